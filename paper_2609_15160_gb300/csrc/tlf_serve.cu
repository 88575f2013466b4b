// Entry points of the operators on a caller's paged caches and logits (declared in include/tlf.h): checks of arguments, and
// the launches. Nothing here allocates or synchronises.
#include <cmath>
#include <cstdio>

#include "k_serve.cuh"
#include "tlf.h"

namespace tlf {

static bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// A cache's shape; NULL when it is fine.
static const char* cache_validate(int n, int hkv, int hd, int layers, int page_size, int dtype, int max_pages, int64_t n_pages,
                                  const void* pool, const void* page_table, const void* lens) {
  if (n < 1 || n > SV_MAX_ROWS) return "n must be in 1..1024";
  if (dtype != TLF_DTYPE_F32 && dtype != TLF_DTYPE_BF16) return "unknown dtype";
  if (hkv < 1 || layers < 1) return "n_kv_heads and n_layers must be positive";
  if (!(hd == 32 || hd == 64 || hd == 128 || (hd == 16 && dtype == TLF_DTYPE_F32)))
    return "head_dim must be 32, 64 or 128 (or 16 with float32)";
  if (page_size != SV_PAGE) return "page_size must be 64";
  if ((int64_t)layers * 2 * hkv * SV_PAGE > 0x7fffffff) return "n_layers * n_kv_heads is too large";
  // (the kernels step through entries in strides of up to 2048 and round their number up: room for that below 2^31)
  if (max_pages < 1 || max_pages > 0x7fffffff / SV_PAGE - 64) return "max_pages must be in 1..2^25 - 65";
  if (n_pages < 1 || n_pages > 0x7fffffff) return "n_pages must be in 1..2^31 - 1";
  if (!pool || !page_table || !lens) return "a device pointer is NULL";
  if (!aligned(pool, 16)) return "pool must be aligned to 16 bytes";
  return nullptr;
}

static const char* chunk_validate(const tlf_chunk* c) {
  if (!c) return "the chunk is NULL";
  if (const char* why = cache_validate(c->n, c->n_kv_heads, c->head_dim, c->n_layers, c->page_size, c->dtype, c->max_pages,
                                       c->n_pages, c->pool, c->page_table, c->lens))
    return why;
  if (c->n_tokens < 0 || c->n_tokens > (1 << 26)) return "n_tokens must be in 0..2^26";
  if (c->max_chunk < 0) return "max_chunk must not be negative";
  if (c->n_heads < 1 || c->n_heads % c->n_kv_heads) return "n_kv_heads must divide n_heads";
  if (c->n_heads / c->n_kv_heads > 64) return "at most 64 query heads per kv head";
  if ((int64_t)c->n_heads * c->head_dim > (1 << 24)) return "n_heads * head_dim must be at most 2^24";
  if (c->layer < 0 || c->layer >= c->n_layers) return "layer out of range";
  if (!c->cu_tokens) return "a device pointer is NULL";
  if (c->reserved0) return "reserved0 must be 0";
  return nullptr;
}

static ChunkDev chunk_dev(const tlf_chunk* c) {
  ChunkDev d{};
  d.n = c->n;
  d.T = c->n_tokens;
  d.max_chunk = c->max_chunk && c->max_chunk < c->n_tokens ? c->max_chunk : c->n_tokens;
  d.Hq = c->n_heads;
  d.Hkv = c->n_kv_heads;
  d.G = c->n_heads / c->n_kv_heads;
  d.hd = c->head_dim;
  d.J = c->n_layers;
  d.layer = c->layer;
  d.max_pages = c->max_pages;
  d.n_pages = c->n_pages;
  d.page_elems = (long long)c->n_layers * 2 * c->n_kv_heads * SV_PAGE * c->head_dim;
  d.pool = c->pool;
  d.page_table = c->page_table;
  d.cu = c->cu_tokens;
  d.lens = c->lens;
  d.err = c->err;
  return d;
}

static const char* rope_validate(const tlf_chunk* c, const tlf_rope_args* a) {
  if (!a) return "the arguments are NULL";
  if (!a->q || !a->k || !a->v || !a->positions || !a->table || !a->q_out) return "a device pointer is NULL";
  if (a->rot_dim < 2 || a->rot_dim % 2 || a->rot_dim > c->head_dim) return "rot_dim must be even and in 2..head_dim";
  if (a->max_pos < 1) return "max_pos must be positive";
  if (a->layout != TLF_ROPE_HALF && a->layout != TLF_ROPE_INTERLEAVED) return "unknown layout";
  if (a->q_f32 != 0 && a->q_f32 != 1) return "q_f32 must be 0 or 1";
  if (c->n_tokens > 1 && (a->q_stride < (int64_t)c->n_heads * c->head_dim || a->k_stride < (int64_t)c->n_kv_heads * c->head_dim ||
                          a->v_stride < (int64_t)c->n_kv_heads * c->head_dim))
    return "a stride is smaller than a token's heads";
  if (!aligned(a->table, 8)) return "table must be aligned to 8 bytes";
  return nullptr;
}

static const char* attn_validate(const tlf_chunk* c, const tlf_attn_chunk_args* a) {
  if (const char* why = chunk_validate(c)) return why;
  if (!a) return "the arguments are NULL";
  if (!a->q || !a->out) return "a device pointer is NULL";
  const int64_t row = (int64_t)c->n_heads * c->head_dim;
  if ((a->q_stride && a->q_stride < row) || (a->out_stride && a->out_stride < row))
    return "a stride is smaller than a token's heads";
  if (a->weight_in && !a->weight_out) return "weight_in without weight_out";
  if (!(a->scale >= 0.f) || a->scale > 2e38f) return "scale must be in 0..2e38";  // (finite times log2 e too)
  if (a->reserved0) return "reserved0 must be 0";
  return nullptr;
}

static const char* evict_validate(const tlf_evict_args* a) {
  if (!a) return "the arguments are NULL";
  if (const char* why = cache_validate(a->n, a->n_kv_heads, a->head_dim, a->n_layers, a->page_size, a->dtype, a->max_pages,
                                       a->n_pages, a->pool, a->page_table, a->lens))
    return why;
  if (!a->next_pos || !a->pos_in || !a->pos_out || !a->weight_in || !a->weight_out || !a->lens_out)
    return "a device pointer is NULL";
  if (a->budget < 1 || a->n_first < 0 || a->n_recent < 0 || (int64_t)a->n_first + a->n_recent > a->budget)
    return "budget must be positive and hold n_first + n_recent entries";
  return nullptr;
}

static const char* sample_validate(const tlf_sample_args* a) {
  if (!a) return "the arguments are NULL";
  if (a->n < 1 || a->n > 65535) return "n must be in 1..65535";
  if (a->vocab < 1 || a->vocab > (1 << 22)) return "vocab must be in 1..2^22";
  if (!a->logits || !a->noise || !a->tokens) return "a device pointer is NULL";
  if (a->n > 1 && (a->logits_stride < a->vocab || a->noise_stride < a->vocab)) return "a stride is smaller than vocab";
  return nullptr;
}

static int refuse(const char* who, const char* why) {
  char msg[256];
  snprintf(msg, sizeof msg, "%s: %s", who, why);
  return set_thread_error(TLF_ERR_INVALID_ARG, msg);
}
static int done(cudaError_t e) { return e == cudaSuccess ? TLF_OK : set_thread_error(TLF_ERR_CUDA, cudaGetErrorString(e)); }

// No C++ exception leaves an entry point (the messages and the table of kernel attributes allocate host memory).
template <typename F>
static int guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return TLF_ERR_CUDA;
  }
}

}  // namespace tlf

using namespace tlf;

extern "C" int tlf_rope_table(const tlf_rope_config* cfg, int32_t max_pos, float* table, void* stream) {
  return guarded([&] {
    const char* who = "tlf_rope_table";
    if (!cfg) return refuse(who, "the config is NULL");
    if (cfg->rot_dim < 2 || cfg->rot_dim % 2 || cfg->rot_dim > 256) return refuse(who, "rot_dim must be even and in 2..256");
    if (cfg->scaling < TLF_ROPE_NONE || cfg->scaling > TLF_ROPE_RAMP) return refuse(who, "unknown scaling");
    if (!(cfg->base > 1.0) || !std::isfinite(cfg->base)) return refuse(who, "base must be larger than 1");
    if (!std::isfinite(cfg->magnitude)) return refuse(who, "magnitude must be finite");
    if (cfg->scaling != TLF_ROPE_NONE && (!(cfg->factor >= 1.0) || !std::isfinite(cfg->factor)))
      return refuse(who, "factor must be at least 1");
    if (cfg->scaling == TLF_ROPE_NTK && cfg->rot_dim == 2) return refuse(who, "NTK needs rot_dim > 2");
    if (cfg->scaling == TLF_ROPE_RAMP &&
        (!(cfg->original_len > 0.0) || !std::isfinite(cfg->original_len) || !(cfg->low_turns >= 0.0) ||
         !(cfg->high_turns > cfg->low_turns) || !std::isfinite(cfg->high_turns)))
      return refuse(who, "RAMP needs original_len > 0 and 0 <= low_turns < high_turns");
    if (max_pos < 1) return refuse(who, "max_pos must be positive");
    if (!table || !aligned(table, 8)) return refuse(who, "table must be a device pointer aligned to 8 bytes");
    return done(launch_rope_scaled_table(*cfg, max_pos, table, static_cast<cudaStream_t>(stream)));
  });
}

extern "C" int tlf_rope_append(const tlf_chunk* c, const tlf_rope_args* a, void* stream) {
  return guarded([&] {
    if (const char* why = chunk_validate(c)) return refuse("tlf_rope_append", why);
    if (const char* why = rope_validate(c, a)) return refuse("tlf_rope_append", why);
    if (c->n_tokens == 0) return (int)TLF_OK;
    const int sms = current_num_sms();
    if (sms <= 0) return set_thread_error(TLF_ERR_CUDA, "no current CUDA device");
    return done(launch_rope_chunk(chunk_dev(c), c->dtype, *a, sms, static_cast<cudaStream_t>(stream)));
  });
}

extern "C" size_t tlf_attn_chunk_scratch_bytes(const tlf_chunk* c, const tlf_attn_chunk_args* a) {
  if (attn_validate(c, a)) return 0;
  const int sms = current_num_sms();
  return sms <= 0 ? 0 : chunk_attn_scratch(chunk_dev(c), c->dtype, *a, sms);
}

extern "C" int tlf_attn_chunk(const tlf_chunk* c, const tlf_attn_chunk_args* a, void* scratch, size_t scratch_bytes,
                              void* stream) {
  return guarded([&] {
    if (const char* why = attn_validate(c, a)) return refuse("tlf_attn_chunk", why);
    const int sms = current_num_sms();
    if (sms <= 0) return set_thread_error(TLF_ERR_CUDA, "no current CUDA device");
    const ChunkDev d = chunk_dev(c);
    if (!scratch || !aligned(scratch, 16) || scratch_bytes < chunk_attn_scratch(d, c->dtype, *a, sms))
      return refuse("tlf_attn_chunk", "scratch too small or not aligned to 16 bytes");
    return done(launch_chunk_attn(d, c->dtype, *a, scratch, sms, static_cast<cudaStream_t>(stream)));
  });
}

extern "C" size_t tlf_cache_evict_scratch_bytes(const tlf_evict_args* a) { return evict_validate(a) ? 0 : evict_scratch(*a); }

extern "C" int tlf_cache_evict(const tlf_evict_args* a, void* scratch, size_t scratch_bytes, void* stream) {
  return guarded([&] {
    if (const char* why = evict_validate(a)) return refuse("tlf_cache_evict", why);
    if (!scratch || !aligned(scratch, 16) || scratch_bytes < evict_scratch(*a))
      return refuse("tlf_cache_evict", "scratch too small or not aligned to 16 bytes");
    const int sms = current_num_sms();
    if (sms <= 0) return set_thread_error(TLF_ERR_CUDA, "no current CUDA device");
    return done(launch_evict(*a, scratch, sms, static_cast<cudaStream_t>(stream)));
  });
}

extern "C" int tlf_sample(const tlf_sample_args* a, void* stream) {
  return guarded([&] {
    if (const char* why = sample_validate(a)) return refuse("tlf_sample", why);
    const int sms = current_num_sms();
    if (sms <= 0) return set_thread_error(TLF_ERR_CUDA, "no current CUDA device");
    return done(launch_sample(*a, sms, static_cast<cudaStream_t>(stream)));
  });
}
