"""Generation for a batch of sequences whose paged caches are kept under a budget of entries.

Runs the operators of tlf as a serving loop does: every step puts the new tokens' rotated keys and values into their pages
(tlf_rope_append), attends from them to the rows' caches and keeps account of what was looked at (tlf_attn_chunk), cuts the
caches that have grown past the budget back to it (tlf_cache_evict) and draws the next tokens (tlf_sample). Prompts go through
the same calls as chunks of many tokens, in pieces of --piece tokens, so that a long prompt never needs a cache longer than the
budget and a piece.

The model is a small pre-norm transformer with grouped-query attention and seeded random weights (synth.make_weights; its
block applied once); projections are torch products.

    python examples/serve_budget.py --rows 4 --prompt 700 --steps 64 --budget 256
"""
import argparse
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2609_15160_gb300 import synth, tlf  # noqa: E402

PAGE = 64


def small_model():
    return synth.tiny_config(vocab=512, d_model=256, n_heads=8, n_kv_heads=2, head_dim=64, n_layers=2, ffn_hidden=512, max_loops=1,
                             dtype="bf16")


class Session:
    """Caches and buffers of `rows` sequences; a row may have up to `budget` entries and the tokens of one call."""

    def __init__(self, model, rows, budget, most_new, max_pos, recent=32, first=4, seed=0, **sampling):
        self.m, self.rows, self.budget, self.most_new = model, rows, budget, most_new
        dev = "cuda"
        w = synth.make_weights(model)
        put = lambda name, t=torch.bfloat16: torch.tensor(np.asarray(w[name], np.float32)).to(dev, t)  # noqa: E731
        self.w = {n: put(n) for n in ("embedding", "wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")}
        self.w.update({n: put(n, torch.float32) for n in ("attn_norm", "mlp_norm", "final_norm")})
        self.wqkv = torch.cat([self.w["wq"], self.w["wk"], self.w["wv"]], 1)
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)  # noqa: E731
        per_row = (budget + most_new + PAGE - 1) // PAGE
        self.pool = torch.zeros(rows * per_row, model.n_layers, 2, model.n_kv_heads, PAGE, model.head_dim, dtype=torch.bfloat16,
                                device=dev)
        self.page_table = torch.arange(rows * per_row, dtype=torch.int32, device=dev).view(rows, per_row)
        self.pos, self.weight = i32(rows * per_row, PAGE), torch.zeros(rows * per_row, PAGE, device=dev)
        self.lens, self.next_pos, self.err = i32(rows), i32(rows), i32(1)
        self.table = torch.empty(max_pos, model.head_dim // 2, 2, device=dev)
        tlf.tlf_rope_table(tlf.rope_config(model.head_dim, base=model.rope_base), max_pos, self.table)
        self.gen = torch.Generator(device=dev).manual_seed(seed)
        self.sampling = {k: torch.full((rows,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device=dev)
                         for k, v in sampling.items()}
        self.evict = tlf.evict_args(self.pool, self.page_table, self.lens, self.next_pos, self.pos, self.pos, self.weight,
                                    self.weight, self.lens, budget=budget, n_first=first, n_recent=recent, err=self.err)
        self.evict_scratch = torch.empty(tlf.tlf_cache_evict_scratch_bytes(self.evict), dtype=torch.uint8, device=dev)

    def norm(self, x, gain):
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.m.norm_eps) * gain).bfloat16()

    def forward(self, chunks):
        """chunks: the new token ids of every row (lists, possibly empty). Appends them and returns the hidden state of every
        new token [tokens, d] (float32) and the rows' offsets into them."""
        m, dev, stream = self.m, "cuda", torch.cuda.current_stream()
        new = np.array([len(c) for c in chunks])
        assert new.max() <= self.most_new
        offsets = np.concatenate([[0], np.cumsum(new)])
        T = int(offsets[-1])
        cu = torch.tensor(offsets, dtype=torch.int32, device=dev)
        count = torch.tensor(new, dtype=torch.int32, device=dev)
        ids = torch.tensor(np.concatenate([np.asarray(c, np.int64) for c in chunks]), device=dev)
        row = torch.repeat_interleave(torch.arange(self.rows, device=dev), count)
        positions = (self.next_pos[row] + torch.arange(T, device=dev) - cu[row]).int()
        self.lens += count
        self.next_pos += count
        x = self.w["embedding"][ids].float()
        hq, hk = m.n_heads * m.head_dim, m.n_kv_heads * m.head_dim
        q = torch.empty(T, m.n_heads, m.head_dim, dtype=torch.bfloat16, device=dev)
        o = torch.empty_like(q)
        attn = tlf.attn_chunk_args(q, o, weight_in=self.weight, weight_out=self.weight)
        scratch = None
        for j in range(m.n_layers):
            qkv = self.norm(x, self.w["attn_norm"][j]) @ self.wqkv[j].T
            batch = tlf.chunk_args(self.pool, self.page_table, cu, self.lens, m.n_heads, T, layer=j, max_chunk=int(new.max()),
                                   err=self.err)
            # the first layer also notes the entries' positions and starts their account
            rope = tlf.rope_args(qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], positions, self.table, q,
                                 entry_pos=self.pos if j == 0 else None, entry_weight=self.weight if j == 0 else None)
            tlf.tlf_rope_append(batch, rope, stream)
            if scratch is None:
                scratch = torch.empty(tlf.tlf_attn_chunk_scratch_bytes(batch, attn), dtype=torch.uint8, device=dev)
            tlf.tlf_attn_chunk(batch, attn, scratch, scratch.numel(), stream)
            x = x + (o.view(T, hq) @ self.w["wo"][j].T).float()
            h = self.norm(x, self.w["mlp_norm"][j])
            x = x + ((torch.nn.functional.silu(h @ self.w["w_gate"][j].T) * (h @ self.w["w_up"][j].T)) @ self.w["w_down"][j].T).float()
        return x, offsets

    def step(self, chunks):
        """The rows' new tokens in, the next token of every row out (rows without new tokens draw from nothing: -1)."""
        x, offsets = self.forward(chunks)
        tlf.tlf_cache_evict(self.evict, self.evict_scratch, self.evict_scratch.numel(), torch.cuda.current_stream())
        new = np.diff(offsets)
        last = torch.tensor(np.maximum(offsets[1:] - 1, 0), device="cuda")
        logits = (self.norm(x[last], self.w["final_norm"]) @ self.w["embedding"].T).float()
        logits[torch.tensor(new == 0, device="cuda")] = -torch.inf
        noise = torch.rand(logits.shape, device="cuda", generator=self.gen)
        tokens = torch.empty(self.rows, dtype=torch.int32, device="cuda")
        logprobs = torch.empty(self.rows, device="cuda")
        tlf.tlf_sample(tlf.sample_args(logits, noise, tokens, logprobs, **self.sampling), torch.cuda.current_stream())
        return tokens, logprobs, logits

    def generate(self, prompts, steps):
        """Prompts in pieces, then `steps` tokens a row; returns the tokens [rows][steps]."""
        longest = max(len(p) for p in prompts)
        tokens = torch.full((self.rows,), -1, dtype=torch.int32, device="cuda")
        for at in range(0, longest, self.most_new):
            t, _, _ = self.step([p[at:at + self.most_new] for p in prompts])
            tokens = torch.where(t >= 0, t, tokens)  # a prompt that has ended keeps its token
        out = [tokens]
        for _ in range(steps - 1):
            out.append(self.step([[int(t)] for t in out[-1].tolist()])[0])
        if int(self.err.item()):
            raise RuntimeError(f"device error word {int(self.err.item())}")
        return torch.stack(out, 1).cpu().numpy()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rows", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--budget", type=int, default=256)
    ap.add_argument("--piece", type=int, default=128)
    ap.add_argument("--temperature", type=float, default=0.8)
    ap.add_argument("--top-p", type=float, default=0.95)
    a = ap.parse_args()
    m = small_model()
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, m.vocab, n).tolist() for n in rng.integers(max(1, a.prompt // 2), a.prompt + 1, a.rows)]
    s = Session(m, a.rows, a.budget, a.piece, a.prompt + a.steps + 1, temperature=a.temperature, top_p=a.top_p, top_k=0)
    tokens = s.generate(prompts, a.steps)
    for b in range(a.rows):
        print(f"row {b}: prompt {len(prompts[b])} tokens, cache {int(s.lens[b])} entries, tokens {tokens[b][:16].tolist()} ...")


if __name__ == "__main__":
    main()
