"""The example's serving loop against a plain forward pass, without and with a budget that bites."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import serve_budget
    return serve_budget


def _plain_logits(s, ids):
    """Logits behind the last of `ids` in float64, the whole sequence at once."""
    import torch
    m, w = s.m, {k: v.double() for k, v in s.w.items()}
    norm = lambda x, g: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + m.norm_eps) * g  # noqa: E731
    n, G = len(ids), m.n_heads // m.n_kv_heads
    x = w["embedding"][torch.tensor(ids, device="cuda")]
    f = m.rope_base ** (-2.0 * torch.arange(m.head_dim // 2, device="cuda", dtype=torch.float64) / m.head_dim)
    ang = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * f
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]

    def turn(y):
        a, b = y[..., :m.head_dim // 2], y[..., m.head_dim // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    mask = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    for j in range(m.n_layers):
        h = norm(x, w["attn_norm"][j])
        q = turn((h @ w["wq"][j].T).view(n, m.n_heads, -1))
        k = turn((h @ w["wk"][j].T).view(n, m.n_kv_heads, -1)).repeat_interleave(G, 1)
        v = (h @ w["wv"][j].T).view(n, m.n_kv_heads, -1).repeat_interleave(G, 1)
        p = torch.softmax((torch.einsum("qhd,khd->hqk", q, k) / m.head_dim ** 0.5).masked_fill(~mask, -torch.inf), -1)
        x = x + torch.einsum("hqk,khd->qhd", p, v).reshape(n, -1) @ w["wo"][j].T
        h = norm(x, w["mlp_norm"][j])
        x = x + (torch.nn.functional.silu(h @ w["w_gate"][j].T) * (h @ w["w_up"][j].T)) @ w["w_down"][j].T
    return norm(x[-1:], w["final_norm"]) @ w["embedding"].T


def test_without_eviction_the_loop_is_the_plain_model(E):
    """Prompts in pieces, then single tokens: logits of the plain float64 model within bfloat16's rounding. Two layers round
    a dozen times each at 2^-8 relative, partly cancelling: 3 % of the largest logit is twice what that leaves."""
    import torch
    m = E.small_model()
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, m.vocab, n).tolist() for n in (150, 1, 97)]
    s = E.Session(m, 3, 400, 64, 300, temperature=0.0)
    for at in (0, 64, 128):
        tokens, _, logits = s.step([p[at:at + 64] for p in prompts])
        for b, p in enumerate(prompts):
            if len(p) <= at:
                assert int(tokens[b]) == -1
                continue
            want = _plain_logits(s, p[:at + 64])
            assert float((logits[b].double() - want[0]).abs().max() / want.abs().max()) < 0.03
            assert int(tokens[b]) == int(logits[b].argmax())
    seqs = [list(p) for p in prompts]
    for _ in range(3):
        for b in range(3):
            seqs[b].append(int(rng.integers(0, m.vocab)))
        _, _, logits = s.step([[q[-1]] for q in seqs])
        for b in range(3):
            want = _plain_logits(s, seqs[b])
            assert float((logits[b].double() - want[0]).abs().max() / want.abs().max()) < 0.03
    assert s.lens.tolist() == [len(q) for q in seqs] and int(s.err.item()) == 0
    # every query of every layer and head gave away 1 in all
    total = sum(len(q) for q in seqs) * m.n_layers * m.n_heads
    held = torch.zeros((), device="cuda")
    for b, q in enumerate(seqs):
        e = torch.arange(len(q), device="cuda")
        held += s.weight[s.page_table[b].long()[e // 64], e % 64].sum()
    assert abs(float(held) / total - 1) < 1e-3


def test_under_a_budget_caches_stay_short_and_keep_what_is_protected(E):
    m = E.small_model()
    rng = np.random.default_rng(2)
    prompts = [rng.integers(0, m.vocab, n).tolist() for n in (500, 40, 333, 200)]
    s = E.Session(m, 4, 96, 64, 700, recent=16, first=4, temperature=0.8, top_k=40, top_p=0.95)
    tokens = s.generate(prompts, 80)
    assert tokens.shape == (4, 80) and (tokens >= 0).all() and (tokens < m.vocab).all()
    assert s.lens.tolist() == [96] * 4
    assert s.next_pos.tolist() == [len(p) + 79 for p in prompts]
    pos = s.pos.cpu().numpy().reshape(4, -1)
    for b in range(4):
        held = sorted(pos[b, :96].tolist())
        assert len(set(held)) == 96 and held[:4] == [0, 1, 2, 3]
        assert held[-16:] == list(range(int(s.next_pos[b]) - 16, int(s.next_pos[b])))
