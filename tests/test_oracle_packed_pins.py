"""The oracle of the packed-sequence operators against independent facts: torch
in float64, closed forms and central differences (CPU)."""

import numpy as np
import pytest
import torch

from oracle import packed as P

RNG = np.random.default_rng


def _attn_case(seed, cu, heads, kv, d):
    r = RNG(seed)
    return r.standard_normal((cu[-1] + 2, (heads + 2 * kv) * d)), r.standard_normal((cu[-1] + 2, heads * d))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv", [(2, 2), (4, 2), (3, 1)])
def test_attention_matches_torch(heads, kv, causal):
    d, cu = 8, [1, 6, 6, 7, 16]
    qkv, do = _attn_case(0, cu, heads, kv, d)
    o, lse, _, _ = P.packed_attention_fwd(qkv, cu, heads, kv, d, causal)
    dqkv, _ = P.packed_attention_bwd(qkv, cu, heads, kv, d, causal, do)
    x = torch.tensor(qkv, requires_grad=True)
    total = 0.0
    for b, e in zip(cu[:-1], cu[1:]):
        if b == e:
            continue
        v = x[b:e].view(e - b, heads + 2 * kv, d).transpose(0, 1)
        q, k, w = v[:heads], v[heads:heads + kv], v[heads + kv:]
        k, w = (t.repeat_interleave(heads // kv, 0) for t in (k, w))
        s = q @ k.transpose(1, 2) / d ** 0.5
        if causal:
            s = s.masked_fill(torch.ones(e - b, e - b, dtype=torch.bool).triu(1), float("-inf"))
        ref = (s.softmax(-1) @ w).transpose(0, 1).reshape(e - b, -1)
        assert np.allclose(o[b:e], ref.detach().numpy(), atol=1e-12)
        assert np.allclose(lse[:, b:e], s.logsumexp(-1).detach().numpy(), atol=1e-12)
        total = total + (ref * torch.tensor(do[b:e])).sum()
    total.backward()
    inside = slice(cu[0], cu[-1])
    assert np.allclose(dqkv[inside], x.grad.numpy()[inside], atol=1e-11)
    # rows of no sequence have no result
    assert np.isnan(o[:1]).all() and np.isnan(o[cu[-1]:]).all() and np.isnan(dqkv[cu[-1]:]).all()


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradient_matches_differences(causal):
    heads, kv, d, cu = 2, 1, 4, [0, 1, 6]
    qkv, do = _attn_case(1, cu, heads, kv, d)
    dqkv, _ = P.packed_attention_bwd(qkv, cu, heads, kv, d, causal, do)
    f = lambda x: (P.packed_attention_fwd(x, cu, heads, kv, d, causal)[0][:6] * do[:6]).sum()  # noqa: E731
    for r in range(6):
        for c in range(qkv.shape[1]):
            x = qkv.copy()
            x[r, c] += 1e-5
            up = f(x)
            x[r, c] -= 2e-5
            assert abs((up - f(x)) / 2e-5 - dqkv[r, c]) < 1e-7


def test_attention_of_one_token_is_its_value():
    qkv, _ = _attn_case(2, [0, 1, 2], 2, 2, 8)
    o, lse, _, _ = P.packed_attention_fwd(qkv, [0, 1, 2], 2, 2, 8, False)
    assert np.allclose(o[:2], qkv[:2, 32:])
    assert np.allclose(lse[0, :2], (qkv[:2, :8] * qkv[:2, 16:24]).sum(1) / np.sqrt(8))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope(interleaved):
    heads, kv, d, M, sec = 3, 1, 16, 5, (2, 3, 1)
    r = RNG(3)
    x = r.standard_normal((M, (heads + 2 * kv) * d))
    pos = r.integers(0, 50, (M, 3))
    f = r.random(d // 2)
    y = P.rope(x, heads, kv, d, pos, f, sec, interleaved)
    # as a product of complex numbers
    v = x.reshape(M, -1, d)
    a, b = (v[..., 0::2], v[..., 1::2]) if interleaved else (v[..., :d // 2], v[..., d // 2:])
    ang = np.stack([pos[:, ax] * f[i] for i, ax in enumerate([0, 0, 1, 1, 1, 2])], 1)
    ang = np.concatenate([ang, np.zeros((M, 2))], 1)[:, None]
    z = (a + 1j * b) * np.where(np.arange(heads + 2 * kv)[None, :, None] < heads + kv, np.exp(1j * ang), 1.0)
    w = y.reshape(M, -1, d)
    got = (w[..., 0::2] + 1j * w[..., 1::2]) if interleaved else (w[..., :d // 2] + 1j * w[..., d // 2:])
    assert np.allclose(got, z, atol=1e-12)
    # turned back it is x again, and position 0 turns nothing
    assert np.allclose(P.rope(y, heads, kv, d, pos, f, sec, interleaved, back=True), x, atol=1e-12)
    assert np.array_equal(P.rope(x, heads, kv, d, 0 * pos, f, sec, interleaved), x)
    # scores depend on the difference of positions alone
    k = heads * d
    shifted = P.rope(x, heads, kv, d, pos + 7, f, sec, interleaved)
    assert np.allclose(shifted[0, :d] @ shifted[1, k:k + d], y[0, :d] @ y[1, k:k + d], atol=1e-10)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_glu_matches_torch(act):
    r = RNG(4)
    M, H, F = 7, 12, 10
    y, w, b, w2, dout = (r.standard_normal(s) for s in ((M, H), (2 * F, H), (2 * F,), (H, F), (M, H)))
    gu, h, _, _ = P.glu_fwd(y, w, b, act)
    t = torch.tensor(y) @ torch.tensor(w).T + torch.tensor(b)
    t.requires_grad_(True)
    fn = torch.nn.functional.silu if act == "silu" else torch.nn.functional.gelu
    ref = fn(t[:, :F]) * t[:, F:]
    assert np.allclose(gu, t.detach().numpy(), atol=1e-12) and np.allclose(h, ref.detach().numpy(), atol=1e-12)
    (ref @ torch.tensor(w2).T * torch.tensor(dout)).sum().backward()
    dgu, _ = P.glu_bwd(dout, w2, gu, act)
    assert np.allclose(dgu, t.grad.numpy(), atol=1e-11)


def test_planted_mistakes_are_seen():
    """The bounds are far smaller than what a wrong formula gives."""
    heads, kv, d, cu = 4, 2, 64, [0, 40, 60]
    qkv, do = _attn_case(5, cu, heads, kv, d)
    qkv, do = qkv[:60], do[:60]
    o, _, ob, _ = P.packed_attention_fwd(qkv, cu, heads, kv, d, False)
    dqkv, db = P.packed_attention_bwd(qkv, cu, heads, kv, d, False, do)
    outside = lambda x, ref, bound: np.mean(np.abs(x - ref) > bound)  # noqa: E731
    assert outside(P.packed_attention_fwd(qkv, cu, heads, kv, d, True)[0], o, ob) > 0.5
    assert outside(P.packed_attention_fwd(qkv, [0, 39, 60], heads, kv, d, False)[0], o, ob) > 0.5
    assert outside(P.packed_attention_bwd(qkv, cu, heads, kv, d, True, do)[0], dqkv, db) > 0.3
    # the key gradient of only one of the heads that share it
    one = do.copy().reshape(60, heads, d)
    one[:, 1::2] = 0
    part, _ = P.packed_attention_bwd(qkv, cu, heads, kv, d, False, one.reshape(60, -1))
    assert outside(part[:, heads * d:], dqkv[:, heads * d:], db[:, heads * d:]) > 0.5
    y, w, w2 = RNG(6).standard_normal((9, 64)), RNG(7).standard_normal((48, 64)) / 8, RNG(8).standard_normal((64, 24))
    gu, h, _, hb = P.glu_fwd(y, w, None, "silu")
    assert outside(P.glu_fwd(y, w, None, "gelu")[1], h, hb) > 0.5
    assert outside(P.glu_fwd(y, np.roll(w, 24, 0), None, "silu")[1], h, hb) > 0.5
    dgu, gb = P.glu_bwd(y, w2, gu, "silu")
    assert outside(np.roll(dgu, 24, 1), dgu, gb) > 0.5
    x, pos, f = RNG(9).standard_normal((9, 8 * 16)), RNG(10).integers(1, 30, (9, 3)), RNG(11).random(8)
    y0 = P.rope(x, 4, 2, 16, pos, f, (2, 3, 3), False)
    b0 = P.rope_bound(x, y0, 4, 2, 16, pos, f, (2, 3, 3), False)
    for wrong in (P.rope(x, 4, 2, 16, pos, f, (2, 3, 3), True), P.rope(x, 4, 2, 16, pos, f, (3, 2, 3), False),
                  P.rope(x, 4, 2, 16, pos, f, (2, 3, 3), False, back=True)):
        assert outside(wrong, y0, b0) > 0.05
    assert (b0[:, 96:] == 0).all()  # values are copied
