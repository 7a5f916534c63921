"""Rotary positions, the packed work list and packed attention on the GPU,
against the float64 oracle within its elementwise bounds, and a packed layer
that uses them together with the gated feed-forward block."""

import numpy as np
import pytest
import torch

import oracle
from helpers import TOL_ACT, TOL_GRAD, announce, cuda, f64, guard_intact, guarded, max_rel
from oracle import packed as P
from paper_2408_03505_amd import binding as B
from paper_2408_03505_amd.synthetic import random_bf16

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

BF = torch.bfloat16


def within(got, ref, bound, rows=None):
    """Every element of got (of these rows) within its bound of ref."""
    got = f64(got)
    sel = slice(None) if rows is None else rows
    off = np.abs(got[sel] - ref[sel])
    assert np.isfinite(got[sel]).all()
    worst = float((off / np.maximum(bound[sel], 1e-300)).max()) if off.size else 0.0
    assert (off <= bound[sel]).all(), f"worst error is {worst:.2f} of its bound"


# ------------------------------------------------------------------ rotary positions

def _rope_inputs(M, heads, kv, d, sec, far, seed):
    x = random_bf16((M, (heads + 2 * kv) * d), seed)
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, far, (M, 3), generator=g, dtype=torch.int32)
    f = []
    for n in sec:
        f += [10000.0 ** (-i / n) for i in range(n)]
    f += [float("nan")] * (d // 2 - len(f))  # pairs of no axis: their frequency is not read
    return x, pos, torch.tensor(f, dtype=torch.float32)


ROPE = [(1, 1, 1, 64, (0, 16, 16), 16), (5, 3, 3, 64, (8, 12, 12), 2 ** 20), (257, 16, 16, 80, (0, 20, 20), 16),
        (33, 8, 2, 128, (16, 24, 20), 2 ** 31 - 1), (300, 6, 1, 80, (10, 0, 7), 1000), (7, 48, 48, 128, (0, 0, 0), 9),
        (64, 4, 4, 128, (64, 0, 0), 4096)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("M,heads,kv,d,sec,far", ROPE)
def test_rope(M, heads, kv, d, sec, far, interleaved, back):
    announce(f"rope M={M} heads={heads}/{kv} d={d} sections={sec} far={far} interleaved={interleaved} back={back}")
    x, pos, f = _rope_inputs(M, heads, kv, d, sec, far, 1)
    out, buf = guarded(x.shape, BF)
    call = B.enc_rope_bwd if back else B.enc_rope_fwd
    call(heads, kv, d, cuda(x), cuda(pos), cuda(f), sec, interleaved, out)
    torch.cuda.synchronize()
    ref = P.rope(f64(x), heads, kv, d, pos.numpy(), f.numpy(), sec, interleaved, back)
    within(out, ref, P.rope_bound(f64(x), ref, heads, kv, d, pos.numpy(), f.numpy(), sec, interleaved))
    assert guard_intact(buf, out.numel())
    # in place: the same bits
    y = cuda(x)
    call(heads, kv, d, y, cuda(pos), cuda(f), sec, interleaved, y)
    assert torch.equal(y.view(torch.int16), out.view(torch.int16))


def test_rope_of_negative_positions():
    x, pos, f = _rope_inputs(9, 2, 2, 64, (8, 12, 12), 1000, 2)
    pos = -pos
    announce("rope negative positions")
    y = B.enc_rope_fwd(2, 2, 64, cuda(x), cuda(pos), cuda(f), (8, 12, 12))
    ref = P.rope(f64(x), 2, 2, 64, pos.numpy(), f.numpy(), (8, 12, 12), False)
    within(y, ref, P.rope_bound(f64(x), ref, 2, 2, 64, pos.numpy(), f.numpy(), (8, 12, 12), False))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d, sec", [(64, (0, 0, 0)), (80, (3, 0, 8)), (128, (16, 24, 23))])
def test_rope_copies_pairs_without_an_axis_bit_for_bit(d, sec, interleaved):
    """Signed zeros, infinities and NaN among them, which a turn by no angle would not keep."""
    x, pos, f = _rope_inputs(5, 3, 1, d, sec, 50, 3)
    used, i = sum(sec), torch.arange(sum(sec), d // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
    heads = x.view(5, 5, d)
    heads[:, :, a] = -0.0
    heads[0, :, b], heads[1, :, b], heads[2, :, b], heads[3, :, b] = float("inf"), float("nan"), float("-inf"), 0.0
    announce(f"rope d={d} sections={sec} interleaved={interleaved} non-finite pairs without an axis")
    for call in (B.enc_rope_fwd, B.enc_rope_bwd):
        y = call(3, 1, d, cuda(x), cuda(pos), cuda(f), sec, interleaved).cpu().view(5, 5, d)
        for c in (a, b):
            assert torch.equal(y[:, :, c].view(torch.int16), heads[:, :, c].view(torch.int16))
        turned = [c for c in range(d) if c not in a.tolist() + b.tolist()]
        assert len(turned) == 2 * used and torch.isfinite(y[:, :, turned]).all()


# ------------------------------------------------------------------ work list

def _items(plan):
    w = plan.view(torch.int32).cpu().numpy()
    n = int(w[0])
    return w[4:4 + 4 * n].reshape(n, 4)[:, :3]


def _plan(cu, tokens):
    return B.enc_packed_plan(torch.tensor(cu, dtype=torch.int32, device="cuda"), tokens)


@pytest.mark.parametrize("lens", [[1], [0, 0, 5], [128, 129, 127, 256], list(range(0, 700, 3)), [3] * 513, [100000]])
def test_plan_lists_every_tile_longest_sequence_first(lens):
    cu = np.concatenate([[2], 2 + np.cumsum(lens)])
    tokens = int(cu[-1]) + 3
    announce(f"plan of {len(lens)} sequences")
    items = _items(_plan(cu.tolist(), tokens))
    tiles = [-(-n // 128) for n in lens]
    order = sorted(range(len(lens)), key=lambda i: (-tiles[i], i))
    want = [(cu[i], lens[i], 128 * (tiles[i] - 1 - k)) for i in order for k in range(tiles[i])]
    assert np.array_equal(items, np.array(want).reshape(-1, 3))


def test_plan_at_its_largest_size():
    """As many rows as an attention call takes, nearly all in one sequence; the memory in
    front of the plan and behind it stays as it was."""
    tokens, n = (2 ** 31 - 1) // 192, 4096
    announce(f"plan of {tokens} tokens")
    size = B.packed_plan_bytes(tokens, 2)
    buf = torch.full((size + 2 * n,), 0x5a, dtype=torch.uint8, device="cuda")
    plan = buf[n:n + size]
    B.enc_packed_plan(torch.tensor([0, 5, tokens], dtype=torch.int32, device="cuda"), tokens, plan)
    items, tiles = _items(plan), -(-(tokens - 5) // 128)
    want = [(5, tokens - 5, 128 * (tiles - 1 - k)) for k in range(tiles)] + [(0, 5, 0)]
    assert np.array_equal(items, np.array(want))
    assert (buf[:n] == 0x5a).all() and (buf[n + size:] == 0x5a).all()


@pytest.mark.parametrize("cu", [[0, 700, 20, 900, 5, 1000], [-50, 10, 400], [0, 2000, 3000], [2 ** 31 - 1, -2 ** 31, 7]])
def test_plan_of_bad_offsets_stays_inside_the_tensors(cu):
    announce(f"plan of offsets {cu}")
    plan = _plan(cu, 1000)
    items = _items(plan)
    assert len(items) <= 1000 // 128 + len(cu) - 1
    first, n, row = items.T
    assert (first >= 0).all() and (n >= 0).all() and (first + n <= 1000).all() and (row >= 0).all() and (row < n).all()


# ------------------------------------------------------------------ attention

def _attn_inputs(cu, tokens, heads, kv, d, seed, scale=1.0):
    qkv = (random_bf16((tokens, (heads + 2 * kv) * d), seed).float() * scale).to(BF)
    do = random_bf16((tokens, heads * d), seed + 1)
    # rows of no sequence hold what no kernel may read
    inside = torch.zeros(tokens, dtype=torch.bool)
    inside[cu[0]:cu[-1]] = True
    qkv[~inside] = float("nan")
    do[~inside] = float("inf")
    return qkv, do, inside.numpy()


LENS = {
    "one": [1],
    "short": [17, 1, 0, 9, 30],
    "tiles": [32, 31, 33, 64, 65, 128, 129, 127],
    "long": [700, 3, 260],
    "many": [int(x) for x in np.random.default_rng(0).integers(0, 90, 40)],
}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,d", [(3, 3, 64), (4, 2, 80), (8, 1, 128), (16, 16, 64), (16, 8, 80), (6, 3, 128),
                                        (16, 2, 128), (32, 8, 64), (4, 1, 80), (12, 3, 128)])
@pytest.mark.parametrize("lens", sorted(LENS))
def test_attention(lens, heads, kv, d, causal):
    lens = LENS[lens]
    cu = [3] + [3 + int(x) for x in np.cumsum(lens)]
    tokens = cu[-1] + 5
    announce(f"packed attention lens={lens} heads={heads}/{kv} d={d} causal={causal}")
    qkv, do, inside = _attn_inputs(cu, tokens, heads, kv, d, 11)
    g, plan = cuda(qkv), _plan(cu, tokens)
    o, ob = guarded((tokens, heads * d), BF)
    lse, lb = guarded((heads, tokens), torch.float32)
    dqkv, db = guarded(qkv.shape, BF)
    for t in (o, lse, dqkv):
        t.fill_(7.0)
    B.enc_attn_packed_fwd(len(lens), heads, kv, d, g, plan, causal, o, lse)
    B.enc_attn_packed_bwd(len(lens), heads, kv, d, g, o, lse, cuda(do), plan, causal, dqkv)
    torch.cuda.synchronize()
    x = np.where(inside[:, None], f64(qkv), 0.0)
    dd = np.where(inside[:, None], f64(do), 0.0)
    ref, rlse, bound, lbound = P.packed_attention_fwd(x, cu, heads, kv, d, causal)
    within(o, ref, bound, inside)
    within(lse.t(), rlse.T, lbound.T, inside)
    ref, bound = P.packed_attention_bwd(x, cu, heads, kv, d, causal, dd)
    within(dqkv, ref, bound, inside)
    # rows of no sequence are as they were, and nothing is written behind the tensors
    for t in (o, lse.t(), dqkv):
        assert (f64(t)[~inside] == 7.0).all()
    for t, b in ((o, ob), (lse, lb), (dqkv, db)):
        assert guard_intact(b, t.numel())


@pytest.mark.parametrize("d", [64, 80, 128])
def test_attention_of_large_logits(d):
    """Logits that spread over hundreds: the maximum moves from tile to tile."""
    heads, cu = 2, [0, 300]
    announce(f"packed attention large logits d={d}")
    qkv, do, inside = _attn_inputs(cu, 300, heads, heads, d, 21, scale=6.0)
    x = f64(qkv)
    x[:, heads * d:2 * heads * d] *= np.linspace(0.1, 1.0, 300)[:, None]
    qkv = torch.tensor(x).to(BF)
    plan = _plan(cu, 300)
    o, lse = B.enc_attn_packed_fwd(1, heads, heads, d, cuda(qkv), plan)
    dqkv = B.enc_attn_packed_bwd(1, heads, heads, d, cuda(qkv), o, lse, cuda(do), plan)
    ref, rlse, bound, lbound = P.packed_attention_fwd(f64(qkv), cu, heads, heads, d, False)
    within(o, ref, bound)
    within(lse, rlse, lbound)
    ref, bound = P.packed_attention_bwd(f64(qkv), cu, heads, heads, d, False, f64(do))
    within(dqkv, ref, bound)


@pytest.mark.parametrize("heads,kv,d", [(2, 2, 64), (4, 1, 80), (3, 1, 128)])
def test_causal_attention_whose_unseen_logits_overflow(heads, kv, d):
    """Keys that grow within each tile of 32: those that a query does not see exceed its
    log-sum-exp by so much that their weights, formed before the mask, are infinite."""
    T, cu = 300, [0, 300]
    announce(f"packed causal attention heads={heads}/{kv} d={d} large unseen logits")
    qkv, do, _ = _attn_inputs(cu, T, heads, kv, d, 25, scale=10.0)
    x = qkv.view(T, heads + 2 * kv, d)
    x[:, heads:heads + kv] *= ((torch.arange(T) % 32 + 1) / 32).to(BF)[:, None, None]
    plan = _plan(cu, T)
    o, lse = B.enc_attn_packed_fwd(1, heads, kv, d, cuda(qkv), plan, True)
    dqkv = B.enc_attn_packed_bwd(1, heads, kv, d, cuda(qkv), o, lse, cuda(do), plan, True)
    ref, rlse, bound, lbound = P.packed_attention_fwd(f64(qkv), cu, heads, kv, d, True)
    v = f64(x)
    for h in range(heads):
        over = v[:32, h] @ v[:32, heads + h // (heads // kv)].T / np.sqrt(d) - rlse[h, :32, None]
        assert (np.triu(over, 1) > 129 * np.log(2)).any()
    within(o, ref, bound)
    within(lse, rlse, lbound)
    ref, bound = P.packed_attention_bwd(f64(qkv), cu, heads, kv, d, True, f64(do))
    # Gradients go down to 1e-90 here, where the oracle's bounds, relative to the terms,
    # know no smallest number.  A weight P below 2^-126 is dropped, which is off by less
    # than that; dS = P (dP - D), |dP - D| <= E, is then off by 2^-126 E, and by 2^-126
    # once more where it is dropped itself; and a product of P or dS with an element of
    # at most X, or the result of the n of them that are added, by 2^-126 where it is.
    n, X = T * (heads // kv), max(np.abs(v).max(), np.abs(f64(do)).max())
    E = 2 * np.abs(f64(do)).reshape(T, heads, d).sum(2).max() * np.abs(v[:, heads + kv:]).max()
    within(dqkv, ref, bound + 2.0 ** -126 * (n * ((1 + E) * X + 1) + 1))


@pytest.mark.parametrize("low", [torch.finfo(BF).min, float("-inf")])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,d", [(2, 2, 64), (4, 1, 80), (2, 1, 128)])
def test_leading_keys_with_logits_of_minus_infinity(heads, kv, d, causal, low):
    """The first 72 keys' logits are -inf (beyond fp32, with the lowest bf16 value): for
    every query after them two whole tiles and a part of one weigh nothing."""
    T, lead = 150, 72
    announce(f"packed attention heads={heads}/{kv} d={d} causal={causal} leading keys {low}")
    qkv, do, _ = _attn_inputs([0, T], T, heads, kv, d, 23)
    x = qkv.view(T, heads + 2 * kv, d)
    x[:, :heads, 0] = 16.0
    x[:lead, heads:heads + kv] = 0.0
    x[:lead, heads:heads + kv, 0] = low
    plan = _plan([0, T], T)
    o, lse = B.enc_attn_packed_fwd(1, heads, kv, d, cuda(qkv), plan, causal)
    v = f64(x)
    rows = slice(lead, T) if causal else slice(0, T)  # (with causal the others see no finite logit)
    seen = np.tril(np.ones((T, T), dtype=bool)) if causal else np.ones((T, T), dtype=bool)
    seen[:, :lead] = False
    for h in range(heads):
        q, k, w = v[:, h], v[lead:, heads + h // (heads // kv)], v[lead:, heads + kv + h // (heads // kv)]
        s = np.where(seen[:, lead:], q @ k.T / np.sqrt(d), -np.inf)[rows]
        m = s.max(1, keepdims=True)
        p = np.exp(s - m)
        total = p.sum(1, keepdims=True)
        p /= total
        # the oracle's bounds, over the keys that weigh something
        size = (np.abs(q[rows]) @ np.abs(k).T / np.sqrt(d)).max(1, keepdims=True)
        ds = P.FP32 * ((d + 4) * size + 4 * np.abs(m) + 8)
        ref, rlse = p @ w, (m + np.log(total))[:, 0]
        bound = (P.BF16 + 2 * ds + 2 * (T + 16) * P.FP32) * (p @ np.abs(w)) + P.BF16 * np.abs(ref) * (1 + P.BF16)
        within(o[rows, h * d:(h + 1) * d], ref, bound)
        within(lse[h, rows], rlse, (2 * ds + (T + 16) * P.FP32)[:, 0] + 4 * P.FP32 * np.abs(rlse))
    if causal or low == float("-inf"):  # (0 times -inf in the backward's products)
        return
    dqkv = B.enc_attn_packed_bwd(1, heads, kv, d, cuda(qkv), o, lse, cuda(do), plan)
    got = f64(dqkv).reshape(T, heads + 2 * kv, d)
    assert np.isfinite(got).all() and (got[:lead, heads:] == 0).all()


@pytest.mark.parametrize("heads,kv,d", [(2, 2, 64), (4, 1, 80), (2, 1, 128)])
def test_a_later_token_reaches_no_earlier_tile(heads, kv, d):
    """With causal attention, non-finite keys and values from token 200 on leave the
    queries of the 32-token tiles before it as they are."""
    announce(f"packed attention heads={heads}/{kv} d={d} non-finite later tokens")
    qkv, _, _ = _attn_inputs([0, 300], 300, heads, kv, d, 27)
    plan = _plan([0, 300], 300)
    want, wlse = B.enc_attn_packed_fwd(1, heads, kv, d, cuda(qkv), plan, True)
    for bad in (float("inf"), float("-inf"), float("nan")):
        qkv[200:, heads * d:] = bad
        o, lse = B.enc_attn_packed_fwd(1, heads, kv, d, cuda(qkv), plan, True)
        assert torch.equal(o[:192], want[:192]) and torch.equal(lse[:, :192], wlse[:, :192])


def test_attention_equals_the_dense_kernels_results():
    """One batch of equal sequences: the dense entry points' numbers, up to the
    order of fp32 sums."""
    b, s, heads, d = 3, 197, 12, 64
    announce("packed attention against dense")
    qkv, do = cuda(random_bf16((b * s, 3 * heads * d), 31)), cuda(random_bf16((b * s, heads * d), 32))
    o, lse = B.enc_attn_fwd(b, s, heads, d, qkv)
    dqkv = B.enc_attn_bwd(b, s, heads, d, qkv, o, lse, do)
    plan = _plan([i * s for i in range(b + 1)], b * s)
    po, plse = B.enc_attn_packed_fwd(b, heads, heads, d, qkv, plan)
    pdqkv = B.enc_attn_packed_bwd(b, heads, heads, d, qkv, po, plse, do, plan)
    assert max_rel(f64(po), f64(o)) < 2 ** -6 and max_rel(f64(pdqkv), f64(dqkv)) < 2 ** -6
    assert max_rel(f64(plse), f64(lse.permute(1, 0, 2).reshape(heads, -1))) < 1e-5


def test_attention_is_deterministic_and_replays_from_a_graph():
    lens = [333, 64, 0, 1, 517]
    cu = [0] + [int(x) for x in np.cumsum(lens)]
    heads, kv, d, T = 8, 4, 80, cu[-1]
    announce("packed attention determinism and graph")
    qkv, do, _ = _attn_inputs(cu, T, heads, kv, d, 41)
    qkv, do = cuda(qkv), cuda(do)
    cug = torch.tensor(cu, dtype=torch.int32, device="cuda")
    plan = B.enc_packed_plan(cug, T)
    o, lse = B.enc_attn_packed_fwd(5, heads, kv, d, qkv, plan)
    ws = torch.empty(B.attn_packed_bwd_workspace_bytes(T, heads), dtype=torch.uint8, device="cuda")
    dqkv = B.enc_attn_packed_bwd(5, heads, kv, d, qkv, o, lse, do, plan, ws=ws)
    bits = lambda *ts: [t.clone().view(torch.int16 if t.dtype == BF else torch.int32) for t in ts]  # noqa: E731
    want = bits(o, lse, dqkv)
    plan2, o2, lse2, dqkv2 = (torch.empty_like(t) for t in (plan, o, lse, dqkv))
    pos = torch.randint(0, 100, (T, 3), dtype=torch.int32, device="cuda")
    freq, sec = torch.rand(d // 2, device="cuda"), (10, 15, 15)
    roped = torch.empty_like(qkv)

    def chain(stream):
        B.enc_rope_fwd(heads, kv, d, qkv, pos, freq, sec, qkvr=roped, stream=stream)
        B.enc_packed_plan(cug, T, plan=plan2, stream=stream)
        B.enc_attn_packed_fwd(5, heads, kv, d, qkv, plan2, o=o2, lse=lse2, stream=stream)
        B.enc_attn_packed_bwd(5, heads, kv, d, qkv, o2, lse2, do, plan2, dqkv=dqkv2, ws=ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    chain(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(bits(o2, lse2, dqkv2), want))
    want_roped = bits(roped)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(torch.cuda.current_stream())
    for _ in range(3):
        for t in (o2, lse2, dqkv2, roped):
            t.fill_(0.5)
        plan2.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bits(o2, lse2, dqkv2, roped), want + want_roped))
        B.enc_attn_packed_fwd(5, heads, kv, d, qkv, plan)  # eager work between the replays
        torch.cuda.synchronize()


def test_a_stream_of_the_callers_gets_memory_of_its_own():
    """Outputs and workspaces of a call on another stream lie in none of the current
    stream's memory: there the writes of a freed tensor may still be on their way."""
    heads, d, T = 16, 128, 4096
    announce("packed attention on a side stream, outputs not given")
    qkv, do = cuda(random_bf16((T, 3 * heads * d), 43)), cuda(random_bf16((T, heads * d), 44))
    plan = _plan([0, T], T)
    o, lse = B.enc_attn_packed_fwd(1, heads, heads, d, qkv, plan)
    dqkv = B.enc_attn_packed_bwd(1, heads, heads, d, qkv, o, lse, do, plan)
    y, w = do[:256].contiguous(), cuda(random_bf16((4096, heads * d), 45))
    gu, h = B.enc_glu_up_fwd(y, w)
    torch.cuda.synchronize()
    want = [t.cpu() for t in (o, lse, dqkv, gu, h)]
    shapes = [(t.shape, t.dtype) for t in (o, lse, dqkv, gu, h)]
    side = torch.cuda.Stream()
    old = [torch.empty(s, dtype=t, device="cuda") for s, t in shapes]
    for _ in range(200):
        for t in old:
            t.fill_(1.5)
    del old, t
    po, plse = B.enc_attn_packed_fwd(1, heads, heads, d, qkv, plan, stream=side)
    pdqkv = B.enc_attn_packed_bwd(1, heads, heads, d, qkv, po, plse, do, plan, stream=side)
    pgu, ph = B.enc_glu_up_fwd(y, w, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(t.cpu(), v) for t, v in zip((po, plse, pdqkv, pgu, ph), want))


def test_tensors_of_another_device_are_refused(monkeypatch):
    """(This process has one device: the current one is made to look like another.)"""
    qkv = cuda(random_bf16((4, 3 * 64), 46))
    plan = _plan([0, 4], 4)
    o, lse = B.enc_attn_packed_fwd(1, 1, 1, 64, qkv, plan)
    torch.cuda.synchronize()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    x, w = o, torch.zeros(16, 64, dtype=BF, device=o.device)
    pos, freq = torch.zeros(4, 3, dtype=torch.int32, device=o.device), torch.ones(32, device=o.device)
    cu = torch.tensor([0, 4], dtype=torch.int32, device=o.device)
    side = torch.cuda.Stream(device=0)
    for call in (lambda s: B.enc_rope_fwd(1, 1, 64, qkv, pos, freq, (8, 8, 8), stream=s),
                 lambda s: B.enc_rope_bwd(1, 1, 64, qkv, pos, freq, (8, 8, 8), stream=s),
                 lambda s: B.enc_packed_plan(cu, 4, stream=s),
                 lambda s: B.enc_attn_packed_fwd(1, 1, 1, 64, qkv, plan, stream=s),
                 lambda s: B.enc_attn_packed_bwd(1, 1, 1, 64, qkv, o, lse, o, plan, stream=s),
                 lambda s: B.enc_glu_up_fwd(x, w, stream=s),
                 lambda s: B.enc_glu_down_bwd_data(x, w[:8].t().contiguous(), torch.cat([x, x])[:4, :16].contiguous(),
                                                   stream=s),
                 lambda s: B.enc_glu_up_bwd_data(x[:, :16].contiguous(), w, stream=s),
                 lambda s: B.enc_glu_up_bwd_weight(x[:, :16].contiguous(), x, torch.zeros(16, 64, device=o.device),
                                                   stream=s)):
        for s in (None, side):
            with pytest.raises(ValueError, match="the current device is 1"):
                call(s)


def test_attention_at_the_end_of_the_largest_tensor():
    """The last rows of a qkv of nearly 2^31 elements (4 GiB), whose last tile
    would reach past 32-bit byte offsets."""
    heads, d = 48, 128
    width = 3 * heads * d
    T = (2 ** 31 - 1) // width
    announce(f"packed attention at the end of {T} rows")
    cu = [T - 160, T - 100, T]
    n = T - cu[0]
    part = random_bf16((n, width), 51)
    dpart = random_bf16((n, heads * d), 52)
    qkv = torch.zeros(T, width, dtype=BF, device="cuda")
    do = torch.zeros(T, heads * d, dtype=BF, device="cuda")
    qkv[cu[0]:], do[cu[0]:] = cuda(part), cuda(dpart)
    plan = _plan(cu, T)
    o, lse = B.enc_attn_packed_fwd(2, heads, heads, d, qkv, plan)
    dqkv = B.enc_attn_packed_bwd(2, heads, heads, d, qkv, o, lse, do, plan)
    local = [c - cu[0] for c in cu]
    ref, rlse, bound, lbound = P.packed_attention_fwd(f64(part), local, heads, heads, d, False)
    within(o[cu[0]:], ref, bound)
    within(lse[:, cu[0]:], rlse, lbound)
    ref, bound = P.packed_attention_bwd(f64(part), local, heads, heads, d, False, f64(dpart))
    within(dqkv[cu[0]:], ref, bound)


def test_attention_of_a_sequence_beyond_2_gib():
    """One sequence whose rows span more than 2^31 bytes, heads of 80, whose tiles' last
    columns lie past the head: queries and keys from its first to its last rows, in
    64 bits from the kernel's own log-sum-exp."""
    heads, kv, d, T = 96, 24, 80, 100003
    A, W = heads * d, (heads + 2 * kv) * d
    assert T * W * 2 > 2 ** 31
    announce(f"packed attention of one sequence of {T} rows, {T * W * 2} bytes")
    g = torch.Generator(device="cuda").manual_seed(61)
    qkv = torch.randn(T, W, generator=g, dtype=BF, device="cuda")
    do = torch.randn(T, A, generator=g, dtype=BF, device="cuda")
    plan = _plan([0, T], T)
    o, lse = B.enc_attn_packed_fwd(1, heads, kv, d, qkv, plan)
    dqkv = B.enc_attn_packed_bwd(1, heads, kv, d, qkv, o, lse, do, plan)
    rows = torch.tensor([0, 1, 46603, 93206, 93207, 99999, T - 1], device="cuda")
    n, F = T, P.FP32
    for h in (0, heads - 1):
        j = h // (heads // kv)
        col = lambda t, i: t[:, i * d:(i + 1) * d].double()  # noqa: E731
        q, k, v, dh, oh = col(qkv, h), col(qkv, heads + j), col(qkv, heads + kv + j), col(do, h), col(o, h)
        s = q[rows] @ k.t() / d ** 0.5
        size = (q[rows].abs() @ k.abs().t() / d ** 0.5).amax(1, keepdim=True)
        rlse = torch.logsumexp(s, 1)
        p = (s - rlse[:, None]).exp()
        # the oracle's bounds (oracle/packed.py)
        ds = F * ((d + 4) * size + 4 * s.amax(1, keepdim=True).abs() + 8)
        ro, lb = p @ v, (2 * ds + (n + 16) * F)[:, 0] + 4 * F * rlse.abs()
        ob = (P.BF16 + 2 * ds + 2 * (n + 16) * F) * (p @ v.abs()) + P.BF16 * ro.abs() * (1 + P.BF16)
        within(o[rows, h * d:(h + 1) * d], f64(ro), f64(ob))
        within(lse[h, rows], f64(rlse), f64(lb))
        rel = F * ((d + 4) * size + 8 * rlse[:, None].abs() + 8) + lb[:, None]
        dP, D = dh[rows] @ v.t(), (dh[rows] * ro).sum(1, keepdim=True)
        e = p * (dP - D)
        edd = (dh[rows].abs() * (ob + (d + 4) * F * ro.abs())).sum(1, keepdim=True)
        eds = (P.BF16 + rel) * e.abs() + p * (1 + rel) * ((d + 4) * F * (dh[rows].abs() @ v.abs().t()) + edd)
        ref, b = e @ k / d ** 0.5, (eds + (n + 16) * F * e.abs()) @ k.abs() / d ** 0.5
        within(dqkv[rows, h * d:(h + 1) * d], f64(ref), f64(b + P.BF16 * (ref.abs() + b)))
    # dK and dV of these rows, over the queries of the four heads that share them, from the
    # kernel's own o and lse
    for j in (0, kv - 1):
        dk, dv = torch.zeros(len(rows), d, dtype=torch.float64, device="cuda"), None
        dv, kb, vb = dk.clone(), dk.clone(), dk.clone()
        k, v = col(qkv, heads + j)[rows], col(qkv, heads + kv + j)[rows]
        for h in range(j * heads // kv, (j + 1) * heads // kv):
            q, dh, oh, L = col(qkv, h), col(do, h), col(o, h), lse[h].double()
            s = q @ k.t() / d ** 0.5
            p = (s - L[:, None]).exp()
            dP, D = dh @ v.t(), (dh * oh).sum(1, keepdim=True)
            e = p * (dP - D)
            rel = F * ((d + 4) * (q.abs() @ k.abs().t() / d ** 0.5) + 12 * L.abs()[:, None] + 8)
            eds = (P.BF16 + rel) * e.abs() + p * (1 + rel) * (d + 4) * F * (
                dh.abs() @ v.abs().t() + (dh.abs() * oh.abs()).sum(1, keepdim=True))
            add = (heads // kv * n + 16) * F
            dk += e.t() @ q / d ** 0.5
            dv += p.t() @ dh
            kb += (eds + add * e.abs()).t() @ q.abs() / d ** 0.5
            vb += ((P.BF16 + rel + add) * p).t() @ dh.abs()
        for i, ref, b in ((heads + j, dk, kb), (heads + kv + j, dv, vb)):
            within(dqkv[rows, i * d:(i + 1) * d], f64(ref), f64(b + P.BF16 * (ref.abs() + b)))


# ------------------------------------------------------------------ a packed layer

@pytest.mark.parametrize("heads,kv,d,act", [(3, 3, 64, "silu"), (4, 1, 80, "gelu")])
def test_packed_layer(heads, kv, d, act):
    """One pre-LN layer on a packed batch: LN, QKV projection, rotary positions,
    packed attention, out-projection, LN, gated feed-forward; forward and
    backward against the oracle's chain, from the same inputs."""
    H, F = 256, 344
    lens = [50, 1, 130, 0, 17]
    cu = [0] + [int(x) for x in np.cumsum(lens)]
    T, A, W = cu[-1], heads * d, (heads + 2 * kv) * d
    announce(f"packed layer heads={heads}/{kv} d={d} {act}")
    std = 0.05
    shapes = dict(ln1_g=(H,), ln1_b=(H,), w_qkv=(W, H), b_qkv=(W,), w_o=(H, A), b_o=(H,), ln2_g=(H,), ln2_b=(H,),
                  w_gu=(2 * F, H), b_gu=(2 * F,), w_2=(H, F), b_2=(H,))
    p = {n: (random_bf16(s, 60 + i).float() * std + (1.0 if n in ("ln1_g", "ln2_g") else 0.0)).to(BF)
         for i, (n, s) in enumerate(shapes.items())}
    x, dout = random_bf16((T, H), 90), random_bf16((T, H), 91)
    sec = (d // 8, d // 4, d // 8)
    pos = torch.stack([torch.arange(T) // 64, torch.arange(T) % 64 // 8, torch.arange(T) % 8], 1).to(torch.int32)
    freq = torch.tensor([100.0 ** (-i / (d // 2)) for i in range(d // 2)], dtype=torch.float32)
    eps, actc = 1e-6, B.GLU_SILU if act == "silu" else B.GLU_GELU
    # ---- the library
    g = {n: cuda(t) for n, t in p.items()}
    gx, gd, gpos, gf, plan = cuda(x), cuda(dout), cuda(pos), cuda(freq), _plan(cu, T)
    y1, m1, r1 = B.enc_ln_fwd(gx, g["ln1_g"], g["ln1_b"], eps)
    qkv = B.enc_qkv_fwd(y1, g["w_qkv"], g["b_qkv"])
    B.enc_rope_fwd(heads, kv, d, qkv, gpos, gf, sec, qkvr=qkv)
    o, lse = B.enc_attn_packed_fwd(len(lens), heads, kv, d, qkv, plan)
    h1 = B.enc_oproj_fwd(o, g["w_o"], g["b_o"], gx)
    y2, m2, r2 = B.enc_ln_fwd(h1, g["ln2_g"], g["ln2_b"], eps)
    gu, h = B.enc_glu_up_fwd(y2, g["w_gu"], g["b_gu"], act=actc)
    out = B.enc_mlp_down_fwd(h, g["w_2"], g["b_2"], h1)
    f32 = lambda n: torch.empty(shapes[n], dtype=torch.float32, device="cuda")  # noqa: E731
    gr = {n: f32(n) for n in shapes}
    dgu = B.enc_glu_down_bwd_data(gd, g["w_2"], gu, act=actc)
    B.enc_mlp_down_bwd_weight(gd, h, gr["w_2"], gr["b_2"])
    dy2 = B.enc_glu_up_bwd_data(dgu, g["w_gu"])
    B.enc_glu_up_bwd_weight(dgu, y2, gr["w_gu"], gr["b_gu"])
    dh1, _, _ = B.enc_ln_bwd(dy2, h1, m2, r2, g["ln2_g"], gd, dgamma=gr["ln2_g"], dbeta=gr["ln2_b"])
    do = B.enc_oproj_bwd_data(dh1, g["w_o"])
    B.enc_oproj_bwd_weight(dh1, o, gr["w_o"], gr["b_o"])
    dqkv = B.enc_attn_packed_bwd(len(lens), heads, kv, d, qkv, o, lse, do, plan)
    B.enc_rope_bwd(heads, kv, d, dqkv, gpos, gf, sec, dqkv=dqkv)
    dy1 = B.enc_qkv_bwd_data(dqkv, g["w_qkv"])
    B.enc_qkv_bwd_weight(dqkv, y1, gr["w_qkv"], gr["b_qkv"])
    dx, _, _ = B.enc_ln_bwd(dy1, gx, m1, r1, g["ln1_g"], dh1, dgamma=gr["ln1_g"], dbeta=gr["ln1_b"])
    torch.cuda.synchronize()
    # ---- the oracle
    q = {n: f64(t) for n, t in p.items()}
    X, D, npos, nf = f64(x), f64(dout), pos.numpy(), freq.numpy()
    Y1, M1, R1 = oracle.layernorm_fwd(X, q["ln1_g"], q["ln1_b"], eps)
    QKV = P.rope(Y1 @ q["w_qkv"].T + q["b_qkv"], heads, kv, d, npos, nf, sec, False)
    O = P.packed_attention_fwd(QKV, cu, heads, kv, d, False)[0]  # noqa: E741
    H1 = X + O @ q["w_o"].T + q["b_o"]
    Y2, M2, R2 = oracle.layernorm_fwd(H1, q["ln2_g"], q["ln2_b"], eps)
    GU, HH, _, _ = P.glu_fwd(Y2, q["w_gu"], q["b_gu"], act)
    OUT = H1 + HH @ q["w_2"].T + q["b_2"]
    G = {}
    DGU = P.glu_bwd(D, q["w_2"], GU, act)[0]
    G["w_2"], G["b_2"] = D.T @ HH, D.sum(0)
    G["w_gu"], G["b_gu"] = DGU.T @ Y2, DGU.sum(0)
    dH1, G["ln2_g"], G["ln2_b"] = oracle.layernorm_bwd(DGU @ q["w_gu"], H1, M2, R2, q["ln2_g"])
    dH1 = dH1 + D
    G["w_o"], G["b_o"] = dH1.T @ O, dH1.sum(0)
    DQKV = P.packed_attention_bwd(QKV, cu, heads, kv, d, False, dH1 @ q["w_o"])[0]
    DQKV = P.rope(DQKV, heads, kv, d, npos, nf, sec, False, back=True)
    G["w_qkv"], G["b_qkv"] = DQKV.T @ Y1, DQKV.sum(0)
    DX, G["ln1_g"], G["ln1_b"] = oracle.layernorm_bwd(DQKV @ q["w_qkv"], X, M1, R1, q["ln1_g"])
    DX = DX + dH1
    for n, got, ref in (("qkv", qkv, QKV), ("o", o, O), ("h1", h1, H1), ("gu", gu, GU), ("h", h, HH), ("out", out, OUT)):
        assert max_rel(f64(got), ref) < TOL_ACT, n
    for n, got, ref in [("dgu", dgu, DGU), ("dqkv", dqkv, DQKV), ("dx", dx, DX)] + [(n, gr[n], G[n]) for n in shapes]:
        assert max_rel(f64(got), ref) < TOL_GRAD, n


@pytest.mark.parametrize("heads,kv,d,act", [(8, 1, 64, "silu"), (12, 4, 80, "gelu"), (4, 2, 128, "silu")])
def test_packed_layer_whose_qkv_is_no_multiple_of_3_wide(heads, kv, d, act):
    assert (heads + 2 * kv) % 3
    test_packed_layer(heads, kv, d, act)
