"""The work of a packed-sequence encoder layer's own operators, as measurable cases.

Encoders that take images, video and text of any size lay the sequences of a
micro-batch end to end without padding, place their tokens with rotary
positions of several axes and use a gated feed-forward block.  `kind`:

  rope   rotary positions (time, height, width) on the queries and keys of a
         packed qkv, forward or backward
  attn   attention within each sequence of a packed batch: the forward, or the
         forward and the backward (`step`)
  glu    a gated feed-forward block's up-projections with their activation and
         product, or (`bwd`) the input gradients of its down- and up-projections

`run` computes them from the formulas in elementary operations, and where `own`
is set with the library's kernels.
"""

import math
import random

import torch

own = False

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


# ------------------------------------------------------------------ cases

def _rope(name, tokens, heads, kv_heads, head_dim, sections, pairs, bwd, far):
    t, h, w = sections
    return dict(name=name, kind="rope", tokens=tokens, heads=heads, kv_heads=kv_heads, head_dim=head_dim, sec_t=t,
                sec_h=h, sec_w=w, interleaved=pairs == "interleaved", bwd=bwd, far=far)


def _attn(name, lens, pad, heads, kv_heads, head_dim, causal, step):
    return dict(name=name, kind="attn", lens=",".join(map(str, lens)), pad=pad, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, causal=causal, step=step)


def _glu(name, rows, hidden, mlp, act, bias, save, bwd):
    return dict(name=name, kind="glu", rows=rows, hidden=hidden, mlp=mlp, act=act, bias=bias, save=save, bwd=bwd)


def _lens(seed, n, lo, hi):
    """n sequence lengths between lo and hi, spread over their logarithm."""
    r = random.Random(seed)
    return [_logint(r, lo, hi) for _ in range(n)]


def listed():
    return [
        # One 224-pixel image of a ViT-Huge encoder (256 patches and a class
        # token), positions by row and column: a few microseconds, latency.
        _rope("rope_fwd_one_image", 257, 16, 16, 80, (0, 20, 20), "halves", False, 16),
        # Video clips at ViT-22B's attention width, all three axes; clips from
        # far into a long recording.
        _rope("rope_fwd_video", 8192, 48, 48, 128, (16, 24, 24), "halves", False, 1 << 20),
        # Backward of a ViT-Base batch of images of several sizes.
        _rope("rope_bwd_images", 5003, 12, 12, 64, (0, 16, 16), "interleaved", True, 64),
        # Backward with shared key heads and four pairs that no axis turns.
        _rope("rope_bwd_grouped", 12289, 32, 8, 128, (16, 24, 20), "interleaved", True, 4096),
        # A handful of short texts for a small encoder, one of them a single
        # token and one empty: the smallest call.
        _attn("attn_fwd_few_tokens", [17, 1, 0, 9, 30], 0, 12, 12, 64, False, False),
        # A text encoder serving a batch of prompts: causal, shared key heads.
        _attn("attn_fwd_text_causal", _lens(1, 24, 30, 2048), 0, 32, 8, 128, True, False),
        # Training on 40 images from 8 x 8 to 32 x 32 patches (ViT-Huge heads),
        # with the batch's last rows unused.
        _attn("attn_step_images", _lens(2, 40, 64, 1024), 77, 16, 16, 80, False, True),
        # Training on one long video clip, a still and a single token
        # (1/3 of ViT-22B's heads): the largest.
        _attn("attn_step_video", [7936, 515, 1], 0, 16, 16, 128, False, True),
        # One token through a ViT-Huge sized block, served: reading the weights.
        _glu("glu_fwd_one_token", 1, 1280, 3416, "silu", False, False, False),
        # A ViT-22B sized block in training, 2048 tokens.
        _glu("glu_fwd_22b", 2048, 6144, 16384, "silu", False, True, False),
        # Input gradients of a ViT-Huge sized block, a ragged number of tokens
        # and of columns, GELU gate.
        _glu("glu_bwd_images", 5003, 1280, 3416, "gelu", True, True, True),
        # Input gradients on one GPU's 1/8 tensor-parallel shard of the ViT-22B
        # sized block.
        _glu("glu_bwd_22b_tp8", 2048, 6144, 2048, "silu", False, True, True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width between lo and hi: a multiple of 64 mostly, of 8 now and then."""
    q = 64 if rng.random() < 0.75 else 8
    return max(1, round(_logint(rng, lo, hi) / q)) * q


def _heads(rng, most):
    heads = _logint(rng, 1, most)
    group = rng.choice([g for g in (1, 1, 1, 2, 4, 8) if heads % g == 0])
    return heads, heads // group


def _draw_once(rng):
    kind = rng.choice(["rope", "attn", "attn", "glu", "glu"])
    head_dim = rng.choice([64, 80, 128])
    heads, kv_heads = _heads(rng, 48)
    if kind == "rope":
        half = head_dim // 2
        t = rng.choice([0, half // 4])
        h = rng.randint(0, half - t)
        w = rng.randint(0, half - t - h) if rng.random() < 0.3 else half - t - h
        return _rope("", _logint(rng, 1, 16384), heads, kv_heads, head_dim, (t, h, w),
                     rng.choice(["halves", "interleaved"]), rng.random() < 0.5, _logint(rng, 2, 1 << 20))
    if kind == "attn":
        n, hi = _logint(rng, 1, 64), _logint(rng, 4, 8192)
        lo = _logint(rng, 1, hi)
        lens = [0 if rng.random() < 0.03 else _logint(rng, lo, hi) for _ in range(n)]
        return _attn("", lens, rng.choice([0, 0, rng.randint(1, 200)]), heads, kv_heads, head_dim,
                     rng.random() < 0.4, rng.random() < 0.6)
    hidden = _width(rng, 192, 6144)
    return _glu("", _logint(rng, 1, 8192), hidden, _width(rng, 256, 4 * hidden), rng.choice(["silu", "silu", "gelu"]),
                rng.random() < 0.4, rng.random() < 0.7, rng.random() < 0.5)


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        m = most.setdefault(c["kind"], [0, 0])
        m[0], m[1] = max(m[0], w["flops"]), max(m[1], w["bytes"])
    while True:
        case = _draw_once(rng)
        case.pop("name")
        w = work(case)
        if w["flops"] > most[case["kind"]][0] or w["bytes"] > most[case["kind"]][1]:
            continue
        if case["kind"] == "attn":  # the plain form pads every sequence to the longest
            lens = _case_lens(case)
            if sum(lens) == 0 or len(lens) * case["heads"] * max(lens) ** 2 > 2.5e9:
                continue
        return case


def _case_lens(case):
    return [int(v) for v in case["lens"].split(",")]


# ------------------------------------------------------------------ inputs

class _Rand:
    """Seeded normal draws on the GPU, rounded once to bf16."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def __call__(self, shape, std=1.0):
        t = torch.randn(shape, generator=self.g, dtype=F32, device="cuda")
        return t.mul_(std).to(BF)


def _inv_freq(case):
    """Frequency of each pair: each axis has a geometric series of its own, and
    the pairs of no axis have none."""
    f = []
    for n in (case["sec_t"], case["sec_h"], case["sec_w"]):
        f += [10000.0 ** (-i / n) for i in range(n)]
    f += [0.0] * (case["head_dim"] // 2 - len(f))
    return torch.tensor(f, dtype=F32, device="cuda")


def _sections(case):
    return case["sec_t"], case["sec_h"], case["sec_w"]


def _inputs(case, seed):
    """The random inputs of a case, the same for the kernels and for exact()."""
    rnd = _Rand(seed)
    kind = case["kind"]
    if kind == "glu":
        M, H, F = case["rows"], case["hidden"], case["mlp"]
        if case["bwd"]:
            return dict(dout=rnd((M, H)), w_2=rnd((H, F), 0.02), gu=rnd((M, 2 * F)), w_gu=rnd((2 * F, H), 0.02))
        return dict(y=rnd((M, H)), w_gu=rnd((2 * F, H), 0.02), b_gu=rnd((2 * F,), 0.02) if case["bias"] else None)
    heads, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
    width = (heads + 2 * kv) * d
    if kind == "rope":
        M, far = case["tokens"], case["far"]
        # frames of 16 x 16 patches in order, starting at a random frame
        i = torch.arange(M, device="cuda")
        t0 = torch.randint(0, far, (1,), generator=rnd.g, device="cuda")
        pos = torch.stack([i // 256 + t0, i % 256 // 16, i % 16], 1).to(torch.int32)
        return dict(x=rnd((M, width)), pos=pos, inv_freq=_inv_freq(case))
    lens = _case_lens(case)
    M = sum(lens) + case["pad"]
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    inp = dict(qkv=rnd((M, width)), cu=torch.tensor(cu, dtype=torch.int32, device="cuda"))
    if case["step"]:
        inp["do"] = rnd((M, heads * d))
    return inp


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    if case["kind"] == "attn":
        lens = _case_lens(case)
        heads, d, M = case["heads"], case["head_dim"], st["qkv"].shape[0]
        # outputs that the program keeps: rows behind the last sequence stay zero
        st["o"] = torch.zeros(M, heads * d, dtype=BF, device="cuda")
        st["lse"] = torch.zeros(heads, M, dtype=F32, device="cuda")
        if case["step"]:
            st["dqkv"] = torch.zeros_like(st["qkv"])
        if own:
            from paper_2408_03505_amd import binding as B
            st["plan"] = B.enc_packed_plan(st["cu"], M)
            if case["step"]:
                st["ws"] = torch.empty(B.attn_packed_bwd_workspace_bytes(M, heads), dtype=torch.uint8, device="cuda")
        else:
            # where each token lies in the sequences padded to the longest
            L = max(lens)
            s = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens))
            i = torch.arange(sum(lens)) - st["cu"].cpu().long()[s]
            st["slot"] = (s * L + i).cuda()
    elif case["kind"] == "glu" and own:
        from paper_2408_03505_amd import binding as B
        M, H, F = case["rows"], case["hidden"], case["mlp"]
        if case["bwd"]:
            need = max(B.glu_workspace_bytes(M, F, H), B.glu_workspace_bytes(M, H, 2 * F))
        else:
            need = B.glu_workspace_bytes(M, 2 * F, H)
        st["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    case = st["case"]
    if own:
        return _run_own(st)
    if case["kind"] == "rope":
        return dict(x=_rope_plain(case, st["x"], st["pos"], st["inv_freq"], F32).to(BF))
    if case["kind"] == "attn":
        return _attn_plain(st)
    if case["bwd"]:
        dgu = _glu_bwd(case, st["dout"].float(), st["w_2"].float(), st["gu"].float()).to(BF)
        return dict(dgu=dgu, dy=(dgu.float() @ st["w_gu"].float()).to(BF))
    gu, h = _glu_fwd(case, st["y"].float(), st["w_gu"].float(), st["b_gu"].float() if case["bias"] else None)
    return dict(gu=gu.to(BF), h=h.to(BF)) if case["save"] else dict(h=h.to(BF))


def _run_own(st):
    from paper_2408_03505_amd import binding as B
    case = st["case"]
    if case["kind"] == "glu":
        act = B.GLU_SILU if case["act"] == "silu" else B.GLU_GELU
        if case["bwd"]:
            dgu = B.enc_glu_down_bwd_data(st["dout"], st["w_2"], st["gu"], act=act, ws=st["ws"])
            return dict(dgu=dgu, dy=B.enc_glu_up_bwd_data(dgu, st["w_gu"], ws=st["ws"]))
        gu, h = B.enc_glu_up_fwd(st["y"], st["w_gu"], st["b_gu"], act=act, save=case["save"], ws=st["ws"])
        return dict(gu=gu, h=h) if case["save"] else dict(h=h)
    shape = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "rope":
        call = B.enc_rope_bwd if case["bwd"] else B.enc_rope_fwd
        return dict(x=call(*shape, st["x"], st["pos"], st["inv_freq"], _sections(case),
                           interleaved=case["interleaved"]))
    seqs = st["cu"].shape[0] - 1
    B.enc_attn_packed_fwd(seqs, *shape, st["qkv"], st["plan"], causal=case["causal"], o=st["o"], lse=st["lse"])
    if not case["step"]:
        return dict(o=st["o"], lse=st["lse"])
    B.enc_attn_packed_bwd(seqs, *shape, st["qkv"], st["o"], st["lse"], st["do"], st["plan"], causal=case["causal"],
                          dqkv=st["dqkv"], ws=st["ws"])
    return dict(o=st["o"], lse=st["lse"], dqkv=st["dqkv"])


# ------------------------------------------------------------------ plain forms

def _rope_plain(case, x, pos, inv_freq, dtype):
    """Each pair (a, b) of a query or key turned by its angle (backward: back)."""
    heads, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
    n = case["sec_t"], case["sec_h"], case["sec_w"]
    half, used, M = d // 2, sum(n), x.shape[0]
    axis = torch.tensor([0] * n[0] + [1] * n[1] + [2] * n[2] + [0] * (half - used), device=x.device)
    angle = pos.to(F64)[:, axis] * inv_freq.to(F64)  # far positions: 32 bits would lose the angle
    angle[:, used:] = 0
    cos, sin = angle.cos().to(dtype)[:, None], angle.sin().to(dtype)[:, None]
    sin = -sin if case["bwd"] else sin
    qk = x[:, :(heads + kv) * d].to(dtype).view(M, heads + kv, d)
    if case["interleaved"]:
        a, b = qk[..., 0::2], qk[..., 1::2]
        out = torch.stack([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = qk[..., :half], qk[..., half:]
        out = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([out.reshape(M, -1), x[:, (heads + kv) * d:].to(dtype)], 1)


def _padded(rows, slot, n, L, heads, d):
    """Packed rows [tokens, heads * d] as [n, heads, L, d], zero where there is none."""
    t = torch.zeros(n * L, heads * d, dtype=rows.dtype, device=rows.device)
    t[slot] = rows[:slot.shape[0]]
    return t.view(n, L, heads, d).transpose(1, 2)


def _packed(t, slot, out):
    """The rows of [n, heads, L, d] back into their places in `out`, rounded."""
    n, heads, L, d = t.shape
    out[:slot.shape[0]] = t.transpose(1, 2).reshape(n * L, heads * d)[slot].to(out.dtype)
    return out


def _attn_plain(st):
    case, slot = st["case"], st["slot"]
    heads, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
    g, scale = heads // kv, 1.0 / math.sqrt(d)
    lens = st["cu"][1:] - st["cu"][:-1]
    text = _case_lens(case)
    n, L = len(text), max(text)
    qkv = st["qkv"].float()
    q, k, v = qkv.split([heads * d, kv * d, kv * d], 1)
    q = _padded(q, slot, n, L, heads, d)
    k = _padded(k, slot, n, L, kv, d).repeat_interleave(g, 1)
    v = _padded(v, slot, n, L, kv, d).repeat_interleave(g, 1)
    j = torch.arange(L, device="cuda")
    # keys that a query sees: of its sequence, and with `causal` none after it;
    # a query past its sequence sees none
    seen = (j[None, None, :] < lens[:, None, None]) & (j[None, :, None] < lens[:, None, None])
    if case["causal"]:
        seen = seen & (j[None, None, :] <= j[None, :, None])
    seen = seen[:, None]
    s = (q @ k.transpose(-1, -2)).mul_(scale).masked_fill_(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total == 0, torch.ones_like(total), total)
    lse = m + torch.where(total == 0, torch.ones_like(total), total).log()
    out = dict(o=_packed(o, slot, torch.zeros_like(st["o"])))
    out["lse"] = torch.zeros_like(st["lse"])
    out["lse"][:, :slot.shape[0]] = lse[..., 0].transpose(0, 1).reshape(heads, n * L)[:, slot]
    if not case["step"]:
        return out
    del s, p, o, lse
    # backward, from the forward's o and lse
    lse = _padded(out["lse"].t(), slot, n, L, heads, 1)
    o = _padded(out["o"].float(), slot, n, L, heads, d)
    do = _padded(st["do"].float(), slot, n, L, heads, d)
    p = (q @ k.transpose(-1, -2)).mul_(scale).sub_(lse).exp_().masked_fill_(~seen, 0.0)
    dv = p.transpose(-1, -2) @ do
    ds = (do @ v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    del p
    dq = (ds @ k).mul_(scale)
    dk = (ds.transpose(-1, -2) @ q).mul_(scale)
    dk, dv = (t.reshape(n, kv, g, L, d).sum(2) for t in (dk, dv))
    dq, dk, dv = (_packed(t, slot, torch.zeros(st["qkv"].shape[0], t.shape[1] * d, dtype=BF, device="cuda"))
                  for t in (dq, dk, dv))
    out["dqkv"] = torch.cat([dq, dk, dv], 1)
    return out


def _act(case, g):
    """The gate's activation and its derivative."""
    if case["act"] == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    phi = 0.5 * (1.0 + torch.erf(g / math.sqrt(2.0)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def _glu_fwd(case, y, w_gu, b_gu):
    gu = y @ w_gu.t()
    if b_gu is not None:
        gu = gu + b_gu
    F = case["mlp"]
    return gu, _act(case, gu[:, :F])[0] * gu[:, F:]


def _glu_bwd(case, dout, w_2, gu):
    F = case["mlp"]
    dh = dout @ w_2
    a, da = _act(case, gu[:, :F])
    return torch.cat([dh * gu[:, F:] * da, dh * a], 1)


# ------------------------------------------------------------------ work

def work(case):
    """Inputs read once, outputs written once, and the products' operations (of
    attention: two in the forward, four in the backward, over the pairs of a
    query and a key that it sees)."""
    if case["kind"] == "glu":
        M, H, F = case["rows"], case["hidden"], case["mlp"]
        if case["bwd"]:
            return dict(bytes=2 * (2 * M * H + 3 * H * F + 4 * M * F), flops=6 * M * H * F)
        return dict(bytes=2 * (M * H + 2 * F * H + M * F * (3 if case["save"] else 1)), flops=4 * M * H * F)
    heads, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
    width = (heads + 2 * kv) * d
    if case["kind"] == "rope":
        M = case["tokens"]
        return dict(bytes=4 * M * width + 12 * M + 2 * d, flops=3 * M * (heads + kv) * d)
    lens = _case_lens(case)
    M = sum(lens)
    pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lens)
    fwd = 4 * pairs * d * heads
    read_write = 2 * M * width + 2 * M * heads * d + 4 * M * heads
    if not case["step"]:
        return dict(bytes=read_write, flops=fwd)
    return dict(bytes=read_write + 2 * M * heads * d + 2 * M * width, flops=3 * fwd)


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    inp = _inputs(case, seed)
    if case["kind"] == "rope":
        return dict(x=_exact_rope(case, inp))
    if case["kind"] == "attn":
        return _exact_attn(case, inp)
    F = case["mlp"]
    if case["bwd"]:
        g, u = (t.to(F64) for t in inp["gu"].split(F, 1))
        dh = inp["dout"].to(F64) @ inp["w_2"].to(F64)
        dgu = torch.empty(case["rows"], 2 * F, dtype=F64, device="cuda")
        if case["act"] == "silu":
            s = torch.sigmoid(g)
            dgu[:, :F], dgu[:, F:] = dh * u * (s + g * s * (1 - s)), dh * g * s
        else:
            c = torch.special.ndtr(g)
            dgu[:, :F] = dh * u * (c + g * torch.exp(-g * g / 2) * (2 * math.pi) ** -0.5)
            dgu[:, F:] = dh * g * c
        return dict(dgu=dgu, dy=dgu @ inp["w_gu"].to(F64))
    gu = inp["y"].to(F64) @ inp["w_gu"].to(F64).t()
    if case["bias"]:
        gu += inp["b_gu"].to(F64)
    g, u = gu.split(F, 1)
    h = u * g * (torch.sigmoid(g) if case["act"] == "silu" else torch.special.ndtr(g))
    return dict(gu=gu, h=h) if case["save"] else dict(h=h)


def _exact_rope(case, inp):
    heads, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
    x = inp["x"].to(F64)
    out = x.clone()
    sign = -1.0 if case["bwd"] else 1.0
    first = 0
    for axis, count in enumerate(_sections(case)):
        for i in range(first, first + count):
            ang = sign * inp["pos"][:, axis].to(F64) * inp["inv_freq"][i].to(F64)
            c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
            lo, hi = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + d // 2)
            lo = slice(lo, (heads + kv) * d, d)
            hi = slice(hi, (heads + kv) * d, d)
            out[:, lo] = x[:, lo] * c - x[:, hi] * s
            out[:, hi] = x[:, hi] * c + x[:, lo] * s
        first += count
    return out


def _exact_attn(case, inp):
    """Sequence by sequence and head by head."""
    heads, kv, d = case["heads"], case["kv_heads"], case["head_dim"]
    M = inp["qkv"].shape[0]
    o = torch.zeros(M, heads * d, dtype=F64, device="cuda")
    lse = torch.zeros(heads, M, dtype=F64, device="cuda")
    dqkv = torch.zeros(inp["qkv"].shape, dtype=F64, device="cuda")
    at = 0
    for n in _case_lens(case):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        later = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1) if case["causal"] else None
        for h in range(heads):
            def cols(base, i):
                return rows, slice((base + i) * d, (base + i + 1) * d)
            at_q, at_k, at_v = cols(0, h), cols(heads, h * kv // heads), cols(heads + kv, h * kv // heads)
            q, k, v = (inp["qkv"][c].to(F64) for c in (at_q, at_k, at_v))
            s = q @ k.t() / math.sqrt(d)
            if later is not None:
                s.masked_fill_(later, -math.inf)
            lse[h, rows] = torch.logsumexp(s, 1)
            p = s.sub_(lse[h, rows][:, None]).exp_()
            o[at_q] = p @ v
            if case["step"]:
                do = inp["do"][at_q].to(F64)
                dqkv[at_v] += p.t() @ do
                ds = p * (do @ v.t() - (do * o[at_q]).sum(1, keepdim=True))
                dqkv[at_q] = ds @ k / math.sqrt(d)
                dqkv[at_k] += ds.t() @ q / math.sqrt(d)
    return dict(o=o, lse=lse, dqkv=dqkv) if case["step"] else dict(o=o, lse=lse)
