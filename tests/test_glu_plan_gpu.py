"""The gated feed-forward products by their own launch plan (enc_glu_plan): the small
tiles of the forward, which only more rows than the few-token kernel takes reach, and
splits of the contraction into every number of parts that a workspace leaves."""

import random

import numpy as np
import pytest
import torch

from helpers import announce, cuda, f64, guard_intact, guarded
from oracle import packed as P
from paper_2408_03505_amd import binding as B
from paper_2408_03505_amd.synthetic import random_bf16
from test_glu_gpu import ACTS, STEPS, _forward, _within

gpu = pytest.mark.gpu
BF = torch.bfloat16

# (whole 64-wide steps, columns of one more)
CONTRACTIONS = [(s, 0) for s in STEPS] + [(0, 8), (0, 56), (1, 8), (1, 40), (2, 24), (3, 56), (4, 8), (5, 32), (8, 16)]
# rows past the few-token kernel's; one tile, several, and tiles that end inside the output
SMALL = [(33, 8), (40, 72), (64, 32), (129, 104), (200, 136)]


def _dims(product, M, H, F):
    """Output columns and contraction."""
    return {B.GLU_UP_FWD: (2 * F, H), B.GLU_DOWN_BWD_DATA: (F, H), B.GLU_UP_BWD_DATA: (H, 2 * F)}[product]


# ------------------------------------------------------------------ the plan (no GPU)

def test_plan_of_few_tokens_and_of_unsplit_products():
    assert B.glu_plan(B.GLU_UP_FWD, 4, 64, 64) == B.glu_plan(B.GLU_UP_FWD, 1, 6144, 16384) == (0, 0, 1)
    # a tile's rows and columns, and those of a product with as long an epilogue
    layouts = {B.GLU_UP_FWD: B.LAYOUT_FWD_GELU, B.GLU_DOWN_BWD_DATA: B.LAYOUT_DGRAD_GELU, B.GLU_UP_BWD_DATA: B.LAYOUT_DGRAD}
    rng = random.Random(9)
    for _ in range(500):
        M, H, F = rng.randint(33, 8192), 64 * rng.randint(1, 64), 64 * rng.randint(1, 64)
        for product, layout in layouts.items():
            N, K = _dims(product, M, H, F)
            bm, bn, parts = B.linear_plan(layout, M, N, K)
            if parts == 1:
                assert B.glu_plan(product, M, H, F) == (bm, bn, 1), (product, M, H, F)
            assert B.glu_plan(product, M, H, F, 0)[2] == 1
            assert B.glu_plan(product, M, H, F)[2] <= parts


def test_the_small_sizes_reach_the_small_tile():
    for steps, more in CONTRACTIONS:
        for M, F in SMALL:
            assert B.glu_plan(B.GLU_UP_FWD, M, 64 * steps + more, F) == (64, 64, 1), (steps, more, M, F)


# sizes whose first products are split, their contractions ending inside a step
SPLIT = [(B.GLU_UP_FWD, 40, 4104, 1000), (B.GLU_UP_FWD, 200, 6152, 264), (B.GLU_UP_FWD, 70, 6152, 2056),
         (B.GLU_DOWN_BWD_DATA, 40, 4104, 1000), (B.GLU_DOWN_BWD_DATA, 200, 6152, 264),
         (B.GLU_DOWN_BWD_DATA, 70, 6152, 2056), (B.GLU_UP_BWD_DATA, 33, 2040, 2056), (B.GLU_UP_BWD_DATA, 64, 1304, 3416)]


@pytest.mark.parametrize("product,M,H,F", SPLIT)
def test_a_smaller_workspace_means_fewer_parts(product, M, H, F):
    N, K = _dims(product, M, H, F)
    full = B.glu_plan(product, M, H, F)[2]
    parts = [B.glu_plan(product, M, H, F, 4 * M * N * room)[2] for room in range(full + 1)]
    assert K % 64 and full >= 7 and parts[full] == full and parts[0] == parts[1] == 1
    assert all(p <= max(room, 1) for room, p in enumerate(parts))
    assert len({p for p in parts if 1 < p < full}) >= 2  # fewer, and still split


@pytest.mark.parametrize("product,M,H,F,rooms", [
    (B.GLU_UP_BWD_DATA, 33, 1280, 3416, (2, 3)), (B.GLU_UP_BWD_DATA, 64, 1304, 3416, (2, 3)),
    (B.GLU_UP_FWD, 40, 4104, 1000, (2, 3, 4)), (B.GLU_DOWN_BWD_DATA, 40, 4104, 1000, (2, 3))])
def test_a_split_cut_to_the_workspace_is_weighed_again(product, M, H, F, rooms):
    """In a few parts these took longer on the tile of their many parts (128x128) than
    the product in one launch (16 to 34 us, not 15 to 22)."""
    N, _ = _dims(product, M, H, F)
    assert B.glu_plan(product, M, H, F)[:2] == (128, 128)
    for room in rooms:
        bm, bn, parts = B.glu_plan(product, M, H, F, 4 * M * N * room)
        assert parts == 1 or (bm, bn) == (64, 64), (room, bm, bn, parts)


# ------------------------------------------------------------------ the products

@gpu
@pytest.mark.parametrize("steps,more", CONTRACTIONS)
def test_forward_on_the_small_tile(steps, more):
    for i, (M, F) in enumerate(SMALL):
        _forward(M, 64 * steps + more, F, "gelu" if (i + steps) % 2 else "silu", bias=i % 3 != 0, save=i != 2, seed=100 * i)


def _in_parts(product, M, H, F, act, rooms):
    """With workspaces for these numbers of parts: within the oracle's bounds, and nothing
    written behind the workspace or the outputs."""
    N, K = _dims(product, M, H, F)
    x, w = random_bf16((M, K), 1), random_bf16((N, K) if product == B.GLU_UP_FWD else (K, N), 2, 1.5 / K ** 0.5)
    if product == B.GLU_UP_FWD:
        b = random_bf16((N,), 3)
        rgu, rh, gb, hb = P.glu_fwd(f64(x), f64(w), f64(b), act)
        refs = [(rgu, gb), (rh, hb)]
        gb = cuda(b)
    elif product == B.GLU_DOWN_BWD_DATA:
        gu = random_bf16((M, 2 * F), 3, 2.0)
        refs = [P.glu_bwd(f64(x), f64(w), f64(gu), act)]
        gu = cuda(gu)
    else:
        ref, err = f64(x) @ f64(w), (K + 4) * P.FP32 * (np.abs(f64(x)) @ np.abs(f64(w)))
        refs = [(ref, P.BF16 * (np.abs(ref) + err) + err)]
    gx, gw = cuda(x), cuda(w)
    for room in rooms:
        size = max(4 * M * N * room, 16)
        parts = B.glu_plan(product, M, H, F, size)[2]
        announce(f"gated product {product} M={M} H={H} F={F} {act} workspace for {room} parts: {parts}")
        ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
        outs = [guarded(r.shape, BF) for r, _ in refs]
        if product == B.GLU_UP_FWD:
            B.enc_glu_up_fwd(gx, gw, gb, act=ACTS[act], gu=outs[0][0], h=outs[1][0], ws=ws[:size])
        elif product == B.GLU_DOWN_BWD_DATA:
            B.enc_glu_down_bwd_data(gx, gw, gu, act=ACTS[act], dgu=outs[0][0], ws=ws[:size])
        else:
            B.enc_glu_up_bwd_data(gx, gw, dy2=outs[0][0], ws=ws[:size])
        torch.cuda.synchronize()
        for (ref, bound), (out, buf) in zip(refs, outs):
            _within(out, ref, bound, f"product {product} {M}x{H}x{F} {act} in {parts} parts")
            assert guard_intact(buf, out.numel())
        assert (ws[size:] == 0x7f).all()
        # the partials are where the plan says: parts of them, and none unsplit
        used = 0 if parts == 1 else 4 * M * N * parts
        assert (ws[used:] == 0x7f).all() and (parts == 1 or not (ws[:used] == 0x7f).all())


@gpu
@pytest.mark.parametrize("product,M,H,F,act", [(*c, act) for c in SPLIT for act in ACTS
                                               if c[0] != B.GLU_UP_BWD_DATA or act == "silu"])  # (without one, that is)
def test_every_number_of_parts(product, M, H, F, act):
    """From the whole workspace down to none."""
    _in_parts(product, M, H, F, act, range(B.glu_plan(product, M, H, F)[2], -1, -1))


@gpu
@pytest.mark.parametrize("product,M,H,F,room,tile", [
    (B.GLU_UP_FWD, 40, 3408, 208, 3, (64, 64)), (B.GLU_UP_FWD, 136, 3984, 1368, 4, (64, 128)),
    (B.GLU_UP_FWD, 129, 3544, 1424, 4, (64, 192)), (B.GLU_UP_FWD, 61, 3496, 128, 6, (128, 128)),
    (B.GLU_DOWN_BWD_DATA, 36, 3208, 272, 2, (64, 64)), (B.GLU_DOWN_BWD_DATA, 679, 3624, 528, 4, (64, 128)),
    (B.GLU_DOWN_BWD_DATA, 717, 3728, 1408, 2, (64, 192)), (B.GLU_DOWN_BWD_DATA, 252, 5656, 160, 10, (128, 128)),
    (B.GLU_UP_BWD_DATA, 36, 536, 2384, 4, (64, 64)), (B.GLU_UP_BWD_DATA, 51, 4464, 1832, 6, (64, 128)),
    (B.GLU_UP_BWD_DATA, 86, 4768, 2760, 4, (64, 192)), (B.GLU_UP_BWD_DATA, 56, 1240, 1832, 7, (128, 128))])
def test_every_tile_of_a_split(product, M, H, F, room, tile):
    N, _ = _dims(product, M, H, F)
    plan = B.glu_plan(product, M, H, F, 4 * M * N * room)
    assert plan[:2] == tile and plan[2] > 1
    _in_parts(product, M, H, F, "silu" if M % 2 else "gelu", [room])
