"""Calls on a stream of the caller's take outputs and workspaces that they are not given
from that stream's memory: a workspace is freed when the call returns, and memory of
the current stream could then be given to its next call while the kernels on the other
stream still write there."""

import contextlib
import inspect

import pytest
import torch

from helpers import announce
from paper_2408_03505_amd import binding as B

BF, F32 = torch.bfloat16, torch.float32

# calls that allocate nothing
GIVEN = {"enc_attn_bwd_noalloc", "enc_calib_copy"}


def _args(*args, **kw):
    return args, kw


def _cases(dev):
    """Arguments of every wrapper that takes a stream, without those that it can allocate."""
    bf = lambda *s: torch.zeros(s, dtype=BF, device=dev)  # noqa: E731
    f32 = lambda *s: torch.zeros(s, dtype=F32, device=dev)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
    M, W, T = 8, 1024, 1024  # a contraction and a number of rows that are split
    cfg = dict(batch=1, seq=16, hidden=128, heads=2, head_dim=64, mlp=256, ln_eps=1e-6)
    p = {n: bf(*s) for n, s in B.param_shapes(cfg).items()}
    pp = {n: bf(*s) for n, s in B.parallel_param_shapes(cfg).items()}
    x = bf(16, 128)
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8, device=dev)  # noqa: E731
    saved, psaved = u8(B.saved_layout(cfg)["total"]), u8(B.parallel_saved_layout(cfg)["total"])
    cu = torch.tensor([0, M], dtype=torch.int32, device=dev)
    plan, qkv = u8(B.packed_plan_bytes(M, 1)), bf(M, 192)  # (a plan of zeros: no sequences)
    pos, freq = i32(M, 3), f32(32)
    return {
        "encoder_layer_fwd": _args(cfg, p, x),
        "encoder_layer_bwd": _args(cfg, p, x, saved, x),
        "enc_ln_fwd": _args(x, bf(128), bf(128), 1e-6),
        "enc_qkv_fwd": _args(bf(M, W), bf(3 * 64, W), bf(3 * 64)),
        "enc_attn_fwd": _args(1, M, 1, 64, qkv),
        "enc_oproj_fwd": _args(bf(M, W), bf(64, W), bf(64), bf(M, 64)),
        "enc_mlp_up_fwd": _args(bf(M, W), bf(64, W), bf(64)),
        "enc_mlp_down_fwd": _args(bf(M, W), bf(64, W), bf(64), bf(M, 64)),
        "enc_mlp_down_bwd_data": _args(bf(M, W), bf(W, 64), bf(M, 64)),
        "enc_mlp_up_bwd_data": _args(bf(M, W), bf(W, 64)),
        "enc_oproj_bwd_data": _args(bf(M, W), bf(W, 64)),
        "enc_qkv_bwd_data": _args(bf(M, 1536), bf(1536, 64)),
        "enc_qkv_bwd_data_add": _args(bf(M, 1536), bf(1536, 64), bf(M, 64)),
        "enc_linear_bwd_weight": _args(bf(T, 64), bf(T, 64)),
        "enc_mlp_down_bwd_weight": _args(bf(T, 64), bf(T, 64), f32(64, 64), f32(64)),
        "enc_mlp_up_bwd_weight": _args(bf(T, 64), bf(T, 64), f32(64, 64), f32(64)),
        "enc_oproj_bwd_weight": _args(bf(T, 64), bf(T, 64), f32(64, 64), f32(64)),
        "enc_qkv_bwd_weight": _args(bf(T, 192), bf(T, 64), f32(192, 64), f32(192)),
        "enc_ln_bwd": _args(x, x, f32(16), f32(16), bf(128)),
        "enc_attn_bwd": _args(1, M, 1, 64, qkv, bf(M, 64), f32(1, 1, M), bf(M, 64)),
        "enc_calib_mfma": _args(1, 1, device=dev),
        "encoder_parallel_fwd": _args(cfg, pp, x),
        "encoder_parallel_bwd": _args(cfg, pp, x, psaved, x),
        "enc_qk_norm_fwd": _args(1, 64, qkv, *(bf(64) for _ in range(4)), 1e-6),
        "enc_qk_norm_bwd": _args(1, 64, qkv, qkv, f32(M, 1, 4), bf(64), bf(64)),
        "enc_rope_fwd": _args(1, 1, 64, qkv, pos, freq, (8, 8, 8)),
        "enc_rope_bwd": _args(1, 1, 64, qkv, pos, freq, (8, 8, 8)),
        "enc_packed_plan": _args(cu, M),
        "enc_attn_packed_fwd": _args(1, 1, 1, 64, qkv, plan),
        "enc_attn_packed_bwd": _args(1, 1, 1, 64, qkv, bf(M, 64), f32(1, M), bf(M, 64), plan),
        "enc_glu_up_fwd": _args(bf(M, W), bf(128, W)),
        "enc_glu_down_bwd_data": _args(bf(M, W), bf(W, 64), bf(M, 128)),
        "enc_glu_up_bwd_data": _args(bf(M, W), bf(W, 64)),
        "enc_glu_up_bwd_weight": _args(bf(T, 128), bf(T, 64), f32(128, 64), f32(128)),
        "enc_patch_embed_fwd": _args(bf(1, 16, 16, 16), 8, bf(64, W), bf(64), bf(5, 64), bf(64)),
        "enc_patch_embed_bwd": _args((1, 16, 16, 16), 8, bf(5, 64), bf(4, W), True),
        "encoder_stack_fwd": _args(cfg, [p, p], bf(128), bf(128), x),
        "encoder_stack_bwd": _args(cfg, [p, p], bf(128), x, u8(B.stack_saved_bytes(cfg, 2)), x),
    }


NAMES = sorted(n for n, f in inspect.getmembers(B, inspect.isfunction)
               if not n.startswith("_") and "stream" in inspect.signature(f).parameters and n not in GIVEN)


def _record(monkeypatch, made):
    """Notes every tensor that the wrappers allocate while `made` is not None."""
    for owner, name in ((torch, "empty"), (torch.Tensor, "new_empty")):
        real = getattr(owner, name)

        def noted(*args, _real=real, **kw):
            t = _real(*args, **kw)
            if made[0] is not None:
                made[0].append(t)
            return t
        monkeypatch.setattr(owner, name, noted)


class _Stream:  # stands in for a stream: nothing is launched
    device_index, cuda_stream = 0, 0x5000


@pytest.mark.parametrize("name", NAMES)
def test_nothing_is_allocated_outside_the_stream(name, monkeypatch):
    """On host tensors, with the launches left out."""
    (args, kw), made, inside = _cases("cpu")[name], [None], [False]
    real = B._call

    @contextlib.contextmanager
    def entered(stream):
        assert stream is _Stream
        inside[0] = True
        yield
        inside[0] = False

    launched = []

    def called(n, *a):
        return real(n, *a) if n.endswith(("_bytes", "_layout")) else launched.append(n)
    monkeypatch.setattr(B, "_call", called)
    monkeypatch.setattr(B, "_check", lambda t, *a, **k: t)
    monkeypatch.setattr(torch.cuda, "stream", entered)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    _record(monkeypatch, made)

    class Notes(list):
        def append(self, t):
            super().append((tuple(t.shape), inside[0]))
    made[0] = notes = Notes()
    getattr(B, name)(*args, **kw, stream=_Stream)
    made[0] = None
    assert launched == [name]
    assert notes and all(at for _, at in notes), notes


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_memory_is_the_streams(name, monkeypatch):
    announce(f"{name} on a side stream, nothing given")
    (args, kw), made = _cases("cuda")[name], [None]
    _record(monkeypatch, made)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    made[0] = notes = []
    getattr(B, name)(*args, **kw, stream=side)
    made[0] = None
    torch.cuda.synchronize()
    stream_of = {}
    for seg in torch.cuda.memory_snapshot():
        stream_of[(seg["address"], seg["address"] + seg["total_size"])] = seg["stream"]
    mine = [t for t in notes if t.numel()]
    assert mine
    for t in mine:
        own = [s for (a, e), s in stream_of.items() if a <= t.data_ptr() < e]
        assert own == [side.cuda_stream], (name, tuple(t.shape), own)
