"""Host side of the packed-sequence and gated feed-forward entry points: sizes,
refusals before anything is launched, and the whole of it once more in a child
process on the library's host code under AddressSanitizer and
UndefinedBehaviorSanitizer (stand-in launchers, no device code)."""

import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2408_03505_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, ODD = 0x10000, 0x10004  # never dereferenced
P, S0 = ctypes.c_void_p(FAKE), ctypes.c_void_p(0)
BIG = 1 << 40
STUB = hasattr(B.lib(), "enc_host_stub_build")

no_gpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer cases run only without a GPU")


def _st(name, *args):
    return getattr(B.lib(), name)(*args)


ROPE = [4, 4, 2, 64, 8, 12, 12, 0, P, P, P, P, S0]
FWD = [64, 3, 4, 2, 64, 0, P, BIG, P, P, P, S0]
BWD = [64, 3, 4, 2, 64, 0, P, BIG, P, P, P, P, P, P, BIG, S0]
UP = [16, 64, 40, 0, P, P, P, P, P, S0, 0, S0]
DOWN = [16, 40, 64, 0, P, P, P, P, S0, 0, S0]
UPB = [16, 64, 40, P, P, P, S0, 0, S0]
UPW = [16, 64, 40, P, P, P, P, 0, S0, 0, S0]
PLAN = [64, 3, P, P, BIG, S0]

INV, UNS, ALI, WSP = B.ENC_ERR_INVALID, B.ENC_ERR_UNSUPPORTED, B.ENC_ERR_ALIGN, B.ENC_ERR_WORKSPACE


def _bad(name, base, changes):
    for at, value, want in changes:
        args = list(base)
        args[at] = value
        assert _st(name, *args) == want, (name, at, value, want, B.lib().enc_last_error())


def _pointers(name, base, optional=()):
    """Every pointer but the stream: NULL is refused unless optional, a misaligned one always."""
    for at, v in enumerate(base[:-1]):
        if isinstance(v, ctypes.c_void_p) and v.value == FAKE:
            if at not in optional:
                _bad(name, base, [(at, S0, INV)])
            _bad(name, base, [(at, ctypes.c_void_p(ODD), ALI)])


@no_gpu_only
def test_rope_refusals():
    for name in ("enc_rope_fwd", "enc_rope_bwd"):
        _bad(name, ROPE, [(0, 0, INV), (0, -1, INV), (1, 0, INV), (2, 0, INV), (3, 96, UNS), (3, 0, INV), (2, 3, UNS),
                          (4, -1, INV), (5, 13, INV), (6, 2 ** 31 - 1, INV), (7, 2, INV), (7, -1, INV),
                          (0, 2 ** 31 // 512, UNS), (1, 65538, UNS)])
        _pointers(name, ROPE)


@no_gpu_only
def test_plan_refusals():
    _bad("enc_packed_plan", PLAN, [(0, 0, INV), (1, 0, INV), (1, -4, INV), (1, 65537, UNS), (4, 0, WSP),
                                   (4, B.packed_plan_bytes(64, 3) - 1, WSP)])
    _pointers("enc_packed_plan", PLAN)
    n = ctypes.c_size_t()
    assert _st("enc_packed_plan_bytes", 64, 3, None) == INV
    assert _st("enc_packed_plan_bytes", 0, 3, ctypes.byref(n)) == INV
    assert _st("enc_packed_plan_bytes", 64, 65537, ctypes.byref(n)) == UNS


@no_gpu_only
def test_plans_of_more_rows_than_attention_takes_are_refused():
    most = (2 ** 31 - 1) // (3 * 64)  # rows of one query, key and value head of 64
    narrow = list(FWD)
    narrow[1], narrow[2], narrow[3] = 1, 1, 1
    _bad("enc_attn_packed_fwd", narrow, [(0, most + 1, UNS), (0, 2 ** 31 - 1, UNS)])
    for tokens in (most + 1, 2 ** 31 - 127, 2 ** 31 - 1):
        _bad("enc_packed_plan", PLAN, [(0, tokens, UNS)])
    if STUB:  # (the product library would launch on fake pointers)
        for name, base in (("enc_packed_plan", PLAN), ("enc_attn_packed_fwd", narrow)):
            args = list(base)
            args[0] = most
            assert _st(name, *args) == B.ENC_OK, B.lib().enc_last_error()


@no_gpu_only
def test_projection_refusals():
    fwd = [16, 64, 640, P, P, P, P, S0, 0, S0]  # eight query heads and one key and value head of 64
    bwd = [16, 64, 640, P, P, P, S0, 0, S0]
    for name, base, optional in (("enc_packed_qkv_fwd", fwd, (5,)), ("enc_packed_qkv_bwd_data", bwd, ())):
        _bad(name, base, [(0, 0, INV), (1, 0, INV), (2, -8, INV), (1, 60, UNS), (2, 644, UNS), (0, 2 ** 31 // 640 + 1, UNS)])
        _pointers(name, base, optional)
        big = list(base)
        big[0], big[1], big[2] = 64, 1024, 1280
        at = len(base) - 3
        need = B.linear_workspace_bytes(64, *((1280, 1024) if at == 7 else (1024, 1280)))
        big[at], big[at + 1] = P, need - 1
        assert need > 0 and _st(name, *big) == WSP
        if STUB:  # (the product library would launch on fake pointers)
            big[at + 1] = need
            assert _st(name, *big) == _st(name, *base) == B.ENC_OK, B.lib().enc_last_error()


def test_plan_sizes():
    # a header and one 16-byte item per 128 rows and sequence
    for tokens, seqs in ((1, 1), (128, 1), (129, 7), (100000, 40), (2 ** 31 - 1, 65536)):
        items = tokens // 128 + seqs
        assert B.packed_plan_bytes(tokens, seqs) == (16 * (1 + items) + 255) // 256 * 256
    assert B.attn_packed_bwd_workspace_bytes(1000, 12) == 96000  # two vectors
    n = ctypes.c_size_t()
    assert _st("enc_attn_packed_bwd_workspace_bytes", 2 ** 30, 4, ctypes.byref(n)) == UNS
    assert _st("enc_attn_packed_bwd_workspace_bytes", 0, 4, ctypes.byref(n)) == INV
    assert _st("enc_attn_packed_bwd_workspace_bytes", 4, 4, None) == INV


def test_glu_workspace_sizes():
    # the other products' where the contraction is a multiple of 64, and never less
    for M, N, K in ((1, 512, 1280), (64, 3416, 1280), (200, 768, 6144), (5003, 1280, 6848), (2048, 6144, 4096)):
        assert B.glu_workspace_bytes(M, N, K) == B.linear_workspace_bytes(M, N, K)
        assert B.linear_workspace_bytes(M, N, K - 8) == 0
        assert B.glu_workspace_bytes(M, N, K - 8) == B.linear_workspace_bytes(M, N, K)
    assert B.glu_workspace_bytes(64, 3416, 1272) > 0
    n = ctypes.c_size_t()
    assert _st("enc_glu_workspace_bytes", 0, 8, 8, ctypes.byref(n)) == INV
    assert _st("enc_glu_workspace_bytes", 8, 12, 8, ctypes.byref(n)) == UNS
    assert _st("enc_glu_workspace_bytes", 8, 8, 8, None) == INV


def test_glu_plan_refusals():
    n = ctypes.c_int()
    out = ctypes.byref(n)
    base = [0, 16, 64, 64, 0, out, out, out]
    _bad("enc_glu_plan", base, [(0, 3, INV), (0, -1, INV), (1, 0, INV), (2, 60, UNS), (3, 12, UNS), (3, 2 ** 30 + 8, UNS),
                                (5, None, INV), (6, None, INV), (7, None, INV)])
    for product in (0, 1, 2):
        for M, H, F in ((1, 8, 8), (2048, 6144, 16384), (70, 6152, 2056), (262000, 8192, 2048)):
            for ws in (0, 1, 4 * M * 2 * F, 2 ** 62):
                assert _st("enc_glu_plan", product, M, H, F, ws, out, out, out) == B.ENC_OK and n.value >= 1
    with pytest.raises(B.EncError):
        B.glu_plan(7, 16, 64, 64)


@no_gpu_only
def test_attention_refusals():
    need = B.packed_plan_bytes(64, 3)
    for name, base in (("enc_attn_packed_fwd", FWD), ("enc_attn_packed_bwd", BWD)):
        _bad(name, base, [(0, 0, INV), (1, 0, INV), (2, 0, INV), (3, 0, INV), (4, 72, UNS), (3, 3, UNS), (5, 2, INV),
                          (5, -1, INV), (7, need - 1, WSP), (1, 65537, UNS), (0, 2 ** 31 // 512, UNS)])
        # more workgroups than a launch takes
        big = list(base)
        big[0], big[1], big[2], big[3] = 8, 65536, 128, 128
        assert _st(name, *big) == UNS
        _pointers(name, base)
    _bad("enc_attn_packed_bwd", BWD, [(14, 2 * 64 * 4 * 4 - 1, WSP)])


@no_gpu_only
def test_glu_refusals():
    _bad("enc_glu_up_fwd", UP, [(0, 0, INV), (1, 0, INV), (2, -8, INV), (1, 60, UNS), (2, 44, UNS), (3, 2, INV),
                                (3, -1, INV), (0, 2 ** 31 // 80 + 1, UNS), (2, (1 << 30) + 8, UNS), (2, 2 ** 24, UNS)])
    _bad("enc_glu_down_bwd_data", DOWN, [(0, 0, INV), (1, 12, UNS), (2, 12, UNS), (3, 7, INV)])
    _bad("enc_glu_up_bwd_data", UPB, [(0, 0, INV), (1, 12, UNS), (2, 12, UNS)])
    _bad("enc_glu_up_bwd_weight", UPW, [(0, 0, INV), (1, 12, UNS), (2, 12, UNS), (2, 2 ** 24, UNS)])
    _pointers("enc_glu_up_fwd", UP, optional=(6, 7))
    _pointers("enc_glu_down_bwd_data", DOWN)
    _pointers("enc_glu_up_bwd_data", UPB)
    _pointers("enc_glu_up_bwd_weight", UPW, optional=(6,))
    # a given workspace that is too small, or misaligned
    M, H, F = 200, 1280, 2048
    for name, base, at, need in (("enc_glu_up_fwd", UP, 9, B.linear_workspace_bytes(M, 2 * F, H)),
                                 ("enc_glu_down_bwd_data", DOWN, 8, B.linear_workspace_bytes(M, F, H)),
                                 ("enc_glu_up_bwd_data", UPB, 6, B.linear_workspace_bytes(M, H, 2 * F))):
        assert need > 0
        args = list(base)
        args[0], args[1], args[2] = (M, F, H) if name == "enc_glu_down_bwd_data" else (M, H, F)
        args[at], args[at + 1] = P, need - 1
        assert _st(name, *args) == WSP, name
        args[at], args[at + 1] = ctypes.c_void_p(ODD), need
        assert _st(name, *args) == ALI, name


@pytest.mark.skipif(not STUB, reason="only on stand-in launchers: the product library would launch on fake pointers")
def test_calls_reach_their_launchers():
    for name, args in (("enc_rope_fwd", ROPE), ("enc_rope_bwd", ROPE), ("enc_packed_plan", PLAN),
                       ("enc_attn_packed_fwd", FWD), ("enc_attn_packed_bwd", BWD), ("enc_glu_up_fwd", UP),
                       ("enc_glu_down_bwd_data", DOWN), ("enc_glu_up_bwd_data", UPB), ("enc_glu_up_bwd_weight", UPW)):
        assert _st(name, *args) == B.ENC_OK, (name, B.lib().enc_last_error())
    # what may be left out, in place, and the largest sizes
    for name, base, at in (("enc_glu_up_fwd", UP, 6), ("enc_glu_up_fwd", UP, 7), ("enc_glu_up_bwd_weight", UPW, 6)):
        args = list(base)
        args[at] = S0
        assert _st(name, *args) == B.ENC_OK
    for name, base in (("enc_attn_packed_fwd", FWD), ("enc_attn_packed_bwd", BWD)):
        args = list(base)
        args[0], args[1], args[2], args[3], args[4] = 116508, 65535, 48, 48, 128
        assert _st(name, *args) == B.ENC_OK, B.lib().enc_last_error()


def test_wrappers_check_their_tensors():
    """The binding refuses host tensors, wrong types and shapes by name."""
    t = torch.zeros(4, 8 * 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU tensor"):
        B.enc_rope_fwd(4, 2, 64, t, torch.zeros(4, 3, dtype=torch.int32), torch.zeros(32), (8, 12, 12))
    with pytest.raises(ValueError, match="offsets"):
        B.enc_packed_plan(torch.zeros(1, dtype=torch.int32), 4)
    with pytest.raises(ValueError, match="offsets"):
        B.enc_packed_plan([0, 4], 4)
    with pytest.raises(ValueError, match="2\\*F"):
        B.enc_glu_up_fwd(torch.zeros(4, 8), torch.zeros(7, 8))
    with pytest.raises(ValueError, match="2\\*F"):
        B.enc_glu_up_bwd_data(torch.zeros(4, 7), torch.zeros(7, 8))


@pytest.mark.skipif(STUB, reason="the child process itself")
@pytest.mark.skipif(not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="needs the HIP headers")
def test_host_code_is_clean_under_asan_and_ubsan():
    from paper_2408_03505_amd import build
    asan = subprocess.run([build.CXX, "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    if not (os.path.isabs(asan) and os.path.exists(asan)):
        pytest.skip("the host compiler has no AddressSanitizer runtime")
    lib = build.build_host_sanitized(verbose=False)
    env = dict(os.environ, OPTIMUS_ENC_LIB=lib, LD_PRELOAD=asan,
               ASAN_OPTIONS="detect_leaks=0:alloc_dealloc_mismatch=0:halt_on_error=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", CUDA_VISIBLE_DEVICES="", HIP_VISIBLE_DEVICES="")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", os.path.abspath(__file__)],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "ERROR: AddressSanitizer" not in tail and "runtime error:" not in tail, tail
    assert " passed" in r.stdout, tail
