"""Microscaled 4-bit matrices without a GPU: the oracle against values worked out by hand, the sizes of containers, and what the
entry points refuse (nothing is launched on a refusal)."""
import ctypes as C
import itertools

import numpy as np
import pytest

import paper_2105_04246_amd as hq
from oracle import mx4

P = C.c_void_p(0x10000)                                          # aligned; nothing dereferences it
ODD, NUL = C.c_void_p(0x10008), C.c_void_p(0)


# ---- the oracle ---------------------------------------------------------------------------

def test_codes_of_the_grid_and_of_ties():
    grid = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    c, s = mx4.quantize_block(grid + [-float(v) for v in grid])
    assert s == 127 and list(c) == list(range(16))               # 6 -> exponent 2, scale 1
    #      0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4: ties to the even code
    c, s = mx4.quantize_block([4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, 7.9])
    assert s == 127 and list(c) == [6, 0, 2, 2, 4, 4, 6, 6, 7, 7]
    c, s = mx4.quantize_block(np.ldexp([4, 0.25, -5.5], 20))
    assert s == 147 and list(c) == [6, 0, 15]


def test_scales_of_zero_small_and_broken_blocks():
    assert mx4.quantize_block(np.zeros(32)) [1] == 0
    assert list(mx4.quantize_block([0.0, -0.0])[0]) == [0, 8]
    c, s = mx4.quantize_block([2.0 ** -126, 2.0 ** -127, 2.0 ** -129])          # scale 2^-127: 2, 1 and a quarter
    assert s == 0 and list(c) == [4, 2, 0]
    for bad in (np.inf, -np.inf, np.nan):
        c, s = mx4.quantize_block([1.0, bad, 2.0])
        assert s == 255 and not c.any()


def test_stochastic_scale_leaves_nothing_above_6():
    low = np.zeros(2, np.uint32)
    high = np.full(2, (1 << 24) - 1, np.uint32)
    assert mx4.quantize_block([6.0, 5.0], low)[1] == 127 and mx4.quantize_block([6.001, 5.0], low)[1] == 128
    assert list(mx4.quantize_block([6.0, 5.0], low)[0]) == [7, 7]               # share 0.5 > 0
    assert list(mx4.quantize_block([6.0, 5.0], high)[0]) == [7, 6]              # share 0.5 < 1 - 2^-24
    half = np.full(2, 1 << 23, np.uint32)
    assert list(mx4.quantize_block([6.0, 5.0], half)[0]) == [7, 6]              # up only if the share exceeds the draw


def test_draws_are_those_of_the_8_bit_path():
    import oracle
    seed = 0x123456789ABCDEF
    for i in (0, 1, 77, 1 << 20, (1 << 32) - 1, 1 << 32, (5 << 32) + 9):
        assert int(mx4.random_bits([i], seed)[0]) == int(oracle.sr_bits(i, seed)) >> 8


def test_containers_go_back_to_values():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 300))
    Q, S = mx4.quantize_rows(x)
    assert Q.shape == (2, 5, 128) and S.shape == (2, 5, 8)
    v = mx4.values(Q, S)
    assert (v[:, 300:] == 0).all()
    top = np.abs(np.pad(x, ((0, 0), (0, 20))).reshape(5, 10, 32)).max(-1).repeat(32, -1)[:, :300]
    assert (np.abs(v[:, :300] - x) <= top / 4).all()              # half the widest step, or what lies above 6
    y, size = mx4.product((Q, S), (Q[:, :2], S[:, :2]))
    assert np.allclose(y, v @ v[:2].T) and (size >= np.abs(y)).all()


# ---- sizes --------------------------------------------------------------------------------

def test_chunks_hold_every_distribution():
    """The bound is reached, and no distribution of n rows over the segments passes it."""
    for n, e in itertools.product((0, 1, 2, 5, 255, 256, 257, 511, 512, 513, 1024, 1537), (1, 2, 3, 4)):
        cap = hq.hq_mx4_chunks(n, e)
        steps = sorted({k for m in range(0, n + 1, 256) for k in (m - 1, m, m + 1) if 0 <= k <= n} | {n})
        most = 0
        for head in itertools.product(steps, repeat=e - 1):
            if sum(head) <= n:
                most = max(most, sum(-(-k // 256) for k in head + (n - sum(head),)))
        assert most == cap, (n, e, most, cap)
    assert hq.hq_mx4_chunks(3, 4096) == 3
    for n, e in ((-1, 1), (5, 0), (5, -3), (5, hq.HQ_MX4_MAX_SEGMENTS + 1), (1 << 31, 1)):
        assert hq.hq_mx4_chunks(n, e) == 0


def test_container_buffers():
    q, s = hq.new_mx4(7, 300, 3, 1, device="cpu")
    assert q.shape == (4, 7, 128) and s.shape == (4, 7, 8)
    q, s = hq.new_mx4(7, 300, batch=5, device="cpu")
    assert q.shape == (10, 7, 128) and s.shape == (10, 7, 8)
    import torch
    assert [hq.mx4_type(t) for t in (torch.float32, torch.bfloat16, torch.float16)] == [hq.HQ_FP32, hq.HQ_BF16, hq.HQ_FP16]
    with pytest.raises(ValueError):
        hq.mx4_type(torch.float64)


def test_struct_matches_the_header():
    class MP(C.Structure):
        _fields_ = [(n, C.c_int32) for n in ("M", "N", "K", "experts", "out_type")]
    assert C.sizeof(hq.hq_mx4_problem) == C.sizeof(MP) == 20


# ---- refusals -----------------------------------------------------------------------------

def test_quantize_refuses():
    L = hq.lib()
    good = [hq.HQ_FP32, P, 8, 8, 1, NUL, P, P, P, P, NUL]

    def both(**change):
        a = list(good)
        for k, v in change.items():
            a[int(k[1:])] = v
        rc = L.hq_mx4_quantize(*a)
        assert L.hq_mx4_quantize_sr(*a[:6], 5, *a[6:]) == rc
        return rc
    for t in (-1, 3):
        assert both(a0=t) == hq.HQ_E_BADARG
    assert both(a1=NUL) == both(a6=NUL) == both(a7=NUL) == both(a8=NUL) == both(a9=NUL) == hq.HQ_E_BADARG
    assert both(a6=NUL, a7=NUL, a8=NUL, a9=NUL) == hq.HQ_E_BADARG                # nothing to write
    for k in (1, 6, 7, 8, 9):
        assert both(**{"a%d" % k: ODD}) == hq.HQ_E_BADARG
    assert both(a5=C.c_void_p(0x10002)) == hq.HQ_E_BADARG
    for k, v in ((2, -1), (3, 0), (3, -4), (4, 0), (4, -1), (2, 0x7fffffff), (3, 0x7fffffff)):
        assert both(**{"a%d" % k: v}) == hq.HQ_E_BADSHAPE, (k, v)
    assert both(a4=hq.HQ_MX4_MAX_SEGMENTS + 1, a5=P) == hq.HQ_E_BADSHAPE
    assert both(a2=1 << 30, a3=1 << 30, a4=1 << 20) == hq.HQ_E_BADSHAPE          # more workgroups than a launch has
    assert both(a2=0, a1=NUL) == hq.HQ_OK                                        # no rows: nothing to do


def test_dequantize_refuses():
    L = hq.lib()
    good = [P, P, 8, 8, 1, NUL, hq.HQ_BF16, P, NUL]
    for k, v, rc in ((0, NUL, hq.HQ_E_BADARG), (1, NUL, hq.HQ_E_BADARG), (7, NUL, hq.HQ_E_BADARG), (0, ODD, hq.HQ_E_BADARG),
                     (7, ODD, hq.HQ_E_BADARG), (6, 7, hq.HQ_E_BADARG), (2, -1, hq.HQ_E_BADSHAPE), (3, -1, hq.HQ_E_BADSHAPE),
                     (4, 0, hq.HQ_E_BADSHAPE), (3, 0x7fffffff, hq.HQ_E_BADSHAPE)):
        a = list(good)
        a[k] = v
        assert L.hq_mx4_dequantize(*a) == rc, (k, v)
    assert L.hq_mx4_dequantize(NUL, NUL, 0, 8, 1, NUL, 0, NUL, NUL) == hq.HQ_OK
    assert L.hq_mx4_dequantize(NUL, NUL, 8, 0, 1, NUL, 0, NUL, NUL) == hq.HQ_OK


def test_products_refuse():
    L = hq.lib()
    big = 1 << 40
    calls = {"gemm": lambda p, A=P, As=P, B=P, Bs=P, offs=P, out=P, ws=P, n=big: L.hq_mx4_gemm(p, A, As, B, Bs, out, ws, n, NUL),
             "rows": lambda p, A=P, As=P, B=P, Bs=P, offs=P, out=P, ws=P, n=big: L.hq_mx4_gemm_grouped(p, A, As, B, Bs, offs, out, NUL),
             "wgrad": lambda p, A=P, As=P, B=P, Bs=P, offs=P, out=P, ws=P, n=big: L.hq_mx4_wgrad_grouped(p, A, As, B, Bs, offs, out, ws, n, NUL)}
    ref = lambda *f: C.byref(hq.mx4_problem(*f))                                  # noqa: E731
    for name, call in calls.items():
        good = ref(64, 64, 64, 1, hq.HQ_FP32)
        assert call(None) == hq.HQ_E_BADARG
        for k in ("A", "As", "B", "Bs", "out"):
            assert call(good, **{k: NUL}) == hq.HQ_E_BADARG, (name, k)
            assert call(good, **{k: ODD}) == hq.HQ_E_BADARG, (name, k)
        if name != "gemm":
            assert call(good, offs=NUL) == hq.HQ_E_BADARG and call(good, offs=C.c_void_p(0x10001)) == hq.HQ_E_BADARG
        for f in ((64, 64, 64, 1, 3), (64, 64, 64, 1, -1)):
            assert call(ref(*f)) == hq.HQ_E_BADARG
        for f in ((-1, 64, 64, 1, 0), (64, -1, 64, 1, 0), (64, 64, -1, 1, 0), (64, 64, 64, 0, 0), (64, 64, 64, hq.HQ_MX4_MAX_SEGMENTS + 1, 0),
                  (0x7fffffff, 64, 64, 1, 0), (64, 0x7fffffff, 64, 1, 0), (64, 64, 0x7fffffff, 1, 0)):
            assert call(ref(*f)) == hq.HQ_E_BADSHAPE, (name, f)
        for f in ((0, 64, 64, 1, 0), (64, 0, 64, 1, 0)):
            assert call(ref(*f), A=NUL, B=NUL, out=NUL) == hq.HQ_OK
        assert call(ref(0x7ffffe00, 0x7ffffe00, 64, 1, 0)) == hq.HQ_E_BADSHAPE   # more workgroups than a launch has
    assert calls["gemm"](ref(64, 64, 64, 2, 0)) == hq.HQ_E_BADSHAPE


def test_split_contractions_ask_for_their_workspace():
    L = hq.lib()
    for entry, p in ((hq.HQ_ENTRY_MX4_GEMM, hq.mx4_problem(256, 256, 1 << 15)), (hq.HQ_ENTRY_MX4_WGRAD_GROUPED, hq.mx4_problem(128, 128, 1 << 15, 2))):
        need = hq.hq_mx4_workspace_bytes(entry, p)
        assert need > 0 and need % (4 * p.M * p.N * p.experts) == 0
        for ws, n in ((NUL, need), (P, need - 1), (ODD, need)):
            rc = (L.hq_mx4_gemm(C.byref(p), P, P, P, P, P, ws, n, NUL) if entry == hq.HQ_ENTRY_MX4_GEMM else
                  L.hq_mx4_wgrad_grouped(C.byref(p), P, P, P, P, P, P, ws, n, NUL))
            assert rc == hq.HQ_E_WORKSPACE
    for entry in (0, 4, 7, -1):
        assert hq.hq_mx4_workspace_bytes(entry, hq.mx4_problem(256, 256, 1 << 15)) == 0
    assert hq.hq_mx4_workspace_bytes(hq.HQ_ENTRY_MX4_GEMM, hq.mx4_problem(256, 256, 1 << 15, 2)) == 0
    assert hq.hq_workspace_bytes(hq.HQ_ENTRY_MX4_GEMM, hq.problem(hq.HQ_LINEAR, 8, 1, 1, 8, 1, 1, 1, 0, 8)) == 0
