"""Microscaled 4-bit operators whose workgroups are more than one launch takes (HIP: fewer than 2^32 threads a launch), without a GPU: every launch
stays below that, and together they have all workgroups, each run of them a multiple of 8 long but the last (the XCDs' turns go on)."""
import json
import os
import subprocess
import sys

import pytest

import launches

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = """
import ctypes as C, json, sys
rec = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL | 2)
rec.recorder_lines.restype = C.c_char_p
sys.path.insert(0, sys.argv[2])
import paper_2105_04246_amd as hq
P = 0x10000
op, args = json.load(sys.stdin)
rec.recorder_reset(0)
if op == "quantize":
    rows, cols, batch, q, t, type, seed = args
    a, b = (type, P, rows, cols, batch, None), (P if q else None,) * 2 + (P if t else None,) * 2 + (0,)
    hq.hq_mx4_quantize(*a, *b) if seed is None else hq.hq_mx4_quantize_sr(*a, seed, *b)
elif op == "dequantize":
    rows, n, batch, type = args
    hq.hq_mx4_dequantize(P, P, rows, n, batch, None, type, P, 0)
else:
    p = hq.mx4_problem(*args)
    if op == "gemm":
        hq.hq_mx4_gemm(p, P, P, P, P, P, P, 1 << 40, 0)
    elif op == "rows":
        hq.hq_mx4_gemm_grouped(p, P, P, P, P, P, P, 0)
    else:
        hq.hq_mx4_wgrad_grouped(p, P, P, P, P, P, P, P, 1 << 40, 0)
print(json.dumps([l.split("\\t") for l in rec.recorder_lines().decode().splitlines()]))
"""

LIMIT = 1 << 32
B16, F32 = 1, 0
N = 9_000_000                                              # x 512 threads: past the limit
DEQUANTIZE = 17_000_000                                    # x 256 threads: past the limit

# (operation, arguments, kernel, workgroups, threads of one)
CASES = [
    # one row and 32 columns a matrix, along the rows; 32 rows and one column, along the columns; one value, both ways in one reading
    ("quantize", (1, 32, N, 1, 0, B16, None), "mx4_quantize_pieces_kernel<1, false>", N, 512),
    ("quantize", (32, 1, N, 0, 1, B16, None), "mx4_quantize_pieces_kernel<1, false>", N, 512),
    ("quantize", (1, 1, N, 1, 1, F32, None), "mx4_quantize_kernel<0>", N, 512),
    ("quantize", (1, 1, N, 1, 1, F32, 5), "mx4_quantize_pieces_kernel<0, true>", 2 * N, 512),
    ("quantize", (1, 32, N, 1, 1, F32, 5), "mx4_quantize_pieces_kernel<0, true>", 2 * N, 512),
    # one matrix: 2^28 rows of 32 columns are 2^23 workgroups of 512 threads
    ("quantize", (1 << 28, 32, 1, 1, 0, B16, None), "mx4_quantize_pieces_kernel<1, false>", 1 << 23, 512),
    ("quantize", ((1 << 28) - 32, 32, 1, 1, 0, B16, None), "mx4_quantize_pieces_kernel<1, false>", (1 << 23) - 1, 512),
    ("dequantize", (1, 8, DEQUANTIZE, F32), "mx4_dequantize_kernel<0>", DEQUANTIZE, 256),
    ("dequantize", (1 << 28, 8, 1, B16), "mx4_dequantize_kernel<1>", 1 << 24, 256),
    ("dequantize", ((1 << 28) - 16, 8, 1, B16), "mx4_dequantize_kernel<1>", (1 << 24) - 1, 256),
    # products by expert: few rows, 64 threads for a contraction of at most 256
    ("rows", (1, 1 << 18, 0, 4096, F32), "mx4_row_kernel<1, 1>", 1 << 26, 64),
    ("rows", (1, (1 << 18) - 16, 0, 4096, F32), "mx4_row_kernel<1, 1>", (1 << 26) - 4096, 64),
    ("rows", (1 << 15, 1 << 20, 0, 4096, B16), "mx4_tile_kernel<64, 64, 2, 1, 1>", None, 128),
    ("wgrad", (1, (1 << 19) + 64, 3, 4096, B16), "mx4_tile_kernel<64, 64, 2, 1, 2>", 8193 * 4096, 128),
    ("wgrad", (1, 1 << 20, 1, 4096, B16), "mx4_tile_kernel<64, 64, 2, 1, 2>", 1 << 26, 128),
]


def launched(op, args):
    r = subprocess.run([sys.executable, "-c", CHILD, launches.recorder(), ROOT], input=json.dumps((op, args)), capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in (c[0],) + c[1]))
def test_launches_stay_below_their_limit(case):
    op, args, kernel, blocks, threads = case
    got = launched(op, args)
    assert got
    runs = [int(l[1]) for l in got]
    for l in got:
        assert l[0].startswith(kernel) and int(l[2]) == threads, (l, kernel, threads)
        assert int(l[1]) * int(l[2]) < LIMIT, l
    assert all(n % 8 == 0 for n in runs[:-1])
    assert blocks is None or sum(runs) == blocks
    assert (len(runs) == 1) == (sum(runs) * threads < LIMIT)


# ---- which kernels the sizes of the GPU tests take

TILE = "mx4_tile_kernel<%d, %d, "
SPLIT = [([12000, 0, 200], 3, 65, 67, 64, 1), ([16000, 300, 0], 3, 130, 200, 64, 4), ([16000, 1, 0, 255], 4, 65, 68, 64, 4),
         ([0, 5000, 0, 11111], 3, 64, 128, 64, 4), ([14000, 2384], 0, 510, 1022, 128, 4), ([16000, 381], 6, 509, 1021, 128, 1),
         ([12000, 0, 200], 0, 64, 96, 64, 4), ([300, 15000, 1], 0, 130, 64, 64, 4), ([7000, 5100, 0], 0, 40, 50, 64, 4)]


@pytest.mark.parametrize("counts,beside,M,N,side,width", SPLIT)
@pytest.mark.parametrize("out", (0, 1, 2))
def test_weight_gradients_that_split(counts, beside, M, N, side, width, out):
    """Sizes of tests/test_gpu_mx4_split.py: more parts than the shortest segments have chunks, joined 4 outputs at a time or one by one."""
    E = len(counts)
    got = launched("wgrad", (M, N, sum(counts) + beside, E, out))
    assert [l[0].startswith(w) for l, w in zip(got, (TILE % (side, side), "mx4_join_kernel<%d, %d" % (out, width)))] == [True, True] and len(got) == 2
    parts = int(got[0][1]) // (-(-M // side) * -(-N // side) * E)
    assert parts >= 2 and (E == 2 or any(-(-n // 256) < parts for n in counts))


def test_kernels_of_operands_beyond_4_gb():
    """Sizes of tests/test_gpu_mx4_far.py."""
    for op, args, side in (("rows", (72, 131072, 8192, 9, 0), 64), ("rows", (2000, 131072, 8192, 9, 0), 256), ("gemm", (40, 1 << 22, 9 * 256, 1, 0), 64),
                           ("gemm", (300, 1 << 22, 9 * 256, 1, 0), 128), ("wgrad", (1 << 22, 40, 2560, 2, 0), 64),
                           ("wgrad", (1 << 22, 300, 2560, 2, 0), 128)):
        got = launched(op, args)
        assert len(got) == 1 and got[0][0].startswith(TILE % (side, side)), (op, args, got)
