"""Microscaled 4-bit products without a GPU: which kernel takes a call on either side of each line of the dispatch, and the compiled
code's loads into LDS (tests/lds_loads.py)."""
import json
import os
import subprocess
import sys

import launches
import lds_loads

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = """
import ctypes as C, json, sys
rec = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL | 2)
rec.recorder_lines.restype = C.c_char_p
sys.path.insert(0, sys.argv[2])
import paper_2105_04246_amd as hq
P, out = 0x10000, []
for op, args in json.load(sys.stdin):
    rec.recorder_reset(0)
    if op == "quantize":
        rows, cols, batch, offs, q, t, type, seed = args
        a = (type, P, rows, cols, batch, P if offs else None)
        b = (P if q else None,) * 2 + (P if t else None,) * 2 + (0,)
        hq.hq_mx4_quantize(*a, *b) if seed is None else hq.hq_mx4_quantize_sr(*a, seed, *b)
    else:
        p = hq.mx4_problem(*args)
        if op == "gemm":
            hq.hq_mx4_gemm(p, P, P, P, P, P, P, 1 << 40, 0)
        elif op == "rows":
            hq.hq_mx4_gemm_grouped(p, P, P, P, P, P, P, 0)
        else:
            hq.hq_mx4_wgrad_grouped(p, P, P, P, P, P, P, P, 1 << 40, 0)
    out.append([l.split("\\t") for l in rec.recorder_lines().decode().splitlines()])
print(json.dumps(out))
"""


def calls(wanted):
    r = subprocess.run([sys.executable, "-c", CHILD, launches.recorder(), ROOT], input=json.dumps(wanted), capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout)


def check(cases):
    for (op, args, want), got in zip(cases, calls([c[:2] for c in cases])):
        names = [l[0] for l in got]
        assert len(names) == len(want) and all(n.startswith(w) for n, w in zip(names, want)), (op, args, names, "expected", want)
        for l in got:
            assert int(l[1]) >= 1


ROW1, ROW2 = "mx4_row_kernel<1", "mx4_row_kernel<2"
TILE = {n: "mx4_tile_kernel<%d, %d" % (n, n) for n in (64, 128, 256)}
JOIN = "mx4_join_kernel"


def test_products():
    check([("gemm", (1, 4096, 4096, 1, 1), [ROW1]), ("gemm", (16, 4096, 4096, 1, 1), [ROW1]), ("gemm", (17, 4096, 4096, 1, 1), [ROW2]),
           ("gemm", (32, 64, 100, 1, 0), [ROW2]), ("gemm", (33, 64, 100, 1, 0), [TILE[64]]), ("gemm", (300, 300, 0, 1, 0), [TILE[64]]),
           ("gemm", (256, 4096, 4096, 1, 1), [TILE[64]]), ("gemm", (1024, 4096, 4096, 1, 1), [TILE[128]]), ("gemm", (2048, 4096, 4096, 1, 1), [TILE[128]]),
           ("gemm", (4096, 4096, 4096, 1, 1), [TILE[256]]), ("gemm", (8192, 4096, 4096, 1, 2), [TILE[256]]),
           ("gemm", (1024, 1024, 16384, 1, 0), [TILE[128], JOIN + "<0, 4"]), ("gemm", (100, 101, 16384, 1, 1), [TILE[64], JOIN + "<1, 4"]),
           ("gemm", (101, 101, 16384, 1, 2), [TILE[64], JOIN + "<2, 1"])])


def test_sizes_of_the_gpu_tests_reach_the_larger_tiles():
    check([("gemm", (1030, 4100, 700, 1, 0), [TILE[128]]), ("gemm", (4100, 4133, 300, 1, 0), [TILE[256]]),
           ("gemm", (1000, 1003, 16000, 1, 0), [TILE[128], JOIN + "<0, 4"]), ("gemm", (3300, 3050, 4000, 1, 0), [TILE[256]]),
           ("rows", (3095, 1100, 600, 4, 0), [TILE[128]]), ("rows", (4205, 4100, 520, 4, 0), [TILE[256]]),
           ("wgrad", (1030, 1100, 1713, 4, 0), [TILE[128]]), ("wgrad", (4100, 2060, 1500, 3, 0), [TILE[256]])])


def test_products_by_expert():
    check([("rows", (63, 512, 512, 8, 1), [ROW1]), ("rows", (64, 512, 512, 8, 1), [TILE[64]]), ("rows", (32, 4096, 1024, 2, 1), [ROW2]),
           ("rows", (16, 4096, 1024, 2, 1), [ROW1]), ("rows", (33, 4096, 1024, 2, 1), [TILE[64]]), ("rows", (8192, 4096, 1024, 8, 1), [TILE[256]]),
           ("wgrad", (4096, 1024, 16384, 16, 0), [TILE[256]]), ("wgrad", (256, 512, 300, 4, 0), [TILE[64]]),
           ("wgrad", (256, 512, 16384, 2, 0), [TILE[64], JOIN + "<0, 4"]), ("wgrad", (64, 64, 0, 4, 1), [TILE[64]])])


def test_quantization():
    both, pieces = "mx4_quantize_kernel<", "mx4_quantize_pieces_kernel<"
    check([("quantize", (4096, 2048, 1, 0, 1, 1, 0, None), [both + "0"]), ("quantize", (4095, 2048, 1, 0, 1, 1, 0, None), [pieces + "0, false"]),
           ("quantize", (4096, 4096, 1, 0, 1, 1, 1, None), [both + "1"]), ("quantize", (4096, 4095, 1, 0, 1, 1, 1, None), [pieces + "1, false"]),
           ("quantize", (4096, 4096, 1, 0, 1, 1, 2, 5), [pieces + "2, true"]), ("quantize", (16384, 4096, 1, 0, 1, 0, 0, None), [pieces + "0, false"]),
           ("quantize", (16384, 4096, 1, 0, 0, 1, 0, None), [pieces + "0, false"]), ("quantize", (1024, 2048, 4, 0, 1, 1, 0, None), [both + "0"]),
           ("quantize", (1024, 2048, 4, 1, 1, 1, 0, None), [pieces + "0, false"])])
    # workgroups: 32 rows of 256 columns each along the rows, 256 rows of 64 columns along the columns; ragged segments: as many as any distribution needs
    got = calls([("quantize", (100, 300, 1, 0, 1, 1, 0, None)), ("quantize", (100, 300, 7, 1, 1, 1, 0, None)), ("quantize", (3, 300, 7, 1, 0, 1, 0, None)),
                 ("quantize", (8192, 4096, 1, 0, 1, 1, 0, None))])
    assert [int(g[0][1]) for g in got] == [4 * 2 + 1 * 5, (2 + 7) * 2 + 7 * 5, 3 * 5, 32 * 16]


def test_no_load_into_lds_is_under_way_when_a_wavefront_of_a_product_ends():
    found = {name: code for name, code in lds_loads.kernels("hq_mx4_gemm.hip").items() if "mx4_tile_kernel" in name}
    assert len(found) == 9                                         # three tiles of three kinds
    for name, code in found.items():
        assert sum(l.startswith("global_load_lds") for _, l in code) >= 10, name
        ends = [(n, l) for n, l in lds_loads.under_way(code) if l == "s_endpgm"]
        assert not ends, (name, ends)
