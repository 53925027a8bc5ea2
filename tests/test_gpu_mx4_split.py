"""Microscaled 4-bit weight gradients by expert whose contraction is split: experts without a row or with fewer chunks than parts, edges, every way to
join, workspaces that hold what is not a number, replays.  Which kernels these sizes take: tests/test_mx4_launches.py."""
import numpy as np
import pytest
import torch

import paper_2105_04246_amd as hq
from oracle import mx4
from test_gpu_mx4 import TYPES, check, dev, guarded, margins_untouched, offsets, random_container
from test_gpu_mx4_steps import Experts, drawn, equal

pytestmark = pytest.mark.gpu

# (rows by expert, rows before the first, rows behind the last, M, N)
SPLIT = [([12000, 0, 200], 1, 2, 65, 67), ([16000, 300, 0], 3, 0, 130, 200), ([16000, 1, 0, 255], 0, 4, 65, 68), ([0, 5000, 0, 11111], 2, 1, 64, 128),
         ([14000, 2384], 0, 0, 510, 1022), ([16000, 381], 2, 4, 509, 1021)]
STEPS = [([12000, 0, 200], 64, 96), ([300, 15000, 1], 130, 64)]                     # rows by expert, N, K of a layer


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("counts,before,behind,M,N", SPLIT)
def test_split_weight_gradients_by_expert(counts, before, behind, M, N, dtype):
    E, T = len(counts), before + sum(counts) + behind
    rng = np.random.default_rng(T + N)
    o, offs = offsets(counts, before)
    cap = hq.hq_mx4_chunks(T, E)
    A, B = ([np.full((cap, r, k), 255, np.uint8) for k in (128, 8)] for r in (M, N))       # chunks of no segment: not a number
    at, parts = 0, []
    for n in counts:
        part = [[t[0] for t in random_container(rng, r, n)] for r in (M, N)]
        for whole, p in zip((A, B), part):
            for k in (0, 1):
                whole[k][at:at + mx4.chunks(n)] = p[k]
        at += mx4.chunks(n)
        parts.append(part)
    p = hq.mx4_problem(M, N, T, E, hq.mx4_type(TYPES[dtype]))
    need = hq.hq_mx4_workspace_bytes(hq.HQ_ENTRY_MX4_WGRAD_GROUPED, p)
    assert need >= 2 * 4 * E * M * N
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")                 # as fp32: not a number
    a, b = dev(A), dev(B)
    first = None
    for turn in range(2):                                                                   # the second one in a used workspace
        flat, out = guarded((E, M, N), TYPES[dtype])
        hq.hq_mx4_wgrad_grouped(p, *a, *b, offs, out, ws, need)
        torch.cuda.synchronize()
        assert margins_untouched(flat) and bool((ws[need:] == 255).all())
        assert first is None or torch.equal(out, first)
        first = out
    for e, (x, y) in enumerate(parts):
        if counts[e]:
            want, size = mx4.product(x, y)
            check(out[e], want, size, -(-counts[e] // 32), TYPES[dtype], "expert %d" % e)
        else:
            assert bool((out[e] == 0).all()), "expert %d has no rows" % e


def test_captured_steps_with_split_weight_gradients():
    """Two layers in graphs of their own that share one workspace, replayed one after the other with other inputs and segments, eager work between."""
    rng = np.random.default_rng(21)
    layers = [Experts(*s) for s in STEPS]
    ws = torch.full((max(L.need for L in layers),), 255, dtype=torch.uint8, device="cuda")
    graphs = []
    for L in layers:
        assert L.need > 0
        L.ws = ws
        L.set(*drawn(rng, L))
        L.step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L.step()
        graphs.append(g)
    eager = Experts([7000, 5100, 0], 40, 50)
    assert eager.need > 0
    for turn in range(4):
        data = []
        for L, g in zip(layers, graphs):
            data.append(drawn(rng, L))
            L.set(*data[-1])
            L.o = np.concatenate([[0], np.sort(rng.integers(0, L.T + 1, L.E - 1)), [L.T]])
            L.offs.copy_(torch.tensor(L.o, dtype=torch.int32))
            g.replay()
        mixed = drawn(rng, eager)
        eager.set(*mixed)
        eager.step()
        equal(eager.results(), eager.expected(*mixed), "eager, turn %d" % turn)
        for L, d in zip(layers, data):
            equal(L.results(), L.expected(*d), "replay, turn %d" % turn)
