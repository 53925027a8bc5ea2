"""Microscaled 4-bit matrices on the CPU, in 64 bits: what hq_mx4_quantize, hq_mx4_dequantize and the products of include/hq.h
compute, written from their definition there.  Test infrastructure only."""
import numpy as np

BLOCK, CHUNK = 32, 256
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def random_bits(index, seed):
    """The 24 random bits of elements `index` (an array) under a 64-bit seed."""
    m = 0xFFFFFFFF
    out = np.empty(len(index), np.uint32)
    for k, i in enumerate(int(v) for v in index):
        low, high = i & m, i >> 32
        h = ((low ^ (low >> 16)) * 0x85EBCA6B + (seed & m)) & m
        h ^= (high * 0x85EBCA77 + (seed >> 32)) & m
        h = ((h ^ (h >> 13)) * 0xC2B2AE35) & m
        h = ((h ^ (h >> 16)) * 0x9E3779B1) & m
        out[k] = (h ^ (h >> 15)) >> 8
    return out


def quantize_block(x, bits=None):
    """(codes, scale byte) of up to 32 values; bits: their random bits, None: to nearest even."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return np.zeros(len(x), np.uint8), 255
    a = np.abs(x)
    top = a.max() if len(a) else 0.0
    byte = 0
    if top > 0:
        e = int(np.floor(np.log2(top)))
        e += int(top >= 2.0 ** (e + 1)) - int(top < 2.0 ** e)
        if bits is not None and top > 1.5 * 2.0 ** e:
            e += 1
        byte = max(e - 2 + 127, 0)
    t = np.ldexp(a, 127 - byte)
    codes = np.empty(len(x), np.uint8)
    for i, v in enumerate(t):
        lo = int(np.searchsorted(GRID, v, side="right")) - 1
        if lo == 7:
            codes[i] = 7
        elif bits is None:
            mid = (GRID[lo] + GRID[lo + 1]) / 2
            codes[i] = lo + int(v > mid or (v == mid and lo % 2 == 1))
        else:
            share = (v - GRID[lo]) / (GRID[lo + 1] - GRID[lo])
            codes[i] = lo + int(share > int(bits[i]) / 2.0 ** 24)
    return codes | (np.signbit(x).astype(np.uint8) << 3), byte


def chunks(n):
    return -(-n // CHUNK)


def quantize_rows(x, bits=None):
    """(codes [chunks, rows, 128], scales [chunks, rows, 8]) of x [rows, n] along n; bits [rows, n]."""
    rows, n = x.shape
    Q, S = np.zeros((chunks(n), rows, 128), np.uint8), np.zeros((chunks(n), rows, 8), np.uint8)
    for r in range(rows):
        for b in range(-(-n // BLOCK)):
            at = slice(b * BLOCK, min(n, (b + 1) * BLOCK))
            c, s = quantize_block(x[r, at], None if bits is None else bits[r, at])
            c = np.concatenate([c, np.zeros(BLOCK - len(c), np.uint8)])
            ch, k = divmod(b, 8)
            Q[ch, r, 16 * k:16 * k + 16] = c[0::2] | (c[1::2] << 4)
            S[ch, r, k] = s
    return Q, S


def values(Q, S):
    """float64 [rows, chunks * 256] of a container."""
    c = np.stack([Q & 15, Q >> 4], -1).reshape(*Q.shape[:2], CHUNK)
    v = np.where(c & 8, -1.0, 1.0) * GRID[c & 7]
    scale = np.where(S == 255, np.nan, np.ldexp(1.0, S.astype(np.int64) - 127))
    return (v * np.repeat(scale, BLOCK, -1)).transpose(1, 0, 2).reshape(Q.shape[1], Q.shape[0] * CHUNK)


def product(A, B):
    """(sum over k of a b, sum of |a| |b|) of two containers (codes, scales) with as many chunks."""
    a, b = values(*A), values(*B)
    return a @ b.T, np.abs(a) @ np.abs(b).T
