"""The microscaled 4-bit operators of ``include/hq.h`` as cases that can be timed and whose outputs can be compared.

A matrix is held as 4-bit codes (E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) with one 8-bit power of two (E8M0, exponent
byte - 127, 255 = not a number) for every 32 values along the axis that a product sums over.  That axis is cut into chunks of
256: codes [chunks][rows][128 bytes], two to a byte, the even element low; scales [chunks][rows][8]; what lies behind the axis'
end has code 0.  Several matrices (experts' weights) follow each other; ragged segments along the axis start a chunk each.

Kinds of case
  quantize  a real tensor into codes along its rows, its columns or both, and back into the values that the codes stand for
  product   out[m][n] = sum_k A[m][k] B[n][k] of two matrices
  experts   rows sorted by expert, each times its expert's matrix: a forward pass or an input gradient
  wgrad     one product per expert that sums over the expert's rows: their weight gradients

Sizes are this repository's (512, 1000, 1024, 4096) or generic; values follow ``perf/cases.py``: half-normal or normal
activations, He-normal weights, Laplace gradients with outliers.  Where ``own`` is false the operators are computed in their
plain form, in 32 bits.
"""
import math

import numpy as np
import torch

own = False

BLOCK, CHUNK = 32, 256
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------

def _quantize(rows, cols, experts, type, rounding, along, values, **more):
    """experts: 0 = one matrix, otherwise the rows are sorted by expert and codes along columns keep experts apart."""
    return dict(more, kind="quantize", rows=rows, cols=cols, experts=experts, type=type, rounding=rounding, along=along, values=values)


def _product(M, N, K, out, **more):
    return dict(more, kind="product", M=M, N=N, K=K, out=out)


def _experts(rows, N, K, experts, out, **more):
    return dict(more, kind="experts", rows=rows, N=N, K=K, experts=experts, out=out)


def _wgrad(rows, M, N, experts, out, **more):
    return dict(more, kind="wgrad", rows=rows, M=M, N=N, experts=experts, out=out)


def listed():
    return [
        # weights of a small linear layer after an optimizer update: both directions, launch-bound
        _quantize(512, 512, 0, "fp32", "nearest", "both", "weights", name="quantize_weights_512"),
        # the input of a large linear layer: rows for the forward pass, columns for the weight gradient
        _quantize(16384, 4096, 0, "bf16", "nearest", "both", "activation", name="quantize_activation_16k"),
        # an output gradient of a layer of experts, rounded stochastically, nothing aligned
        _quantize(2111, 1000, 6, "fp32", "stochastic", "both", "gradient", name="quantize_gradient_ragged_sr"),
        # one new token through a linear layer: the weights' bytes and latency count
        _product(1, 4096, 4096, "bf16", name="product_one_token"),
        # an ordinary batch with no size a multiple of anything
        _product(777, 1001, 1100, "fp32", name="product_odd"),
        # the forward pass of a large linear layer
        _product(8192, 4096, 4096, "bf16", name="product_8k"),
        # a weight gradient: few outputs, a sum over all tokens
        _product(1024, 1024, 16384, "fp32", name="product_weight_gradient"),
        # a few tokens in flight, most experts idle or with one row
        _experts(16, 2048, 1024, 32, "bf16", name="experts_serving"),
        # forward pass of a training batch, one expert without a row
        _experts(8192, 4096, 1024, 8, "bf16", name="experts_8k"),
        # small experts off every multiple
        _experts(1501, 500, 300, 5, "fp16", name="experts_odd"),
        # weight gradients of few rows: bound by the gradients written
        _wgrad(300, 256, 512, 4, "fp32", name="wgrad_small"),
        # weight gradients of a training batch over many experts
        _wgrad(16384, 4096, 1024, 16, "fp32", name="wgrad_16k"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _size(rng, lo, hi):
    """Uniform over the logarithm; half of the sizes are multiples of 64 where that leaves one."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if n >= 64 and rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(("quantize", "product", "product", "experts", "experts", "wgrad"))
    if kind == "quantize":
        cols, type = _size(rng, 64, 8192), rng.choice(("fp32", "bf16", "fp16"))
        rows = _size(rng, 1, max(1, min(16384, 48_000_000 // cols)))
        values = rng.choice(("activation", "gradient", "weights"))
        experts = rng.choice((0, 0, _log_int(rng, 2, 64)))
        return _quantize(rows, cols, experts, type, "stochastic" if values == "gradient" else "nearest",
                         rng.choice(("rows", "columns", "both", "both")), values)
    out = rng.choice(("fp32", "bf16", "bf16", "fp16"))
    if kind == "product":
        N, K = _size(rng, 64, 8192), _size(rng, 64, 16384)
        M = _size(rng, 1, max(1, min(16384, int(1.2e11 / (N * K)))))
        return _product(M, N, K, out)
    experts = _log_int(rng, 2, 64)
    if kind == "experts":
        N, K = _size(rng, 64, 4096), _size(rng, 64, 4096)
        experts = max(2, min(experts, int(1.2e8 / (N * K))))
        rows = _size(rng, 1, max(1, min(16384, int(3e10 / (N * K)))))
        return _experts(rows, N, K, experts, out)
    M, N = _size(rng, 64, 4096), _size(rng, 64, 4096)
    experts = max(2, min(experts, int(6e7 / (M * N))))
    rows = _size(rng, 1, max(1, min(16384, int(6e10 / (M * N)))))
    return _wgrad(rows, M, N, experts, out)


# ---------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------

_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_VALUES = torch.tensor(_MAGNITUDES + tuple(-v for v in _MAGNITUDES), dtype=torch.float32)
_POWERS = torch.from_numpy(np.append(np.ldexp(1.0, np.arange(-127, 128)), np.nan).astype(np.float32))   # by scale byte


def _random24(index, seed):
    """The 24 random bits of an element: its index and a 64-bit seed through a multiply and xor-shift generator."""
    u32 = 0xFFFFFFFF
    low, high = index & u32, index >> 32
    h = ((low ^ (low >> 16)) * 0x85EBCA6B + (seed & u32)) & u32
    h = h ^ ((high * 0x85EBCA77 + (seed >> 32)) & u32)
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & u32
    h = ((h ^ (h >> 16)) * 0x9E3779B1) & u32
    return (h ^ (h >> 15)) >> 8


def _to_codes(x, random=None):
    """Codes 0..15 and scale bytes of blocks along the last axis, x [..., blocks, 32] in fp32; random: 24 bits for each value."""
    amax = x.abs().amax(-1)
    bits = amax.view(torch.int32)
    byte = (bits >> 23) - 2
    if random is not None:
        byte = byte + ((bits & 0x7FFFFF) > 0x400000)                       # nothing may lie beyond 6
    finite = torch.isfinite(amax)
    byte = byte.clamp(min=0)
    factor = ((254 - byte) << 23).view(torch.float32).unsqueeze(-1)        # 2^(127 - byte)
    t = torch.where(finite.unsqueeze(-1), x.abs() * factor, 0.0)
    step = torch.where(t >= 4.0, 2.0, torch.where(t >= 2.0, 1.0, 0.5))
    q = t / step
    q = torch.round(q) if random is None else torch.floor(q) + (q - torch.floor(q) > random.to(torch.float32) * 2.0 ** -24)
    v = (q * step).clamp(max=6.0)
    # magnitudes by number: 2 v up to 2, then 2 + v up to 4, then 4 + v / 2
    code = torch.where(v <= 2.0, 2.0 * v, torch.where(v <= 4.0, 2.0 + v, 4.0 + 0.5 * v)).to(torch.uint8)
    sign = torch.signbit(x) & finite.unsqueeze(-1)
    return code | (sign.to(torch.uint8) << 3), torch.where(finite, byte, 255).to(torch.uint8)


def _blocks(x):
    """x [..., n] as [..., chunks * 8, 32] with zeros behind the end."""
    n = x.shape[-1]
    whole = -(-n // CHUNK) * CHUNK
    return torch.nn.functional.pad(x, (0, whole - n)).unflatten(-1, (whole // BLOCK, BLOCK))


def _container(x):
    """(codes, scales) of x [..., rows, n] along n as they lie in memory: [..., chunks, rows, 128] and [..., chunks, rows, 8]."""
    code, byte = _to_codes(_blocks(x.float()))
    code = code.flatten(-2).unflatten(-1, (-1, CHUNK // 2, 2))
    packed = code[..., 0] | (code[..., 1] << 4)                            # [..., rows, chunks, 128]
    return packed.transpose(-3, -2).contiguous(), byte.unflatten(-1, (-1, CHUNK // BLOCK)).transpose(-3, -2).contiguous()


def _values(codes, scales):
    """[..., chunks, rows, 128] codes and their scales -> fp32 [..., rows, chunks * 256]"""
    both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    v = _VALUES.to(codes.device)[both.int()].unflatten(-1, (CHUNK // BLOCK, BLOCK)) * _POWERS.to(codes.device)[scales.int()].unsqueeze(-1)
    return v.flatten(-2).transpose(-3, -2).flatten(-2)


def _padded(counts, first):
    """[experts, most rows]: each expert's row numbers from first[e] on, and which of them it has."""
    at = torch.arange(int(counts.max()) if counts.numel() else 0)
    return (first[:, None] + at).cuda(), (at < counts[:, None]).cuda()


def _plain_quantize(s):
    c, x = s["case"], s["X"].float()
    random = None
    if c["rounding"] == "stochastic":
        random = _random24(torch.arange(x.numel(), device=x.device).view_as(x), s["seed"])
    out = {}
    if c["along"] != "columns":
        n = c["cols"]
        code, byte = _to_codes(_blocks(x), None if random is None else _blocks(random))
        out["rows"] = (_VALUES.cuda()[code.int()] * _POWERS.cuda()[byte.int()].unsqueeze(-1)).flatten(-2)[:, :n].to(s["X"].dtype)
    if c["along"] != "rows":
        # each expert's rows in blocks of their own, then back to where they were
        rows, has = _padded(s["counts"], s["first"])
        flat, has = rows.clamp(max=c["rows"] - 1), has.unsqueeze(-1)
        part = torch.where(has, x[flat], 0.0).transpose(-2, -1)
        code, byte = _to_codes(_blocks(part), None if random is None else _blocks(random[flat].transpose(-2, -1)))
        v = (_VALUES.cuda()[code.int()] * _POWERS.cuda()[byte.int()].unsqueeze(-1)).flatten(-2)[..., :rows.shape[1]]
        out["columns"] = v.transpose(-2, -1)[has.squeeze(-1)].t().contiguous().to(s["X"].dtype)
    return out


def _plain_product(s):
    c = s["case"]
    return (_values(*s["A"]) @ _values(*s["B"]).t()).to(TYPES[c["out"]])


def _plain_experts(s):
    c = s["case"]
    rows, has = _padded(s["counts"], s["first"])
    a = _values(*s["A"])[rows.clamp(max=c["rows"] - 1)]
    return torch.matmul(a, _values(*s["B"]).transpose(-2, -1))[has].to(TYPES[c["out"]])


def _plain_wgrad(s):
    c = s["case"]
    at, has = _padded((s["counts"] + CHUNK - 1) // CHUNK, s["first_chunk"])
    at = at.clamp(max=max(0, s["A"][0].shape[0] - 1))

    def part(codes, scales):
        v = _values(codes[at.flatten()].unsqueeze(1), scales[at.flatten()].unsqueeze(1))             # [experts * chunks, rows, 256]
        v = torch.where(has.flatten()[:, None, None], v, 0.0).unflatten(0, at.shape)
        return v.transpose(1, 2).flatten(-2)                                                       # [experts, rows, chunks * 256]

    return torch.matmul(part(*s["A"]), part(*s["B"]).transpose(-2, -1)).to(TYPES[c["out"]])


# ---------------------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------------------

def _own_quantize(s):
    import paper_2105_04246_amd as hq
    c, x = s["case"], s["X"]
    rows, cols, experts = c["rows"], c["cols"], c["experts"]
    q, qs = hq.new_mx4(rows, cols) if c["along"] != "columns" else (None, None)
    t, ts = hq.new_mx4(cols, rows, experts) if c["along"] != "rows" else (None, None)
    args = (hq.mx4_type(x.dtype), x, rows, cols, max(1, experts), s["offsets"] if experts else None)
    if c["rounding"] == "stochastic":
        hq.hq_mx4_quantize_sr(*args, s["seed"], q, qs, t, ts)
    else:
        hq.hq_mx4_quantize(*args, q, qs, t, ts)
    out = {}
    if q is not None:
        out["rows"] = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        hq.hq_mx4_dequantize(q, qs, rows, cols, 1, None, hq.mx4_type(x.dtype), out["rows"])
    if t is not None:
        out["columns"] = torch.empty((cols, rows), dtype=x.dtype, device=x.device)
        hq.hq_mx4_dequantize(t, ts, cols, rows, max(1, experts), s["offsets"] if experts else None, hq.mx4_type(x.dtype), out["columns"])
    return out


def _own_product(s):
    import paper_2105_04246_amd as hq
    c = s["case"]
    p = hq.mx4_problem(c["M"], c["N"], c["K"], 1, hq.mx4_type(TYPES[c["out"]]))
    out = torch.empty((c["M"], c["N"]), dtype=TYPES[c["out"]], device="cuda")
    need = hq.hq_mx4_workspace_bytes(hq.HQ_ENTRY_MX4_GEMM, p)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    hq.hq_mx4_gemm(p, *s["A"], *s["B"], out, ws, need)
    return out


def _own_experts(s):
    import paper_2105_04246_amd as hq
    c = s["case"]
    p = hq.mx4_problem(c["rows"], c["N"], c["K"], c["experts"], hq.mx4_type(TYPES[c["out"]]))
    out = torch.empty((c["rows"], c["N"]), dtype=TYPES[c["out"]], device="cuda")
    hq.hq_mx4_gemm_grouped(p, *s["A"], *s["B"], s["offsets"], out)
    return out


def _own_wgrad(s):
    import paper_2105_04246_amd as hq
    c = s["case"]
    p = hq.mx4_problem(c["M"], c["N"], c["rows"], c["experts"], hq.mx4_type(TYPES[c["out"]]))
    out = torch.empty((c["experts"], c["M"], c["N"]), dtype=TYPES[c["out"]], device="cuda")
    need = hq.hq_mx4_workspace_bytes(hq.HQ_ENTRY_MX4_WGRAD_GROUPED, p)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    hq.hq_mx4_wgrad_grouped(p, *s["A"], *s["B"], s["offsets"], out, ws, need)
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"quantize": _own_quantize, "product": _own_product, "experts": _own_experts, "wgrad": _own_wgrad}[kind](state)
    return {"quantize": _plain_quantize, "product": _plain_product, "experts": _plain_experts, "wgrad": _plain_wgrad}[kind](state)


# ---------------------------------------------------------------------------------------
# what a training or serving program has in hand before the call
# ---------------------------------------------------------------------------------------

def _real(g, shape, values):
    x = torch.randn(shape, generator=g, device="cuda")
    if values == "weights":
        return x.mul_(math.sqrt(2.0 / shape[-1]))
    if values == "activation":
        return x.clamp_(min=0.0)
    u = torch.rand(shape, generator=g, device="cuda").sub_(0.5)            # Laplace(0, 1e-3), 1 % of the values 20 times as large
    x = u.sign() * torch.log1p(u.abs_().clamp_(max=0.4999999).mul_(-2.0)) * -1e-3
    return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.01, x * 20.0, x)


def _counts(rows, experts, seed):
    """Rows per expert of a router that prefers some: every eighth expert (one at least) gets none."""
    r = np.random.RandomState(seed % (1 << 31))
    share = r.gamma(2.0, size=experts)
    share[r.permutation(experts)[:max(1, experts // 8)]] = 0.0
    return torch.from_numpy(r.multinomial(rows, share / share.sum()))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    state = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 1) % 2 ** 63}
    if kind != "product":
        rows, experts = case["rows"], case["experts"]
        counts = _counts(rows, experts, seed) if experts else torch.tensor([rows])
        ends = counts.cumsum(0)
        state.update(counts=counts, first=ends - counts,
                     offsets=torch.nn.functional.pad(ends, (1, 0)).to(torch.int32).cuda())
    if kind == "quantize":
        state["X"] = _real(g, (rows, case["cols"]), case["values"]).to(TYPES[case["type"]])
    elif kind == "product":
        state["A"] = _container(_real(g, (case["M"], case["K"]), "normal" if case["M"] < 64 else "gradient"))
        state["B"] = _container(_real(g, (case["N"], case["K"]), "weights"))
    elif kind == "experts":
        state["A"] = _container(_real(g, (rows, case["K"]), "gradient"))
        state["B"] = _container(_real(g, (experts, case["N"], case["K"]), "weights"))
    else:
        chunks = (counts + CHUNK - 1) // CHUNK
        state["first_chunk"] = chunks.cumsum(0) - chunks
        # each expert's rows behind zeros up to a whole chunk: one matrix along all chunks
        place = torch.repeat_interleave(state["first_chunk"] * CHUNK - state["first"], counts) + torch.arange(rows)
        most = (rows - min(experts, rows)) // CHUNK + min(experts, rows)
        for name, n, values in (("A", case["M"], "gradient"), ("B", case["N"], "activation")):
            x = torch.zeros((most * CHUNK, n), device="cuda")
            x[place.cuda()] = _real(g, (rows, n), values)
            state[name] = _container(x.t())
    return state


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------

_SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
_HELD = 0.5 + 1 / BLOCK                                                    # bytes of a value as code and scale


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        ways = 2 if case["along"] == "both" else 1
        n = case["rows"] * case["cols"]
        return {"bytes": (1.0 + ways) * _SIZE[case["type"]] * n, "flops": 0.0}
    if kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": _HELD * (M + N) * K + _SIZE[case["out"]] * M * N, "flops": 2.0 * M * N * K}
    rows, E = case["rows"], case["experts"]
    if kind == "experts":
        N, K = case["N"], case["K"]
        busy = min(E - max(1, E // 8), rows)                               # experts that can have a row
        return {"bytes": _HELD * (rows + busy * N) * K + _SIZE[case["out"]] * rows * N, "flops": 2.0 * rows * N * K}
    M, N = case["M"], case["N"]
    return {"bytes": _HELD * rows * (M + N) + _SIZE[case["out"]] * E * M * N, "flops": 2.0 * rows * M * N}


# ---------------------------------------------------------------------------------------
# the operators' definition in 64 bits
# ---------------------------------------------------------------------------------------

def _exact_bits(n, seed):
    """Random bits of elements 0 .. n - 1 (n < 2^32), in 32-bit words."""
    with np.errstate(over="ignore"):
        h = np.arange(n, dtype=np.uint32)
        h ^= h >> np.uint32(16)
        h *= np.uint32(0x85EBCA6B)
        h += np.uint32(seed & 0xFFFFFFFF)
        h ^= np.uint32(seed >> 32)
        for shift, factor in ((13, 0xC2B2AE35), (16, 0x9E3779B1)):
            h ^= h >> np.uint32(shift)
            h *= np.uint32(factor)
        h ^= h >> np.uint32(15)
    return h >> np.uint32(8)


def _exact_blocks(x, r):
    """Values of blocks x [n, 32] after quantization, all finite, by comparison with the borders between neighbouring grid values."""
    grid = torch.tensor(_MAGNITUDES, dtype=torch.float64, device=x.device)
    a = x.abs()
    top = a.amax(1)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -126))) - 2            # where log2 was rounded over a border, the next line mends it
    e = e + (top >= 2.0 ** (e + 3)).double() - (top < 2.0 ** (e + 2)).double()
    if r is not None:
        e = e + (top > 6.0 * 2.0 ** e).double()
    unit = 2.0 ** e.clamp(min=-127).unsqueeze(1)
    t = a / unit
    if r is None:
        # codes with an odd number give ties away
        borders = (grid[1:] + grid[:-1]) / 2
        low = torch.bucketize(t, borders, right=False)                     # a border belongs to the value below it
        low = low + ((low < 7) & (t == borders[low.clamp(max=6)]) & (low % 2 == 1))
        v = grid[low]
    else:
        low = (torch.bucketize(t, grid, right=True) - 1).clamp(max=6)
        share = (t - grid[low]) / (grid[low + 1] - grid[low])
        v = torch.where(share > r.double() / 2 ** 24, grid[low + 1], grid[low])
    return torch.copysign(v * unit, x)


def _exact_along(x, r):
    """Quantized along the last axis."""
    n = x.shape[-1]
    pad = (0, -n % BLOCK)
    f = torch.nn.functional.pad
    v = _exact_blocks(f(x, pad).reshape(-1, BLOCK), None if r is None else f(r, pad).reshape(-1, BLOCK))
    return v.view(*x.shape[:-1], -1)[..., :n]


def _exact_matrix(codes, scales):
    """fp64 [rows, chunks * 256] from [chunks, rows, 128] codes: sign, exponent and mantissa taken apart."""
    c = torch.stack((codes % 16, codes // 16), -1).flatten(-2).double()
    sign = 1 - 2 * torch.floor(c / 8)
    m = c % 8
    e, f = torch.floor(m / 2), m % 2
    v = sign * torch.where(e == 0, f / 2, (1 + f / 2) * 2.0 ** (e - 1))
    v = v.unflatten(-1, (-1, BLOCK)) * (2.0 ** (scales.double() - 127)).unsqueeze(-1)
    return v.flatten(-2).permute(1, 0, 2).flatten(1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "product":
        return _exact_matrix(*s["A"]) @ _exact_matrix(*s["B"]).t()
    counts = s["counts"].tolist()
    if kind == "quantize":
        x, r = s["X"].double(), None
        if case["rounding"] == "stochastic":
            r = torch.from_numpy(_exact_bits(x.numel(), s["seed"]).astype(np.int32)).cuda().view_as(x)
        out = {}
        if case["along"] != "columns":
            out["rows"] = _exact_along(x, r)
        if case["along"] != "rows":
            parts = zip(x.split(counts), [None] * len(counts) if r is None else r.split(counts))
            out["columns"] = torch.cat([_exact_along(a.t().contiguous(), None if b is None else b.t().contiguous()) for a, b in parts if len(a)], 1)
        return out
    if kind == "experts":
        parts = _exact_matrix(*s["A"]).split(counts)
        return torch.cat([a @ _exact_matrix(c, q).t() for a, c, q in zip(parts, *s["B"])])
    got = torch.zeros((case["experts"], case["M"], case["N"]), dtype=torch.float64, device="cuda")
    for e, (n, at) in enumerate(zip(counts, s["first_chunk"].tolist())):
        here = slice(at, at + -(-n // CHUNK))
        if n:
            got[e] = _exact_matrix(*(t[here] for t in s["A"])) @ _exact_matrix(*(t[here] for t in s["B"])).t()
    return got
