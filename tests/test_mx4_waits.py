"""The compiled code of the microscaled 4-bit products: what a matrix instruction has written is read by nothing but the next matrix instruction for as
long as the pipe takes.  (The compiler has left those wait states out before stores to LDS, so the source asks for them; this holds the built code to it.)"""
import re

import lds_loads

NEED = 8                                                        # wait states after a scaled 16 x 16 x 128 product of 4-bit codes, 4 passes of the pipe


def registers(operand):
    """{"v3", "v4"} of v[3:4], {"a7"} of a7."""
    m = re.fullmatch(r"([va])(\d+)|([va])\[(\d+):(\d+)\]", operand)
    if not m:
        return set()
    if m.group(1):
        return {operand}
    return {m.group(3) + str(i) for i in range(int(m.group(4)), int(m.group(5)) + 1)}


def operands(line):
    return re.findall(r"[va]\[\d+:\d+\]|\b[va]\d+\b", line.split(None, 1)[1] if " " in line else "")


def early_reads(code):
    """[(matrix instruction, instruction)]: reached within NEED wait states on some path, and naming a register that the former writes."""
    lines = [l for _, l in code]
    labels = {l[:-1]: i for i, l in enumerate(lines) if l.endswith(":")}
    found = []
    for start, line in enumerate(lines):
        if not line.startswith("v_mfma"):
            continue
        written = registers(operands(line)[0])
        todo, best = [(start + 1, 0)], {}
        while todo:
            i, waited = todo.pop()
            while i < len(lines) and waited < NEED and best.get(i, NEED) > waited:
                best[i] = waited
                l = lines[i]
                if not l.endswith(":"):
                    op = l.split()[0]
                    if not op.startswith("v_mfma") and any(registers(o) & written for o in operands(l)):
                        found.append((line, l))
                    target = labels.get(l.split()[-1]) if op.startswith(("s_branch", "s_cbranch")) else None
                    waited += int(l.split()[1]) + 1 if op == "s_nop" else 1
                    if target is not None:
                        todo.append((target, waited))
                    if op in ("s_branch", "s_endpgm"):
                        break
                i += 1
    return found


def test_the_reader_finds_what_is_missing():
    mfma = "v_mfma_scale_f32_16x16x128_f8f6f4 v[2:5], v[28:31], v[36:39], v[2:5], v7, v40 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
    code = lambda *l: list(enumerate((mfma,) + l))                                            # noqa: E731
    assert early_reads(code("s_nop 6", "ds_write_b32 v1, v2", "s_endpgm"))
    assert not early_reads(code("s_nop 7", "ds_write_b32 v1, v2", "s_endpgm"))
    assert not early_reads(code("ds_write_b32 v1, v6", mfma, "s_endpgm"))
    assert early_reads(code("s_cbranch_scc1 .L", "s_nop 15", "s_endpgm", ".L:", "v_mov_b32_e32 v9, v5", "s_endpgm"))
    assert early_reads(code("s_nop 3", "global_store_dwordx4 v[10:11], v[4:7], off", "s_endpgm"))


def test_results_of_matrix_instructions_are_waited_for():
    kernels = {n: c for n, c in lds_loads.kernels("hq_mx4_gemm.hip").items() if any(l.startswith("v_mfma") for _, l in c)}
    assert len(kernels) == 13                                    # nine tiles, two kernels of few rows for each of two kinds
    for name, code in kernels.items():
        assert not early_reads(code), (name, early_reads(code)[:3])
