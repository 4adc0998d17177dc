"""CPU-only: the 8-bit products in the compiler's listing.  gemm_fp8.hip issues its matrix instructions from assembly blocks, which the compiler does not look into, so the waits around
them have to come from the code."""
import os
import re
import subprocess

import pytest

from paper_2211_05953_amd import build

WRITTEN, READY = 2, 19  # slots between a vector instruction and a product that reads what it writes; between a product of 16 passes and anything else on its sums


def _registers(operand):
    m = re.match(r"-?\|?([av])(?:\[(\d+):(\d+)\]|(\d+)\b)", operand)
    if not m:
        return frozenset()
    lo, hi = (m.group(2), m.group(3)) if m.group(2) else (m.group(4), m.group(4))
    return frozenset((m.group(1), r) for r in range(int(lo), int(hi) + 1))


def _kernels(text, name):
    """Instructions and labels of the listing's kernels whose name contains `name`: (text, opcode, operands' registers)."""
    out, code = [], None
    for line in text.split("\n"):
        m = re.match(r"(_Z\w+):", line)
        if m:
            code = []
            if name in m.group(1):
                out.append(code)
        t = line.split(";")[0].strip()
        if code is not None and t and (not t.startswith(".") or re.match(r"\.LBB\w+:$", t)):
            op, _, rest = t.partition(" ")
            code.append((t, op, [_registers(a) for a in re.split(r",\s*", rest.strip())]))
    return out


def _too_close(code):
    """What of a kernel violates the distances, along every path through its branches, each instruction at the earliest it can issue (one slot, s_nop n as n + 1).  A path is
    known by what vector instructions wrote in each of the last slots, and by the slots since the last product; where paths meet, by the worst of both."""
    sums = frozenset().union(*[a[0] for _, op, a in code if op.startswith("v_mfma")])
    label = {t[:-1]: i for i, (t, _, _) in enumerate(code) if t.endswith(":")}
    merge = lambda a, b: (tuple(x | y for x, y in zip(a[0], b[0])), min(a[1], b[1]))  # noqa: E731
    nothing = (frozenset(),) * WRITTEN
    entry, todo, bad = {0: (nothing, READY)}, [0], set()
    while todo:
        i = todo.pop()
        state = entry[i]
        while i < len(code):
            t, op, args = code[i]
            if t.endswith(":"):
                merged = merge(entry[i], state) if i in entry else state
                if i in entry and merged == entry[i] and state != entry[i]:
                    break
                entry[i] = state = merged
            else:
                recent, since = state
                slots, wrote = 1, frozenset()
                if op == "s_nop":
                    slots = int(t.split()[1]) + 1
                elif op.startswith("v_mfma"):
                    bad.update((t, r) for r in frozenset().union(*args) & frozenset().union(*recent))
                    since = -1
                elif since < READY and not op.startswith("s_"):
                    bad.update((t, r) for r in frozenset().union(*args) & sums)
                if op.startswith("v_") and not op.startswith(("v_mfma", "v_cmp")):
                    wrote = args[0]
                state = ((nothing + recent + (wrote,) + (frozenset(),) * (slots - 1))[-WRITTEN:], min(since + slots, READY))
                if "branch" in op:
                    j = label[t.split()[1]]
                    merged = merge(entry[j], state) if j in entry else state
                    if entry.get(j) != merged:
                        entry[j] = merged
                        todo.append(j)
                if op in ("s_branch", "s_endpgm"):
                    break
            i += 1
    return sorted(bad, key=str)


def test_products_keep_their_distance(tmp_path):
    out = tmp_path / "fp8.s"
    src = os.path.join(build.CSRC, "gemm_fp8.hip")
    subprocess.run([build._hipcc()] + build.FLAGS + ["-x", "hip", "-S", "--cuda-device-only", src, "-o", str(out)], check=True, capture_output=True)
    kernels = _kernels(out.read_text(), "gemm_fp8_kernel")
    assert len(kernels) == 40  # 10 tiles by 4 pairs of formats
    for code in kernels:
        assert sum(op.startswith("v_mfma") for _, op, _ in code) >= 16
        assert not _too_close(code), _too_close(code)[:5]
        # and what is written before the first product is held away from it by the code itself: behind the last write of a sum an s_nop 1 or more, before any product
        first = [op.startswith("v_mfma") for _, op, _ in code].index(True)
        sums = frozenset().union(*[a[0] for _, op, a in code if op.startswith("v_mfma")])
        last = max(i for i in range(first) if code[i][1].startswith("v_accvgpr") and code[i][2][0] & sums)
        assert any(op == "s_nop" and int(t.split()[1]) >= WRITTEN - 1 for t, op, _ in code[last:first])


SCALED = "v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[0:7], v[8:15], a[0:3], v16, v17 op_sel:[0,1,0] op_sel_hi:[0,0,0] cbsz:1 blgp:0\n"


@pytest.mark.parametrize("code,n", [
    ("v_accvgpr_write_b32 a3, 0\ns_nop 0\n" + SCALED, 1),      # a sum written one slot in front
    ("v_accvgpr_write_b32 a3, 0\ns_nop 1\n" + SCALED, 0),
    ("v_mov_b32_e32 v17, v90\n" + SCALED, 1),                  # a scale
    ("v_mov_b32_e32 v8, v90\nv_mov_b32_e32 v91, v90\n" + SCALED, 1),
    ("v_mov_b32_e32 v8, v90\nv_mov_b32_e32 v91, v90\ns_nop 0\n" + SCALED, 0),
    (SCALED + "s_nop 15\nv_accvgpr_read_b32 v20, a0", 1),      # a result read
    (SCALED + "s_nop 15\ns_nop 2\nv_accvgpr_read_b32 v20, a0", 0),
    (SCALED + "v_accvgpr_read_b32 v20, a9", 0),
    (".LBB0_1:\n" + SCALED + "v_mov_b32_e32 v0, v90\ns_cbranch_scc1 .LBB0_1", 1),  # over a loop's end
    (".LBB0_1:\n" + SCALED + "v_mov_b32_e32 v0, v90\ns_nop 0\ns_cbranch_scc1 .LBB0_1", 0),
    ("v_mov_b32_e32 v0, v90\ns_branch .LBB0_2\n.LBB0_1:\ns_nop 7\n.LBB0_2:\n" + SCALED, 1),
])
def test_what_is_too_close_is_found(code, n):
    (kernel,) = _kernels("_Zkernel:\n" + code + "\ns_endpgm\n", "kernel")
    assert len(_too_close(kernel)) == n
