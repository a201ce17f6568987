"""The attention backward's generated code, what the compiler does not look
after around the inline MFMAs: their operands are complete two wait states
before them.  A register copy or a conversion that the compiler places between
settle() and the product would break it."""
import re

from test_attn_backward_code import kernels  # noqa: F401  (fixture)

WAIT_STATES = 2


def registers(text):
    """VGPRs named in an operand list: v7, v[8:11]."""
    regs = set()
    for m in re.finditer(r"\bv(?:(\d+)\b|\[(\d+):(\d+)\])", text):
        lo, hi = (m.group(1), m.group(1)) if m.group(1) else m.groups()[1:]
        regs.update(range(int(lo), int(hi) + 1))
    return regs


def written(instruction):
    """VGPRs that a vector instruction writes (its first operand, both of a
    swap); none for other instructions."""
    op, _, rest = instruction.partition(" ")
    if not op.startswith("v_") or op.startswith("v_mfma"):
        return set()
    operands = re.split(r",\s*(?![^\[]*\])", rest)
    return registers(",".join(operands[:2] if "swap" in op else operands[:1]))


def late_operands(lines):
    """(line of an inline product, line that writes an operand too late)."""
    code = [l.split(";")[0].strip() for l in lines]
    bad, products = [], 0
    for i, l in enumerate(code):
        m = re.match(r"v_mfma\S+ a\[[^,]*, (v\S+), (v\S+), a\[", l)
        if not m:
            continue
        products += 1
        needs = registers(m.group(1)) | registers(m.group(2))
        states = 0
        for j in range(i - 1, -1, -1):
            assert not code[j].endswith(":"), (l, code[j])  # a branch's end
            if not code[j] or code[j].startswith("."):
                continue
            nop = re.match(r"s_nop (\d+)", code[j])
            if written(code[j]) & needs:
                bad.append((l, code[j]))
            states += int(nop.group(1)) + 1 if nop else 1
            if states >= WAIT_STATES:
                break
    return bad, products


def test_operands_are_complete(kernels):  # noqa: F811
    for name, lines in kernels.items():
        D = int(re.search(r"ILi(\d+)E", name).group(1))
        bad, products = late_operands(lines)
        # dq: one, dk and dv: two of two groups of keys, D/16 products each
        assert products == (4 if "dkv" in name else 1) * (D // 16), name
        assert not bad, (name, bad)


def test_late_operands_are_seen():
    product = "v_mfma_f32_32x32x16_bf16 a[0:15], v[8:11], v[4:7], a[0:15]"
    for before, late in ((["v_mov_b32_e32 v9, v2"], 1),
                         (["v_mov_b32_e32 v9, v2", "s_nop 0"], 1),
                         (["v_mov_b32_e32 v9, v2", "s_nop 1"], 0),
                         (["v_mov_b32_e32 v9, v2", "s_add_i32 s0, s0, 1",
                           "ds_read_b128 v[20:23], v9"], 0),
                         (["v_permlane32_swap_b32_e32 v30, v6"], 1),
                         (["v_cvt_pk_bf16_f32 v4, v20, v21"], 1),
                         (["v_add_f32_e32 v12, v8, v4"], 0)):
        lines = ["s_nop 7"] + [x + " ; note" for x in before] + [
            "\t;;#ASMSTART", "\t" + product, "\t;;#ASMEND"]
        assert len(late_operands(lines)[0]) == late, before
