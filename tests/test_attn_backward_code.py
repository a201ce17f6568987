"""The attention backward's generated code.  Its accumulators are held by
inline MFMAs that the compiler does not know as such, which is only right as
long as nothing else in a tile loop reads or moves them, and only fast as long
as nothing spills there; both are the register allocator's to break.  Compiles
the source to assembly for gfx950 (no GPU needed) and looks."""
import os
import re
import subprocess

import pytest

from paper_2512_22737_amd import build as B

SRC = "attn_backward.hip"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "k.s")
    try:
        cc = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    subprocess.run([cc, *B.HIPCC_FLAGS, *B.FILE_FLAGS[SRC], "-I", B.INCLUDE,
                    "-I", B.CSRC, "-S", "--cuda-device-only",
                    os.path.join(B.CSRC, SRC), "-o", out], check=True,
                   capture_output=True, timeout=600)
    text = open(out).read()
    found = {}
    for m in re.finditer(r"^(\S*(?:dq|dkv)_kernelILi\d+E\S*):", text, re.M):
        body = text[m.end():]
        found[m.group(1)] = body[:body.index("s_endpgm")].split("\n")
    assert len(found) == 4, list(found)
    return found


def tile_loop(lines):
    """(index, line) of the loop with the products: all blocks of its header."""
    blocks, cur = [], None
    for i, l in enumerate(lines):
        if re.match(r"\.LBB\S+:", l):
            cur = dict(label=l.split(":")[0].lstrip("."), head=l, lines=[])
            blocks.append(cur)
        elif cur is not None:
            if l.strip().startswith(";") and not cur["lines"]:
                cur["head"] += l
            cur["lines"].append((i, l))

    def header(b):
        m = re.search(r"in Loop: Header=(BB\S+)", b["head"])
        if m:
            return m.group(1)
        return b["label"].lstrip("L") if "Loop Header" in b["head"] else None

    count = {}
    for b in blocks:
        n = sum("v_mfma" in l for _, l in b["lines"])
        count[header(b)] = count.get(header(b), 0) + n
    best = max((h for h in count if h), key=lambda h: count[h])
    assert count[best] >= 12, count
    return [x for b in blocks if header(b) == best for x in b["lines"]]


def accumulators(lines):
    regs = set()
    for l in lines:
        m = re.search(r"v_mfma\S+ a\[(\d+):(\d+)\]", l)
        if m:
            regs.update(range(int(m.group(1)), int(m.group(2)) + 1))
    return regs


def test_loops_leave_the_accumulators_alone(kernels):
    for name, lines in kernels.items():
        loop = tile_loop(lines)
        regs = accumulators(l for _, l in loop)
        # D/32 tiles of 16 for dq's 32 rows, for 64 keys of dk and of dv
        D = int(re.search(r"ILi(\d+)E", name).group(1))
        assert len(regs) == (4 if "dkv" in name else 1) * (D // 32) * 16
        for _, l in loop:
            assert "scratch_" not in l, (name, l)
            for m in re.finditer(r"v_accvgpr\S+ .*", l):
                used = {int(x) for x in re.findall(r"\ba(\d+)\b", m.group(0))}
                assert not used & regs, (name, l)


def test_accumulators_are_read_after_a_wait(kernels):
    """Between the last product and the first read of an accumulator there are
    18 wait states."""
    for name, lines in kernels.items():
        loop = tile_loop(lines)
        regs = accumulators(l for _, l in loop)
        waited = False
        for l in lines[max(i for i, _ in loop) + 1:]:
            if re.search(r"s_nop 15", l):
                waited = True
            m = (re.search(r"v_accvgpr_read\S* \S+ a(\d+)", l) or
                 re.search(r"(?:store|write)\S* .*\ba\[?(\d+)", l))
            if m and int(m.group(1)) in regs:
                assert waited, (name, l)
                break
        else:
            raise AssertionError(f"{name}: no accumulator is read")
