"""What the compiler made of the kernels, from the instructions of the built library: the result of a matrix product is not there at
once, nothing in the hardware waits for it, and the compiler, which keeps the distance, counts the instructions of one way only where
several lead to the first use.  Here all of them are walked."""
import re

import pytest

from test_kernel_code_cpu import _code

REGISTERS = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)")


def _registers(text):
    """The vector registers of an instruction, operand by operand: (file, first, last)."""
    return [(m.group(1), int(m.group(2) or m.group(4)), int(m.group(3) or m.group(4))) for m in REGISTERS.finditer(text)]


def _distance(op):
    """Instructions between a product and the first that reads its result: its passes and three (two for fp32)."""
    if "16x16x4_f32" in op:
        return 8 + 2
    m = re.match(r"v_mfma_f32_16x16x(16|32)_bf16", op)
    assert m, op
    return 4 + 3


def early_uses(code):
    """[(address, instruction, address of the use, the use)] of (address, instruction) pairs."""
    index = {at: i for i, (at, _) in enumerate(code)}
    follow, wait, operands = [], [], []
    for i, (_, text) in enumerate(code):
        op = text.split()[0]
        nxt = [i + 1] if i + 1 < len(code) else []
        if op == "s_endpgm":
            nxt = []
        elif op.startswith(("s_branch", "s_cbranch")):
            to = index[int(re.search(r"<[^+>]+(?:\+0x([0-9a-f]+))?>", text).group(1) or "0", 16)]
            nxt = [to] if op == "s_branch" else nxt + [to]
        follow.append(nxt)
        wait.append(int(text.split()[1]) + 1 if op == "s_nop" else 1)
        operands.append(_registers(re.sub(r"<.*", "", text)))
    early = []
    for i, (at, text) in enumerate(code):
        if not text.startswith("v_mfma"):
            continue
        need, (kind, lo, hi) = _distance(text), operands[i][0]
        best, todo = {}, [(k, 0) for k in follow[i]]
        while todo:
            k, waited = todo.pop()
            if waited >= need or best.get(k, need) <= waited:
                continue
            best[k] = waited
            # (products that add to it, or take its place, wait by themselves: their two factors count)
            seen = operands[k][1:3] if code[k][1].startswith("v_mfma") else operands[k]
            if any(f == kind and a <= hi and b >= lo for f, a, b in seen):
                early.append((at, text, code[k][0], code[k][1]))
                continue
            todo += [(x, waited + wait[k]) for x in follow[k]]
    return early


def test_the_walk_finds_an_early_use():
    """A use ten instructions behind a product on one way and one behind it on the other."""
    mfma = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], 0 00"
    code = [(0, mfma), (8, "s_cbranch_vccnz 9 BF <kernel+0x38>")] + [(12 + 4 * i, "s_nop 0 BF") for i in range(11)]
    code += [(0x38, "v_mul_f32_e32 v4, s0, v2 0A"), (0x3c, "s_endpgm BF")]
    assert [x[2] for x in early_uses(code)] == [0x38]
    assert not early_uses([c for c in code if "cbranch" not in c[1]])


@pytest.mark.parametrize("part", ["window_", "decode_", "prefill_"])
def test_no_product_is_used_before_it_is_there(part):
    kernels = _code(part)
    assert any("v_mfma" in x for code in kernels.values() for _, x in code)
    for name, code in kernels.items():
        assert not early_uses(code), (name, early_uses(code)[:2])
