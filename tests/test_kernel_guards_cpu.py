"""Of the windowed tiles' kernels, from the instructions of the built library: no product whose result is soon used is on its way where the
control flow parts.  There the compiler has been seen to count the instructions up to the use on one way only, so that nothing but how long
the others happened to be kept a result from being read early (test_kernel_hazards_cpu walks them all)."""
import os
import re

import paper_2410_18248_amd as P
from paper_2410_18248_amd import build
from test_kernel_code_cpu import OBJDUMP, _code
from test_kernel_hazards_cpu import _registers

NEED, FAR = 8, 16                                   # instructions until a product of 16x16x32 is there; a use not far behind that


def parted(code):
    """[(address, product, address of the use, the use, instructions between)] for products that are not there yet at a branch in front of a
    use that is not FAR."""
    index = {at: i for i, (at, _) in enumerate(code)}
    follow, wait, operands, parts = [], [], [], []
    for i, (_, text) in enumerate(code):
        op = text.split()[0]
        nxt = [i + 1] if i + 1 < len(code) and op != "s_endpgm" else []
        if op.startswith(("s_branch", "s_cbranch")):
            to = index[int(re.search(r"<[^+>]+(?:\+0x([0-9a-f]+))?>", text).group(1) or "0", 16)]
            nxt = [to] if op == "s_branch" else nxt + [to]
        follow.append(nxt)
        parts.append(op.startswith(("s_branch", "s_cbranch")))
        wait.append(int(text.split()[1]) + 1 if op == "s_nop" else 1)
        operands.append(_registers(re.sub(r"<.*", "", text)))
    found = []
    for i, (at, text) in enumerate(code):
        if not text.startswith("v_mfma"):
            continue
        kind, lo, hi = operands[i][0]
        best, todo = {}, [(k, 0, False) for k in follow[i]]
        while todo:
            k, waited, early = todo.pop()
            if waited >= FAR or best.get((k, early), FAR) <= waited:
                continue
            best[k, early] = waited
            product = code[k][1].startswith("v_mfma")
            seen = operands[k][1:3] if product else operands[k]
            if any(f == kind and a <= hi and b >= lo for f, a, b in seen):
                if early:
                    found.append((hex(at), text, hex(code[k][0]), code[k][1], waited))
                continue
            if product and operands[k][0][:2] == (kind, lo):
                continue                            # (added to: that product's turn)
            todo += [(x, waited + wait[k], early or (parts[k] and waited < NEED)) for x in follow[k]]
    return found


def test_what_counts_as_parted():
    mfma = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], 0 00"

    def way(nops, behind):
        code = [(0, mfma), (8, "s_nop %d BF" % nops), (12, "s_cbranch_vccnz 9 BF <kernel+0x38>")] + [(16 + 4 * i, "s_nop 0 BF") for i in range(8)]
        return code + [(0x34, "s_nop 0 BF"), (0x38, "s_nop %d BF" % behind), (0x3c, "v_mul_f32_e32 v4, s0, v2 0A"), (0x40, "s_endpgm BF")]
    assert parted(way(0, 3)) and parted(way(6, 3))
    assert not parted(way(7, 0))                    # there at the branch
    assert not parted(way(0, 15))                   # not soon used
    assert not parted([c for c in way(0, 3) if "cbranch" not in c[1]])


def test_scores_are_there_where_the_way_parts():
    for part, many in (("window_tiles", 20), ("window_teams", 2)):
        kernels = {n: c for n, c in _code(part).items() if "window_tiles_f32" not in n}
        assert len(kernels) == many
        for name, code in kernels.items():
            assert sum(x.startswith("v_mfma_f32_16x16x32_bf16") for _, x in code) > 8, name
            assert not parted(code), (name, parted(code)[:2])


def test_the_instructions_can_be_read_where_the_library_is_built():
    """Without it the tests that walk through the kernels would pass over everything."""
    assert os.path.exists(P.lib_path()) and os.path.exists(build.HIPCC) and os.path.exists(OBJDUMP)
