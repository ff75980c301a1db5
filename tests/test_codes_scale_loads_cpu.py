"""Where a block's scales come from in the kernels of attention over a cache of 8 bits: scalar loads inside the walk, not one of each lane's own."""
import re

import pytest

from test_kernel_code_cpu import _code


def _walks(code):
    """Instructions of the innermost loops that have products of the matrix cores and loads of codes in them."""
    loops = []
    for at, (address, x) in enumerate(code):
        m = re.match(r"s_c?branch\S*\s.*<[^>]*\+0x([0-9a-f]+)>", x)
        if m and int(m.group(1), 16) <= address:
            first = next(i for i, (a, _) in enumerate(code) if a >= int(m.group(1), 16))
            text = [y for _, y in code[first:at + 1]]
            if any(y.startswith("v_mfma") for y in text) and any(y.startswith("global_load_dwordx4") for y in text):
                loops.append((first, at, text))
    return [text for first, last, text in loops if not any((f, e) != (first, last) and f >= first and e <= last for f, e, _ in loops)]


@pytest.fixture(scope="module")
def walks():
    out = {n: _walks(c) for n, c in _code("kv8_").items() if re.search(r"kv8_(decodeI|rows|tiles)", n)}
    assert len(out) > 12 and all(out.values()), [n for n, w in out.items() if not w]
    return out


def _scales(text, load):
    return [x for x in text if re.match(load, x)]


def test_scales_come_by_scalar_loads_in_the_walk(walks):
    """Eight bytes, for keys and values, behind no constant offset (a kernel's own arguments have one, or come in front of the loop)."""
    for name, loops in walks.items():
        for text in loops:
            assert _scales(text, r"s_load_dwordx2 s\[\d+:\d+\], s\[\d+:\d+\], 0x0\b"), name


def test_no_lane_loads_scales_of_its_own(walks):
    for name, loops in walks.items():
        for text in loops:
            assert not _scales(text, r"(global|flat)_load_dwordx2\b|(global|flat)_load_dword\b"), (name, _scales(text, r"(global|flat)_load_dwordx?2?\b")[:2])


def test_a_walk_with_loads_by_lanes_would_be_found():
    """The look at the code itself, on a few lines: one loop inside another, the inner one with products."""
    lines = ["s_load_dwordx2 s[4:5], s[0:1], 0x0", "v_mov_b32 v0, 0", "global_load_dwordx4 v[0:3], v4, s[2:3]", "global_load_dwordx2 v[6:7], v4, s[2:3]", "v_mfma_f32_16x16x32_bf16 a, b, c, d",
             "s_cbranch_scc1 65531 <kernel+0x8>", "s_cbranch_scc1 65530 <kernel+0x0>"]
    (text,) = _walks([(4 * i, x) for i, x in enumerate(lines)])
    assert text == lines[2:6]
    assert not _scales(text, r"s_load_dwordx2 s\[\d+:\d+\], s\[\d+:\d+\], 0x0\b") and _scales(text, r"(global|flat)_load_dwordx2\b")
