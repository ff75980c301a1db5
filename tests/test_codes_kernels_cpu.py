"""What the compiler made of the kernels of a cache of 8 bits: no product is used before it is there on any way through the control flow, conversions of
codes are the instructions for two at a time, and registers leave room for the workgroups that the launches count on."""
import re

import pytest

from test_kernel_code_cpu import _code
from test_kernel_hazards_cpu import early_uses
from test_kernel_resources_cpu import _workgroups, kernels  # noqa: F401


@pytest.fixture(scope="module")
def code():
    out = _code("kv8_")
    assert sum("v_mfma" in x for c in out.values() for _, x in c) > 100
    return out


def test_no_product_is_used_before_it_is_there(code):
    for name, c in code.items():
        assert not early_uses(c), (name, early_uses(c)[:2])


def test_codes_are_converted_two_at_a_time(code):
    for name, c in code.items():
        text = [x for _, x in c]
        if re.search(r"kv8_(decodeI|rows|tiles|read)", name):
            assert sum(x.startswith("v_cvt_scalef32_pk_bf16_fp8") for x in text) >= 8, name
        if re.search(r"kv8_append", name):
            assert any(x.startswith("v_cvt_pk_fp8_f32") for x in text), name


def test_scales_come_by_scalar_loads(code):
    """One load for both of a block's scales, which no lane waits for by itself."""
    for name, c in code.items():
        if re.search(r"kv8_(decodeI|tiles)", name):
            assert sum(x.startswith("s_load_dwordx2") for _, x in c) >= 2, name


def test_workgroups_per_cu(kernels):  # noqa: F811
    least = {"kv8_decodeILi64": 4, "kv8_decodeILi128": 3, "kv8_decodeILi256": 1, "kv8_tilesILi64ELi2ELi2": 3, "kv8_tilesILi64ELi2ELi1": 3,
             "kv8_tilesILi128ELi2ELi2": 2, "kv8_tilesILi128ELi2ELi1": 2, "kv8_tilesILi256ELi1ELi1": 2, "kv8_tilesILi256ELi2ELi1": 1}
    seen = set()
    for name, k in kernels.items():
        for part, n in least.items():
            if part in name:
                assert _workgroups(k) >= n and k[".private_segment_fixed_size"] == 0, (name, k[".vgpr_count"])
                seen.add(part)
    assert seen == set(least)
