"""The cache of 8 bits without a GPU: sizes, refusals, and the plain form of its codes against torch's conversions."""
import ctypes

import numpy as np
import pytest
import torch

import codes_forms as F
import paper_2410_18248_amd as P
from test_boundary_cpu import _cfg
from test_operators_cpu import A, _refused


@pytest.fixture
def lam():
    buf = ctypes.create_string_buffer(4096)
    a = (ctypes.addressof(buf) + 255) & ~255
    x = P.Lamps(_cfg(dtype=P.LAMPS_E4M3), a, a, a)  # "device" memory that is never looked at
    x._buf = buf
    yield x
    x.destroy()


def test_plain_codes_are_torchs():
    c = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(F.VALUES, c.view(torch.float8_e4m3fn).double().numpy())
    x = np.concatenate([F.VALUES[:127], F.MIDDLES, F.MIDDLES * (1 + 2 ** -20), F.MIDDLES * (1 - 2 ** -20), [1e-9]]).astype(np.float32)
    x = np.concatenate([x, -x])
    np.testing.assert_array_equal(F.codes_of(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert (F.codes_of(np.array([460.0, 1e30, -1e30])) == [126, 126, 254]).all()
    assert F.codes_of(np.array([np.nan]))[0] & 127 == 127 and F.codes_of(np.array([np.inf]))[0] & 127 == 127


def test_plain_scales_are_the_smallest_that_hold():
    for most in (448.0, 448.0 * (1 + 2 ** -7), 447.0, 1.0, 1.75, 1.7578125, 3.0, 2.0 ** -60, 1e20):
        s = F.scale_of(np.array([0.1 * most, -most]))
        assert most <= 448 * s and most > 448 * s / 2 and np.log2(s) == int(np.log2(s))
    assert F.scale_of(np.zeros(3)) == 2.0 ** -110 and F.scale_of(np.array([np.nan, np.inf, 1.0])) == F.scale_of(np.array([1.0]))
    assert F.scale_of(np.array([1e-40])) == 2.0 ** -110 and F.scale_of(np.array([3.3e38])) == 2.0 ** 119


def test_every_code_times_every_scale_is_a_bf16_number():
    for e in range(F.LEAST, F.MOST + 1):
        x = F.NUMBERS * 2.0 ** e
        assert (torch.from_numpy(x).bfloat16().double().numpy() == x).all() and np.isfinite(torch.from_numpy(x).bfloat16().float().numpy()).all()


@pytest.mark.parametrize("bs,D", [(16, 64), (32, 128), (64, 256)])
def test_places_are_a_permutation(bs, D):
    for at in F.places(bs, D):
        assert (np.sort(at.reshape(-1)) == np.arange(bs * D)).all()


@pytest.mark.parametrize("heads,Hkv,D,bs,tail", [(8, 2, 128, 16, 128), (32, 8, 128, 32, 128), (40, 40, 64, 16, 384), (16, 16, 256, 64, 128), (17, 17, 64, 16, 256)])
def test_sizes(heads, Hkv, D, bs, tail):
    c = _cfg(num_q_heads=heads, num_kv_heads=Hkv, head_dim=D, block_size=bs, dtype=P.LAMPS_E4M3)
    half = 2 * (Hkv * bs * D + tail)
    assert P.lamps_block_bytes(c) == 2 * half and P.lamps_pool_bytes(c) == 32 * half
    assert P.lamps_kv_layout(c) == P.LAMPS_LAYOUT_CODES
    assert P.lamps_kv_bytes_per_token(c) == -(-2 * half // bs)
    wide = _cfg(num_q_heads=heads, num_kv_heads=Hkv, head_dim=D, block_size=bs)
    assert P.lamps_kv_bytes_per_token(c) < 0.6 * P.lamps_kv_bytes_per_token(wide)


def test_configurations_refuse():
    for kw in (dict(head_dim=32), dict(head_dim=96), dict(part_tokens=32), dict(dtype=3), dict(block_size=8)):
        c = dict(dtype=P.LAMPS_E4M3)
        c.update(kw)
        assert P.lamps_pool_bytes(_cfg(**c)) == 0, kw
        with pytest.raises(P.LampsError) as e:
            P.Lamps(_cfg(**c), 4096, 4096, 4096)
        assert e.value.status == -1


def test_read_refuses(lam):
    def read(layer=0, n=2, total=4, start=A, table=A, lens=A, k=2 * A, v=3 * A):
        lam.kv_read_tokens(layer, n, total, start, table, lens, k, v)
    for kw, status, word in [(dict(start=0), -1, "null"), (dict(table=0), -1, "null"), (dict(lens=0), -1, "null"), (dict(k=0), -1, "null"), (dict(v=0), -1, "null"),
                             (dict(k=2 * A + 8), -1, "aligned"), (dict(v=3 * A + 2), -1, "aligned"), (dict(v=2 * A), -1, "overlap"), (dict(v=2 * A + 4 * 2 * 128 * 2 - 16), -1, "overlap"),
                             (dict(layer=2), -2, "layer"), (dict(layer=-1), -2, "layer"), (dict(n=5), -2, "n_req"), (dict(n=-1), -2, "n_req"), (dict(total=-1), -2, "total")]:
        _refused(lambda: read(**kw), status, word)
    read(n=0)
    read(total=0)


def test_appends_refuse(lam):
    for kw in (dict(k=0), dict(v=0), dict(table=0), dict(lens=0), dict(k=A + 8)):
        x = dict(k=A, v=A, table=A, lens=A)
        x.update(kw)
        _refused(lambda: lam.kv_append(0, 2, x["k"], x["v"], x["table"], x["lens"], A, False), -1, "lamps_kv_append")
        _refused(lambda: lam.kv_append_tokens(0, 2, 4, x["k"], x["v"], A, x["table"], x["lens"]), -1, "lamps_kv_append_tokens")
