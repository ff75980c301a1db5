"""The operators around the cache without a GPU: what they refuse, with nothing enqueued, and the frequencies."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2410_18248_amd as P
from test_boundary_cpu import _cfg


@pytest.fixture
def lam():
    buf = ctypes.create_string_buffer(4096)
    a = (ctypes.addressof(buf) + 255) & ~255
    x = P.Lamps(_cfg(), a, a, a)                    # "device" memory that is never looked at
    x._buf = buf
    yield x
    x.destroy()


def _refused(call, status, word):
    with pytest.raises(P.LampsError) as e:
        call()
    assert e.value.status == status and word in str(e.value), str(e.value)


A = 1 << 20                                         # addresses of nothing


def test_window_calls_refuse(lam):
    def decode(layer=0, batch=2, window=8, sinks=1, q=A, table=A, lens=A, mask=A, out=2 * A):
        lam.decode_attn_window(layer, batch, window, sinks, q, table, lens, mask, out)

    def prefill(layer=0, n=2, total=4, window=8, sinks=1, q=A, start=A, table=A, lens=A, out=2 * A):
        lam.prefill_attn_window(layer, n, total, window, sinks, q, start, table, lens, out)
    for call, own in ((decode, "mask"), (prefill, "start")):
        for kw, status, word in [(dict(q=0), -1, "null"), (dict(table=0), -1, "null"), (dict(lens=0), -1, "null"), (dict(out=0), -1, "null"),
                                 ({own: 0}, -1, "null"), (dict(q=A + 8), -1, "aligned"), (dict(out=A + 2), -1, "aligned"), (dict(window=0), -1, "window"),
                                 (dict(window=-5), -1, "window"), (dict(sinks=-1), -1, "sinks"), (dict(layer=2), -2, "layer"), (dict(layer=-1), -2, "layer")]:
            _refused(lambda: call(**kw), status, word)
    _refused(lambda: decode(batch=5), -2, "batch")
    _refused(lambda: decode(batch=-1), -2, "batch")
    _refused(lambda: prefill(n=5), -2, "n_req")
    _refused(lambda: prefill(total=-1), -2, "total")
    decode(batch=0)
    prefill(n=0)
    prefill(total=0)


def test_rope_calls_refuse(lam):
    def rope(**kw):
        x = dict(rotary_dim=64, frequencies=A, normalise=True, q_weight=A, k_weight=A)
        x.update(kw)
        return P.LampsRope(**x)

    def one(r=None, layer=0, batch=2, q=A, k=2 * A, v=3 * A, table=A, lens=A, mask=A, out=4 * A, strides=(0, 0, 0)):
        lam.rope_append(layer, batch, r or rope(), q, k, v, table, lens, mask, False, out, *strides)

    def many(r=None, layer=0, batch=2, total=4, q=A, k=2 * A, v=3 * A, start=A, table=A, lens=A, out=4 * A, strides=(0, 0, 0)):
        lam.rope_append_tokens(layer, batch, total, r or rope(), q, k, v, start, table, lens, out, *strides)
    row = 8 * 128
    for call, own in ((one, "mask"), (many, "start")):
        for kw, status, word in [
                (dict(q=0), -1, "null"), (dict(k=0), -1, "null"), (dict(v=0), -1, "null"), (dict(table=0), -1, "null"), (dict(lens=0), -1, "null"),
                (dict(out=0), -1, "null"), ({own: 0}, -1, "null"), (dict(q=A + 8), -1, "aligned"), (dict(v=A + 4), -1, "aligned"),
                (dict(r=rope(rotary_dim=24)), -1, "rotary_dim"), (dict(r=rope(rotary_dim=-16)), -1, "rotary_dim"),
                (dict(r=rope(rotary_dim=144)), -1, "rotary_dim"), (dict(r=rope(pairs=2)), -1, "pairs"), (dict(r=rope(frequencies=None)), -1, "frequencies"),
                (dict(r=rope(frequencies=A + 4)), -1, "frequencies"), (dict(r=rope(q_weight=A + 8)), -1, "weight"),
                (dict(r=rope(norm_eps=-1.0)), -1, "norm_eps"), (dict(r=rope(norm_eps=math.nan)), -1, "norm_eps"),
                (dict(r=rope(amplitude=math.inf)), -1, "amplitude"), (dict(strides=(row - 8, 0, 0)), -1, "stride"), (dict(strides=(0, 8, 0)), -1, "stride"),
                (dict(strides=(0, 0, -256)), -1, "stride"), (dict(strides=(row + 4, 0, 0)), -1, "16 bytes"), (dict(strides=(1 << 62, 0, 0)), -1, "stride"),
                (dict(out=A, strides=(row + 8, 0, 0)), -1, "overlaps"), (dict(out=A + 16), -1, "overlaps"), (dict(out=2 * A), -1, "overlaps"),
                (dict(out=3 * A - 16), -1, "overlaps"), (dict(layer=2), -2, "layer"), (dict(layer=-1), -2, "layer")]:
            _refused(lambda: call(**kw), status, word)
    for kw in (dict(batch=5), dict(batch=-1)):
        _refused(lambda: one(**kw), -2, "batch")
        _refused(lambda: many(**kw), -2, "n_req")
    _refused(lambda: many(total=-1), -2, "total")
    one(batch=0)
    many(total=0)
    many(batch=0)
    assert lam.lib.lamps_rope_append(lam.h, 0, 1, None, A, 0, A, 0, A, 0, A, A, A, 0, 2 * A) == -1


def test_rope_strides_beyond_what_64_bits_hold(lam):
    # 2^30 rows of 2^40 elements: the end of such rows has no address, and rows of 2^28 elements that do not overlap must not seem to
    rope = P.LampsRope(64, frequencies=A)
    for at in range(3):
        strides = [0, 0, 0]
        strides[at] = 1 << 40
        _refused(lambda: lam.rope_append_tokens(0, 2, 1 << 30, rope, A, 2 * A, 3 * A, A, A, A, 1 << 61, *strides), -1, "2^28")
        _refused(lambda: lam.rope_append(0, 2, rope, A, 2 * A, 3 * A, A, A, A, False, 1 << 61, *strides), -1, "2^28")
    _refused(lambda: lam.rope_append_tokens(2, 2, 1 << 30, rope, A, 2 * A, 3 * A, A, A, A, 1 << 61, 1 << 28, 1 << 28, 1 << 28), -2, "layer")
    _refused(lambda: lam.rope_append_tokens(2, 2, 1 << 30, rope, A, 2 * A, 3 * A, A, A, A, 1 << 50, 1 << 28, 1 << 28, 1 << 28), -1, "overlaps")


def test_rope_tensors_of_another_form_refuse():
    f = torch.tensor(P.lamps_rope_frequencies(64, 10000.0), dtype=torch.float64)
    P.LampsRope(64, frequencies=f)
    P.LampsRope(32, frequencies=f)                  # (more than it reads)
    for bad in (f.float(), f[:31], f.view(torch.int64), torch.stack([f, f], 1)[:, 0]):
        _refused(lambda: P.LampsRope(64, frequencies=bad), -1, "float64")
    w = torch.ones(128, 2)
    for kw in (dict(q_weight=w[:, 0]), dict(k_weight=w[:, 1])):
        _refused(lambda: P.LampsRope(64, frequencies=f, normalise=True, **kw), -1, "contiguous")


def test_tables_refuse(lam):
    def call(n=3, total=4, cached=A, new=2 * A, ids=3 * A, n_ids=5, grow=False, table=4 * A, lens=5 * A, start=6 * A, slots=7 * A, report=8 * A):
        lam.batch_tables(n, total, cached, new, ids, n_ids, grow, table, lens, start, slots, report)
    for kw, status, word in [
            (dict(cached=0), -1, "null"), (dict(new=0), -1, "null"), (dict(ids=0), -1, "null"), (dict(table=0), -1, "null"), (dict(lens=0), -1, "null"),
            (dict(start=0), -1, "null"), (dict(lens=A), -1, "overlaps"), (dict(lens=A + 8), -1, "overlaps"), (dict(start=2 * A - 4), -1, "overlaps"),
            (dict(table=3 * A - 4), -1, "overlaps"), (dict(slots=4 * A + 8), -1, "overlap"), (dict(report=7 * A), -1, "overlap"),
            (dict(slots=7 * A + 4), -1, "aligned"), (dict(cached=A + 2), -1, "aligned"), (dict(report=8 * A + 1), -1, "aligned"),
            (dict(n=5), -2, "n_req"), (dict(n=-1), -2, "n_req"), (dict(total=-1), -2, "total"), (dict(n_ids=-1), -2, "n_ids"), (dict(n_ids=33), -2, "blocks")]:
        _refused(lambda: call(**kw), status, word)


def test_frequencies():
    n, base, s, length, lo, hi = 64, 10000.0, 8.0, 4096.0, 1.0, 32.0
    f = np.array([base ** (-2.0 * i / n) for i in range(n // 2)])
    close = lambda a, b: np.testing.assert_allclose(a, b, rtol=1e-14)
    close(P.lamps_rope_frequencies(n, base), f)
    close(P.lamps_rope_frequencies(n, base, P.LAMPS_ROPE_LINEAR, s), f / s)
    close(P.lamps_rope_frequencies(n, base, P.LAMPS_ROPE_BASE, s), [(base * s ** (n / (n - 2))) ** (-2.0 * i / n) for i in range(n // 2)])
    # with the changed base the slowest pair turns as interpolated positions would, the fastest as before
    g = P.lamps_rope_frequencies(n, base, P.LAMPS_ROPE_BASE, s)
    assert abs(g[0] - 1.0) < 1e-15 and abs(g[-1] / (f[-1] / s) - 1) < 1e-12
    g = np.array(P.lamps_rope_frequencies(n, base, P.LAMPS_ROPE_BY_PARTS, s, length, lo, hi))
    turns = length * f / (2 * math.pi)
    assert (g[turns >= hi] == f[turns >= hi]).all()
    close(g[turns <= lo], f[turns <= lo] / s)
    between = (turns > lo) & (turns < hi)
    assert between.sum() >= 5
    k = (turns[between] - lo) / (hi - lo)
    close(g[between], k * f[between] + (1 - k) * f[between] / s)
    assert P.lamps_rope_frequencies(0, base) == []
    for bad in [dict(rotary_dim=24), dict(rotary_dim=-16), dict(base=1.0), dict(base=math.inf), dict(base=math.nan), dict(scaling=4), dict(scaling=-1),
                dict(scaling=1, factor=0.5), dict(scaling=2, factor=math.nan), dict(scaling=3, factor=2.0, original_positions=0.0, low_turns=1.0, high_turns=2.0),
                dict(scaling=3, factor=2.0, original_positions=9.0, low_turns=2.0, high_turns=2.0),
                dict(scaling=3, factor=2.0, original_positions=9.0, low_turns=1.0, high_turns=math.inf)]:
        kw = dict(rotary_dim=64, base=10000.0)
        kw.update(bad)
        with pytest.raises(P.LampsError):
            P.lamps_rope_frequencies(**kw)
