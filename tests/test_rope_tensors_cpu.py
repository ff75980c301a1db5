"""What a call of lamps_rope_append finds wrong with the tensors that it is given, before anything reaches the library."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2410_18248_amd as P
from test_boundary_cpu import _cfg
from test_operators_cpu import A, _refused


class OnDevice:
    """What the binding asks of a tensor on the device."""
    is_cuda = True

    def __init__(self, x):
        self.x, self.dtype = x, x.dtype

    def __getattr__(self, name):
        return getattr(self.x, name)


@pytest.fixture(params=[P.LAMPS_BF16, P.LAMPS_F32])
def lam(request):
    buf = ctypes.create_string_buffer(4096)
    a = (ctypes.addressof(buf) + 255) & ~255
    cfg = _cfg()
    cfg.dtype = request.param
    x = P.Lamps(cfg, a, a, a)
    x._buf = buf
    yield x
    x.destroy()


def _calls(lam, rope=None, q=A, k=2 * A, v=3 * A, out=4 * A, strides=(0, 0, 0)):
    rope = rope or P.LampsRope(64, frequencies=A)
    lam.rope_append(0, 0, rope, q, k, v, A, A, A, False, out, *strides)                  # (of no requests: nothing is enqueued)
    lam.rope_append_tokens(0, 0, 0, rope, q, k, v, A, A, A, out, *strides)


def test_weights_are_a_heads_in_the_caches_type(lam):
    D = lam.cfg.head_dim
    mine, other = (torch.bfloat16, torch.float32) if lam.cfg.dtype == P.LAMPS_BF16 else (torch.float32, torch.bfloat16)
    for name in ("q_weight", "k_weight"):
        good = P.LampsRope(64, frequencies=A, normalise=True, **{name: OnDevice(torch.ones(D, dtype=mine))})
        _calls(lam, good)
        _calls(lam, good)
        for bad in (torch.ones(D, dtype=other), torch.ones(D, dtype=torch.float16), torch.ones(D // 2, dtype=mine), torch.ones(2, D, dtype=mine)):
            for normalise in (True, False):                  # (read in both cases)
                rope = P.LampsRope(64, frequencies=A, normalise=normalise, **{name: OnDevice(bad)})
                for _ in range(2):
                    _refused(lambda: _calls(lam, rope), -1, name)


def test_a_rope_that_suits_one_cache_is_looked_at_again_for_another(lam):
    rope = P.LampsRope(64, frequencies=A, q_weight=OnDevice(torch.ones(lam.cfg.head_dim, dtype=torch.bfloat16)))
    suits = lam.cfg.dtype == P.LAMPS_BF16
    cfg = _cfg()
    cfg.dtype = P.LAMPS_F32 if suits else P.LAMPS_BF16
    other = P.Lamps(cfg, *lam._keep)
    good, bad = (lam, other) if suits else (other, lam)
    for _ in range(2):
        _calls(good, rope)
        _refused(lambda: _calls(bad, rope), -1, "q_weight")
    other.destroy()


def test_tensors_in_host_memory(lam):
    D, mine = lam.cfg.head_dim, torch.bfloat16 if lam.cfg.dtype == P.LAMPS_BF16 else torch.float32
    f = torch.tensor(P.lamps_rope_frequencies(64, 10000.0), dtype=torch.float64)
    _calls(lam, P.LampsRope(64, frequencies=OnDevice(f)))
    for kw in (dict(frequencies=f), dict(frequencies=f.numpy()), dict(frequencies=A, q_weight=torch.ones(D, dtype=mine)),
               dict(frequencies=A, k_weight=torch.ones(D, dtype=mine)), dict(frequencies=A, k_weight=np.ones(D, dtype=np.float32))):
        _refused(lambda: _calls(lam, P.LampsRope(64, **kw)), -1, "host memory")


def test_rows_apart_need_their_stride(lam):
    H, Hkv, D = lam.cfg.num_q_heads, lam.cfg.num_kv_heads, lam.cfg.head_dim
    x = torch.zeros((3, H + 2 * Hkv, D), dtype=torch.bfloat16 if lam.cfg.dtype == P.LAMPS_BF16 else torch.float32)
    parts = dict(q=x[:, :H], k=x[:, H:H + Hkv], v=x[:, H + Hkv:])
    step = x.stride(0)
    for at, (name, part) in enumerate(parts.items()):
        _refused(lambda: _calls(lam, **{name: part}), -1, "stride")
        strides = [0, 0, 0]
        strides[at] = step
        _calls(lam, strides=strides, **{name: part})
        _calls(lam, **{name: part[:1]})                      # (one row follows nothing)
        _calls(lam, **{name: part.contiguous()})
    _refused(lambda: _calls(lam, out=parts["q"]), -1, "q_out must be contiguous")
    _calls(lam, out=parts["q"].contiguous())
