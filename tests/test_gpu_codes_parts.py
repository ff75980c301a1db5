"""GPU parity of attention over a cache of 8 bits where its launches are cut into many parts: plain heads, heads of 256, wide groups; against plain numpy
in 64 bits over the numbers that the codes stand for."""
import numpy as np
import pytest
import torch

import codes_forms as F
import test_gpu_codes_decode as decoding
import test_gpu_codes_prefill as prefilling

pytestmark = pytest.mark.gpu

#        H   Hkv D    bs   (context, new tokens) per request
FORMS = [
    (32, 32, 128, 16, [(3600, 512)]),
    (8, 8, 128, 16, [(6000, 130), (900, 300)]),
    (16, 16, 64, 32, [(5000, 200)]),
    (8, 8, 256, 16, [(2500, 100), (31, 31)]),
    (5, 5, 128, 16, [(4000, 40), (4000, 64), (4000, 65)]),
    (17, 1, 256, 16, [(1500, 60)]),                              # tiles of 128 columns of 256
    (32, 1, 256, 32, [(700, 90), (40, 40)]),
]


@pytest.mark.parametrize("window,sinks", [(None, 0), (2000, 5)])
@pytest.mark.parametrize("H,Hkv,D,bs,reqs", FORMS)
def test_many_tokens_on_long_contexts(H, Hkv, D, bs, reqs, window, sinks):
    """Twice, with the same bits, and rows behind the last request's are left as they were."""
    rig, table = decoding.cache(H, Hkv, D, bs, [c for c, _ in reqs], 41)
    total, most = sum(n for _, n in reqs), max(n for _, n in reqs)
    q = F.normal(9, total + 2, H, D)
    out = torch.full((total + 2, H, D), 2.5, dtype=torch.bfloat16, device=rig.dev)
    again = out.clone()
    start = prefilling.prefill(rig, 1, q, reqs, table, out, most, window, sinks)
    prefilling.prefill(rig, 1, q, reqs, table, again, most, window, sinks)
    assert torch.equal(out, again) and (out[total:] == 2.5).all()
    prefilling.check(rig, 1, q, reqs, table, start, out, prefilling.rounded, window or prefilling.ALL, sinks)
    rig.close()


@pytest.mark.parametrize("H,Hkv,D,ctx", [(16, 1, 256, [3000, 1, 40]), (32, 2, 256, [300, 5000]), (32, 1, 256, [64] * 70)])
def test_one_token_with_sixteen_heads_of_256_in_a_pass(H, Hkv, D, ctx):
    """The most that a workgroup's waves hand over: 66 048 bytes."""
    rig, table = decoding.cache(H, Hkv, D, 16, ctx, 42)
    q, running = F.normal(3, len(ctx), H, D), np.ones(len(ctx), dtype=int)
    out = decoding.decode(rig, 1, q, table, ctx, running)
    assert torch.equal(out, decoding.decode(rig, 1, q, table, ctx, running))
    decoding.check(rig, 1, q, table, ctx, running, out)
    rig.close()
