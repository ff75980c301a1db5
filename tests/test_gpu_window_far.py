"""Windowed attention over scores near the ends of what 32 bits hold: every kernel that a call may be sent to treats them alike."""
import numpy as np
import pytest
import torch

import lamps_workloads as W
import paper_2410_18248_amd as P
from operator_forms import f64, seen
from rig import Rig, n2t, to_f64

pytestmark = pytest.mark.gpu

# Every product of a query and a key is 1.875 2^119 (head size 128), their sum 1.875 2^126, and times scale and log2(e), which make a power of two
# together, the score is 1.875 2^127 = 3.19e38 or 1.875 2^100: all of it exact.  All scores of a row are equal, so its weights are: a row is the mean of
# the values that it sees.
LOG2E = np.float32(1.4426950408889634)


def _scale(power):
    """A scale whose product with log2(e) is 2^power in 32 bits."""
    x = np.float32(2.0 ** power / 1.4426950408889634)
    near = [np.nextafter(x, np.float32(0)), x, np.nextafter(x, np.float32(np.inf))]
    return next(float(y) for y in near if np.float32(y * LOG2E) == np.float32(2.0 ** power))


@pytest.mark.parametrize("sign,power", [(-1, 1), (-1, -26), (1, 1)])
@pytest.mark.parametrize("H,Hkv,D,reqs,window,sinks", [
    (16, 8, 128, [(2600, 2500), (2300, 2300)], 1100, 3),       # two teams of waves
    (16, 8, 128, [(300, 300), (77, 20)], 40, 3),
    (4, 2, 256, [(300, 300), (130, 50)], 40, 3),               # two teams, heads of 256
    (8, 2, 64, [(900, 20), (700, 9)], 600, 3),                 # tiles in parts
    (4, 4, 128, [(300, 300), (77, 20)], 40, 3),
])
def test_equal_scores_of_any_size(H, Hkv, D, reqs, window, sinks, sign, power):
    ctx = [c for c, _ in reqs]
    geom = W.Geometry(1, H, Hkv, D, 16, sum((c + 15) // 16 for c in ctx) + 2, max((c + 15) // 16 for c in ctx), "bf16")
    rig = Rig(geom, len(reqs), scale=_scale(power))
    table, _ = W.deal_block_table(W.permutation(3, geom.num_blocks), ctx, geom)
    K, V = zip(*[W.logical_kv(5 + r, geom, c) for r, c in enumerate(ctx)])
    bits = lambda x: W.f32_to_bf16_bits(np.array([x], dtype=np.float32))[0]
    K = [np.full_like(k, bits(2.0 ** 60)) for k in K]
    rig.page_requests(0, table, K, V)
    total = sum(n for _, n in reqs)
    q = np.full((total, H, D), bits(sign * 1.875 * 2.0 ** 66 / D), dtype=np.uint16)
    start = np.concatenate([[0], np.cumsum([n for _, n in reqs])])
    dev = rig.dev
    args = n2t(q, dev), torch.tensor(start, dtype=torch.int32, device=dev), torch.as_tensor(table, device=dev), torch.tensor(ctx, dtype=torch.int32, device=dev)
    for most in (0, -1):
        out = torch.zeros((total, H, D), dtype=rig.tdtype, device=dev)
        torch.cuda.synchronize()
        rig.lamps.prefill_attn_window(0, len(reqs), total, window, sinks, *args, out, max_new_tokens=most)
        torch.cuda.synchronize()
        got = to_f64(out)
        for r, (c, n) in enumerate(reqs):
            v = f64(V[r])
            for i in [i for i in range(n) if n <= 60 or i % 97 in (0, 50) or n - i < 5]:
                on = seen(c - n + i, c, window, sinks)
                ref, size = v[on].mean(0), np.abs(v[on]).mean(0)
                # (the weights are ones; a mean of up to 1 100 values in 32 bits, 1 100 2^-24 = 6.6e-5 of their sizes, and half a step of bf16)
                off = 2.0 ** -8 * np.abs(ref) + 7e-5 * (size + np.abs(ref)) + 1e-6
                for g in range(H):
                    good = np.abs(got[start[r] + i, g] - ref[g * Hkv // H]) <= off[g * Hkv // H]
                    assert bool(good.all()), (most, r, i, g)
    rig.close()
