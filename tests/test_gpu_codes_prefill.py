"""GPU parity of attention of many new tokens per request over a cache of 8 bits, against plain numpy in 64 bits over the numbers that the
codes stand for."""
import numpy as np
import pytest
import torch

import codes_forms as F
from operator_forms import seen, window_attn
from test_gpu_codes_decode import ACC, STEP, bound, cache

pytestmark = pytest.mark.gpu

ALL = 1 << 30
#        H  Hkv D    bs   (context, new tokens) per request
FORMS = [
    (8, 2, 128, 16, [(130, 130), (47, 5), (16, 16), (1, 1), (200, 64), (33, 0)]),
    (4, 4, 128, 32, [(130, 130), (47, 5), (95, 31), (1, 1)]),
    (8, 2, 64, 32, [(95, 95), (64, 33), (300, 2)]),
    (3, 3, 64, 64, [(150, 150), (400, 20)]),
    (16, 1, 256, 16, [(70, 70), (131, 2)]),
    (4, 4, 256, 32, [(90, 90), (50, 6)]),
    (6, 2, 128, 16, [(100, 100), (77, 10)]),                     # groups of 3
    (32, 1, 128, 16, [(45, 45), (90, 3)]),                       # 32 heads per kv head
    (40, 1, 64, 16, [(40, 40)]),                                 # 40
    (8, 2, 128, 16, [(700, 700), (1200, 37), (5, 5)]),           # several tiles
    (8, 1, 64, 16, [(4000, 3), (30, 30), (2500, 40), (700, 1)]),  # walks that are cut
    (16, 2, 256, 16, [(3000, 9), (2000, 2000)]),
    (2, 1, 128, 64, [(9000, 70)]),
    (32, 2, 128, 16, [(1100, 1100), (1500, 1000), (40, 40)]),     # many tiles
    (16, 16, 128, 32, [(2100, 2100), (2600, 2050), (1, 1)]),
    (8, 2, 64, 64, [(928, 928)]),                                # parts that the last of them adds up: short rows
    (16, 4, 256, 16, [(1000, 1000), (7, 3)]),
    (32, 32, 64, 16, [(5000, 5)] + [(30, 30)] * 16),             # and one long context beside many tiles
    (8, 2, 128, 16, [(3000, 70), (800, 70)]),
]


def rounded(out, size):
    """Where weights are rounded to bf16: half a step of each and of their sum, besides what `bound` has."""
    return bound(out, size) + STEP * (size + np.abs(out))


def prefill(rig, layer, q, reqs, table, out, most=0, window=None, sinks=0):
    start = np.concatenate([[0], np.cumsum([n for _, n in reqs])])
    args = rig.ints(start), rig.ints(table), rig.ints([c for c, _ in reqs])
    total, q = int(start[-1]), q.to(rig.dev)
    torch.cuda.synchronize()
    if window is None:
        rig.lamps.prefill_attn(layer, len(reqs), total, q, *args, out, max_new_tokens=most)
    else:
        rig.lamps.prefill_attn_window(layer, len(reqs), total, window, sinks, q, *args, out, max_new_tokens=most)
    torch.cuda.synchronize()
    return start


def check(rig, layer, q, reqs, table, start, out, limit, window=ALL, sinks=0, scale=None):
    pools, got, q = rig.host(), F.f64(out), F.f64(q)
    for r, (c, n) in enumerate(reqs):
        if n == 0:
            continue
        K, V = pools.logical(layer, table[r], c)
        # (of long prompts the first and the last of 100 rows and some between, and all of the last tile)
        for i in [i for i in range(n) if n <= 150 or i % 100 in (0, 41, 99) or n - i < 20]:
            at = start[r] + i
            ref, size = window_attn(q[at:at + 1], K[:c - n + i + 1], V[:c - n + i + 1], c - n + i, window, sinks, scale)
            off = np.abs(got[at] - ref[0]) - limit(ref[0], size[0])
            assert (off <= 0).all(), (r, c, n, i, off.max())


@pytest.mark.parametrize("most", [0, 1, -1])                     # max_new_tokens: unknown, exact, a wavefront per token
@pytest.mark.parametrize("H,Hkv,D,bs,reqs", FORMS)
def test_prefill(H, Hkv, D, bs, reqs, most):
    """Rows behind the last request's are left as they were."""
    rig, table = cache(H, Hkv, D, bs, [c for c, _ in reqs], 31)
    total = sum(n for _, n in reqs)
    q = F.normal(9, total + 3, H, D)
    out = torch.full((total + 3, H, D), 2.5, dtype=torch.bfloat16, device=rig.dev)
    again = out.clone()
    most = max(n for _, n in reqs) if most == 1 else most
    start = prefill(rig, 1, q, reqs, table, out, most)
    prefill(rig, 1, q, reqs, table, again, most)
    assert torch.equal(out, again) and (out[total:] == 2.5).all()
    check(rig, 1, q, reqs, table, start, out, bound if most < 0 or H // Hkv > 32 else rounded)
    rig.close()


@pytest.mark.parametrize("most", [0, -1])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (50, 40), (300, 7)])
@pytest.mark.parametrize("H,Hkv,D,bs,reqs", FORMS)
def test_prefill_window(H, Hkv, D, bs, reqs, window, sinks, most):
    """Entries of blocks that no new token sees name no block; codes that none sees are NaN."""
    rig, table = cache(H, Hkv, D, bs, [c for c, _ in reqs], 32)
    pools, holes = rig.host(), table.copy()
    for r, (c, n) in enumerate(reqs):
        any_sees = np.zeros(c, dtype=bool)
        for p in range(c - max(n, 1), c):
            any_sees |= seen(p, c, window, sinks)
        for b in range((c + bs - 1) // bs):
            if not any_sees[b * bs:(b + 1) * bs].any():
                holes[r, b] = -7
            else:
                for t in range(b * bs, min(c, (b + 1) * bs)):
                    if not any_sees[t]:
                        for which in (0, 1):
                            pools.codes(which, int(table[r, b]), 1)[:, pools.at[which][t % bs]] = 0x7F
    rig.k_pool.copy_(torch.from_numpy(pools.k))
    rig.v_pool.copy_(torch.from_numpy(pools.v))
    q = F.normal(9, sum(n for _, n in reqs), H, D)
    out = torch.full(q.shape, 2.5, dtype=torch.bfloat16, device=rig.dev)
    start = prefill(rig, 1, q, reqs, holes, out, most, window, sinks)
    check(rig, 1, q, reqs, table, start, out, bound if most < 0 or H // Hkv > 32 else rounded, window, sinks)
    rig.close()


@pytest.mark.parametrize("H,Hkv,D,c,n,at", [(8, 2, 128, 130, 100, 77), (4, 4, 64, 130, 100, 77), (8, 4, 256, 130, 100, 77), (32, 2, 128, 2200, 2150, 1407)])
@pytest.mark.parametrize("window", [ALL, 24])
@pytest.mark.parametrize("most", [0, -1])
def test_values_that_are_nan_reach_those_that_see_them(H, Hkv, D, c, n, at, window, most):
    """One NaN value at a position: rows from there on (in the window) are NaN in its dim and head, others are not; a NaN key: in all dims."""
    rig, table = cache(H, Hkv, D, 16, [c], 5)
    q = F.normal(9, n, H, D)
    clean = torch.zeros(n, H, D, dtype=torch.bfloat16, device=rig.dev)
    prefill(rig, 1, q, [(c, n)], table, clean, most, window)
    assert not torch.isnan(clean).any()
    pools = rig.host()
    pools.codes(1, int(table[0, at // 16]), 1)[1, pools.at[1][at % 16, 9]] = 0xFF
    rig.v_pool.copy_(torch.from_numpy(pools.v))
    out = torch.zeros_like(clean)
    prefill(rig, 1, q, [(c, n)], table, out, most, window)
    G, p = H // Hkv, np.arange(c - n, c)
    sees = torch.tensor((p >= at) & (p - window < at), device=rig.dev)
    bad = torch.zeros(n, H, D, dtype=torch.bool, device=rig.dev)
    bad[sees, G:2 * G, 9] = True
    assert torch.equal(torch.isnan(out), bad)
    assert torch.equal(out[~bad], clean[~bad])
    pools.codes(0, int(table[0, at // 16]), 1)[0, pools.at[0][at % 16, 3]] = 0x7F
    rig.k_pool.copy_(torch.from_numpy(pools.k))
    prefill(rig, 1, q, [(c, n)], table, out, most, window)
    bad[sees, :G] = True
    assert torch.equal(torch.isnan(out), bad)
    rig.close()


@pytest.mark.parametrize("scale", [0.02, -0.1, 1.0])
def test_other_scales(scale):
    reqs = [(300, 70), (1500, 20), (33, 33)]
    rig, table = cache(8, 2, 128, 16, [c for c, _ in reqs], 21, scale=scale)
    q = F.normal(3, 123, 8, 128)
    out = torch.zeros(123, 8, 128, dtype=torch.bfloat16, device=rig.dev)
    start = prefill(rig, 1, q, reqs, table, out)
    # (scores to |scale| 340 in size: see test_gpu_codes_decode)
    acc = 2 ** -24 * 12 * abs(scale) * 340 + 4e-5
    check(rig, 1, q, reqs, table, start, out, lambda o, z: STEP * np.abs(o) + (STEP + acc) * (z + np.abs(o)) + 1e-6, scale=scale)
    rig.close()


@pytest.mark.parametrize("n_req", [64, 65, 256, 257, 500])
def test_many_requests(n_req):
    rng = np.random.RandomState(n_req)
    new = rng.randint(0, 9, n_req)
    ctx = new + rng.randint(0, 40, n_req)
    for r in rng.choice(n_req, 4, replace=False):
        new[r] = rng.randint(20, 60)
        ctx[r] = new[r] + 1500
    reqs = list(zip(ctx.tolist(), new.tolist()))
    rig, table = cache(4, 2, 64, 16, ctx.tolist(), n_req)
    q = F.normal(3, int(new.sum()), 4, 64)
    out = torch.full(q.shape, 2.5, dtype=torch.bfloat16, device=rig.dev)
    start = prefill(rig, 1, q, reqs, table, out, int(new.max()))
    check(rig, 1, q, reqs, table, start, out, rounded)
    rig.close()


def test_requests_that_mean_nothing_are_left_alone():
    """Contexts shorter than their new tokens, longer than the row, negative; entries outside the pool; tokens behind total_tokens."""
    ctx = [60, 40, 50, 33, 70]
    rig, table = cache(8, 2, 128, 16, ctx, 5, spare_row=0)
    counts, said = [20, 10, 12, 9, 30], [60, 9, 1 << 30, -1, 70]
    bad = table.copy()
    bad[4, 1] = 1 << 20
    q = F.normal(3, 81, 8, 128)
    for most in (0, -1):
        out = torch.full((81, 8, 128), 2.5, dtype=torch.bfloat16, device=rig.dev)
        start = prefill(rig, 1, q, list(zip(said, counts)), bad, out, most)
        assert (out[20:51] == 2.5).all() and not (out[51:] == 2.5).all(-1).any()
        check(rig, 1, q, [(60, 20)], table, start, out, rounded)
        small = torch.full((81, 8, 128), 2.5, dtype=torch.bfloat16, device=rig.dev)
        rig.lamps.prefill_attn(1, 1, 7, q.to(rig.dev), rig.ints([0, 20]), rig.ints(table), rig.ints([60]), small, max_new_tokens=most)
        torch.cuda.synchronize()
        # (a launch of fewer tokens may take other tiles, whose sums have another order: the first seven rows by the formula, as those of a context of 47)
        assert (small[7:] == 2.5).all()
        check(rig, 1, q, [(47, 7)], table, [0], small, rounded)
    rig.close()


def test_a_prompt_attends_as_its_tokens_do_one_by_one():
    """Prefill's last row and decode's, the same equation by two kernels."""
    ctx = [77, 600]
    rig, table = cache(8, 2, 128, 16, ctx, 8)
    q = F.normal(3, 2, 8, 128)
    one, many = (torch.zeros(2, 8, 128, dtype=torch.bfloat16, device=rig.dev) for _ in range(2))
    rig.lamps.decode_attn(1, 2, q.to(rig.dev), rig.ints(table), rig.ints(ctx), torch.ones(2, dtype=torch.uint8, device=rig.dev), one)
    prefill(rig, 1, q, [(c, 1) for c in ctx], table, many, 1)
    assert ((one.float() - many.float()).abs() <= 3 * STEP * (one.float().abs() + 0.2)).all()
    rig.close()


assert ACC < STEP
