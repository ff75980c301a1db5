"""GPU parity of attention of one new token per request over a cache of 8 bits, against plain numpy in 64 bits over the numbers that the
codes stand for."""
import numpy as np
import pytest
import torch

import codes_forms as F
import paper_2410_18248_amd as P
from operator_forms import window_attn

pytestmark = pytest.mark.gpu

# Half a step of bf16, 2^-8 of the value, for the output's rounding; weights are pairs of bf16 and off by 2^-17 = 8e-6.  A score is a sum of D products, at
# most 12 roundings deep, of |q||k| scale < 30 for normal vectors, so off by 12 2^-24 30 = 2e-5, which is the relative error of a weight; and the reference of
# the exponentials lies up to 8 below the largest score, which changes no relative error.
STEP, ACC = 2.0 ** -8, 6e-5


def bound(out, size):
    return STEP * np.abs(out) + ACC * (size + np.abs(out)) + 1e-6


#        H   Hkv D    bs  context lengths
FORMS = [
    (8, 2, 128, 16, [1, 0, 15, 16, 17, 31, 32, 33, 100, 333, 1000]),
    (4, 4, 128, 32, [1, 40, 129, 500, 64]),                    # plain heads
    (8, 8, 64, 16, [63, 1, 200, 7]),
    (16, 2, 64, 64, [130, 1, 64]),
    (16, 4, 256, 16, [90, 3, 47]),
    (3, 3, 256, 64, [70, 200]),
    (6, 2, 128, 16, [45, 130]),                                # groups of 3
    (32, 1, 128, 16, [300, 20]),                               # two passes of 16 heads
    (40, 1, 64, 16, [100]),                                    # 10 heads a pass
    (17, 1, 128, 16, [80, 5]),                                 # 17 passes of one
    (8, 2, 128, 16, [5000, 30, 900, 1, 2500, 64]),             # cut
    (2, 1, 64, 32, [9000]),
    (8, 8, 64, 16, [(37 * i) % 129 for i in range(150)]),        # many short ranges: a wave each
    (40, 40, 128, 32, [(17 * i) % 97 for i in range(30)]),
    (32, 8, 128, 16, [(29 * i) % 129 for i in range(131)]),
    (16, 16, 256, 16, [(53 * i) % 127 for i in range(67)]),
    (96, 3, 64, 16, [5] * 200 + [128] * 70),                     # the same in two passes, and a second launch for 14 requests
]


def cache(H, Hkv, D, bs, ctx, seed, layers=2, scale=0.0, size=1.0, max_batch=0, spare_row=1):
    rig = F.CodesRig(layers, H, Hkv, D, bs, sum((c + bs - 1) // bs for c in ctx) + 3, (max(ctx) + bs - 1) // bs + spare_row, max_batch or len(ctx), scale=scale, seed=seed)
    table = rig.deal(ctx, seed)
    k, v = F.normal(seed + 1, sum(ctx), Hkv, D, size=size), F.normal(seed + 2, sum(ctx), Hkv, D)
    if sum(ctx):
        rig.append_tokens(layers - 1, k, v, ctx, table, ctx)
    return rig, table


def decode(rig, layer, q, table, ctx, running, window=None, sinks=0):
    out = torch.full(q.shape, 2.5, dtype=torch.bfloat16, device=rig.dev)
    args = q.to(rig.dev), rig.ints(table), rig.ints(ctx), torch.tensor(running, dtype=torch.uint8, device=rig.dev)
    torch.cuda.synchronize()
    if window is None:
        rig.lamps.decode_attn(layer, len(ctx), *args, out)
    else:
        rig.lamps.decode_attn_window(layer, len(ctx), window, sinks, *args, out)
    torch.cuda.synchronize()
    return out


def check(rig, layer, q, table, ctx, running, out, window=1 << 30, sinks=0, scale=None, rows=None):
    pools, got = rig.host(), F.f64(out)
    for r in range(len(ctx)) if rows is None else rows:
        if not running[r]:
            assert (got[r] == 2.5).all()
        elif ctx[r] == 0:
            assert (got[r] == 0).all()
        else:
            K, V = pools.logical(layer, table[r], ctx[r])
            ref, size = window_attn(F.f64(q[r:r + 1]), K, V, ctx[r] - 1, window, sinks, scale)
            off = np.abs(got[r] - ref[0]) - bound(ref[0], size[0])
            assert (off <= 0).all(), (r, ctx[r], off.max())


@pytest.mark.parametrize("H,Hkv,D,bs,ctx", FORMS)
def test_decode(H, Hkv, D, bs, ctx):
    rig, table = cache(H, Hkv, D, bs, ctx, 11)
    q, running = F.normal(3, len(ctx), H, D), np.ones(len(ctx), dtype=int)
    running[2:3] = 0
    out = decode(rig, 1, q, table, ctx, running)
    check(rig, 1, q, table, ctx, running, out)
    assert torch.equal(out, decode(rig, 1, q, table, ctx, running))
    # the same bits from the library's own scratch memory
    again = torch.full_like(out, 2.5)
    args = q.to(rig.dev), rig.k_pool, rig.v_pool, rig.ints(table), rig.ints(ctx), torch.tensor(running, dtype=torch.uint8, device=rig.dev)
    torch.cuda.synchronize()
    P.lamps_decode_attn_static(rig.cfg, rig.compute.cuda_stream, 1, len(ctx), *args, again)
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    rig.close()


@pytest.mark.parametrize("H,Hkv,D,bs,ctx", FORMS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 3), (50, 40), (400, 16), (1 << 30, 1 << 30)])
def test_decode_window(H, Hkv, D, bs, ctx, window, sinks):
    """Table entries of blocks that nothing sees name no block."""
    rig, table = cache(H, Hkv, D, bs, ctx, 12)
    holes = table.copy()
    for r, c in enumerate(ctx):
        for b in range((c + bs - 1) // bs):
            t = np.arange(b * bs, min(c, (b + 1) * bs))
            if not ((t >= c - window) | (t < sinks)).any():
                holes[r, b] = -5
    q, running = F.normal(4, len(ctx), H, D), np.ones(len(ctx), dtype=int)
    out = decode(rig, 1, q, holes, ctx, running, window, sinks)
    check(rig, 1, q, table, ctx, running, out, window, sinks)
    rig.close()


@pytest.mark.parametrize("scale", [0.02, -0.1, 2.0])
def test_other_scales_and_numbers_of_other_sizes(scale):
    """Scores to some 100; keys of 2^-20 and 2^10 times the usual size under softmax scales that make up for it."""
    for size in (1.0, 2.0 ** -20, 2.0 ** 10):
        ctx = [70, 1500, 33]
        rig, table = cache(8, 2, 128, 16, ctx, 21, scale=scale / size, size=size)
        q = F.normal(3, 3, 8, 128)
        out = decode(rig, 1, q, table, ctx, [1, 1, 1])
        # (a score is up to |scale| 30 sqrt(128) ~ 340 |scale| in size: its error, as derived above, in proportion)
        pools, got = rig.host(), F.f64(out)
        acc = 2 ** -24 * 12 * abs(scale) * 340 + 4e-5
        for r in range(3):
            K, V = pools.logical(1, table[r], ctx[r])
            ref, sz = window_attn(F.f64(q[r:r + 1]), K, V, ctx[r] - 1, 1 << 30, 0, scale / size)
            off = np.abs(got[r] - ref[0]) - (STEP * np.abs(ref[0]) + acc * (sz[0] + np.abs(ref[0])) + 1e-6)
            assert (off <= 0).all(), (size, r, off.max())
        rig.close()


def test_a_score_that_stands_out_anywhere():
    """One key that fits the query, at the first position, the last, and where units and parts end."""
    ctx = [2500]
    for at in (0, 15, 16, 31, 32, 255, 256, 1249, 2495, 2499):
        rig = F.CodesRig(1, 8, 2, 128, 16, 160, 158, 1)
        table = rig.deal(ctx)
        k, v, q = F.normal(1, 2500, 2, 128), F.normal(2, 2500, 2, 128), F.normal(3, 1, 8, 128)
        k[at] = (q[0, ::4] * 3).bfloat16()
        rig.append_tokens(0, k, v, ctx, table, ctx)
        check(rig, 0, q, table, ctx, [1], decode(rig, 0, q, table, ctx, [1]))
        rig.close()


def test_what_is_behind_the_context_or_outside_the_window_does_not_count():
    """NaN codes in slots behind the context, outside the window, and in other heads; a NaN that counts makes its row NaN."""
    ctx, window, sinks = [37, 70, 16], 20, 3
    rig, table = cache(4, 2, 64, 16, [48, 80, 16], 9)
    pools = rig.host()
    for r, c in enumerate(ctx):
        for b in range((c + 15) // 16):
            for s in range(16):
                t = b * 16 + s
                if not (t < c and (t >= c - window or t < sinks)):
                    for which in (0, 1):
                        pools.codes(which, int(table[r, b]), 1)[:, pools.at[which][s]] = 0x7F + 0x80 * (s & 1)
    rig.k_pool.copy_(torch.from_numpy(pools.k))
    rig.v_pool.copy_(torch.from_numpy(pools.v))
    q = F.normal(3, 3, 4, 64)
    out = decode(rig, 1, q, table, ctx, [1, 1, 1], window, sinks)
    check(rig, 1, q, table, ctx, [1, 1, 1], out, window, sinks)
    pools.codes(1, int(table[1, 4]), 1)[0, pools.at[1][5, 7]] = 0xFF      # position 69, head 0, dim 7
    rig.v_pool.copy_(torch.from_numpy(pools.v))
    got = decode(rig, 1, q, table, ctx, [1, 1, 1], window, sinks)
    nan = torch.isnan(got)
    assert nan[1, :2, 7].all() and nan.sum() == 2
    pools.codes(0, int(table[1, 4]), 1)[1, pools.at[0][5, 7]] = 0x7F
    rig.k_pool.copy_(torch.from_numpy(pools.k))
    nan = torch.isnan(decode(rig, 1, q, table, ctx, [1, 1, 1], window, sinks))
    assert nan[1, 2:].all() and not nan[0].any() and not nan[2].any()
    rig.close()


@pytest.mark.parametrize("batch,long", [(64, 3000), (65, 3000), (255, 2000), (256, 0), (257, 1000), (600, 700)])
def test_many_requests(batch, long):
    """Short contexts with a few long ones among them, some waiting; more than one launch holds."""
    rng = np.random.RandomState(batch)
    ctx = rng.randint(0, 60, batch)
    if long:
        ctx[rng.choice(batch, 3, replace=False)] = [long, long - 17, long // 2]
    running = (rng.rand(batch) < 0.8).astype(int)
    rig, table = cache(4, 2, 64, 16, ctx.tolist(), batch)
    q = F.normal(3, batch, 4, 64)
    check(rig, 1, q, table, ctx.tolist(), running, decode(rig, 1, q, table, ctx.tolist(), running))
    rig.close()


def test_lengths_and_entries_that_mean_nothing_do_no_harm():
    """Lengths behind the row are cut to it, negative ones are empty, entries outside the pool are not followed; other rows are as they are."""
    ctx = [40, 70, 33, 20]
    rig, table = cache(8, 2, 128, 16, ctx, 5, spare_row=0)
    bad_table, bad_ctx = table.copy(), [1 << 30, -3, 33, 20]
    bad_table[0, 1:], bad_table[2, 1] = 1 << 30, -1
    q = F.normal(3, 4, 8, 128)
    out = decode(rig, 1, q, bad_table, bad_ctx, [1, 1, 1, 1])
    check(rig, 1, q, table, ctx, [1] * 4, out, rows=[3])
    assert (out[1] == 0).all()
    rig.close()


def test_out_and_rows_that_lie_oddly():
    """out 2 bytes off a word, as lamps_decode_attn allows."""
    ctx = [40, 700]
    rig, table = cache(8, 2, 64, 16, ctx, 5)
    q = F.normal(3, 2, 8, 64)
    room = torch.zeros(2 * 8 * 64 + 1, dtype=torch.bfloat16, device=rig.dev)
    rig.lamps.decode_attn(1, 2, q.to(rig.dev), rig.ints(table), rig.ints(ctx), torch.ones(2, dtype=torch.uint8, device=rig.dev), room[1:])
    torch.cuda.synchronize()
    check(rig, 1, q, table, ctx, [1, 1], room[1:].view(2, 8, 64))
    assert room[0] == 0
    rig.close()
