"""GPU parity of lamps_decode_attn_window and lamps_prefill_attn_window: every new token over the last positions up to its own and
the first few, against plain numpy in 64 bits."""
import numpy as np
import pytest
import torch

import lamps_workloads as W
import paper_2410_18248_amd as P
from operator_forms import f64, seen, window_attn
from rig import Rig, n2t, to_f64

pytestmark = pytest.mark.gpu

#        dtype  H  Hkv D    bs  (context, new tokens) per request                    windows and sinks
CASES = [
    ("bf16", 8, 2, 128, 16, [(130, 130), (47, 5), (16, 16), (1, 1), (200, 64), (33, 0)], [(1, 0), (16, 4), (50, 17), (129, 3), (1000, 0)]),
    ("bf16", 4, 4, 128, 16, [(130, 130), (47, 5), (16, 16), (1, 1), (95, 31)], [(1, 1), (15, 0), (40, 16), (500, 7)]),
    ("bf16", 8, 2, 64, 32, [(95, 95), (64, 33), (300, 2)], [(7, 5), (64, 40)]),
    ("bf16", 3, 3, 64, 64, [(150, 150), (400, 20)], [(33, 1), (100, 70)]),
    ("bf16", 16, 1, 256, 16, [(70, 70), (131, 2)], [(20, 2), (65, 33)]),
    ("bf16", 4, 4, 256, 32, [(90, 90), (50, 6)], [(31, 4)]),
    ("bf16", 6, 2, 128, 16, [(100, 100), (77, 10)], [(32, 0)]),                    # groups of 3
    ("bf16", 32, 1, 128, 16, [(45, 45), (90, 3)], [(17, 3)]),                      # 32 heads per kv head
    ("bf16", 40, 1, 64, 16, [(40, 40)], [(9, 2)]),                                 # 40
    ("bf16", 8, 2, 128, 16, [(700, 700), (1200, 37)], [(260, 4), (97, 70)]),       # several tiles of new tokens
    ("bf16", 4, 4, 128, 16, [(700, 700), (1200, 37)], [(260, 4)]),
    ("bf16", 8, 4, 64, 16, [(900, 30), (700, 1), (1500, 100)], [(512, 16)]),
    ("bf16", 16, 8, 128, 16, [(3000, 2500), (2800, 2800), (500, 1), (40, 0), (1700, 1600)], [(150, 20), (1000, 3)]),   # two teams of waves
    ("bf16", 10, 10, 128, 32, [(3000, 2500), (2900, 2900), (700, 700), (1700, 1600)], [(33, 0), (700, 40)]),
    ("f32", 4, 4, 64, 16, [(40, 40), (117, 3), (64, 1), (9, 0), (33, 33)], [(1, 0), (13, 3), (30, 20), (200, 5)]),
    ("f32", 8, 2, 32, 16, [(150, 150), (80, 7)], [(11, 2), (64, 16)]),
    ("f32", 8, 2, 128, 32, [(130, 130), (300, 9)], [(50, 4)]),
    ("f32", 3, 1, 64, 64, [(170, 100)], [(33, 4)]),                                # groups of 3
]
# Half a step of bf16 (2^-8 of the value): once for the output, and where the weights are rounded to it, once for each of them and their
# sum.  On top the sums in 32 bits.  A score is a sum of D products: at most 12 roundings deep, of |q||k| scale < 30 for normal vectors, so off
# by 12 2^-24 30 = 2e-5, which is the relative error of a weight; values of the pair (high part and remainder) are off by 2^-17 = 8e-6.
STEP = 2.0 ** -8
ACC = 6e-5


def bound(dtype, out, size, rounded):
    if dtype == "f32":
        return ACC * (size + np.abs(out)) + 1e-6
    return STEP * np.abs(out) + (STEP * (size + np.abs(out)) if rounded else 0.0) + ACC * (size + np.abs(out)) + 1e-6


def _setup(dtype, H, Hkv, D, bs, reqs, window, sinks, seed, layers=2, clean=True):
    """Pools in which what no new token sees is NaN, and table entries of blocks of nothing else name no block."""
    ctx = [c for c, _ in reqs]
    geom = W.Geometry(layers, H, Hkv, D, bs, sum((c + bs - 1) // bs for c in ctx) + 4, max((c + bs - 1) // bs for c in ctx) + 1, dtype)
    rig = Rig(geom, len(reqs))
    table, _ = W.deal_block_table(W.permutation(seed, geom.num_blocks), ctx, geom)
    K, V = zip(*[W.logical_kv(seed + 17 * r, geom, c) for r, c in enumerate(ctx)])
    KN, VN = [k.copy() for k in K], [v.copy() for v in V]
    holes = table.copy()
    for r, (c, n) in enumerate(reqs):
        any_sees = np.zeros(c, dtype=bool)
        for p in range(c - max(n, 1), c):
            any_sees |= seen(p, c, window, sinks)
        if clean:
            nan = np.uint16(0x7FC0) if dtype == "bf16" else np.float32("nan")
            KN[r][~any_sees], VN[r][~any_sees] = nan, nan
            for b in range((c + bs - 1) // bs):
                if not any_sees[b * bs:(b + 1) * bs].any():
                    holes[r, b] = -7
    rig.page_requests(layers - 1, table, KN, VN)
    return geom, rig, holes, K, V, ctx


@pytest.mark.parametrize("dtype,H,Hkv,D,bs,reqs,looks", CASES)
def test_decode(dtype, H, Hkv, D, bs, reqs, looks):
    for w, (window, sinks) in enumerate(looks):
        one = [(c, 1) for c, _ in reqs] + [(0, 0)]
        geom, rig, table, K, V, ctx = _setup(dtype, H, Hkv, D, bs, one, window, sinks, 31 + D + w)
        B = len(ctx)
        q = W.queries(5 + w, geom, B)
        running = np.ones(B, dtype=np.uint8)
        running[1:2] = 0
        dev = rig.dev
        out = torch.full((B, H, D), 2.5, dtype=rig.tdtype, device=dev)
        args = n2t(q, dev), torch.as_tensor(table, device=dev), torch.tensor(ctx, dtype=torch.int32, device=dev), torch.as_tensor(running, device=dev)
        torch.cuda.synchronize()
        rig.lamps.decode_attn_window(1, B, window, sinks, *args, out)
        again = torch.full_like(out, 2.5)
        torch.cuda.synchronize()
        rig.lamps.decode_attn_window(1, B, window, sinks, *args, again)
        torch.cuda.synchronize()
        assert torch.equal(out, again)
        got = to_f64(out)
        for r in range(B):
            if not running[r]:
                assert (got[r] == 2.5).all()
            elif ctx[r] == 0:
                assert (got[r] == 0).all()
            else:
                ref, size = window_attn(f64(q[r:r + 1]), f64(K[r]), f64(V[r]), ctx[r] - 1, window, sinks)
                off = np.abs(got[r] - ref[0]) - bound(dtype, ref[0], size[0], False)
                assert (off <= 0).all(), (window, sinks, r, ctx[r], off.max())
        rig.close()


def _prefill(rig, layer, q, reqs, table, window, sinks, out, most):
    dev = rig.dev
    start = np.concatenate([[0], np.cumsum([n for _, n in reqs])])
    args = torch.tensor(start, dtype=torch.int32, device=dev), torch.as_tensor(table, device=dev), \
        torch.tensor([c for c, _ in reqs], dtype=torch.int32, device=dev)
    qd = q if torch.is_tensor(q) else n2t(q, dev)
    torch.cuda.synchronize()
    rig.lamps.prefill_attn_window(layer, len(reqs), qd.shape[0], window, sinks, qd, *args, out, max_new_tokens=most)
    torch.cuda.synchronize()
    return start


@pytest.mark.parametrize("rows", [False, True])
@pytest.mark.parametrize("dtype,H,Hkv,D,bs,reqs,looks", CASES)
def test_prefill(dtype, H, Hkv, D, bs, reqs, looks, rows):
    """Rows behind the last request's are left as they were."""
    for w, (window, sinks) in enumerate(looks):
        geom, rig, table, K, V, ctx = _setup(dtype, H, Hkv, D, bs, reqs, window, sinks, 77 + D + w)
        total = sum(n for _, n in reqs)
        q = W.queries(9 + w, geom, total + 3)
        out = torch.full((total + 3, H, D), 2.5, dtype=rig.tdtype, device=rig.dev)
        again = out.clone()
        most = -1 if rows else (max(n for _, n in reqs) if w % 2 else 0)
        start = _prefill(rig, 1, q, reqs, table, window, sinks, out, most)
        _prefill(rig, 1, q, reqs, table, window, sinks, again, most)
        assert torch.equal(out, again)
        got = to_f64(out)
        assert (got[total:] == 2.5).all()
        for r, (c, n) in enumerate(reqs):
            # (of long prompts the first and the last of 100 rows and some between, and all of the last tile)
            pick = [i for i in range(n) if n <= 300 or i % 100 in (0, 41, 99) or n - i < 20]
            if n:
                kd, vd = f64(K[r]), f64(V[r])
                for i in pick:
                    at = start[r] + i
                    ref, size = window_attn(f64(q[at:at + 1]), kd, vd, c - n + i, window, sinks)
                    off = np.abs(got[at] - ref[0]) - bound(dtype, ref[0], size[0], not rows)
                    assert (off <= 0).all(), (window, sinks, r, c, n, i, off.max())
        rig.close()


@pytest.mark.parametrize("what", ["nan", "inf"])
@pytest.mark.parametrize("dtype,H,Hkv,D,bs", [("bf16", 8, 2, 128, 16), ("bf16", 4, 4, 128, 16), ("bf16", 8, 2, 64, 16), ("bf16", 4, 4, 64, 16),
                                              ("bf16", 8, 1, 256, 16), ("bf16", 2, 2, 256, 16), ("f32", 4, 2, 64, 16), ("f32", 4, 4, 128, 16),
                                              ("f32", 4, 1, 32, 16)])
def test_what_a_token_does_not_see_has_no_part_in_its_row(dtype, H, Hkv, D, bs, what):
    """Keys and values that are no finite numbers, at one position: the rows that see it are no finite numbers, all others as without."""
    reqs, window, sinks, at = [(150, 150), (90, 20)], 40, 3, (60, 75)
    geom, rig, table, K, V, ctx = _setup(dtype, H, Hkv, D, bs, reqs, window, sinks, 3, clean=False)
    total = sum(n for _, n in reqs)
    q = W.queries(4, geom, total)
    bad = {"nan": (0x7FC0, np.nan), "inf": (0x7F80, np.inf)}[what][0 if dtype == "bf16" else 1]
    for keys in (True, False):
        for rows in (0, -1):
            rig.page_requests(1, table, K, V)
            clean = torch.zeros((total, H, D), dtype=rig.tdtype, device=rig.dev)
            _prefill(rig, 1, q, reqs, table, window, sinks, clean, rows)
            Kb, Vb = [k.copy() for k in K], [v.copy() for v in V]
            for r, p in enumerate(at):
                (Kb if keys else Vb)[r][p] = bad
            rig.page_requests(1, table, Kb, Vb)
            out = torch.zeros_like(clean)
            start = _prefill(rig, 1, q, reqs, table, window, sinks, out, rows)
            for r, (c, n) in enumerate(reqs):
                sees = np.array([seen(p, c, window, sinks)[at[r]] for p in range(c - n, c)])
                a, b = clean[start[r]:start[r + 1]].cpu(), out[start[r]:start[r + 1]].cpu()
                assert torch.equal(a[~sees], b[~sees]), (keys, rows, r)
                if what == "nan" or not keys:             # (an infinite key may give weights of 0)
                    assert not torch.isfinite(b[sees]).any(), (keys, rows, r)
    rig.close()


def test_a_full_window_is_the_whole_attention():
    for dtype, H, Hkv, D in [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 64)]:
        reqs = [(300, 300), (77, 1)]
        geom, rig, table, K, V, ctx = _setup(dtype, H, Hkv, D, 16, reqs, 1 << 30, 0, 8)
        total = sum(n for _, n in reqs)
        q = n2t(W.queries(1, geom, total), rig.dev)
        outs = [torch.zeros((total, H, D), dtype=rig.tdtype, device=rig.dev) for _ in range(2)]
        start = _prefill(rig, 1, q, reqs, table, 2 ** 31 - 1, 2 ** 31 - 1, outs[0], 0)
        rig.lamps.prefill_attn(1, 2, total, q, torch.tensor(start, dtype=torch.int32, device=rig.dev), torch.as_tensor(table, device=rig.dev),
                               torch.tensor(ctx, dtype=torch.int32, device=rig.dev), outs[1])
        torch.cuda.synchronize()
        a, b = to_f64(outs[0]), to_f64(outs[1])
        for r, (c, n) in enumerate(reqs):
            at = slice(start[r], start[r + 1])
            ref, size = window_attn(f64(W.queries(1, geom, total)[at]), f64(K[r]), f64(V[r]), c - n, 1 << 30, 0)
            assert (np.abs(a[at] - b[at]) <= 2 * bound(dtype, ref, size, True)).all()
        rig.close()


@pytest.mark.parametrize("dtype,H,Hkv,D,bs,layers,batch", [("bf16", 8, 2, 128, 16, 1, 1), ("bf16", 4, 4, 128, 16, 3, 3), ("f32", 8, 2, 64, 32, 1, 2)])
def test_long_contexts_in_parts(dtype, H, Hkv, D, bs, layers, batch):
    """Few ranges of wide windows, which workgroups share."""
    window, sinks = 2000, 33
    reqs = [(5000 - 700 * r, 1) for r in range(batch)]
    geom, rig, table, K, V, ctx = _setup(dtype, H, Hkv, D, bs, reqs, window, sinks, 91, layers=layers)
    q = W.queries(2, geom, batch)
    out = torch.zeros((batch, H, D), dtype=rig.tdtype, device=rig.dev)
    rig.lamps.decode_attn_window(layers - 1, batch, window, sinks, n2t(q, rig.dev), torch.as_tensor(table, device=rig.dev),
                                 torch.tensor(ctx, dtype=torch.int32, device=rig.dev), torch.ones(batch, dtype=torch.uint8, device=rig.dev), out)
    torch.cuda.synchronize()
    for r in range(batch):
        ref, size = window_attn(f64(q[r:r + 1]), f64(K[r]), f64(V[r]), ctx[r] - 1, window, sinks)
        assert (np.abs(to_f64(out)[r] - ref[0]) <= bound(dtype, ref[0], size[0], False)).all()
    rig.close()


def test_lengths_beyond_the_row_are_clamped():
    for dtype, H, Hkv, D in [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 32)]:
        geom, rig, table, K, V, ctx = _setup(dtype, H, Hkv, D, 16, [(64, 1), (64, 1), (30, 1)], 20, 2, 4)
        full = np.ascontiguousarray(table[:, :4])                        # (a row of 64 positions, all of them there)
        rig.lamps.destroy()
        cfg = P.LampsConfig(2, H, Hkv, D, 16, geom.num_blocks, 4, 3, rig.cfg.dtype)
        rig.lamps = P.Lamps(cfg, rig.k_pool, rig.v_pool, rig.workspace)
        q = n2t(W.queries(1, geom, 3), rig.dev)
        outs = []
        for lens in ([64, 64, 30], [65, 2 ** 31 - 1, 30], [64, 64, -1]):
            out = torch.full((3, H, D), 2.5, dtype=rig.tdtype, device=rig.dev)
            rig.lamps.decode_attn_window(1, 3, 20, 2, q, torch.as_tensor(full, device=rig.dev), torch.tensor(lens, dtype=torch.int32, device=rig.dev),
                                         torch.ones(3, dtype=torch.uint8, device=rig.dev), out)
            torch.cuda.synchronize()
            outs.append(out)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0][:2], outs[2][:2]) and bool((outs[2][2] == 0).all())
        rig.close()


def test_bad_lengths_and_entries_are_harmless():
    """A context longer than its row is clamped (decode) or ignored (many tokens), one shorter than its new tokens ignored; a row whose
    entries name no block of the pool is written with something, the others are as without it."""
    for dtype, H, Hkv, D in [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 32)]:
        reqs = [(70, 70), (60, 30), (50, 50)]
        geom, rig, table, K, V, ctx = _setup(dtype, H, Hkv, D, 16, reqs, 40, 2, 8)
        total = sum(n for _, n in reqs)
        q = W.queries(1, geom, total)
        good = torch.full((total, H, D), 2.5, dtype=rig.tdtype, device=rig.dev)
        start = _prefill(rig, 1, q, reqs, table, 40, 2, good, 0)
        for lens in ([70, 100000, 50], [70, 29, 50]):
            out = torch.full_like(good, 2.5)
            rig.lamps.prefill_attn_window(1, 3, total, 40, 2, n2t(q, rig.dev), torch.tensor(start, dtype=torch.int32, device=rig.dev),
                                          torch.as_tensor(table, device=rig.dev), torch.tensor(lens, dtype=torch.int32, device=rig.dev), out)
            torch.cuda.synchronize()
            assert (out[start[1]:start[2]] == 2.5).all()
            assert torch.equal(out[:start[1]], good[:start[1]]) and torch.equal(out[start[2]:], good[start[2]:])
        wild = table.copy()
        wild[1] = geom.num_blocks + 5
        out = torch.full_like(good, 2.5)
        _prefill(rig, 1, q, reqs, wild, 40, 2, out, 0)
        assert torch.equal(out[:start[1]], good[:start[1]]) and torch.equal(out[start[2]:], good[start[2]:])
        rig.close()


#          many tiles of 32-bit values under short windows: a tile to a wave
WAVES = [
    ("f32", 8, 2, 32, 16, [(3000, 3000), (2500, 2403), (5, 0), (1900, 1797), (20, 0)], [(33, 3), (490, 20)]),
    ("f32", 32, 8, 128, 32, [(1000, 1000), (900, 801), (31, 31)], [(17, 2), (300, 5)]),
    ("f32", 8, 8, 64, 16, [(4000, 4000), (3500, 3141)], [(100, 0)]),
]


@pytest.mark.parametrize("dtype,H,Hkv,D,bs,reqs,looks", WAVES)
def test_prefill_of_many_tiles(dtype, H, Hkv, D, bs, reqs, looks):
    test_prefill(dtype, H, Hkv, D, bs, reqs, looks, False)


@pytest.mark.parametrize("dtype,H,Hkv,D,reqs,window,at", [
    ("bf16", 16, 8, 128, [(2500, 2500), (2300, 2003)], 1030, (1000, 700)),       # two teams of waves
    ("bf16", 8, 2, 128, [(900, 20), (700, 9)], 600, (895, 100)),                 # tiles in parts
    ("bf16", 4, 4, 64, [(900, 20), (700, 9)], 600, (300, 695)),
    ("f32", 32, 8, 128, [(1000, 1000), (900, 850)], 40, (500, 899)),             # a tile to a wave
    ("f32", 8, 2, 32, [(4000, 4000), (3500, 3300)], 100, (1, 3411)),
])
def test_values_and_keys_that_are_no_numbers_in_large_and_shared_launches(dtype, H, Hkv, D, reqs, window, at):
    """As test_what_a_token_does_not_see_has_no_part_in_its_row, one position of each request."""
    sinks = 3
    geom, rig, table, K, V, ctx = _setup(dtype, H, Hkv, D, 16, reqs, window, sinks, 6, clean=False)
    total = sum(n for _, n in reqs)
    q = W.queries(4, geom, total)
    clean = torch.zeros((total, H, D), dtype=rig.tdtype, device=rig.dev)
    _prefill(rig, 1, q, reqs, table, window, sinks, clean, 0)
    for keys in (True, False):
        Kb, Vb = [k.copy() for k in K], [v.copy() for v in V]
        for r, p in enumerate(at):
            (Kb if keys else Vb)[r][p] = 0x7FC0 if dtype == "bf16" else np.nan
        rig.page_requests(1, table, Kb, Vb)
        out = torch.zeros_like(clean)
        start = _prefill(rig, 1, q, reqs, table, window, sinks, out, 0)
        for r, (c, n) in enumerate(reqs):
            sees = np.array([seen(p, c, window, sinks)[at[r]] for p in range(c - n, c)])
            a, b = clean[start[r]:start[r + 1]].cpu(), out[start[r]:start[r + 1]].cpu()
            assert sees.any()
            assert torch.equal(a[~sees], b[~sees]), (keys, r)
            assert not torch.isfinite(b[sees]).any(), (keys, r)
    rig.close()


#          heads of 256 in groups: two teams of waves, and tiles of 128 columns in parts
TEAMS_256 = [
    ("bf16", 4, 2, 256, 16, [(300, 300), (1, 1), (0, 0), (130, 50), (700, 41)], [(1, 0), (40, 3), (128, 33)]),
    ("bf16", 16, 1, 256, 32, [(400, 90), (70, 70)], [(33, 0), (400, 7)]),
    ("bf16", 6, 2, 256, 16, [(140, 140), (77, 10)], [(50, 4)]),                    # groups of 3
    ("bf16", 16, 4, 256, 16, [(1500, 33), (900, 5)], [(64, 1), (1000, 4)]),
]


@pytest.mark.parametrize("dtype,H,Hkv,D,bs,reqs,looks", TEAMS_256)
def test_prefill_heads_of_256_in_groups(dtype, H, Hkv, D, bs, reqs, looks):
    test_prefill(dtype, H, Hkv, D, bs, reqs, looks, False)


@pytest.mark.parametrize("reqs,window,at", [([(300, 300), (200, 20)], 40, (100, 185)), ([(900, 20), (700, 9)], 600, (895, 100))])
def test_values_and_keys_that_are_no_numbers_heads_of_256(reqs, window, at):
    test_values_and_keys_that_are_no_numbers_in_large_and_shared_launches("bf16", 8, 4, 256, reqs, window, at)


#          few tiles with long walks, in two to four parts that the last workgroup of a tile adds up
SHARED = [
    ("bf16", 32, 8, 128, 16, [(1500, 40), (900, 37), (30, 30), (1200, 64), (800, 1), (1100, 40)], [(1000, 4), (2000, 0)]),
    ("bf16", 32, 8, 128, 32, [(1500, 150), (900, 141), (300, 300)], [(1000, 4)]),
    ("bf16", 8, 8, 128, 16, [(1300, 300), (900, 290), (1700, 310)], [(700, 33)]),
    ("bf16", 16, 8, 64, 16, [(1500, 150), (1100, 140), (900, 170)], [(800, 3)]),
    ("bf16", 16, 8, 256, 16, [(3500, 832)], [(3000, 5)]),
    ("bf16", 8, 8, 256, 16, [(1500, 460), (1200, 440)], [(600, 2)]),
]


@pytest.mark.parametrize("dtype,H,Hkv,D,bs,reqs,looks", SHARED)
def test_prefill_of_shared_tiles(dtype, H, Hkv, D, bs, reqs, looks):
    test_prefill(dtype, H, Hkv, D, bs, reqs, looks, False)


def test_values_and_keys_that_are_no_numbers_in_shared_tiles():
    test_values_and_keys_that_are_no_numbers_in_large_and_shared_launches(
        "bf16", 32, 8, 128, [(1500, 40), (900, 37), (30, 30), (1200, 64), (800, 9), (1100, 40)], 1000, (490, 890, 3, 180, 795, 1070))


def test_shared_tiles_replayed():
    """A captured call whose tiles are shared, replayed with other calls of the same workspace in between."""
    reqs, window, sinks = [(1500, 40), (900, 37), (30, 30), (1200, 64), (800, 1), (1100, 40)], 1000, 4
    geom, rig, table, K, V, ctx = _setup("bf16", 32, 8, 128, 16, reqs, window, sinks, 12)
    dev, total, lam = rig.dev, sum(n for _, n in reqs), rig.lamps
    start = torch.tensor(np.concatenate([[0], np.cumsum([n for _, n in reqs])]), dtype=torch.int32, device=dev)
    td, cd = torch.as_tensor(table, device=dev), torch.tensor(ctx, dtype=torch.int32, device=dev)
    queries = [n2t(W.queries(s, geom, total), dev) for s in range(3)]
    with torch.cuda.stream(rig.compute):
        want = [torch.zeros_like(q) for q in queries]
        for q, out in zip(queries, want):
            lam.prefill_attn_window(1, 6, total, window, sinks, q, start, td, cd, out, max_new_tokens=64)
        q, out, other, ones = queries[0].clone(), torch.zeros_like(queries[0]), torch.zeros_like(queries[0]), torch.ones(6, dtype=torch.uint8, device=dev)
        rig.compute.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=rig.compute):
            lam.prefill_attn_window(1, 6, total, window, sinks, q, start, td, cd, out, max_new_tokens=64)
            lam.prefill_attn_window(1, 6, total, window, sinks, out, start, td, cd, other, max_new_tokens=64)
        for it in range(6):
            q.copy_(queries[it % 3])
            out.zero_()
            graph.replay()
            again = torch.zeros_like(q)
            lam.prefill_attn_window(1, 6, total, window, sinks, out, start, td, cd, again, max_new_tokens=64)
            rig.compute.synchronize()
            assert torch.equal(out, want[it % 3]) and torch.equal(other, again), it
            lam.decode_attn_window(1, 6, 900, 0, q[:6], td, cd, ones, torch.zeros_like(q[:6]))
            if it % 2:
                lam.prefill_attn_window(1, 6, total, 300, 0, q, start, td, cd, torch.zeros_like(q), max_new_tokens=64)
    torch.cuda.synchronize()
    rig.close()
