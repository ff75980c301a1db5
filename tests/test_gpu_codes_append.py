"""GPU parity of appends into a cache of 8 bits and of reading back: byte by byte against plain numpy."""
import numpy as np
import pytest
import torch

import codes_forms as F
import lamps_workloads as W
import paper_2410_18248_amd as P
from rig import Rig, n2t, t2n

pytestmark = pytest.mark.gpu

#        H  Hkv D    bs   new tokens per request, call by call
FORMS = [
    (8, 2, 128, 16, [[5, 1, 40, 0, 16], [11, 3, 1, 2, 17], [1, 1, 23, 31, 1]]),
    (4, 4, 64, 16, [[1, 15, 64], [16, 1, 3]]),
    (4, 4, 64, 32, [[33, 2], [30, 70]]),
    (6, 2, 256, 16, [[19, 4], [1, 12]]),
    (8, 4, 128, 64, [[70, 3, 64], [1, 130, 5]]),
    (8, 2, 256, 64, [[61, 90], [70, 1]]),
    (2, 1, 128, 256, [[300, 5], [30, 300]]),
    (40, 40, 128, 32, [[40, 7], [5, 5]]),
    (3, 3, 64, 16, [[9, 20], [8, 1]]),
]
# sizes of a call's numbers: as drawn; growing from call to call, so that scales move; shrinking; far apart within a vector
SIZES = {"alike": lambda c: 1.0, "growing": lambda c: 7.0 ** c, "much larger": lambda c: 1e4 ** c, "shrinking": lambda c: 20.0 ** -c}


def _numbers(seed, total, Hkv, D, size, wide):
    x = F.normal(seed, total, Hkv, D, size=size)
    if wide:
        x = (x.float() * 2.0 ** torch.randint(-12, 6, x.shape, generator=torch.Generator().manual_seed(seed + 1)).float()).bfloat16()
    return x


@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("H,Hkv,D,bs,calls", FORMS)
def test_many_tokens(H, Hkv, D, bs, calls, sizes):
    """Call after call onto what is there; what no call reaches stays as it was; read back, the numbers are the codes' own."""
    n = len(calls[0])
    ctx, after = np.zeros(n, dtype=int), np.sum(calls, 0)
    row = (after.max() + bs - 1) // bs + 1
    rig = F.CodesRig(2, H, Hkv, D, bs, int(sum((t + bs - 1) // bs for t in after)) + 2, int(row), n)
    table, expected = rig.deal(after), rig.host()
    for c, counts in enumerate(calls):
        total = sum(counts)
        k, v = (_numbers(100 * c + i, total, Hkv, D, SIZES[sizes](c), sizes == "alike") for i in (0, 1))
        ctx = ctx + counts
        rig.append_tokens(1, k, v, counts, table, ctx)
        at = 0
        for r, m in enumerate(counts):
            if m:
                expected.append(1, table[r], ctx[r] - m, F.f64(k[at:at + m]), F.f64(v[at:at + m]))
            at += m
        F.same(rig.host(), expected)
    # all of it, and the last few of each
    for counts in (after, np.minimum(after, 5)):
        total = int(sum(counts))
        out = [torch.full((total + 2, Hkv, D), 2.5, dtype=torch.bfloat16, device=rig.dev) for _ in range(2)]
        rig.lamps.kv_read_tokens(1, n, total, rig.ints(np.concatenate([[0], np.cumsum(counts)])), rig.ints(table), rig.ints(after), *out)
        torch.cuda.synchronize()
        for x, which in zip(out, (0, 1)):
            want = np.concatenate([expected.logical(1, table[r], after[r])[which][after[r] - counts[r]:] for r in range(n)])
            np.testing.assert_array_equal(F.f64(x[:total]), want)
            assert (x[total:] == 2.5).all()
    rig.close()


@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("H,Hkv,D,bs,calls", FORMS)
def test_one_token(H, Hkv, D, bs, calls, sizes):
    """Token by token from what a first call left; some requests wait; lengths go up where the call says so."""
    first = [max(1, x) for x in calls[0]] + [0, bs - 1]
    n, steps = len(first), 2 * bs + 3 if bs <= 16 else 6
    rig = F.CodesRig(2, H, Hkv, D, bs, int(sum((t + steps + bs - 1) // bs for t in first)) + 2, (max(first) + steps) // bs + 2, n)
    ctx = np.array(first)
    table, expected = rig.deal(ctx + steps), rig.host()
    k, v = F.normal(1, int(ctx.sum()), Hkv, D), F.normal(2, int(ctx.sum()), Hkv, D)
    rig.append_tokens(0, k, v, first, table, ctx)
    at = 0
    for r, m in enumerate(first):
        if m:
            expected.append(0, table[r], 0, F.f64(k[at:at + m]), F.f64(v[at:at + m]))
        at += m
    td, cd = rig.ints(table), rig.ints(ctx)
    for step in range(steps):
        advance = step % 3 > 0
        running = np.ones(n, dtype=np.uint8)
        running[step % n] = 0
        k, v = (_numbers(50 * step + i, n, Hkv, D, SIZES[sizes](step / 8), step % 2 == 0) for i in (3, 4))
        args = k.to(rig.dev), v.to(rig.dev), td, cd, torch.tensor(running, device=rig.dev)
        torch.cuda.synchronize()
        rig.lamps.kv_append(0, n, *args, advance)
        torch.cuda.synchronize()
        for r in range(n):
            if running[r]:
                expected.append(0, table[r], int(ctx[r]), F.f64(k[r:r + 1]), F.f64(v[r:r + 1]))
                ctx[r] += advance
        assert (cd.cpu().numpy() == ctx).all()
        F.same(rig.host(), expected)
    rig.close()


def test_every_number_rounds_as_torch_rounds_it():
    """All bf16 numbers, 65 536 of them, each beside the largest that its scale holds, and NaN and infinities among others."""
    D, Hkv = 64, 1
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = bits.view(1024, 1, 64)
    rig = F.CodesRig(1, 1, Hkv, D, 16, 65, 64, 1)
    table, expected = rig.deal([1024]), rig.host()
    rig.append_tokens(0, x, x.flip(0), [1024], table, [1024])
    expected.append(0, table[0], 0, F.f64(x), F.f64(x.flip(0)))
    F.same(rig.host(), expected)
    rig.close()
    # 448 in front of each block: a scale of 1 wherever the rest is not larger
    small = bits[(bits.float().abs() <= 448) | bits.isnan()]
    small = small[:len(small) // 960 * 960].view(-1, 15, 64)
    y = torch.cat([torch.full((len(small), 1, 64), 448.0).bfloat16(), small], 1).view(-1, 1, 64)
    n = y.shape[0]
    rig = F.CodesRig(1, 1, Hkv, D, 16, n // 16, n // 16, 1)
    table = rig.deal([n])
    rig.append_tokens(0, y, -y, [n], table, [n])
    got = rig.host()
    for b in range(n // 16):
        assert (got.scales(int(table[0, b]), 0) == 1.0).all()
    flat = np.concatenate([got.codes(0, int(table[0, b]), 0)[0][got.at[0]] for b in range(n // 16)])
    np.testing.assert_array_equal(F.no_sign(flat), F.no_sign(y.view(n, 64).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()))
    rig.close()


def test_numbers_that_are_not_finite_stay_with_themselves():
    """A token with NaN and infinities has NaN in their places; the scale goes by the rest, and a token of nothing else has the least one."""
    rig = F.CodesRig(1, 4, 2, 128, 16, 4, 4, 2)
    table, expected = rig.deal([20, 3]), rig.host()
    k, v = F.normal(5, 23, 2, 128), F.normal(6, 23, 2, 128)
    k[3, 0, 5], k[3, 1, 7:20], v[4, 0, 0], v[17] = float("nan"), float("inf"), -float("inf"), float("nan")
    k[20:], v[20:] = float("inf"), 0.0
    rig.append_tokens(0, k, v, [20, 3], table, [20, 3])
    expected.append(0, table[0], 0, F.f64(k[:20]), F.f64(v[:20]))
    expected.append(0, table[1], 0, F.f64(k[20:]), F.f64(v[20:]))
    got = rig.host()
    F.same(got, expected)
    assert (got.scales(int(table[1, 0]), 0) == 2.0 ** -110).all() and (got.scales(int(table[0, 0]), 0) < 0.1).all()
    one = torch.full((2, 2, 128), float("nan"), dtype=torch.bfloat16)
    one[1] = 3.0
    rig.lamps.kv_append(0, 2, one.to(rig.dev), one.to(rig.dev), rig.ints(table), rig.ints([20, 3]), torch.ones(2, dtype=torch.uint8, device=rig.dev), False)
    expected.append(0, table[0], 20, F.f64(one[:1]), F.f64(one[:1]))
    expected.append(0, table[1], 3, F.f64(one[1:]), F.f64(one[1:]))
    F.same(rig.host(), expected)
    rig.close()


def test_what_names_no_place_writes_nothing():
    """Blocks outside the pool, positions behind the table row, contexts shorter than their new tokens or longer than the row, rows behind the last."""
    rig = F.CodesRig(1, 4, 2, 64, 16, 6, 3, 6)
    table, before = rig.deal([32, 16, 0, 16, 32, 0]), rig.host()
    table[0, 1], table[2] = 6, -9
    counts, ctx = [20, 4, 3, 9, 2, 5], [30, 3, 10, 60, 17, -4]
    k, v = F.normal(1, 48, 2, 64), F.normal(2, 48, 2, 64)
    rig.append_tokens(0, k, v, counts, table, ctx)
    expected = before
    at = np.concatenate([[0], np.cumsum(counts)])
    # the first six of request 0's (positions 10 to 15 of a block that nothing was put into: only their own codes and the scales are said), and request 4's
    got = rig.host()
    touched = {int(table[0, 0]), int(table[4, 0]), int(table[4, 1])}
    for b in range(6):
        if b not in touched:
            assert (got.k[b] == expected.k[b]).all() and (got.v[b] == expected.v[b]).all()
    out = [torch.full((43, 2, 64), 2.5, dtype=torch.bfloat16, device=rig.dev) for _ in range(2)]
    rig.lamps.kv_read_tokens(0, 6, 43, rig.ints(at), rig.ints(table), rig.ints(ctx), *out)
    torch.cuda.synchronize()
    for x in out:
        for r in (1, 2, 3, 5):
            assert (x[at[r]:at[r + 1]] == 2.5).all()
        assert (x[6:20] == 2.5).all() and not (x[at[4]:at[5]] == 2.5).all()
    td, cd = rig.ints(table), rig.ints([48, -1, 5, 47, 1 << 30, 31])
    snap, ones = rig.host(), torch.ones(6, dtype=torch.uint8, device=rig.dev)
    ones[4:] = 0
    rig.lamps.kv_append(0, 6, k.to(rig.dev), v.to(rig.dev), td, cd, ones, True)
    after = rig.host()
    assert (after.k == snap.k).all() and (after.v == snap.v).all()
    assert cd.tolist() == [48, -1, 5, 47, 1 << 30, 31]
    # rows that q_start claims behind total_tokens are neither read nor written
    q_start = rig.ints([0, 10])
    small = [torch.full((4, 2, 64), 2.5, dtype=torch.bfloat16, device=rig.dev) for _ in range(2)]
    rig.lamps.kv_read_tokens(0, 1, 2, q_start, rig.ints(table[4:5]), rig.ints([17]), *small)
    torch.cuda.synchronize()
    assert all((x[2:] == 2.5).all() for x in small)
    rig.close()


@pytest.mark.parametrize("dtype,H,Hkv,D,bs", [("bf16", 8, 2, 128, 16), ("bf16", 4, 4, 64, 32), ("bf16", 16, 4, 256, 64), ("f32", 4, 2, 32, 16), ("f32", 3, 3, 128, 32)])
def test_read_out_of_wide_pools(dtype, H, Hkv, D, bs):
    """Rows read back are the rows that were appended."""
    counts, ctx = [45, 1, 17, 0, 16], [45, 30, 33, 5, 16]
    geom = W.Geometry(2, H, Hkv, D, bs, 16, 4, dtype)
    rig = Rig(geom, 5)
    table, _ = W.deal_block_table(W.permutation(3, 16), ctx, geom)
    total = sum(counts)
    k, v = (torch.randn(total, Hkv, D, generator=torch.Generator().manual_seed(i)).to(rig.tdtype).to(rig.dev) for i in (1, 2))
    start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=rig.dev)
    args = start, torch.tensor(table, device=rig.dev), torch.tensor(ctx, dtype=torch.int32, device=rig.dev)
    torch.cuda.synchronize()
    rig.lamps.kv_append_tokens(1, 5, total, k, v, *args)
    out = [torch.full((total + 1, Hkv, D), 2.5, dtype=rig.tdtype, device=rig.dev) for _ in range(2)]
    torch.cuda.synchronize()
    rig.lamps.kv_read_tokens(1, 5, total, *args, *out)
    torch.cuda.synchronize()
    for x, y in zip(out, (k, v)):
        assert torch.equal(x[:total], y) and (x[total:] == 2.5).all()
    rig.close()


@pytest.mark.parametrize("layered,kw", [(False, {}), (True, {}), (False, dict(zero_copy_workgroups=8)), (False, dict(direct_copy_bytes=1))])
def test_swapped_blocks_take_their_scales_along(layered, kw):
    rig = F.CodesRig(3, 8, 2, 128, 16, 12, 4, 2, staging_bytes=0, **kw)
    blocks = rig.lamps.alloc_blocks(4)
    table = np.array([blocks, [-1] * 4], dtype=np.int32)
    for layer in range(3):
        rig.append_tokens(layer, F.normal(layer, 50, 2, 128, size=10.0 ** layer), F.normal(9 + layer, 50, 2, 128), [50, 0], table, [50, 0])
    before = rig.host()
    buf = torch.empty(4 * P.lamps_block_bytes(rig.cfg), dtype=torch.uint8).pin_memory()
    rig.lamps.ticket_wait(rig.lamps.swap_out(blocks, buf, layered=layered))
    rig.lamps.free_blocks(blocks)
    rig.lamps.alloc_blocks(3)                           # (others in between)
    again = rig.lamps.alloc_blocks(4)
    assert again != blocks
    rig.lamps.ticket_wait(rig.lamps.swap_in(buf, again, layered=layered))
    after = rig.host()
    row = np.array(again)
    for layer in range(3):
        for x, y in zip(before.logical(layer, table[0], 50), after.logical(layer, row, 50)):
            np.testing.assert_array_equal(x, y)
    rig.close()
