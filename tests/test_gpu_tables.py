"""GPU parity of lamps_batch_tables: whole numbers, equal to the plain form's."""
import numpy as np
import pytest
import torch

import lamps_workloads as W
from operator_forms import tables
from rig import Rig

pytestmark = pytest.mark.gpu


def _run(bs, row, cached, new, ids, grow, total, table, num_blocks, slots=True, report=True, odd=0):
    n = len(cached)
    geom = W.Geometry(1, 2, 2, 64, bs, num_blocks, row, "f32")
    rig = Rig(geom, max(n, 1), poison=False)
    ints = lambda x: torch.tensor(np.asarray(x, dtype=np.int32), dtype=torch.int32, device=rig.dev)
    room = torch.full((n * row + odd + 4,), -9, dtype=torch.int32, device=rig.dev)
    td = room[odd:odd + n * row].view(n, row)             # (rows that are not 16-byte aligned)
    td.copy_(ints(table).view(n, row))
    cd, qd = torch.full((n + 2,), -9, dtype=torch.int32, device=rig.dev), torch.full((n + 3,), -9, dtype=torch.int32, device=rig.dev)
    sd = torch.full((total + 2,), -9, dtype=torch.int64, device=rig.dev)
    rd = torch.full((6,), -9, dtype=torch.int32, device=rig.dev)
    torch.cuda.synchronize()
    c, w, i = ints(cached), ints(new), ints(ids)
    # (an empty tensor has no address: any other stands for it, of which nothing is read)
    c, w = (c, w) if n else (ints([7]), ints([7]))
    for _ in range(2):                                    # (a second time: the same)
        rig.lamps.batch_tables(n, total, c, w, i if len(ids) else None, len(ids), grow, td if n else room, cd, qd, sd if slots else None,
                               rd if report else None)
    torch.cuda.synchronize()
    assert (room[:odd] == -9).all() and (room[odd + n * row:] == -9).all() and (cd[n:] == -9).all() and (qd[n + 1:] == -9).all()
    assert (sd[total if slots else 0:] == -9).all() and (rd[4 if report else 0:] == -9).all()
    got = td.cpu().numpy(), cd[:n].cpu().tolist(), qd[:n + 1].cpu().tolist(), sd[:total].cpu().tolist(), rd[:4].cpu().tolist()
    rig.close()
    return got


def _check(bs, row, cached, new, ids, grow, total, table, num_blocks, **kw):
    t, c, q, s, rep = _run(bs, row, cached, new, ids, grow, total, table, num_blocks, **kw)
    wt, wc, wq, ws, wr = tables(cached, new, ids, grow, np.asarray(table), bs, total)
    assert (t == wt).all() and c == wc and q == wq
    if kw.get("slots", True):
        want = [b * bs + o if 0 <= b < num_blocks else -1 for b, o in ws]
        assert s == want + [-1] * (total - len(want))
    if kw.get("report", True):
        assert rep == wr


@pytest.mark.parametrize("grow", [False, True])
@pytest.mark.parametrize("n,bs,row,most", [(1, 16, 1, 16), (1, 16, 2000, 3000), (5, 16, 7, 100), (64, 32, 33, 40), (256, 16, 128, 30),
                                           (257, 16, 61, 300), (1000, 64, 20, 9), (1025, 16, 9, 20), (8192, 16, 5, 3)])
def test_batches(n, bs, row, most, grow):
    rng = np.random.default_rng(n + row)
    new = rng.integers(0, most + 1, n)
    cached = rng.integers(0, row * bs + 1, n)
    new = np.minimum(new, row * bs - cached)
    held = -(-cached // bs) if grow else 0 * cached
    need = -(-(cached + new) // bs) - held
    num_blocks = int(held.sum() + need.sum()) + 5
    perm = rng.permutation(num_blocks).astype(np.int32)
    table = rng.integers(-5, num_blocks, (n, row)).astype(np.int32)
    ids = perm[:need.sum()]
    _check(bs, row, cached.tolist(), new.tolist(), ids, grow, int(new.sum()), table, num_blocks)
    _check(bs, row, cached.tolist(), new.tolist(), perm[:need.sum() + 5], grow, int(new.sum()) + 9, table, num_blocks, odd=1, report=False)


@pytest.mark.parametrize("grow", [False, True])
def test_requests_that_cannot_be_served(grow):
    rng = np.random.default_rng(3)
    bs, row, blocks = 16, 6, 500
    table = rng.integers(0, blocks, (9, row)).astype(np.int32)
    cached = [10, -1, 30, 90, 2 ** 31 - 1, 16, 0, 5, 96]
    new = [7, 5, 20, 7, 2 ** 31 - 1, 16, 0, -3, 0]
    for n_ids in (0, 1, 2, 4, 5, 20):
        for total in (0, 7, 26, 27, 60):
            _check(bs, row, cached, new, np.arange(100, 100 + n_ids, dtype=np.int32), grow, total, table, blocks)
    # entries kept that name no block have no slot
    table[:] = blocks
    _check(bs, row, [5] * 9, [3] * 9, np.arange(9, dtype=np.int32), grow, 27, table, blocks)


def test_sums_beyond_32_bits():
    """40 requests that want 2^26 blocks and 2^30 tokens each: no sum wraps around and serves one."""
    bs, row = 16, 1 << 26
    geom = W.Geometry(1, 1, 1, 32, bs, 4, row, "f32")
    rig = Rig(geom, 70, poison=False)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=rig.dev)
    td = torch.full((42, row), 3, dtype=torch.int32, device=rig.dev)
    cached, new = ints([0] * 42), ints([5] + [1 << 30] * 40 + [0])
    ctx, start, rep = ints([-9] * 42), ints([-9] * 43), ints([-9] * 4)
    torch.cuda.synchronize()
    rig.lamps.batch_tables(42, 100, cached, new, ints([2, 1, 0]), 3, False, td, ctx, start, None, rep)
    torch.cuda.synchronize()
    assert ctx.tolist() == [5] + [0] * 41 and start.tolist() == [0] + [5] * 42 and rep.tolist() == [1, 40, 1, 5]
    assert td[0, 0] == 2 and bool((td[0, 1:] == -1).all()) and bool((td[1:41] == 3).all()) and bool((td[41] == -1).all())
    rig.close()


def test_empty_batch():
    t, c, q, s, rep = _run(16, 3, [], [], [], False, 4, np.zeros((0, 3)), 5)
    assert c == [] and q == [0] and s == [-1] * 4 and rep == [0, 0, -1, 0]
