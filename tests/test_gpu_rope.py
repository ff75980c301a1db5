"""GPU parity of lamps_rope_append and lamps_rope_append_tokens: queries and keys normalised and turned, keys and values in the cache,
everything else in the pools as it was, against plain numpy in 64 bits."""
import numpy as np
import pytest
import torch

import lamps_workloads as W
import paper_2410_18248_amd as P
from operator_forms import f64, turned
from rig import Rig, n2t, t2n, to_f64

pytestmark = pytest.mark.gpu

# Results are rounded once: half a step of the type, relative to the value.  In front of it: the mean of D squares and its root (at most 10
# roundings deep), the weight, two products and a sum of a pair, whose error goes by the pair's length, not by the result: 16 roundings of 2^-24.
# (cos, sin) are good to 2^-23.
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
ACC = 18 * 2.0 ** -24


def bound(dtype, ref, length):
    return HALF[dtype] * np.abs(ref) + ACC * length + 1e-12


class Rope:
    def __init__(self, geom, dev, rotary, pairs, norm, scaling, weights=True, seed=1):
        rng = np.random.default_rng(seed)
        self.freq = P.lamps_rope_frequencies(rotary, 10000.0, scaling, 4.0, 2048.0, 1.0, 32.0)
        self.near, self.norm, self.eps = pairs == P.LAMPS_ROPE_NEIGHBOURS, norm, 1e-5
        self.amplitude = 1.25 if scaling == P.LAMPS_ROPE_BY_PARTS else 1.0
        self.w = [None, None]
        if norm and weights:
            w = (1 + 0.3 * rng.standard_normal((2, geom.head_dim))).astype(np.float32)
            self.w = [W.f32_to_bf16_bits(x) if geom.dtype == "bf16" else x for x in w]
        on = [None if x is None else n2t(x, dev) for x in self.w]
        self.args = P.LampsRope(rotary, pairs, torch.tensor(self.freq, dtype=torch.float64, device=dev) if rotary else None,
                                amplitude=0.0 if self.amplitude == 1.0 else self.amplitude, normalise=norm, norm_eps=self.eps,
                                q_weight=on[0], k_weight=on[1])

    def __call__(self, x, p, which):
        """Exact heads, and the largest a pair can be: its length behind the norm (a plain dim: its own)."""
        w = None if self.w[which] is None else f64(self.w[which])
        eps = self.eps if self.norm else None
        y = turned(f64(x), p, self.freq, self.near, self.amplitude, eps, w)
        plain = turned(f64(x), p, [], False, 1.0, eps, w)
        other = turned(plain, p * 0, np.zeros(len(self.freq)), self.near)    # (turned by nothing)
        n = 2 * len(self.freq)
        if n:
            a = plain[..., :n].reshape(*plain.shape[:-1], n // 2, 2) if self.near else plain[..., :n].reshape(*plain.shape[:-1], 2, n // 2)
            length = self.amplitude * np.sqrt((a * a).sum(-1 if self.near else -2))
            other = np.abs(other)
            other[..., :n] = np.repeat(length, 2, -1) if self.near else np.concatenate([length, length], -1)
        return y, np.abs(other)


#        dtype  H  Hkv D    bs  rotary pairs norm scaling
FORMS = [
    ("bf16", 8, 2, 128, 16, 128, 0, True, 0), ("bf16", 8, 2, 128, 32, 64, 1, True, 3), ("bf16", 4, 4, 128, 16, 128, 1, False, 1),
    ("bf16", 4, 4, 128, 16, 48, 0, True, 2), ("bf16", 6, 2, 64, 16, 64, 0, True, 3), ("bf16", 8, 8, 64, 64, 16, 1, False, 0),
    ("bf16", 16, 1, 256, 16, 256, 0, True, 0), ("bf16", 2, 2, 256, 16, 80, 1, True, 1), ("bf16", 3, 3, 64, 16, 0, 0, True, 0),
    ("bf16", 8, 2, 128, 16, 0, 0, False, 0), ("f32", 4, 4, 64, 16, 64, 0, True, 0), ("f32", 8, 2, 32, 16, 32, 1, True, 3),
    ("bf16", 40, 40, 128, 16, 128, 0, True, 0),                          # more than a workgroup's threads have in one turn
    ("f32", 3, 1, 128, 32, 128, 0, False, 1), ("f32", 2, 2, 128, 16, 112, 1, True, 2), ("f32", 5, 5, 32, 16, 16, 0, True, 0),
]


def _rig(dtype, H, Hkv, D, bs, ctx, row, seed, layers=2):
    """Pools of numbers, a table that names blocks only where the new positions are."""
    used = [sorted(x) for x in ctx]
    geom = W.Geometry(layers, H, Hkv, D, bs, sum(len(x) for x in used) + 3, row, dtype)
    rig = Rig(geom, max(1, len(ctx)), poison=False)
    g = torch.Generator(device=rig.dev).manual_seed(seed)
    rig.k_pool.normal_(generator=g)
    rig.v_pool.normal_(generator=g)
    table = np.full((len(ctx), row), -1, dtype=np.int32)
    perm, at = W.permutation(seed, geom.num_blocks), 0
    for r, blocks in enumerate(used):
        for b in blocks:
            table[r, b] = perm[at]
            at += 1
    return geom, rig, table


def _vectors(geom, dev, n, packed, seed):
    """q, k, v rows as device tensors and as numpy, and their stride."""
    H, Hkv, D = geom.num_q_heads, geom.num_kv_heads, geom.head_dim
    q, (k, v) = W.queries(seed, geom, n), W.logical_kv(seed + 1, geom, n)
    if not packed:
        return (q, k, v), (n2t(q, dev), n2t(k, dev), n2t(v, dev)), (0, 0, 0)
    x = n2t(np.concatenate([q, k, v], axis=1), dev)
    return (q, k, v), (x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]), ((H + 2 * Hkv) * D,) * 3


def _check(rig, geom, layer, dtype, rope, before, where, k, v, q, q_out, p):
    """where: (block, slot) of each row of q, k, v and q_out that was written; p their positions."""
    kp, vp = t2n(rig.k_pool), t2n(rig.v_pool)
    want, size = rope(q, p, 0)
    assert (np.abs(q_out - want) <= bound(dtype, want, size)).all()
    want, size = rope(k, p, 1)
    for i, (block, slot) in enumerate(where):
        got = f64(kp[block, layer][:, rig.k_index[slot]])
        assert (np.abs(got - want[i]) <= bound(dtype, want[i], size[i])).all(), i
        assert (vp[block, layer][:, rig.v_index[slot]] == v[i]).all(), i
        kp[block, layer][:, rig.k_index[slot]] = before[0][block, layer][:, rig.k_index[slot]]
        vp[block, layer][:, rig.v_index[slot]] = before[1][block, layer][:, rig.v_index[slot]]
    assert (kp == before[0]).all() and (vp == before[1]).all()        # nothing else was touched


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,H,Hkv,D,bs,rotary,pairs,norm,scaling", FORMS)
def test_one_token(dtype, H, Hkv, D, bs, rotary, pairs, norm, scaling, packed):
    ctx = [0, 1, 15, 16, 77, 20001, 131071, 64, 5]
    running = np.array([1, 1, 1, 1, 1, 1, 1, 0, 1], dtype=np.uint8)
    row = 131072 // bs
    geom, rig, table = _rig(dtype, H, Hkv, D, bs, [{c // bs} for c in ctx], row, 7 + D)
    table[8, ctx[8] // bs] = geom.num_blocks                              # no block of the pool: nothing of the request is written
    dev, B = rig.dev, len(ctx)
    rope = Rope(geom, dev, rotary, pairs, norm, scaling, weights=D != 256)
    before = [t2n(rig.k_pool).copy(), t2n(rig.v_pool).copy()]
    (q, k, v), (qd, kd, vd), strides = _vectors(geom, dev, B, packed, 3)
    td, cd, md = torch.as_tensor(table, device=dev), torch.tensor(ctx, dtype=torch.int32, device=dev), torch.as_tensor(running, device=dev)
    for advance in (False, True):
        out = torch.full((B, H, D), 2.5, dtype=rig.tdtype, device=dev)
        torch.cuda.synchronize()
        rig.lamps.rope_append(1, B, rope.args, qd, kd, vd, td, cd, md, advance, out, *strides)
        torch.cuda.synchronize()
        on = [r for r in range(B) if r < 7]
        got = to_f64(out)
        assert (got[7:] == 2.5).all()
        _check(rig, geom, 1, dtype, rope, before, [(table[r, ctx[r] // bs], ctx[r] % bs) for r in on], k[on], v[on], q[on], got[on],
               np.array([ctx[r] for r in on]))
        assert cd.cpu().tolist() == [c + (1 if advance and r in on else 0) for r, c in enumerate(ctx)]
    # positions outside the row write nothing
    before = [t2n(rig.k_pool).copy(), t2n(rig.v_pool).copy()]
    cd = torch.tensor([-1, row * bs, 2 ** 31 - 1] + [-5] * (B - 3), dtype=torch.int32, device=dev)
    out.fill_(2.5)
    torch.cuda.synchronize()
    rig.lamps.rope_append(1, B, rope.args, qd, kd, vd, td, cd, md, True, out, *strides)
    torch.cuda.synchronize()
    assert (out == 2.5).all() and (t2n(rig.k_pool) == before[0]).all() and (t2n(rig.v_pool) == before[1]).all()
    assert cd.cpu().tolist()[:3] == [-1, row * bs, 2 ** 31 - 1]
    rig.close()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,H,Hkv,D,bs,rotary,pairs,norm,scaling", FORMS)
def test_many_tokens(dtype, H, Hkv, D, bs, rotary, pairs, norm, scaling, packed):
    reqs = [(40, 40), (17, 3), (100, 0), (1, 1), (30020, 19), (64, 32), (33, 33)]       # (context with them, new tokens)
    row = 30032 // bs + 1
    geom, rig, table = _rig(dtype, H, Hkv, D, bs, [{p // bs for p in range(c - n, c)} for c, n in reqs], row, 9 + D)
    dev, total = rig.dev, sum(n for _, n in reqs)
    rope = Rope(geom, dev, rotary, pairs, norm, scaling, weights=H != 4)
    before = [t2n(rig.k_pool).copy(), t2n(rig.v_pool).copy()]
    (q, k, v), (qd, kd, vd), strides = _vectors(geom, dev, total + 2, packed, 5)
    start = np.concatenate([[0], np.cumsum([n for _, n in reqs])])
    p = np.concatenate([np.arange(c - n, c) for c, n in reqs]).astype(np.int64)
    r_of = np.concatenate([[r] * n for r, (_, n) in enumerate(reqs)]).astype(int)
    sd, td = torch.tensor(start, dtype=torch.int32, device=dev), torch.as_tensor(table, device=dev)
    out = torch.full((total + 2, H, D), 2.5, dtype=rig.tdtype, device=dev)
    cd = torch.tensor([c for c, _ in reqs], dtype=torch.int32, device=dev)
    torch.cuda.synchronize()
    rig.lamps.rope_append_tokens(1, len(reqs), total + 2, rope.args, qd, kd, vd, sd, td, cd, out, *strides)
    torch.cuda.synchronize()
    got = to_f64(out)
    assert (got[total:] == 2.5).all()
    _check(rig, geom, 1, dtype, rope, before, [(table[r, x // bs], x % bs) for r, x in zip(r_of, p)], k[:total], v[:total], q[:total], got[:total], p)
    # lengths that cannot be, and entries that name no block, write nothing of theirs
    rig.upload_pools(*before)
    lens, wild = [c for c, _ in reqs], table.copy()
    lens[0], lens[5] = row * bs + 1, 31
    wild[6, 0] = -3
    out.fill_(2.5)
    torch.cuda.synchronize()
    rig.lamps.rope_append_tokens(1, len(reqs), total + 2, rope.args, qd, kd, vd, sd, torch.as_tensor(wild, device=dev),
                                 torch.tensor(lens, dtype=torch.int32, device=dev), out, *strides)
    torch.cuda.synchronize()
    fine = np.array([r not in (0, 5) and not (r == 6 and x < bs) for r, x in zip(r_of, p)])
    got2 = to_f64(out)
    assert (got2[:total][fine] == got[:total][fine]).all() and (got2[:total][~fine] == 2.5).all()
    at = [(table[r, x // bs], x % bs) for r, x in zip(r_of[fine], p[fine])]
    _check(rig, geom, 1, dtype, rope, before, at, k[:total][fine], v[:total][fine], q[:total][fine], got2[:total][fine], p[fine])
    rig.close()


@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("dtype,H,Hkv,D", [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 64)])
def test_queries_in_place(dtype, H, Hkv, D, tokens):
    """q_out may be q."""
    geom, rig, table = _rig(dtype, H, Hkv, D, 16, [{0, 1, 2}], 4, 11)
    dev, n = rig.dev, 40 if tokens else 1
    rope = Rope(geom, dev, D, 0, True, 0)
    _, (qd, kd, vd), _ = _vectors(geom, dev, n, False, 5)
    td, sd = torch.as_tensor(table, device=dev), torch.tensor([0, n], dtype=torch.int32, device=dev)
    cd, md = torch.tensor([n if tokens else 17], dtype=torch.int32, device=dev), torch.ones(1, dtype=torch.uint8, device=dev)
    outs = [torch.zeros_like(qd), qd.clone()]
    torch.cuda.synchronize()
    for out in outs:
        src = qd if out is outs[0] else out
        if tokens:
            rig.lamps.rope_append_tokens(0, 1, n, rope.args, src, kd, vd, sd, td, cd, out)
        else:
            rig.lamps.rope_append(0, 1, rope.args, src, kd, vd, td, cd, md, False, out)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    rig.close()


def test_infinities_stay_where_they_are():
    """A number that is none makes its own pair none, nothing else of its head, without a norm; heads beside it are not touched by it."""
    geom, rig, table = _rig("bf16", 4, 2, 64, 16, [{0}], 4, 11)
    dev = rig.dev
    rope = Rope(geom, dev, 32, 0, False, 0)
    _, (qd, kd, vd), _ = _vectors(geom, dev, 1, False, 5)
    qd[0, 1, 3] = float("inf")
    qd[0, 2, 40] = float("-inf")                                          # (not turned)
    out = torch.zeros_like(qd)
    torch.cuda.synchronize()
    rig.lamps.rope_append(0, 1, rope.args, qd, kd, vd, torch.as_tensor(table, device=dev), torch.tensor([5], dtype=torch.int32, device=dev),
                          torch.ones(1, dtype=torch.uint8, device=dev), False, out)
    torch.cuda.synchronize()
    bad = ~torch.isfinite(out[0]).cpu()
    assert bad.nonzero().tolist() == [[1, 3], [1, 19], [2, 40]] and out[0, 2, 40] == float("-inf")
    rig.close()


@pytest.mark.parametrize("dtype,H,Hkv,D", [("bf16", 8, 2, 128), ("f32", 4, 4, 64)])
def test_positions_at_the_end_of_the_longest_row(dtype, H, Hkv, D):
    """A row of 2^30 positions.  On top of the bound above: an angle of 2^30 radians is rounded to 2^-24 here and by the kernel, which takes
    2^27.4 turns off it, rounded to 2^-26 of a turn (1e-7 radians), by 1 / (2 pi), off by half a step (1.2e-7): 4e-7 together."""
    bs, row = 64, 1 << 24
    new, p0 = 37, (1 << 30) - 37
    blocks = {p // bs for p in range(p0, p0 + new)} | {(1 << 29) // bs}
    geom, rig, table = _rig(dtype, H, Hkv, D, bs, [blocks], row, 23, layers=1)
    dev, rope = rig.dev, Rope(geom, rig.dev, D, 0, True, 0)
    td = torch.as_tensor(table, device=dev)
    far = lambda x: (np.abs(x[0]) <= bound(dtype, x[1], x[2]) + 4e-7 * x[2]).all()
    (q, k, v), (qd, kd, vd), _ = _vectors(geom, dev, new, False, 5)
    out = torch.zeros((new, H, D), dtype=rig.tdtype, device=dev)
    torch.cuda.synchronize()
    rig.lamps.rope_append_tokens(0, 1, new, rope.args, qd, kd, vd, torch.tensor([0, new], dtype=torch.int32, device=dev), td,
                                 torch.tensor([1 << 30], dtype=torch.int32, device=dev), out)
    one = torch.zeros((1, H, D), dtype=rig.tdtype, device=dev)
    torch.cuda.synchronize()
    rig.lamps.rope_append(0, 1, rope.args, qd, kd, vd, td, torch.tensor([(1 << 29) + 7], dtype=torch.int32, device=dev),
                          torch.ones(1, dtype=torch.uint8, device=dev), False, one)
    torch.cuda.synchronize()
    p = np.arange(p0, p0 + new)
    want, size = rope(q, p, 0)
    assert far((to_f64(out) - want, want, size))
    want, size = rope(q[:1], np.array([(1 << 29) + 7]), 0)
    assert far((to_f64(one) - want, want, size))
    kp, vp = t2n(rig.k_pool), t2n(rig.v_pool)
    places = [(i, x) for i, x in enumerate(p)]
    want, size = rope(k, p, 1)
    for i, x in places:
        at = table[0, x // bs], 0
        assert far((f64(kp[at][:, rig.k_index[x % bs]]) - want[i], want[i], size[i])), i
        assert (vp[at][:, rig.v_index[x % bs]] == v[i]).all(), i
    rig.close()
