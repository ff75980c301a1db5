"""A cache of 8 bits in plain numpy, from its formulas: e4m3 codes, scales, where they lie, and what appends make of a pool's bytes."""
import numpy as np
import torch

import paper_2410_18248_amd as P
from rig import Rig, t2n

# the numbers that codes 0 .. 126 stand for: 3 bits of fraction, exponents from -6, then subnormal ones
NUMBERS = np.array([((c & 7) / 8 + (1 if c >> 3 else 0)) * 2.0 ** (max(c >> 3, 1) - 7) for c in range(127)])
MIDDLES = (NUMBERS[1:] + NUMBERS[:-1]) / 2
VALUES = np.concatenate([NUMBERS, [np.nan], -NUMBERS, [np.nan]])
LEAST, MOST = -110, 119                             # exponents of scales


def codes_of(y):
    """Numbers rounded to codes, ties to the even one; beyond the largest: the largest."""
    size = np.abs(y)
    c = np.searchsorted(MIDDLES, size, side="left")
    tie = (c < 126) & (MIDDLES[np.minimum(c, 125)] == size)
    c = np.where(tie & (c % 2 == 1), c + 1, c)
    c = np.where(np.isfinite(y), c, 127).astype(np.uint8)
    return c | (np.signbit(y) << 7).astype(np.uint8)


def scale_of(x):
    """Of numbers along the last axis, those of a block's new tokens."""
    most = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.where(most > 0, np.ceil(np.log2(np.where(most > 0, most, 1.0) / 448.0)), LEAST)
    e = np.where(most > 448.0 * 2.0 ** e, e + 1, e)
    e = np.where((most > 0) & (most <= 448.0 * 2.0 ** (e - 1)), e - 1, e)
    return 2.0 ** np.clip(e, LEAST, MOST)


def places(bs, D):
    """Byte of (slot, dim) in a tile, of keys and of values."""
    s, d = np.arange(bs)[:, None], np.arange(D)[None, :]
    base, t = s // 16 * 16 * D, s % 16
    return base + (d // 16 * 16 + t) * 16 + d % 16, base + ((d // 64 * 4 + t // 4) * 16 + d % 16) * 16 + d % 64 // 16 * 4 + t % 4


class Pools:
    """The bytes of both pools on the host, [blocks][layers][slice]."""

    def __init__(self, k, v, heads, bs, D):
        self.k, self.v, self.heads, self.bs, self.D = k, v, heads, bs, D
        self.at = places(bs, D)
        self.tiles = heads * bs * D

    def scales(self, block, layer):
        """[head][keys, values]"""
        return self.k[block, layer, self.tiles:self.tiles + 8 * self.heads].view(np.float32).reshape(self.heads, 2)

    def codes(self, which, block, layer):
        return (self.k, self.v)[which][block, layer, :self.tiles].reshape(self.heads, self.bs * self.D)

    def append(self, layer, row, first, k, v):
        """k, v [n][heads][D] in float64, positions first and up of the request with this table row."""
        n, bs = k.shape[0], self.bs
        for b in range(first // bs, (first + n - 1) // bs + 1):
            lo, hi, block = max(first, b * bs), min(first + n, (b + 1) * bs), int(row[b])
            for which, x in enumerate((k, v)):
                new = x[lo - first:hi - first]
                scale = scale_of(new.transpose(1, 0, 2).reshape(self.heads, -1))
                codes, scales = self.codes(which, block, layer), self.scales(block, layer)
                if lo % bs:
                    old = scales[:, which].astype(np.float64)
                    scale = np.maximum(scale, old)
                    there = self.at[which][:lo % bs].reshape(-1)
                    for g in range(self.heads):
                        if scale[g] != old[g]:
                            codes[g, there] = codes_of(VALUES[codes[g, there]] * (old[g] / scale[g]))
                for g in range(self.heads):
                    y = np.where(np.isfinite(new[:, g]), new[:, g], np.nan) / scale[g]
                    y = np.where(np.isfinite(new[:, g]), y, np.copysign(np.nan, new[:, g]))
                    codes[g, self.at[which][lo % bs:lo % bs + hi - lo]] = codes_of(y)
                scales[:, which] = scale

    def logical(self, layer, row, count):
        """Keys and values of positions 0 .. count - 1, [count][heads][D] in float64."""
        out = []
        for which in (0, 1):
            x = np.empty((count, self.heads, self.D))
            for b in range((count + self.bs - 1) // self.bs):
                n = min(self.bs, count - b * self.bs)
                y = VALUES[self.codes(which, int(row[b]), layer)[:, self.at[which][:n]]] * self.scales(int(row[b]), layer)[:, which, None, None].astype(np.float64)
                x[b * self.bs:b * self.bs + n] = y.transpose(1, 0, 2)
            out.append(x)
        return out


def no_sign(codes):
    """Codes with one NaN instead of two."""
    return np.where(codes & 127 == 127, 127, codes)


class CodesRig(Rig):
    """Pools of 8 bits, workspace, streams and a Lamps context; the pools' first bytes are noise (which holds NaN)."""

    def __init__(self, layers, H, Hkv, D, bs, blocks, row, max_batch, scale=0.0, seed=1, **kw):
        self.dev, self.tdtype = torch.device("cuda:0"), torch.bfloat16
        self.cfg = P.LampsConfig(layers, H, Hkv, D, bs, blocks, row, max_batch, P.LAMPS_E4M3, scale, 0, kw.pop("staging_bytes", 0),
                                 kw.pop("direct_copy_bytes", 0), kw.pop("zero_copy_workgroups", 0))
        assert not kw and P.lamps_kv_layout(self.cfg) == P.LAMPS_LAYOUT_CODES
        size = P.lamps_pool_bytes(self.cfg)
        g = torch.Generator().manual_seed(seed)
        self.k_pool, self.v_pool = (torch.randint(0, 256, (blocks, layers, size // blocks // layers), generator=g, dtype=torch.uint8).to(self.dev) for _ in range(2))
        self.workspace = torch.empty(P.lamps_workspace_bytes(self.cfg), dtype=torch.uint8, device=self.dev)
        self.compute = torch.cuda.current_stream(self.dev)
        self.s_out, self.s_in = (torch.cuda.Stream(self.dev) for _ in range(2))
        torch.cuda.synchronize()
        self.lamps = P.Lamps(self.cfg, self.k_pool, self.v_pool, self.workspace, self.compute.cuda_stream, self.s_out.cuda_stream, self.s_in.cuda_stream)

    def host(self):
        torch.cuda.synchronize()
        return Pools(self.k_pool.cpu().numpy().copy(), self.v_pool.cpu().numpy().copy(), self.cfg.num_kv_heads, self.cfg.block_size, self.cfg.head_dim)

    def ints(self, x):
        return torch.tensor(np.asarray(x), dtype=torch.int32, device=self.dev)

    def deal(self, tokens, seed=7):
        """A table of random blocks for requests of so many tokens, -1 behind them; on the host."""
        bs, ids, at = self.cfg.block_size, np.random.RandomState(seed).permutation(self.cfg.num_blocks), 0
        table = np.full((len(tokens), self.cfg.max_blocks_per_req), -1, dtype=np.int32)
        for r, t in enumerate(tokens):
            n = (t + bs - 1) // bs
            table[r, :n] = ids[at:at + n]
            at += n
        assert at <= self.cfg.num_blocks
        return table

    def append_tokens(self, layer, k, v, counts, table, ctx):
        start = np.concatenate([[0], np.cumsum(counts)])
        args = [x.to(self.dev) for x in (k, v)] + [self.ints(start), self.ints(table), self.ints(ctx)]
        torch.cuda.synchronize()
        self.lamps.kv_append_tokens(layer, len(counts), int(start[-1]), *args)
        torch.cuda.synchronize()


def normal(seed, *shape, size=1.0):
    """bf16 numbers, on the host."""
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * size).bfloat16()


def f64(t):
    return t.detach().cpu().double().numpy()


def same(pools, expected):
    """Bytes of both pools, but for the sign of NaN and the bytes that nothing uses."""
    n = pools.tiles
    for a, b in ((pools.k, expected.k), (pools.v, expected.v)):
        bad = np.argwhere(no_sign(a[:, :, :n]) != no_sign(b[:, :, :n]))
        assert len(bad) == 0, (len(bad), bad[:4])
    m = n + 8 * pools.heads
    a, b = pools.k[:, :, n:m], expected.k[:, :, n:m]
    assert (a == b).all(), np.argwhere(a != b)[:4]
    assert (pools.k[:, :, m:] == expected.k[:, :, m:]).all() and (pools.v[:, :, n:] == expected.v[:, :, n:]).all()
