"""The operators around the cache as they are used, one behind the other: tables from lengths, queries and keys normalised and turned on
their way into the cache, attention over windows -- by the calls, out of a captured graph, and in the serving loop -- against plain
numpy in 64 bits."""
import math

import numpy as np
import pytest
import torch

import lamps_workloads as W
import paper_2410_18248_amd as P
from operator_forms import f64, turned, window_attn
from paper_2410_18248_amd.engine import LiveEngine, RandomSource
from rig import Rig, n2t, to_f64

pytestmark = pytest.mark.gpu


def rounded(x, dtype):
    """float64 -> what the cache and the queries hold, as float64."""
    x = x.astype(np.float32)
    return f64(W.f32_to_bf16_bits(x.reshape(-1)).reshape(x.shape)) if dtype == "bf16" else x.astype(np.float64)


# What the rows are off by: as in test_gpu_window, and in bf16 a turned element within 2^-20 of a tie may be rounded the other way, a step of
# 2^-7: of 64 to 128 products of a score, |q||k| 2^-7 / sqrt(D) < 9 / 128 / 8 = 0.009 for one of them, which is the relative error of that weight.
def close(got, ref, size, dtype):
    off = 2e-5 * (size + np.abs(ref)) + 1e-6 if dtype == "f32" else (3 * 2.0 ** -8 + 0.02) * (size + np.abs(ref)) + 1e-5
    assert (np.abs(got - ref) <= off).all(), np.abs(got - ref).max()


class Model:
    """What a serving program keeps for one layer of each kind, and the numpy form of it."""

    def __init__(self, dtype, H, Hkv, D, bs, batch, row, window, sinks, seed):
        self.dtype, self.H, self.Hkv, self.D, self.bs, self.seed, self.looks = dtype, H, Hkv, D, bs, seed, [(window, sinks), (1 << 30, 0)]
        self.geom = W.Geometry(2, H, Hkv, D, bs, batch * row + 2, row, dtype)
        self.rig = Rig(self.geom, batch)
        self.freq = P.lamps_rope_frequencies(D // 2, 10000.0, P.LAMPS_ROPE_BY_PARTS, 4.0, 512.0, 1.0, 8.0)
        rng = np.random.default_rng(seed)
        self.w = [(1 + 0.2 * rng.standard_normal(D)).astype(np.float32) for _ in range(2)]
        if dtype == "bf16":
            self.w = [W.f32_to_bf16_bits(x) for x in self.w]
        self.rope = P.LampsRope(D // 2, P.LAMPS_ROPE_NEIGHBOURS, torch.tensor(self.freq, dtype=torch.float64, device=self.rig.dev), amplitude=1.1,
                                normalise=True, norm_eps=1e-6, q_weight=n2t(self.w[0], self.rig.dev), k_weight=n2t(self.w[1], self.rig.dev))
        self.K = [[np.zeros((0, Hkv, D)) for _ in range(batch)] for _ in range(2)]
        self.V = [[np.zeros((0, Hkv, D)) for _ in range(batch)] for _ in range(2)]

    def turn(self, x, p, which):
        return rounded(turned(f64(x), np.asarray(p), self.freq, True, 1.1, 1e-6, f64(self.w[which])), self.dtype)

    def expect(self, layer, r, q, k, v, first):
        """Rows of one request: its new keys and values join the cache; outputs and sizes."""
        p = np.arange(first, first + len(q))
        self.K[layer][r] = np.concatenate([self.K[layer][r], self.turn(k, p, 1)])
        self.V[layer][r] = np.concatenate([self.V[layer][r], f64(v)])
        return window_attn(self.turn(q, p, 0), self.K[layer][r], self.V[layer][r], first, *self.looks[layer])


@pytest.mark.parametrize("dtype,H,Hkv,D,bs", [("bf16", 8, 2, 128, 16), ("bf16", 4, 4, 64, 32), ("f32", 4, 2, 64, 16)])
def test_prompts_and_steps(dtype, H, Hkv, D, bs):
    """Prompts of three requests, then eight decode iterations of which the last six are replayed from one graph; the tables grow from a list of
    spare blocks on the device, whatever the host knows."""
    new, steps, row = [37, 1, 90], 8, 8 if bs == 16 else 4
    m = Model(dtype, H, Hkv, D, bs, 3, row, 25, 3, 17 + D)
    rig, lam, dev, B = m.rig, m.rig.lamps, m.rig.dev, 3
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    spare = torch.as_tensor(W.permutation(5, m.geom.num_blocks).astype(np.int32), device=dev)
    total = sum(new)
    with torch.cuda.stream(rig.compute):
        table = torch.full((B, row), -1, dtype=torch.int32, device=dev)
        cached, counts, ctx, start, report = ints([0] * B), ints(new), ints([0] * B), ints([0] * (B + 1)), ints([0] * 4)
        slots = torch.zeros(total, dtype=torch.int64, device=dev)
        lam.batch_tables(B, total, cached, counts, spare, spare.numel(), False, table, ctx, start, slots, report)
        at = np.concatenate([[0], np.cumsum(new)])
        for layer, (window, sinks) in enumerate(m.looks):
            q, (k, v) = W.queries(3 + layer, m.geom, total), W.logical_kv(9 + layer, m.geom, total)
            qd = n2t(q, dev)
            out = torch.zeros_like(qd)
            lam.rope_append_tokens(layer, B, total, m.rope, qd, n2t(k, dev), n2t(v, dev), start, table, ctx, qd)
            if layer == 0:
                lam.prefill_attn_window(layer, B, total, window, sinks, qd, start, table, ctx, out, max_new_tokens=max(new))
            else:
                lam.prefill_attn(layer, B, total, qd, start, table, ctx, out, max_new_tokens=max(new))
            rig.compute.synchronize()
            for r in range(B):
                s = slice(at[r], at[r + 1])
                close(to_f64(out)[s], *m.expect(layer, r, q[s], k[s], v[s], 0), dtype)
        taken = int(report[0])
        assert taken == sum(-(-n // bs) for n in new) and report.tolist()[1:] == [0, -1, total]
        # the slot map is where the values are
        values = rig.v_pool.view(m.geom.num_blocks, 2, Hkv, -1)[slots // bs, 0][torch.arange(total, device=dev)[:, None, None], torch.arange(
            Hkv, device=dev)[None, :, None], torch.as_tensor(rig.v_index, device=dev)[slots % bs][:, None]]
        assert torch.equal(values.cpu(), n2t(W.logical_kv(9, m.geom, total)[1], "cpu"))

    # decode: everything an iteration touches lives in tensors allocated once
    with torch.cuda.stream(rig.compute):
        left = spare[taken:].clone()
        ones, running = ints([1] * B), torch.ones(B, dtype=torch.uint8, device=dev)
        q_s = torch.zeros((2, B, H, D), dtype=rig.tdtype, device=dev)
        k_s, v_s, out_s = torch.zeros((2, B, Hkv, D), dtype=rig.tdtype, device=dev), torch.zeros((2, B, Hkv, D), dtype=rig.tdtype, device=dev), torch.zeros_like(q_s)
        cached.copy_(ctx)

    def iteration():
        lam.batch_tables(B, B, cached, ones, left, left.numel(), True, table, ctx, start, None, report)
        for layer, (window, sinks) in enumerate(m.looks):
            lam.rope_append(layer, B, m.rope, q_s[layer], k_s[layer], v_s[layer], table, cached, running, False, q_s[layer])
            if layer == 0:
                lam.decode_attn_window(layer, B, window, sinks, q_s[layer], table, ctx, running, out_s[layer])
            else:
                lam.decode_attn(layer, B, q_s[layer], table, ctx, running, out_s[layer])

    graph, lens = None, list(new)
    for it in range(steps):
        given = [(W.queries(50 * it + l, m.geom, B), *W.logical_kv(70 * it + l + 1, m.geom, B)) for l in range(2)]
        with torch.cuda.stream(rig.compute):              # the program's own eager work between replays
            for l in range(2):
                q_s[l].copy_(n2t(given[l][0], dev))
                k_s[l].copy_(n2t(given[l][1], dev))
                v_s[l].copy_(n2t(given[l][2], dev))
            if it < 2:
                iteration()
            else:
                if graph is None:
                    rig.compute.synchronize()
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=rig.compute):
                        iteration()
                graph.replay()
        rig.compute.synchronize()
        took = sum(c % bs == 0 for c in lens)
        assert report.tolist() == [took, 0, -1, B] and ctx.tolist() == [c + 1 for c in lens]
        for l in range(2):
            q, k, v = given[l]
            for r in range(B):
                close(to_f64(out_s)[l, r:r + 1], *m.expect(l, r, q[r:r + 1], k[r:r + 1], v[r:r + 1], lens[r]), dtype)
        lens = [c + 1 for c in lens]
        with torch.cuda.stream(rig.compute):
            left.copy_(torch.cat([left[took:], left[:took]]))      # (ids taken go out of the list's front)
            cached.copy_(ctx)
    rig.close()


def test_two_contexts_on_two_streams():
    """Each with its workspace: calls of both at once are as calls of each alone."""
    models = [Model("bf16", 8, 2, 128, 16, 2, 200, 1500, 4, s) for s in (1, 2)]
    outs = []
    for m in models:
        table, _ = W.deal_block_table(W.permutation(m.seed, m.geom.num_blocks), [3100, 2000], m.geom)
        for pool in (m.rig.k_pool, m.rig.v_pool):
            pool.normal_(generator=torch.Generator(device=m.rig.dev).manual_seed(m.seed))
        m.args = [n2t(W.queries(m.seed, m.geom, 2), m.rig.dev), torch.as_tensor(table, device=m.rig.dev),
                  torch.tensor([3100, 2000], dtype=torch.int32, device=m.rig.dev), torch.ones(2, dtype=torch.uint8, device=m.rig.dev)]
        m.q = n2t(W.queries(m.seed + 9, m.geom, 30), m.rig.dev)
        m.start = torch.tensor([0, 11, 30], dtype=torch.int32, device=m.rig.dev)

    def run(m, out, rows):
        m.rig.lamps.decode_attn_window(1, 2, 1500, 4, *m.args, out)
        m.rig.lamps.prefill_attn_window(1, 2, 30, 1500, 4, m.q, m.start, m.args[1], m.args[2], rows)
    new = lambda m: (torch.zeros_like(m.args[0]), torch.zeros_like(m.q))
    for m in models:
        outs.append(new(m))
        torch.cuda.synchronize()
        run(m, *outs[-1])
        torch.cuda.synchronize()
    both = [[new(m) for m in models] for _ in range(10)]
    torch.cuda.synchronize()
    for pair in both:
        for m, o in zip(models, pair):
            run(m, *o)
    torch.cuda.synchronize()
    for pair in both:
        for o, e in zip(pair, outs):
            assert torch.equal(o[0], e[0]) and torch.equal(o[1], e[1])
    for m in models:
        m.rig.close()


@pytest.mark.parametrize("dtype,H,Hkv", [("bf16", 8, 2), ("f32", 4, 4)])
def test_served_with_rotary_positions_and_windows(dtype, H, Hkv):
    """The serving loop of a model with rotary positions, every other layer with a window: prompts, API responses, swaps, discards and
    recomputes, and every token's attention."""
    L, D, bs, tdt = 2, 64, 16, torch.bfloat16 if dtype == "bf16" else torch.float32
    memory_tokens, n_req, looks = 400, 6, [(20, 3), None]
    nb = memory_tokens // bs + n_req + 2
    cfg = P.LampsConfig(L, H, Hkv, D, bs, nb, 16, 8, P.LAMPS_BF16 if dtype == "bf16" else P.LAMPS_F32, 0.0, 0, 0)
    scfg = P.LampsSchedConfig(P.LAMPS_POLICY_LAMPS, 4, memory_tokens, 20, 1, 1 << 20, 50.0, 1.0, P.LampsCostModel(1e-3, 1e-7, 1e-4, 1e-5, 1e-4, 1e-6, 0, 0))
    src = RandomSource(7, H, Hkv, D, tdt)
    freq = P.lamps_rope_frequencies(D, 10000.0)
    rope = P.LampsRope(D, P.LAMPS_ROPE_HALVES, torch.tensor(freq, dtype=torch.float64, device="cuda:0"), normalise=True)
    tokens = [0]

    def observer(kind, rid, layer, first_pos, rows):
        n = rows.shape[0]
        q, k, v = (x.double().numpy() for x in src.rows(rid, 0, first_pos + n, layer))
        turn = lambda x, p: rounded(turned(x, p, freq, False, 1.0, 1e-6), dtype)
        ref, size = window_attn(turn(q[first_pos:], np.arange(first_pos, first_pos + n)), turn(k, np.arange(first_pos + n)), v, first_pos,
                                *(looks[layer] or (1 << 30, 0)))
        close(rows.double().numpy(), ref, size, dtype)
        tokens[0] += n

    eng = LiveEngine(cfg, scfg, src, observer=observer, rope=rope, windows=looks)
    strategies = [P.LAMPS_PRESERVE, P.LAMPS_DISCARD, P.LAMPS_SWAP]
    for i in range(n_req):
        eng.add(i, 0.001 * i, 10 + 9 * i, [(3 + i, 0.003, 5, strategies[i % 3]), (6, None, 0, None)])
    stats = eng.run(max_iterations=2000)
    assert eng.lam.num_free() == nb and stats["swapped_in_blocks"] > 0 and stats["discarded_blocks"] > 0
    assert tokens[0] >= L * sum(10 + 9 * i + 3 + i + 5 + 6 for i in range(n_req))
    assert math.isfinite(stats["gpu_s"])
    eng.close()
