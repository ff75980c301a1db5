"""A cache of 8 bits as a serving program has it: the scheduler's loop over it, iterations captured and replayed, other streams than the current one,
appends and reads beside attention."""
import numpy as np
import pytest
import torch

import codes_forms as F
import lamps_workloads as W
import paper_2410_18248_amd as P
from operator_forms import window_attn
from paper_2410_18248_amd.engine import LiveEngine, RandomSource
from test_gpu_codes_decode import bound
from test_gpu_codes_prefill import rounded

pytestmark = pytest.mark.gpu
ALL = 1 << 30


class Model:
    """What a request's cache holds, layer by layer, from the numbers that were appended to it: blocks in its own order."""

    def __init__(self, layers, heads, bs, D, blocks):
        self.pools = F.Pools(*(np.zeros((blocks, layers, heads * bs * D + -(-heads * 8 // 128) * 128), dtype=np.uint8) for _ in range(2)), heads, bs, D)
        self.row = np.arange(blocks)

    def append(self, layer, first, k, v):
        self.pools.append(layer, self.row, first, F.f64(k), F.f64(v))

    def attend(self, layer, first, q, window, sinks):
        K, V = self.pools.logical(layer, self.row, first + q.shape[0])
        return window_attn(F.f64(q), K, V, first, window, sinks)


@pytest.mark.parametrize("H,Hkv,layered,windows", [(8, 2, False, None), (4, 4, True, None), (8, 2, False, [(20, 4), None])])
def test_trace_served_over_8_bits(H, Hkv, layered, windows):
    """Every attention output of a small trace with all three strategies, against the codes that its own appends make: swapped blocks bring codes and scales back,
    discarded contexts begin anew, in blocks that others have left."""
    L, D, bs, memory_tokens, n_req = 2, 64, 16, 400, 9
    nb = memory_tokens // bs + n_req + 2
    cfg = P.LampsConfig(L, H, Hkv, D, bs, nb, 16, 8, P.LAMPS_E4M3, 0.0, 0, 0)
    cost = P.LampsCostModel(1e-3, 1e-7, 1e-4, 1e-5, 1e-4, 1e-6, 0, 0)
    scfg = P.LampsSchedConfig(P.LAMPS_POLICY_LAMPS, 4, memory_tokens, 20, 1, 1 << 20, 50.0, 1.0, cost)
    src = RandomSource(78, H, Hkv, D, torch.bfloat16)
    models = [Model(L, Hkv, bs, D, 16) for _ in range(n_req)]
    seen = {}

    def observer(kind, rid, layer, first, rows):
        n = rows.shape[0]
        q, k, v = src.rows(rid, first, n, layer)
        models[rid].append(layer, first, k, v)
        window, sinks = (windows[layer] if windows and windows[layer] else (ALL, 0))
        ref, size = models[rid].attend(layer, first, q, window, sinks)
        off = np.abs(rows.double().numpy() - ref) - (bound if kind == "decode" else rounded)(ref, size)
        assert (off <= 0).all(), (kind, rid, layer, first, off.max())
        seen[rid, layer] = seen.get((rid, layer), 0) + n
    eng = LiveEngine(cfg, scfg, src, observer=observer, layered_swap=layered, windows=windows)
    u = W.uniform01(6, 10 * n_req)
    strategies, want = [P.LAMPS_PRESERVE, P.LAMPS_DISCARD, P.LAMPS_SWAP], {}
    for i in range(n_req):
        x = u[10 * i:10 * i + 10]
        prompt, segs = int(x[0] * 30), []
        for k in range(1 + int(x[1] * 2)):
            segs.append((1 + int(x[2 + k] * 12), 0.002 + 0.01 * x[6 + k], int(x[4 + k] * 8), strategies[(i + k) % 3]))
        segs.append((1 + int(x[8] * 10), None, 0, None))
        want[i] = prompt + sum(s[0] + s[2] for s in segs)
        eng.add(i, 0.001 * i, prompt, segs)
    stats = eng.run(max_iterations=5000)
    assert eng.lam.num_free() == nb and all(seen[i, l] >= want[i] for i in range(n_req) for l in range(L))
    assert stats["swapped_out_blocks"] > 0 and stats["swapped_in_blocks"] > 0 and stats["discarded_blocks"] > 0
    eng.close()


def test_rotary_positions_refuse():
    cfg = P.LampsConfig(1, 4, 2, 64, 16, 4, 4, 2, P.LAMPS_E4M3, 0.0, 0, 0)
    f = torch.tensor(P.lamps_rope_frequencies(64, 10000.0), dtype=torch.float64, device="cuda:0")
    with pytest.raises(ValueError, match="8 bits"):
        LiveEngine(cfg, None, None, rope=P.LampsRope(64, frequencies=f))
    rig = F.CodesRig(1, 4, 2, 64, 16, 4, 4, 2)
    x = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device=rig.dev)
    args = x, x[:, :2].contiguous(), x[:, 2:].contiguous(), rig.ints([[0] * 4] * 2), rig.ints([0, 0])
    for call in (lambda: rig.lamps.rope_append(0, 2, P.LampsRope(64, frequencies=f), *args, torch.ones(2, dtype=torch.uint8, device=rig.dev), False, x),
                 lambda: rig.lamps.rope_append_tokens(0, 2, 2, P.LampsRope(64, frequencies=f), *args[:3], rig.ints([0, 1, 2]), *args[3:], x)):
        with pytest.raises(P.LampsError, match="8 bits") as e:
            call()
        assert e.value.status == -1
    rig.close()


@pytest.mark.parametrize("H,Hkv,D,ctx", [(8, 2, 128, [15, 16, 47, 3, 200]), (4, 4, 64, [31, 1, 64, 4000]), (16, 1, 256, [700, 33])])
def test_decode_iterations_replayed_from_a_graph(H, Hkv, D, ctx):
    """Append and attention of two layers, lengths advanced on the device, and the last few positions read back: one eager iteration, then replays, each
    against the formulas, with eager work of the program's own between them."""
    L, bs, steps, B = 2, 16, 5, len(ctx)
    rig = F.CodesRig(L, H, Hkv, D, bs, sum((c + steps + bs - 1) // bs for c in ctx) + 2, (max(ctx) + steps) // bs + 1, B)
    lam, dev = rig.lamps, rig.dev
    table = rig.deal([c + steps for c in ctx])
    for layer in range(L):
        rig.append_tokens(layer, F.normal(layer, sum(ctx), Hkv, D), F.normal(9 + layer, sum(ctx), Hkv, D), ctx, table, ctx)
    expected = rig.host()
    stream = torch.cuda.Stream(dev)
    lam2 = P.Lamps(rig.cfg, rig.k_pool, rig.v_pool, rig.workspace, stream.cuda_stream)
    td, cd, md = rig.ints(table), rig.ints(ctx), torch.ones(B, dtype=torch.uint8, device=dev)
    md[0] = 0
    cd1, start = torch.zeros_like(cd), rig.ints(np.arange(B + 1))
    q, k, v = (torch.zeros(L, B, n, D, dtype=torch.bfloat16, device=dev) for n in (H, Hkv, Hkv))
    out, kr, vr = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)

    def iteration():
        torch.add(cd, 1, out=cd1)
        for layer in range(L):
            lam2.kv_append(layer, B, k[layer], v[layer], td, cd, md, layer == L - 1)
            lam2.decode_attn(layer, B, q[layer], td, cd1, md, out[layer])
            lam2.kv_read_tokens(layer, B, B, start, td, cd1, kr[layer], vr[layer])
    graph, now = None, list(ctx)
    for step in range(steps):
        new = [[F.normal(100 * step + 10 * i + layer, B, n, D, size=1.0 if step < 3 else 9.0) for layer in range(L)] for i, n in enumerate((H, Hkv, Hkv))]
        for x, y in zip((q, k, v), new):
            x.copy_(torch.stack(y))
        out.fill_(2.5)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            if step == 0:
                iteration()
            else:
                if graph is None:
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=stream):
                        iteration()
                graph.replay()
        stream.synchronize()
        got, back = F.f64(out), (F.f64(kr), F.f64(vr))
        for layer in range(L):
            for r in range(1, B):
                expected.append(layer, table[r], now[r], F.f64(new[1][layer][r:r + 1]), F.f64(new[2][layer][r:r + 1]))
                K, V = expected.logical(layer, table[r], now[r] + 1)
                ref, size = window_attn(F.f64(new[0][layer][r:r + 1]), K, V, now[r], ALL, 0)
                assert (np.abs(got[layer, r] - ref[0]) <= bound(ref[0], size[0])).all(), (step, layer, r)
                assert (back[0][layer, r] == K[-1]).all() and (back[1][layer, r] == V[-1]).all()
        for r in range(1, B):
            now[r] += 1
        assert (got[:, 0] == 2.5).all() and cd.tolist() == now
        F.same(rig.host(), expected)
    torch.cuda.synchronize()
    lam2.destroy()
    rig.close()


def test_prompts_replayed_from_a_graph():
    """Tables, append and attention of prompts and responses, cut and whole, in a graph: every replay the eager call's bits."""
    rig = F.CodesRig(1, 8, 2, 128, 16, 330, 260, 4)
    dev, lam = rig.dev, rig.lamps
    stream = torch.cuda.Stream(dev)
    lam2 = P.Lamps(rig.cfg, rig.k_pool, rig.v_pool, rig.workspace, stream.cuda_stream)
    cached, new = [4000, 0, 30, 500], [20, 90, 1, 17]
    total = sum(new)
    first = rig.deal([c + n for c, n in zip(cached, new)])
    rig.append_tokens(0, F.normal(1, sum(cached), 2, 128), F.normal(2, sum(cached), 2, 128), cached, first, cached)
    ids = np.concatenate([first[r][:(c + n + 15) // 16] for r, (c, n) in enumerate(zip(cached, new))])
    table, ctx, start = torch.zeros(4, 260, dtype=torch.int32, device=dev), rig.ints([0] * 4), rig.ints([0] * 5)
    have, bring, given = rig.ints(cached), rig.ints(new), rig.ints(ids)
    q, k, v = (torch.zeros(total, n, 128, dtype=torch.bfloat16, device=dev) for n in (8, 2, 2))
    out = torch.zeros_like(q)

    def run():
        lam2.batch_tables(4, total, have, bring, given, len(ids), False, table, ctx, start)
        lam2.kv_append_tokens(0, 4, total, k, v, start, table, ctx)
        lam2.prefill_attn(0, 4, total, q, start, table, ctx, out, max_new_tokens=90)
    snap, graph = (rig.k_pool.clone(), rig.v_pool.clone()), None
    for step in range(4):
        for x, n in ((q, 8), (k, 2), (v, 2)):
            x.copy_(F.normal(50 * step + n, total, n, 128))
        results = []
        for how in ("eager", "graph"):
            rig.k_pool.copy_(snap[0])
            rig.v_pool.copy_(snap[1])
            out.fill_(2.5)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                if how == "eager":
                    run()
                else:
                    if graph is None:
                        graph = torch.cuda.CUDAGraph()
                        with torch.cuda.graph(graph, stream=stream):
                            run()
                    graph.replay()
            torch.cuda.synchronize()
            results.append((out.clone(), rig.k_pool.clone(), rig.v_pool.clone()))
        assert all(torch.equal(a, b) for a, b in zip(*results)) and not (results[0][0] == 2.5).all(-1).any()
    lam2.destroy()
    rig.close()


def test_far_blocks_of_a_long_cache():
    """Offsets beyond 32 bits: a pool of more than 4 GiB, the request's blocks at its end."""
    Hkv, D, bs, ctx = 8, 128, 64, 200
    slice_ = Hkv * bs * D + 128
    blocks = (5 << 30) // slice_
    cfg = P.LampsConfig(1, 16, Hkv, D, bs, blocks, 4, 1, P.LAMPS_E4M3)
    dev = torch.device("cuda:0")
    k_pool, v_pool = (torch.zeros(P.lamps_pool_bytes(cfg), dtype=torch.uint8, device=dev) for _ in range(2))
    lam = P.Lamps(cfg, k_pool, v_pool, torch.empty(P.lamps_workspace_bytes(cfg), dtype=torch.uint8, device=dev))
    table = [blocks - 1, blocks - 3, 0, blocks - 2]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    q, k, v = F.normal(1, ctx, 16, D), F.normal(2, ctx, Hkv, D), F.normal(3, ctx, Hkv, D)
    args = ints([0, ctx]), ints([table]), ints([ctx])
    lam.kv_append_tokens(0, 1, ctx, k.to(dev), v.to(dev), *args)
    model = Model(1, Hkv, bs, D, 4)
    model.append(0, 0, k, v)
    back = [torch.zeros(ctx, Hkv, D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    lam.kv_read_tokens(0, 1, ctx, *args, *back)
    many, one = torch.zeros(ctx, 16, D, dtype=torch.bfloat16, device=dev), torch.zeros(1, 16, D, dtype=torch.bfloat16, device=dev)
    lam.prefill_attn(0, 1, ctx, q.to(dev), *args, many)
    lam.decode_attn(0, 1, q[-1:].to(dev), *args[1:], torch.ones(1, dtype=torch.uint8, device=dev), one)
    torch.cuda.synchronize()
    for x, y in zip(back, model.pools.logical(0, model.row, ctx)):
        np.testing.assert_array_equal(F.f64(x), y)
    ref, size = model.attend(0, 0, q, ALL, 0)
    assert (np.abs(F.f64(many) - ref) <= rounded(ref, size)).all()
    assert (np.abs(F.f64(one[0]) - ref[-1]) <= bound(ref[-1], size[-1])).all()
    lam.destroy()


def test_blocks_4_gib_apart():
    """A block whose layers take more than 4 GiB of a pool: the tiles' kernel, which keeps that distance in 32 bits, is not taken."""
    L, Hkv, D, bs = 520, 32, 256, 1024
    cfg = P.LampsConfig(L, Hkv, Hkv, D, bs, 3, 2, 1, P.LAMPS_E4M3, 0.0, 0, 0)
    size = P.lamps_pool_bytes(cfg)
    assert size // 3 > 1 << 32
    dev = torch.device("cuda:0")
    k_pool, v_pool = (torch.zeros(size, dtype=torch.uint8, device=dev) for _ in range(2))
    cfg.staging_bytes = 0
    lam = P.Lamps(cfg, k_pool, v_pool, torch.empty(P.lamps_workspace_bytes(cfg), dtype=torch.uint8, device=dev))
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    ctx, n = 1030, 9
    k, v, q = F.normal(2, ctx, Hkv, D), F.normal(3, ctx, Hkv, D), F.normal(1, n, Hkv, D)
    table = ints([[2, 1]])
    lam.kv_append_tokens(L - 1, 1, ctx, k.to(dev), v.to(dev), ints([0, ctx]), table, ints([ctx]))
    out = torch.zeros(n, Hkv, D, dtype=torch.bfloat16, device=dev)
    lam.prefill_attn(L - 1, 1, n, q.to(dev), ints([0, n]), table, ints([ctx]), out)
    torch.cuda.synchronize()
    model = Model(1, Hkv, bs, D, 2)
    model.append(0, 0, k, v)
    K, V = model.pools.logical(0, model.row, ctx)
    for h in (0, 17, 31):
        ref, size = window_attn(F.f64(q[:, h:h + 1]), K[:, h:h + 1], V[:, h:h + 1], ctx - n, ALL, 0)
        assert (np.abs(F.f64(out[:, h:h + 1]) - ref) <= bound(ref, size)).all()
    lam.destroy()
