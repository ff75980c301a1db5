"""How many launches a call on a cache of 8 bits is: counted in a captured graph, which then is replayed."""
import ctypes

import numpy as np
import pytest
import torch

import codes_forms as F
import paper_2410_18248_amd as P
import test_gpu_codes_decode as decoding
import test_gpu_codes_prefill as prefilling

pytestmark = pytest.mark.gpu


def _captured(rig, call, out):
    """(nodes, outputs of an eager call and of two replays)"""
    stream = torch.cuda.Stream(rig.dev)
    lam = P.Lamps(rig.cfg, rig.k_pool, rig.v_pool, rig.workspace, stream.cuda_stream)
    call(lam)
    torch.cuda.synchronize()
    results, graph = [out.clone()], torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.stream(stream):
        graph.capture_begin(capture_error_mode="relaxed")
        call(lam)
        graph.capture_end()
    nodes = ctypes.c_size_t()
    hip = ctypes.CDLL("libamdhip64.so")
    assert hip.hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(nodes)) == 0
    graph.instantiate()
    for _ in range(2):
        out.fill_(2.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        results.append(out.clone())
    lam.destroy()
    return nodes.value, results


@pytest.mark.parametrize("window,sinks,launches", [(256, 4, 1), (1000, 24, 1), (1000, 25, 2), (1 << 30, 0, 2)])
def test_one_token(window, sinks, launches):
    """A window that leaves nothing to cut, on a long row: no launch behind it that adds parts up."""
    ctx = [4000, 3000]
    rig, table = decoding.cache(8, 2, 128, 16, ctx, 51)
    q = F.normal(3, 2, 8, 128)
    out = torch.full(q.shape, 2.5, dtype=torch.bfloat16, device=rig.dev)
    args = q.to(rig.dev), rig.ints(table), rig.ints(ctx), torch.ones(2, dtype=torch.uint8, device=rig.dev), out
    torch.cuda.synchronize()
    nodes, results = _captured(rig, lambda lam: lam.decode_attn_window(1, 2, window, sinks, *args), out)
    assert nodes == launches
    for x in results:
        assert torch.equal(x, results[0])
    decoding.check(rig, 1, q, table, ctx, [1, 1], results[0], window, sinks)
    rig.close()


@pytest.mark.parametrize("window,sinks,launches", [(256, 4, 1), (700, 40, 1), (2000, 0, 2), (1 << 30, 0, 2)])
def test_many_tokens(window, sinks, launches):
    reqs = [(4000, 12), (2500, 30)]
    rig, table = decoding.cache(8, 2, 128, 16, [c for c, _ in reqs], 52)
    q = F.normal(3, 42, 8, 128)
    out = torch.full(q.shape, 2.5, dtype=torch.bfloat16, device=rig.dev)
    start = np.array([0, 12, 42])
    args = q.to(rig.dev), rig.ints(start), rig.ints(table), rig.ints([c for c, _ in reqs]), out
    torch.cuda.synchronize()
    nodes, results = _captured(rig, lambda lam: lam.prefill_attn_window(1, 2, 42, window, sinks, *args, max_new_tokens=30), out)
    assert nodes == launches
    for x in results:
        assert torch.equal(x, results[0])
    prefilling.check(rig, 1, q, reqs, table, start, results[0], prefilling.rounded, window, sinks)
    rig.close()
