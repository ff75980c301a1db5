"""Windowed attention under other softmax scales, negative ones among them, and with scores of a wide range, whose largest stands anywhere: the
reference of the exponentials moves in the middle of a walk, and parts and waves come with references far apart."""
import numpy as np
import pytest
import torch

import lamps_workloads as W
import paper_2410_18248_amd as P
from operator_forms import f64, seen
from rig import Rig, n2t, to_f64

pytestmark = pytest.mark.gpu

#        form             dtype  H   Hkv D   bs  (context, new tokens) per request                                              window, sinks
FORMS = {
    "narrow":          ("bf16", 8, 2, 128, 16, [(47, 5), (200, 64), (130, 20)], 50, 17),
    "wide":            ("bf16", 32, 8, 128, 16, [(400, 400), (330, 170)], 97, 20),
    "plain":           ("bf16", 4, 4, 128, 16, [(300, 300), (95, 31)], 60, 16),
    "heads of 64":     ("bf16", 8, 2, 64, 32, [(300, 250), (95, 40)], 64, 40),
    "teams":           ("bf16", 16, 8, 128, 16, [(2600, 2500), (2300, 2300)], 1100, 20),
    "teams of 256":    ("bf16", 4, 2, 256, 16, [(300, 300), (130, 50)], 100, 33),
    "plain of 256":    ("bf16", 4, 4, 256, 32, [(90, 90), (150, 50)], 70, 4),
    "shared":          ("bf16", 32, 8, 128, 16, [(1500, 40), (900, 37), (30, 30), (1200, 64), (800, 1), (1100, 40)], 1000, 20),
    "shared, 64":      ("bf16", 16, 8, 64, 16, [(1500, 150), (1100, 140), (900, 170)], 800, 3),
    "many parts":      ("bf16", 8, 2, 128, 16, [(3000, 16)], 2500, 33),
    "fp32":            ("f32", 8, 2, 64, 16, [(117, 60), (33, 33), (300, 100)], 80, 20),
    "fp32 to a wave":  ("f32", 8, 2, 32, 16, [(3000, 3000), (2500, 2403), (1900, 1797)], 300, 20),
    "rows":            ("bf16", 8, 2, 128, 16, [(200, 64), (130, 20)], 50, 17),
    "rows, plain":     ("bf16", 4, 4, 64, 16, [(200, 64), (130, 20)], 50, 17),
    "rows, fp32":      ("f32", 8, 2, 64, 16, [(200, 64), (130, 20)], 50, 17),
}
DECODE = {
    "grouped":         ("bf16", 8, 2, 128, 16, [130, 16, 1, 200, 333], 90, 17),
    "plain":           ("bf16", 4, 4, 128, 16, [130, 16, 1, 200, 333], 90, 17),
    "of 256":          ("bf16", 16, 1, 256, 16, [70, 131], 65, 33),
    "fp32":            ("f32", 8, 2, 64, 16, [130, 16, 1, 200, 333], 90, 17),
    "fp32, plain":     ("f32", 4, 4, 128, 16, [130, 16, 1, 200, 333], 90, 17),
    "parts":           ("bf16", 8, 2, 128, 16, [5000], 2000, 33),
    "parts, plain":    ("bf16", 4, 4, 64, 16, [5000, 2500], 2000, 33),
    "parts, fp32":     ("f32", 8, 2, 64, 32, [5000], 2000, 33),
}
# Keys of what stands out are a u / 2, u of ones and minus ones, and the queries 2 u more than N(0, 1): scores a sqrt(D) (1 + N(0, 1 / D)),
# 8 to 45 at these heights, in units of 1 / sqrt(D); those of the others N(0, 1 + 4).
#          where (share of the positions that the last token sees, < 0: sinks first) and heights
SCENES = {
    "wide":       None,                                                             # queries 16 times as large: scores N(0, 256)
    "late":       [(0.93, 4.0)],
    "sink":       [(-1, 4.0), (0.93, 1.0)],
    "rising":     [(0.1, 1.0), (0.35, 1.9), (0.6, 2.8), (0.85, 3.7)],
    "falling":    [(0.1, 3.7), (0.35, 2.8), (0.6, 1.9), (0.85, 1.0)],
    "two alike":  [(0.2, 3.0), (0.8, 3.0)],
}
SCALES = [1.0, -1.0, 0.3, -2.5]                                                     # times 1 / sqrt(head size)
STEP = 2.0 ** -8


def _made(dtype, H, Hkv, D, ctx, rows, scene, sign, window, sinks, seed, geom):
    """Keys, values, queries: what stands out lies where every request's last token sees it."""
    rng = np.random.default_rng(seed)
    u = np.sign(rng.standard_normal(D))
    store = (lambda x: W.f32_to_bf16_bits(x.astype(np.float32).reshape(-1)).reshape(x.shape)) if dtype == "bf16" else (lambda x: x.astype(np.float32))
    K, V = [], []
    for c in ctx:
        k = rng.standard_normal((c, Hkv, D))
        if SCENES[scene]:
            on = np.flatnonzero(seen(c - 1, c, window, sinks))
            for where, height in SCENES[scene]:
                at = min(1, c - 1) if where < 0 else on[int(where * len(on))]
                k[at] = sign * height * u / 2
        K.append(store(k))
        V.append(store(rng.standard_normal((c, Hkv, D))))
    q = rng.standard_normal((rows, H, D))
    return K, V, store(q + 2 * u if SCENES[scene] else 16 * q)


def _rig(dtype, H, Hkv, D, bs, ctx, scale):
    geom = W.Geometry(1, H, Hkv, D, bs, sum((c + bs - 1) // bs for c in ctx) + 2, max((c + bs - 1) // bs for c in ctx), dtype)
    rig = Rig(geom, len(ctx), scale=scale)
    table, _ = W.deal_block_table(W.permutation(11, geom.num_blocks), ctx, geom)
    return geom, rig, table


def _close(got, q, K, V, p, window, sinks, scale, dtype, rounded, what):
    """One row, [H][D], against 64 bits.  A score is a sum of D products in 32 bits, at most 12 roundings deep, times the scale (a rounding of the scale and two
    of log2 e come on top), less the reference: off by 16 2^-24 of the sum of the sizes of its products, which is a relative error of the weight; sums of
    weights and of values and the exponential as in test_gpu_window, 6e-5; half a step of bf16 for the output, and for weights that are
    rounded to it once for each and once for their sum."""
    on = seen(p, K.shape[0], window, sinks)
    k, v = K[on], V[on]
    G = q.shape[0] // K.shape[1]
    for g in range(K.shape[1]):
        x = q[g * G:(g + 1) * G]
        s = x @ k[:, g].T * scale
        reach = (np.abs(x) @ np.abs(k[:, g]).T).max(1, keepdims=True) * abs(scale)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        ref, size = w @ v[:, g], w @ np.abs(v[:, g]) + np.abs(w @ v[:, g])
        bound = (6e-5 + 16 * 2.0 ** -24 * reach + (STEP if rounded else 0.0)) * size + 1e-6
        if dtype == "bf16":
            bound = bound + STEP * np.abs(ref)
        off = np.abs(got[g * G:(g + 1) * G] - ref) - bound
        assert off.max() <= 0, (what, p, g, off.max())


@pytest.mark.parametrize("scene", SCENES)
@pytest.mark.parametrize("form", FORMS)
def test_prefill(form, scene):
    dtype, H, Hkv, D, bs, reqs, window, sinks = FORMS[form]
    ctx, total, rows = [c for c, _ in reqs], sum(n for _, n in reqs), form.startswith("rows")
    start = np.concatenate([[0], np.cumsum([n for _, n in reqs])])
    for factor in SCALES:
        scale = float(np.float32(factor / np.sqrt(D)))
        geom, rig, table = _rig(dtype, H, Hkv, D, bs, ctx, scale)
        K, V, q = _made(dtype, H, Hkv, D, ctx, total, scene, np.sign(factor), window, sinks, 5, geom)
        rig.page_requests(0, table, K, V)
        dev = rig.dev
        out = torch.zeros((total, H, D), dtype=rig.tdtype, device=dev)
        args = n2t(q, dev), torch.tensor(start, dtype=torch.int32, device=dev), torch.as_tensor(table, device=dev), torch.tensor(ctx, dtype=torch.int32, device=dev)
        torch.cuda.synchronize()
        rig.lamps.prefill_attn_window(0, len(reqs), total, window, sinks, *args, out, max_new_tokens=-1 if rows else max(n for _, n in reqs))
        torch.cuda.synchronize()
        got = to_f64(out)
        for r, (c, n) in enumerate(reqs):
            kd, vd, qd = f64(K[r]), f64(V[r]), f64(q[start[r]:start[r + 1]])
            for i in [i for i in range(n) if n <= 40 or i % max(1, n // 24) == 0 or n - i < 5]:
                _close(got[start[r] + i], qd[i], kd, vd, c - n + i, window, sinks, scale, dtype, dtype == "bf16" and not rows, (factor, r))
        rig.close()


@pytest.mark.parametrize("scene", SCENES)
@pytest.mark.parametrize("form", DECODE)
def test_decode(form, scene):
    dtype, H, Hkv, D, bs, ctx, window, sinks = DECODE[form]
    for factor in SCALES:
        scale = float(np.float32(factor / np.sqrt(D)))
        geom, rig, table = _rig(dtype, H, Hkv, D, bs, ctx, scale)
        K, V, q = _made(dtype, H, Hkv, D, ctx, len(ctx), scene, np.sign(factor), window, sinks, 7, geom)
        rig.page_requests(0, table, K, V)
        dev = rig.dev
        out = torch.zeros((len(ctx), H, D), dtype=rig.tdtype, device=dev)
        args = n2t(q, dev), torch.as_tensor(table, device=dev), torch.tensor(ctx, dtype=torch.int32, device=dev), torch.ones(len(ctx), dtype=torch.uint8, device=dev)
        torch.cuda.synchronize()
        rig.lamps.decode_attn_window(0, len(ctx), window, sinks, *args, out)
        torch.cuda.synchronize()
        got = to_f64(out)
        for r, c in enumerate(ctx):
            _close(got[r], f64(q[r]), f64(K[r]), f64(V[r]), c - 1, window, sinks, scale, dtype, False, (factor, r))
        rig.close()
