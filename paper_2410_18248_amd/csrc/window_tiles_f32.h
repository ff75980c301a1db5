// Windowed attention of many new tokens on the fp32 matrix instruction.  Device code; part of window_attn.hip.
#pragma once

// One workgroup = one (request, heads of a pass, tile of new tokens): 16 columns, (new token, head) pairs of one kv head, as in prefill_tiles_f32, whose
// operands and sums (MfmaF32Tile) these are; its four waves take every fourth of the units that the tile's tokens see and add their states up in LDS.
// Units that some column does not see whole are masked, and values there that are no finite numbers kept from the columns that do not see them.
// In large launches with short walks a wave has a tile of its own.
// Bound by the walk on short prompts (6 of 17 to 700 tokens, 8 heads of 64, window 100: 16 us, 4 of them bytes), by keys and values out of L2 on long ones: a wave
// loads a unit's for its own 16 columns alone, 8 flops a byte at head size 128.  4 of 700 tokens on 500, 32 / 8 heads, 173 us under a window of 250 and 481 under one of
// everything, 0.44 and 0.53 of the fp32 matrix rate; 16 of 700, 8 heads of 64, window 250, 97, 0.39.
template <int DIM>
struct WindowF32Tile : MfmaF32Tile<DIM> {
    typedef MfmaF32Tile<DIM> Base;
    typedef typename Base::State State;
    typedef typename Base::vvec vvec;
    using Base::D, Base::NK, Base::VW, Base::NC;

    // Every `stride`-th unit of `see` from u0 on.  q: the row of the lane's column (nullptr: none), at position pos (-1); the tile's tokens are at p_first ..
    // p_last.
    static __device__ __forceinline__ void reduce(const DecodeArgs &a, int r, int g, const float *q, int pos, int p_first, int p_last, int window, int sinks,
                                                  const Sight<16> &see, int u0, int stride, State &st)
    {
        const int lane = threadIdx.x & 63, j = lane & 15, qd = lane >> 4;
        f32x4 qb[NK];
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            qb[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (q) qb[i] = *reinterpret_cast<const f32x4 *>(q + 16 * i + 4 * qd);
        }
        float m = kLeast, l = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int v = 0; v < VW; ++v) st.o[c][v] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int n = (see.units - u0 + stride - 1) / stride;
        const int32_t *table = a.block_table + (size_t)r * a.max_blocks;
        const size_t tile = (size_t)a.block_size * D, block_stride = (size_t)a.num_layers * a.num_kv_heads * tile;
        const size_t head_off = ((size_t)a.layer * a.num_kv_heads + g) * tile;
        const float *kp = static_cast<const float *>(a.k_pool) + head_off + j * D + 4 * qd;
        const float *vp = static_cast<const float *>(a.v_pool) + head_off + 4 * qd * D + VW * j;
        const auto place = [&](int c) { return see.at(u0 + min(c, n - 1) * stride); };
        const auto entry = [&](int c) -> int { return table[place(c) >> a.log2_block_size]; };
        const auto issue = [&](int c, int block, f32x4 (&kx)[NK], vvec (&vx)[4][NC]) {
            // (an entry that names no block of the pool reads the last one; the rows are meaningless)
            const size_t off = (size_t)min((unsigned)block, (unsigned)a.num_blocks - 1) * block_stride + (size_t)(place(c) & (a.block_size - 1)) * D;
#pragma unroll
            for (int i = 0; i < NK; ++i) kx[i] = *reinterpret_cast<const f32x4 *>(kp + off + 16 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int c2 = 0; c2 < NC; ++c2) vx[e][c2] = *reinterpret_cast<const vvec *>(vp + off + e * D + 16 * VW * c2);
        };
        const auto visible = [&](int p, int t) { return (t <= p) & ((t > p - window) | (t < sinks)); };
        const int hi = p_last - window + 1;
        const auto consume = [&](int c, f32x4 (&kx)[NK], vvec (&vx)[4][NC]) {
            __builtin_amdgcn_sched_barrier(0);        // (the loads above stay above what waits for the ones before them)
            const int t0 = place(c);
            const bool masked = (t0 + 15 > p_first) | ((t0 < hi) & (t0 + 16 > sinks));   // uniform
            f32x4 p8[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p8[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NK; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f32x4 &x = p8[4 * (i & 1) + e];
                    x = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[i][e], qb[i][e], x, 0, 0, 0);
                }
            float s[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[e] = (((p8[0][e] + p8[1][e]) + (p8[2][e] + p8[3][e])) + ((p8[4][e] + p8[5][e]) + (p8[6][e] + p8[7][e]))) * a.scale_log2e;
#pragma unroll
            for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(s[e]));
            bool wild = false;                        // uniform: a value that not every column sees is no finite number
            if (masked) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!visible(pos, t0 + 4 * qd + e)) s[e] = -INFINITY;
                float z = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c2 = 0; c2 < NC; ++c2)
#pragma unroll
                        for (int v = 0; v < VW; ++v) z = fmaf(vx[e][c2][v], 0.0f, z);
                wild = __any(z != 0.0f);              // (NaN)
            }
            float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float mn = fmaxf(m, mx), sc = fast_exp2(m - mn);
            m = mn;
            float ps = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[e] = fast_exp2(s[e] - mn);
                ps += s[e];
            }
            l = l * sc + ps;
            if (!wild) {
#pragma unroll
                for (int c2 = 0; c2 < NC; ++c2)
#pragma unroll
                    for (int v = 0; v < VW; ++v) {
                        f32x4 t[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            t[e >> 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(vx[e][c2][v], s[e], t[e >> 1], 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) st.o[c2][v][e] = fmaf(st.o[c2][v][e], sc, t[0][e] + t[1][e]);
                    }
            } else {                                  // once per token, what it does not see zeroed, kept by its columns (summed as above)
#pragma unroll
                for (int c2 = 0; c2 < NC; ++c2)
#pragma unroll
                    for (int v = 0; v < VW; ++v) {
                        f32x4 kept = {0.f, 0.f, 0.f, 0.f};
                        for (int p = p_first; p <= p_last; ++p) {
                            f32x4 t[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                t[e >> 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(visible(p, t0 + 4 * qd + e) ? vx[e][c2][v] : 0.0f, s[e], t[e >> 1], 0, 0, 0);
                            if (pos == p) kept = t[0] + t[1];
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) st.o[c2][v][e] = fmaf(st.o[c2][v][e], sc, kept[e]);
                    }
            }
        };
        if (n > 0) {
            f32x4 ka[NK], kb[NK];
            vvec va[4][NC], vb[4][NC];
            int c = 0, e1, e2;
            if ((n & 1) == 0) {                       // the last one is to be one that `ka` holds
                const int e0 = entry(0);
                e1 = entry(1);
                issue(0, e0, kb, vb);
                issue(1, e1, ka, va);
                e1 = entry(2);
                e2 = entry(3);
                consume(0, kb, vb);
                c = 1;
            } else {
                issue(0, entry(0), ka, va);
                e1 = entry(1);
                e2 = entry(2);
            }
            for (; c + 1 < n; c += 2) {
                issue(c + 1, e1, kb, vb);
                e1 = entry(c + 3);
                consume(c, ka, va);
                issue(c + 2, e2, ka, va);
                e2 = entry(c + 4);
                consume(c + 1, kb, vb);
            }
            consume(c, ka, va);
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        st.m = m;
        st.l = l;
    }
};

// Heads of a group that share a tile: the largest divisor up to 16.
__host__ __device__ __forceinline__ int f32_heads(int group)
{
    int gh = group < 16 ? group : 16;
    while (group % gh) --gh;
    return gh;
}

// ALONE: a wave has a tile of its own, and no sum to make.
template <int D, bool ALONE>
__global__ __launch_bounds__(kThreads, D == 128 ? 2 : 1) void window_tiles_f32(const WindowArgs w)
{
    typedef WindowF32Tile<D> R;
    constexpr int ROW = D + 4;                        // floats; 16-byte aligned, rows in different banks
    const DecodeArgs &a = w.d;
    const int G = a.num_q_heads / a.num_kv_heads, GH = f32_heads(G), passes = G / GH, TW = 16 / GH;
    const int lane = threadIdx.x & 63, j = lane & 15, qd = lane >> 4, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    TileAt at;
    const unsigned all = (unsigned)w.items * (unsigned)(a.num_kv_heads * passes), per = ((all + kWaves - 1) / kWaves + 7) / 8;   // ALONE: workgroups to an XCD
    const unsigned mine = ((blockIdx.x & 7) * per + (blockIdx.x >> 3)) * kWaves + wv;
    if (!tile_at(w, TW, at, !ALONE ? tile_item(w, blockIdx.x, a.num_kv_heads * passes) : blockIdx.x >> 3 < per && mine < all ? (int)mine : -1)) return;
    const int g = at.g / passes, h0 = at.g * GH, base_pos = at.ctx - at.n_new, n_new = min(at.n_new, w.total_tokens - at.first);
    const int toks = min(TW, n_new - at.tile * TW), tok = j / GH;   // this lane's column: token tile * TW + tok, head h0 + j % GH
    const bool ok = tok < toks;
    const int p_first = base_pos + at.tile * TW, p_last = p_first + toks - 1;
    const float *q = static_cast<const float *>(a.q) + ((size_t)(at.first + at.tile * TW + tok) * a.num_q_heads + h0 + j % GH) * D;
    const Sight<16> see(p_last + 1, max(0, p_first - w.window + 1), w.sinks, std::true_type{});
    typename R::State st;
    R::reduce(a, at.r, g, ok ? q : nullptr, ok ? p_first + tok : -1, p_first, p_last, w.window, w.sinks, see, ALONE ? 0 : wv, ALONE ? 1 : kWaves, st);
    if constexpr (ALONE) {
        if (!ok) return;
        const float inv = 1.0f / st.l;
        float *out = static_cast<float *>(a.out) + (q - static_cast<const float *>(a.q));
#pragma unroll
        for (int c = 0; c < R::NC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                typename R::vvec x;
#pragma unroll
                for (int v = 0; v < R::VW; ++v) x[v] = st.o[c][v][e] * inv;
                *reinterpret_cast<typename R::vvec *>(out + 16 * R::VW * c + R::VW * (4 * qd + e)) = x;
            }
        return;
    }
    __shared__ __align__(16) float part[kWaves][16][ROW];
    __shared__ float2 stat[kWaves][16];
    if (qd == 0) stat[wv][j] = make_float2(st.m, st.l);
#pragma unroll
    for (int c = 0; c < R::NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int v = 0; v < R::VW; ++v) part[wv][j][16 * R::VW * c + R::VW * (4 * qd + e) + v] = st.o[c][v][e];
    __syncthreads();
    const int col = threadIdx.x >> 4, x = threadIdx.x & 15, t = col / GH;
    if (t >= toks) return;
    float M = kLeast, L = 0.0f, f[kWaves];
#pragma unroll
    for (int k = 0; k < kWaves; ++k) M = fmaxf(M, stat[k][col].x);
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        f[k] = fast_exp2(stat[k][col].x - M);
        L += stat[k][col].y * f[k];
    }
    const float inv = 1.0f / L;
    float *out = static_cast<float *>(a.out) + ((size_t)(at.first + at.tile * TW + t) * a.num_q_heads + h0 + col % GH) * D;
    for (int d = 4 * x; d < D; d += 64) {
        f32x4 A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const f32x4 o = *reinterpret_cast<const f32x4 *>(&part[k][col][d]);
#pragma unroll
            for (int e = 0; e < 4; ++e) A[e] += o[e] * f[k];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) A[e] *= inv;
        *reinterpret_cast<f32x4 *>(out + d) = A;
    }
}
