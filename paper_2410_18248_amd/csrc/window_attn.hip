// Attention over the last `window` positions of a request's cache and its first `sinks`: decode and many new tokens.
//
//   out = softmax(q K^T * scale) V  over the positions t < end with t >= lo or t < sinks,  lo = end - window
//
// for the new token at position end - 1.  What this leaves of a long context is two short stretches, so the work of a call is bounded by what the
// host knows: ranges of about the same size, and no more of them cut than the chip needs.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attn_reducers.h"
#include "handover.h"
#include "internal.h"
#include "requests.h"
#include "tile_parts.h"

namespace lamps {
namespace {

// ---------------------------------------------------------------- what a token sees

// A state without a position is (kLeast, 0, 0).  A row of no positions is zero; one whose weights are not numbers is none either.
__device__ __forceinline__ float reciprocal(float L, bool none) { return none ? 0.0f : 1.0f / L; }

// ---------------------------------------------------------------- vector ALUs

// One wavefront reduces units u0 .. u1 - 1 of a token's sight (plain layout): as ValuReducer, whose loads these are, with a place for each
// unit and a mask where a unit is seen in part.
template <bool BF16, int LPT, int GH, int NH>
struct WindowValu : ValuReducer<BF16, LPT, GH, NH> {
    typedef ValuReducer<BF16, LPT, GH, NH> Base;
    using Base::VEC, Base::D, Base::ES, Base::TPW, Base::kLoads, Base::HT, Base::NL;
    static constexpr int U = HT;

    template <typename Sink>
    static __device__ __forceinline__ void run(const DecodeArgs &a, int r, size_t qrow, int g, int h0, int, const Sight<U> &see, int u0, int u1, Sink sink)
    {
        const int lane = threadIdx.x & 63, row = lane / LPT, col = lane % LPT;
        uint4 qv[GH];
#pragma unroll
        for (int h = 0; h < GH; ++h)
            qv[h] = *reinterpret_cast<const uint4 *>(static_cast<const char *>(a.q) + ((qrow * a.num_q_heads + h0 + h) * D + col * VEC) * ES);
        float m[GH], l[GH], acc[GH][VEC];
#pragma unroll
        for (int h = 0; h < GH; ++h) {
            m[h] = kLeast;
            l[h] = 0.0f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[h][e] = 0.0f;
        }
        const int32_t *table = a.block_table + (size_t)r * a.max_blocks;
        const size_t tile_bytes = (size_t)a.block_size * D * ES, block_stride = (size_t)a.num_layers * a.num_kv_heads * tile_bytes;
        const size_t head_off = ((size_t)a.layer * a.num_kv_heads + g) * tile_bytes;
        const char *kp = static_cast<const char *>(a.k_pool) + head_off + lane * 16;
        const char *vp = static_cast<const char *>(a.v_pool) + head_off + lane * 16;
        int pb[NH], pbn[NH];
#pragma unroll
        for (int f = 0; f < NH; ++f) pb[f] = u0 + f < u1 ? table[see.at(u0 + f) >> a.log2_block_size] : -1;
        for (int u = u0; u < u1; u += NH) {
            uint4 kx[NL], vx[NL];
            int t0[NH];
#pragma unroll
            for (int f = 0; f < NH; ++f) {
                t0[f] = see.at(u + f);
                // (uniform; an entry that names no block of the pool reads nothing: its positions are zeros, the row is meaningless)
                const bool in = (unsigned)pb[f] < (unsigned)a.num_blocks;
                const size_t off = (size_t)(in ? pb[f] : 0) * block_stride + (size_t)(t0[f] & (a.block_size - 1)) * D * ES;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) kx[f * kLoads + i] = in ? load_stream16(kp + off + i * 1024) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) vx[f * kLoads + i] = in ? load_stream16(vp + off + i * 1024) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int f = 0; f < NH; ++f) pbn[f] = u + NH + f < u1 ? table[see.at(u + NH + f) >> a.log2_block_size] : -1;
            float s[GH][NL];
#pragma unroll
            for (int h = 0; h < GH; ++h)
#pragma unroll
                for (int i = 0; i < NL; ++i) s[h][i] = sum_token_lanes<LPT>(dot16<BF16>(qv[h], kx[i])) * a.scale_log2e;
#pragma unroll
            for (int f = 0; f < NH; ++f)
                if (u + f >= u1 || !see.sees_all(t0[f])) {   // uniform
#pragma unroll
                    for (int i = 0; i < kLoads; ++i)
                        if (u + f >= u1 || !see.sees(t0[f] + i * TPW + row)) {
#pragma unroll
                            for (int h = 0; h < GH; ++h) s[h][f * kLoads + i] = -INFINITY;
                            vx[f * kLoads + i] = make_uint4(0, 0, 0, 0);
                        }
                }
#pragma unroll
            for (int h = 0; h < GH; ++h) {
                float mn = m[h];
#pragma unroll
                for (int i = 0; i < NL; ++i) mn = fmaxf(mn, s[h][i]);
                const float sc = fast_exp2(m[h] - mn);
                float ps = 0.0f;
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    s[h][i] = fast_exp2(s[h][i] - mn);
                    ps += s[h][i];
                }
                l[h] = l[h] * sc + ps;
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[h][e] *= sc;
                m[h] = mn;
            }
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                float vf[VEC];
                unpack<BF16, VEC>(vx[i], vf);
#pragma unroll
                for (int h = 0; h < GH; ++h)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[h][e] = fmaf(s[h][i], vf[e], acc[h][e]);
            }
#pragma unroll
            for (int f = 0; f < NH; ++f) pb[f] = pbn[f];
        }
#pragma unroll
        for (int h = 0; h < GH; ++h) {
#pragma unroll
            for (int stride = LPT; stride < 64; stride *= 2) {
                const float mo = __shfl_xor(m[h], stride), lo = __shfl_xor(l[h], stride);
                float ao[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) ao[e] = __shfl_xor(acc[h][e], stride);
                merge_state<VEC>(m[h], l[h], acc[h], mo, lo, ao);
            }
            if (row == 0) sink(h, col * VEC, m[h], l[h], acc[h]);
        }
    }
};

// ---------------------------------------------------------------- matrix cores

// As MfmaReducer (bf16, tiled layout, up to 16 heads of a group), with a place for each sub-tile and a mask where one is seen in part.
template <int DIM>
struct WindowMfma : MfmaReducer<DIM> {
    typedef MfmaReducer<DIM> Base;
    using Base::D, Base::NK, Base::NS;
    static constexpr int U = 16;

    template <typename Sink>
    static __device__ __forceinline__ void run(const DecodeArgs &a, int r, size_t qrow, int g, int h0, int heads, const Sight<U> &see, int u0, int u1, Sink sink)
    {
        const int lane = threadIdx.x & 63, j = lane & 15, qd = lane >> 4;
        bf16x8 qb[NK];
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            uint4 t = make_uint4(0, 0, 0, 0);
            if (j < heads)
                t = *reinterpret_cast<const uint4 *>(static_cast<const char *>(a.q) + ((qrow * a.num_q_heads + h0 + j) * D + 32 * i + 8 * qd) * 2);
            qb[i] = __builtin_bit_cast(bf16x8, t);
        }
        float m = kLeast, l = 0.0f;
        f32x4 o[2 * NS];
#pragma unroll
        for (int s = 0; s < 2 * NS; ++s) o[s] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int n = u1 - u0;
        const int32_t *table = a.block_table + (size_t)r * a.max_blocks;
        const size_t tile_bytes = (size_t)a.block_size * D * 2, block_stride = (size_t)a.num_layers * a.num_kv_heads * tile_bytes;
        const size_t head_off = ((size_t)a.layer * a.num_kv_heads + g) * tile_bytes;
        const char *kp = static_cast<const char *>(a.k_pool) + head_off + lane * 16;
        const char *vp = static_cast<const char *>(a.v_pool) + head_off + lane * 16;
        const auto place = [&](int c) { return see.at(u0 + min(c, n - 1)); };
        const auto entry = [&](int c) -> int { return table[place(c) >> a.log2_block_size]; };
        const auto issue = [&](int c, int block, uint4 (&kx)[NK], uint4 (&vx)[NS]) {
            // (an entry that names no block of the pool reads the last one; the row is meaningless)
            const size_t off = (size_t)min((unsigned)block, (unsigned)a.num_blocks - 1) * block_stride +
                               (size_t)((place(c) & (a.block_size - 1)) >> 4) * (16 * D * 2);
#pragma unroll
            for (int i = 0; i < NK; ++i) kx[i] = load_stream16(kp + off + i * 1024);
#pragma unroll
            for (int i = 0; i < NS; ++i) vx[i] = load_stream16(vp + off + i * 1024);
        };
        const auto consume = [&](int c, uint4 (&kx)[NK], uint4 (&vx)[NS]) {
            __builtin_amdgcn_sched_barrier(0);     // (the loads above stay above what waits for the ones before them)
            const int t0 = place(c);
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NK; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kx[i]), qb[i], s, 0, 0, 0);
            // The scores are taken out of the matrix cores in front of the branch.  Where two ways lead from a product to the first use of its
            // result, the compiler counts the instructions of one of them only, and by the shorter one the result was not there yet: rows
            // wrong by a tenth, where the condition below was two branches.
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] *= a.scale_log2e;
            asm volatile("" : "+v"(s));
            if (!see.sees_all(t0)) {               // uniform
                bool on[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    on[e] = see.sees(t0 + 4 * qd + e);
                    if (!on[e]) s[e] = -INFINITY;
                }
                const uint32_t m01 = (on[0] ? 0x0000FFFFu : 0u) | (on[1] ? 0xFFFF0000u : 0u), m23 = (on[2] ? 0x0000FFFFu : 0u) | (on[3] ? 0xFFFF0000u : 0u);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    vx[i].x &= m01; vx[i].z &= m01;
                    vx[i].y &= m23; vx[i].w &= m23;
                }
            }
            float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float mn = fmaxf(m, mx), sc = fast_exp2(m - mn);
            m = mn;
            float p[4], ps = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[e] = fast_exp2(s[e] - mn);
                ps += p[e];
            }
            l = l * sc + ps;
            // the weights as pairs, the high part and what it leaves: fp32's accuracy for a second, nearly free, product
            union { s16x4 v; uint16_t u[4]; } ph, pl;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ph.u[e] = to_bf16_rne(p[e]);
                pl.u[e] = to_bf16_rne(p[e] - __uint_as_float((uint32_t)ph.u[e] << 16));
            }
#pragma unroll
            for (int x = 0; x < 2 * NS; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[x][e] *= sc;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                union { uint2 u; s16x4 v; } a0, a1;
                a0.u = make_uint2(vx[i].x, vx[i].y);
                a1.u = make_uint2(vx[i].z, vx[i].w);
                o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a0.v, ph.v, o[2 * i], 0, 0, 0);
                o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a0.v, pl.v, o[2 * i], 0, 0, 0);
                o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a1.v, ph.v, o[2 * i + 1], 0, 0, 0);
                o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a1.v, pl.v, o[2 * i + 1], 0, 0, 0);
            }
        };
        if (n > 0) {
            uint4 ka[NK], va[NS], kb[NK], vb[NS];
            int c = 0, e1, e2;
            if ((n & 1) == 0) {                    // the last one is to be one that `ka` holds
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
        if (j < heads) {
#pragma unroll
            for (int x = 0; x < 2 * NS; ++x) {
                const float A[4] = {o[x][0], o[x][1], o[x][2], o[x][3]};
                sink(j, 16 * x + 4 * qd, m, l, A);
            }
        }
    }
};

// N outputs, element i and up, times inv
template <bool BF16, int N>
__device__ __forceinline__ void put_out(void *out, size_t i, float inv, const float (&A)[N])
{
    float o[N];
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = A[e] * inv;
    if constexpr (BF16) {
        uint32_t w[N / 2];
#pragma unroll
        for (int e = 0; e < N; e += 2) w[e / 2] = pack_bf16(o[e], o[e + 1]);
        uint16_t *at = static_cast<uint16_t *>(out) + i;
        if constexpr (N == 2) *reinterpret_cast<uint32_t *>(at) = w[0];
        if constexpr (N == 4) *reinterpret_cast<uint2 *>(at) = make_uint2(w[0], w[1]);
        if constexpr (N == 8) *reinterpret_cast<uint4 *>(at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int e = 0; e < N; e += 2) *reinterpret_cast<float2 *>(static_cast<float *>(out) + i + e) = make_float2(o[e], o[e + 1]);
    }
}

// ---------------------------------------------------------------- one new token per request

// A workgroup takes a range, one (request, kv head / pass), or one of the parts of it that the host has counted: its waves a stretch of the units each,
// added up in LDS.  Parts leave their states to a second launch.  Bound by memory where the launch is large (230 of 256 requests on 32 / 8 heads of 128, window 1 024:
// 89 us, 5.7 TB/s; 51 of 64 on 32 plain heads, 2 048: 184 us, 5.9 TB/s), otherwise by the round trips
// of one walk: length, table entries, K / V, the sum (one request, window 1 024: 5.6 us, and 3.1 of adding the parts up).
template <typename R>
__global__ __launch_bounds__(kThreads, R::kLeastPerCu) void window_decode(const WindowArgs w)
{
    constexpr int D = R::D;
    extern __shared__ __align__(16) float states[];   // [wave][head][D + 2]
    const DecodeArgs &a = w.d;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int GH = a.heads_per_pass, HC = a.num_kv_heads * a.passes;
    const int item = blockIdx.x, part = item / (HC * a.batch), range = item - part * HC * a.batch;
    const int r = range / HC, hc = range - r * HC, h0 = hc * GH;
    const int running = a.running[r], C = ctx_len(a, r);
    if (!running) return;
    const Sight<R::U> see(C, w.window, w.sinks);
    const int each = (see.units + w.parts - 1) / w.parts, p0 = min(see.units, part * each), p1 = min(see.units, p0 + each);
    const int per = (p1 - p0 + kWaves - 1) / kWaves, u0 = min(p1, p0 + wv * per);
    R::run(a, r, (size_t)r, hc / a.passes, h0, GH, see, u0, min(p1, u0 + per),
           [&](int h, int d, float M, float L, const auto &A) { store_partial(states + (size_t)(wv * GH + h) * (D + 2), D, d, M, L, A); });
    __syncthreads();
    for (int i = 2 * (64 * wv + lane); i < GH * D; i += 128 * kWaves) {
        const int h = i / D, d = i % D;
        const float *x = states + h * (D + 2);
        float M = kLeast, L = 0.0f, A[2] = {0.0f, 0.0f};
        float2 ml[kWaves];
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            ml[k] = *reinterpret_cast<const float2 *>(x + k * GH * (D + 2) + D);
            M = fmaxf(M, ml[k].x);
        }
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const float f = fast_exp2(ml[k].x - M);
            const float2 o = *reinterpret_cast<const float2 *>(x + k * GH * (D + 2) + d);
            L += ml[k].y * f;
            A[0] += o.x * f;
            A[1] += o.y * f;
        }
        if (w.parts == 1) put_out<R::kBF16>(a.out, ((size_t)r * a.num_q_heads + h0 + h) * D + d, reciprocal(L, see.units == 0), A);
        else store_partial(a.partials + (((size_t)range * w.parts + part) * GH + h) * (D + 2), D, d, M, L, A);
    }
}

// Adds the parts of a range up: 128 (head, dim) outputs a workgroup, two per lane, its waves every eighth part.
constexpr int kMergeWaves = 8, kMostParts = 64;
template <bool BF16>
__global__ __launch_bounds__(64 * kMergeWaves) void window_merge(const WindowArgs w)
{
    constexpr int N = kMostParts / kMergeWaves;
    __shared__ float4 sums[kMergeWaves][64];
    const DecodeArgs &a = w.d;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int D = a.head_dim, GH = a.heads_per_pass, HC = a.num_kv_heads * a.passes;
    const int range = blockIdx.x, r = range / HC, hc = range - r * HC;
    const int idx = min((int)blockIdx.y * 128 + 2 * lane, GH * D - 2), h = idx / D, d = idx - h * D;
    float2 ml[N], ao[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        ml[k] = make_float2(kLeast, 0.0f);
        ao[k] = make_float2(0.0f, 0.0f);
        const int part = wv + kMergeWaves * k;
        if (part < w.parts) {
            const float2 *x = reinterpret_cast<const float2 *>(a.partials + (((size_t)range * w.parts + part) * GH + h) * (D + 2));
            ml[k] = x[D / 2];
            ao[k] = x[d / 2];
        }
    }
    if (!a.running[r]) return;                        // (nothing was written)
    const bool none = a.ctx_lens[r] <= 0;
    float M = kLeast, L = 0.0f, A[2] = {0.0f, 0.0f};
    const auto add = [&](float m, float l, float x, float y) {
        const float Mn = fmaxf(M, m), f0 = fast_exp2(M - Mn), f = fast_exp2(m - Mn);
        L = L * f0 + l * f;
        A[0] = A[0] * f0 + x * f;
        A[1] = A[1] * f0 + y * f;
        M = Mn;
    };
#pragma unroll
    for (int k = 0; k < N; ++k) add(ml[k].x, ml[k].y, ao[k].x, ao[k].y);
    sums[wv][lane] = make_float4(M, L, A[0], A[1]);
    __syncthreads();
    if (wv > 0) return;
#pragma unroll
    for (int k = 1; k < kMergeWaves; ++k) {
        const float4 o = sums[k][lane];
        add(o.x, o.y, o.z, o.w);
    }
    if (blockIdx.y * 128 + 2 * lane < GH * D) put_out<BF16>(a.out, ((size_t)r * a.num_q_heads + hc * GH + h) * D + d, reciprocal(L, none), A);
}

// ---------------------------------------------------------------- many new tokens: a wavefront per token

template <typename R>
__global__ __launch_bounds__(kThreads) void window_rows(const WindowArgs w)
{
    constexpr int D = R::D;
    const DecodeArgs &a = w.d;
    const int GH = a.heads_per_pass, HC = a.num_kv_heads * a.passes;
    const long long item = (long long)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= (long long)w.total_tokens * HC) return;
    const int n = (int)(item / HC), hc = (int)(item - (long long)n * HC), h0 = hc * GH;
    const auto [r, first, count, ctx] = new_tokens_at(w.q_start, a.ctx_lens, a.batch, n, [](int q, int) { return q; });
    // (a context shorter than its new tokens, or longer than the table row: nothing is read or written)
    if (n < first || n >= first + count || ctx < count || ctx > a.max_blocks * a.block_size) return;
    const Sight<R::U> see(ctx - count + (n - first) + 1, w.window, w.sinks);
    R::run(a, r, (size_t)n, hc / a.passes, h0, GH, see, 0, see.units, [&](int h, int d, float, float L, const auto &A) {
        put_out<R::kBF16>(a.out, ((size_t)n * a.num_q_heads + h0 + h) * D + d, reciprocal(L, false), A);
    });
}

#include "window_tiles.h"
#include "window_tiles_f32.h"

// ---------------------------------------------------------------- launches

// Positions that the sight of one token can have: of `span` tokens together so many more.
long long most_positions(const WindowArgs &w, int unit)
{
    const long long row = (long long)w.d.max_blocks * w.d.block_size;
    return std::min(row, (long long)w.window + w.sinks + 2 * unit);
}

// Parts of a range: as many as give every wave of the chip a walk, but two units to a wave at least, or the sum is longer than the walk; none where a workgroup's own walk
// is about as long as the way through a second launch (one request, window 256, 32 / 8 heads of 128: 5.9 us whole, 9.2 in two parts; 1 024 9.0 in eight parts,
// 9.1 in four).
template <typename R>
int count_parts(const WindowArgs &w)
{
    const DecodeArgs &a = w.d;
    const long long ranges = (long long)a.batch * a.num_kv_heads * a.passes, units = most_positions(w, R::U) / R::U;
    if (units <= 9 * kWaves) return 1;
    const long long chip = 256LL * std::min(R::kMostPerCu, 4);
    const size_t state = (size_t)a.heads_per_pass * (a.head_dim + 2) * sizeof(float);
    long long parts = std::min(chip / ranges, units / (2 * kWaves));
    parts = std::min(parts, (long long)(a.partial_capacity / (state * ranges)));
    return (int)std::max(1LL, std::min(parts, (long long)kMostParts));
}

template <typename R>
hipError_t launch_one(WindowArgs w, hipStream_t s)
{
    const DecodeArgs &a = w.d;
    const long long ranges = (long long)a.batch * a.num_kv_heads * a.passes;
    if (w.q_start) {
        const long long items = (long long)w.total_tokens * a.num_kv_heads * a.passes;
        if (items > 0x7fffffffLL * kWaves) return hipErrorInvalidValue;
        hipLaunchKernelGGL(window_rows<R>, dim3((unsigned)((items + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, w);
        return hipGetLastError();
    }
    w.parts = count_parts<R>(w);
    if (ranges * w.parts > 0x7fffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL(window_decode<R>, dim3((unsigned)(ranges * w.parts)), dim3(kThreads), (size_t)kWaves * a.heads_per_pass * (R::D + 2) * sizeof(float), s, w);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || w.parts == 1) return e;
    hipLaunchKernelGGL(window_merge<R::kBF16>, dim3((unsigned)ranges, (unsigned)((a.heads_per_pass * a.head_dim + 127) / 128)), dim3(64 * kMergeWaves), 0, s, w);
    return hipGetLastError();
}

template <int D, bool TILED, int kCB>
hipError_t launch_tiles(WindowArgs w, hipStream_t s)
{
    const DecodeArgs &a = w.d;
    const int WT = kWaves * (16 * kCB / (a.num_q_heads / a.num_kv_heads));
    const long long items = (long long)w.total_tokens / WT + a.batch, tiles = items * a.num_kv_heads;
    const long long stages = (std::min((long long)a.max_blocks * a.block_size, (long long)w.window + w.sinks + WT) + 31) / 32 + 1;
    const long long state = (long long)tile_state_floats(D, kWaves * 16 * kCB) * (long long)sizeof(float);
    // Two workgroups fit a CU, 512 the chip: with half as many parts more 12 responses of 4 to 64 tokens, window 2 048, took 46 us, 40 so, and one prompt of 2 000 (504
    // tiles) in two 55 us, 31 whole.  Four stages at least to a part: a part's way to its first product is as long as four.
    // (about as many tiles as there are: half of the requests' last ones are there besides the full ones)
    const long long there = std::max(1LL, ((long long)w.total_tokens / WT + a.batch / 2) * a.num_kv_heads);
    long long parts = std::min(512 / there, stages / 4);
    parts = std::max(1LL, std::min({parts, (long long)kMostParts, (long long)a.partial_capacity / ((state + 8) * tiles)}));
    const long long grid = (tiles * parts + 7) / 8 * 8, join = (tiles + 7) / 8 * 8;
    if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
    w.items = (int)items;
    w.parts = (int)parts;
    if (parts == 1) {
        hipLaunchKernelGGL((window_tiles<D, TILED, kCB, false>), dim3((unsigned)grid), dim3(kThreads), 0, s, w);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((window_tiles<D, TILED, kCB, true>), dim3((unsigned)grid), dim3(kThreads), 0, s, w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts <= kHandedParts) return e;
    hipLaunchKernelGGL((window_join<D, kCB>), dim3((unsigned)join, kWaves * kCB, D / 32), dim3(kThreads), 0, s, w);
    return hipGetLastError();
}

template <int D, int kCB>
hipError_t launch_teams(WindowArgs w, hipStream_t s)
{
    const int WT = 8 * (16 * kCB / (w.d.num_q_heads / w.d.num_kv_heads));
    const long long items = (long long)w.total_tokens / WT + w.d.batch, grid = (items * w.d.num_kv_heads + 7) / 8 * 8;
    if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
    w.items = (int)items;
    w.parts = 1;
    hipLaunchKernelGGL((window_teams<D, kCB>), dim3((unsigned)grid), dim3(512), 128 << 10, s, w);
    return hipGetLastError();
}

template <int D, bool TILED>
hipError_t launch_tiles(const WindowArgs &w, hipStream_t s)
{
    const int G = w.d.num_q_heads / w.d.num_kv_heads;
    const long long walk = std::min((long long)w.window, (long long)w.d.max_blocks * w.d.block_size);
    if constexpr (D == 128 && TILED) {
        // Two teams: with grouped heads, where a walk is eight times a tile's own tokens and more, requests fill four tiles and there is one to a CU (time over that of tiles
        // of 128 columns, 32 / 8 heads, window 1 024 / 256: one prompt of 4 096 0.89 / 1.08, 16 of 512 0.95 / 1.01, 8 of 256 on 3 000 0.86 / 1.0,
        // 16 of 128 on 3 000 1.13 / 1.34; 40 plain heads, prompts, windows of 64 to 4 096: 1.03 to 1.3).
        const int WT = 256 / G;
        if (G <= 32 && w.d.scale_log2e > 0.0f && walk >= 8 * WT && w.total_tokens >= 4LL * WT * w.d.batch && w.d.num_kv_heads * ((long long)w.total_tokens / WT) >= 256)
            return launch_teams<D, 2>(w, s);
    }
    if constexpr (D >= 256) {
        if constexpr (TILED) {
            // Two teams, but where so few tiles have so long a walk that workgroups would share one (time over that of tiles of 128 columns by window_tiles, 16 heads of 256 on
            // 1 to 8: windows of 64, 256 and 1 024, prompts and chunks on cached tokens, 0.68 to 1.0, one of 1.11; 8 of 128 on 3 000, window 3 000, 1.09; plain
            // heads, whose other tiles are of 64 columns, 0.84 to 1.16).
            const int WT = 128 / G;
            if (G <= 16 && w.d.scale_log2e > 0.0f && w.d.num_kv_heads * ((long long)w.total_tokens / WT) * 16 >= walk) return launch_teams<D, 1>(w, s);
        }
        // (as in prefill_mfma)
        return launch_tiles<D, TILED, TILED ? 2 : 1>(w, s);
    } else {
        // Tiles of 64 columns, of which more fit a CU: where requests have few columns, and where a tile's own tokens are a large part of what it walks over (time over that
        // of 128, prompts: window 64, 40 plain heads 0.88, 32 / 8 heads 0.91 to 0.96; 256, 0.93 and 1.03 to 1.07; 1 024, 1.04 and 1.07 to 1.13;
        // 8 of 256 on 3 000, 32 / 8 heads, 1.2 to 1.3).
        const bool narrow = G <= 16 && ((long long)w.max_new_tokens * G <= 512 || walk * G <= 512);
        return narrow ? launch_tiles<D, TILED, 1>(w, s) : launch_tiles<D, TILED, 2>(w, s);
    }
}

template <int D>
hipError_t launch_tiles_f32(WindowArgs w, hipStream_t s)
{
    const int GH = f32_heads(w.d.num_q_heads / w.d.num_kv_heads), TW = 16 / GH;
    const long long items = (long long)w.total_tokens / TW + w.d.batch, all = items * (w.d.num_q_heads / GH);
    if (all > 0x7ffffff8LL) return hipErrorInvalidValue;
    w.items = (int)items;
    w.parts = 1;
    // A tile to a wave where that keeps all of them at work and a walk is short, so that its latency is not what the launch takes (time over that of a tile to four
    // waves: 5 600 tiles, 8 plain heads of 64, windows of 50 / 250 / 500 / 1 000 0.74 / 0.91 / 0.98 / 1.09, 32 / 8 heads of 128, 50 / 250 / 1 000, 0.76 / 0.89 /
    // 1.01; 4 000 of 8 / 2 heads of 32, 50 / 250 / 1 000, 0.69 / 0.86 / 1.14; 2 100 of 64, 50 / 250, 0.97 / 1.13; 600, 1.2 to 1.5).
    const bool alone = (w.total_tokens / TW) * (long long)(w.d.num_q_heads / GH) >= 3500 && most_positions(w, 16) <= 512 + 32;
    if (alone) hipLaunchKernelGGL((window_tiles_f32<D, true>), dim3((unsigned)(((all + kWaves - 1) / kWaves + 7) / 8 * 8)), dim3(kThreads), 0, s, w);
    else hipLaunchKernelGGL((window_tiles_f32<D, false>), dim3((unsigned)((all + 7) / 8 * 8)), dim3(kThreads), 0, s, w);
    return hipGetLastError();
}

template <int LPT>
hipError_t launch_f32(const WindowArgs &w, hipStream_t s)
{
    switch (w.d.heads_per_pass) {
    case 1: return launch_one<WindowValu<false, LPT, 1, kHalves>>(w, s);
    case 2: return launch_one<WindowValu<false, LPT, 2, kHalves>>(w, s);
    case 4: return launch_one<WindowValu<false, LPT, 4, 1>>(w, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_window(const WindowArgs &w, hipStream_t s)
{
    const DecodeArgs &a = w.d;
    const int lpt = a.head_dim * (a.bf16 ? 2 : 4) / 16;
    if (decode_uses_tiled_layout(a.bf16, a.num_q_heads / a.num_kv_heads)) {
        if (a.head_dim == 64) return launch_one<WindowMfma<64>>(w, s);
        if (a.head_dim == 128) return launch_one<WindowMfma<128>>(w, s);
        if (a.head_dim == 256) return launch_one<WindowMfma<256>>(w, s);
    } else if (a.bf16) {
        if (lpt == 8) return launch_one<WindowValu<true, 8, 1, kHalves>>(w, s);
        if (lpt == 16) return launch_one<WindowValu<true, 16, 1, kHalves>>(w, s);
        if (lpt == 32) return launch_one<WindowValu<true, 32, 1, kHalves>>(w, s);
    } else {
        if (lpt == 8) return launch_f32<8>(w, s);
        if (lpt == 16) return launch_f32<16>(w, s);
        if (lpt == 32) return launch_f32<32>(w, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_decode_window(const WindowArgs &w, hipStream_t stream)
{
    if (w.d.batch == 0) return hipSuccess;
    return launch_window(w, stream);
}

hipError_t launch_prefill_window(const WindowArgs &w, hipStream_t stream)
{
    const DecodeArgs &a = w.d;
    if (a.batch == 0 || w.total_tokens == 0) return hipSuccess;
    const int G = a.num_q_heads / a.num_kv_heads;
    // (the kernels of tiles keep the distance between two blocks of a pool in 32 bits)
    const unsigned long long stride = 2ull * a.num_layers * a.num_kv_heads * a.block_size * a.head_dim;
    if (a.bf16 && G <= 32 && !w.force_rows && stride <= 0xffffffffull) {
        const bool tiled = decode_uses_tiled_layout(a.bf16, G);
        if (a.head_dim == 64) return tiled ? launch_tiles<64, true>(w, stream) : launch_tiles<64, false>(w, stream);
        if (a.head_dim == 128) return tiled ? launch_tiles<128, true>(w, stream) : launch_tiles<128, false>(w, stream);
        if (a.head_dim == 256) return tiled ? launch_tiles<256, true>(w, stream) : launch_tiles<256, false>(w, stream);
    }
    if (!a.bf16 && !w.force_rows) {
        if (a.head_dim == 32) return launch_tiles_f32<32>(w, stream);
        if (a.head_dim == 64) return launch_tiles_f32<64>(w, stream);
        if (a.head_dim == 128) return launch_tiles_f32<128>(w, stream);
    }
    return launch_window(w, stream);
}

}  // namespace lamps
