// Queries and keys normalised head by head and turned to their position, keys and values into the cache: what stands between a
// layer's projections and its attention, in one pass.
//
//   x <- x / sqrt(mean(x^2) + eps) * w ;   (a, b) <- A (a cos u - b sin u, a sin u + b cos u),  u = p f_i
//
// The norm, and the turn behind it, are in fp32 and rounded once.  The angle is in fp64: at position 100 000 an fp32 product is off by
// 4e-3 radians; whole turns are taken off before anything is rounded to 32 bits.  (fp64 multiplies run at half the rate of fp32
// ones here, and an angle serves all heads of a token.)
#include <hip/hip_runtime.h>

#include "attn_reducers.h"
#include "internal.h"
#include "requests.h"

namespace lamps {
namespace {

// (cos u, sin u) of u = p f.  u is brought to r in [-pi/4, pi/4] and a quarter; there the series of both end where the next term
// is below 2^-28: r^11 / 11! = 2e-9 and r^12 / 12! = 1e-10.
__device__ __forceinline__ float2 turn(int p, double f)
{
    const double turns = (double)p * f * 0.15915494309189533577;      // 1 / (2 pi)
    const double part = turns - rint(turns), quarter = rint(4.0 * part);
    const float r = (float)((part - 0.25 * quarter) * 6.28318530717958647692);
    const float z = r * r;
    const float s = fmaf(r * z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), r);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
    const int q = (int)quarter;
    const float cs = q & 1 ? s : c, sn = q & 1 ? c : s;
    return make_float2((q + 1) & 2 ? -cs : cs, q & 2 ? -sn : sn);
}

// How a thread treats its 16 bytes of a head, N elements, which are of the same dims in all heads that it sees.
template <bool BF16, int LPH>
struct Turner {
    static constexpr int N = BF16 ? 8 : 4;
    float c[N], s[N];                                 // y = c x + s (the pair's other); not turned: y = x
    int other;                                        // the lane that holds the others, HALVES (its own: neighbours)
    bool turned;

    // cs: (cos, sin) of the token's pairs, amplitude included
    __device__ __forceinline__ void init(const RopeArgs &a, const float2 *cs, int col)
    {
        const int lane = threadIdx.x & 63, half = a.rotary_dim / 2, d = col * N;
        turned = d < a.rotary_dim;
        other = lane;
        const bool low = d < half;
        if (!a.neighbours && turned) other = low ? lane + half / N : lane - half / N;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int i = a.neighbours ? (d + e) / 2 : low ? d + e : d + e - half;
            const float2 x = turned ? cs[i] : make_float2(1.0f, 0.0f);
            c[e] = x.x;
            s[e] = (a.neighbours ? (e & 1) == 0 : low) ? -x.y : x.y;
        }
    }
    // What the lane half a head away has: without LDS.
    static __device__ __forceinline__ float across(float x)
    {
        if constexpr (LPH == 32) return __shfl_xor(x, 16);
        const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), LPH == 16 ? 0x128 : 0x141, 0xF, 0xF, true);   // row_ror 8; row_half_mirror
        if constexpr (LPH == 16) return __int_as_float(y);
        return __int_as_float(__builtin_amdgcn_update_dpp(0, y, 0x1B, 0xF, 0xF, true));                               // quad_perm [3, 2, 1, 0]
    }
    // One head's: by the LPH lanes that hold it together.
    __device__ __forceinline__ uint4 apply(const RopeArgs &a, uint4 x, const float (&w)[N]) const
    {
        float f[N];
        unpack<BF16, N>(x, f);
        if (a.normalise) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) sum = fmaf(f[e], f[e], sum);
            sum = sum_token_lanes<LPH>(sum);
            const float inv = rsqrtf(sum * a.inv_dim + a.norm_eps);
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] = f[e] * inv * w[e];
        }
        if (a.rotary_dim > 0) {
            float o[N];
            if (a.neighbours) {                       // uniform
#pragma unroll
                for (int e = 0; e < N; ++e) o[e] = f[e ^ 1];
            } else if (a.rotary_dim == LPH * N) {
#pragma unroll
                for (int e = 0; e < N; ++e) o[e] = across(f[e]);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) o[e] = __shfl(f[e], other);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] = turned ? fmaf(f[e], c[e], o[e] * s[e]) : f[e];
        }
        if constexpr (BF16) return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        else return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

template <bool BF16, int N>
__device__ __forceinline__ void weights_of(const void *w, int d, float (&f)[N])
{
    if (w) {
        unpack<BF16, N>(*reinterpret_cast<const uint4 *>(static_cast<const char *>(w) + d * (BF16 ? 2 : 4)), f);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = 1.0f;
    }
}

// ---------------------------------------------------------------- one new token per request

// Workgroups (request, slice of its heads): 16 bytes of a head per thread, queries, then keys, then values.  Bound by the
// round trips: length, mask, the vectors and the frequencies are asked for together, then the table entry; the angles go through LDS (32 / 8 heads of 128: 4.0 us for
// one request, 6.0 for 230 of 256, whose bytes are 1.1 us of a copy).
// With `advance` one workgroup takes a request, for the others might read the new length.
template <bool BF16, int D, bool TILED>
__global__ __launch_bounds__(1024) void rope_append(const RopeArgs a)
{
    constexpr int ES = BF16 ? 2 : 4, N = 16 / ES, LPH = D / N;
    __shared__ float2 cs[D / 2];
    const int r = blockIdx.x, tid = threadIdx.x, H = a.num_q_heads, Hkv = a.num_kv_heads;
    const int units = (H + 2 * Hkv) * LPH, step = gridDim.y * blockDim.x;
    const auto source = [&](int i) {
        const int head = i / LPH, at = (i % LPH) * 16;
        const char *x = head < H ? static_cast<const char *>(a.q) + ((size_t)r * a.q_stride + (size_t)head * D) * ES
                        : head < H + Hkv ? static_cast<const char *>(a.k_new) + ((size_t)r * a.k_stride + (size_t)(head - H) * D) * ES
                                         : static_cast<const char *>(a.v_new) + ((size_t)r * a.v_stride + (size_t)(head - H - Hkv) * D) * ES;
        return *reinterpret_cast<const uint4 *>(x + at);
    };
    int i = blockIdx.y * blockDim.x + tid;
    uint4 x = i < units ? source(i) : make_uint4(0, 0, 0, 0);
    const int t = a.ctx_lens[r];
    if (!a.running[r]) return;                        // uniform over the workgroup, as what follows
    const int lb = t >> a.log2_block_size, slot = t & (a.block_size - 1);
    if (t < 0 || lb >= a.max_blocks) return;
    const int block = a.block_table[(size_t)r * a.max_blocks + lb];
    for (int j = tid; j < a.rotary_dim / 2; j += blockDim.x) {
        const float2 y = turn(t, a.frequencies[j]);
        cs[j] = make_float2(y.x * a.amplitude, y.y * a.amplitude);
    }
    if (block < 0 || block >= a.num_blocks) return;
    __syncthreads();
    const size_t tile = (size_t)a.block_size * D, at0 = (((size_t)block * a.num_layers + a.layer) * Hkv) * tile;
    const int col = i % LPH;                          // (the step is a multiple of LPH)
    Turner<BF16, LPH> turner;
    turner.init(a, cs, col);
    for (; i < units; i += step) {
        const int head = i / LPH, d = col * N;
        if (head < H + Hkv) {
            const bool key = head >= H;
            float w[N];
            weights_of<BF16, N>(key ? a.k_weight : a.q_weight, d, w);
            const uint4 y = turner.apply(a, x, w);
            if (!key) {
                *reinterpret_cast<uint4 *>(static_cast<char *>(a.q_out) + (((size_t)r * H + head) * D + d) * ES) = y;
            } else {
                const size_t o = TILED ? (size_t)(slot >> 4) * 16 * D + (size_t)((d >> 3) * 16 + (slot & 15)) * 8 : (size_t)slot * D + d;
                *reinterpret_cast<uint4 *>(static_cast<char *>(a.k_pool) + (at0 + (head - H) * tile + o) * ES) = y;
            }
        } else if constexpr (!TILED) {
            *reinterpret_cast<uint4 *>(static_cast<char *>(a.v_pool) + (at0 + (head - H - Hkv) * tile + (size_t)slot * D + d) * ES) = x;
        } else {
            // (a unit of the value tile is four slots of two dims: one token's are 16 bits each)
            uint16_t *v = static_cast<uint16_t *>(a.v_pool) + at0 + (head - H - Hkv) * tile + (size_t)(slot >> 4) * 16 * D;
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int dd = d + e;
                v[((((dd >> 5) * 4 + ((slot & 15) >> 2)) * 16 + (dd & 15)) * 2 + ((dd & 31) >> 4)) * 4 + (slot & 3)] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
            }
        }
        if (i + step < units) x = source(i + step);
    }
    if (a.advance && tid == 0) a.ctx_lens[r] = t + 1;
}

// ---------------------------------------------------------------- many new tokens

// Workgroups (request, 16 positions that a sub-tile of the cache has, kv heads): kv head by kv head the G queries of its group, its key
// and its value.  A thread keeps one of the 16 positions and 16 bytes of a head (HS heads side by side where heads are short), so the angles of its
// dims stay in registers, and asks for four heads before it turns the four before them.  Bound by memory: 4 x 4 096 tokens on 32 / 8 heads of 128 out of packed rows 94 us,
// 4.3 TB/s read and written; 24 of 16 to 700 on 40 plain heads 119, 4.8 TB/s.  (Non-temporal loads, or six or eight heads ahead, are as fast.)
template <int D, bool BF16>
constexpr int rope_threads() { return 16 * D * (BF16 ? 2 : 4) / 16 > 256 ? 16 * D * (BF16 ? 2 : 4) / 16 : 256; }

template <bool BF16, int D, bool TILED>
__global__ __launch_bounds__((rope_threads<D, BF16>())) void rope_append_tokens(const RopeArgs a)
{
    constexpr int ES = BF16 ? 2 : 4, N = 16 / ES, LPH = D / N, THREADS = rope_threads<D, BF16>(), HS = THREADS / (16 * LPH);
    constexpr int AHEAD = 4;                          // heads asked for together
    __shared__ float2 cs[16][D / 2 + 1];
    const int w = blockIdx.x, tid = threadIdx.x;
    const auto [r, first, count, ctx] = new_tokens_at(a.q_start, a.ctx_lens, a.batch, w, [](int q, int i) { return (q >> 4) + 2 * i; });
    const int p0 = ctx - count;                       // position of the request's first new token
    if (first < 0 || count <= 0 || p0 < 0) return;
    const int sub = (p0 >> 4) + (w - ((first >> 4) + 2 * r));
    const int t_lo = max(p0, sub * 16), t_hi = min(p0 + min(count, a.total_tokens - first), sub * 16 + 16);
    if (t_lo >= t_hi || ctx > a.max_blocks * a.block_size) return;
    const int bs = a.block_size, block = a.block_table[(size_t)r * a.max_blocks + ((sub * 16) >> a.log2_block_size)];
    if (block < 0 || block >= a.num_blocks) return;

    const int half = a.rotary_dim / 2;
    for (int j = tid; j < 16 * half; j += THREADS) {
        const int token = j / half, i = j - token * half;
        const float2 y = turn(sub * 16 + token, a.frequencies[i]);
        cs[token][i] = make_float2(y.x * a.amplitude, y.y * a.amplitude);
    }
    __syncthreads();
    const int col = tid % LPH, slot = tid / LPH % 16, hs = tid / (16 * LPH), d = col * N;
    const int t = sub * 16 + slot;
    const bool live = t >= t_lo && t < t_hi;          // (the same for all lanes of a head)
    const size_t n = (size_t)first + (live ? t - p0 : t_lo - p0);
    Turner<BF16, LPH> turner;
    turner.init(a, cs[slot], col);
    float qw[N], kw[N];
    weights_of<BF16, N>(a.q_weight, d, qw);
    weights_of<BF16, N>(a.k_weight, d, kw);

    const int H = a.num_q_heads, Hkv = a.num_kv_heads, G = H / Hkv, heads = a.heads_each;
    const int g0 = blockIdx.y * heads, g1 = min(Hkv, g0 + heads);
    const size_t tile = (size_t)bs * D, sub_at = (size_t)(((sub * 16) & (bs - 1)) >> 4) * 16 * D;
    const char *q = static_cast<const char *>(a.q) + (n * a.q_stride + d) * ES, *k = static_cast<const char *>(a.k_new) + (n * a.k_stride + d) * ES;
    char *q_out = static_cast<char *>(a.q_out) + (n * H * D + d) * ES;
    // Values.  Plain layout: as keys.  Tiled layout: a wave takes four slots, a quad, of up to 128 dims, 16 bytes of a slot to a lane, and brings them into
    // the tile's units, four slots of two dims each, by the transposing LDS read (lane j of 16 receives dim j of four rows); a quad that is not all
    // new goes by 16 bits.
    constexpr int VROW = D < 128 ? D : 128, VL = VROW / 8;   // dims of a row in a wave's LDS, and the lanes that load one
    const int lane = tid & 63, wave = tid >> 6;
    const int vchunk = TILED ? (D < 128 ? 0 : wave % (D / 128)) : 0;                  // which 128 dims
    const int vfirst = TILED ? (D < 128 ? wave % 2 * 8 : wave / (D / 128) % 4 * 4) : 0;   // the wave's first slot
    const int vd = TILED ? vchunk * 128 + lane % VL * 8 : d, vslot = TILED ? vfirst + lane / VL : slot;
    const int vt = sub * 16 + vslot;
    const bool vlive = vt >= t_lo && vt < t_hi;
    const char *v = static_cast<const char *>(a.v_new) + (((size_t)first + (vlive ? vt - p0 : t_lo - p0)) * a.v_stride + vd) * ES;
    __shared__ __align__(16) uint16_t quads[TILED ? THREADS / 64 : 1][TILED ? 512 : 8];
    const auto put_values = [&](uint4 x, int g) {
        const size_t at = (((size_t)block * a.num_layers + a.layer) * Hkv + g) * tile + sub_at;
        if constexpr (!TILED) {
            if (live) *reinterpret_cast<uint4 *>(static_cast<char *>(a.v_pool) + (at + (size_t)slot * D + d) * ES) = x;
        } else {
            typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
            uint16_t *mine = quads[wave];
            *reinterpret_cast<uint4 *>(mine + lane * 8) = x;
            const int i16 = lane & 15, group = lane >> 4;    // the 16 lanes' quad and 32 dims of the wave's
            const int quad = D < 128 ? group >> 1 : 0, i32 = D < 128 ? group & 1 : group;
            const uint16_t *from = mine + (quad * 4 + (i16 >> 2)) * VROW + 32 * i32 + 4 * (i16 & 3);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(from + 16));
            uint16_t *to = static_cast<uint16_t *>(a.v_pool) + at;
            const int q0 = vfirst + quad * 4, t0 = sub * 16 + q0;
            if (t0 >= t_lo && t0 + 4 <= t_hi) {
                const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
                *reinterpret_cast<uint4 *>(to + (size_t)(((vchunk * 4 + i32) * 4 + (q0 >> 2)) * 16 + i16) * 8) = make_uint4(l.x, l.y, h.x, h.y);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t0 + e >= t_lo && t0 + e < t_hi) {
                        uint16_t *unit = to + (size_t)(((vchunk * 4 + i32) * 4 + (q0 >> 2)) * 16 + i16) * 8 + e;
                        unit[0] = (uint16_t)lo[e];
                        unit[4] = (uint16_t)hi[e];
                    }
            }
        }
    };
    // queries of heads g0 G .. g1 G - 1, keys and values g0 .. g1 - 1: a batch of heads is asked for while the one before it is turned
    const int nq = (g1 - g0) * G, nk = nq + g1 - g0, all = nk + g1 - g0;
    const auto from = [&](int i) {
        return *reinterpret_cast<const uint4 *>(i < nq ? q + (size_t)(g0 * G + i) * D * ES : i < nk ? k + (size_t)(g0 + i - nq) * D * ES : v + (size_t)(g0 + i - nk) * D * ES);
    };
    uint4 x[AHEAD], y[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) x[u] = from(min(hs + u * HS, all - 1));
    for (int i0 = hs; i0 < all; i0 += AHEAD * HS) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) y[u] = from(min(i0 + (AHEAD + u) * HS, all - 1));
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = i0 + u * HS;                // (the same for a wave)
            if (i >= all) break;
            if (i < nq) {
                const uint4 z = turner.apply(a, x[u], qw);
                if (live) *reinterpret_cast<uint4 *>(q_out + (size_t)(g0 * G + i) * D * ES) = z;
            } else if (i < nk) {
                const uint4 z = turner.apply(a, x[u], kw);
                const size_t at = (((size_t)block * a.num_layers + a.layer) * Hkv + g0 + i - nq) * tile + sub_at;
                const size_t o = TILED ? (size_t)((d >> 3) * 16 + slot) * 8 : (size_t)slot * D + d;
                if (live) *reinterpret_cast<uint4 *>(static_cast<char *>(a.k_pool) + (at + o) * ES) = z;
            } else {
                put_values(x[u], g0 + i - nk);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) x[u] = y[u];
    }
}

template <bool BF16, int D, bool TILED>
hipError_t launch(RopeArgs a, int total_tokens, hipStream_t stream)
{
    constexpr int ES = BF16 ? 2 : 4;
    if (total_tokens < 0) {
        const int units = (a.num_q_heads + 2 * a.num_kv_heads) * (D * ES / 16);
        if (a.advance) {
            const int threads = units < 1024 ? (units + 63) / 64 * 64 : 1024;
            hipLaunchKernelGGL((rope_append<BF16, D, TILED>), dim3((unsigned)a.batch), dim3((unsigned)threads), 0, stream, a);
        } else {
            hipLaunchKernelGGL((rope_append<BF16, D, TILED>), dim3((unsigned)a.batch, (unsigned)((units + 255) / 256)), dim3(256), 0, stream, a);
        }
        return hipGetLastError();
    }
    // The angles of 16 positions are as much work as turning a head or two: a workgroup takes as many kv heads as leave the chip four workgroups to a CU.
    const long long subs = (total_tokens >> 4) + 2LL * a.batch;
    a.heads_each = 1;
    while (a.heads_each * 2 <= a.num_kv_heads && subs * ((a.num_kv_heads + 2 * a.heads_each - 1) / (2 * a.heads_each)) >= 1024) a.heads_each *= 2;
    hipLaunchKernelGGL((rope_append_tokens<BF16, D, TILED>), dim3((unsigned)subs, (unsigned)((a.num_kv_heads + a.heads_each - 1) / a.heads_each)),
                       dim3(rope_threads<D, BF16>()), 0, stream, a);
    return hipGetLastError();
}

template <bool BF16, int D>
hipError_t launch(const RopeArgs &a, int total_tokens, int tiled, hipStream_t stream)
{
    if constexpr (BF16)
        if (tiled) return launch<BF16, D, true>(a, total_tokens, stream);
    return launch<BF16, D, false>(a, total_tokens, stream);
}

}  // namespace

hipError_t launch_rope_append(const RopeArgs &a, int total_tokens, int tiled, hipStream_t stream)
{
    if (a.batch == 0 || total_tokens == 0) return hipSuccess;
    if (a.bf16) {
        if (a.head_dim == 64) return launch<true, 64>(a, total_tokens, tiled, stream);
        if (a.head_dim == 128) return launch<true, 128>(a, total_tokens, tiled, stream);
        if (a.head_dim == 256) return launch<true, 256>(a, total_tokens, tiled, stream);
    } else {
        if (a.head_dim == 32) return launch<false, 32>(a, total_tokens, tiled, stream);
        if (a.head_dim == 64) return launch<false, 64>(a, total_tokens, tiled, stream);
        if (a.head_dim == 128) return launch<false, 128>(a, total_tokens, tiled, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace lamps
