// Keys and values into a cache of 8 bits, and back out of a cache of any type.
//
// A block has one scale for the keys of a head and one for its values, which the largest of its tokens decides.  Tokens come one or
// many at a time; slot 0 begins a block anew, and where a later token is larger than the scale holds, the codes that are there are
// rounded to the new one.  Scales, codes and the rounding: kv8.h.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "internal.h"
#include "kv8.h"
#include "requests.h"

namespace lamps {
namespace {

constexpr int kThreads = 256;
constexpr int kAdvanceThreads = 1024;

// Largest of a value over the lanes of a wave, in all of them.
__device__ __forceinline__ uint32_t wave_most(uint32_t x)
{
#pragma unroll
    for (int k = 1; k < 64; k *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, k));
    return x;
}
// The same over rows of 16 lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t row_max(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true)); }
__device__ __forceinline__ uint32_t row_most(uint32_t x) { return row_max<0x121>(row_max<0x122>(row_max<0x124>(row_max<0x128>(x)))); }   // (turned by 8, 4, 2, 1 lanes)

// ---------------------------------------------------------------- one token per request

// Sixteen lanes take the keys, or the values, of one head; unit 2 g + (0 or 1).  Bound by the launch and the round trips in front of the stores: length,
// mask and vectors are asked for together, then the table entry, then the block's scales.  256 requests of 40 heads of 128, a tenth of them masked out, us: 6.4 (a wave to a head's
// keys or values, 18 000 waves on a chip that holds 8 192 of them: 9.0); one request of 8 heads 4.8, of which the kernel is 2.6.
template <int D>
__global__ __launch_bounds__(kAdvanceThreads) void kv8_append(const AppendArgs a)
{
    constexpr int E = D / 16;                            // dims of a lane
    const int r = blockIdx.x, lane = threadIdx.x & 63, waves = blockDim.x >> 6, quarter = lane >> 4, d0 = (lane & 15) * E;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), units = 2 * a.num_kv_heads;
    const auto vector = [&](int u, uint32_t (&x)[E / 2]) {   // its dims
        const uint16_t *p = static_cast<const uint16_t *>(u & 1 ? a.v_new : a.k_new) + ((size_t)r * a.num_kv_heads + (u >> 1)) * D + d0;
#pragma unroll
        for (int e = 0; e < E / 2; e += 2) {
            const uint2 y = *reinterpret_cast<const uint2 *>(p + 2 * e);
            x[e] = y.x; x[e + 1] = y.y;
        }
    };
    int u0 = (blockIdx.y * waves + wv) * 4;              // the wave's first
    uint32_t x[E / 2];
    vector(min(u0 + quarter, units - 1), x);
    const int t = a.ctx_lens[r], running = a.running[r];
    if (!running) return;                                // uniform over the workgroup
    if (a.advance) __syncthreads();                      // (all of its waves have read the length)
    const int lb = t >> a.log2_block_size, slot = t & (a.block_size - 1);
    if (t < 0 || lb >= a.max_blocks) return;
    const int block = a.block_table[(size_t)r * a.max_blocks + lb];
    if (block < 0 || block >= a.num_blocks) return;
    const size_t tile = (size_t)a.block_size * D, slice = codes_slice(a.num_kv_heads, a.block_size, D);
    const size_t at = ((size_t)block * a.num_layers + a.layer) * slice;
    char *const k_codes = static_cast<char *>(a.k_pool) + at, *const v_codes = static_cast<char *>(a.v_pool) + at;
    float *scales = reinterpret_cast<float *>(k_codes + a.num_kv_heads * tile);
    for (; u0 < units; u0 += 4 * waves * gridDim.y) {
        const int u = u0 + quarter;
        const bool on = u < units;
        const float old = on && slot > 0 ? scales[u] : 0.0f;
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < E / 2; ++e) most = max(most, max(finite_size(x[e]), finite_size(x[e] >> 16)));
        const float scale = fmaxf(scale_for(row_most(most)), old), inv = inverse(scale);
        // what is there, by the new scale: the wave together, a unit at a time
        uint64_t grown = __ballot(on && slot > 0 && old != scale) & 0x0001000100010001ull;
        if (grown) {                                     // uniform
            const float factor = old * inv;
            do {
                const int from = __builtin_ctzll(grown), v = u0 + (from >> 4);
                grown &= grown - 1;
                const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(factor), from));
                char *codes = (v & 1 ? v_codes : k_codes) + (v >> 1) * tile;
                for (int i = lane; i < ((slot + 15) >> 4) * D; i += 64) {
                    const int sub = i / D, c = i & (D - 1);
                    // a unit of keys is one slot's, of values four slots'
                    const int s0 = sub * 16 + (v & 1 ? (c >> 4 & 3) * 4 : c & 15);
                    if (s0 >= slot) continue;
                    uint4 *p = reinterpret_cast<uint4 *>(codes) + i;
                    const uint4 w = *p;
                    uint4 y = make_uint4(recode(w.x, f), recode(w.y, f), recode(w.z, f), recode(w.w, f));
                    if ((v & 1) && s0 + 4 > slot) {
                        const uint32_t keep = 0xFFFFFFFFu << (8 * (slot - s0));   // slots that hold nothing: as they were
                        y.x = (y.x & ~keep) | (w.x & keep);
                        y.y = (y.y & ~keep) | (w.y & keep);
                        y.z = (y.z & ~keep) | (w.z & keep);
                        y.w = (y.w & ~keep) | (w.w & keep);
                    }
                    *p = y;
                }
            } while (grown);
            __builtin_amdgcn_s_waitcnt(0);               // (the token's own codes lie in the same units)
        }
        uint32_t w[E / 4];
#pragma unroll
        for (int e = 0; e < E / 4; ++e)
            w[e] = to_codes(__uint_as_float(x[2 * e] << 16), __uint_as_float(x[2 * e] & 0xFFFF0000u), __uint_as_float(x[2 * e + 1] << 16), __uint_as_float(x[2 * e + 1] & 0xFFFF0000u), inv);
        if (on) {
            char *sub = (u & 1 ? v_codes : k_codes) + (u >> 1) * tile + (size_t)(slot >> 4) * 16 * D;
            if (u & 1) {
#pragma unroll
                for (int e = 0; e < E; ++e) sub[value_code(slot & 15, d0 + e)] = (char)(w[e / 4] >> (8 * (e & 3)));
            } else {
                uint32_t *p = reinterpret_cast<uint32_t *>(sub + key_code(slot & 15, d0));
#pragma unroll
                for (int e = 0; e < E / 4; ++e) p[e] = w[e];
            }
            if ((lane & 15) == 0) scales[u] = scale;
        }
        const int next = u0 + 4 * waves * gridDim.y;
        if (next < units) vector(min(next + quarter, units - 1), x);
    }
    // (a workgroup to a request: its waves have read the length)
    if (a.advance && threadIdx.x == 0) a.ctx_lens[r] = t + 1;
}

// ---------------------------------------------------------------- many tokens per request

// Four lanes that follow each other hold rows of a matrix of 4 by 4, and then its columns.
template <int CTRL>
__device__ __forceinline__ uint32_t quad_swap(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true); }
__device__ __forceinline__ void transpose4(uint32_t (&w)[4])
{
    const int lane = threadIdx.x & 3;
    // neighbours exchange w[1] of the even one for w[0] of the odd one, and w[3] for w[2]; then pairs
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        const uint32_t give = lane & 1 ? w[k] : w[k + 1], got = quad_swap<0xB1>(give);
        if (lane & 1) w[k] = got; else w[k + 1] = got;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t give = lane & 2 ? w[k] : w[k + 2], got = quad_swap<0x4E>(give);
        if (lane & 2) w[k] = got; else w[k + 2] = got;
    }
}

// Where the tokens of a workgroup are: the w'th (request, block that holds new tokens).  Request r touches at most (count >> log2) + 2 blocks, and the
// first workgroups of consecutive requests are that far apart.
struct BlockAt {
    int first, p0, t_lo, t_hi, lb, block;                // row and position of the request's first token; the block's new positions
};
__device__ __forceinline__ bool block_at(const CodesArgs &a, int w, int log2, BlockAt &x)
{
    const auto begin = [log2](int q, int i) { return (q >> log2) + 2 * i; };
    const NewTokens n = new_tokens_at(a.q_start, a.ctx_lens, a.batch, w, begin);
    x.p0 = n.ctx - n.count;
    x.first = n.first;
    // (a context shorter than its new tokens, or longer than the table row: nothing is read or written for it)
    if (n.count <= 0 || n.first < 0 || x.p0 < 0 || n.ctx > a.max_blocks * a.block_size) return false;
    const int b = (x.p0 >> log2) + (w - begin(n.first, n.r)), size = 1 << log2;
    x.t_lo = max(x.p0, b << log2);
    x.t_hi = min(x.p0 + min(n.count, a.total_tokens - n.first), (b << log2) + size);
    x.lb = (b << log2) >> a.log2_block_size;
    if (x.t_lo >= x.t_hi || x.lb >= a.max_blocks) return false;
    x.block = a.block_table[(size_t)n.r * a.max_blocks + x.lb];
    return x.block >= 0 && x.block < a.num_blocks;
}

// One workgroup per (block that holds new tokens, kv head), which alone decides its two scales and writes it.  A unit is 16 bytes of codes: of
// keys 16 dims of a slot; of values, for four slots, dims j + 16 s of a group of 64, which four lanes, one for each s, load four dims j at a time of
// and transpose among themselves.  The numbers are loaded for the largest of them, kept (HOLD units to a thread, where a block has no more; else they are loaded
// again, out of L2) and rounded.  Bound by memory: 4 prompts of 4 096 tokens, 8 heads of 128, 101 MB, 21.9 to 23.7 us, 4.3 to 4.6 TB/s; 12 responses of 4 to 64 tokens 4.8, the launch and the
// round trips.
template <int D, int HOLD>
__global__ __launch_bounds__(kThreads) void kv8_append_tokens(const CodesArgs a)
{
    __shared__ uint32_t sizes[2][kThreads / 64];
    BlockAt b;
    if (!block_at(a, blockIdx.x, a.log2_block_size, b)) return;
    const int g = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), base = b.lb << a.log2_block_size;
    const size_t tile = (size_t)a.block_size * D, slice = codes_slice(a.num_kv_heads, a.block_size, D);
    const size_t at = ((size_t)b.block * a.num_layers + a.layer) * slice;
    float *scales = reinterpret_cast<float *>(static_cast<char *>(a.k_pool) + at + a.num_kv_heads * tile) + 2 * g;
    const bool begins = b.t_lo == base;
    const float old_k = begins ? 0.0f : scales[0], old_v = begins ? 0.0f : scales[1];
    const int row = a.num_kv_heads * D;
    // units of a sub-tile: D of keys, D of values (a wave's are of one kind)
    const int sub0 = (b.t_lo - base) >> 4, subs = ((b.t_hi - 1 - base) >> 4) + 1, last = subs * 2 * D;
    // Unit i: its four words of codes' worth of numbers, by slots (values) or dims (keys): 4 x 4 bf16 in 8 words.
    const auto slot_of = [&](int i) { const int c = i & (D - 1); return (i / (2 * D)) * 16 + (i & D ? (c >> 4 & 3) * 4 : c & 15); };
    const auto load = [&](int i, uint32_t (&x)[8]) {
        const int c = i & (D - 1);
        const auto src = [&](const void *p, int slot) {  // (slots that hold no new token: the nearest that does)
            const int t = min(max(base + slot, b.t_lo), b.t_hi - 1);
            return static_cast<const uint16_t *>(p) + (size_t)(b.first + (t - b.p0)) * row + g * D;
        };
        if (i & D) {
            const int s = c & 3, jg = c >> 2 & 3;        // c = ((i64 * 4 + q) * 4 + jg) * 4 + s
            const int d = (c >> 6) * 64 + 16 * s + 4 * jg, slot = slot_of(i);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint2 w = *reinterpret_cast<const uint2 *>(src(a.v_new, slot + k) + d);
                x[2 * k] = w.x;
                x[2 * k + 1] = w.y;
            }
        } else {
            const uint16_t *p = src(a.k_new, slot_of(i)) + (c >> 4) * 16;
            const uint4 w0 = *reinterpret_cast<const uint4 *>(p), w1 = *reinterpret_cast<const uint4 *>(p + 8);
            x[0] = w0.x; x[1] = w0.y; x[2] = w0.z; x[3] = w0.w;
            x[4] = w1.x; x[5] = w1.y; x[6] = w1.z; x[7] = w1.w;
        }
    };
    const auto largest = [&](int i, const uint32_t (&x)[8], uint32_t &k, uint32_t &v) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, max(finite_size(x[e]), finite_size(x[e] >> 16)));
        if (i & D) v = max(v, m); else k = max(k, m);
    };
    const int first = sub0 * 2 * D + tid;
    uint32_t held[HOLD > 0 ? HOLD : 1][8], most_k = 0, most_v = 0;
    if constexpr (HOLD > 0) {
#pragma unroll
        for (int k = 0; k < HOLD; ++k) {
            const int i = first + k * kThreads;
            if (i < last) load(i, held[k]);
        }
#pragma unroll
        for (int k = 0; k < HOLD; ++k) {
            const int i = first + k * kThreads;
            if (i < last) largest(i, held[k], most_k, most_v);
        }
    } else {
        for (int i = first; i < last; i += kThreads) {
            load(i, held[0]);
            largest(i, held[0], most_k, most_v);
        }
    }
    most_k = wave_most(most_k);
    most_v = wave_most(most_v);
    if (lane == 0) {
        sizes[0][wv] = most_k;
        sizes[1][wv] = most_v;
    }
    __syncthreads();
    most_k = most_v = 0;
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) {
        most_k = max(most_k, sizes[0][k]);
        most_v = max(most_v, sizes[1][k]);
    }
    const float scale_k = fmaxf(scale_for(most_k), old_k), scale_v = fmaxf(scale_for(most_v), old_v);
    if (tid == 0) *reinterpret_cast<float2 *>(scales) = make_float2(scale_k, scale_v);
    char *kt = static_cast<char *>(a.k_pool) + at + g * tile, *vt = static_cast<char *>(a.v_pool) + at + g * tile;
    const auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    const auto hi = [](uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); };
    const auto store = [&](int i, const uint32_t (&x)[8]) {
        const int c = i & (D - 1), slot = slot_of(i);
        const bool value = (i & D) != 0;
        const float scale = value ? scale_v : scale_k, old = value ? old_v : old_k, inv = inverse(scale);
        const bool moved = !begins && old != scale;
        uint32_t w[4];
        int place;
        if (value) {
            // x[2 k], x[2 k + 1]: dims 4 jg .. + 3 of slot k; word e: dim 4 jg + e of the four slots
            w[0] = to_codes(lo(x[0]), lo(x[2]), lo(x[4]), lo(x[6]), inv);
            w[1] = to_codes(hi(x[0]), hi(x[2]), hi(x[4]), hi(x[6]), inv);
            w[2] = to_codes(lo(x[1]), lo(x[3]), lo(x[5]), lo(x[7]), inv);
            w[3] = to_codes(hi(x[1]), hi(x[3]), hi(x[5]), hi(x[7]), inv);
            transpose4(w);                               // lane s: the unit of dims 4 jg + s + 16 (0 .. 3)
            place = c;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = to_codes(lo(x[2 * k]), hi(x[2 * k]), lo(x[2 * k + 1]), hi(x[2 * k + 1]), inv);
            place = c;
        }
        uint4 *to = reinterpret_cast<uint4 *>((value ? vt : kt) + (size_t)(i / (2 * D)) * 16 * D) + place;
        const int n = value ? 4 : 1, lo_t = b.t_lo - base, hi_t = b.t_hi - base;
        if (slot >= lo_t && slot + n <= hi_t) {
            *to = make_uint4(w[0], w[1], w[2], w[3]);
        } else if (value && slot + n > lo_t && slot < hi_t) {
            // four slots that are not all new: those in front by the new scale, those behind as they were
            const uint4 was = *to;
            const uint32_t y[4] = {was.x, was.y, was.z, was.w};
            const uint32_t fresh = (0xFFFFFFFFu << (8 * max(lo_t - slot, 0))) & (0xFFFFFFFFu >> (8 * max(slot + 4 - hi_t, 0)));
            const uint32_t before = lo_t > slot ? ~(0xFFFFFFFFu << (8 * (lo_t - slot))) : 0;
            const float f = old * inv;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t z = moved ? recode(y[k], f) : y[k];
                w[k] = (w[k] & fresh) | (z & before) | (y[k] & ~(fresh | before));
            }
            *to = make_uint4(w[0], w[1], w[2], w[3]);
        }
    };
    if constexpr (HOLD > 0) {
#pragma unroll
        for (int k = 0; k < HOLD; ++k) {
            const int i = first + k * kThreads;
            if (i < last) store(i, held[k]);
        }
    } else {
        for (int i = first; i < last; i += kThreads) {
            load(i, held[0]);
            store(i, held[0]);
        }
    }
    // what the block held before, where its scale has grown (units with a new token in them are done)
    if (begins) return;
    const float fk = old_k * inverse(scale_k), fv = old_v * inverse(scale_v);
    if (old_k == scale_k && old_v == scale_v) return;
    const int held_to = b.t_lo - base;
    for (int i = tid; i < ((held_to + 15) >> 4) * 2 * D; i += kThreads) {
        const int slot = slot_of(i);
        const bool value = (i & D) != 0;
        if ((value ? old_v == scale_v : old_k == scale_k) || slot + (value ? 4 : 1) > held_to) continue;
        uint4 *p = reinterpret_cast<uint4 *>((value ? vt : kt) + (size_t)(i / (2 * D)) * 16 * D) + (i & (D - 1));
        const float f = value ? fv : fk;
        const uint4 w = *p;
        *p = make_uint4(recode(w.x, f), recode(w.y, f), recode(w.z, f), recode(w.w, f));
    }
}

// ---------------------------------------------------------------- reading back

// One workgroup per (request, 16 positions of which some are asked for, kv head).  Bound by memory: 383 MB of 40 heads of 128, two thirds of them written, 85 us, 4.5 TB/s.
template <int D>
__global__ __launch_bounds__(kThreads) void kv8_read_tokens(const CodesArgs a, uint16_t *k_out, uint16_t *v_out)
{
    BlockAt b;
    if (!block_at(a, blockIdx.x, 4, b)) return;
    const int g = blockIdx.y, base = b.t_lo & ~15, sub = (base & (a.block_size - 1)) >> 4;
    const size_t tile = (size_t)a.block_size * D, slice = codes_slice(a.num_kv_heads, a.block_size, D);
    const size_t at = ((size_t)b.block * a.num_layers + a.layer) * slice;
    const float2 scale = reinterpret_cast<const float2 *>(static_cast<const char *>(a.k_pool) + at + a.num_kv_heads * tile)[g];
    const size_t from = at + g * tile + (size_t)sub * 16 * D, row = (size_t)a.num_kv_heads * D;
    const auto out = [&](uint16_t *p, int slot) { return p + (size_t)(b.first + (base + slot - b.p0)) * row + g * D; };
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        const int c = i & (D - 1);
        const bool value = (i & D) != 0;
        const uint4 w4 = reinterpret_cast<const uint4 *>(static_cast<const char *>(value ? a.v_pool : a.k_pool) + from)[c];
        uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
        if (value) {
            transpose4(w);                               // (as in kv8_append_tokens, the other way round)
            const int s = c & 3, jg = c >> 2 & 3, q = c >> 4 & 3, d = (c >> 6) * 64 + 16 * s + 4 * jg;
            uint32_t x[4][2];                            // [dim][slots 0, 1 and 2, 3]
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e][0] = from_codes<false>(w[e], scale.y);
                x[e][1] = from_codes<true>(w[e], scale.y);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = base + 4 * q + k, h = k >> 1, sh = 16 * (k & 1);
                if (t >= b.t_lo && t < b.t_hi)
                    *reinterpret_cast<uint2 *>(out(v_out, 4 * q + k) + d) =
                        make_uint2((x[0][h] >> sh & 0xFFFFu) | (x[1][h] >> sh) << 16, (x[2][h] >> sh & 0xFFFFu) | (x[3][h] >> sh) << 16);
            }
        } else {
            const int slot = c & 15, t = base + slot;
            if (t < b.t_lo || t >= b.t_hi) continue;
            uint4 *to = reinterpret_cast<uint4 *>(out(k_out, slot) + (c >> 4) * 16);
            to[0] = make_uint4(from_codes<false>(w[0], scale.x), from_codes<true>(w[0], scale.x), from_codes<false>(w[1], scale.x), from_codes<true>(w[1], scale.x));
            to[1] = make_uint4(from_codes<false>(w[2], scale.x), from_codes<true>(w[2], scale.x), from_codes<false>(w[3], scale.x), from_codes<true>(w[3], scale.x));
        }
    }
}

// Out of pools of the rows' own type: 16 bytes of a row at a time.
template <typename T, bool TILED>
__global__ __launch_bounds__(kThreads) void kv_read_tokens(const CodesArgs a, T *k_out, T *v_out)
{
    constexpr int N = 16 / (int)sizeof(T);
    BlockAt b;
    if (!block_at(a, blockIdx.x, 4, b)) return;
    const int D = a.head_dim, g = blockIdx.y, base = b.t_lo & ~15, row = a.num_kv_heads * D;
    const size_t tile = (size_t)a.block_size * D;
    const size_t from = (((size_t)b.block * a.num_layers + a.layer) * a.num_kv_heads + g) * tile + (size_t)(base & (a.block_size - 1)) * D;
    const T *kt = static_cast<const T *>(a.k_pool) + from, *vt = static_cast<const T *>(a.v_pool) + from;
    for (int i = threadIdx.x; i < 16 * (D / N); i += kThreads) {
        const int slot = i / (D / N), d = (i - slot * (D / N)) * N, t = base + slot;
        if (t < b.t_lo || t >= b.t_hi) continue;
        const size_t to = (size_t)(b.first + (t - b.p0)) * row + g * D + d;
        if constexpr (TILED) {
            *reinterpret_cast<uint4 *>(k_out + to) = *reinterpret_cast<const uint4 *>(kt + ((d >> 3) * 16 + slot) * 8);
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const auto at = [&](int x) { return ((((x >> 5) * 4 + (slot >> 2)) * 16 + (x & 15)) * 2 + ((x & 31) >> 4)) * 4 + (slot & 3); };
                w[e >> 1] = vt[at(d + e)] | (uint32_t)vt[at(d + e + 1)] << 16;
            }
            *reinterpret_cast<uint4 *>(v_out + to) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            *reinterpret_cast<uint4 *>(k_out + to) = *reinterpret_cast<const uint4 *>(kt + slot * D + d);
            *reinterpret_cast<uint4 *>(v_out + to) = *reinterpret_cast<const uint4 *>(vt + slot * D + d);
        }
    }
}

template <int D>
hipError_t append_tokens(const CodesArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.total_tokens >> a.log2_block_size) + 2 * a.batch), (unsigned)a.num_kv_heads), block(kThreads);
    const int units = a.block_size / 16 * 2 * D;         // of a block
    if (units <= kThreads) hipLaunchKernelGGL((kv8_append_tokens<D, 1>), grid, block, 0, s, a);
    else if (units <= 2 * kThreads) hipLaunchKernelGGL((kv8_append_tokens<D, 2>), grid, block, 0, s, a);
    else if (units <= 4 * kThreads) hipLaunchKernelGGL((kv8_append_tokens<D, 4>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((kv8_append_tokens<D, 0>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv8_append(const AppendArgs &a, hipStream_t s)
{
    if (a.batch == 0) return hipSuccess;
    // (where the call advances the lengths a request is one workgroup's: another may have yet to read them)
    const int threads = a.advance ? std::min(kAdvanceThreads, (2 * a.num_kv_heads + 3) / 4 * 64) : kThreads, waves = threads / 64;
    const dim3 grid((unsigned)a.batch, a.advance ? 1u : (unsigned)((2 * a.num_kv_heads + 4 * waves - 1) / (4 * waves))), block((unsigned)threads);
    if (a.head_dim == 64) hipLaunchKernelGGL(kv8_append<64>, grid, block, 0, s, a);
    else if (a.head_dim == 128) hipLaunchKernelGGL(kv8_append<128>, grid, block, 0, s, a);
    else if (a.head_dim == 256) hipLaunchKernelGGL(kv8_append<256>, grid, block, 0, s, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

hipError_t launch_kv8_append_tokens(const CodesArgs &a, hipStream_t s)
{
    if (a.batch == 0 || a.total_tokens == 0) return hipSuccess;
    if (a.head_dim == 64) return append_tokens<64>(a, s);
    if (a.head_dim == 128) return append_tokens<128>(a, s);
    if (a.head_dim == 256) return append_tokens<256>(a, s);
    return hipErrorInvalidValue;
}

hipError_t launch_kv_read_tokens(const CodesArgs &a, int form, void *k_out, void *v_out, hipStream_t s)
{
    if (a.batch == 0 || a.total_tokens == 0) return hipSuccess;
    const dim3 grid((unsigned)((a.total_tokens >> 4) + 2 * a.batch), (unsigned)a.num_kv_heads), block(kThreads);
    uint16_t *k = static_cast<uint16_t *>(k_out), *v = static_cast<uint16_t *>(v_out);
    if (form == LAMPS_LAYOUT_CODES) {
        if (a.head_dim == 64) hipLaunchKernelGGL(kv8_read_tokens<64>, grid, block, 0, s, a, k, v);
        else if (a.head_dim == 128) hipLaunchKernelGGL(kv8_read_tokens<128>, grid, block, 0, s, a, k, v);
        else if (a.head_dim == 256) hipLaunchKernelGGL(kv8_read_tokens<256>, grid, block, 0, s, a, k, v);
        else return hipErrorInvalidValue;
    } else if (!a.bf16) {
        hipLaunchKernelGGL((kv_read_tokens<float, false>), grid, block, 0, s, a, static_cast<float *>(k_out), static_cast<float *>(v_out));
    } else if (form == LAMPS_LAYOUT_TILED) {
        hipLaunchKernelGGL((kv_read_tokens<uint16_t, true>), grid, block, 0, s, a, k, v);
    } else {
        hipLaunchKernelGGL((kv_read_tokens<uint16_t, false>), grid, block, 0, s, a, k, v);
    }
    return hipGetLastError();
}

}  // namespace lamps
