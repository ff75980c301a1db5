// Attention of many new tokens per request over a cache of 8 bits, everything up to each one's own position or a window of it and its first positions.
//
//   out[n] = softmax(q[n] K^T * scale) V  over the positions t <= p with t > p - window or t < sinks, K and V the numbers that the codes stand for
//
// One workgroup = one (request, kv head, tile of new tokens), or one of the parts of its walk: four waves of kCB blocks of 16 columns, (new token, head-of-group)
// pairs.  A stage is 32 cached positions: their codes are converted once, on the way into LDS, by all four waves, to the operands of the
// products that every wave reads (by each wave for itself it would be 64 conversions a stage and wave at head size 128, half as much again as the softmax takes of the
// vector ALUs).  Codes of a later stage are in registers meanwhile.  The softmax keeps a running maximum that moves only
// where a weight would pass 2^8; weights are rounded to bf16 for the second product and summed as rounded.
//
// Bound, where walks are long, by the issue of products, softmax and conversions on two waves to a SIMD: 2 prompts of 8 192, 32 / 8 heads of 128, 955 to 1 010 us by the card, 1.09 to 1.15 PFLOP/s, the
// matrix cores busy 0.48 of it, the vector ALUs 0.45, LDS 0.40 (a large bf16 product of the library on the same card 1.14 to 1.28; the same attention over bf16, which has nothing to convert,
// 880 to 910 us); 4 of 4 096 517 to 534 (475 to 494).  Short walks by a tile's beginning, three round trips, 4 us, and its stores: 24 prompts of 16 to 700 on 40 plain heads 105 to 109 us, of which 54 are
// their bytes (over bf16 110).  12 responses of 4 to 64 tokens on 300 to 30 000, 32 / 8 heads, 78 to 81 us (over bf16 575).  Heads of 256, one product to a read of LDS: 2 prompts of 4 096, 16 / 4 heads,
// 400 us, LDS busy 0.47 of it and the matrix cores 0.28; 4 of 1 024 84 us, 0.27 and 0.15, with 1.3 of 2 waves to a SIMD.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_reducers.h"
#include "handover.h"
#include "internal.h"
#include "kv8.h"
#include "kv8_cut.h"
#include "requests.h"
#include "tile_parts.h"
#include "kv8_decode.h"

namespace lamps {
namespace {

struct Tiling {
    int items;                                           // parts that there is room for
    int log2_places;                                     // 2^it: workgroups that all work is dealt to evenly where requests are cut; -1: none is
    int later;                                           // parts are added up by a second launch
};
// Requests of a launch that cuts: a lane holds four.  (257 of 4 to 32 tokens, 32 / 8 heads, one of them 40 on 30 000: 645 us, which no other workgroup shares, where 256 take 82; by lanes that hold
// sixteen 108, but 69 in place of 53 where all are short, and 400 of them 101 in place of 75.)
constexpr int kMostRequests = 256;

// What a workgroup takes.
struct TilePiece {
    int r, g, tile, first, n_new, ctx;                   // the tile's tokens: rows first + tile * WT and up of n_new
    int runs, at, item;                                  // part `at` of up to `runs`; the item of the first
};

// Sum of whole numbers below 2^48 over the lanes of a wave, in all of them.
__device__ __forceinline__ uint64_t wave_sum(uint64_t x)
{
    const int low = wave_scan((int)(x & 0xFFFFFF)), high = wave_scan((int)(x >> 24));
    return ((uint64_t)(unsigned)__builtin_amdgcn_readlane(high, 63) << 24) + (unsigned)__builtin_amdgcn_readlane(low, 63);
}

// How a launch that cuts divides its work (kv8_cut.h), by every wave for itself, K consecutive requests per lane.
template <int K, bool WINDOW>
struct TilePlan {
    bool any;                                            // request's tiles may be cut
    int first[K], count[K], ctx[K], tiles[K], runs[K];   // first row, new tokens, length; tiles, and parts of each (1: not cut)

    __device__ __forceinline__ TilePlan(const WindowArgs &w, const Tiling &c, int WT)
    {
        const DecodeArgs &a = w.d;
        const int lane = threadIdx.x & 63;
        int stages[K];
        uint64_t work = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = min(K * lane + k, a.batch - 1);
            first[k] = w.q_start[i];
            count[k] = w.q_start[i + 1];
            ctx[k] = a.ctx_lens[i];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            count[k] -= first[k];
            // (a context shorter than its new tokens, or longer than the table row: nothing is read or written for it; rows past the last: none)
            const bool on = K * lane + k < a.batch && first[k] >= 0 && count[k] > 0 && ctx[k] >= count[k] && ctx[k] <= a.max_blocks * a.block_size;
            const int rows = on ? min(count[k], w.total_tokens - first[k]) : 0;
            tiles[k] = max(0, (rows + WT - 1) / WT);
            const int p = ctx[k] - count[k] + rows;      // (the last tile's end, and what its first token sees)
            if constexpr (WINDOW) stages[k] = tiles[k] > 0 ? Sight<32>(p, max(0, p - min(rows, WT) - w.window + 1), w.sinks, std::true_type{}).units : 0;
            else stages[k] = tiles[k] > 0 ? (p + 31) / 32 : 0;
            work += cut8::work_of(stages[k], tiles[k]);
        }
        any = false;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            runs[k] = 1;
            any |= __any(stages[k] > cut8::least_cut(cut8::kLeastStages, c.later)) != 0;
        }
        if (!any) return;                                // (short walks: whatever the share is)
        int size = cut8::first_size(wave_sum(work), a.num_kv_heads, c.log2_places);
        const int least = cut8::least_cut(size, c.later);
        any = false;
#pragma unroll
        for (int k = 0; k < K; ++k) any |= __any(stages[k] > least) != 0;
        if (!any) return;                                // (most launches of many tiles)
        for (int tries = c.later ? cut8::kTries : 0;; --tries) {
            const int worth = c.later ? size : least;
            int sum = 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                runs[k] = cut8::runs_of(stages[k], size, worth);
                sum += tiles[k] * runs[k];
            }
            if (tries == 0 || __builtin_amdgcn_readlane(wave_scan(sum), 63) * a.num_kv_heads <= 1 << c.log2_places) break;
            size = cut8::next_size(size);
        }
    }
    __device__ __forceinline__ bool cut(int k) const { return runs[k] > 1; }
    // Request k of lane l.
    __device__ __forceinline__ void take(int k, int l, TilePiece &x) const
    {
        x.r = K * l + k;
        x.first = __builtin_amdgcn_readlane(first[k], l);
        x.n_new = __builtin_amdgcn_readlane(count[k], l);
        x.ctx = __builtin_amdgcn_readlane(ctx[k], l);
        x.runs = __builtin_amdgcn_readlane(runs[k], l);
    }
};
// The number of request (k of lane l) that `at` falls to, `at` of its own then: mine[k] of each.
template <int K>
__device__ __forceinline__ bool find_request(const int (&mine)[K], int &at, int &k_of, int &l_of)
{
    int own = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) own += mine[k];
    const int upto = wave_scan(own);
    if (at >= __builtin_amdgcn_readlane(upto, 63)) return false;
    l_of = __popcll(__ballot(upto <= at));
    at -= __builtin_amdgcn_readlane(upto - own, l_of);
    k_of = -1;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int n = __builtin_amdgcn_readlane(mine[k], l_of);
        if (k_of < 0) {
            if (at < n) k_of = k; else at -= n;
        }
    }
    return true;
}
// The piece'th of all parts, cut requests' first, of each request the longest tile first.
template <int K, bool WINDOW>
__device__ __forceinline__ bool find_tile(const WindowArgs &w, const Tiling &c, int WT, int piece, TilePiece &x)
{
    const TilePlan<K, WINDOW> plan(w, c, WT);
    int cuts[K], others[K], sum = 0, at = piece, k_of = 0, l_of = 0;
    if (!plan.any) {
        if (!find_request<K>(plan.tiles, at, k_of, l_of)) return false;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k == k_of) {
                plan.take(k, l_of, x);
                x.runs = 1;
                x.at = 0;
                x.item = piece;
                x.tile = __builtin_amdgcn_readlane(plan.tiles[k], l_of) - 1 - at;
            }
        return true;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        cuts[k] = plan.cut(k) ? plan.tiles[k] * plan.runs[k] : 0;
        others[k] = plan.cut(k) ? 0 : plan.tiles[k];
        sum += cuts[k];
    }
    const int all = __builtin_amdgcn_readlane(wave_scan(sum), 63);
    if (piece >= all) at -= all;
    if (!(piece < all ? find_request<K>(cuts, at, k_of, l_of) : find_request<K>(others, at, k_of, l_of))) return false;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (k == k_of) {
            plan.take(k, l_of, x);
            const int t = (int)((unsigned)at / (unsigned)x.runs);
            x.at = at - t * x.runs;
            x.item = piece - x.at;
            x.tile = __builtin_amdgcn_readlane(plan.tiles[k], l_of) - 1 - t;
        }
    return true;
}
// The nth tile that is cut: its request, and the number of its first part.
template <int K, bool WINDOW>
__device__ __forceinline__ bool find_cut_tile(const WindowArgs &w, const Tiling &c, int WT, int nth, TilePiece &x)
{
    const TilePlan<K, WINDOW> plan(w, c, WT);
    int cuts[K], own = 0, at = nth, k_of = 0, l_of = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        cuts[k] = plan.cut(k) ? plan.tiles[k] : 0;
        own += cuts[k] * plan.runs[k];
    }
    if (!find_request<K>(cuts, at, k_of, l_of)) return false;
    int before = __builtin_amdgcn_readlane(wave_scan(own) - own, l_of);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (k < k_of) before += __builtin_amdgcn_readlane(cuts[k] * plan.runs[k], l_of);
        if (k == k_of) {
            plan.take(k, l_of, x);
            x.at = 0;
            x.item = before + at * x.runs;
            x.tile = __builtin_amdgcn_readlane(plan.tiles[k], l_of) - 1 - at;
        }
    }
    return true;
}
// Without: any number of requests, none cut.
__device__ __forceinline__ bool find_whole_tile(const WindowArgs &w, int WT, int piece, TilePiece &x)
{
    const DecodeArgs &a = w.d;
    const NewTokens n = new_tokens_at(w.q_start, a.ctx_lens, a.batch, piece, [WT](int q, int r) { return q / WT + r; });
    x.r = __builtin_amdgcn_readfirstlane(n.r);
    x.first = __builtin_amdgcn_readfirstlane(n.first);
    x.n_new = __builtin_amdgcn_readfirstlane(n.count);
    x.ctx = __builtin_amdgcn_readfirstlane(n.ctx);
    x.tile = __builtin_amdgcn_readfirstlane(piece - (x.first / WT + x.r));
    x.runs = 1;
    x.at = 0;
    x.item = piece;
    if (x.first < 0 || x.tile < 0 || x.ctx < x.n_new || x.ctx > a.max_blocks * a.block_size) return false;
    return (long long)x.tile * WT < min(x.n_new, w.total_tokens - x.first);
}

constexpr size_t tile_state(int D, int columns) { return (size_t)columns * (D + 2); }   // floats

template <int D, int kCB, int PS, bool WINDOW>
__global__ __launch_bounds__(kThreads, D >= 256 && kCB > 1 ? 1 : 2) void kv8_tiles(const WindowArgs w, const Tiling c)
{
    constexpr int kCols = 16 * kCB, CG = kWaves / PS, NK = D / 32, NS = D / 16;   // columns of a wave; waves with columns of their own
    constexpr int SUBK = 16 * D * 2, VOFF = 2 * SUBK, STAGE = 4 * SUBK;   // bytes of a sub-tile of keys, where values begin, of a stage
    constexpr bool kHold = D <= 128;                     // operands of a stage are held in registers
    constexpr int RING = kHold && PS == 1 ? 4 : 2;       // rounds that there are buffers for
    __shared__ __align__(16) char lds[RING * PS * STAGE];
    constexpr int SUBS = D == 256 ? 2 : 1, KINDS = D == 64 ? 1 : 2;   // of a thread's units: sub-tiles, keys and values
    __shared__ uint32_t wild_at[RING * PS][kWaves * SUBS];

    const DecodeArgs &a = w.d;
    const int G = a.num_q_heads / a.num_kv_heads, TW = kCols / G, WT = CG * TW;
    TilePiece at;
    // (heads next to each other: with 8 of them and more all tiles of one go to one XCD, whose L2 has its keys and values)
    const int piece = __builtin_amdgcn_readfirstlane((int)((unsigned)blockIdx.x / (unsigned)a.num_kv_heads));
    at.g = blockIdx.x - piece * a.num_kv_heads;
    if (c.log2_places < 0 ? !find_whole_tile(w, WT, piece, at) : a.batch <= 64 ? !find_tile<1, WINDOW>(w, c, WT, piece, at) : !find_tile<4, WINDOW>(w, c, WT, piece, at)) return;
    const int g = at.g, first = at.first, base_pos = at.ctx - at.n_new, n_new = min(at.n_new, w.total_tokens - first);
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 15, qd = lane >> 4;

    // what the tile walks over, and the part of it that is this workgroup's
    const int p_first = base_pos + at.tile * WT, p_last = base_pos + min(n_new, (at.tile + 1) * WT) - 1;
    const Sight<32> see = WINDOW ? Sight<32>(p_last + 1, max(0, p_first - w.window + 1), w.sinks, std::true_type{}) : Sight<32>(p_last + 1, 0, 0, std::true_type{});
    const auto position = [&](int st) { return WINDOW ? see.at(st) : st * 32; };
    int st0 = 0, st1 = see.units, runs = 1;
    if (at.runs > 1) {
        const cut8::Parts parts = cut8::parts_of(see.units, at.runs);
        runs = parts.count;
        if (at.at >= runs) return;
        st0 = at.at * parts.each;
        st1 = min(see.units, st0 + parts.each);
    }
    st0 = __builtin_amdgcn_readfirstlane(st0);
    st1 = __builtin_amdgcn_readfirstlane(st1);
    // the wave's own tokens; none: positions that see nothing
    const int cg = wv / PS, ps = wv % PS;                // its columns, and which of PS stages it takes
    const int wave_tok = at.tile * WT + cg * TW;
    const bool none = wave_tok >= n_new;
    const int wave_min = __builtin_amdgcn_readfirstlane(none ? 0x3fffffff : base_pos + wave_tok);
    const int wave_max = __builtin_amdgcn_readfirstlane(none ? -1 : base_pos + min(n_new, wave_tok + TW) - 1);
    const int wave_hi = wave_max - w.window + 1, wave_lo = wave_min - w.window + 1;   // where the windows of the wave's last and first token begin

    // Thread's units of a stage, 16 bytes of codes.  Heads of 128: a wave half of a sub-tile's keys and the same of its values; of 64: its keys or its values; of
    // 256: a quarter of both sub-tiles' of both.
    const int wave_sub = D == 64 ? wv & 1 : D == 128 ? wv >> 1 : 0, wave_kind = D == 64 ? wv >> 1 : 0;
    const int u = D == 64 ? lane : D == 128 ? (wv & 1) * 64 + lane : tid;   // of the sub-tile
    const table_ptr table = (table_ptr)(uintptr_t)(a.block_table + (size_t)at.r * a.max_blocks);
    const uint32_t tile_bytes = (uint32_t)a.block_size * D, slice = (uint32_t)codes_slice(a.num_kv_heads, a.block_size, D), stride = a.num_layers * slice;   // (the launcher has checked that it fits)
    const char *k0 = static_cast<const char *>(a.k_pool) + (size_t)a.layer * slice;
    const char *kp = k0 + (size_t)g * tile_bytes, *vp = static_cast<const char *>(a.v_pool) + (size_t)a.layer * slice + (size_t)g * tile_bytes;
    const char *sp = k0 + (size_t)a.num_kv_heads * tile_bytes + g * 8;
    const uint32_t last_block = (uint32_t)a.num_blocks - 1, u16 = u * 16;
    const int last_stage = see.units - 1, in_block = (a.block_size - 1) & ~15;
    struct Places {
        uint32_t block[SUBS], at[SUBS];                  // where a sub-tile is: a block, and where in its tile
    };
    const auto lookup = [&](int st) __attribute__((always_inline)) {
        const int t = position(min(st, last_stage));
        Places x;
#pragma unroll
        for (int i = 0; i < SUBS; ++i) {
            const int sub = SUBS == 2 ? i : wave_sub;
            int p;
            if constexpr (WINDOW) {
                const int2 both = sub_tiles(see, t);
                p = sub ? both.y : both.x;
            } else {
                p = t + 16 * sub < see.end ? t + 16 * sub : t;
            }
            x.block[i] = (uint32_t)table[p >> a.log2_block_size];
            x.at[i] = (uint32_t)(p & in_block) * D;
        }
        return x;
    };
    struct Codes {
        uint4 raw[SUBS][KINDS];
        float2 scale[SUBS];
    };
    const auto load = [&](const Places &x, Codes &y) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < SUBS; ++i) {
            // (an entry that names no block of the pool reads the last one: the rows are meaningless.  Not looked at before it is used: nothing waits for it)
            const uint64_t block = (uint64_t)min(x.block[i], last_block) * stride, off = block + x.at[i];
            y.scale[i] = __builtin_bit_cast(float2, *(scales_ptr)(uintptr_t)(sp + block));
            if constexpr (KINDS == 2) {
                y.raw[i][0] = *reinterpret_cast<const uint4 *>(kp + off + u16);
                y.raw[i][1] = *reinterpret_cast<const uint4 *>(vp + off + u16);
            } else {
                y.raw[i][0] = *reinterpret_cast<const uint4 *>((wave_kind ? vp : kp) + off + u16);
            }
        }
    };
    // Converts them to operands.  Values behind the tile's last position, which the cache may hold anything at, and those of a sub-tile that no token sees,
    // become zeros; whether one that is left is NaN matters where a stage is not seen by all.
    const int wg_min = p_first, wg_hi = p_last - w.window + 1;
    const uint32_t key_to = (u >> 4) * 512 + (u & 15) * 16, value_to = VOFF + ((u >> 6) * 256 + (u >> 4 & 3) * 16 + (u & 15)) * 16;
    const auto put = [&](int st, int buf, const Codes &from) __attribute__((always_inline)) {
        char *to = lds + buf * STAGE;
        const int t0 = position(min(st, last_stage));
        const bool edge = (t0 + 31 > wg_min) | (WINDOW && t0 < wg_hi);
#pragma unroll
        for (int i = 0; i < SUBS; ++i)
#pragma unroll
            for (int k = 0; k < KINDS; ++k) {
                const int sub = SUBS == 2 ? i : wave_sub;
                const uint4 y = from.raw[i][k];
                if (KINDS == 2 ? k == 0 : wave_kind == 0) {
                    const float s = from.scale[i].x;
                    uint4 *p = reinterpret_cast<uint4 *>(to + sub * SUBK + key_to);
                    p[0] = make_uint4(from_codes<false>(y.x, s), from_codes<true>(y.x, s), from_codes<false>(y.y, s), from_codes<true>(y.y, s));
                    p[16] = make_uint4(from_codes<false>(y.z, s), from_codes<true>(y.z, s), from_codes<false>(y.w, s), from_codes<true>(y.w, s));
                } else {
                    const float s = from.scale[i].y;
                    uint32_t x[4] = {y.x, y.y, y.z, y.w};
                    if (edge) {                          // uniform
                        int left = see.end - (t0 + 16 * sub + (u >> 4 & 3) * 4);   // of the unit's four positions
                        if constexpr (WINDOW) {
                            const int2 both = sub_tiles(see, t0);
                            if ((sub ? both.y : both.x) != t0 + 16 * sub) left = 0;
                        }
                        const uint32_t keep = left >= 4 ? 0xFFFFFFFFu : left <= 0 ? 0u : ~(0xFFFFFFFFu << (8 * left));
                        bool bad = false;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[e] &= keep;
                            bad |= any_nan(x[e]);
                        }
                        const bool any = __any(bad);
                        if (lane == 0) wild_at[buf][kWaves * i + wv] = any;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *reinterpret_cast<uint2 *>(to + value_to + e * 1024 + sub * 8) = make_uint2(from_codes<false>(x[e], s), from_codes<true>(x[e], s));
                }
            }
    };

    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < SUBS; ++i) for (int k = 0; k < RING * PS; ++k) wild_at[k][kWaves * i + wv] = 0;
    }
    // A round of the walk is PS stages, one for each of the waves that share columns.  Codes are asked for a round ahead of their conversion, the first in front of the
    // queries (two rounds ahead was no faster with two buffers: 12 responses 84 us, 2 prompts of 8 192 1 008, either way).
    Places next[PS];
    Codes codes[PS], early[RING == 4 ? 2 : 1][PS];
    const auto lookup_round = [&](int st) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < PS; ++k) next[k] = lookup(st + k);
    };
    const auto load_round = [&](Codes (&x)[PS]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < PS; ++k) load(next[k], x[k]);
    };
    const auto put_round = [&](int st, int buf, const Codes (&x)[PS]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < PS; ++k) put(st + k, buf * PS + k, x[k]);
    };
    if (st0 < st1) {
        lookup_round(st0);
        load_round(codes);
        lookup_round(st0 + PS);
        if constexpr (RING == 4) {
            load_round(early[0]);
            lookup_round(st0 + 2 * PS);
            load_round(early[1]);
            lookup_round(st0 + 3 * PS);
        }
    }

    // this lane's column in each block: (token, head), its position, its queries (of a negative scale: their negatives)
    int pos[kCB];
    size_t orow[kCB];
    bf16x8 qb[kCB][NK];
    const float scale = fabsf(a.scale_log2e);
    const uint32_t flip = a.scale_log2e < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int b = 0; b < kCB; ++b) {
        const int col = b * 16 + j, tl = col / G, hd = col - tl * G, tok = wave_tok + tl;
        const bool ok = col < TW * G && tok < n_new;
        pos[b] = ok ? base_pos + tok : -1;
        orow[b] = ((size_t)(first + (ok ? tok : 0)) * a.num_q_heads + g * G + hd) * D;
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            uint4 t = make_uint4(0, 0, 0, 0);
            if (ok) t = *reinterpret_cast<const uint4 *>(static_cast<const char *>(a.q) + (orow[b] + 32 * i + 8 * qd) * 2);
            t.x ^= flip; t.y ^= flip; t.z ^= flip; t.w ^= flip;
            qb[b][i] = __builtin_bit_cast(bf16x8, t);
        }
    }
    float m[kCB];
    f32x4 o[kCB][NS], l[kCB];
#pragma unroll
    for (int b = 0; b < kCB; ++b) {
        m[b] = kLeast;
        l[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) o[b][s] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));

    f32x4 sc0[kCB], sc1[kCB];                            // scores: positions t + 4 qd + e and t + 16 + 4 qd + e of the lane's column
    bf16x8 pw[kCB];
    // Position p sees t + 4 qd + e: e <= lim and (e > lim - window or e < sinks - t - 4 qd), lim = p - t - 4 qd.
    const auto visible = [&](int p, int t, int e) {
        const int lim = p - t - 4 * qd;
        return WINDOW ? (e <= lim) & ((e > lim - w.window) | (e < w.sinks - t - 4 * qd)) : e <= lim;
    };
    // The weights of block b, by the reference that it has; the largest of them, found by packed maxima of pairs: they are not negative, so their bits compare as
    // they do, and as those of fp16 numbers.  One of 2^kSlack and more, or no finite one, asks for another reference: rare after the first stages.
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    const auto weigh = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            pw[b][e] = (__bf16)fast_exp2(fmaf(sc0[b][e], scale, -m[b]));
            pw[b][4 + e] = (__bf16)fast_exp2(fmaf(sc1[b][e], scale, -m[b]));
        }
        uint4 y = __builtin_bit_cast(uint4, pw[b]);
        asm("" : "+v"(y.x), "+v"(y.y), "+v"(y.z), "+v"(y.w));   // (pairs from here on: carried over the branch one by one, they are converted twice)
        pw[b] = __builtin_bit_cast(bf16x8, y);
        uint32_t most;
        asm("v_pk_maximum3_f16 %0, %1, %2, %3" : "=v"(most) : "v"(y.x), "v"(y.y), "v"(y.z));
        asm("v_pk_maximum3_f16 %0, %1, %2, %2" : "=v"(most) : "v"(most), "v"(y.w));
        return most;
    };
    const auto over = [](uint32_t most) {
        constexpr unsigned short kBelow = ((127 + (int)kSlack) << 7) - 1;   // the bf16 in front of 2^kSlack
        return __any(__builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, most), u16x2{kBelow, kBelow})) != 0);
    };
    const auto softmax = [&](int t0, bool masked) __attribute__((always_inline)) {
        if (masked) {
#pragma unroll
            for (int b = 0; b < kCB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!visible(pos[b], t0, e)) sc0[b][e] = -INFINITY;
                    if (!visible(pos[b], t0 + 16, e)) sc1[b][e] = -INFINITY;
                }
        }
        uint32_t most[kCB], all = 0;
#pragma unroll
        for (int b = 0; b < kCB; ++b) {
            most[b] = weigh(b);
            if (b == 0) all = most[0];
            else asm("v_pk_maximum3_f16 %0, %1, %2, %2" : "=v"(all) : "v"(all), "v"(most[b]));
        }
        if (over(all)) {                                 // wave-uniform
#pragma unroll
            for (int b = 0; b < kCB; ++b) {
                if (kCB > 1 && !over(most[b])) continue;
                float mx = sc0[b][0];                    // (the median with infinity: the maximum)
#pragma unroll
                for (int e = 1; e < 8; ++e) mx = __builtin_amdgcn_fmed3f(mx, e < 4 ? sc0[b][e & 3] : sc1[b][e & 3], INFINITY);
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale;
                const float mn = mx - m[b] > kSlack ? mx : m[b], f = fast_exp2(m[b] - mn);
                m[b] = mn;
#pragma unroll
                for (int e = 0; e < 4; ++e) l[b][e] *= f;
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[b][s][e] *= f;
                weigh(b);
            }
        }
    };

    // A value that is NaN must not reach the columns that do not see it, and a zero weight does not silence it: where a stage that is seen in part has one,
    // the products are taken without, and those of (is NaN) by (is seen) tell which outputs it makes NaN.
    const auto set_apart = [&](int s, int t0, uint4 &v) __attribute__((always_inline)) {
        uint32_t x[4] = {v.x, v.y, v.z, v.w}, is[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t nan = ((((x[k] & 0x7FFF7FFFu) + 0x007F007Fu) & 0x80008000u) >> 15) * 0xFFFFu;
            x[k] &= ~nan;
            is[k] = nan & 0x3F803F80u;
        }
        v = make_uint4(x[0], x[1], x[2], x[3]);
#pragma unroll
        for (int b = 0; b < kCB; ++b) {
            uint32_t y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = k < 2 ? t0 : t0 + 16;
                y[k] = (visible(pos[b], t, 2 * (k & 1)) ? 0x3F80u : 0u) | (visible(pos[b], t, 2 * (k & 1) + 1) ? 0x3F800000u : 0u);
            }
            const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(is[0], is[1], is[2], is[3]), operand(y[0], y[1], y[2], y[3]), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[b][s][e] += hit[e] > 0.0f ? __uint_as_float(0x7FC00000u) : 0.0f;
        }
    };

    // Operands of keys for the stage at hand are in registers where its iteration begins, those of values are asked for in front of its products
    // (heads of 256: both where they are used, for want of registers).  Behind the softmax a barrier: everyone has what the stage's buffer held, and the next one is
    // whole; the next keys are read, and a later stage is converted, while the matrix cores multiply values.  With four buffers a barrier in every second round does: the third round
    // ahead is converted into the buffer that two rounds, and a barrier since, have left (two buffers and a barrier a round / so: 2 prompts of 8 192, 32 / 8 heads, 993 us and 970, 24 of 16 to
    // 700 on 40 plain ones 115 and 111).
    bf16x8 kop[kHold ? NK : 1][2];
    uint4 vheld[kHold ? NS : 1];
    const char *mine = lds + lane * 16;                  // (unit qd * 16 + j)
    const auto key = [&](const char *buf, int i, int h) { return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(buf + h * SUBK + i * 1024)); };
    const auto read_k = [&](const char *buf) __attribute__((always_inline)) {
        if constexpr (kHold) {
#pragma unroll
            for (int i = 0; i < NK; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) kop[i][h] = key(buf, i, h);
        }
    };
    if (st0 < st1) {
        put_round(st0, 0, codes);
        if constexpr (RING == 4) {
            put_round(st0 + PS, 1, early[0]);
            put_round(st0 + 2 * PS, 2, early[1]);
            load_round(codes);
            lookup_round(st0 + 4 * PS);
        } else if constexpr (kHold) {
            load_round(codes);
            lookup_round(st0 + 2 * PS);
            put_round(st0 + PS, 1, codes);               // (past the last stage: the last one once more, which nobody reads)
            load_round(codes);
            lookup_round(st0 + 3 * PS);
        } else {
            load_round(codes);
            lookup_round(st0 + 2 * PS);
        }
    }
    if constexpr (kHold) {
        __syncthreads();
        if (st0 < st1) read_k(mine + ps * STAGE);
    }
    // The round from stage rd on, whose buffer is `cur`; past the last stage the last one is converted once more, which nobody reads.
    const auto round = [&](int rd, auto parity) __attribute__((always_inline)) {
        constexpr int cur = parity;
        if constexpr (!kHold) {
            __syncthreads();
            put_round(rd + PS, cur ^ 1, codes);
            load_round(codes);
            lookup_round(rd + 3 * PS);
        }
        const int st = rd + ps;
        const char *buf = mine + (cur * PS + ps) * STAGE;
        const int t0 = position(PS > 1 ? min(st, last_stage) : st);
        const bool live = (t0 <= wave_max) & (!WINDOW | (t0 + 31 >= wave_lo) | (t0 < w.sinks)) & (PS == 1 | st < st1);   // uniform over the wave, as what follows
        const bool masked = !((t0 + 31 <= wave_min) & (!WINDOW | (t0 >= wave_hi) | (t0 + 32 <= w.sinks)));
        const auto values = [&](int s) { return *reinterpret_cast<const uint4 *>(buf + VOFF + s * 1024); };
        const auto vop = [&](int s) { return kHold ? vheld[kHold ? s : 0] : values(s); };
        bool apart = false;
        if (live) {
            if constexpr (kHold) {
#pragma unroll
                for (int s = 0; s < NS; ++s) vheld[s] = values(s);
            }
#pragma unroll
            for (int b = 0; b < kCB; ++b) sc0[b] = sc1[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                const bf16x8 ka = kHold ? kop[kHold ? i : 0][0] : key(buf, i, 0), kb = kHold ? kop[kHold ? i : 0][1] : key(buf, i, 1);
#pragma unroll
                for (int b = 0; b < kCB; ++b) {
                    sc0[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qb[b][i], sc0[b], 0, 0, 0);
                    sc1[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qb[b][i], sc1[b], 0, 0, 0);
                }
            }
            // (they are there before the way parts: see window_attn.hip)
            if constexpr (kCB == 1) asm volatile("s_nop 7" : "+v"(sc0[0]), "+v"(sc1[0]));
            else asm volatile("s_nop 7" : "+v"(sc0[0]), "+v"(sc1[0]), "+v"(sc0[1]), "+v"(sc1[1]));
            softmax(t0, masked);
            if (masked) {
                uint32_t any = 0;
#pragma unroll
                for (int k = 0; k < kWaves * SUBS; ++k) any |= wild_at[cur * PS + ps][k];
                apart = __builtin_amdgcn_readfirstlane(any) != 0;
            }
            if constexpr (kHold) {
                if (apart) {
#pragma unroll
                    for (int s = 0; s < NS; ++s) set_apart(s, t0, vheld[s]);
                }
            }
        }
        if constexpr (kHold) {
            if (RING == 2 || (cur & 1)) __syncthreads();
            read_k(mine + ((cur + 1) % RING * PS + ps) * STAGE);
            constexpr int far = RING == 4 ? 3 : 2;
            put_round(rd + far * PS, (cur + far) % RING, codes);
            load_round(codes);
            lookup_round(rd + (far + 2) * PS);
        }
        if (!live) return;
#pragma unroll
        for (int b = 0; b < kCB; ++b) l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pw[b], l[b], 0, 0, 0);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            uint4 v = vop(s);
            if (!kHold && apart) set_apart(s, t0, v);    // uniform
#pragma unroll
            for (int b = 0; b < kCB; ++b) o[b][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), pw[b], o[b][s], 0, 0, 0);
        }
    };
    // (heads of 256: the first round is converted by itself, and the second's codes come first)
    for (int rd = st0; rd < st1; rd += RING * PS) {
        round(rd, std::integral_constant<int, 0>{});
        if (rd + PS < st1) round(rd + PS, std::integral_constant<int, 1>{});
        if constexpr (RING == 4) {
            if (rd + 2 * PS < st1) round(rd + 2 * PS, std::integral_constant<int, 2>{});
            if (rd + 3 * PS < st1) round(rd + 3 * PS, std::integral_constant<int, 3>{});
        }
    }
    // (the last products are there before what adds them up or stores them: see window_tiles.h)
    asm volatile("s_nop 7" ::: "memory");
#pragma unroll
    for (int b = 0; b < kCB; ++b) asm volatile("" : "+v"(l[b]), "+v"(o[b][NS - 1]));

    if constexpr (PS > 1) {
        // the waves of the same columns: their states through LDS to the first of them
        constexpr int kState = kCols * (D + 2) * 4;      // bytes
        static_assert(CG * (PS - 1) * kState <= 2 * PS * STAGE, "the states fit into the stages' place");
        __syncthreads();
        char *there = lds + (cg * (PS - 1) + ps - 1) * kState + lane * 16;
        if (ps > 0 && !none) {
#pragma unroll
            for (int b = 0; b < kCB; ++b) {
#pragma unroll
                for (int s = 0; s < NS; ++s) *reinterpret_cast<f32x4 *>(there + (b * NS + s) * 1024) = o[b][s];
                if (qd == 0) *reinterpret_cast<float2 *>(there - lane * 16 + kCols * D * 4 + (b * 16 + j) * 8) = make_float2(m[b], l[b][0]);
            }
        }
        __syncthreads();
        if (ps == 0 && !none) {
#pragma unroll
            for (int k = 0; k < PS - 1; ++k)
#pragma unroll
                for (int b = 0; b < kCB; ++b) {
                    const char *from = lds + (cg * (PS - 1) + k) * kState;
                    const float2 ml = *reinterpret_cast<const float2 *>(from + kCols * D * 4 + (b * 16 + j) * 8);
                    const float Mn = fmaxf(m[b], ml.x), f0 = fast_exp2(m[b] - Mn), f = fast_exp2(ml.x - Mn);
                    m[b] = Mn;
                    l[b][0] = l[b][0] * f0 + ml.y * f;
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const f32x4 y = *reinterpret_cast<const f32x4 *>(from + lane * 16 + (b * NS + s) * 1024);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[b][s][e] = o[b][s][e] * f0 + y[e] * f;
                    }
                }
        }
    }
    const bool holds = ps == 0 && !none;                 // the wave has a state to hand on
    if (runs == 1) {
        if (PS > 1 && !holds) return;
#pragma unroll
        for (int b = 0; b < kCB; ++b) store_column<NS>(static_cast<uint16_t *>(a.out) + orow[b], qd, pos[b] >= 0, 1.0f / l[b][0], o[b]);
        return;
    }
    // the columns of each block as the wave holds them, and their (reference, sum); the last part to arrive adds them up, or a second launch
    constexpr int kAll = CG * kCols;
    constexpr size_t state = tile_state(D, kAll);
    const size_t item = (size_t)at.item * a.num_kv_heads + g, step = (size_t)a.num_kv_heads * state;
    float *first_part = a.partials + item * state, *to = first_part + at.at * step;
    if (c.later) {                                       // (a second launch adds them up)
        if (!holds) return;
#pragma unroll
        for (int b = 0; b < kCB; ++b) {
            const int block = cg * kCB + b;
#pragma unroll
            for (int s = 0; s < NS; ++s) *reinterpret_cast<f32x4 *>(to + block * 16 * D + s * 256 + 4 * lane) = o[b][s];
            if (qd == 0) *reinterpret_cast<float2 *>(to + kAll * D + 2 * (block * 16 + j)) = make_float2(m[b], l[b][0]);
        }
        return;
    }
    uint64_t *flags = reinterpret_cast<uint64_t *>(a.partials + (size_t)c.items * state) + item;
    if (holds) {
#pragma unroll
        for (int b = 0; b < kCB; ++b) {
            const int block = cg * kCB + b;
#pragma unroll
            for (int s = 0; s < 2 * NS; ++s)
                put_shared(to + block * 16 * D + s * 128 + 2 * lane, o[b][s >> 1][2 * (s & 1)], o[b][s >> 1][2 * (s & 1) + 1]);
            if (qd == 0) put_shared(to + kAll * D + 2 * (block * 16 + j), m[b], l[b][0]);
        }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();                                     // the workgroup's stores have arrived, and its LDS is free
    int *is_last = reinterpret_cast<int *>(lds);
    if (wv == 0) {
        const bool all = report_run<true>(flags, a.num_kv_heads, at.at, runs, w.tag);
        if (lane == 0) *is_last = all;
    }
    __syncthreads();
    if (!*is_last || !holds) return;
    // the parts in order, whichever workgroup this is: bit-reproducible
#pragma unroll 1
    for (int b = 0; b < kCB; ++b) {
        const int block = cg * kCB + b;
        float M = kLeast, L = 0.0f;
        f32x4 A[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) A[s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int k = 0; k < runs; ++k) {
            const float *from = first_part + k * step;
            const float2 ml = get_shared(from + kAll * D + 2 * (block * 16 + j));
            float2 x[2 * NS];
#pragma unroll
            for (int s = 0; s < 2 * NS; ++s) x[s] = get_shared(from + block * 16 * D + s * 128 + 2 * lane);
            const float Mn = fmaxf(M, ml.x), f0 = fast_exp2(M - Mn), f = fast_exp2(ml.x - Mn);
            L = L * f0 + ml.y * f;
#pragma unroll
            for (int s = 0; s < 2 * NS; ++s) {
                A[s >> 1][2 * (s & 1)] = A[s >> 1][2 * (s & 1)] * f0 + x[s].x * f;
                A[s >> 1][2 * (s & 1) + 1] = A[s >> 1][2 * (s & 1) + 1] * f0 + x[s].y * f;
            }
            M = Mn;
        }
        const int col = b * 16 + j, tl = col / G, tok = wave_tok + tl;
        const bool ok = col < TW * G && tok < n_new;
        store_column<NS>(static_cast<uint16_t *>(a.out) + ((size_t)(first + (ok ? tok : 0)) * a.num_q_heads + g * G + (ok ? col - tl * G : 0)) * D, qd, ok, 1.0f / L, A);
    }
}

// Adds the parts of a tile up behind a launch with `later`: a workgroup takes a block of 16 columns, its waves every fourth part.
template <int D, int kCB, int CG, bool WINDOW>
__global__ __launch_bounds__(kThreads) void kv8_join(const WindowArgs w, const Tiling c)
{
    constexpr int kCols = 16 * kCB, kAll = CG * kCols, NS = D / 16, N = D >= 256 ? 1 : 2, SLABS = D == 64 ? 2 : NS / kWaves;
    __shared__ __align__(16) float sums[kWaves][16 * D];
    __shared__ float2 stats[kWaves][16];
    const DecodeArgs &a = w.d;
    const int G = a.num_q_heads / a.num_kv_heads, TW = kCols / G, WT = CG * TW;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 15, qd = lane >> 4;
    const int nth = __builtin_amdgcn_readfirstlane((int)((unsigned)blockIdx.x / (unsigned)a.num_kv_heads)), g = blockIdx.x - nth * a.num_kv_heads, block = blockIdx.y;
    TilePiece at;
    if (a.batch <= 64 ? !find_cut_tile<1, WINDOW>(w, c, WT, nth, at) : !find_cut_tile<4, WINDOW>(w, c, WT, nth, at)) return;
    const int base_pos = at.ctx - at.n_new, n_new = min(at.n_new, w.total_tokens - at.first), wave_tok = at.tile * WT + block / kCB * TW;
    if (wave_tok >= n_new) return;                       // (the wave had no tokens and has left nothing)
    const int p_first = base_pos + at.tile * WT, p_last = base_pos + min(n_new, (at.tile + 1) * WT) - 1;
    const Sight<32> see(p_last + 1, WINDOW ? max(0, p_first - w.window + 1) : 0, WINDOW ? w.sinks : 0, std::true_type{});
    const int runs = cut8::parts_of(see.units, at.runs).count;
    if (runs == 1) return;                               // (written already)
    constexpr size_t state = tile_state(D, kAll);
    const size_t step = (size_t)a.num_kv_heads * state;
    const float *parts = a.partials + ((size_t)at.item * a.num_kv_heads + g) * state;
    float M = kLeast, L = 0.0f;
    f32x4 A[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) A[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int p0 = wv; p0 < runs; p0 += N * kWaves) {
        float2 ml[N];
        f32x4 y[N][NS];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float *from = parts + (size_t)min(p0 + k * kWaves, runs - 1) * step;
            ml[k] = *reinterpret_cast<const float2 *>(from + kAll * D + 2 * (block * 16 + j));
#pragma unroll
            for (int s = 0; s < NS; ++s) y[k][s] = *reinterpret_cast<const f32x4 *>(from + block * 16 * D + s * 256 + 4 * lane);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (p0 + k * kWaves >= runs) break;          // uniform
            const float Mn = fmaxf(M, ml[k].x), f0 = fast_exp2(M - Mn), f = fast_exp2(ml[k].x - Mn);
            L = L * f0 + ml[k].y * f;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) A[s][e] = A[s][e] * f0 + y[k][s][e] * f;
            M = Mn;
        }
    }
#pragma unroll
    for (int s = 0; s < NS; ++s) *reinterpret_cast<f32x4 *>(&sums[wv][s * 256 + 4 * lane]) = A[s];
    if (qd == 0) stats[wv][j] = make_float2(M, L);
    __syncthreads();
    // each wave some of the outputs, the parts' sums in order
    if (wv * SLABS >= NS) return;
    float2 ml[kWaves];
    M = kLeast;
    L = 0.0f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        ml[k] = stats[k][j];
        M = fmaxf(M, ml[k].x);
    }
    f32x4 B[SLABS];
#pragma unroll
    for (int s = 0; s < SLABS; ++s) B[s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        const float f = fast_exp2(ml[k].x - M);
        L += ml[k].y * f;
#pragma unroll
        for (int s = 0; s < SLABS; ++s) {
            const f32x4 y = *reinterpret_cast<const f32x4 *>(&sums[k][(wv * SLABS + s) * 256 + 4 * lane]);
#pragma unroll
            for (int e = 0; e < 4; ++e) B[s][e] += y[e] * f;
        }
    }
    const int col = block % kCB * 16 + j, tl = col / G, tok = wave_tok + tl;
    const bool ok = col < TW * G && tok < n_new;
    store_column<SLABS>(static_cast<uint16_t *>(a.out) + ((size_t)(at.first + (ok ? tok : 0)) * a.num_q_heads + g * G + (ok ? col - tl * G : 0)) * D + 16 * wv * SLABS, qd, ok, 1.0f / L, B);
}

// A wavefront per token and kv head (or pass), weights as pairs of bf16: for more than 32 heads to a kv head, and where a caller asks for it.
template <int D>
__global__ __launch_bounds__(kThreads, D >= 256 ? 1 : 2) void kv8_rows(const WindowArgs w)
{
    const DecodeArgs &a = w.d;
    const int GH = a.heads_per_pass, HC = a.num_kv_heads * a.passes;
    const long long item = (long long)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= (long long)w.total_tokens * HC) return;
    const int n = (int)(item / HC), hc = (int)(item - (long long)n * HC), h0 = hc * GH;
    const auto [r, first, count, ctx] = new_tokens_at(w.q_start, a.ctx_lens, a.batch, n, [](int q, int) { return q; });
    // (a context shorter than its new tokens, or longer than the table row: nothing is read or written)
    if (n < first || n >= first + count || ctx < count || ctx > a.max_blocks * a.block_size) return;
    const Sight<32> see(__builtin_amdgcn_readfirstlane(ctx - count + (n - first) + 1), w.window, w.sinks);
    uint16_t *out = static_cast<uint16_t *>(a.out) + ((size_t)n * a.num_q_heads + h0) * D;
    CodesReducer<D>::run(a, __builtin_amdgcn_readfirstlane(r), (size_t)n, hc / a.passes, h0, GH, see, 0, see.units, [&](int h, int d, float, float L, const auto &A) {
        const float inv = 1.0f / L;
        *reinterpret_cast<uint2 *>(out + h * D + d) = make_uint2(pack_bf16(A[0] * inv, A[1] * inv), pack_bf16(A[2] * inv, A[3] * inv));
    });
}

template <int D, int kCB, int PS>
hipError_t launch_tiles(const WindowArgs &w, hipStream_t s)
{
    const DecodeArgs &a = w.d;
    constexpr int CG = kWaves / PS;
    const int WT = CG * (16 * kCB / (a.num_q_heads / a.num_kv_heads));
    const long long tiles = (long long)w.total_tokens / WT + a.batch, heads = a.num_kv_heads;
    Tiling c = {0, -1, 0};
    if (a.batch <= kMostRequests) {
        // (parts are fewer than twice the places)
        const long long state = (long long)tile_state(D, CG * 16 * kCB) * (long long)sizeof(float), room = (long long)a.partial_capacity / (state + 8);
        c.log2_places = cut8::kLog2Places;
        while (c.log2_places >= 0 && (2LL << c.log2_places) > room) --c.log2_places;
        c.items = c.log2_places < 0 ? 0 : 2 << c.log2_places;
        c.later = c.log2_places >= 0 && cut8::tiles_later(tiles * heads, cut8::most_seen((long long)a.max_blocks * a.block_size, w.window, w.sinks, WT));
    }
    const long long grid = (tiles * heads + c.items + heads - 1) / heads * heads;
    if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
    const bool window = w.window < (long long)a.max_blocks * a.block_size;
    if (window) hipLaunchKernelGGL((kv8_tiles<D, kCB, PS, true>), dim3((unsigned)grid), dim3(kThreads), 0, s, w, c);
    else hipLaunchKernelGGL((kv8_tiles<D, kCB, PS, false>), dim3((unsigned)grid), dim3(kThreads), 0, s, w, c);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !c.later) return e;
    // (a tile that is cut has two parts at least)
    const dim3 join((unsigned)(heads * std::min(tiles, (1LL << c.log2_places) / heads + 1)), CG * kCB);
    if (window) hipLaunchKernelGGL((kv8_join<D, kCB, CG, true>), join, dim3(kThreads), 0, s, w, c);
    else hipLaunchKernelGGL((kv8_join<D, kCB, CG, false>), join, dim3(kThreads), 0, s, w, c);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const WindowArgs &w, hipStream_t s)
{
    const DecodeArgs &a = w.d;
    const int G = a.num_q_heads / a.num_kv_heads;
    // (the tiles' kernel keeps the distance between two blocks of a pool in 32 bits)
    const bool far = a.num_layers * codes_slice(a.num_kv_heads, a.block_size, D) > 0xffffffffull;
    if (G > 32 || w.force_rows || far) {
        const long long items = (long long)w.total_tokens * a.num_kv_heads * a.passes;
        if (items > 0x7fffffffLL * kWaves) return hipErrorInvalidValue;
        hipLaunchKernelGGL(kv8_rows<D>, dim3((unsigned)((items + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, w);
        return hipGetLastError();
    }
    if constexpr (D >= 256) {
        // (of 64 columns two workgroups fit a CU, of 128 one: 4 prompts of 1 024, 16 / 4 heads, 88 us and 119)
        return G <= 16 ? launch_tiles<D, 1, 1>(w, s) : launch_tiles<D, 2, 1>(w, s);
    } else {
        // Four waves on 64 columns and two stages at a time where a request has no more columns, or few more and the launch few tiles; else each 32 of 128.  By 64 / 128, us, all
        // on 3 000 cached: 64 requests of 16 tokens, 32 / 8 heads, 85 / 99, of 24 142 / 106, of 64 267 / 218; 16 of 48 69 / 84; 4 of 192 on 40 plain heads 72 / 106, 64 of 32 368 / 414, of
        // 128 725 / 598.  (Without contexts by 128 always, 64 of 16 10.2 and 13.3; but the host does not know.)  12 of 4 to 64 on 300 to 30 000 80 / 85.
        const long long columns = (long long)w.max_new_tokens * G, tiles = (long long)w.total_tokens * G / 64 + a.batch;
        const bool narrow = columns <= 64 || (columns <= 256 && tiles * a.num_kv_heads <= 1024);
        return narrow ? launch_tiles<D, 2, 2>(w, s) : launch_tiles<D, 2, 1>(w, s);
    }
}

}  // namespace

size_t kv8_parts_bytes(int head_dim, int group)
{
    if (group > 32) return 0;                            // (a wavefront per token)
    return ((size_t)2 << cut8::kLog2Places) * (tile_state(head_dim, head_dim >= 256 && group <= 16 ? 64 : 128) * sizeof(float) + 8);
}

hipError_t launch_kv8_prefill(const WindowArgs &w, hipStream_t stream)
{
    if (w.d.batch == 0 || w.total_tokens == 0) return hipSuccess;
    if (w.d.head_dim == 64) return launch<64>(w, stream);
    if (w.d.head_dim == 128) return launch<128>(w, stream);
    if (w.d.head_dim == 256) return launch<256>(w, stream);
    return hipErrorInvalidValue;
}

}  // namespace lamps
