// Attention of one new token per request over a cache of 8 bits, everything or a window of it and its first positions.
//
//   out = softmax(q K^T * scale) V  over the positions t < end with t >= end - window or t < sinks, K and V the numbers that the codes stand for
//
// A stream over the codes, half as many bytes as of bf16.  A range is one (request, kv head / pass); ranges of about an even share of all work go whole to
// a workgroup, the longest first, longer ones are cut, each part a workgroup's, in front of them, and the last part of a range to arrive adds them up, or, where ranges are
// few, a second launch.  Bound by memory where the launch is large (230 of 256 requests of 32 to 8 192 tokens on 32 / 8 heads of 128, 97.6 us, 6.1 TB/s of codes; 51 of 64 of
// 128 to 4 096 on 40 plain heads 104, 6.4 TB/s; bf16 caches of the same 190 and 217 us), otherwise by a walk's round trips: lengths, entries, codes, sums.
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

struct Split {
    uint64_t tag;
    int log2_places;                                     // 2^it: workgroups that all work is dealt to evenly, if it is cut
};
// What a workgroup takes: units u0 .. u1 - 1 of a range, one of `runs` parts of it (the at'th; `first`: the item of the first).
struct Piece {
    int r, hc, C, u0, u1, runs, at, first;
    bool single;                                         // a range of the wave's own
};
constexpr int kLeastUnits = 2 * kWaves;                  // of a part
constexpr int kMostRequests = 256;                       // of a launch
constexpr int kMostUnits = 1 << 26;
// So many ranges of no more units go to a wave each, which needs no other (a workgroup / a wave, us: 256 requests of 60 on 40 plain heads 62.5 / 41.5, of 120 77.8 / 63.9, of 60 on
// 32 / 8 heads 15.6 / 10.6; 202 of 60 on 16 plain heads of 256 65.7 / 41.1): the workgroups that are too many leave at once.
constexpr int kShortUnits = 4, kManyRanges = 1024;

__device__ __forceinline__ int divided(int a, int b) { return (int)((unsigned)a / (unsigned)b); }

// How a launch is cut, by every wave for itself, K consecutive requests per lane.
template <int K>
struct Plan {
    int n[K], C[K], np[K];                               // units of a request's ranges, its length, parts of each (0: not cut)
    int own, upto, cuts, whole;                          // parts of the lane's requests' ranges per head / pass, and of all up to them; all parts; requests that are not cut
    int longest, worth;

    __device__ __forceinline__ Plan(const WindowArgs &w, const Split &c)
    {
        const DecodeArgs &a = w.d;
        const int lane = threadIdx.x & 63, HC = a.num_kv_heads * a.passes;
        int running[K], low = 0, high = 0;
        longest = whole = own = upto = cuts = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = min(K * lane + k, a.batch - 1);
            running[k] = a.running[i];
            C[k] = a.ctx_lens[i];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) asm volatile("" : "+v"(running[k]), "+v"(C[k]));   // (asked for together)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            C[k] = min(C[k], a.max_blocks * a.block_size);
            n[k] = K * lane + k < a.batch && running[k] ? max(1, Sight<32>(C[k], w.window, w.sinks).units) : 0;   // (an empty context: its row of zeros)
            np[k] = 0;
            low += n[k] & 0xFFFF;
            high += n[k] >> 16;
            longest = max(longest, n[k]);
            whole += __popcll(__ballot(n[k] > 0));
        }
        longest = __builtin_amdgcn_readlane(wave_max_to(longest), 63);
        const unsigned long long all = ((unsigned long long)(unsigned)__builtin_amdgcn_readlane(wave_scan(high), 63) << 16) + (unsigned)__builtin_amdgcn_readlane(wave_scan(low), 63);
        // An even share of all units, so that the parts beyond the first of their ranges are no more than the places; what is up to half as long again is not worth
        // the hand-over.
        const unsigned long long even = (all * (unsigned)HC >> c.log2_places) + 1;
        const int size = max((int)min(even, (unsigned long long)kMostUnits), kLeastUnits);
        worth = size + size / 2;
        if (longest <= worth) return;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            np[k] = n[k] > worth ? divided(n[k] + size - 1, size) : 0;
            own += np[k];
            whole -= __popcll(__ballot(np[k] > 0));
        }
        upto = wave_scan(own);
        cuts = __builtin_amdgcn_readlane(upto, 63) * HC;
    }
};
// Units of each part of a range that is cut into so many, and how many of these there are then.
__device__ __forceinline__ int2 parts_of(int n, int parts)
{
    const int each = divided(n + parts - 1, parts);
    return make_int2(each, divided(n + each - 1, each));
}

// What workgroup `item` takes.  False: nothing.
template <int K>
__device__ __forceinline__ bool find_piece(const WindowArgs &w, const Split &c, int item, Piece &it)
{
    const DecodeArgs &a = w.d;
    const int lane = threadIdx.x & 63, HC = a.num_kv_heads * a.passes;
    const Plan<K> plan(w, c);
    const auto &[n, C, np, own, upto, cuts, whole, longest, worth] = plan;
    it.single = longest <= kShortUnits && whole * HC >= kManyRanges;
    if (it.single) item = item * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= cuts + whole * HC) return false;
    if (item < cuts) {                                   // (none, where `single`: a part has kLeastUnits and more)
        int at = divided(item, HC);
        it.hc = item - at * HC;
        const int l = __popcll(__ballot(upto <= at));
        at -= __builtin_amdgcn_readlane(upto - own, l);
        int k = 0, of = __builtin_amdgcn_readlane(np[0], l), nr = __builtin_amdgcn_readlane(n[0], l);
        it.C = __builtin_amdgcn_readlane(C[0], l);
#pragma unroll
        for (int j = 1; j < K; ++j)
            if (k == j - 1 && at >= of) {
                at -= of;
                k = j;
                of = __builtin_amdgcn_readlane(np[j], l);
                nr = __builtin_amdgcn_readlane(n[j], l);
                it.C = __builtin_amdgcn_readlane(C[j], l);
            }
        it.r = K * l + k;
        const int2 parts = parts_of(nr, of);
        it.runs = parts.y;
        it.at = at;
        it.first = item - at * HC;
        it.u0 = at * parts.x;
        it.u1 = min(nr, it.u0 + parts.x);
        return it.at < it.runs;
    }
    // the request with the nth longest sight of those that run and are not cut (ties by place): the bits of its length from the highest on
    int nth = divided(item - cuts, HC);
    it.hc = item - cuts - nth * HC;
    unsigned long long in[K];
#pragma unroll
    for (int k = 0; k < K; ++k) in[k] = __ballot(n[k] > 0 && np[k] == 0);
    for (int bit = 31 - __builtin_clz((unsigned)min(longest, worth)); bit >= 0; --bit) {
        unsigned long long set[K];
        int m = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            set[k] = in[k] & __ballot(n[k] >> bit & 1);
            m += __popcll(set[k]);
        }
        const bool have = nth < m;
        if (!have) nth -= m;
#pragma unroll
        for (int k = 0; k < K; ++k) in[k] = have ? set[k] : in[k] & ~set[k];
    }
    it.r = it.C = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int m = __popcll(in[k]);
        if (nth >= 0 && nth < m) {
            // (the lane with nth of them in front of it)
            const unsigned long long mine = __ballot((in[k] >> lane & 1) && __builtin_amdgcn_mbcnt_hi((unsigned)(in[k] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)in[k], 0)) == (unsigned)nth);
            const int l = __ffsll((long long)mine) - 1;
            it.r = K * l + k;
            it.C = __builtin_amdgcn_readlane(C[k], l);
            nth = -1;
        } else if (nth >= 0) {
            nth -= m;
        }
    }
    it.u0 = 0;
    it.u1 = kMostUnits;                                  // (all there are)
    it.runs = 1;
    it.at = it.first = 0;
    return true;
}

// Two outputs, element i and up; wide: out is 4-byte aligned there.
__device__ __forceinline__ void put_pair(void *out, size_t i, bool wide, float x, float y)
{
    const uint32_t w = pack_bf16(x, y);
    uint16_t *at = static_cast<uint16_t *>(out) + i;
    if (wide) {
        *reinterpret_cast<uint32_t *>(at) = w;
    } else {
        at[0] = (uint16_t)w;
        at[1] = (uint16_t)(w >> 16);
    }
}

template <int D, bool LATER>
__global__ __launch_bounds__(kThreads, D >= 256 ? 1 : 2) void kv8_decode(const WindowArgs w, const Split c)
{
    typedef CodesReducer<D> R;
    extern __shared__ __align__(16) float states[];      // [wave][head][D + 2]
    __shared__ int is_last;
    const DecodeArgs &a = w.d;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int GH = a.heads_per_pass, HC = a.num_kv_heads * a.passes;
    Piece it;
    if (a.batch <= 64 ? !find_piece<1>(w, c, blockIdx.x, it) : !find_piece<4>(w, c, blockIdx.x, it)) return;
    const Sight<32> see(it.C, w.window, w.sinks);
    const int u1 = min(it.u1, see.units), n = max(u1 - it.u0, 0), each = it.single ? n : (n + kWaves - 1) / kWaves, from = it.single ? 0 : min(n, wv * each);
    const bool wide = ((uintptr_t)a.out & 3) == 0;
    const size_t slot = (size_t)GH * (D + 2), row = ((size_t)it.r * a.num_q_heads + it.hc * GH) * D;
    R::run(a, it.r, (size_t)it.r, it.hc / a.passes, it.hc * GH, GH, see, it.u0 + from, it.u0 + min(n, from + each), [&](int h, int d, float M, float L, const auto &A) {
        if (it.single) {                                 // uniform
            const float inv = see.units == 0 ? 0.0f : 1.0f / L;
            put_pair(a.out, row + h * D + d, wide, A[0] * inv, A[1] * inv);
            put_pair(a.out, row + h * D + d + 2, wide, A[2] * inv, A[3] * inv);
        } else {
            store_partial(states + (size_t)(wv * GH + h) * (D + 2), D, d, M, L, A);
        }
    });
    if (it.single) return;
    __syncthreads();
    // the waves' states added up: pair i of outputs, of head h from dim d on
    const auto add_up = [&](auto out) {
        for (int i = 2 * (64 * wv + lane); i < GH * D; i += 128 * kWaves) {
            const int h = i / D, d = i % D;
            const float *x = states + h * (D + 2);
            float M = kLeast, L = 0.0f, A[2] = {0.0f, 0.0f};
            float2 ml[kWaves];
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                ml[k] = *reinterpret_cast<const float2 *>(x + k * slot + D);
                M = fmaxf(M, ml[k].x);
            }
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                const float f = fast_exp2(ml[k].x - M);
                const float2 o = *reinterpret_cast<const float2 *>(x + k * slot + d);
                L += ml[k].y * f;
                A[0] += o.x * f;
                A[1] += o.y * f;
            }
            out(i, h, d, M, L, A);
        }
    };
    const auto finish = [&](int i, int, int, float, float L, const float (&A)[2]) {
        const float inv = see.units == 0 ? 0.0f : 1.0f / L;   // (no positions: zeros)
        put_pair(a.out, row + i, wide, A[0] * inv, A[1] * inv);
    };
    if (it.runs == 1) {
        add_up(finish);
        return;
    }
    float *mine = a.partials + (size_t)(it.first + it.at * HC) * slot;
    if constexpr (LATER) {                               // (a second launch adds them up)
        add_up([&](int, int h, int d, float M, float L, const float (&A)[2]) { store_partial(mine + h * (D + 2), D, d, M, L, A); });
        return;
    }
    add_up([&](int, int h, int d, float M, float L, const float (&A)[2]) {
        put_shared(mine + h * (D + 2) + d, A[0], A[1]);
        if (d == 0) put_shared(mine + h * (D + 2) + D, M, L);
    });
    uint64_t *flags = reinterpret_cast<uint64_t *>(a.partials + ((size_t)2 << c.log2_places) * slot);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (wv == 0) {
        const bool last = report_run<true>(flags + it.first, HC, it.at, it.runs, c.tag);
        if (lane == 0) is_last = last;
    }
    __syncthreads();
    if (!is_last) return;
    // the parts in order, whichever workgroup this is: bit-reproducible
    for (int i = 2 * (64 * wv + lane); i < GH * D; i += 128 * kWaves) {
        const int h = i / D, d = i % D;
        const float *x = a.partials + (size_t)it.first * slot + h * (D + 2);
        float M = kLeast, L = 0.0f, A[2] = {0.0f, 0.0f};
        for (int p0 = 0; p0 < it.runs; p0 += 8) {
            float2 ml[8], o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float *y = x + (size_t)min(p0 + k, it.runs - 1) * HC * slot;
                ml[k] = get_shared(y + D);
                o[k] = get_shared(y + d);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (p0 + k >= it.runs) break;
                const float Mn = fmaxf(M, ml[k].x), f0 = fast_exp2(M - Mn), f = fast_exp2(ml[k].x - Mn);
                L = L * f0 + ml[k].y * f;
                A[0] = A[0] * f0 + o[k].x * f;
                A[1] = A[1] * f0 + o[k].y * f;
                M = Mn;
            }
        }
        finish(i, h, d, M, L, A);
    }
}

// Adds the parts of a range up behind a LATER launch: 128 outputs a workgroup, two per lane, its waves every eighth part, eight of them asked for together.
constexpr int kJoinWaves = 8;
template <int K>
__global__ __launch_bounds__(64 * kJoinWaves) void kv8_decode_join(const WindowArgs w, const Split c)
{
    constexpr int N = 8;
    __shared__ float4 sums[kJoinWaves][64];
    const DecodeArgs &a = w.d;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = a.head_dim;
    const int GH = a.heads_per_pass, HC = a.num_kv_heads * a.passes, r = divided(blockIdx.x, HC), hc = blockIdx.x - r * HC;
    const Plan<K> p(w, c);
    int n = 0, of = 0, before = __builtin_amdgcn_readlane(p.upto - p.own, r / K);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int x = __builtin_amdgcn_readlane(p.np[k], r / K);
        if (k < r % K) before += x;
        if (k == r % K) {
            of = x;
            n = __builtin_amdgcn_readlane(p.n[k], r / K);
        }
    }
    if (of == 0) return;                                 // does not run, or written already
    const int runs = parts_of(n, of).y, i = min((int)blockIdx.y * 128 + 2 * lane, GH * D - 2), h = i / D, d = i - h * D;
    const size_t slot = (size_t)GH * (D + 2);
    const float *x = a.partials + ((size_t)before * HC + hc) * slot + h * (D + 2);
    float M = kLeast, L = 0.0f, A[2] = {0.0f, 0.0f};
    const auto add = [&](float m, float l, float y0, float y1) {
        const float Mn = fmaxf(M, m), f0 = fast_exp2(M - Mn), f = fast_exp2(m - Mn);
        L = L * f0 + l * f;
        A[0] = A[0] * f0 + y0 * f;
        A[1] = A[1] * f0 + y1 * f;
        M = Mn;
    };
    for (int p0 = wv; p0 < runs; p0 += N * kJoinWaves) {
        float2 ml[N], o[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float *y = x + (size_t)min(p0 + k * kJoinWaves, runs - 1) * HC * slot;
            ml[k] = *reinterpret_cast<const float2 *>(y + D);
            o[k] = *reinterpret_cast<const float2 *>(y + d);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (p0 + k * kJoinWaves >= runs) break;      // uniform
            add(ml[k].x, ml[k].y, o[k].x, o[k].y);
        }
    }
    sums[wv][lane] = make_float4(M, L, A[0], A[1]);
    __syncthreads();
    if (wv > 0) return;
#pragma unroll
    for (int k = 1; k < kJoinWaves; ++k) {
        const float4 y = sums[k][lane];
        add(y.x, y.y, y.z, y.w);
    }
    const float inv = 1.0f / L;
    if (blockIdx.y * 128 + 2 * lane < GH * D) put_pair(a.out, ((size_t)r * a.num_q_heads + hc * GH) * D + i, ((uintptr_t)a.out & 3) == 0, A[0] * inv, A[1] * inv);
}

template <int D>
hipError_t launch(WindowArgs w, hipStream_t s)
{
    DecodeArgs &a = w.d;
    const int HC = a.num_kv_heads * a.passes;
    const size_t state = (size_t)a.heads_per_pass * (D + 2) * sizeof(float), per_share = decode_share_bytes(a.heads_per_pass, D);
    // Parts are no more than 5 / 3 of the places: n / size + 1 of a range, which has more than 1.5 size.  Places by what any memory for the geometry has room for (a context's and
    // lamps_decode_attn_static's), so that results go by the arguments alone.
    const size_t room = std::min((size_t)decode_max_shares(a.heads_per_pass, D) * per_share, (size_t)LAMPS_STATIC_SCRATCH_BYTES - ((size_t)1 << 20));
    // 256 places, or 512 where there are hundreds of ranges (256 / 512 / 1 024: 16 of 2 000 15.2 / 16.1 / 22.6, 32 of 100 to 4 000 on 16 / 4 heads of 256 20.4 / 25.0 / 24.9; 200 of 100 to 4 000 on
    // 8 / 2 heads of 64 14.7 / 13.5 / 15.7, 230 of 32 to 8 192 on 32 / 8 heads 104.5 / 97.4 / 100.0).
    const long long ranges = (long long)a.batch * HC;
    const bool later = cut8::ranges_later(ranges, cut8::most_seen((long long)a.max_blocks * a.block_size, w.window, w.sinks, 1));
    int log2_places = ranges < 384 ? 8 : 9;
    while (log2_places > 0 && ((size_t)2 << log2_places) * (state + 8) > room) --log2_places;
    if (((size_t)2 << log2_places) * (state + 8) > std::min(room, a.partial_capacity)) return hipErrorInvalidValue;
    // A wave holds 256 requests: larger batches by several launches.  (HC may be thousands: no more workgroups than a grid has.)
    const long long most = 0x7fffffffLL - (1LL << log2_places);
    const int step = (int)std::max(1LL, std::min((long long)kMostRequests, most / HC));
    const int batch = a.batch;
    for (int r0 = 0; r0 < batch; r0 += step) {
        WindowArgs x = w;
        const size_t rows = (size_t)r0 * a.num_q_heads * D * 2;
        x.d.batch = std::min(step, batch - r0);
        x.d.q = static_cast<const char *>(a.q) + rows;
        x.d.out = static_cast<char *>(a.out) + rows;
        x.d.block_table = a.block_table + (size_t)r0 * a.max_blocks;
        x.d.ctx_lens = a.ctx_lens + r0;
        x.d.running = a.running + r0;
        const Split c = {next_launch_tag(), log2_places};
        const unsigned grid = (unsigned)((long long)x.d.batch * HC + (1LL << log2_places));
        if (!later) {
            hipLaunchKernelGGL((kv8_decode<D, false>), dim3(grid), dim3(kThreads), (size_t)kWaves * state, s, x, c);
        } else {
            hipLaunchKernelGGL((kv8_decode<D, true>), dim3(grid), dim3(kThreads), (size_t)kWaves * state, s, x, c);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            const dim3 join((unsigned)(x.d.batch * HC), (unsigned)((a.heads_per_pass * D + 127) / 128));
            if (x.d.batch <= 64) hipLaunchKernelGGL(kv8_decode_join<1>, join, dim3(64 * kJoinWaves), 0, s, x, c);
            else hipLaunchKernelGGL(kv8_decode_join<4>, join, dim3(64 * kJoinWaves), 0, s, x, c);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_kv8_decode(const WindowArgs &w, hipStream_t stream)
{
    if (w.d.batch == 0) return hipSuccess;
    if (w.d.head_dim == 64) return launch<64>(w, stream);
    if (w.d.head_dim == 128) return launch<128>(w, stream);
    if (w.d.head_dim == 256) return launch<256>(w, stream);
    return hipErrorInvalidValue;
}

}  // namespace lamps
