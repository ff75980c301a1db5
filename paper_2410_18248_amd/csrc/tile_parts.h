// What the kernels of tiles of new tokens share, with a window and without.  Device code; include from a .hip file only, behind attn_reducers.h.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cfloat>
#include <type_traits>

namespace lamps {
namespace {

constexpr int kStage = 32;               // cached positions per LDS stage
constexpr float kSlack = 8.0f;           // log2 of the largest weight before the reference moves
constexpr float kLeast = -FLT_MAX;       // a reference below which no finite score lies

typedef __attribute__((address_space(4))) const int32_t *table_ptr;   // read-only: scalar loads

// s_waitcnt immediate: wait until at most n of the wave's vector memory operations are outstanding
constexpr int vmcnt(int n) { return 0x0F70 | (n & 15) | (n >> 4) << 14; }

// The positions that one token sees, in aligned units of U: those of the sinks, then those of the window.
template <int U>
struct Sight {
    int end, lo, sinks;                  // sees t < end if t >= lo or t < sinks; lo = 0 where the two stretches meet
    int first, start, units;             // units of sinks; position of the first unit behind them; all units

    __device__ __forceinline__ Sight(int C, int window, int want) : Sight(max(C, 0), max(0, max(C, 0) - window), want, std::true_type{}) {}
    // (of several tokens together: `from` the first one's, C the last one's)
    __device__ __forceinline__ Sight(int C, int from, int want, std::true_type)
    {
        end = C;
        lo = from;
        sinks = min(want, lo);
        if (lo <= sinks) lo = sinks = 0;
        first = (sinks + U - 1) / U;
        start = max(lo / U, first) * U;
        units = first + (max(end - start, 0) + U - 1) / U;
    }
    __device__ __forceinline__ int at(int u) const { return u < first ? u * U : start + (u - first) * U; }
    __device__ __forceinline__ int unit_of(int t) const { return t < start ? t / U : first + (t - start) / U; }   // of a position that lies in one
    // (no branches: see window_attn.hip)
    __device__ __forceinline__ bool sees(int t) const { return (t < end) & ((t >= lo) | (t < sinks)); }
    __device__ __forceinline__ bool sees_all(int t) const { return (t + U <= end) & ((t >= lo) | (t + U <= sinks)); }   // of the unit at t
};

// Stores a column's N slabs of 16 outputs, those of quarter qd being 4 qd .. of each.  Odd and even quarters exchange halves of
// two slabs, so that a lane stores 16 bytes and an instruction 64 of a row: by 8 and 32, 24 prompts of 16 to 700 tokens on 40 heads took
// 42.0 us, 39.2 so; 12 of 100 to 700 on 32 / 8 heads 30.4 and 27.5.  By a whole wave, which leaves where none of its columns is a row (8 tokens, 16 / 8
// heads of 256: 6.2 us with all blocks exchanged, 5.7 so).
template <int N, typename Slabs>
__device__ __forceinline__ void store_column(uint16_t *dst, int qd, bool mine, float inv, const Slabs &o)
{
    static_assert(N % 2 == 0, "slabs go in pairs");
    if (!__any(mine)) return;
#pragma unroll
    for (int s = 0; s < N; s += 2) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = pack_bf16(o[s + (k >> 1)][2 * (k & 1)] * inv, o[s + (k >> 1)][2 * (k & 1) + 1] * inv);
        const auto x0 = __builtin_amdgcn_permlane16_swap(w[0], w[2], false, false);
        const auto x1 = __builtin_amdgcn_permlane16_swap(w[1], w[3], false, false);
        if (mine) *reinterpret_cast<uint4 *>(dst + 16 * (s + (qd & 1)) + 8 * (qd >> 1)) = make_uint4(x0[0], x1[0], x0[1], x1[1]);
    }
}

}  // namespace
}  // namespace lamps
