// What the kernels of tiles of new tokens share, with a window and without.  Device code; include from a .hip file only, behind attn_reducers.h.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lamps {
namespace {

constexpr int kStage = 32;               // cached positions per LDS stage
constexpr float kSlack = 8.0f;           // log2 of the largest weight before the reference moves

typedef __attribute__((address_space(4))) const int32_t *table_ptr;   // read-only: scalar loads

// s_waitcnt immediate: wait until at most n of the wave's vector memory operations are outstanding
constexpr int vmcnt(int n) { return 0x0F70 | (n & 15) | (n >> 4) << 14; }

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
