// A cache held in 8 bits: where codes and scales lie, and how they come and go.  Device code; include from a .hip file only.
//
// Of each (block, layer, kv head) the keys, and apart from them the values, are e4m3 codes times one scale s = 2^e:
//   e = the smallest whole number with a <= 448 2^e,  a the largest finite magnitude of the block's tokens,  held within [-110, 119]
//   code = rne_e4m3(x / s)   (448 where x is larger; NaN for what is no finite number)
// Powers of two, because then x / s is exact and the rounding to a code the only one; another scale moves a code's exponent and
// changes nothing else, but for codes that leave the normal numbers; and code * s is a bf16 number, for every code and e, which one
// conversion instruction makes of two codes.  (A scale of a / 448 would use half a binade more at the top, where e4m3, a floating point
// type, has no more digits than elsewhere: nothing is gained.)
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lamps {
namespace {

constexpr int kLeastExp = -110, kMostExp = 119;          // of scales: every code times its scale is a normal bf16 number, or zero
constexpr float kMostCode = 448.0f;

typedef __attribute__((ext_vector_type(2))) float codes_f32x2;

// The scale of a block whose largest finite magnitude has these bits (fp32).
__device__ __forceinline__ float scale_for(uint32_t most)
{
    // (448 = 1.75 * 2^8: a carry out of the fraction where it is beyond 1.75)
    const int e = (int)((most + 0x1FFFFFu) >> 23) - 8;
    return __uint_as_float((uint32_t)min(max(e, kLeastExp + 127), kMostExp + 127) << 23);
}
// 1 / s of such a scale.
__device__ __forceinline__ float inverse(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// Magnitude bits (fp32) of a bf16 number if it is finite, else 0: the larger ones are the larger numbers.
__device__ __forceinline__ uint32_t finite_size(uint32_t bf16_bits)
{
    const uint32_t x = (bf16_bits & 0x7FFFu) << 16;
    return x < 0x7F800000u ? x : 0;
}

// Four numbers to four codes, times 1 / s.
__device__ __forceinline__ float bounded(float x, float inv)
{
    const float y = __builtin_amdgcn_fmed3f(x * inv, -kMostCode, kMostCode);
    return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : y;
}
__device__ __forceinline__ uint32_t to_codes(float x0, float x1, float x2, float x3, float inv)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(bounded(x0, inv), bounded(x1, inv), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(bounded(x2, inv), bounded(x3, inv), w, true);
    return (uint32_t)w;
}
// Four codes rounded to a scale 1 / f times theirs, f <= 1.
__device__ __forceinline__ uint32_t recode(uint32_t codes, float f)
{
    const codes_f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(b[0] * f, b[1] * f, w, true);
    return (uint32_t)w;
}
// Codes 0, 1 or 2, 3 of four, times s, as a pair of bf16: exact.
template <bool HIGH>
__device__ __forceinline__ uint32_t from_codes(uint32_t codes, float s)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, s, HIGH));
}
// Whether one of four codes is NaN: all seven bits of its magnitude set.
__device__ __forceinline__ bool any_nan(uint32_t codes) { return (((codes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0; }

// A block's slice of a pool in one layer: the tiles of its heads, block_size * head_dim codes each, and behind them room for two scales
// (fp32) of each head, of its keys and of its values.  Both are in the key pool's slice, next to each other, so that a block's
// scales are one line of memory for a reader; the room in the value pool's slice is not used.
__host__ __device__ __forceinline__ uint32_t codes_tail(int kv_heads) { return ((uint32_t)kv_heads * 8 + 127) & ~127u; }
__host__ __device__ __forceinline__ uint64_t codes_slice(int kv_heads, int block_size, int head_dim)
{
    return (uint64_t)kv_heads * block_size * head_dim + codes_tail(kv_heads);
}
// Inside a tile, sub-tiles of 16 slots: keys by units of 16 dims of one slot, values by units of 4 slots of dims j, j + 16, j + 32 and j + 48 --
// 16 bytes that a lane of the attention kernels loads and converts to operands of the matrix cores.  Byte offsets in a sub-tile.
__device__ __forceinline__ int key_code(int t, int d) { return ((d >> 4) * 16 + t) * 16 + (d & 15); }
__device__ __forceinline__ int value_code(int t, int d) { return (((d >> 6) * 4 + (t >> 2)) * 16 + (d & 15)) * 16 + (d >> 4 & 3) * 4 + (t & 3); }

}  // namespace
}  // namespace lamps
