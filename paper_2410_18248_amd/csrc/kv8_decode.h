// One wavefront's walk over a cache of 8 bits: up to 16 query heads of one kv head over units of 32 positions.  Device code; include from a .hip file
// only, behind attn_reducers.h, kv8.h and tile_parts.h.
#pragma once

namespace lamps {
namespace {

typedef __attribute__((address_space(4))) const uint64_t *scales_ptr;   // read-only: scalar loads

__device__ __forceinline__ bf16x8 operand(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return __builtin_bit_cast(bf16x8, make_uint4(x, y, z, w)); }

// Where the two sub-tiles of the unit at t are read: one that nothing is seen of, whose block may be anyone's, in the other one's place.
__device__ __forceinline__ int2 sub_tiles(const Sight<32> &see, int t)
{
    const bool first = (t + 15 >= see.lo) | (t < see.sinks), second = (t + 16 < see.end) & ((t + 31 >= see.lo) | (t + 16 < see.sinks));
    return make_int2(first ? t : t + 16, second ? t + 16 : t);
}

// As MfmaReducer, with codes for operands: a lane's 16 bytes are 16 dims of a key, two operands of 16x16x32 products (the contraction
// index is permuted, and the queries with it), or four positions of four values' dims, which with the four of the unit's other sub-tile are the
// operands of four products over 32 positions.  A unit of 32 positions is two sub-tiles of 16, in one block or two, each with its block's scales, which
// the conversion to bf16 takes.  Plain heads (one query head to a kv head) go the same way: of the products' 16 columns one is used, but the
// matrix cores have 6 times what the stream asks of them.  Weights are pairs of bf16, the high part and what it leaves.
template <int DIM>
struct CodesReducer {
    static constexpr int D = DIM, U = 32;
    static constexpr int NL = D / 64, NK = D / 32, NS = D / 16;   // loads of a sub-tile and pool; operands of keys, of values
    struct Unit {
        uint4 k[2][NL], v[2][NL];
        float2 scale[2];                                 // of keys and of values
    };

    // Units u0 .. u1 - 1 of a token's sight; sink(h, d, M, L, A): as for MfmaReducer.
    template <typename Sink>
    static __device__ __forceinline__ void run(const DecodeArgs &a, int r, size_t qrow, int g, int h0, int heads, const Sight<U> &see, int u0, int u1, Sink sink)
    {
        const int lane = threadIdx.x & 63, j = lane & 15, qd = lane >> 4;
        bf16x8 qb[NK];                                   // [2 i + h]: dims 64 i + 16 qd + 8 h and up of head h0 + j
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            uint4 t = make_uint4(0, 0, 0, 0);
            if (j < heads)
                t = *reinterpret_cast<const uint4 *>(static_cast<const char *>(a.q) + ((qrow * a.num_q_heads + h0 + j) * D + 64 * (i >> 1) + 16 * qd + 8 * (i & 1)) * 2);
            qb[i] = __builtin_bit_cast(bf16x8, t);
        }
        float m = kLeast, l = 0.0f;                      // m is the same in the 4 lanes of a head
        f32x4 o[NS];                                     // out^T: dims 16 s + 4 qd + e, head j
#pragma unroll
        for (int s = 0; s < NS; ++s) o[s] = f32x4{0.f, 0.f, 0.f, 0.f};

        const int n = u1 - u0;
        const table_ptr table = (table_ptr)(uintptr_t)(a.block_table + (size_t)r * a.max_blocks);
        const size_t tile = (size_t)a.block_size * D, slice = codes_slice(a.num_kv_heads, a.block_size, D), stride = a.num_layers * slice;
        const char *k0 = static_cast<const char *>(a.k_pool) + a.layer * slice;
        const char *kp = k0 + g * tile + lane * 16, *vp = static_cast<const char *>(a.v_pool) + a.layer * slice + g * tile + lane * 16;
        const char *sp = k0 + a.num_kv_heads * tile + g * 8;
        const auto place = [&](int c) { return see.at(u0 + min(c, n - 1)); };
        const auto entry = [&](int c) {
            const int2 t = sub_tiles(see, place(c));
            return make_int2(table[t.x >> a.log2_block_size], table[t.y >> a.log2_block_size]);
        };
        const auto issue = [&](int c, int2 blocks, Unit &x) {
            const int2 t = sub_tiles(see, place(c));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // (an entry that names no block of the pool reads the last one; the row is meaningless)
                const size_t block = (size_t)min((unsigned)(h ? blocks.y : blocks.x), (unsigned)a.num_blocks - 1) * stride;
                const size_t off = block + (size_t)(((h ? t.y : t.x) & (a.block_size - 1)) >> 4) * (16 * D);
                x.scale[h] = __builtin_bit_cast(float2, *(scales_ptr)(uintptr_t)(sp + block));
#pragma unroll
                for (int i = 0; i < NL; ++i) x.k[h][i] = load_stream16(kp + off + i * 1024);
#pragma unroll
                for (int i = 0; i < NL; ++i) x.v[h][i] = load_stream16(vp + off + i * 1024);
            }
        };
        const auto consume = [&](int c, Unit &x) {
            __builtin_amdgcn_sched_barrier(0);           // (the loads above stay above what waits for the ones before them)
            const int t0 = place(c);
            f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};   // positions t0 + 16 h + 4 qd + e, head j
#pragma unroll
            for (int i = 0; i < NL; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 w = x.k[h][i];
                    const float f = x.scale[h].x;
                    s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(from_codes<false>(w.x, f), from_codes<true>(w.x, f), from_codes<false>(w.y, f), from_codes<true>(w.y, f)),
                                                                   qb[2 * i], s[h], 0, 0, 0);
                    s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(from_codes<false>(w.z, f), from_codes<true>(w.z, f), from_codes<false>(w.w, f), from_codes<true>(w.w, f)),
                                                                   qb[2 * i + 1], s[h], 0, 0, 0);
                }
            // (taken out of the matrix cores in front of the branch: see window_attn.hip)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[h][e] *= a.scale_log2e;
            asm volatile("" : "+v"(s[0]), "+v"(s[1]));
            if (!see.sees_all(t0)) {                     // uniform
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t keep = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool on = see.sees(t0 + 16 * h + 4 * qd + e);
                        if (!on) s[h][e] = -INFINITY;
                        keep |= on ? 0xFFu << (8 * e) : 0u;
                    }
#pragma unroll
                    for (int i = 0; i < NL; ++i) {
                        x.v[h][i].x &= keep; x.v[h][i].y &= keep;
                        x.v[h][i].z &= keep; x.v[h][i].w &= keep;
                    }
                }
            }
            float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            if (__any(mx - m > kSlack)) {                // rare after the first units
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float mn = mx - m > kSlack ? mx : m, f = fast_exp2(m - mn);
                m = mn;
                l *= f;
#pragma unroll
                for (int i = 0; i < NS; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][e] *= f;
            }
            uint32_t ph[4], pl[4];                       // pairs of weights: positions 4 qd + 0, 1 and 2, 3 of each sub-tile
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p0 = fast_exp2(s[k >> 1][2 * (k & 1)] - m), p1 = fast_exp2(s[k >> 1][2 * (k & 1) + 1] - m);
                l += p0 + p1;
                ph[k] = pack_bf16(p0, p1);
                pl[k] = pack_bf16(p0 - bf16_lo(ph[k]), p1 - bf16_hi(ph[k]));
            }
            const bf16x8 high = operand(ph[0], ph[1], ph[2], ph[3]), low = operand(pl[0], pl[1], pl[2], pl[3]);
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const uint32_t w0[4] = {x.v[0][i].x, x.v[0][i].y, x.v[0][i].z, x.v[0][i].w}, w1[4] = {x.v[1][i].x, x.v[1][i].y, x.v[1][i].z, x.v[1][i].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bf16x8 v = operand(from_codes<false>(w0[k], x.scale[0].y), from_codes<true>(w0[k], x.scale[0].y),
                                             from_codes<false>(w1[k], x.scale[1].y), from_codes<true>(w1[k], x.scale[1].y));
                    o[4 * i + k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, high, o[4 * i + k], 0, 0, 0);
                    o[4 * i + k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, low, o[4 * i + k], 0, 0, 0);
                }
            }
        };
        if (n > 0) {
            Unit x, y;
            int c = 0;
            int2 e1, e2;
            if ((n & 1) == 0) {                          // the last one is to be one that `x` holds
                const int2 e0 = entry(0);
                e1 = entry(1);
                issue(0, e0, y);
                issue(1, e1, x);
                e1 = entry(2);
                e2 = entry(3);
                consume(0, y);
                c = 1;
            } else {
                issue(0, entry(0), x);
                e1 = entry(1);
                e2 = entry(2);
            }
            for (; c + 1 < n; c += 2) {
                issue(c + 1, e1, y);
                e1 = entry(c + 3);
                consume(c, x);
                issue(c + 2, e2, x);
                e2 = entry(c + 4);
                consume(c + 1, y);
            }
            consume(c, x);
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (j < heads) {
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const float A[4] = {o[s][0], o[s][1], o[s][2], o[s][3]};
                sink(j, 16 * s + 4 * qd, m, l, A);
            }
        }
    }
};

}  // namespace
}  // namespace lamps
