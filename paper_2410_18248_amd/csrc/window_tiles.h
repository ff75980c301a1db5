// Windowed attention of many new tokens on the matrix cores, bf16.  Device code; part of window_attn.hip.
#pragma once

// One workgroup = one (request, kv head, tile of new tokens): four waves of kCB blocks of 16 columns, (new token, head-of-group) pairs, as in
// prefill_mfma, whose products, operand layouts and lazily moved reference these are.  What differs is what a tile walks over: the units of 16
// positions that any of its tokens sees -- of the sinks, then of the windows, which begin where the first token's does -- two units to a stage,
// wherever they lie.  Units that all columns of a wave see need no mask; the others get one by position, and there a value that is no finite number must
// not reach the columns that do not see it (a zero weight does not silence it): stages that hold one, which is found by a product of the values
// with zeros, multiply once per token of the wave, with what that one does not see zeroed.
//
// Weights are rounded to bf16 for the second product and summed up as rounded, in fp32: outputs of normal values are off by 0.0021 to 0.0023 of their size, 0.0016 to
// 0.0017 of that by their own rounding.  As pairs of bf16, which decode has, they are off by that alone, and launches take 1.03 to 1.33 times as long
// (4 x 8 192 tokens, window 1 024, 588 / 743 us; 12 responses 37.6 / 43.5); a wavefront per token, which a caller can ask for, has them in fp32.
//
// Bound by the matrix cores and the vector ALUs on long prompts, as prefill_mfma is, and by the walk where few tokens leave the chip idle: then
// the stages of a tile are shared by up to `parts` workgroups, as many as the host counts from window and sinks.  Up to four parts are added up by the last of them to
// arrive, more by a second launch (us, so / by a second launch always: 12 responses of 4 to 64 tokens on 32 / 8 heads, window 2 048, in two 40.3 / 43.5;
// 12 of 6 to 35 on 345 to 2 490, window of everything, 30.3 / 33.4; 4 of 16, 40 plain heads, 40.3 / 44.8; one of 16 tokens on 32 / 8, in 16, 18.6 / 13.8).

// Which workgroup does what: items -- tiles of one head, numbered by the row that they begin at, at most one for nothing per request -- head by
// head, and of these an eighth, one after the other, to each of the eight XCDs: neighbours in time and place share most of their windows in an L2.
struct TileAt {
    int r, g, tile, first, n_new, ctx, part, item;    // (g: of `heads` that tiles are dealt for)
};
// The number of a workgroup's item, part by part; < 0: none.
__device__ __forceinline__ int tile_item(const WindowArgs &w, unsigned block, int heads)
{
    const unsigned all = (unsigned)w.items * (unsigned)heads * (unsigned)w.parts, per = (all + 7) / 8, i = (block & 7) * per + (block >> 3);
    return block >> 3 < per && i < all ? (int)i : -1;
}
__device__ __forceinline__ bool tile_at(const WindowArgs &w, int WT, TileAt &at, int i0)
{
    const DecodeArgs &a = w.d;
    const unsigned items = (unsigned)w.items;
    if (i0 < 0) return false;
    const unsigned i = (unsigned)i0;
    // (uniform, and said to be: divisions go through the vector ALUs, and addresses of loads into LDS are scalars)
    const unsigned run = (unsigned)__builtin_amdgcn_readfirstlane((int)(i / (unsigned)w.parts));
    at.part = (int)(i - run * (unsigned)w.parts);
    at.g = __builtin_amdgcn_readfirstlane((int)(run / items));
    const int k = (int)(run - (unsigned)at.g * items);
    at.item = (int)run;
    const NewTokens x = new_tokens_at(w.q_start, a.ctx_lens, a.batch, k, [WT](int q, int r) { return q / WT + r; });
    at.r = __builtin_amdgcn_readfirstlane(x.r);
    at.first = __builtin_amdgcn_readfirstlane(x.first);
    at.ctx = __builtin_amdgcn_readfirstlane(x.ctx);
    at.n_new = __builtin_amdgcn_readfirstlane(x.count);
    at.tile = __builtin_amdgcn_readfirstlane(k - (at.first / WT + at.r));
    // a context shorter than its new tokens, or longer than the table row: nothing is read or written for it; rows past the last: none
    if (at.first < 0 || at.tile < 0 || at.ctx < at.n_new || at.ctx > a.max_blocks * a.block_size) return false;
    return (long long)at.tile * WT < min(at.n_new, w.total_tokens - at.first);
}

constexpr size_t tile_state_floats(int D, int columns) { return (size_t)columns * (D + 2); }

// Narrow tiles, of 64 columns, whole: one stage per barrier, operands read one after the other, for three or four workgroups to a CU.  Shared ones
// keep four stages in LDS instead (12 responses, added up by a second launch, 43.6 us, 45.2 as whole ones have it).
template <int D, int kCB, bool SPLIT>
constexpr bool tile_small() { return D <= 128 && kCB == 1 && !SPLIT; }
constexpr int kHandedParts = 4;
// Stages per barrier, and groups of them that LDS holds.
template <int D, int kCB>
constexpr int tile_groups() { return D <= 128 && kCB > 1 ? 2 : 1; }
template <int D, int kCB, bool SPLIT>
constexpr int tile_buffers() { return D <= 128 && SPLIT && kCB == 1 ? 4 : 2; }

// Behind a loop: its last products are there before what adds them up or stores them.  (Which way leads from one to the other is the loop's
// own matter: the compiler may count the instructions of another, see window_attn.hip.)
template <int kCB, int NS>
__device__ __forceinline__ void products_there(f32x4 (&l)[kCB], f32x4 (&o)[kCB][NS])
{
    asm volatile("s_nop 7" ::: "memory");
#pragma unroll
    for (int b = 0; b < kCB; ++b) asm volatile("" : "+v"(l[b]), "+v"(o[b][NS - 1]));
}

template <int D, bool TILED, int kCB, bool SPLIT>
__global__ __launch_bounds__(kThreads, D >= 256 && kCB > 1 ? 1 : (tile_small<D, kCB, SPLIT>()) ? (D == 128 && TILED ? 3 : 4) : 2) void window_tiles(const WindowArgs w)
{
    constexpr int kCols = 16 * kCB, GRP = tile_groups<D, kCB>(), NB = tile_buffers<D, kCB, SPLIT>();
    constexpr int NK = D / 32, NS = D / 16, U = D * 2, NU = D / 8;
    constexpr int LPT = (2 * U) / kThreads;           // 16-byte units per thread, pool and stage
    constexpr int SUBB = 16 * D * 2, VOFF = 2 * SUBB, STAGE = 4 * SUBB, GSTAGE = GRP * STAGE;
    constexpr bool kLean = D >= 256 || (D == 128 && tile_small<D, kCB, SPLIT>());   // operands are read one after the other: registers
    constexpr int kLoads = GRP * 2 * LPT;             // of a group, of one wave; all groups have as many
    static_assert(NB * GSTAGE <= 65536 && LPT >= 1 && (2 * U) % kThreads == 0, "head_dim");
    __shared__ __align__(16) char lds[NB * GSTAGE];

    const DecodeArgs &a = w.d;
    const int G = a.num_q_heads / a.num_kv_heads, TW = kCols / G, WT = kWaves * TW;
    TileAt at;
    if (!tile_at(w, WT, at, tile_item(w, blockIdx.x, a.num_kv_heads))) return;
    const int r = at.r, g = at.g, first = at.first, base_pos = at.ctx - at.n_new;
    const int n_new = min(at.n_new, w.total_tokens - first);
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 15, qd = lane >> 4;

    // what the tile walks over, and the part of it that is this workgroup's
    const int p_first = base_pos + at.tile * WT, p_last = base_pos + min(n_new, (at.tile + 1) * WT) - 1;
    const Sight<16> see(p_last + 1, max(0, p_first - w.window + 1), w.sinks, std::true_type{});
    const int last_unit = see.units - 1, n_stages = (see.units + 1) / 2;
    int st0 = 0, st1 = n_stages, runs = 1;
    if constexpr (SPLIT) {
        // (parts are whole groups; handed over in here, eight stages at least, or twelve, whose states are twice as large: 4 of 64 tokens, 16 plain heads of 256, 35.8 us by
        // eight, 30.6 so; of 128 all the same)
        const bool handed = w.parts <= kHandedParts;
        runs = handed ? max(1, min(w.parts, n_stages / (D >= 256 ? 12 : 8))) : w.parts;
        const int each = ((n_stages + runs - 1) / runs + GRP - 1) / GRP * GRP;
        if (handed) runs = (n_stages + each - 1) / each;
        if (at.part >= runs) return;
        st0 = min(n_stages, at.part * each);
        st1 = min(n_stages, st0 + each);
    }
    // the wave's own tokens; none: positions that see nothing
    const int wave_tok = at.tile * WT + wv * TW;
    const bool none = wave_tok >= n_new;
    const int wave_min = __builtin_amdgcn_readfirstlane(none ? 0x3fffffff : base_pos + wave_tok);
    const int wave_max = __builtin_amdgcn_readfirstlane(none ? -1 : base_pos + min(n_new, wave_tok + TW) - 1);
    const int wave_hi = wave_max - w.window + 1;      // the first position of the window of the wave's last token
    // units that all of its columns see (of the windows), and those that some see: of the sinks, and those
    const int full0 = __builtin_amdgcn_readfirstlane(see.first + (max(wave_hi - see.start, 0) + 15) / 16);
    const int full1 = __builtin_amdgcn_readfirstlane(none ? 0 : see.first + max(wave_min + 1 - see.start, 0) / 16);
    const int some0 = __builtin_amdgcn_readfirstlane(see.first + max(wave_min - w.window + 1 - see.start, 0) / 16);
    const int some1 = __builtin_amdgcn_readfirstlane(none ? 0 : see.unit_of(wave_max) + 1);
    const int sunk = see.start > 0 ? see.first : (min(w.sinks, see.end) + 15) / 16;   // (where the first token's window reaches the sinks, positions are units)

    const table_ptr table = (table_ptr)(uintptr_t)(a.block_table + (size_t)r * a.max_blocks);
    const uint32_t tile_bytes = (uint32_t)a.block_size * D * 2;
    const uint32_t block_stride = (uint32_t)a.num_layers * a.num_kv_heads * tile_bytes;   // (the launcher has checked that it fits)
    const size_t head_off = ((size_t)a.layer * a.num_kv_heads + g) * tile_bytes;
    const char *kp = static_cast<const char *>(a.k_pool) + head_off, *vp = static_cast<const char *>(a.v_pool) + head_off;
    const uint32_t last_block = (uint32_t)a.num_blocks - 1;
    // A group's units: the blocks they lie in, looked up an iteration before the loads that use them, and where in a block's tile.
    struct Places {
        uint32_t block[2 * GRP], at[2 * GRP];
    };
    const auto lookup = [&](int grp) {
        Places x;
#pragma unroll
        for (int i = 0; i < 2 * GRP; ++i) {
            const int t = see.at(min(grp * 2 * GRP + i, last_unit));
            // (an entry that names no block of the pool reads the last one: the rows are meaningless)
            x.block[i] = min((uint32_t)table[t >> a.log2_block_size], last_block);
            x.at[i] = (uint32_t)((t & (a.block_size - 1)) >> 4) * SUBB;
        }
        return x;
    };
    // This lane's part of a load: unit x of a sub-tile to LDS slot x (tiled layout), or slot s of row r takes unit s ^ r of a key row and s ^ 2 r of a
    // value row (plain), so that the rows that an operand read touches lie in different banks.
    uint32_t lane_k[LPT], lane_v[LPT];
#pragma unroll
    for (int k = 0; k < LPT; ++k) {
        const int x = (kThreads * k + 64 * wv) % U + lane, row = x / NU, sl = x % NU;
        lane_k[k] = (uint32_t)(TILED ? x : row * NU + (sl ^ (row & (NU - 1)))) * 16;
        lane_v[k] = (uint32_t)(TILED ? x : row * NU + (sl ^ ((2 * row) & (NU - 1)))) * 16;
    }
    const auto dma_group = [&](char *buf, const Places &x) {
#pragma unroll
        for (int h = 0; h < GRP; ++h)
#pragma unroll
            for (int k = 0; k < LPT; ++k) {
                const int x0 = kThreads * k + 64 * wv;   // the wave's first unit: sub-tile x0 / U
                const bool second = U >= kThreads ? (kThreads * k) / U != 0 : __builtin_amdgcn_readfirstlane(x0 / U) != 0;
                const uint32_t block = __builtin_amdgcn_readfirstlane((int)(second ? x.block[2 * h + 1] : x.block[2 * h]));
                const uint64_t off = (uint64_t)block * block_stride + (second ? x.at[2 * h + 1] : x.at[2 * h]);
                typedef __attribute__((address_space(3))) char *lptr;
                const uint32_t lk = (uint32_t)(uintptr_t)(lptr)(buf + h * STAGE + x0 * 16), lv = lk + VOFF;
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lk), "v"(lane_k[k]), "s"(kp + off) : "memory");
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lv), "v"(lane_v[k]), "s"(vp + off) : "memory");
            }
    };
    const int grp0 = st0 / GRP, grp1 = st0 < st1 ? (st1 + GRP - 1) / GRP : grp0;   // (a part that is not empty begins with a group)
    const auto ask_first = [&]() {
        Places x[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) x[i] = lookup(grp0 + i);
#pragma unroll
        for (int i = 0; i < NB; ++i) dma_group(lds + i * GSTAGE, x[i]);
    };
    // The first tiles in front of the queries, or, where four groups are on their way, behind them.
    if constexpr (NB == 2) ask_first();

    // this lane's column in each block: (token, head), its position, its queries (of a negative scale: their negatives)
    int pos[kCB];
    size_t orow[kCB];
    bf16x8 qb[kCB][NK];
    const float scale = fabsf(a.scale_log2e);
    const uint32_t flip = a.scale_log2e < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int b = 0; b < kCB; ++b) {
        const int c = b * 16 + j, tl = c / G, hd = c - tl * G, tok = wave_tok + tl;
        const bool ok = c < TW * G && tok < n_new;
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
    if constexpr (NB > 2) ask_first();
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

    const int koff = qd * 256 + j * 16, voff = VOFF + (qd * 16 + j) * 16;
    int kslot[NK], vslot[NS];
#pragma unroll
    for (int i = 0; i < NK; ++i) kslot[i] = (j * NU + ((4 * i + qd) ^ (j & (NU - 1)))) * 16;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int rv = 4 * qd + (j >> 2);
        vslot[s] = VOFF + (rv * NU + ((2 * s + ((j & 3) >> 1)) ^ ((2 * rv) & (NU - 1)))) * 16 + (j & 1) * 8;
    }
    bf16x8 kop[NK][2], vop[NS];
    const auto read_k = [&](const char *buf) {
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                kop[i][h] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(buf + (TILED ? koff + i * 1024 : kslot[i]) + h * SUBB));
    };
    const auto read_v = [&](const char *buf) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if constexpr (TILED) {
                const char *src = buf + voff + (s >> 1) * 1024 + (s & 1) * 8;
                const uint2 h0 = *reinterpret_cast<const uint2 *>(src), h1 = *reinterpret_cast<const uint2 *>(src + SUBB);
                vop[s] = __builtin_bit_cast(bf16x8, make_uint4(h0.x, h0.y, h1.x, h1.y));
            } else {
                typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
                const s16x4 h0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(buf + vslot[s]));
                const s16x4 h1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(buf + vslot[s] + SUBB));
                vop[s] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(h0, h1, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        }
    };
    f32x4 sc0[kCB], sc1[kCB];                         // scores: positions t0 + 4 qd + e and t1 + 4 qd + e of the lane's column
    bf16x8 pw[kCB];
    const auto scores = [&]() {
#pragma unroll
        for (int b = 0; b < kCB; ++b) sc0[b] = sc1[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int b = 0; b < kCB; ++b) {
                sc0[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[i][0], qb[b][i], sc0[b], 0, 0, 0);
                sc1[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[i][1], qb[b][i], sc1[b], 0, 0, 0);
            }
        // (they are there before the way parts: up to 1.3 % of a launch on 31 of prompts, chunks and responses, 0.1 on average)
        if constexpr (kCB == 1) asm volatile("s_nop 7" : "+v"(sc0[0]), "+v"(sc1[0]));
        else asm volatile("s_nop 7" : "+v"(sc0[0]), "+v"(sc1[0]), "+v"(sc0[1]), "+v"(sc1[1]));
    };
    // Position p sees t + 4 qd + e of a unit: e <= lim and (e > lim - window or e < sinks - t - 4 qd), lim = p - t - 4 qd.
    const auto visible = [&](int p, int t, int e) {
        const int lim = p - t - 4 * qd;
        return (e <= lim) & ((e > lim - w.window) | (e < w.sinks - t - 4 * qd));
    };
    // The mask of a unit: by what it takes for the wave's columns, most often one of the two comparisons or none.
    const auto mask = [&](f32x4 (&x)[kCB], int t) {
        const bool late = t + 15 > wave_min, early = t < wave_hi, sunk = t < w.sinks;
        if (early & sunk) {
#pragma unroll
            for (int b = 0; b < kCB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!visible(pos[b], t, e)) x[b][e] = -INFINITY;
            return;
        }
        if (late) {
#pragma unroll
            for (int b = 0; b < kCB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e > pos[b] - t - 4 * qd) x[b][e] = -INFINITY;
        }
        if (early) {
#pragma unroll
            for (int b = 0; b < kCB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e <= pos[b] - t - 4 * qd - w.window) x[b][e] = -INFINITY;
        }
    };
    const auto position = [&](int u) { return u <= last_unit ? see.at(u) : 0x40000000; };   // (past the last unit: where nobody looks)
    const auto softmax = [&](int u, bool masked) {
        if (masked) {
            mask(sc0, position(u));
            mask(sc1, position(u + 1));
        }
#pragma unroll
        for (int b = 0; b < kCB; ++b) {
            float sc[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[e] = e < 4 ? sc0[b][e] : sc1[b][e - 4];
            float mx = sc[0];                         // (the median with infinity: the maximum)
#pragma unroll
            for (int e = 1; e < 8; ++e) mx = __builtin_amdgcn_fmed3f(mx, sc[e], INFINITY);
            mx *= scale;
            if (__any(mx - m[b] > kSlack)) {          // wave-uniform, rare after the first stages
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float mn = mx - m[b] > kSlack ? mx : m[b];
                const float f = fast_exp2(m[b] - mn);
                m[b] = mn;
#pragma unroll
                for (int e = 0; e < 4; ++e) l[b][e] *= f;
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[b][s][e] *= f;
            }
            const float mn = m[b];
#pragma unroll
            for (int e = 0; e < 8; ++e) pw[b][e] = (__bf16)fast_exp2(fmaf(sc[e], scale, -mn));
        }
    };
    // Whether one of the stage's values is no finite number: those give NaN times zero, which the matrix cores find for a few cycles
    // (by exponents, two operations on each of the registers, a masked stage took 1.3 times as long).
    const auto wild = [&]() {
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        const bf16x8 zero = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
#pragma unroll
        for (int s = 0; s < NS; ++s) y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop[s], zero, y, 0, 0, 0);
        return __any((y[0] + y[1]) + (y[2] + y[3]) != 0.0f) != 0;
    };
    const auto sums = [&]() {
#pragma unroll
        for (int b = 0; b < kCB; ++b) l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pw[b], l[b], 0, 0, 0);
    };
    const auto accumulate = [&]() {
        sums();
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int b = 0; b < kCB; ++b) o[b][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop[s], pw[b], o[b][s], 0, 0, 0);
    };
    // Token by token: what one does not see is zeroed, and its columns take the result.
    const auto accumulate_apart = [&](int u) {
        const int t0 = position(u), t1 = position(u + 1);
        sums();
#pragma unroll 1
        for (int tok = 0; tok < TW; ++tok) {
            const int p = wave_tok + tok < n_new ? base_pos + wave_tok + tok : -1;
            uint32_t keep[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                keep[k] = (visible(p, k < 2 ? t0 : t1, 2 * (k & 1)) ? 0x0000FFFFu : 0u) | (visible(p, k < 2 ? t0 : t1, 2 * (k & 1) + 1) ? 0xFFFF0000u : 0u);
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                uint4 v = __builtin_bit_cast(uint4, vop[s]);
                v.x &= keep[0]; v.y &= keep[1]; v.z &= keep[2]; v.w &= keep[3];
#pragma unroll
                for (int b = 0; b < kCB; ++b) {
                    const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), pw[b], o[b][s], 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[b][s][e] = pos[b] == p ? y[e] : o[b][s][e];
                }
            }
        }
    };

    Places next = lookup(grp0 + NB);
    // Group `ahead` behind it on its way, this one is there, for everyone.
    const auto landed = [&](auto ahead) {
        __builtin_amdgcn_s_waitcnt(vmcnt(ahead * kLoads));
        __syncthreads();
    };
    landed(std::integral_constant<int, NB == 2 ? 0 : NB - 1>{});
    if (!kLean) read_k(lds);
    for (int grp = grp0; grp < grp1; ++grp) {
        char *cur = lds + ((grp - grp0) & (NB - 1)) * GSTAGE, *nxt = lds + ((grp - grp0 + 1) & (NB - 1)) * GSTAGE;
#pragma unroll
        for (int h = 0; h < GRP; ++h) {
            const int st = grp * GRP + h;
            char *buf = cur + h * STAGE;
            const int u = 2 * st;                     // its first unit; what follows is uniform over the wave
            const bool live = (st < st1) & (u < some1) & ((u + 1 >= some0) | (u < sunk));
            const bool masked = (u < full0) | (u + 2 > full1);
            bool apart = false;
            if (live) {
                if (kLean) read_k(buf);
                else read_v(buf);                     // needed after the next K operands are asked for
                scores();
                if (kLean) read_v(buf);
                softmax(u, masked);
                // (here, where no keys are held in registers)
                apart = masked && wild();
                if (apart) accumulate_apart(u);
            }
            if (h == GRP - 1) {
                landed(std::integral_constant<int, NB - 2>{});   // this group's operands are in registers: its place is free
                dma_group(cur, next);
                next = lookup(grp + NB + 1);
            }
            if (!kLean && st + 1 < grp1 * GRP) read_k(h == GRP - 1 ? nxt : buf + STAGE);
            if (live && !apart) accumulate();
        }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt(0));             // no load is left on its way to LDS
    products_there(l, o);

    if (SPLIT && w.parts > kHandedParts) {
        // the columns of each block as the wave holds them, by whole lines, and their (reference, sum)
        if (none) return;
        float *mine = a.partials + ((size_t)at.item * w.parts + at.part) * tile_state_floats(D, kWaves * kCols);
#pragma unroll
        for (int b = 0; b < kCB; ++b) {
            float *to = mine + (size_t)(wv * kCB + b) * 16 * D;
#pragma unroll
            for (int s = 0; s < NS; ++s) *reinterpret_cast<f32x4 *>(to + s * 256 + 4 * lane) = o[b][s];
            if (qd == 0) *reinterpret_cast<float2 *>(mine + (size_t)kWaves * kCols * D + 2 * ((wv * kCB + b) * 16 + j)) = make_float2(m[b], l[b][0]);
        }
        return;
    }
    if (SPLIT && runs > 1) {
        // the columns of each block as the wave holds them, and their (reference, sum); the last part to arrive adds them up
        constexpr int kAll = kWaves * kCols;
        const size_t state = tile_state_floats(D, kAll);
        float *first_part = a.partials + (size_t)at.item * w.parts * state, *to = first_part + at.part * state;
        uint64_t *flags = reinterpret_cast<uint64_t *>(a.partials + (size_t)w.items * a.num_kv_heads * w.parts * state) + (size_t)at.item * w.parts;
        if (!none) {
#pragma unroll
            for (int b = 0; b < kCB; ++b) {
                const int block = wv * kCB + b;
#pragma unroll
                for (int s = 0; s < 2 * NS; ++s)
                    put_shared(to + block * 16 * D + s * 128 + 2 * lane, o[b][s >> 1][2 * (s & 1)], o[b][s >> 1][2 * (s & 1) + 1]);
                if (qd == 0) put_shared(to + kAll * D + 2 * (block * 16 + j), m[b], l[b][0]);
            }
        }
        __builtin_amdgcn_s_waitcnt(vmcnt(0));
        __syncthreads();                              // the workgroup's stores have arrived, and its LDS is free
        int *is_last = reinterpret_cast<int *>(lds);
        if (wv == 0) {
            const bool all = report_run<false>(flags, 1, at.part, runs, w.tag);
            if (lane == 0) *is_last = all;
        }
        __syncthreads();
        if (!*is_last) return;
        // The parts in order, whichever workgroup this is: bit-reproducible.  The waves share the blocks that have columns, by halves of their dims.
        constexpr int HS = NS / 2, N = kHandedParts;
        int me = lane;
        asm volatile("" : "+v"(me));                  // (worked out here, not kept over the loop)
        const int j = me & 15, qd = me >> 4;
        const int blocks = (min(WT, n_new - at.tile * WT) + TW - 1) / TW * kCB;
#pragma unroll 1
        for (int u = wv; u < 2 * blocks; u += kWaves) {
            const int block = u >> 1, half = u & 1;
            float2 ml[N], x[N][2 * HS];
            float M = kLeast, L = 0.0f;
            f32x4 A[HS];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (k > 1 && k >= runs) {             // uniform
                    ml[k] = make_float2(kLeast, 0.0f);
#pragma unroll
                    for (int s = 0; s < 2 * HS; ++s) x[k][s] = make_float2(0.0f, 0.0f);
                    continue;
                }
                const float *from = first_part + k * state;
                ml[k] = get_shared(from + kAll * D + 2 * (block * 16 + j));
#pragma unroll
                for (int s = 0; s < 2 * HS; ++s) x[k][s] = get_shared(from + block * 16 * D + (half * 2 * HS + s) * 128 + 2 * me);
            }
#pragma unroll
            for (int k = 0; k < N; ++k) M = fmaxf(M, ml[k].x);
#pragma unroll
            for (int s = 0; s < HS; ++s) A[s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float f = fast_exp2(ml[k].x - M);
                L += ml[k].y * f;
#pragma unroll
                for (int s = 0; s < 2 * HS; ++s) {
                    A[s >> 1][2 * (s & 1)] += x[k][s].x * f;
                    A[s >> 1][2 * (s & 1) + 1] += x[k][s].y * f;
                }
            }
            const int c = block % kCB * 16 + j, t = c / G, tok = at.tile * WT + block / kCB * TW + t;
            const bool mine = c < TW * G && tok < n_new;
            store_column<HS>(static_cast<uint16_t *>(a.out) + ((size_t)(first + (mine ? tok : 0)) * a.num_q_heads + g * G + (mine ? c - t * G : 0)) * D + 16 * half * HS, qd,
                             mine, 1.0f / L, A);
        }
        return;
    }
#pragma unroll
    for (int b = 0; b < kCB; ++b) store_column<NS>(static_cast<uint16_t *>(a.out) + orow[b], qd, pos[b] >= 0, 1.0f / l[b][0], o[b]);
}

// Adds more than kHandedParts parts of a tile up, two slabs of 16 columns to a workgroup, every fourth part to a wave.  What they add is asked for in front of
// the lengths that say which rows it is (where it lies goes by the launch alone).
template <int D, int kCB>
__global__ __launch_bounds__(kThreads) void window_join(const WindowArgs w0)
{
    constexpr int kCols = 16 * kCB, N = 4, MOST = kMostParts / kWaves;
    __shared__ float4 sums[kWaves][2][64];
    __shared__ float2 stats[kWaves][64];
    const DecodeArgs &a = w0.d;
    WindowArgs w = w0;
    w.parts = 1;
    const int G = a.num_q_heads / a.num_kv_heads, TW = kCols / G, WT = kWaves * TW, parts = w0.parts;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 15, qd = lane >> 4;
    const int block = blockIdx.y, slab = 2 * blockIdx.z;
    const size_t state = tile_state_floats(D, kWaves * kCols);
    const int item = tile_item(w, blockIdx.x, a.num_kv_heads);
    if (item < 0) return;
    const float *x = a.partials + (size_t)item * parts * state;
    float M = kLeast, L = 0.0f;
    f32x4 A[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    const auto add = [&](float2 ml, f32x4 y0, f32x4 y1) {
        const float Mn = fmaxf(M, ml.x), f0 = fast_exp2(M - Mn), f = fast_exp2(ml.x - Mn);
        L = L * f0 + ml.y * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            A[0][e] = A[0][e] * f0 + y0[e] * f;
            A[1][e] = A[1][e] * f0 + y1[e] * f;
        }
        M = Mn;
    };
    TileAt at;
    bool on = false;
    for (int k0 = 0; k0 < MOST; k0 += N) {
        float2 ml[N];
        f32x4 y[N][2];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float *from = x + (size_t)min(wv + kWaves * (k0 + k), parts - 1) * state;
            ml[k] = *reinterpret_cast<const float2 *>(from + (size_t)kWaves * kCols * D + 2 * (block * 16 + j));
#pragma unroll
            for (int s = 0; s < 2; ++s) y[k][s] = *reinterpret_cast<const f32x4 *>(from + (size_t)block * 16 * D + (slab + s) * 256 + 4 * lane);
        }
        if (k0 == 0) {
            on = tile_at(w, WT, at, item);
            if (!on) return;
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (wv + kWaves * (k0 + k) < parts) add(ml[k], y[k][0], y[k][1]);
        if (kWaves * (k0 + N) >= parts) break;
    }
    sums[wv][0][lane] = make_float4(A[0][0], A[0][1], A[0][2], A[0][3]);
    sums[wv][1][lane] = make_float4(A[1][0], A[1][1], A[1][2], A[1][3]);
    stats[wv][lane] = make_float2(M, L);
    __syncthreads();
    if (wv > 0) return;
#pragma unroll
    for (int k = 1; k < kWaves; ++k) {
        const float4 y0 = sums[k][0][lane], y1 = sums[k][1][lane];
        add(stats[k][lane], f32x4{y0.x, y0.y, y0.z, y0.w}, f32x4{y1.x, y1.y, y1.z, y1.w});
    }
    const int n_new = min(at.n_new, w.total_tokens - at.first);
    const int wave_tok = at.tile * WT + block / kCB * TW, c = block % kCB * 16 + j, tl = c / G;
    // (a wave that had no tokens has left nothing)
    const bool mine = c < TW * G && wave_tok + tl < n_new;
    uint16_t *to = static_cast<uint16_t *>(a.out) + ((size_t)(at.first + (mine ? wave_tok + tl : 0)) * a.num_q_heads + at.g * G + (mine ? c - tl * G : 0)) * D + 16 * slab;
    store_column<2>(to, qd, mine, 1.0f / L, A);
}

// ---------------------------------------------------------------- two teams of waves

// prefill_teams' way through a tile of 256 columns (128 at head size 256), for launches with many new tokens (grouped heads: plain ones are as fast or faster by
// window_tiles).
// Bound by the two teams' phases in turn, matrix cores and vector ALUs; what a tile costs beyond its stages, its queries and outputs, two masked ends and the filling of
// the pipeline, is 11 of 35 us under a window of 1 024: 4 prompts of 8 192 on 32 / 8 heads take 555 to 600 us from card to card, 860 to 930 TFLOP/s of the positions seen.  Tiles in
// chains, the next one's first stages asked for behind the last one's, took 580 to 600.
template <int D, int kCB>
__global__ __launch_bounds__(512, 2) void window_teams(const WindowArgs w)
{
    constexpr bool WINDOW = true, TILED = true;
    constexpr int W = 8, kCols = 16 * kCB;
    constexpr int NK = D / 32, NS = D / 16, U = D * 2, NU = D / 8;
    constexpr int SUBB = 16 * D * 2, VOFF = 2 * SUBB, STAGE = 4 * SUBB;
    constexpr int NB = 131072 / STAGE;
    constexpr int VA = NB - 2, KA = NB == 4 ? NB : NB - 2;
    constexpr int NE = U / 256;
    extern __shared__ __align__(16) char lds[];

    const DecodeArgs &a = w.d;
    const int G = a.num_q_heads / a.num_kv_heads, TW = kCols / G, WT = W * TW, window = w.window, sinks = w.sinks;
    TileAt at;
    if (!tile_at(w, WT, at, tile_item(w, blockIdx.x, a.num_kv_heads))) return;
    const int r = at.r, g = at.g, tile = at.tile, first = at.first, n_new = min(at.n_new, w.total_tokens - first), C = at.ctx - at.n_new + n_new;
#include "teams_body.h"
}
