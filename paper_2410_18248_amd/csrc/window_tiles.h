// Windowed attention of many new tokens on the matrix cores, bf16.  Device code; part of window_attn.hip.
#pragma once

// One workgroup = one (request, kv head, tile of new tokens): four waves of kCB blocks of 16 columns, (new token, head-of-group) pairs, as in
// prefill_mfma, whose products, operand layouts and lazily moved reference these are.  What differs is what a tile walks over: the units of 16
// positions that any of its tokens sees -- of the sinks, then of the windows, which begin where the first token's does -- two units to a stage,
// wherever they lie.  Units that all columns of a wave see need no mask; the others get one by position, and there a value that is no finite number must
// not reach the columns that do not see it (a zero weight does not silence it): stages that hold one, which is found with two packed
// operations per register, multiply once per token of the wave, with what that one does not see zeroed.
//
// Bound by the matrix cores and the vector ALUs on long prompts, as prefill_mfma is, and by the walk where few tokens leave the chip idle: then
// the stages of a tile are shared by `parts` workgroups, as many as the host counts from window and sinks, and a second launch adds them up.

// Which workgroup does what: items -- tiles of one head, numbered by the row that they begin at, at most one for nothing per request -- head by
// head, and of these an eighth, one after the other, to each of the eight XCDs: neighbours in time and place share most of their windows in an L2.
struct TileAt {
    int r, g, tile, first, n_new, ctx, part, item;
};
template <int THREADS>
__device__ __forceinline__ bool tile_at(const WindowArgs &w, int WT, TileAt &at)
{
    const DecodeArgs &a = w.d;
    const unsigned items = (unsigned)w.items, all = items * (unsigned)a.num_kv_heads * (unsigned)w.parts, per = (all + 7) / 8;
    unsigned i = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per || i >= all) return false;
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

// The kernels that keep to 256 registers: two workgroups to a CU.
template <int D, int kCB>
constexpr int tile_groups() { return D <= 128 ? 2 : 1; }   // stages per barrier: two where they fit

template <int D, bool TILED, int kCB, bool SPLIT>
__global__ __launch_bounds__(kThreads, D >= 256 && kCB > 1 ? 1 : 2) void window_tiles(const WindowArgs w)
{
    constexpr int kCols = 16 * kCB, GRP = tile_groups<D, kCB>(), NB = 2;
    constexpr int NK = D / 32, NS = D / 16, U = D * 2, NU = D / 8;
    constexpr int LPT = (2 * U) / kThreads;           // 16-byte units per thread, pool and stage
    constexpr int SUBB = 16 * D * 2, VOFF = 2 * SUBB, STAGE = 4 * SUBB, GSTAGE = GRP * STAGE;
    constexpr bool kLean = D >= 256;                  // operands are read one after the other: registers
    static_assert(NB * GSTAGE <= 65536 && LPT >= 1 && (2 * U) % kThreads == 0, "head_dim");
    __shared__ __align__(16) char lds[NB * GSTAGE];

    const DecodeArgs &a = w.d;
    const int G = a.num_q_heads / a.num_kv_heads, TW = kCols / G, WT = kWaves * TW;
    TileAt at;
    if (!tile_at<kThreads>(w, WT, at)) return;
    const int r = at.r, g = at.g, first = at.first, base_pos = at.ctx - at.n_new;
    const int n_new = min(at.n_new, w.total_tokens - first);
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 15, qd = lane >> 4;

    // what the tile walks over, and the part of it that is this workgroup's
    const int p_first = base_pos + at.tile * WT, p_last = base_pos + min(n_new, (at.tile + 1) * WT) - 1;
    const Sight<16> see(p_last + 1, max(0, p_first - w.window + 1), w.sinks, std::true_type{});
    const int last_unit = see.units - 1, n_stages = (see.units + 1) / 2;
    int st0 = 0, st1 = n_stages;
    if constexpr (SPLIT) {
        const int each = (((n_stages + w.parts - 1) / w.parts) + GRP - 1) / GRP * GRP;
        st0 = min(n_stages, at.part * each);
        st1 = min(n_stages, st0 + each);
    }
    // the wave's own tokens; none: positions that see nothing
    const int wave_tok = at.tile * WT + wv * TW;
    const bool none = wave_tok >= n_new;
    const int wave_min = __builtin_amdgcn_readfirstlane(none ? 0x3fffffff : base_pos + wave_tok);
    const int wave_max = __builtin_amdgcn_readfirstlane(none ? -1 : base_pos + min(n_new, wave_tok + TW) - 1);
    const int wave_lo = wave_min - w.window + 1, wave_hi = wave_max - w.window + 1;   // the first position of the first token's window, the last's

    const table_ptr table = (table_ptr)(uintptr_t)(a.block_table + (size_t)r * a.max_blocks);
    const uint32_t tile_bytes = (uint32_t)a.block_size * D * 2;
    const uint32_t block_stride = (uint32_t)a.num_layers * a.num_kv_heads * tile_bytes;   // (the launcher has checked that it fits)
    const size_t head_off = ((size_t)a.layer * a.num_kv_heads + g) * tile_bytes;
    const char *kp = static_cast<const char *>(a.k_pool) + head_off, *vp = static_cast<const char *>(a.v_pool) + head_off;
    const uint32_t last_block = (uint32_t)a.num_blocks - 1;
    const auto unit_at = [&](int u) { return see.at(min(u, last_unit)); };
    uint32_t ent[2 * GRP];
    // (an entry that names no block of the pool reads the last one: the rows are meaningless)
    const auto lookup = [&](int grp, uint32_t (&e)[2 * GRP]) {
#pragma unroll
        for (int i = 0; i < 2 * GRP; ++i) e[i] = min((uint32_t)table[unit_at(grp * 2 * GRP + i) >> a.log2_block_size], last_block);
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
    const auto dma = [&](int st, char *buf, uint32_t e0, uint32_t e1) {
#pragma unroll
        for (int k = 0; k < LPT; ++k) {
            const int x0 = kThreads * k + 64 * wv, sub = U >= kThreads ? (kThreads * k) / U : __builtin_amdgcn_readfirstlane(x0 / U);
            const int t = __builtin_amdgcn_readfirstlane(unit_at(2 * st + sub));
            const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(sub ? e1 : e0)) * block_stride + (uint32_t)(((t & (a.block_size - 1)) >> 4) * SUBB);
            typedef __attribute__((address_space(3))) char *lptr;
            const uint32_t lk = (uint32_t)(uintptr_t)(lptr)(buf + x0 * 16), lv = lk + VOFF;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lk), "v"(lane_k[k]), "s"(kp + off) : "memory");
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lv), "v"(lane_v[k]), "s"(vp + off) : "memory");
        }
    };
    const auto dma_group = [&](int grp, char *buf, const uint32_t (&e)[2 * GRP]) {
#pragma unroll
        for (int h = 0; h < GRP; ++h) dma(grp * GRP + h, buf + h * STAGE, e[2 * h], e[2 * h + 1]);
    };
    const int grp0 = st0 / GRP, grp1 = st0 < st1 ? (st1 + GRP - 1) / GRP : grp0;   // (a part that is not empty begins with a group)
    {
        uint32_t e0[2 * GRP], e1[2 * GRP];
        lookup(grp0, e0);
        lookup(grp0 + 1, e1);
        dma_group(grp0, lds, e0);
        dma_group(grp0 + 1, lds + GSTAGE, e1);
    }

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
    };
    // Position p sees t + 4 qd + e of a unit: e <= lim and (e > lim - window or e < sinks - t - 4 qd), lim = p - t - 4 qd.
    const auto visible = [&](int p, int t, int e) {
        const int lim = p - t - 4 * qd;
        return (e <= lim) & ((e > lim - w.window) | (e < w.sinks - t - 4 * qd));
    };
    const auto softmax = [&](int t0, int t1, bool masked) {
#pragma unroll
        for (int b = 0; b < kCB; ++b) {
            float sc[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[e] = e < 4 ? sc0[b][e] : sc1[b][e - 4];
            if (masked) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!visible(pos[b], e < 4 ? t0 : t1, e & 3)) sc[e] = -INFINITY;
            }
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
    // Whether one of the stage's values is no finite number: exponents of all ones, two to a word.
    const auto wild = [&]() {
        typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
        u16x2 most = {0, 0};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const uint4 u = __builtin_bit_cast(uint4, vop[s]);
            const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[k] & 0x7FFF7FFFu));
        }
        return __any((most[0] >= 0x7F80) | (most[1] >= 0x7F80)) != 0;
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
    const auto accumulate_apart = [&](int t0, int t1) {
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
                uint4 u = __builtin_bit_cast(uint4, vop[s]);
                u.x &= keep[0]; u.y &= keep[1]; u.z &= keep[2]; u.w &= keep[3];
#pragma unroll
                for (int b = 0; b < kCB; ++b) {
                    const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u), pw[b], o[b][s], 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[b][s][e] = pos[b] == p ? y[e] : o[b][s][e];
                }
            }
        }
    };

    lookup(grp0 + NB, ent);
    __builtin_amdgcn_s_waitcnt(vmcnt(0));
    __syncthreads();
    if (!kLean) read_k(lds);
    for (int grp = grp0; grp < grp1; ++grp) {
        char *cur = lds + ((grp - grp0) & 1) * GSTAGE, *nxt = lds + ((grp - grp0 + 1) & 1) * GSTAGE;
#pragma unroll
        for (int h = 0; h < GRP; ++h) {
            const int st = grp * GRP + h;
            char *buf = cur + h * STAGE;
            // the stage's units; one past the last: positions that nobody sees
            const int t0 = unit_at(2 * st), t1 = 2 * st + 1 <= last_unit ? see.at(2 * st + 1) : 0x40000000;
            const auto some = [&](int t) { return (t <= wave_max) & ((t + 15 >= wave_lo) | (t < w.sinks)); };
            const auto every = [&](int t) { return (t + 15 <= wave_min) & ((t >= wave_hi) | (t + 16 <= w.sinks)); };
            const bool live = (st < st1) & (some(t0) | some(t1));   // wave-uniform: its columns see something of it
            const bool masked = !(every(t0) & every(t1));
            bool apart = false;
            if (live) {
                if (kLean) read_k(buf);
                else read_v(buf);                     // needed after the next K operands are asked for
                scores();
                if (kLean) read_v(buf);
                softmax(t0, t1, masked);
                // (here, where no keys are held in registers)
                apart = masked && wild();
                if (apart) accumulate_apart(t0, t1);
            }
            if (h == GRP - 1) {
                __builtin_amdgcn_s_waitcnt(vmcnt(0)); // the next group is there, for everyone; this one's operands are in registers
                __syncthreads();
                dma_group(grp + NB, cur, ent);
                lookup(grp + NB + 1, ent);
            }
            if (!kLean && st + 1 < grp1 * GRP) read_k(h == GRP - 1 ? nxt : buf + STAGE);
            if (live && !apart) accumulate();
        }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt(0));             // no load is left on its way to LDS

    if constexpr (SPLIT) {
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
    } else {
#pragma unroll
        for (int b = 0; b < kCB; ++b) store_column<NS>(static_cast<uint16_t *>(a.out) + orow[b], qd, pos[b] >= 0, 1.0f / l[b][0], o[b]);
    }
}

// Adds the parts of a tile up: a workgroup takes 16 columns of one, its waves a quarter of the dims each (a slab at least).
template <int D, int kCB>
__global__ __launch_bounds__(kThreads) void window_join(const WindowArgs w0)
{
    constexpr int kCols = 16 * kCB, NS = D / 16, EACH = NS / kWaves < 2 ? 2 : NS / kWaves, N = 4;
    const DecodeArgs &a = w0.d;
    WindowArgs w = w0;
    w.parts = 1;
    const int G = a.num_q_heads / a.num_kv_heads, TW = kCols / G, WT = kWaves * TW, parts = w0.parts;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 15, qd = lane >> 4;
    TileAt at;
    if (wv * EACH >= NS || !tile_at<kThreads>(w, WT, at)) return;
    const int n_new = min(at.n_new, w.total_tokens - at.first), block = blockIdx.y;
    const int wave = block / kCB, c = block % kCB * 16 + j, tl = c / G, tok = at.tile * WT + wave * TW + tl;
    if (at.tile * WT + wave * TW >= n_new) return;    // (a wave that had no tokens has left nothing)
    const bool mine = c < TW * G && tok < n_new;
    const size_t state = tile_state_floats(D, kWaves * kCols);
    const float *x = a.partials + (size_t)at.item * parts * state;
    float M = kLeast, L = 0.0f;
    f32x4 A[EACH];
#pragma unroll
    for (int s = 0; s < EACH; ++s) A[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < parts; k0 += N) {
        float2 ml[N];
        f32x4 y[N][EACH];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float *from = x + (size_t)min(k0 + k, parts - 1) * state;
            ml[k] = *reinterpret_cast<const float2 *>(from + (size_t)kWaves * kCols * D + 2 * (block * 16 + j));
#pragma unroll
            for (int s = 0; s < EACH; ++s) y[k][s] = *reinterpret_cast<const f32x4 *>(from + (size_t)block * 16 * D + (wv * EACH + s) * 256 + 4 * lane);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (k0 + k >= parts) break;
            const float Mn = fmaxf(M, ml[k].x), f0 = fast_exp2(M - Mn), f = fast_exp2(ml[k].x - Mn);
            L = L * f0 + ml[k].y * f;
#pragma unroll
            for (int s = 0; s < EACH; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) A[s][e] = A[s][e] * f0 + y[k][s][e] * f;
            M = Mn;
        }
    }
    uint16_t *to = static_cast<uint16_t *>(a.out) + ((size_t)(at.first + (mine ? tok : 0)) * a.num_q_heads + at.g * G + (mine ? c - tl * G : 0)) * D + 16 * wv * EACH;
    store_column<EACH>(to, qd, mine, 1.0f / L, A);
}
