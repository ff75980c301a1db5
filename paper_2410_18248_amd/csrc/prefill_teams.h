// Prompt attention by two teams of waves that take turns at the matrix cores: prefill_mfma's contraction for launches with many
// new tokens.  Device code; part of prefill_attn.hip.
#pragma once

// One workgroup = one (request, kv head, tile of 256 columns; 128 at head size 256): eight waves of kCB blocks of 16 (new token,
// head-of-group) columns, one workgroup to a CU, two waves to a SIMD, one of either team.  While one team is in its matrix phase -- the scores of
// stage s and the outputs of stage s - 1, back to back, with the LDS reads of the next operands between them -- the
// other is in its softmax phase -- weights of its stage, the next loads from the pools -- and a barrier ends each phase.  Left to themselves,
// as in prefill_mfma, the two waves of a SIMD fall into step: both want the matrix cores, then both the vector ALUs (which share
// one issue port with them besides), and a wave-stage of 32 x 32 takes 1 100 to 1 300 cycles for 544 of matrix work; here 830.  The stages'
// tiles come by global_load_lds into a ring of 128 KiB, up to six stages ahead, and serve twice the columns.
//
// Bound by the two phases -- matrix pipe busy 0.56 of the launch, LDS 0.66, 0.4 of that conflicts of the tiled layout's 8-byte value reads -- and by
// power: the chip runs this at 2.2 GHz (prefill_mfma, matrix pipe 0.46, at 2.3), and what takes fewer cycles at more energy loses.  With
// 32x32x16 products, 1 600 cycles to a pair of wave-stages in place of 1 665, it ran at 1.95 GHz: 4 prompts of 4 096, 32 / 8 heads of
// 128, 501 us against 482.  Waves whose columns see no more of the positions do no products (ragged prompts -6 %).  Attention
// alone, us, tiles of 128 by prefill_mfma / so: those 550 / 486, one of 8 000 511 / 438, 4 of 1 000 52 / 43, 16 of 500 on 2 000 to 4 000 cached
// 444 / 386; 40 plain heads, 4 of 2 048, 215 / 198; heads of 256, 4 of 512 on 500 to 2 000 (attention of a recompute's chunk) 76 / 68, 8 of 1 000
// to 2 000 237 / 198.
//
// What each phase holds is measured (cycles of a matrix / softmax phase): all operand reads at the start of the softmax phase 780 /
// 1 100, for the wave waits for room in the LDS queue before its first weight; reads among the products, loads there too 770 / 550; loads, with
// their address arithmetic, in the softmax phase 640 / 780, the least together.  Grouped layout: a value operand is two 8-byte reads, half of
// a unit each; 16-byte reads want 8 register swaps (500 cycles) or, with values brought in by 4 bytes such that they lie as operands, three more
// loads a wave (+3 %).
//
// The reference point of the exponentials moves where prefill_mfma's does and to the same value, so that a row has the same bits whichever of the two
// kernels a call's totals choose.  That it has to is found after the fact, by a weight of 2^kSlack and more: the largest by packed maxima of
// three (two instructions to eight weights; by packed maxima of two the phase is 5 % longer).  A move is far from rare where scores are
// peaked, and all eight waves wait for it at the barrier; only the block that asks for it is weighed again, and lanes compare without LDS.  4 prompts
// of 4 096, 32 / 8 heads, us, queries of N(0, 1) / N(0, 16) by prefill_mfma 549 / 579, with the reference looked for in both blocks through LDS
// 483 / 640, so 482 / 551; 4 of 2 048 on 40 plain heads 207 / 216, 200 / 270, 195 / 229.
template <int D, bool TILED, int kCB>
__global__ __launch_bounds__(512, 2) void prefill_teams(const PrefillArgs p, const int tiles, const int full_groups)
{
    constexpr int W = 8, kCols = 16 * kCB;
    constexpr int NK = D / 32, NS = D / 16, U = D * 2, NU = D / 8;
    constexpr int SUBB = 16 * D * 2, VOFF = 2 * SUBB, STAGE = 4 * SUBB;
    constexpr int NB = 131072 / STAGE;
    constexpr int VA = NB - 2, KA = NB == 4 ? NB : NB - 2;
    constexpr int NE = U / 256;                      // sub-tiles a wave loads from: half of the waves a sub-tile, or each a part of both
    static_assert(NB * STAGE == 131072 && (NE == 1 || NE == 2), "head_dim");
    extern __shared__ __align__(16) char lds[];

    const DecodeArgs &a = p.d;
    const int G = a.num_q_heads / a.num_kv_heads, TW = kCols / G, WT = W * TW;
    Place at;
    if (!place<false>(p, a.num_kv_heads, tiles, full_groups, WT, false, at)) return;
    const int r = at.r, g = at.head, tile = at.tile, first = at.first, n_new = at.n_new, C = at.ctx;
    constexpr bool WINDOW = false;
    constexpr int window = 0, sinks = 0;
#include "teams_body.h"
}
