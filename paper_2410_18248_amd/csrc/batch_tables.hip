// A batch's block table, lengths, first rows and slot map from the lengths of its requests, on the device.
//
// With c_r cached and n_r new tokens of request r, blocks of b positions and h_r = ceil(c_r / b) of them held already (or none):
//   need_r = ceil((c_r + n_r) / b) - h_r        before_r = need_0 + .. + need_(r-1)        first_r = n_0 + .. + n_(r-1)
//   table[r][h_r + j] = ids[before_r + j], j < need_r, and -1 behind;   slots[first_r + i] = table[r][(c_r + i) / b] b + (c_r + i) % b
// A request that cannot be served (lamps.h) counts no tokens, and where the tokens go beyond the rows there are, no request
// behind that one counts any: so the rows of those served follow each other.
//
// Bound by the launch and the round trips: lengths, the sums, ids (and kept entries), stores.  One launch: every workgroup sums the
// whole batch up for itself, which is a load per request of a thread and two scans, and then writes its own part of the table
// (2 048 entries) or of the slots (1 024); the first one writes lengths and first rows.  A second launch behind one that sums
// costs more than the sums do.
#include <hip/hip_runtime.h>

#include "attn_reducers.h"
#include "internal.h"

namespace lamps {
namespace {

constexpr int kTableThreads = 256, kTableEntries = 2048, kTableSlots = 1024;

// Inclusive sums over the threads of the workgroup that stop at the type's largest number: a sum that does not fit stays too large.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
__device__ __forceinline__ uint32_t wave_scan_sat(uint32_t x)
{
    x = add_sat(x, (uint32_t)dpp_shifted<0x111, 0xF>((int)x));
    x = add_sat(x, (uint32_t)dpp_shifted<0x112, 0xF>((int)x));
    x = add_sat(x, (uint32_t)dpp_shifted<0x114, 0xF>((int)x));
    x = add_sat(x, (uint32_t)dpp_shifted<0x118, 0xF>((int)x));
    x = add_sat(x, (uint32_t)dpp_shifted<0x142, 0xA>((int)x));
    return add_sat(x, (uint32_t)dpp_shifted<0x143, 0xC>((int)x));
}
// What lies in front of this thread's x.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t *waves)
{
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const uint32_t upto = wave_scan_sat(x);
    if (lane == 63) waves[wv] = upto;
    __syncthreads();
    // (the lane before: a sum that stopped cannot be taken apart again)
    uint32_t before = (uint32_t)__shfl_up((int)upto, 1);
    if (lane == 0) before = 0;
    for (int w = 0; w < wv; ++w) before = add_sat(before, waves[w]);
    return before;
}

struct Lengths {
    int cached, fresh, held, need;                    // need < 0: lengths that no row can have
};
__device__ __forceinline__ Lengths lengths_of(const TableArgs &a, int r)
{
    Lengths x = {0, 0, 0, 0};
    if (r < a.n_req) {
        x.cached = a.cached[r];
        x.fresh = a.new_tokens[r];
        const long long after = (long long)x.cached + x.fresh, row = (long long)a.max_blocks << a.log2_block_size;
        if (x.cached < 0 || x.fresh < 0 || after > row) {
            x.need = -1;
        } else {
            const int round = (1 << a.log2_block_size) - 1;
            x.held = a.grow ? (x.cached + round) >> a.log2_block_size : 0;
            x.need = (int)((after + round) >> a.log2_block_size) - x.held;
        }
    }
    return x;
}

// K requests per thread, in order.  Dynamic LDS: ids before each request, then rows before each request and behind the last; bit 31 of
// the former: not served.
template <int K>
__global__ __launch_bounds__(kTableThreads) void batch_tables(const TableArgs a)
{
    extern __shared__ uint32_t sums[];
    __shared__ uint32_t waves[3][kTableThreads / 64];
    __shared__ int missing[2];                        // requests not served, the lowest
    __shared__ uint32_t taken;
    const int tid = threadIdx.x, n = a.n_req;
    uint32_t *ids_before = sums, *rows_before = sums + n;
    Lengths x[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = lengths_of(a, tid * K + k);
    if (tid == 0) {
        missing[0] = 0;
        missing[1] = 0x7fffffff;
        taken = 0;
    }
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) mine = add_sat(mine, (uint32_t)max(x[k].need, 0));
    uint32_t at = sum_before(mine, waves[0]), before[K], tokens[K];
    mine = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        before[k] = at;
        at = add_sat(at, (uint32_t)max(x[k].need, 0));
        tokens[k] = x[k].need == 0 || (x[k].need > 0 && at <= (uint32_t)a.n_ids) ? (uint32_t)x[k].fresh : 0xffffffffu;   // (all ones: no ids)
        if (tokens[k] != 0xffffffffu) mine = add_sat(mine, tokens[k]);
    }
    at = sum_before(mine, waves[1]);
    uint32_t rows[K], most = 0;                       // rows in front of each; of all that are served
#pragma unroll
    for (int k = 0; k < K; ++k) {
        rows[k] = at;
        if (tokens[k] == 0xffffffffu) continue;
        at = add_sat(at, tokens[k]);
        if (at <= (uint32_t)a.total_tokens) most = at;
        else if (tokens[k] > 0) tokens[k] = 0xffffffffu;
    }
    most = (uint32_t)wave_max_to((int)most);          // (no more than total_tokens: not negative)
    if ((tid & 63) == 63) waves[2][tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTableThreads / 64; ++w) most = max(most, waves[2][w]);
    int lost = 0, lowest = 0x7fffffff;
    uint32_t used = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = tid * K + k;
        if (r >= n) break;
        const bool served = tokens[k] != 0xffffffffu;
        ids_before[r] = served ? (x[k].need > 0 ? before[k] : 0u) : 0x80000000u;
        rows_before[r] = min(rows[k], most);
        if (served) used += (uint32_t)x[k].need;
        else {
            ++lost;
            lowest = min(lowest, r);
        }
        if (blockIdx.x == 0) {
            a.ctx_lens[r] = served ? x[k].cached + x[k].fresh : 0;
            a.q_start[r] = (int)min(rows[k], most);
        }
    }
    if (tid == 0) rows_before[n] = most;
    if (blockIdx.x == 0) {
        if (tid == 0) a.q_start[n] = (int)most;
        if (a.report) {
            if (lost) {
                atomicAdd(&missing[0], lost);
                atomicMin(&missing[1], lowest);
            }
            if (used) atomicAdd(&taken, used);
            __syncthreads();
            if (tid == 0) {
                a.report[0] = (int)taken;
                a.report[1] = missing[0];
                a.report[2] = missing[0] ? missing[1] : -1;
                a.report[3] = (int)most;
            }
        }
        return;
    }
    __syncthreads();
    const int item = blockIdx.x - 1;
    if (item < a.table_items) {                       // a stretch of the table: four entries at a time
        const long long all = (long long)n * a.max_blocks;
        for (int i = 0; i < kTableEntries / (4 * kTableThreads); ++i) {
            const long long e0 = (long long)item * kTableEntries + 4 * (i * kTableThreads + tid);
            if (e0 >= all) break;
            int r = (int)(e0 / a.max_blocks), col = (int)(e0 - (long long)r * a.max_blocks);
            int v[4];
            bool put[4];
            int held = 0, need = 0, from = 0;
            bool served = false;
            const auto enter = [&]() {
                const Lengths y = lengths_of(a, r);
                served = !(ids_before[r] >> 31);
                from = (int)(ids_before[r] & 0x7fffffffu);
                held = y.held;
                need = y.need;
            };
            enter();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = col - held;
                put[e] = e0 + e < all && served && j >= 0;
                v[e] = put[e] && j < need ? a.block_ids[from + j] : -1;
                if (++col == a.max_blocks && e < 3 && e0 + e + 1 < all) {
                    col = 0;
                    ++r;
                    enter();
                }
            }
            int32_t *to = a.block_table + e0;
            if (put[0] && put[1] && put[2] && put[3] && a.wide) {
                *reinterpret_cast<int4 *>(to) = make_int4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (put[e]) to[e] = v[e];
            }
        }
        return;
    }
    const int n0 = (item - a.table_items) * kTableSlots;
#pragma unroll
    for (int i = 0; i < kTableSlots / kTableThreads; ++i) {
        const uint32_t row = (uint32_t)n0 + i * kTableThreads + tid;
        if (row >= (uint32_t)a.total_tokens) break;
        long long slot = -1;
        if (row < most) {
            int lo = 0, hi = n;                       // the last request whose rows begin at or in front of it: that one has some
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (rows_before[mid] <= row) lo = mid; else hi = mid;
            }
            const Lengths y = lengths_of(a, lo);
            const int p = y.cached + (int)(row - rows_before[lo]), j = (p >> a.log2_block_size) - y.held;
            const int block = j < 0 ? a.block_table[(size_t)lo * a.max_blocks + j + y.held] : a.block_ids[(ids_before[lo] & 0x7fffffffu) + j];
            if ((unsigned)block < (unsigned)a.num_blocks) slot = ((long long)block << a.log2_block_size) + (p & ((1 << a.log2_block_size) - 1));
        }
        a.slots[row] = slot;
    }
}

}  // namespace

hipError_t launch_batch_tables(TableArgs a, hipStream_t stream)
{
    const long long entries = (long long)a.n_req * a.max_blocks;
    const long long items = (entries + kTableEntries - 1) / kTableEntries;
    const long long slots = a.slots ? ((long long)a.total_tokens + kTableSlots - 1) / kTableSlots : 0;
    if (items + slots >= 0x7fffffffLL) return hipErrorInvalidValue;
    a.table_items = (int)items;
    a.wide = ((uintptr_t)a.block_table & 15) == 0;
    const dim3 grid((unsigned)(1 + items + slots)), block(kTableThreads);
    const size_t lds = (2 * (size_t)a.n_req + 1) * sizeof(uint32_t);
    if (a.n_req <= kTableThreads)
        hipLaunchKernelGGL(batch_tables<1>, grid, block, lds, stream, a);
    else if (a.n_req <= 4 * kTableThreads)
        hipLaunchKernelGGL(batch_tables<4>, grid, block, lds, stream, a);
    else
        hipLaunchKernelGGL(batch_tables<32>, grid, block, lds, stream, a);
    return hipGetLastError();
}

}  // namespace lamps
