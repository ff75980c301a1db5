// A batch's block table, lengths, first rows and slot map from the lengths of its requests, on the device.
//
// With c_r cached and n_r new tokens of request r, blocks of b positions and h_r = ceil(c_r / b) of them held already (or none):
//   need_r = ceil((c_r + n_r) / b) - h_r        before_r = need_0 + .. + need_(r-1)        first_r = n_0 + .. + n_(r-1)
//   table[r][h_r + j] = ids[before_r + j], j < need_r, and -1 behind;   slots[first_r + i] = table[r][(c_r + i) / b] b + (c_r + i) % b
// A request that cannot be served (lamps.h) counts no tokens, and where the tokens go beyond the rows there are, no request
// behind that one counts any: so the rows of those served follow each other.
//
// Bound by the launch and the round trips: lengths, the sums, ids (and kept entries), stores.  One launch: every workgroup sums the
// whole batch up for itself, which is a load per request of a thread and two scans, keeps what its own part asks for in LDS, and writes that part:
// 2 048 entries of the table, a request's whole row at most, or 1 024 slots; the first one writes lengths and first rows.  A second launch behind one that sums
// costs more than the sums do, up to 1 024 requests: 64 with rows of 512 4.8 us; 1 024 with rows of 2 048, 8 MB of table, and 206 000 slots, 9.5.  Beyond, a thread sums up to 32 requests
// and every part does so again: 1 025 with rows of 512 / 2 048 take 23 / 56 us (1 024: 5.6 / 7.9), 8 192 180 / 660, of which the stores are 3 / 13.
#include <hip/hip_runtime.h>

#include <algorithm>

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

// What a part of the table or of the slots asks for of a request.
struct Held {
    int before, held, need;                           // first id, entries held, entries taken (-1: not served, the row is left alone)
};

// K requests per thread, in order.  Dynamic LDS: workgroups of the table, Held of the rows they write; of the slots, all requests' first rows and ids and
// cached tokens.
template <int K>
__global__ __launch_bounds__(kTableThreads) void batch_tables(const TableArgs a)
{
    extern __shared__ int kept[];
    __shared__ uint32_t waves[3][kTableThreads / 64];
    __shared__ int missing[2];                        // requests not served, the lowest
    __shared__ uint32_t taken;
    const int tid = threadIdx.x, n = a.n_req, item = (int)blockIdx.x - 1;
    // the part: rows r0 .. r1 of the table, from entry e0 (of r0's row) on
    const bool lengths = item < 0, rows_part = !lengths && item < a.table_items;
    int r0 = 0, r1 = -1, e0 = 0;
    if (rows_part) {
        const long long from = (long long)item * kTableEntries;
        r0 = (int)(from / a.max_blocks);
        e0 = (int)(from - (long long)r0 * a.max_blocks);
        r1 = min(n - 1, r0 + (e0 + kTableEntries - 1) / a.max_blocks);
    }
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
    uint32_t first[K], most = 0;                      // rows in front of each; of all that are served
#pragma unroll
    for (int k = 0; k < K; ++k) {
        first[k] = at;
        if (tokens[k] == 0xffffffffu) continue;
        at = add_sat(at, tokens[k]);
        if (at <= (uint32_t)a.total_tokens) most = at;
        else if (tokens[k] > 0) tokens[k] = 0xffffffffu;
    }
    if (rows_part) {
        Held *own = reinterpret_cast<Held *>(kept);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int r = tid * K + k;
            if (r >= r0 && r <= r1) own[r - r0] = Held{(int)before[k], x[k].held, tokens[k] != 0xffffffffu ? x[k].need : -1};
        }
        __syncthreads();
        // four entries at a time; all that a thread writes is asked for before the first is stored
        constexpr int TURNS = kTableEntries / (4 * kTableThreads);
        int v[TURNS][4];
        bool put[TURNS][4];
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const unsigned at0 = (unsigned)e0 + 4 * (i * kTableThreads + tid);     // entries behind the start of r0's row (below 2^27)
            int r = (int)(at0 / (unsigned)a.max_blocks), col = (int)(at0 - (unsigned)r * (unsigned)a.max_blocks);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = r <= r1 - r0;
                const Held h = own[in ? r : 0];
                const int j = col - h.held;
                put[i][e] = in && h.need >= 0 && j >= 0;
                v[i][e] = put[i][e] && j < h.need ? a.block_ids[h.before + j] : -1;
                if (++col == a.max_blocks) {
                    col = 0;
                    ++r;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            int32_t *to = a.block_table + (long long)item * kTableEntries + 4 * (i * kTableThreads + tid);
            if (put[i][0] && put[i][1] && put[i][2] && put[i][3] && a.wide) {
                *reinterpret_cast<int4 *>(to) = make_int4(v[i][0], v[i][1], v[i][2], v[i][3]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (put[i][e]) to[e] = v[i][e];
            }
        }
        return;
    }
    most = (uint32_t)wave_max_to((int)most);          // (no more than total_tokens: not negative)
    if ((tid & 63) == 63) waves[2][tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTableThreads / 64; ++w) most = max(most, waves[2][w]);
    if (lengths) {
        int lost = 0, lowest = 0x7fffffff;
        uint32_t used = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int r = tid * K + k;
            if (r >= n) break;
            const bool served = tokens[k] != 0xffffffffu;
            if (served) {
                used += (uint32_t)x[k].need;
            } else {
                ++lost;
                lowest = min(lowest, r);
            }
            a.ctx_lens[r] = served ? x[k].cached + x[k].fresh : 0;
            a.q_start[r] = (int)min(first[k], most);
        }
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
    // slots, four rows to a thread: the last request whose rows begin at or in front of the first (that one has some) is searched for, the others' follow it
    int *starts = kept, *ids_before = starts + n + 1, *cached = ids_before + n;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = tid * K + k;
        if (r < n) {
            starts[r] = (int)min(first[k], most);
            ids_before[r] = (int)before[k];
            cached[r] = x[k].cached;
        }
    }
    if (tid == 0) starts[n] = (int)most;
    __syncthreads();
    constexpr int TURNS = kTableSlots / kTableThreads;
    const int row0 = (item - a.table_items) * kTableSlots + tid * TURNS;
    if (row0 < 0 || row0 >= a.total_tokens) return;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= row0) lo = mid; else hi = mid;
    }
    const int round = (1 << a.log2_block_size) - 1;
    int block[TURNS], slot[TURNS];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        block[i] = -1;
        slot[i] = 0;
        if ((uint32_t)row0 + i < most) {
            while (starts[lo + 1] <= row0 + i) ++lo;  // (ends: the last start is `most`)
            const int c = cached[lo], p = c + (row0 + i - starts[lo]), entry = p >> a.log2_block_size, held = a.grow ? (c + round) >> a.log2_block_size : 0;
            slot[i] = p & round;
            block[i] = entry < held ? a.block_table[(size_t)lo * a.max_blocks + entry] : a.block_ids[ids_before[lo] + entry - held];
        }
    }
#pragma unroll
    for (int i = 0; i < TURNS; ++i)
        if ((uint32_t)row0 + i < (uint32_t)a.total_tokens) a.slots[row0 + i] = (unsigned)block[i] < (unsigned)a.num_blocks ? ((long long)block[i] << a.log2_block_size) + slot[i] : -1;
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
    const size_t rows = std::min((size_t)a.n_req, (size_t)kTableEntries / a.max_blocks + 2);
    const size_t lds = std::max(a.slots ? (3 * (size_t)a.n_req + 1) * sizeof(int) : 0, rows * sizeof(Held));
    if (a.n_req <= kTableThreads)
        hipLaunchKernelGGL(batch_tables<1>, grid, block, lds, stream, a);
    else if (a.n_req <= 4 * kTableThreads)
        hipLaunchKernelGGL(batch_tables<4>, grid, block, lds, stream, a);
    else
        hipLaunchKernelGGL(batch_tables<32>, grid, block, lds, stream, a);
    return hipGetLastError();
}

}  // namespace lamps
