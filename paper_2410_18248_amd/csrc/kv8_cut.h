// How a launch of many new tokens over a cache of 8 bits divides its work: the arithmetic alone, the same in the kernel of the tiles, in the one that adds
// their parts up behind it, and on the host (where a test walks through it).  The two kernels find the same parts each for itself, so it is whole numbers
// throughout: nothing that a compiler may round or contract one way in one of them and another way in the other.
#pragma once
#include <stdint.h>

#ifndef __HIP__
#define __host__
#define __device__
#endif

namespace lamps {
namespace cut8 {

constexpr int kLog2Places = 9;           // 512 workgroups are what the chip holds at once, two to a CU
constexpr int kLeastStages = 8;          // of a part
constexpr int kWorth = 16;               // by which a tile is longer, where it is worth a sum of parts
constexpr int kTries = 12;
constexpr int kMostSize = 1 << 26;       // stages: as many as a row can have
constexpr int kMostTiles = 1 << 20;      // of a request that count: with more an even share is longer than any of them

// Stages of a request's tiles, each taken as long as its last one: below 2^46.
__host__ __device__ inline uint64_t work_of(int stages, int tiles) { return (uint64_t)(unsigned)stages * (unsigned)(tiles < kMostTiles ? tiles : kMostTiles); }
// Of all requests' work and kv heads an even share of 2^log2_places, and a part's size to begin with: more than that share, so that parts, n / size + 1 of a
// tile with n > size stages, are fewer than twice the places.
__host__ __device__ inline int first_size(uint64_t work, int heads, int log2_places)
{
    if (work >= (uint64_t)kMostSize << log2_places) return kMostSize;
    const uint64_t even = (work * (unsigned)heads >> log2_places) + 1;
    return even > kMostSize ? kMostSize : even > kLeastStages ? (int)even : kLeastStages;
}
// Nothing is cut where no tile has more stages than this.  Parts cost their beginnings and a sum.  By a size of 1.5 shares (few tiles: one) and more / so, us, 32 / 8 heads:
// one prompt of 1 000 37 / 26, 4 of 400 27 / 19, 12 of 30 tokens on 500 22 / 16; 16 / 4 heads of 256, 1 000 39 / 33.  Few tiles by 2 shares and 32 more: 4 of 128 on 2 000 53 / 40.
__host__ __device__ inline int least_cut(int size, bool later) { return later ? 2 * size + kWorth : size + size / 2 > kWorth + 4 ? size + size / 2 : kWorth + 4; }
// Parts of a tile that is cut if it has more than `worth` stages.
__host__ __device__ inline int runs_of(int stages, int size, int worth) { return stages > worth ? (int)((unsigned)(stages + size - 1) / (unsigned)size) : 1; }
// Where the parts are added up by a second launch they are of about one size, and the chip holds all of them at once: from an even share their size goes up until there are no
// more of them than places (12 responses of 4 to 64 tokens on 300 to 30 000, 32 / 8 heads, by tiles that had two buffers yet: 853 parts of an even share and up to half as much again, 114 us; 504
// so, 84; the line of all tiles in even shares, the ends of tiles in the middle of one, 90 to 96: two workgroups of a CU share what they wait for, and a tile's beginning and end cost
// what 8 stages do).
__host__ __device__ inline int next_size(int size) { return size + size / 16 + 1; }

// Stages of each part of a tile of `units`, and parts that there are then: one of earlier tokens may have fewer stages than the request's last one, by which
// the parts are counted.
struct Parts {
    int each, count;
};
__host__ __device__ inline Parts parts_of(int units, int runs)
{
    const int most = units / (kLeastStages / 2), want = runs < most ? runs : most, n = want > 1 ? want : 1;
    const int each = (int)((unsigned)(units + n - 1) / (unsigned)n);
    return Parts{each, (int)((unsigned)(units + each - 1) / (unsigned)each)};
}

// Positions that anything of a launch sees at most: a table row, or a window, the first positions, and what the other tokens of a tile see beside the first one's.
inline long long most_seen(long long row, int window, int sinks, int tokens)
{
    const long long seen = (long long)window + sinks + tokens - 1;
    return seen < row ? seen : row;
}
// Whether the parts of tiles of new tokens are added up by a second launch: few tiles (`tiles`: of all kv heads), where contexts may be seen that it cuts.  The last part to arrive adds
// up: the responses 109 us, 16 tokens on 8 000 49; a second launch: 84 and 21.  (Behind a launch that cuts nothing it is time lost: 12 tokens that see the last 256 and 512 of 8 000
// 16.4 and 20.5, without it 14.4 and 18.5.)
inline bool tiles_later(long long tiles, long long seen) { return tiles < 1 << kLog2Places && seen > 32 * (2 * kLeastStages + kWorth); }
// The same of one new token per request, by ranges: (request, kv head or pass).  Few, all of which may be cut: parts for one workgroup to a CU, and a second launch for the sums, whose
// workgroups share the parts of a range: by the last of them to arrive, which is alone with them, / so, us: one request of 30 000 on 32 / 8 heads 19.6 / 17.0, 60 000 on 32 / 4 28.0 /
// 18.1, 8 000 14.1 / 10.9, 1 999 10.0 / 9.5; 16 of 2 000 15.2 / 16.6, 200 of 100 to 4 000 on 8 / 2 heads of 64 14.8 / 21.1.  No gain where 1 024 positions at most are seen: 100 6.1 / 7.3, 700
// 8.3 / 8.6 (all by the last / by a second launch); the last 256 of 8 000 5.9 / 8.6.
inline bool ranges_later(long long ranges, long long seen) { return ranges < 128 && seen > 1024; }

}  // namespace cut8
}  // namespace lamps
