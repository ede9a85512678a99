// The rows of a matrix, or of its groups, cut into tiles, one workgroup each: which rows a
// workgroup of agcn_qlinear.hip's kernels works on. The groups' offsets are device memory
// that the caller may fill with anything; whatever they hold, a tile lies inside the matrix.
//
// Needs HIP's device functions (hip_runtime.h) or, on the host, stand-ins for them.
#pragma once

#include <algorithm>
#include <cstdint>

namespace agcn {

// Workgroups of a launch, at most: 2^31 - 1 threads of 256.
constexpr int64_t kMostTiles = INT32_MAX / 256;

// Rows of `blocks` blocks of 128 columns that one launch quantises, at most: 16 blocks a
// workgroup of 256 threads.
constexpr int64_t most_quantized_rows(int64_t blocks) {
  return std::max<int64_t>(1, kMostTiles * 16 / blocks);
}

// The rows a tile of at most BM rows works on: rows [row, row + count) of group
// `group`, or rows of no group (group -1), which are set to 0.
struct Rows {
  int64_t row;
  int32_t count, group;
};

// The rows cut at the groups' offsets, in tiles of BM. The rows before the first
// offset and after the last are parts of their own without a group, so that the
// parts cover all rows. Offsets are clamped to [0, n] and a part that would be
// negative is empty, so no offsets reach past the matrices. Every lane of a wave makes the
// calls, with 64 parts looked at per step.
//
// Up to kScanned parts each workgroup adds their tiles up, and the tiles there are go to the
// first workgroups, so that all XCDs have as many: 32768 x 4096 -> 2048 over 64 groups 306 us,
// 318 with a search. But that costs groups times tiles. With more parts the workgroups are
// slots with a place for every tile that any offsets may make, some of them empty, and a
// slot's part is searched for among 64 at a time: 32,000 x 2048 -> 1024 over 250 groups 112 us, 116
// added up; 300 rows x 128 -> 128 for each of 250 groups 11.4 and 15.8, of 1000 groups 29 and 95, of
// 5000 174 and 1867.
//
// Offsets that decrease make parts that overlap, with any number of tiles in all: sums of
// tiles end at what is asked of them, so they stay in 32 bits (64 lanes of 2^23 tiles at
// most, kMostTiles).
constexpr int kScanned = 128;
template <int BM>
struct GroupTiles {
  const int32_t* offsets;
  int n, parts;
  template <class Args>  // with the members n, offsets and groups
  __device__ __forceinline__ explicit GroupTiles(const Args& p)
      : offsets(p.offsets), n((int)p.n), parts(p.groups + 2) {}
  // The lane's part of a step: rows [*lo, *hi), and its tiles.
  __device__ __forceinline__ int part(int base, int* lo, int* hi) const {
    const int i = base + (int)(threadIdx.x % 64);
    *lo = *hi = 0;
    if (i < parts) {
      *lo = i == 0 ? 0 : min(max(offsets[i - 1], 0), n);
      *hi = i == parts - 1 ? n : min(max(offsets[i], 0), n);
    }
    return *hi > *lo ? (int)(((int64_t)(*hi - *lo) + BM - 1) / BM) : 0;
  }
  // The tiles of all parts, or `most` where they are more.
  __device__ __forceinline__ int total(int most) const {
    int sum = 0;
    for (int base = 0; base < parts; base += 64) {
      int lo, hi;
      sum += min(part(base, &lo, &hi), most - sum);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    return __builtin_amdgcn_readfirstlane(min(sum, most));
  }
  // Tile `tile` >= 0 of all parts' tiles. (A part's tiles past that one do not change what is
  // found.)
  __device__ __forceinline__ Rows find(int tile) const {
    const int lane = threadIdx.x % 64;
    for (int base = 0; base < parts; base += 64) {
      int lo, hi;
      const int tiles = min(part(base, &lo, &hi), tile + 1);
      int end = tiles;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int up = __shfl_up(end, d);
        if (lane >= d) end += up;
      }
      const uint64_t hit = __ballot(tile < end);
      if (hit != 0) {
        const int at = __ffsll((unsigned long long)hit) - 1;
        const int first = __shfl(end, at) - __shfl(tiles, at), i = base + at;
        const int row = __shfl(lo, at) + (tile - first) * BM;
        return {__builtin_amdgcn_readfirstlane(row),
                __builtin_amdgcn_readfirstlane(min(BM, __shfl(hi, at) - row)),
                __builtin_amdgcn_readfirstlane(i == 0 || i == parts - 1 ? -1 : i - 1)};
      }
      tile -= __shfl(end, 63);
    }
    return {0, 0, -1};
  }
  // The first slot of part i. Neighbouring parts' slots are rows / BM apart and one more, as
  // many as a part can have tiles (without the one for SKIP = 1). Few rows among many parts:
  // a slot per row, and a tile at the slot of its first row.
  template <int SKIP>
  __device__ __forceinline__ int64_t slot(int i, bool by_row) const {
    const int lo = i == 0 ? 0 : min(max(offsets[i - 1], 0), n);
    return by_row ? lo : lo / BM + (SKIP == 0 ? i : 0);
  }
  // The tile of slot `at`, as find() gives it, or none: the last part that starts at the slot
  // or before has it.
  template <int SKIP>
  __device__ __forceinline__ Rows search(uint32_t at) const {
    const bool by_row = SKIP == 0 && n < n / BM + (int64_t)parts;
    int first = 0, count = parts;  // it is among these
    while (count > 1) {
      const int step = (count + 63) / 64, i = first + (int)(threadIdx.x % 64) * step;
      const uint64_t from = __ballot(i < first + count && slot<SKIP>(i, by_row) <= at);
      const int last = __builtin_amdgcn_readfirstlane(from == 0 ? 0 : 63 - __clzll((long long)from)) * step;
      count = min(step, count - last);
      first += last;
    }
    const int64_t lo = first == 0 ? 0 : min(max(offsets[first - 1], 0), n);
    const int64_t hi = first == parts - 1 ? n : min(max(offsets[first], 0), n);
    const int64_t past = (int64_t)at - slot<SKIP>(first, by_row);
    if (past < 0 || (by_row && past % BM != 0)) return {0, 0, -1};
    const int64_t row = lo + (by_row ? past : (SKIP + past) * BM);
    if (row >= hi) return {0, 0, -1};
    return {__builtin_amdgcn_readfirstlane((int)row),
            __builtin_amdgcn_readfirstlane((int)min((int64_t)BM, hi - row)),
            first == 0 || first == parts - 1 ? -1 : first - 1};
  }
};

// The rows of workgroup y where groups have few: the first BM of part y, found without
// a search; tiles past a part's first have slots after the parts' workgroups.
template <int BM, bool GROUPED, class Args>
__device__ __forceinline__ Rows few_rows(const Args& p) {
  if constexpr (!GROUPED) {
    const int64_t row = (int64_t)blockIdx.y * BM;
    return {row, (int32_t)min((int64_t)BM, p.n - row), 0};
  } else {
    const int n = (int)p.n, i = blockIdx.y, last = p.groups + 1;
    if (i > last) return GroupTiles<BM>(p).template search<1>((uint32_t)(i - last - 1));
    const int lo = i == 0 ? 0 : min(max(p.offsets[i - 1], 0), n);
    const int hi = i == last ? n : min(max(p.offsets[i], 0), n);
    return {__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(min(BM, hi - lo)),
            i == 0 || i == last ? -1 : i - 1};
  }
}
inline int64_t few_rows_grid(int64_t n, int32_t groups, int64_t bm, bool grouped) {
  return grouped ? groups + 2 + n / bm : (n + bm - 1) / bm;
}

// Tiles that any offsets cut n rows into, at most.
inline int64_t most_slots(int64_t n, int32_t groups, int64_t bm) {
  return std::min<int64_t>(n, n / bm + groups + 2);
}

// Workgroup `i` of `total` as the tile that keeps neighbouring tiles on one of the 8
// XCDs (workgroups go to them in turn), each with its own L2.
__device__ __forceinline__ uint32_t xcd_tile(uint32_t i, uint32_t total) {
  const uint32_t q = total / 8, r = total % 8, x = i % 8;
  return x * q + min(x, r) + i / 8;
}

// The rows and the column tile of this workgroup: bands of group_m row tiles, in each
// the row tiles of one column tile after another. The grid of a grouped product
// has room for any offsets.
template <int BM, bool GROUPED, class Args>
__device__ __forceinline__ Rows tile_rows(const Args& p, uint32_t tiles_n, uint32_t group_m,
                                          uint32_t* tn) {
  uint32_t tiles_m = gridDim.x / tiles_n;
  if constexpr (GROUPED) {
    if (p.groups + 2 <= kScanned) tiles_m = (uint32_t)GroupTiles<BM>(p).total((int)tiles_m);
    if (blockIdx.x >= tiles_m * tiles_n) return {0, 0, -1};
  }
  const uint32_t tile = xcd_tile(blockIdx.x, tiles_m * tiles_n);
  const uint32_t band = tile / (group_m * tiles_n), in = tile % (group_m * tiles_n);
  const uint32_t high = min(group_m, tiles_m - band * group_m);
  // (Divisions are vector code; the buffers built on their results must be scalar.)
  const uint32_t tm = __builtin_amdgcn_readfirstlane(band * group_m + in % high);
  *tn = __builtin_amdgcn_readfirstlane(in / high);
  if constexpr (GROUPED)
    return p.groups + 2 <= kScanned ? GroupTiles<BM>(p).find((int)tm)
                                    : GroupTiles<BM>(p).template search<0>(tm);
  const int64_t row = (int64_t)tm * BM;
  return {row, (int32_t)min((int64_t)BM, p.n - row), 0};
}

}  // namespace agcn
