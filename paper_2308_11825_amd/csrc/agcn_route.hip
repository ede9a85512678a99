// Rows sent to groups (experts, types) and back.
//
// A row t has k slots j = t k + c, each with the id of a group. k_group_* sort the slots
// by group, stably: place[j] = number of slots of lower groups + number of earlier slots
// of the same group. Slots whose id is no group come after all others; their place p is
// written as -1 - p. k_dispatch lays the rows out that way, k_combine adds them up per
// row again, with weights, and k_combine_grad gives that sum's gradients.
#include <algorithm>

#include "agcn_rows.hpp"
#include "agcn_row_tiles.hpp"

namespace agcn {

namespace {

struct SortArgs {
  uint32_t slots;
  int32_t k, groups;
  const void* ids;
  int64_t ldi;
  int32_t* offsets;  // groups + 1
  int32_t* place;
  int64_t ldp;
  int32_t* counts;  // [tiles][groups + 1], and [groups + 1] sums over the tiles
  int32_t tiles;
  uint32_t chunk;  // slots of a wave, whole steps of 64
};

template <class ID>
__device__ __forceinline__ int32_t group_of(const SortArgs& a, uint32_t slot) {
  const uint32_t t = slot / (uint32_t)a.k, c = slot % (uint32_t)a.k;
  const ID id = static_cast<const ID*>(a.ids)[(int64_t)t * a.ldi + c];
  return id >= 0 && id < (ID)a.groups ? (int32_t)id : a.groups;
}
__device__ __forceinline__ void write_place(const SortArgs& a, uint32_t slot, int32_t key, int32_t p) {
  const uint32_t t = slot / (uint32_t)a.k, c = slot % (uint32_t)a.k;
  a.place[(int64_t)t * a.ldp + c] = key == a.groups ? -1 - p : p;
}

// The lanes of `active` with this lane's key, of `bits` bits.
__device__ __forceinline__ uint64_t same_key(int32_t key, uint64_t active, int bits) {
  uint64_t same = active;
  for (int b = 0; b < bits; ++b) {
    const uint64_t ones = __ballot(key >> b & 1);
    same &= (key >> b & 1) ? ones : ~ones;
  }
  return same;
}
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// What the wave's lanes wrote to LDS before is what they read after.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ int wave_scan(int v) {  // inclusive
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int up = __shfl_up(v, d);
    if (lane >= d) v += up;
  }
  return v;
}
// Exclusive sums over the workgroup's threads, and the sum of all in *total. `part` holds
// a value per wave.
template <int THREADS>
__device__ __forceinline__ int block_scan(int v, int* part, int* total) {
  const int in = wave_scan(v), wave = threadIdx.x / 64;
  if (threadIdx.x % 64 == 63) part[wave] = in;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    before += w < wave ? part[w] : 0;
    sum += part[w];
  }
  __syncthreads();
  *total = sum;
  return before + in - v;
}

// Sorting takes its launches' time and little more: 192 slots 3.6 us, 262,144 11.6 in two launches
// (16.6 in three), 10^6 18.
//
// Up to kSmallSlots slots: one workgroup, each wave a run of the slots. A slot's rank among its
// wave's slots of its group, then the waves' and the groups' sums. TILED: a workgroup for each
// tile of up to that many slots, the groups' counts in all tiles having been written before;
// each adds up those of the tiles before its own and of all.
constexpr int kMostSortTiles = 256, kSmallBins = 1024, kSmallSteps = 8, kSmallSlots = 1024 * kSmallSteps;
template <class ID, bool TILED>
__global__ __launch_bounds__(1024) void k_group_small(SortArgs a, int bits) {
  __shared__ int32_t count[16][kSmallBins];
  __shared__ int32_t tile_sum[TILED ? 2 : 1][TILED ? kSmallBins : 1];
  __shared__ int part[16];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, bins = a.groups + 1;
  for (int i = threadIdx.x; i < 16 * bins; i += 1024) count[i / bins][i % bins] = 0;
  if constexpr (TILED) tile_sum[0][threadIdx.x] = tile_sum[1][threadIdx.x] = 0;
  __syncthreads();
  int32_t key[kSmallSteps], rank[kSmallSteps];
  const uint32_t first = (blockIdx.x * 16 + wave) * a.chunk;
#pragma unroll
  for (int s = 0; s < kSmallSteps; ++s) {
    const uint32_t j = first + s * 64 + lane;
    key[s] = s * 64 < a.chunk && j < a.slots ? group_of<ID>(a, j) : -1;
  }
  if constexpr (TILED) {
    const int width = 1 << bits, bin = threadIdx.x % width;
    int before = 0, all = 0;
    if (bin < bins) {
#pragma unroll 8
      for (int t = threadIdx.x / width; t < a.tiles; t += 1024 / width) {
        const int c = a.counts[(int64_t)t * bins + bin];
        before += t < (int)blockIdx.x ? c : 0;
        all += c;
      }
      atomicAdd(&tile_sum[0][bin], before);  // sums of integers: any order
      atomicAdd(&tile_sum[1][bin], all);
    }
  }
#pragma unroll
  for (int s = 0; s < kSmallSteps; ++s) {
    if (s * 64 >= a.chunk) break;
    const uint64_t same = same_key(key[s], __ballot(key[s] >= 0), bits);
    const int before = lanes_before(same), at = key[s] >= 0 ? count[wave][key[s]] : 0;
    rank[s] = at + before;
    wave_order();
    if (key[s] >= 0 && before == 0) count[wave][key[s]] = at + __popcll(same);
    wave_order();
  }
  __syncthreads();
  int sum = 0;
  if ((int)threadIdx.x < bins) {
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      const int c = count[w][threadIdx.x];
      count[w][threadIdx.x] = sum;
      sum += c;
    }
  }
  int total, start;
  if constexpr (TILED) {
    start = block_scan<1024>((int)threadIdx.x < bins ? tile_sum[1][threadIdx.x] : 0, part, &total);
  } else {
    start = block_scan<1024>(sum, part, &total);
  }
  if ((int)threadIdx.x < bins) {
    if (blockIdx.x == 0) a.offsets[threadIdx.x] = start;
    if constexpr (TILED) start += tile_sum[0][threadIdx.x];
#pragma unroll
    for (int w = 0; w < 16; ++w) count[w][threadIdx.x] += start;
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < kSmallSteps; ++s)
    if (key[s] >= 0) write_place(a, first + s * 64 + lane, key[s], count[wave][key[s]] + rank[s]);
}

// Many slots, in three launches: the groups' counts in each tile of slots, their sums over
// the tiles before, and the places. Groups are taken kBins at a time.
constexpr int kBins = 2048, kSortThreads = 256, kSortWaves = kSortThreads / 64;

template <class ID, int THREADS>
__global__ __launch_bounds__(THREADS) void k_group_count(SortArgs a) {
  __shared__ int32_t count[kBins];
  const uint32_t tile = THREADS / 64 * a.chunk, first = blockIdx.x * tile;
  const uint32_t end = min(a.slots, first + tile);
  const int bins = a.groups + 1;
  for (int base = 0; base < bins; base += kBins) {
    const int here = min(kBins, bins - base);
    for (int i = threadIdx.x; i < here; i += THREADS) count[i] = 0;
    __syncthreads();
    for (uint32_t j = first + threadIdx.x; j < end; j += THREADS) {
      const int key = group_of<ID>(a, j) - base;
      if (key >= 0 && key < here) atomicAdd(&count[key], 1);  // a sum of ones: any order
    }
    __syncthreads();
    for (int i = threadIdx.x; i < here; i += THREADS)
      a.counts[(int64_t)blockIdx.x * bins + base + i] = count[i];
    __syncthreads();
  }
}

// 16 groups a workgroup, 16 threads for the tiles of each.
__global__ __launch_bounds__(256) void k_group_tiles(SortArgs a) {
  constexpr int kEach = kMostSortTiles / 16;
  __shared__ int32_t sums[16][17];
  const int bins = a.groups + 1, bin = blockIdx.x * 16 + threadIdx.x % 16, s = threadIdx.x / 16;
  int32_t v[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int tile = s * kEach + i;
    v[i] = bin < bins && tile < a.tiles ? a.counts[(int64_t)tile * bins + bin] : 0;
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) sum += v[i];
  sums[s][threadIdx.x % 16] = sum;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) before += i < s ? sums[i][threadIdx.x % 16] : 0;
  if (bin >= bins) return;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int tile = s * kEach + i;
    if (tile < a.tiles) a.counts[(int64_t)tile * bins + bin] = before;
    before += v[i];
  }
  if (s == 15) a.counts[(int64_t)a.tiles * bins + bin] = before;
}

template <class ID>
__global__ __launch_bounds__(kSortThreads) void k_group_place(SortArgs a, int bits) {
  __shared__ int32_t next[kSortWaves][kBins];
  __shared__ int part[kSortWaves];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, bins = a.groups + 1;
  const uint32_t first = (blockIdx.x * kSortWaves + wave) * a.chunk;
  const uint32_t end = min(a.slots, first + a.chunk);
  const int32_t* before = a.counts + (int64_t)blockIdx.x * bins;
  const int32_t* sums = a.counts + (int64_t)a.tiles * bins;
  int32_t start = 0;  // of the groups from `base` on
  for (int base = 0; base < bins; base += kBins) {
    const int here = min(kBins, bins - base);
    for (int i = threadIdx.x; i < kSortWaves * kBins; i += kSortThreads) next[i / kBins][i % kBins] = 0;
    __syncthreads();
    for (uint32_t j = first + lane; j < end; j += 64) {
      const int key = group_of<ID>(a, j) - base;
      if (key >= 0 && key < here) atomicAdd(&next[wave][key], 1);
    }
    __syncthreads();
    for (int b = 0; b < here; b += kSortThreads) {
      const int i = b + threadIdx.x;
      int total;
      const int from = start + block_scan<kSortThreads>(i < here ? sums[base + i] : 0, part, &total);
      start += total;
      if (i < here) {
        if (blockIdx.x == 0) a.offsets[base + i] = from;
        int at = from + before[base + i];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
          const int c = next[w][i];
          next[w][i] = at;
          at += c;
        }
      }
    }
    __syncthreads();
    for (uint32_t j0 = first; j0 < end; j0 += 64) {
      const uint32_t j = j0 + lane;
      const int key = j < end ? group_of<ID>(a, j) : -1, in = key - base;
      const bool mine = key >= 0 && in >= 0 && in < here;
      const uint64_t same = same_key(in, __ballot(mine), bits);
      const int n = lanes_before(same), at = mine ? next[wave][in] : 0;
      wave_order();
      if (mine) {
        write_place(a, j, key, at + n);
        if (n == 0) next[wave][in] = at + __popcll(same);
      }
      wave_order();
    }
    __syncthreads();
  }
}

// --- rows -------------------------------------------------------------------------

struct RowArgs {
  int64_t n, f;  // rows of one per token, and their columns (k_dispatch: bytes)
  int32_t k;
  const int32_t* place;
  int64_t ldp;
  const float* w;  // or NULL
  int64_t ldw;
  const void* X;  // of a token
  int64_t ldx;
  const void* R;  // of a slot, n k of them
  int64_t ldr;
  void* out;  // of a token, or of a slot
  int64_t ldo;
  float* dw;
  int64_t lddw;
  bool past;  // the slots' rows and the results start on lines
};

// The row that a place names, and whether its slot is kept; places outside the matrix name
// row 0 and are not.
struct Slot {
  int64_t row;
  bool kept, inside;
  __device__ __forceinline__ Slot(const RowArgs& a, int64_t t, int c) {
    const int32_t p = a.place[t * a.ldp + c], r = p < 0 ? -1 - p : p;
    inside = r < a.n * a.k;
    row = inside ? r : 0;
    kept = p >= 0 && inside;
  }
};

// Few tokens: a token's columns (k_combine_grad: slots) over gridDim.y workgroups, `each` of them
// a workgroup and turn.
__device__ __forceinline__ int64_t part_start(int first, int each) { return first + (int64_t)blockIdx.y * each; }
__device__ __forceinline__ int64_t part_step(int each) { return (int64_t)gridDim.y * each; }

// The token of a group of G lanes: one for the whole wave in scalar registers.
template <int G>
__device__ __forceinline__ int64_t token_of(int64_t i) {
  const int64_t t = i * (256 / G) + threadIdx.x / G;
  if constexpr (G < 64) return t;
  return (int64_t)__builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)t >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)t);
}

// A row read once and written k times, U pieces of W bytes a lane at a time (the last piece of
// a row ends where the row does). Reading a row for each place costs more: the writes are in order,
// but the same row is fetched k times (32768 rows of 8 KB to 8 places each 570 us, 416 this way, 5.8
// TB/s; 478 with ordinary stores). Rows that share lines: neighbours in group order come from neighbouring
// rows, which go to one XCD, and their parts of a line meet in its L2 (100,000 x 6 x 600 bytes 93 us, 127
// with workgroups as they come).
template <int W>
using Bytes = std::conditional_t<W == 16, v4i_any, std::conditional_t<W == 4, uint32_t, uint8_t>>;
template <int W, int G, int U>
__global__ __launch_bounds__(256) void k_dispatch(RowArgs a) {
  const int lane = threadIdx.x % G;
  for (int64_t i = xcd_tile(blockIdx.x, gridDim.x); i * (256 / G) < a.n; i += gridDim.x) {
    const int64_t t = token_of<G>(i);
    if (t >= a.n) continue;
    const uint8_t* x = static_cast<const uint8_t*>(a.X) + t * a.ldx;
    for (int64_t at = part_start(lane, G * U) * W; at < a.f; at += part_step(G * U) * W) {
      Bytes<W> v[U];
      int64_t from[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        from[u] = std::min<int64_t>(at + u * G * W, a.f - W);
        v[u] = load_any<Bytes<W>>(x + from[u]);
      }
      for (int c = 0; c < a.k; ++c) {
        const Slot s(a, t, c);
        if (!s.inside) continue;
        uint8_t* to = static_cast<uint8_t*>(a.out) + s.row * a.ldo;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (u > 0 && at + u * G * W >= a.f) break;
          store_row(to + from[u], s.kept ? v[u] : Bytes<W>{}, a.past);
        }
      }
    }
  }
}

// out[t] = sum over c of w[t][c] R[place[t][c]], in c's order, A rows and U pieces of each on
// their way at a time. Bound by memory: 32768 x 8 slots x 4096 bfloat16 423 us, 5.7 TB/s.
template <class T, int V, int G, int U, int A>
__global__ __launch_bounds__(256) void k_combine(RowArgs a) {
  using P = Piece<T, V>;
  const int lane = threadIdx.x % G;
  for (int64_t i = xcd_tile(blockIdx.x, gridDim.x); i * (256 / G) < a.n; i += gridDim.x) {
    const int64_t t = token_of<G>(i);
    if (t >= a.n) continue;
    for (int64_t at = part_start(lane, G * U) * V; at < a.f; at += part_step(G * U) * V) {
      int64_t from[U];
      float sum[U][V];
#pragma unroll
      for (int x = 0; x < U; ++x) {
        from[x] = std::min<int64_t>(at + x * G * V, a.f - V);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[x][e] = 0.0f;
      }
      for (int c0 = 0; c0 < a.k; c0 += A) {
        P v[A][U];
        float w[A];
        bool kept[A];
#pragma unroll
        for (int u = 0; u < A; ++u) {
          const int c = min(c0 + u, a.k - 1);
          const Slot s(a, t, c);
          kept[u] = s.kept && c0 + u < a.k;
          w[u] = a.w != nullptr ? a.w[t * a.ldw + c] : 1.0f;
          load_row(v[u], static_cast<const T*>(a.R) + s.row * a.ldr, from, a.past);
        }
#pragma unroll
        for (int u = 0; u < A; ++u)
#pragma unroll
          for (int x = 0; x < U; ++x)
#pragma unroll
            for (int e = 0; e < V; ++e)
              sum[x][e] = kept[u] ? fmaf(w[u], to_float(v[u][x].e[e]), sum[x][e]) : sum[x][e];
      }
#pragma unroll
      for (int x = 0; x < U; ++x) {
        if (x > 0 && at + x * G * V >= a.f) break;
        P o;
#pragma unroll
        for (int e = 0; e < V; ++e) o.e[e] = (T)sum[x][e];
        store_row(static_cast<T*>(a.out) + t * a.ldo + from[x], o, a.past);
      }
    }
  }
}

// dR[place[t][c]] = w[t][c] X[t] and dw[t][c] = X[t] . R[place[t][c]], X the gradient of
// k_combine's sum. A group of lanes has a whole token, A slots and U pieces of each at a time: 16384
// x 8 slots x 4096 bfloat16 438 us, 5.2 TB/s of reads and writes of rows in no order.
template <class T, int V, int G, int U, int A>
__global__ __launch_bounds__(256) void k_combine_grad(RowArgs a) {
  using P = Piece<T, V>;
  const int lane = threadIdx.x % G;
  for (int64_t i = xcd_tile(blockIdx.x, gridDim.x); i * (256 / G) < a.n; i += gridDim.x) {
    const int64_t t = token_of<G>(i);
    if (t >= a.n) continue;
    for (int64_t c0 = part_start(0, A); c0 < a.k; c0 += part_step(A)) {
      int64_t row[A];
      float w[A], dot[A];
      bool kept[A], inside[A];
#pragma unroll
      for (int u = 0; u < A; ++u) {
        const int c = (int)std::min<int64_t>(c0 + u, a.k - 1);
        const Slot s(a, t, c);
        row[u] = s.row;
        kept[u] = s.kept;
        inside[u] = s.inside && c0 + u < a.k;
        w[u] = s.kept ? a.w[t * a.ldw + c] : 0.0f;
        dot[u] = 0.0f;
      }
      for (int64_t at = lane * V; at < a.f; at += G * V * U) {
        P x[U], r[A][U];
        int64_t from[U];
#pragma unroll
        for (int y = 0; y < U; ++y) {
          from[y] = std::min<int64_t>(at + y * G * V, a.f - V);
          x[y] = load_any<P>(static_cast<const T*>(a.X) + t * a.ldx + from[y]);
        }
#pragma unroll
        for (int u = 0; u < A; ++u) load_row(r[u], static_cast<const T*>(a.R) + row[u] * a.ldr, from, a.past);
#pragma unroll
        for (int y = 0; y < U; ++y) {
          if (y > 0 && at + y * G * V >= a.f) break;
          const int shared = (int)(at + y * G * V - from[y]);
#pragma unroll
          for (int u = 0; u < A; ++u) {
            P o;
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float g = to_float(x[y].e[e]);
              o.e[e] = (T)(kept[u] ? w[u] * g : 0.0f);
              dot[u] = e >= shared ? fmaf(g, to_float(r[u][y].e[e]), dot[u]) : dot[u];
            }
            if (inside[u]) store_row(static_cast<T*>(a.out) + row[u] * a.ldo + from[y], o, a.past);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < A; ++u) {
        const float d = lanes_sum<G>(dot[u]);
        if (lane == 0 && c0 + u < a.k) a.dw[t * a.lddw + c0 + u] = kept[u] ? d : 0.0f;
      }
    }
  }
}

// Workgroups of a launch, at most; rows past them are looped over.
constexpr int64_t kMostGroups = 1 << 20;
template <int G>
dim3 row_grid(int64_t n, int64_t parts) {
  const int64_t groups = std::max<int64_t>(1, std::min<int64_t>(kMostGroups, ceil_div64(n, 256 / G)));
  // Up to four workgroups a compute unit, as far as a token has `parts`: a workgroup's pieces of its columns (512
  // of 16 bytes where rows are over 4 KB: 48 x 4096 bfloat16 stay 48 workgroups) or, for k_combine_grad, A of its
  // slots (two parts of 8). k_combine of 200 x 8 slots x 8192 bfloat16 6.8 us, 9.6 with a workgroup a token;
  // k_combine_grad 22 and 37 (100 workgroups: four tokens each, in two parts), of 48 x 8 x 4096 9.5 and 16.5; k_dispatch
  // 6.0 and 7.0.
  return dim3((unsigned)groups, (unsigned)std::max<int64_t>(1, std::min<int64_t>(parts, 1024 / groups)));
}

int bits_of(int bins) {
  int bits = 0;
  while (1 << bits < bins) ++bits;
  return bits;
}

// How a sort is cut: tiles, and slots of a wave of each, whole steps of 64.
struct SortShape {
  bool small;  // a tile is kSmallSlots slots at most, for k_group_small
  int32_t tiles;
  uint32_t chunk;
};
SortShape sort_shape(int64_t slots, int32_t groups) {
  auto steps = [slots](int64_t waves) { return ceil_div64(slots, 64 * waves); };
  if (groups < kSmallBins && slots <= kSmallSlots) return {true, 1, (uint32_t)steps(16) * 64};
  if (groups < kSmallBins && slots <= (int64_t)kSmallSlots * kMostSortTiles) {
    const int64_t chunk = std::min<int64_t>(kSmallSteps, steps(16 * 64)) * 64;  // about 64 tiles, or more
    return {true, (int32_t)ceil_div64(slots, 16 * chunk), (uint32_t)chunk};
  }
  const int64_t chunk = std::max<int64_t>(4, steps(kMostSortTiles * kSortWaves)) * 64;
  return {false, (int32_t)std::max<int64_t>(1, ceil_div64(slots, kSortWaves * chunk)), (uint32_t)chunk};
}

template <class ID>
int sort_typed(SortArgs a, hipStream_t st) {
  const int bins = a.groups + 1;
  const SortShape s = sort_shape(a.slots, a.groups);
  a.tiles = s.tiles;
  a.chunk = s.chunk;
  if (s.small && s.tiles == 1) {
    k_group_small<ID, false><<<1, 1024, 0, st>>>(a, bits_of(bins));
    return launched("k_group_small launch");
  }
  if (s.small) {
    k_group_count<ID, 1024><<<(unsigned)a.tiles, 1024, 0, st>>>(a);
    if (int rc = launched("k_group_count launch")) return rc;
    k_group_small<ID, true><<<(unsigned)a.tiles, 1024, 0, st>>>(a, bits_of(bins));
    return launched("k_group_small launch");
  }
  k_group_count<ID, kSortThreads><<<(unsigned)a.tiles, kSortThreads, 0, st>>>(a);
  if (int rc = launched("k_group_count launch")) return rc;
  k_group_tiles<<<(unsigned)ceil_div64(bins, 16), 256, 0, st>>>(a);
  if (int rc = launched("k_group_tiles launch")) return rc;
  k_group_place<ID><<<(unsigned)a.tiles, kSortThreads, 0, st>>>(a, bits_of(std::min(bins, kBins)));
  return launched("k_group_place launch");
}

// Lanes a token (G) and pieces a lane at a time (NV) by a row's pieces, and slots at a time
// (A) by k. Short rows take few lanes, so that a wave has several tokens' loads on their way: us on
// one MI355X, 60,000 x 2 slots x 601 float16 45 in 32 lanes of 3 pieces, 48 in 64 of 2, 60 in 256
// of 1; 200,000 x 128 float32 37 in 16 of 2, 56 in 64 of 1.
template <bool SHORT, class F>  // SHORT: 8 pieces at most
void token_shape(int64_t p, F use) {
  if constexpr (SHORT) {
    use(Shape<8, 1>{});
  } else {
    if (p <= 4) use(Shape<4, 1>{});
    else if (p <= 8) use(Shape<8, 1>{});
    else if (p <= 16) use(Shape<16, 1>{});
    else if (p <= 32) use(Shape<16, 2>{});
    else if (p <= 48) use(Shape<16, 3>{});
    else if (p <= 64) use(Shape<16, 4>{});
    else if (p <= 96) use(Shape<32, 3>{});
    else if (p <= 128) use(Shape<32, 4>{});
    else use(Shape<64, 4>{});
  }
}
template <class F>
void slots_at_once(int32_t k, F use) {
  if (k <= 1) use(std::integral_constant<int, 1>{});
  else if (k == 2) use(std::integral_constant<int, 2>{});
  else if (k % 3 == 0 && k % 4 != 0) use(std::integral_constant<int, 3>{});
  else use(std::integral_constant<int, 4>{});
}

template <class T, int V>
int combine_pieces(const RowArgs& a, hipStream_t st) {
  const int64_t pieces = ceil_div64(a.f, V);
  slots_at_once(a.k, [&](auto at_once) {
    constexpr int A = decltype(at_once)::value;
    // Rows over 4 KB: the lanes of four waves, two pieces each.
    if (V > 1 && pieces > 256) {
      k_combine<T, V, 256, 2, A><<<row_grid<256>(a.n, ceil_div64(pieces, 512)), 256, 0, st>>>(a);
      return;
    }
    token_shape<V == 1>(pieces, [&](auto shape) {
      constexpr int G = decltype(shape)::kG, U = decltype(shape)::kNV;
      k_combine<T, V, G, U, A><<<row_grid<G>(a.n, ceil_div64(pieces, G * U)), 256, 0, st>>>(a);
    });
  });
  return launched("k_combine launch");
}
template <class T, int V>
int combine_grad_pieces(const RowArgs& a, hipStream_t st) {
  slots_at_once(a.k, [&](auto at_once) {
    constexpr int A = decltype(at_once)::value;
    token_shape<V == 1>(ceil_div64(a.f, V), [&](auto shape) {
      constexpr int G = decltype(shape)::kG, U = decltype(shape)::kNV;
      k_combine_grad<T, V, G, U, A><<<row_grid<G>(a.n, ceil_div64(a.k, A)), 256, 0, st>>>(a);
    });
  });
  return launched("k_combine_grad launch");
}

template <class T>
int combine_typed(RowArgs a, bool grad, hipStream_t st) {
  constexpr int V = kPiece<T>;
  a.past = on_lines(a.R, a.ldr, sizeof(T)) && on_lines(a.out, a.ldo, sizeof(T));
  if (a.f < V) return grad ? combine_grad_pieces<T, 1>(a, st) : combine_pieces<T, 1>(a, st);
  return grad ? combine_grad_pieces<T, V>(a, st) : combine_pieces<T, V>(a, st);
}
int combine_any(const RowArgs& a, int32_t dtype, bool grad, hipStream_t st) {
  if (dtype == AGCN_FLOAT) return combine_typed<float>(a, grad, st);
  return dtype == AGCN_BFLOAT ? combine_typed<bf16_t>(a, grad, st) : combine_typed<f16_t>(a, grad, st);
}

template <int W>
int dispatch_pieces(const RowArgs& a, hipStream_t st) {
  const int64_t pieces = ceil_div64(a.f, W);
  if (pieces <= 1) k_dispatch<W, 1, 1><<<row_grid<1>(a.n, ceil_div64(pieces, 1)), 256, 0, st>>>(a);
  else if (pieces <= 4) k_dispatch<W, 4, 1><<<row_grid<4>(a.n, ceil_div64(pieces, 4)), 256, 0, st>>>(a);
  else if (pieces <= 16 || W < 16) k_dispatch<W, 16, 1><<<row_grid<16>(a.n, ceil_div64(pieces, 16)), 256, 0, st>>>(a);
  else if (pieces <= 64) k_dispatch<W, 64, 1><<<row_grid<64>(a.n, ceil_div64(pieces, 64)), 256, 0, st>>>(a);
  else if (pieces <= 128) k_dispatch<W, 64, 2><<<row_grid<64>(a.n, ceil_div64(pieces, 128)), 256, 0, st>>>(a);
  else k_dispatch<W, 256, 2><<<row_grid<256>(a.n, ceil_div64(pieces, 512)), 256, 0, st>>>(a);
  return launched("k_dispatch launch");
}

}  // namespace

size_t sort_workspace_bytes(int64_t slots, int32_t groups) {
  const SortShape s = sort_shape(slots, groups);
  if (s.small && s.tiles <= 1) return 0;
  return (size_t)(s.tiles + 1) * ((size_t)groups + 1) * sizeof(int32_t);
}

int run_sort_groups(int64_t n, int32_t k, int32_t groups, const void* ids, int32_t id_bytes, int64_t ldi,
                    int32_t* offsets, int32_t* place, int64_t ldp, void* ws, hipStream_t st) {
  const SortArgs a{(uint32_t)(n * k), std::max(k, 1), groups, ids, ldi, offsets, place, ldp,
                   static_cast<int32_t*>(ws), 0, 0};
  return id_bytes == 8 ? sort_typed<int64_t>(a, st) : sort_typed<int32_t>(a, st);
}

int run_dispatch(int64_t n, int32_t k, int64_t bytes, const void* X, int64_t ldx, const int32_t* place, int64_t ldp,
                 void* Y, int64_t ldy, hipStream_t st) {
  if (n == 0 || k == 0 || bytes == 0) return AGCN_OK;
  RowArgs a{};
  a.n = n, a.f = bytes, a.k = k, a.place = place, a.ldp = ldp, a.X = X, a.ldx = ldx, a.out = Y, a.ldo = ldy;
  a.past = on_lines(Y, ldy, 1);
  if (bytes >= 16) return dispatch_pieces<16>(a, st);
  return bytes >= 4 ? dispatch_pieces<4>(a, st) : dispatch_pieces<1>(a, st);
}

int run_combine(int64_t n, int32_t k, int32_t f, int32_t dtype, const void* R, int64_t ldr, const int32_t* place,
                int64_t ldp, const float* w, int64_t ldw, void* out, int64_t ldo, hipStream_t st) {
  if (n == 0 || f == 0) return AGCN_OK;
  RowArgs a{};
  a.n = n, a.f = f, a.k = k, a.place = place, a.ldp = ldp, a.w = w, a.ldw = ldw, a.R = R, a.ldr = ldr;
  a.out = out, a.ldo = ldo;
  return combine_any(a, dtype, false, st);
}

int run_combine_backward(int64_t n, int32_t k, int32_t f, int32_t dtype, const void* dOut, int64_t lddo,
                         const void* R, int64_t ldr, const int32_t* place, int64_t ldp, const float* w, int64_t ldw,
                         void* dR, int64_t lddr, float* dw, int64_t lddw, hipStream_t st) {
  if (n == 0 || k == 0) return AGCN_OK;
  RowArgs a{};
  a.n = n, a.f = f, a.k = k, a.place = place, a.ldp = ldp, a.w = w, a.ldw = ldw, a.X = dOut, a.ldx = lddo;
  a.R = R, a.ldr = ldr, a.out = dR, a.ldo = lddr, a.dw = dw, a.lddw = lddw;
  return combine_any(a, dtype, true, st);
}

}  // namespace agcn
