// Shared by the kernels that hold a row in registers (agcn_norm.hip, agcn_quant.hip) or walk
// over rows (agcn_route.hip).
//
// Lanes take 16 bytes of a row at a time. In rows that do not end on such a piece the last
// lane's piece is the row's last 16 bytes; the columns that it shares with the lane before
// count there only, and both lanes write the same values, so no lane has a shorter way of
// its own. Rows shorter than a piece are taken value by value.
#pragma once

#include <algorithm>

#include "agcn_quant.hpp"

namespace agcn {

template <class T, int V>
struct alignas(sizeof(T)) Piece {
  T e[V];
};

// Where lane `lane`'s v-th piece of V columns starts, and how many of its first columns
// belong to another lane (V: all of them).
template <int G, int V>
struct Column {
  int start, shared;
  __device__ __forceinline__ Column(int v, int lane, int f) {
    const int c = (v * G + lane) * V;
    start = max(min(c, f - V), 0);
    shared = min(c - start, V);
  }
};

// Sums over the G lanes of a row that one wave has (all of them for G <= 64).
template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
  v = sum16(v);
  if constexpr (G >= 32) v += __shfl_xor(v, 16);
  if constexpr (G >= 64) v += __shfl_xor(v, 32);
  return v;
}

// Lanes a row and pieces a lane by the row's pieces: the fewest idle lanes, and one piece a
// lane as long as a workgroup has the lanes. Calls use(Shape), or returns false for rows that
// are too long.
template <int G, int NV>
struct Shape {
  static constexpr int kG = G, kNV = NV;
};
template <class F>
bool row_shape(int64_t pieces, F use) {
  if (pieces <= 16) use(Shape<16, 1>{});
  else if (pieces <= 32) use(Shape<32, 1>{});
  else if (pieces <= 48) use(Shape<16, 3>{});
  else if (pieces <= 64) use(Shape<64, 1>{});
  else if (pieces <= 96) use(Shape<32, 3>{});
  else if (pieces <= 128) use(Shape<64, 2>{});
  else if (pieces <= 192) use(Shape<64, 3>{});
  else if (pieces <= 256) use(Shape<256, 1>{});
  else if (pieces <= 512) use(Shape<512, 1>{});
  else if (pieces <= 1024) use(Shape<1024, 1>{});
  else if (pieces <= 2048) use(Shape<1024, 2>{});
  else return false;
  return true;
}
template <class T>
inline constexpr int kPiece = 16 / (int)sizeof(T);

inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AGCN_OK : hip_fail(e, what);
}

}  // namespace agcn
