// Shared by the kernels that hold a row in registers (agcn_norm.hip, agcn_quant.hip) or walk
// over rows (agcn_route.hip).
//
// Lanes take 16 bytes of a row at a time. In rows that do not end on such a piece the last
// lane's piece is the row's last 16 bytes; the columns that it shares with the lane before
// count there only, and both lanes write the same values, so no lane has a shorter way of
// its own. Rows shorter than a piece are taken value by value.
#pragma once

#include <algorithm>
#include <type_traits>

#include "agcn_quant.hpp"

namespace agcn {

template <class T, int V>
struct alignas(sizeof(T)) Piece {
  T e[V];
};

// A piece read or written past the caches that will not see it again (PAST, where rows start
// on 128-byte lines: a line that two rows share is better put together in L2).
typedef int v4i_any __attribute__((ext_vector_type(4), aligned(1)));
template <class V, bool PAST, class T>
__device__ __forceinline__ V load_row(const T* p) {
  if constexpr (PAST && sizeof(V) == 16)
    return __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const v4i_any*>(p)));
  else
    return load_any<V>(p);
}
template <bool PAST, class T, class V>
__device__ __forceinline__ void store_row(T* p, const V& v) {
  if constexpr (PAST && sizeof(V) == 16) {
    v4i_any t;
    __builtin_memcpy(&t, &v, 16);
    __builtin_nontemporal_store(t, reinterpret_cast<v4i_any*>(p));
  } else {
    store_any(p, v);
  }
}
// The same decided when it runs, for kernels of many shapes. (Between the two empty statements
// nothing is moved: the compiler would make one access of both ways, and an ordinary one.)
template <int N, class V, class T, class At>
__device__ __forceinline__ void load_row(V (&v)[N], const T* p, const At (&at)[N], bool past) {
  if (past) {
    asm volatile("");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = load_row<V, true>(p + at[i]);
    asm volatile("");
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = load_any<V>(p + at[i]);
  }
}
template <class T, class V>
__device__ __forceinline__ void store_row(T* p, const V& v, bool past) {
  if (past) {
    asm volatile("");
    store_row<true>(p, v);
    asm volatile("");
  } else {
    store_any(p, v);
  }
}
// Rows of `size` bytes a value that start on lines; no row there, or one of them only, are in line.
inline bool on_lines(const void* p, int64_t ld, int64_t size) {
  return p == nullptr || (reinterpret_cast<uintptr_t>(p) % 128 == 0 && ld * size % 128 == 0);
}

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

// Sums over the G lanes of a row that one wave has (all of them for G <= 64). Neighbours of
// 4 by quads, then halves of 8 and rows of 16 with their mirror images.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  const int b = __builtin_bit_cast(int, v);
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, 0xf, 0xf, false));
}
template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
  v = dpp_add<0x4e>(dpp_add<0xb1>(v));
  if constexpr (G >= 8) v = dpp_add<0x141>(v);
  if constexpr (G >= 16) v = dpp_add<0x140>(v);
  if constexpr (G >= 32) v += __shfl_xor(v, 16);
  if constexpr (G >= 64) v += __shfl_xor(v, 32);
  return v;
}

// Lanes a row (G) and pieces a lane (NV) by the row's pieces: few idle lanes, and few waves
// that wait for each other. GRAD: the kernel also keeps two sums a column and does best with a
// row in as few lanes as its registers allow. us on one MI355X of layer_norm with residual and
// of its gradients: 60,000 x 608 float16 59 in 64 lanes of 2 pieces and 63 in 32 of 3 (60 and 61);
// 50,000 x 2048 bfloat16 134 in 128 of 2, 167 in 64 of 4, 140 in 256 of 1 (198, 143, 176); 57,522 x
// 2432 209 in 64 of 5, 241 in 128 of 3, 285 in 512 of 1 (240, 331, 254); 16384 x 4096 91 in 256 of 2, 97 in
// 512 of 1 (105 and 121); 20,000 x 5120 153 in 256 of 3, 160 in 512 of 2 (177, and 169 in 256 of 4); 32768 x
// 8192 381 in 512 of 2, 393 in 1024 of 1, 411 in 256 of 4 (395, 396, 360). Rows of 16 and 32 values in 4 and 8 lanes: 400,000 x 64
// bfloat16 38, and 54 in 16 lanes. Calls use(Shape), or returns false for rows that are too long.
template <int G, int NV>
struct Shape {
  static constexpr int kG = G, kNV = NV;
};
constexpr int row_threads(int g) { return g > 64 ? g : 256; }  // of a workgroup
template <int V, bool GRAD, class F>  // V: columns of a piece; 1 for rows of less than a piece
bool row_shape(int64_t pieces, F use) {
  if constexpr (V == 1) {
    use(Shape<8, 1>{});
  } else {
    if (pieces <= 4) use(Shape<4, 1>{});
    else if (pieces <= 8) use(Shape<8, 1>{});
    else if (pieces <= 16) use(Shape<16, 1>{});
    else if (pieces <= 32) use(Shape<32, 1>{});
    else if (pieces <= 48) use(Shape<16, 3>{});
    else if (pieces <= 64) use(Shape<64, 1>{});
    else if (pieces <= 96) use(std::conditional_t<GRAD, Shape<32, 3>, Shape<64, 2>>{});
    else if (pieces <= 128) use(Shape<64, 2>{});
    else if (pieces <= 192) use(Shape<64, 3>{});
    else if (pieces <= 256) use(std::conditional_t<GRAD, Shape<64, 4>, Shape<128, 2>>{});
    else if (pieces <= 320) use(Shape<64, 5>{});
    else if (pieces <= 384) use(std::conditional_t<GRAD, Shape<256, 2>, Shape<128, 3>>{});
    else if (pieces <= 512) use(Shape<256, 2>{});
    else if (pieces <= 768) use(Shape<256, 3>{});
    else if (pieces <= 1024) use(std::conditional_t<GRAD, Shape<256, 4>, Shape<512, 2>>{});
    else if (pieces <= 1536) use(std::conditional_t<GRAD, Shape<1024, 2>, Shape<512, 3>>{});
    else if (pieces <= 2048) use(std::conditional_t<GRAD, Shape<1024, 2>, Shape<512, 4>>{});
    else if (pieces <= 3 * 1024) use(Shape<1024, 3>{});
    else {
      if constexpr (!GRAD || V <= 4) {  // (no registers for two sums of 32 columns)
        if (pieces <= 4096) {
          use(Shape<1024, 4>{});
          return true;
        }
      }
      return false;
    }
  }
  return true;
}
template <class T>
inline constexpr int kPiece = 16 / (int)sizeof(T);

inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AGCN_OK : hip_fail(e, what);
}

}  // namespace agcn
