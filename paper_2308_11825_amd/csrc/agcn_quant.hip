// Rows and weights in 8 bits: e4m3 values, and for each block one scale, the
// power of two 2^e with the least e >= -126 that brings the block's largest
// finite value to 448 or less. A block is 128 columns of a row, or 128 x 128 of
// a weight. A power of two costs no precision (e4m3 keeps 4 bits at any
// exponent but the lowest), multiplying by it is exact, and the matrix
// instruction takes it as it is held, one byte (exponent + 127).
//
// k_rms_norm: h = x + r, y = h / sqrt(mean(h^2) + eps) * g, then y's blocks.
// k_quantize_rows: the blocks of x itself. k_quantize_weight: those of W^T.
//
// All have little to do but read and write: each value is read once and held in registers
// from the sum of squares to the 8 bits, and 16 lanes of 8 values make one block, so
// a block's largest value needs four DPP steps and no LDS. Rows of one vector a lane are bound
// by memory. 16-bit rows of several are not yet: the compiler waits for a vector's
// values before it asks for the next one's, as they are converted where they are loaded
// (60,000 x 601 float16 26 us, 4.2 TB/s), and so for the 64 values of k_quantize_weight.
#include <algorithm>

#include "agcn_quant.hpp"
#include "agcn_row_tiles.hpp"
#include "agcn_rows.hpp"

namespace agcn {

namespace {

// `valid` of 8 consecutive values, zeros in the others' place.
template <class T>
__device__ __forceinline__ void load8(const T* p, int valid, float (&v)[8]) {
  struct alignas(sizeof(T)) Raw {
    T e[8];
  };
  if (valid >= 8) {
    const Raw r = load_any<Raw>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float(r.e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? to_float(p[i]) : 0.0f;
  }
}
template <class T>
__device__ __forceinline__ void store8(T* p, int valid, const float (&v)[8]) {
  if (valid >= 8) {
    struct alignas(sizeof(T)) Raw {
      T e[8];
    } r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.e[i] = (T)v[i];
    store_any(p, r);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) p[i] = (T)v[i];
  }
}

// The 8 bits of a lane's 8 values (16 lanes make a block) and the block's scale.
__device__ __forceinline__ void quantize8(const float (&y)[8], int valid, bool first_lane, uint8_t* q,
                                          uint8_t* s) {
  float a = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(y[i]));  // the larger number: NaN does not count
  a = max16(a);
  if (a == __builtin_inff()) {  // the same for the block's 16 lanes
    a = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = fmaxf(a, finite_abs(y[i]));
    a = max16(a);
  }
  const int code = scale_code(a);
  const float inv = inverse_scale(code);
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = pack_e4m3(y[4 * i] * inv, y[4 * i + 1] * inv, y[4 * i + 2] * inv, y[4 * i + 3] * inv);
  if (valid >= 8) {
    store_any(q, uint2{w[0], w[1]});
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) q[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
  if (first_lane && valid > 0) *s = (uint8_t)code;
}

// Squares past fp32's range: a row whose mean of squares + eps is not finite is summed again
// with its values scaled by this, so that only infinities and NaN in it remain.
constexpr float kTiny = 0x1p-80f;

__device__ __forceinline__ float mean_eps(float ss, int32_t f, float eps) { return ss / (float)f + eps; }

// Sum over the G lanes (G <= 64) or the workgroup (G = its threads) of a row.
// `part`: two rows of partial sums, used in turn, so that one barrier a row is
// enough.
template <int G>
__device__ __forceinline__ float row_sum(float v, float (*part)[16], int turn) {
  v = sum16(v);
  if constexpr (G >= 32) v += __shfl_xor(v, 16);
  if constexpr (G >= 64) v += __shfl_xor(v, 32);
  if constexpr (G > 64) {
    if (threadIdx.x % 64 == 0) part[turn][threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < G / 64; ++i) v += part[turn][i];
  }
  return v;
}

struct NormArgs {
  int64_t n;
  int32_t f;
  const void* X;
  int64_t ldx;
  const void* R;  // residual, or NULL
  int64_t ldr;
  void* H;  // x + r, or NULL
  int64_t ldh;
  const void* g;
  float eps;
  uint8_t* Q;
  int64_t ldq;
  uint8_t* S;
  int64_t lds;
};

// One row per G lanes, NV vectors of 8 columns per lane (f <= G * NV * 8), the
// row's values and the weights of its columns in registers.
template <class T, class TG, int G, int NV>
__global__ __launch_bounds__(G > 256 ? G : 256) void k_rms_norm(NormArgs a) {
  constexpr int kThreads = G > 256 ? G : 256, kRows = kThreads / G;
  __shared__ float part[4][16];
  const int lane = threadIdx.x % G;
  float g[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * G + lane) * 8;
    load8(static_cast<const TG*>(a.g) + c, a.f - c, g[v]);
  }
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G; row < a.n;
       row += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
    float h[NV][8];
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * 8;
      load8(x + c, a.f - c, h[v]);
    }
    if (a.R != nullptr) {
      const T* r = static_cast<const T*>(a.R) + row * a.ldr;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * 8;
        float t[8];
        load8(r + c, a.f - c, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] += t[i];
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(h[v][i], h[v][i], ss);
    if (a.H != nullptr) {
      T* to = static_cast<T*>(a.H) + row * a.ldh;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + lane) * 8;
        store8(to + c, a.f - c, h[v]);
      }
    }
    ss = row_sum<G>(ss, part, turn);
    float m = mean_eps(ss, a.f, a.eps), rs = 1.0f / sqrtf(m);
    if (!(m <= FLT_MAX)) {  // the same for every lane of the row
      ss = 0.0f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float t = h[v][i] * kTiny;
          ss = fmaf(t, t, ss);
        }
      m = mean_eps(row_sum<G>(ss, part + 2, turn), a.f, a.eps * kTiny * kTiny);
      rs = kTiny * (1.0f / sqrtf(m));
    }
    uint8_t* q = a.Q + row * a.ldq;
    uint8_t* s = a.S + row * a.lds;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + lane) * 8;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = h[v][i] * rs * g[v][i];
      quantize8(y, a.f - c, lane % 16 == 0, q + c, s + c / kQBlock);
    }
  }
}

// Rows too long for registers: one workgroup a row, its values read twice (H is
// written by the second pass, so that it may lie on X or R).
template <class T, class TG>
__global__ __launch_bounds__(1024) void k_rms_norm_long(NormArgs a) {
  constexpr int G = 1024;
  __shared__ float part[4][16];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x, turn ^= 1) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
    const T* r = static_cast<const T*>(a.R) + row * a.ldr;
    auto load = [&](int c, float(&h)[8]) {
      load8(x + c, a.f - c, h);
      if (a.R != nullptr) {
        float t[8];
        load8(r + c, a.f - c, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += t[i];
      }
    };
    auto squares = [&](float scale) {
      float ss = 0.0f;
      for (int64_t c = threadIdx.x * 8; c < a.f; c += G * 8) {
        float h[8];
        load((int)c, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float t = h[i] * scale;
          ss = fmaf(t, t, ss);
        }
      }
      return ss;
    };
    float m = mean_eps(row_sum<G>(squares(1.0f), part, turn), a.f, a.eps), rs = 1.0f / sqrtf(m);
    if (!(m <= FLT_MAX)) {
      m = mean_eps(row_sum<G>(squares(kTiny), part + 2, turn), a.f, a.eps * kTiny * kTiny);
      rs = kTiny * (1.0f / sqrtf(m));
    }
    uint8_t* q = a.Q + row * a.ldq;
    uint8_t* s = a.S + row * a.lds;
    for (int64_t c0 = 0; c0 < a.f; c0 += G * 8) {  // whole waves: the blocks' DPP steps
      const int64_t c = c0 + threadIdx.x * 8;
      const int valid = (int)std::min<int64_t>(8, a.f - c);
      float h[8] = {}, g[8] = {}, y[8];
      if (valid > 0) {
        load((int)c, h);
        load8(static_cast<const TG*>(a.g) + c, valid, g);
        if (a.H != nullptr) store8(static_cast<T*>(a.H) + row * a.ldh + c, valid, h);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = h[i] * rs * g[i];
      quantize8(y, valid, threadIdx.x % 16 == 0, q + c, s + c / kQBlock);
    }
  }
}

// 16 lanes a block; blocks of all rows in a row.
template <class T>
__global__ __launch_bounds__(256) void k_quantize_rows(uint32_t total, uint32_t blocks, int32_t f,
                                                       const T* X, int64_t ldx, uint8_t* Q,
                                                       int64_t ldq, uint8_t* S, int64_t lds) {
  const uint32_t at = blockIdx.x * 16 + threadIdx.x / 16;
  if (at >= total) return;  // whole blocks of 16 lanes
  const int64_t row = at / blocks;
  const int b = (int)(at % blocks), c = b * kQBlock + (threadIdx.x % 16) * 8;
  float x[8];
  load8(X + row * ldx + c, f - c, x);
  quantize8(x, f - c, threadIdx.x % 16 == 0, Q + row * ldq + c, S + row * lds + b);
}

// One workgroup a 128 x 128 block of W (fin x fout), written as W^T. A thread
// holds 64 consecutive k of one column: its loads run along W's rows with its
// neighbours', and its 64 bytes are one piece of W^T's row.
template <class T>
__global__ __launch_bounds__(256) void k_quantize_weight(int32_t fin, int32_t fout, const T* W,
                                                         int64_t ldw, int64_t group_w, uint8_t* Q,
                                                         int64_t ldq, int64_t group_q, uint8_t* S,
                                                         int64_t lds, int64_t group_s) {
  __shared__ float part[4];
  const int kb = blockIdx.x, nb = blockIdx.y;
  const int64_t e = blockIdx.z;
  const int n = nb * kQBlock + threadIdx.x % 128, k0 = kb * kQBlock + (threadIdx.x / 128) * 64;
  W += e * group_w;
  float w[64], a = 0.0f;
#pragma unroll
  for (int i = 0; i < 64; ++i) {
    w[i] = n < fout && k0 + i < fin ? to_float(W[(int64_t)(k0 + i) * ldw + n]) : 0.0f;
    a = fmaxf(a, finite_abs(w[i]));
  }
  a = max16(a);
  a = fmaxf(a, __shfl_xor(a, 16));
  a = fmaxf(a, __shfl_xor(a, 32));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = a;
  __syncthreads();
  const int code = scale_code(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
  const float inv = inverse_scale(code);
  if (threadIdx.x == 0) S[e * group_s + (int64_t)nb * lds + kb] = (uint8_t)code;
  if (n >= fout) return;
  uint8_t* q = Q + e * group_q + (int64_t)n * ldq + k0;
#pragma unroll
  for (int i = 0; i < 64; i += 4) {
    const uint32_t v = pack_e4m3(w[i] * inv, w[i + 1] * inv, w[i + 2] * inv, w[i + 3] * inv);
    if (k0 + i + 4 <= fin) {
      store_any(q + i, v);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k0 + i + j < fin) q[i + j] = (uint8_t)(v >> (8 * j));
    }
  }
}

// --- 8-bit integers ---------------------------------------------------------------
//
// A row (of X, or of W^T) as integers of -127 to 127 and one float: with a its largest
// |x|, q = x (127 / a) rounded to nearest even, 127 / a and the product rounded to fp32, and
// s = a / 127. A row that holds an infinity or NaN has s = NaN, which its results then are;
// a row of zeros s = 0.

// Bits of |v|: they order as the values do, with infinities and NaN above all numbers.
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_xor(uint32_t v) {
  return std::max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false));
}
template <int ROR>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  return dpp_max_xor<0x120 + ROR>(v);
}
__device__ __forceinline__ uint32_t magnitude16(uint32_t v) {
  return dpp_max<1>(dpp_max<2>(dpp_max<4>(dpp_max<8>(v))));
}

// x as an integer is rint(x up factor); up keeps 127 / a inside fp32's range.
struct IntScale {
  float up, factor, scale;
  __device__ __forceinline__ explicit IntScale(uint32_t top) {
    const float a = __builtin_bit_cast(float, top);
    const bool number = top < 0x7f800000u;
    up = a < 0x1p-100f ? 0x1p100f : 1.0f;
    factor = number && a > 0.0f ? 127.0f / (a * up) : 0.0f;
    scale = number ? a / 127.0f : __builtin_nanf("");
  }
  __device__ __forceinline__ uint32_t operator()(float x) const {
    return (uint32_t)(int)rintf(x * up * factor) & 0xffu;  // (0 for NaN, and for 0 times an infinity)
  }
};

// One row per G lanes, NV pieces of V columns a lane, in registers from the largest value to
// the 8 bits. Bound by memory: 16384 x 8192 bfloat16 70 us, 5.7 TB/s; a row of 4096 2 us.
template <class T, int G, int NV, int V>
__global__ __launch_bounds__(row_threads(G)) void k_quantize_int(int64_t n, int32_t f, const T* X, int64_t ldx,
                                                                  int8_t* Q, int64_t ldq, float* S) {
  constexpr int kThreads = row_threads(G), kRows = kThreads / G, kWaves = G > 64 ? G / 64 : 1;
  __shared__ uint32_t part[2][16];
  const int lane = threadIdx.x % G;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G; row < n; row += (int64_t)gridDim.x * kRows,
               turn ^= 1) {
    Piece<T, V> x[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) x[v] = load_any<Piece<T, V>>(X + row * ldx + Column<G, V>(v, lane, f).start);
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < V; ++i) top = std::max(top, magnitude(to_float(x[v].e[i])));
    if constexpr (G == 4) top = dpp_max_xor<0x4e>(dpp_max_xor<0xb1>(top));
    else if constexpr (G == 8) top = dpp_max_xor<0x141>(dpp_max_xor<0x4e>(dpp_max_xor<0xb1>(top)));
    else top = magnitude16(top);
    if constexpr (G >= 32) top = std::max(top, (uint32_t)__shfl_xor((int)top, 16));
    if constexpr (G >= 64) top = std::max(top, (uint32_t)__shfl_xor((int)top, 32));
    if constexpr (kWaves > 1) {
      if (threadIdx.x % 64 == 0) part[turn][threadIdx.x / 64] = top;
      __syncthreads();
      top = magnitude16(part[turn][threadIdx.x % kWaves % 16]);
    }
    const IntScale s(top);
    if (lane == 0) S[row] = s.scale;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Column<G, V> c(v, lane, f);
      if (c.shared == V) continue;
      uint32_t q[V];
#pragma unroll
      for (int i = 0; i < V; ++i) q[i] = s(to_float(x[v].e[i]));
      int8_t* to = Q + row * ldq + c.start;
      if constexpr (V == 1) {
        *to = (int8_t)q[0];
      } else {
        uint32_t w[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; ++i) w[i] = q[4 * i] | q[4 * i + 1] << 8 | q[4 * i + 2] << 16 | q[4 * i + 3] << 24;
        __builtin_memcpy(to, w, V);
      }
    }
  }
}

// Rows too long for registers, or of no columns: one workgroup a row, its values read twice.
template <class T>
__global__ __launch_bounds__(1024) void k_quantize_int_long(int64_t n, int32_t f, const T* X, int64_t ldx, int8_t* Q,
                                                            int64_t ldq, float* S) {
  __shared__ uint32_t part[16];
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const T* x = X + row * ldx;
    uint32_t top = 0;
    for (int c = threadIdx.x; c < f; c += 1024) top = std::max(top, magnitude(to_float(x[c])));
    top = magnitude16(top);
    top = std::max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = std::max(top, (uint32_t)__shfl_xor((int)top, 32));
    __syncthreads();  // the row before has been read
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = top;
    __syncthreads();
    const IntScale s(magnitude16(part[threadIdx.x % 16]));
    if (threadIdx.x == 0) S[row] = s.scale;
    for (int c = threadIdx.x; c < f; c += 1024) Q[row * ldq + c] = (int8_t)s(to_float(x[c]));
  }
}

// W (fin x fout) as W^T: one workgroup 64 columns of W, read once for their largest values and
// once more to be written, 256 rows at a time through LDS. A thread has 16 rows of a column,
// and then 16 bytes of a row of W^T. Bound by each workgroup's own loads, one a compute unit:
// 8192 x 8192 bfloat16 217 us in 128 workgroups, 0.9 TB/s (a weight is cut to 8 bits once).
template <class T>
__global__ __launch_bounds__(1024) void k_quantize_weight_int(int32_t fin, int32_t fout, const T* W, int64_t ldw,
                                                              int64_t group_w, int8_t* Q, int64_t ldq,
                                                              int64_t group_q, float* S, int64_t group_s) {
  constexpr int kRows = 256, kRow = kRows + 16;
  __shared__ uint32_t part[16][64];
  __shared__ __align__(16) uint8_t tile[64][kRow];  // [column of W][row]
  const int at = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t e = blockIdx.y, n0 = (int64_t)blockIdx.x * 64, n = n0 + at;
  W += e * group_w;
  Q += e * group_q;
  const bool inside = n < fout;
  const T* column = W + (inside ? n : 0);
  uint32_t top = 0;
  if (inside) {
#pragma unroll 16
    for (int k = wave; k < fin; k += 16) top = std::max(top, magnitude(to_float(column[(int64_t)k * ldw])));
  }
  part[wave][at] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) top = std::max(top, part[w][at]);
  const IntScale s(top);
  if (inside && wave == 0) S[e * group_s + n] = s.scale;
  for (int k0 = 0; k0 < fin; k0 += kRows) {
    T x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int k = k0 + wave * 16 + i;
      x[i] = inside && k < fin ? column[(int64_t)k * ldw] : (T)0.0f;
    }
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      q[i] = s(to_float(x[4 * i])) | s(to_float(x[4 * i + 1])) << 8 | s(to_float(x[4 * i + 2])) << 16 |
             s(to_float(x[4 * i + 3])) << 24;
    __builtin_memcpy(&tile[at][wave * 16], q, 16);
    __syncthreads();
    const int c = threadIdx.x / 16, k = threadIdx.x % 16 * 16;
    if (n0 + c < fout) {
      int8_t* to = Q + (n0 + c) * ldq + k0 + k;
      if (k0 + k + 16 <= fin) {
        __builtin_memcpy(to, &tile[c][k], 16);
      } else {
        for (int i = 0; k0 + k + i < fin; ++i) to[i] = (int8_t)tile[c][k + i];
      }
    }
    __syncthreads();
  }
}

// Workgroups resident at once, about: rows past them are looped over, with the
// columns' weights kept in registers. Four short rows a wave have little to keep: 230,000 x
// 128 floats 67.6 us with 16384 workgroups, 73.7 with 2048; 100,000 x 256 bfloat16 34.8 and 30.7.
constexpr int64_t kNormGroups = 2048, kNormGroupsShort = 16384;

template <class T, class TG, int G, int NV>
int launch_norm(const NormArgs& a, hipStream_t st) {
  constexpr int kThreads = G > 256 ? G : 256, kRows = kThreads / G;
  const int64_t grid = std::min<int64_t>(G * NV == 16 ? kNormGroupsShort : kNormGroups, ceil_div64(a.n, kRows));
  k_rms_norm<T, TG, G, NV><<<(unsigned)grid, kThreads, 0, st>>>(a);
  return launched("k_rms_norm launch");
}

// Lanes a row and vectors a lane: the fewest idle lanes, and past 2048 columns one
// vector a lane as long as a workgroup has the lanes (more rows' loads are on their way
// than with four). us at 60,000 rows of float16: 601 columns 26.8 with 32 lanes and 3
// vectors, 34.1 with 64 and 2; 300 columns 17.5 with 16 and 3, 21.0 with 64 and 1; 20,000 x
// 1500 22.7 with 64 and 3, 27.1 with 256 and 1; 32768 x 8192 bfloat16 with residual 342 with 1024
// and 1, 393 with 256 and 4; 16384 x 4096 87 with 512 and 1, 98 with 256 and 2.
template <class T, class TG>
int norm_typed(const NormArgs& a, hipStream_t st) {
  if (a.f <= 128) return launch_norm<T, TG, 16, 1>(a, st);
  if (a.f <= 256) return launch_norm<T, TG, 32, 1>(a, st);
  if (a.f <= 384) return launch_norm<T, TG, 16, 3>(a, st);
  if (a.f <= 512) return launch_norm<T, TG, 64, 1>(a, st);
  if (a.f <= 768) return launch_norm<T, TG, 32, 3>(a, st);
  if (a.f <= 1024) return launch_norm<T, TG, 64, 2>(a, st);
  if (a.f <= 1536) return launch_norm<T, TG, 64, 3>(a, st);
  if (a.f <= 2048) return launch_norm<T, TG, 256, 1>(a, st);
  if (a.f <= 4096) return launch_norm<T, TG, 512, 1>(a, st);
  if (a.f <= 8192) return launch_norm<T, TG, 1024, 1>(a, st);
  if (a.f <= 16384) return launch_norm<T, TG, 1024, 2>(a, st);
  if (a.f <= 32768) return launch_norm<T, TG, 1024, 4>(a, st);
  k_rms_norm_long<T, TG><<<(unsigned)std::min<int64_t>(kNormGroups, a.n), 1024, 0, st>>>(a);
  return launched("k_rms_norm_long launch");
}

template <class T>
int quantize_typed(int64_t n, int32_t f, const void* X, int64_t ldx, uint8_t* Q, int64_t ldq,
                   uint8_t* S, int64_t lds, hipStream_t st) {
  const int64_t blocks = ceil_div64(f, kQBlock), most = most_quantized_rows(blocks);
  for (int64_t r = 0; r < n; r += most) {
    const int64_t rows = std::min(most, n - r), total = rows * blocks;
    k_quantize_rows<T><<<(unsigned)ceil_div64(total, 16), 256, 0, st>>>(
        (uint32_t)total, (uint32_t)blocks, f, static_cast<const T*>(X) + r * ldx, ldx, Q + r * ldq,
        ldq, S + r * lds, lds);
    if (int rc = launched("k_quantize_rows launch")) return rc;
  }
  return AGCN_OK;
}

template <class T, int V>
int quantize_int_pieces(int64_t n, int32_t f, const T* X, int64_t ldx, int8_t* Q, int64_t ldq, float* S,
                        hipStream_t st) {
  const bool fits = f > 0 && row_shape<V, false>(ceil_div64(f, V), [&](auto shape) {
    constexpr int G = decltype(shape)::kG, NV = decltype(shape)::kNV, kThreads = row_threads(G);
    const int64_t grid = std::min<int64_t>(kNormGroupsShort, ceil_div64(n, kThreads / G));
    k_quantize_int<T, G, NV, V><<<(unsigned)grid, kThreads, 0, st>>>(n, f, X, ldx, Q, ldq, S);
  });
  if (!fits)
    k_quantize_int_long<T><<<(unsigned)std::min<int64_t>(kNormGroups, n), 1024, 0, st>>>(n, f, X, ldx, Q, ldq, S);
  return launched("k_quantize_int launch");
}
template <class T>
int quantize_int_typed(int64_t n, int32_t f, const void* X, int64_t ldx, void* Q, int64_t ldq, float* S,
                       hipStream_t st) {
  const T* x = static_cast<const T*>(X);
  int8_t* q = static_cast<int8_t*>(Q);
  return f < kPiece<T> ? quantize_int_pieces<T, 1>(n, f, x, ldx, q, ldq, S, st)
                       : quantize_int_pieces<T, kPiece<T>>(n, f, x, ldx, q, ldq, S, st);
}
template <class T>
int quantize_weight_int_typed(int32_t groups, int32_t fin, int32_t fout, const void* W, int64_t ldw, int64_t group_w,
                              void* Q, int64_t ldq, int64_t group_q, float* S, int64_t group_s, hipStream_t st) {
  constexpr int32_t kMost = 65535;  // a grid's y
  for (int32_t e = 0; e < groups; e += kMost) {
    const dim3 grid((unsigned)ceil_div64(fout, 64), (unsigned)std::min(kMost, groups - e));
    k_quantize_weight_int<T><<<grid, 1024, 0, st>>>(fin, fout, static_cast<const T*>(W) + e * group_w, ldw, group_w,
                                                    static_cast<int8_t*>(Q) + e * group_q, ldq, group_q,
                                                    S + e * group_s, group_s);
    if (int rc = launched("k_quantize_weight_int launch")) return rc;
  }
  return AGCN_OK;
}

}  // namespace

int run_rms_norm(int64_t n, int32_t f, int32_t dtype, const void* X, int64_t ldx, const void* R,
                 int64_t ldr, void* H, int64_t ldh, const void* g, int32_t g_dtype, float eps,
                 void* Q, int64_t ldq, void* S, int64_t lds, hipStream_t st) {
  if (n == 0 || f == 0) return AGCN_OK;
  const NormArgs a{n, f, X, ldx, R, ldr, H, ldh, g, eps, static_cast<uint8_t*>(Q), ldq,
                   static_cast<uint8_t*>(S), lds};
  if (dtype == AGCN_FLOAT) return norm_typed<float, float>(a, st);
  if (dtype == AGCN_BFLOAT)
    return g_dtype == AGCN_FLOAT ? norm_typed<bf16_t, float>(a, st) : norm_typed<bf16_t, bf16_t>(a, st);
  return g_dtype == AGCN_FLOAT ? norm_typed<f16_t, float>(a, st) : norm_typed<f16_t, f16_t>(a, st);
}

int run_quantize_rows(int64_t n, int32_t f, int32_t dtype, const void* X, int64_t ldx, void* Q,
                      int64_t ldq, void* S, int64_t lds, hipStream_t st) {
  if (n == 0 || f == 0) return AGCN_OK;
  uint8_t* q = static_cast<uint8_t*>(Q);
  uint8_t* s = static_cast<uint8_t*>(S);
  if (dtype == AGCN_FLOAT) return quantize_typed<float>(n, f, X, ldx, q, ldq, s, lds, st);
  if (dtype == AGCN_BFLOAT) return quantize_typed<bf16_t>(n, f, X, ldx, q, ldq, s, lds, st);
  return quantize_typed<f16_t>(n, f, X, ldx, q, ldq, s, lds, st);
}

int run_quantize_weight(int32_t groups, int32_t fin, int32_t fout, int32_t dtype, const void* W,
                        int64_t ldw, int64_t group_w, void* Q, int64_t ldq, int64_t group_q, void* S,
                        int64_t lds, int64_t group_s, hipStream_t st) {
  if (groups == 0 || fin == 0 || fout == 0) return AGCN_OK;
  const int64_t kb = ceil_div64(fin, kQBlock), nb = ceil_div64(fout, kQBlock);
  if (nb > 65535) return fail(AGCN_ERR_UNSUPPORTED, "fout is over 65535 blocks of 128");
  constexpr int32_t kMost = 65535;  // a grid's z
  for (int32_t e = 0; e < groups; e += kMost) {
    const dim3 grid((unsigned)kb, (unsigned)nb, (unsigned)std::min(kMost, groups - e));
    uint8_t* q = static_cast<uint8_t*>(Q) + e * group_q;
    uint8_t* s = static_cast<uint8_t*>(S) + e * group_s;
    if (dtype == AGCN_FLOAT)
      k_quantize_weight<<<grid, 256, 0, st>>>(fin, fout, static_cast<const float*>(W) + e * group_w,
                                              ldw, group_w, q, ldq, group_q, s, lds, group_s);
    else if (dtype == AGCN_BFLOAT)
      k_quantize_weight<<<grid, 256, 0, st>>>(fin, fout, static_cast<const bf16_t*>(W) + e * group_w,
                                              ldw, group_w, q, ldq, group_q, s, lds, group_s);
    else
      k_quantize_weight<<<grid, 256, 0, st>>>(fin, fout, static_cast<const f16_t*>(W) + e * group_w,
                                              ldw, group_w, q, ldq, group_q, s, lds, group_s);
    if (int rc = launched("k_quantize_weight launch")) return rc;
  }
  return AGCN_OK;
}

int run_quantize_int(int64_t n, int32_t f, int32_t dtype, const void* X, int64_t ldx, void* Q, int64_t ldq, float* S,
                     hipStream_t st) {
  if (n == 0) return AGCN_OK;
  if (dtype == AGCN_FLOAT) return quantize_int_typed<float>(n, f, X, ldx, Q, ldq, S, st);
  if (dtype == AGCN_BFLOAT) return quantize_int_typed<bf16_t>(n, f, X, ldx, Q, ldq, S, st);
  return quantize_int_typed<f16_t>(n, f, X, ldx, Q, ldq, S, st);
}

int run_quantize_weight_int(int32_t groups, int32_t fin, int32_t fout, int32_t dtype, const void* W, int64_t ldw,
                            int64_t group_w, void* Q, int64_t ldq, int64_t group_q, float* S, int64_t group_s,
                            hipStream_t st) {
  if (groups == 0 || fout == 0) return AGCN_OK;
  if (dtype == AGCN_FLOAT)
    return quantize_weight_int_typed<float>(groups, fin, fout, W, ldw, group_w, Q, ldq, group_q, S, group_s, st);
  if (dtype == AGCN_BFLOAT)
    return quantize_weight_int_typed<bf16_t>(groups, fin, fout, W, ldw, group_w, Q, ldq, group_q, S, group_s, st);
  return quantize_weight_int_typed<f16_t>(groups, fin, fout, W, ldw, group_w, Q, ldq, group_q, S, group_s, st);
}

}  // namespace agcn
