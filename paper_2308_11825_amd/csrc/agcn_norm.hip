// Layer norm of rows and its gradients.
//
//   h = x + r,  mean = sum h / f,  var = sum (h - mean)^2 / f,  rs = 1 / sqrt(var + eps)
//   y = (h - mean) rs g + b
// and for a gradient dy of y, with xh = (h - mean) rs and d = dy g,
//   dx = rs (d - sum d / f - xh sum(d xh) / f) + dh,  dg = sum over rows of dy xh,
//   db = sum over rows of dy.
//
// Little to do but read and write: a row is read once and held in registers, and memory bounds
// the time of more rows than a chip holds. us on one MI355X: 32768 x 8192 bfloat16 with residual 377
// (5.7 TB/s), 230,000 x 128 float32 76 (6.2); gradients with the residual stream's 362 and 77 (5.9, 6.1),
// 60,000 x 601 float16 without 49 (4.4: its rows share lines); 40,000 columns, past registers, 2.3 to 3. A copy of 2^30 bytes reaches 5.1, one
// that goes past the caches with a workgroup for every 4 KB 6.4.
#include <algorithm>
#include <cfloat>

#include "agcn_rows.hpp"

namespace agcn {

namespace {

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
  const void* b;  // or NULL
  bool p_float;   // g and b are float32, else of the rows' type
  float eps;
  void* Y;
  int64_t ldy;
  float* stats;  // mean and rs of each row, or NULL
  int64_t lds;
};

// (h scale - pivot - shift) rs is the normalised h: the mean is a pivot near it and the
// rest, so that rows far from 0 and rows of one value keep their differences' bits.
struct RowStats {
  float scale, pivot, shift, rs;
  __device__ __forceinline__ float operator()(float h) const {
    return (fmaf(h, scale, -pivot) - shift) * rs;
  }
};

// Values whose squares pass fp32's range are scaled by this; eps is nothing next to them
// unless they are all the same, and then the row is b.
constexpr float kTiny = 0x1p-80f;

// Columns of a row that wave w holds.
template <int G, int NV, int V>
__device__ __forceinline__ int wave_columns(int w, int f) {
  int c = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) c += min(max(f - (v * G + w * 64) * V, 0), 64 * V);
  return c;
}

// rs from the sum of squares s2; false where a sum left fp32's range, or is NaN.
__device__ __forceinline__ bool finish_stats(float s2, float over, float eps, RowStats* to) {
  const float var = (s2 < 0.0f ? 0.0f : s2) * over + eps * to->scale * to->scale;
  to->rs = var == 0.0f ? 0.0f : 1.0f / sqrtf(var);
  return s2 <= FLT_MAX && var <= FLT_MAX;
}

__device__ __forceinline__ float first_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// Mean and variance of h scale over a row: around the wave's own mean, whose rounding is
// put right by the sum of the differences, and the waves' sums then joined. That mean is
// itself the first value and the mean difference to it, so values that are all the same
// have no differences.
template <int G, int NV, int V>
__device__ __forceinline__ bool row_stats(const float (&h)[NV][V], const int (&shared)[NV], int f, float scale,
                                          float eps, float (*part)[4], RowStats* to) {
  constexpr int kWaves = G > 64 ? G / 64 : 1;
  const int own = kWaves > 1 ? wave_columns<G, NV, V>(threadIdx.x / 64, f) : f;
  const float first = (G >= 64 ? first_lane(h[0][0]) : __shfl(h[0][0], 0, G < 64 ? G : 64)) * scale;
  float s = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < V; ++i) s += i >= shared[v] ? fmaf(h[v][i], scale, -first) : 0.0f;
  const float m = first + lanes_sum<G>(s) / (float)max(own, 1);
  float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = i >= shared[v] ? fmaf(h[v][i], scale, -m) : 0.0f;
      s1 += d;
      s2 = fmaf(d, d, s2);
    }
  s1 = lanes_sum<G>(s1);
  s2 = lanes_sum<G>(s2);
  const float over = 1.0f / (float)f;
  to->scale = scale;
  if constexpr (kWaves == 1) {
    to->pivot = m;
    to->shift = s1 * over;
    s2 = fmaf(-s1, to->shift, s2);
  } else {
    if (threadIdx.x % 64 == 0) {
      float* p = part[threadIdx.x / 64];
      p[0] = m;
      p[1] = s1;
      p[2] = s2;
    }
    __syncthreads();
    const int w = threadIdx.x % 16;
    const float count = w < kWaves ? (float)wave_columns<G, NV, V>(w, f) : 0.0f;
    const float* p = part[min(w, kWaves - 1)];
    const float p1 = w < kWaves ? p[1] : 0.0f, p2 = w < kWaves ? p[2] : 0.0f;
    to->pivot = part[0][0];
    float a = count > 0.0f ? p[0] - to->pivot : 0.0f;
    to->shift = sum16(fmaf(count, a, p1)) * over;
    a = count > 0.0f ? a - to->shift : 0.0f;
    s2 = sum16(fmaf(a, fmaf(count, a, 2.0f * p1), p2));
  }
  return finish_stats(s2, over, eps, to);
}

__device__ __forceinline__ void write_stats(float* to, const RowStats& s, float eps) {
  to[0] = (s.pivot + s.shift) / s.scale;
  to[1] = s.rs == 0.0f ? 1.0f / sqrtf(eps) : s.rs * s.scale;
}

// Parameters of V columns from `at` on.
template <class T, int V>
__device__ __forceinline__ void load_params(float (&to)[V], const void* p, int at, bool p_float) {
  if (p_float) {
    const auto v = load_any<Piece<float, V>>(static_cast<const float*>(p) + at);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = v.e[i];
  } else {
    const auto v = load_any<Piece<T, V>>(static_cast<const T*>(p) + at);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = to_float(v.e[i]);
  }
}
template <class T>
__device__ __forceinline__ float load_param(const void* p, int64_t at, bool p_float) {
  return p_float ? static_cast<const float*>(p)[at] : to_float(static_cast<const T*>(p)[at]);
}

// One row per G lanes, NV pieces of V columns a lane (V <= f <= G * NV * V, or V = 1); the
// parameters of its columns stay in registers too.
template <class T, class TP, int G, int NV, int V, bool PAST>
__global__ __launch_bounds__(row_threads(G)) void k_layer_norm(NormArgs a) {
  constexpr int kThreads = row_threads(G), kRows = kThreads / G;
  constexpr bool kKeep = G < 1024 || NV == 1;
  using In = Piece<T, V>;
  using Param = Piece<TP, V>;
  __shared__ float part[4][16][4];
  const int lane = threadIdx.x % G;
  int start[NV], shared[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Column<G, V> c(v, lane, a.f);
    start[v] = c.start;
    shared[v] = c.shared;
  }
  Param g[NV], b[NV];
  auto params = [&](int v) {
    g[v] = load_any<Param>(static_cast<const TP*>(a.g) + start[v]);
    if (a.b != nullptr) b[v] = load_any<Param>(static_cast<const TP*>(a.b) + start[v]);
  };
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int i = 0; i < V; ++i) b[v].e[i] = (TP)0.0f;
    if (kKeep) params(v);
  }
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G; row < a.n;
       row += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
    In raw[NV];
    float h[NV][V];
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = load_row<In, PAST>(x + start[v]);
    if (a.R != nullptr) {
      const T* r = static_cast<const T*>(a.R) + row * a.ldr;
      In add[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) add[v] = load_row<In, PAST>(r + start[v]);
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < V; ++i) h[v][i] = to_float(raw[v].e[i]) + to_float(add[v].e[i]);
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < V; ++i) h[v][i] = to_float(raw[v].e[i]);
    }
    RowStats s;
    if (!row_stats<G, NV, V>(h, shared, a.f, 1.0f, a.eps, part[turn], &s))  // the same for the row's lanes
      row_stats<G, NV, V>(h, shared, a.f, kTiny, a.eps, part[2 + turn], &s);
    if (a.stats != nullptr && lane == 0) write_stats(a.stats + row * a.lds, s, a.eps);
    T* y = static_cast<T*>(a.Y) + row * a.ldy;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if constexpr (!kKeep) {
        if (NV * V >= 32) asm volatile("" ::: "memory");  // (not all pieces' at once: no registers for them)
        params(v);
      }
      if (shared[v] == V) continue;
      // (H after the statistics: where it lies on X or R, all lanes have read their columns.)
      if (a.H != nullptr) {
        In o;
#pragma unroll
        for (int i = 0; i < V; ++i) o.e[i] = (T)h[v][i];
        store_row<PAST>(static_cast<T*>(a.H) + row * a.ldh + start[v], o);
      }
      In o;
#pragma unroll
      for (int i = 0; i < V; ++i) o.e[i] = (T)fmaf(s(h[v][i]), to_float(g[v].e[i]), to_float(b[v].e[i]));
      store_row<PAST>(y + start[v], o);
    }
  }
}

// Rows too long for registers: one workgroup a row, its values read three times.
template <class T>
__global__ __launch_bounds__(1024) void k_layer_norm_long(NormArgs a) {
  constexpr int G = 1024, V = kPiece<T>;
  using In = Piece<T, V>;
  __shared__ float part[2][16];
  auto block_sum = [&](float v, int at) {
    v = lanes_sum<64>(v);
    if (threadIdx.x % 64 == 0) part[at][threadIdx.x / 64] = v;
    __syncthreads();
    return sum16(part[at][threadIdx.x % 16]);
  };
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.X) + row * a.ldx;
    const T* r = static_cast<const T*>(a.R) + row * a.ldr;
    auto each = [&](auto use) {
      for (int64_t c = threadIdx.x * V; c < a.f; c += G * V) {
        const int valid = (int)std::min<int64_t>(V, a.f - c);
        float h[V];
        if (valid == V) {
          const In v = load_any<In>(x + c);
          In add = {};
          if (a.R != nullptr) add = load_any<In>(r + c);
#pragma unroll
          for (int i = 0; i < V; ++i) h[i] = to_float(v.e[i]) + (a.R != nullptr ? to_float(add.e[i]) : 0.0f);
        } else {
          for (int i = 0; i < V; ++i)
            h[i] = i < valid ? to_float(x[c + i]) + (a.R != nullptr ? to_float(r[c + i]) : 0.0f) : 0.0f;
        }
        use(c, valid, h);
      }
    };
    const float over = 1.0f / (float)a.f;
    auto stats = [&](float scale, RowStats* to) {
      const float first = (to_float(x[0]) + (a.R != nullptr ? to_float(r[0]) : 0.0f)) * scale;
      float s = 0.0f;
      each([&](int64_t, int valid, const float(&h)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) s += i < valid ? fmaf(h[i], scale, -first) : 0.0f;
      });
      const float m = first + block_sum(s, 0) * over;
      float s1 = 0.0f, s2 = 0.0f;
      each([&](int64_t, int valid, const float(&h)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = i < valid ? fmaf(h[i], scale, -m) : 0.0f;
          s1 += d;
          s2 = fmaf(d, d, s2);
        }
      });
      s1 = block_sum(s1, 1);
      __syncthreads();
      s2 = block_sum(s2, 0);
      __syncthreads();
      to->scale = scale;
      to->pivot = m;
      to->shift = s1 * over;
      s2 = fmaf(-s1, to->shift, s2);
      return finish_stats(s2, over, a.eps, to);
    };
    RowStats s;
    if (!stats(1.0f, &s)) stats(kTiny, &s);
    if (a.stats != nullptr && threadIdx.x == 0) write_stats(a.stats + row * a.lds, s, a.eps);
    each([&](int64_t c, int valid, const float(&h)[V]) {
      T* to = static_cast<T*>(a.Y) + row * a.ldy + c;
      T* hidden = static_cast<T*>(a.H) + row * a.ldh + c;
      if (valid == V) {
        float g[V], b[V] = {};
        load_params<T>(g, a.g, (int)c, a.p_float);
        if (a.b != nullptr) load_params<T>(b, a.b, (int)c, a.p_float);
        In y, o;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          o.e[i] = (T)h[i];
          y.e[i] = (T)fmaf(s(h[i]), g[i], b[i]);
        }
        if (a.H != nullptr) store_any(hidden, o);
        store_any(to, y);
      } else {
        for (int i = 0; i < valid; ++i) {
          if (a.H != nullptr) hidden[i] = (T)h[i];
          const float b = a.b != nullptr ? load_param<T>(a.b, c + i, a.p_float) : 0.0f;
          to[i] = (T)fmaf(s(h[i]), load_param<T>(a.g, c + i, a.p_float), b);
        }
      }
    });
  }
}

// --- gradients --------------------------------------------------------------------

struct GradArgs {
  int64_t n;
  int32_t f;
  const void* dY;
  int64_t lddy;
  const void* H;
  int64_t ldh;
  const void* dH;  // the residual stream's own gradient, or NULL
  int64_t lddh;
  const float* stats;
  int64_t lds;
  const void* g;
  bool p_float;  // g is float32, else of the rows' type
  void* dX;
  int64_t lddx;
  float* part;  // [workgroups][2][f]: the workgroup's sums of dy xh and of dy
};

// xh of a row; half the difference cannot leave fp32's range.
struct Normalised {
  float half, rs2, rs;
  __device__ __forceinline__ explicit Normalised(const float* stats)
      : half(0.5f * stats[0]), rs2(2.0f * stats[1]), rs(stats[1]) {}
  __device__ __forceinline__ float operator()(float h) const { return fmaf(h, 0.5f, -half) * rs2; }
};

// Rows as in k_layer_norm, each workgroup over every gridDim.x-th; the columns' sums stay in
// registers until the end, and k_layer_norm_sums adds the workgroups' up: 4 to 6 us more, a
// third of the time of 2048 x 4096 (25 us).
template <class T, int G, int NV, int V, bool PAST>
__global__ __launch_bounds__(row_threads(G)) void k_layer_norm_grad(GradArgs a) {
  constexpr int kThreads = row_threads(G), kRows = kThreads / G, kWaves = G > 64 ? G / 64 : 1;
  using In = Piece<T, V>;
  __shared__ float part[2][16][2];
  const int lane = threadIdx.x % G;
  int start[NV], shared[NV];
  float g[NV][V], dg[NV][V], db[NV][V];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Column<G, V> c(v, lane, a.f);
    start[v] = c.start;
    shared[v] = c.shared;
    load_params<T>(g[v], a.g, c.start, a.p_float);
#pragma unroll
    for (int i = 0; i < V; ++i) dg[v][i] = db[v][i] = 0.0f;
  }
  const float over = 1.0f / (float)a.f;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G; row < a.n;
       row += (int64_t)gridDim.x * kRows, turn ^= 1) {
    In dy[NV], h[NV], dh[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      dy[v] = load_row<In, PAST>(static_cast<const T*>(a.dY) + row * a.lddy + start[v]);
      h[v] = load_row<In, PAST>(static_cast<const T*>(a.H) + row * a.ldh + start[v]);
    }
    if (a.dH != nullptr) {
#pragma unroll
      for (int v = 0; v < NV; ++v) dh[v] = load_row<In, PAST>(static_cast<const T*>(a.dH) + row * a.lddh + start[v]);
    }
    const Normalised norm(a.stats + row * a.lds);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float y = to_float(dy[v].e[i]), xh = norm(to_float(h[v].e[i]));
        const float d = i >= shared[v] ? y * g[v][i] : 0.0f;
        s1 += d;
        s2 += i >= shared[v] ? d * xh : 0.0f;  // (0 times an infinity would count)
        dg[v][i] = fmaf(y, xh, dg[v][i]);
        db[v][i] += y;
      }
    s1 = lanes_sum<G>(s1);
    s2 = lanes_sum<G>(s2);
    if constexpr (kWaves > 1) {
      if (threadIdx.x % 64 == 0) {
        part[turn][threadIdx.x / 64][0] = s1;
        part[turn][threadIdx.x / 64][1] = s2;
      }
      __syncthreads();
      const int w = threadIdx.x % 16;
      s1 = sum16(w < kWaves ? part[turn][w % kWaves][0] : 0.0f);
      s2 = sum16(w < kWaves ? part[turn][w % kWaves][1] : 0.0f);
    }
    s1 *= over;
    s2 *= over;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (shared[v] == V) continue;
      In o;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float xh = norm(to_float(h[v].e[i]));
        float d = norm.rs * (fmaf(to_float(dy[v].e[i]), g[v][i], -s1) - xh * s2);
        if (a.dH != nullptr) d += to_float(dh[v].e[i]);
        o.e[i] = (T)d;
      }
      store_row<PAST>(static_cast<T*>(a.dX) + row * a.lddx + start[v], o);
    }
  }
  if (a.part == nullptr) return;
  float* to = a.part + (int64_t)blockIdx.x * 2 * a.f;
  if constexpr (kRows == 1) {
    struct Sums {
      float s[V];
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (shared[v] == 0) {
        store_any(to + start[v], __builtin_bit_cast(Sums, dg[v]));
        store_any(to + a.f + start[v], __builtin_bit_cast(Sums, db[v]));
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i >= shared[v]) {
            to[start[v] + i] = dg[v][i];
            to[a.f + start[v] + i] = db[v][i];
          }
      }
    }
  } else {
    // The rows of a wave, and then the waves in their order.
    constexpr int kWidth = G * NV * V;
    __shared__ float sums[kThreads / 64][kWidth];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float x = k == 0 ? dg[v][i] : db[v][i];
          if constexpr (G < 8) x += __shfl_xor(x, 4);
          if constexpr (G < 16) x += __shfl_xor(x, 8);
          if constexpr (G < 32) x += __shfl_xor(x, 16);
          if constexpr (G < 64) x += __shfl_xor(x, 32);
          if (threadIdx.x % 64 < G) sums[threadIdx.x / 64][(v * V + i) * G + lane] = x;
        }
      __syncthreads();
      for (int c = threadIdx.x; c < kWidth; c += kThreads) {
        const int at = c / G, l = c % G, v = at / V, i = at % V;
        const Column<G, V> col(v, l, a.f);
        if (i < col.shared) continue;
        float x = sums[0][c];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) x += sums[w][c];
        to[k * a.f + col.start + i] = x;
      }
      __syncthreads();
    }
  }
}

// V columns of a row from `at` on, `valid` of them its own.
template <class T, int V>
__device__ __forceinline__ void load_columns(float (&to)[V], const T* row, int at, int valid) {
  if (valid == V) {
    const auto v = load_any<Piece<T, V>>(row + at);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = to_float(v.e[i]);
  } else {
    for (int i = 0; i < V; ++i) to[i] = i < valid ? to_float(row[at + i]) : 0.0f;
  }
}

// Rows too long for registers: dx, one workgroup a row (with the sums below 8000 x 30720 bfloat16 883
// us, 1190 by single elements),
template <class T>
__global__ __launch_bounds__(1024) void k_layer_norm_grad_long(GradArgs a) {
  constexpr int V = kPiece<T>;
  __shared__ float part[2][16];
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* dy = static_cast<const T*>(a.dY) + row * a.lddy;
    const T* h = static_cast<const T*>(a.H) + row * a.ldh;
    const Normalised norm(a.stats + row * a.lds);
    auto each = [&](auto use) {
      for (int c = threadIdx.x * V; c < a.f; c += 1024 * V) {
        const int valid = min(V, a.f - c);
        float y[V], x[V], g[V];
        load_columns(y, dy, c, valid);
        load_columns(x, h, c, valid);
        if (valid == V) {
          load_params<T>(g, a.g, c, a.p_float);
        } else {
          for (int i = 0; i < V; ++i) g[i] = i < valid ? load_param<T>(a.g, c + i, a.p_float) : 0.0f;
        }
        use(c, valid, y, x, g);
      }
    };
    float s1 = 0.0f, s2 = 0.0f;
    each([&](int, int valid, const float(&y)[V], const float(&x)[V], const float(&g)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = y[i] * g[i];
        s1 += i < valid ? d : 0.0f;
        s2 += i < valid ? d * norm(x[i]) : 0.0f;
      }
    });
    s1 = lanes_sum<64>(s1);
    s2 = lanes_sum<64>(s2);
    __syncthreads();  // the row before has been read
    if (threadIdx.x % 64 == 0) {
      part[0][threadIdx.x / 64] = s1;
      part[1][threadIdx.x / 64] = s2;
    }
    __syncthreads();
    const float over = 1.0f / (float)a.f;
    s1 = sum16(part[0][threadIdx.x % 16]) * over;
    s2 = sum16(part[1][threadIdx.x % 16]) * over;
    each([&](int c, int valid, const float(&y)[V], const float(&x)[V], const float(&g)[V]) {
      float dh[V] = {};
      if (a.dH != nullptr) load_columns(dh, static_cast<const T*>(a.dH) + row * a.lddh, c, valid);
      T* to = static_cast<T*>(a.dX) + row * a.lddx + c;
      Piece<T, V> o;
#pragma unroll
      for (int i = 0; i < V; ++i) o.e[i] = (T)(norm.rs * (fmaf(y[i], g[i], -s1) - norm(x[i]) * s2) + dh[i]);
      if (valid == V) {
        store_any(to, o);
      } else {
        for (int i = 0; i < valid; ++i) to[i] = o.e[i];
      }
    });
  }
}
// and the columns' sums, a thread V columns over every gridDim.y-th row.
template <class T>
__global__ __launch_bounds__(256) void k_layer_norm_columns(GradArgs a) {
  constexpr int V = kPiece<T>;
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
  if (c >= a.f) return;
  const int valid = (int)std::min<int64_t>(V, a.f - c);
  float dg[V] = {}, db[V] = {};
#pragma unroll 2
  for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
    const Normalised norm(a.stats + row * a.lds);
    float y[V], x[V];
    load_columns(y, static_cast<const T*>(a.dY) + row * a.lddy, (int)c, valid);
    load_columns(x, static_cast<const T*>(a.H) + row * a.ldh, (int)c, valid);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      dg[i] = fmaf(y[i], norm(x[i]), dg[i]);
      db[i] += y[i];
    }
  }
  float* to = a.part + (int64_t)blockIdx.y * 2 * a.f + c;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < valid) {
      to[i] = dg[i];
      to[a.f + i] = db[i];
    }
}

// Column sums of `parts` rows of 2 f values: 32 columns a workgroup, every 32nd row a
// thread, and the threads' sums in their order.
template <class TP>
__global__ __launch_bounds__(1024) void k_layer_norm_sums(int32_t parts, int32_t f, const float* part, TP* dg,
                                                          TP* db) {
  __shared__ float sums[32][33];
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
  const int at = threadIdx.x / 32;
  float s = 0.0f;
  if (c < 2 * (int64_t)f) {
#pragma unroll 4
    for (int p = at; p < parts; p += 32) s += part[(int64_t)p * 2 * f + c];
  }
  sums[at][threadIdx.x % 32] = s;
  __syncthreads();
  if (at != 0 || c >= 2 * (int64_t)f) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) s += sums[i][threadIdx.x];
  if (c < f) {
    if (dg != nullptr) dg[c] = (TP)s;
  } else if (db != nullptr) {
    db[c - f] = (TP)s;
  }
}

// Workgroups of a launch, at most; rows past them are looped over, with the parameters kept in
// registers. That pays where the parameters are more than half of what a row moves (50,000 x 2048
// bfloat16 without residual 75 us with 2048 workgroups and 103 with one a row; 60,000 x 640 of one wave a
// row 37 with 4096 and 46), where rows share lines, which L2 puts together as long as they are written
// close by (60,000 x 601 float16 69 and 76), and for wide rows of 16 bits with their long chains of
// loads (16384 x 8192 bfloat16 184 with 1024 and 202; 57,522 x 2432 203 with 2048 and 243). Other rows do better with a
// workgroup for every few (50,000 x 1024 float32 130 us, and 145 with 2048; 20,000 x 5120 269 and 299).
constexpr int64_t kMostNormGroups = 1 << 20, kLongRowGroups = 1024;
template <class T, int G, int NV>
int64_t most_groups(const NormArgs& a, bool past) {
  if (G * NV > 256 && sizeof(T) < 4) return G <= 256 ? 2048 : 1024;
  const int64_t row = (int64_t)(a.R != nullptr ? 4 : 2) * a.f * (int64_t)sizeof(T);
  const int64_t params = (int64_t)(a.b != nullptr ? 2 : 1) * a.f * (int64_t)(a.p_float ? sizeof(float) : sizeof(T));
  if (past && row >= 2 * params) return kMostNormGroups;
  return G <= 64 ? 4096 : G <= 256 ? 2048 : 1024;
}

template <class T, class TP, int V, bool PAST>
int norm_pieces(const NormArgs& a, hipStream_t st) {
  const bool fits = row_shape<V, false>(ceil_div64(a.f, V), [&](auto shape) {
    constexpr int G = decltype(shape)::kG, NV = decltype(shape)::kNV, kThreads = row_threads(G);
    const int64_t grid = std::min(most_groups<T, G, NV>(a, PAST), ceil_div64(a.n, kThreads / G));
    k_layer_norm<T, TP, G, NV, V, PAST><<<(unsigned)grid, kThreads, 0, st>>>(a);
  });
  if (!fits) k_layer_norm_long<T><<<(unsigned)std::min(kLongRowGroups, a.n), 1024, 0, st>>>(a);
  return launched("k_layer_norm launch");
}

template <class T, class TP>
int norm_typed(const NormArgs& a, hipStream_t st) {
  if (a.f < kPiece<T>) return norm_pieces<T, TP, 1, false>(a, st);
  const bool past = on_lines(a.X, a.ldx, sizeof(T)) && on_lines(a.R, a.ldr, sizeof(T)) &&
                    on_lines(a.H, a.ldh, sizeof(T)) && on_lines(a.Y, a.ldy, sizeof(T));
  return past ? norm_pieces<T, TP, kPiece<T>, true>(a, st) : norm_pieces<T, TP, kPiece<T>, false>(a, st);
}

// Workgroups of the gradients, whose column sums are kept apart: two or one a compute unit (230,000 x 128
// float32 76 us with 512 workgroups, 92 with 1024, 105 with 256; 8192 x 16384 float16 190 with 256 and 223 with
// 512), and at least two steps of rows each, so that few wide rows leave compute units idle: 64 x 4096
// bfloat16 7.7 us with the sums' launch, 256 rows 9.6 in 128 workgroups, 400 11.6, 1024 20.
int64_t grad_groups(int64_t n, int32_t f, int64_t v) {
  int64_t groups = 0;
  auto set = [&](auto shape) {
    constexpr int G = decltype(shape)::kG, kRows = row_threads(G) / G;
    groups = std::min<int64_t>(G == 1024 ? 256 : 512, ceil_div64(n, 2 * kRows));
  };
  const int64_t pieces = ceil_div64(f, v);
  if (v == 1 ? row_shape<1, true>(pieces, set) : v == 4 ? row_shape<4, true>(pieces, set) : row_shape<8, true>(pieces, set))
    return groups;
  return std::min<int64_t>(n, std::max<int64_t>(1, 1024 * v / ceil_div64(f, 256)));
}

template <class T>
int column_sums(const GradArgs& a, int64_t groups, void* dg, void* db, hipStream_t st) {
  const unsigned grid = (unsigned)ceil_div64(2 * (int64_t)a.f, 32);
  if (a.p_float)
    k_layer_norm_sums<<<grid, 1024, 0, st>>>((int32_t)groups, a.f, a.part, static_cast<float*>(dg),
                                             static_cast<float*>(db));
  else
    k_layer_norm_sums<<<grid, 1024, 0, st>>>((int32_t)groups, a.f, a.part, static_cast<T*>(dg), static_cast<T*>(db));
  return launched("k_layer_norm_sums launch");
}

template <class T, int V, bool PAST>
int grad_pieces(const GradArgs& a, void* dg, void* db, hipStream_t st) {
  const int64_t groups = grad_groups(a.n, a.f, V);
  const bool fits = row_shape<V, true>(ceil_div64(a.f, V), [&](auto shape) {
    constexpr int G = decltype(shape)::kG, NV = decltype(shape)::kNV;
    k_layer_norm_grad<T, G, NV, V, PAST><<<(unsigned)groups, row_threads(G), 0, st>>>(a);
  });
  if (!fits) {
    k_layer_norm_grad_long<T><<<(unsigned)std::min(kLongRowGroups, a.n), 1024, 0, st>>>(a);
    if (int rc = launched("k_layer_norm_grad_long launch")) return rc;
    if (a.part != nullptr)
      k_layer_norm_columns<T><<<dim3((unsigned)ceil_div64(a.f, 256 * kPiece<T>), (unsigned)groups), 256, 0, st>>>(a);
  }
  if (int rc = launched("k_layer_norm_grad launch")) return rc;
  if (a.part == nullptr) return AGCN_OK;
  return column_sums<T>(a, groups, dg, db, st);
}

template <class T>
int grad_typed(const GradArgs& a, void* dg, void* db, hipStream_t st) {
  if (a.f < kPiece<T>) return grad_pieces<T, 1, false>(a, dg, db, st);
  const bool past = on_lines(a.dY, a.lddy, sizeof(T)) && on_lines(a.H, a.ldh, sizeof(T)) &&
                    on_lines(a.dH, a.lddh, sizeof(T)) && on_lines(a.dX, a.lddx, sizeof(T));
  return past ? grad_pieces<T, kPiece<T>, true>(a, dg, db, st) : grad_pieces<T, kPiece<T>, false>(a, dg, db, st);
}

template <class TP>
__global__ __launch_bounds__(256) void k_zeros(int32_t f, TP* a, TP* b) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= f) return;
  if (a != nullptr) a[c] = (TP)0.0f;
  if (b != nullptr) b[c] = (TP)0.0f;
}
template <class TP>
int zeros(int32_t f, void* a, void* b, hipStream_t st) {
  k_zeros<TP><<<(unsigned)ceil_div64(f, 256), 256, 0, st>>>(f, static_cast<TP*>(a), static_cast<TP*>(b));
  return launched("k_zeros launch");
}

}  // namespace

size_t layer_norm_workspace_bytes(int64_t n, int32_t f, int32_t dtype) {
  if (n == 0 || f == 0) return 0;
  int64_t v = dtype == AGCN_FLOAT ? 4 : 8;
  if (f < v) v = 1;
  return (size_t)grad_groups(n, f, v) * 2 * (size_t)f * sizeof(float);
}

int run_layer_norm(int64_t n, int32_t f, int32_t dtype, const void* X, int64_t ldx, const void* R, int64_t ldr,
                   void* H, int64_t ldh, const void* g, const void* b, int32_t p_dtype, float eps, void* Y,
                   int64_t ldy, float* stats, int64_t lds, hipStream_t st) {
  if (n == 0 || f == 0) return AGCN_OK;
  const NormArgs a{n, f, X, ldx, R, ldr, H, ldh, g, b, p_dtype == AGCN_FLOAT, eps, Y, ldy, stats, lds};
  if (dtype == AGCN_FLOAT) return norm_typed<float, float>(a, st);
  if (dtype == AGCN_BFLOAT) return a.p_float ? norm_typed<bf16_t, float>(a, st) : norm_typed<bf16_t, bf16_t>(a, st);
  return a.p_float ? norm_typed<f16_t, float>(a, st) : norm_typed<f16_t, f16_t>(a, st);
}

int run_layer_norm_backward(int64_t n, int32_t f, int32_t dtype, const void* dY, int64_t lddy, const void* H,
                            int64_t ldh, const void* dH, int64_t lddh, const float* stats, int64_t lds,
                            const void* g, int32_t p_dtype, void* dX, int64_t lddx, void* dg, void* db, void* ws,
                            hipStream_t st) {
  if (f == 0) return AGCN_OK;
  const bool sums = dg != nullptr || db != nullptr;
  if (n == 0) {
    if (!sums) return AGCN_OK;
    if (p_dtype == AGCN_FLOAT) return zeros<float>(f, dg, db, st);
    return p_dtype == AGCN_BFLOAT ? zeros<bf16_t>(f, dg, db, st) : zeros<f16_t>(f, dg, db, st);
  }
  const GradArgs a{n, f, dY, lddy, H, ldh, dH, lddh, stats, lds, g, p_dtype == AGCN_FLOAT, dX, lddx,
                   sums ? static_cast<float*>(ws) : nullptr};
  if (dtype == AGCN_FLOAT) return grad_typed<float>(a, dg, db, st);
  return dtype == AGCN_BFLOAT ? grad_typed<bf16_t>(a, dg, db, st) : grad_typed<f16_t>(a, dg, db, st);
}

}  // namespace agcn
