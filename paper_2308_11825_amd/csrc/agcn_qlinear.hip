// Products of matrices held in 8 bits (agcn_quant.hip's form):
//   Y = act(A W^T),  Y[m][n] = sum over blocks b of 128 k of
//       s_a[m][b] s_w[n / 128][b] sum over k in b of a[m][k] w[n][k],
// with one W, or with a W for each group of rows (agcn_grouped_linear).
//
// The matrix instruction for 8-bit floats (16 x 16 x 128, one block of 128 k at
// a time) takes both scales as they are held and adds to fp32 accumulators. Of
// eight neighbouring products it cuts off what lies more than 13 bits below the largest,
// and adds those sums with fp32's bits. So an element is off by at most 7 * 2^-13 of the
// largest of each eight, which is under a quarter of bfloat16's rounding (2^-8) where
// nothing cancels, and 1.4e-5 in the 2-norm for normal values, a hundredth of that rounding
// (1.7e-3): bfloat16 outputs are computed with it. float16 rounds by 2^-11, less than
// that bound. For it and for float32 the values times their scales are turned into bf16,
// which holds them exactly, and multiplied on the bf16 matrix cores: 8e-8 at K = 4096, for twice
// the time where the matrix cores bound it (4096 x 4096 -> 4096 58 us and 119, 16384 x 8192 -> 8192
// 858 and 1735) and little where memory does (1 x 4096 -> 4096 5.4 and 5.9).
//
// W's rows are the instruction's rows and A's its columns: a lane then holds
// four neighbouring outputs of one row of Y, and the scale of one row of A.
#include <algorithm>
#include <type_traits>

#include "agcn_quant.hpp"
#include "agcn_row_tiles.hpp"

namespace agcn {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef v4f v4f_any __attribute__((aligned(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

struct LinearArgs {
  int64_t n;  // rows of A and Y
  int32_t fin, fout;
  const uint8_t* A;
  int64_t lda;
  const uint8_t* SA;
  int64_t ldsa;
  const uint8_t* W;  // fout x fin
  int64_t ldw, group_w;
  const uint8_t* SW;
  int64_t ldsw, group_sw;
  const int32_t* offsets;  // groups + 1, or NULL
  int32_t groups;
  void* Y;
  int64_t ldy;
  int32_t act;
};

// `valid` of 16 bytes, zeros in the others' place.
__device__ __forceinline__ v4i load16(const uint8_t* p, int valid) {
  if (valid >= 16) return load_any<v4i>(p);
  v4i v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < valid) v[i / 4] |= (int)((uint32_t)p[i] << (8 * (i % 4)));
  return v;
}

__device__ __forceinline__ v8i join(v4i a, v4i b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Eight of a lane's 32 values (words 2 j and 2 j + 1) times their scale as bf16, which
// holds them exactly down to 2^-133 (its last subnormal; only values below 2^-129 with
// one of the three least scales have bits there). The conversion takes a scale as a
// float's exponent, code 0 as 2^-127 and 255 as NaN.
__device__ __forceinline__ v8b to_bf16(v8i v, int j, uint32_t code) {
  const float scale = __builtin_bit_cast(float, code << 23);
  v8b r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * j + h], scale, false);
    const v2b b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * j + h], scale, true);
    r[4 * h] = a[0];
    r[4 * h + 1] = a[1];
    r[4 * h + 2] = b[0];
    r[4 * h + 3] = b[1];
  }
  return r;
}

// acc[j][t] += scaled w[j] a[t] for one block of 128 k. `w` and `a` give the 32 values
// that a lane holds of row lane % 16; which 32 does not matter as long as both
// agree. EXACT: on the bf16 matrix cores.
template <bool EXACT, int NT, int MT, class GetW, class GetA>
__device__ __forceinline__ void block_products(v4f (&acc)[NT][MT], GetW w, GetA a, uint32_t sw,
                                               const uint32_t (&sa)[MT]) {
  if constexpr (EXACT) {
    v8b ab[MT][4];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const v8i av = a(t);
#pragma unroll
      for (int i = 0; i < 4; ++i) ab[t][i] = to_bf16(av, i, sa[t]);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const v8i wv = w(j);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const v8b wb = to_bf16(wv, i, sw);
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, ab[t][i], acc[j][t], 0, 0, 0);
      }
    }
  } else {
    v8i av[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) av[t] = a(t);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const v8i wv = w(j);
#pragma unroll
      for (int t = 0; t < MT; ++t)
        acc[j][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av[t], acc[j][t], 0, 0, 0,
                                                                     (int)sw, 0, (int)sa[t]);
    }
  }
}

// --- few rows, any alignment: straight from memory ---------------------------------------

// One workgroup: 16 outputs by MT * 16 rows. Its NW waves take the blocks of k in turn, U
// at a time so that their loads are on their way together; their sums are added in
// the waves' order.
template <int MT, int NW, int U, bool EXACT, class TY, bool GROUPED>
__global__ __launch_bounds__(64 * NW) void k_qlinear_thin(LinearArgs p) {
  constexpr int BM = MT * 16;
  __shared__ float part[NW][BM][20];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, g = lane / 16;
  const int n0 = blockIdx.x * 16;
  const Rows rows = few_rows<BM, GROUPED>(p);
  if (rows.count <= 0) return;
  v4f acc[1][MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[0][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  if (rows.group >= 0) {
    // Rows past the last are read as the last; their results are not written.
    const uint8_t* w =
        p.W + rows.group * p.group_w + (int64_t)min(n0 + r, p.fout - 1) * p.ldw + g * 32;
    const uint8_t* sw = p.SW + rows.group * p.group_sw + (int64_t)(n0 / kQBlock) * p.ldsw;
    const uint8_t *a[MT], *sa[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int64_t m = rows.row + min(t * 16 + r, rows.count - 1);
      a[t] = p.A + m * p.lda + g * 32;
      sa[t] = p.SA + m * p.ldsa;
    }
    struct Block {
      v8i w, a[MT];
      uint32_t sw, sa[MT];
    };
    auto load = [&](Block& v, int b, int valid) {
      const int64_t k = (int64_t)b * kQBlock;
      v.w = join(load16(w + k, valid), load16(w + k + 16, valid - 16));
      v.sw = sw[b];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        v.a[t] = join(load16(a[t] + k, valid), load16(a[t] + k + 16, valid - 16));
        v.sa[t] = sa[t][b];
      }
    };
    auto multiply = [&](const Block& v) {
      block_products<EXACT>(acc, [&](int) { return v.w; }, [&](int t) { return v.a[t]; }, v.sw, v.sa);
    };
    const int whole = p.fin / kQBlock, left = p.fin % kQBlock;
    int b = wave;
    for (; b + (U - 1) * NW < whole; b += U * NW) {
      Block v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) load(v[u], b + u * NW, 32);
#pragma unroll
      for (int u = 0; u < U; ++u) multiply(v[u]);
    }
    for (; b < whole; b += NW) {
      Block v;
      load(v, b, 32);
      multiply(v);
    }
    if (left != 0 && b == whole) {
      Block v;
      load(v, b, left - g * 32);
      multiply(v);
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) *reinterpret_cast<v4f*>(&part[wave][t * 16 + r][g * 4]) = acc[0][t];
  __syncthreads();
  TY* y = static_cast<TY*>(p.Y) + rows.row * p.ldy + n0;
  for (int i = threadIdx.x; i < rows.count * 16; i += 64 * NW) {
    const int m = i / 16, n = i % 16;
    float v = part[0][m][n];
#pragma unroll
    for (int k = 1; k < NW; ++k) v += part[k][m][n];
    if (n0 + n < p.fout) y[m * p.ldy + n] = (TY)q_act(v, p.act);
  }
}

// --- tiles through LDS -------------------------------------------------------------

typedef __attribute__((address_space(3))) uint8_t lds_byte;

// A tile of A or W in LDS: rows of one block of 128 k, 128 bytes. Row R's 16-byte
// piece c lies at position c ^ key(R). LDS has 64 banks, two rows, and serves 16 lanes'
// 16 bytes at a time: the 16 rows of a fragment that go together take all 16 places of
// two rows. PERM: the order in which fragments take the rows of W, so that a lane's
// outputs are neighbours: 0 as they are, 16 rows 0-3, 8-11, 16-19, 24-27 and then 4-7, ...
// of 32 for two fragments of 16, 32 rows 0-3, 8-11, 4-7, 12-15, 16-19, ... for one of 32.
template <int PERM>
__device__ __forceinline__ int swizzle_key(int row) {
  return PERM == 16 ? (row >> 1 & 1) | (row >> 2 & 6) : row >> 1 & 7;
}

// Ones in the first `valid` of 16 bytes.
__device__ __forceinline__ v4i bytes_kept(int valid) {
  v4i keep;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int b = valid - 4 * w;
    keep[w] = b <= 0 ? 0 : b >= 4 ? -1 : (1 << (8 * b)) - 1;
  }
  return keep;
}

// The part of a tile that one wave stages: every WAVES-th eight rows, 16 bytes a
// lane. Rows past `count` are zeros (the buffer's end); their results are not written.
template <int ROWS, int WAVES, int PERM>
struct Stage {
  static constexpr int kSteps = ROWS / 8 / WAVES;
  // The lane's piece is the same in all its rows.
  static_assert(ROWS % (8 * WAVES) == 0 && WAVES % 4 == 0, "whole steps of the swizzle's period");
  const uint8_t* base;
  uint32_t bytes;  // to the end of the 4 bytes that hold the last row's last value
  int32_t ld, count, first, piece;

  __device__ __forceinline__ void init(const uint8_t* p, int64_t stride, int rows, int fin, int wave,
                                       int lane) {
    base = p;
    ld = (int32_t)stride;
    count = rows;
    bytes = (uint32_t)(rows - 1) * (uint32_t)ld + (((uint32_t)fin + 3) & ~3u);
    const int row = wave * 8 + lane / 8;
    piece = ((lane % 8) ^ swizzle_key<PERM>(row)) * 16;
    first = row * ld + piece;
  }
  static __device__ __forceinline__ int place(int i, int wave) { return (i * WAVES + wave) * 1024; }

  // Straight into LDS. The whole offset is the lanes', so that the buffer's end bounds it.
  __device__ __forceinline__ void issue(uint8_t* lds, int k, int wave) const {
    const auto res = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          res, (__attribute__((address_space(3))) void*)(lds + place(i, wave)), 16,
          first + (i * WAVES * 8 * ld + k), 0, 0, 0);
  }
  // Zeros in the lane's own bytes past a row's end, `left` bytes into the last block.
  __device__ __forceinline__ void mask(uint8_t* lds, int left, int wave, int lane) const {
    const v4i keep = bytes_kept(left - piece);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      *reinterpret_cast<v4i*>(lds + place(i, wave) + lane * 16) &= keep;
  }
  // Through registers, for rows that do not start on 16 bytes.
  __device__ __forceinline__ void load(v4i (&v)[kSteps], int fin, int k, int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int row = min((i * WAVES + wave) * 8 + lane / 8, count - 1);
      v[i] = load16(base + row * ld + piece + k, fin - k - piece);
    }
  }
  __device__ __forceinline__ void store(uint8_t* lds, const v4i (&v)[kSteps], int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) *reinterpret_cast<v4i*>(lds + place(i, wave) + lane * 16) = v[i];
  }
};

// Half of a tile of 4 H rows for 4 waves: of every 2 H rows H from `h` H on.
template <int H, int PERM>
struct HalfStage {
  static constexpr int kSteps = 2 * H / 32;
  const uint8_t* base;
  uint32_t bytes, first;
  int32_t ld, piece;
  __device__ __forceinline__ void init(const uint8_t* p, int64_t stride, int rows, int fin, int wave,
                                       int lane) {
    base = p;
    ld = (int32_t)stride;
    bytes = (uint32_t)(rows - 1) * (uint32_t)ld + (((uint32_t)fin + 3) & ~3u);
    const int row = wave * 8 + lane / 8;
    piece = ((lane % 8) ^ swizzle_key<PERM>(row)) * 16;
    first = (uint32_t)(row * ld + piece);
  }
  static __device__ __forceinline__ int place(int i, int wave) { return (i * 4 + wave) * 1024; }
  __device__ __forceinline__ void issue(uint8_t* lds, uint32_t k, int h, int i, int wave) const {
    const auto res = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, 0x00020000);
    const int row = i * 32 / H * 2 * H + i * 32 % H + h * H;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        res, (__attribute__((address_space(3))) void*)(lds + place(i, wave)), 16,
        first + ((uint32_t)(row * ld) + k), 0, 0, 0);
  }
  __device__ __forceinline__ void mask(uint8_t* lds, int left, int wave, int lane) const {
    const v4i keep = bytes_kept(left - piece);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) *reinterpret_cast<v4i*>(lds + place(i, wave) + lane * 16) &= keep;
  }
};

// The scales of a wave's MT * TILE rows of A for one block: lane r holds those of
// rows r, TILE + r, ...; 0 past the last row.
template <int TILE>
struct RowScales {
  const uint8_t* base;
  uint32_t bytes;
  int32_t ld, first;
  __device__ __forceinline__ void init(const uint8_t* p, int64_t stride, int rows, int blocks, int row) {
    base = p;
    ld = (int32_t)stride;
    bytes = (uint32_t)(rows - 1) * (uint32_t)ld + (uint32_t)blocks;
    first = row * ld;
  }
  __device__ __forceinline__ uint32_t load(int t, int b) const {
    const auto res = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, 0x00020000);
    return __builtin_amdgcn_raw_buffer_load_b8(res, first + (t * TILE * ld + b), 0, 0);
  }
};

// Writes RUN neighbouring outputs of a row from column n on, of `count` columns. ALL:
// the caller knows that they are all there.
template <bool ALL, int RUN, class TY>
__device__ __forceinline__ void store_run(const float (&v)[RUN], TY* to, int n, int count) {
  struct alignas(sizeof(TY)) Run {
    TY e[RUN];
  } o;
#pragma unroll
  for (int i = 0; i < RUN; ++i) o.e[i] = (TY)v[i];
  if (ALL || n + RUN <= count) {
    store_any(to + n, o);
  } else {
#pragma unroll
    for (int i = 0; i < RUN; ++i)
      if (n + i < count) to[n + i] = o.e[i];
  }
}

// Calls write(all, relu) with both as compile-time constants: whole tiles without
// activation, most of them, then write nothing but their values.
template <class F>
__device__ __forceinline__ void write_tile(bool whole, int32_t act, F write) {
  using Yes = std::true_type;
  using No = std::false_type;
  if (whole && act == 0) write(Yes{}, No{});
  else if (whole) write(Yes{}, Yes{});
  else if (act == 0) write(No{}, No{});
  else write(No{}, Yes{});
}

// BM x BN outputs per workgroup of WM x WN waves, TM x TN a wave, one block of 128 k
// at a time: while the waves multiply one block from LDS, the next is on its way
// into the other half. For outputs too narrow or too few for k_qlinear_ring, where the
// time is memory's or the latency of the loads: 230,000 x 128 -> 41 13.5 us, 3.6 TB/s.
template <int TM, int TN, int WM, int WN, bool EXACT, class TY, bool GROUPED, bool ASYNC>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_qlinear_tile(LinearArgs p, uint32_t tiles_n,
                                                               uint32_t group_m) {
  constexpr int BM = TM * WM, BN = TN * WN, WAVES = WM * WN, MT = TM / 16, NT = TN / 16;
  constexpr int PERM = sizeof(TY) == 2 ? 16 : 0;
  __shared__ __align__(1024) uint8_t lds0[(BM + BN) * kQBlock];
  __shared__ __align__(1024) uint8_t lds1[(BM + BN) * kQBlock];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, g = lane / 16, wm = wave % WM, wn = wave / WM;
  uint32_t tn;
  const Rows rows = tile_rows<BM, GROUPED>(p, tiles_n, group_m, &tn);
  if (rows.count <= 0) return;
  const int n0 = (int)tn * BN, count_n = min(BN, p.fout - n0);
  v4f acc[NT][MT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[j][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  const int blocks = rows.group < 0 ? 0 : (p.fin + kQBlock - 1) / kQBlock;
  if (blocks > 0) {
    Stage<BM, WAVES, 0> sa;
    Stage<BN, WAVES, PERM> sw;
    sa.init(p.A + rows.row * p.lda, p.lda, rows.count, p.fin, wave, lane);
    sw.init(p.W + rows.group * p.group_w + (int64_t)n0 * p.ldw, p.ldw, count_n, p.fin, wave, lane);
    RowScales<16> scale_a;
    scale_a.init(p.SA + rows.row * p.ldsa, p.ldsa, rows.count, blocks, wm * TM + r);
    const uint8_t* scale_w =
        p.SW + rows.group * p.group_sw +
        (int64_t)min((n0 + wn * TN) / kQBlock, (p.fout - 1) / kQBlock) * p.ldsw;
    // Fragments: row r of the tile, pieces g and g + 4.
    const int row_w = PERM ? 8 * (r / 4) + r % 4 : r;
    const int frag_a = (wm * TM + r) * kQBlock + ((g ^ swizzle_key<0>(r)) * 16);
    const int frag_w = BM * kQBlock + (wn * TN + row_w) * kQBlock + ((g ^ swizzle_key<PERM>(row_w)) * 16);

    v4i pre_a[Stage<BM, WAVES, 0>::kSteps], pre_w[Stage<BN, WAVES, PERM>::kSteps];
    uint32_t code_a[MT], next_a[MT], code_w, next_w = 0;
    auto fetch = [&](uint8_t* to, int b) {
#pragma unroll
      for (int t = 0; t < MT; ++t) next_a[t] = scale_a.load(t, b);
      next_w = scale_w[b];
      if constexpr (ASYNC) {
        sa.issue(to, b * kQBlock, wave);
        sw.issue(to + BM * kQBlock, b * kQBlock, wave);
      } else {
        sa.load(pre_a, p.fin, b * kQBlock, wave, lane);
        sw.load(pre_w, p.fin, b * kQBlock, wave, lane);
      }
    };
    auto arrive = [&](uint8_t* to, int b) {
      if constexpr (ASYNC) {
        __builtin_amdgcn_s_waitcnt(0);
        const int left = p.fin - b * kQBlock;
        if (left < kQBlock) {
          sa.mask(to, left, wave, lane);
          sw.mask(to + BM * kQBlock, left, wave, lane);
        }
      } else {
        sa.store(to, pre_a, wave, lane);
        sw.store(to + BM * kQBlock, pre_w, wave, lane);
      }
#pragma unroll
      for (int t = 0; t < MT; ++t) code_a[t] = next_a[t];
      code_w = next_w;
      __syncthreads();
    };
    auto multiply = [&](const uint8_t* lds) {
      auto read = [&](int at) {
        return join(*reinterpret_cast<const v4i*>(lds + at), *reinterpret_cast<const v4i*>(lds + (at ^ 64)));
      };
      block_products<EXACT>(
          acc, [&](int j) { return read(frag_w + (PERM ? j / 2 * 32 + j % 2 * 4 : j * 16) * kQBlock); },
          [&](int t) { return read(frag_a + t * 16 * kQBlock); }, code_w, code_a);
    };
    fetch(lds0, 0);
    arrive(lds0, 0);
    for (int b = 0; b < blocks; b += 2) {
      if (b + 1 < blocks) fetch(lds1, b + 1);
      multiply(lds0);
      if (b + 1 >= blocks) break;
      arrive(lds1, b + 1);
      if (b + 2 < blocks) fetch(lds0, b + 2);
      multiply(lds1);
      if (b + 2 < blocks) arrive(lds0, b + 2);
    }
  }

  TY* y = static_cast<TY*>(p.Y) + rows.row * p.ldy + n0;
  write_tile(rows.count == BM && count_n == BN, p.act, [&](auto all, auto relu) {
    constexpr bool ALL = decltype(all)::value, RELU = decltype(relu)::value;
    constexpr int kRun = PERM ? 8 : 4;  // neighbouring outputs of a lane
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int m = wm * TM + t * 16 + r;
      if (!ALL && m >= rows.count) continue;
#pragma unroll
      for (int j = 0; j < NT; j += kRun / 4) {
        float v[kRun];
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[i] = q_act(acc[j + i / 4][t][i % 4], RELU);
        store_run<ALL>(v, y + m * p.ldy, wn * TN + (PERM ? j / 2 * 32 + 8 * g : j * 16 + 4 * g), count_n);
      }
    }
  });
}

// --- few rows: every wave streams blocks of k of its own ------------------------------

// ROWS rows of a block of 128 k, staged by one wave for itself.
template <int ROWS>
struct WaveStage {
  const uint8_t* base;
  uint32_t bytes, first;
  int32_t ld, piece;
  __device__ __forceinline__ void init(const uint8_t* p, int64_t stride, int rows, int fin, int lane) {
    base = p;
    ld = (int32_t)stride;
    bytes = (uint32_t)(rows - 1) * (uint32_t)ld + (((uint32_t)fin + 3) & ~3u);
    first = (uint32_t)(lane / 8 * ld);
  }
  // Eight rows further the swizzle is another.
  static __device__ __forceinline__ int piece_of(int i, int lane) {
    return ((lane % 8) ^ swizzle_key<0>(i * 8 + lane / 8)) * 16;
  }
  __device__ __forceinline__ void issue(uint8_t* lds, uint32_t k, int lane) const {
    const auto res = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < ROWS / 8; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          res, (__attribute__((address_space(3))) void*)(lds + i * 1024), 16,
          first + ((uint32_t)(i * 8 * ld) + k) + piece_of(i, lane), 0, 0, 0);
  }
  __device__ __forceinline__ void mask(uint8_t* lds, int left, int lane) const {
#pragma unroll
    for (int i = 0; i < ROWS / 8; ++i)
      *reinterpret_cast<v4i*>(lds + i * 1024 + lane * 16) &= bytes_kept(left - piece_of(i, lane));
  }
};

// One workgroup: NT * 16 outputs by MT * 16 rows. Its NW waves take the blocks of k in
// turn, each through S slots of LDS of its own that are filled S - 1 blocks ahead, so no
// wave waits for another before the end, where their sums are added in the waves'
// order. Bound by the loads on their way: through LDS 8 lanes read 128 neighbouring
// bytes, where a fragment read straight into registers takes 16 bytes of 16 rows per 16
// lanes and its time from the address unit (64 x 4096 -> 4096 17.5 us, and 8.5 here).
template <int MT, int NT, int NW, int S, bool EXACT, class TY, bool GROUPED>
__global__ __launch_bounds__(64 * NW) void k_qlinear_stream(LinearArgs p) {
  constexpr int BM = MT * 16, BN = NT * 16, kStage = (BM + BN) * kQBlock;
  constexpr int kLoads = (BM + BN) / 8 + MT + 1;  // of a block: into LDS, and scales
  constexpr int kSums = NW * BM * (BN + 4) * 4;
  static_assert(kQBlock % BN == 0 && kLoads * (S - 1) < 64, "one scale of W, and vmcnt's range");
  __shared__ __align__(1024) uint8_t lds[NW * S * kStage > kSums ? NW * S * kStage : kSums];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, g = lane / 16, n0 = blockIdx.x * BN;
  const Rows rows = few_rows<BM, GROUPED>(p);
  if (rows.count <= 0) return;
  const int blocks = rows.group < 0 ? 0 : (p.fin + kQBlock - 1) / kQBlock;
  const int mine = blocks > wave ? (blocks - wave + NW - 1) / NW : 0;
  v4f acc[NT][MT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[j][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  if (mine > 0) {
    uint8_t* own = lds + wave * S * kStage;
    WaveStage<BN> sw;
    sw.init(p.W + rows.group * p.group_w + (int64_t)n0 * p.ldw, p.ldw, min(BN, p.fout - n0), p.fin, lane);
    const uint8_t* scale_w = p.SW + rows.group * p.group_sw + (int64_t)(n0 / kQBlock) * p.ldsw;
    WaveStage<BM> sa;
    sa.init(p.A + rows.row * p.lda, p.lda, rows.count, p.fin, lane);
    RowScales<16> scale_a;
    scale_a.init(p.SA + rows.row * p.ldsa, p.ldsa, rows.count, blocks, r);
    const int frag = r * kQBlock + ((g ^ swizzle_key<0>(r)) * 16);
    uint32_t code_a[S][MT], code_w[S];
    // The wave's i-th block, into slot u = i % S; past the last one zeros.
    auto fetch = [&](int i, int u) {
      const int b = wave + i * NW;
      const uint32_t k = i < mine ? (uint32_t)(b * kQBlock) : 0x80000000u;
      sw.issue(own + u * kStage, k, lane);
      sa.issue(own + u * kStage + BN * kQBlock, k, lane);
      const int c = min(b, blocks - 1);
#pragma unroll
      for (int t = 0; t < MT; ++t) code_a[u][t] = scale_a.load(t, c);
      code_w[u] = scale_w[c];
    };
#pragma unroll
    for (int u = 0; u < S - 1; ++u) fetch(u, u);
    for (int i0 = 0; i0 < mine; i0 += S) {
#pragma unroll
      for (int u = 0; u < S; ++u) {
        fetch(i0 + u + S - 1, (u + S - 1) % S);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads*(S - 1)) : "memory");
        uint8_t* slot = own + u * kStage;
        const int left = p.fin - (wave + (i0 + u) * NW) * kQBlock;
        if (left < kQBlock) {
          sw.mask(slot, left, lane);
          sa.mask(slot + BN * kQBlock, left, lane);
        }
        auto read = [&](int at) {
          return join(*reinterpret_cast<const v4i*>(slot + at), *reinterpret_cast<const v4i*>(slot + (at ^ 64)));
        };
        block_products<EXACT>(
            acc, [&](int j) { return read(frag + j * 16 * kQBlock); },
            [&](int t) { return read(frag + (BN + t * 16) * kQBlock); }, code_w[u], code_a[u]);
        // The slot is filled again by the next fetch: its reads are over.
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0);  // what was fetched past the last block
  __syncthreads();
  auto part = reinterpret_cast<float(*)[BM][BN + 4]>(lds);
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int t = 0; t < MT; ++t)
      *reinterpret_cast<v4f*>(&part[wave][t * 16 + r][j * 16 + g * 4]) = acc[j][t];
  __syncthreads();
  TY* y = static_cast<TY*>(p.Y) + rows.row * p.ldy + n0;
  for (int i = threadIdx.x; i < rows.count * BN; i += 64 * NW) {
    const int m = i / BN, n = i % BN;
    float v = part[0][m][n];
#pragma unroll
    for (int k = 1; k < NW; ++k) v += part[k][m][n];
    if (n0 + n < p.fout) y[m * p.ldy + n] = (TY)q_act(v, p.act);
  }
}

// 4 H x 4 H outputs per workgroup of 4 waves, 2 H x 2 H a wave. With H = 64 the
// accumulators fill half of the registers and one wave a SIMD is left, so nothing but the
// order of its own instructions hides LDS and memory. A block of 128 k is multiplied in
// four quarters of H x H, and a quarter needs one new half of A or W, which is read
// from LDS during the quarter before:
//   A0 W0 | read W1,   A0 W1 | read A1,   A1 W1 | read A0',   A1 W0 | read W1'
// (' the next block, which starts with the other half of W). So LDS is filled and
// emptied in halves of a block, of A and of W together: five slots (32 KB each, or 16 KB and
// two workgroups a compute unit), one being read and four on their way, which are
// two blocks' time to arrive. EXACT: a half becomes bf16 when it has been read.
// H = 64: 4096 x 4096 -> 4096 58 us, 16384 x 8192 -> 8192 850 us, 2.4 and 2.6 PFLOP/s, where the chip
// lowers its clock to about 2 GHz. H = 32: 16384 x 1024 -> 4096 75 us, 1.8 PFLOP/s, bound by LDS;
// 230,000 x 128 -> 128 17 us, 5.1 TB/s.
template <int H, bool EXACT, class TY, bool GROUPED>
__global__ __launch_bounds__(256, H == 64 ? 1 : 2) void k_qlinear_ring(LinearArgs p, uint32_t tiles_n,
                                                                       uint32_t group_m) {
  constexpr int BM = 4 * H, BN = 4 * H, T = H / 32, kSlots = 5, kPart = 2 * H * kQBlock, kSlot = 2 * kPart;
  constexpr int kLoads = H / 8, kCodes = 2 * T + 1;  // a wave's loads of half a block, and of scales
  __shared__ __align__(1024) uint8_t lds[kSlots * kSlot];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 32, g = lane / 32, wm = wave % 2, wn = wave / 2;
  uint32_t tn;
  const Rows rows = tile_rows<BM, GROUPED>(p, tiles_n, group_m, &tn);
  if (rows.count <= 0) return;
  const int n0 = (int)tn * BN, count_n = min(BN, p.fout - n0);
  v16f acc[2 * T][2 * T];
#pragma unroll
  for (int j = 0; j < 2 * T; ++j)
#pragma unroll
    for (int t = 0; t < 2 * T; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[j][t][i] = 0.0f;

  const int blocks = rows.group < 0 ? 0 : (p.fin + kQBlock - 1) / kQBlock;
  if (blocks > 0) {
    // Two blocks a round; an odd number starts with a round's second, so that the last
    // block, which may be a part of one, always comes second in the last round. (H = 64
    // has no registers for a way into the middle and takes a block of zeros first.)
    constexpr bool kSkip = H < 64;
    const int none = blocks & 1, total = blocks + none, begin = kSkip ? none : 0;
    HalfStage<H, 0> sa;
    HalfStage<H, 32> sw;
    sa.init(p.A + rows.row * p.lda, p.lda, rows.count, p.fin, wave, lane);
    sw.init(p.W + rows.group * p.group_w + (int64_t)n0 * p.ldw, p.ldw, count_n, p.fin, wave, lane);
    RowScales<32> scale_a;
    scale_a.init(p.SA + rows.row * p.ldsa, p.ldsa, rows.count, blocks, wm * 2 * H + r);
    const uint8_t* scale_w =
        p.SW + rows.group * p.group_sw +
        (int64_t)min((n0 + wn * 2 * H) / kQBlock, (p.fout - 1) / kQBlock) * p.ldsw;
    // Fragments: pieces g, g + 2 (the first 64 k), g + 4 and g + 6 of a row.
    const int row_w = r / 16 * 16 + r / 4 % 2 * 8 + r / 8 % 2 * 4 + r % 4;
    const int frag_a = (wm * H + r) * kQBlock + ((g ^ swizzle_key<0>(r)) * 16);
    const int frag_w = kPart + (wn * H + row_w) * kQBlock + ((g ^ swizzle_key<32>(row_w)) * 16);

    uint32_t code_a[2 * T], next_a[2][2 * T], code_w, next_w[2];
    int to = 0, from = 0;  // slots to fill and to read next
    auto advance = [](int& slot) { slot = slot == (kSlots - 1) * kSlot ? 0 : slot + kSlot; };
    // Load l of a wave's for half h of block i: rows H h on of every 2 H of A, and of W the
    // other half in odd blocks. Past the last block nothing is read (zeros arrive).
    auto issue = [&](int i, int h, int l) {
      const uint32_t k = i < total ? (uint32_t)((i - none) * kQBlock) : 0x80000000u;
      if (l < kLoads / 2) sa.issue(lds + to, k, h, l, wave);
      else sw.issue(lds + to + kPart, k, h ^ (i & 1), l - kLoads / 2, wave);
      if (l == kLoads - 1) advance(to);
    };
    auto issue_all = [&](int i, int h) {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) issue(i, h, l);
    };
    // Two blocks ahead: loads arrive in their order, and a block's scales are asked for
    // after the values of the first half of the block after the next.
    auto code = [&](int i, int u, int l) {
      const int b = min(max(i - none, 0), blocks - 1);
      if (l < 2 * T) next_a[u][l] = scale_a.load(l, b);
      else next_w[u] = scale_w[b];
    };
    auto mask = [&](int slot, int left) {
      sa.mask(lds + slot, left, wave, lane);
      sw.mask(lds + slot + kPart, left, wave, lane);
    };
    // The half at `from` is in LDS and the one before it has been read, by all waves.
    // `young` later ones have been asked for and may be on their way.
    auto arrive = [&](int left, auto young) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(young)::value * kLoads) : "memory");
      if (left < kQBlock) mask(from, left);
      // (A fence would wait for every load into LDS.)
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    // Half an operand: [64 k][tile of 32 rows], as read and as multiplied.
    struct Half {
      v8i q[2 * T];
      v8b b[EXACT ? 2 * T : 1][EXACT ? 4 : 1];
    };
    Half a0, a1, w0, w1;
    auto read = [&](Half& v, int at, int c) {
      const int x = at + c % T * 32 * kQBlock, h = c / T * 64;
      v.q[c] = join(*reinterpret_cast<const v4i*>(lds + from + (x ^ h)),
                    *reinterpret_cast<const v4i*>(lds + from + (x ^ (h + 32))));
    };
    auto convert = [&](Half& v, const uint32_t* scale, int step) {
      if constexpr (EXACT) {
#pragma unroll
        for (int c = 0; c < 2 * T; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) v.b[c][i] = to_bf16(v.q[c], i, scale[c % T * step]);
      }
    };
    // A quarter in eight parts, and after each what `between` issues in its shadow.
    auto quarter = [&](const Half& w, const Half& a, int hw, int ha, auto between) {
      constexpr int kProducts = T * T * 2 * (EXACT ? 4 : 1);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
#pragma unroll
        for (int x = k * kProducts / 8; x < (k + 1) * kProducts / 8; ++x) {
          const int j = x / T % T, t = x % T, y = x / (T * T);  // y: the step of k
          v16f& c = acc[hw * T + j][ha * T + t];
          if constexpr (EXACT)
            c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.b[y / 4 * T + j][y % 4], a.b[y / 4 * T + t][y % 4], c,
                                                        0, 0, 0);
          else
            c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w.q[y * T + j], a.q[y * T + t], c, 0, 0, 0,
                                                                (int)code_w, 0, (int)code_a[ha * T + t]);
        }
        between(k);
        if (H == 64) __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    // Block i, its first half of W (number `first`) in wf; the other goes to wo. WHICH: 0 a
    // block in the middle, 1 the one before the last, 2 the last.
    auto step = [&](int i, int first, Half& wf, Half& wo, auto which) {
      constexpr int WHICH = decltype(which)::value;
      const int left = WHICH == 0 ? kQBlock : p.fin - (blocks - 1) * kQBlock;
#pragma unroll
      for (int t = 0; t < 2 * T; ++t) code_a[t] = next_a[first][t];
      code_w = next_w[first];
      // At most one load after a product: the four waves' loads are taken in turn.
      convert(wf, &code_w, 0);
      convert(a0, code_a, 1);
      quarter(wf, a0, first, 0, [&](int k) {
        if (k == 0) arrive(WHICH == 2 ? left : kQBlock, std::integral_constant<int, WHICH == 2 ? 1 : 3>{});
        else if (k <= 2 * T) read(wo, frag_w, k - 1);
        if (WHICH > 0) return;
        if (k >= 1 && k <= kCodes) code(i + 2, first, k - 1);
        if (k >= 6 && k - 6 < kLoads) issue(i + 2, 1, k - 6);
      });
      convert(wo, &code_w, 0);
      quarter(wo, a0, 1 - first, 0, [&](int k) {
        if (k < 2 * T) read(a1, frag_a, k);
        if (k == 4) advance(from);
        if (k >= 2 && k < kLoads && WHICH == 0) issue(i + 2, 1, k);
      });
      convert(a1, code_a + T, 1);
      quarter(wo, a1, 1 - first, 1, [&](int k) {
        if (WHICH == 2) return;
        if (k == 0) arrive(WHICH == 1 ? left : kQBlock, std::integral_constant<int, WHICH == 1 ? 2 : 3>{});
        else if (k <= 2 * T) read(a0, frag_a, k - 1);
        if (k >= 5 && k - 5 < kLoads && WHICH == 0) issue(i + 3, 0, k - 5);
      });
      quarter(wf, a1, first, 1, [&](int k) {
        if (WHICH == 2) return;
        if (k < 2 * T) read(wo, frag_w, k);
        if (k == 4) advance(from);
        if (k >= 3 && k < kLoads && WHICH == 0) issue(i + 3, 0, k);
      });
    };
    if (!kSkip && none) {
      mask(0, 0);
      mask(kSlot, 0);
      to = 2 * kSlot;
    } else {
      issue_all(begin, 0);
      issue_all(begin, 1);
    }
    const bool one = kSkip && blocks == 1;
    if (!one) {
      issue_all(begin + 1, 0);
      issue_all(begin + 1, 1);
    }
#pragma unroll
    for (int l = 0; l < 2 * kCodes; ++l) code(l / kCodes, l / kCodes, l % kCodes);
    if (one) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    arrive(one ? p.fin : kQBlock, std::integral_constant<int, 2>{});
#pragma unroll
    for (int c = 0; c < 2 * T; ++c) {
      read(a0, frag_a, c);
      read(w0, frag_w, c);
      if (kSkip) read(w1, frag_w, c);
    }
    if (!one) issue_all(begin + 2, 0);
    advance(from);
    using Middle = std::integral_constant<int, 0>;
    using Before = std::integral_constant<int, 1>;
    using Last = std::integral_constant<int, 2>;
    int i = 0;
    if (one) {
      step(1, 1, w1, w0, Last{});
    } else {
      if (kSkip && none) {
#pragma unroll
        for (int l = 0; l < kCodes; ++l) code(2, 0, l);
        step(1, 1, w1, w0, Middle{});
        i = 2;
      }
      for (; i + 2 < total; i += 2) {
        step(i, 0, w0, w1, Middle{});
        step(i + 1, 1, w1, w0, Middle{});
      }
      step(i, 0, w0, w1, Before{});
      step(i + 1, 1, w1, w0, Last{});
    }
    __builtin_amdgcn_s_waitcnt(0);  // what was fetched past the last block
  }
  // 32 rows at a time through the wave's own part of LDS, so that 16 lanes write 256
  // neighbouring bytes of Y (a lane's own 16 bytes of 32 rows made 3 TB/s of the
  // whole chip's writes). Rows are 16 bytes apart from a multiple of the banks. float32 is
  // written past L2, which then keeps A's rows for the other column tiles: 230,000 x 602 ->
  // 256 122 us, otherwise 134; 16384 x 1024 -> 4096 149 and 159. 16-bit outputs gain as often as they
  // lose (bfloat16 78 and 83; 82 and 75; float16 96 and 104; 20.4 and 19.0).
  __syncthreads();
  constexpr int kRun = 16 / sizeof(TY), kRow = 2 * H * sizeof(TY) + 16, kLanes = 2 * H / kRun;
  uint8_t* own = lds + wave * 32 * kRow;
  TY* y = static_cast<TY*>(p.Y) + rows.row * p.ldy + n0;
  write_tile(rows.count == BM && count_n == BN, p.act, [&](auto all, auto relu) {
    constexpr bool ALL = decltype(all)::value, RELU = decltype(relu)::value;
    struct alignas(16) Run {
      TY e[kRun];
    };
#pragma unroll
    for (int t = 0; t < 2 * T; ++t) {
#pragma unroll
      for (int j = 0; j < 2 * T; ++j)
#pragma unroll
        for (int c = 0; c < 16; c += kRun) {
          Run v;
#pragma unroll
          for (int i = 0; i < kRun; ++i) v.e[i] = (TY)q_act(acc[j][t][c + i], RELU);
          *reinterpret_cast<Run*>(own + r * kRow + (j * 32 + c / 8 * 16 + 8 * g + c % 8) * sizeof(TY)) = v;
        }
      const int n = lane % kLanes * kRun, left = count_n - wn * 2 * H - n, row0 = wm * 2 * H + t * 32 + lane / kLanes;
      TY* to = y + row0 * p.ldy + wn * 2 * H + n;
      auto each = [&](auto store) {
#pragma unroll
        for (int i = 0; i < kLanes / 2; ++i) {
          const int m = i * (64 / kLanes);
          const Run v = *reinterpret_cast<const Run*>(own + (m + lane / kLanes) * kRow + lane % kLanes * 16);
          if (ALL || row0 + m < rows.count) store(to + m * p.ldy, v);
        }
      };
      if (ALL || left >= kRun) {
        each([](TY* at, const Run& v) {
          if constexpr (sizeof(TY) == 4) __builtin_nontemporal_store(__builtin_bit_cast(v4f, v), (v4f_any*)at);
          else store_any(at, v);
        });
      } else if (left > 0) {
        each([&](TY* at, const Run& v) {
#pragma unroll
          for (int k = 0; k < kRun; ++k)
            if (k < left) at[k] = v.e[k];
        });
      }
    }
  });
}

// Grid of a launch over BM x BN tiles; rows of a band: square patches of about 32
// tiles, what the 32 CUs of an XCD work on at a time.
struct TileGrid {
  int64_t tiles, tiles_n, group_m;
};
template <int BM, int BN, bool GROUPED>
TileGrid tile_grid(const LinearArgs& p) {
  const int64_t tiles_m = GROUPED ? most_slots(p.n, p.groups, BM) : ceil_div64(p.n, BM);
  const int64_t tiles_n = ceil_div64(p.fout, BN);
  return {tiles_m * tiles_n, tiles_n, std::min<int64_t>(tiles_m, 8)};
}

int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AGCN_OK : hip_fail(e, what);
}

template <int TM, int TN, int WM, int WN, bool EXACT, class TY, bool GROUPED, bool ASYNC>
int launch_tile(const LinearArgs& p, hipStream_t st) {
  const TileGrid t = tile_grid<TM * WM, TN * WN, GROUPED>(p);
  if (t.tiles > kMostTiles) return fail(AGCN_ERR_UNSUPPORTED, "matrix too large for one launch");
  k_qlinear_tile<TM, TN, WM, WN, EXACT, TY, GROUPED, ASYNC>
      <<<(unsigned)t.tiles, 64 * WM * WN, 0, st>>>(p, (uint32_t)t.tiles_n, (uint32_t)t.group_m);
  return launched("k_qlinear_tile launch");
}

template <int H, bool EXACT, class TY, bool GROUPED>
int launch_ring(const LinearArgs& p, hipStream_t st) {
  const TileGrid t = tile_grid<4 * H, 4 * H, GROUPED>(p);
  if (t.tiles > kMostTiles) return fail(AGCN_ERR_UNSUPPORTED, "matrix too large for one launch");
  k_qlinear_ring<H, EXACT, TY, GROUPED>
      <<<(unsigned)t.tiles, 256, 0, st>>>(p, (uint32_t)t.tiles_n, (uint32_t)t.group_m);
  return launched("k_qlinear_ring launch");
}

template <int MT, int U, bool EXACT, class TY, bool GROUPED>
int launch_thin(const LinearArgs& p, hipStream_t st) {
  constexpr int NW = 8;
  const dim3 grid((unsigned)ceil_div64(p.fout, 16), (unsigned)few_rows_grid(p.n, p.groups, MT * 16, GROUPED));
  k_qlinear_thin<MT, NW, U, EXACT, TY, GROUPED><<<grid, 64 * NW, 0, st>>>(p);
  return launched("k_qlinear_thin launch");
}

template <int MT, int NT, int NW, int S, bool EXACT, class TY, bool GROUPED>
int launch_stream(const LinearArgs& p, hipStream_t st) {
  const dim3 grid((unsigned)ceil_div64(p.fout, NT * 16),
                  (unsigned)few_rows_grid(p.n, p.groups, MT * 16, GROUPED));
  k_qlinear_stream<MT, NT, NW, S, EXACT, TY, GROUPED><<<grid, 64 * NW, 0, st>>>(p);
  return launched("k_qlinear_stream launch");
}

// Which kernel. Figures are us on one MI355X, bfloat16 outputs; k_qlinear_ring by its H,
// k_qlinear_tile by its outputs. float16 goes as float32: its products are the same.
template <bool EXACT, class TY, bool GROUPED>
int linear_typed(const LinearArgs& p, hipStream_t st) {
  constexpr int64_t kUnits = 256;  // compute units
  // Into LDS directly: rows that start on 16 bytes.
  const bool async = aligned16(p.A) && aligned16(p.W) && p.lda % 16 == 0 && p.ldw % 16 == 0 &&
                     (!GROUPED || p.group_w % 16 == 0);
  // Offsets inside a tile are 32-bit.
  const bool near = std::max({p.lda, p.ldw, p.ldsa}) <= (INT32_MAX - kMostWidth) / 256;
  const int64_t rows = GROUPED ? p.n / std::max(1, p.groups) : p.n;  // of a group, on average
  const bool fits_y = few_rows_grid(p.n, p.groups, 16, GROUPED) <= 65535;  // a grid's y
  // Row and column tiles together, half a row tile more per group.
  auto tiles = [&](int64_t bm, int64_t bn) {
    const int64_t m = GROUPED ? p.n / bm + (p.groups + 1) / 2 : ceil_div64(p.n, bm);
    return m * ceil_div64(p.fout, bn);
  };
  if (!near || !async) {
    if (fits_y && (!near || rows <= 64)) {
      if (rows <= 16) return launch_thin<1, 4, EXACT, TY, GROUPED>(p, st);
      return launch_thin<2, 2, EXACT, TY, GROUPED>(p, st);
    }
    if (!near) return fail(AGCN_ERR_UNSUPPORTED, "row strides over 8 million bytes and over 65535 row tiles");
    if (tiles(64, 64) <= 4 * kUnits) return launch_tile<32, 32, 2, 2, EXACT, TY, GROUPED, false>(p, st);
    return launch_tile<32, 64, 4, 1, EXACT, TY, GROUPED, false>(p, st);
  }
  if constexpr (GROUPED) {
    // Few rows a group: bound by the weights, which are read once per row tile. 512 x 4096
    // -> 2048 over 64 groups 93 with 32 x 32 outputs, 99 with 64 x 64; 2048 rows 151, 117 and
    // 130 in k_qlinear_ring<32>; 4096 rows 236, 159 and 148.
    if (fits_y && rows <= 12) return launch_stream<2, 2, 4, 2, EXACT, TY, true>(p, st);
    if (fits_y && rows < 64) return launch_stream<4, 4, 4, 1, EXACT, TY, true>(p, st);
  } else if (tiles(64, 64) <= kUnits) {
    // Few outputs: the largest tile of which there are not more than compute units, each
    // read by a workgroup that splits k over its waves. 16, 64, 128 and 256 x 4096 -> 4096:
    // 6.6, 11.2, 19.8, 36 with 16 x 32 outputs; 7.2, 8.5, 13.2, 22 with 32 x 32; 8.6, 10.0, 10.9,
    // 18 with 32 x 64; 10.7, 13.7, 13.9, 14.5 with 64 x 64; 2048 x 4096 -> 512 18.1, ring<32> 20.1.
    // A short k has too few blocks to split: 4096 x 256 -> 256 6.8 in 64 x 64 outputs, 4.3 in
    // k_qlinear_tile's; 1024 x 1024 -> 1024 7.1 and 6.2; 1024 x 2048 -> 1024 9.6 and 9.0, float32 11.5 and 11.9.
    if (tiles(16, 32) <= kUnits) return launch_stream<1, 2, 8, 2, EXACT, TY, false>(p, st);
    if (tiles(32, 32) <= kUnits) return launch_stream<2, 2, 4, 2, EXACT, TY, false>(p, st);
    if (tiles(32, 64) <= kUnits) return launch_stream<2, 4, 4, 2, EXACT, TY, false>(p, st);
    if (p.fin < 2048) return launch_tile<32, 32, 2, 2, EXACT, TY, false, true>(p, st);
    return launch_stream<4, 4, 4, 2, EXACT, TY, false>(p, st);
  }
  // A full chip and a long k: half the reads of LDS and cache per product. 4096 x 4096 -> 4096
  // ring<64> 60 and ring<32> 81; 8192 x 2048 -> 2048 36 and 38; 65536 x 1536 -> 512 57 and 66. Short k
  // end before its loads are under way, unless there are few columns and A is most
  // of the reading: 65536 x 512 -> 512 37 and 28; 16384 x 1024 -> 4096 88 and 79; 65536 x 1024 -> 512 46
  // and 41; 230,000 x 602 -> 256 84 and 93, x 1024 100 and 105, x 512 73 and 63. Half a tile per compute
  // unit is too few (2048 x 4096 -> 4096 48 and 43), and half-empty column tiles cost what
  // full ones do (230,000 x 200 -> 200 51 and 40).
  if constexpr (!EXACT) {
    const int64_t large = tiles(256, 256);
    if (rows >= 256 && large >= kUnits && large * 16 <= tiles(128, 128) * 5 &&
        (p.fin >= 1536 || (p.fin > 512 && p.fout <= 512 && large > 3 * kUnits)))
      return launch_ring<64, false, TY, GROUPED>(p, st);
  }
  // Narrow outputs fill narrow tiles: 230,000 x 128 -> 41 13.7 with 64 columns, 22.5 with 128;
  // 230,000 x 256 -> 16 13.6 with 32 columns, 16.8 with 64.
  if (p.fout <= 32 && tiles(128, 32) >= kUnits) return launch_tile<32, 32, 4, 1, EXACT, TY, GROUPED, true>(p, st);
  // Half a tile per compute unit is enough where the loads bound it, and one where the
  // conversions do. ring<32> and the smaller tile: 512 x 4096 -> 4096 21.5 and 23.4
  // (k_qlinear_stream); 1024 x 2048 -> 2048 11.6 and 12.8 (64 x 64); 16384 x 512 -> 512 10.8 and 13.0 (128 x
  // 64); 4096 x 1024 -> 1024 9.2 and 11.3. float32: 512 x 4096 -> 4096 33.4 and 25.6 (stream), 1024 x 2048
  // -> 2048 19.4 and 15.6.
  if (p.fout > 64 && tiles(128, 128) >= (EXACT ? kUnits : kUnits / 2))
    return launch_ring<32, EXACT, TY, GROUPED>(p, st);
  // Two workgroups a compute unit, each wave with blocks of its own.
  if constexpr (!GROUPED)
    if (tiles(64, 64) <= 2 * kUnits && p.fin >= (EXACT ? 2048 : 4096))
      return launch_stream<4, 4, 4, 1, EXACT, TY, false>(p, st);
  // 65536 x 602 -> 64 12.2 in 128 x 64 outputs; 2000 x 512 -> 512 over 8 groups 6.6.
  if (tiles(128, 64) > kUnits) return launch_tile<32, 64, 4, 1, EXACT, TY, GROUPED, true>(p, st);
  return launch_tile<32, 32, 2, 2, EXACT, TY, GROUPED, true>(p, st);
}

template <bool EXACT, class TY>
int linear_pieces(const LinearArgs& p, hipStream_t st) {
  if (p.offsets != nullptr) return linear_typed<EXACT, TY, true>(p, st);
  // A launch's row tiles (at least of 16 rows): longer matrices go in pieces.
  constexpr int64_t kMost = 65535 * 16;
  for (int64_t r = 0; r < p.n; r += kMost) {
    LinearArgs q = p;
    q.n = std::min(kMost, p.n - r);
    q.A += r * p.lda;
    q.SA += r * p.ldsa;
    q.Y = static_cast<TY*>(p.Y) + r * p.ldy;
    if (int rc = linear_typed<EXACT, TY, false>(q, st)) return rc;
  }
  return AGCN_OK;
}

}  // namespace

int run_quantized_linear(int64_t n, int32_t fin, int32_t fout, int32_t groups, const void* A,
                         int64_t lda, const void* SA, int64_t ldsa, const void* W, int64_t ldw,
                         int64_t group_w, const void* SW, int64_t ldsw, int64_t group_sw,
                         const int32_t* offsets, int32_t dtype, void* Y, int64_t ldy, hipStream_t st,
                         int32_t act) {
  if (n == 0 || fout == 0) return AGCN_OK;
  const LinearArgs p{n, fin, fout, static_cast<const uint8_t*>(A), lda,
                     static_cast<const uint8_t*>(SA), ldsa, static_cast<const uint8_t*>(W), ldw,
                     group_w, static_cast<const uint8_t*>(SW), ldsw, group_sw, offsets, groups, Y,
                     ldy, act};
  if (dtype == AGCN_FLOAT) return linear_pieces<true, float>(p, st);
  if (dtype == AGCN_BFLOAT) return linear_pieces<false, bf16_t>(p, st);
  return linear_pieces<true, f16_t>(p, st);
}

}  // namespace agcn
