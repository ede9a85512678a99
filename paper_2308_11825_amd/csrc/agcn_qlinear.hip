// Products of matrices held in 8 bits (agcn_quant.hip's form):
//   Y = act(A W^T),  Y[m][n] = sum over blocks b of 128 k of
//       s_a[m][b] s_w[n / 128][b] sum over k in b of a[m][k] w[n][k],
// with one W, or with a W for each group of rows (agcn_grouped_linear).
//
// The matrix instruction for 8-bit floats (16 x 16 x 128, one block of 128 k at
// a time) takes both scales as they are held and adds to fp32 accumulators. It
// adds a few products at a time with about 16 bits below the largest: against 64
// bits its sums are off by 1.4e-5 (2-norm, normal values, K = 128 to 4096; 5e-5 where
// all bit patterns are equally likely), a hundredth of the rounding to
// bfloat16 (1.7e-3) and less than a tenth of that to float16 (2.1e-4): those
// outputs are computed with it. For float32 outputs the values are turned into
// bf16, which holds every e4m3 value, and multiplied on the bf16 matrix cores
// from zero for each block; the block's sum is scaled and added in fp32:
// 8e-8 at K = 4096.
//
// W's rows are the instruction's rows and A's its columns: a lane then holds
// four neighbouring outputs of one row of Y, and the scale of one row of A.
#include <algorithm>

#include "agcn_quant.hpp"

namespace agcn {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
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

// The product of two scales, 2^(code + code - 254), as two factors: it may be out
// of float's range where the scaled sum is not. A code of 255 is NaN.
struct TwoFactors {
  float a, b;
};
__device__ __forceinline__ TwoFactors scale_product(uint32_t sw, uint32_t sa) {
  const int e = (int)(sw + sa) - 254, half = e >> 1;  // -254 to 254
  const float a = __builtin_amdgcn_ldexpf(1.0f, half), b = __builtin_amdgcn_ldexpf(1.0f, e - half);
  return {sw == 255 || sa == 255 ? __builtin_nanf("") : a, b};
}

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

// Eight of a lane's 32 values (words 2 j and 2 j + 1) as bf16, exactly.
__device__ __forceinline__ v8b to_bf16(v8i v, int j) {
  v8b r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * j + h], 1.0f, false);
    const v2b b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * j + h], 1.0f, true);
    r[4 * h] = a[0];
    r[4 * h + 1] = a[1];
    r[4 * h + 2] = b[0];
    r[4 * h + 3] = b[1];
  }
  return r;
}

// acc += s_w s_a (w a) for one block of 128 k. A lane holds 32 k of row
// lane % 16 of both; which 32 does not matter as long as both agree.
template <bool EXACT>
__device__ __forceinline__ void block_product(v4f& acc, v8i w, v8i a, uint32_t sw, uint32_t sa) {
  if constexpr (EXACT) {
    v4f part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(to_bf16(w, j), to_bf16(a, j), part, 0, 0, 0);
    const TwoFactors f = scale_product(sw, sa);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = fmaf(part[i] * f.a, f.b, acc[i]);
  } else {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, acc, 0, 0, 0, (int)sw, 0, (int)sa);
  }
}

// The rows a tile of at most BM rows works on: rows [row, row + count) of group
// `group`, or rows of no group (group -1), which are set to 0.
struct Rows {
  int64_t row;
  int32_t count, group;
};

// Tile `slot` of the rows cut at the groups' offsets. The rows before the first
// offset and after the last are parts of their own without a group, so that the
// parts cover all rows. Offsets are clamped to [0, n] and a part that would be
// negative is empty, so no offsets reach past the matrices. Every lane of a wave
// calls it, with 64 parts looked at per step.
template <int BM>
__device__ __forceinline__ Rows find_rows(const LinearArgs& p, int32_t slot) {
  const int lane = threadIdx.x % 64, n = (int32_t)p.n;
  const int parts = p.groups + 2;
  for (int base = 0; base < parts; base += 64) {
    const int i = base + lane;
    int lo = 0, hi = 0;
    if (i < parts) {
      lo = i == 0 ? 0 : min(max(p.offsets[i - 1], 0), n);
      hi = i == parts - 1 ? n : min(max(p.offsets[i], 0), n);
    }
    const int tiles = hi > lo ? (int)(((int64_t)(hi - lo) + BM - 1) / BM) : 0;
    int end = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int up = __shfl_up(end, d);
      if (lane >= d) end += up;
    }
    const uint64_t hit = __ballot(slot < end);
    if (hit != 0) {
      const int at = __ffsll((unsigned long long)hit) - 1;
      const int from = __shfl(lo, at), to = __shfl(hi, at);
      const int tile = slot - (__shfl(end, at) - __shfl(tiles, at));
      const int row = from + tile * BM, part = base + at;
      return {row, min(BM, to - row), part == 0 || part == parts - 1 ? -1 : part - 1};
    }
    slot -= __shfl(end, 63);
  }
  return {0, 0, -1};
}

// Tiles that any offsets cut n rows into, at most.
int64_t most_slots(int64_t n, int32_t groups, int64_t bm) {
  return std::min<int64_t>(n, n / bm + groups + 2);
}

// One workgroup: 16 outputs by MT * 16 rows, its waves taking the blocks of k in
// turn, each straight from memory; their sums are added in the waves' order.
template <int MT, int NW, bool EXACT, class TY, bool GROUPED>
__global__ __launch_bounds__(64 * NW) void k_qlinear_thin(LinearArgs p) {
  __shared__ float part[NW][MT * 16][16];
  constexpr int BM = MT * 16;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, g = lane / 16;
  const int n0 = blockIdx.x * 16;
  Rows rows;
  if constexpr (GROUPED) {
    rows = find_rows<BM>(p, blockIdx.y);
  } else {
    rows.row = (int64_t)blockIdx.y * BM;
    rows.count = (int32_t)min((int64_t)BM, p.n - rows.row);
    rows.group = 0;
  }
  if (rows.count <= 0) return;
  v4f acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  if (rows.group >= 0) {
    // Rows past the last are read as the last; their results are not written.
    const uint8_t* w = p.W + rows.group * p.group_w + (int64_t)min(n0 + r, p.fout - 1) * p.ldw + g * 32;
    const uint8_t* sw = p.SW + rows.group * p.group_sw + (int64_t)(n0 / kQBlock) * p.ldsw;
    const uint8_t *a[MT], *sa[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int64_t m = rows.row + min(t * 16 + r, rows.count - 1);
      a[t] = p.A + m * p.lda + g * 32;
      sa[t] = p.SA + m * p.ldsa;
    }
    const int whole = p.fin / kQBlock, blocks = (p.fin + kQBlock - 1) / kQBlock;
    for (int b = wave; b < blocks; b += NW) {
      const int valid = b < whole ? 32 : p.fin - b * kQBlock - g * 32;
      const int64_t k = (int64_t)b * kQBlock;
      const v8i wv = join(load16(w + k, valid), load16(w + k + 16, valid - 16));
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const v8i av = join(load16(a[t] + k, valid), load16(a[t] + k + 16, valid - 16));
        block_product<EXACT>(acc[t], wv, av, sw[b], sa[t][b]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) store_any(&part[wave][t * 16 + r][g * 4], acc[t]);
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

template <int MT, int NW, bool EXACT, class TY, bool GROUPED>
int launch_thin(const LinearArgs& p, hipStream_t st) {
  const int64_t y = GROUPED ? most_slots(p.n, p.groups, MT * 16) : ceil_div64(p.n, MT * 16);
  const dim3 grid((unsigned)ceil_div64(p.fout, 16), (unsigned)y);
  k_qlinear_thin<MT, NW, EXACT, TY, GROUPED><<<grid, 64 * NW, 0, st>>>(p);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AGCN_OK : hip_fail(e, "k_qlinear_thin launch");
}

// Row tiles are a grid's y, 65,535 at most: longer matrices go in pieces.
template <bool EXACT, class TY>
int linear_typed(const LinearArgs& p, hipStream_t st) {
  if (p.offsets != nullptr) {
    if (most_slots(p.n, p.groups, 64) > 65535)
      return fail(AGCN_ERR_UNSUPPORTED, "over 65535 tiles of 64 rows");
    return launch_thin<4, 4, EXACT, TY, true>(p, st);
  }
  constexpr int64_t kMost = 65535 * 64;
  for (int64_t r = 0; r < p.n; r += kMost) {
    LinearArgs q = p;
    q.n = std::min(kMost, p.n - r);
    q.A += r * p.lda;
    q.SA += r * p.ldsa;
    q.Y = static_cast<TY*>(p.Y) + r * p.ldy;
    if (int rc = launch_thin<4, 4, EXACT, TY, false>(q, st)) return rc;
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
  if (dtype == AGCN_FLOAT) return linear_typed<true, float>(p, st);
  if (dtype == AGCN_BFLOAT) return linear_typed<false, bf16_t>(p, st);
  return linear_typed<false, f16_t>(p, st);
}

}  // namespace agcn
