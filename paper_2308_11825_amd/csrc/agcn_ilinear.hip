// Products of matrices held in 8-bit integers with a scale per row (agcn_quant.hip's form):
//   Y = act(A W^T),  Y[m][n] = s_a[m] s_w[n] sum over k of a[m][k] w[n][k],
// with one W, or with a W for each group of rows (agcn_grouped_int_linear). The sum is
// exact in 32 bits for fewer than 2^17 values of k (each product is 2^14 at most), and is
// rounded once to fp32 and once by each scale.
//
// The kernels are those of agcn_products.hpp with the matrix cores' integer instructions, as many
// cycles as the e4m3 ones. Where the matrix cores bound them, power does: 16384 x 8192 -> 8192 818 to 900 us, 2.4
// to 2.7 POP/s, with the matrix cores at work in 77 % of the cycles of a clock that falls to 1.6 GHz;
// 32768 x 4096 -> 2048 with one weight 248 us, and 168 for zeros. 1 x 4096 -> 4096 4.9 us, 3.4 TB/s of
// weights: 128 workgroups of 32 columns, which leave half of the compute units without loads.
#include "agcn_products.hpp"

namespace agcn {

int run_int_linear(int64_t n, int32_t fin, int32_t fout, int32_t groups, const void* A, int64_t lda,
                   const float* SA, const void* W, int64_t ldw, int64_t group_w, const float* SW,
                   int64_t group_sw, const int32_t* offsets, int32_t dtype, void* Y, int64_t ldy,
                   hipStream_t st, int32_t act) {
  if (n == 0 || fout == 0) return AGCN_OK;
  const LinearArgs p{n, fin, fout, static_cast<const uint8_t*>(A), lda, nullptr, 0,
                     static_cast<const uint8_t*>(W), ldw, group_w, nullptr, 0, 0, offsets, groups,
                     Y, ldy, act, SA, SW, group_sw, dtype == AGCN_HALF};
  if (dtype == AGCN_FLOAT) return linear_pieces<kInteger, float>(p, st);
  return linear_pieces<kInteger, uint16_t>(p, st);
}

}  // namespace agcn
