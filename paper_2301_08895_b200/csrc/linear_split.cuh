// fp32 matrices for the tensor cores: every element as the exact sum of three bf16 numbers.
//
// a1 = bf16(a), a2 = bf16(a - a1), a3 = a - a1 - a2: the differences are exact, each piece is at most 2^-8 of the one before and eight bits
// long, so 24 bits fit.  A product of two such numbers is taken as six of the nine products of pieces; the three left out are below
// 2^-23 |a b| together, the error of a single fp32 rounding and a half at the most.  The sum over k runs through the six pairs one after
// the other, the smallest first, so that only the last pass adds to sums of the result's size; its own additions are linear_tc.cuh's, 256 terms
// at a time.  The whole sum is off by less than fused multiply-adds one after the other (4096 terms of both signs: 2.4e-7 of its size for 8.1e-7).
//
// Pieces are those of 2^16 a, so that all 24 bits of any small a, denormal ones included, are multiples of 2^-133, bf16's smallest number; the epilogue
// takes 2^-32 of the sums.  The scaled sums overflow before those of fp32 do: infinities, NaN and elements of 2^L and more, 2 L = 94 - log2 of the terms
// (rounded up), raise their block's flag.  The product is then taken from the fp32 matrices by fused multiply-adds instead: the results are
// fp32's whatever the data, and the cost of such data is time (4096^3: 3.3 ms for 0.71).
//
// 4096^3 with GELU: splitting 67 us (335 MB, 5 TB/s), products 590 us (1.40 PFLOP/s in bf16), epilogue 50; the plain kernel takes 2507.
//
// Layout: pieces [3][rows to a multiple of 64][columns to a multiple of 8], zeros behind the matrix: a block of 64 terms never reaches
// into the next piece, whichever way the sum runs.
#pragma once
#include "layerops.cuh"

namespace absb {
namespace split3 {

constexpr int PAIRS = 6;                                  // (a1 b3) (a3 b1) (a2 b2) (a1 b2) (a2 b1) (a1 b1)
constexpr uint32_t A_PIECE = 0x010120u, B_PIECE = 0x001102u;     // the pairs' pieces, four bits each, first pair lowest

struct Matrix {
  const float* src; long long ld, rows; int cols;
  __nv_bfloat16* dst; uint32_t rows_p; int cols_p;
  int vec;                                                // rows start on 16 bytes
  layer::Divisor per_row;                                 // groups of eight columns
  uint32_t end;                                           // groups of this matrix and the ones before it
};
struct Args { Matrix m[3]; uint32_t n; uint32_t* flags; float limit; };     // limit: 2^L
constexpr float UP = 0x1p16f, DOWN = 0x1p-32f;

// Whether any block of the split raised its flag; all threads of the block take part.
__device__ __forceinline__ bool any_flag(const uint32_t* flags, int n) {
  int bad = 0;
  for (int i = threadIdx.x; i < n; i += blockDim.x) bad |= (int)flags[i];
  return __syncthreads_or(bad) != 0;
}

__global__ void __launch_bounds__(256) split_kernel(const __grid_constant__ Args a) {
  grid_dependency_sync();
  int bad = 0;
  for (uint32_t u = blockIdx.x * 256u + threadIdx.x; u < a.n; u += gridDim.x * 256u) {
    const int w = u < a.m[0].end ? 0 : u < a.m[1].end ? 1 : 2;
    const Matrix& m = a.m[w];
    const uint32_t q = w ? u - a.m[w - 1].end : u, r = m.per_row.div(q);
    const int c = (int)(q - r * m.per_row.d) * 8;
    float v[8];
    if (r < m.rows && m.vec && c + 8 <= m.cols) {
      const float4* s = reinterpret_cast<const float4*>(m.src + (long long)r * m.ld + c);
      const float4 x = s[0], y = s[1];
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    } else {
      const float* s = m.src + (long long)r * m.ld + c;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = r < m.rows && c + e < m.cols ? s[e] : 0.f;
    }
    __nv_bfloat16 p[3][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      bad |= !(fabsf(v[e]) < a.limit);
      const float up = v[e] * UP;
      p[0][e] = __float2bfloat16_rn(up);
      const float rest = up - __bfloat162float(p[0][e]);
      p[1][e] = __float2bfloat16_rn(rest);
      p[2][e] = __float2bfloat16_rn(rest - __bfloat162float(p[1][e]));
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
      *reinterpret_cast<uint4*>(m.dst + ((size_t)k * m.rows_p + r) * m.cols_p + c) = *reinterpret_cast<const uint4*>(p[k]);
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) a.flags[blockIdx.x] = (uint32_t)(bad != 0);
}

}  // namespace split3
}  // namespace absb
