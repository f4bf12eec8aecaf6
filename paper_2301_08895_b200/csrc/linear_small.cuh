// The affine layer where its size makes the tiled products wasteful: few rows, or few outputs.
#pragma once
#include "layerops.cuh"

namespace absb {
namespace small {

using layer::Lanes;
using layer::Pack;

struct Args {
  const void* x; const void* w; const void* bias; const void* res; void* y; void* pre;
  long long ldx, ldw, ldr, ldy, ldp;
  long long rows;
  int K, N, act;
};

// result of one output from its sum over k, in two halves: what is loaded, and what is stored.  (A store may alias a load for all the
// compiler knows; several outputs' loads come first.)
template <typename T> __device__ __forceinline__ void fetch(const Args& a, long long m, int j, float& bias, float& res) {
  bias = a.bias ? ldf((const T*)a.bias, j) : 0.f;
  res = a.res ? ldf((const T*)a.res, m * a.ldr + j) : 0.f;
}
template <typename T, int ACT> __device__ __forceinline__ void finish(const Args& a, long long m, int j, float z, float bias, float res) {
  z += bias;
  if (a.pre) stf((T*)a.pre, m * a.ldp + j, z);
  stf((T*)a.y, m * a.ldy + j, layer::act_value<ACT>(z) + res);
}

// ---- a few rows: a pass over W, whose bytes bound the call (or its latency).  L neighbouring lanes take L VE columns of
// one k, the CTA's 256 / L groups of lanes take every (256 / L)-th k, so that all loads of a short sum are under way at once; the partial
// sums are added over the warp by shuffles and over the warps in shared memory.  Few columns per CTA (32 to 256 bytes of a row of W)
// spread a small W over many SMs: 784 -> 256 runs on 16 of them without splitting the sum over CTAs.
constexpr int NT = 256;

template <typename T, int VE, int M, int ACT>
__global__ void __launch_bounds__(NT) few_rows_kernel(const Args a, int log_l) {
  extern __shared__ __align__(16) float red[];                   // [warp][M][L VE]
  // With more than two rows a stretch of x goes through shared memory, k by k: the loads of x would be half of all instructions.
  constexpr bool STAGED = M > 2;
  constexpr int KC = STAGED ? 1024 : 1;
  __shared__ __align__(16) float xs[STAGED ? KC * M : 1];
  const int L = 1 << log_l, G = NT >> log_l, cols = L * VE;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int l = threadIdx.x & (L - 1), g = threadIdx.x >> log_l;
  const int j0 = blockIdx.x * (L * VE), j = j0 + l * VE;
  grid_dependency_sync();
  Lanes<VE> acc[M];
#pragma unroll
  for (int m = 0; m < M; ++m) acc[m].fill(0.f);
  const T* w = (const T*)a.w + (long long)g * a.ldw + j;
  const long long step = G * a.ldw;
  constexpr int U = M <= 2 ? 8 : 4;
  auto multiply = [&](const Pack<T, VE>& q, const float (&xv)[M]) {
    float f[VE];
    q.get(f);
    Lanes<VE> wl;
    wl.set(f);
#pragma unroll
    for (int m = 0; m < M; ++m) {
      Lanes<VE> xl;
      xl.fill(xv[m]);
      acc[m] = fma(xl, wl, acc[m]);
    }
  };
  if constexpr (!STAGED) {
    const T* x = (const T*)a.x + g;
    if (j < a.N)
      for (int k = g; k < a.K; k += U * G, w += U * step, x += U * G) {
        Pack<T, VE> q[U];
        float xv[U][M];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k + u * G < a.K) {
            q[u].load(w + u * step);
#pragma unroll
            for (int m = 0; m < M; ++m) xv[u][m] = m < a.rows ? ldf(x, m * a.ldx + u * G) : 0.f;
          }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k + u * G < a.K) multiply(q[u], xv[u]);
      }
  } else {
    for (int k0 = 0; k0 < a.K; k0 += KC) {
      const int n = min(KC, a.K - k0);
      if (k0 > 0) __syncthreads();
#pragma unroll
      for (int m = 0; m < M; ++m)
        for (int k = threadIdx.x; k < n; k += NT) xs[k * M + m] = m < a.rows ? ldf((const T*)a.x, m * a.ldx + k0 + k) : 0.f;
      __syncthreads();
      if (j < a.N)
        for (int k = g; k < n; k += U * G) {
          Pack<T, VE> q[U];
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (k + u * G < n) q[u].load(w + (long long)(k0 + k - g + u * G) * a.ldw);
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (k + u * G < n) {
              float xv[M];
#pragma unroll
              for (int m = 0; m < M; ++m) xv[m] = xs[(k + u * G) * M + m];
              multiply(q[u], xv);
            }
        }
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m) {
    float v[VE];
    acc[m].get(v);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      for (int o = 16; o >= L; o >>= 1) v[e] += __shfl_xor_sync(0xffffffffu, v[e], o);
      if (lane < L) red[(warp * M + m) * cols + l * VE + e] = v[e];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < M * cols; i += NT) {
    const int m = i / cols, c = i - m * cols;
    if (m < a.rows && j0 + c < a.N) {
      float z = 0.f, bias, res;
      fetch<T>(a, m, j0 + c, bias, res);
#pragma unroll
      for (int q = 0; q < NT / 32; ++q) z += red[(q * M + m) * cols + c];
      finish<T, ACT>(a, m, j0 + c, z, bias, res);
    }
  }
}

// ---- at most 16 outputs of at most 512 inputs, bf16, many rows: a pass over x.  A warp takes 16 rows on mma.sync.m16n8k16 (the products are a few per cent of
// the time that the rows need from HBM; tcgen05's tile of 128 rows x 64 columns per CTA spends it on operands of W and on an
// epilogue of 54 columns that do not exist: 60000 x 256 -> 10 took 16 us).  A lane loads 16 bytes = eight neighbouring k of a row; as the order
// of the sum is free, those eight serve as the eight k that the lane holds of two products, and W's operands, which lie in shared
// memory as each lane needs them, follow that order.
constexpr int WARPS = 8, MAX_N = 16;

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NTILES: n8 tiles; blocks of 32 k are padded with zeros
template <int NTILES, int ACT>
__global__ void __launch_bounds__(WARPS * 32) few_outputs_kernel(const Args a, int n_blocks, int groups) {
  extern __shared__ __align__(16) uint8_t dyn[];
  uint4* wf = reinterpret_cast<uint4*>(dyn);                     // [block][n8 tile][lane]: operands of the block's two products
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r = lane >> 2, q = lane & 3;                         // row (and row + 8) of A, column r of B; eight k: 8 q ...
  float* stage = reinterpret_cast<float*>(wf + n_blocks * NTILES * 32) + warp * 16 * (NTILES * 8 + 1);
  grid_dependency_sync();
  for (int i = threadIdx.x; i < n_blocks * NTILES * 32; i += WARPS * 32) {
    const int ln = i & 31, t = i >> 5, nt = t % NTILES, blk = t / NTILES;
    const int n = nt * 8 + (ln >> 2), k0 = blk * 32 + 8 * (ln & 3);
    uint16_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = n < a.N && k0 + e < a.K ? __bfloat16_as_ushort(((const __nv_bfloat16*)a.w)[(long long)(k0 + e) * a.ldw + n]) : (uint16_t)0;
    wf[i] = make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16);
  }
  __syncthreads();
  for (int g = blockIdx.x * WARPS + warp; g < groups; g += gridDim.x * WARPS) {
    const long long m0 = 16ll * g;
    const __nv_bfloat16* x0 = (const __nv_bfloat16*)a.x + (m0 + r) * a.ldx + 8 * q;
    const bool in0 = m0 + r < a.rows, in1 = m0 + r + 8 < a.rows;
    float c[NTILES][4];
#pragma unroll
    for (int t = 0; t < NTILES; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) c[t][e] = 0.f;
    constexpr int U = 4;                                         // (eight take registers from other CTAs and are no faster)
    for (int b = 0; b < n_blocks; b += U) {
      uint4 p0[U], p1[U];
      const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = b + u < n_blocks && 32 * (b + u) + 8 * q < a.K;
        p0[u] = in && in0 ? __ldg(reinterpret_cast<const uint4*>(x0 + 32 * (b + u))) : zero;
        p1[u] = in && in1 ? __ldg(reinterpret_cast<const uint4*>(x0 + 32 * (b + u) + 8 * a.ldx)) : zero;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (b + u < n_blocks) {
#pragma unroll
          for (int t = 0; t < NTILES; ++t) {
            const uint4 w = wf[((b + u) * NTILES + t) * 32 + lane];
            mma16816(c[t], p0[u].x, p1[u].x, p0[u].y, p1[u].y, w.x, w.y);
            mma16816(c[t], p0[u].z, p1[u].z, p0[u].w, p1[u].w, w.z, w.w);
          }
        }
    }
    // through shared memory, so that a row's results leave together
    constexpr int P = NTILES * 8 + 1;
#pragma unroll
    for (int t = 0; t < NTILES; ++t) {
      stage[r * P + 8 * t + 2 * q] = c[t][0];
      stage[r * P + 8 * t + 2 * q + 1] = c[t][1];
      stage[(r + 8) * P + 8 * t + 2 * q] = c[t][2];
      stage[(r + 8) * P + 8 * t + 2 * q + 1] = c[t][3];
    }
    __syncwarp();
    const int n_rows = (int)min(16ll, a.rows - m0);
    int m = lane / a.N, j = lane - m * a.N;                      // element lane, lane + 32, ... of the group's results
    const int dm = 32 / a.N, dj = 32 - dm * a.N;
    while (m < n_rows) {
      float bias, res;
      fetch<__nv_bfloat16>(a, m0 + m, j, bias, res);
      finish<__nv_bfloat16, ACT>(a, m0 + m, j, stage[m * P + j], bias, res);
      m += dm;
      j += dj;
      if (j >= a.N) { j -= a.N; ++m; }
    }
    __syncwarp();
  }
}

}  // namespace small
}  // namespace absb
