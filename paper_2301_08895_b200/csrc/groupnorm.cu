// Group normalisation of channels-last maps with an activation, and its gradients.
#include <atomic>

#include "layerops.cuh"

using namespace absb;
using namespace absb::layer;

// A sample's maps are cut into chunks of whole groups (at least 128 bytes of channels where there are as many), and a cluster of
// Q CTAs takes one chunk of one sample: every CTA copies its share of the positions into shared memory, where it stays, so that
// HBM sees each element once.  Thread (r, v) owns vector v of rows r, r + R, ...; sums are kept per channel in registers, added
// over the R thread rows by a tree in shared memory and over a group's channels by a warp.  Forward: mean of the CTA's part,
// then squares of the deviations from it; the parts are joined over the cluster by Chan's formula (exact weights, no
// cancellation).  Backward: the channel sums of g and g xh give dw and db, and weighted with w the two group means that dx needs.
// Maps too large for that (or rows of more than NT vectors) are read twice by the streaming kernels below.

namespace {

constexpr int NT = 512;

struct GnArgs {
  const void* x; const void* dy; const void* w; const void* b;
  void* y;                               // forward: y; backward: dx (may be null)
  void* dw; void* db;
  float* mean; float* rstd;
  float* part;                           // scratch
  long long xs, xp, ys, yp, ds, dp;      // pitches of x, y (dx), dy
  long long samples;
  uint32_t positions;
  int C, G, D;                           // channels, groups, channels per group
  float eps;
  int gpc, chunks, Q, ppc;               // groups per chunk, chunks, CTAs per chunk, positions per CTA
  int parts;                             // streaming: position ranges per sample
};

__device__ __forceinline__ void cp16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp4(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.commit_group;" ::: "memory");
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}
// VE elements from global to shared memory, without a detour through registers where the hardware has one
template <typename T, int VE> __device__ __forceinline__ void copy_in(T* dst, const T* src) {
  if (sizeof(T) * VE == 16) cp16(dst, src);
  else if (sizeof(T) * VE == 4) cp4(dst, src);
  else *dst = *src;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float ld_peer(const float* p, int rank) {       // *p of CTA `rank` of the cluster
  uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(r) : "memory");
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <typename T> __device__ __forceinline__ float param(const void* p, int c, float none) { return p ? ldf((const T*)p, c) : none; }

// red[r][c] of R thread rows -> red[0][c], every thread adding its own vector v of rows r and r + h.  Ends with a barrier.
template <int VE>
__device__ __forceinline__ void tree_rows(float* red, const float (&mine)[VE], int r, int R, int v, int cw, bool active) {
  float* at = red + r * cw + v * VE;
  if (active) {
#pragma unroll
    for (int j = 0; j < VE; ++j) at[j] = mine[j];
  }
  __syncthreads();
  int h = 1;
  while (h < R) h <<= 1;
  for (h >>= 1; h > 0; h >>= 1) {
    if (active && r < h && r + h < R) {
#pragma unroll
      for (int j = 0; j < VE; ++j) at[j] += at[h * cw + j];
    }
    __syncthreads();
  }
}

// The slope of the activation at u = xh w + b.  Which side of zero u lies on is decided in 64 bits where 32 leave it open.
template <int ACT>
__device__ __forceinline__ float slope_at(float xv, float mean, float rstd, float xh, float w, float b) {
  const float u = fmaf(xh, w, b);
  if (ACT == ABS_ACT_RELU && fabsf(u) <= 4e-7f * fabsf(xh * w))      // (xh: two roundings, u: one; 2^-23 + 2^-24 = 1.8e-7)
    return ((double)xv - (double)mean) * (double)rstd * (double)w + (double)b > 0.0 ? 1.f : 0.f;
  return act_slope<ACT>(u);
}

// Shape of a CTA's work.
struct Share {
  int rank, ch, c0, cw, groups, lv, R, r, v, np;
  long long n, p0;
  bool active;
};
template <int VE> __device__ __forceinline__ Share share_of(const GnArgs& a) {
  Share s;
  s.rank = (int)(blockIdx.x % a.Q);
  const uint32_t u = blockIdx.x / a.Q;
  s.n = u / a.chunks;
  s.ch = (int)(u % a.chunks);
  s.groups = min(a.gpc, a.G - s.ch * a.gpc);
  s.c0 = s.ch * a.gpc * a.D;
  s.cw = s.groups * a.D;
  s.lv = s.cw / VE;
  s.R = NT / s.lv;
  s.r = (int)threadIdx.x / s.lv;
  s.v = (int)threadIdx.x - s.r * s.lv;
  s.active = s.r < s.R;
  s.p0 = (long long)s.rank * a.ppc;
  s.np = (int)min((long long)a.ppc, (long long)a.positions - s.p0);
  return s;
}

template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(NT) gn_forward_kernel(const GnArgs a) {
  extern __shared__ __align__(16) uint8_t gsm[];
  const Share s = share_of<VE>(a);
  const int maxcw = a.gpc * a.D;
  float* red = reinterpret_cast<float*>(gsm);                    // [NT * VE]
  float* own = red + NT * VE;                                    // [2][gpc] this CTA's means and squared deviations
  float* fin = own + 2 * a.gpc;                                  // [2][gpc] the sample's means and 1 / standard deviations
  T* data = reinterpret_cast<T*>(gsm + round_up_sz((size_t)(NT * VE + 4 * a.gpc) * 4, 16));      // [ppc][cw]
  (void)maxcw;
  grid_dependency_sync();
  const T* x = (const T*)a.x + s.n * a.xs + s.p0 * a.xp + s.c0 + s.v * VE;
  T* mine = data + (size_t)s.v * VE;
  if (s.active)
    for (int p = s.r; p < s.np; p += s.R) copy_in<T, VE>(mine + (size_t)p * s.cw, x + (long long)p * a.xp);
  cp_wait();
  float acc[VE], mu[VE];
  int grp[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) { acc[j] = 0.f; grp[j] = (s.v * VE + j) / a.D; }
  if (s.active)
    for (int p = s.r; p < s.np; p += s.R) {
      Pack<T, VE> q;
      float f[VE];
      q.load(mine + (size_t)p * s.cw);
      q.get(f);
#pragma unroll
      for (int j = 0; j < VE; ++j) acc[j] += f[j];
    }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float cnt = (float)s.np * (float)a.D;
  tree_rows<VE>(red, acc, s.r, s.R, s.v, s.cw, s.active);
  for (int g = warp; g < s.groups; g += NT / 32) {
    float t = 0.f;
    for (int c = lane; c < a.D; c += 32) t += red[g * a.D + c];
    t = warp_sum(t);
    if (lane == 0) own[g] = t / cnt;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < VE; ++j) { acc[j] = 0.f; mu[j] = s.active ? own[grp[j]] : 0.f; }
  if (s.active)
    for (int p = s.r; p < s.np; p += s.R) {
      Pack<T, VE> q;
      float f[VE];
      q.load(mine + (size_t)p * s.cw);
      q.get(f);
#pragma unroll
      for (int j = 0; j < VE; ++j) { const float d = f[j] - mu[j]; acc[j] = fmaf(d, d, acc[j]); }
    }
  tree_rows<VE>(red, acc, s.r, s.R, s.v, s.cw, s.active);
  for (int g = warp; g < s.groups; g += NT / 32) {
    float t = 0.f;
    for (int c = lane; c < a.D; c += 32) t += red[g * a.D + c];
    t = warp_sum(t);
    if (lane == 0) own[a.gpc + g] = t;
  }
  if (a.Q > 1) { cluster_arrive(); cluster_wait(); }
  else __syncthreads();
  for (int g = threadIdx.x; g < s.groups; g += NT) {
    // M = sum n_i m_i / N, V = sum (v_i + n_i (m_i - M)^2) / N
    float mean = 0.f, var = 0.f;
    const float total = (float)a.positions * (float)a.D;
    for (int q = 0; q < a.Q; ++q) {
      const float nq = (float)min((long long)a.ppc, (long long)a.positions - (long long)q * a.ppc) * (float)a.D;
      mean = fmaf(nq / total, a.Q > 1 ? ld_peer(own + g, q) : own[g], mean);
    }
    for (int q = 0; q < a.Q; ++q) {
      const float nq = (float)min((long long)a.ppc, (long long)a.positions - (long long)q * a.ppc) * (float)a.D;
      const float d = (a.Q > 1 ? ld_peer(own + g, q) : own[g]) - mean;
      var += fmaf(nq * d, d, a.Q > 1 ? ld_peer(own + a.gpc + g, q) : own[a.gpc + g]);
    }
    const float rstd = 1.f / sqrtf(var / total + a.eps);
    fin[g] = mean;
    fin[a.gpc + g] = rstd;
    if (s.rank == 0 && a.mean) {
      a.mean[s.n * a.G + s.ch * a.gpc + g] = mean;
      a.rstd[s.n * a.G + s.ch * a.gpc + g] = rstd;
    }
  }
  __syncthreads();
  if (a.Q > 1) cluster_arrive();                                 // (nobody leaves while a peer reads its sums: waited for at the end)
  if (s.active) {
    float sc[VE], sh[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const int c = s.c0 + s.v * VE + j;
      mu[j] = fin[grp[j]];
      sc[j] = fin[a.gpc + grp[j]] * param<T>(a.w, c, 1.f);
      sh[j] = param<T>(a.b, c, 0.f);
    }
    T* y = (T*)a.y + s.n * a.ys + s.p0 * a.yp + s.c0 + s.v * VE;
    for (int p = s.r; p < s.np; p += s.R) {
      Pack<T, VE> q;
      float f[VE];
      q.load(mine + (size_t)p * s.cw);
      q.get(f);
#pragma unroll
      for (int j = 0; j < VE; ++j) f[j] = act_value<ACT>(fmaf(f[j] - mu[j], sc[j], sh[j]));
      q.set(f);
      q.store(y + (long long)p * a.yp);
    }
  }
  __syncwarp();
  if (a.Q > 1) cluster_wait();
}

template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(NT) gn_backward_kernel(const GnArgs a) {
  extern __shared__ __align__(16) uint8_t gsm[];
  const Share s = share_of<VE>(a);
  const int maxcw = a.gpc * a.D;
  float* red = reinterpret_cast<float*>(gsm);                    // [NT * VE]
  float* own = red + NT * VE;                                    // [2][cw] this CTA's channel sums of g and g xh
  float* tot = own + 2 * maxcw;                                  // [2][cw] the sample's, times w
  float* fin = tot + 2 * maxcw;                                  // [2][gpc] the two group means
  T* data = reinterpret_cast<T*>(gsm + round_up_sz((size_t)(NT * VE + 4 * maxcw + 2 * a.gpc) * 4, 16));      // [2][ppc][cw]
  T* data2 = data + round_up_sz((size_t)a.ppc * s.cw, 16);
  grid_dependency_sync();
  const T* x = (const T*)a.x + s.n * a.xs + s.p0 * a.xp + s.c0 + s.v * VE;
  const T* dy = (const T*)a.dy + s.n * a.ds + s.p0 * a.dp + s.c0 + s.v * VE;
  T* mx = data + (size_t)s.v * VE;
  T* mg = data2 + (size_t)s.v * VE;
  if (s.active)
    for (int p = s.r; p < s.np; p += s.R) {
      copy_in<T, VE>(mx + (size_t)p * s.cw, x + (long long)p * a.xp);
      copy_in<T, VE>(mg + (size_t)p * s.cw, dy + (long long)p * a.dp);
    }
  float sb[VE], sw[VE], mu[VE], rs[VE], wv[VE], bv[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int c = s.c0 + s.v * VE + j;
    sb[j] = sw[j] = mu[j] = rs[j] = wv[j] = bv[j] = 0.f;
    if (s.active) {
      mu[j] = a.mean[s.n * a.G + c / a.D];
      rs[j] = a.rstd[s.n * a.G + c / a.D];
      wv[j] = param<T>(a.w, c, 1.f);
      bv[j] = param<T>(a.b, c, 0.f);
    }
  }
  cp_wait();
  if (s.active)
    for (int p = s.r; p < s.np; p += s.R) {
      Pack<T, VE> q, d;
      float f[VE], g[VE];
      q.load(mx + (size_t)p * s.cw);
      d.load(mg + (size_t)p * s.cw);
      q.get(f);
      d.get(g);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float xh = (f[j] - mu[j]) * rs[j];
        const float gj = g[j] * slope_at<ACT>(f[j], mu[j], rs[j], xh, wv[j], bv[j]);
        sb[j] += gj;
        sw[j] = fmaf(gj, xh, sw[j]);
      }
    }
  tree_rows<VE>(red, sb, s.r, s.R, s.v, s.cw, s.active);
  for (int c = threadIdx.x; c < s.cw; c += NT) own[c] = red[c];
  __syncthreads();
  tree_rows<VE>(red, sw, s.r, s.R, s.v, s.cw, s.active);
  for (int c = threadIdx.x; c < s.cw; c += NT) own[maxcw + c] = red[c];
  if (a.Q > 1) { cluster_arrive(); cluster_wait(); }
  else __syncthreads();
  for (int i = threadIdx.x; i < 2 * s.cw; i += NT) {
    const int k = i >= s.cw ? 1 : 0, c = i - k * s.cw;
    float t = 0.f;
    for (int q = 0; q < a.Q; ++q) t += a.Q > 1 ? ld_peer(own + k * maxcw + c, q) : own[k * maxcw + c];
    if (s.rank == 0 && a.part) a.part[((size_t)s.n * 2 + k) * a.C + s.c0 + c] = t;
    tot[k * maxcw + c] = t * param<T>(a.w, s.c0 + c, 1.f);
  }
  __syncthreads();
  if (a.Q > 1) cluster_arrive();
  if (a.y != nullptr) {                                          // (uniform)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float total = (float)a.positions * (float)a.D;
    for (int i = warp; i < 2 * s.groups; i += NT / 32) {
      const int k = i >= s.groups ? 1 : 0, g = i - k * s.groups;
      float t = 0.f;
      for (int c = lane; c < a.D; c += 32) t += tot[k * maxcw + g * a.D + c];
      t = warp_sum(t);
      if (lane == 0) fin[k * a.gpc + g] = t / total;
    }
    __syncthreads();
    if (s.active) {
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const int g = (s.v * VE + j) / a.D;
        sb[j] = fin[g];
        sw[j] = fin[a.gpc + g];
      }
      T* dx = (T*)a.y + s.n * a.ys + s.p0 * a.yp + s.c0 + s.v * VE;
      for (int p = s.r; p < s.np; p += s.R) {
        Pack<T, VE> q, d;
        float f[VE], g[VE];
        q.load(mx + (size_t)p * s.cw);
        d.load(mg + (size_t)p * s.cw);
        q.get(f);
        d.get(g);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          const float xh = (f[j] - mu[j]) * rs[j];
          const float gj = g[j] * slope_at<ACT>(f[j], mu[j], rs[j], xh, wv[j], bv[j]) * wv[j];
          f[j] = rs[j] * (gj - fmaf(xh, sw[j], sb[j]));
        }
        q.set(f);
        q.store(dx + (long long)p * a.yp);
      }
    }
  }
  __syncwarp();
  if (a.Q > 1) cluster_wait();
}

// ---- streaming form: CTA = (sample, range of positions, 32 vectors of channels); 16 rows of threads

constexpr int SNT = 512, SROWS = SNT / 32;
struct Range { long long n; int c; uint32_t p0, p1; };
template <int VE> __device__ __forceinline__ Range range_of(const GnArgs& a) {
  Range r;
  r.n = blockIdx.x / a.parts;
  const uint32_t part = blockIdx.x % a.parts;
  r.c = (int)(blockIdx.y * 32 + (threadIdx.x & 31)) * VE;
  r.p0 = part * (uint32_t)a.ppc;
  r.p1 = (uint32_t)min((long long)a.positions, (long long)r.p0 + a.ppc);
  return r;
}

// part[n][s][0 | 1][c]: mean and squared deviations of channel c over the range
template <typename T, int VE>
__global__ void __launch_bounds__(SNT) gn_stats_kernel(const GnArgs a) {
  __shared__ float red[SROWS][32][VE];
  const Range r = range_of<VE>(a);
  const int row = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dependency_sync();
  const T* x = (const T*)a.x + r.n * a.xs + r.c;
  const bool in = r.c < a.C;
  float acc[VE], mu[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) acc[j] = mu[j] = 0.f;
  for (int pass = 0; pass < 2; ++pass) {
    if (in)
#pragma unroll 4
      for (uint32_t p = r.p0 + row; p < r.p1; p += SROWS) {
        Pack<T, VE> q;
        float f[VE];
        q.load(x + (long long)p * a.xp);
        q.get(f);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          if (pass == 0) acc[j] += f[j];
          else { const float d = f[j] - mu[j]; acc[j] = fmaf(d, d, acc[j]); }
        }
      }
#pragma unroll
    for (int j = 0; j < VE; ++j) red[row][lane][j] = acc[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      float t = 0.f;
      for (int k = 0; k < SROWS; ++k) t += red[k][lane][j];
      if (pass == 0) mu[j] = t / (float)(r.p1 - r.p0);
      acc[j] = pass == 0 ? 0.f : t;
    }
    __syncthreads();
  }
  if (in && row < 2)
#pragma unroll
    for (int j = 0; j < VE; ++j) a.part[((size_t)blockIdx.x * 2 + row) * a.C + r.c + j] = row ? acc[j] : mu[j];
}

__device__ __forceinline__ float block_sum(float v, float* sm) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
  for (int i = 0; i < 8; ++i) t += sm[i];
  return t;
}

// mean and rstd of a group from its channels' parts: CTA = (sample, group)
__global__ void __launch_bounds__(256) gn_join_kernel(const GnArgs a, float* stat) {
  __shared__ float sm[8];
  grid_dependency_sync();
  const long long n = blockIdx.x / a.G;
  const int g = (int)(blockIdx.x % a.G);
  const long long items = (long long)a.parts * a.D;
  const float total = (float)a.positions * (float)a.D;
  auto weight = [&](long long s) { return (float)min((long long)a.ppc, (long long)a.positions - s * a.ppc); };
  auto at = [&](long long s, int k, int c) { return a.part[((size_t)(n * a.parts + s) * 2 + k) * a.C + g * a.D + c]; };
  float t = 0.f;
  for (long long i = threadIdx.x; i < items; i += 256) t = fmaf(weight(i / a.D) / total, at(i / a.D, 0, (int)(i % a.D)), t);
  const float mean = block_sum(t, sm);
  t = 0.f;
  for (long long i = threadIdx.x; i < items; i += 256) {
    const float d = at(i / a.D, 0, (int)(i % a.D)) - mean;
    t += fmaf(weight(i / a.D) * d, d, at(i / a.D, 1, (int)(i % a.D)));
  }
  const float rstd = 1.f / sqrtf(block_sum(t, sm) / total + a.eps);
  if (threadIdx.x == 0) {
    stat[2 * (size_t)blockIdx.x] = mean;
    stat[2 * (size_t)blockIdx.x + 1] = rstd;
    if (a.mean) { a.mean[blockIdx.x] = mean; a.rstd[blockIdx.x] = rstd; }
  }
}

template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(SNT) gn_apply_kernel(const GnArgs a, const float* stat) {
  const Range r = range_of<VE>(a);
  const int row = threadIdx.x >> 5;
  grid_dependency_sync();
  if (r.c >= a.C) return;
  float mu[VE], sc[VE], sh[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const size_t g = 2 * ((size_t)r.n * a.G + (r.c + j) / a.D);
    mu[j] = stat[g];
    sc[j] = stat[g + 1] * param<T>(a.w, r.c + j, 1.f);
    sh[j] = param<T>(a.b, r.c + j, 0.f);
  }
  const T* x = (const T*)a.x + r.n * a.xs + r.c;
  T* y = (T*)a.y + r.n * a.ys + r.c;
#pragma unroll 4
  for (uint32_t p = r.p0 + row; p < r.p1; p += SROWS) {
    Pack<T, VE> q;
    float f[VE];
    q.load(x + (long long)p * a.xp);
    q.get(f);
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = act_value<ACT>(fmaf(f[j] - mu[j], sc[j], sh[j]));
    q.set(f);
    q.store(y + (long long)p * a.yp);
  }
}

// part[n][s][0 | 1][c]: sums of g and g xh over the range
template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(SNT) gn_sums_kernel(const GnArgs a) {
  __shared__ float red[SROWS][32][VE];
  const Range r = range_of<VE>(a);
  const int row = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dependency_sync();
  const T* x = (const T*)a.x + r.n * a.xs + r.c;
  const T* dy = (const T*)a.dy + r.n * a.ds + r.c;
  float sb[VE], sw[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) sb[j] = sw[j] = 0.f;
  if (r.c < a.C) {
    float mu[VE], rs[VE], wv[VE], bv[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      mu[j] = a.mean[r.n * a.G + (r.c + j) / a.D];
      rs[j] = a.rstd[r.n * a.G + (r.c + j) / a.D];
      wv[j] = param<T>(a.w, r.c + j, 1.f);
      bv[j] = param<T>(a.b, r.c + j, 0.f);
    }
#pragma unroll 2
    for (uint32_t p = r.p0 + row; p < r.p1; p += SROWS) {
      Pack<T, VE> q, d;
      float f[VE], g[VE];
      q.load(x + (long long)p * a.xp);
      d.load(dy + (long long)p * a.dp);
      q.get(f);
      d.get(g);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float xh = (f[j] - mu[j]) * rs[j];
        const float gj = g[j] * slope_at<ACT>(f[j], mu[j], rs[j], xh, wv[j], bv[j]);
        sb[j] += gj;
        sw[j] = fmaf(gj, xh, sw[j]);
      }
    }
  }
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int j = 0; j < VE; ++j) red[row][lane][j] = k ? sw[j] : sb[j];
    __syncthreads();
    if (row == 0 && r.c < a.C)
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        float t = 0.f;
        for (int q = 0; q < SROWS; ++q) t += red[q][lane][j];
        a.part[((size_t)blockIdx.x * 2 + k) * a.C + r.c + j] = t;
      }
    __syncthreads();
  }
}

// the two group means of g w and g w xh: CTA = (sample, group)
template <typename T>
__global__ void __launch_bounds__(256) gn_join_sums_kernel(const GnArgs a, float* stat) {
  __shared__ float sm[8];
  grid_dependency_sync();
  const long long n = blockIdx.x / a.G;
  const int g = (int)(blockIdx.x % a.G);
  const long long items = (long long)a.parts * a.D;
  for (int k = 0; k < 2; ++k) {
    float t = 0.f;
    for (long long i = threadIdx.x; i < items; i += 256) {
      const int c = g * a.D + (int)(i % a.D);
      t = fmaf(a.part[((size_t)(n * a.parts + i / a.D) * 2 + k) * a.C + c], param<T>(a.w, c, 1.f), t);
    }
    t = block_sum(t, sm) / ((float)a.positions * (float)a.D);
    if (threadIdx.x == 0) stat[2 * (size_t)blockIdx.x + k] = t;
  }
}

template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(SNT) gn_dx_kernel(const GnArgs a, const float* stat) {
  const Range r = range_of<VE>(a);
  const int row = threadIdx.x >> 5;
  grid_dependency_sync();
  if (r.c >= a.C) return;
  float mu[VE], rs[VE], wv[VE], bv[VE], s1[VE], s2[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const size_t g = (size_t)r.n * a.G + (r.c + j) / a.D;
    mu[j] = a.mean[g];
    rs[j] = a.rstd[g];
    s1[j] = stat[2 * g];
    s2[j] = stat[2 * g + 1];
    wv[j] = param<T>(a.w, r.c + j, 1.f);
    bv[j] = param<T>(a.b, r.c + j, 0.f);
  }
  const T* x = (const T*)a.x + r.n * a.xs + r.c;
  const T* dy = (const T*)a.dy + r.n * a.ds + r.c;
  T* dx = (T*)a.y + r.n * a.ys + r.c;
  for (uint32_t p = r.p0 + row; p < r.p1; p += SROWS) {
    Pack<T, VE> q, d;
    float f[VE], g[VE];
    q.load(x + (long long)p * a.xp);
    d.load(dy + (long long)p * a.dp);
    q.get(f);
    d.get(g);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float xh = (f[j] - mu[j]) * rs[j];
      const float gj = g[j] * slope_at<ACT>(f[j], mu[j], rs[j], xh, wv[j], bv[j]) * wv[j];
      f[j] = rs[j] * (gj - fmaf(xh, s2[j], s1[j]));
    }
    q.set(f);
    q.store(dx + (long long)p * a.yp);
  }
}

// out[s][0 | 1][c] = sum of rows s per, ... of part[rows][2][C]; the last stage writes db and dw: block = 32 columns x 8 rows of threads
template <typename T>
__global__ void __launch_bounds__(256) gn_param_kernel(const float* part, long long rows, long long per, int C, float* out, void* dw, void* db) {
  __shared__ float red[8][33];
  grid_dependency_sync();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long j = (long long)blockIdx.x * 32 + lane, width = 2ll * C;
  const long long r1 = min(rows, (long long)(blockIdx.y + 1) * per);
  float t = 0.f;
  if (j < width) {
#pragma unroll 8
    for (long long r = blockIdx.y * per + w; r < r1; r += 8) t += part[r * width + j];
  }
  red[w][lane] = t;
  __syncthreads();
  if (w == 0 && j < width) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) v += red[k][lane];
    if (out) out[blockIdx.y * width + j] = v;
    else if (j < C) { if (db) stf((T*)db, j, v); }
    else if (dw) stf((T*)dw, j - C, v);
  }
}

typedef void (*GnFn)(const GnArgs);
typedef void (*GnStatFn)(const GnArgs, const float*);
#define GN_ACT(type, name, T, VE, act)                                                                              \
  ((act) == ABS_ACT_RELU ? (type)name<T, VE, ABS_ACT_RELU> : (act) == ABS_ACT_GELU ? (type)name<T, VE, ABS_ACT_GELU> \
   : (act) == ABS_ACT_SILU ? (type)name<T, VE, ABS_ACT_SILU> : (type)name<T, VE, ABS_ACT_NONE>)
#define GN_PICK(type, name, dtype, vec, act)                                                                        \
  ((dtype) == ABS_FP32 ? ((vec) ? GN_ACT(type, name, float, 4, act) : GN_ACT(type, name, float, 1, act))            \
                       : ((vec) ? GN_ACT(type, name, __nv_bfloat16, 8, act) : GN_ACT(type, name, __nv_bfloat16, 1, act)))

constexpr size_t CTA_BYTES = 72 * 1024, MOST_BYTES = 200 * 1024;

// How a call is cut up; `vec`: 16-byte accesses.  The scratch of a call is the larger of the two forms'.
struct Plan {
  bool resident;
  int gpc, chunks, Q, ppc;               // resident form
  size_t smem;
  int parts, sppc;                       // streaming form
};
size_t smem_bytes(int gpc, int D, long long ppc, int VE, size_t esz, bool grad) {
  const size_t cw = (size_t)gpc * D;
  const size_t head = round_up_sz(((size_t)NT * VE + (grad ? 4 * cw + 2 * gpc : 4 * (size_t)gpc)) * 4, 16);
  return head + (grad ? 2 : 1) * round_up_sz((size_t)ppc * cw, 16) * esz;
}
Plan plan(long long samples, long long positions, int C, int G, int dtype, bool grad, bool vec) {
  Plan p = {};
  const int D = C / G;
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  const int VE = vec ? (int)(16 / esz) : 1;
  // streaming: ranges of at least 64 positions, about 8 CTAs per SM in all
  const long long cols = (C + 32 * VE - 1) / (32 * VE);
  long long parts = (8 * PLAN_SMS + samples * cols - 1) / (samples * cols);
  if (parts > (positions + 63) / 64) parts = (positions + 63) / 64;
  if (parts < 1) parts = 1;
  p.sppc = (int)((positions + parts - 1) / parts);
  p.parts = (int)((positions + p.sppc - 1) / p.sppc);
  // resident: the smallest chunk of whole groups and whole vectors with 128 bytes of channels
  int unit = 1;
  while ((long long)unit * D % VE) ++unit;
  int gpc = unit;
  while (gpc < G && (size_t)gpc * D * esz < 128) gpc += unit;
  if (gpc > G) gpc = G;
  for (;; gpc = unit) {
    if ((long long)gpc * D / VE <= NT) {
      for (long long q = 1; q <= 8; ++q) {
        const long long ppc = (positions + q - 1) / q;
        if ((q - 1) * ppc >= positions) break;
        const size_t need = ppc < (1 << 24) ? smem_bytes(gpc, D, ppc, VE, esz, grad) : ~(size_t)0;
        const long long chunks = (G + gpc - 1) / gpc;
        const bool busy = samples * chunks * q >= PLAN_SMS || (size_t)ppc * gpc * D * esz <= 8192;
        if (need <= CTA_BYTES && busy) { p.resident = true; }
        else if (need <= MOST_BYTES && q == 8) { p.resident = true; }
        else if (need <= MOST_BYTES && (q + 1 > 8 || q * ((positions + q) / (q + 1)) >= positions)) { p.resident = true; }
        if (p.resident) {
          p.gpc = gpc; p.chunks = (int)chunks; p.Q = (int)q; p.ppc = (int)ppc; p.smem = need;
          if (samples * chunks * q > 0x7fffffff) p.resident = false;
          return p;
        }
      }
    }
    if (gpc == unit) return p;
  }
}

// floats of scratch in front of the partial sums: [samples * groups][2] statistics of the streaming form
size_t stat_floats(long long samples, int G) { return round_up_sz((size_t)samples * G * 2, 64); }
constexpr int PARAM_SPLIT = 64;          // rows of the first stage of the parameter sums when there are more than PARAM_ROWS
constexpr long long PARAM_ROWS = 512;
size_t scratch_floats(const Plan& p, long long samples, int C, int G, bool grad) {
  if (!grad) return p.resident ? 0 : stat_floats(samples, G) + (size_t)samples * p.parts * 2 * C;
  const long long rows = p.resident ? samples : samples * p.parts;
  return (p.resident ? 0 : stat_floats(samples, G)) + (size_t)rows * 2 * C + (rows > PARAM_ROWS ? (size_t)PARAM_SPLIT * 2 * C : 0);
}

cudaError_t run_params(const GnArgs& a, long long rows, int dtype, float* second, cudaStream_t s) {
  auto* kernel = dtype == ABS_FP32 ? gn_param_kernel<float> : gn_param_kernel<__nv_bfloat16>;
  const unsigned cols = (unsigned)((2ll * a.C + 31) / 32);
  const float* from = a.part;
  cudaError_t e = cudaSuccess;
  if (rows > PARAM_ROWS) {
    const long long per = (rows + PARAM_SPLIT - 1) / PARAM_SPLIT;
    e = launch(kernel, dim3(cols, PARAM_SPLIT), 256, 0, 1, s, from, rows, per, a.C, second, (void*)nullptr, (void*)nullptr);
    from = second;
    rows = PARAM_SPLIT;
  }
  if (e == cudaSuccess) e = launch(kernel, dim3(cols), 256, 0, 1, s, from, rows, rows, a.C, (float*)nullptr, a.dw, a.db);
  return e;
}

cudaError_t launch_resident(GnFn fn, const Plan& p, long long samples, cudaStream_t s, const GnArgs& a) {
  // the kernels' shared memory is raised to the most any plan asks for, once per device
  static std::atomic<uint64_t> ready;
  int device, sms;
  if (current_device(&device, &sms) != ABS_OK) return cudaErrorInvalidDevice;
  if (!(ready.load(std::memory_order_acquire) >> device & 1)) {
    for (int dtype = 0; dtype < 2; ++dtype)
      for (int act = ABS_ACT_NONE; act <= ABS_ACT_SILU; ++act)
        for (int vec = 0; vec < 2; ++vec) {
          cudaError_t e = allow_smem(GN_PICK(GnFn, gn_forward_kernel, dtype, vec, act), MOST_BYTES);
          if (e == cudaSuccess) e = allow_smem(GN_PICK(GnFn, gn_backward_kernel, dtype, vec, act), MOST_BYTES);
          if (e != cudaSuccess) return e;
        }
    ready.fetch_or(1ull << device, std::memory_order_release);
  }
  return launch(fn, dim3((unsigned)(samples * p.chunks * p.Q)), NT, p.smem, p.Q, s, a);
}

bool on16(const void* p) { return (uintptr_t)p % 16 == 0; }
bool pitch16(long long samples, long long positions, long long s, long long p, size_t esz) {
  return (samples == 1 || s * (long long)esz % 16 == 0) && (positions == 1 || p * (long long)esz % 16 == 0);
}

int check(long long samples, long long positions, int channels, int groups, int act, int dtype) {
  if (dtype != ABS_FP32 && dtype != ABS_BF16_FP32MASTER) return fail(ABS_EUNSUPPORTED, "unknown dtype %d", dtype);
  if (act < ABS_ACT_NONE || act > ABS_ACT_SILU) return fail(ABS_EUNSUPPORTED, "unknown activation %d", act);
  if (samples < 0 || samples >= (1ll << 31)) return fail(ABS_EINVAL, "samples %lld outside [0, 2^31)", samples);
  if (positions < 0 || positions >= (1ll << 31)) return fail(ABS_EINVAL, "positions %lld outside [0, 2^31)", positions);
  if (channels < 1 || channels > (1 << 20)) return fail(ABS_EINVAL, "channels %d outside [1, 2^20]", channels);
  if (groups < 1 || groups > channels || channels % groups) return fail(ABS_EINVAL, "channels %d is not a multiple of groups %d", channels, groups);
  if (samples * groups >= (1ll << 31)) return fail(ABS_EINVAL, "samples x groups = %lld outside [0, 2^31)", samples * groups);
  return ABS_OK;
}

int check_scratch(const void* scratch, size_t have, size_t need) {
  if (need == 0) return ABS_OK;
  if (have < need) return fail(ABS_ENOSPACE, "scratch holds %zu bytes, %zu needed", have, need);
  if (!scratch || (uintptr_t)scratch % 256) return fail(ABS_EINVAL, "scratch is null or not 256-byte aligned");
  return ABS_OK;
}

// maps [samples][positions][C] with pitches s, p
int check_maps(const char* name, const void* ptr, long long s, long long p, long long samples, long long positions, int C, size_t esz) {
  if (!ptr) return fail(ABS_EINVAL, "%s is null", name);
  if ((uintptr_t)ptr % esz) return fail(ABS_EINVAL, "%s is not aligned to its type", name);
  if (positions > 1 && p < C) return fail(ABS_EINVAL, "%s: position pitch %lld below the %d channels", name, p, C);
  if (samples > 1 && s < (positions - 1) * (positions > 1 ? p : 0) + C) return fail(ABS_EINVAL, "%s: samples overlap (pitch %lld)", name, s);
  return ABS_OK;
}

Span maps_span(const void* ptr, long long s, long long p, long long samples, long long positions, int C, size_t esz) {
  Span r = {(uintptr_t)ptr, (uintptr_t)ptr, (long long)(p * (long long)esz), (long long)(C * (long long)esz)};
  if (ptr) r.hi += (uintptr_t)(((samples - 1) * s + (positions - 1) * p + C) * (long long)esz);
  if (samples > 1 && s % (p > 0 ? p : 1)) r.ld = 0;      // (rows of different samples are not a multiple of the pitch apart)
  return r;
}

}  // namespace

extern "C" int abs_group_norm_scratch_bytes(long long samples, long long positions, int channels, int groups, int dtype, int grad,
                                            size_t* out) {
  if (!out) return fail(ABS_EINVAL, "out is null");
  const int rc = check(samples, positions, channels, groups, 0, dtype);
  if (rc != ABS_OK) return rc;
  const size_t a = samples == 0 || positions == 0 ? 0 : scratch_floats(plan(samples, positions, channels, groups, dtype, grad, true), samples, channels, groups, grad);
  const size_t b = samples == 0 || positions == 0 ? 0 : scratch_floats(plan(samples, positions, channels, groups, dtype, grad, false), samples, channels, groups, grad);
  *out = (a > b ? a : b) * 4;
  return ABS_OK;
}

extern "C" int abs_group_norm(const void* x, long long xs, long long xp, const void* w, const void* b, void* y, long long ys,
                              long long yp, float* mean, float* rstd, long long samples, long long positions, int channels,
                              int groups, float eps, int act, int dtype, void* scratch, size_t scratch_bytes, void* stream) {
  int rc = check(samples, positions, channels, groups, act, dtype);
  if (rc != ABS_OK) return rc;
  if (!(eps > 0.f)) return fail(ABS_EINVAL, "eps %g is not positive", (double)eps);
  if (!mean != !rstd) return fail(ABS_EINVAL, "mean and rstd go together");
  if (samples == 0 || positions == 0) return ABS_OK;
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  if ((rc = check_maps("x", x, xs, xp, samples, positions, channels, esz)) != ABS_OK) return rc;
  if ((rc = check_maps("y", y, ys, yp, samples, positions, channels, esz)) != ABS_OK) return rc;
  if (!(x == y && (samples == 1 || xs == ys) && (positions == 1 || xp == yp)) &&
      overlap(maps_span(x, xs, xp, samples, positions, channels, esz), maps_span(y, ys, yp, samples, positions, channels, esz)))
    return fail(ABS_EINVAL, "y overlaps x without being the same maps");
  GnArgs a = {};
  a.x = x; a.y = y; a.w = w; a.b = b; a.mean = mean; a.rstd = rstd;
  a.xs = xs; a.xp = xp; a.ys = ys; a.yp = yp;
  a.samples = samples; a.positions = (uint32_t)positions;
  a.C = channels; a.G = groups; a.D = channels / groups; a.eps = eps;
  const bool vec = (size_t)channels * esz % 16 == 0 && on16(x) && on16(y) && pitch16(samples, positions, xs, xp, esz) && pitch16(samples, positions, ys, yp, esz);
  const Plan p = plan(samples, positions, channels, groups, dtype, false, vec);
  if ((rc = check_scratch(scratch, scratch_bytes, scratch_floats(p, samples, channels, groups, false) * 4)) != ABS_OK) return rc;
  a.gpc = p.gpc; a.chunks = p.chunks; a.Q = p.Q; a.ppc = p.resident ? p.ppc : p.sppc;
  a.parts = p.parts;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e;
  if (p.resident) {
    e = launch_resident(GN_PICK(GnFn, gn_forward_kernel, dtype, vec, act), p, samples, s, a);
  } else {
    float* stat = (float*)scratch;
    a.part = stat + stat_floats(samples, groups);
    const int VE = vec ? (int)(16 / esz) : 1;
    const dim3 grid((unsigned)(samples * p.parts), (unsigned)((channels + 32 * VE - 1) / (32 * VE)));
    const GnFn stats = dtype == ABS_FP32 ? (vec ? (GnFn)gn_stats_kernel<float, 4> : (GnFn)gn_stats_kernel<float, 1>)
                                         : (vec ? (GnFn)gn_stats_kernel<__nv_bfloat16, 8> : (GnFn)gn_stats_kernel<__nv_bfloat16, 1>);
    e = launch(stats, grid, SNT, 0, 1, s, a);
    if (e == cudaSuccess) e = launch(gn_join_kernel, dim3((unsigned)(samples * groups)), 256, 0, 1, s, a, stat);
    if (e == cudaSuccess) e = launch(GN_PICK(GnStatFn, gn_apply_kernel, dtype, vec, act), grid, SNT, 0, 1, s, a, (const float*)stat);
  }
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}

extern "C" int abs_group_norm_grad(const void* dy, long long dys, long long dyp, const void* x, long long xs, long long xp,
                                   const void* w, const void* b, const float* mean, const float* rstd, void* dx, long long dxs,
                                   long long dxp, void* dw, void* db, long long samples, long long positions, int channels,
                                   int groups, int act, int dtype, void* scratch, size_t scratch_bytes, void* stream) {
  int rc = check(samples, positions, channels, groups, act, dtype);
  if (rc != ABS_OK) return rc;
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  cudaError_t e = cudaSuccess;
  if (samples == 0 || positions == 0) {
    if (dw) e = cudaMemsetAsync(dw, 0, channels * esz, (cudaStream_t)stream);
    if (db && e == cudaSuccess) e = cudaMemsetAsync(db, 0, channels * esz, (cudaStream_t)stream);
    return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "memset: %s", cudaGetErrorString(e));
  }
  if (!mean || !rstd) return fail(ABS_EINVAL, "mean and rstd of the forward pass are needed");
  if ((rc = check_maps("dy", dy, dys, dyp, samples, positions, channels, esz)) != ABS_OK) return rc;
  if ((rc = check_maps("x", x, xs, xp, samples, positions, channels, esz)) != ABS_OK) return rc;
  if (dx) {
    if ((rc = check_maps("dx", dx, dxs, dxp, samples, positions, channels, esz)) != ABS_OK) return rc;
    const Span sd = maps_span(dx, dxs, dxp, samples, positions, channels, esz);
    if (overlap(sd, maps_span(x, xs, xp, samples, positions, channels, esz))) return fail(ABS_EINVAL, "dx overlaps x");
    if (!(dx == dy && (samples == 1 || dxs == dys) && (positions == 1 || dxp == dyp)) &&
        overlap(sd, maps_span(dy, dys, dyp, samples, positions, channels, esz)))
      return fail(ABS_EINVAL, "dx overlaps dy without being the same maps");
  }
  GnArgs a = {};
  a.x = x; a.dy = dy; a.y = dx; a.w = w; a.b = b; a.dw = dw; a.db = db;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.xs = xs; a.xp = xp; a.ys = dxs; a.yp = dxp; a.ds = dys; a.dp = dyp;
  a.samples = samples; a.positions = (uint32_t)positions;
  a.C = channels; a.G = groups; a.D = channels / groups;
  const bool vec = (size_t)channels * esz % 16 == 0 && on16(x) && on16(dy) && on16(dx) && pitch16(samples, positions, xs, xp, esz) &&
                   pitch16(samples, positions, dys, dyp, esz) && (!dx || pitch16(samples, positions, dxs, dxp, esz));
  const Plan p = plan(samples, positions, channels, groups, dtype, true, vec);
  if (!dx && !dw && !db) return ABS_OK;
  if ((rc = check_scratch(scratch, scratch_bytes, scratch_floats(p, samples, channels, groups, true) * 4)) != ABS_OK) return rc;
  a.gpc = p.gpc; a.chunks = p.chunks; a.Q = p.Q; a.ppc = p.resident ? p.ppc : p.sppc;
  a.parts = p.parts;
  cudaStream_t s = (cudaStream_t)stream;
  const long long rows = p.resident ? samples : samples * p.parts;
  if (p.resident) {
    a.part = dw || db ? (float*)scratch : nullptr;
    e = launch_resident(GN_PICK(GnFn, gn_backward_kernel, dtype, vec, act), p, samples, s, a);
  } else {
    float* stat = (float*)scratch;
    a.part = stat + stat_floats(samples, groups);
    const int VE = vec ? (int)(16 / esz) : 1;
    const dim3 grid((unsigned)(samples * p.parts), (unsigned)((channels + 32 * VE - 1) / (32 * VE)));
    e = launch(GN_PICK(GnFn, gn_sums_kernel, dtype, vec, act), grid, SNT, 0, 1, s, a);
    if (dx && e == cudaSuccess) {
      auto* join = dtype == ABS_FP32 ? gn_join_sums_kernel<float> : gn_join_sums_kernel<__nv_bfloat16>;
      e = launch(join, dim3((unsigned)(samples * groups)), 256, 0, 1, s, a, stat);
      if (e == cudaSuccess) e = launch(GN_PICK(GnStatFn, gn_dx_kernel, dtype, vec, act), grid, SNT, 0, 1, s, a, (const float*)stat);
    }
  }
  if ((dw || db) && e == cudaSuccess) e = run_params(a, rows, dtype, a.part + (size_t)rows * 2 * channels, s);
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}
