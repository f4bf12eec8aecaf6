// Group normalisation of channels-last maps with an activation, and its gradients.
#include <algorithm>
#include <atomic>

#include "layerops.cuh"

using namespace absb;
using namespace absb::layer;

// A sample's maps are cut into chunks of whole groups (at least 128 bytes of channels where there are as many), and a cluster of
// Q CTAs takes one chunk of one sample: every CTA copies its share of the positions into shared memory, where it stays, so that
// HBM sees each element once.  Thread (r, v) owns vector v of rows r, r + R, ...; statistics are kept per channel in registers
// and joined in shared memory, a warp to a group.  Forward: each thread's means and squared deviations (about its own first
// element: the cancellation is at most 1 + n, n <= 32 rows), then the CTA's mean and squared deviations of a group, then the
// cluster's, by Chan's formula.  Backward: the channel sums of g and g xh give dw and db, and weighted with w the two group means that dx needs.
// Larger batches and maps are read twice by the streaming kernels below, the second time from L2.

namespace {

constexpr int NT = 256;

struct GnArgs {
  const void* x; const void* dy; const void* w; const void* b;
  void* y;                               // forward: y; backward: dx (may be null)
  void* dw; void* db;
  float* mean; float* rstd;
  float* part; float* stat;              // scratch: channel sums of the backward pass; entries of the streaming form
  long long xs, xp, ys, yp, ds, dp;      // pitches of x, y (dx), dy
  long long samples;
  uint32_t positions;
  int C, G, D;                           // channels, groups, channels per group
  float eps;
  int gpc, chunks, Q, ppc;               // groups per chunk, chunks, CTAs per chunk, positions per CTA
  int cw, R, last;                       // channels of a chunk, thread rows, positions of a chunk's last CTA
  int segments;                          // row segments that sum a channel
  Divisor by_Q, by_chunks, by_D, by_lv, by_R, by_cw;
  int parts;                             // streaming: position ranges per sample
  Divisor by_parts;
};

__device__ __forceinline__ void cp16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp4(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// the copies of a thread's block `b` of four have arrived
__device__ __forceinline__ void cp_wait(int b) {
  if (b == 0) asm volatile("cp.async.wait_group 3;" ::: "memory");
  else if (b == 1) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (b == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}
// VE elements from global to shared memory, without a detour through registers where the hardware has one
template <typename T, int VE> __device__ __forceinline__ void copy_in(T* dst, const T* src) {
  if (sizeof(T) * VE == 16) cp16(dst, src);
  else if (sizeof(T) * VE == 4) cp4(dst, src);
  else *dst = *src;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float eight_sum(float v) {              // over the aligned eight lanes
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <typename T> __device__ __forceinline__ float param(const void* p, int c, float none) { return p ? ldf((const T*)p, c) : none; }

// Sums of red[r][c] over the thread rows, in S = N / cw segments of rows (at least one): col[s][c].
template <int N> __device__ __forceinline__ void column_sums(const float* red, float* col, const GnArgs& a) {
  if (a.segments > 1) {
    const int sg = (int)a.by_cw.div(threadIdx.x), c = (int)threadIdx.x - sg * a.cw;
    if (sg < a.segments) {
      float t = 0.f;
#pragma unroll 4
      for (int r = sg; r < a.R; r += a.segments) t += red[r * a.cw + c];
      col[threadIdx.x] = t;
    }
  } else {
    for (int c = threadIdx.x; c < a.cw; c += N) {
      float t = 0.f;
#pragma unroll 4
      for (int r = 0; r < a.R; ++r) t += red[r * a.cw + c];
      col[c] = t;
    }
  }
}
// f(g, sum of channels [lo, hi) of group g over all segments) for each group of the CTA: a thread to a group of few terms, else
// a warp.  range(g, lo, hi) gives the channels.
template <int N, typename Range, typename F>
__device__ __forceinline__ void group_sums(const float* col, int segments, int cw, int groups, int D, Range range, F f) {
  if (segments * D <= 16) {
    for (int g = threadIdx.x; g < groups; g += N) {
      int lo, hi;
      range(g, lo, hi);
      float t = 0.f;
      for (int s = 0; s < segments; ++s)
#pragma unroll 4
        for (int c = lo; c < hi; ++c) t += col[s * cw + c];
      f(g, t);
    }
  } else {
    const int lane = threadIdx.x & 31;
    for (int g = threadIdx.x >> 5; g < groups; g += N / 32) {
      int lo, hi;
      range(g, lo, hi);
      float t = 0.f;
      if (D <= 16) {                     // several segments at a time
        const int k = 32 / D, s0 = lane / D, c = lo + lane - s0 * D;
        if (s0 < k && c < hi)
          for (int s = s0; s < segments; s += k) t += col[s * cw + c];
      } else {
        for (int s = 0; s < segments; ++s)
          for (int c = lo + lane; c < hi; c += 32) t += col[s * cw + c];
      }
      t = warp_sum(t);
      if (lane == 0) f(g, t);
    }
  }
}

// w or b of VE neighbouring channels
template <typename T, int VE> __device__ __forceinline__ void params(const void* p, int c, float none, float (&v)[VE]) {
  if (p == nullptr) {
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = none;
  } else if (VE > 1 && ((uintptr_t)p & 15) == 0) {               // (c is a multiple of VE)
    Pack<T, VE> q;
    q.load((const T*)p + c);
    q.get(v);
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = ldf((const T*)p, c + j);
  }
}
// v[j] = from(group of channel c + j)
template <int VE, typename F> __device__ __forceinline__ void per_group(int c, const GnArgs& a, F from, float (&v)[VE]) {
  int g = (int)a.by_D.div((uint32_t)c), left = a.D - (c - g * a.D);
  float t = from(g);
  if (left >= VE) {
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = t;
  } else if (a.D >= VE) {                                        // two groups
    const float t1 = from(g + 1);
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = j < left ? t : t1;
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      if (left == 0) { t = from(++g); left = a.D; }
      v[j] = t;
      --left;
    }
  }
}

// VE neighbouring channels of a sample in the backward pass: e = x - mean, u = e (rstd w) + b, g = dy act'(u).  (rstd is a factor of
// a whole channel's sum, and of all of dx, so that xh = e rstd itself is not needed.)
template <typename T, int VE, int ACT> struct Point {
  Lanes<VE> nmu, rw, b;
  __device__ __forceinline__ void init(const GnArgs& a, long long n, int c, bool in) {
    float m[VE], r[VE], v[VE];
    if (in) {
      params<T, VE>(a.w, c, 1.f, v);
      per_group<VE>(c, a, [&](int g) { return a.rstd[n * a.G + g]; }, r);
      per_group<VE>(c, a, [&](int g) { return a.mean[n * a.G + g]; }, m);
#pragma unroll
      for (int j = 0; j < VE; ++j) { r[j] *= v[j]; m[j] = -m[j]; }
      params<T, VE>(a.b, c, 0.f, v);
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j) m[j] = r[j] = v[j] = 0.f;
    }
    nmu.set(m); rw.set(r); b.set(v);
  }
  __device__ __forceinline__ void at(const GnArgs& a, long long n, int c, const Pack<T, VE>& x, const Pack<T, VE>& dy, Lanes<VE>& e, Lanes<VE>& g) const {
    float f[VE], d[VE];
    x.get(f);
    dy.get(d);
    e.set(f);
    e = add(e, nmu);
    g.set(d);
    if constexpr (ACT == ABS_ACT_NONE) return;
    const Lanes<VE> u = fma(e, rw, b);
    if constexpr (ACT != ABS_ACT_RELU) { g = mul(g, act_slopes<ACT>(u)); return; }
    // Which side of zero u lies on is decided in 64 bits where 32 leave it open (three roundings of e rstd w: 2^-22).
    float uv[VE], ev[VE], rv[VE];
    u.get(uv); e.get(ev); rw.get(rv);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      bool on = uv[j] > 0.f;
      if (fabsf(uv[j]) <= 4e-7f * fabsf(ev[j] * rv[j])) {
        const long long i = n * a.G + (c + j) / a.D;
        on = ((double)f[j] - (double)a.mean[i]) * (double)a.rstd[i] * (double)param<T>(a.w, c + j, 1.f) + (double)param<T>(a.b, c + j, 0.f) > 0.0;
      }
      d[j] = on ? d[j] : 0.f;
    }
    g.set(d);
  }
};
// dx = rstd (g w - s1 - xh s2) = g (rstd w) + n1 + e n2 with n1 = -rstd s1, n2 = -rstd^2 s2
template <int VE> __device__ __forceinline__ Lanes<VE> dx_of(const Lanes<VE>& e, const Lanes<VE>& g, const Lanes<VE>& rw, const Lanes<VE>& n1, const Lanes<VE>& n2) {
  return fma(g, rw, fma(e, n2, n1));
}

// Shape of a CTA's work.  Thread rows and columns are those of a full chunk; the last chunk of a sample can be narrower.
struct Share {
  int rank, ch, c0, cw, groups, r, v, np, rows;
  long long n, p0;
  bool active;
};
template <int VE> __device__ __forceinline__ Share share_of(const GnArgs& a) {
  Share s;
  const uint32_t u = a.by_Q.div(blockIdx.x), n = a.by_chunks.div(u);
  s.rank = (int)(blockIdx.x - u * a.by_Q.d);
  s.n = n;
  s.ch = (int)(u - n * a.by_chunks.d);
  s.groups = min(a.gpc, a.G - s.ch * a.gpc);
  s.c0 = s.ch * a.cw;
  s.cw = s.groups * a.D;
  s.r = (int)a.by_lv.div(threadIdx.x);
  s.v = (int)threadIdx.x - s.r * (int)a.by_lv.d;
  s.active = s.r < a.R && s.v * VE < s.cw;
  s.p0 = (long long)s.rank * a.ppc;
  s.np = s.rank == a.Q - 1 ? a.last : a.ppc;
  s.rows = s.active && s.r < s.np ? (int)a.by_R.div((uint32_t)(s.np - s.r + a.R - 1)) : 0;
  return s;
}
// Mean and squared deviations of VE channels over rows that come one by one, in stretches of at most 32: sums about the
// stretch's first row (whose own deviation is part of the result, so that cancellation costs at most a factor of 1 + 32), joined
// to what was there by Chan's formula.
template <int VE> struct Moments {
  float mean[VE], dev[VE], seen;
  Lanes<VE> nk, s1, s2;                                          // minus the first row; sums
  __device__ __forceinline__ Moments() : seen(0.f) {
#pragma unroll
    for (int j = 0; j < VE; ++j) mean[j] = dev[j] = 0.f;
  }
  template <typename T> __device__ __forceinline__ void begin(const Pack<T, VE>& q) {
    float f[VE];
    q.get(f);
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = -f[j];
    nk.set(f);
    s1.fill(0.f);
    s2.fill(0.f);
  }
  template <typename T> __device__ __forceinline__ void row(const Pack<T, VE>& q) {
    float f[VE];
    q.get(f);
    Lanes<VE> l;
    l.set(f);
    l = add(l, nk);
    s1 = add(s1, l);
    s2 = fma(l, l, s2);
  }
  __device__ __forceinline__ void end(float n) {
    float a1[VE], a2[VE], k0[VE];
    s1.get(a1); s2.get(a2); nk.get(k0);
    const float inv = 1.f / n;
    if (seen == 0.f) {
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        mean[j] = fmaf(a1[j], inv, -k0[j]);
        dev[j] = fmaxf(fmaf(-a1[j] * inv, a1[j], a2[j]), 0.f);
      }
    } else {
      const float share = n / (seen + n);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float delta = fmaf(a1[j], inv, -k0[j]) - mean[j];
        dev[j] += fmaxf(fmaf(-a1[j] * inv, a1[j], a2[j]), 0.f) + delta * delta * (seen * share);
        mean[j] = fmaf(delta, share, mean[j]);
      }
    }
    seen += n;
  }
};

// VE floats to shared memory, 16 bytes at a time where there are as many
template <int VE> __device__ __forceinline__ void put(float* d, const float (&v)[VE]) {
  Lanes<VE> l;
  l.set(v);
  l.store(d);
}

template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(NT, 3) gn_forward_kernel(const GnArgs a) {
  extern __shared__ __align__(16) uint8_t gsm[];
  const Share s = share_of<VE>(a);
  float* red = reinterpret_cast<float*>(gsm);                    // [R][cw]
  float* col = red + NT * VE;                                    // [segments][cw]
  float* own = col + max(NT, a.cw);                              // [2][gpc] this CTA's means and squared deviations
  float* fin = own + 2 * a.gpc;                                  // [2][gpc] the sample's means and 1 / standard deviations
  T* data = reinterpret_cast<T*>(gsm + round_up_sz((size_t)(NT * VE + max(NT, a.cw) + 4 * a.gpc) * 4, 16));      // [ppc][cw]
  grid_dependency_sync();
  T* mine = data + s.r * a.cw + s.v * VE;
  const int step = a.R * a.cw;                                   // elements between a thread's rows
  const int rows = s.rows;
  const int quarter = (rows + 3) >> 2;                           // rows of a block: the first is worked on while the others arrive
  {
    const T* x = (const T*)a.x + s.n * a.xs + (s.p0 + s.r) * a.xp + s.c0 + s.v * VE;
    T* d = mine;
    const long long xstep = a.R * a.xp;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int n = min(quarter, rows - b * quarter);
#pragma unroll 2
      for (int i = 0; i < n; ++i, x += xstep, d += step) copy_in<T, VE>(d, x);
      cp_commit();
    }
  }
  // mean and squared deviations of each of the thread's channels, 32 rows at a time
  Moments<VE> mo;
  const T* d = mine;
  cp_wait(0);
  for (int i = 0, b = 0; i < rows;) {
    const int n = min(32, rows - i);
    while (i >= (b + 1) * quarter) cp_wait(++b);
    Pack<T, VE> q;
    q.load(d);
    mo.begin(q);
    for (const int end = i + n; i < end;) {
      while (i >= (b + 1) * quarter) cp_wait(++b);
      const int stop = min(end, (b + 1) * quarter);
#pragma unroll 2
      for (; i < stop; ++i, d += step) {
        q.load(d);
        mo.row(q);
      }
    }
    mo.end((float)n);
  }
  const float (&me)[VE] = mo.mean, (&mm)[VE] = mo.dev;
  const float seen = mo.seen;
  const int S = max(1, a.segments);
  auto range = [&](int g, int& lo, int& hi) { lo = g * a.D; hi = lo + a.D; };
  float* at = red + s.r * a.cw + s.v * VE;
  float out[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) out[j] = me[j] * seen;
  if (s.active) put<VE>(at, out);
  __syncthreads();
  const float cnt = (float)s.np * (float)a.D;
  column_sums<NT>(red, col, a);
  __syncthreads();
  group_sums<NT>(col, S, a.cw, s.groups, a.D, range, [&](int g, float t) { own[g] = t / cnt; });
  __syncthreads();
  if (s.active) {
    float mu[VE];
    per_group<VE>(s.v * VE, a, [&](int g) { return own[g]; }, mu);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float e = me[j] - mu[j];
      out[j] = seen > 0.f ? fmaf(e * e, seen, mm[j]) : 0.f;      // (a thread without rows: no 0 times infinity)
    }
    put<VE>(at, out);
  }
  __syncthreads();
  column_sums<NT>(red, col, a);
  __syncthreads();
  group_sums<NT>(col, S, a.cw, s.groups, a.D, range, [&](int g, float t) { own[a.gpc + g] = t; });
  if (a.Q > 1) { __syncwarp(); cluster_arrive(); cluster_wait(); }
  else __syncthreads();
  for (int g = threadIdx.x; g < s.groups; g += NT) {
    // M = m_0 + sum n_i (m_i - m_0) / N (equal means stay what they are), V = sum (v_i + n_i (m_i - M)^2) / N; all CTAs but the last
    // have the same count
    float pm[8], pv[8], M = 0.f, V = 0.f;
    const float inv_total = 1.f / (float)a.positions, n0 = (float)a.ppc * inv_total, n1 = (float)a.last * inv_total;
    const float inv_all = inv_total / (float)a.D;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      pm[q] = pv[q] = 0.f;
      if (q < a.Q) {
        pm[q] = a.Q > 1 ? ld_peer(own + g, q) : own[g];
        pv[q] = a.Q > 1 ? ld_peer(own + a.gpc + g, q) : own[a.gpc + g];
      }
    }
    M = pm[0];
#pragma unroll
    for (int q = 1; q < 8; ++q)
      if (q < a.Q) M = fmaf(q == a.Q - 1 ? n1 : n0, pm[q] - pm[0], M);
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < a.Q) {
        const float e = pm[q] - M;
        V = fmaf(pv[q], inv_all, fmaf((q == a.Q - 1 ? n1 : n0) * e, e, V));
      }
    const float rstd = 1.f / sqrtf(V + a.eps);
    fin[g] = M;
    fin[a.gpc + g] = rstd;
    if (s.rank == 0 && a.mean) {
      a.mean[s.n * a.G + s.ch * a.gpc + g] = M;
      a.rstd[s.n * a.G + s.ch * a.gpc + g] = rstd;
    }
  }
  __syncthreads();
  if (a.Q > 1) cluster_arrive();                                 // (nobody leaves while a peer reads its sums: waited for at the end)
  if (rows > 0) {
    Lanes<VE> nmu, sc, sh;
    float f0[VE], f1[VE], f2[VE];
    params<T, VE>(a.w, s.c0 + s.v * VE, 1.f, f2);
    per_group<VE>(s.v * VE, a, [&](int g) { return fin[g]; }, f0);
    per_group<VE>(s.v * VE, a, [&](int g) { return fin[a.gpc + g]; }, f1);
#pragma unroll
    for (int j = 0; j < VE; ++j) { f0[j] = -f0[j]; f1[j] *= f2[j]; }
    params<T, VE>(a.b, s.c0 + s.v * VE, 0.f, f2);
    nmu.set(f0); sc.set(f1); sh.set(f2);
    T* y = (T*)a.y + s.n * a.ys + (s.p0 + s.r) * a.yp + s.c0 + s.v * VE;
    d = mine;
    const long long ystep = a.R * a.yp;
#pragma unroll 2
    for (int i = 0; i < rows; ++i, d += step, y += ystep) {
      Pack<T, VE> q;
      float f[VE];
      q.load(d);
      q.get(f);
      Lanes<VE> l;
      l.set(f);
      act_values<ACT>(fma(add(l, nmu), sc, sh)).get(f);
      q.set(f);
      q.store(y);
    }
  }
  __syncwarp();
  if (a.Q > 1) cluster_wait();
}

template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(NT, 3) gn_backward_kernel(const GnArgs a) {
  extern __shared__ __align__(16) uint8_t gsm[];
  const Share s = share_of<VE>(a);
  const int maxcw = a.cw;
  float* red = reinterpret_cast<float*>(gsm);                    // [2][R][cw]
  const int cols = max(NT, a.cw);
  float* col = red + 2 * NT * VE;                                // [2][segments][cw]
  float* own = col + 2 * cols;                                    // [2][cw] this CTA's channel sums of g and g xh
  float* tot = own + 2 * maxcw;                                  // [2][cw] the sample's, times w
  float* fin = tot + 2 * maxcw;                                  // [2][gpc] the two group means
  // [ppc][cw] dy as it arrives, then g in fp32, vector by vector in the same place; [ppc][cw] x
  float* gs = reinterpret_cast<float*>(gsm + round_up_sz((size_t)(2 * NT * VE + 2 * cols + 4 * maxcw + 2 * a.gpc) * 4, 16));
  T* data = reinterpret_cast<T*>(gs + round_up_sz((size_t)a.ppc * a.cw, 16));
  grid_dependency_sync();
  const int first = s.r * a.cw + s.v * VE;
  const int step = a.R * a.cw;
  const int rows = s.rows;
  const int quarter = (rows + 3) >> 2;
  {
    const T* x = (const T*)a.x + s.n * a.xs + (s.p0 + s.r) * a.xp + s.c0 + s.v * VE;
    const T* dy = (const T*)a.dy + s.n * a.ds + (s.p0 + s.r) * a.dp + s.c0 + s.v * VE;
    int o = first;
    const long long xstep = a.R * a.xp, dstep = a.R * a.dp;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int n = min(quarter, rows - b * quarter);
      for (int i = 0; i < n; ++i, x += xstep, dy += dstep, o += step) {
        copy_in<T, VE>(data + o, x);
        copy_in<T, VE>(reinterpret_cast<T*>(gs + o), dy);
      }
      cp_commit();
    }
  }
  Point<T, VE, ACT> pt;
  pt.init(a, s.n, s.c0 + s.v * VE, s.active);
  Lanes<VE> sb, sw;
  sb.fill(0.f);
  sw.fill(0.f);
  for (int b = 0, i = 0, o = first; b < 4; ++b) {
    cp_wait(b);
#pragma unroll 2
    for (const int end = min(rows, (b + 1) * quarter); i < end; ++i, o += step) {
      Pack<T, VE> q, d;
      q.load(data + o);
      d.load(reinterpret_cast<const T*>(gs + o));
      Lanes<VE> e, g;
      pt.at(a, s.n, s.c0 + s.v * VE, q, d, e, g);
      sb = add(sb, g);
      sw = fma(g, e, sw);
      g.store(gs + o);
    }
  }
  float v0[VE], v1[VE];
  sb.get(v0);
  sw.get(v1);
  if (s.active) {
    put<VE>(red + first, v0);
    put<VE>(red + NT * VE + first, v1);
  }
  __syncthreads();
  column_sums<NT>(red, col, a);
  column_sums<NT>(red + NT * VE, col + cols, a);
  __syncthreads();
  const int S = max(1, a.segments);
  for (int i = threadIdx.x; i < 2 * s.cw; i += NT) {
    const int k = i >= s.cw ? 1 : 0, c = i - k * s.cw;
    float t = 0.f;
#pragma unroll 4
    for (int g = 0; g < S; ++g) t += col[k * cols + g * a.cw + c];
    own[k * maxcw + c] = t;
  }
  if (a.Q > 1) { __syncwarp(); cluster_arrive(); cluster_wait(); }
  else __syncthreads();
  for (int i = threadIdx.x; i < 2 * s.cw; i += NT) {
    const int k = i >= s.cw ? 1 : 0, c = i - k * s.cw;
    float pq[8], t = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) pq[q] = q < a.Q ? (a.Q > 1 ? ld_peer(own + k * maxcw + c, q) : own[k * maxcw + c]) : 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) t += pq[q];
    if (k) t *= a.rstd[s.n * a.G + s.ch * a.gpc + a.by_D.div((uint32_t)c)];            // (the sums of g xh were kept as those of g (x - mean))
    if (s.rank == 0 && a.part) a.part[((size_t)s.n * 2 + k) * a.C + s.c0 + c] = t;
    tot[k * maxcw + c] = t * param<T>(a.w, s.c0 + c, 1.f);
  }
  __syncthreads();
  if (a.Q > 1) cluster_arrive();
  if (a.y != nullptr) {                                          // (uniform)
    const float inv_total = 1.f / ((float)a.positions * (float)a.D);
    group_sums<NT>(tot, 1, 0, 2 * s.groups, a.D,
                   [&](int i, int& lo, int& hi) { lo = i < s.groups ? i * a.D : maxcw + (i - s.groups) * a.D; hi = lo + a.D; },
                   [&](int i, float t) { fin[i < s.groups ? i : a.gpc + i - s.groups] = t * inv_total; });
    __syncthreads();
    if (rows > 0) {
      Lanes<VE> n1, n2;
      float rs[VE];
      per_group<VE>(s.v * VE, a, [&](int g) { return a.rstd[s.n * a.G + s.ch * a.gpc + g]; }, rs);
      per_group<VE>(s.v * VE, a, [&](int g) { return -fin[g]; }, v0);
      per_group<VE>(s.v * VE, a, [&](int g) { return -fin[a.gpc + g]; }, v1);
#pragma unroll
      for (int j = 0; j < VE; ++j) { v0[j] *= rs[j]; v1[j] *= rs[j] * rs[j]; }
      n1.set(v0);
      n2.set(v1);
      T* dx = (T*)a.y + s.n * a.ys + (s.p0 + s.r) * a.yp + s.c0 + s.v * VE;
      int o = first;
      const long long ystep = a.R * a.yp;
#pragma unroll 2
      for (int i = 0; i < rows; ++i, o += step, dx += ystep) {
        Pack<T, VE> q;
        float f[VE];
        q.load(data + o);
        q.get(f);
        Lanes<VE> e, g;
        e.set(f);
        g.load(gs + o);
        dx_of(add(e, pt.nmu), g, pt.rw, n1, n2).get(f);
        q.set(f);
        q.store(dx);
      }
    }
  }
  __syncwarp();
  if (a.Q > 1) cluster_wait();
}

// ---- streaming form: a CTA takes a range of positions of a sample and a block of channels (all of them up to SNT vectors), reads it
// in a first kernel for the statistics and in a second one for the result, which starts with the samples that were read last.
// What bounds it is instructions (two conversions, five packed operations and SiLU's special functions per pair), not HBM: batches of
// samples that stay in L2 between the two kernels were no faster (64 x 64 x 64 x 320 bf16: 93.6 us in one go, 95 in halves, 113 in thirds).

constexpr int SNT = 256;                 // threads
// Rows a thread has under way, each in a slot of its own in shared memory (asynchronous copies: loads into registers that far ahead
// cost the registers, and the compiler waits for several of them at once: statistics of 64 x 64 x 64 x 320 bf16 51 us with
// four loads in a batch, 81 us with a register ring).
constexpr int AHEAD = 8, AHEAD2 = 6;     // one matrix; two
template <int N> __device__ __forceinline__ void cp_wait_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

struct Range {
  long long n;
  int part, e, c0, cw, r, v, g0, groups; // range, entry; channels; thread row and column; groups that the block touches
  uint32_t p0, p1;
  bool active;
};
template <int VE> __device__ __forceinline__ Range range_of(const GnArgs& a, uint32_t bx) {
  Range s;
  const uint32_t ln = a.by_parts.div(bx);
  s.n = ln;
  s.part = (int)(bx - ln * a.by_parts.d);
  s.e = s.part * (int)gridDim.y + (int)blockIdx.y;
  s.c0 = (int)blockIdx.y * a.cw;
  s.cw = min(a.cw, a.C - s.c0);
  s.r = (int)a.by_lv.div(threadIdx.x);
  s.v = (int)threadIdx.x - s.r * (int)a.by_lv.d;
  s.active = s.r < a.R && s.v * VE < s.cw;
  s.p0 = (uint32_t)s.part * (uint32_t)a.ppc;
  s.p1 = (uint32_t)min((long long)a.positions, (long long)s.p0 + a.ppc);
  s.g0 = (int)a.by_D.div((uint32_t)s.c0);
  s.groups = (int)a.by_D.div((uint32_t)(s.c0 + s.cw - 1)) - s.g0 + 1;
  return s;
}
// channels [lo, hi) of the block that belong to its group g
__device__ __forceinline__ void group_range(const GnArgs& a, const Range& s, int g, int& lo, int& hi) {
  lo = max(0, (s.g0 + g) * a.D - s.c0);
  hi = min(s.cw, (s.g0 + g + 1) * a.D - s.c0);
}
// entry[n][g][e] = (count, mean, squared deviations) of the block's part of group g
template <typename T, int VE>
__global__ void __launch_bounds__(SNT, 3) gn_stats_kernel(const GnArgs a) {
  extern __shared__ __align__(16) float red[];                   // [AHEAD][SNT] vectors, then [R][cw]
  __shared__ float col[SNT * VE], own[SNT * VE];                 // channel sums; means of the block's groups
  const Range s = range_of<VE>(a, blockIdx.x);
  T* slot = reinterpret_cast<T*>(red) + threadIdx.x * VE;
  grid_dependency_sync();
  Moments<VE> mo;
  if (s.active && s.p0 + s.r < s.p1) {
    const T* x = (const T*)a.x + s.n * a.xs + (long long)(s.p0 + s.r) * a.xp + s.c0 + s.v * VE;
    const long long step = a.R * a.xp;
    const int rows = (int)a.by_R.div(s.p1 - s.p0 - s.r + a.R - 1);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u, x += step) {
      if (u < rows) copy_in<T, VE>(slot + u * SNT * VE, x);
      cp_commit();
    }
    for (int i = 0; i < rows; i += AHEAD) {                      // (32 is a multiple of AHEAD)
#pragma unroll
      for (int u = 0; u < AHEAD; ++u, x += step)
        if (i + u < rows) {
          cp_wait_but<AHEAD - 1>();
          Pack<T, VE> q;
          q.load(slot + u * SNT * VE);
          if (u == 0 && (i & 31) == 0) {
            if (i > 0) mo.end(32.f);
            mo.begin(q);
          }
          mo.row(q);
          if (i + u + AHEAD < rows) copy_in<T, VE>(slot + u * SNT * VE, x);
          cp_commit();
        }
    }
    mo.end((float)(rows - ((rows - 1) & ~31)));
  }
  float* at = red + s.r * a.cw + s.v * VE;
  float out[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) out[j] = mo.mean[j] * mo.seen;
  __syncthreads();                                               // (everybody has left the rows' slots)
  if (s.active) put<VE>(at, out);
  __syncthreads();
  const float np = (float)(s.p1 - s.p0);
  const int E = a.parts * (int)gridDim.y;
  float* entry = a.stat + ((size_t)s.n * a.G + s.g0) * E * 3 + (size_t)s.e * 3;
  const int S = max(1, a.segments);
  auto range = [&](int g, int& lo, int& hi) { group_range(a, s, g, lo, hi); };
  column_sums<SNT>(red, col, a);
  __syncthreads();
  group_sums<SNT>(col, S, a.cw, s.groups, a.D, range, [&](int g, float t) {
    int lo, hi;
    group_range(a, s, g, lo, hi);
    const float cnt = np * (float)(hi - lo), m = t / cnt;
    entry[(size_t)g * E * 3] = cnt;
    entry[(size_t)g * E * 3 + 1] = own[g] = m;
  });
  __syncthreads();
  if (s.active) {
    float mu[VE];
    per_group<VE>(s.c0 + s.v * VE, a, [&](int g) { return own[g - s.g0]; }, mu);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float e = mo.mean[j] - mu[j];
      out[j] = mo.seen > 0.f ? fmaf(e * e, mo.seen, mo.dev[j]) : 0.f;      // (a thread without rows: no 0 times infinity)
    }
    put<VE>(at, out);
  }
  __syncthreads();
  column_sums<SNT>(red, col, a);
  __syncthreads();
  group_sums<SNT>(col, S, a.cw, s.groups, a.D, range, [&](int g, float t) { entry[(size_t)g * E * 3 + 2] = t; });
}

// entries of a group that other blocks than this one hold are zero
__global__ void __launch_bounds__(256) gn_clear_kernel(float* p, size_t n) {
  grid_dependency_sync();
  for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < n; i += gridDim.x * 256ull) p[i] = 0.f;
}

template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(SNT, 3) gn_apply_kernel(const GnArgs a) {
  extern __shared__ __align__(16) float ring[];                  // [AHEAD][SNT] vectors
  const Range s = range_of<VE>(a, gridDim.x - 1 - blockIdx.x);
  T* slot = reinterpret_cast<T*>(ring) + threadIdx.x * VE;
  float* fin = reinterpret_cast<float*>(reinterpret_cast<T*>(ring) + AHEAD * SNT * VE);     // [2][groups of the block] mean, 1 / standard deviation
  const int sub = threadIdx.x & 7;
  grid_dependency_sync();
  const int E = a.parts * (int)gridDim.y;
  const float inv_total = 1.f / ((float)a.positions * (float)a.D);
  for (int g0 = threadIdx.x >> 5 << 2; g0 < s.groups; g0 += SNT / 8) {       // eight lanes to a group
    const int g = g0 + ((threadIdx.x & 31) >> 3);
    const float* entry = a.stat + ((size_t)s.n * a.G + s.g0 + g) * E * 3;
    const int n = g < s.groups ? E : 0;
    const int first = n > 0 ? s.e % (int)gridDim.y : 0;          // (an entry of this block: its range may be empty elsewhere)
    const float m0 = n > 0 ? entry[3 * first + 1] : 0.f;
    float m = 0.f, v = 0.f;
    for (int e = sub; e < n; e += 8) m = fmaf(entry[3 * e] * inv_total, entry[3 * e + 1] - m0, m);
    m = eight_sum(m) + m0;                                       // (relative to one of them: equal means stay what they are)
    for (int e = sub; e < n; e += 8) {
      const float d = entry[3 * e + 1] - m;
      v += fmaf(entry[3 * e] * d, d, entry[3 * e + 2]);
    }
    v = eight_sum(v);
    const float rstd = 1.f / sqrtf(fmaf(v, inv_total, a.eps));
    if (sub == 0 && g < s.groups) {
      fin[g] = m;
      fin[s.groups + g] = rstd;
      if (a.mean && s.part == 0 && (s.g0 + g) * a.D >= s.c0) {
        a.mean[s.n * a.G + s.g0 + g] = m;
        a.rstd[s.n * a.G + s.g0 + g] = rstd;
      }
    }
  }
  __syncthreads();
  if (!s.active || s.p0 + s.r >= s.p1) return;
  const int c = s.c0 + s.v * VE;
  Lanes<VE> nmu, sc, sh;
  float f0[VE], f1[VE], f2[VE];
  params<T, VE>(a.w, c, 1.f, f2);
  per_group<VE>(c, a, [&](int g) { return fin[g - s.g0]; }, f0);
  per_group<VE>(c, a, [&](int g) { return fin[s.groups + g - s.g0]; }, f1);
#pragma unroll
  for (int j = 0; j < VE; ++j) { f0[j] = -f0[j]; f1[j] *= f2[j]; }
  params<T, VE>(a.b, c, 0.f, f2);
  nmu.set(f0);
  sc.set(f1); sh.set(f2);
  const T* x = (const T*)a.x + s.n * a.xs + (long long)(s.p0 + s.r) * a.xp + c;
  T* y = (T*)a.y + s.n * a.ys + (long long)(s.p0 + s.r) * a.yp + c;
  const long long xstep = a.R * a.xp, ystep = a.R * a.yp;
  const int rows = (int)a.by_R.div(s.p1 - s.p0 - s.r + a.R - 1);
#pragma unroll
  for (int u = 0; u < AHEAD; ++u, x += xstep) {
    if (u < rows) copy_in<T, VE>(slot + u * SNT * VE, x);
    cp_commit();
  }
  for (int i = 0; i < rows; i += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u, x += xstep, y += ystep)
      if (i + u < rows) {
        cp_wait_but<AHEAD - 1>();
        Pack<T, VE> q;
        float f[VE];
        q.load(slot + u * SNT * VE);
        q.get(f);
        Lanes<VE> l;
        l.set(f);
        act_values<ACT>(fma(add(l, nmu), sc, sh)).get(f);
        if (i + u + AHEAD < rows) copy_in<T, VE>(slot + u * SNT * VE, x);
        cp_commit();
        q.set(f);
        q.store(y);
      }
  }
}

// part[n][range][0 | 1][c]: sums of g and g xh over the range; entry[n][g][e]: those times w, over the block's part of the group
template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(SNT, 3) gn_sums_kernel(const GnArgs a) {
  extern __shared__ __align__(16) float red[];                   // [R][cw], [2][cw], [segments][cw]
  const Range s = range_of<VE>(a, blockIdx.x);
  float* tot = red + SNT * VE;
  float* col = tot + 2 * a.cw;
  T* slot = reinterpret_cast<T*>(col + round_up(max(SNT, a.cw) + 2 * a.cw, 4) - 2 * a.cw) + threadIdx.x * VE;     // [AHEAD2][2][SNT] vectors
  grid_dependency_sync();
  Lanes<VE> sb, sw;
  sb.fill(0.f);
  sw.fill(0.f);
  const int c = s.c0 + s.v * VE;
  if (s.active && s.p0 + s.r < s.p1) {
    Point<T, VE, ACT> pt;
    pt.init(a, s.n, c, true);
    const T* x = (const T*)a.x + s.n * a.xs + (long long)(s.p0 + s.r) * a.xp + c;
    const T* dy = (const T*)a.dy + s.n * a.ds + (long long)(s.p0 + s.r) * a.dp + c;
    const long long xstep = a.R * a.xp, dstep = a.R * a.dp;
    const int rows = (int)a.by_R.div(s.p1 - s.p0 - s.r + a.R - 1);
#pragma unroll
    for (int u = 0; u < AHEAD2; ++u, x += xstep, dy += dstep) {
      if (u < rows) { copy_in<T, VE>(slot + 2 * u * SNT * VE, x); copy_in<T, VE>(slot + (2 * u + 1) * SNT * VE, dy); }
      cp_commit();
    }
    for (int i = 0; i < rows; i += AHEAD2) {
#pragma unroll
      for (int u = 0; u < AHEAD2; ++u, x += xstep, dy += dstep)
        if (i + u < rows) {
          cp_wait_but<AHEAD2 - 1>();
          Pack<T, VE> q, d;
          q.load(slot + 2 * u * SNT * VE);
          d.load(slot + (2 * u + 1) * SNT * VE);
          Lanes<VE> e, g;
          pt.at(a, s.n, c, q, d, e, g);
          if (i + u + AHEAD2 < rows) { copy_in<T, VE>(slot + 2 * u * SNT * VE, x); copy_in<T, VE>(slot + (2 * u + 1) * SNT * VE, dy); }
          cp_commit();
          sb = add(sb, g);
          sw = fma(g, e, sw);
        }
    }
  }
  const int E = a.parts * (int)gridDim.y;
  const long long row = s.n * a.parts + s.part;
  const int S = max(1, a.segments);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float v[VE];
    if (k) sw.get(v); else sb.get(v);
    if (s.active) put<VE>(red + s.r * a.cw + s.v * VE, v);
    __syncthreads();
    column_sums<SNT>(red, col, a);
    __syncthreads();
    for (int i = threadIdx.x; i < s.cw; i += SNT) {
      float t = 0.f;
#pragma unroll 4
      for (int g = 0; g < S; ++g) t += col[g * a.cw + i];
      if (k) t *= a.rstd[s.n * a.G + a.by_D.div((uint32_t)(s.c0 + i))];        // (kept as the sums of g (x - mean))
      a.part[((size_t)row * 2 + k) * a.C + s.c0 + i] = t;
      tot[k * a.cw + i] = t * param<T>(a.w, s.c0 + i, 1.f);
    }
    __syncthreads();
  }
  if (a.y == nullptr) return;
  group_sums<SNT>(tot, 1, 0, 2 * s.groups, a.D,
                  [&](int i, int& lo, int& hi) {
                    const int k = i >= s.groups ? 1 : 0;
                    group_range(a, s, i - k * s.groups, lo, hi);
                    lo += k * a.cw;
                    hi += k * a.cw;
                  },
                  [&](int i, float t) {
                    const int k = i >= s.groups ? 1 : 0;
                    a.stat[(((size_t)s.n * a.G + s.g0 + i - k * s.groups) * E + s.e) * 2 + k] = t;
                  });
}

template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(SNT, 3) gn_dx_kernel(const GnArgs a) {
  extern __shared__ __align__(16) float ring[];                  // [AHEAD2][2][SNT] vectors
  const Range s = range_of<VE>(a, gridDim.x - 1 - blockIdx.x);
  T* slot = reinterpret_cast<T*>(ring) + threadIdx.x * VE;
  float* fin = reinterpret_cast<float*>(reinterpret_cast<T*>(ring) + AHEAD2 * 2 * SNT * VE);     // [2][groups of the block] the two group means
  const int sub = threadIdx.x & 7;
  grid_dependency_sync();
  const int E = a.parts * (int)gridDim.y;
  const float inv_total = 1.f / ((float)a.positions * (float)a.D);
  for (int g0 = threadIdx.x >> 5 << 2; g0 < s.groups; g0 += SNT / 8) {       // eight lanes to a group
    const int g = g0 + ((threadIdx.x & 31) >> 3);
    const float* entry = a.stat + ((size_t)s.n * a.G + s.g0 + g) * E * 2;
    const int n = g < s.groups ? E : 0;
    float t0 = 0.f, t1 = 0.f;
    for (int e = sub; e < n; e += 8) { t0 += entry[2 * e]; t1 += entry[2 * e + 1]; }
    t0 = eight_sum(t0);
    t1 = eight_sum(t1);
    if (sub == 0 && g < s.groups) { fin[g] = t0 * inv_total; fin[s.groups + g] = t1 * inv_total; }
  }
  __syncthreads();
  if (!s.active || s.p0 + s.r >= s.p1) return;
  const int c = s.c0 + s.v * VE;
  Point<T, VE, ACT> pt;
  pt.init(a, s.n, c, true);
  Lanes<VE> n1, n2;
  float v0[VE], v1[VE], rs[VE];
  per_group<VE>(c, a, [&](int g) { return a.rstd[s.n * a.G + g]; }, rs);
  per_group<VE>(c, a, [&](int g) { return -fin[g - s.g0]; }, v0);
  per_group<VE>(c, a, [&](int g) { return -fin[s.groups + g - s.g0]; }, v1);
#pragma unroll
  for (int j = 0; j < VE; ++j) { v0[j] *= rs[j]; v1[j] *= rs[j] * rs[j]; }
  n1.set(v0);
  n2.set(v1);
  const T* x = (const T*)a.x + s.n * a.xs + (long long)(s.p0 + s.r) * a.xp + c;
  const T* dy = (const T*)a.dy + s.n * a.ds + (long long)(s.p0 + s.r) * a.dp + c;
  T* dx = (T*)a.y + s.n * a.ys + (long long)(s.p0 + s.r) * a.yp + c;
  const long long xstep = a.R * a.xp, dstep = a.R * a.dp, ystep = a.R * a.yp;
  const int rows = (int)a.by_R.div(s.p1 - s.p0 - s.r + a.R - 1);
#pragma unroll
  for (int u = 0; u < AHEAD2; ++u, x += xstep, dy += dstep) {
    if (u < rows) { copy_in<T, VE>(slot + 2 * u * SNT * VE, x); copy_in<T, VE>(slot + (2 * u + 1) * SNT * VE, dy); }
    cp_commit();
  }
  for (int i = 0; i < rows; i += AHEAD2) {
#pragma unroll
    for (int u = 0; u < AHEAD2; ++u, x += xstep, dy += dstep, dx += ystep)
      if (i + u < rows) {
        cp_wait_but<AHEAD2 - 1>();
        Pack<T, VE> q, d;
        q.load(slot + 2 * u * SNT * VE);
        d.load(slot + (2 * u + 1) * SNT * VE);
        Lanes<VE> e, g;
        pt.at(a, s.n, c, q, d, e, g);
        if (i + u + AHEAD2 < rows) { copy_in<T, VE>(slot + 2 * u * SNT * VE, x); copy_in<T, VE>(slot + (2 * u + 1) * SNT * VE, dy); }
        cp_commit();
        float f[VE];
        dx_of(e, g, pt.rw, n1, n2).get(f);
        q.set(f);
        q.store(dx);
      }
  }
}

// out[s][0 | 1][c] = sum of rows s per, ... of part[rows][2][C]; the last stage writes db and dw: block = 32 columns x 32 rows of threads
template <typename T>
__global__ void __launch_bounds__(1024) gn_param_kernel(const float* part, long long rows, long long per, int C, float* out, void* dw, void* db) {
  __shared__ float red[32][33];
  grid_dependency_sync();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long j = (long long)blockIdx.x * 32 + lane, width = 2ll * C;
  const long long r1 = min(rows, (long long)(blockIdx.y + 1) * per);
  float t = 0.f;
  if (j < width) {
#pragma unroll 8
    for (long long r = blockIdx.y * per + w; r < r1; r += 32) t += part[r * width + j];
  }
  red[w][lane] = t;
  __syncthreads();
  const float v = warp_sum(red[lane][w]);                        // (column w of the block)
  const long long c = (long long)blockIdx.x * 32 + w;
  if (lane == 0 && c < width) {
    if (out) out[blockIdx.y * width + c] = v;
    else if (c < C) { if (db) stf((T*)db, c, v); }
    else if (dw) stf((T*)dw, c - C, v);
  }
}

typedef void (*GnFn)(const GnArgs);
#define GN_ACT(type, name, T, VE, act)                                                                              \
  ((act) == ABS_ACT_RELU ? (type)name<T, VE, ABS_ACT_RELU> : (act) == ABS_ACT_GELU ? (type)name<T, VE, ABS_ACT_GELU> \
   : (act) == ABS_ACT_SILU ? (type)name<T, VE, ABS_ACT_SILU> : (type)name<T, VE, ABS_ACT_NONE>)
#define GN_PICK(type, name, dtype, vec, act)                                                                        \
  ((dtype) == ABS_FP32 ? ((vec) ? GN_ACT(type, name, float, 4, act) : GN_ACT(type, name, float, 1, act))            \
                       : ((vec) ? GN_ACT(type, name, __nv_bfloat16, 8, act) : GN_ACT(type, name, __nv_bfloat16, 1, act)))

constexpr double RESIDENT_BYTES = 12e6;
constexpr size_t CTA_BYTES = 110 * 1024, MOST_BYTES = 200 * 1024, STREAM_BYTES = 112 * 1024;

// How a call is cut up; `vec`: 16-byte accesses.  The scratch of a call is the larger of the two forms'.
struct Plan {
  bool resident;
  int gpc, chunks, Q, ppc;               // resident form
  size_t smem;
  int cw, blocks, R, parts, sppc;        // streaming form
};
size_t smem_bytes(int gpc, int D, long long ppc, int VE, size_t esz, bool grad) {
  const size_t cw = (size_t)gpc * D;
  const size_t head = round_up_sz((grad ? 2 * (size_t)NT * VE + 2 * (cw > NT ? cw : NT) + 4 * cw + 2 * gpc : (size_t)NT * VE + (cw > NT ? cw : NT) + 4 * (size_t)gpc) * 4, 16);
  return head + round_up_sz((size_t)ppc * cw, 16) * (grad ? 4 + esz : esz);
}
Plan plan(long long samples, long long positions, int C, int G, int dtype, bool grad, bool vec) {
  Plan p = {};
  const int D = C / G;
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  const int VE = vec && (size_t)C * esz % 16 == 0 ? (int)(16 / esz) : 1;      // (a position of fewer channels, or a part more, has no whole vectors)
  int unit = 1;                          // groups that make whole vectors
  while ((long long)unit * D % VE) ++unit;
  const double sample_bytes = (double)positions * C * esz * (grad ? 2 : 1);
  // resident: chunks of whole groups and whole vectors, with 128 bytes of channels, else with 64, else the smallest there are;
  // one that leaves room for two CTAs per SM is sought first, then any that fits
  if (samples * sample_bytes <= RESIDENT_BYTES)
    for (size_t most : {CTA_BYTES, MOST_BYTES})
      for (size_t least : {(size_t)128, (size_t)64, (size_t)1}) {
        int gpc = unit;
        while (gpc < G && (size_t)gpc * D * esz < least) gpc += unit;
        if (gpc > G) gpc = G;
        if ((long long)gpc * D / VE > NT) continue;
        const long long chunks = (G + gpc - 1) / gpc;
        long long best = 0;
        for (long long q = 1; q <= 8; ++q) {
          const long long ppc = (positions + q - 1) / q;
          if ((q - 1) * ppc >= positions) break;                 // (the last CTA would have nothing)
          if (ppc >= (1 << 24) || smem_bytes(gpc, D, ppc, VE, esz, grad) > most) continue;
          best = q;
          if (samples * chunks * q >= PLAN_SMS || (size_t)ppc * gpc * D * esz <= 8192) break;    // enough CTAs, or too little for each
        }
        if (best == 0 || samples * chunks * best > 0x7fffffff) continue;
        p.resident = true;
        p.gpc = gpc; p.chunks = (int)chunks; p.Q = (int)best; p.ppc = (int)((positions + best - 1) / best);
        p.smem = smem_bytes(gpc, D, p.ppc, VE, esz, grad);
        return p;
      }
  // streaming: blocks of whole groups if a group fits
  const long long width = (long long)unit * D, most = (long long)SNT * VE;
  p.cw = C <= most ? C : (int)(width <= most ? most / width * width : most);
  p.blocks = (C + p.cw - 1) / p.cw;
  p.R = SNT / (p.cw / VE);
  // ranges of positions: as many as keep the waves of CTAs (three per SM) short, a CTA costing about as much as 12 rows
  // besides its own
  const long long units = samples * p.blocks, slots = 3 * PLAN_SMS;
  const long long most_parts = std::min({(positions + 8 * p.R - 1) / (8 * p.R), 4096ll, 12 * PLAN_SMS / units + 1});
  long long parts = 1;
  double least = 1e300;
  // among the numbers of ranges with as many waves the largest has the fewest rows; the smallest with as few rows is as good
  for (long long waves = (units + slots - 1) / slots, last = 0; last < most_parts; ++waves) {
    const long long n = std::min(most_parts, waves * slots / units);
    if (n == last) continue;                                     // (a wave too many for the units, and too few for another range)
    const long long rows = ((positions + n - 1) / n + p.R - 1) / p.R, few = (positions + rows * p.R - 1) / (rows * p.R);
    const double cost = (double)waves * (double)(rows + 12);
    if (cost < least) { least = cost; parts = std::max(few, last + 1); }
    last = n;
  }
  p.sppc = (int)((positions + parts - 1) / parts);
  p.parts = (int)((positions + p.sppc - 1) / p.sppc);
  return p;
}

constexpr int PARAM_SPLIT = 64;          // rows of the first stage of the parameter sums when there are more than PARAM_ROWS
constexpr long long PARAM_ROWS = 1024;
// floats of scratch: [entries][channel sums of all samples][first stage of the parameter sums]
size_t entry_floats(const Plan& p, long long samples, int G, bool grad) {
  return p.resident ? 0 : round_up_sz((size_t)samples * G * p.parts * p.blocks * (grad ? 2 : 3), 64);
}
size_t scratch_floats(const Plan& p, long long samples, int C, int G, bool grad) {
  if (!grad) return entry_floats(p, samples, G, grad);
  const long long rows = p.resident ? samples : samples * p.parts;
  return entry_floats(p, samples, G, grad) + (size_t)rows * 2 * C + (rows > PARAM_ROWS ? (size_t)PARAM_SPLIT * 2 * C : 0);
}

cudaError_t run_params(const GnArgs& a, long long rows, int dtype, float* second, cudaStream_t s) {
  auto* kernel = dtype == ABS_FP32 ? gn_param_kernel<float> : gn_param_kernel<__nv_bfloat16>;
  const unsigned cols = (unsigned)((2ll * a.C + 31) / 32);
  const float* from = a.part;
  cudaError_t e = cudaSuccess;
  if (rows > PARAM_ROWS) {
    const long long per = (rows + PARAM_SPLIT - 1) / PARAM_SPLIT;
    e = launch(kernel, dim3(cols, PARAM_SPLIT), 1024, 0, 1, s, from, rows, per, a.C, second, (void*)nullptr, (void*)nullptr);
    from = second;
    rows = PARAM_SPLIT;
  }
  if (e == cudaSuccess) e = launch(kernel, dim3(cols), 1024, 0, 1, s, from, rows, rows, a.C, (float*)nullptr, a.dw, a.db);
  return e;
}

GnFn stats_fn(int dtype, bool vec) {
  return dtype == ABS_FP32 ? (vec ? (GnFn)gn_stats_kernel<float, 4> : (GnFn)gn_stats_kernel<float, 1>)
                           : (vec ? (GnFn)gn_stats_kernel<__nv_bfloat16, 8> : (GnFn)gn_stats_kernel<__nv_bfloat16, 1>);
}
// The kernels' shared memory is raised to the most any plan asks for, once per device.
cudaError_t raise_smem() {
  static std::atomic<uint64_t> ready;
  int device, sms;
  if (current_device(&device, &sms) != ABS_OK) return cudaErrorInvalidDevice;
  if (ready.load(std::memory_order_acquire) >> device & 1) return cudaSuccess;
  for (int dtype = 0; dtype < 2; ++dtype)
    for (int vec = 0; vec < 2; ++vec) {
      cudaError_t e = allow_smem(stats_fn(dtype, vec), STREAM_BYTES);
      for (int act = ABS_ACT_NONE; act <= ABS_ACT_SILU && e == cudaSuccess; ++act) {
        e = allow_smem(GN_PICK(GnFn, gn_forward_kernel, dtype, vec, act), MOST_BYTES);
        if (e == cudaSuccess) e = allow_smem(GN_PICK(GnFn, gn_backward_kernel, dtype, vec, act), MOST_BYTES);
        if (e == cudaSuccess) e = allow_smem(GN_PICK(GnFn, gn_apply_kernel, dtype, vec, act), STREAM_BYTES);
        if (e == cudaSuccess) e = allow_smem(GN_PICK(GnFn, gn_sums_kernel, dtype, vec, act), STREAM_BYTES);
        if (e == cudaSuccess) e = allow_smem(GN_PICK(GnFn, gn_dx_kernel, dtype, vec, act), STREAM_BYTES);
      }
      if (e != cudaSuccess) return e;
    }
  ready.fetch_or(1ull << device, std::memory_order_release);
  return cudaSuccess;
}

cudaError_t launch_resident(GnFn fn, const Plan& p, long long samples, int VE, cudaStream_t s, const GnArgs& a) {
  const cudaError_t ready = raise_smem();
  if (ready != cudaSuccess) return ready;
  GnArgs b = a;
  b.by_Q = Divisor((uint32_t)p.Q);
  b.by_chunks = Divisor((uint32_t)p.chunks);
  b.cw = p.gpc * a.D;
  b.R = NT / (b.cw / VE);
  b.last = (int)((long long)a.positions - (long long)(p.Q - 1) * p.ppc);
  b.segments = NT / b.cw;
  b.by_lv = Divisor((uint32_t)(b.cw / VE));
  b.by_R = Divisor((uint32_t)b.R);
  b.by_cw = Divisor((uint32_t)b.cw);
  return launch(fn, dim3((unsigned)(samples * p.chunks * p.Q)), NT, p.smem, p.Q, s, b);
}

// The first kernel's statistics, the second kernel's results.
struct StreamFns { GnFn first, second; };
cudaError_t launch_streaming(const StreamFns& f, const Plan& p, long long samples, int VE, size_t esz, bool grad, cudaStream_t s, const GnArgs& call) {
  const cudaError_t ready = raise_smem();
  if (ready != cudaSuccess) return ready;
  GnArgs a = call;
  a.cw = p.cw; a.R = p.R; a.parts = p.parts; a.ppc = p.sppc;
  a.by_parts = Divisor((uint32_t)p.parts);
  a.by_lv = Divisor((uint32_t)(p.cw / VE));
  a.by_R = Divisor((uint32_t)p.R);
  a.by_cw = Divisor((uint32_t)p.cw);
  a.segments = SNT / p.cw;
  const size_t vec_bytes = (size_t)VE * esz * SNT, wide = (size_t)(p.cw > SNT ? p.cw : SNT) + 2 * (size_t)p.cw;
  const size_t sums = grad ? ((size_t)SNT * VE + round_up_sz(wide, 4)) * 4 + AHEAD2 * 2 * vec_bytes : AHEAD * vec_bytes;            // (the sums of four bytes per element fit into the slots)
  const size_t two = (grad ? AHEAD2 * 2 : AHEAD) * vec_bytes + 2 * ((size_t)(p.cw + a.D - 1) / a.D + 1) * 4;     // (groups that a block touches)
  const dim3 grid((unsigned)(samples * p.parts), (unsigned)p.blocks);
  cudaError_t e = cudaSuccess;
  if (p.blocks > 1) {
    const size_t n = (size_t)samples * a.G * p.parts * p.blocks * (grad ? 2 : 3);
    e = launch(gn_clear_kernel, dim3((unsigned)((n + 255) / 256 < 1024 ? (n + 255) / 256 : 1024)), 256, 0, 1, s, a.stat, n);
  }
  if (e == cudaSuccess) e = launch(f.first, grid, SNT, sums, 1, s, a);
  if (e == cudaSuccess && f.second) e = launch(f.second, grid, SNT, two, 1, s, a);
  return e;
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

// maps [samples][positions][C] with pitches s, p
int check_maps(const char* name, const void* ptr, long long s, long long p, long long samples, long long positions, int C, size_t esz) {
  if (!ptr) return fail(ABS_EINVAL, "%s is null", name);
  if ((uintptr_t)ptr % esz) return fail(ABS_EINVAL, "%s is not aligned to its type", name);
  if (positions > 1 && p < C) return fail(ABS_EINVAL, "%s: position pitch %lld below the %d channels", name, p, C);
  if (samples > 1 && s < (positions - 1) * (positions > 1 ? p : 0) + C) return fail(ABS_EINVAL, "%s: samples overlap (pitch %lld)", name, s);
  return ABS_OK;
}

Span flat(const void* ptr, long long bytes) { return Span{(uintptr_t)ptr, (uintptr_t)ptr + (ptr ? (uintptr_t)bytes : 0), 0, 0}; }
Span maps_span(const void* ptr, long long s, long long p, long long samples, long long positions, int C, size_t esz) {
  Span r = {(uintptr_t)ptr, (uintptr_t)ptr, (long long)(p * (long long)esz), (long long)(C * (long long)esz)};
  if (ptr && samples > 0) r.hi += (uintptr_t)(((samples - 1) * s + (positions - 1) * p + C) * (long long)esz);
  if (samples > 1 && s % (p > 0 ? p : 1)) r.ld = 0;      // (rows of different samples are not a multiple of the pitch apart)
  return r;
}

// Two maps of one shape share a byte.  With equal pitches they do not if each position of the one lies in the gap behind (in front of) that of the
// other, as channel ranges of one buffer do.
struct Maps { const void* p; long long s, i; Span span; };        // pitches of samples and positions
bool maps_overlap(const Maps& a, const Maps& b, long long samples, long long positions, int C, size_t esz) {
  if (!overlap(a.span, b.span)) return false;
  if ((samples > 1 && a.s != b.s) || (positions > 1 && a.i != b.i)) return true;
  const unsigned long long row = C * (unsigned long long)esz, pitch = a.i * (unsigned long long)esz, sample = a.s * (unsigned long long)esz;
  const unsigned long long d = (uintptr_t)a.p < (uintptr_t)b.p ? (uintptr_t)b.p - (uintptr_t)a.p : (uintptr_t)a.p - (uintptr_t)b.p;
  return d < row || (positions > 1 && d + row > pitch) || (samples > 1 && (positions - 1) * pitch + d + row > sample);
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
  if ((rc = check_vector("w", w, esz)) != ABS_OK || (rc = check_vector("b", b, esz)) != ABS_OK) return rc;
  if ((rc = check_vector("mean", mean, 4)) != ABS_OK || (rc = check_vector("rstd", rstd, 4)) != ABS_OK) return rc;
  const Span sx = maps_span(x, xs, xp, samples, positions, channels, esz), sy = maps_span(y, ys, yp, samples, positions, channels, esz);
  const Span sw = flat(w, channels * esz), sb = flat(b, channels * esz), sm = flat(mean, samples * groups * 4), sr = flat(rstd, samples * groups * 4);
  if (!(x == y && (samples == 1 || xs == ys) && (positions == 1 || xp == yp)) && maps_overlap({x, xs, xp, sx}, {y, ys, yp, sy}, samples, positions, channels, esz)) return fail(ABS_EINVAL, "y overlaps x without being the same maps");
  if (overlap(sy, sw) || overlap(sy, sb)) return fail(ABS_EINVAL, "y overlaps w or b");
  if (overlap(sm, sr)) return fail(ABS_EINVAL, "mean overlaps rstd");
  for (const Span& st : {sm, sr})
    if (overlap(st, sx) || overlap(st, sy) || overlap(st, sw) || overlap(st, sb)) return fail(ABS_EINVAL, "mean or rstd overlaps another argument");
  GnArgs a = {};
  a.x = x; a.y = y; a.w = w; a.b = b; a.mean = mean; a.rstd = rstd;
  a.xs = xs; a.xp = xp; a.ys = ys; a.yp = yp;
  a.samples = samples; a.positions = (uint32_t)positions;
  a.C = channels; a.G = groups; a.D = channels / groups; a.eps = eps;
  a.by_D = Divisor((uint32_t)a.D);
  const bool vec = (size_t)channels * esz % 16 == 0 && on16(x) && on16(y) && pitch16(samples, positions, xs, xp, esz) && pitch16(samples, positions, ys, yp, esz);
  const Plan p = plan(samples, positions, channels, groups, dtype, false, vec);
  if ((rc = check_scratch(scratch, scratch_bytes, scratch_floats(p, samples, channels, groups, false) * 4, {sx, sy, sw, sb, sm, sr})) != ABS_OK) return rc;
  a.gpc = p.gpc; a.chunks = p.chunks; a.Q = p.Q; a.ppc = p.ppc;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e;
  if (p.resident) {
    e = launch_resident(GN_PICK(GnFn, gn_forward_kernel, dtype, vec, act), p, samples, vec ? (int)(16 / esz) : 1, s, a);
  } else {
    a.stat = (float*)scratch;
    const StreamFns fns = {stats_fn(dtype, vec), GN_PICK(GnFn, gn_apply_kernel, dtype, vec, act)};
    e = launch_streaming(fns, p, samples, vec ? (int)(16 / esz) : 1, esz, false, s, a);
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
    if ((rc = check_vector("dw", dw, esz)) != ABS_OK || (rc = check_vector("db", db, esz)) != ABS_OK) return rc;
    if (dw) e = cudaMemsetAsync(dw, 0, channels * esz, (cudaStream_t)stream);
    if (db && e == cudaSuccess) e = cudaMemsetAsync(db, 0, channels * esz, (cudaStream_t)stream);
    return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "memset: %s", cudaGetErrorString(e));
  }
  if (!mean || !rstd) return fail(ABS_EINVAL, "mean and rstd of the forward pass are needed");
  if ((rc = check_vector("dw", dw, esz)) != ABS_OK || (rc = check_vector("db", db, esz)) != ABS_OK) return rc;
  if ((rc = check_maps("dy", dy, dys, dyp, samples, positions, channels, esz)) != ABS_OK) return rc;
  if ((rc = check_maps("x", x, xs, xp, samples, positions, channels, esz)) != ABS_OK) return rc;
  if (dx && (rc = check_maps("dx", dx, dxs, dxp, samples, positions, channels, esz)) != ABS_OK) return rc;
  if ((rc = check_vector("w", w, esz)) != ABS_OK || (rc = check_vector("b", b, esz)) != ABS_OK) return rc;
  if ((rc = check_vector("mean", mean, 4)) != ABS_OK || (rc = check_vector("rstd", rstd, 4)) != ABS_OK) return rc;
  const Span sx = maps_span(x, xs, xp, samples, positions, channels, esz), sg = maps_span(dy, dys, dyp, samples, positions, channels, esz);
  const Span sd = maps_span(dx, dxs, dxp, dx ? samples : 0, positions, channels, esz), s1 = flat(dw, channels * esz), s2 = flat(db, channels * esz);
  const Span fixed[4] = {flat(w, channels * esz), flat(b, channels * esz), flat(mean, samples * groups * 4), flat(rstd, samples * groups * 4)};
  const Maps mx = {x, xs, xp, sx}, mg = {dy, dys, dyp, sg}, md = {dx, dxs, dxp, sd};
  if (maps_overlap(md, mx, samples, positions, channels, esz)) return fail(ABS_EINVAL, "dx overlaps x");
  if (!(dx == dy && (samples == 1 || dxs == dys) && (positions == 1 || dxp == dyp)) && maps_overlap(md, mg, samples, positions, channels, esz))
    return fail(ABS_EINVAL, "dx overlaps dy without being the same maps");
  if (overlap(s1, s2) || overlap(s1, sd) || overlap(s2, sd)) return fail(ABS_EINVAL, "two gradients overlap");
  for (const Span& o : {sd, s1, s2})
    for (const Span& f : fixed)
      if (overlap(o, f)) return fail(ABS_EINVAL, "a gradient overlaps an operand");
  if (overlap(s1, sx) || overlap(s1, sg) || overlap(s2, sx) || overlap(s2, sg)) return fail(ABS_EINVAL, "a gradient overlaps an operand");
  GnArgs a = {};
  a.x = x; a.dy = dy; a.y = dx; a.w = w; a.b = b; a.dw = dw; a.db = db;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.xs = xs; a.xp = xp; a.ys = dxs; a.yp = dxp; a.ds = dys; a.dp = dyp;
  a.samples = samples; a.positions = (uint32_t)positions;
  a.C = channels; a.G = groups; a.D = channels / groups;
  a.by_D = Divisor((uint32_t)a.D);
  const bool vec = (size_t)channels * esz % 16 == 0 && on16(x) && on16(dy) && on16(dx) && pitch16(samples, positions, xs, xp, esz) &&
                   pitch16(samples, positions, dys, dyp, esz) && (!dx || pitch16(samples, positions, dxs, dxp, esz));
  const Plan p = plan(samples, positions, channels, groups, dtype, true, vec);
  if (!dx && !dw && !db) return ABS_OK;
  if ((rc = check_scratch(scratch, scratch_bytes, scratch_floats(p, samples, channels, groups, true) * 4,
                          {sx, sg, sd, s1, s2, fixed[0], fixed[1], fixed[2], fixed[3]})) != ABS_OK) return rc;
  a.gpc = p.gpc; a.chunks = p.chunks; a.Q = p.Q; a.ppc = p.ppc;
  cudaStream_t s = (cudaStream_t)stream;
  const long long rows = p.resident ? samples : samples * p.parts;
  if (p.resident) {
    a.part = dw || db ? (float*)scratch : nullptr;
    e = launch_resident(GN_PICK(GnFn, gn_backward_kernel, dtype, vec, act), p, samples, vec ? (int)(16 / esz) : 1, s, a);
  } else {
    a.stat = (float*)scratch;
    a.part = a.stat + entry_floats(p, samples, groups, true);
    const StreamFns fns = {GN_PICK(GnFn, gn_sums_kernel, dtype, vec, act), dx ? GN_PICK(GnFn, gn_dx_kernel, dtype, vec, act) : nullptr};
    e = launch_streaming(fns, p, samples, vec ? (int)(16 / esz) : 1, esz, true, s, a);
  }
  if ((dw || db) && e == cudaSuccess) e = run_params(a, rows, dtype, a.part + (size_t)rows * 2 * channels, s);
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}
