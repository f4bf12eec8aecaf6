// Group normalisation of channels-last maps with an activation, and its gradients.
#include "layerops.cuh"

using namespace absb;
using namespace absb::layer;

namespace {

constexpr int GN_NT = 256;

struct GnArgs {
  const void* x; const void* dy; const void* w; const void* b;
  void* y;                               // forward: y; backward: dx
  void* dw; void* db;
  float* mean; float* rstd;
  long long xs, xp, ys, yp, ds, dp;      // pitches of x, y (dx), dy
  long long samples;
  uint32_t positions;
  int C, G, D;                           // channels, groups, channels per group
  float eps;
};

__device__ __forceinline__ float block_sum(float v, float* sm) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < GN_NT / 32; ++i) t += sm[i];
  return t;
}

template <typename T> __device__ __forceinline__ float param(const void* p, int c, float none) { return p ? ldf((const T*)p, c) : none; }

// One CTA per sample and group, three passes over the group (the later two from L2).
template <typename T, int ACT>
__global__ void __launch_bounds__(GN_NT) gn_simple_kernel(GnArgs a) {
  grid_dependency_sync();
  __shared__ float sm[GN_NT / 32];
  const long long n = blockIdx.x / a.G;
  const int g = blockIdx.x % a.G, c0 = g * a.D;
  const T* x = (const T*)a.x + n * a.xs + c0;
  T* y = (T*)a.y + n * a.ys + c0;
  const long long cnt = (long long)a.positions * a.D;
  float s = 0.f;
  for (long long i = threadIdx.x; i < cnt; i += GN_NT) s += ldf(x, (i / a.D) * a.xp + i % a.D);
  const float mean = block_sum(s, sm) / (float)cnt;
  s = 0.f;
  for (long long i = threadIdx.x; i < cnt; i += GN_NT) {
    const float d = ldf(x, (i / a.D) * a.xp + i % a.D) - mean;
    s = fmaf(d, d, s);
  }
  const float rstd = 1.f / sqrtf(block_sum(s, sm) / (float)cnt + a.eps);
  for (long long i = threadIdx.x; i < cnt; i += GN_NT) {
    const int c = (int)(i % a.D);
    const long long p = i / a.D;
    const float xh = (ldf(x, p * a.xp + c) - mean) * rstd;
    stf(y, p * a.yp + c, act_value<ACT>(fmaf(xh, param<T>(a.w, c0 + c, 1.f), param<T>(a.b, c0 + c, 0.f))));
  }
  if (threadIdx.x == 0 && a.mean) {
    a.mean[n * a.G + g] = mean;
    a.rstd[n * a.G + g] = rstd;
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

template <typename T, int ACT>
__global__ void __launch_bounds__(GN_NT) gn_grad_simple_kernel(GnArgs a) {
  grid_dependency_sync();
  __shared__ float sm[GN_NT / 32];
  const long long n = blockIdx.x / a.G;
  const int gi = blockIdx.x % a.G, c0 = gi * a.D;
  const T* x = (const T*)a.x + n * a.xs + c0;
  const T* dy = (const T*)a.dy + n * a.ds + c0;
  T* dx = (T*)a.y + n * a.ys + c0;
  const long long cnt = (long long)a.positions * a.D;
  const float mean = a.mean[n * a.G + gi], rstd = a.rstd[n * a.G + gi];
  float s1 = 0.f, s2 = 0.f;
  for (int pass = 0; pass < 2; ++pass) {
    for (long long i = threadIdx.x; i < cnt; i += GN_NT) {
      const int c = (int)(i % a.D);
      const long long p = i / a.D;
      const float w = param<T>(a.w, c0 + c, 1.f), b = param<T>(a.b, c0 + c, 0.f);
      const float xv = ldf(x, p * a.xp + c), xh = (xv - mean) * rstd;
      const float g = ldf(dy, p * a.dp + c) * slope_at<ACT>(xv, mean, rstd, xh, w, b) * w;
      if (pass == 0) { s1 += g; s2 = fmaf(g, xh, s2); }
      else stf(dx, p * a.yp + c, rstd * (g - s1 - xh * s2));
    }
    if (pass == 0) {
      s1 = block_sum(s1, sm) / (float)cnt;
      s2 = block_sum(s2, sm) / (float)cnt;
    }
  }
}

// dw, db: block = 32 channels x 8 rows of threads
template <typename T, int ACT>
__global__ void __launch_bounds__(GN_NT) gn_param_simple_kernel(GnArgs a) {
  grid_dependency_sync();
  __shared__ float red[2][8][33];
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float sw = 0.f, sb = 0.f;
  if (c < a.C) {
    const float w = param<T>(a.w, c, 1.f), b = param<T>(a.b, c, 0.f);
    for (long long n = 0; n < a.samples; ++n) {
      const float mean = a.mean[n * a.G + c / a.D], rstd = a.rstd[n * a.G + c / a.D];
      for (uint32_t p = r; p < a.positions; p += 8) {
        const float xv = ldf((const T*)a.x, n * a.xs + (long long)p * a.xp + c), xh = (xv - mean) * rstd;
        const float g = ldf((const T*)a.dy, n * a.ds + (long long)p * a.dp + c) * slope_at<ACT>(xv, mean, rstd, xh, w, b);
        sb += g;
        sw = fmaf(g, xh, sw);
      }
    }
  }
  red[0][r][lane] = sw;
  red[1][r][lane] = sb;
  __syncthreads();
  if (r < 2 && c < a.C) {
    float t = 0.f;
    for (int k = 0; k < 8; ++k) t += red[r][k][lane];
    void* out = r == 0 ? a.dw : a.db;
    if (out) stf((T*)out, c, t);
  }
}

typedef void (*GnFn)(GnArgs);
#define GN_PICK(name, T, act) \
  ((act) == ABS_ACT_RELU ? (GnFn)name<T, ABS_ACT_RELU> : (act) == ABS_ACT_GELU ? (GnFn)name<T, ABS_ACT_GELU> \
   : (act) == ABS_ACT_SILU ? (GnFn)name<T, ABS_ACT_SILU> : (GnFn)name<T, ABS_ACT_NONE>)

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
  (void)grad;
  *out = 0;
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
  (void)scratch; (void)scratch_bytes;
  const GnFn fn = dtype == ABS_FP32 ? GN_PICK(gn_simple_kernel, float, act) : GN_PICK(gn_simple_kernel, __nv_bfloat16, act);
  const cudaError_t e = launch(fn, dim3((unsigned)(samples * groups)), GN_NT, 0, 1, (cudaStream_t)stream, a);
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
  (void)scratch; (void)scratch_bytes;
  if (dw || db) {                          // (in front of dx, which may take dy's place)
    const GnFn fn = dtype == ABS_FP32 ? GN_PICK(gn_param_simple_kernel, float, act) : GN_PICK(gn_param_simple_kernel, __nv_bfloat16, act);
    e = launch(fn, dim3((unsigned)((channels + 31) / 32)), GN_NT, 0, 1, (cudaStream_t)stream, a);
  }
  if (dx && e == cudaSuccess) {
    const GnFn fn = dtype == ABS_FP32 ? GN_PICK(gn_grad_simple_kernel, float, act) : GN_PICK(gn_grad_simple_kernel, __nv_bfloat16, act);
    e = launch(fn, dim3((unsigned)(samples * groups)), GN_NT, 0, 1, (cudaStream_t)stream, a);
  }
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}
