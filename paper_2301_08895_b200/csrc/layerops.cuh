// What the stand-alone layer operations share: argument checks, launches, activations, vector loads.
#pragma once
#include <math.h>

#include <initializer_list>

#include "common.cuh"

namespace absb {

void set_last_error(const char* text);   // abs_api.cu: text returned by abs_last_error()

namespace layer {

constexpr int MAX_DEVICES = 64;

int fail(int code, const char* fmt, ...);            // linear.cu
// Properties of the current device, looked up once per device: ABS_OK, or an error with its text.
int current_device(int* device, int* sms);           // linear.cu

// A kernel that uses more than 48 KB of dynamic shared memory says so once per device.
template <typename... KArgs>
cudaError_t allow_smem(void (*kernel)(KArgs...), size_t bytes) {
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}

// Launch that may start while the kernel in front of it drains: every kernel of these operations waits for that one
// before it reads or writes anything.
template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
  if (e != cudaSuccess) cudaGetLastError();            // (reported by this call; not to be found by the caller's next one)
  return e;
}

// ---- device memory of a matrix: rows of `cols` elements, `ld` apart
struct Span {
  uintptr_t lo, hi;        // first byte and the byte behind the last one
  long long ld, row;       // pitch and row length in bytes
};
inline Span span(const void* p, long long rows, long long cols, long long ld, size_t esz) {
  Span s = {(uintptr_t)p, (uintptr_t)p, (long long)(ld * (long long)esz), (long long)(cols * (long long)esz)};
  if (p && rows > 0) s.hi += (uintptr_t)((rows - 1) * s.ld + s.row);
  return s;
}
// Whether two matrices share a byte; column ranges of one buffer (equal pitches) do not.
inline bool overlap(const Span& a, const Span& b) {
  if (a.lo == a.hi || b.lo == b.hi || a.hi <= b.lo || b.hi <= a.lo) return false;
  if (a.ld != b.ld || a.ld <= 0) return true;
  const long long d = (long long)((b.lo >= a.lo ? b.lo - a.lo : a.ld - (a.lo - b.lo) % a.ld) % a.ld);   // b's column offset from a
  return d < a.row || d + b.row > a.ld;
}

// Scratch: large enough, aligned, apart from the call's other memory; vectors: aligned to their type (linear.cu).
int check_scratch(const void* scratch, size_t have, size_t need, std::initializer_list<Span> others);
int check_vector(const char* name, const void* p, size_t esz);

// ---- activations.  Exponential and reciprocal are the hardware's approximations (2^-22 each, denormal results are zero):
// two instructions of the special-function unit per value, where expf and a division cost some twenty instructions.
__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// z held at -41.5 from below, a NaN kept: SiLU and its slope are evaluated there, and below it they are those of -41.5, which are smaller than
// 4e-17.  (Its exponential stays below 2^60, which the vectors' shared reciprocals need; -infinity gets a finite value.)
__device__ __forceinline__ float silu_held(float z) {
  float h;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(h) : "f"(z), "f"(-41.5f));
  return h;
}
// Phi(z) and exp(-z^2 / 2).  With x = |z| / sqrt(2), exp(x^2) erfc(x) is a polynomial of degree eight in t - 0.62318, t = 1 / (1 + 0.322 x), but for
// 2^-24.9 of itself: the least such error over 0 <= x <= 9.5, by reweighted least squares (Lawson's method).  Phi is then good to 2^-21, and left of zero
// to 2^-19 of itself at z = -5 and 2^-16 at -12, where exp(-z^2 / 2) loses the roundings of z^2.
__device__ __forceinline__ float normal_cdf(float z, float& bell) {
  const float s = rcp_approx(fmaf(0.22768838f, fabsf(z), 1.f)) - 0.62318307f;
  bell = ex2_approx(-0.72134752044448170f * z * z);
  float p = fmaf(-0.0858301465f, s, -0.0936853988f);
  p = fmaf(p, s, 0.168758458f);
  p = fmaf(p, s, 0.60961558f);
  p = fmaf(p, s, 0.950146763f);
  p = fmaf(p, s, 0.996267036f);
  p = fmaf(p, s, 0.779021849f);
  p = fmaf(p, s, 0.470782062f);
  p = fmaf(p, s, 0.134547527f);
  const float tail = p * bell;                       // Phi(-|z|)
  return z >= 0.f ? 1.f - tail : tail;
}

template <int ACT> __device__ __forceinline__ float act_value(float z) {
  if (ACT == ABS_ACT_RELU) return fmaxf(z, 0.f);
  if (ACT == ABS_ACT_GELU) {
    float bell;
    return z * normal_cdf(z, bell);
  }
  if (ACT == ABS_ACT_SILU) {
    const float h = silu_held(z);
    return h * rcp_approx(1.f + ex2_approx(-1.4426950408889634f * h));
  }
  return z;
}
template <int ACT> __device__ __forceinline__ float act_slope(float z) {
  if (ACT == ABS_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (ACT == ABS_ACT_GELU) {
    float bell;
    const float c = normal_cdf(z, bell);
    return fmaf(0.39894228040143268f * z, bell, c);
  }
  if (ACT == ABS_ACT_SILU) {                           // s (1 + z (1 - s)) with 1 - s = exp(-z) s: far above zero 1 - s would be s's rounding
    const float h = silu_held(z), e = ex2_approx(-1.4426950408889634f * h), s = rcp_approx(1.f + e);
    return s * fmaf(h * e, s, 1.f);
  }
  return 1.f;
}

// ---- N floats in pairs: the packed FP32 instructions of sm_100 work on two at a time
template <int N> struct Lanes {
  static_assert(N % 2 == 0, "pairs");
  unsigned long long p[N / 2];
  __device__ __forceinline__ void fill(float v) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) put(i, v, v);
  }
  __device__ __forceinline__ void put(int i, float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(p[i]) : "f"(a), "f"(b)); }
  __device__ __forceinline__ void set(const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) put(i, v[2 * i], v[2 * i + 1]);
  }
  __device__ __forceinline__ void get(float (&v)[N]) const {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) asm("mov.b64 {%0, %1}, %2;" : "=f"(v[2 * i]), "=f"(v[2 * i + 1]) : "l"(p[i]));
  }
  // 16-byte accesses (N a multiple of four)
  __device__ __forceinline__ void load(const float* s) {
#pragma unroll
    for (int i = 0; i < N / 2; i += 2) {
      const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(s + 2 * i);
      p[i] = q.x;
      p[i + 1] = q.y;
    }
  }
  __device__ __forceinline__ void store(float* d) const {
#pragma unroll
    for (int i = 0; i < N / 2; i += 2) *reinterpret_cast<ulonglong2*>(d + 2 * i) = make_ulonglong2(p[i], p[i + 1]);
  }
};
template <> struct Lanes<1> {
  float v0;
  __device__ __forceinline__ void fill(float v) { v0 = v; }
  __device__ __forceinline__ void set(const float (&v)[1]) { v0 = v[0]; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = v0; }
  __device__ __forceinline__ void load(const float* s) { v0 = *s; }
  __device__ __forceinline__ void store(float* d) const { *d = v0; }
};
template <int N> __device__ __forceinline__ Lanes<N> add(const Lanes<N>& a, const Lanes<N>& b) {
  Lanes<N> r;
  if constexpr (N == 1) r.v0 = a.v0 + b.v0;
  else
#pragma unroll
    for (int i = 0; i < N / 2; ++i) asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.p[i]) : "l"(a.p[i]), "l"(b.p[i]));
  return r;
}
template <int N> __device__ __forceinline__ Lanes<N> mul(const Lanes<N>& a, const Lanes<N>& b) {
  Lanes<N> r;
  if constexpr (N == 1) r.v0 = a.v0 * b.v0;
  else
#pragma unroll
    for (int i = 0; i < N / 2; ++i) asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.p[i]) : "l"(a.p[i]), "l"(b.p[i]));
  return r;
}
template <int N> __device__ __forceinline__ Lanes<N> fma(const Lanes<N>& a, const Lanes<N>& b, const Lanes<N>& c) {
  Lanes<N> r;
  if constexpr (N == 1) r.v0 = fmaf(a.v0, b.v0, c.v0);
  else
#pragma unroll
    for (int i = 0; i < N / 2; ++i) asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.p[i]) : "l"(a.p[i]), "l"(b.p[i]), "l"(c.p[i]));
  return r;
}
// 1 / (1 + exp(-z)) of N values, and e = exp(-z).  Two values share a reciprocal, 1 / a = b / (a b): a value then costs the special-function unit one
// and a half instructions instead of two, which bounds a pass of SiLU over bf16 (64 x 64 x 64 x 320: 63.6 -> 55.6 us).
// held: z as silu_held gives it, so that the product of two values of 1 + exp(-z) <= 2^60 stays finite; the reciprocals take a NaN's exponential
// for 2^60 instead, since it would reach its partner through them, and the NaN comes back by the caller's product with held.
template <int N> __device__ __forceinline__ Lanes<N> sigmoids(const Lanes<N>& z, Lanes<N>& held, Lanes<N>& e) {
  static_assert(N % 4 == 0, "pairs of pairs");
  float v[N];
  Lanes<N> k, one, a;
  k.fill(-1.4426950408889634f);
  one.fill(1.f);
  z.get(v);
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = silu_held(v[j]);
  held.set(v);
  mul(held, k).get(v);
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = fminf(ex2_approx(v[j]), 0x1p60f);
  e.set(v);
  a = add(e, one);
  Lanes<N> r;
#pragma unroll
  for (int i = 0; i < N / 2; i += 2) {
    Lanes<2> x, y, q;
    float w[2];
    x.p[0] = a.p[i];
    y.p[0] = a.p[i + 1];
    mul(x, y).get(w);
    w[0] = rcp_approx(w[0]);
    w[1] = rcp_approx(w[1]);
    q.set(w);
    r.p[i] = mul(q, y).p[0];
    r.p[i + 1] = mul(q, x).p[0];
  }
  return r;
}
template <int ACT, int N> __device__ __forceinline__ Lanes<N> act_values(const Lanes<N>& z) {
  if constexpr (ACT == ABS_ACT_NONE) return z;
  if constexpr (ACT == ABS_ACT_SILU && N > 1) {
    Lanes<N> held, e;
    const Lanes<N> s = sigmoids(z, held, e);
    return mul(held, s);
  }
  float v[N];
  Lanes<N> r;
  z.get(v);
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = act_value<ACT>(v[j]);
  r.set(v);
  return r;
}
template <int ACT, int N> __device__ __forceinline__ Lanes<N> act_slopes(const Lanes<N>& z) {
  if constexpr (ACT == ABS_ACT_SILU && N > 1) {
    Lanes<N> held, e, one;
    one.fill(1.f);
    const Lanes<N> s = sigmoids(z, held, e);
    return mul(s, fma(mul(held, e), s, one));          // (as act_slope)
  }
  float v[N];
  Lanes<N> r;
  z.get(v);
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = act_slope<ACT>(v[j]);
  r.set(v);
  return r;
}

// ---- VE consecutive stored values in one access (16 bytes, or one element), and as binary32
template <typename T, int VE> struct Pack;
template <> struct Pack<float, 4> {
  float4 q;
  __device__ __forceinline__ void load(const float* p) { q = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = q; }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w; }
  __device__ __forceinline__ void set(const float (&v)[4]) { q = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Pack<__nv_bfloat16, 8> {
  uint4 q;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { q = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = q; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(u[j] << 16); v[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
      u[j] = *reinterpret_cast<const uint32_t*>(&b);
    }
    q = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <typename T> struct Pack<T, 1> {
  T q;
  __device__ __forceinline__ void load(const T* p) { q = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = q; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = (float)q; }
  __device__ __forceinline__ void set(const float (&v)[1]) { q = (T)v[0]; }
};

template <typename T> __device__ __forceinline__ T round_to(float v);
template <> __device__ __forceinline__ float round_to<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 round_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Division of x < 2^32 by a fixed d >= 1 (Granlund and Montgomery): q = (t + ((x - t) >> 1)) >> (l - 1) with
// t = floor(m x / 2^32), l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1.
struct Divisor {
  uint32_t d, m;
  int sh;
  Divisor() = default;
  __host__ explicit Divisor(uint32_t div) : d(div) {
    int l = 0;
    while (l < 32 && (1ull << l) < div) ++l;
    m = (uint32_t)(((1ull << 32) * ((1ull << l) - div)) / div + 1);
    sh = l;
  }
  __device__ __forceinline__ uint32_t div(uint32_t x) const {
    if (sh == 0) return x;
    const uint32_t t = __umulhi(m, x);
    return (t + ((x - t) >> 1)) >> (sh - 1);
  }
};

}  // namespace layer
}  // namespace absb
