// Dropout from the counter-based generator: the mask is a function of (row, column, call, seed) and is never stored.
#include "layerops.cuh"
#include "philox.cuh"

using namespace absb;
using namespace absb::layer;

namespace {

constexpr int DROP_NT = 256;                 // threads; a thread takes U blocks of eight columns, all loaded before the first is used

struct DropArgs {
  const void* x; const void* r; void* y;
  long long ldx, ldr, ldy;
  uint32_t row0;                             // first row of this launch
  uint32_t units, cols;                      // blocks of eight columns in this launch; columns
  Divisor per_row;                           // blocks of a row
  uint32_t thr, call, key0, key1;            // thr = T << 16 (T < 65536)
  int none;                                  // T = 65536: nothing is kept
  float scale;
};

// Eight columns (fewer at a row's end) as loaded.
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
  Pack<__nv_bfloat16, 8> p;
  __device__ __forceinline__ void load(const __nv_bfloat16* s) { p.load(s); }
  __device__ __forceinline__ void store(__nv_bfloat16* d) const { p.store(d); }
  __device__ __forceinline__ void get(float (&v)[8]) const { p.get(v); }
  __device__ __forceinline__ void set(const float (&v)[8]) { p.set(v); }
};
template <> struct Eight<float> {
  Pack<float, 4> a, b;
  __device__ __forceinline__ void load(const float* s) { a.load(s); b.load(s + 4); }
  __device__ __forceinline__ void store(float* d) const { a.store(d); b.store(d + 4); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const float u[8] = {a.q.x, a.q.y, a.q.z, a.q.w, b.q.x, b.q.y, b.q.z, b.q.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = u[j];
  }
  __device__ __forceinline__ void set(const float (&v)[8]) { a.q = make_float4(v[0], v[1], v[2], v[3]); b.q = make_float4(v[4], v[5], v[6], v[7]); }
};

template <typename T, bool VEC>
__device__ __forceinline__ void load8(Eight<T>& e, const T* p, int n) {
  if (VEC && n == 8) { e.load(p); return; }
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < n ? ldf(p, j) : 0.f;
  e.set(v);
}

template <typename T, bool VEC, bool RES, int U>
__global__ void __launch_bounds__(DROP_NT) dropout_kernel(DropArgs a) {
  grid_dependency_sync();
  const T* x = (const T*)a.x;
  const T* r = (const T*)a.r;
  T* y = (T*)a.y;
  const uint32_t u0 = blockIdx.x * (uint32_t)(DROP_NT * U) + threadIdx.x;
  Eight<T> ex[U], er[U];
  uint32_t row[U], blk[U];
  int n[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const uint32_t u = u0 + k * DROP_NT;
    const bool in = u < a.units;
    const uint32_t q = a.per_row.div(in ? u : 0u);
    row[k] = a.row0 + q;
    blk[k] = (in ? u : 0u) - q * a.per_row.d;
    n[k] = in ? (int)min(8u, a.cols - 8u * blk[k]) : 0;
    load8<T, VEC>(ex[k], x + (long long)row[k] * a.ldx + 8ll * blk[k], n[k]);
    if (RES) load8<T, VEC>(er[k], r + (long long)row[k] * a.ldr + 8ll * blk[k], n[k]);
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    if (n[k] == 0) break;
    uint32_t w[4];
    philox4x32_10(blk[k], row[k], 2u, a.call, a.key0, a.key1, w);
    float v[8], rv[8];
    ex[k].get(v);
    if (RES) er[k].get(rv);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool keep = !a.none && ((j & 1) ? w[j >> 1] : w[j >> 1] << 16) >= a.thr;
      v[j] = keep ? v[j] * a.scale : 0.f;          // (selected, so that a dropped infinity or NaN is gone)
      if (RES) v[j] += rv[j];
    }
    T* d = y + (long long)row[k] * a.ldy + 8ll * blk[k];
    if (VEC && n[k] == 8) {
      Eight<T> o;
      o.set(v);
      o.store(d);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n[k]) stf(d, j, v[j]);
    }
  }
}

template <typename T, int U> void (*dropout_fn(bool vec, bool res))(DropArgs) {
  if (vec) return res ? dropout_kernel<T, true, true, U> : dropout_kernel<T, true, false, U>;
  return res ? dropout_kernel<T, false, true, U> : dropout_kernel<T, false, false, U>;
}

}  // namespace

extern "C" int abs_dropout(const void* x, long long ldx, const void* residual, long long ldr, void* y, long long ldy,
                           long long rows, long long cols, double p, unsigned long long seed, unsigned int call, int dtype,
                           void* stream) {
  if (dtype != ABS_FP32 && dtype != ABS_BF16_FP32MASTER) return fail(ABS_EUNSUPPORTED, "unknown dtype %d", dtype);
  if (rows < 0 || rows >= (1ll << 32)) return fail(ABS_EINVAL, "rows %lld outside [0, 2^32)", rows);
  if (cols < 1 || cols >= (1ll << 31)) return fail(ABS_EINVAL, "cols %lld outside [1, 2^31)", cols);
  if (!(p >= 0.0 && p <= 1.0)) return fail(ABS_EINVAL, "p %g outside [0, 1]", p);
  if (rows == 0) return ABS_OK;
  if (!x || !y) return fail(ABS_EINVAL, "null pointer argument");
  if (rows == 1) { ldx = ldy = cols; ldr = cols; }
  if (ldx < cols || ldy < cols || (residual && ldr < cols)) return fail(ABS_EINVAL, "a row pitch is below the %lld columns", cols);
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  if (((uintptr_t)x | (uintptr_t)y | (uintptr_t)residual) % esz) return fail(ABS_EINVAL, "a matrix is not aligned to its type");
  const Span sx = span(x, rows, cols, ldx, esz), sr = span(residual, rows, cols, ldr, esz), sy = span(y, rows, cols, ldy, esz);
  if (overlap(sx, sy) && !(x == y && ldx == ldy)) return fail(ABS_EINVAL, "y overlaps x without being the same matrix");
  if (residual && overlap(sr, sy) && !(residual == y && ldr == ldy)) return fail(ABS_EINVAL, "y overlaps residual without being the same matrix");
  DropArgs a;
  a.x = x; a.r = residual; a.y = y;
  a.ldx = ldx; a.ldr = ldr; a.ldy = ldy;
  a.cols = (uint32_t)cols;
  const uint32_t per_row = (uint32_t)((cols + 7) / 8);
  a.per_row = Divisor(per_row);
  const uint32_t T = (uint32_t)floor(p * 65536.0 + 0.5);
  a.none = T == 65536u;
  a.thr = a.none ? 0u : T << 16;
  a.scale = a.none ? 0.f : 65536.f / (float)(65536u - T);
  a.call = call;
  a.key0 = (uint32_t)seed;
  a.key1 = (uint32_t)(seed >> 32);
  const bool vec = (((uintptr_t)x | (uintptr_t)y | (uintptr_t)residual | (uintptr_t)(ldx * (long long)esz) | (uintptr_t)(ldy * (long long)esz) |
                     (residual ? (uintptr_t)(ldr * (long long)esz) : 0)) & 15) == 0;
  // four blocks per thread, or one where that leaves SMs without work (128 x 256: 2.1 us, and 1.1 with one)
  const int U = rows * per_row > 2ll * PLAN_SMS * DROP_NT * 4 ? 4 : 1;
  void (*kernel)(DropArgs) = dtype == ABS_FP32 ? (U == 4 ? dropout_fn<float, 4>(vec, residual != nullptr) : dropout_fn<float, 1>(vec, residual != nullptr))
                                               : (U == 4 ? dropout_fn<__nv_bfloat16, 4>(vec, residual != nullptr) : dropout_fn<__nv_bfloat16, 1>(vec, residual != nullptr));
  // unit numbers are 32-bit: at most 2^30 blocks per launch
  const long long step = (1ll << 30) / per_row;
  for (long long r0 = 0; r0 < rows; r0 += step) {
    const long long nr = rows - r0 < step ? rows - r0 : step;
    a.row0 = (uint32_t)r0;
    a.units = (uint32_t)(nr * per_row);
    const cudaError_t e = launch(kernel, dim3((a.units + DROP_NT * U - 1) / (DROP_NT * U)), DROP_NT, 0, 1, (cudaStream_t)stream, a);
    if (e != cudaSuccess) return fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
  }
  return ABS_OK;
}
