// Affine layer with bias, activation and residual in the epilogue of its matrix product, and its gradients.
#include <atomic>
#include <cstdarg>
#include <cstdio>

#include "layerops.cuh"

using namespace absb;
using namespace absb::layer;

namespace absb {
namespace layer {

int fail(int code, const char* fmt, ...) {
  char buf[384];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return code;
}

int current_device(int* device, int* sms) {
  static std::atomic<int> known[MAX_DEVICES];
  cudaError_t e = cudaGetDevice(device);
  if (e != cudaSuccess) return fail(ABS_ECUDA, "cudaGetDevice: %s", cudaGetErrorString(e));
  if (*device < 0 || *device >= MAX_DEVICES) return fail(ABS_EUNSUPPORTED, "device index %d not supported", *device);
  int n = known[*device].load(std::memory_order_relaxed);
  if (n == 0) {
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, *device);
    if (e != cudaSuccess) return fail(ABS_ECUDA, "cudaDeviceGetAttribute: %s", cudaGetErrorString(e));
    known[*device].store(n, std::memory_order_relaxed);
  }
  *sms = n;
  return ABS_OK;
}

}  // namespace layer
}  // namespace absb

namespace {

// C[i][j] = sum_k A(i, k) B(k, j) on FP32 FMAs; A and B by element strides, so that the three products of the layer are one kernel.
struct ProdArgs {
  const void* a; const void* b;
  long long a_i, a_k, b_k, b_j;          // element strides
  long long I; int J; long long K;
  const void* bias; const void* res; void* out; void* pre;
  long long ldr, ldo, ldp;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(256) product_kernel(ProdArgs p) {
  grid_dependency_sync();
  __shared__ float sa[16][65], sb[16][65];
  const long long i0 = (long long)blockIdx.x * 64;
  const int j0 = blockIdx.y * 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  for (long long k0 = 0; k0 < p.K; k0 += 16) {
    for (int e = threadIdx.x; e < 1024; e += 256) {
      const int ka = p.a_k == 1 ? e & 15 : e >> 6, ia = p.a_k == 1 ? e >> 4 : e & 63;
      sa[ka][ia] = (i0 + ia < p.I && k0 + ka < p.K) ? ldf((const T*)p.a, (i0 + ia) * p.a_i + (k0 + ka) * p.a_k) : 0.f;
      const int kb = p.b_k == 1 ? e & 15 : e >> 6, jb = p.b_k == 1 ? e >> 4 : e & 63;
      sb[kb][jb] = (j0 + jb < p.J && k0 + kb < p.K) ? ldf((const T*)p.b, (k0 + kb) * p.b_k + (j0 + jb) * p.b_j) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] = fmaf(sa[k][ty + 16 * u], sb[k][tx + 16 * v], acc[u][v]);
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const long long i = i0 + ty + 16 * u;
      const int j = j0 + tx + 16 * v;
      if (i >= p.I || j >= p.J) continue;
      const float z = acc[u][v] + (p.bias ? ldf((const T*)p.bias, j) : 0.f);
      if (p.pre) stf((T*)p.pre, i * p.ldp + j, z);
      float y = act_value<ACT>(z);
      if (p.res) y += ldf((const T*)p.res, i * p.ldr + j);
      stf((T*)p.out, i * p.ldo + j, y);
    }
}

// dz = dy act'(pre), rounded to storage, and the column sums of the unrounded dz over each block of rows
template <typename T, int ACT>
__global__ void __launch_bounds__(256) slope_kernel(const void* dy, long long lddy, const void* pre, long long ldp, void* dz, float* part,
                                                    long long rows, int n, int chunk) {
  grid_dependency_sync();
  __shared__ float red[8][33];
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
  const long long m0 = (long long)blockIdx.y * chunk, m1 = min(rows, m0 + chunk);
  float s = 0.f;
  if (j < n)
    for (long long m = m0 + r; m < m1; m += 8) {
      float g = ldf((const T*)dy, m * lddy + j);
      if (ACT != ABS_ACT_NONE) {
        g *= act_slope<ACT>(ldf((const T*)pre, m * ldp + j));
        stf((T*)dz, m * n + j, g);
      }
      s += g;
    }
  red[r][lane] = s;
  __syncthreads();
  if (r == 0 && j < n && part) {
    float t = 0.f;
    for (int k = 0; k < 8; ++k) t += red[k][lane];
    part[(size_t)blockIdx.y * n + j] = t;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) column_kernel(const float* part, int chunks, int n, void* db) {
  grid_dependency_sync();
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= n) return;
  float t = 0.f;
  for (int c = 0; c < chunks; ++c) t += part[(size_t)c * n + j];
  stf((T*)db, j, t);
}

typedef void (*ProdFn)(ProdArgs);
template <typename T> ProdFn product_fn(int act) {
  return act == ABS_ACT_RELU ? (ProdFn)product_kernel<T, ABS_ACT_RELU> : act == ABS_ACT_GELU ? (ProdFn)product_kernel<T, ABS_ACT_GELU>
         : act == ABS_ACT_SILU ? (ProdFn)product_kernel<T, ABS_ACT_SILU> : (ProdFn)product_kernel<T, ABS_ACT_NONE>;
}
typedef void (*SlopeFn)(const void*, long long, const void*, long long, void*, float*, long long, int, int);
template <typename T> SlopeFn slope_fn(int act) {
  return act == ABS_ACT_RELU ? (SlopeFn)slope_kernel<T, ABS_ACT_RELU> : act == ABS_ACT_GELU ? (SlopeFn)slope_kernel<T, ABS_ACT_GELU>
         : act == ABS_ACT_SILU ? (SlopeFn)slope_kernel<T, ABS_ACT_SILU> : (SlopeFn)slope_kernel<T, ABS_ACT_NONE>;
}

int run_product(const ProdArgs& p, int act, int dtype, cudaStream_t s) {
  const dim3 grid((unsigned)((p.I + 63) / 64), (unsigned)((p.J + 63) / 64));
  const cudaError_t e = launch(dtype == ABS_FP32 ? product_fn<float>(act) : product_fn<__nv_bfloat16>(act), grid, 256, 0, 1, s, p);
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}

int check(long long rows, int n_in, int n_out, int act, int dtype) {
  if (dtype != ABS_FP32 && dtype != ABS_BF16_FP32MASTER) return fail(ABS_EUNSUPPORTED, "unknown dtype %d", dtype);
  if (act < ABS_ACT_NONE || act > ABS_ACT_SILU) return fail(ABS_EUNSUPPORTED, "unknown activation %d", act);
  if (rows < 0 || rows >= (1ll << 31)) return fail(ABS_EINVAL, "rows %lld outside [0, 2^31)", rows);
  if (n_in < 1 || n_in > (1 << 20)) return fail(ABS_EINVAL, "n_in %d outside [1, 2^20]", n_in);
  if (n_out < 1 || n_out > (1 << 20)) return fail(ABS_EINVAL, "n_out %d outside [1, 2^20]", n_out);
  return ABS_OK;
}
int check_matrix(const char* name, const void* p, long long rows, long long cols, long long ld, size_t esz) {
  if (!p) return fail(ABS_EINVAL, "%s is null", name);
  if (ld < cols) return fail(ABS_EINVAL, "%s: row pitch %lld below its %lld columns", name, ld, cols);
  if ((uintptr_t)p % esz) return fail(ABS_EINVAL, "%s is not aligned to its type", name);
  return ABS_OK;
}

size_t round256(size_t v) { return (v + 255) / 256 * 256; }

struct GradPlan { size_t dz, part, total; int chunk, chunks; };
GradPlan grad_plan(long long rows, int n_out, int act, int dtype) {
  GradPlan g = {};
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  long long chunk = 64;
  while ((rows + chunk - 1) / chunk > 128) chunk *= 2;
  g.chunk = (int)chunk;
  g.chunks = (int)((rows + chunk - 1) / chunk);
  g.dz = 0;
  g.part = act == ABS_ACT_NONE ? 0 : round256((size_t)rows * n_out * esz);
  g.total = g.part + round256((size_t)g.chunks * n_out * 4);
  return g;
}

}  // namespace

extern "C" int abs_linear_scratch_bytes(long long rows, int n_in, int n_out, int act, int dtype, int grad, int aligned, size_t* out) {
  if (!out) return fail(ABS_EINVAL, "out is null");
  const int rc = check(rows, n_in, n_out, act, dtype);
  if (rc != ABS_OK) return rc;
  (void)aligned;
  *out = grad ? grad_plan(rows, n_out, act, dtype).total : 0;
  return ABS_OK;
}

extern "C" int abs_linear(const void* x, long long ldx, const void* w, long long ldw, const void* bias, const void* residual,
                          long long ldr, void* y, long long ldy, void* pre, long long ldp, long long rows, int n_in, int n_out,
                          int act, int dtype, void* scratch, size_t scratch_bytes, void* stream) {
  int rc = check(rows, n_in, n_out, act, dtype);
  if (rc != ABS_OK) return rc;
  if (rows == 0) return ABS_OK;
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  if ((rc = check_matrix("x", x, rows, n_in, ldx, esz)) != ABS_OK) return rc;
  if ((rc = check_matrix("w", w, n_in, n_out, ldw, esz)) != ABS_OK) return rc;
  if ((rc = check_matrix("y", y, rows, n_out, ldy, esz)) != ABS_OK) return rc;
  if (residual && (rc = check_matrix("residual", residual, rows, n_out, ldr, esz)) != ABS_OK) return rc;
  if (pre && (rc = check_matrix("pre", pre, rows, n_out, ldp, esz)) != ABS_OK) return rc;
  const Span sx = span(x, rows, n_in, ldx, esz), sw = span(w, n_in, n_out, ldw, esz), sb = span(bias, bias ? 1 : 0, n_out, n_out, esz);
  const Span sr = span(residual, residual ? rows : 0, n_out, ldr, esz), sy = span(y, rows, n_out, ldy, esz), sp = span(pre, pre ? rows : 0, n_out, ldp, esz);
  if (overlap(sy, sx) || overlap(sy, sw) || overlap(sy, sb)) return fail(ABS_EINVAL, "y overlaps an operand");
  if (overlap(sp, sx) || overlap(sp, sw) || overlap(sp, sb) || overlap(sp, sr) || overlap(sp, sy)) return fail(ABS_EINVAL, "pre overlaps another matrix");
  if (overlap(sy, sr) && !(y == residual && ldy == ldr)) return fail(ABS_EINVAL, "y overlaps residual without being the same matrix");
  (void)scratch; (void)scratch_bytes;
  const ProdArgs p = {x, w, ldx, 1, ldw, 1, rows, n_out, n_in, bias, residual, y, pre, ldr, ldy, ldp};
  return run_product(p, act, dtype, (cudaStream_t)stream);
}

extern "C" int abs_linear_grad(const void* dy, long long lddy, const void* x, long long ldx, const void* w, long long ldw,
                               const void* pre, long long ldp, void* dx, long long lddx, void* dw, long long lddw, void* db,
                               long long rows, int n_in, int n_out, int act, int dtype, void* scratch, size_t scratch_bytes,
                               void* stream) {
  int rc = check(rows, n_in, n_out, act, dtype);
  if (rc != ABS_OK) return rc;
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  cudaStream_t s = (cudaStream_t)stream;
  if (dw && (rc = check_matrix("dw", dw, n_in, n_out, lddw, esz)) != ABS_OK) return rc;
  if (rows == 0) {
    cudaError_t e = cudaSuccess;
    if (dw) e = cudaMemset2DAsync(dw, (size_t)lddw * esz, 0, (size_t)n_out * esz, (size_t)n_in, s);
    if (db && e == cudaSuccess) e = cudaMemsetAsync(db, 0, (size_t)n_out * esz, s);
    return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "memset: %s", cudaGetErrorString(e));
  }
  if ((rc = check_matrix("dy", dy, rows, n_out, lddy, esz)) != ABS_OK) return rc;
  if (dw && (rc = check_matrix("x", x, rows, n_in, ldx, esz)) != ABS_OK) return rc;
  if (dx && (rc = check_matrix("w", w, n_in, n_out, ldw, esz)) != ABS_OK) return rc;
  if (dx && (rc = check_matrix("dx", dx, rows, n_in, lddx, esz)) != ABS_OK) return rc;
  if (act != ABS_ACT_NONE && (rc = check_matrix("pre", pre, rows, n_out, ldp, esz)) != ABS_OK) return rc;
  const Span ins[4] = {span(dy, rows, n_out, lddy, esz), span(x, x ? rows : 0, n_in, ldx, esz), span(w, w ? n_in : 0, n_out, ldw, esz),
                       span(pre, act != ABS_ACT_NONE ? rows : 0, n_out, ldp, esz)};
  const Span outs[3] = {span(dx, dx ? rows : 0, n_in, lddx, esz), span(dw, dw ? n_in : 0, n_out, lddw, esz), span(db, db ? 1 : 0, n_out, n_out, esz)};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 4; ++j)
      if (overlap(outs[i], ins[j])) return fail(ABS_EINVAL, "a gradient overlaps an operand");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return fail(ABS_EINVAL, "two gradients overlap");
  }
  const GradPlan g = grad_plan(rows, n_out, act, dtype);
  if (scratch_bytes < g.total) return fail(ABS_ENOSPACE, "scratch holds %zu bytes, %zu needed", scratch_bytes, g.total);
  if (!scratch || (uintptr_t)scratch % 256) return fail(ABS_EINVAL, "scratch is null or not 256-byte aligned");
  void* dz = act == ABS_ACT_NONE ? const_cast<void*>(dy) : scratch;
  const long long lddz = act == ABS_ACT_NONE ? lddy : n_out;
  float* part = db ? (float*)((char*)scratch + g.part) : nullptr;
  cudaError_t e = cudaSuccess;
  if (act != ABS_ACT_NONE || db)
    e = launch(dtype == ABS_FP32 ? slope_fn<float>(act) : slope_fn<__nv_bfloat16>(act), dim3((unsigned)((n_out + 31) / 32), (unsigned)g.chunks), 256, 0, 1, s,
               dy, lddy, pre, ldp, dz, part, rows, n_out, g.chunk);
  if (db && e == cudaSuccess)
    e = launch(dtype == ABS_FP32 ? column_kernel<float> : column_kernel<__nv_bfloat16>, dim3((unsigned)((n_out + 255) / 256)), 256, 0, 1, s,
               (const float*)part, g.chunks, n_out, db);
  if (e != cudaSuccess) return fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
  if (dx) {
    const ProdArgs p = {dz, w, lddz, 1, 1, ldw, rows, n_in, n_out, nullptr, nullptr, dx, nullptr, 0, lddx, 0};
    if ((rc = run_product(p, ABS_ACT_NONE, dtype, s)) != ABS_OK) return rc;
  }
  if (dw) {
    const ProdArgs p = {x, dz, 1, ldx, lddz, 1, n_in, n_out, rows, nullptr, nullptr, dw, nullptr, 0, lddw, 0};
    if ((rc = run_product(p, ABS_ACT_NONE, dtype, s)) != ABS_OK) return rc;
  }
  return ABS_OK;
}
