// Affine layer with bias, activation and residual in the epilogue of its matrix product, and its gradients.
#include <atomic>
#include <cstdarg>
#include <cstdio>

#include "layerops.cuh"
#include "linear_tc.cuh"
#include "linear_fma.cuh"
#include "linear_small.cuh"

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

int check_scratch(const void* scratch, size_t have, size_t need, std::initializer_list<Span> others) {
  if (need == 0) return ABS_OK;
  if (have < need) return fail(ABS_ENOSPACE, "scratch holds %zu bytes, %zu needed", have, need);
  if (!scratch || (uintptr_t)scratch % 256) return fail(ABS_EINVAL, "scratch is null or not 256-byte aligned");
  const Span mine = {(uintptr_t)scratch, (uintptr_t)scratch + need, 0, 0};
  for (const Span& o : others)
    if (overlap(mine, o)) return fail(ABS_EINVAL, "scratch overlaps an operand or a result");
  return ABS_OK;
}

int check_vector(const char* name, const void* p, size_t esz) {
  return p && (uintptr_t)p % esz ? fail(ABS_EINVAL, "%s is not aligned to its type", name) : ABS_OK;
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

constexpr int BK_TERMS = tc::BK;

// dz = dy act'(pre), rounded to storage, and the column sums of the unrounded dz over each chunk of rows: one pass at HBM's pace
// (8192 x 4096 bf16 GELU: 201 MB in 45 us).  A thread takes VE columns of every R-th row, four rows' loads of both matrices under way.
struct SlopeArgs {
  const void* dy; const void* pre; void* dz; float* part;
  long long lddy, ldp, lddz, rows;
  int n, chunk, lv, R;                   // vectors of columns per CTA, thread rows
  Divisor by_lv;
};
template <typename T, int VE, int ACT>
__global__ void __launch_bounds__(256) slope_kernel(const SlopeArgs a) {
  __shared__ __align__(16) float red[256 * VE];
  const int r = (int)a.by_lv.div(threadIdx.x), v = (int)threadIdx.x - r * a.lv;
  const int c = (blockIdx.x * a.lv + v) * VE;
  const bool active = r < a.R && c < a.n;
  grid_dependency_sync();
  Lanes<VE> sum;
  sum.fill(0.f);
  if (active) {
    const long long m0 = (long long)blockIdx.y * a.chunk, m1 = min(a.rows, m0 + a.chunk);
    const T* dy = (const T*)a.dy + (m0 + r) * a.lddy + c;
    const T* pre = (const T*)a.pre + (m0 + r) * a.ldp + c;
    T* dz = (T*)a.dz + (m0 + r) * a.lddz + c;
    const long long s0 = a.R * a.lddy, s1 = a.R * a.ldp, s2 = a.R * a.lddz;
    constexpr int U = 4;
    for (long long m = m0 + r; m < m1; m += U * a.R, dy += U * s0, pre += U * s1, dz += U * s2) {
      Pack<T, VE> g[U], z[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (m + u * a.R < m1) {
          g[u].load(dy + u * s0);
          if (ACT != ABS_ACT_NONE) z[u].load(pre + u * s1);
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (m + u * a.R < m1) {
          float f[VE];
          Lanes<VE> l;
          g[u].get(f);
          l.set(f);
          if (ACT != ABS_ACT_NONE) {
            Lanes<VE> zl;
            z[u].get(f);
            zl.set(f);
            l = mul(l, act_slopes<ACT>(zl));
          }
          sum = add(sum, l);
          if (a.dz) {
            l.get(f);
            g[u].set(f);
            g[u].store(dz + u * s2);
          }
        }
    }
  }
  if (a.part == nullptr) return;
  const int cb = a.lv * VE;
  float f[VE];
  sum.get(f);
  if (active)
#pragma unroll
    for (int e = 0; e < VE; ++e) red[r * cb + v * VE + e] = f[e];
  __syncthreads();
  for (int i = threadIdx.x; i < cb && blockIdx.x * cb + i < a.n; i += 256) {
    float t = 0.f;
#pragma unroll 4
    for (int k = 0; k < a.R; ++k) t += red[k * cb + i];
    a.part[(size_t)blockIdx.y * a.n + blockIdx.x * cb + i] = t;
  }
}

// db = sum of the chunks' column sums: block = 32 columns x 8 rows of threads
template <typename T>
__global__ void __launch_bounds__(256) column_kernel(const float* part, int chunks, int n, void* db) {
  __shared__ float red[8][33];
  grid_dependency_sync();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
  float t = 0.f;
  if (j < n) {
#pragma unroll 8
    for (int c = w; c < chunks; c += 8) t += part[(size_t)c * n + j];
  }
  red[w][lane] = t;
  __syncthreads();
  if (w == 0 && j < n) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) v += red[k][lane];
    stf((T*)db, j, v);
  }
}

// Partial results of a split sum: C = epilogue(sum over splits), in order.
struct FinishArgs {
  const float* part;
  int splits, I, J, Jp;                  // Jp: pitch of a partial row
  const void* bias; const void* res; void* out; void* pre;
  long long ldr, ldo, ldp;
  Divisor quads;                         // groups of four columns per row
  uint32_t n;                            // groups
};
template <typename T, int ACT>
__global__ void __launch_bounds__(256) finish_kernel(FinishArgs a) {
  grid_dependency_sync();
  for (uint32_t q = blockIdx.x * 256u + threadIdx.x; q < a.n; q += gridDim.x * 256u) {
    const uint32_t i = a.quads.div(q), j = 4u * (q - i * a.quads.d);
    const float* p = a.part + (size_t)i * a.Jp + j;
    const size_t step = (size_t)a.I * a.Jp;
    float4 s = *reinterpret_cast<const float4*>(p);
#pragma unroll 4
    for (int k = 1; k < a.splits; ++k) {
      const float4 t = *reinterpret_cast<const float4*>(p + k * step);
      s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
    }
    const float z[4] = {s.x, s.y, s.z, s.w};
    float bias[4], res[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {                        // (all loads in front of the stores, which may alias them)
      const bool in = (int)j + e < a.J;
      bias[e] = a.bias && in ? ldf((const T*)a.bias, j + e) : 0.f;
      res[e] = a.res && in ? ldf((const T*)a.res, (long long)i * a.ldr + j + e) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((int)j + e >= a.J) break;
      const float v = z[e] + bias[e];
      if (a.pre) stf((T*)a.pre, (long long)i * a.ldp + j + e, v);
      stf((T*)a.out, (long long)i * a.ldo + j + e, act_value<ACT>(v) + res[e]);
    }
  }
}

// Copy of a matrix with a row pitch that TMA can address (a multiple of eight elements, the start on 16 bytes).
__global__ void __launch_bounds__(256) pack_kernel(const __nv_bfloat16* src, long long ld, long long rows, int cols, __nv_bfloat16* dst, int pitch) {
  grid_dependency_sync();
  const int per = pitch / 8;
  const long long n = rows * per;
  for (long long u = blockIdx.x * 256ll + threadIdx.x; u < n; u += gridDim.x * 256ll) {
    const long long r = u / per;
    const int c = (int)(u - r * per) * 8;
    const __nv_bfloat16* s = src + r * ld + c;
    __nv_bfloat16 v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? s[e] : __float2bfloat16_rn(0.f);
    *reinterpret_cast<uint4*>(dst + r * pitch + c) = *reinterpret_cast<const uint4*>(v);
  }
}

typedef void (*SlopeFn)(const SlopeArgs);
#define ACT_FN(type, name, act, ...)                                                                                       \
  ((act) == ABS_ACT_RELU ? (type)name<__VA_ARGS__, ABS_ACT_RELU> : (act) == ABS_ACT_GELU ? (type)name<__VA_ARGS__, ABS_ACT_GELU> \
   : (act) == ABS_ACT_SILU ? (type)name<__VA_ARGS__, ABS_ACT_SILU> : (type)name<__VA_ARGS__, ABS_ACT_NONE>)
SlopeFn slope_fn(int dtype, bool vec, int act) {
  if (dtype == ABS_FP32) return vec ? ACT_FN(SlopeFn, slope_kernel, act, float, 4) : ACT_FN(SlopeFn, slope_kernel, act, float, 1);
  return vec ? ACT_FN(SlopeFn, slope_kernel, act, __nv_bfloat16, 8) : ACT_FN(SlopeFn, slope_kernel, act, __nv_bfloat16, 1);
}
size_t round256(size_t v) { return (v + 255) / 256 * 256; }

struct Operand { const void* p; long long rows, cols, ld; };     // a stored matrix that TMA can address
struct Result {
  const void* bias; const void* res; long long ldr;
  void* out; long long ldo; void* pre; long long ldp;
  int act;
};

typedef void (*FinishFn)(FinishArgs);
template <typename T> cudaError_t finish(const float* part, int splits, int I, int J, const Result& r, int sms, cudaStream_t s) {
  FinishArgs f = {};
  f.part = part; f.splits = splits; f.I = I; f.J = J; f.Jp = (J + 3) / 4 * 4;
  f.bias = r.bias; f.res = r.res; f.out = r.out; f.pre = r.pre;
  f.ldr = r.ldr; f.ldo = r.ldo; f.ldp = r.ldp;
  f.quads = Divisor((uint32_t)(f.Jp / 4));
  f.n = (uint32_t)((size_t)I * (f.Jp / 4));              // (at most 2^31: plan_product)
  const unsigned blocks = (f.n + 255) / 256;
  return launch(ACT_FN(FinishFn, finish_kernel, r.act, T), dim3(blocks < 8u * sms ? blocks : 8u * sms), 256, 0, 1, s, f);
}

// ------------------------------------------------------------------ tensor-core products (bf16)

// How a product C[I][J] = sum over K terms is cut up.
struct Plan { int bn, cg, splits, kb_per; size_t part_bytes; double t; bool stretches; };     // stretches: of sums too long for tensor memory in one

// The cheapest of the five tiles and of the ways to split the sum, by a model in microseconds: a block of 64 terms of a tile (measured
// at 8192 x 4096 x 4096: 178 us with 256 x 256 tiles of CTA pairs; the narrow tiles wait for operands, not for the tensor cores), the
// tiles a unit (CTA or CTA pair) takes in turn, 4.1 us for launch, filling the pipeline and the last tile's epilogue, and for split sums the
// partial results' way through L2 and a second launch.
// partial: the results stay fp32 sums in scratch even if the sum is not split.
Plan plan_product(long long I, int J, long long K, bool partial = false) {
  struct Opt { int bn, cg; double kb; };
  static const Opt opts[5] = {{256, 2, 0.40}, {256, 1, 0.45}, {128, 1, 0.29}, {128, 2, 0.29}, {64, 1, 0.28}};
  const long long n_kb = (K + BK_TERMS - 1) / BK_TERMS;
  const long long Jp = (J + 3) / 4 * 4;
  Plan best = {};
  double best_t = 1e30;
  for (const Opt& o : opts) {
    const long long tiles = (I + 128 * o.cg - 1) / (128 * o.cg) * ((J + o.bn - 1) / o.bn);
    const long long units = PLAN_SMS / o.cg;
    for (int s = 1; s <= 64 && s <= n_kb; ++s) {
      const long long per = (n_kb + s - 1) / s;
      if (s > 1 && ((s - 1) * per >= n_kb || (size_t)s * I * Jp * 4 > (256u << 20))) continue;
      double t = (double)((tiles * s + units - 1) / units) * per * o.kb + 4.1;
      if (s > 1 || partial) t += 2.5 + (double)s * I * Jp * 8.0 / 6e6;
      if (t < best_t) {
        best_t = t;
        best = Plan{o.bn, o.cg, s, (int)per, s > 1 || partial ? round256((size_t)s * I * Jp * 4) : 0, t, partial};
      }
      if (tiles * s >= 2 * units) break;
    }
  }
  // (so that finish_kernel's numbers stay below 2^32; with larger results, a device of 180 GB holds operands of fewer than 7000 blocks)
  if (best.kb_per > dense::LONG_SUM && I * Jp <= 1ll << 33) {
    best.stretches = true;
    best.part_bytes = round256((size_t)best.splits * I * Jp * 4);
  }
  return best;
}

// The same for a product of pieces: six passes over the terms.
Plan plan_pieces(long long I, int J, long long K) { return plan_product(I, J, split3::PAIRS * ((K + BK_TERMS - 1) / BK_TERMS * BK_TERMS), true); }

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static std::atomic<EncodeTiledFn> known;
  EncodeTiledFn fn = known.load(std::memory_order_acquire);
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess) {
      fn = (EncodeTiledFn)p;
      known.store(fn, std::memory_order_release);
    }
  }
  return fn;
}
// bf16 matrix [rows][cols], 128-byte swizzle, boxes of 64 columns x box_rows
bool matrix_map(CUtensorMap* map, const void* p, long long rows, long long cols, long long ld, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, one[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// fp32 partial results [splits][I][Jp], boxes of 32 x 32
bool partial_map(CUtensorMap* map, const void* p, int I, int J, int Jp, int splits) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)J, (cuuint64_t)I, (cuuint64_t)splits};
  const cuuint64_t strides[2] = {(cuuint64_t)Jp * 4, (cuuint64_t)Jp * 4 * I};
  const cuuint32_t box[3] = {32, 32, 1}, one[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool tma_able(const void* p, long long rows, long long ld) { return (uintptr_t)p % 16 == 0 && (rows == 1 || ld % 8 == 0); }
long long tma_pitch(long long rows, long long cols, long long ld) { return rows == 1 ? (cols + 7) / 8 * 8 : ld; }
size_t pack_bytes(long long rows, long long cols) { return round256((size_t)rows * ((cols + 7) / 8 * 8) * 2); }

template <int BN, int CG, bool STRETCHES>
cudaError_t launch_dense(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, const CUtensorMap& z, const dense::Args& p, int sms, int device,
                         cudaStream_t s) {
  static std::atomic<uint64_t> ready;
  auto* kernel = dense::dense_kernel<BN, CG, STRETCHES>;
  if (!(ready.load(std::memory_order_acquire) >> device & 1)) {
    const cudaError_t e = allow_smem(kernel, dense::Cfg<BN, CG>::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    ready.fetch_or(1ull << device, std::memory_order_release);
  }
  const int units = sms / CG < p.n_tiles ? sms / CG : p.n_tiles;
  return launch(kernel, dim3((unsigned)(units * CG)), dense::THREADS, dense::Cfg<BN, CG>::SMEM_BYTES, CG, s, a, b, o, z, p);
}

template <bool STRETCHES>
cudaError_t launch_tile(const Plan& pl, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, const CUtensorMap& z, const dense::Args& p, int sms,
                        int device, cudaStream_t s) {
  if (pl.cg == 2) return pl.bn == 256 ? launch_dense<256, 2, STRETCHES>(a, b, o, z, p, sms, device, s) : launch_dense<128, 2, STRETCHES>(a, b, o, z, p, sms, device, s);
  return pl.bn == 256 ? launch_dense<256, 1, STRETCHES>(a, b, o, z, p, sms, device, s)
         : pl.bn == 128 ? launch_dense<128, 1, STRETCHES>(a, b, o, z, p, sms, device, s) : launch_dense<64, 1, STRETCHES>(a, b, o, z, p, sms, device, s);
}

__device__ unsigned g_status;            // how often a CTA's bounded wait ran out: only ever counted up, so that no report is lost to a reader
std::atomic<unsigned> g_status_seen[MAX_DEVICES];      // what abs_op_status has reported of it
unsigned* status_word(int device) {
  static std::atomic<unsigned*> known[MAX_DEVICES];
  unsigned* p = known[device].load(std::memory_order_acquire);
  if (!p && cudaGetSymbolAddress((void**)&p, g_status) == cudaSuccess) known[device].store(p, std::memory_order_release);
  return p;
}

// C[I][J] = sum_t A(i, t) B(j, t) for stored operands; a_mn / b_mn: the operand is stored [t][i] / [t][j].
// pieces: the operands are fp32 in three pieces each, and the result is left as the plan's partial sums.
int tc_product(const Operand& a, int a_mn, const Operand& b, int b_mn, int I, int J, long long K, const Result& r, const Plan& pl, bool pieces, float* part,
               int sms, int device, cudaStream_t s) {
  const int Jp = (J + 3) / 4 * 4;
  dense::Args p = {};
  p.a_mn = a_mn; p.b_mn = b_mn;
  p.I = I; p.J = J;
  p.kb_pass = (int)((K + BK_TERMS - 1) / BK_TERMS);
  p.n_kb = p.kb_pass;
  if (pieces) {
    p.n_kb *= split3::PAIRS;
    p.a_step = (int)(a.rows / 3); p.b_step = (int)(b.rows / 3);
  }
  p.splits = pl.splits; p.kb_per = pl.kb_per;
  p.stretch = pieces ? dense::STRETCH : dense::LONG_STRETCH;
  p.n_it = (I + 128 * pl.cg - 1) / (128 * pl.cg);
  p.n_jt = (J + pl.bn - 1) / pl.bn;
  const long long n_tiles = (long long)p.n_it * p.n_jt * pl.splits;
  if (n_tiles > 0x7fffffff) return fail(ABS_EUNSUPPORTED, "%lld tiles in one product", n_tiles);
  p.n_tiles = (int)n_tiles;
  p.status = status_word(device);
  if (!p.status) return fail(ABS_ECUDA, "cudaGetSymbolAddress(status) failed");
  CUtensorMap ma, mb, mo, mz;
  bool ok = matrix_map(&ma, a.p, a.rows, a.cols, a.ld, a_mn ? 64 : 128) && matrix_map(&mb, b.p, b.rows, b.cols, b.ld, b_mn ? 64 : pl.bn / pl.cg);
  const bool partial = pl.splits > 1 || pl.stretches;
  if (partial) {
    p.partial = 1;
    ok = ok && partial_map(&mo, part, I, J, Jp, pl.splits);
  } else {
    p.bias = (const __nv_bfloat16*)r.bias; p.res = (const __nv_bfloat16*)r.res; p.out = (__nv_bfloat16*)r.out; p.pre = (__nv_bfloat16*)r.pre;
    p.ldr = r.ldr; p.ldo = r.ldo; p.ldp = r.ldp;
    p.act = r.act;
    p.res_vec = r.res && (uintptr_t)r.res % 16 == 0 && (r.ldr % 8 == 0 || I == 1);
    p.bias_vec = r.bias && (uintptr_t)r.bias % 16 == 0;
    p.out_tma = tma_able(r.out, I, r.ldo);
    p.pre_tma = r.pre && tma_able(r.pre, I, r.ldp);
    mo = ma;
    if (p.out_tma) ok = ok && matrix_map(&mo, r.out, I, J, tma_pitch(I, J, r.ldo), 32);
  }
  mz = mo;
  if (p.pre_tma) ok = ok && matrix_map(&mz, r.pre, I, J, tma_pitch(I, J, r.ldp), 32);
  if (!ok) return fail(ABS_ECUDA, "cuTensorMapEncodeTiled failed");
  auto* go = pl.stretches ? &launch_tile<true> : &launch_tile<false>;
  cudaError_t e = go(pl, ma, mb, mo, mz, p, sms, device, s);
  if (e == cudaSuccess && partial && !pieces) e = finish<__nv_bfloat16>(part, pl.splits, I, J, r, sms, s);
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}

int pack(const void* src, long long rows, long long cols, long long ld, void* dst, int sms, cudaStream_t s) {
  const int pitch = (int)((cols + 7) / 8 * 8);
  const long long blocks = (rows * (pitch / 8) + 255) / 256;
  const cudaError_t e = launch(pack_kernel, dim3((unsigned)(blocks < 16 * sms ? blocks : 16 * sms)), 256, 0, 1, s, (const __nv_bfloat16*)src, ld, rows, (int)cols,
                               (__nv_bfloat16*)dst, pitch);
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}

// ------------------------------------------------------------------ fp32 products

// clusters of q CTAs that the GPU runs at a time, as the driver's occupancy query tells, with two CTAs per SM (72 clusters of four ran in two
// rounds, 150 us, pairs 126) and with one
const int CLUSTERS[9] = {0, 296, 148, 93, 71, 56, 45, 37, 33}, ALONE[9] = {0, 148, 74, 45, 33, 26, 22, 15, 15};

struct FmaPlan { int bm, Q, splits, kb_per; size_t part_bytes; double t; bool alone; };    // alone: one CTA per SM, by its shared memory
// 64 x 64 or 128 x 128 tiles, how many CTAs of a cluster share a tile's sum, and into how many parts that go through scratch it is cut
// besides.  A block of 32 k takes a CTA that is alone on its SM 0.95 or 3.3 us, two of them together 1.7 or 5.8 us (4096^3: 54
// TFLOP/s); a round of CTAs costs 3 to 5 us for filling and results, a microsecond more in clusters, parts their way through L2 and a
// launch.
FmaPlan plan_fma(long long I, int J, int K, int most = 64) {
  FmaPlan best = {};
  double least = 1e300;
  const int n_kb = (K + fp32::BK - 1) / fp32::BK;
  const long long Jp = (J + 3) / 4 * 4;
  for (int bm : {64, 128}) {
    const long long tiles = (I + bm - 1) / bm * ((J + bm - 1) / bm);
    const double one = bm == 64 ? 0.95 : 3.3, two = bm == 64 ? 1.7 : 5.8;
    for (int split = 1; split <= most; split *= 2) {
      const size_t bytes = split > 1 ? round256((size_t)split * (I * Jp + J) * 4) : 0;
      if (split > 1 && (bytes > (64u << 20) || tiles * (split / 2) > 2 * PLAN_SMS)) break;
      for (int q = 1; q <= 8; ++q) {
        const int chunks = q * split, per = (n_kb + chunks - 1) / chunks;
        if ((long long)(chunks - 1) * per >= n_kb) continue;     // (a part would be empty)
        const long long n = tiles * split, full = n / CLUSTERS[q], rest = n - full * CLUSTERS[q];
        const double around = (bm == 64 ? 3.0 : 5.0) + (q > 1 ? 1.0 : 0.0);
        const bool alone = full == 0 && rest <= ALONE[q], apart = alone || (q == 1 && rest <= ALONE[1]);
        const double last = rest == 0 ? 0.0 : (apart ? one : two) * per + around;
        const double t = (double)full * (two * per + around) + last + (split > 1 ? 2.5 + (double)bytes * 2.0 / 6e6 : 0.0);
        if (t < least) { least = t; best = FmaPlan{bm, q, split, per, bytes, t, alone}; }
      }
    }
  }
  return best;
}
// Two small products that run at a time, dx (rows x n_in, sums over n_out) and dw (n_in x n_out, sums over the rows, in as many parts as
// find a place): one launch if all CTAs of both are on the GPU together.  On their own each leaves most of it idle, and a second kernel
// behind the first costs about 4 us more than alone (1111 x 401 x 123: 26 us, together 19.5).
bool plan_fma_pair(long long rows, int n_in, int n_out, FmaPlan* dx, FmaPlan* dw) {
  constexpr int BM = 64;
  const int kx = (n_out + fp32::BK - 1) / fp32::BK, kw = (int)((rows + fp32::BK - 1) / fp32::BK);
  const long long tx = (rows + BM - 1) / BM * ((n_in + BM - 1) / BM), tw = (long long)((n_in + BM - 1) / BM) * ((n_out + BM - 1) / BM);
  const long long Jp = (n_out + 3) / 4 * 4;
  double least = dx->t + dw->t + 4.0;
  bool together = false;
  for (int q = 1; q <= 8 && tx + tw <= CLUSTERS[q]; ++q) {
    const int room = (int)((CLUSTERS[q] - tx) / tw);
    const int px = (kx + q - 1) / q, pw = (kw + room * q - 1) / (room * q), split = (kw + pw * q - 1) / (pw * q);
    if ((q - 1) * px >= kx || (split * q - 1) * pw >= kw) continue;      // (a part would be empty)
    const size_t bytes = split > 1 ? round256((size_t)split * (n_in * Jp + n_out) * 4) : 0;
    const bool alone = tx + tw * split <= ALONE[q];
    const double t = (px > pw ? px : pw) * (alone ? 0.95 : 1.7) + 3.0 + (q > 1 ? 1.0 : 0.0) +
                     (split > 1 ? 2.5 + (double)bytes * 2.0 / 6e6 : 0.0);
    if (t < least) {
      least = t;
      together = true;
      *dx = FmaPlan{BM, q, 1, px, 0, t, alone};
      *dw = FmaPlan{BM, q, split, pw, bytes, 0.0, alone};
    }
  }
  return together;
}

typedef void (*FmaFn)(const fp32::Pair);
template <int BM> FmaFn fma_fn(int act) {
  return act == ABS_ACT_RELU ? (FmaFn)fp32::fma_kernel<BM, BM, ABS_ACT_RELU> : act == ABS_ACT_GELU ? (FmaFn)fp32::fma_kernel<BM, BM, ABS_ACT_GELU>
         : act == ABS_ACT_SILU ? (FmaFn)fp32::fma_kernel<BM, BM, ABS_ACT_SILU> : (FmaFn)fp32::fma_kernel<BM, BM, ABS_ACT_NONE>;
}
// One fp32 product: its matrices, its plan and where its parts go.
struct Fma { fp32::Args p; FmaPlan pl; int I, J, K, act; float* part; };

// More than half of an SM's shared memory: CTAs of a cluster otherwise share SMs while others idle (1000 x 784 x 128 on 128 CTAs: 15.9 us in
// pairs, 12.9 alone).
constexpr size_t ALONE_SMEM = 120 * 1024;
static_assert(ALONE_SMEM >= fp32::Cfg<64, 64>::SMEM && ALONE_SMEM >= fp32::Cfg<128, 128>::SMEM, "");

int fma_products(std::initializer_list<Fma> products, int sms, int device, cudaStream_t s) {
  static std::atomic<uint64_t> ready;
  cudaError_t e = cudaSuccess;
  if (!(ready.load(std::memory_order_acquire) >> device & 1)) {
    for (int i = ABS_ACT_NONE; i <= ABS_ACT_SILU && e == cudaSuccess; ++i) {
      e = allow_smem(fma_fn<64>(i), ALONE_SMEM);
      if (e == cudaSuccess) e = allow_smem(fma_fn<128>(i), ALONE_SMEM);
    }
    if (e != cudaSuccess) return fail(ABS_ECUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    ready.fetch_or(1ull << device, std::memory_order_release);
  }
  fp32::Pair pair = {};
  long long ctas = 0;
  int n = 0;
  for (const Fma& f : products) {
    const FmaPlan& pl = f.pl;
    fp32::Args& p = pair.a[n++];
    p = f.p;
    p.I = f.I; p.J = f.J; p.K = f.K;
    p.n_kb = (f.K + fp32::BK - 1) / fp32::BK;
    p.n_jt = (f.J + pl.bm - 1) / pl.bm;
    p.Q = pl.Q; p.kb_per = pl.kb_per;
    p.by_Q = Divisor((uint32_t)pl.Q);
    p.by_njt = Divisor((uint32_t)p.n_jt);
    const long long tiles = ((long long)f.I + pl.bm - 1) / pl.bm * p.n_jt;
    if (pl.splits > 1) {
      p.bias = p.res = nullptr;
      p.pre = nullptr;
      p.ldo = (f.J + 3) / 4 * 4;
      p.out = f.part;
      p.out_step = f.I * p.ldo;
      p.col_step = f.J;
      if (p.colsum) p.colsum = f.part + pl.splits * p.out_step;
    }
    p.by_tiles = Divisor((uint32_t)(tiles < 0x7fffffff ? tiles : 1));
    ctas += tiles * pl.splits * pl.Q;
    if (ctas > 0x7fffffff) return fail(ABS_EUNSUPPORTED, "%lld tiles in one product", ctas);
    if (n == 1) pair.first = (uint32_t)ctas;
  }
  const Fma& one = *products.begin();                    // (two products have one tile, one cluster and no activation)
  const int in_kernel = one.pl.splits > 1 ? ABS_ACT_NONE : one.act;
  const size_t smem = one.pl.alone ? ALONE_SMEM : one.pl.bm == 64 ? fp32::Cfg<64, 64>::SMEM : fp32::Cfg<128, 128>::SMEM;
  e = launch(one.pl.bm == 64 ? fma_fn<64>(in_kernel) : fma_fn<128>(in_kernel), dim3((unsigned)ctas), fp32::NT, smem, one.pl.Q, s, pair);
  n = 0;
  for (const Fma& f : products) {
    const float* sums = pair.a[n++].colsum;
    if (e != cudaSuccess || f.pl.splits == 1) continue;
    const Result r = {f.p.bias, f.p.res, f.p.ldr, f.p.out, f.p.ldo, f.p.pre, f.p.ldp, f.act};
    e = finish<float>(f.part, f.pl.splits, f.I, f.J, r, sms, s);
    if (e == cudaSuccess && sums)
      e = launch(column_kernel<float>, dim3((unsigned)((f.J + 31) / 32)), 256, 0, 1, s, sums, f.pl.splits, f.J, (void*)f.p.colsum);
  }
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}
int check_pitches(std::initializer_list<long long> pitches) {
  for (long long pitch : pitches)
    if (pitch > (1ll << 24)) return fail(ABS_EUNSUPPORTED, "fp32: row pitch %lld above 2^24", pitch);
  return ABS_OK;
}

// ------------------------------------------------------------------ fp32 products on the tensor cores

constexpr int SPLIT_BLOCKS = 4 * PLAN_SMS;
constexpr size_t FLAG_BYTES = (SPLIT_BLOCKS * 4 + 255) / 256 * 256;
long long rows64(long long rows) { return (rows + 63) / 64 * 64; }
size_t piece_bytes(long long rows, int cols) { return round256((size_t)rows64(rows) * ((cols + 7) / 8 * 8) * 6); }
// The pieces' way is taken where its time by the models is less; plan_fma leaves out what every launch costs.  Around the border, us as plain
// fused multiply-adds and in pieces: 256 x 512 x 512 10.8, 13.3; 512 x 512 x 512 13.9, 14.4; 1000 x 784 x 128 12.9, 15.9; 400 x 1024 x 512 23.4, 17.6;
// 20000 x 128 x 128 32.4, 28.0; 1024 x 785 x 512 32.3, 20.8; gradients of 512 x 512 x 512 22.7, 28.2, of 1024 x 512 x 512 45.5, 34.4.
constexpr double PLAIN_START = 3.0;
double split_time(size_t bytes) { return 3.0 + (double)bytes * (10.0 / 6.0) / 4e6; }
// matrices whose pieces and results stay well inside scratch and the copies' coordinates
bool pieces_fit(long long I, int J, const Plan& pl, size_t bytes) {
  return bytes <= (2ull << 30) && pl.part_bytes <= (1ull << 30) && (size_t)I * ((J + 3) / 4 * 4) <= (1ull << 28);
}

struct Flags { uint32_t* p; int n; };
split3::Matrix in_pieces(const void* src, long long ld, long long rows, int cols, void* dst) {
  split3::Matrix m = {};
  m.src = (const float*)src; m.ld = ld; m.rows = rows; m.cols = cols;
  m.dst = (__nv_bfloat16*)dst; m.rows_p = (uint32_t)rows64(rows); m.cols_p = (cols + 7) / 8 * 8;
  m.vec = (uintptr_t)src % 16 == 0 && ld % 4 == 0;
  m.per_row = Divisor((uint32_t)(m.cols_p / 8));
  return m;
}
// terms: of the longest sum over these matrices
cudaError_t split(std::initializer_list<split3::Matrix> ms, long long terms, Flags* flags, cudaStream_t s) {
  split3::Args a = {};
  int log_terms = 0;
  while ((1ll << log_terms) < terms) ++log_terms;
  a.limit = ldexpf(1.f, (94 - log_terms) / 2);
  uint32_t n = 0, i = 0;
  for (const split3::Matrix& m : ms) {
    a.m[i] = m;
    n += m.rows_p * (uint32_t)(m.cols_p / 8);            // (at most 2^27 groups in 2 GB)
    a.m[i++].end = n;
  }
  a.n = n;
  a.flags = flags->p;
  const uint32_t blocks = (n + 255) / 256;
  flags->n = (int)(blocks < SPLIT_BLOCKS ? blocks : SPLIT_BLOCKS);
  return launch(split3::split_kernel, dim3((unsigned)flags->n), 256, 0, 1, s, a);
}
// C = epilogue(A B) from pieces: their product, then the plain kernel, which only adds the epilogue unless a flag is raised.
int pieces_product(const split3::Matrix& a, int a_mn, const split3::Matrix& b, int b_mn, fp32::Args plain, const Plan& pl, int I, int J, int K, int act,
                   const Flags& flags, float* part, int sms, int device, cudaStream_t s) {
  const Operand oa = {a.dst, 3ll * a.rows_p, a.cols_p, a.cols_p}, ob = {b.dst, 3ll * b.rows_p, b.cols_p, b.cols_p};
  const int rc = tc_product(oa, a_mn, ob, b_mn, I, J, K, Result{}, pl, true, part, sms, device, s);
  if (rc != ABS_OK) return rc;
  plain.flags = flags.p; plain.n_flags = flags.n;
  plain.sums = part; plain.parts = pl.splits;
  auto whole = [](const void* p, long long ld) { return !p || ((uintptr_t)p % 16 == 0 && ld % 4 == 0); };
  plain.vec = whole(plain.res, plain.ldr) && whole(plain.out, plain.ldo) && whole(plain.pre, plain.ldp);
  return fma_products({{plain, plan_fma(I, J, K, 1), I, J, K, act, nullptr}}, sms, device, s);
}

// ------------------------------------------------------------------ few rows, few outputs

// Rows up to which a pass over W on FP32 FMAs is faster than the tiled products: 784 -> 256 bf16 with 1, 2, 4 rows 3.5, 5.3, 8.9 us
// against 6.8 us of the tensor-core product; 785 -> 501 fp32 with 8 rows 11.1 us, the FMA tiles as much.
int few_rows_limit(int dtype) { return dtype == ABS_FP32 ? 8 : 2; }

typedef void (*RowsFn)(const small::Args, int);
template <typename T, int VE> RowsFn few_rows_fn(long long rows, int act) {
  if constexpr (sizeof(T) == 4) {
    if (rows > 4) return ACT_FN(RowsFn, small::few_rows_kernel, act, T, VE, 8);
    if (rows > 2) return ACT_FN(RowsFn, small::few_rows_kernel, act, T, VE, 4);
  }
  return rows == 1 ? ACT_FN(RowsFn, small::few_rows_kernel, act, T, VE, 1) : ACT_FN(RowsFn, small::few_rows_kernel, act, T, VE, 2);
}
int few_rows(const small::Args& a, int dtype, cudaStream_t s) {
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  const bool vec = (uintptr_t)a.w % 16 == 0 && (a.K == 1 || a.ldw * (long long)esz % 16 == 0) && (size_t)a.N * esz % 16 == 0;
  const int VE = vec ? (int)(16 / esz) : 1;
  // lanes per row of W: 32 bytes at least (vectors), more where two CTAs per SM remain, at most 256 bytes
  int log_l = vec ? 1 : 3;
  while (log_l < (vec ? 4 : 5) && (a.N + (VE << log_l) - 1) / (VE << log_l) > 2 * PLAN_SMS) ++log_l;
  const unsigned blocks = (unsigned)((a.N + (VE << log_l) - 1) / (VE << log_l));
  const RowsFn fn = dtype == ABS_FP32 ? (vec ? few_rows_fn<float, 4>(a.rows, a.act) : few_rows_fn<float, 1>(a.rows, a.act))
                                      : (vec ? few_rows_fn<__nv_bfloat16, 8>(a.rows, a.act) : few_rows_fn<__nv_bfloat16, 1>(a.rows, a.act));
  const int M = a.rows <= 2 ? (int)a.rows : a.rows <= 4 ? 4 : 8;
  const size_t smem = (size_t)(small::NT / 32) * M * (VE << log_l) * 4;          // (at most 16 KB)
  const cudaError_t e = launch(fn, dim3(blocks), small::NT, smem, 1, s, a, log_l);
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}

typedef void (*OutputsFn)(const small::Args, int, int);
OutputsFn few_outputs_fn(int tiles, int act) {
  return tiles == 1 ? ACT_FN(OutputsFn, small::few_outputs_kernel, act, 1) : ACT_FN(OutputsFn, small::few_outputs_kernel, act, 2);
}
int output_tiles(int N) { return N <= 8 ? 1 : 2; }
size_t outputs_smem(int K, int N) {
  const int t = output_tiles(N);
  return (size_t)((K + 31) / 32) * t * 32 * 16 + (size_t)small::WARPS * 16 * (t * 8 + 1) * 4;
}
// Sizes for which that pass is faster than tiles of 128 x 64 (60000 rows: 256 -> 10 9.9 us against 18, 512 -> 10 16 against 21, 256 -> 16
// 10.3 against 12.3, 512 -> 16 17.2 against 15.4); x has to be on 16 bytes.
bool few_outputs_size(long long rows, int K, int N) { return N <= small::MAX_N && K <= (N % 8 ? 512 : 256) && rows >= 256 && K % 8 == 0; }
int few_outputs(const small::Args& a, int sms, cudaStream_t s) {
  const size_t smem = outputs_smem(a.K, a.N);            // (at most 25 KB)
  const int groups = (int)((a.rows + 15) / 16);
  const int per_sm = (int)((220 * 1024) / (smem + 1024)) < 4 ? (int)((220 * 1024) / (smem + 1024)) : 4;
  const int blocks = (groups + small::WARPS - 1) / small::WARPS, most = sms * per_sm;
  const cudaError_t e = launch(few_outputs_fn(output_tiles(a.N), a.act), dim3((unsigned)(blocks < most ? blocks : most)), small::WARPS * 32, smem, 1, s, a,
                               (a.K + 31) / 32, groups);
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}

int check(long long rows, int n_in, int n_out, int act, int dtype) {
  if (dtype != ABS_FP32 && dtype != ABS_BF16_FP32MASTER) return fail(ABS_EUNSUPPORTED, "unknown dtype %d", dtype);
  if (act < ABS_ACT_NONE || act > ABS_ACT_SILU) return fail(ABS_EUNSUPPORTED, "unknown activation %d", act);
  if (rows < 0 || rows > (1ll << 30)) return fail(ABS_EINVAL, "rows %lld outside [0, 2^30]", rows);
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

// Scratch of a call.  need_*: the operand is copied to a pitch that TMA can address (bf16).
struct FwdPlan { size_t w, part, total, flags; Plan tc; FmaPlan fma; bool pieces; };   // (x comes first)
FwdPlan fwd_plan(long long rows, int n_in, int n_out, int dtype, bool pack_x, bool pack_w) {
  FwdPlan f = {};
  if (dtype == ABS_FP32) {
    f.fma = plan_fma(rows, n_out, n_in);
    f.total = f.fma.part_bytes;
    f.tc = plan_pieces(rows, n_out, n_in);
    const size_t bx = piece_bytes(rows, n_in), bw = piece_bytes(n_in, n_out);
    f.pieces = pieces_fit(rows, n_out, f.tc, bx + bw) && f.tc.t + split_time(bx + bw) < f.fma.t + PLAIN_START;
    if (f.pieces) {
      f.w = bx;
      f.part = bx + bw;
      f.flags = f.part + f.tc.part_bytes;
      f.total = f.flags + FLAG_BYTES;
    }
    return f;
  }
  f.w = pack_x ? pack_bytes(rows, n_in) : 0;
  f.part = f.w + (pack_w ? pack_bytes(n_in, n_out) : 0);
  f.tc = plan_product(rows, n_out, n_in);
  f.total = f.part + f.tc.part_bytes;
  return f;
}
struct GradPlan { size_t dz, sums, x, w, part, total; long long ld_dz; int chunk, chunks; FmaPlan dx, dw, dx2, dw2; Plan tx, tw; bool together, pieces; size_t pz, px, pw, flags; };
GradPlan grad_plan(long long rows, int n_in, int n_out, int dtype, bool need_dz, bool pack_x, bool pack_w) {
  GradPlan g = {};
  const size_t esz = dtype == ABS_FP32 ? 4 : 2;
  // rows whose column sums a CTA adds: enough CTAs for a few on every SM, at most 1024 chunks
  const long long vecs = (n_out + 7) / 8, cols = (vecs + 63) / 64;
  long long chunk = 32;
  while ((rows + chunk - 1) / chunk > 1024 || (rows + chunk - 1) / chunk * cols > 16 * PLAN_SMS) chunk *= 2;
  g.chunk = (int)chunk;
  g.chunks = (int)((rows + chunk - 1) / chunk);
  g.ld_dz = (n_out + 7) / 8 * 8;
  g.sums = need_dz ? round256((size_t)rows * g.ld_dz * esz) : 0;
  g.x = g.sums + round256((size_t)g.chunks * n_out * 4);
  g.w = g.x + (pack_x ? pack_bytes(rows, n_in) : 0);
  g.part = g.w + (pack_w ? pack_bytes(n_in, n_out) : 0);
  size_t a, b;
  if (dtype == ABS_FP32) {
    g.dx = plan_fma(rows, n_in, n_out); g.dw = plan_fma(n_in, n_out, (int)rows);
    g.dx2 = g.dx; g.dw2 = g.dw;
    g.together = plan_fma_pair(rows, n_in, n_out, &g.dx2, &g.dw2);
    a = g.dx.part_bytes; b = g.dw.part_bytes > g.dw2.part_bytes ? g.dw.part_bytes : g.dw2.part_bytes;
    g.tx = plan_pieces(rows, n_in, n_out);
    g.tw = plan_pieces(n_in, n_out, rows);
    const size_t bz = piece_bytes(rows, n_out), bx = piece_bytes(rows, n_in), bw = piece_bytes(n_in, n_out);
    g.pieces = pieces_fit(rows, n_in, g.tx, bz + bx + bw) && pieces_fit(n_in, n_out, g.tw, 0) &&
               g.tx.t + g.tw.t + split_time(bz + bx + bw) < (g.together ? g.dx2.t : g.dx.t + g.dw.t) + PLAIN_START;
    if (g.pieces) {
      g.pz = g.part; g.px = g.pz + bz; g.pw = g.px + bx;
      g.flags = g.pw + bw;
      g.part = g.flags + FLAG_BYTES;
      a = g.tx.part_bytes; b = g.tw.part_bytes;
    }
  } else {
    g.tx = plan_product(rows, n_in, n_out);
    g.tw = plan_product(n_in, n_out, rows);
    a = g.tx.part_bytes; b = g.tw.part_bytes;
  }
  g.total = g.part + (a > b ? a : b);
  return g;
}


}  // namespace

extern "C" int abs_linear_scratch_bytes(long long rows, int n_in, int n_out, int act, int dtype, int grad, int aligned, size_t* out) {
  if (!out) return fail(ABS_EINVAL, "out is null");
  const int rc = check(rows, n_in, n_out, act, dtype);
  if (rc != ABS_OK) return rc;
  *out = 0;
  if (rows == 0) return ABS_OK;
  const bool bf16 = dtype != ABS_FP32, px = bf16 && !(aligned & 1), pw = bf16 && !(aligned & 2), pg = bf16 && !(aligned & 4);
  if (grad) *out = grad_plan(rows, n_in, n_out, dtype, act != ABS_ACT_NONE || pg, px, pw).total;
  else if (rows > few_rows_limit(dtype) && !(bf16 && !px && few_outputs_size(rows, n_in, n_out))) *out = fwd_plan(rows, n_in, n_out, dtype, px, pw).total;
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
  if ((rc = check_vector("bias", bias, esz)) != ABS_OK) return rc;
  if (rows == 1) { ldx = n_in; ldr = ldy = ldp = n_out; }      // (a single row has no pitch)
  if (n_in == 1) ldw = n_out;
  const Span sx = span(x, rows, n_in, ldx, esz), sw = span(w, n_in, n_out, ldw, esz), sb = span(bias, bias ? 1 : 0, n_out, n_out, esz);
  const Span sr = span(residual, residual ? rows : 0, n_out, ldr, esz), sy = span(y, rows, n_out, ldy, esz), sp = span(pre, pre ? rows : 0, n_out, ldp, esz);
  if (overlap(sy, sx) || overlap(sy, sw) || overlap(sy, sb)) return fail(ABS_EINVAL, "y overlaps an operand");
  if (overlap(sp, sx) || overlap(sp, sw) || overlap(sp, sb) || overlap(sp, sr) || overlap(sp, sy)) return fail(ABS_EINVAL, "pre overlaps another matrix");
  if (overlap(sy, sr) && !(y == residual && ldy == ldr)) return fail(ABS_EINVAL, "y overlaps residual without being the same matrix");
  const bool few = rows <= few_rows_limit(dtype), bf16 = dtype != ABS_FP32;
  const bool pack_x = bf16 && !tma_able(x, rows, ldx), pack_w = bf16 && !tma_able(w, n_in, ldw);
  const bool narrow = !few && bf16 && !pack_x && few_outputs_size(rows, n_in, n_out);
  const FwdPlan f = few || narrow ? FwdPlan{} : fwd_plan(rows, n_in, n_out, dtype, pack_x, pack_w);
  if (!bf16 && !few && (rc = check_pitches({ldx, ldw})) != ABS_OK) return rc;
  if ((rc = check_scratch(scratch, scratch_bytes, f.total, {sx, sw, sb, sr, sy, sp})) != ABS_OK) return rc;
  cudaStream_t s = (cudaStream_t)stream;
  int device, sms;
  if ((rc = current_device(&device, &sms)) != ABS_OK) return rc;
  const small::Args sa = {x, w, bias, residual, y, pre, ldx, ldw, ldr, ldy, ldp, rows, n_in, n_out, act};
  if (few) return few_rows(sa, dtype, s);
  if (narrow) return few_outputs(sa, sms, s);
  if (dtype == ABS_FP32) {
    fp32::Args p = {};
    p.a = (const float*)x; p.a_i = ldx; p.a_k = 1;
    p.b = (const float*)w; p.b_k = ldw; p.b_j = 1;
    p.bias = (const float*)bias; p.res = (const float*)residual; p.out = (float*)y; p.pre = (float*)pre;
    p.ldr = ldr; p.ldo = ldy; p.ldp = ldp;
    if (f.pieces) {
      char* sc = (char*)scratch;
      Flags flags = {(uint32_t*)(sc + f.flags), 0};
      const split3::Matrix mx = in_pieces(x, ldx, rows, n_in, sc), mw = in_pieces(w, ldw, n_in, n_out, sc + f.w);
      const cudaError_t e = split({mx, mw}, n_in, &flags, s);
      if (e != cudaSuccess) return fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
      return pieces_product(mx, 0, mw, 1, p, f.tc, (int)rows, n_out, n_in, act, flags, (float*)(sc + f.part), sms, device, s);
    }
    return fma_products({{p, f.fma, (int)rows, n_out, n_in, act, (float*)scratch}}, sms, device, s);
  }
  char* sc = (char*)scratch;
  Operand a = {x, rows, n_in, tma_pitch(rows, n_in, ldx)}, b = {w, n_in, n_out, tma_pitch(n_in, n_out, ldw)};
  if (pack_x) {
    if ((rc = pack(x, rows, n_in, ldx, sc, sms, s)) != ABS_OK) return rc;
    a.p = sc; a.ld = (n_in + 7) / 8 * 8;
  }
  if (pack_w) {
    if ((rc = pack(w, n_in, n_out, ldw, sc + f.w, sms, s)) != ABS_OK) return rc;
    b.p = sc + f.w; b.ld = (n_out + 7) / 8 * 8;
  }
  const Result r = {bias, residual, ldr, y, ldy, pre, ldp, act};
  return tc_product(a, 0, b, 1, (int)rows, n_out, n_in, r, f.tc, false, (float*)(sc + f.part), sms, device, s);
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
  if ((rc = check_vector("db", db, esz)) != ABS_OK) return rc;
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
  if (rows == 1) { lddy = ldp = n_out; ldx = lddx = n_in; }
  if (n_in == 1) ldw = lddw = n_out;
  const Span ins[4] = {span(dy, rows, n_out, lddy, esz), span(x, x ? rows : 0, n_in, ldx, esz), span(w, w ? n_in : 0, n_out, ldw, esz),
                       span(pre, act != ABS_ACT_NONE ? rows : 0, n_out, ldp, esz)};
  const Span outs[3] = {span(dx, dx ? rows : 0, n_in, lddx, esz), span(dw, dw ? n_in : 0, n_out, lddw, esz), span(db, db ? 1 : 0, n_out, n_out, esz)};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 4; ++j)
      if (overlap(outs[i], ins[j])) return fail(ABS_EINVAL, "a gradient overlaps an operand");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return fail(ABS_EINVAL, "two gradients overlap");
  }
  const bool bf16 = dtype != ABS_FP32;
  const bool need_dz = act != ABS_ACT_NONE || (bf16 && (dx || dw) && !tma_able(dy, rows, lddy));
  const bool pack_x = bf16 && dw && !tma_able(x, rows, ldx), pack_w = bf16 && dx && !tma_able(w, n_in, ldw);
  const GradPlan g = grad_plan(rows, n_in, n_out, dtype, need_dz, pack_x, pack_w);
  const long long lddz = need_dz ? g.ld_dz : lddy;
  if (!bf16 && (rc = check_pitches({dx || dw ? lddz : 0, dw ? ldx : 0, dx ? ldw : 0})) != ABS_OK) return rc;
  if ((rc = check_scratch(scratch, scratch_bytes, g.total, {ins[0], ins[1], ins[2], ins[3], outs[0], outs[1], outs[2]})) != ABS_OK) return rc;
  int device, sms;
  if ((rc = current_device(&device, &sms)) != ABS_OK) return rc;
  char* sc = (char*)scratch;
  const void* dz = need_dz ? sc + g.dz : dy;
  const bool with_dw = !bf16 && !g.pieces && dw && db; // the column sums come with the product
  float* part = db && !with_dw ? (float*)(sc + g.sums) : nullptr;
  cudaError_t e = cudaSuccess;
  if (need_dz || part) {
    SlopeArgs q = {dy, pre, need_dz ? (void*)(sc + g.dz) : (void*)nullptr, part, lddy, ldp, lddz, rows, n_out, g.chunk, 0, 0, Divisor()};
    const bool vec = tma_able(dy, rows, lddy * (long long)esz / 2) && (act == ABS_ACT_NONE || tma_able(pre, rows, ldp * (long long)esz / 2)) &&
                     (size_t)n_out * esz % 16 == 0;
    const int VE = vec ? (int)(16 / esz) : 1, vecs = (n_out + VE - 1) / VE;
    q.lv = vecs < 64 ? vecs : 64;
    q.R = 256 / q.lv;
    q.by_lv = Divisor((uint32_t)q.lv);
    e = launch(slope_fn(dtype, vec, act), dim3((unsigned)((vecs + q.lv - 1) / q.lv), (unsigned)g.chunks), 256, 0, 1, s, q);
  }
  if (part && e == cudaSuccess)
    e = launch(dtype == ABS_FP32 ? column_kernel<float> : column_kernel<__nv_bfloat16>, dim3((unsigned)((n_out + 31) / 32)), 256, 0, 1, s,
               (const float*)part, g.chunks, n_out, db);
  if (e != cudaSuccess) return fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
  if (!bf16) {
    const split3::Matrix none = {};
    const split3::Matrix mz = in_pieces(dz, lddz, rows, n_out, sc + g.pz), mx = dw ? in_pieces(x, ldx, rows, n_in, sc + g.px) : none;
    const split3::Matrix mw = dx ? in_pieces(w, ldw, n_in, n_out, sc + g.pw) : none;
    Flags flags = {(uint32_t*)(sc + g.flags), 0};
    if (g.pieces && (dx || dw)) {
      const long long terms = dw && (rows > n_out || !dx) ? rows : n_out;
      e = dx && dw ? split({mz, mx, mw}, terms, &flags, s) : dw ? split({mz, mx}, terms, &flags, s) : split({mz, mw}, terms, &flags, s);
      if (e != cudaSuccess) return fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
    }
    fp32::Args px = {}, pw = {};
    px.a = (const float*)dz; px.a_i = lddz; px.a_k = 1;
    px.b = (const float*)w; px.b_k = 1; px.b_j = ldw;
    px.out = (float*)dx; px.ldo = lddx;
    pw.a = (const float*)x; pw.a_i = 1; pw.a_k = ldx;
    pw.b = (const float*)dz; pw.b_k = lddz; pw.b_j = 1;
    pw.out = (float*)dw; pw.ldo = lddw;
    pw.colsum = with_dw ? (float*)db : nullptr;
    float* sums = (float*)(sc + g.part);
    if (g.pieces) {
      if (dx && (rc = pieces_product(mz, 0, mw, 0, px, g.tx, (int)rows, n_in, n_out, ABS_ACT_NONE, flags, sums, sms, device, s)) != ABS_OK) return rc;
      return dw ? pieces_product(mx, 1, mz, 1, pw, g.tw, n_in, n_out, (int)rows, ABS_ACT_NONE, flags, sums, sms, device, s) : ABS_OK;
    }
    if (dx && dw && g.together)
      return fma_products({{px, g.dx2, (int)rows, n_in, n_out, ABS_ACT_NONE, nullptr}, {pw, g.dw2, n_in, n_out, (int)rows, ABS_ACT_NONE, sums}}, sms, device, s);
    if (dx && (rc = fma_products({{px, g.dx, (int)rows, n_in, n_out, ABS_ACT_NONE, sums}}, sms, device, s)) != ABS_OK) return rc;
    if (dw && (rc = fma_products({{pw, g.dw, n_in, n_out, (int)rows, ABS_ACT_NONE, sums}}, sms, device, s)) != ABS_OK) return rc;
    return ABS_OK;
  }
  const Operand od = {dz, rows, n_out, tma_pitch(rows, n_out, lddz)};
  float* split = (float*)(sc + g.part);
  if (dx) {
    Operand ow = {w, n_in, n_out, tma_pitch(n_in, n_out, ldw)};
    if (pack_w) {
      if ((rc = pack(w, n_in, n_out, ldw, sc + g.w, sms, s)) != ABS_OK) return rc;
      ow.p = sc + g.w; ow.ld = (n_out + 7) / 8 * 8;
    }
    const Result r = {nullptr, nullptr, 0, dx, lddx, nullptr, 0, ABS_ACT_NONE};
    if ((rc = tc_product(od, 0, ow, 0, (int)rows, n_in, n_out, r, g.tx, false, split, sms, device, s)) != ABS_OK) return rc;
  }
  if (dw) {
    Operand ox = {x, rows, n_in, tma_pitch(rows, n_in, ldx)};
    if (pack_x) {
      if ((rc = pack(x, rows, n_in, ldx, sc + g.x, sms, s)) != ABS_OK) return rc;
      ox.p = sc + g.x; ox.ld = (n_in + 7) / 8 * 8;
    }
    const Result r = {nullptr, nullptr, 0, dw, lddw, nullptr, 0, ABS_ACT_NONE};
    if ((rc = tc_product(ox, 1, od, 1, n_in, n_out, rows, r, g.tw, false, split, sms, device, s)) != ABS_OK) return rc;
  }
  return ABS_OK;
}

// One warp waits for an arrival that never comes, as the kernels of these operations wait, and reports it as they do.
namespace {
__global__ void op_wait_selftest_kernel(unsigned* status, unsigned long long limit_ns) {
  __shared__ uint64_t bar;
  __shared__ int gave_up;
  grid_dependency_sync();
  if (threadIdx.x == 0) {
    tc::mbar_init(&bar, 1);
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (threadIdx.x == 0 && !tc::mbar_wait(&bar, 0u, &gave_up, limit_ns)) atomicAdd(status, 1u);
}
}  // namespace

extern "C" int abs_op_selftest_wait_timeout(int limit_us, void* stream) {
  if (limit_us < 1 || limit_us > 1000000) return fail(ABS_EINVAL, "limit_us %d outside [1, 1000000]", limit_us);
  int device, sms;
  const int rc = current_device(&device, &sms);
  if (rc != ABS_OK) return rc;
  unsigned* word = status_word(device);
  if (!word) return fail(ABS_ECUDA, "cudaGetSymbolAddress(status) failed");
  const cudaError_t e = launch(op_wait_selftest_kernel, dim3(1), 32, 0, 1, (cudaStream_t)stream, word, 1000ull * (unsigned long long)limit_us);
  return e == cudaSuccess ? ABS_OK : fail(ABS_ECUDA, "kernel launch: %s", cudaGetErrorString(e));
}

extern "C" int abs_op_status(void* stream) {
  int device, sms;
  const int rc = current_device(&device, &sms);
  if (rc != ABS_OK) return rc;
  unsigned* word = status_word(device);
  if (!word) return fail(ABS_ECUDA, "cudaGetSymbolAddress(status) failed");
  unsigned v = 0;
  cudaError_t e = cudaMemcpyAsync(&v, word, sizeof v, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e != cudaSuccess) return fail(ABS_ECUDA, "status: %s", cudaGetErrorString(e));
  unsigned seen = g_status_seen[device].load();
  while ((int)(v - seen) > 0 && !g_status_seen[device].compare_exchange_weak(seen, v)) {}
  return (int)(v - seen) > 0 ? fail(ABS_ETIMEOUT, "a bounded wait in a layer operation ran out: its results are not valid") : ABS_OK;
}
