// The products of the affine layer in fp32, on FP32 FMAs (no rounding of operands), two per instruction.
//
// C[i][j] = sum_k A(i, k) B(k, j); either operand has its sum index or its other index contiguous.  A CTA of 256 threads takes a
// BM x BN tile; blocks of 32 k are copied a few ahead by 4-byte asynchronous copies, which take any pitch and alignment, put both
// operands k-major into shared memory and fill what lies outside with zeros.  A thread holds 8 x 8 sums as pairs of neighbouring j: a
// k costs four 16-byte shared loads and eight doublings of an operand of A per 32 packed FMAs.  (Products alone, without copies, by a
// loop over shared memory: 61 TFLOP/s in this form, 59 with single FMAs, 50 to 57 with pairs of even and odd k, which need no doubling.)
// 64 x 64 tiles have four groups of 64 threads that take eight k of a block each (KG = 4), added at
// the end; and a cluster of Q CTAs can share a tile's sum: each leaves its part in shared memory, takes 1 / Q of the tile's rows,
// adds the parts in the order of the ranks and applies the epilogue.  A long sum of few tiles is cut into parts besides, which a second
// kernel adds.
#pragma once
#include "layerops.cuh"
#include "linear_split.cuh"

namespace absb {
namespace fp32 {

constexpr int NT = 256, BK = 32;

struct Args {
  const float* a; const float* b;
  long long a_i, a_k, b_k, b_j;          // element pitches; one of each pair is 1
  int I, J, K;
  int n_jt, Q, kb_per, n_kb;             // column tiles; CTAs per tile, blocks of 32 k of each
  const float* bias; const float* res; float* out; float* pre;
  long long ldr, ldo, ldp;
  float* colsum;                         // sums of B's columns (null: none), by the CTAs of the first row tile
  long long out_step; int col_step;      // part number s of a sum cut in parts goes to out + s out_step, colsum + s col_step
  layer::Divisor by_Q, by_njt, by_tiles; // by_tiles: tiles of one part
  const uint32_t* flags; int n_flags;    // if given and none is raised: the sums are ready, `parts` of them, [parts][I][J to a multiple of 4]
  const float* sums; int parts, vec;     // vec: rows of res, out and pre start on 16 bytes
};

struct Pair { Args a[2]; uint32_t first; };          // CTAs of the first product; those behind them work on the second

template <int BM, int BN> struct Cfg {
  static constexpr int LDA = BM + 4, LDB = BN + 4;       // (4 modulo 32; with the swizzle no bank is hit twice, or twice at most)
  static constexpr int STAGES = 3;
  static constexpr int KG = NT / ((BM / 8) * (BN / 8));
  static constexpr int STAGE = BK * (LDA + LDB);
  static constexpr int RING = STAGES * STAGE, PARTS = KG * BM * BN + BN;           // floats: stages; the groups' sums, column sums
  static constexpr size_t SMEM = (size_t)(RING > PARTS ? RING : PARTS) * 4;
};

// Shared memory holds element (k, x) of an operand at [k][x ^ swizzle(k)]: where the sum index is contiguous in memory, a warp copies 32 k
// of one x (whole lines), and would hit the same eight banks four times over.  Neighbouring pairs of B's columns stay pairs.
__host__ __device__ constexpr int swizzle_a(int k) { return k >> 3; }
__host__ __device__ constexpr int swizzle_b(int k) { return (k >> 4) << 1; }

// This thread's part of one operand's copies: element n of a block goes from src + n * hop to its place in the tile.
template <int W, bool B> struct Mover {
  static constexpr int N = BK * W / NT, LD = W + 4;
  static constexpr uint32_t ALL = N == 32 ? 0xffffffffu : (1u << N) - 1u;
  const float* src;
  long long advance;
  int hop;                               // (a pitch that does not fit is refused by the host)
  int k, x0;                             // k of element 0 inside a block, index along the tile of element 0
  uint32_t rows;                         // k contiguous: which elements lie inside the matrix; else all or none
  bool kmajor;
  // X: elements of the matrix from the tile's start on
  __device__ __forceinline__ Mover(const float* base, long long px, long long pk, long long x_tile, int X) {
    kmajor = pk == 1;
    if (kmajor) {                        // element n: x0 + 8 n
      k = threadIdx.x & 31;
      x0 = threadIdx.x >> 5;
      hop = 8 * (int)px;
      const int n = x0 < X ? (X - x0 + 7) / 8 : 0;
      rows = n >= N ? ALL : (1u << n) - 1u;
    } else {                             // element n: k + (NT / W) n
      x0 = (int)threadIdx.x % W;
      k = (int)threadIdx.x / W;
      hop = (NT / W) * (int)pk;
      rows = x0 < X ? ALL : 0u;
    }
    src = base + (x_tile + x0) * px + (long long)k * pk;
    advance = BK * pk;
  }
  __device__ __forceinline__ void copy(float* tile, const float* any, int kb, int K) const {
    const float* s = src + (long long)kb * advance;
    const int left = K - kb * BK - k;    // (elements of the sum from this thread's first one on)
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(tile);
    if (kmajor) {
      const uint32_t d0 = d + 4u * (uint32_t)(k * LD + (x0 ^ (B ? swizzle_b(k) : swizzle_a(k))));
      put(s, any, left > 0 ? rows : 0u, [&](int n) { return d0 + 32u * (uint32_t)n; });
    } else {
      uint32_t in = rows;
      if (left < BK) {
        const int n = left > 0 ? (left + NT / W - 1) / (NT / W) : 0;
        in = n >= N ? in : in & ((1u << n) - 1u);
      }
      const uint32_t d0 = d + 4u * (uint32_t)(k * LD);
      put(s, any, in, [&](int n) {       // (k < NT / W <= 4 does not reach the swizzle's bits)
        const int up = (NT / W) * n;
        return d0 + 4u * (uint32_t)(up * LD + (x0 ^ (B ? swizzle_b(up) : swizzle_a(up))));
      });
    }
  }
  template <typename F> __device__ __forceinline__ void put(const float* s, const float* any, uint32_t in, F at) const {
    if (in == ALL) {
#pragma unroll
      for (int n = 0; n < N; ++n) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at(n)), "l"(s + (long long)hop * n) : "memory");
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;"
                     ::"r"(at(n)), "l"(in >> n & 1u ? s + (long long)hop * n : any), "r"(in >> n & 1u ? 4 : 0) : "memory");
    }
  }
};

// The epilogue of a tile whose sums are ready, in groups of four columns; the CTAs of a cluster take turns.
template <int BN, int ACT> __device__ __noinline__ void finish_tile(const Args& p, long long i0, int j0, int X, int Y, int rank) {
  constexpr int U = 4, PER = BN / 4;
  const long long pitch = (p.J + 3) / 4 * 4, step = p.I * pitch;
  const int j = j0 + (int)threadIdx.x % PER * 4, left = Y - (int)threadIdx.x % PER * 4;       // (NT is a multiple of PER: the same columns all the way)
  if (left <= 0) return;
  const bool vec = p.vec && left >= 4;
  float bias[4] = {0.f, 0.f, 0.f, 0.f};
  if (p.bias)
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[e] = e < left ? p.bias[j + e] : 0.f;
  const int hop = NT / PER * p.Q;
#pragma unroll 1
  for (int r0 = (int)threadIdx.x / PER + rank * (NT / PER); r0 < X; r0 += U * hop) {
    float4 z[U], res[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * hop;
      z[u] = res[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r >= X) continue;
      const long long i = i0 + r;
      z[u] = *reinterpret_cast<const float4*>(p.sums + i * pitch + j);
      if (p.res) {
        const float* s = p.res + i * p.ldr + j;
        if (vec) res[u] = *reinterpret_cast<const float4*>(s);
        else res[u] = make_float4(s[0], left > 1 ? s[1] : 0.f, left > 2 ? s[2] : 0.f, left > 3 ? s[3] : 0.f);
      }
    }
    for (int k = 1; k < p.parts; ++k)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + u * hop;
        if (r >= X) continue;
        const float4 o = *reinterpret_cast<const float4*>(p.sums + k * step + (i0 + r) * pitch + j);
        z[u].x += o.x; z[u].y += o.y; z[u].z += o.z; z[u].w += o.w;
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * hop;
      if (r >= X) continue;
      const long long i = i0 + r;
      const float v[4] = {fmaf(z[u].x, split3::DOWN, bias[0]), fmaf(z[u].y, split3::DOWN, bias[1]), fmaf(z[u].z, split3::DOWN, bias[2]),
                          fmaf(z[u].w, split3::DOWN, bias[3])};
      const float y[4] = {layer::act_value<ACT>(v[0]) + res[u].x, layer::act_value<ACT>(v[1]) + res[u].y, layer::act_value<ACT>(v[2]) + res[u].z,
                          layer::act_value<ACT>(v[3]) + res[u].w};
      float* out = p.out + i * p.ldo + j;
      float* pre = p.pre ? p.pre + i * p.ldp + j : nullptr;
      if (vec) {
        if (pre) *reinterpret_cast<float4*>(pre) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(out) = make_float4(y[0], y[1], y[2], y[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < left) {
            if (pre) pre[e] = v[e];
            out[e] = y[e];
          }
      }
    }
  }
}

template <int BM, int BN, int ACT>
__global__ void __launch_bounds__(NT, 2) fma_kernel(const __grid_constant__ Pair pair) {
  using C = Cfg<BM, BN>;
  constexpr int STAGES = C::STAGES, KG = C::KG, KPG = BK / KG, TX = BN / 8;
  extern __shared__ __align__(16) float sm[];
  const bool second = blockIdx.x >= pair.first;
  const Args& p = pair.a[second];
  const uint32_t block = second ? blockIdx.x - pair.first : blockIdx.x;
  const uint32_t work = p.by_Q.div(block), part = p.out_step ? p.by_tiles.div(work) : 0u, tile = work - part * p.by_tiles.d;
  const int rank = (int)(block - work * p.by_Q.d);
  const uint32_t it = p.by_njt.div(tile);
  const long long i0 = (long long)it * BM;
  const int j0 = (int)(tile - it * p.by_njt.d) * BN;
  const int kb0 = ((int)part * p.Q + rank) * p.kb_per, nkb = min(p.kb_per, p.n_kb - kb0);
  grid_dependency_sync();
  const int X = (int)min((long long)BM, p.I - i0), Y = min(BN, p.J - j0);
  if (p.flags && !split3::any_flag(p.flags, p.n_flags)) {          // (the whole grid alike)
    finish_tile<BN, ACT>(p, i0, j0, X, Y, rank);
    return;
  }
  const Mover<BM, false> ma(p.a, p.a_i, p.a_k, i0, X);
  const Mover<BN, true> mb(p.b, p.b_j, p.b_k, j0, Y);
  auto fetch = [&](int kb) {
    if (kb < nkb) {
      float* st = sm + (kb % STAGES) * C::STAGE;
      ma.copy(st, p.a, kb0 + kb, p.K);
      mb.copy(st + BK * C::LDA, p.b, kb0 + kb, p.K);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const int g = (int)threadIdx.x / (NT / KG), t = (int)threadIdx.x % (NT / KG);
  const int tx = t % TX, ty = t / TX;
  layer::Lanes<2> acc[8][4];
#pragma unroll
  for (int u = 0; u < 8; ++u)
#pragma unroll
    for (int v = 0; v < 4; ++v) acc[u][v].fill(0.f);
  float cs = 0.f;
  const bool sums = p.colsum != nullptr && it == 0 && (int)threadIdx.x < BN;
#pragma unroll 1
  for (int kb = 1 - STAGES; kb < nkb; ++kb) {                    // (the first steps only fetch: one copy of that code)
    if (kb >= 0) {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      __syncthreads();                   // the block is there, and everybody has left the one that is overwritten next
    }
    fetch(kb + STAGES - 1);
    if (kb < 0) continue;
    const float* sa = sm + (kb % STAGES) * C::STAGE + g * KPG * C::LDA + 4 * ty;
    const float* sb = sm + (kb % STAGES) * C::STAGE + BK * C::LDA + g * KPG * C::LDB + 4 * tx;
    // eight k have one swizzle: with one group of threads it is known here, with four it is the group's and goes into row_of, col_of
#pragma unroll
    for (int o = 0; o < KPG / 8; ++o) {
      const int xa = KG == 1 ? swizzle_a(8 * o) : 0, xb = KG == 1 ? swizzle_b(8 * o) >> 1 : 0;
#pragma unroll
      for (int k = 0; k < 8; ++k, sa += C::LDA, sb += C::LDB) {
        const float4 a0 = *reinterpret_cast<const float4*>(sa), a1 = *reinterpret_cast<const float4*>(sa + BM / 2);
        layer::Lanes<4> b0, b1;
        b0.load(sb);
        b1.load(sb + BN / 2);
        const float av[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
        layer::Lanes<2> bv[4];
        bv[0].p[0] = b0.p[0]; bv[1].p[0] = b0.p[1]; bv[2].p[0] = b1.p[0]; bv[3].p[0] = b1.p[1];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          layer::Lanes<2> aa;
          aa.fill(av[(u & 4) | ((u & 3) ^ xa)]);
#pragma unroll
          for (int v = 0; v < 4; ++v) acc[u][v] = layer::fma(aa, bv[(v & 2) | ((v & 1) ^ xb)], acc[u][v]);
        }
      }
    }
    if (sums) {
      const float* col = sm + (kb % STAGES) * C::STAGE + BK * C::LDA;
#pragma unroll 8
      for (int k = 0; k < BK; ++k) cs += col[k * C::LDB + ((int)threadIdx.x ^ swizzle_b(k))];
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();

  // every group of threads leaves its sums, then all threads add them up (in place of the first group's): sm[BM][BN]
  float* tile_sm = sm;
  float* cs_sm = sm + KG * BM * BN;      // [BN]
  {
    const int ga = KG == 1 ? 0 : swizzle_a(g * KPG), gb = KG == 1 ? 0 : swizzle_b(g * KPG) >> 1;
    float* mine = sm + g * BM * BN + tx * 4;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      float* row = mine + ((u < 4 ? 0 : BM / 2) + ty * 4 + ((u & 3) ^ ga)) * BN;
#pragma unroll
      for (int v = 0; v < 4; v += 2) {
        layer::Lanes<4> q;
        q.p[0] = gb ? acc[u][v + 1].p[0] : acc[u][v].p[0];
        q.p[1] = gb ? acc[u][v].p[0] : acc[u][v + 1].p[0];
        q.store(row + (v < 2 ? 0 : BN / 2));
      }
    }
  }
  if (sums) cs_sm[threadIdx.x] = cs;
  if (KG > 1) {
    __syncthreads();
#pragma unroll
    for (int e = (int)threadIdx.x * 4; e < BM * BN; e += NT * 4) {
      layer::Lanes<4> z;
      z.load(sm + e);
#pragma unroll
      for (int h = 1; h < KG; ++h) {
        layer::Lanes<4> o;
        o.load(sm + h * BM * BN + e);
        z = layer::add(z, o);
      }
      z.store(sm + e);
    }
  }
  if (p.Q > 1) {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
  const int share = (BM + p.Q - 1) / p.Q, r0 = rank * share, r1 = min(min(BM, r0 + share), X);
  // a few elements at a time, all their loads in front of the first store (which the compiler has to take for an alias of theirs)
  auto finish = [&](int e, const float z, float bias, float res) {
    const int r = r0 + e / BN, c = e % BN;
    const long long i = i0 + r;
    const float v = z + bias;
    if (p.pre) p.pre[i * p.ldp + j0 + c] = v;
    p.out[part * p.out_step + i * p.ldo + j0 + c] = layer::act_value<ACT>(v) + res;
  };
  constexpr int U = 4;
#pragma unroll 1
  for (int e0 = (int)threadIdx.x; e0 < (r1 - r0) * BN; e0 += U * NT) {
    float z[U], bias[U], res[U];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = e0 + u * NT, r = r0 + e / BN, c = e % BN;
      in[u] = r < r1 && c < Y;
      z[u] = in[u] && p.Q == 1 ? tile_sm[r * BN + c] : 0.f;
      bias[u] = in[u] && p.bias ? p.bias[j0 + c] : 0.f;
      res[u] = in[u] && p.res ? p.res[(i0 + r) * p.ldr + j0 + c] : 0.f;
    }
    if (p.Q > 1) {
#pragma unroll 4
      for (int q = 0; q < p.Q; ++q)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (in[u]) z[u] += ld_peer(tile_sm + r0 * BN + e0 + u * NT, q);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (in[u]) finish(e0 + u * NT, z[u], bias[u], res[u]);
  }
  if (sums && rank == 0 && (int)threadIdx.x < Y) {
    float z = cs;
    for (int q = 1; q < p.Q; ++q) z += ld_peer(cs_sm + threadIdx.x, q);
    p.colsum[(size_t)part * p.col_step + j0 + threadIdx.x] = z;
  }
  if (p.Q > 1) {                         // nobody leaves while a peer reads its part
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}

}  // namespace fp32
}  // namespace absb
