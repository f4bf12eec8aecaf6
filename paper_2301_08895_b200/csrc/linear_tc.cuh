// The three products of the affine layer in bf16 on the 5th-generation tensor cores.
//
//   forward     Y[m][n]  = act( sum_k X[m][k] W[k][n] + b[n] ) + R[m][n]      X: k contiguous, W: n contiguous
//   operand     dX[m][k] = sum_n dZ[m][n] W[k][n]                             both: n contiguous
//   weights     dW[k][n] = sum_m X[m][k] dZ[m][n]                             neither: the sum runs over rows
//
// are one kernel: C[i][j] = sum_t A(i, t) B(j, t), each operand either with t contiguous ("K-major": one box of 64 t per
// 128 rows) or with i (j) contiguous ("MN-major": boxes of 64 columns x 64 t).  Both arrive by TMA in the 128-byte swizzle
// that tcgen05.mma reads; sizes that do not fill a tile are filled with zeros by the copies and clipped by the stores.
//
// Products of fp32 matrices come here as three bf16 pieces of each (linear_split.cuh): the sum runs over six pairs of pieces, which lie
// a_step and b_step rows apart.
//
// Persistent and warp-specialised: warp 0 issues the copies of a ring of stages, warp 1 the products into two alternating
// accumulators in tensor memory, warps 2..9 take the other accumulator through the epilogue meanwhile: registers, a box of 32
// rows x 128 bytes per warp in shared memory, one bulk store per box.  CG = 2: a cluster of two CTAs shares a tile of 256 x BN,
// each loads its own rows of A and half of B.  A sum can be split over `splits` tiles that leave fp32 partial results, and products of pieces leave
// tensor memory in stretches (below).
// Every wait is bounded: on expiry the CTA counts up the operations' status word, drains its copies, frees tensor memory and returns.
#pragma once
#include "layerops.cuh"
#include "linear_split.cuh"
#include "tcprim.cuh"

namespace absb {
namespace dense {

using namespace tc;

constexpr int EPI_WARPS = 8;
constexpr int THREADS = 64 + 32 * EPI_WARPS;

// An addition in tensor memory truncates, a step of 2^-23 of the sum towards zero, and in a long sum the steps add up: a product of pieces over 20000
// terms of one sign was off by 9.7e-5.  So products of pieces add up there over a stretch of blocks only; the epilogue's warps take each stretch out
// and add it in registers, rounding to nearest, while the next one runs.  SMALL_STRETCH in the passes of the smaller pairs, whose steps count 2^-7 and
// less, STRETCH in the last pass: with 8, 4 or 2 blocks that product is off by 2.6e-7, 1.4e-7 or 2.0e-7 (one of both signs by 4.9e-7, 2.8e-7 or 2.6e-7
// of its size; on FP32 FMAs 1.1e-6 and 1.8e-6) and takes (2048 x 20000 x 1024) 470, 490 or 515 us, 460 in one stretch.
// A sum in bf16 is rounded by up to 2^-8 and left in one stretch up to LONG_SUM blocks (65536 terms of one sign: off by 4e-4); longer ones go in
// stretches of LONG_STRETCH (off by 8e-6; 134 million terms 1.4e-2 before), which also keeps the epilogue's wait for a stretch below half a millisecond
// (4096 x 65600 x 4096: 1605 us, 1500 in one stretch).
constexpr int SMALL_STRETCH = 64, STRETCH = 4, LONG_SUM = 1024, LONG_STRETCH = 64;      // (stretches: powers of two)

struct Args {
  int a_mn, b_mn;                        // operand layouts: 0 K-major, 1 MN-major
  int I, J, n_kb;                        // rows and columns of C; blocks of 64 terms of the sum
  int splits, kb_per;                    // tiles that share a sum, blocks of each
  int kb_pass, a_step, b_step;           // blocks of one pair of pieces; rows from a piece to the next (0: bf16, one pass)
  int stretch;                           // STRETCHES: blocks of a stretch of the last pass
  int n_it, n_jt, n_tiles;
  // final results (splits = 1)
  const __nv_bfloat16* bias; const __nv_bfloat16* res; __nv_bfloat16* out; __nv_bfloat16* pre;
  long long ldr, ldo, ldp;
  int act, out_tma, pre_tma, res_vec, bias_vec;   // stores by TMA; residual rows, bias on 16-byte boundaries
  int partial;                           // 1: fp32 partial results through map_out instead
  unsigned* status;                      // counts CTAs whose wait ran out
};

template <int BN, int CG> struct Cfg {
  static constexpr int STAGES = (BN == 256 && CG == 1) ? 4 : 6;
  static constexpr int A_BYTES = BM * BK * 2;
  static constexpr int B_BYTES = (BN / CG) * BK * 2;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int TMEM_COLS = 2 * BN;
  static constexpr int OUT_BYTES = EPI_WARPS * 4096;
  static constexpr size_t SMEM_BYTES = (size_t)STAGES * STAGE_BYTES + OUT_BYTES + 1024 /*alignment*/ + 256 /*barriers*/;
};

template <int ACT> __device__ __forceinline__ void activate(float (&z)[64]) {
#pragma unroll
  for (int i = 0; i < 64; ++i) z[i] = layer::act_value<ACT>(z[i]);
}

// lane's row of a swizzled box of 32 rows x 64 bf16
__device__ __forceinline__ void box_put(uint8_t* my_row, int sw, const float (&z)[64]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(z[8 * j + 2 * e], z[8 * j + 2 * e + 1]);
      u[e] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(my_row + ((j ^ sw) << 4)) = make_uint4(u[0], u[1], u[2], u[3]);
  }
}

__device__ __forceinline__ void store_box_2d(const CUtensorMap* map, const void* box, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(box)), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// The box's rows to a matrix that TMA cannot address (row pitch or start not on 16 bytes, a ragged last column): two columns per lane,
// row by row, or, where few columns are left, element by element over all rows.
__device__ __forceinline__ void box_rows_out(const uint8_t* box, int lane, __nv_bfloat16* out, long long ld, int i0, int j0, int I, int J) {
  const int rows = min(32, I - i0), width = J - j0;
  if (width <= 16) {
    int r = lane / width, c = lane - r * width;
    const int dr = 32 / width, dc = 32 - dr * width;
    while (r < rows) {
      out[(long long)(i0 + r) * ld + j0 + c] = *reinterpret_cast<const __nv_bfloat16*>(box + r * 128 + (((c >> 3) ^ (r & 7)) << 4) + ((c & 7) << 1));
      r += dr;
      c += dc;
      if (c >= width) { c -= width; ++r; }
    }
    return;
  }
  const int j = j0 + 2 * lane;
  for (int r = 0; r < rows; ++r) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(box + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + ((lane & 3) << 2));
    __nv_bfloat16* d = out + (long long)(i0 + r) * ld + j;
    const __nv_bfloat162 b = *reinterpret_cast<const __nv_bfloat162*>(&w);
    if (j < J) d[0] = b.x;
    if (j + 1 < J) d[1] = b.y;
  }
}

// First block behind the stretch that starts with block kb, of a tile's blocks in front of `end`.
__device__ __forceinline__ int stretch_end(const Args& p, int kb, int end) {
  const int small = p.n_kb - p.kb_pass;
  if (kb < small) return min(min(kb + SMALL_STRETCH - (kb & (SMALL_STRETCH - 1)), small), end);
  return min(kb + p.stretch - ((kb - small) & (p.stretch - 1)), end);
}

// STRETCHES: sums that leave tensor memory in stretches, partial results: fp32 operands in pieces, long sums in bf16; an own instance, since the
// bookkeeping costs the other bf16 products 3 % (8192 x 4096 x 4096: 205 us for 199, in turn on one box).
template <int BN, int CG, bool STRETCHES>
__global__ void __launch_bounds__(THREADS, 1)
dense_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
             const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_pre, const __grid_constant__ Args p) {
  using C = Cfg<BN, CG>;
  constexpr int ROWS = BM * CG;
  extern __shared__ uint8_t smem_raw[];
  const int rank = (CG == 2) ? (int)cluster_rank() : 0;
  const int unit = (int)blockIdx.x / CG, n_units = (int)gridDim.x / CG;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - smem_u32(smem_raw));
  uint8_t* stage_out = smem + (size_t)C::STAGES * C::STAGE_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(stage_out + C::OUT_BYTES);
  uint64_t* full = bars;                     // [STAGES] bytes landed
  uint64_t* empty = bars + C::STAGES;        // [STAGES] products that read the stage are done
  uint64_t* acc_full = bars + 2 * C::STAGES; // [2] accumulator complete
  uint64_t* acc_empty = acc_full + 2;        // [2] accumulator drained
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], EPI_WARPS * CG); }
    *abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_a); prefetch_map(&map_b); prefetch_map(&map_out);
  }
  if (warp == 1) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::TMEM_COLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::TMEM_COLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();              // the peer's barriers exist before anything signals them
  tc_fence_after();
  const uint32_t full0_addr = (CG == 2) ? map_to_cta(smem_u32(&full[0]), 0) : smem_u32(&full[0]);
  const uint32_t acc_empty0_addr = (CG == 2) ? map_to_cta(smem_u32(&acc_empty[0]), 0) : smem_u32(&acc_empty[0]);
  const uint32_t tmem_base = *tmem_slot;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  struct Tile { int i0, j0, split, kb0, n_kb; };
  auto tile_of = [&](int t) -> Tile {
    Tile c;
    const int per = p.n_it * p.n_jt;
    c.split = t / per;
    const int rem = t - c.split * per;
    const int it = rem / p.n_jt;
    c.i0 = it * ROWS + rank * BM;
    c.j0 = (rem - it * p.n_jt) * BN;
    c.kb0 = c.split * p.kb_per;
    c.n_kb = min(p.kb_per, p.n_kb - c.kb0);      // (at least 1: the host takes no more splits than that)
    return c;
  };

  if (warp == 0) {
    // ------------------------------------------------------------------ copies
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      int armed[C::STAGES];
      for (int s = 0; s < C::STAGES; ++s) armed[s] = -1;
      bool ok = true;
      auto load = [&](void* dst, const CUtensorMap* map, int st, int x, int y) {
        if (CG == 2) tma2_load_2d(dst, map, full0_addr + 8u * (uint32_t)st, x, y);
        else tma_load_2d(dst, map, &full[st], x, y);
      };
      constexpr int BH = BN / CG;
      for (int t = unit; t < p.n_tiles && ok; t += n_units) {
        const Tile c = tile_of(t);
        const int j0 = c.j0 + rank * BH;
        int pass = 0, at = c.kb0, ra = 0, rb = 0;      // pair of pieces, block in its pass, rows to the pieces
        auto pieces = [&] {
          ra = p.a_step * (int)(split3::A_PIECE >> 4 * pass & 15u);
          rb = p.b_step * (int)(split3::B_PIECE >> 4 * pass & 15u);
        };
        if (STRETCHES) {
          pass = at / p.kb_pass;
          at -= pass * p.kb_pass;
          pieces();
        }
        for (int kb = 0; kb < c.n_kb; ++kb) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, abort)) { ok = false; break; }
          uint8_t* sa = smem + (size_t)stage * C::STAGE_BYTES;
          uint8_t* sb = sa + C::A_BYTES;
          if (rank == 0) {
            mbar_expect_tx(&full[stage], CG * C::STAGE_BYTES);
            armed[stage] = (int)phase;
          }
          const int k0 = STRETCHES ? at * BK : (c.kb0 + kb) * BK;
          if (p.a_mn) {
            for (int j = 0; j < BM / 64; ++j) load(sa + j * 8192, &map_a, stage, c.i0 + 64 * j, k0 + ra);
          } else {
            load(sa, &map_a, stage, k0, c.i0 + ra);
          }
          if (p.b_mn) {
            for (int j = 0; j < BH / 64; ++j) load(sb + j * 8192, &map_b, stage, j0 + 64 * j, k0 + rb);
          } else {
            load(sb, &map_b, stage, k0, j0 + rb);
          }
          if (STRETCHES && ++at == p.kb_pass) {
            at = 0;
            ++pass;
            pieces();
          }
          if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
        }
      }
      // every stage's release must have landed before this CTA's shared memory goes away
      for (int s = 0; s < C::STAGES && ok; ++s) {
        if (!mbar_wait(&empty[stage], phase ^ 1u, abort)) ok = false;
        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
      }
      if (!ok) {
        for (int s = 0; s < C::STAGES; ++s)
          if (armed[s] >= 0) {
            const unsigned long long t0 = global_ns();
            while (!mbar_test(&full[s], (uint32_t)armed[s]) && global_ns() - t0 < WAIT_LIMIT_NS) {}
          }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    if (lane == 0 && rank == 0) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      const uint32_t idesc = instr_desc(p.a_mn, p.b_mn, BN, ROWS);
      const uint32_t a_lbo = p.a_mn ? 8192u : 16u, b_lbo = p.b_mn ? 8192u : 16u;
      const uint32_t a_kstep = p.a_mn ? 2048u : 32u, b_kstep = p.b_mn ? 2048u : 32u;
      for (int t = unit; t < p.n_tiles && ok; t += n_units) {
        const Tile c = tile_of(t);
        for (int kb = 0; kb < c.n_kb && ok;) {
          const int first = kb, stop = STRETCHES ? stretch_end(p, c.kb0 + kb, c.kb0 + c.n_kb) - c.kb0 : c.n_kb;
          if (!mbar_wait(&acc_empty[acc], acc_phase ^ 1u, abort)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + (uint32_t)(acc * BN);
          for (; kb < stop; ++kb) {
            if (!mbar_wait(&full[stage], phase, abort)) { ok = false; break; }
            tc_fence_after();
            const uint32_t sa = base + (uint32_t)stage * C::STAGE_BYTES, sb = sa + C::A_BYTES;
#pragma unroll
            for (int kk = 0; kk < BK / UK; ++kk) {
              const uint64_t da = smem_desc(sa + kk * a_kstep, a_lbo, 1024u);
              const uint64_t db = smem_desc(sb + kk * b_kstep, b_lbo, 1024u);
              if (CG == 2) umma2(d_tmem, da, db, idesc, (kb > first || kk > 0) ? 1u : 0u);
              else umma(d_tmem, da, db, idesc, (kb > first || kk > 0) ? 1u : 0u);
            }
            if (CG == 2) umma2_commit_both(&empty[stage]);
            else umma_commit(&empty[stage]);
            if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
          }
          if (!ok) break;
          if (CG == 2) umma2_commit_both(&acc_full[acc]);
          else umma_commit(&acc_full[acc]);
          acc ^= 1;
          if (acc == 0) acc_phase ^= 1u;
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    const int q = warp & 3;                    // tensor-memory lane quarter this warp may read
    const int half = (warp - 2) >> 2;
    constexpr int N_HALF = (BN >= 128) ? 2 : 1;
    constexpr int HALF_COLS = BN / N_HALF;
    const bool works = half < N_HALF;
    const int sw = lane & 7;
    uint8_t* my_box = stage_out + ((warp - 2) << 12);
    uint8_t* my_row = my_box + lane * 128;
    int acc = 0;
    uint32_t acc_phase = 0;
    auto release = [&] {                       // the accumulator is drained; its barrier lives in the leader CTA
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CG == 2) mbar_arrive_cluster(acc_empty0_addr + 8u * (uint32_t)acc);
        else mbar_arrive(&acc_empty[acc]);
      }
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
    };
    auto partial_box = [&](const uint32_t* v, int col, int row0, int split) {      // 32 columns of a partial result
      if (lane == 0) bulk_wait_read();         // the box is free once the store issued from it has read it
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<uint4*>(my_row + ((j ^ sw) << 4)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
      fence_async();
      __syncwarp();
      if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                     ::"l"(reinterpret_cast<uint64_t>(&map_out)), "r"(smem_u32(my_box)), "r"(col), "r"(row0), "r"(split) : "memory");
        bulk_commit();
      }
    };
    for (int t = unit; t < p.n_tiles; t += n_units) {
      const Tile c = tile_of(t);
      const int row0 = c.i0 + q * 32, row = row0 + lane;
      if constexpr (STRETCHES) {
        const int j0 = c.j0 + half * HALF_COLS;
        constexpr int LD = HALF_COLS < 128 ? 64 : 32;      // (columns under way: 168 registers)
        uint32_t sum[HALF_COLS];               // (binary32)
#pragma unroll
        for (int i = 0; i < HALF_COLS; ++i) sum[i] = 0u;
        bool ok = true;
        for (int kb = 0; kb < c.n_kb;) {
          kb = stretch_end(p, c.kb0 + kb, c.kb0 + c.n_kb) - c.kb0;
          ok = mbar_wait(&acc_full[acc], acc_phase, abort);
          if (!ok) break;
          tc_fence_after();
          if (works && row0 < p.I) {           // (uniform in the warp)
            const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN + half * HALF_COLS);
#pragma unroll
            for (int c0 = 0; c0 < HALF_COLS; c0 += LD)
              if (j0 + c0 < p.J) {
                uint32_t v[LD];
                if constexpr (LD == 64) tmem_ld64(t_row + (uint32_t)c0, v);
                else tmem_ld32(t_row + (uint32_t)c0, v);
#pragma unroll
                for (int i = 0; i < LD; ++i) sum[c0 + i] = __float_as_uint(__uint_as_float(sum[c0 + i]) + __uint_as_float(v[i]));
              }
          }
          release();
        }
        if (!ok) break;
        if (works && row0 < p.I) {
#pragma unroll
          for (int c0 = 0; c0 < HALF_COLS; c0 += 32)
            if (j0 + c0 < p.J) partial_box(&sum[c0], j0 + c0, row0, c.split);
        }
        continue;
      }
      if (!mbar_wait(&acc_full[acc], acc_phase, abort)) break;
      tc_fence_after();
      const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN);
      if (works && row0 < p.I) {               // (uniform in the warp)
        if (p.partial) {
#pragma unroll 1
          for (int c0 = half * HALF_COLS; c0 < (half + 1) * HALF_COLS && c.j0 + c0 < p.J; c0 += 32) {
            uint32_t v[32];
            tmem_ld32(t_row + (uint32_t)c0, v);
            partial_box(v, c.j0 + c0, row0, c.split);
          }
        } else {
#pragma unroll 1
          for (int c0 = half * HALF_COLS; c0 < (half + 1) * HALF_COLS && c.j0 + c0 < p.J; c0 += 64) {
            const int j0 = c.j0 + c0;
            // (a bulk store leaves out what lies behind the last column in units of 16 bytes only)
            const bool whole = j0 + 64 <= p.J || (p.J & 7) == 0;
            uint4 rv[8];
            const bool res_fast = p.res != nullptr && p.res_vec && j0 + 64 <= p.J;
            if (res_fast) {
              const uint4* r = reinterpret_cast<const uint4*>(p.res + (long long)row * p.ldr + j0);
#pragma unroll
              for (int j = 0; j < 8; ++j) rv[j] = row < p.I ? r[j] : make_uint4(0u, 0u, 0u, 0u);
            }
            float z[64];
            {
              uint32_t v[32];
              tmem_ld32(t_row + (uint32_t)c0, v);
#pragma unroll
              for (int i = 0; i < 32; ++i) z[i] = __uint_as_float(v[i]);
              tmem_ld32(t_row + (uint32_t)(c0 + 32), v);
#pragma unroll
              for (int i = 0; i < 32; ++i) z[32 + i] = __uint_as_float(v[i]);
            }
            if (p.bias_vec && j0 + 64 <= p.J) {      // (the same addresses in all lanes)
#pragma unroll
              for (int i = 0; i < 64; i += 8) {
                float b[8];
                layer::Pack<__nv_bfloat16, 8> bp;
                bp.load(p.bias + j0 + i);
                bp.get(b);
#pragma unroll
                for (int e = 0; e < 8; ++e) z[i + e] += b[e];
              }
            } else if (p.bias != nullptr) {
#pragma unroll
              for (int i = 0; i < 64; ++i) z[i] += j0 + i < p.J ? __bfloat162float(p.bias[j0 + i]) : 0.f;
            }
            if (lane == 0) bulk_wait_read();
            __syncwarp();
            if (p.pre != nullptr) {
              box_put(my_row, sw, z);
              if (p.pre_tma && whole) {
                fence_async();
                __syncwarp();
                if (lane == 0) { store_box_2d(&map_pre, my_box, j0, row0); bulk_commit(); }
              } else {
                __syncwarp();
                box_rows_out(my_box, lane, p.pre, p.ldp, row0, j0, p.I, p.J);
              }
            }
            if (p.act == ABS_ACT_RELU) activate<ABS_ACT_RELU>(z);
            else if (p.act == ABS_ACT_GELU) activate<ABS_ACT_GELU>(z);
            else if (p.act == ABS_ACT_SILU) activate<ABS_ACT_SILU>(z);
            if (res_fast) {
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const uint32_t u[4] = {rv[j].x, rv[j].y, rv[j].z, rv[j].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  z[8 * j + 2 * e] += __uint_as_float(u[e] << 16);
                  z[8 * j + 2 * e + 1] += __uint_as_float(u[e] & 0xffff0000u);
                }
              }
            } else if (p.res != nullptr && row < p.I) {
              const __nv_bfloat16* r = p.res + (long long)row * p.ldr + j0;
#pragma unroll
              for (int i = 0; i < 64; ++i)
                if (j0 + i < p.J) z[i] += __bfloat162float(r[i]);
            }
            if (p.pre != nullptr) {
              if (lane == 0) bulk_wait_read();
              __syncwarp();
            }
            box_put(my_row, sw, z);
            if (p.out_tma && whole) {
              fence_async();
              __syncwarp();
              if (lane == 0) { store_box_2d(&map_out, my_box, j0, row0); bulk_commit(); }
            } else {
              __syncwarp();
              box_rows_out(my_box, lane, p.out, p.ldo, row0, j0, p.I, p.J);
              __syncwarp();
            }
          }
        }
      }
      release();
    }
    if (lane == 0) bulk_wait_read();           // shared memory may go once the stores have read it
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();              // neither CTA leaves while the pair still uses its memory
  if (warp == 1) {
    tc_fence_after();
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
  }
  if (threadIdx.x == 0 && *abort) atomicAdd(p.status, 1u);
}

}  // namespace dense
}  // namespace absb
