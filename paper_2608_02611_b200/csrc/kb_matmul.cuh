// Product of two 8-bit matrices with a binary32 scale per block of 128 along K (contract in
// include/kb_ops.h):
//     D[m][n] = sum_kb SA[kb][m] * SB[kb][n or n/128] * sum_{k in kb} A[m][k] * B[n][k]
//
// The scales differ from one K block of 128 to the next, so the tensor cores cannot add across
// blocks: each block's 128-deep product goes to an accumulator of its own in tensor memory, and
// the epilogue warps multiply it with its scales and add it to running sums in registers while
// the tensor cores are at the next blocks.  K blocks are also the unit of the copies: a stage of
// the shared-memory ring is one block of both operands, 128 bytes per row in the 128-byte
// swizzle, and takes 4 matrix instructions.
//
// Roles: warp 0 copies (tensor maps; rows and columns outside a matrix read as zero), warp 1 (and 3
// in the pair kernel) issues matrix instructions, warp 2 fetches scales (and, in the pair kernel, sees to
// the rows with extreme scales at the end), warps from 4 on scale and add.  Every wait on a barrier in
// shared memory is bounded.
#pragma once

#include "kb_block8.cuh"
#include "kb_tcgen05.cuh"

namespace kb {

struct MatmulParams {
  const float* a_scale;      // [KB][M]
  const float* b_scale;      // [KB][N] or [KB][ceil(N/128)]
  void* d;
  uint64_t ldd;
  uint32_t M, N, KB;
  uint32_t b_scale_ld;       // N or ceil(N/128)
  uint32_t b_scale_shift;    // 0 or 7
  uint32_t tiles_m;          // column tiles (of A's rows)
  uint32_t splits;           // CTAs per tile along K (a cluster)
  uint32_t idesc;
  const unsigned char* a;    // the codes themselves, for the rows that recompute_wide_rows takes
  const unsigned char* b;
  uint64_t lda, ldb;
  uint32_t K;
  bool a_e5m2, b_e5m2;
  int out;                   // kb_dtype of D
  bool vec_out;              // rows of D start on 16-byte boundaries
  unsigned int* status;
};

// v[0..n) to column `col` of the rows row0, row0 + 1, ... of D, where they exist
template <int DT, int N>
__device__ __forceinline__ void store_down(const MatmulParams& p, uint32_t row0, uint32_t col, const float* v) {
  constexpr int kBytes = DT == KB_F32 ? 4 : 2;
  unsigned char* at = static_cast<unsigned char*>(p.d) + ((uint64_t)row0 * p.ldd + col) * kBytes;
  const uint64_t step = p.ldd * kBytes;
#pragma unroll
  for (int j = 0; j < N; ++j, at += step)
    if (row0 + j < p.M) store_elem<DT>(at, 0, v[j]);
}
template <int N>
__device__ __forceinline__ void store_down(const MatmulParams& p, uint32_t row0, uint32_t col, const float* v) {
  if (p.out == KB_BF16)
    store_down<KB_BF16, N>(p, row0, col, v);
  else if (p.out == KB_F16)
    store_down<KB_F16, N>(p, row0, col, v);
  else
    store_down<KB_F32, N>(p, row0, col, v);
}

// After a wait has run out: let the copies already issued land, for a second at most.
__device__ __forceinline__ void drain_copies(uint64_t* full, uint32_t stages, uint64_t issued) {
  const uint64_t back = issued < stages ? issued : stages;
  for (uint64_t m = issued - back; m < issued; ++m) {
    const unsigned long long t0 = global_ns();
    while (!mbar_try_wait(&full[m % stages], (uint32_t)((m / stages) & 1ull)))
      if (global_ns() - t0 > 1000000000ull) break;
  }
}

// ---- few rows of A ---------------------------------------------------------------------------
// The rows of B (weights) take the 128 lanes of the tile and BN rows of A its columns, so that a
// single token wastes no lanes and the weights stream through once.  A cluster of `splits` CTAs
// shares a tile's K blocks; the partial sums are added over distributed shared memory in rank
// order.  Bound by the weights' bytes: 16 KB of weights per K block and CTA, up to ten blocks on
// their way.  The scales come through a ring of their own, several blocks ahead: fetched when they
// are needed, their latency would stand in every block.
constexpr uint32_t kScaleStep = 4;          // K blocks whose scales share a slot of shared memory
template <int BN>
struct LaneTile {
  static constexpr uint32_t kStageBytes = (128 + BN) * 128;
  static constexpr uint32_t kStages = BN == 128 ? 4 : BN == 64 ? 6 : 9;
  static constexpr uint32_t kAcc = BN == 128 ? 2 : 4;          // accumulators in tensor memory
  static constexpr uint32_t kTmemCols = kAcc * BN;
  // the cluster's partial sums for this CTA's share of the columns, 8 CTAs at most
  // (in groups of 4 columns: 16 bytes per row)
  static constexpr uint32_t kGroups = BN / 4;
  static constexpr uint32_t kSumBytes = (kGroups + 8) * 2048;
  static constexpr uint32_t kSmem = 1024 + kStages * kStageBytes + kSumBytes;
  static constexpr uint32_t kScaleSlots = 4;
  static constexpr int kEpiWarps = BN >= 64 ? 8 : 4;           // each adds 32 rows x kEpiCols columns
  static constexpr int kEpiCols = BN / (kEpiWarps / 4);
  static constexpr int kThreads = 32 * (4 + kEpiWarps);        // and four warps that copy, issue, fetch scales
};

// A cluster of `splits` CTAs divides a tile's `groups` of columns: CTA o finishes those from cluster_first(o) up
// to cluster_first(o + 1), none if they are equal, and holds cluster_share places for each CTA's part.
__host__ __device__ constexpr uint32_t cluster_first(uint32_t groups, uint32_t splits, uint32_t o) {
  return (groups * o + splits - 1) / splits;
}
__host__ __device__ constexpr uint32_t cluster_owner(uint32_t groups, uint32_t splits, uint32_t g) { return g * splits / groups; }
__host__ __device__ constexpr uint32_t cluster_share(uint32_t groups, uint32_t splits) { return (groups + splits - 1) / splits; }

// c0 += v0 * s0, c1 += v1 * s1 as one packed instruction
__device__ __forceinline__ void fma_pair(float& c0, float& c1, float v0, float v1, float s0, float s1) {
  asm("{\n.reg .b64 c, v, s;\n"
      "mov.b64 c, {%0, %1};\nmov.b64 v, {%2, %3};\nmov.b64 s, {%4, %5};\n"
      "fma.rn.f32x2 c, v, s, c;\nmov.b64 {%0, %1}, c;\n}"
      : "+f"(c0), "+f"(c1)
      : "f"(v0), "f"(v1), "f"(s0), "f"(s1));
}

// ---- scales at the ends of binary32's range ------------------------------------------------------
// A block's sum is 0 or between 2^-32 and 2^39 in magnitude.  With a first scale in [2^-94, 2^88] its
// product with that stays a normal number, and the second scale overflows or underflows only where the
// result does.  Of a first scale outside ("wide"), a power of two goes over to the second: where that one
// then leaves the range, the result does too.  Rows whose scale is not wide get 1 and add as ever.
__device__ __forceinline__ bool scale_is_wide(float s) {   // 0, Inf and NaN are not
  const float a = fabsf(s);
  return (a > 0.0f && a < 0x1p-94f) || (a > 0x1p88f && a <= 0x1.fffffep127f);
}
__device__ __forceinline__ float take_over(float& first) {   // returns the second scale's factor
  if (!scale_is_wide(first)) return 1.0f;
  const bool up = fabsf(first) < 1.0f;
  first *= up ? 0x1p40f : 0x1p-40f;
  return up ? 0x1p-40f : 0x1p40f;
}
// Tile scales are multiplied with each other first, which takes a product that is a normal number.
__device__ __forceinline__ bool product_is_wide(float s, float s1, float s2) {   // s = s1 * s2
  return !(fabsf(s) >= 0x1p-126f && fabsf(s) <= 0x1.fffffep127f) && s1 != 0.0f && s2 != 0.0f && isfinite(s1) && isfinite(s2);
}

// BROWS: B has one scale per row (per lane of the tile) instead of one per 128 rows.
template <int BN, bool BROWS>
__global__ void __launch_bounds__(LaneTile<BN>::kThreads, 1)
    matmul_lanes_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a,
                        const MatmulParams p) {
  using T = LaneTile<BN>;
  extern __shared__ unsigned char dyn[];
  __shared__ uint64_t full[T::kStages], empty[T::kStages], acc_full[T::kAcc], acc_empty[T::kAcc], drained;
  __shared__ uint64_t sc_full[T::kScaleSlots], sc_empty[T::kScaleSlots];
  __shared__ uint32_t tmem_base, first_group[9];
  __shared__ unsigned int abort_word;
  __shared__ float lane_scale[T::kScaleSlots][kScaleStep][BROWS ? 128 : 1];
  __shared__ __align__(16) float col_scale[T::kScaleSlots][kScaleStep][BN];
  volatile unsigned int* abort_flag = &abort_word;
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dyn) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = p.splits > 1 ? cluster_rank() : 0;
  const uint32_t tile = blockIdx.x / p.splits;
  const uint32_t n0 = tile / p.tiles_m * 128, m0 = tile % p.tiles_m * BN;
  const uint32_t kb0 = (uint32_t)((uint64_t)p.KB * rank / p.splits);
  const uint32_t nkb = (uint32_t)((uint64_t)p.KB * (rank + 1) / p.splits) - kb0;

  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < T::kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (uint32_t i = 0; i < T::kAcc; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], T::kEpiWarps);
    }
    for (uint32_t i = 0; i < T::kScaleSlots; ++i) {
      mbar_init(&sc_full[i], 32);
      mbar_init(&sc_empty[i], T::kEpiWarps);
    }
    mbar_init(&drained, 1);
    abort_word = 0u;
    mbar_fence_init();
  }
  if (warp == 2 && lane < 9) first_group[lane] = cluster_first(T::kGroups, p.splits, lane);
  if (p.splits > 1) cluster_arrive();   // "this CTA runs": waited for before the first write to another's memory
  if (warp == 1) tmem_alloc<1>(&tmem_base, T::kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;

  float acc[T::kEpiCols];
  bool ok = true;
  if (warp == 0) {
    uint32_t st = 0, phase = 0, issued = 0;
    for (uint32_t i = 0; i < nkb; ++i) {
      if (!__all_sync(0xFFFFFFFFu, mbar_wait_bounded(&empty[st], phase ^ 1u, abort_flag, p.status))) {
        drain_copies(full, T::kStages, issued);
        __syncwarp();
        break;
      }
      const uint32_t s = smem_u32(stages + st * T::kStageBytes), bar = smem_u32(&full[st]);
      const int x = (int)((kb0 + i) * 128);
      expect_tx_elect(bar, T::kStageBytes);
      tma_load_2d(s, &map_b, x, (int)n0, bar);
      tma_load_2d(s + 128 * 128, &map_a, x, (int)m0, bar);
      ++issued;
      if (++st == T::kStages) {
        st = 0;
        phase ^= 1u;
      }
    }
  } else if (warp == 1) {
    uint32_t st = 0, phase = 0;
    for (uint32_t i = 0; i < nkb; ++i) {
      const uint32_t a = i % T::kAcc, a_phase = (i / T::kAcc) & 1u;
      const bool go = mbar_wait_bounded(&acc_empty[a], a_phase ^ 1u, abort_flag, p.status) &&
                      mbar_wait_bounded(&full[st], phase, abort_flag, p.status);
      if (!__all_sync(0xFFFFFFFFu, go)) {
        mma_commit(&drained);   // what has been issued ends before tensor memory is freed
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(&drained, 0))
          if (global_ns() - t0 > 1000000000ull) break;
        __syncwarp();
        break;
      }
      tc_fence_after();
      const uint32_t s = smem_u32(stages + st * T::kStageBytes);
      mma_f8_block<1>(tmem + a * BN, smem_desc_k128(s), smem_desc_k128(s + 128 * 128), p.idesc);
      mma_commit(&empty[st]);
      mma_commit(&acc_full[a]);
      if (++st == T::kStages) {
        st = 0;
        phase ^= 1u;
      }
    }
  } else if (warp == 2) {
    uint32_t slot = 0, phase = 0;
    for (uint32_t i = 0; i < nkb; i += kScaleStep) {
      if (!__all_sync(0xFFFFFFFFu, mbar_wait_bounded(&sc_empty[slot], phase ^ 1u, abort_flag, p.status))) break;
#pragma unroll
      for (uint32_t k = 0; k < kScaleStep; ++k) {
        const bool k_in = i + k < nkb;
        const float* as = p.a_scale + (uint64_t)(kb0 + i + k) * p.M;
        const float* bs = p.b_scale + (uint64_t)(kb0 + i + k) * p.b_scale_ld;
#pragma unroll
        for (int c = 0; c < BN; c += 32) {
          const uint32_t m = m0 + c + lane;
          const bool in = k_in && m < p.M;
          if (c + lane < BN) cp_async_f32(&col_scale[slot][k][c + lane], in ? as + m : p.a_scale, in);
        }
        if constexpr (BROWS) {
#pragma unroll
          for (int c = 0; c < 128; c += 32) {
            const bool in = k_in && n0 + c + lane < p.N;
            cp_async_f32(&lane_scale[slot][k][c + lane], in ? bs + n0 + c + lane : p.b_scale, in);
          }
        } else if (lane == 0) {
          cp_async_f32(&lane_scale[slot][k][0], k_in ? bs + (n0 >> 7) : p.b_scale, k_in);
        }
      }
      cp_async_arrive(&sc_full[slot]);
      if (++slot == T::kScaleSlots) {
        slot = 0;
        phase ^= 1u;
      }
    }
    cp_async_wait_all();
    __syncwarp();
  } else if (warp >= 4) {
    const int quarter = warp & 3;                       // the lanes of tensor memory this warp may read
    const int col0 = ((warp - 4) >> 2) * T::kEpiCols;   // and its columns
    const uint32_t n = n0 + quarter * 32 + lane;
    const bool n_in = n < p.N;
    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + col0;
    uint32_t slot = 0, slot_phase = 0;
#pragma unroll
    for (int j = 0; j < T::kEpiCols; ++j) acc[j] = 0.0f;
    // after a wait has run out every later one returns at once: the loop runs to its end, because
    // reads of tensor memory are collective
    for (uint32_t i = 0; i < nkb; ++i) {
      const uint32_t a = i % T::kAcc, a_phase = (i / T::kAcc) & 1u, k = i % kScaleStep;
      if (k == 0) ok &= mbar_wait_bounded(&sc_full[slot], slot_phase, abort_flag, p.status);
      const float ls = lane_scale[slot][k][BROWS ? quarter * 32 + lane : 0];
      const float* c = &col_scale[slot][k][col0];
      ok &= mbar_wait_bounded(&acc_full[a], a_phase, abort_flag, p.status);
      __syncwarp();
      tc_fence_after();
      auto add_block = [&](float first, auto over) {
        constexpr int kCols = T::kEpiCols < 32 ? 16 : 32;
#pragma unroll
        for (int j0 = 0; j0 < T::kEpiCols; j0 += kCols) {
          float v[kCols];
          if constexpr (kCols == 16)
            tmem_ld16(taddr + a * BN + j0, v);
          else
            tmem_ld32(taddr + a * BN + j0, v);
          tmem_wait_ld(v);
          if (j0 + kCols == T::kEpiCols) {   // all of this accumulator is in registers
            tc_fence_before();
            mbar_arrive_if(&acc_empty[a], lane == 0);
          }
#pragma unroll
          for (int j = 0; j < kCols; j += 4) {
            const float4 f = over(*reinterpret_cast<const float4*>(c + j0 + j));
            fma_pair(acc[j0 + j], acc[j0 + j + 1], v[j] * first, v[j + 1] * first, f.x, f.y);
            fma_pair(acc[j0 + j + 2], acc[j0 + j + 3], v[j + 2] * first, v[j + 3] * first, f.z, f.w);
          }
        }
      };
      if (!__any_sync(0xFFFFFFFFu, scale_is_wide(ls))) {   // the reads of tensor memory are the whole warp's
        add_block(ls, [](float4 f) { return f; });
      } else {
        float first = ls;
        const float t = take_over(first);
        add_block(first, [t](float4 f) { return make_float4(f.x * t, f.y * t, f.z * t, f.w * t); });
      }
      if (k == kScaleStep - 1) {
        __syncwarp();
        mbar_arrive_if(&sc_empty[slot], lane == 0);
        if (++slot == T::kScaleSlots) {
          slot = 0;
          slot_phase ^= 1u;
        }
      }
    }
    if (p.splits == 1 && ok && n_in) store_down<T::kEpiCols>(p, m0 + col0, n, acc);
  }
  if (p.splits > 1) {
    // The cluster adds its partial sums: each CTA owns a share of the tile's columns and gets every
    // CTA's sums for them written into its shared memory, then adds them in rank order.
    cluster_wait();
    const uint32_t share = cluster_share(T::kGroups, p.splits);          // places per CTA and owner
    const uint32_t row = (warp & 3) * 32 + lane;
    unsigned char* sum_buf = stages + T::kStages * T::kStageBytes;
    if (warp >= 4) {
      const uint32_t g0 = ((warp - 4) >> 2) * (T::kEpiCols / 4);
      const uint32_t mine = smem_u32(sum_buf) + (rank * share * 128 + row) * 16;
      uint32_t owner = cluster_owner(T::kGroups, p.splits, g0), next = first_group[owner + 1];
      uint32_t at = map_to_rank(mine, owner) + (g0 - first_group[owner]) * 2048;
#pragma unroll
      for (uint32_t g = 0; g < T::kEpiCols / 4; ++g, at += 2048) {
        while (g0 + g == next) {   // more than once where an owner has no group
          next = first_group[++owner + 1];
          at = map_to_rank(mine, owner);
        }
        if (m0 + (g0 + g) * 4 < p.M) st_cluster_f32x4(at, acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]);
      }
    }
    cluster_sync_all();
    if (warp >= 4 && ok && n0 + row < p.N) {
      const uint32_t first = first_group[rank], last = first_group[rank + 1];
      const float4* sums = reinterpret_cast<const float4*>(sum_buf) + row;
      for (uint32_t g = first + ((warp - 4) >> 2); g < last && m0 + 4 * g < p.M; g += T::kEpiWarps / 4) {
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r) {
          if (r < p.splits) {
            const float4 f = sums[(r * share + g - first) * 128];
            v[0] += f.x;
            v[1] += f.y;
            v[2] += f.z;
            v[3] += f.w;
          }
        }
        store_down<4>(p, m0 + 4 * g, n0 + row, v);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_free<1>(tmem, T::kTmemCols);
}

// ---- many rows of A ------------------------------------------------------------------------
// A pair of CTAs shares a tile of 256 rows of A and 256 rows of B: each holds its own 128 rows of
// either operand, the pair's matrix instructions (issued by the first CTA) read both halves of B,
// and each CTA's tensor memory gets 128 rows x 256 columns.  Per K block of 128 the pair's tensor
// cores are busy for 512 cycles at the 8-bit rate, while 32 KB per CTA have to arrive and 32,768
// accumulators per CTA have to be scaled and added: half of the SM's binary32 rate.  Two
// accumulators fill tensor memory, so the scaling of one block runs under the products of the
// next.  Persistent: a pair walks over tiles, and a tile's last scaling and its stores run under
// the next tile's first products.
struct PairTile {
  static constexpr uint32_t kHalfBytes = 128 * 128;             // one operand's share of a CTA
  static constexpr uint32_t kStageBytes = 2 * kHalfBytes;
  static constexpr uint32_t kStages = 5;
  static constexpr uint32_t kScaleSlots = 3;
  static constexpr uint32_t kTmemCols = 512;
  static constexpr int kEpiWarps = 8;
  // three warpgroups: one copies and issues, two scale and add.  168 registers per thread at
  // launch are split 56 / 224 / 224: 128 running sums and 32 values on their way need that many
  // before the compiler stops moving them about (8192^3, when the split was chosen: 548 us, with
  // 104 / 200 / 200 570; 570 now, with scales safe at both ends of the range).
  static constexpr int kThreads = 128 + 32 * kEpiWarps;
  static constexpr int kRegsLaunch = 168, kRegsControl = 56, kRegsEpi = 224;
  static_assert(128 * kRegsControl + (kThreads - 128) * kRegsEpi <= kThreads * kRegsLaunch, "register shares");
  // results leave through shared memory, 64 bytes of 32 rows per warp at a time, so that every
  // store of a warp covers whole 32-byte sectors; 80-byte rows keep the 16-byte accesses apart
  static constexpr uint32_t kOutPitch = 80;
  static constexpr uint32_t kOutBytes = 32 * kOutPitch;
  static constexpr uint32_t kSmem = 1024 + kStages * kStageBytes + kEpiWarps * kOutBytes;
  static constexpr uint32_t kGroupM = 8;                        // tiles of A that neighbouring pairs share
};

// Tile coordinates of item `t`: down kGroupM tiles of A, then along B, so that the pairs that run
// together read few different rows of either.
__host__ __device__ __forceinline__ void pair_tile(uint32_t t, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
  const uint32_t per = PairTile::kGroupM * tiles_n;
  const uint32_t g = t / per, r = t % per;
  const uint32_t h = min(PairTile::kGroupM, tiles_m - g * PairTile::kGroupM);
  tm = g * PairTile::kGroupM + r % h;
  tn = r / h;
}

// A warp's 32 rows x 128 columns of results (lane = row) to D at row m0 and column n0.
template <int DT>
__device__ __forceinline__ void store_warp_tile(const MatmulParams& p, unsigned char* buf, int lane, uint32_t m0,
                                                uint32_t n0, const float (&acc)[128]) {
  constexpr int kBytes = DT == KB_F32 ? 4 : 2;
  constexpr int kCols = 64 / kBytes;        // columns per round: 64 bytes
  constexpr int kUnit = 16 / kBytes;        // columns per 16 bytes
#pragma unroll
  for (int c = 0; c < 128; c += kCols) {
    if (n0 + c >= p.N) break;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float* v = acc + c + u * kUnit;
      uint4 w;
      if constexpr (DT == KB_F32)
        w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      else
        w = make_uint4(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]), pack2<DT>(v[4], v[5]), pack2<DT>(v[6], v[7]));
      *reinterpret_cast<uint4*>(buf + lane * PairTile::kOutPitch + u * 16) = w;
    }
    __syncwarp();
    if (p.vec_out && n0 + c + kCols <= p.N) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t row = i * 8 + (lane >> 2), unit = lane & 3;
        if (m0 + row < p.M)
          *reinterpret_cast<uint4*>(static_cast<unsigned char*>(p.d) +
                                    ((uint64_t)(m0 + row) * p.ldd + n0 + c + unit * kUnit) * kBytes) =
              *reinterpret_cast<const uint4*>(buf + row * PairTile::kOutPitch + unit * 16);
      }
    } else {
      for (int i = lane; i < 32 * kCols; i += 32) {
        const uint32_t row = i / kCols, col = i % kCols;
        if (m0 + row < p.M && n0 + c + col < p.N) {
          const uint64_t at = (uint64_t)(m0 + row) * p.ldd + n0 + c + col;
          const unsigned char* src = buf + row * PairTile::kOutPitch + col * kBytes;
          if constexpr (DT == KB_F32)
            static_cast<uint32_t*>(p.d)[at] = *reinterpret_cast<const uint32_t*>(src);
          else
            static_cast<unsigned short*>(p.d)[at] = *reinterpret_cast<const unsigned short*>(src);
        }
      }
    }
    __syncwarp();
  }
}

// Tile scales: the rows, of 32 rows x 128 columns of D (one tile of B), for which some K block's product of
// scales is no normal number, once more by one warp.  Such scales come from values around 2^-60, or 2^60, on
// both sides at once, so nothing of this stands in the loops of the kernel: a second path there cost 11%
// of 8192^3, and four branches per K block 4%.  Rows whose codes are 0 wherever the product underflows are
// left alone.  Codes are exact in binary16, so the block sums come from warp-wide matrix instructions on
// 16 rows x 8 columns (2048 x 2560 x 1024 with every row taken: 90 ms element by element, so 5.7).
// Eight codes of a row from column k (a multiple of 8) on, 0 past its K columns
__device__ __forceinline__ uint2 code_pair(const unsigned char* row, uint32_t k, uint32_t K) {
  if (k + 8 <= K) return *reinterpret_cast<const uint2*>(row + k);   // rows start on 16-byte boundaries
  uint2 w = make_uint2(0u, 0u);
  for (uint32_t j = 0; k + j < K; ++j) (j < 4 ? w.x : w.y) |= (uint32_t)row[k + j] << (8 * (j & 3));
  return w;
}
__device__ __forceinline__ void widen_codes(uint32_t w, bool e5m2, uint32_t& lo, uint32_t& hi) {
  if (e5m2)
    ElemF8<true>::widen4(w, lo, hi);
  else
    ElemF8<false>::widen4(w, lo, hi);
}
__device__ __forceinline__ void recompute_wide_rows(const MatmulParams& p, uint32_t m0, uint32_t n0, int lane) {
  if (n0 >= p.N) return;
  const float* bs = p.b_scale + (n0 >> 7);
  const uint32_t row = m0 + lane;
  const unsigned char* codes = p.a + row * p.lda;
  bool need = false;
  for (uint32_t kb = 0; row < p.M && kb < p.KB && !need; ++kb) {
    const float r = p.a_scale[(uint64_t)kb * p.M + row], c = bs[(uint64_t)kb * p.b_scale_ld], s = r * c;
    if (!product_is_wide(s, r, c)) continue;
    need = fabsf(s) > 1.0f;
    for (uint32_t k = kb * 128; k < kb * 128 + 128 && !need; k += 8) {
      const uint2 w = code_pair(codes, k, p.K);
      need = ((w.x | w.y) & 0x7F7F7F7Fu) != 0;
    }
  }
  const uint32_t rows = __ballot_sync(0xFFFFFFFFu, need);
#pragma unroll 1
  for (uint32_t half = 0; half < 2; ++half) {
    if (((rows >> (16 * half)) & 0xFFFFu) == 0) continue;
    // this lane's rows of the fragments (rows and columns outside D repeat the last one and are not stored)
    const uint32_t g = half * 16 + (lane >> 2), r0 = min(m0 + g, p.M - 1), r1 = min(m0 + g + 8, p.M - 1);
    const unsigned char *a0 = p.a + r0 * p.lda, *a1 = p.a + r1 * p.lda;
#pragma unroll 1
    for (uint32_t nt = n0; nt < n0 + 128 && nt < p.N; nt += 8) {
      const unsigned char* b = p.b + min(nt + (lane >> 2), p.N - 1) * p.ldb;
      float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
      for (uint32_t kb = 0; kb < p.KB; ++kb) {
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
        for (uint32_t h = 0; h < 4; ++h) {
          // four lanes hold 32 columns, 8 each: the order of the contraction is the same for both operands
          const uint32_t k = kb * 128 + h * 32 + (lane & 3) * 8;
          const uint2 wa = code_pair(a0, k, p.K), wc = code_pair(a1, k, p.K), wb = code_pair(b, k, p.K);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            uint32_t x0, x1, y0, y1, z0, z1;
            widen_codes(w ? wa.y : wa.x, p.a_e5m2, x0, x1);
            widen_codes(w ? wc.y : wc.x, p.a_e5m2, y0, y1);
            widen_codes(w ? wb.y : wb.x, p.b_e5m2, z0, z1);
            asm volatile(
                "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3])
                : "r"(x0), "r"(y0), "r"(x1), "r"(y1), "r"(z0), "r"(z1));
          }
        }
        const float c = bs[(uint64_t)kb * p.b_scale_ld];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float first = p.a_scale[(uint64_t)kb * p.M + (i ? r1 : r0)], second = c;
          if (product_is_wide(first * c, first, c)) {
            second *= take_over(first);
          } else {
            second *= first;
            first = 1.0f;
          }
          d[2 * i] = fmaf(v[2 * i] * first, second, d[2 * i]);
          d[2 * i + 1] = fmaf(v[2 * i + 1] * first, second, d[2 * i + 1]);
        }
      }
      const uint32_t col = nt + (lane & 3) * 2;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (((rows >> (g + 8 * i)) & 1u) == 0) continue;
        if (col < p.N) store_down<1>(p, i ? r1 : r0, col, &d[2 * i]);
        if (col + 1 < p.N) store_down<1>(p, i ? r1 : r0, col + 1, &d[2 * i + 1]);
      }
    }
  }
}

// BROWS: B has one scale per row (per column of the tile) instead of one per 128 rows.
template <bool BROWS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairTile::kThreads, 1)
    matmul_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                       const MatmulParams p) {
  using T = PairTile;
  extern __shared__ unsigned char dyn[];
  __shared__ uint64_t full[T::kStages], done[T::kStages], acc_empty[2], drained[2];
  __shared__ uint64_t sc_full[T::kScaleSlots], sc_empty[T::kScaleSlots];
  __shared__ uint64_t stored;
  __shared__ uint32_t tmem_base;
  __shared__ unsigned int abort_word, redo_word;
  __shared__ __align__(16) float row_scale[T::kScaleSlots][128][kScaleStep];
  __shared__ __align__(16) float col_scale[T::kScaleSlots][BROWS ? kScaleStep * 256 : 2 * kScaleStep];
  volatile unsigned int* abort_flag = &abort_word;
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dyn) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const uint32_t tiles_n = (p.N + 255) / 256, tiles = p.tiles_m * tiles_n;
  const uint32_t first = blockIdx.x >> 1, step = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < T::kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&done[i], 1);
    }
    for (uint32_t i = 0; i < 2; ++i) {
      mbar_init(&acc_empty[i], 2 * T::kEpiWarps);
      mbar_init(&drained[i], 1);
    }
    for (uint32_t i = 0; i < T::kScaleSlots; ++i) {
      mbar_init(&sc_full[i], 32);
      mbar_init(&sc_empty[i], T::kEpiWarps);
    }
    mbar_init(&stored, T::kEpiWarps);
    abort_word = redo_word = 0u;
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc<2>(&tmem_base, T::kTmemCols);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();   // both CTAs' barriers are ready and their tensor memory is allocated
  tc_fence_after();
  const uint32_t tmem = tmem_base;

  if (warp < 4) regs_shrink<T::kRegsControl>();
  if (warp == 0) {
    uint32_t st = 0, phase = 0;
    uint64_t issued = 0;
    bool go = true;
    for (uint32_t t = first; t < tiles && go; t += step) {
      uint32_t tm, tn;
      pair_tile(t, p.tiles_m, tiles_n, tm, tn);
      const int ya = (int)(tm * 256 + rank * 128), yb = (int)(tn * 256 + rank * 128);
      for (uint32_t kb = 0; kb < p.KB; ++kb) {
        go = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&done[st], phase ^ 1u, abort_flag, p.status));
        if (!go) break;
        const uint32_t s = smem_u32(stages + st * T::kStageBytes);
        const uint32_t bar = map_to_rank(smem_u32(&full[st]), 0);
        if (rank == 0) expect_tx_elect(smem_u32(&full[st]), 2 * T::kStageBytes);
        tma_load_2d_pair(s, &map_a, (int)(kb * 128), ya, bar);
        tma_load_2d_pair(s + T::kHalfBytes, &map_b, (int)(kb * 128), yb, bar);
        ++issued;
        if (++st == T::kStages) {
          st = 0;
          phase ^= 1u;
        }
      }
    }
    if (!go) {
      // let the copies in flight land: the first CTA's barriers count both CTAs' bytes, the
      // second CTA cannot see them and waits far longer than a copy takes
      if (rank == 0) drain_copies(full, T::kStages, issued);
      const unsigned long long t0 = global_ns();
      while (global_ns() - t0 < 20000000ull) {
      }
      __syncwarp();
    }
  } else if (warp == 1 || warp == 3) {
    // Matrix instructions: one thread takes the even K blocks and their accumulator, another the
    // odd ones, so that what a thread spends on its waits hides under the other's products.
    const uint32_t a = warp >> 1;
    if (rank == 0) {
      const uint32_t nkb = tiles > first ? ((tiles - first + step - 1) / step) * p.KB : 0;
      uint32_t st = a, phase = 0, acc_phase = 1;   // stage a, a + 2, ... of the ring
      for (uint32_t it = a; it < nkb; it += 2) {
        const bool go = mbar_wait_bounded(&full[st], phase, abort_flag, p.status) &&
                        mbar_wait_bounded(&acc_empty[a], acc_phase, abort_flag, p.status);
        if (!__all_sync(0xFFFFFFFFu, go)) {
          // what has been issued ends before tensor memory is freed
          mma_commit_pair(&drained[a]);
          const unsigned long long t0 = global_ns();
          while (!mbar_try_wait(&drained[a], 0))
            if (global_ns() - t0 > 1000000000ull) break;
          __syncwarp();
          break;
        }
        tc_fence_after();
        const uint32_t s = smem_u32(stages + st * T::kStageBytes);
        mma_f8_block<2>(tmem + a * 256, smem_desc_k128(s), smem_desc_k128(s + T::kHalfBytes), p.idesc);
        mma_commit_pair(&done[st]);   // frees the stage and hands over the accumulator
        acc_phase ^= 1u;
        st += 2;
        if (st >= T::kStages) {
          st -= T::kStages;
          phase ^= 1u;
        }
      }
    }
  } else if (warp == 2) {
    // the scales of kScaleStep K blocks at a time, one or two steps ahead of their use
    uint32_t slot = 0, phase = 0;
    bool ok = true;
    for (uint32_t t = first; t < tiles && ok; t += step) {
      uint32_t tm, tn;
      pair_tile(t, p.tiles_m, tiles_n, tm, tn);
      const uint32_t m0 = tm * 256 + rank * 128, n0 = tn * 256;
      for (uint32_t kb0 = 0; kb0 < p.KB; kb0 += kScaleStep) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&sc_empty[slot], phase ^ 1u, abort_flag, p.status));
        if (!ok) break;
#pragma unroll
        for (uint32_t k = 0; k < kScaleStep; ++k) {
          const bool k_in = kb0 + k < p.KB;
          const float* as = p.a_scale + (uint64_t)(kb0 + k) * p.M;
          const float* bs = p.b_scale + (uint64_t)(kb0 + k) * p.b_scale_ld;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t m = m0 + i * 32 + lane;
            const bool in = k_in && m < p.M;
            cp_async_f32(&row_scale[slot][i * 32 + lane][k], in ? as + m : p.a_scale, in);
          }
          if constexpr (BROWS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t n = n0 + i * 32 + lane;
              const bool in = k_in && n < p.N;
              cp_async_f32(&col_scale[slot][k * 256 + i * 32 + lane], in ? bs + n : p.b_scale, in);
            }
          } else if (lane < 2) {
            const uint32_t n = n0 + lane * 128;
            const bool in = k_in && n < p.N;
            cp_async_f32(&col_scale[slot][lane * kScaleStep + k], in ? bs + (n >> 7) : p.b_scale, in);
          }
        }
        cp_async_arrive(&sc_full[slot]);
        if (++slot == T::kScaleSlots) {
          slot = 0;
          phase ^= 1u;
        }
      }
    }
    cp_async_wait_all();
    __syncwarp();
    if constexpr (!BROWS) {
      // once everything is stored (nothing waits for this warp any more): the rows with scales that need it
      ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&stored, 0, abort_flag, p.status)) && !*abort_flag;
      for (uint32_t t = first; t < tiles && ok && redo_word; t += step) {
        uint32_t tm, tn;
        pair_tile(t, p.tiles_m, tiles_n, tm, tn);
        for (uint32_t part = 0; part < 8; ++part)
          recompute_wide_rows(p, tm * 256 + rank * 128 + (part & 3) * 32, tn * 256 + (part >> 2) * 128, lane);
      }
    }
  } else if (warp >= 4) {
    regs_grow<T::kRegsEpi>();
    const int quarter = warp & 3, cols = ((warp - 4) >> 2) * 128;   // 32 rows and 128 columns of the tile
    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + cols;
    unsigned char* out_buf = stages + T::kStages * T::kStageBytes + (warp - 4) * T::kOutBytes;
    const uint32_t release0 = map_to_rank(smem_u32(&acc_empty[0]), 0);
    uint32_t a = 0, st = 0, st_phase = 0, slot = 0, slot_phase = 0;
    // After a wait has run out every later one returns at once, so the loops just run to their end;
    // no lane leaves its warp, whose reads of tensor memory are collective.
    bool ok = true;
    for (uint32_t t = first; t < tiles; t += step) {
      float acc[128];
#pragma unroll
      for (int j = 0; j < 128; ++j) acc[j] = 0.0f;
      for (uint32_t kb0 = 0; kb0 < p.KB; kb0 += kScaleStep) {
        ok &= mbar_wait_bounded(&sc_full[slot], slot_phase, abort_flag, p.status);
        const float4 rs = *reinterpret_cast<const float4*>(row_scale[slot][quarter * 32 + lane]);
        float s4[4] = {rs.x, rs.y, rs.z, rs.w};
        bool wide = false;
        if constexpr (BROWS) {
#pragma unroll
          for (int k = 0; k < 4; ++k) wide |= scale_is_wide(s4[k]);
          wide = __any_sync(0xFFFFFFFFu, wide);   // one path for the warp, whose reads of tensor memory are collective
        } else {
          const float4 cs = *reinterpret_cast<const float4*>(&col_scale[slot][(cols >> 7) * kScaleStep]);
          const float c4[4] = {cs.x, cs.y, cs.z, cs.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float r = s4[k];
            s4[k] *= c4[k];
            wide |= product_is_wide(s4[k], r, c4[k]);
          }
          if (wide) redo_word = 1u;
        }
#pragma unroll 1
        for (uint32_t k = 0; k < kScaleStep && kb0 + k < p.KB; ++k) {
          ok &= mbar_wait_bounded(&done[st], st_phase, abort_flag, p.status);
          __syncwarp();
          tc_fence_after();
          const float s = s4[0];
          s4[0] = s4[1];
          s4[1] = s4[2];
          s4[2] = s4[3];
          const float* c = &col_scale[slot][BROWS ? k * 256 + cols : 0];
          if (++st == T::kStages) {
            st = 0;
            st_phase ^= 1u;
          }
          auto add_block = [&](float first, auto second) {   // acc += (v * first) * second, tile scales: v * first
#pragma unroll
            for (int j0 = 0; j0 < 128; j0 += 32) {
              float v[32];
              tmem_ld32(taddr + a * 256 + j0, v);
              tmem_wait_ld(v);
              if (j0 == 96) {   // all of this accumulator is in registers
                tc_fence_before();
                mbar_arrive_cluster_if(release0 + a * 8, lane == 0);
              }
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const float4 f = BROWS ? second(*reinterpret_cast<const float4*>(c + j0 + j)) : make_float4(first, first, first, first);
                fma_pair(acc[j0 + j], acc[j0 + j + 1], BROWS ? v[j] * first : v[j], BROWS ? v[j + 1] * first : v[j + 1], f.x, f.y);
                fma_pair(acc[j0 + j + 2], acc[j0 + j + 3], BROWS ? v[j + 2] * first : v[j + 2],
                         BROWS ? v[j + 3] * first : v[j + 3], f.z, f.w);
              }
            }
          };
          if (!BROWS || !wide) {
            add_block(s, [](float4 f) { return f; });
          } else {
            float first = s;
            const float t = take_over(first);
            add_block(first, [t](float4 f) { return make_float4(f.x * t, f.y * t, f.z * t, f.w * t); });
          }
          a ^= 1u;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sc_empty[slot]);
        if (++slot == T::kScaleSlots) {
          slot = 0;
          slot_phase ^= 1u;
        }
      }
      uint32_t tm, tn;
      pair_tile(t, p.tiles_m, tiles_n, tm, tn);
      if (__all_sync(0xFFFFFFFFu, ok)) {
        const uint32_t m0 = tm * 256 + rank * 128 + quarter * 32, n0 = tn * 256 + cols;
        if (p.out == KB_BF16)
          store_warp_tile<KB_BF16>(p, out_buf, lane, m0, n0, acc);
        else if (p.out == KB_F16)
          store_warp_tile<KB_F16>(p, out_buf, lane, m0, n0, acc);
        else
          store_warp_tile<KB_F32>(p, out_buf, lane, m0, n0, acc);
      }
    }
    if constexpr (!BROWS) {
      __syncwarp();
      mbar_arrive_if(&stored, lane == 0);
    }
  }
  tc_fence_before();
  cluster_sync_all();   // neither CTA leaves while the other's instructions use its memory
  tc_fence_after();
  if (warp == 1) tmem_free<2>(tmem, T::kTmemCols);
}

}  // namespace kb
