// Attention over whole prompts (contract in include/kb_attention.h).
//
// A CTA takes two tiles of 128 queries against the keys and values that they share, 128 keys at a
// time: two neighbouring heads of a group at the same 128 queries, or 256 queries of one head where groups
// are odd.  Per tile and step the tensor cores make S = Q K^T (128 x 128, accumulated in tensor memory), a
// warpgroup with one thread per query turns S into P = 2^(S c - r) in registers and writes it back over S
// in 16 bits, and the tensor cores add P V to the output, which stays in tensor memory to the end.
// While one tile's warpgroup is at its exponentials the tensor cores work for the other tile.
//
// The running reference r of a query (shared with the paged kernel: kRoom, kLazy) is raised only where a score
// exceeds it by more than 2^kLazy, so the output in tensor memory is rescaled a few times per query and
// not once per step.  Bound by the exponentials and the tensor cores together: a tile's step is 1024 cycles
// of 128 x 128 x 128 products (two at dim 128) and 16384 exponentials, 1024 cycles at 16 a cycle.
//
// What a query does not see never enters its sums: scores behind a mask become -infinity before anything is
// done with them, and values of keys behind a sequence's end are zeroed in shared memory before they
// are multiplied (0 times NaN is not 0).  Values of a causal tile's later keys are ordinary numbers in all but
// broken inputs: where a query's output is not finite although its sum is, the values it does not see are looked
// at, and if one of them is not finite the query is computed again without them (repair).
//
// Roles: warp 0 copies, warp 1 issues matrix instructions, warps 2 and 3 idle; warps 4 to 7 and 8 to 11
// are the tiles' warpgroups.  Every wait is bounded.
#pragma once

#include "kb_paged.cuh"
#include "kb_tcgen05.cuh"

namespace kb {

struct PromptParams {
  const int *q_offsets, *k_offsets;   // NULL: one sequence of all tokens
  uint32_t sequences, q_tokens, k_tokens;
  uint32_t hq, group, dim;
  bool pair;                          // tiles are two heads (else: two pieces of 128 queries)
  bool causal, vec_out;
  float scale_log2;
  const void *q, *k, *v;              // for repair
  uint64_t q_row, q_head, k_row, k_head, v_row, v_head;
  void* out;
  uint64_t o_row, o_head;
  float* lse;
  unsigned int* status;
};

template <int DP>   // dim rounded up to 64 or 128
struct PromptTile {
  static constexpr uint32_t kChunks = DP / 64;                  // of 64 elements = 128 bytes
  static constexpr uint32_t kTileBytes = 128 * DP * 2;          // 128 rows of q, k or v
  static constexpr uint32_t kStages = DP == 128 ? 4 : 8;        // of the ring of k and v tiles
  static constexpr uint32_t kSmem = 1024 + (2 + kStages) * kTileBytes;
  static constexpr uint32_t kTmemS = 0, kTmemO = 256, kTmemCols = 512;   // per tile: S 128 columns, O DP columns
  static constexpr int kThreads = 384;
  // 168 registers per thread at launch, shared out 56 / 224 / 224 to the three warpgroups
  static constexpr int kRegsLaunch = 168, kRegsControl = 56, kRegsSoftmax = 224;
  static_assert(128 * kRegsControl + 256 * kRegsSoftmax <= kThreads * kRegsLaunch, "register shares");
};

// Tiles of 128 keys that the queries [row, row + rows) of a sequence see: causal ones see the keys up to
// their place plus nk - nq.
__host__ __device__ __forceinline__ uint32_t prompt_tiles(uint32_t row, uint32_t rows, uint32_t nq, uint32_t nk, bool causal) {
  if (row >= nq || rows == 0) return 0;
  const uint32_t last = row + rows < nq ? row + rows - 1 : nq - 1;
  long long seen = nk;
  if (causal && (long long)last + nk - nq + 1 < seen) seen = (long long)last + nk - nq + 1;
  return seen <= 0 ? 0u : (uint32_t)((seen + 127) / 128);
}
// Keys that query `row` sees
__host__ __device__ __forceinline__ uint32_t prompt_seen(uint32_t row, uint32_t nq, uint32_t nk, bool causal) {
  if (!causal) return nk;
  const long long seen = (long long)row + nk - nq + 1;
  return seen <= 0 ? 0u : seen < nk ? (uint32_t)seen : nk;
}

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// x * c - r for two numbers as one packed instruction
__device__ __forceinline__ void scale_pair(float& x0, float& x1, float c, float minus_r) {
  asm("{\n.reg .b64 x, c, r;\nmov.b64 x, {%0, %1};\nmov.b64 c, {%2, %2};\nmov.b64 r, {%3, %3};\n"
      "fma.rn.f32x2 x, x, c, r;\nmov.b64 {%0, %1}, x;\n}"
      : "+f"(x0), "+f"(x1)
      : "f"(c), "f"(minus_r));
}
__device__ __forceinline__ void add_pair(float& s0, float& s1, float x0, float x1) {
  asm("{\n.reg .b64 s, x;\nmov.b64 s, {%0, %1};\nmov.b64 x, {%2, %3};\nadd.rn.f32x2 s, s, x;\nmov.b64 {%0, %1}, s;\n}"
      : "+f"(s0), "+f"(s1)
      : "f"(x0), "f"(x1));
}

// A query's output once more from global memory, by one warp, over the keys that it sees alone.
template <int DT>
__device__ __noinline__ void repair_row(const PromptParams& p, uint32_t q_at, uint32_t k0, uint32_t keys, uint32_t h, float r, float by, int lane) {
  const uint32_t hk = h / p.group;
  const uint64_t qa = q_at * p.q_row + h * p.q_head;
  float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // elements lane, 32 + lane, ...
  for (uint32_t j0 = 0; j0 < keys; j0 += 32) {
    float s = 0.0f;
    if (j0 + lane < keys) {
      const uint64_t ka = (uint64_t)(k0 + j0 + lane) * p.k_row + hk * p.k_head;
      for (uint32_t d = 0; d < p.dim; ++d) s = fmaf(load_elem<DT>(p.q, qa + d), load_elem<DT>(p.k, ka + d), s);
    }
    const float e = exp2_fast(fmaf(s, p.scale_log2, -r));
    for (uint32_t j = 0; j < 32 && j0 + j < keys; ++j) {
      const float w = __shfl_sync(0xFFFFFFFFu, e, j);
      const uint64_t va = (uint64_t)(k0 + j0 + j) * p.v_row + hk * p.v_head;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i * 32 + lane < (int)p.dim) o[i] = fmaf(w, load_elem<DT>(p.v, va + i * 32 + lane), o[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i * 32 + lane < (int)p.dim) store_elem<DT>(p.out, q_at * p.o_row + h * p.o_head + i * 32 + lane, o[i] * by);
}

template <int DT, int DP>
__global__ void __launch_bounds__(PromptTile<DP>::kThreads, 1)
    attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const PromptParams p) {
  using T = PromptTile<DP>;
  extern __shared__ unsigned char dyn[];
  __shared__ uint64_t q_full[2], full[T::kStages], empty[T::kStages], s_full[2], p_full[2], o_full[2], drained;
  __shared__ uint32_t tmem_base, scan[12], found[5];
  __shared__ unsigned int abort_word;
  volatile unsigned int* abort_flag = &abort_word;
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dyn) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // Which item: the queries [row, row + rows_per) of a sequence.  Later pieces of a sequence, which see more keys, come first.
  const uint32_t units = p.pair ? p.hq / 2 : p.hq;
  const uint32_t item = blockIdx.x / units, unit = blockIdx.x % units;
  const uint32_t rows_per = p.pair ? 128 : 256;
  if (threadIdx.x == 0) found[4] = 0;
  uint32_t before = 0;
  bool here = false;
  for (uint32_t s0 = 0; s0 < p.sequences && !here; s0 += T::kThreads) {
    const uint32_t s = s0 + threadIdx.x;
    uint32_t qa = 0, nq = 0, ka = 0, nk = 0;
    if (s < p.sequences) {
      if (p.q_offsets) {
        const int a = p.q_offsets[s], b = p.q_offsets[s + 1], c = p.k_offsets[s], d = p.k_offsets[s + 1];
        if (a >= 0 && a <= b && (uint32_t)b <= p.q_tokens && c >= 0 && c <= d && (uint32_t)d <= p.k_tokens) {
          qa = a;
          nq = b - a;
          ka = c;
          nk = d - c;
        } else if (blockIdx.x == 0) {
          set_status(p.status, (unsigned int)KB_ERR_INVALID_ARG);
        }
      } else {
        nq = p.q_tokens;
        nk = p.k_tokens;
      }
    }
    const uint32_t mine = (nq + rows_per - 1) / rows_per;
    uint32_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, sum, o);
      if (lane >= o) sum += up;
    }
    __syncthreads();
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    uint32_t all = 0, mine_before = before + sum - mine;
#pragma unroll
    for (int w = 0; w < T::kThreads / 32; ++w) {
      if (w < warp) mine_before += scan[w];
      all += scan[w];
    }
    const bool mine_here = item >= mine_before && item < mine_before + mine;
    if (mine_here) {
      found[0] = qa;
      found[1] = nq;
      found[2] = ka;
      found[3] = nk;
      found[4] = mine - (item - mine_before);   // 1 + the piece
    }
    here = __syncthreads_or(mine_here);
    before += all;
  }
  __syncthreads();
  if (found[4] == 0) return;   // fewer items than the host had to allow for
  const uint32_t q0 = found[0], nq = found[1], k0 = found[2], nk = found[3], row0 = (found[4] - 1) * rows_per;
  const uint32_t head0 = p.pair ? 2 * unit : unit;
  // per tile: first query, number of key tiles
  const uint32_t n0 = prompt_tiles(row0, 128, nq, nk, p.causal);
  const uint32_t n1 = p.pair ? n0 : prompt_tiles(row0 + 128, 128, nq, nk, p.causal);
  const uint32_t steps = max(n0, n1);

  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < T::kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], 4);
      mbar_init(&o_full[i], 1);
    }
    mbar_init(&drained, 1);
    abort_word = 0u;
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc<1>(&tmem_base, T::kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  unsigned char* ring = base + 2 * T::kTileBytes;

  if (warp < 4) regs_shrink<T::kRegsControl>();
  if (warp == 0) {
    // the ring takes K0, V0, K1, V1, ...: the order in which the matrix instructions want them
    const int hk = (int)(head0 / p.group);
    uint32_t st = 0, phase = 0, issued = 0;
    bool go = true;
    if (steps) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if ((t ? n1 : n0) == 0) continue;
        const uint32_t bar = smem_u32(&q_full[t]);
        expect_tx_elect(bar, T::kTileBytes);
        for (uint32_t c = 0; c < T::kChunks; ++c)
          tma_load_3d(smem_u32(base + t * T::kTileBytes) + c * 16384, &map_q, (int)(c * 64), (int)(q0 + row0 + (p.pair ? 0 : t * 128)),
                      (int)(head0 + (p.pair ? t : 0)), bar);
      }
    }
    for (uint32_t i = 0; i < 2 * steps; ++i) {
      go = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(&empty[st], phase ^ 1u, abort_flag, p.status));
      if (!go) break;
      const uint32_t s = smem_u32(ring + st * T::kTileBytes), bar = smem_u32(&full[st]);
      expect_tx_elect(bar, T::kTileBytes);
      for (uint32_t c = 0; c < T::kChunks; ++c)
        tma_load_3d(s + c * 16384, i & 1 ? &map_v : &map_k, (int)(c * 64), (int)(k0 + i / 2 * 128), hk, bar);
      ++issued;
      if (++st == T::kStages) {
        st = 0;
        phase ^= 1u;
      }
    }
    if (!go) {   // what is on its way lands before the CTA ends
      drain_copies(full, T::kStages, issued);
      for (int t = 0; t < 2; ++t)
        if (t ? n1 : n0) drain_copies(&q_full[t], 1, 1);
      __syncwarp();
    }
  } else if (warp == 1 && steps) {
    const uint32_t idesc_s = mma_idesc_f16(DT == KB_BF16, false, 128, 128), idesc_o = mma_idesc_f16(DT == KB_BF16, true, 128, DP);
    uint32_t st = 0, phase = 0;
    bool go = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (go) go = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity, abort_flag, p.status));
      tc_fence_after();
    };
    auto scores = [&](int t, uint32_t stage) {
      const uint32_t a = smem_u32(base + t * T::kTileBytes), b = smem_u32(ring + stage * T::kTileBytes);
      for (uint32_t c = 0; c < T::kChunks; ++c)
        mma_f16_block(tmem + T::kTmemS + t * 128, smem_desc_k128(a + c * 16384), smem_desc_k128(b + c * 16384), idesc_s, c > 0);
      mma_commit(&s_full[t]);
    };
    auto next = [&]() {
      if (++st == T::kStages) {
        st = 0;
        phase ^= 1u;
      }
    };
    wait(&full[st], phase);
    for (int t = 0; t < 2; ++t) {
      if ((t ? n1 : n0) == 0) continue;
      wait(&q_full[t], 0);
      if (go) scores(t, st);
    }
    if (go) mma_commit(&empty[st]);
    next();
    for (uint32_t j = 0; j < steps && go; ++j) {
      const uint32_t vst = st;
      wait(&full[vst], phase);
      if (!go) break;
      const uint32_t rest = nk - j * 128;
      if (rest < 128) {   // values behind the sequence's end: another's, or anything
        for (uint32_t i = lane; i < (128 - rest) * 8 * T::kChunks; i += 32) {
          const uint32_t unit16 = i & 7, row = rest + (i >> 3) % (128 - rest), c = (i >> 3) / (128 - rest);
          *reinterpret_cast<uint4*>(ring + vst * T::kTileBytes + c * 16384 + row * 128 + unit16 * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }
      next();
      const uint32_t kst = st;
      const bool more = j + 1 < steps;
      if (more) wait(&full[kst], phase);
      for (int t = 0; t < 2 && go; ++t) {
        const uint32_t n = t ? n1 : n0;
        if (j >= n) continue;
        wait(&p_full[t], j & 1u);
        if (!go) break;
        const uint32_t v = smem_u32(ring + vst * T::kTileBytes);
#pragma unroll
        for (uint32_t c = 0; c < 2; ++c)   // 64 keys each
          mma_f16_block_ts(tmem + T::kTmemO + t * DP, tmem + T::kTmemS + t * 128 + c * 32, smem_desc_n128(v + c * 8192, 16384), idesc_o, j > 0 || c > 0);
        mma_commit(&o_full[t]);
        if (j + 1 < n) {
          // the next scores go where P is read from: that has to be over
          wait(&o_full[t], j & 1u);
          if (go) scores(t, kst);
        }
      }
      if (!go) break;
      mma_commit(&empty[vst]);
      if (more) {
        mma_commit(&empty[kst]);
        next();
      }
    }
    if (!go) {   // what has been issued ends before tensor memory is freed
      mma_commit(&drained);
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(&drained, 0))
        if (global_ns() - t0 > 1000000000ull) break;
      __syncwarp();
    }
  } else if (warp >= 4) {
    regs_grow<T::kRegsSoftmax>();
    const int t = (warp - 4) >> 2, quarter = warp & 3;
    const uint32_t n = t ? n1 : n0, row = row0 + (p.pair ? 0 : t * 128) + quarter * 32 + lane, h = head0 + (p.pair ? t : 0);
    const uint32_t at_s = tmem + T::kTmemS + t * 128 + ((uint32_t)(quarter * 32) << 16);
    const uint32_t at_o = tmem + T::kTmemO + t * DP + ((uint32_t)(quarter * 32) << 16);
    const uint32_t seen = row < nq ? prompt_seen(row, nq, nk, p.causal) : 0;
    const uint32_t seen_by_all = __reduce_min_sync(0xFFFFFFFFu, seen);
    const float c = p.scale_log2;
    float r = -INFINITY, l0 = 0.0f, l1 = 0.0f;
    // after a wait has run out every later one returns at once: the loop runs to its end, because reads of
    // tensor memory are collective
    bool ok = true;
    for (uint32_t j = 0; j < n; ++j) {
      ok &= mbar_wait_bounded(&s_full[t], j & 1u, abort_flag, p.status);
      __syncwarp();
      tc_fence_after();
      float s[4][32];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld32(at_s + i * 32, s[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_wait_ld(s[i]);
      if (j * 128 + 128 > seen_by_all) {
        const int left = (int)seen - (int)(j * 128);   // keys of this tile that the query sees
#pragma unroll
        for (int i = 0; i < 128; ++i) s[i / 32][i % 32] = i < left ? s[i / 32][i % 32] : -INFINITY;
      }
      float m[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
      for (int i = 4; i < 128; ++i) m[i % 4] = max_nan(m[i % 4], s[i / 32][i % 32]);
      const float top = max_nan(max_nan(m[0], m[1]), max_nan(m[2], m[3])) * c;   // scale > 0; NaN stays
      if (__any_sync(0xFFFFFFFFu, top - kRoom > r + kLazy)) {
        const float raised = fmaxf(r, top - kRoom), f = r == -INFINITY ? 0.0f : exp2_fast(r - raised);
        r = raised;
        l0 *= f;
        l1 *= f;
        if (j > 0) {
          ok &= mbar_wait_bounded(&o_full[t], (j - 1) & 1u, abort_flag, p.status);
          __syncwarp();
          tc_fence_after();
#pragma unroll 1
          for (int i = 0; i < DP; i += 32) {
            float o[32];
            tmem_ld32(at_o + i, o);
            tmem_wait_ld(o);
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] *= f;
            tmem_st32(at_o + i, reinterpret_cast<const uint32_t*>(o));
          }
        }
      }
      const float minus_r = -known(r);
      uint32_t w[64];
#pragma unroll
      for (int i = 0; i < 128; i += 2) {
        float &x = s[i / 32][i % 32], &y = s[i / 32][i % 32 + 1];
        scale_pair(x, y, c, minus_r);
        x = exp2_fast(x);
        y = exp2_fast(y);
        add_pair(l0, l1, x, y);
        w[i / 2] = pack2<DT>(x, y);
      }
      tmem_st32(at_s, w);
      tmem_st32(at_s + 32, w + 32);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      mbar_arrive_if(&p_full[t], lane == 0);
    }
    const float l = l0 + l1;
    const bool none = l == 0.0f;
    const float by = 1.0f / l;
    if (n) {
      ok &= mbar_wait_bounded(&o_full[t], (n - 1) & 1u, abort_flag, p.status);
      __syncwarp();
      tc_fence_after();
    }
    if (__all_sync(0xFFFFFFFFu, ok)) {
      const bool in = row < nq;
      if (in && p.lse) p.lse[(uint64_t)(q0 + row) * p.hq + h] = none ? -INFINITY : (r + log2f(l)) * 0.69314718055994531f;
      // rows go through shared memory (the tile's queries are not needed any more), so that a warp's stores cover whole rows
      constexpr int kUnits = DP / 8;   // of 16 bytes
      unsigned char* rows = base + t * T::kTileBytes + quarter * 32 * DP * 2;
      bool odd = false;                // an element that is not finite
#pragma unroll
      for (int i = 0; i < DP; i += 32) {
        float o[32];
        if (n) {
          tmem_ld32(at_o + i, o);
          tmem_wait_ld(o);
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          o[k] = none ? 0.0f : o[k] * by;
          odd |= !(fabsf(o[k]) <= 3.402823466e38f);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float* v = o + 8 * u;
          const int at = (i / 8 + u) ^ (lane & 7);
          *reinterpret_cast<uint4*>(rows + lane * DP * 2 + at * 16) =
              make_uint4(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]), pack2<DT>(v[4], v[5]), pack2<DT>(v[6], v[7]));
        }
      }
      __syncwarp();
      const uint32_t first = row - lane;
      for (int i = lane; i < 32 * kUnits; i += 32) {
        const uint32_t rr = i / kUnits, u = i % kUnits;
        if (first + rr >= nq || u * 8 >= p.dim) continue;
        const unsigned char* from = rows + rr * DP * 2 + ((u ^ (rr & 7)) * 16);
        unsigned short* to = static_cast<unsigned short*>(p.out) + (uint64_t)(q0 + first + rr) * p.o_row + h * p.o_head + u * 8;
        if (p.vec_out) {
          *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) to[e] = reinterpret_cast<const unsigned short*>(from)[e];
        }
      }
      // rows that are not finite although their sums are: values that they do not see?
      const bool ask = in && odd && l > 0.0f && l <= 3.402823466e38f && seen < min(nk, n * 128);
      if (__any_sync(0xFFFFFFFFu, ask)) {
        const uint32_t least = __reduce_min_sync(0xFFFFFFFFu, ask ? seen : 0xFFFFFFFFu);
        uint32_t last_bad = 0;   // 1 + the last key with a value that is not finite, of those some row does not see
        const uint32_t hk = h / p.group;
        for (uint32_t k = least; k < min(nk, n * 128); ++k) {
          bool bad = false;
          for (uint32_t d = lane; d < p.dim; d += 32)
            bad |= !(fabsf(load_elem<DT>(p.v, (uint64_t)(k0 + k) * p.v_row + hk * p.v_head + d)) <= 3.402823466e38f);
          if (__any_sync(0xFFFFFFFFu, bad)) last_bad = k + 1;
        }
        uint32_t todo = __ballot_sync(0xFFFFFFFFu, ask && seen < last_bad);
        __syncwarp();
        while (todo) {
          const int src = __ffs(todo) - 1;
          todo &= todo - 1;
          repair_row<DT>(p, q0 + first + src, k0, __shfl_sync(0xFFFFFFFFu, seen, src), h, __shfl_sync(0xFFFFFFFFu, r, src),
                         __shfl_sync(0xFFFFFFFFu, by, src), lane);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_free<1>(tmem, T::kTmemCols);
}

}  // namespace kb
