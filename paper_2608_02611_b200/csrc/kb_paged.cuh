// Attention of one new token per sequence over a paged cache (contract in include/kb_attention.h).
//
// Bound by the cache's bytes: every key and value is read once for the query heads that share it, up to
// 16 of them, and the rest has to stay out of the way.  Work is divided evenly whatever the lengths: steps
// of 128 keys (64 with 4 warps) are the units, those of all sequences form one row, and the row is cut into pieces, as many
// as let the card run a CTA for each piece and group of heads at the same time.  A CTA takes the sequences that its
// piece touches one after the other; CTAs of the same piece are neighbours, so that the groups'
// heads, which lie side by side in the cache, are read at about the same time.  A sequence that lies in
// one piece is finished there; otherwise each piece leaves its part in the workspace, and the CTA that comes
// last adds the parts up in the order of the keys.
//
// A warp takes 16 keys of a step at a time, which a ring of its own in shared memory gets by tensor-map copies
// (boxes of up to 16 keys of a page, 64 elements after another, in the 128-byte swizzle), kPagedStages tiles ahead and
// on into the next sequence: 192 KB are on their way per SM at dim 128.  Straight from global memory into
// registers, with 16 warps per SM, 128 x 4096 keys of 8 heads took 486 us; so 331 (6.5 TB/s).  From there they go into warp-wide
// matrix instructions without any rearrangement, because the order of a contraction and of an operand's rows is
// free as long as the other operand and the result's readers have the same:
//   scores  S^T[16 keys][8 heads] = K Q^T: lane (g, t) = (lane / 4, lane % 4) reads the elements 32 h + 8 t .. + 7
//     of keys kappa(g) and kappa(g) + 8, 16 bytes each, as its part of the first operand's rows g and g + 8; q
//     is held in the same order.
//   out  O^T[dim][8 heads] = V^T P^T: P^T comes from S^T by transposing 8 x 8 matrices of 16-bit numbers
//     between lanes, so lane (g, t) has the keys kappa(2t), kappa(2t + 1) and those + 8; it reads their elements
//     64 c + 8 g .. + 7, pairs two keys' by byte permutes, and the rows of the product are whatever elements
//     its reads brought.
// kappa(g) = g, with bit 2 flipped where g is odd: then the 8 lanes of a phase read from 8 different bank groups in
// both places.
// The 8-column tile of the instruction holds the heads: fewer than 8 waste matrix work, which is not
// what bounds this kernel.  The exponentials are relative to a running value that is raised only where
// a score, in powers of two, is more than kLazy above the largest there was when it was last raised; p is rounded to the
// storage type for the matrix instruction, the sum is of p before that, in binary32.
#pragma once

#include "kb_block8.cuh"
#include "kb_tcgen05.cuh"

namespace kb {

// exp(s) is taken relative to r, as 2^(s' - r) with s' = s * log2(e).  r = (largest s' when it was last raised) - kRoom: the
// largest p is between 2^kRoom and 2^(kRoom + kLazy) <= 2^15, so that binary16 holds it and small p keep their digits.
constexpr float kRoom = 7.0f, kLazy = 8.0f;

struct PagedParams {
  const void* q;
  uint64_t q_row, q_head;
  uint64_t pages;
  uint32_t page_size, page_shift, max_pages;   // page_shift: log2 of page_size, 32 where it is no power of two
  uint32_t box;                             // keys of a copy: 16, or the power of two that divides page_size
  uint32_t copies;                          // of the keys' 64 elements each: 1 where a copy takes all of whole 64s
  const int* table;
  uint64_t table_row;
  const int* lengths;
  uint32_t sequences, hkv, group, chunks;   // group: query heads per kv head; chunks: pieces of at most 8 NT of them
  uint32_t dim;
  float scale_log2;
  void* out;
  uint64_t o_row, o_head;
  float* lse;
  uint32_t q_heads;
  bool vec_out;
  float* part;                              // [2 * CTAs][8 NT][DP] sums of p v
  float* part_rl;                           // [2 * CTAs][8 NT][2]: r, sum of p
  unsigned int* arrived;                    // [CTAs], zero between calls
  unsigned int* status;
};

constexpr uint32_t kPagedStages = 3;
constexpr uint32_t kPagedWaves = 3;                // of CTAs that run together, at most
// W warps: 8, and one CTA per SM, or 4 and two
template <int DP, int NT, int W>
struct PagedTile {
  static constexpr int kThreads = 32 * W, kPerSm = 8 / W;
  static constexpr uint32_t kHalf = DP / 64 * 2048;                      // 16 keys, or values
  static constexpr uint32_t kRing = W * kPagedStages * 2 * kHalf;
  static constexpr uint32_t kSmem = 1024 + kRing;
  static_assert(8 * NT * DP * 4 <= 2 * kHalf, "a warp's sums fit a tile");
};
__host__ __device__ __forceinline__ uint32_t paged_kappa(uint32_t g) { return g ^ ((g & 1) << 2); }

// A sequence's keys as the table can hold them, and units per group of heads: one at least, for the zeros of an
// empty sequence
__host__ __device__ __forceinline__ uint32_t paged_length(int length, uint32_t max_pages, uint32_t page_size) {
  const uint64_t most = (uint64_t)max_pages * page_size;
  return length <= 0 ? 0u : (uint64_t)length > most ? (uint32_t)most : (uint32_t)length;
}
__host__ __device__ __forceinline__ uint32_t paged_units(uint32_t keys, uint32_t step) { return keys ? (keys + step - 1) / step : 1u; }
// A row of n units in pieces: the first `more` of them have size + 1 units, the others size.  As few as keep the longest
// as short as `most` pieces would; each has a unit.
struct PagedPieces {
  uint32_t count, size, more;
  __host__ __device__ __forceinline__ PagedPieces(uint32_t n, uint32_t most) {
    const uint32_t longest = (n + most - 1) / most;
    count = (n + longest - 1) / longest;
    size = n / count;
    more = n - size * count;
  }
  __host__ __device__ __forceinline__ uint32_t first(uint32_t c) const { return size * c + (c < more ? c : more); }   // unit that piece c starts at
  __host__ __device__ __forceinline__ uint32_t of(uint32_t u) const {                                                 // piece that unit u lies in
    const uint32_t bigger = more * (size + 1);
    return u < bigger ? u / (size + 1) : more + (u - bigger) / size;
  }
};

template <int DT>
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (DT == KB_BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {   // 2^x, 2 ulp; 0 for -inf, NaN for NaN
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// The reference of a row's exponentials as it enters an exponent: 0 while no score above -infinity was met
__device__ __forceinline__ float known(float r) { return r == -INFINITY ? 0.0f : r; }

// DP: 64 or 128, dim rounded up.  NT: tiles of 8 heads.
template <int DT, int DP, int NT, int W>
__global__ void __launch_bounds__(32 * W, 8 / W)
    attention_paged_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const PagedParams p) {
  using T = PagedTile<DP, NT, W>;
  constexpr int kH = DP / 32, kC = DP / 64, kHeads = 8 * NT;
  constexpr uint32_t kS = kPagedStages, kStepKeys = 16 * W, kThreads = T::kThreads;
  extern __shared__ unsigned char dyn[];
  __shared__ uint64_t full[W][kS];
  __shared__ float warp_r[W][kHeads], warp_l[W][kHeads];
  __shared__ uint4 q_lanes[2][NT * kH * 32];   // of this sequence and of the next one
  __shared__ const float4* sums_of[W];
  __shared__ uint32_t scan[W], found_seq, found_before, join_word[2];
  __shared__ unsigned int abort_word;
  volatile unsigned int* abort_flag = &abort_word;
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dyn) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  if (threadIdx.x < W * kS) {
    mbar_init(&full[threadIdx.x / kS][threadIdx.x % kS], 1);
    mbar_fence_init();   // each thread's own barrier, for the copies
  }
  if (threadIdx.x == 0) {
    abort_word = 0u;
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  after_the_kernel_before();
  const uint32_t item = blockIdx.x, per_seq = gridDim.x, hk = item / p.chunks, h0 = hk * p.group + item % p.chunks * kHeads;
  const uint32_t heads = min((uint32_t)kHeads, (hk + 1) * p.group - h0);   // query heads h0 .. of this CTA

  // Units of all sequences, then the sequence that this piece starts in.  (Rolled loops throughout: a short call takes as
  // long as its instructions take to arrive.)
  PagedPieces pieces(1, 1);
  uint32_t u0 = 0, u1 = 0;
  bool found = false;
#pragma unroll 1
  for (int pass = 0; pass < 2 && !found; ++pass) {
    uint32_t sum_before = 0;
#pragma unroll 1
    for (uint32_t s0 = 0; s0 < p.sequences && !found; s0 += kThreads) {
      const uint32_t s = s0 + threadIdx.x, units = s < p.sequences ? paged_units(paged_length(p.lengths[s], p.max_pages, p.page_size), kStepKeys) : 0;
      uint32_t sum = units;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, sum, o);
        if (lane >= o) sum += up;
      }
      __syncthreads();
      if (lane == 31) scan[warp] = sum;
      __syncthreads();
      uint32_t before = sum_before + sum - units;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        if (w < warp) before += scan[w];
        sum_before += scan[w];
      }
      if (pass == 0 && s0 + kThreads < p.sequences) continue;
      if (pass == 0) {
        pieces = PagedPieces(sum_before, gridDim.y);
        if (blockIdx.y >= pieces.count) return;
        u0 = pieces.first(blockIdx.y);
        u1 = pieces.first(blockIdx.y + 1);
      }
      if (pass == 1 || p.sequences <= kThreads) {
        const bool here = units && u0 >= before && u0 < before + units;
        if (here) {
          found_seq = s;
          found_before = before;
        }
        found = __syncthreads_or(here);
      }
    }
  }
  if (!found) return;   // lengths that changed in between
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (uint32_t s = threadIdx.x; s < p.sequences; s += kThreads)
      if (p.lengths[s] < 0 || (uint64_t)p.lengths[s] > (uint64_t)p.max_pages * p.page_size) set_status(p.status, (unsigned int)KB_ERR_INVALID_ARG);
  uint32_t seq = found_seq, seq_first = found_before;   // the sequence and its first unit

  // ---- this warp's copies: the tiles of the piece's sequences one after the other, up to kS ahead of their use
  unsigned char* ring = base + warp * kS * 2 * T::kHalf;
  uint32_t p_seq = seq, p_first = seq_first, p_key = (u0 - seq_first) * kStepKeys + warp * 16, p_end = 0;
  uint32_t p_stage = 0, issued = 0, used = 0, pages_at = 0;
  int pages = -1;                                 // lane i: the page of the key (box = 16: of the step i on) pages_at + ...
  bool p_known = false, bad = false;              // p_end and pages are p_seq's
  unsigned long long there = 0;                   // 16 bits per tile on its way, the next one lowest: keys that are there
  bool ok = true;                                 // no wait has run out
  auto by_page = [&](uint32_t key) { return p.page_shift < 32 ? key >> p.page_shift : key / p.page_size; };
  auto produce = [&]() {
    if (!ok) return;
#pragma unroll 1
    for (;;) {
      if (!p_known) {
        if (p_seq >= p.sequences || p_first >= u1) return;
        const uint32_t keys = paged_length(p.lengths[p_seq], p.max_pages, p.page_size), n = paged_units(keys, kStepKeys);
        p_end = u1 - p_first >= n ? keys : (u1 - p_first) * kStepKeys;
        p_known = true;
        pages_at = p_key + 32 * kStepKeys;        // none yet
      }
      if (p_key < p_end) break;
      p_first += paged_units(paged_length(p.lengths[p_seq], p.max_pages, p.page_size), kStepKeys);
      ++p_seq;
      p_key = warp * 16;
      p_known = false;
    }
    // pages of the next 32 steps at once, or of the 16 keys of this one
    const bool whole = p.box == 16;
    if (!whole || p_key - pages_at >= 32 * kStepKeys) {
      pages_at = p_key;
      const uint32_t key = whole ? p_key + lane * kStepKeys : p_key + (lane & 15);
      pages = -1;
      if (key < p_end) {
        const int page = p.table[p_seq * p.table_row + by_page(key)];
        if (page >= 0 && (uint64_t)page < p.pages)
          pages = page;
        else
          bad = true;
      }
    }
    const uint32_t left = p_end - p_key;
    uint32_t mask;
    if (whole)
      mask = __shfl_sync(0xFFFFFFFFu, pages, (p_key - pages_at) / kStepKeys) >= 0 ? 0xFFFFu : 0u;
    else
      mask = __ballot_sync(0xFFFFFFFFu, pages >= 0) & 0xFFFFu;
    if (left < 16) mask &= (1u << left) - 1;
    there |= (unsigned long long)mask << (16 * (issued - used));
    const uint32_t bar = smem_u32(&full[warp][p_stage]), to = smem_u32(ring + p_stage * 2 * T::kHalf);
    uint32_t boxes = 0;
#pragma unroll 1
    for (uint32_t i = 0; i < 16; i += p.box) boxes += (mask >> i) & 1u;
    expect_tx_elect(bar, boxes * p.box * 128 * kC * 2);
#pragma unroll 1
    for (uint32_t i = 0; i < 16; i += p.box) {
      const int page = __shfl_sync(0xFFFFFFFFu, pages, whole ? (p_key - pages_at) / kStepKeys : i);
      if (((mask >> i) & 1u) == 0) continue;
      const int row = (int)(p_key + i - by_page(p_key + i) * p.page_size);
#pragma unroll 1
      for (uint32_t c = 0; c < p.copies; ++c) {
        tma_load_5d(to + c * 2048 + i * 128, &map_k, (int)(c * 64), row, 0, (int)hk, page, bar);
        tma_load_5d(to + T::kHalf + c * 2048 + i * 128, &map_v, (int)(c * 64), row, 0, (int)hk, page, bar);
      }
    }
    ++issued;
    p_stage = p_stage + 1 == kS ? 0 : p_stage + 1;
    p_key += kStepKeys;
  };
  uint32_t wanted = kS;                           // tiles that are free for copies
  // q as the second operand of the scores, in the lanes' order: heads h0 + 8 n + g
  constexpr uint32_t kQ = NT * kH * 32, kQEach = (kQ + kThreads - 1) / kThreads;
  uint4 q_next[kQEach];
  auto load_q = [&](uint32_t of) {
#pragma unroll
    for (uint32_t e = 0; e < kQEach; ++e) {
      const uint32_t i = e * kThreads + threadIdx.x, head = i / (kH * 32) * 8 + (i & 31) / 4, d = i / 32 % kH * 32 + (i & 3) * 8;
      q_next[e] = make_uint4(0u, 0u, 0u, 0u);
      if (i < kQ && head < heads && d < p.dim)
        q_next[e] = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(p.q) + of * p.q_row + (h0 + head) * p.q_head + d);
    }
  };
  auto store_q = [&](uint32_t to) {
#pragma unroll
    for (uint32_t e = 0; e < kQEach; ++e)
      if (e * kThreads + threadIdx.x < kQ) q_lanes[to][e * kThreads + threadIdx.x] = q_next[e];
  };
  uint32_t q_at = 0;
  // Sequences that this piece has a part of, the one that began earlier and the one that goes on: first unit, units
  uint32_t part_first[2] = {0, 0}, part_units[2] = {0, 0}, part_seq[2] = {0, 0};
  // places in the workspace: a sequence that began in an earlier piece is its piece's first, another its last
  auto place = [&](uint32_t piece, bool began) { return (uint64_t)2 * (piece * per_seq + item) + (began ? 1 : 0); };
  // Four elements d .. of a head's output: o / sum, and its lse
  auto finish = [&](uint32_t of, uint32_t head, uint32_t d, float4 o, float top, float sum) {
    if (head >= heads) return;
    const bool none = sum == 0.0f;   // no score above -infinity
    const float by = 1.0f / sum;
    const float v[4] = {none ? 0.0f : o.x * by, none ? 0.0f : o.y * by, none ? 0.0f : o.z * by, none ? 0.0f : o.w * by};
    unsigned short* to = static_cast<unsigned short*>(p.out) + of * p.o_row + (h0 + head) * p.o_head + d;
    if (p.vec_out && d + 4 <= p.dim) {
      *reinterpret_cast<uint2*>(to) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
    } else {
#pragma unroll 1
      for (int i = 0; i < 4; ++i)
        if (d + i < p.dim) store_elem<DT>(to, i, i < 2 ? (i ? v[1] : v[0]) : (i == 2 ? v[2] : v[3]));
    }
    if (d == 0 && p.lse) p.lse[(uint64_t)of * p.q_heads + h0 + head] = none ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
  };

  uint32_t stage = 0, phase = 0;
  const uint32_t key_of[2] = {paged_kappa(g), paged_kappa(g) + 8};                              // rows g and g + 8 of the scores
  const uint32_t val_of[4] = {2u * t, (2u * t + 1) ^ 4u, 2u * t + 8, ((2u * t + 1) ^ 4u) + 8};   // kappa(2t), kappa(2t + 1), and + 8
#pragma unroll 1
  for (uint32_t u = u0; u < u1 && seq < p.sequences; ++seq) {

    const uint32_t keys = paged_length(p.lengths[seq], p.max_pages, p.page_size), seq_units = paged_units(keys, kStepKeys);
    const uint32_t unit0 = u - seq_first, unit1 = min(seq_units, u1 - seq_first);
    const uint32_t key_end = unit1 == seq_units ? keys : unit1 * kStepKeys;
    float acc[NT][kC][4][4], r[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      r[n][0] = r[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < kC * 16; ++i) acc[n][i / 16][i / 4 % 4][i % 4] = 0.0f;
    }
    unsigned char* scratch = nullptr;          // the tile that this warp used last
    bool fresh = true;
#pragma unroll 1
    for (uint32_t key0 = unit0 * kStepKeys + warp * 16;; key0 += kStepKeys) {
      // copies into tiles that are free: all at first, then the one used before this one; the last one used of this sequence
      // holds the warp's sums before it is free
      if (scratch && key0 < key_end) wanted = 1;
#pragma unroll 1
      for (; wanted; --wanted) produce();
      if (fresh) {
        fresh = false;
        if (u == u0) {   // later sequences' were loaded while the one before was worked on
          load_q(seq);
          store_q(0);
          __syncthreads();
        }
        if (seq_first + seq_units < u1 && seq + 1 < p.sequences) load_q(seq + 1);
      }
      if (key0 >= key_end) break;
      ok = ok && mbar_wait_bounded(&full[warp][stage], phase, abort_flag, p.status);
      __syncwarp();
      const unsigned char* tile = ring + stage * 2 * T::kHalf;
      scratch = ring + stage * 2 * T::kHalf;
      const uint32_t mask = (uint32_t)there & 0xFFFFu;
      there >>= 16;
      ++used;
      if (++stage == kS) {
        stage = 0;
        phase ^= 1u;
      }
      if (!ok) continue;
      auto read = [&](uint32_t at, uint32_t row, int c, uint32_t unit) {   // 16 bytes of a swizzled row
        return *reinterpret_cast<const uint4*>(tile + at + c * 2048 + row * 128 + ((unit ^ (row & 7)) * 16));
      };
      float s[NT][4], s2[NT][4];   // two chains of products
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][i] = s2[n][i] = 0.0f;
#pragma unroll
      for (int h = 0; h < kH; ++h) {
        const uint4 k0 = read(0, key_of[0], h / 2, h % 2 * 4 + t), k1 = read(0, key_of[1], h / 2, h % 2 * 4 + t);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4 qv = q_lanes[q_at][(n * kH + h) * 32 + lane];
          mma_16816<DT>(s[n], k0.x, k1.x, k0.y, k1.y, qv.x, qv.y);
          mma_16816<DT>(s2[n], k0.z, k1.z, k0.w, k1.w, qv.z, qv.w);
        }
      }
      const bool seen0 = (mask >> key_of[0]) & 1u, seen1 = (mask >> key_of[1]) & 1u;
      uint32_t pb[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float x[4];   // keys of rows g, g, g + 8, g + 8; heads 2t, 2t + 1, 2t, 2t + 1
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (i < 2 ? seen0 : seen1) ? (s[n][i] + s2[n][i]) * p.scale_log2 : -INFINITY;
        const float top0 = fmaxf(x[0], x[2]), top1 = fmaxf(x[1], x[3]);
        // r is -infinity until a score was met
        if (__any_sync(0xFFFFFFFFu, top0 - kRoom > r[n][0] + kLazy || top1 - kRoom > r[n][1] + kLazy)) {
          float m0 = top0, m1 = top1;
#pragma unroll
          for (int o = 4; o < 32; o *= 2) {
            m0 = fmaxf(m0, __shfl_xor_sync(0xFFFFFFFFu, m0, o));
            m1 = fmaxf(m1, __shfl_xor_sync(0xFFFFFFFFu, m1, o));
          }
          const float n0 = fmaxf(r[n][0], m0 - kRoom), n1 = fmaxf(r[n][1], m1 - kRoom);
          const float f0 = r[n][0] == -INFINITY ? 0.0f : exp2_fast(r[n][0] - n0), f1 = r[n][1] == -INFINITY ? 0.0f : exp2_fast(r[n][1] - n1);
          r[n][0] = n0;
          r[n][1] = n1;
          l[n][0] *= f0;
          l[n][1] *= f1;
#pragma unroll
          for (int i = 0; i < kC * 16; ++i) acc[n][i / 16][i / 4 % 4][i % 4] *= i % 2 ? f1 : f0;
        }
        const float r0 = known(r[n][0]), r1 = known(r[n][1]);
        const float p0 = exp2_fast(x[0] - r0), p1 = exp2_fast(x[1] - r1), p2 = exp2_fast(x[2] - r0), p3 = exp2_fast(x[3] - r1);
        l[n][0] += p0 + p2;
        l[n][1] += p1 + p3;
        pb[n][0] = transpose_8x8(pack2<DT>(p0, p1));
        pb[n][1] = transpose_8x8(pack2<DT>(p2, p3));
      }
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        uint4 v4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v4[i] = read(T::kHalf, val_of[i], c, g);
          if (((mask >> val_of[i]) & 1u) == 0) v4[i] = make_uint4(0u, 0u, 0u, 0u);   // 0 times NaN is not 0
        }
        const uint32_t w[4][4] = {{v4[0].x, v4[0].y, v4[0].z, v4[0].w}, {v4[1].x, v4[1].y, v4[1].z, v4[1].w},
                                  {v4[2].x, v4[2].y, v4[2].z, v4[2].w}, {v4[3].x, v4[3].y, v4[3].z, v4[3].w}};
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // rows g: element i of the lane's 8, rows g + 8: element 4 + i
          const uint32_t pick = i & 1 ? 0x7632u : 0x5410u;
          const uint32_t a0 = __byte_perm(w[0][i >> 1], w[1][i >> 1], pick), a1 = __byte_perm(w[0][2 + (i >> 1)], w[1][2 + (i >> 1)], pick);
          const uint32_t a2 = __byte_perm(w[2][i >> 1], w[3][i >> 1], pick), a3 = __byte_perm(w[2][2 + (i >> 1)], w[3][2 + (i >> 1)], pick);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_16816<DT>(acc[n][c][i], a0, a1, a2, a3, pb[n][0], pb[n][1]);
        }
      }
      __syncwarp();   // the tile is read
    }

    // The warps' sums meet in shared memory, those of p v in the tile that the warp used last; warps without a tile of this
    // sequence have none.
    const uint32_t warps = min((uint32_t)W, (key_end - unit0 * kStepKeys + 15) / 16);
    const bool whole = unit0 == 0 && unit1 == seq_units;
    if (scratch) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t head = 8 * n + 2 * t + i;
#pragma unroll
          for (int o = 4; o < 32; o *= 2) l[n][i] += __shfl_xor_sync(0xFFFFFFFFu, l[n][i], o);
          if (g == 0) {
            warp_r[warp][head] = r[n][i];
            warp_l[warp][head] = l[n][i];
          }
#pragma unroll
          for (int c = 0; c < kC; ++c) {
            float* to = reinterpret_cast<float*>(scratch) + head * DP + 64 * c + 8 * g;
            *reinterpret_cast<float4*>(to) = make_float4(acc[n][c][0][i], acc[n][c][1][i], acc[n][c][2][i], acc[n][c][3][i]);
            *reinterpret_cast<float4*>(to + 4) = make_float4(acc[n][c][0][2 + i], acc[n][c][1][2 + i], acc[n][c][2][2 + i], acc[n][c][3][2 + i]);
          }
        }
      if (lane == 0) sums_of[warp] = reinterpret_cast<const float4*>(scratch);
    }
    store_q(q_at ^ 1u);
    __syncthreads();
    const uint64_t here = place(blockIdx.y, unit0 == 0);
#pragma unroll 1
    for (uint32_t j = threadIdx.x; j < kHeads * DP / 4; j += kThreads) {
      const uint32_t head = j / (DP / 4), d = j % (DP / 4) * 4;
      float top = -INFINITY, sum = 0.0f;
      float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, w < (int)warps ? warp_r[w][head] : -INFINITY);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        if (w >= (int)warps) break;
        const float4 v = sums_of[w][j];
        const float f = exp2_fast(warp_r[w][head] - known(top));
        sum = fmaf(warp_l[w][head], f, sum);
        o.x = fmaf(v.x, f, o.x);
        o.y = fmaf(v.y, f, o.y);
        o.z = fmaf(v.z, f, o.z);
        o.w = fmaf(v.w, f, o.w);
      }
      if (whole) {
        finish(seq, head, d, o, top, sum);
      } else {
        __stcg(reinterpret_cast<float4*>(p.part) + here * (kHeads * DP / 4) + j, o);
        if (d == 0) __stcg(reinterpret_cast<float2*>(p.part_rl) + here * kHeads + head, make_float2(top, sum));
      }
    }
    if (!whole) {
      const int which = unit0 == 0;
      part_first[which] = seq_first;
      part_units[which] = seq_units;
      part_seq[which] = seq;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the sums were read before copies come in their place
    __syncthreads();                                               // shared memory is used again
    if (scratch) wanted = 1;
    q_at ^= 1u;
    u = seq_first + unit1;
    seq_first += seq_units;
  }

  // Parts are counted once all of the piece is done; the CTA that counts a sequence's last one adds them up.
  uint32_t c0[2], parts[2];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    c0[which] = part_units[which] ? pieces.of(part_first[which]) : 0;
    parts[which] = part_units[which] ? pieces.of(part_first[which] + part_units[which] - 1) - c0[which] + 1 : 0;
    if (threadIdx.x == 32 * which) {
      join_word[which] = 0u;
      if (parts[which]) {
        __threadfence();                                                // the CTA's part is there before it is counted
        unsigned int* count = p.arrived + c0[which] * per_seq + item;   // a sequence that goes on is the last of the piece it began in
        const bool all = atomicAdd(count, 1u) == parts[which] - 1;
        if (all) {
          *count = 0u;                                                  // as the next call expects it
          __threadfence();
        }
        join_word[which] = all;
      }
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    if (!join_word[which]) continue;
    const uint32_t from = which ? c0[1] : c0[0], count = which ? parts[1] : parts[0], of = which ? part_seq[1] : part_seq[0];
#pragma unroll 1
    for (uint32_t j = threadIdx.x; j < kHeads * DP / 4; j += kThreads) {
      const uint32_t head = j / (DP / 4);
      // the parts in the order of the keys, eight on their way at a time
      float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      float top = -INFINITY, sum = 0.0f;
#pragma unroll 1
      for (uint32_t i0 = 0; i0 < count; i0 += 8) {
        float4 v[8];
        float2 rl[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          rl[i] = make_float2(-INFINITY, 0.0f);
          v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (i0 + i >= count) continue;
          const uint64_t at = place(from + i0 + i, i0 + i == 0);
          v[i] = __ldcg(reinterpret_cast<const float4*>(p.part) + at * (kHeads * DP / 4) + j);
          rl[i] = __ldcg(reinterpret_cast<const float2*>(p.part_rl) + at * kHeads + head);
        }
        float higher = top;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) higher = fmaxf(higher, rl[i].x);
        const float f0 = exp2_fast(top - known(higher));     // 0 at first
        o = make_float4(o.x * f0, o.y * f0, o.z * f0, o.w * f0);
        sum *= f0;
        top = higher;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          const float f = exp2_fast(rl[i].x - known(top));
          o.x = fmaf(v[i].x, f, o.x);
          o.y = fmaf(v[i].y, f, o.y);
          o.z = fmaf(v[i].z, f, o.z);
          o.w = fmaf(v[i].w, f, o.w);
          sum = fmaf(rl[i].y, f, sum);
        }
      }
      finish(of, head, j % (DP / 4) * 4, o, top, sum);
    }
  }
  if (bad) set_status(p.status, (unsigned int)KB_ERR_INVALID_ARG);
  if (!ok) {   // what is on its way lands before the CTA ends
#pragma unroll 1
    for (uint32_t i = 0; i < kS; ++i) {
      const unsigned long long t0 = global_ns();
      while (issued > i && !mbar_try_wait(&full[warp][(issued - 1 - i) % kS], ((issued - 1 - i) / kS) & 1u))
        if (global_ns() - t0 > 1000000000ull) break;
    }
  }
}

}  // namespace kb
