// Attention of one new token per sequence over a paged cache (contract in include/kb_attention.h).
//
// Bound by the cache's bytes: every key and value is read once for the query heads that share it, up to
// 16 of them, and the rest has to stay out of the way.  Work is divided evenly whatever the lengths: an
// item is a (sequence, group of heads), its units are steps of 128 keys, the units of all items form
// one row that is cut into as many pieces as CTAs fit the card, and a CTA takes the items that its piece
// touches one after the other.  An item that lies in one piece is finished there; otherwise each piece
// leaves its part in the workspace, and the CTA that comes last adds the parts up in the order of the keys.
//
// A warp takes 16 keys of a step at a time, straight from global memory into the registers of
// the warp-wide matrix instructions, with no staging in between.  What makes that possible: the order of a
// contraction is free as long as both operands have the same.
//   scores  S^T[16 keys][8 heads] = K Q^T: lane (g, t) = (lane / 4, lane % 4) holds the elements
//     32 h + 8 t .. + 7 of keys g and g + 8, so that every load is 16 bytes and four lanes read 64 in a row;
//     q is held in the same order.
//   out  O^T[dim][8 heads] = V^T P^T: lane (g, t) holds the elements 64 c + 8 g .. + 7 of the keys 2t, 2t + 1,
//     2t + 8, 2t + 9; two keys' elements are paired by byte permutes, and the rows of the product are
//     whatever elements the lanes' loads brought.  P^T comes from S^T by transposing 8 x 8 matrices of
//     16-bit numbers between lanes.
// The 8-column tile of the instruction holds the heads: fewer than 8 waste matrix work, which is not
// what bounds this kernel.  The exponentials are relative to a running value that is raised only where
// a score exceeds it by more than 2^kLazy; p is rounded to the storage type for the matrix
// instruction, the sum of the rounded p is kept in binary32.
#pragma once

#include "kb_block8.cuh"

namespace kb {

// exp(s) is taken relative to r, as 2^(s' - r) with s' = s * log2(e).  r = (largest s' when it was last raised) - kRoom: the
// largest p is between 2^kRoom and 2^(kRoom + kLazy) <= 2^15, so that binary16 holds it and small p keep their digits.
constexpr float kRoom = 7.0f, kLazy = 8.0f;

struct PagedParams {
  const void* q;
  uint64_t q_row, q_head;
  const void *k, *v;
  uint64_t k_page, k_row, k_head, v_page, v_row, v_head;
  uint64_t pages;
  uint32_t page_size, max_pages;
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
  float* part;                              // [2 * grid][8 NT][DP] sums, then [2 * grid][8 NT][2] (r, sum of p)
  float* part_rl;
  unsigned int* arrived;                    // [grid], zero between calls
  unsigned int* status;
};

constexpr int kPagedWarps = 8, kPagedThreads = 32 * kPagedWarps;
constexpr uint32_t kStepKeys = 16 * kPagedWarps;   // keys of a unit

// A sequence's keys as the table can hold them, and units per group of heads: one at least, for the zeros of an
// empty sequence
__host__ __device__ __forceinline__ uint32_t paged_length(int length, uint32_t max_pages, uint32_t page_size) {
  const uint64_t most = (uint64_t)max_pages * page_size;
  return length <= 0 ? 0u : (uint64_t)length > most ? (uint32_t)most : (uint32_t)length;
}
__host__ __device__ __forceinline__ uint32_t paged_units(uint32_t keys) { return keys ? (keys + kStepKeys - 1) / kStepKeys : 1u; }
// Piece c of `pieces` of a row of n units starts here
__host__ __device__ __forceinline__ unsigned long long piece_first(unsigned long long n, uint32_t c, uint32_t pieces) {
  return n / pieces * c + (n % pieces) * c / pieces;
}
// The piece that unit u lies in
__host__ __device__ __forceinline__ uint32_t piece_of(unsigned long long n, unsigned long long u, uint32_t pieces) {
  uint32_t lo = 0, hi = pieces - 1;
  while (lo < hi) {
    const uint32_t mid = (lo + hi + 1) / 2;
    if (piece_first(n, mid, pieces) <= u)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

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
__device__ __forceinline__ uint4 load_once(const void* p) {   // read through once: not kept in the first-level cache
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// The reference of a row's exponentials as it enters an exponent: 0 while no score above -infinity was met
__device__ __forceinline__ float known(float r) { return r == -INFINITY ? 0.0f : r; }

// DP: 64 or 128, dim rounded up.  NT: tiles of 8 heads.  PAGE16: pages are multiples of 16 keys, so that the 16
// keys of a warp's step lie on one page.
template <int DT, int DP, int NT, bool PAGE16>
__global__ void __launch_bounds__(kPagedThreads, NT == 1 ? 2 : 1) attention_paged_kernel(const PagedParams p) {
  constexpr int kH = DP / 32, kC = DP / 64, kHeads = 8 * NT;
  extern __shared__ float sums[];                 // [warps][heads][DP], and the join's weights
  __shared__ float warp_r[kPagedWarps][kHeads], warp_l[kPagedWarps][kHeads], item_r[kHeads], item_l[kHeads];
  __shared__ unsigned long long scan[kPagedWarps];
  __shared__ uint32_t found_seq, last_word;
  __shared__ unsigned long long found_before;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t per_seq = p.hkv * p.chunks;

  // Units of all items, and the sequence that this piece starts in.
  unsigned long long total = 0, u0 = 0, u1 = 0;
  uint32_t pieces = 1;
  for (int pass = 0; pass < 2; ++pass) {
    unsigned long long before = 0;
    bool found = false;
    for (uint32_t base = 0; base < p.sequences && !found; base += kPagedThreads) {
      const uint32_t s = base + threadIdx.x;
      const uint32_t keys = s < p.sequences ? paged_length(p.lengths[s], p.max_pages, p.page_size) : 0;
      const unsigned long long mine = s < p.sequences ? (unsigned long long)paged_units(keys) * per_seq : 0;
      unsigned long long sum = mine;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const unsigned long long up = __shfl_up_sync(0xFFFFFFFFu, sum, o);
        if (lane >= o) sum += up;
      }
      __syncthreads();
      if (lane == 31) scan[warp] = sum;
      __syncthreads();
      unsigned long long all = 0, mine_before = before + sum - mine;
#pragma unroll
      for (int w = 0; w < kPagedWarps; ++w) {
        if (w < warp) mine_before += scan[w];
        all += scan[w];
      }
      if (pass == 1) {
        const bool here = mine && u0 >= mine_before && u0 < mine_before + mine;
        if (here) {
          found_seq = s;
          found_before = mine_before;
        }
        found = __syncthreads_or(here);
      } else if (blockIdx.x == 0 && s < p.sequences && (p.lengths[s] < 0 || (uint64_t)p.lengths[s] > (uint64_t)p.max_pages * p.page_size)) {
        set_status(p.status, (unsigned int)KB_ERR_INVALID_ARG);
      }
      before += all;
    }
    if (pass == 0) {
      total = before;
      pieces = (uint32_t)min((unsigned long long)gridDim.x, total);   // every piece has a unit
      if (blockIdx.x >= pieces) return;
      u0 = piece_first(total, blockIdx.x, pieces);
      u1 = piece_first(total, blockIdx.x + 1, pieces);
    }
  }
  __syncthreads();
  uint32_t seq = found_seq;
  unsigned long long seq_first = found_before;   // the first unit of the sequence's first item

  for (unsigned long long u = u0; u < u1;) {
    const uint32_t keys = paged_length(p.lengths[seq], p.max_pages, p.page_size), units = paged_units(keys);
    const uint32_t item = (uint32_t)((u - seq_first) / units), unit0 = (uint32_t)((u - seq_first) % units);
    const uint32_t unit1 = (uint32_t)min((unsigned long long)units, unit0 + (u1 - u));
    const unsigned long long item_first = u - unit0;
    const uint32_t hk = item / p.chunks, h0 = hk * p.group + item % p.chunks * kHeads;   // first query head
    const uint32_t heads = min((uint32_t)kHeads, (hk + 1) * p.group - h0);

    // q as the second operand of the scores: heads h0 + 8 n + g
    uint32_t qb[NT][kH][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < kH; ++h) {
        const uint32_t head = 8 * n + g, d = 32 * h + 8 * t;
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (head < heads && d < p.dim)
          w = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(p.q) + seq * p.q_row + (h0 + head) * p.q_head + d);
        qb[n][h][0] = w.x;
        qb[n][h][1] = w.y;
        qb[n][h][2] = w.z;
        qb[n][h][3] = w.w;
      }
    float acc[NT][kC][4][4], r[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      r[n][0] = r[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < kC * 16; ++i) acc[n][i / 16][i / 4 % 4][i % 4] = 0.0f;
    }

    const int* table = p.table + seq * p.table_row;
    const uint32_t key_end = min(keys, unit1 * kStepKeys);
    const unsigned short* kh = static_cast<const unsigned short*>(p.k) + hk * p.k_head;
    const unsigned short* vh = static_cast<const unsigned short*>(p.v) + hk * p.v_head;
    bool bad = false;
    // Page of key `key`, -1 where there is none or the table names one that is not there
    auto page_of = [&](uint32_t key) -> int {
      if (key >= key_end) return -1;
      const int page = table[key / p.page_size];
      if (page >= 0 && (uint64_t)page < p.pages) return page;
      bad = true;
      return -1;
    };
    uint4 kr[2][kH], vr[4][kC];
    // The pages of a warp's next 32 steps (PAGE16: lane i has step i's) or of the next step's 16 keys (lane i has key i's)
    uint32_t key0 = unit0 * kStepKeys + warp * 16;
    int pages = -1;
    uint32_t ahead = 0;                       // PAGE16: steps whose pages the lanes hold
    uint32_t pages_at = key0;                 // the key that lane 0's page belongs to
    auto fetch_pages = [&](uint32_t key) {
      pages_at = key;
      pages = PAGE16 ? page_of(key + lane * kStepKeys) : page_of(key + (lane & 15));
      ahead = 32;
    };
    // Page and place on it of key key0 + i
    auto row_of = [&](uint32_t key, int i, int& page, uint32_t& off) {
      if constexpr (PAGE16) {
        page = __shfl_sync(0xFFFFFFFFu, pages, (key - pages_at) / kStepKeys);
        off = key % p.page_size + i;
        if (key + i >= key_end) page = -1;
      } else {
        page = __shfl_sync(0xFFFFFFFFu, pages, i);
        off = (key + i) % p.page_size;
      }
    };
    auto load_k = [&](uint32_t key, bool (&there)[2]) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int page;
        uint32_t off;
        row_of(key, g + 8 * i, page, off);
        there[i] = page >= 0;
        const unsigned short* at = kh + (uint64_t)(uint32_t)page * p.k_page + (uint64_t)off * p.k_row + 8 * t;
#pragma unroll
        for (int h = 0; h < kH; ++h)
          kr[i][h] = there[i] && 32 * h + 8 * t < (int)p.dim ? load_once(at + 32 * h) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    auto load_v = [&](uint32_t key) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int page;
        uint32_t off;
        row_of(key, 2 * t + (i & 1) + 8 * (i >> 1), page, off);
        const unsigned short* at = vh + (uint64_t)(uint32_t)page * p.v_page + (uint64_t)off * p.v_row + 8 * g;
#pragma unroll
        for (int c = 0; c < kC; ++c)
          vr[i][c] = page >= 0 && 64 * c + 8 * g < (int)p.dim ? load_once(at + 64 * c) : make_uint4(0u, 0u, 0u, 0u);
      }
    };

    bool there[2] = {false, false};
    if (key0 < key_end) {
      fetch_pages(key0);
      load_k(key0, there);
    }
    for (; key0 < key_end; key0 += kStepKeys) {
      load_v(key0);
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
        for (int h = 0; h < kH; ++h) {
          mma_16816<DT>(s[n], kr[0][h].x, kr[1][h].x, kr[0][h].y, kr[1][h].y, qb[n][h][0], qb[n][h][1]);
          mma_16816<DT>(s[n], kr[0][h].z, kr[1][h].z, kr[0][h].w, kr[1][h].w, qb[n][h][2], qb[n][h][3]);
        }
      }
      const bool seen0 = there[0], seen1 = there[1];
      if (key0 + kStepKeys < key_end) {   // the next keys are on their way while these are worked on
        if (!PAGE16 || (key0 + kStepKeys - pages_at) / kStepKeys >= ahead) fetch_pages(key0 + kStepKeys);
        load_k(key0 + kStepKeys, there);
      }
      uint32_t pb[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float x[4];   // keys g, g, g + 8, g + 8; heads 2t, 2t + 1, 2t, 2t + 1
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (i < 2 ? seen0 : seen1) ? s[n][i] * p.scale_log2 : -INFINITY;
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
        const uint32_t* v0 = reinterpret_cast<const uint32_t*>(&vr[0][c]);
        const uint32_t* v1 = reinterpret_cast<const uint32_t*>(&vr[1][c]);
        const uint32_t* v2 = reinterpret_cast<const uint32_t*>(&vr[2][c]);
        const uint32_t* v3 = reinterpret_cast<const uint32_t*>(&vr[3][c]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // rows g: element i of the lane's 8, rows g + 8: element 4 + i
          const uint32_t pick = i & 1 ? 0x7632u : 0x5410u;
          const uint32_t a0 = __byte_perm(v0[i >> 1], v1[i >> 1], pick), a1 = __byte_perm(v0[2 + (i >> 1)], v1[2 + (i >> 1)], pick);
          const uint32_t a2 = __byte_perm(v2[i >> 1], v3[i >> 1], pick), a3 = __byte_perm(v2[2 + (i >> 1)], v3[2 + (i >> 1)], pick);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_16816<DT>(acc[n][c][i], a0, a1, a2, a3, pb[n][0], pb[n][1]);
        }
      }
    }
    if (bad) set_status(p.status, (unsigned int)KB_ERR_INVALID_ARG);

    // The warps' parts: one reference for all, sums of p over the lanes, sums of p v over the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int o = 4; o < 32; o *= 2) l[n][i] += __shfl_xor_sync(0xFFFFFFFFu, l[n][i], o);
        if (g == 0) {
          warp_r[warp][8 * n + 2 * t + i] = r[n][i];
          warp_l[warp][8 * n + 2 * t + i] = l[n][i];
        }
      }
    __syncthreads();
    if (threadIdx.x < kHeads) {
      float top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kPagedWarps; ++w) top = fmaxf(top, warp_r[w][threadIdx.x]);
#pragma unroll
      for (int w = 0; w < kPagedWarps; ++w) {
        const float f = warp_r[w][threadIdx.x] == -INFINITY ? 0.0f : exp2_fast(warp_r[w][threadIdx.x] - top);
        sum += warp_l[w][threadIdx.x] * f;
      }
      item_r[threadIdx.x] = top;
      item_l[threadIdx.x] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t head = 8 * n + 2 * t + i;
        const float f = r[n][i] == -INFINITY ? 0.0f : exp2_fast(r[n][i] - item_r[head]);
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          float* to = sums + ((uint32_t)warp * kHeads + head) * DP + 64 * c + 8 * g;
          *reinterpret_cast<float4*>(to) = make_float4(acc[n][c][0][i] * f, acc[n][c][1][i] * f, acc[n][c][2][i] * f, acc[n][c][3][i] * f);
          *reinterpret_cast<float4*>(to + 4) =
              make_float4(acc[n][c][0][2 + i] * f, acc[n][c][1][2 + i] * f, acc[n][c][2][2 + i] * f, acc[n][c][3][2 + i] * f);
        }
      }
    __syncthreads();

    // Four elements of a head, of sum l and reference r, to the outputs
    auto finish = [&](uint32_t head, uint32_t d, float4 o, float top, float sum) {
      if (head >= heads) return;
      const float by = 1.0f / sum;
      const bool none = sum == 0.0f;   // no score above -infinity
      const float v[4] = {none ? 0.0f : o.x * by, none ? 0.0f : o.y * by, none ? 0.0f : o.z * by, none ? 0.0f : o.w * by};
      unsigned short* to = static_cast<unsigned short*>(p.out) + seq * p.o_row + (h0 + head) * p.o_head + d;
      if (p.vec_out && d + 4 <= p.dim) {
        *reinterpret_cast<uint2*>(to) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (d + i < p.dim) store_elem<DT>(to, i, v[i]);
      }
      if (d == 0 && p.lse) p.lse[(uint64_t)seq * p.q_heads + h0 + head] = none ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
    };
    const bool whole = unit0 == 0 && unit1 == units;
    // this piece's place in the workspace: an item that began earlier is the piece's first, the other its last
    float* mine = p.part + (uint64_t)(2 * blockIdx.x + (unit0 == 0)) * kHeads * DP;
    for (uint32_t i = threadIdx.x; i < kHeads * DP / 4; i += kPagedThreads) {
      float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kPagedWarps; ++w) {
        const float4 x = reinterpret_cast<const float4*>(sums)[w * (kHeads * DP / 4) + i];
        o.x += x.x;
        o.y += x.y;
        o.z += x.z;
        o.w += x.w;
      }
      if (whole)
        finish(i / (DP / 4), i % (DP / 4) * 4, o, item_r[i / (DP / 4)], item_l[i / (DP / 4)]);
      else
        __stcg(reinterpret_cast<float4*>(mine) + i, o);
    }
    if (!whole) {
      if (threadIdx.x < kHeads)
        __stcg(reinterpret_cast<float2*>(p.part_rl) + (uint64_t)(2 * blockIdx.x + (unit0 == 0)) * kHeads + threadIdx.x,
               make_float2(item_r[threadIdx.x], item_l[threadIdx.x]));
      const uint32_t c0 = piece_of(total, item_first, pieces), c1 = piece_of(total, item_first + units - 1, pieces);
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        const bool last = atomicAdd(p.arrived + c0, 1u) == c1 - c0;
        if (last) p.arrived[c0] = 0u;   // as the next call expects it
        last_word = last;
        __threadfence();
      }
      __syncthreads();
      if (last_word) {
        const uint32_t parts = c1 - c0 + 1;
        auto place = [&](uint32_t i) { return (uint64_t)(2 * (c0 + i) + (i == 0)); };
        if (threadIdx.x < kHeads) {
          const float2* rl = reinterpret_cast<const float2*>(p.part_rl) + threadIdx.x;
          float top = -INFINITY, sum = 0.0f;
          for (uint32_t i = 0; i < parts; ++i) top = fmaxf(top, __ldcg(rl + place(i) * kHeads).x);
          for (uint32_t i = 0; i < parts; ++i) {
            const float2 x = __ldcg(rl + place(i) * kHeads);
            const float f = x.x == -INFINITY ? 0.0f : exp2_fast(x.x - top);
            sums[i * kHeads + threadIdx.x] = f;
            sum += x.y * f;
          }
          item_r[threadIdx.x] = top;
          item_l[threadIdx.x] = sum;
        }
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < kHeads * DP / 4; j += kPagedThreads) {
          const uint32_t head = j / (DP / 4);
          float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
          for (uint32_t i = 0; i < parts; ++i) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(p.part) + place(i) * (kHeads * DP / 4) + j);
            const float f = sums[i * kHeads + head];
            o.x = fmaf(x.x, f, o.x);
            o.y = fmaf(x.y, f, o.y);
            o.z = fmaf(x.z, f, o.z);
            o.w = fmaf(x.w, f, o.w);
          }
          finish(head, j % (DP / 4) * 4, o, item_r[head], item_l[head]);
        }
      }
    }
    __syncthreads();   // shared memory is used again
    u += unit1 - unit0;
    if (u - seq_first == (unsigned long long)units * per_seq && u < u1) {
      seq_first = u;
      ++seq;
    }
  }
}

}  // namespace kb
