// Attention over whole prompts (contract in include/kb_attention.h).
//
// A CTA takes two tiles of 128 queries against the keys and values that they share, 64 keys at a
// time: two neighbouring heads of a group at the same 128 queries, or 256 queries of one head where groups
// are odd (where there are fewer such items than SMs: one tile).  Per tile and step the tensor cores make S = Q K^T (128 x 64, accumulated in tensor memory), a
// warpgroup with one thread per query turns S into P = 2^(S c - r) in registers and writes it back over S
// in 16 bits, and the tensor cores add P V to the output, which stays in tensor memory to the end.
// S has two places per tile: the next step's scores are there when a warpgroup is done with this one's, and
// no product waits for the one before it (one place for 128 keys: 3830 cycles for 128 keys of both tiles, of which the
// warpgroups computed for 1720 and waited for the rest).
//
// The running reference r of a query (shared with the paged kernel: kRoom, kLazy) is raised only where a score, in powers of
// two, is more than kLazy above the largest there was when it was last raised (kRoom + kLazy above r), so the output in
// tensor memory is rescaled a few times per query and not once per step.
//
// What a query does not see never enters its sums: scores behind a mask become -infinity before anything is
// done with them, and values of keys behind a sequence's end are zeroed in shared memory before they
// are multiplied (0 times NaN is not 0).  So are the values that are not finite of an item's last steps, whose keys only some of
// its queries see (two or three steps of an item, five at most): two warps look at them while the step's scores are
// worked on, and the queries that see such values get them back as their outputs are stored (add_taken_out).  The cost is the
// same however long the text is: of 8 x 2048 tokens 384 us, without the look 379; 16384 tokens of 8 heads with a NaN near
// the end 0.50 ms, without it 0.48.  Looking only where an output is not finite would be free, but the rows would have to be computed
// again over all their keys (0.83 s for that NaN), or the item a second time, for which each CTA would wait at its end (77 tokens: 8.9 us, so 7.9).
//
// CTAs are persistent: one per SM takes items off a common count, those with the most keys first, and its copies and
// score products run ahead into the next item while the last one's outputs are stored.
//
// Bound by the tensor cores and the exponentials together: a step's 4 products of both tiles and its 16384 exponentials take
// 1024 cycles each, and the two warpgroups, which feed one with the other's results, keep either busy 63% of the time
// in long prompts and 45% in short ones, where items begin and end.  16384 tokens of 32 heads on 8, causal: 1787 us alone at the full
// clock (1230 TFLOP/s), 2040 in a long run under the power cap, at 1.5 GHz; 8192 tokens without a mask 900 us (1220 TFLOP/s).
//
// Roles: warp 0 copies, warps 1 to 4 issue matrix instructions, warp 5 hands out the items, warps 6 and 7 look at
// values, warps 8 to 11 and 12 to 15 are the tiles' warpgroups, warps 16 to 19 divide and store the outputs of both tiles (4000
// cycles per item, in which the tiles' warpgroups begin the next one).  Every wait is bounded.  The warps' instructions share
// one cache: the look and the outputs' loop are the shorter for it (8 x 2048 tokens: 388 us with the outputs' 64 columns unrolled, so 384).
#pragma once

#include "kb_paged.cuh"
#include "kb_tcgen05.cuh"

namespace kb {

struct PromptParams {
  const int *q_offsets, *k_offsets;   // NULL: one sequence of all tokens
  unsigned int* next;                 // [0] items handed out beyond the first of each CTA, [1] CTAs that have ended; 0 between calls
  uint32_t sequences, q_tokens, k_tokens;
  uint32_t hq, group, dim;
  bool pair;                          // an item's tiles are two heads (else: of one head)
  uint32_t second;                    // queries from an item's first tile to its second: 0, 128, or kPromptNoSecond
  bool causal, vec_out;
  uint32_t phase_keys;                // keys of a phase's sequences; 0: all sequences are one phase
  float scale_log2;
  const void* v;                      // for the values that were taken out
  uint64_t v_row, v_head;
  void* out;
  uint64_t o_row, o_head;
  float* lse;
  unsigned int* status;
};

constexpr uint32_t kPromptKeys = 64;   // keys of a step: two reads of tensor memory, one block of a product's contraction
constexpr uint32_t kPromptNoSecond = 1u << 30;   // past the end of any sequence
// Keys of a sequence, and sequences, at most.  The last warpgroup waits for an item as long as its keys take (16 ns each with two
// tiles at the clock under the power cap: 0.3 s), the others for the next item as long as empty sequences take to be passed over (32
// in half a microsecond), and every wait is given up after 2 s.  It also keeps a number of keys and one of queries, added, within an int.
constexpr uint32_t kPromptMostKeys = 1u << 24, kPromptMostSequences = 1u << 24;
template <int DP>   // dim rounded up to 64 or 128
struct PromptTile {
  static constexpr uint32_t kChunks = DP / 64;                  // of 64 elements = 128 bytes
  static constexpr uint32_t kTileBytes = 128 * DP * 2;          // 128 rows of q
  static constexpr uint32_t kStepBytes = kPromptKeys * DP * 2;  // of k or v
  static constexpr uint32_t kChunkBytes = kPromptKeys * 128;    // of which 64 elements
  static constexpr uint32_t kStages = 256 / kPromptKeys;        // of the rings of k and of v tiles
  static constexpr uint32_t kOutPitch = 144, kOutBytes = 32 * kOutPitch;   // a warp's way out: 128 bytes of 32 rows at a time
  static constexpr uint32_t kSmem = 1024 + 2 * kTileBytes + 2 * kStages * kStepBytes + 4 * kOutBytes;
  // tensor memory: per tile 128 columns for S, in places of kPromptKeys, and DP columns of O
  static constexpr uint32_t kPlaces = 128 / kPromptKeys;
  static constexpr uint32_t kTmemS = 0, kTmemO = 256, kTmemCols = 512;
  static constexpr int kThreads = 640;
  // 96 registers per thread at launch, shared out 48 to the first two warpgroups, 152 to the next two and 80 to the last
  static constexpr int kRegsLaunch = 96, kRegsControl = 48, kRegsSoftmax = 152, kRegsOut = 80;
  static_assert(256 * kRegsControl + 256 * kRegsSoftmax + 128 * kRegsOut <= kThreads * kRegsLaunch, "register shares");
};
static_assert(PromptTile<128>::kSmem <= 227 * 1024 - 1024, "shared memory");

// Steps of kPromptKeys keys that the queries [row, row + rows) of a sequence see: causal ones see the keys up to
// their place plus nk - nq.
__host__ __device__ __forceinline__ uint32_t prompt_steps(uint32_t row, uint32_t rows, uint32_t nq, uint32_t nk, bool causal) {
  if (row >= nq || rows == 0) return 0;
  const int last = (int)(row + rows < nq ? row + rows : nq);           // nq at most 2^30, nk kPromptMostKeys
  const int seen = causal ? min(last + (int)nk - (int)nq, (int)nk) : (int)nk;
  return seen <= 0 ? 0u : ((uint32_t)seen + kPromptKeys - 1) / kPromptKeys;
}
// Keys that query `row` sees
__host__ __device__ __forceinline__ uint32_t prompt_seen(uint32_t row, uint32_t nq, uint32_t nk, bool causal) {
  if (!causal) return nk;
  const int seen = (int)(row + 1) + (int)nk - (int)nq;
  return seen <= 0 ? 0u : min((uint32_t)seen, nk);
}

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
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

// A whole warp waits; false if the wait ran out.
__device__ __noinline__ bool wait_long(uint64_t* bar, uint32_t parity, volatile unsigned int* abort_flag, unsigned int* status) {
  return mbar_wait_bounded(bar, parity, abort_flag, status);
}
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile unsigned int* abort_flag, unsigned int* status) {
  if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xFFFFFFFFu, wait_long(bar, parity, abort_flag, status));
}

// An item: what a CTA's roles have to know of it
struct PromptItem {
  uint32_t q0, nq, k0, nk, row0, head0;   // the sequence, the item's first query and head
  uint32_t n[2];                          // steps of either tile
  uint32_t steps;                         // the larger of the two
  uint32_t look;                          // from this step on: keys that some query does not see, or behind the sequence's end
  uint32_t live;                          // 0: no more items
};
// True if one of the 16-bit numbers of n vectors of 16 bytes (a multiple of 256) is not finite (a warp's work): 0 times it is NaN.
template <int DT>
__device__ __forceinline__ bool some_not_finite(const unsigned char* at, uint32_t n, int lane) {
  uint32_t sum[4] = {0u, 0u, 0u, 0u};
  auto add = [&](uint32_t& to, uint32_t w) {
    if constexpr (DT == KB_BF16)
      asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(to) : "r"(w), "r"(0u));
    else
      asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(to) : "r"(w), "r"(0u));
  };
#pragma unroll 1
  for (const unsigned char *v = at + lane * 16, *end = at + n * 16; v < end; v += 8 * 512)
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      const uint4 w = *reinterpret_cast<const uint4*>(v + i * 512);
      add(sum[0], w.x);
      add(sum[1], w.y);
      add(sum[2], w.z);
      add(sum[3], w.w);
    }
  return __any_sync(0xFFFFFFFFu, ((sum[0] | sum[1] | sum[2] | sum[3]) & 0x7FFF7FFFu) != 0);   // else zeros of either sign
}
// Sets those numbers to zero
template <int DT>
__device__ __noinline__ void take_out(unsigned char* at, uint32_t n, int lane) {
  constexpr uint32_t kInfinity = DT == KB_BF16 ? 0x7F80u : 0x7C00u;
#pragma unroll 1
  for (uint32_t i = lane; i < n * 8; i += 32) {
    unsigned short* e = reinterpret_cast<unsigned short*>(at) + i;
    if ((*e & kInfinity) == kInfinity) *e = 0;
  }
}
// What the outputs' warps have to know of an item's values
struct PromptLooked {
  uint32_t nq, nk, k0, key;   // the sequence; the first key that was looked at
  uint32_t taken_out[2];      // not 0: the even (odd) places of the ring had values that are not finite
};
// 64 columns (from `col` on) of the outputs of a warp's 32 queries (from `first` on; a lane's sum is l) in shared memory: adds
// the values that are not finite and that the products left out, those of the looked-at keys that a query sees.
// With one of them the output is infinite or NaN, whatever the probabilities.  Each key is the last that one query sees.
template <int DT>
__device__ __forceinline__ void add_taken_out(const PromptParams& p, const PromptLooked& x, uint32_t first, float l, uint32_t h, uint32_t col,
                                              unsigned char* rows, uint32_t pitch, int lane) {
  constexpr uint32_t kAtOnce = 4;
  const uint32_t c = col + 2 * lane, last = prompt_seen(min(first + 31, x.nq - 1), x.nq, x.nk, true);
  const uint32_t some = __ballot_sync(0xFFFFFFFFu, l != 0.0f);   // nothing is added to the zeros of a query without a sum
  const unsigned short* v = static_cast<const unsigned short*>(p.v) + (uint64_t)x.k0 * p.v_row + h / p.group * p.v_head + c;
  float sum[2] = {0.0f, 0.0f};
#pragma unroll 1
  for (uint32_t key = x.key; key < last; key += kAtOnce) {
    uint32_t w[kAtOnce];
#pragma unroll
    for (uint32_t u = 0; u < kAtOnce; ++u) w[u] = key + u < last && c < p.dim ? *reinterpret_cast<const uint32_t*>(v + (key + u) * p.v_row) : 0u;
#pragma unroll
    for (uint32_t u = 0; u < kAtOnce; ++u) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float one = load_elem<DT>(&w[u], e);
        if (!(fabsf(one) <= 3.402823466e38f)) sum[e] += one;
      }
      const uint32_t row = key + u + x.nq - x.nk - first;   // of the query that sees all up to this key
      if (row < 32 && (some >> row & 1u) && key + u < last) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (!(sum[e] == 0.0f)) store_elem<DT>(rows + row * pitch, 2 * lane + e, load_elem<DT>(rows + row * pitch, 2 * lane + e) + sum[e]);
      }
    }
  }
}

// Which item has number `it`: a warp's answer.  Up to 32 sequences: the items with the most keys of a phase (mostly there is
// one phase) come first, whatever their sequence, so that no CTA begins a long one when the others are about to end (8192 tokens of
// 32 heads on 8 in 8, 16 and 32 equal prompts 102, 79 and 66 us, one after the other 114, 91 and 74; of ragged lengths 165, 109 and 97, 195, 124
// and 114).  Piece j of a sequence (128 or 256
// queries) is on level base + j of the number of keys (causal), all pieces of it on level base (not causal); the
// level of item `it` is the largest that has more than `it` items on it or above.  More sequences: one after the
// other, the later pieces of each first.
struct PromptSequences {
  uint32_t shift;                 // pieces have 1 << shift queries
  bool causal, held;              // held: all sequences, one per lane
  uint32_t q0, nq, k0, nk;        // of sequence at + lane; with phases of the lane-th longest
  uint32_t phase, phase_first;    // of the sequence, and its first piece
  uint32_t units;                 // heads or pairs of heads of a piece
  uint32_t total, top;            // pieces of all; no level is above
  uint32_t at, before;            // not held: where the search goes on, pieces before that
  __device__ __forceinline__ uint32_t pieces() const { return (nq + (1u << shift) - 1) >> shift; }
  __device__ __forceinline__ uint32_t base() const { return causal ? (nk > nq ? (nk - nq) >> shift : 0u) : nk >> shift; }
  __device__ __forceinline__ uint32_t on_or_above(uint32_t level) const {
    if (!causal) return base() >= level ? pieces() : 0u;
    const uint32_t end = base() + pieces();
    return end <= level ? 0u : min(pieces(), end - level);
  }
};
__device__ __forceinline__ uint32_t warp_prefix(uint32_t v, int lane) {   // sum up to and with this lane
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, v, o);
    if (lane >= o) v += up;
  }
  return v;
}
__device__ __forceinline__ void prompt_load(const PromptParams& p, PromptSequences& q, uint32_t s, bool& bad) {
  q.q0 = q.nq = q.k0 = q.nk = 0;
  if (s >= p.sequences) return;
  if (!p.q_offsets) {
    q.nq = p.q_tokens;
    q.nk = p.k_tokens;
    return;
  }
  const int a = p.q_offsets[s], b = p.q_offsets[s + 1], c = p.k_offsets[s], d = p.k_offsets[s + 1];
  if (a < 0 || a > b || (uint32_t)b > p.q_tokens || c < 0 || c > d || (uint32_t)d > p.k_tokens || (uint32_t)(d - c) > kPromptMostKeys) {
    bad = true;
    return;
  }
  q.q0 = a;
  q.nq = b - a;
  q.k0 = c;
  q.nk = d - c;
}
// Sequences in phases, the longest first, each of as many as have about p.phase_keys keys, so that the keys and values that
// the card is at work on stay in the second-level cache (why and when: prompt_phase_keys).
__device__ __forceinline__ void prompt_phases(const PromptParams& p, PromptSequences& q, int lane) {
  const uint32_t key = q.pieces() ? q.base() + q.pieces() : 0u;
  uint32_t rank = 0;
#pragma unroll 1
  for (int j = 0; j < 32; ++j) {
    const uint32_t other = __shfl_sync(0xFFFFFFFFu, key, j);
    rank += other > key || (other == key && j < lane) ? 1u : 0u;
  }
  PromptSequences sorted = q;
#pragma unroll 1
  for (int j = 0; j < 32; ++j) {
    const bool here = __shfl_sync(0xFFFFFFFFu, rank, j) == (uint32_t)lane;
    const uint32_t q0 = __shfl_sync(0xFFFFFFFFu, q.q0, j), nq = __shfl_sync(0xFFFFFFFFu, q.nq, j);
    const uint32_t k0 = __shfl_sync(0xFFFFFFFFu, q.k0, j), nk = __shfl_sync(0xFFFFFFFFu, q.nk, j);
    if (here) sorted.q0 = q0, sorted.nq = nq, sorted.k0 = k0, sorted.nk = nk;
  }
  q = sorted;
  const uint32_t keys = warp_prefix(q.nk, lane) - q.nk, pieces = warp_prefix(q.pieces(), lane) - q.pieces();   // before this one
  q.phase = keys / p.phase_keys;
  const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, q.phase, 1);
  const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, lane == 0 || before != q.phase);
  const int first = 31 - __clz(firsts & (0xFFFFFFFFu >> (31 - lane)));   // lane of the phase's first sequence
  q.phase_first = __shfl_sync(0xFFFFFFFFu, pieces, first);
}
__device__ __forceinline__ void prompt_begin(const PromptParams& p, PromptSequences& q, int lane, bool report) {
  q.shift = p.second == 128 ? 8 : 7;
  q.causal = p.causal;
  q.held = p.sequences <= 32;
  q.total = q.at = q.before = q.phase = q.phase_first = 0;
  q.units = p.pair ? p.hq / 2 : p.hq;
  bool bad = false;
#pragma unroll 1
  for (uint32_t s0 = 0; s0 < p.sequences; s0 += 32) {
    prompt_load(p, q, s0 + lane, bad);
    q.total += __reduce_add_sync(0xFFFFFFFFu, q.pieces());
  }
  q.top = __reduce_max_sync(0xFFFFFFFFu, q.base() + q.pieces());
  if (!q.held)
    prompt_load(p, q, lane, bad);
  else if (p.phase_keys)
    prompt_phases(p, q, lane);
  if (bad && report) set_status(p.status, (unsigned int)KB_ERR_INVALID_ARG);
}
// The sequence, first query and first head of item `number` < total * units
__device__ __forceinline__ void prompt_find(const PromptParams& p, PromptSequences& q, uint32_t number, int lane, PromptItem& x) {
  uint32_t it = number / q.units;   // among the pieces of all; below: among those of the phase
  x.head0 = (number - it * q.units) * (p.pair ? 2 : 1);
  bool in_phase = true;             // the lane's sequence is
  if (q.held && p.phase_keys) {
    const int src = 31 - __clz(__ballot_sync(0xFFFFFFFFu, q.phase_first <= it));   // the last sequence of a phase that has begun by then
    in_phase = q.phase == __shfl_sync(0xFFFFFFFFu, q.phase, src);
    it -= __shfl_sync(0xFFFFFFFFu, q.phase_first, src);
  }
  // items before those of this round, and lane's among them, of which it leaves out the last `over` pieces
  uint32_t before = 0, mine, over = 0;
  if (q.held) {
    uint32_t lo = 0, hi = q.top;   // more than `it` items on or above lo, not so many on or above hi
#pragma unroll 1
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (__reduce_add_sync(0xFFFFFFFFu, in_phase ? q.on_or_above(mid) : 0u) > it)
        lo = mid;
      else
        hi = mid;
    }
    over = in_phase ? q.on_or_above(lo + 1) : 0u;
    before = __reduce_add_sync(0xFFFFFFFFu, over);
    mine = in_phase ? q.on_or_above(lo) - over : 0u;
  } else {
#pragma unroll 1
    for (;;) {
      mine = q.pieces();
      const uint32_t all = __reduce_add_sync(0xFFFFFFFFu, mine);
      before = q.before;
      if (it < before + all || q.at + 32 >= p.sequences) break;
      q.before += all;
      q.at += 32;
      bool bad = false;
      prompt_load(p, q, q.at + lane, bad);
    }
  }
  const uint32_t first = before + warp_prefix(mine, lane) - mine;
  const int src = max(0, __ffs(__ballot_sync(0xFFFFFFFFu, it >= first && it < first + mine)) - 1);
  x.row0 = __shfl_sync(0xFFFFFFFFu, q.pieces() - 1 - over - (it - first), src) << q.shift;
  x.q0 = __shfl_sync(0xFFFFFFFFu, q.q0, src);
  x.nq = __shfl_sync(0xFFFFFFFFu, q.nq, src);
  x.k0 = __shfl_sync(0xFFFFFFFFu, q.k0, src);
  x.nk = __shfl_sync(0xFFFFFFFFu, q.nk, src);
}

// A warp hands out the CTA's items.  A function of its own: inlined, it took 60 KB of the kernel's instructions, which
// did not fit their cache any more.
__device__ __noinline__ void hand_out_items(const PromptParams& p, PromptSequences q, int lane, PromptItem* items, uint64_t* item_full,
                                            uint64_t* item_empty, uint64_t* want, volatile unsigned int* abort_flag) {
  const uint32_t total = q.total * q.units;
  uint32_t number = blockIdx.x;
#pragma unroll 1
  for (uint32_t taken = 0;;) {
    const uint32_t slot = taken & 1;
    PromptItem x = {};
    if (number < total) {
      prompt_find(p, q, number, lane, x);
      x.n[0] = prompt_steps(x.row0, 128, x.nq, x.nk, p.causal);
      x.n[1] = p.pair ? x.n[0] : prompt_steps(x.row0 + p.second, 128, x.nq, x.nk, p.causal);
      x.steps = max(x.n[0], x.n[1]);
      x.look = prompt_seen(x.row0, x.nq, x.nk, p.causal) / kPromptKeys;
      x.live = 1;
    }
    if (!wait_warp(&item_empty[slot], ((taken >> 1) & 1u) ^ 1u, abort_flag, p.status)) break;
    if (lane == 0) items[slot] = x;
    __syncwarp();
    mbar_arrive_if(&item_full[slot], lane == 0);
    ++taken;
    // towards the end the next one is taken when the last copy of this one is under way, not before: others may be free earlier
    if (!x.live) break;
    if (number + 2 * gridDim.x >= total && !wait_warp(want, (taken - 1) & 1u, abort_flag, p.status)) break;
    if (lane == 0) number = gridDim.x + atomicAdd(p.next, 1u);
    number = __shfl_sync(0xFFFFFFFFu, number, 0);
  }
  // the last CTA leaves the counts as the next call expects them
  if (lane == 0 && atomicAdd(p.next + 1, 1u) == gridDim.x - 1) {
    p.next[0] = 0u;
    p.next[1] = 0u;
  }
}

template <int DT, int DP>
__global__ void __launch_bounds__(PromptTile<DP>::kThreads, 1)
    attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const PromptParams p) {
  using T = PromptTile<DP>;
  constexpr uint32_t kS = T::kStages, kP = T::kPlaces;
  extern __shared__ unsigned char dyn[];
  __shared__ uint64_t q_full[2], q_empty[2], k_full[kS], k_empty[kS], v_full[kS], v_empty[kS], v_tail[kS];
  __shared__ uint64_t s_full[2][kP], p_full[2][kP], o_full[2][kP], item_full[2], item_empty[2], want, drained[5];
  __shared__ uint64_t sum_full[2], o_free[2], looked[4];
  __shared__ PromptLooked values_of[4];   // by the item's number; looked: it is there
  __shared__ float2 row_sum[2][128];   // r and l of the tiles' queries
  __shared__ PromptItem items[2];
  __shared__ uint32_t tmem_base;
  __shared__ unsigned int abort_word;
  volatile unsigned int* abort_flag = &abort_word;
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dyn) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    prefetch_map(&map_q);
    prefetch_map(&map_k);
    prefetch_map(&map_v);
    for (uint32_t i = 0; i < kS; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 2);
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 2);
      mbar_init(&v_tail[i], 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&q_full[t], 1);
      mbar_init(&q_empty[t], 1);
      mbar_init(&item_full[t], 1);
      mbar_init(&item_empty[t], 19);   // all warps but the one that hands them out
      mbar_init(&sum_full[t], 4);
      mbar_init(&o_free[t], 4);
      for (uint32_t b = 0; b < kP; ++b) {
        mbar_init(&s_full[t][b], 1);
        mbar_init(&p_full[t][b], 4);
        mbar_init(&o_full[t][b], 1);
      }
    }
    mbar_init(&want, 1);
    for (int i = 0; i < 4; ++i) mbar_init(&looked[i], 2);
    for (int i = 1; i < 5; ++i) mbar_init(&drained[i], 1);
    abort_word = 0u;
    mbar_fence_init();
  }
  // before the kernel before this one is over: no CTA with tensor memory of its own runs beside this one, whose
  // registers leave no room
  if (warp == 1) tmem_alloc<1>(&tmem_base, T::kTmemCols);
  after_the_kernel_before();
  PromptSequences q;
  if (warp == 5) prompt_begin(p, q, lane, blockIdx.x == 0);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  unsigned char *ring = base + 2 * T::kTileBytes, *ring_v = ring + kS * T::kStepBytes, *way_out = ring_v + kS * T::kStepBytes;
  bool go = true;   // no wait has run out
  auto wait = [&](uint64_t* bar, uint32_t parity) { return go = go && wait_warp(bar, parity & 1u, abort_flag, p.status); };
  uint32_t taken = 0;
  auto next_item = [&](PromptItem& x, auto how) {   // the next item, in order, for a role's warp
    const uint32_t slot = taken & 1;
    if (!how(&item_full[slot], taken >> 1)) return false;
    x = items[slot];
    __syncwarp();
    mbar_arrive_if(&item_empty[slot], lane == 0);
    ++taken;
    return x.live != 0;
  };

  if (warp < 8) regs_shrink<T::kRegsControl>();
  if (warp == 5) {
    hand_out_items(p, q, lane, items, item_full, item_empty, &want, abort_flag);
  } else if (warp == 0) {
    uint32_t k_issued = 0, v_issued = 0, q_items[2] = {0, 0};
    PromptItem x;
#pragma unroll 1
    while (next_item(x, wait)) {
      const int hk = (int)(x.head0 / p.group);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (x.n[t] == 0 || !wait(&q_empty[t], q_items[t] + 1)) continue;
        ++q_items[t];
        const uint32_t bar = smem_u32(&q_full[t]);
        expect_tx_elect(bar, T::kTileBytes);
#pragma unroll
        for (uint32_t c = 0; c < T::kChunks; ++c)
          tma_load_3d(smem_u32(base) + t * T::kTileBytes + c * 16384, &map_q, (int)(c * 64), (int)(x.q0 + x.row0 + t * p.second),
                      (int)(x.head0 + (p.pair ? t : 0)), bar);
      }
      auto copy = [&](const CUtensorMap* map, unsigned char* to, uint64_t* full, uint64_t* empty, uint32_t& issued, uint32_t step) {
        const uint32_t st = issued % kS;
        if (!wait(&empty[st], issued / kS + 1)) return;
        const uint32_t s = smem_u32(to) + st * T::kStepBytes, bar = smem_u32(&full[st]);
        expect_tx_elect(bar, T::kStepBytes);
#pragma unroll
        for (uint32_t c = 0; c < T::kChunks; ++c)
          tma_load_3d(s + c * T::kChunkBytes, map, (int)(c * 64), (int)(x.k0 + step * kPromptKeys), hk, bar);
        ++issued;
      };
      // values that some query does not see have to be looked at first: warps 6 and 7 hand those tiles on
      auto values = [&](uint32_t step) { copy(&map_v, ring_v, step >= x.look ? v_tail : v_full, v_empty, v_issued, step); };
      if (x.steps) copy(&map_k, ring, k_full, k_empty, k_issued, 0);
#pragma unroll 1
      for (uint32_t i = 0; i < x.steps && go; ++i) {
        if (i + 1 < x.steps) copy(&map_k, ring, k_full, k_empty, k_issued, i + 1);
        values(i);
      }
      mbar_arrive_if(&want, lane == 0);
    }
    if (!go) {   // what is on its way lands before the CTA ends
      drain_copies(k_full, kS, k_issued);
      drain_copies(v_full, kS, v_issued);
      for (int t = 0; t < 2; ++t) drain_copies(&q_full[t], 1, q_items[t]);
      __syncwarp();
    }
  } else if (warp == 6 || warp == 7) {
    // Values behind a sequence's end are another's, or anything: zeros.  Those of keys that only some queries see must be finite
    // where they meet the others' zeros.  Each of the two warps has every other place of the ring, which is every other step, and
    // always the same ones: a wait that passes over a phase which is not complete would not wait.
    // (values_of: an item is here once the last warpgroup has taken the item before the last, so what is overwritten was read.)
    uint32_t v_used = 0, phases = 0;
    PromptItem x;
#pragma unroll 1
    while (next_item(x, wait)) {
      uint32_t odd = 0;
#pragma unroll 1
      for (uint32_t i = x.look; i < x.steps; ++i) {
        const uint32_t st = (v_used + i) % kS, rows = min(kPromptKeys, x.nk - i * kPromptKeys);
        if (((st ^ warp) & 1) != 0) continue;
        if (!wait(&v_tail[st], phases >> st)) break;
        phases ^= 1u << st;
        unsigned char* tile = ring_v + st * T::kStepBytes;
        if (rows < kPromptKeys) {
#pragma unroll 1
          for (uint32_t k = rows * 8 + lane; k < kPromptKeys * 8; k += 32)
#pragma unroll
            for (uint32_t c = 0; c < T::kChunks; ++c) *reinterpret_cast<uint4*>(tile + c * T::kChunkBytes + k * 16) = make_uint4(0u, 0u, 0u, 0u);
          __syncwarp();
        }
        if (p.causal && some_not_finite<DT>(tile, T::kStepBytes / 16, lane)) {
          take_out<DT>(tile, T::kStepBytes / 16, lane);
          odd = 1;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        mbar_arrive_if(&v_full[st], lane == 0);
      }
      v_used += x.steps;
      PromptLooked& to = values_of[(taken - 1) & 3];
      if (lane == 0) {
        if (warp == 6) to.nq = x.nq, to.nk = x.nk, to.k0 = x.k0, to.key = x.look * kPromptKeys;
        to.taken_out[warp & 1] = odd;
      }
      __syncwarp();
      if (go) mbar_arrive_if(&looked[(taken - 1) & 3], lane == 0);
    }
  } else if (warp >= 1 && warp < 5) {
    // Four warps issue matrix instructions, so that what one spends on its waits hides under the others' products: warps 1
    // and 2 a tile's scores, warps 3 and 4 a tile's outputs.
    const int t = (warp - 1) & 1;
    uint32_t used = 0, done = 0, q_items = 0;   // tiles of the ring; steps of this tile; items (scores: those with steps of it)
    PromptItem x;
    if (warp < 3) {
      const uint32_t idesc = mma_idesc_f16(DT == KB_BF16, false, 128, kPromptKeys);
      const uint32_t a = smem_u32(base) + t * T::kTileBytes;
#pragma unroll 1
      while (next_item(x, wait)) {
        const uint32_t n = t ? x.n[1] : x.n[0];
        if (n) wait(&q_full[t], q_items++);
#pragma unroll 1
        for (uint32_t i = 0; i < x.steps && go; ++i, ++used) {
          const uint32_t st = used % kS, b = smem_u32(ring) + st * T::kStepBytes;
          wait(&k_full[st], used / kS);   // of steps past the tile's, too: both tiles release K
          if (i < n && go) {
            const uint32_t place = done % kP;
            if (done >= kP && !wait(&o_full[t][place], done / kP - 1)) break;   // S goes where P of kP steps ago was
            tc_fence_after();
#pragma unroll
            for (uint32_t c = 0; c < T::kChunks; ++c)
              mma_f16_block(tmem + T::kTmemS + t * 128 + place * kPromptKeys, smem_desc_k128(a + c * 16384), smem_desc_k128(b + c * T::kChunkBytes),
                            idesc, c > 0);
            mma_commit(&s_full[t][place]);
            if (i + 1 == n) mma_commit(&q_empty[t]);
            ++done;
          }
          if (go) mma_commit(&k_empty[st]);
        }
      }
    } else {
      const uint32_t idesc = mma_idesc_f16(DT == KB_BF16, true, 128, DP);
#pragma unroll 1
      while (next_item(x, wait)) {
        const uint32_t n = t ? x.n[1] : x.n[0];
#pragma unroll 1
        for (uint32_t i = 0; i < x.steps && go; ++i, ++used) {
          const uint32_t st = used % kS, v = smem_u32(ring_v) + st * T::kStepBytes;
          wait(&v_full[st], used / kS);
          if (i < n && go) {
            const uint32_t place = done % kP;
            if (!wait(&p_full[t][place], done / kP)) break;
            // The last item's outputs have been read.  Items without steps of this tile skip this wait, so it stands behind the one
            // for P: that comes from a warpgroup that has waited for the item before the last, and a phase more than one behind
            // would pass for the next.
            if (i == 0 && !wait(&o_free[t], q_items + 1)) break;
            tc_fence_after();
            mma_f16_block_ts(tmem + T::kTmemO + t * DP, tmem + T::kTmemS + t * 128 + place * kPromptKeys, smem_desc_n128(v, T::kChunkBytes),
                             idesc, i > 0);
            mma_commit(&o_full[t][place]);
            ++done;
          }
          if (go) mma_commit(&v_empty[st]);
        }
        ++q_items;
      }
    }
    if (!go) {   // what has been issued ends before tensor memory is freed
      mma_commit(&drained[warp]);
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(&drained[warp], 0))
        if (global_ns() - t0 > 1000000000ull) break;
      __syncwarp();
    }
  } else if (warp >= 8 && warp < 16) {
    regs_grow<T::kRegsSoftmax>();
    const int t = (warp - 8) >> 2, quarter = warp & 3;
    const uint32_t at_s = tmem + T::kTmemS + t * 128 + ((uint32_t)(quarter * 32) << 16);
    const uint32_t at_o = tmem + T::kTmemO + t * DP + ((uint32_t)(quarter * 32) << 16);
    const float c = p.scale_log2;
    // no call between reads of tensor memory and their use: everything is in registers there
    auto wait_here = [&](uint64_t* bar, uint32_t parity) {
      return go = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity & 1u, abort_flag, p.status));
    };
    uint32_t done = 0, items_done = 0;
    PromptItem x;
#pragma unroll 1
    while (next_item(x, wait_here)) {
      const uint32_t n = t ? x.n[1] : x.n[0], nq = x.nq, nk = x.nk;
      const uint32_t row = x.row0 + t * p.second + quarter * 32 + lane;
      const uint32_t seen = row < nq ? prompt_seen(row, nq, nk, p.causal) : 0;
      const uint32_t seen_by_all = __reduce_min_sync(0xFFFFFFFFu, seen);
      float r = -INFINITY, l0 = 0.0f, l1 = 0.0f;
#pragma unroll 1
      for (uint32_t i = 0; i < n; ++i, ++done) {
        const uint32_t place = done % kP, at = at_s + place * kPromptKeys;
        if (!wait_here(&s_full[t][place], done / kP)) break;
        tc_fence_after();
        float s[kPromptKeys];
        tmem_ld32(at, s);
        tmem_ld32(at + 32, s + 32);
        tmem_wait_ld64(s);
        if ((i + 1) * kPromptKeys > seen_by_all) {
          const int left = (int)seen - (int)(i * kPromptKeys);   // keys of this step that the query sees
#pragma unroll
          for (int k = 0; k < (int)kPromptKeys; ++k) s[k] = k < left ? s[k] : -INFINITY;
        }
        float m[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (uint32_t k = 4; k < kPromptKeys - 4; k += 8) {
#pragma unroll
          for (int e = 0; e < 4; ++e) m[e] = max3_nan(m[e], s[k + 2 * e], s[k + 2 * e + 1]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = max_nan(m[e], s[kPromptKeys - 4 + e]);
        const float top = max_nan(max_nan(m[0], m[1]), max_nan(m[2], m[3])) * c;   // scale > 0; NaN stays
        if (__any_sync(0xFFFFFFFFu, !(top - kRoom <= r + kLazy))) {   // raised, or NaN
          float raised = max_nan(r, top - kRoom);
          raised += raised == -INFINITY ? 0.0f : raised - raised;   // +infinity becomes NaN, which all its row becomes
          const float f = r == -INFINITY ? 0.0f : exp2_fast(r - raised);
          r = raised;
          l0 *= f;
          l1 *= f;
          if (i > 0) {
            if (!wait_here(&o_full[t][(done - 1) % kP], (done - 1) / kP)) break;
            tc_fence_after();
#pragma unroll 1
            for (int d = 0; d < DP; d += 32) {
              float o[32];
              tmem_ld32(at_o + d, o);
              tmem_wait_ld(o);
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] *= f;
              tmem_st32(at_o + d, reinterpret_cast<const uint32_t*>(o));
            }
          }
        }
        const float minus_r = -known(r);
        uint32_t w[kPromptKeys / 2];
        // This step's sum: a long row's would round each of its numbers to its own, much larger steps (lse of 131072 keys alike off by
        // 6e-4).  It costs 16384 tokens of dim 128 2040 us, without it 1992, and 4 x 4096 of dim 64 433 us and 419.
        float step0, step1;
#pragma unroll
        for (uint32_t k = 0; k < kPromptKeys; k += 2) {
          float &a = s[k], &b = s[k + 1];
          scale_pair(a, b, c, minus_r);
          a = exp2_fast(a);
          b = exp2_fast(b);
          if (k == 0)
            step0 = a, step1 = b;
          else
            add_pair(step0, step1, a, b);
          w[k / 2] = pack2<DT>(a, b);
        }
        add_pair(l0, l1, step0, step1);
        tmem_st32(at, w);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        mbar_arrive_if(&p_full[t][place], lane == 0);
      }
      // the sums to the last warpgroup, which has taken the last item's by then
      if (!go || !wait_here(&o_free[t], items_done + 1)) break;
      ++items_done;
      row_sum[t][quarter * 32 + lane] = make_float2(r, l0 + l1);
      __syncwarp();
      mbar_arrive_if(&sum_full[t], lane == 0);
    }
  } else if (warp >= 16) {
    // outputs: a tile's sums of p v by its sums of p, while the other warpgroups are at the next item
    regs_shrink<T::kRegsOut>();
    const int quarter = warp & 3;
    unsigned char* rows = way_out + quarter * T::kOutBytes;
    auto wait_here = [&](uint64_t* bar, uint32_t parity) {
      return go = __all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity & 1u, abort_flag, p.status));
    };
    uint32_t done[2] = {0, 0}, items_done = 0;
    PromptItem x;
#pragma unroll 1
    while (next_item(x, wait_here)) {
      if (!wait_here(&looked[items_done & 3], items_done >> 2)) break;
      const PromptLooked& looked_at = values_of[items_done & 3];
#pragma unroll 1
      for (int t = 0; t < 2; ++t) {
        const uint32_t n = t ? x.n[1] : x.n[0], nq = x.nq, h = x.head0 + (p.pair ? t : 0);
        const uint32_t first = x.row0 + t * p.second + quarter * 32, row = first + lane;
        const uint32_t steps = (t ? done[1] : done[0]) + n;
        if (t)
          done[1] = steps;
        else
          done[0] = steps;
        if (!wait_here(&sum_full[t], items_done)) break;
        const float2 rl = row_sum[t][quarter * 32 + lane];
        const float r = rl.x, l = rl.y, by = 1.0f / l;
        const bool none = l == 0.0f, in = row < nq;
        if (n) {
          if (!wait_here(&o_full[t][(steps - 1) % kP], (steps - 1) / kP)) break;
          tc_fence_after();
        }
        // 128 bytes of 32 rows at a time through shared memory, so that a warp's stores cover whole lines
        const uint32_t mask = none ? 0u : 0xFFFFFFFFu, at_o = tmem + T::kTmemO + t * DP + ((uint32_t)(quarter * 32) << 16);
        unsigned short* to = static_cast<unsigned short*>(p.out) + (uint64_t)(x.q0 + first + (lane >> 3)) * p.o_row + h * p.o_head + (lane & 7) * 8;
        const int rows_left = (int)(nq - first) - (lane >> 3);
#pragma unroll 1
        for (int d = 0; d < (int)p.dim && first < nq; d += 64, to += 64) {
#pragma unroll 1
          for (int e = 0; e < 64; e += 32) {
            float o[32];
            uint32_t w[16];
            if (n) {
              tmem_ld32(at_o + d + e, o);
              tmem_wait_ld(o);
            }
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float a = o[k] * by, b = o[k + 1] * by;
              w[k / 2] = pack2<DT>(a, b) & mask;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
              *reinterpret_cast<uint4*>(rows + lane * T::kOutPitch + e * 2 + u * 16) = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
          }
          __syncwarp();
          if (looked_at.taken_out[0] | looked_at.taken_out[1]) {
            add_taken_out<DT>(p, looked_at, first, l, h, d, rows, T::kOutPitch, lane);
            __syncwarp();
          }
          if (d + (lane & 7) * 8 < (int)p.dim) {
            const unsigned char* from = rows + (lane >> 3) * T::kOutPitch + (lane & 7) * 16;
            if (p.vec_out) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (4 * k < rows_left) *reinterpret_cast<uint4*>(to + 4 * k * p.o_row) = *reinterpret_cast<const uint4*>(from + 4 * k * T::kOutPitch);
            } else {
#pragma unroll 1
              for (int k = 0; k < 64; ++k)
                if (k / 8 * 4 < rows_left) to[k / 8 * 4 * p.o_row + k % 8] = reinterpret_cast<const unsigned short*>(from + k / 8 * 4 * T::kOutPitch)[k % 8];
            }
          }
          __syncwarp();
        }
        tc_fence_before();
        __syncwarp();
        mbar_arrive_if(&o_free[t], lane == 0);
        if (in && p.lse) p.lse[(uint64_t)(x.q0 + row) * p.hq + h] = none ? -INFINITY : (r + log2f(l)) * 0.69314718055994531f;
      }
      if (!go) break;
      ++items_done;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_free<1>(tmem, T::kTmemCols);
}

}  // namespace kb
