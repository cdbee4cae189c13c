// Norms of queries and keys for each head with the position rotation, in one pass that also stores the
// turned keys and the values in a paged cache (contract in include/kb_attention.h).
//
// Bound by bytes: every element is read once and written once or twice.  A head's row of dim elements
// belongs to L lanes of a warp (8 elements each), so that its sum of squares takes log2(L) shuffles and
// nothing leaves the registers.  The angles are the same for all heads of a token: a CTA works on
// whole tokens and first puts their cosines and sines into shared memory, one per thread.
//
// An angle is position * inv_freq radians, and only its fraction of a turn matters.  inv_freq / (2 pi) is
// taken to a 64-bit fixed-point fraction; its product with the position, modulo 2^64, is exact, so
// the error is the fraction's own (2^-53 of it) times the position, whatever the position.  The quarter of the turn
// goes off as an integer and at most an eighth of a turn on either side is left for sincospi.
#pragma once

#include <type_traits>

#include "kb_block8.cuh"

namespace kb {

struct RopeParams {
  const void *q, *k, *v;
  uint64_t q_row, q_head, k_row, k_head, v_row, v_head;
  void *q_out, *k_out;
  uint64_t qo_row, qo_head, ko_row, ko_head;
  void *k_cache, *v_cache;             // NULL: no cache
  uint64_t kc_page, kc_row, kc_head, vc_page, vc_row, vc_head;
  uint64_t slots_end;                  // pages * page_size
  uint32_t page_size;
  const long long* positions;
  const long long* slots;
  const double* inv_freq;
  const void *q_weight, *k_weight;     // NULL: 1
  bool param_f32, norm, interleaved;
  float eps;
  uint64_t tokens;
  uint32_t hq, hkv;
  uint32_t dim, half;                  // half: pairs that are turned
  unsigned int* status;
};

constexpr uint32_t kRopeThreads = 256;
constexpr uint32_t kRopeTokens = 8;       // tokens per CTA, at most
constexpr uint32_t kRopeMaxHalf = 128;

// cos and sin of the angle position * freq radians
__host__ __device__ __forceinline__ uint64_t rope_turn(double freq) {   // part of a turn per position, in units of 2^-64
  const double t = freq * 0.15915494309189533577;   // 1 / (2 pi)
  const double part = t - floor(t);
  return part < 1.0 ? (uint64_t)(part * 18446744073709551616.0) : 0ull;
}
__device__ __forceinline__ float2 rope_cos_sin(long long position, double freq) {
  const uint64_t turn = (uint64_t)position * rope_turn(freq);
  const uint32_t quarter = (uint32_t)((turn + (1ull << 61)) >> 62);              // 0..3, 4 wraps to 0
  const long long rest = (long long)(turn - ((uint64_t)(quarter & 3u) << 62));   // within an eighth of a turn
  float s, c;
  sincospif((float)rest * 0x1p-63f, &s, &c);
  const float2 cs = (quarter & 1u) ? make_float2(-s, c) : make_float2(c, s);
  return (quarter & 2u) ? make_float2(-cs.x, -cs.y) : cs;
}

// What both kernels begin with: the CTA's cosines and sines, and where its tokens' keys and values go in the
// cache (-1: nowhere).
struct RopeShared {
  float cos_of[kRopeTokens][kRopeMaxHalf], sin_of[kRopeTokens][kRopeMaxHalf];
  long long at_k[kRopeTokens], at_v[kRopeTokens];
};
__device__ __forceinline__ void rope_begin(const RopeParams& p, RopeShared& s, uint64_t t0, uint32_t ntok) {
  for (uint32_t i = threadIdx.x; i < ntok * p.half; i += kRopeThreads) {
    const uint32_t t = i / p.half, f = i % p.half;
    const float2 cs = rope_cos_sin(p.positions[t0 + t], p.inv_freq[f]);
    s.cos_of[t][f] = cs.x;
    s.sin_of[t][f] = cs.y;
  }
  if (p.k_cache && threadIdx.x < ntok) {
    const long long slot = p.slots[t0 + threadIdx.x];
    const bool in = slot >= 0 && (uint64_t)slot < p.slots_end;
    if (slot >= 0 && !in) set_status(p.status, (unsigned int)KB_ERR_INVALID_ARG);
    const uint64_t page = in ? (uint64_t)slot / p.page_size : 0, off = in ? (uint64_t)slot % p.page_size : 0;
    s.at_k[threadIdx.x] = in ? (long long)(page * p.kc_page + off * p.kc_row) : -1;
    s.at_v[threadIdx.x] = in ? (long long)(page * p.vc_page + off * p.vc_row) : -1;
  }
}
template <int DT>
__device__ __forceinline__ float rope_weight(const RopeParams& p, const void* w, uint32_t e) {
  if (!w || !p.norm || e >= p.dim) return 1.0f;
  return p.param_f32 ? static_cast<const float*>(w)[e] : load_elem<DT>(w, e);
}

// Rows on vector boundaries with dim a multiple of 8 and pairs of which four make a vector.  L lanes hold a
// row, two vectors of four elements each, so that the elements of a pair are in one lane: of halves, lane c
// has 4 c .. + 3 and half + 4 c .. + 3, and the lanes after those have 8 of the elements that are not turned each;
// of neighbours, 8 c .. + 7.  A warp works on 32 / L heads of one kind at a time, so that what differs between
// q, k and v is the same for all its lanes, and has the next kRopeAhead pieces on their way meanwhile
// (16384 tokens of 32 + 8 + 8 heads of 128, bf16, stored in a cache: one row at a time 176 us).
__device__ __forceinline__ void vec_words(uint2 v, uint32_t* w) { w[0] = v.x, w[1] = v.y; }
__device__ __forceinline__ void vec_words(uint4 v, uint32_t* w) { w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w; }
__device__ __forceinline__ void words_vec(const uint32_t* w, uint2& v) { v = make_uint2(w[0], w[1]); }
__device__ __forceinline__ void words_vec(const uint32_t* w, uint4& v) { v = make_uint4(w[0], w[1], w[2], w[3]); }
template <int DT>
struct RopePiece {
  static constexpr int kWords = DT == KB_F32 ? 8 : 4, kAhead = DT == KB_F32 ? 2 : 4;
};
template <int DT, int L>
__global__ void __launch_bounds__(kRopeThreads, 3) qk_norm_rope_kernel(const RopeParams p, const uint32_t per_cta) {
  constexpr int kWarps = kRopeThreads / 32, kBytes = DT == KB_F32 ? 4 : 2, kWords = RopePiece<DT>::kWords, kAhead = RopePiece<DT>::kAhead;
  constexpr uint32_t kHeads = 32 / L;        // heads of a piece
  using Vec = typename std::conditional<DT == KB_F32, uint4, uint2>::type;
  __shared__ __align__(16) RopeShared sh;
  const uint64_t t0 = (uint64_t)blockIdx.x * per_cta;
  const uint32_t ntok = (uint32_t)min((uint64_t)per_cta, p.tokens - t0);
  const uint32_t warp = threadIdx.x >> 5, c = threadIdx.x % L, sub = (threadIdx.x & 31) / L;
  // pieces of a token: queries', keys', values'
  const uint32_t nq = p.q_out ? (p.hq + kHeads - 1) / kHeads : 0, nkv = (p.hkv + kHeads - 1) / kHeads;
  const uint32_t nk = p.k_out || p.k_cache ? nkv : 0, per_token = nq + nk + (p.k_cache ? nkv : 0);
  // the lane's two vectors, and its pairs
  const uint32_t turned = p.interleaved ? p.dim / 8 : p.half / 4;   // lanes with pairs (the rest have cosine 1)
  const bool has = c * 8 < p.dim;
  const uint32_t ea = p.interleaved ? 8 * c : c < turned ? 4 * c : 2 * p.half + 8 * (c - turned);
  const uint32_t eb = p.interleaved || c >= turned ? ea + 4 : p.half + 4 * c;

  struct Place {
    uint32_t t, piece;
  };
  auto forward = [&](Place x) {
    x.piece += kWarps;
    while (x.piece >= per_token) {
      x.piece -= per_token;
      ++x.t;
    }
    return x;
  };
  auto load = [&](Place x, uint32_t* raw) {
    const bool is_q = x.piece < nq, is_k = !is_q && x.piece < nq + nk;
    const uint32_t head = (x.piece - (is_q ? 0 : is_k ? nq : nq + nk)) * kHeads + sub;
    const void* src = is_q ? p.q : is_k ? p.k : p.v;
    const uint64_t row = is_q ? p.q_row : is_k ? p.k_row : p.v_row, step = is_q ? p.q_head : is_k ? p.k_head : p.v_head;
#pragma unroll
    for (int i = 0; i < kWords; ++i) raw[i] = 0u;
    if (x.t < ntok && has && head < (is_q ? p.hq : p.hkv)) {
      const unsigned char* from = static_cast<const unsigned char*>(src) + ((t0 + x.t) * row + head * step) * kBytes;
      const Vec a = *reinterpret_cast<const Vec*>(from + ea * kBytes), b = *reinterpret_cast<const Vec*>(from + eb * kBytes);
      vec_words(a, raw);
      vec_words(b, raw + kWords / 2);
    }
  };
  Place ahead{0, warp};
  while (ahead.piece >= per_token) {
    ahead.piece -= per_token;
    ++ahead.t;
  }
  Place now = ahead;
  uint32_t next[kAhead][kWords];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    load(ahead, next[u]);
    ahead = forward(ahead);
  }
  rope_begin(p, sh, t0, ntok);
  float wq[8], wk[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t e = j < 4 ? ea + j : eb + j - 4;
    wq[j] = rope_weight<DT>(p, p.q_weight, e);
    wk[j] = rope_weight<DT>(p, p.k_weight, e);
  }
  const float per_dim = 1.0f / (float)p.dim;
  __syncthreads();

  while (now.t < ntok) {
    uint32_t raw[kAhead][kWords];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) raw[u][i] = next[u][i];
      load(ahead, next[u]);
      ahead = forward(ahead);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u, now = forward(now)) {
      if (now.t >= ntok) break;   // the same for the whole warp
      const bool is_q = now.piece < nq, is_k = !is_q && now.piece < nq + nk;
      const uint32_t head = (now.piece - (is_q ? 0 : is_k ? nq : nq + nk)) * kHeads + sub;
      const uint64_t token = t0 + now.t;
      auto put = [&](void* dst, uint64_t at) {
        unsigned char* to = static_cast<unsigned char*>(dst) + at * kBytes;
        Vec a, b;
        words_vec(raw[u], a);
        words_vec(raw[u] + kWords / 2, b);
        *reinterpret_cast<Vec*>(to + ea * kBytes) = a;
        *reinterpret_cast<Vec*>(to + eb * kBytes) = b;
      };
      if (is_q || is_k) {
        float v[8];
        if constexpr (DT == KB_F32) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(raw[u][j]);
        } else {
          Elem<DT>::decode(make_uint4(raw[u][0], raw[u][1], raw[u][2], raw[u][3]), v);
        }
        if (p.norm) {
          float sum = 0.0f;
          if (has) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(v[j], v[j], sum);
          }
#pragma unroll
          for (int o = L / 2; o > 0; o /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
          const float by = rsqrtf(fmaf(sum, per_dim, p.eps));
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= by * (is_q ? wq[j] : wk[j]);
        }
        if (c < turned) {
          const float4 cs = *reinterpret_cast<const float4*>(&sh.cos_of[now.t][4 * c]), sn = *reinterpret_cast<const float4*>(&sh.sin_of[now.t][4 * c]);
          const float co[4] = {cs.x, cs.y, cs.z, cs.w}, si[4] = {sn.x, sn.y, sn.z, sn.w};
          if (!p.interleaved) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float a = v[j], b = v[j + 4];
              v[j] = fmaf(a, co[j], -(b * si[j]));
              v[j + 4] = fmaf(b, co[j], a * si[j]);
            }
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float a = v[2 * j], b = v[2 * j + 1];
              if (4 * c + j >= p.half) continue;
              v[2 * j] = fmaf(a, co[j], -(b * si[j]));
              v[2 * j + 1] = fmaf(b, co[j], a * si[j]);
            }
          }
        }
        if constexpr (DT == KB_F32) {
#pragma unroll
          for (int j = 0; j < 8; ++j) raw[u][j] = __float_as_uint(v[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[u][j] = pack2<DT>(v[2 * j], v[2 * j + 1]);
        }
      }
      if (!has || head >= (is_q ? p.hq : p.hkv)) continue;
      if (is_q) {
        put(p.q_out, token * p.qo_row + head * p.qo_head);
      } else if (is_k) {
        if (p.k_out) put(p.k_out, token * p.ko_row + head * p.ko_head);
        if (p.k_cache && sh.at_k[now.t] >= 0) put(p.k_cache, (uint64_t)sh.at_k[now.t] + head * p.kc_head);
      } else if (sh.at_v[now.t] >= 0) {
        put(p.v_cache, (uint64_t)sh.at_v[now.t] + head * p.vc_head);
      }
    }
  }
}

// Any other rows: a row at a time per L lanes, element by element, the pairs' other halves through shared memory.
template <int DT, int L>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_plain_kernel(const RopeParams p, const uint32_t per_cta) {
  constexpr uint32_t kSlots = kRopeThreads / L;
  __shared__ RopeShared sh;
  __shared__ float swap[kRopeThreads * 8];
  const uint64_t t0 = (uint64_t)blockIdx.x * per_cta;
  const uint32_t ntok = (uint32_t)min((uint64_t)per_cta, p.tokens - t0), c = threadIdx.x % L, slot = threadIdx.x / L;
  float* row = swap + slot * (L * 8);
  rope_begin(p, sh, t0, ntok);
  __syncthreads();
  const uint32_t first = p.q_out ? 0 : p.hq, rows = p.hq + (p.k_out || p.k_cache ? p.hkv : 0) + (p.k_cache ? p.hkv : 0);
  for (uint32_t t = 0; t < ntok; ++t)
    for (uint32_t r0 = first; r0 < rows; r0 += kSlots) {   // the same number of times for all lanes: rows take shuffles
      const uint64_t token = t0 + t;
      const uint32_t r = r0 + slot;
      const bool is_q = r < p.hq, is_k = !is_q && r < p.hq + p.hkv, in = r < rows, turn = in && (is_q || is_k);
      const uint32_t h = is_q ? r : is_k ? r - p.hq : r - p.hq - p.hkv;
      const void* src = is_q ? p.q : is_k ? p.k : p.v;
      const uint64_t at = is_q ? token * p.q_row + h * p.q_head : is_k ? token * p.k_row + h * p.k_head : token * p.v_row + h * p.v_head;
      float v[8], sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = in && j * L + c < p.dim ? load_elem<DT>(src, at + j * L + c) : 0.0f;
        sum = fmaf(v[j], v[j], sum);
      }
#pragma unroll
      for (int o = L / 2; o > 0; o /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      if (p.norm && turn) {
        const float by = rsqrtf(sum / (float)p.dim + p.eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= by * rope_weight<DT>(p, is_q ? p.q_weight : p.k_weight, j * L + c);
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 8; ++j) row[j * L + c] = v[j];
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t e = j * L + c;
        if (turn && e < 2 * p.half) {
          const bool lower = p.interleaved ? (e & 1u) == 0 : e < p.half;
          const uint32_t f = p.interleaved ? e / 2 : lower ? e : e - p.half;
          const float other = row[p.interleaved ? e ^ 1u : lower ? e + p.half : e - p.half] * sh.sin_of[t][f];
          v[j] = fmaf(v[j], sh.cos_of[t][f], lower ? -other : other);
        }
        if (!in || e >= p.dim) continue;
        if (is_q) {
          store_elem<DT>(p.q_out, token * p.qo_row + h * p.qo_head + e, v[j]);
        } else if (is_k) {
          if (p.k_out) store_elem<DT>(p.k_out, token * p.ko_row + h * p.ko_head + e, v[j]);
          if (p.k_cache && sh.at_k[t] >= 0) store_elem<DT>(p.k_cache, (uint64_t)sh.at_k[t] + h * p.kc_head + e, v[j]);
        } else if (sh.at_v[t] >= 0) {
          store_elem<DT>(p.v_cache, (uint64_t)sh.at_v[t] + h * p.vc_head + e, v[j]);
        }
      }
    }
}

}  // namespace kb
