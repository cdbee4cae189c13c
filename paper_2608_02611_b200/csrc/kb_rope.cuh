// Norms of queries and keys for each head with the position rotation, in one pass that also stores the
// turned keys and the values in a paged cache (contract in include/kb_attention.h).
//
// Bound by bytes: every element is read once and written once or twice.  A head's row of dim elements
// belongs to L lanes of a warp (8 elements each), so that its sum of squares takes log2(L) shuffles and
// nothing leaves the registers.  The angles are the same for all heads of a token: a CTA works on
// whole tokens and first puts their cosines and sines into shared memory, one per thread, where
// each lane picks up the 8 pairs that it needs for all its rows of the token.
//
// An angle is position * inv_freq radians, and only its fraction of a turn matters.  inv_freq / (2 pi) is
// taken to a 64-bit fixed-point fraction; its product with the position, modulo 2^64, is exact, so
// the error is the fraction's own (2^-53 of it) times the position, whatever the position.  The quarter of the turn
// goes off as an integer and at most an eighth of a turn on either side is left for sincospi.
#pragma once

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
  uint32_t hq, hkv, rows;              // rows of a token: q's and k's heads, and v's with a cache
  uint32_t dim, half;                  // half: pairs that are turned
  uint32_t first_row;                  // hq where no queries are wanted: those rows are passed over
  unsigned int* status;
};

constexpr uint32_t kRopeThreads = 256;
constexpr uint32_t kRopeTokens = 4;       // tokens per CTA, at most
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

// L lanes hold a row.  VEC: 8 consecutive elements per lane, in 16-byte pieces, and pairs that lie 8 k
// apart (or side by side); otherwise the elements c, L + c, ... and pairs through shared memory.
template <int DT, int L, bool VEC>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const RopeParams p, const uint32_t per_cta) {
  constexpr int kSlots = kRopeThreads / L;   // rows at a time
  __shared__ __align__(16) float cos_of[kRopeTokens][kRopeMaxHalf], sin_of[kRopeTokens][kRopeMaxHalf];
  __shared__ long long at_k[kRopeTokens], at_v[kRopeTokens];
  __shared__ float swap[VEC ? 1 : kRopeThreads * 8];
  const uint64_t t0 = (uint64_t)blockIdx.x * per_cta;
  const uint32_t ntok = (uint32_t)min((uint64_t)per_cta, p.tokens - t0);
  const int c = threadIdx.x % L, slot = threadIdx.x / L;
  const int row_lane = (threadIdx.x & 31) & ~(L - 1);   // lane of the row's first element

  for (uint32_t i = threadIdx.x; i < ntok * p.half; i += kRopeThreads) {
    const uint32_t t = i / p.half, f = i % p.half;
    const float2 cs = rope_cos_sin(p.positions[t0 + t], p.inv_freq[f]);
    cos_of[t][f] = cs.x;
    sin_of[t][f] = cs.y;
  }
  if (p.k_cache && threadIdx.x < ntok) {
    const long long s = p.slots[t0 + threadIdx.x];
    const bool in = s >= 0 && (uint64_t)s < p.slots_end;
    if (s >= 0 && !in) set_status(p.status, (unsigned int)KB_ERR_INVALID_ARG);
    const uint64_t page = in ? (uint64_t)s / p.page_size : 0, off = in ? (uint64_t)s % p.page_size : 0;
    at_k[threadIdx.x] = in ? (long long)(page * p.kc_page + off * p.kc_row) : -1;
    at_v[threadIdx.x] = in ? (long long)(page * p.vc_page + off * p.vc_row) : -1;
  }
  // the lane's weights, as binary32
  float wq[8], wk[8];
  auto elem = [&](int j) -> uint32_t { return VEC ? c * 8 + j : j * L + c; };
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t e = elem(j);
    const bool in = e < p.dim && p.norm;
    wq[j] = !in || !p.q_weight ? 1.0f : p.param_f32 ? static_cast<const float*>(p.q_weight)[e] : load_elem<DT>(p.q_weight, e);
    wk[j] = !in || !p.k_weight ? 1.0f : p.param_f32 ? static_cast<const float*>(p.k_weight)[e] : load_elem<DT>(p.k_weight, e);
  }
  __syncthreads();

  for (uint32_t t = 0; t < ntok; ++t) {
    const uint64_t token = t0 + t;
    float cs[8], sn[8];
    int partner = c;             // VEC, halves: the lane of the row with the other element of the pairs
    if constexpr (VEC) {
      const uint32_t chunks = p.half / 8;
      const bool low = (uint32_t)c < chunks, turned = (uint32_t)c < 2 * chunks;
      if (!p.interleaved) {
        partner = turned ? (low ? c + (int)chunks : c - (int)chunks) : c;
        const uint32_t f = (low ? c : c - chunks) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          cs[j] = turned ? cos_of[t][f + j] : 1.0f;
          sn[j] = turned ? (low ? -sin_of[t][f + j] : sin_of[t][f + j]) : 0.0f;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t f = c * 4 + j;
          cs[j] = f < p.half ? cos_of[t][f] : 1.0f;
          sn[j] = f < p.half ? sin_of[t][f] : 0.0f;
        }
      }
    }
    // the trip count is the same for all lanes of a warp: rows take shuffles
    for (uint32_t r0 = p.first_row; r0 < p.rows; r0 += kSlots) {
      const uint32_t r = r0 + slot;
      const bool is_q = r < p.hq, is_k = !is_q && r < p.hq + p.hkv, in = r < p.rows;
      const uint32_t h = is_q ? r : is_k ? r - p.hq : r - p.hq - p.hkv;
      const void* src = is_q ? p.q : is_k ? p.k : p.v;
      const uint64_t at = is_q ? token * p.q_row + h * p.q_head : is_k ? token * p.k_row + h * p.k_head : token * p.v_row + h * p.v_head;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.0f;
      if constexpr (VEC) {
        if (in && c * 8 < (int)p.dim) load8<DT>(src, at + c * 8, v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (in && elem(j) < p.dim) v[j] = load_elem<DT>(src, at + elem(j));
      }
      if (p.norm) {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(v[j], v[j], sum);
#pragma unroll
        for (int o = L / 2; o > 0; o /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const float by = is_q || is_k ? rsqrtf(sum / (float)p.dim + p.eps) : 1.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= by * (is_q ? wq[j] : is_k ? wk[j] : 1.0f);
      }
      if constexpr (VEC) {
        if (!p.interleaved) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float other = __shfl_sync(0xFFFFFFFFu, v[j], row_lane + partner);
            if (is_q || is_k) v[j] = partner == c ? v[j] : fmaf(v[j], cs[j], other * sn[j]);
          }
        } else if (is_q || is_k) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (c * 4 + j >= (int)p.half) continue;
            const float a = v[2 * j], b = v[2 * j + 1];
            v[2 * j] = a * cs[j] - b * sn[j];
            v[2 * j + 1] = fmaf(b, cs[j], a * sn[j]);
          }
        }
      } else {
        float* row = swap + slot * (L * 8);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) row[elem(j)] = v[j];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t e = elem(j);
          if (e >= 2 * p.half || !(is_q || is_k)) continue;
          const bool first = p.interleaved ? (e & 1u) == 0 : e < p.half;
          const uint32_t f = p.interleaved ? e / 2 : first ? e : e - p.half;
          const float other = row[p.interleaved ? e ^ 1u : first ? e + p.half : e - p.half];
          const float s = sin_of[t][f];
          v[j] = fmaf(v[j], cos_of[t][f], first ? -other * s : other * s);
        }
      }
      auto put = [&](void* dst, uint64_t to) {
        if constexpr (VEC) {
          if (c * 8 < (int)p.dim) store8<DT>(dst, to + c * 8, v);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (elem(j) < p.dim) store_elem<DT>(dst, to + elem(j), v[j]);
        }
      };
      if (!in) continue;
      if (is_q) {
        put(p.q_out, token * p.qo_row + h * p.qo_head);
      } else if (is_k) {
        if (p.k_out) put(p.k_out, token * p.ko_row + h * p.ko_head);
        if (p.k_cache && at_k[t] >= 0) put(p.k_cache, (uint64_t)at_k[t] + h * p.kc_head);
      } else if (at_v[t] >= 0) {
        put(p.v_cache, (uint64_t)at_v[t] + h * p.vc_head);
      }
    }
  }
}

}  // namespace kb
