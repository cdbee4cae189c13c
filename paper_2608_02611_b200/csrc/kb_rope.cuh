// Norms of queries and keys for each head with the position rotation, in one pass that also stores the
// turned keys and the values in a paged cache (contract in include/kb_attention.h).
//
// Bound by bytes: every element is read once and written once or twice.  A head's row of dim elements
// belongs to L lanes of a warp (8 elements each), so that its sum of squares takes log2(L) shuffles and
// nothing leaves the registers.  The angles are the same for all heads of a token: a CTA works on
// whole tokens and first puts their cosines and sines into shared memory, one per thread.
//
// An angle is position * inv_freq radians, and only its fraction of a turn matters.  inv_freq / (2 pi) is rounded to
// binary64, whose fraction of a turn is taken in units of 2^-64; its product with the position, modulo 2^64, is exact.  What the
// rounding left, at most 2^-53 of the quotient, is taken in binary32, and so is its product with the position.  So
// the angle is off by 2^-64 of a turn (and 2^-75 of inv_freq) times the position beside what binary32 rounds: by nothing up to 2^36.
// (The rounding left in binary64, and the digits behind the 64th, would do for any position, but cost 16384 tokens
// 2.3 us of 93.7 and 1001 tokens 0.6 of 8.3, for registers and their spills.)  The quarter of the turn
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

// freq / (2 pi), rounded: the product by itself, not part of a fused operation
__host__ __device__ __forceinline__ double rope_quotient(double freq) {
#ifdef __CUDA_ARCH__
  return __dmul_rn(freq, 0.15915494309189535);
#else
  return freq * 0.15915494309189535;
#endif
}
// The part of a turn per position, in units of 2^-64
__host__ __device__ __forceinline__ uint64_t rope_turn(double freq) {
  const double t = rope_quotient(freq);
  const double part = t - floor(t);
  return part < 1.0 ? (uint64_t)(part * 18446744073709551616.0) : 0ull;
}
// What the quotient's rounding left, in turns; 1 / (2 pi) in two parts
__host__ __device__ __forceinline__ float rope_rest(double freq) {
  return fmaf((float)freq, -9.8393383e-18f, (float)fma(freq, 0.15915494309189535, -rope_quotient(freq)));
}
// cos and sin of the angle position * freq radians
__device__ __forceinline__ float2 rope_cos_sin(long long position, double freq) {
  if (freq < 0.0) position = (long long)(0ull - (uint64_t)position);   // a fraction a little below 1 would be rounded
  freq = fabs(freq);
  const float more = (float)position * rope_rest(freq);
  const uint64_t turn = (uint64_t)position * rope_turn(freq) + (uint64_t)__float2ll_rn((more - rintf(more)) * 18446744073709551616.0f);
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
// of neighbours, 8 c .. + 7.  A warp takes 32 / L heads of one kind through the CTA's tokens, four of whose loads are
// under way before the first is used; what depends on the head (weights, addresses but for a step per token) is
// done once for them.  16384 tokens of 32 + 8 + 8 heads of 128, bf16, stored in a cache: a row at a time 176 us;
// heads in turn, which had to be told apart for every row (240 instructions for 512 bytes), 121 us; so 94 (4.6 TB/s; issue
// slots 70% busy, with 43% of the warps, of 64 registers), in binary32 without a cache 115 (5.8 TB/s; there some 100 bytes of the
// registers spill).
__device__ __forceinline__ void vec_words(uint2 v, uint32_t* w) { w[0] = v.x, w[1] = v.y; }
__device__ __forceinline__ void vec_words(uint4 v, uint32_t* w) { w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w; }
__device__ __forceinline__ void words_vec(const uint32_t* w, uint2& v) { v = make_uint2(w[0], w[1]); }
__device__ __forceinline__ void words_vec(const uint32_t* w, uint4& v) { v = make_uint4(w[0], w[1], w[2], w[3]); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 a, b;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 a, a, b, c;\nmov.b64 {%0, %1}, a;\n}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
template <int DT, int L>
__global__ void __launch_bounds__(kRopeThreads, 4) qk_norm_rope_kernel(const RopeParams p, const uint32_t per_cta) {
  constexpr int kWarps = kRopeThreads / 32, kBytes = DT == KB_F32 ? 4 : 2, kWords = 2 * kBytes, kAhead = 4;
  constexpr uint32_t kHeads = 32 / L;        // heads of a piece
  using Vec = typename std::conditional<DT == KB_F32, uint4, uint2>::type;
  __shared__ __align__(16) RopeShared sh;
  const uint64_t t0 = (uint64_t)blockIdx.x * per_cta;
  const uint32_t ntok = (uint32_t)min((uint64_t)per_cta, p.tokens - t0);
  const uint32_t warp = threadIdx.x >> 5, c = threadIdx.x % L, sub = (threadIdx.x & 31) / L;
  // pieces of a token: queries', keys', values'
  const uint32_t nq = p.q_out ? (p.hq + kHeads - 1) / kHeads : 0, nkv = (p.hkv + kHeads - 1) / kHeads;
  const uint32_t nk = p.k_out || p.k_cache ? nkv : 0, pieces = nq + nk + (p.k_cache ? nkv : 0);
  // the lane's two vectors, and its pairs
  const uint32_t turned = p.interleaved ? p.half * 2 : p.half;       // four times the lanes with pairs, or more
  const bool has = c * 8 < p.dim, turns = (p.interleaved ? 8 * c : 4 * c) < turned;
  const uint32_t ea = p.interleaved ? 8 * c : turns ? 4 * c : 2 * p.half + 8 * (c - p.half / 4);
  const uint32_t eb = p.interleaved || !turns ? ea + 4 : p.half + 4 * c;
  const float per_dim = 1.0f / (float)p.dim;
  bool begun = false;
  after_the_kernel_before();

#pragma unroll 1
  for (uint32_t piece = blockIdx.y * kWarps + warp; piece < pieces || !begun; piece += kWarps * gridDim.y) {
    const bool is_q = piece < nq, is_v = piece >= nq + nk;
    const uint32_t head = (piece - (is_q ? 0 : is_v ? nq + nk : nq)) * kHeads + sub;
    const bool mine = piece < pieces && has && head < (is_q ? p.hq : p.hkv);
    const uint64_t in_row = is_q ? p.q_row : is_v ? p.v_row : p.k_row;
    const unsigned char* from = static_cast<const unsigned char*>(is_q ? p.q : is_v ? p.v : p.k) +
                                (t0 * in_row + head * (is_q ? p.q_head : is_v ? p.v_head : p.k_head)) * kBytes;
    unsigned char* to = static_cast<unsigned char*>(is_q ? p.q_out : is_v ? nullptr : p.k_out);
    const uint64_t out_row = is_q ? p.qo_row : p.ko_row;
    if (to) to += (t0 * out_row + head * (is_q ? p.qo_head : p.ko_head) + ea) * kBytes;
    from += ea * kBytes;
    const uint32_t other = (eb - ea) * kBytes;   // from the lane's one vector to the other
    const uint64_t in_step = in_row * kBytes, out_step = out_row * kBytes;
    unsigned char* cache = static_cast<unsigned char*>(is_q ? nullptr : is_v ? p.v_cache : p.k_cache);
    if (cache) cache += (head * (is_v ? p.vc_head : p.kc_head) + ea) * kBytes;
    const long long* slots = is_v ? sh.at_v : sh.at_k;
    float2 w[4];
    const void* weight = is_q ? p.q_weight : p.k_weight;
#pragma unroll 1
    for (uint32_t first = 0; first < ntok; first += kAhead) {
      uint32_t raw[kAhead][kWords];
#pragma unroll
      for (int u = 0; u < kAhead; ++u, from += in_step) {
        Vec a = {}, b = {};
        if (mine && first + u < ntok) {
          a = *reinterpret_cast<const Vec*>(from);
          b = *reinterpret_cast<const Vec*>(from + other);
        }
        vec_words(a, raw[u]);
        vec_words(b, raw[u] + kWords / 2);
      }
      if (!begun) {   // the CTA's angles, while the first rows are on their way
        begun = true;
        rope_begin(p, sh, t0, ntok);
        __syncthreads();
        if (piece >= pieces) break;
      }
      if (first == 0 && !is_v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t e = j < 2 ? ea + 2 * j : eb + 2 * j - 4;
          w[j] = make_float2(rope_weight<DT>(p, weight, e), rope_weight<DT>(p, weight, e + 1));
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint32_t t = first + u;
        if (t >= ntok) break;
        if (!is_v) {
          float v[8];
          if constexpr (DT == KB_F32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(raw[u][j]);
          } else {
            Elem<DT>::decode(make_uint4(raw[u][0], raw[u][1], raw[u][2], raw[u][3]), v);
          }
          float2 x[4] = {{v[0], v[1]}, {v[2], v[3]}, {v[4], v[5]}, {v[6], v[7]}};
          if (p.norm) {
            float2 sums = mul2(x[0], x[0]);
#pragma unroll
            for (int j = 1; j < 4; ++j) sums = fma2(x[j], x[j], sums);
            float sum = sums.x + sums.y;
#pragma unroll
            for (int o = L / 2; o > 0; o /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            const float by = rsqrtf(fmaf(sum, per_dim, p.eps));
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = mul2(mul2(x[j], make_float2(by, by)), w[j]);
          }
          if (turns) {
            const float4 co = *reinterpret_cast<const float4*>(&sh.cos_of[t][4 * c]), si = *reinterpret_cast<const float4*>(&sh.sin_of[t][4 * c]);
            if (!p.interleaved) {
              const float2 cs[2] = {{co.x, co.y}, {co.z, co.w}}, sn[2] = {{si.x, si.y}, {si.z, si.w}};
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const float2 a = x[j], b = x[j + 2];
                x[j] = fma2(a, cs[j], mul2(b, make_float2(-sn[j].x, -sn[j].y)));
                x[j + 2] = fma2(b, cs[j], mul2(a, sn[j]));
              }
            } else {
              const float cs[4] = {co.x, co.y, co.z, co.w}, sn[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (4 * c + j >= p.half) continue;
                x[j] = make_float2(fmaf(x[j].x, cs[j], -(x[j].y * sn[j])), fmaf(x[j].y, cs[j], x[j].x * sn[j]));
              }
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (DT == KB_F32) {
              raw[u][2 * j] = __float_as_uint(x[j].x);
              raw[u][2 * j + 1] = __float_as_uint(x[j].y);
            } else {
              raw[u][j] = pack2<DT>(x[j].x, x[j].y);
            }
          }
        }
        if (!mine) continue;
        Vec a, b;
        words_vec(raw[u], a);
        words_vec(raw[u] + kWords / 2, b);
        if (to) {
          *reinterpret_cast<Vec*>(to) = a;
          *reinterpret_cast<Vec*>(to + other) = b;
          to += out_step;
        }
        if (cache) {
          const long long slot = slots[t];
          if (slot >= 0) {
            unsigned char* d = cache + slot * kBytes;
            *reinterpret_cast<Vec*>(d) = a;
            *reinterpret_cast<Vec*>(d + other) = b;
          }
        }
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
  after_the_kernel_before();
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
