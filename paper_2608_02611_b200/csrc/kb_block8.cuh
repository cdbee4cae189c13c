// What the model operators share: a warp's view of a row in groups of 256 elements, and the
// quantisation of blocks of 128 to 8-bit floating point.
//
// A warp handles a row in groups of 256 consecutive elements, 8 per lane, i.e. two quantisation
// blocks.  Rows that start on 16-byte boundaries and are a multiple of 8 long (VEC) give lane l
// the elements 8l..8l+7, so that it loads and stores 16-byte vectors and 16 lanes hold a block.
// All other rows give it the elements l, 32+l, ..., 224+l: every load and store of the warp is
// still one contiguous piece, and elements j < 4 and j >= 4 of all lanes hold a block each.
#pragma once

#include <cuda_bf16.h>

#include "kb_common.cuh"

namespace kb {

constexpr uint32_t kGroup = 256;

template <bool VEC>
__host__ __device__ __forceinline__ uint32_t group_col(uint32_t g, int lane, int j) {
  return g * kGroup + (VEC ? lane * 8 + j : j * 32 + lane);
}

// ---- storage types ------------------------------------------------------------------------
template <int DT>
__device__ __forceinline__ float load_elem(const void* p, uint64_t i) {
  return Elem<DT>::load(p, i);
}
template <int DT>
__device__ __forceinline__ void store_elem(void* p, uint64_t i, float v) {
  if constexpr (DT == KB_F32)
    reinterpret_cast<float*>(p)[i] = v;
  else if constexpr (DT == KB_BF16)
    reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else
    reinterpret_cast<__half*>(p)[i] = __float2half_rn(v);
}
template <int DT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {   // 16-bit types
  if constexpr (DT == KB_BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}
// 8 consecutive elements from / to a 16-byte aligned place
template <int DT>
__device__ __forceinline__ void load8(const void* p, uint64_t i, float (&v)[8]) {
  if constexpr (DT == KB_F32) {
    const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(p) + i);
    const uint4 a = q[0], b = q[1];
    Elem<DT>::decode(a, v);
    Elem<DT>::decode(b, v + 4);
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned short*>(p) + i);
    Elem<DT>::decode(a, v);
  }
}
template <int DT>
__device__ __forceinline__ void store8(void* p, uint64_t i, const float (&v)[8]) {
  if constexpr (DT == KB_F32) {
    float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + i);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(reinterpret_cast<unsigned short*>(p) + i) =
        make_uint4(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]), pack2<DT>(v[4], v[5]), pack2<DT>(v[6], v[7]));
  }
}

// The n (1..8) elements from element i on, of a matrix that holds `span` elements from `base` (its gaps
// between rows included), as raw words with zeros after the n; E bytes per element, any alignment.
// Where a granule reaches past the matrix's ends the elements are read one by one.
template <int E>
__device__ __forceinline__ void load_shifted(const void* base, uint64_t span, uint64_t i, int n, uint32_t (&w)[2 * E]) {
  constexpr int kGranules = E / 2 + 1;         // 16-byte granules that 8 elements can lie in
  const uintptr_t first = reinterpret_cast<uintptr_t>(base), at = first + i * E, from = at & ~(uintptr_t)15;
  if (from >= first && from + 16 * kGranules <= first + span * E) {
    uint32_t u[4 * kGranules];
#pragma unroll
    for (int k = 0; k < kGranules; ++k) {
      const uint4 t = *reinterpret_cast<const uint4*>(from + 16 * k);
      u[4 * k] = t.x;
      u[4 * k + 1] = t.y;
      u[4 * k + 2] = t.z;
      u[4 * k + 3] = t.w;
    }
    const uint32_t off = (uint32_t)(at & 15);
    constexpr int kWords = 2 * E + (E == 2 ? 1 : 0);   // words that still matter after the word shifts
#pragma unroll
    for (int k = 0; k < kWords + 1; ++k) u[k] = (off & 8) && k + 2 < 4 * kGranules ? u[k + 2] : u[k];
#pragma unroll
    for (int k = 0; k < kWords; ++k) u[k] = (off & 4) ? u[k + 1] : u[k];
#pragma unroll
    for (int k = 0; k < 2 * E; ++k) {
      if constexpr (E == 2)
        w[k] = (off & 2) ? __funnelshift_r(u[k], u[k + 1], 16) : u[k];
      else
        w[k] = u[k];
    }
    if (n < 8) {
#pragma unroll
      for (int k = 0; k < 2 * E; ++k) {
        if constexpr (E == 2)
          w[k] = 2 * k + 1 < n ? w[k] : 2 * k < n ? w[k] & 0xFFFFu : 0u;
        else
          w[k] = k < n ? w[k] : 0u;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2 * E; ++k) w[k] = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) {
        if constexpr (E == 2)
          w[j >> 1] |= (uint32_t) static_cast<const unsigned short*>(base)[i + j] << (16 * (j & 1));
        else
          w[j] = static_cast<const uint32_t*>(base)[i + j];
      }
  }
}

// A lane's 8 elements of group g of a row that starts at element `row0`; elements past the row's
// end read as `fill`.
template <int DT, bool VEC>
__device__ __forceinline__ void load_group(const void* base, uint64_t row0, uint32_t g, int lane, uint32_t cols,
                                           float (&v)[8], float fill = 0.0f) {
  if constexpr (VEC) {
    const uint32_t c = group_col<true>(g, lane, 0);
    if (c < cols) {
      load8<DT>(base, row0 + c, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = fill;
    }
  } else if ((g + 1) * kGroup <= cols) {   // a whole group: no test per element
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = load_elem<DT>(base, row0 + group_col<false>(g, lane, j));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t c = group_col<false>(g, lane, j);
      v[j] = c < cols ? load_elem<DT>(base, row0 + c) : fill;
    }
  }
}
// Sets a lane's elements past the row's end.
template <bool VEC>
__device__ __forceinline__ void fill_tail(uint32_t g, int lane, uint32_t cols, float value, float (&v)[8]) {
  if ((g + 1) * kGroup <= cols) return;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (group_col<VEC>(g, lane, j) >= cols) v[j] = value;
}
template <int DT, bool VEC>
__device__ __forceinline__ void store_group(void* base, uint64_t row0, uint32_t g, int lane, uint32_t cols,
                                            const float (&v)[8]) {
  if constexpr (VEC) {
    const uint32_t c = group_col<true>(g, lane, 0);
    if (c < cols) store8<DT>(base, row0 + c, v);
  } else if ((g + 1) * kGroup <= cols) {
#pragma unroll
    for (int j = 0; j < 8; ++j) store_elem<DT>(base, row0 + group_col<false>(g, lane, j), v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t c = group_col<false>(g, lane, j);
      if (c < cols) store_elem<DT>(base, row0 + c, v[j]);
    }
  }
}
// Parameters [cols] of the row's own type or of binary32 (f32), or none (value `none`).
template <int DT, bool VEC>
__device__ __forceinline__ void load_params(const void* base, bool f32, uint32_t g, int lane, uint32_t cols,
                                            float none, float (&v)[8]) {
  if (base == nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = none;
  } else if (DT == KB_F32 || f32) {
    load_group<KB_F32, VEC>(base, 0, g, lane, cols, v);
  } else {
    load_group<DT, VEC>(base, 0, g, lane, cols, v);
  }
}

// ---- two binary32 values in one register pair: one instruction for two operations ------------------
// (The norms are bound by the number of instructions beside memory.)
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(Pair v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ float fold(Pair v) {
  float lo, hi;
  unpair(v, lo, hi);
  return lo + hi;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// ---- 8-bit quantisation ---------------------------------------------------------------------
// A block with largest magnitude a >= 2^-100 has the scale S = a / F, and its codes are the quotients
// v F / a rounded.  Inputs of 8 or 11 significant bits make quotients that lie exactly between two
// codes, and a product with a rounded F / a would send some of them the wrong way; so the quotient is
// rounded correctly, as (v L * 0.875) / (a 2^-kShift L) with F = 1.75 * 2^(kShift - 1).  The remainder of that
// division is a multiple of 2^-79 a L (quotients from 2^-17 on, half the smallest e5m2 step, and 23 bits
// below each leading bit) and has to stay above binary32's smallest step, 2^-149.  So L = 2^40 for a
// under kSmallMax, and 1 elsewhere.  Such blocks and those with an Inf are rare: one test per block finds
// both, and only there the values are treated first.
template <bool E5M2>
struct Fp8 {
  static constexpr float kTop = E5M2 ? 57344.0f : 448.0f;
  static constexpr float kUnscale = E5M2 ? 0x1p-16f : 0x1p-9f;   // 2^-kShift
};
struct BlockScale {
  float scale, den, inv;   // S, a 2^-kShift L, 1 / den
};
constexpr float kLeastMax = 0x1p-100f, kSmallMax = 0x1p-60f;
__device__ __forceinline__ float block_lift(float amax) { return amax < kSmallMax ? 0x1p40f : 1.0f; }   // L
__device__ __forceinline__ bool block_is_rare(float amax) { return !(amax >= kSmallMax && amax <= 0x1.fffffep127f); }
template <bool E5M2>
__device__ __forceinline__ BlockScale block_scale(float amax) {
  const float a = fmaxf(amax, kLeastMax), den = a * (Fp8<E5M2>::kUnscale * block_lift(a));
  return {__fdiv_rn(a, Fp8<E5M2>::kTop), den, __fdiv_rn(1.0f, den)};
}
// Two values to two codes (lo in the low byte), saturating; NaN becomes NaN.
template <bool E5M2>
__device__ __forceinline__ uint32_t quant2(float lo, float hi) {
  unsigned short r;
  if (E5M2)
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// (v * 0.875) / den, v and den lifted where the block's maximum is small, rounded correctly from the rounded
// reciprocal (Markstein 1990: a quotient estimate within an ulp, corrected once by its exact remainder)
__device__ __forceinline__ void quotients(float& v0, float& v1, const Pair den, const Pair inv) {
  const Pair num = mul2(pair(v0, v1), pair(0.875f, 0.875f));
  const Pair t = mul2(num, inv);
  const Pair rest = fma2(t, den, num);   // den comes negated
  unpair(fma2(rest, inv, t), v0, v1);
}
template <bool E5M2>
__device__ __forceinline__ uint2 quant8(const float (&v)[8], float den, float inv) {
  const Pair d = pair(-den, -den), r = pair(inv, inv);
  float t[8];
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    t[j] = v[j];
    t[j + 1] = v[j + 1];
    quotients(t[j], t[j + 1], d, r);
  }
  uint2 q;
  q.x = quant2<E5M2>(t[0], t[1]) | quant2<E5M2>(t[2], t[3]) << 16;
  q.y = quant2<E5M2>(t[4], t[5]) | quant2<E5M2>(t[6], t[7]) << 16;
  return q;
}
// Largest magnitude, NaN left out (the maximum of a number and NaN is the number).
template <int J0, int J1>
__device__ __forceinline__ float max_abs(const float (&v)[8]) {
  float m = 0.0f;
#pragma unroll
  for (int j = J0; j < J1; ++j) m = fmaxf(m, fabsf(v[j]));
  return m;
}
// For a block whose maximum may be infinite: Inf becomes NaN; returns the largest finite magnitude.
template <int J0, int J1>
__device__ __forceinline__ float settle_inf(float (&v)[8]) {
  float m = 0.0f;
#pragma unroll
  for (int j = J0; j < J1; ++j) {
    if (isinf(v[j])) v[j] = __uint_as_float(0x7FFFFFFFu);
    m = fmaxf(m, fabsf(v[j]));
  }
  return m;
}
template <int J0, int J1>
__device__ __forceinline__ void lift_values(float (&v)[8], float lift) {
#pragma unroll
  for (int j = J0; j < J1; ++j) v[j] *= lift;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}

// The quotients of a block whose maximum all lanes of `mask` hold: one lane divides for the scale and
// the others for the reciprocal, so the two cost one division.
template <bool E5M2>
__device__ __forceinline__ BlockScale shared_block_scale(float amax, unsigned int mask, int first, int lane) {
  const float a = fmaxf(amax, kLeastMax), den = a * (Fp8<E5M2>::kUnscale * block_lift(a));
  const bool is_first = lane == first;
  const float r = __fdiv_rn(is_first ? a : 1.0f, is_first ? Fp8<E5M2>::kTop : den);
  return {r, den, __shfl_sync(mask, r, first + 1)};   // .scale holds in lane `first` only
}

// Quantise a lane's part of the groups g0, g0 + gstep, ... (NCH of them) of row `row`: codes to q,
// the blocks' scales to scale[block][row].  All 32 lanes take part; elements past the row's end must
// be 0.  `whole`: no lane's 8 elements end past the row's end.  The steps of all groups stand side by
// side, so that their shuffles and divisions overlap.
template <bool E5M2, bool VEC, int NCH>
__device__ __forceinline__ void quant_groups(float (&v)[NCH][8], uint32_t g0, uint32_t gstep, int lane, uint32_t cols,
                                             uint64_t row, uint64_t rows, unsigned char* q, uint64_t ldq,
                                             float* scale, bool whole = true) {
  if constexpr (VEC) {
    const unsigned int half = 0xFFFFu << (lane & 16);
    float m[NCH];
    bool any = false;
#pragma unroll
    for (int i = 0; i < NCH; ++i) m[i] = max_abs<0, 8>(v[i]);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < NCH; ++i) m[i] = fmaxf(m[i], __shfl_xor_sync(half, m[i], o));
#pragma unroll
    for (int i = 0; i < NCH; ++i) any |= block_is_rare(m[i]);
    if (any) {   // the same for the 16 lanes of a block
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        m[i] = settle_inf<0, 8>(v[i]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m[i] = fmaxf(m[i], __shfl_xor_sync(half, m[i], o));
        lift_values<0, 8>(v[i], block_lift(m[i]));
      }
    }
    BlockScale s[NCH];
#pragma unroll
    for (int i = 0; i < NCH; ++i) s[i] = shared_block_scale<E5M2>(m[i], half, lane & 16, lane);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const uint32_t c = group_col<true>(g0 + i * gstep, lane, 0);
      if (c < cols) {
        const uint2 r = quant8<E5M2>(v[i], s[i].den, s[i].inv);
        unsigned char* dst = q + row * ldq + c;
        if (whole || c + 8 <= cols) {
          *reinterpret_cast<uint2*>(dst) = r;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (c + j < cols) dst[j] = (unsigned char)((j < 4 ? r.x : r.y) >> (8 * (j & 3)));
        }
        if ((lane & 15) == 0) scale[(uint64_t)(c >> 7) * rows + row] = s[i].scale;
      }
    }
  } else {
    float m[NCH][2];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      m[i][0] = max_abs<0, 4>(v[i]);
      m[i][1] = max_abs<4, 8>(v[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < 2 * NCH; ++i)
        m[i >> 1][i & 1] = fmaxf(m[i >> 1][i & 1], __shfl_xor_sync(0xFFFFFFFFu, m[i >> 1][i & 1], o));
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const uint32_t g = g0 + i * gstep;
      if (block_is_rare(m[i][0])) {   // the same for the warp
        m[i][0] = warp_max(settle_inf<0, 4>(v[i]));
        lift_values<0, 4>(v[i], block_lift(m[i][0]));
      }
      if (block_is_rare(m[i][1])) {
        m[i][1] = warp_max(settle_inf<4, 8>(v[i]));
        lift_values<4, 8>(v[i], block_lift(m[i][1]));
      }
      // lanes 0..15 work out the first block's quotients, lanes 16..31 the second's
      const unsigned int half = 0xFFFFu << (lane & 16);
      const BlockScale s = shared_block_scale<E5M2>(lane < 16 ? m[i][0] : m[i][1], half, lane & 16, lane);
      const float inv0 = __shfl_sync(0xFFFFFFFFu, s.inv, 0), inv1 = __shfl_sync(0xFFFFFFFFu, s.inv, 16);
      const float den0 = __shfl_sync(0xFFFFFFFFu, s.den, 0), den1 = __shfl_sync(0xFFFFFFFFu, s.den, 16);
      const uint2 r0 = quant8<E5M2>(v[i], den0, inv0), r1 = quant8<E5M2>(v[i], den1, inv1);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = group_col<false>(g, lane, j);
        const uint32_t w = j < 4 ? r0.x : r1.y;
        if (c < cols) q[row * ldq + c] = (unsigned char)(w >> (8 * (j & 3)));
      }
      const uint32_t kb = g * 2 + (lane >> 4);
      if ((lane & 15) == 0 && kb * 128u < cols) scale[(uint64_t)kb * rows + row] = s.scale;
    }
  }
}

}  // namespace kb
