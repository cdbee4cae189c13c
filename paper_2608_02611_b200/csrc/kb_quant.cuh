// Quantisation to 8-bit floating point in blocks of 128 (contract in include/kb_ops.h).
//
// Bound: memory; an element is read once and its code written once.  Blocks along a row need no
// other row and are handled by half a warp each.  Tiles of 128 x 128 and everything that is
// written transposed go through a CTA that holds the whole tile in registers: 16 x 16 threads
// with 8 x 8 elements each, so that a thread's column of 8 codes is one 8-byte piece of a
// transposed row.
#pragma once

#include "kb_block8.cuh"

namespace kb {

struct QuantParams {
  const void* x;
  unsigned char* q;
  float* scale;
  uint64_t rows, cols, ldx, ldq;    // of x
  uint64_t span;                    // elements of x from its first to its last, gaps included
  bool q_vec;                       // rows of q start on 8-byte boundaries
  uint32_t groups;                  // groups of 256 columns per row
  uint32_t rtiles, ctiles;          // tiles of 128 along the rows and columns of x
};

template <int DT>
struct Held8 {   // 8 consecutive elements of one row
  static constexpr int kWords = 2 * Elem<DT>::kBytes;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void* p, uint64_t i) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(p) + i * Elem<DT>::kBytes);
    *reinterpret_cast<uint4*>(w) = q[0];
    if constexpr (DT == KB_F32) *reinterpret_cast<uint4*>(w + 4) = q[1];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < kWords; ++k) w[k] = 0u;
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (DT == KB_F32)
      return __uint_as_float(w[j]);
    else if constexpr (DT == KB_BF16)
      return __uint_as_float((j & 1) ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
    else
      return __half2float(__ushort_as_half((unsigned short)(w[j >> 1] >> (16 * (j & 1)))));
  }
  __device__ __forceinline__ void all(float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = get(j);
  }
};

// 1 x 128 blocks along the rows of x: one warp per row and piece of NG groups.
constexpr int kQuantRowGroups = 4;
// VEC: rows of x and q are aligned and a multiple of 8 long.  Otherwise, with aligned rows of q
// (SHIFT), a lane still takes 8 consecutive elements and shifts the granules they lie in into place
// (8191 x 8191 bf16: 73 us, element by element 90; 2000 x 5003: 11.7 and 15.0); rows of q at any address go
// element by element.  Four CTAs per SM: with three, and registers to spare, 8191 x 8191 takes 89 us.
template <int DT, bool VEC, bool SHIFT, bool E5M2>
__global__ void __launch_bounds__(256, 4) quant_rows_kernel(const QuantParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t row = (uint64_t)blockIdx.x * 8 + warp;
  if (row >= p.rows) return;
  for (uint32_t g0 = blockIdx.y * kQuantRowGroups; g0 < p.groups; g0 += gridDim.y * kQuantRowGroups) {
    float v[kQuantRowGroups][8];
#pragma unroll
    for (int i = 0; i < kQuantRowGroups; ++i) {
      if constexpr (SHIFT) {
        const uint64_t c = (uint64_t)(g0 + i) * kGroup + lane * 8;
        Held8<DT> h;
        if (c < p.cols)
          load_shifted<Elem<DT>::kBytes>(p.x, p.span, row * p.ldx + c, (int)min((uint64_t)8, p.cols - c), h.w);
        else
          h.zero();
        h.all(v[i]);
      } else {
        load_group<DT, VEC>(p.x, row * p.ldx, g0 + i, lane, (uint32_t)p.cols, v[i]);
      }
    }
    quant_groups<E5M2, VEC || SHIFT, kQuantRowGroups>(v, g0, 1, lane, (uint32_t)p.cols, row, p.rows, p.q, p.ldq,
                                                      p.scale, !SHIFT);
  }
}

// One 128 x 128 tile per CTA of 256 threads.  TILES: one scale for the tile, else one per column
// of x (only needed transposed: the block then runs along the rows of x).  A thread keeps its 8 x 8
// elements in their storage type (32 registers for 16-bit types), so that three CTAs fit on an SM
// and 96 KB are on their way while one of them reduces.
// The transposed tile in shared memory: rows of 128 codes; the 8-byte piece k of row r stands at
// place k ^ (r / 8), so that neither the writes (16 rows apart by 8, one piece each) nor the reads
// (one row at a time) meet in a bank.
__host__ __device__ __forceinline__ int transposed_at(int r, int k) { return r * 128 + ((k ^ (r >> 3)) & 15) * 8; }
__device__ __forceinline__ float inf_to_nan(float v) { return isinf(v) ? __uint_as_float(0x7FFFFFFFu) : v; }

template <int DT, bool VEC, bool E5M2, bool TILES, bool TRANSPOSE>
__global__ void __launch_bounds__(256, DT == KB_F32 ? 2 : 3) quant_tile_kernel(const QuantParams p) {
  __shared__ __align__(16) float smax[TILES ? 8 : 8 * 128];
  __shared__ __align__(16) float sinv[TILES ? 4 : 128], sden[TILES ? 4 : 128];
  __shared__ float slift[TILES ? 1 : 128];
  __shared__ int some_small;   // a column's maximum is (only written where TILES does not hold)
  __shared__ __align__(16) unsigned char st[TRANSPOSE ? 128 * 128 : 16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const uint32_t rt = blockIdx.x / p.ctiles, ct = blockIdx.x % p.ctiles;
  const uint64_t row0 = (uint64_t)rt * 128 + ry * 8, col0 = (uint64_t)ct * 128 + cx * 8;
  const int nrow = row0 < p.rows ? (int)min((uint64_t)8, p.rows - row0) : 0;
  const int ncol = col0 < p.cols ? (int)min((uint64_t)8, p.cols - col0) : 0;
  Held8<DT> h[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= nrow || ncol == 0)
      h[i].zero();
    else if constexpr (VEC)
      h[i].load(p.x, (row0 + i) * p.ldx + col0);
    else
      load_shifted<Elem<DT>::kBytes>(p.x, p.span, (row0 + i) * p.ldx + col0, ncol, h[i].w);
  }
  bool rare = false;       // the tile holds an Inf, or a block of it has a small maximum
  __align__(16) float den[TILES ? 4 : 8], inv[TILES ? 4 : 8];   // per column of the thread, or of the tile
  if constexpr (TILES) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(h[i].get(j)));
    m = warp_max(m);
    if (lane == 0) smax[warp] = m;
    __syncthreads();
    m = warp_max(smax[lane & 7]);
    rare = block_is_rare(m);
    if (rare) {   // the same for the whole CTA
      float f = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) f = fmaxf(f, fabsf(inf_to_nan(h[i].get(j))));
      f = warp_max(f);
      __syncthreads();
      if (lane == 0) smax[warp] = f;
      __syncthreads();
      m = warp_max(smax[lane & 7]);
      slift[0] = block_lift(m);   // by every thread: only needed, and read back, where `rare` holds
    }
    const BlockScale s = block_scale<E5M2>(m);
    den[0] = s.den;
    inv[0] = s.inv;
    if (threadIdx.x == 0) {
      if (TRANSPOSE)
        p.scale[(uint64_t)rt * p.ctiles + ct] = s.scale;
      else
        p.scale[(uint64_t)ct * p.rtiles + rt] = s.scale;
    }
  } else {
    auto columns = [&](bool settle) {   // each column's maximum over the warp's 16 rows, to smax[warp][column]
      float m[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = h[i].get(j);
          m[j] = fmaxf(m[j], fabsf(settle ? inf_to_nan(v) : v));
        }
        m[j] = fmaxf(m[j], __shfl_xor_sync(0xFFFFFFFFu, m[j], 16));
      }
      if (lane < 16) {
        float4* dst = reinterpret_cast<float4*>(smax + warp * 128 + cx * 8);
        dst[0] = make_float4(m[0], m[1], m[2], m[3]);
        dst[1] = make_float4(m[4], m[5], m[6], m[7]);
      }
    };
    // one thread per column: the tile's maximum, the scale to memory, the divisor and its
    // reciprocal back to shared memory
    auto column = [&]() {
      float t = 0.0f;
      if (threadIdx.x < 128) {
#pragma unroll
        for (int w = 0; w < 8; ++w) t = fmaxf(t, smax[w * 128 + threadIdx.x]);
        const BlockScale s = block_scale<E5M2>(t);
        sinv[threadIdx.x] = s.inv;
        sden[threadIdx.x] = s.den;
        slift[threadIdx.x] = block_lift(t);
        if (t < kSmallMax) some_small = 1;
        const uint64_t c = (uint64_t)ct * 128 + threadIdx.x;
        if (c < p.cols) p.scale[(uint64_t)rt * p.cols + c] = s.scale;
      }
      return isinf(t);
    };
    if (threadIdx.x == 0) some_small = 0;
    columns(false);
    __syncthreads();
    rare = __syncthreads_or(column());
    if (rare) {
      columns(true);
      __syncthreads();
      column();
      __syncthreads();
    }
    rare |= some_small != 0;
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      *reinterpret_cast<float4*>(inv + j) = *reinterpret_cast<const float4*>(sinv + cx * 8 + j);
      *reinterpret_cast<float4*>(den + j) = *reinterpret_cast<const float4*>(sden + cx * 8 + j);
    }
  }
  if constexpr (!TRANSPOSE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= nrow) break;
      float v[8];
      h[i].all(v);
      if (rare) {
        const float lift = slift[0];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = inf_to_nan(v[j]) * lift;
      }
      const uint2 r = quant8<E5M2>(v, den[0], inv[0]);
      unsigned char* dst = p.q + (row0 + i) * p.ldq + col0;
      if (ncol == 8 && (VEC || p.q_vec)) {
        *reinterpret_cast<uint2*>(dst) = r;
      } else {
        for (int j = 0; j < ncol; ++j) dst[j] = (unsigned char)((j < 4 ? r.x : r.y) >> (8 * (j & 3)));
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = h[i].get(j);
      if (rare) {
        const float lift = slift[TILES ? 0 : cx * 8 + j];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = inf_to_nan(c[i]) * lift;
      }
      const uint2 r = quant8<E5M2>(c, den[TILES ? 0 : j], inv[TILES ? 0 : j]);
      *reinterpret_cast<uint2*>(st + transposed_at(cx * 8 + j, ry)) = r;
    }
    __syncthreads();
    // a warp writes one transposed row (a column of x) at a time
    const uint64_t tcol0 = (uint64_t)rt * 128;   // first column of the transposed tile
    const int left = (int)min((uint64_t)128, p.rows - tcol0);
    for (int c = warp; c < 128; c += 8) {
      const uint64_t trow = (uint64_t)ct * 128 + c;
      if (trow >= p.cols) break;
      unsigned char* dst = p.q + trow * p.ldq + tcol0;
      if ((p.ldq & 3) == 0 && left == 128 && (reinterpret_cast<uintptr_t>(p.q) & 3) == 0) {
        reinterpret_cast<uint32_t*>(dst)[lane] = *reinterpret_cast<const uint32_t*>(st + transposed_at(c, lane >> 1) + (lane & 1) * 4);
      } else {
        for (int b = lane; b < left; b += 32) dst[b] = st[transposed_at(c, b >> 3) + (b & 7)];
      }
    }
  }
}

}  // namespace kb
