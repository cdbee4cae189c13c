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
  uint32_t groups;                  // groups of 256 columns per row
  uint32_t rtiles, ctiles;          // tiles of 128 along the rows and columns of x
};

// 1 x 128 blocks along the rows of x: one warp per row and piece of NG groups.
constexpr int kQuantRowGroups = 4;
template <int DT, bool VEC, bool E5M2>
__global__ void __launch_bounds__(256) quant_rows_kernel(const QuantParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t row = (uint64_t)blockIdx.x * 8 + warp;
  if (row >= p.rows) return;
  for (uint32_t g0 = blockIdx.y * kQuantRowGroups; g0 < p.groups; g0 += gridDim.y * kQuantRowGroups) {
    float v[kQuantRowGroups][8];
#pragma unroll
    for (int i = 0; i < kQuantRowGroups; ++i)
      load_group<DT, VEC>(p.x, row * p.ldx, g0 + i, lane, (uint32_t)p.cols, v[i]);
#pragma unroll
    for (int i = 0; i < kQuantRowGroups; ++i)
      if (g0 + i < p.groups)
        quant_group<E5M2, VEC>(v[i], g0 + i, lane, (uint32_t)p.cols, row, p.rows, p.q, p.ldq, p.scale);
  }
}

// One 128 x 128 tile per CTA of 256 threads.  TILES: one scale for the tile, else one per column
// of x (only needed transposed: the block then runs along the rows of x).
constexpr int kTransposePitch = 132;   // bytes; an odd number of words spreads a column's rows over the banks
template <int DT, bool VEC, bool E5M2, bool TILES, bool TRANSPOSE>
__global__ void __launch_bounds__(256) quant_tile_kernel(const QuantParams p) {
  __shared__ unsigned int smax[TILES ? 8 : 8 * 128];
  __shared__ __align__(16) unsigned char st[TRANSPOSE ? 128 * kTransposePitch : 16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const uint32_t rt = blockIdx.x / p.ctiles, ct = blockIdx.x % p.ctiles;
  const uint64_t row0 = (uint64_t)rt * 128 + ry * 8, col0 = (uint64_t)ct * 128 + cx * 8;
  const int nrow = row0 < p.rows ? (int)min((uint64_t)8, p.rows - row0) : 0;
  const int ncol = col0 < p.cols ? (int)min((uint64_t)8, p.cols - col0) : 0;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (VEC) {
      if (i < nrow && ncol == 8) {
        load8<DT>(p.x, (row0 + i) * p.ldx + col0, v[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[i][j] = (i < nrow && j < ncol) ? load_elem<DT>(p.x, (row0 + i) * p.ldx + col0 + j) : 0.0f;
    }
  }
  float inv[8];   // per column of the thread; all equal for TILES
  if constexpr (TILES) {
    unsigned int m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, max_bits<0, 8>(v[i]));
    m = warp_max_u32(m);
    if (lane == 0) smax[warp] = m;
    __syncthreads();
    m = warp_max_u32(smax[lane & 7]);
    if (m >= kInfBits) {   // the same for the whole CTA
      unsigned int f = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) f = max(f, settle_nonfinite<0, 8>(v[i]));
      f = warp_max_u32(f);
      __syncthreads();
      if (lane == 0) smax[warp] = f;
      __syncthreads();
      m = warp_max_u32(smax[lane & 7]);
    }
    const BlockScale s = block_scale<E5M2>(__uint_as_float(m));
#pragma unroll
    for (int j = 0; j < 8; ++j) inv[j] = s.inv;
    if (threadIdx.x == 0) {
      if (TRANSPOSE)
        p.scale[(uint64_t)rt * p.ctiles + ct] = s.scale;
      else
        p.scale[(uint64_t)ct * p.rtiles + rt] = s.scale;
    }
  } else {
    unsigned int m[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // a finite maximum needs no second look here: the select costs less than a column's barrier
        const unsigned int b = abs_bits(v[i][j]);
        if (b >= kInfBits)
          v[i][j] = __uint_as_float(0x7FFFFFFFu);
        else
          m[j] = max(m[j], b);
      }
      m[j] = max(m[j], __shfl_xor_sync(0xFFFFFFFFu, m[j], 16));
    }
    if (lane < 16) {
#pragma unroll
      for (int j = 0; j < 8; ++j) smax[warp * 128 + cx * 8 + j] = m[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      unsigned int t = 0u;
#pragma unroll
      for (int w = 0; w < 8; ++w) t = max(t, smax[w * 128 + cx * 8 + j]);
      const BlockScale s = block_scale<E5M2>(__uint_as_float(t));
      inv[j] = s.inv;
      if (ry == 0 && j < ncol) p.scale[(uint64_t)rt * p.cols + col0 + j] = s.scale;
    }
  }
  if constexpr (!TRANSPOSE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= nrow) break;
      const uint2 r = quant8<E5M2>(v[i], inv[0]);
      unsigned char* dst = p.q + (row0 + i) * p.ldq + col0;
      if (VEC) {
        if (ncol == 8) *reinterpret_cast<uint2*>(dst) = r;
      } else {
        for (int j = 0; j < ncol; ++j) dst[j] = (unsigned char)((j < 4 ? r.x : r.y) >> (8 * (j & 3)));
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = v[i][j];
      const uint2 r = quant8<E5M2>(c, inv[j]);
      uint32_t* dst = reinterpret_cast<uint32_t*>(st + (cx * 8 + j) * kTransposePitch + ry * 8);
      dst[0] = r.x;
      dst[1] = r.y;
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
        reinterpret_cast<uint32_t*>(dst)[lane] = *reinterpret_cast<const uint32_t*>(st + c * kTransposePitch + lane * 4);
      } else {
        for (int b = lane; b < left; b += 32) dst[b] = st[c * kTransposePitch + b];
      }
    }
  }
}

}  // namespace kb
