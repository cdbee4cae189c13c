// Layer norm, forward and backward (contracts in include/kb_ops.h).
//
// Forward: a row lives in the registers of one warp (short rows) or one CTA, 8 elements per lane
// and group of 256 (kb_block8.cuh).  The mean and then the sum of squared distances from it are
// reduced from the registers, so the row is read once and the variance does not suffer from the
// cancellation of sum(x^2)/n - mean^2.  The same registers then give y and, where asked for, the
// row's 8-bit blocks, so a consumer in 8 bits costs no second pass over y.
//
// Bound: memory.  Each element is read and written once; the parameters stay in L1/L2.
#pragma once

#include "kb_block8.cuh"

namespace kb {

struct NormParams {
  const void* x;
  const void* weight;
  const void* bias;
  void* y;
  float* mean;
  float* rstd;
  unsigned char* q;
  float* scale;
  uint64_t rows, ldx, ldy, ldq;
  uint32_t cols, groups;
  float eps;
  bool param_f32, e5m2;
};

struct NormBwdParams {
  const void* dy;
  const void* x;
  const void* weight;
  const float* mean;
  const float* rstd;
  void* dx;
  float* partial;            // [partial rows][2][cols]: dweight, dbias
  uint64_t rows, lddy, ldx, lddx;
  uint32_t cols, groups;
  bool param_f32, want_param;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
// Sum over the CTA's warps in warp order, the same value in every thread.  `red` holds one float
// per warp and is not reused before the next barrier of another reduction.
__device__ __forceinline__ float cta_sum(float v, float* red, int warp, int lane, int nwarps) {
  v = warp_sum(v);
  if (lane == 0) red[warp] = v;
  __syncthreads();
  return warp_sum(lane < nwarps ? red[lane] : 0.0f);
}

// y and the row's other outputs from a lane's 8 elements of group g
template <int DT, bool VEC>
__device__ __forceinline__ void norm_emit(const NormParams& p, uint64_t row, uint32_t g, int lane, float mean,
                                          float rstd, float (&v)[8]) {
  float w[8], b[8];
  load_params<DT, VEC>(p.weight, p.param_f32, g, lane, p.cols, 1.0f, w);
  load_params<DT, VEC>(p.bias, p.param_f32, g, lane, p.cols, 0.0f, b);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = fmaf((v[j] - mean) * rstd, w[j], b[j]);
  if (p.y) store_group<DT, VEC>(p.y, row * p.ldy, g, lane, p.cols, v);
  if (p.q) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (group_col<VEC>(g, lane, j) >= p.cols) v[j] = 0.0f;
    if (p.e5m2)
      quant_group<true, VEC>(v, g, lane, p.cols, row, p.rows, p.q, p.ldq, p.scale);
    else
      quant_group<false, VEC>(v, g, lane, p.cols, row, p.rows, p.q, p.ldq, p.scale);
  }
}

// One row per warp (WARP) or per CTA, NCH groups per warp in registers.
template <int DT, int NCH, bool VEC, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : NCH == 1 ? 1024 : 512) norm_kernel(const NormParams p) {
  __shared__ float red[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const uint64_t row = WARP ? (uint64_t)blockIdx.x * nwarps + warp : blockIdx.x;
  if (WARP && row >= p.rows) return;
  float v[NCH][8];
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
    load_group<DT, VEC>(p.x, row * p.ldx, WARP ? i : i * nwarps + warp, lane, p.cols, v[i]);
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[i][j];
  const float n = (float)p.cols;
  const float mean = (WARP ? warp_sum(s) : cta_sum(s, red[0], warp, lane, nwarps)) / n;
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = v[i][j] - mean;
      if (group_col<VEC>(WARP ? i : i * nwarps + warp, lane, j) < p.cols) ss = fmaf(d, d, ss);
    }
  const float var = (WARP ? warp_sum(ss) : cta_sum(ss, red[1], warp, lane, nwarps)) / n;
  const float rstd = 1.0f / sqrtf(var + p.eps);
#pragma unroll
  for (int i = 0; i < NCH; ++i)
    norm_emit<DT, VEC>(p, row, WARP ? i : i * nwarps + warp, lane, mean, rstd, v[i]);
  if (lane == 0 && (WARP || warp == 0)) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// Rows too long for the registers of a CTA: three passes, the second and third from L2.
template <int DT, bool VEC>
__global__ void __launch_bounds__(512) norm_long_kernel(const NormParams p) {
  __shared__ float red[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const uint64_t row = blockIdx.x;
  const float n = (float)p.cols;
  float s = 0.0f;
  for (uint32_t g = warp; g < p.groups; g += nwarps) {
    float v[8];
    load_group<DT, VEC>(p.x, row * p.ldx, g, lane, p.cols, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[j];
  }
  const float mean = cta_sum(s, red[0], warp, lane, nwarps) / n;
  float ss = 0.0f;
  for (uint32_t g = warp; g < p.groups; g += nwarps) {
    float v[8];
    load_group<DT, VEC>(p.x, row * p.ldx, g, lane, p.cols, v, mean);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = v[j] - mean;
      ss = fmaf(d, d, ss);
    }
  }
  const float var = cta_sum(ss, red[1], warp, lane, nwarps) / n;
  const float rstd = 1.0f / sqrtf(var + p.eps);
  for (uint32_t g = warp; g < p.groups; g += nwarps) {
    float v[8];
    load_group<DT, VEC>(p.x, row * p.ldx, g, lane, p.cols, v);
    norm_emit<DT, VEC>(p, row, g, lane, mean, rstd, v);
  }
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// Backward, short and middle rows: a warp or a CTA walks over rows with a stride of the grid.
// Each lane keeps its columns' sums of dy * xh and dy in registers over all its rows; they leave
// once, as a partial row per CTA, and norm_param_kernel adds the partial rows in order.  So x and
// dy are read once for all three gradients.
template <int DT, int NCH, bool VEC, bool WARP>
__global__ void __launch_bounds__(512) norm_bwd_kernel(const NormBwdParams p) {
  __shared__ float red[2][2][16];
  extern __shared__ float sum_smem[];   // WARP: [2][cols]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const uint64_t first = WARP ? (uint64_t)blockIdx.x * nwarps + warp : blockIdx.x;
  const uint64_t step = WARP ? (uint64_t)gridDim.x * nwarps : gridDim.x;
  const float rn = 1.0f / (float)p.cols;
  float dw[NCH][8], db[NCH][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = 0.0f;
  int turn = 0;
  for (uint64_t row = first; row < p.rows; row += step, turn ^= 1) {
    float xh[NCH][8], gy[NCH][8];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const uint32_t g = WARP ? i : i * nwarps + warp;
      load_group<DT, VEC>(p.x, row * p.ldx, g, lane, p.cols, xh[i]);
      load_group<DT, VEC>(p.dy, row * p.lddy, g, lane, p.cols, gy[i]);
    }
    const float mean = p.mean[row], rstd = p.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const uint32_t g = WARP ? i : i * nwarps + warp;
      float w[8];
      load_params<DT, VEC>(p.weight, p.param_f32, g, lane, p.cols, 1.0f, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xh[i][j] = (xh[i][j] - mean) * rstd;
        dw[i][j] = fmaf(gy[i][j], xh[i][j], dw[i][j]);
        db[i][j] += gy[i][j];
        gy[i][j] *= w[j];
        if (group_col<VEC>(g, lane, j) < p.cols) {
          s1 += gy[i][j];
          s2 = fmaf(gy[i][j], xh[i][j], s2);
        }
      }
    }
    s1 = warp_sum(s1);
    s2 = warp_sum(s2);
    if constexpr (!WARP) {
      if (lane == 0) {
        red[turn][0][warp] = s1;
        red[turn][1][warp] = s2;
      }
      __syncthreads();   // one barrier per row: the other half of `red` serves the next row
      s1 = warp_sum(lane < nwarps ? red[turn][0][lane] : 0.0f);
      s2 = warp_sum(lane < nwarps ? red[turn][1][lane] : 0.0f);
    }
    if (p.dx) {
      s1 *= rn;
      s2 *= rn;
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        float d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = rstd * (gy[i][j] - s1 - xh[i][j] * s2);
        store_group<DT, VEC>(p.dx, row * p.lddx, WARP ? i : i * nwarps + warp, lane, p.cols, d);
      }
    }
  }
  if (!p.want_param) return;
  float* out = p.partial + (uint64_t)blockIdx.x * 2 * p.cols;
  if constexpr (WARP) {
    for (int w = 0; w < nwarps; ++w) {   // warps add in order
      if (warp == w) {
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t c = group_col<VEC>(i, lane, j);
            if (c < p.cols) {
              sum_smem[c] = w ? sum_smem[c] + dw[i][j] : dw[i][j];
              sum_smem[p.cols + c] = w ? sum_smem[p.cols + c] + db[i][j] : db[i][j];
            }
          }
      }
      __syncthreads();
    }
    for (uint32_t c = threadIdx.x; c < 2 * p.cols; c += blockDim.x) out[c] = sum_smem[c];
  } else {
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t c = group_col<VEC>(i * nwarps + warp, lane, j);
        if (c < p.cols) {
          out[c] = dw[i][j];
          out[p.cols + c] = db[i][j];
        }
      }
  }
}

// Backward, rows too long for the registers: dx by row (two passes over the row) ...
template <int DT, bool VEC>
__global__ void __launch_bounds__(512) norm_bwd_long_kernel(const NormBwdParams p) {
  __shared__ float red[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const uint64_t row = blockIdx.x;
  const float mean = p.mean[row], rstd = p.rstd[row];
  float s1 = 0.0f, s2 = 0.0f;
  for (uint32_t g = warp; g < p.groups; g += nwarps) {
    float x[8], gy[8], w[8];
    load_group<DT, VEC>(p.x, row * p.ldx, g, lane, p.cols, x);
    load_group<DT, VEC>(p.dy, row * p.lddy, g, lane, p.cols, gy);
    load_params<DT, VEC>(p.weight, p.param_f32, g, lane, p.cols, 1.0f, w);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (group_col<VEC>(g, lane, j) < p.cols) {
        const float gw = gy[j] * w[j];
        s1 += gw;
        s2 = fmaf(gw, (x[j] - mean) * rstd, s2);
      }
  }
  const float rn = 1.0f / (float)p.cols;
  s1 = cta_sum(s1, red[0], warp, lane, nwarps) * rn;
  s2 = cta_sum(s2, red[1], warp, lane, nwarps) * rn;
  for (uint32_t g = warp; g < p.groups; g += nwarps) {
    float x[8], gy[8], w[8];
    load_group<DT, VEC>(p.x, row * p.ldx, g, lane, p.cols, x);
    load_group<DT, VEC>(p.dy, row * p.lddy, g, lane, p.cols, gy);
    load_params<DT, VEC>(p.weight, p.param_f32, g, lane, p.cols, 1.0f, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = rstd * (gy[j] * w[j] - s1 - (x[j] - mean) * rstd * s2);
    store_group<DT, VEC>(p.dx, row * p.lddx, g, lane, p.cols, x);
  }
}
// ... and the parameters' partial sums by column: a warp owns a group of columns and walks over
// the rows of its slice (blockIdx.y).
template <int DT, bool VEC>
__global__ void __launch_bounds__(256) norm_bwd_cols_kernel(const NormBwdParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const uint32_t g = blockIdx.x * nwarps + warp;
  if (g >= p.groups) return;
  float dw[8] = {}, db[8] = {};
  for (uint64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
    const float mean = p.mean[row], rstd = p.rstd[row];
    float x[8], gy[8];
    load_group<DT, VEC>(p.x, row * p.ldx, g, lane, p.cols, x);
    load_group<DT, VEC>(p.dy, row * p.lddy, g, lane, p.cols, gy);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dw[j] = fmaf(gy[j], (x[j] - mean) * rstd, dw[j]);
      db[j] += gy[j];
    }
  }
  float* out = p.partial + (uint64_t)blockIdx.y * 2 * p.cols;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t c = group_col<VEC>(g, lane, j);
    if (c < p.cols) {
      out[c] = dw[j];
      out[p.cols + c] = db[j];
    }
  }
}

// Sums of the partial rows per column, in a fixed order: 32 columns per CTA, each warp takes the
// partial rows w, w + 32, ..., then the warps' sums are added in order.  blockIdx.y: dweight, dbias.
template <int PT>
__global__ void __launch_bounds__(1024) norm_param_kernel(const float* partial, uint32_t nparts, uint32_t cols,
                                                          void* dweight, void* dbias) {
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t c = blockIdx.x * 32 + lane;
  const float* src = partial + (uint64_t)blockIdx.y * cols;
  void* out = blockIdx.y ? dbias : dweight;
  if (out == nullptr) return;
  float s = 0.0f;
  if (c < cols)
    for (uint32_t i = warp; i < nparts; i += 32) s += src[(uint64_t)i * 2 * cols + c];
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < cols) {
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < 32; ++w) t += part[w][lane];
    store_elem<PT>(out, c, t);
  }
}

}  // namespace kb
