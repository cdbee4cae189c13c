// Layer norm, forward and backward (contracts in include/kb_ops.h).
//
// Forward: a row lives in the registers of one warp (up to 1024 columns) or one CTA, 8 elements
// per lane and group of 256 (kb_block8.cuh).  The mean and then the sum of squared distances from
// it are reduced from the registers, so the row is read once and the variance does not suffer from
// the cancellation of sum(x^2)/n - mean^2.  The same registers then give y and, where asked for,
// the row's 8-bit blocks, so a consumer in 8 bits costs no second pass over y.
//
// Backward: rows by warp or CTA, walking over rows; each lane keeps its columns' sums of dy * xh and
// dy in registers over all its rows.  They leave once, as a partial row per CTA, and
// norm_param_kernel adds the partial rows in order.  So x and dy are read once for all three
// gradients.  The registers that hold the sums leave too few warps to cover the memory's latency,
// so long walks get their rows through a ring in shared memory, several rows ahead.
//
// Bound: memory; each element is read and written once.
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
  bool param_f32;
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
  uint32_t stages, slot_bytes;   // of the row ring
  bool param_f32, want_param;
  unsigned int* status;
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

// y and the row's blocks from a lane's centred elements (x - mean) of NCH groups.  Q: 0 no blocks,
// 1 e4m3, 2 e5m2.
template <int DT, bool VEC, int NCH, int Q>
__device__ __forceinline__ void norm_emit(const NormParams& p, uint64_t row, uint32_t g0, uint32_t gstep, int lane,
                                          float rstd, float (&v)[NCH][8]) {
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    float w[8], b[8];
    load_params<DT, VEC>(p.weight, p.param_f32, g0 + i * gstep, lane, p.cols, 1.0f, w);
    load_params<DT, VEC>(p.bias, p.param_f32, g0 + i * gstep, lane, p.cols, 0.0f, b);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const Pair t = mul2(pair(v[i][j], v[i][j + 1]), pair(rstd, rstd));
      unpair(fma2(t, pair(w[j], w[j + 1]), pair(b[j], b[j + 1])), v[i][j], v[i][j + 1]);
    }
  }
  if (p.y) {
#pragma unroll
    for (int i = 0; i < NCH; ++i)
      store_group<DT, VEC>(p.y, row * p.ldy, g0 + i * gstep, lane, p.cols, v[i]);
  }
  if constexpr (Q != 0) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) fill_tail<VEC>(g0 + i * gstep, lane, p.cols, 0.0f, v[i]);
    quant_groups<Q == 2, VEC, NCH>(v, g0, gstep, lane, p.cols, row, p.rows, p.q, p.ldq, p.scale);
  }
}

// A row per warp (WARP) or per CTA, NCH groups per warp in registers.
template <int DT, int NCH, bool VEC, bool WARP, int Q>
__global__ void __launch_bounds__(WARP ? 128 : NCH == 1 ? 1024 : 512, WARP ? 8 : NCH == 1 ? 1 : 2)
    norm_kernel(const NormParams p) {   // 64 registers: 32 warps share an SM
  __shared__ float red[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const uint64_t row = WARP ? (uint64_t)blockIdx.x * 4 + warp : blockIdx.x;
  if (WARP && row >= p.rows) return;
  const uint32_t g0 = WARP ? 0 : warp, gstep = WARP ? 1 : nwarps;   // this warp's groups: g0, g0 + gstep, ...
  float v[NCH][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i) load_group<DT, VEC>(p.x, row * p.ldx, g0 + i * gstep, lane, p.cols, v[i]);
  Pair s2 = pair(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < 8; j += 2) s2 = add2(s2, pair(v[i][j], v[i][j + 1]));
  const float s = fold(s2);
  const float n = (float)p.cols;
  const float mean = (WARP ? warp_sum(s) : cta_sum(s, red[0], warp, lane, nwarps)) / n;
  Pair ss2 = pair(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    fill_tail<VEC>(g0 + i * gstep, lane, p.cols, mean, v[i]);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const Pair d = add2(pair(v[i][j], v[i][j + 1]), pair(-mean, -mean));
      ss2 = fma2(d, d, ss2);
      unpair(d, v[i][j], v[i][j + 1]);
    }
  }
  const float ss = fold(ss2);
  const float var = (WARP ? warp_sum(ss) : cta_sum(ss, red[1], warp, lane, nwarps)) / n;
  const float rstd = 1.0f / sqrtf(var + p.eps);
  norm_emit<DT, VEC, NCH, Q>(p, row, g0, gstep, lane, rstd, v);
  if (lane == 0 && (WARP || warp == 0)) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// Rows too long for the registers of a CTA: three passes, the second and third from L2.
template <int DT, bool VEC, int Q>
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
    float v[1][8];
    load_group<DT, VEC>(p.x, row * p.ldx, g, lane, p.cols, v[0]);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[0][j] -= mean;
    norm_emit<DT, VEC, 1, Q>(p, row, g, 1, lane, rstd, v);
  }
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[row] = mean;
    if (p.rstd) p.rstd[row] = rstd;
  }
}

// Rows on their way from global memory: a ring of `stages` slots of `tensors` rows each.
constexpr uint32_t kRowRingStages = 8;   // at most
struct RowRing {
  unsigned char* buf;
  uint64_t* full;
  volatile unsigned int* abort_flag;
  unsigned int* status;
  uint32_t stages, row_bytes, slot_bytes;

  __device__ __forceinline__ void init() {   // one thread
    for (uint32_t i = 0; i < stages; ++i) mbar_init(&full[i], 1);
    *abort_flag = 0u;
    mbar_fence_init();
  }
  // one thread: the rows at s0 (and s1) into slot `slot`
  __device__ __forceinline__ void fetch(uint32_t slot, const void* s0, const void* s1) {
    const uint64_t policy = l2_policy_evict_first();   // read once
    mbar_arrive_expect_tx(&full[slot], s1 ? 2 * row_bytes : row_bytes);
    bulk_g2s(buf + slot * slot_bytes, s0, row_bytes, &full[slot], policy);
    if (s1) bulk_g2s(buf + slot * slot_bytes + slot_bytes / 2, s1, row_bytes, &full[slot], policy);
  }
  __device__ __forceinline__ bool wait(uint32_t slot, uint32_t phase) {
    return mbar_wait_bounded(&full[slot], phase, abort_flag, status);
  }
  // after a wait has run out: let the copies in flight land before the CTA may leave
  __device__ __forceinline__ void drain(uint64_t issued) {
    const uint64_t back = issued < stages ? issued : stages;
    for (uint64_t m = issued - back; m < issued; ++m) {
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(&full[m % stages], (uint32_t)((m / stages) & 1ull)))
        if (global_ns() - t0 > 1000000000ull) break;
    }
  }
};
template <int DT>
__device__ __forceinline__ const unsigned char* row_ptr(const void* base, uint64_t row, uint64_t ld) {
  return static_cast<const unsigned char*>(base) + row * ld * Elem<DT>::kBytes;
}

// Backward, rows by warp (WARP) or by CTA, walking over the rows with the grid's stride.  RING
// (VEC, CTA and two groups per warp only): the rows of x and dy come through shared memory.
template <int DT, int NCH, bool VEC, bool WARP, bool RING>
__global__ void __launch_bounds__(WARP ? 128 : NCH == 1 ? 768 : 512) norm_bwd_kernel(const NormBwdParams p) {
  __shared__ float red[2][2][32];
  __shared__ uint64_t full[kRowRingStages];
  __shared__ unsigned int abort_word;
  extern __shared__ __align__(128) unsigned char dyn[];   // WARP: [2][cols] sums; RING: the ring
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const uint64_t first = WARP ? (uint64_t)blockIdx.x * nwarps + warp : blockIdx.x;
  const uint64_t step = WARP ? (uint64_t)gridDim.x * nwarps : gridDim.x;
  RowRing ring{dyn, full, &abort_word, p.status, p.stages, p.cols * Elem<DT>::kBytes, p.slot_bytes};
  uint64_t issued = 0;
  if constexpr (RING) {
    if (threadIdx.x == 0) {
      ring.init();
      for (uint64_t r = blockIdx.x; r < p.rows && issued < p.stages; r += gridDim.x, ++issued)
        ring.fetch((uint32_t)issued, row_ptr<DT>(p.x, r, p.ldx), row_ptr<DT>(p.dy, r, p.lddy));
    }
    __syncthreads();
  }
  const float rn = 1.0f / (float)p.cols;
  float w[NCH][8], dw[NCH][8], db[NCH][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    load_params<DT, VEC>(p.weight, p.param_f32, WARP ? i : i * nwarps + warp, lane, p.cols, 1.0f, w[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = 0.0f;
  }
  uint32_t slot = 0, phase = 0;
  int turn = 0;
  float next_mean = first < p.rows ? p.mean[first] : 0.0f, next_rstd = first < p.rows ? p.rstd[first] : 0.0f;
  // without a ring, a CTA with one group per warp has the registers to read a row ahead
  constexpr bool kAhead = !RING && !WARP && NCH == 1;
  float xn[NCH][8], gn[NCH][8];
  if (kAhead && first < p.rows) {
    load_group<DT, VEC>(p.x, first * p.ldx, warp, lane, p.cols, xn[0]);
    load_group<DT, VEC>(p.dy, first * p.lddy, warp, lane, p.cols, gn[0]);
  }
  for (uint64_t row = first; row < p.rows; row += step, turn ^= 1) {
    float xh[NCH][8], g[NCH][8];
    const float mean = next_mean, rstd = next_rstd;
    if (row + step < p.rows) {   // a row ahead: their latency would stand at the head of every row
      next_mean = p.mean[row + step];
      next_rstd = p.rstd[row + step];
    }
    if constexpr (RING) {
      ring.wait(slot, phase);   // on failure the loop runs on, quickly, to keep the barriers together
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        load_group<DT, true>(dyn + slot * p.slot_bytes, 0, i * nwarps + warp, lane, p.cols, xh[i], mean);
        load_group<DT, true>(dyn + slot * p.slot_bytes + p.slot_bytes / 2, 0, i * nwarps + warp, lane, p.cols, g[i]);
      }
    } else if constexpr (kAhead) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xh[0][j] = xn[0][j];
        g[0][j] = gn[0][j];
      }
      fill_tail<VEC>(warp, lane, p.cols, mean, xh[0]);
      if (row + step < p.rows) {
        load_group<DT, VEC>(p.x, (row + step) * p.ldx, warp, lane, p.cols, xn[0]);
        load_group<DT, VEC>(p.dy, (row + step) * p.lddy, warp, lane, p.cols, gn[0]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        load_group<DT, VEC>(p.x, row * p.ldx, WARP ? i : i * nwarps + warp, lane, p.cols, xh[i], mean);
        load_group<DT, VEC>(p.dy, row * p.lddy, WARP ? i : i * nwarps + warp, lane, p.cols, g[i]);
      }
    }
    // past the row's end dy is 0 and x is the mean, unless the mean is not finite: the sums of such
    // a row are not finite either, and no column past the end is ever written
    Pair s1p = pair(0.0f, 0.0f), s2p = s1p;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const Pair x = mul2(add2(pair(xh[i][j], xh[i][j + 1]), pair(-mean, -mean)), pair(rstd, rstd));
        Pair gy = pair(g[i][j], g[i][j + 1]);
        unpair(fma2(gy, x, pair(dw[i][j], dw[i][j + 1])), dw[i][j], dw[i][j + 1]);
        unpair(add2(gy, pair(db[i][j], db[i][j + 1])), db[i][j], db[i][j + 1]);
        gy = mul2(gy, pair(w[i][j], w[i][j + 1]));
        s1p = add2(s1p, gy);
        s2p = fma2(gy, x, s2p);
        unpair(x, xh[i][j], xh[i][j + 1]);
        unpair(gy, g[i][j], g[i][j + 1]);
      }
    float s1 = warp_sum(fold(s1p)), s2 = warp_sum(fold(s2p));
    if constexpr (!WARP) {
      if (lane == 0) {
        red[turn][0][warp] = s1;
        red[turn][1][warp] = s2;
      }
      __syncthreads();   // one barrier per row: the other half of `red` serves the next row
      if constexpr (RING) {
        // every thread has read the rows: the slot takes those that are `stages` ahead
        const uint64_t ahead = row + (uint64_t)p.stages * gridDim.x;
        if (threadIdx.x == 0 && ahead < p.rows && !*ring.abort_flag) {
          ring.fetch(slot, row_ptr<DT>(p.x, ahead, p.ldx), row_ptr<DT>(p.dy, ahead, p.lddy));
          ++issued;
        }
        if (++slot == p.stages) {
          slot = 0;
          phase ^= 1u;
        }
      }
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
        for (int j = 0; j < 8; j += 2) {
          const Pair t = fma2(pair(xh[i][j], xh[i][j + 1]), pair(-s2, -s2), pair(g[i][j], g[i][j + 1]));
          unpair(mul2(add2(t, pair(-s1, -s1)), pair(rstd, rstd)), d[j], d[j + 1]);
        }
        store_group<DT, VEC>(p.dx, row * p.lddx, WARP ? i : i * nwarps + warp, lane, p.cols, d);
      }
    }
  }
  if constexpr (RING) {
    if (threadIdx.x == 0 && abort_word) ring.drain(issued);
  }
  if (!p.want_param) return;
  float* out = p.partial + (uint64_t)blockIdx.x * 2 * p.cols;
  if constexpr (WARP) {
    float* sums = reinterpret_cast<float*>(dyn);
    for (int k = 0; k < nwarps; ++k) {   // warps add in order
      if (warp == k) {
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t c = group_col<VEC>(i, lane, j);
            if (c < p.cols) {
              sums[c] = k ? sums[c] + dw[i][j] : dw[i][j];
              sums[p.cols + c] = k ? sums[p.cols + c] + db[i][j] : db[i][j];
            }
          }
      }
      __syncthreads();
    }
    for (uint32_t c = threadIdx.x; c < 2 * p.cols; c += blockDim.x) out[c] = sums[c];
  } else {
    // partial rows start on 16-byte boundaries where the columns of a VEC row do
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      store_group<KB_F32, VEC>(out, 0, i * nwarps + warp, lane, p.cols, dw[i]);
      store_group<KB_F32, VEC>(out, p.cols, i * nwarps + warp, lane, p.cols, db[i]);
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

// Sums of the partial rows per column, in a fixed order: 32 columns per CTA, each of 16 warps takes
// the partial rows w, w + 16, ... with eight loads on their way, then the warps' sums are added in
// order.  blockIdx.y: dweight, dbias.
constexpr int kParamWarps = 16;
template <int PT>
__global__ void __launch_bounds__(32 * kParamWarps) norm_param_kernel(const float* partial, uint32_t nparts,
                                                                      uint32_t cols, void* dweight, void* dbias) {
  __shared__ float part[kParamWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t c = blockIdx.x * 32 + lane;
  const float* src = partial + (uint64_t)blockIdx.y * cols + c;
  void* out = blockIdx.y ? dbias : dweight;
  if (out == nullptr) return;
  float s = 0.0f;
  for (uint32_t i0 = warp; i0 < nparts; i0 += 8 * kParamWarps) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t i = i0 + k * kParamWarps;
      v[k] = i < nparts && c < cols ? src[(uint64_t)i * 2 * cols] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) s += v[k];
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < cols) {
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < kParamWarps; ++w) t += part[w][lane];
    store_elem<PT>(out, c, t);
  }
}

}  // namespace kb
