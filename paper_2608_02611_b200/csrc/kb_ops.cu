// Host side of the model operators: argument checks, choice of kernel, launch.
// Declarations and their contracts are in include/kb_ops.h.
#include <algorithm>
#include <cmath>

#include "../../include/kb_hooks.h"
#include "../../include/kb_ops.h"
#include "kb_ctx.cuh"
#include "kb_matmul.cuh"
#include "kb_norm.cuh"
#include "kb_quant.cuh"

using namespace kb;

namespace {

inline bool is_f8_type(int dt) { return dt == KB_F8E4M3 || dt == KB_F8E5M2; }
// rows of a matrix start on 16-byte boundaries
inline bool rows_aligned(const void* p, uint64_t ld, int bytes) { return aligned16(p) && (ld * bytes) % 16 == 0; }

// A matrix argument: not null, element-aligned, leading dimension at least its columns.
kb_status check_matrix(kb_ctx* ctx, const char* where, const char* name, const void* p, uint64_t cols, uint64_t ld,
                       int bytes) {
  if (!p) return fail(ctx, KB_ERR_INVALID_ARG, "%s: %s is NULL", where, name);
  if (!aligned_to(p, bytes)) return fail(ctx, KB_ERR_ALIGNMENT, "%s: %s is not aligned to its element type", where, name);
  if (ld < cols)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: leading dimension %llu of %s is less than its %llu columns", where,
                (unsigned long long)ld, name, (unsigned long long)cols);
  return KB_OK;
}
kb_status check_vector(kb_ctx* ctx, const char* where, const char* name, const void* p, int bytes) {
  if (!aligned_to(p, bytes)) return fail(ctx, KB_ERR_ALIGNMENT, "%s: %s is not aligned to its element type", where, name);
  return KB_OK;
}

// ---- quantisation ------------------------------------------------------------------------------

template <int DT, bool VEC, bool E5M2>
kb_status launch_quant(kb_ctx* ctx, const QuantParams& p, bool transpose, bool tiles, cudaStream_t st) {
  if (!transpose && !tiles) {
    const uint64_t pieces = (p.groups + kQuantRowGroups - 1) / kQuantRowGroups;
    const dim3 grid((unsigned int)((p.rows + 7) / 8), (unsigned int)std::min<uint64_t>(pieces, 65535));
    if (!VEC && p.q_vec)
      quant_rows_kernel<DT, VEC, !VEC, E5M2><<<grid, 256, 0, st>>>(p);
    else
      quant_rows_kernel<DT, VEC, false, E5M2><<<grid, 256, 0, st>>>(p);
    return launched(ctx);
  }
  const uint64_t n = (uint64_t)p.rtiles * p.ctiles;
  if (n > 0x7FFFFFFFull) return fail(ctx, KB_ERR_UNSUPPORTED, "kb_quantize_blocks: more than 2^31 - 1 tiles");
  const unsigned int grid = (unsigned int)n;
  if (tiles && transpose)
    quant_tile_kernel<DT, VEC, E5M2, true, true><<<grid, 256, 0, st>>>(p);
  else if (tiles)
    quant_tile_kernel<DT, VEC, E5M2, true, false><<<grid, 256, 0, st>>>(p);
  else
    quant_tile_kernel<DT, VEC, E5M2, false, true><<<grid, 256, 0, st>>>(p);
  return launched(ctx);
}
template <int DT>
kb_status launch_quant(kb_ctx* ctx, const QuantParams& p, bool vec, bool e5m2, bool transpose, bool tiles,
                       cudaStream_t st) {
  if (vec)
    return e5m2 ? launch_quant<DT, true, true>(ctx, p, transpose, tiles, st)
                : launch_quant<DT, true, false>(ctx, p, transpose, tiles, st);
  return e5m2 ? launch_quant<DT, false, true>(ctx, p, transpose, tiles, st)
              : launch_quant<DT, false, false>(ctx, p, transpose, tiles, st);
}

// ---- layer norm ----------------------------------------------------------------------------------

// The row ring of a CTA that walks over rows of `bytes` each: as many slots as fit its share of an
// SM's shared memory, 0 if fewer than two do (then the rows are read directly).
constexpr size_t kRingBytes = 220 * 1024;   // of an SM's shared memory
uint32_t ring_stages(size_t bytes, int ctas_per_sm) {
  const size_t share = kRingBytes / ctas_per_sm - 1024;
  return (uint32_t)std::min<size_t>(share / round_up(bytes, 128), kRowRingStages);
}
// CTAs of `threads` threads of a kernel that fit an SM by its registers (the count is fixed at
// compile time, so it is asked for once), at most `most`.
template <auto Kernel>
int ctas_by_registers(unsigned int threads, int most) {
  static const int regs = [] {
    cudaFuncAttributes a = {};
    return cudaFuncGetAttributes(&a, Kernel) == cudaSuccess ? a.numRegs : 255;
  }();
  const int per_warp = (regs + 7) / 8 * 8 * 32;
  return std::max(1, std::min(most, 65536 / per_warp / (int)(threads / 32)));
}
// The limit belongs to the kernel on the device, not to the context: it is raised to the same size by every
// call, so that no other thread's call, with narrower rows on a context of its own, takes it back.
template <class K>
kb_status ring_limits(kb_ctx* ctx, K kernel, size_t smem) {
  if (smem > 40 * 1024)   // static and dynamic shared memory together: 48 KB without asking
    KB_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes));
  return KB_OK;
}

template <int DT, int NCH, bool VEC, int Q>
kb_status launch_norm(kb_ctx* ctx, const NormParams& p, cudaStream_t st) {
  const uint32_t warps = (p.groups + NCH - 1) / NCH;
  if (NCH == 2 || warps == 1)   // two groups per lane are only chosen for rows of two groups
    norm_kernel<DT, NCH, VEC, true, Q><<<(unsigned int)((p.rows + 3) / 4), 128, 0, st>>>(p);
  else if constexpr (NCH != 2)
    norm_kernel<DT, NCH, VEC, false, Q><<<(unsigned int)p.rows, 32 * warps, 0, st>>>(p);
  return launched(ctx);
}
template <int DT, bool VEC, int Q>
kb_status launch_norm(kb_ctx* ctx, const NormParams& p, cudaStream_t st) {
  // one row per SM at most: as many warps as the row has groups, for the shortest time of one row
  if (p.groups == 1 || (p.groups <= 32 && p.rows <= (uint64_t)ctx->sm_count))
    return launch_norm<DT, 1, VEC, Q>(ctx, p, st);
  if (p.groups == 2) return launch_norm<DT, 2, VEC, Q>(ctx, p, st);
  if (p.groups <= 64) return launch_norm<DT, 4, VEC, Q>(ctx, p, st);
  norm_long_kernel<DT, VEC, Q><<<(unsigned int)p.rows, 512, 0, st>>>(p);
  return launched(ctx);
}
template <int DT>
kb_status launch_norm(kb_ctx* ctx, const NormParams& p, bool vec, bool e5m2, cudaStream_t st) {
  if (vec)
    return !p.q ? launch_norm<DT, true, 0>(ctx, p, st)
                : e5m2 ? launch_norm<DT, true, 2>(ctx, p, st) : launch_norm<DT, true, 1>(ctx, p, st);
  return !p.q ? launch_norm<DT, false, 0>(ctx, p, st)
              : e5m2 ? launch_norm<DT, false, 2>(ctx, p, st) : launch_norm<DT, false, 1>(ctx, p, st);
}

// The workspace of partial sums, with room for `need` bytes
kb_status ensure_partials(kb_ctx* ctx, size_t need, cudaStream_t st) {
  ctx->captured |= is_capturing(st);
  return ensure_workspace(ctx, &ctx->ops_ws, &ctx->ops_ws_bytes, need, st, "partial parameter gradients");
}

template <int DT, int NCH, bool VEC, bool WARP>
kb_status launch_norm_bwd(kb_ctx* ctx, NormBwdParams& p, unsigned int threads, uint32_t* nparts, cudaStream_t st) {
  const uint64_t per = WARP ? threads / 32 : 1;
  auto launch = [&](auto kernel, uint64_t resident, size_t smem) {
    const unsigned int grid = (unsigned int)std::min<uint64_t>((p.rows + per - 1) / per, resident);
    *nparts = grid;
    if (p.want_param) {
      KB_TRY(ensure_partials(ctx, (size_t)grid * 2 * p.cols * sizeof(float), st));
      p.partial = reinterpret_cast<float*>(ctx->ops_ws);
    }
    kernel<<<grid, threads, smem, st>>>(p);
    return launched(ctx);
  };
  if constexpr (VEC && !WARP && NCH == 2) {   // with one group per warp the rows are too few for the ring
    constexpr auto kernel = norm_bwd_kernel<DT, NCH, true, false, true>;
    const int per_sm = ctas_by_registers<kernel>(threads, std::max(4, (int)(1024 / threads)));
    const uint64_t resident = (uint64_t)ctx->sm_count * per_sm;
    const size_t bytes = (size_t)p.cols * elem_bytes((kb_dtype)DT);
    const uint32_t stages = ring_stages(2 * round_up(bytes, 128), per_sm);
    if (p.rows >= 2 * resident && stages >= 2) {
      p.stages = stages;
      p.slot_bytes = (uint32_t)(2 * round_up(bytes, 128));
      const size_t smem = (size_t)stages * p.slot_bytes;
      KB_TRY(ring_limits(ctx, kernel, smem));
      return launch(kernel, resident, smem);
    }
  }
  constexpr auto kernel = norm_bwd_kernel<DT, NCH, VEC, WARP, false>;
  return launch(kernel, (uint64_t)ctx->sm_count * ctas_by_registers<kernel>(threads, WARP ? 4 : std::max(2, (int)(1024 / threads))),
                WARP ? 2 * sizeof(float) * p.cols : 0);
}

// Rows too long for the registers: slices of the rows, a partial row each
uint32_t norm_bwd_slices(const kb_ctx* ctx, uint64_t rows, uint32_t groups) {
  const uint64_t want = std::max<uint64_t>(1, 8ull * ctx->sm_count / ((groups + 7) / 8));
  return (uint32_t)std::min<uint64_t>(std::min<uint64_t>(want, (rows + 7) / 8), 65535);
}
// Partial rows of a backward pass over `rows` rows or fewer, at most: the grids below as if registers did not
// limit the CTAs per SM
uint64_t norm_bwd_most_partials(const kb_ctx* ctx, uint64_t rows, uint32_t groups) {
  if (groups > 32) return norm_bwd_slices(ctx, rows, groups);
  const uint32_t threads = 32 * ((groups + 1) / 2);   // two groups per warp: the most CTAs per SM
  return std::min<uint64_t>(rows, (uint64_t)ctx->sm_count * (groups <= 2 ? 4 : std::max(4u, 1024 / threads)));
}

template <int DT, bool VEC>
kb_status launch_norm_bwd(kb_ctx* ctx, NormBwdParams& p, uint32_t* nparts, cudaStream_t st) {
  const uint32_t g = p.groups;
  // a warp per row up to 512 columns (32768 x 512 bf16: 32 us, by CTAs 42; 32768 x 768: 51 and 48)
  if (g == 1) return launch_norm_bwd<DT, 1, VEC, true>(ctx, p, 128, nparts, st);
  if (g == 2) return launch_norm_bwd<DT, 2, VEC, true>(ctx, p, 128, nparts, st);
  // Two groups per warp, through the ring from twice the resident CTAs on (16000 x 4096 bf16: 73 us, with one
  // group per warp 101); one group per warp with a row ahead, up to 24 warps, for fewer than two rows per SM
  // and for rows that cannot take the ring (777 x 5003 fp16: 17 us, with two groups 19).  In between, up to
  // the ring's first row, the two differ either way: 400 x 1024 bf16 8.2 us with two groups and 8.6 with
  // one, 500 x 3000 9.7 and 10.0, 1000 x 2048 12.5 and 11.7, 2000 x 1024 17.0 and 14.1.
  const bool few = !VEC || p.rows < 2ull * ctx->sm_count;
  if (few && g <= 24) return launch_norm_bwd<DT, 1, VEC, false>(ctx, p, 32 * g, nparts, st);
  if (g <= 32) return launch_norm_bwd<DT, 2, VEC, false>(ctx, p, 32 * ((g + 1) / 2), nparts, st);
  const uint32_t gx = (g + 7) / 8, slices = norm_bwd_slices(ctx, p.rows, g);
  if (p.want_param) {   // what can be refused comes before the first launch
    KB_TRY(ensure_partials(ctx, (size_t)slices * 2 * p.cols * sizeof(float), st));
    p.partial = reinterpret_cast<float*>(ctx->ops_ws);
  }
  if (p.dx) {
    norm_bwd_long_kernel<DT, VEC><<<(unsigned int)p.rows, 512, 0, st>>>(p);
    KB_TRY(launched(ctx));
  }
  if (p.want_param) {
    *nparts = slices;
    norm_bwd_cols_kernel<DT, VEC><<<dim3(gx, slices), 256, 0, st>>>(p);
    KB_TRY(launched(ctx));
  }
  return KB_OK;
}

// ---- product ---------------------------------------------------------------------------------------

template <int BN>
void lanes_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* attr, unsigned int grid, uint32_t splits, cudaStream_t st) {
  cfg->gridDim = dim3(grid);
  cfg->blockDim = dim3(LaneTile<BN>::kThreads);
  cfg->dynamicSmemBytes = LaneTile<BN>::kSmem;
  cfg->stream = st;
  attr->id = cudaLaunchAttributeClusterDimension;
  attr->val.clusterDim.x = splits;
  attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
  cfg->attrs = attr;
  cfg->numAttrs = 1;
}
template <int BN>
kb_status lanes_attr(kb_ctx* ctx) {
  KB_CUDA(ctx, cudaFuncSetAttribute(matmul_lanes_kernel<BN, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)LaneTile<BN>::kSmem));
  KB_CUDA(ctx, cudaFuncSetAttribute(matmul_lanes_kernel<BN, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)LaneTile<BN>::kSmem));
  return KB_OK;
}

kb_status prepare_matmul(kb_ctx* ctx) {
  if (ctx->ops_ready) return KB_OK;
  KB_TRY(find_encoder(ctx, "kb_matmul_blocks"));
  KB_TRY(lanes_attr<16>(ctx));
  KB_TRY(lanes_attr<32>(ctx));
  KB_TRY(lanes_attr<64>(ctx));
  KB_TRY(lanes_attr<128>(ctx));
  KB_CUDA(ctx, cudaFuncSetAttribute(matmul_pair_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairTile::kSmem));
  KB_CUDA(ctx, cudaFuncSetAttribute(matmul_pair_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairTile::kSmem));
  // the pair kernel's warps split the registers it was launched with; with fewer, as other compiler
  // options would give it, they would wait for the rest for good
  for (const void* kernel : {reinterpret_cast<const void*>(&matmul_pair_kernel<false>), reinterpret_cast<const void*>(&matmul_pair_kernel<true>)}) {
    cudaFuncAttributes attr = {};
    KB_CUDA(ctx, cudaFuncGetAttributes(&attr, kernel));
    if (attr.numRegs < PairTile::kRegsLaunch)
      return fail(ctx, KB_ERR_UNSUPPORTED, "kb_matmul_blocks: the library was compiled with %d registers for a kernel that splits %d",
                  attr.numRegs, PairTile::kRegsLaunch);
  }
  // every variant takes an SM of its own, so one of them stands for all
  for (uint32_t n = 1; n <= 8; ++n) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    lanes_config<128>(&cfg, attr, n, n, nullptr);
    KB_CUDA(ctx, cudaOccupancyMaxActiveClusters(&ctx->cluster_room[n], matmul_lanes_kernel<128, false>, &cfg));
  }
  ctx->ops_ready = true;
  return KB_OK;
}

// Tensor map of an 8-bit matrix [rows][cols], boxes of 128 columns and `box_rows` rows in the
// 128-byte swizzle; places outside the matrix read as zero.
kb_status encode_map(kb_ctx* ctx, CUtensorMap* map, const void* p, uint64_t rows, uint64_t cols, uint64_t ld,
                     uint32_t box_rows) {
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {ld};
  const cuuint32_t box[2] = {128, box_rows}, step[2] = {1, 1};
  const CUresult rc = reinterpret_cast<EncodeTiled>(ctx->encode_tiled)(
      map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, step,
      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (rc != CUDA_SUCCESS) return fail(ctx, KB_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d", (int)rc);
  return KB_OK;
}

// CTAs per tile of matmul_lanes_kernel: as many as run at the same time, at least two K blocks each,
// 8 at most (the portable cluster size).  A cluster stays within one of the GPU's processing
// clusters, so sizes that do not divide those leave SMs idle, and a second wave costs more than the
// shorter K range saves (512x512x8192: 8 CTAs a tile 19.7 us in two waves, 5 a tile 12.4 us in one).
uint32_t lane_splits(const kb_ctx* ctx, uint64_t tiles, uint32_t KB) {
  uint32_t splits = std::max(1u, std::min(KB / 2, 8u));
  while (splits > 1 && tiles > (uint64_t)ctx->cluster_room[splits]) --splits;
  return splits;
}
// Which kernel takes more than 64 rows of A.  Measured per K block and CTA, long K: 0.47 us for a
// 128 x 128 tile of matmul_lanes_kernel, 0.52 us for a 256 x 256 tile of a pair.  The pair does four
// times the work in it but needs 74 tiles to fill the card and cannot share a tile's K blocks:
// 300x1000x2000 8.5 us by lanes and 18 by pairs, 512x512x8192 12 and 34, 256x4096x4096 14 and 21;
// 1024x2048x4096 19 and 21; 512x8192x8192 85 and 38.
bool lanes_are_faster(const kb_ctx* ctx, uint64_t M, uint64_t N, uint32_t KB) {
  const uint64_t lane_tiles = ((M + 127) / 128) * ((N + 127) / 128), pair_tiles = ((M + 255) / 256) * ((N + 255) / 256);
  const uint64_t sms = (uint64_t)ctx->sm_count, pairs = sms / 2, splits = lane_splits(ctx, lane_tiles, KB);
  const double lanes = 0.47 * (double)((lane_tiles * splits + sms - 1) / sms) * (double)((KB + splits - 1) / splits);
  const double by_pairs = 0.52 * (double)((pair_tiles + pairs - 1) / pairs) * (double)KB;
  return lanes < by_pairs;
}

template <int BN>
kb_status launch_lanes(kb_ctx* ctx, MatmulParams& p, const void* a, uint64_t lda, bool a_e5m2, const void* b,
                       uint64_t ldb, bool b_e5m2, uint64_t K, cudaStream_t st) {
  CUtensorMap map_a, map_b;
  KB_TRY(encode_map(ctx, &map_a, a, p.M, K, lda, BN));
  KB_TRY(encode_map(ctx, &map_b, b, p.N, K, ldb, 128));
  p.idesc = mma_idesc_f8(b_e5m2, a_e5m2, 128, BN);
  p.tiles_m = (p.M + BN - 1) / BN;
  const uint64_t tiles = (uint64_t)p.tiles_m * ((p.N + 127) / 128);
  const uint32_t splits = lane_splits(ctx, tiles, p.KB);
  p.splits = splits;
  if (tiles * splits > 0x7FFFFFFFull) return fail(ctx, KB_ERR_UNSUPPORTED, "kb_matmul_blocks: more than 2^31 - 1 tiles");
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  lanes_config<BN>(&cfg, attr, (unsigned int)(tiles * splits), splits, st);
  if (p.b_scale_shift)
    KB_CUDA(ctx, cudaLaunchKernelEx(&cfg, matmul_lanes_kernel<BN, false>, map_b, map_a, p));
  else
    KB_CUDA(ctx, cudaLaunchKernelEx(&cfg, matmul_lanes_kernel<BN, true>, map_b, map_a, p));
  ctx->product_rows = BN;
  ctx->product_splits = splits;
  return launched(ctx);
}

kb_status launch_pair(kb_ctx* ctx, MatmulParams& p, const void* a, uint64_t lda, bool a_e5m2, const void* b,
                      uint64_t ldb, bool b_e5m2, uint64_t K, cudaStream_t st) {
  CUtensorMap map_a, map_b;
  KB_TRY(encode_map(ctx, &map_a, a, p.M, K, lda, 128));
  KB_TRY(encode_map(ctx, &map_b, b, p.N, K, ldb, 128));
  p.idesc = mma_idesc_f8(a_e5m2, b_e5m2, 256, 256);
  p.tiles_m = (p.M + 255) / 256;
  p.splits = 1;
  const uint64_t tiles = (uint64_t)p.tiles_m * ((p.N + 255) / 256);
  if (tiles > 0x3FFFFFFFull) return fail(ctx, KB_ERR_UNSUPPORTED, "kb_matmul_blocks: more than 2^30 - 1 tiles");
  const unsigned int pairs = (unsigned int)std::min<uint64_t>(tiles, (uint64_t)ctx->sm_count / 2);
  if (p.b_scale_shift)
    matmul_pair_kernel<false><<<2 * pairs, PairTile::kThreads, PairTile::kSmem, st>>>(map_a, map_b, p);
  else
    matmul_pair_kernel<true><<<2 * pairs, PairTile::kThreads, PairTile::kSmem, st>>>(map_a, map_b, p);
  ctx->product_rows = 256;
  ctx->product_splits = 1;
  return launched(ctx);
}

}  // namespace

// ---------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------

extern "C" kb_status kb_ctx_last_product(const kb_ctx* ctx, uint32_t* rows, uint32_t* splits) {
  if (!ctx || !rows || !splits) return KB_ERR_INVALID_ARG;
  *rows = ctx->product_rows;
  *splits = ctx->product_splits;
  return KB_OK;
}

extern "C" kb_status kb_quantize_blocks(kb_ctx* ctx, const void* d_x, uint64_t rows, uint64_t cols, uint64_t ldx,
                                        kb_dtype dtype, int transpose, kb_scale_mode mode, void* d_q, uint64_t ldq,
                                        kb_dtype q_dtype, float* d_scale, void* stream) {
  TraceRange trace("kb_quantize_blocks");
  if (!ctx) return KB_ERR_INVALID_ARG;
  const char* where = "kb_quantize_blocks";
  if (!is_float_type(dtype)) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dtype %d is not fp32, fp16 or bf16", where, (int)dtype);
  if (!is_f8_type(q_dtype)) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: q_dtype %d is not an 8-bit float", where, (int)q_dtype);
  if (mode != KB_SCALE_ROWS && mode != KB_SCALE_TILES) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: unknown mode %d", where, (int)mode);
  if (transpose != 0 && transpose != 1) return fail(ctx, KB_ERR_INVALID_ARG, "%s: transpose must be 0 or 1", where);
  if (rows > KB_OPS_MAX_DIM || cols > KB_OPS_MAX_DIM) return fail(ctx, KB_ERR_INVALID_ARG, "%s: rows or columns beyond 2^30", where);
  if (rows == 0 || cols == 0) return KB_OK;
  const int e = elem_bytes(dtype);
  KB_TRY(check_matrix(ctx, where, "d_x", d_x, cols, ldx, e));
  KB_TRY(check_matrix(ctx, where, "d_q", d_q, transpose ? rows : cols, ldq, 1));
  if (!d_scale) return fail(ctx, KB_ERR_INVALID_ARG, "%s: d_scale is NULL", where);
  KB_TRY(check_vector(ctx, where, "d_scale", d_scale, 4));
  DeviceGuard g(ctx->device);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  QuantParams p;
  p.x = d_x;
  p.q = static_cast<unsigned char*>(d_q);
  p.scale = d_scale;
  p.rows = rows;
  p.cols = cols;
  p.ldx = ldx;
  p.ldq = ldq;
  p.groups = (uint32_t)((cols + kGroup - 1) / kGroup);
  p.rtiles = (uint32_t)((rows + 127) / 128);
  p.ctiles = (uint32_t)((cols + 127) / 128);
  p.span = (rows - 1) * ldx + cols;
  p.q_vec = ldq % 8 == 0 && aligned_to(d_q, 8);
  const bool vec = cols % 8 == 0 && rows_aligned(d_x, ldx, e) && (transpose || p.q_vec);
  const bool e5m2 = q_dtype == KB_F8E5M2, tiles = mode == KB_SCALE_TILES;
  if (dtype == KB_F32) return launch_quant<KB_F32>(ctx, p, vec, e5m2, transpose, tiles, st);
  if (dtype == KB_F16) return launch_quant<KB_F16>(ctx, p, vec, e5m2, transpose, tiles, st);
  return launch_quant<KB_BF16>(ctx, p, vec, e5m2, transpose, tiles, st);
}

extern "C" kb_status kb_layernorm(kb_ctx* ctx, const void* d_x, uint64_t rows, uint64_t cols, uint64_t ldx,
                                  kb_dtype dtype, const void* d_weight, const void* d_bias, kb_dtype param_dtype,
                                  float eps, void* d_y, uint64_t ldy, float* d_mean, float* d_rstd, void* d_q,
                                  uint64_t ldq, kb_dtype q_dtype, float* d_scale, void* stream) {
  TraceRange trace("kb_layernorm");
  if (!ctx) return KB_ERR_INVALID_ARG;
  const char* where = "kb_layernorm";
  if (!is_float_type(dtype)) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dtype %d is not fp32, fp16 or bf16", where, (int)dtype);
  if (param_dtype != dtype && param_dtype != KB_F32)
    return fail(ctx, KB_ERR_UNSUPPORTED, "%s: parameters are of the row's type or binary32", where);
  if (!(eps > 0.0f) || !std::isfinite(eps)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: eps must be finite and > 0", where);
  if (cols == 0 || rows > KB_OPS_MAX_DIM || cols > KB_OPS_MAX_DIM)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: columns outside [1, 2^30] or rows beyond 2^30", where);
  if (!d_y && !d_mean && !d_rstd && !d_q) return fail(ctx, KB_ERR_INVALID_ARG, "%s: no output", where);
  if ((d_q == nullptr) != (d_scale == nullptr)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: d_q and d_scale come together", where);
  if (d_q && !is_f8_type(q_dtype)) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: q_dtype %d is not an 8-bit float", where, (int)q_dtype);
  if (rows == 0) return KB_OK;
  const int e = elem_bytes(dtype), pe = elem_bytes(param_dtype);
  KB_TRY(check_matrix(ctx, where, "d_x", d_x, cols, ldx, e));
  if (d_y) KB_TRY(check_matrix(ctx, where, "d_y", d_y, cols, ldy, e));
  if (d_q) KB_TRY(check_matrix(ctx, where, "d_q", d_q, cols, ldq, 1));
  KB_TRY(check_vector(ctx, where, "d_weight", d_weight, pe));
  KB_TRY(check_vector(ctx, where, "d_bias", d_bias, pe));
  KB_TRY(check_vector(ctx, where, "d_mean", d_mean, 4));
  KB_TRY(check_vector(ctx, where, "d_rstd", d_rstd, 4));
  KB_TRY(check_vector(ctx, where, "d_scale", d_scale, 4));
  DeviceGuard g(ctx->device);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  NormParams p;
  p.x = d_x;
  p.weight = d_weight;
  p.bias = d_bias;
  p.y = d_y;
  p.mean = d_mean;
  p.rstd = d_rstd;
  p.q = static_cast<unsigned char*>(d_q);
  p.scale = d_scale;
  p.rows = rows;
  p.ldx = ldx;
  p.ldy = ldy;
  p.ldq = ldq;
  p.cols = (uint32_t)cols;
  p.groups = (uint32_t)((cols + kGroup - 1) / kGroup);
  p.eps = eps;
  p.param_f32 = param_dtype == KB_F32;
  const bool e5m2 = q_dtype == KB_F8E5M2;
  const bool vec = cols % 8 == 0 && rows_aligned(d_x, ldx, e) && (!d_y || rows_aligned(d_y, ldy, e)) &&
                   (!d_q || (ldq % 8 == 0 && aligned_to(d_q, 8))) && aligned16(d_weight) && aligned16(d_bias);
  if (dtype == KB_F32) return launch_norm<KB_F32>(ctx, p, vec, e5m2, st);
  if (dtype == KB_F16) return launch_norm<KB_F16>(ctx, p, vec, e5m2, st);
  return launch_norm<KB_BF16>(ctx, p, vec, e5m2, st);
}

extern "C" kb_status kb_layernorm_backward_reserve(kb_ctx* ctx, uint64_t rows, uint64_t cols, void* stream) {
  TraceRange trace("kb_layernorm_backward_reserve");
  if (!ctx) return KB_ERR_INVALID_ARG;
  if (cols == 0 || rows > KB_OPS_MAX_DIM || cols > KB_OPS_MAX_DIM)
    return fail(ctx, KB_ERR_INVALID_ARG, "kb_layernorm_backward_reserve: columns outside [1, 2^30] or rows beyond 2^30");
  DeviceGuard g(ctx->device);
  const uint64_t parts = norm_bwd_most_partials(ctx, rows, (uint32_t)((cols + kGroup - 1) / kGroup));
  return ensure_partials(ctx, (size_t)parts * 2 * cols * sizeof(float), reinterpret_cast<cudaStream_t>(stream));
}

extern "C" kb_status kb_layernorm_backward(kb_ctx* ctx, const void* d_dy, uint64_t lddy, const void* d_x,
                                           uint64_t ldx, uint64_t rows, uint64_t cols, kb_dtype dtype,
                                           const void* d_weight, kb_dtype param_dtype, const float* d_mean,
                                           const float* d_rstd, void* d_dx, uint64_t lddx, void* d_dweight,
                                           void* d_dbias, void* stream) {
  TraceRange trace("kb_layernorm_backward");
  if (!ctx) return KB_ERR_INVALID_ARG;
  const char* where = "kb_layernorm_backward";
  if (!is_float_type(dtype)) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dtype %d is not fp32, fp16 or bf16", where, (int)dtype);
  if (param_dtype != dtype && param_dtype != KB_F32)
    return fail(ctx, KB_ERR_UNSUPPORTED, "%s: parameters are of the row's type or binary32", where);
  if (cols == 0 || rows > KB_OPS_MAX_DIM || cols > KB_OPS_MAX_DIM)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: columns outside [1, 2^30] or rows beyond 2^30", where);
  if (!d_dx && !d_dweight && !d_dbias) return fail(ctx, KB_ERR_INVALID_ARG, "%s: no output", where);
  const int e = elem_bytes(dtype), pe = elem_bytes(param_dtype);
  KB_TRY(check_vector(ctx, where, "d_weight", d_weight, pe));
  KB_TRY(check_vector(ctx, where, "d_dweight", d_dweight, pe));
  KB_TRY(check_vector(ctx, where, "d_dbias", d_dbias, pe));
  DeviceGuard g(ctx->device);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (d_dweight) KB_CUDA(ctx, cudaMemsetAsync(d_dweight, 0, cols * pe, st));
    if (d_dbias) KB_CUDA(ctx, cudaMemsetAsync(d_dbias, 0, cols * pe, st));
    return KB_OK;
  }
  KB_TRY(check_matrix(ctx, where, "d_dy", d_dy, cols, lddy, e));
  KB_TRY(check_matrix(ctx, where, "d_x", d_x, cols, ldx, e));
  if (d_dx) KB_TRY(check_matrix(ctx, where, "d_dx", d_dx, cols, lddx, e));
  if (!d_mean || !d_rstd) return fail(ctx, KB_ERR_INVALID_ARG, "%s: d_mean or d_rstd is NULL", where);
  KB_TRY(check_vector(ctx, where, "d_mean", d_mean, 4));
  KB_TRY(check_vector(ctx, where, "d_rstd", d_rstd, 4));
  NormBwdParams p;
  p.dy = d_dy;
  p.x = d_x;
  p.weight = d_weight;
  p.mean = d_mean;
  p.rstd = d_rstd;
  p.dx = d_dx;
  p.partial = nullptr;
  p.rows = rows;
  p.lddy = lddy;
  p.ldx = ldx;
  p.lddx = lddx;
  p.cols = (uint32_t)cols;
  p.groups = (uint32_t)((cols + kGroup - 1) / kGroup);
  p.param_f32 = param_dtype == KB_F32;
  p.want_param = d_dweight || d_dbias;
  p.stages = p.slot_bytes = 0;
  p.status = ctx->d_status;
  const bool vec = cols % 8 == 0 && rows_aligned(d_dy, lddy, e) && rows_aligned(d_x, ldx, e) &&
                   (!d_dx || rows_aligned(d_dx, lddx, e)) && aligned16(d_weight);
  uint32_t nparts = 0;
  if (dtype == KB_F32)
    KB_TRY((vec ? launch_norm_bwd<KB_F32, true>(ctx, p, &nparts, st) : launch_norm_bwd<KB_F32, false>(ctx, p, &nparts, st)));
  else if (dtype == KB_F16)
    KB_TRY((vec ? launch_norm_bwd<KB_F16, true>(ctx, p, &nparts, st) : launch_norm_bwd<KB_F16, false>(ctx, p, &nparts, st)));
  else
    KB_TRY((vec ? launch_norm_bwd<KB_BF16, true>(ctx, p, &nparts, st) : launch_norm_bwd<KB_BF16, false>(ctx, p, &nparts, st)));
  if (!p.want_param) return KB_OK;
  const dim3 grid((unsigned int)((cols + 31) / 32), 2);
  if (param_dtype == KB_F32)
    norm_param_kernel<KB_F32><<<grid, 32 * kParamWarps, 0, st>>>(p.partial, nparts, p.cols, d_dweight, d_dbias);
  else if (param_dtype == KB_F16)
    norm_param_kernel<KB_F16><<<grid, 32 * kParamWarps, 0, st>>>(p.partial, nparts, p.cols, d_dweight, d_dbias);
  else
    norm_param_kernel<KB_BF16><<<grid, 32 * kParamWarps, 0, st>>>(p.partial, nparts, p.cols, d_dweight, d_dbias);
  return launched(ctx);
}

extern "C" kb_status kb_matmul_blocks(kb_ctx* ctx, const void* d_a, uint64_t lda, kb_dtype a_dtype,
                                      const float* d_a_scale, const void* d_b, uint64_t ldb, kb_dtype b_dtype,
                                      const float* d_b_scale, kb_scale_mode b_mode, uint64_t M, uint64_t N,
                                      uint64_t K, void* d_d, uint64_t ldd, kb_dtype d_dtype, void* stream) {
  TraceRange trace("kb_matmul_blocks");
  if (!ctx) return KB_ERR_INVALID_ARG;
  const char* where = "kb_matmul_blocks";
  if (!is_f8_type(a_dtype) || !is_f8_type(b_dtype)) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: operands are 8-bit floats", where);
  if (!is_float_type(d_dtype)) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: d_dtype %d is not fp32, fp16 or bf16", where, (int)d_dtype);
  if (b_mode != KB_SCALE_ROWS && b_mode != KB_SCALE_TILES) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: unknown b_mode %d", where, (int)b_mode);
  if (M > KB_OPS_MAX_DIM || N > KB_OPS_MAX_DIM || K > KB_OPS_MAX_DIM)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: a dimension beyond 2^30", where);
  if (M == 0 || N == 0) return KB_OK;
  const int e = elem_bytes(d_dtype);
  KB_TRY(check_matrix(ctx, where, "d_d", d_d, N, ldd, e));
  DeviceGuard g(ctx->device);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (K == 0) {
    KB_CUDA(ctx, cudaMemset2DAsync(d_d, ldd * e, 0, N * e, M, st));
    return KB_OK;
  }
  KB_TRY(check_matrix(ctx, where, "d_a", d_a, K, lda, 1));
  KB_TRY(check_matrix(ctx, where, "d_b", d_b, K, ldb, 1));
  if (!rows_aligned(d_a, lda, 1) || !rows_aligned(d_b, ldb, 1))
    return fail(ctx, KB_ERR_ALIGNMENT, "%s: operands need 16-byte aligned pointers and row strides", where);
  if (!d_a_scale || !d_b_scale) return fail(ctx, KB_ERR_INVALID_ARG, "%s: d_a_scale or d_b_scale is NULL", where);
  KB_TRY(check_vector(ctx, where, "d_a_scale", d_a_scale, 4));
  KB_TRY(check_vector(ctx, where, "d_b_scale", d_b_scale, 4));
  KB_TRY(prepare_matmul(ctx));
  MatmulParams p;
  p.a_scale = d_a_scale;
  p.b_scale = d_b_scale;
  p.d = d_d;
  p.ldd = ldd;
  p.M = (uint32_t)M;
  p.N = (uint32_t)N;
  p.KB = (uint32_t)((K + KB_BLOCK - 1) / KB_BLOCK);
  p.b_scale_shift = b_mode == KB_SCALE_TILES ? 7 : 0;
  p.b_scale_ld = b_mode == KB_SCALE_TILES ? (p.N + 127) / 128 : p.N;
  p.a = static_cast<const unsigned char*>(d_a);
  p.b = static_cast<const unsigned char*>(d_b);
  p.lda = lda;
  p.ldb = ldb;
  p.K = (uint32_t)K;
  p.a_e5m2 = a_dtype == KB_F8E5M2;
  p.b_e5m2 = b_dtype == KB_F8E5M2;
  p.out = (int)d_dtype;
  p.status = ctx->d_status;
  p.vec_out = rows_aligned(d_d, ldd, e);
  const bool ae = a_dtype == KB_F8E5M2, be = b_dtype == KB_F8E5M2;
  if (M <= 16) return launch_lanes<16>(ctx, p, d_a, lda, ae, d_b, ldb, be, K, st);
  if (M <= 32) return launch_lanes<32>(ctx, p, d_a, lda, ae, d_b, ldb, be, K, st);
  if (M <= 64) return launch_lanes<64>(ctx, p, d_a, lda, ae, d_b, ldb, be, K, st);
  if (!lanes_are_faster(ctx, M, N, p.KB)) return launch_pair(ctx, p, d_a, lda, ae, d_b, ldb, be, K, st);
  return launch_lanes<128>(ctx, p, d_a, lda, ae, d_b, ldb, be, K, st);
}
