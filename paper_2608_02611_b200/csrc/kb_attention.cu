// Host side of the attention operators: argument checks, choice of kernel, launch.
// Declarations and their contracts are in include/kb_attention.h.
#include <algorithm>
#include <cmath>
#include <tuple>

#include "../../include/kb_attention.h"
#include "kb_ctx.cuh"
#include "kb_paged.cuh"
#include "kb_prompt.cuh"
#include "kb_rope.cuh"

using namespace kb;

namespace {

constexpr uint64_t kMaxStride = 1ull << 40;   // elements
constexpr double kLog2e = 1.4426950408889634;

// Heads of a batch, [tokens][heads][dim]: not null, element-aligned, strides that an address can hold.
struct Heads {
  const char* name;
  const void* p;
  uint64_t row, head;
};
kb_status check_heads(kb_ctx* ctx, const char* where, const Heads& t, int bytes) {
  if (!t.p) return fail(ctx, KB_ERR_INVALID_ARG, "%s: %s is NULL", where, t.name);
  if (!aligned_to(t.p, bytes)) return fail(ctx, KB_ERR_ALIGNMENT, "%s: %s is not aligned to its element type", where, t.name);
  if (t.row > kMaxStride || t.head > kMaxStride)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: a stride of %s is beyond 2^40 elements", where, t.name);
  return KB_OK;
}
// No two rows of dim elements are one where axes of these lengths and strides lie within each other, in whatever order
struct Axis {
  uint64_t n, stride;
};
template <size_t N>
bool rows_apart(Axis (&axes)[N], uint64_t dim) {
  std::sort(axes, axes + N, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  unsigned __int128 extent = dim;
  for (const Axis& a : axes) {
    if (a.n <= 1) continue;
    if (a.stride < extent) return false;
    extent += (unsigned __int128)(a.n - 1) * a.stride;
  }
  return true;
}
// The same for an output, no two elements of which may be one
kb_status check_out(kb_ctx* ctx, const char* where, const Heads& t, uint64_t tokens, uint64_t heads, uint64_t dim, int bytes) {
  KB_TRY(check_heads(ctx, where, t, bytes));
  Axis axes[2] = {{tokens, t.row}, {heads, t.head}};
  if (!rows_apart(axes, dim)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: the strides of %s let its rows overlap", where, t.name);
  return KB_OK;
}
// Rows start on 16-byte boundaries
bool heads_aligned(const void* p, uint64_t row, uint64_t head, int bytes) {
  return aligned16(p) && (row * bytes) % 16 == 0 && (head * bytes) % 16 == 0;
}
// The stride of an axis of one element is free: one that suits the copies instead
void settle(Heads& t, uint64_t tokens, uint64_t heads, uint32_t dim) {
  if (heads <= 1) t.head = round_up(dim, 8);
  if (tokens <= 1) t.row = std::max<uint64_t>(1, heads) * round_up(std::max<uint64_t>(t.head, dim), 8);
}
// Number of heads and dim, as every call has them
kb_status check_sizes(kb_ctx* ctx, const char* where, uint32_t q_heads, uint32_t kv_heads, uint32_t dim, uint32_t most) {
  if (dim == 0 || dim > most) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dim %u is not within 1 .. %u", where, dim, most);
  if (q_heads == 0 || kv_heads == 0 || q_heads > 65536 || q_heads % kv_heads != 0)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: %u query heads are not a multiple (up to 65536) of %u key heads", where, q_heads, kv_heads);
  return KB_OK;
}
kb_status check_cache(kb_ctx* ctx, const char* where, const kb_paged_cache& c, int bytes) {
  KB_TRY(check_heads(ctx, where, {"the cache's keys", c.d_k, c.k_row, c.k_head}, bytes));
  KB_TRY(check_heads(ctx, where, {"the cache's values", c.d_v, c.v_row, c.v_head}, bytes));
  if (c.k_page > kMaxStride || c.v_page > kMaxStride)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: a stride of the cache's pages is beyond 2^40 elements", where);
  if (c.page_size == 0 || c.pages > 0x7FFFFFFFull / c.page_size)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: a cache of %llu pages of %u slots (1 .. 2^31 - 1 slots in all)", where,
                (unsigned long long)c.pages, c.page_size);
  return KB_OK;
}

// ---- norms and rotation ------------------------------------------------------------------------

template <int DT, int L>
kb_status launch_rope(kb_ctx* ctx, const RopeParams& p, bool vec, cudaStream_t st) {
  // as many tokens per CTA as leave three CTAs for each SM; with fewer, the heads of a token are shared out as well
  const uint64_t fill = 3ull * ctx->sm_count;
  const uint32_t per = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(kRopeTokens, p.tokens / fill));
  const uint64_t grid = (p.tokens + per - 1) / per;
  const uint64_t turns = ((p.hq + 2ull * p.hkv) * L + kRopeThreads - 1) / kRopeThreads;   // of a CTA's warps through a token
  if (vec)
    return launch_dependent(ctx, qk_norm_rope_kernel<DT, L>, dim3((unsigned int)grid, (unsigned int)std::min<uint64_t>(turns, (fill + grid - 1) / grid)),
                            kRopeThreads, 0, st, p, per);
  return launch_dependent(ctx, qk_norm_rope_plain_kernel<DT, L>, dim3((unsigned int)grid), kRopeThreads, 0, st, p, per);
}
template <int DT>
kb_status launch_rope(kb_ctx* ctx, const RopeParams& p, bool vec, cudaStream_t st) {
  if (p.dim <= 64) return launch_rope<DT, 8>(ctx, p, vec, st);
  if (p.dim <= 128) return launch_rope<DT, 16>(ctx, p, vec, st);
  return launch_rope<DT, 32>(ctx, p, vec, st);
}

// ---- paged attention ---------------------------------------------------------------------------

constexpr uint32_t kPagedMostHeads = 16, kPagedMostDim = 128;

struct PagedSpace {
  size_t part, rl, arrived, bytes;
  explicit PagedSpace(const kb_ctx* ctx) {
    const size_t slots = 2ull * 2 * ctx->sm_count * kPagedWaves;   // two per CTA, of two per SM
    part = 0;
    rl = slots * kPagedMostHeads * kPagedMostDim * sizeof(float);
    arrived = rl + slots * kPagedMostHeads * 2 * sizeof(float);
    bytes = arrived + slots * sizeof(unsigned int);
  }
};
kb_status ensure_paged(kb_ctx* ctx, cudaStream_t st) {
  ctx->captured |= is_capturing(st);
  const PagedSpace space(ctx);
  if (ctx->paged_ws_bytes >= space.bytes) return KB_OK;
  KB_TRY(ensure_workspace(ctx, &ctx->paged_ws, &ctx->paged_ws_bytes, space.bytes, st, "parts of divided sequences"));
  const cudaError_t e = cudaMemset(ctx->paged_ws + space.arrived, 0, space.bytes - space.arrived);
  if (e != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess) {
    ctx_free(ctx, ctx->paged_ws);
    ctx->paged_ws = nullptr;
    ctx->paged_ws_bytes = 0;
    return fail(ctx, KB_ERR_CUDA, "the workspace of paged attention could not be zeroed");
  }
  return KB_OK;
}

// Pieces of the row of units, each of which takes a CTA per group of heads: as many as run at the same time; or,
// where that would leave more than a tenth of the card idle (32 groups: 4 x 32 of 148 SMs), the
// number that fills up to kPagedWaves waves best.
uint32_t paged_pieces(uint64_t resident, uint64_t per_seq, uint64_t most_units) {
  auto use = [&](uint64_t n) { return (double)(n * per_seq) / (double)((n * per_seq + resident - 1) / resident * resident); };
  uint64_t best = std::max<uint64_t>(1, resident / per_seq);
  if (use(best) < 0.9)
    for (uint64_t n = best + 1; n * per_seq <= kPagedWaves * resident; ++n)
      if (use(n) > use(best)) best = n;
  return (uint32_t)std::min(best, most_units);
}

template <int DT, int DP>
kb_status prepare_paged(kb_ctx* ctx) {   // one fixed size each, whatever thread or context calls
  auto raise = [&](auto kernel, uint32_t smem) {
    KB_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    return KB_OK;
  };
  KB_TRY(raise(attention_paged_kernel<DT, DP, 1, 8>, PagedTile<DP, 1, 8>::kSmem));
  KB_TRY(raise(attention_paged_kernel<DT, DP, 2, 8>, PagedTile<DP, 2, 8>::kSmem));
  KB_TRY(raise(attention_paged_kernel<DT, DP, 1, 4>, PagedTile<DP, 1, 4>::kSmem));
  return raise(attention_paged_kernel<DT, DP, 2, 4>, PagedTile<DP, 2, 4>::kSmem);
}
kb_status prepare_paged(kb_ctx* ctx) {
  if (ctx->paged_ready) return KB_OK;
  KB_TRY(find_encoder(ctx, "kb_attention_paged"));
  KB_TRY((prepare_paged<KB_F16, 64>(ctx)));
  KB_TRY((prepare_paged<KB_F16, 128>(ctx)));
  KB_TRY((prepare_paged<KB_BF16, 64>(ctx)));
  KB_TRY((prepare_paged<KB_BF16, 128>(ctx)));
  ctx->paged_ready = true;
  return KB_OK;
}
// Tensor map of a cache [pages][page size][heads][dim], as elements of a head, keys of a page, pieces of a head (of 64 elements, or
// one of all), heads, pages; boxes of 64 elements, `box_rows` keys and all pieces.
kb_status encode_cache(kb_ctx* ctx, CUtensorMap* map, const void* d, uint64_t page, uint64_t row, uint64_t head, const kb_paged_cache& c,
                       uint32_t heads, uint32_t dim, kb_dtype dtype, uint32_t box_rows, uint32_t pieces) {
  const uint64_t any = round_up(dim, 8);   // the stride of an axis of one element is free
  const cuuint64_t dims[5] = {dim / pieces, c.page_size, pieces, heads, std::max<uint64_t>(c.pages, 1)};
  const cuuint64_t strides[4] = {(c.page_size > 1 ? row : any) * 2, 128, (heads > 1 ? head : any) * 2, (c.pages > 1 ? page : any) * 2};
  const cuuint32_t box[5] = {64, box_rows, pieces, 1, 1}, step[5] = {1, 1, 1, 1, 1};
  const CUresult rc = reinterpret_cast<EncodeTiled>(ctx->encode_tiled)(
      map, dtype == KB_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(d), dims, strides,
      box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (rc != CUDA_SUCCESS) return fail(ctx, KB_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d for a cache", (int)rc);
  return KB_OK;
}

template <int DT, int DP, int NT, int W>
kb_status launch_paged(kb_ctx* ctx, const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p, cudaStream_t st) {
  using T = PagedTile<DP, NT, W>;
  const uint64_t most_units = (uint64_t)paged_units(paged_length(0x7FFFFFFF, p.max_pages, p.page_size), 16 * W) * p.sequences;
  if (most_units > 0x7FFFFFFFull) return fail(ctx, KB_ERR_UNSUPPORTED, "kb_attention_paged: sequences * max_pages * page_size is beyond 2^36");
  const uint32_t per_seq = p.hkv * p.chunks, pieces = paged_pieces((uint64_t)ctx->sm_count * T::kPerSm, per_seq, most_units);
  return launch_dependent(ctx, attention_paged_kernel<DT, DP, NT, W>, dim3(per_seq, pieces), T::kThreads, T::kSmem, st, k, v, p);
}
// Four warps and two CTAs per SM instead of eight and one where there are enough sequences to fill the card: what a CTA does
// between two sequences then hides under its neighbour's copies (of 8 heads: 256 x 200 keys 55 us, with eight warps 72; 128 x 200 31 and
// 38.5; 32 x 200 9.4 and 11.3; 64 sequences of 1 to 16384 keys 78.5 and 85).  For fewer the parts would be more and a
// CTA's share of a long sequence later (one of 8192 keys 18.7 us and 16.5; 7 of up to 3001 keys 22.4 and 16.8; 16 x 200 9.9 and 7.5, 18 x 1000
// 16.5 and 14.6).  Not everything past the border gains: 20 x 200 13.7 us and 12.3, 128 x 1000 93 and 88, 128 x 4096 337 and 331.
bool paged_in_fours(const kb_ctx* ctx, const PagedParams& p) {
  return (uint64_t)p.sequences * p.hkv * p.chunks >= (uint64_t)ctx->sm_count;
}
template <int DT, int DP, int NT>
kb_status launch_paged(kb_ctx* ctx, const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p, cudaStream_t st) {
  return paged_in_fours(ctx, p) ? launch_paged<DT, DP, NT, 4>(ctx, k, v, p, st) : launch_paged<DT, DP, NT, 8>(ctx, k, v, p, st);
}
template <int DT>
kb_status launch_paged(kb_ctx* ctx, const CUtensorMap& k, const CUtensorMap& v, const PagedParams& p, cudaStream_t st) {
  if (p.dim > 64) return p.group > 8 ? launch_paged<DT, 128, 2>(ctx, k, v, p, st) : launch_paged<DT, 128, 1>(ctx, k, v, p, st);
  return p.group > 8 ? launch_paged<DT, 64, 2>(ctx, k, v, p, st) : launch_paged<DT, 64, 1>(ctx, k, v, p, st);
}

// ---- attention over prompts ----------------------------------------------------------------------

// Tensor map of heads [tokens][heads][dim], boxes of 64 elements of dim and `rows` tokens of a head in the 128-byte
// swizzle; places outside the tensor read as zero.
kb_status encode_heads(kb_ctx* ctx, CUtensorMap* map, const Heads& t, uint64_t tokens, uint32_t heads, uint32_t dim, kb_dtype dtype,
                       uint32_t rows) {
  const cuuint64_t dims[3] = {dim, tokens, heads}, strides[2] = {t.row * 2, t.head * 2};
  const cuuint32_t box[3] = {64, rows, 1}, step[3] = {1, 1, 1};
  const CUresult rc = reinterpret_cast<EncodeTiled>(ctx->encode_tiled)(
      map, dtype == KB_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(t.p), dims, strides,
      box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (rc != CUDA_SUCCESS) return fail(ctx, KB_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d for %s", (int)rc, t.name);
  return KB_OK;
}

template <int DT, int DP>
kb_status prepare_prompt(kb_ctx* ctx) {
  constexpr auto kernel = attention_kernel<DT, DP>;
  KB_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PromptTile<DP>::kSmem));
  // the warpgroups split the registers that the kernel is launched with; with fewer they would wait for the rest for good
  cudaFuncAttributes attr = {};
  KB_CUDA(ctx, cudaFuncGetAttributes(&attr, kernel));
  if (attr.numRegs < PromptTile<DP>::kRegsLaunch)
    return fail(ctx, KB_ERR_UNSUPPORTED, "kb_attention: the library was compiled with %d registers for a kernel that splits %d",
                attr.numRegs, PromptTile<DP>::kRegsLaunch);
  return KB_OK;
}
kb_status prepare_prompt(kb_ctx* ctx) {
  if (ctx->attention_ready) return KB_OK;
  KB_TRY(find_encoder(ctx, "kb_attention"));
  KB_TRY((prepare_prompt<KB_F16, 64>(ctx)));
  KB_TRY((prepare_prompt<KB_F16, 128>(ctx)));
  KB_TRY((prepare_prompt<KB_BF16, 64>(ctx)));
  KB_TRY((prepare_prompt<KB_BF16, 128>(ctx)));
  ctx->attention_ready = true;
  return KB_OK;
}
// Keys of a phase (prompt_phases).  Items in the order of their lengths alone, whatever their sequence, keep the card even to the
// end, but go through all keys and values once per length: past the second-level cache (126 MB, whose halves both hold
// what both halves of the card read) those come from memory each time.  8 x 2048 tokens of 32 heads read 1309 MB then, in phases
// of 32 MB 455 MB (327 us and 317; 8 x 4096 of 32 heads on 8: 1043 and 985; 8 x 2048 on 16, 134 MB: 312 to 318 and 319 to 353, 16 x 1024 of 32 heads 245
// and 243).  Up to 64 MB they stay there as it is (13 sequences with 43 MB: 272 us, in phases 259 to 268).  By the tensors' sizes, like the tiles.
uint32_t prompt_phase_keys(uint64_t keys, uint64_t kv_heads, uint64_t dim) {
  const uint64_t bytes = 2 * 2 * kv_heads * dim;   // of a key and its value
  return keys * bytes <= (64u << 20) ? 0u : (uint32_t)std::max<uint64_t>(1, (32u << 20) / bytes);
}
template <int DT, int DP>
kb_status launch_prompt(kb_ctx* ctx, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const PromptParams& p,
                        unsigned int grid, cudaStream_t st) {
  return launch_dependent(ctx, attention_kernel<DT, DP>, dim3(grid), PromptTile<DP>::kThreads, PromptTile<DP>::kSmem, st, q, k, v, p);
}

}  // namespace

// ---------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------

extern "C" kb_status kb_qk_norm_rope(kb_ctx* ctx, const void* d_q, uint64_t q_row, uint64_t q_head, uint32_t q_heads,
                                     const void* d_k, uint64_t k_row, uint64_t k_head, uint32_t kv_heads,
                                     uint64_t tokens, uint32_t dim, kb_dtype dtype, int norm, const void* d_q_weight,
                                     const void* d_k_weight, kb_dtype param_dtype, float eps,
                                     const int64_t* d_positions, const double* d_inv_freq, uint32_t rotary_dim,
                                     int interleaved, void* d_q_out, uint64_t q_out_row, uint64_t q_out_head,
                                     void* d_k_out, uint64_t k_out_row, uint64_t k_out_head, const void* d_v,
                                     uint64_t v_row, uint64_t v_head, const kb_paged_cache* cache,
                                     const int64_t* d_slots, void* stream) {
  TraceRange trace("kb_qk_norm_rope");
  if (!ctx) return KB_ERR_INVALID_ARG;
  const char* where = "kb_qk_norm_rope";
  if (!is_float_type(dtype)) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dtype %d is not fp32, fp16 or bf16", where, (int)dtype);
  if (param_dtype != dtype && param_dtype != KB_F32)
    return fail(ctx, KB_ERR_UNSUPPORTED, "%s: weights are of the heads' type or binary32", where);
  KB_TRY(check_sizes(ctx, where, q_heads, kv_heads, dim, KB_ROPE_MAX_DIM));
  if ((norm != 0 && norm != 1) || (interleaved != 0 && interleaved != 1))
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: norm and interleaved must be 0 or 1", where);
  if (norm && (!(eps > 0.0f) || !std::isfinite(eps))) return fail(ctx, KB_ERR_INVALID_ARG, "%s: eps must be finite and > 0", where);
  if (!norm && (d_q_weight || d_k_weight)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: weights without the norm", where);
  if (rotary_dim > dim || rotary_dim % 2 != 0)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: rotary_dim %u is odd or more than dim %u", where, rotary_dim, dim);
  if (tokens > KB_OPS_MAX_DIM) return fail(ctx, KB_ERR_INVALID_ARG, "%s: more than 2^30 tokens", where);
  if (!d_q_out && !d_k_out && !cache && tokens) return fail(ctx, KB_ERR_INVALID_ARG, "%s: no output", where);
  if (tokens == 0) return KB_OK;
  const int e = elem_bytes(dtype), pe = elem_bytes(param_dtype);
  if (d_q_out) {
    KB_TRY(check_heads(ctx, where, {"d_q", d_q, q_row, q_head}, e));
    KB_TRY(check_out(ctx, where, {"d_q_out", d_q_out, q_out_row, q_out_head}, tokens, q_heads, dim, e));
  }
  if (d_k_out || cache) KB_TRY(check_heads(ctx, where, {"d_k", d_k, k_row, k_head}, e));
  if (d_k_out) KB_TRY(check_out(ctx, where, {"d_k_out", d_k_out, k_out_row, k_out_head}, tokens, kv_heads, dim, e));
  // in place means the very same rows: others would be written while they are still to be read
  if (d_q_out && d_q_out == d_q && (q_out_row != q_row || q_out_head != q_head))
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: d_q_out is d_q with other strides", where);
  if (d_k_out && d_k_out == d_k && (k_out_row != k_row || k_out_head != k_head))
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: d_k_out is d_k with other strides", where);
  if (cache) {
    KB_TRY(check_heads(ctx, where, {"d_v", d_v, v_row, v_head}, e));
    KB_TRY(check_cache(ctx, where, *cache, e));
    Axis k_axes[3] = {{cache->pages, cache->k_page}, {cache->page_size, cache->k_row}, {kv_heads, cache->k_head}};
    Axis v_axes[3] = {{cache->pages, cache->v_page}, {cache->page_size, cache->v_row}, {kv_heads, cache->v_head}};
    if (!rows_apart(k_axes, dim) || !rows_apart(v_axes, dim)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: the strides of the cache let its slots overlap", where);
    if (!d_slots) return fail(ctx, KB_ERR_INVALID_ARG, "%s: a cache without d_slots", where);
    if (!aligned_to(d_slots, 8)) return fail(ctx, KB_ERR_ALIGNMENT, "%s: d_slots is not aligned to its element type", where);
  }
  if (!aligned_to(d_q_weight, pe) || !aligned_to(d_k_weight, pe))
    return fail(ctx, KB_ERR_ALIGNMENT, "%s: a weight is not aligned to its element type", where);
  if (rotary_dim && (!d_positions || !d_inv_freq)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: d_positions or d_inv_freq is NULL", where);
  if (!aligned_to(d_positions, 8) || !aligned_to(d_inv_freq, 8))
    return fail(ctx, KB_ERR_ALIGNMENT, "%s: d_positions or d_inv_freq is not aligned to its element type", where);
  DeviceGuard g(ctx->device);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  RopeParams p = {};
  p.q = d_q;
  p.q_row = q_row;
  p.q_head = q_head;
  p.k = d_k;
  p.k_row = k_row;
  p.k_head = k_head;
  p.v = d_v;
  p.v_row = v_row;
  p.v_head = v_head;
  p.q_out = d_q_out;
  p.qo_row = q_out_row;
  p.qo_head = q_out_head;
  p.k_out = d_k_out;
  p.ko_row = k_out_row;
  p.ko_head = k_out_head;
  if (cache) {
    p.k_cache = cache->d_k;
    p.v_cache = cache->d_v;
    p.kc_page = cache->k_page;
    p.kc_row = cache->k_row;
    p.kc_head = cache->k_head;
    p.vc_page = cache->v_page;
    p.vc_row = cache->v_row;
    p.vc_head = cache->v_head;
    p.slots_end = cache->pages * cache->page_size;
    p.page_size = cache->page_size;
    p.slots = reinterpret_cast<const long long*>(d_slots);
  }
  p.positions = reinterpret_cast<const long long*>(d_positions);
  p.inv_freq = d_inv_freq;
  p.q_weight = d_q_weight;
  p.k_weight = d_k_weight;
  p.param_f32 = param_dtype == KB_F32;
  p.norm = norm;
  p.interleaved = interleaved;
  p.eps = eps;
  p.tokens = tokens;
  p.hq = q_heads;
  p.hkv = kv_heads;
  p.dim = dim;
  p.half = rotary_dim / 2;
  p.status = ctx->d_status;
  const bool vec = dim % 8 == 0 && (interleaved || p.half % 4 == 0) && (!d_q_out || (heads_aligned(d_q, q_row, q_head, e) && heads_aligned(d_q_out, q_out_row, q_out_head, e))) &&
                   (!(d_k_out || cache) || heads_aligned(d_k, k_row, k_head, e)) && (!d_k_out || heads_aligned(d_k_out, k_out_row, k_out_head, e)) &&
                   (!cache || (heads_aligned(d_v, v_row, v_head, e) && heads_aligned(cache->d_k, cache->k_row, cache->k_head, e) &&
                               heads_aligned(cache->d_v, cache->v_row, cache->v_head, e) && (cache->k_page * e) % 16 == 0 && (cache->v_page * e) % 16 == 0));
  if (dtype == KB_F32) return launch_rope<KB_F32>(ctx, p, vec, st);
  if (dtype == KB_F16) return launch_rope<KB_F16>(ctx, p, vec, st);
  return launch_rope<KB_BF16>(ctx, p, vec, st);
}

extern "C" kb_status kb_attention(kb_ctx* ctx, const void* d_q, uint64_t q_row, uint64_t q_head, uint32_t q_heads,
                                  uint64_t q_tokens, const void* d_k, uint64_t k_row, uint64_t k_head, const void* d_v,
                                  uint64_t v_row, uint64_t v_head, uint32_t kv_heads, uint64_t k_tokens, uint32_t dim,
                                  kb_dtype dtype, const int32_t* d_q_offsets, const int32_t* d_k_offsets,
                                  uint32_t sequences, int causal, float scale, void* d_out, uint64_t out_row,
                                  uint64_t out_head, float* d_lse, void* stream) {
  TraceRange trace("kb_attention");
  if (!ctx) return KB_ERR_INVALID_ARG;
  const char* where = "kb_attention";
  if (dtype != KB_F16 && dtype != KB_BF16) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dtype %d is not fp16 or bf16", where, (int)dtype);
  KB_TRY(check_sizes(ctx, where, q_heads, kv_heads, dim, KB_ATTENTION_MAX_DIM));
  if (dim % 8 != 0) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dim %u is not a multiple of 8", where, dim);
  if (causal != 0 && causal != 1) return fail(ctx, KB_ERR_INVALID_ARG, "%s: causal must be 0 or 1", where);
  const float scale_log2 = (float)(scale * kLog2e);
  if (!(scale > 0.0f) || !std::isfinite(scale_log2)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: scale must be > 0 and at most 2^127", where);
  if (q_tokens > KB_OPS_MAX_DIM || k_tokens > KB_OPS_MAX_DIM || sequences > kPromptMostSequences)
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: tokens beyond 2^30, or sequences beyond 2^24", where);
  if (!d_k_offsets && k_tokens > kPromptMostKeys) return fail(ctx, KB_ERR_INVALID_ARG, "%s: a sequence of more than 2^24 keys", where);
  if ((d_q_offsets == nullptr) != (d_k_offsets == nullptr) || (!d_q_offsets && sequences != 1))
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: offsets of queries and keys come together, and without them there is one sequence", where);
  if (q_tokens == 0 || sequences == 0) return KB_OK;
  Heads q{"d_q", d_q, q_row, q_head}, k{"d_k", d_k, k_row, k_head}, v{"d_v", d_v, v_row, v_head};
  KB_TRY(check_heads(ctx, where, q, 2));
  KB_TRY(check_out(ctx, where, {"d_out", d_out, out_row, out_head}, q_tokens, q_heads, dim, 2));
  if (k_tokens) {
    KB_TRY(check_heads(ctx, where, k, 2));
    KB_TRY(check_heads(ctx, where, v, 2));
  } else {   // no key anywhere: the copies that are never made still want an address
    k.p = v.p = d_q;
    k.head = v.head = 8;
  }
  settle(q, q_tokens, q_heads, dim);
  settle(k, k_tokens, kv_heads, dim);
  settle(v, k_tokens, kv_heads, dim);
  for (const Heads& t : {q, k, v}) {
    if (!heads_aligned(t.p, t.row, t.head, 2)) return fail(ctx, KB_ERR_ALIGNMENT, "%s: %s needs 16-byte aligned pointers and strides", where, t.name);
    if (t.row == 0 || t.head == 0 || t.row >= kMaxStride / 2 || t.head >= kMaxStride / 2)
      return fail(ctx, KB_ERR_INVALID_ARG, "%s: a stride of %s is 0 or beyond 2^39 elements", where, t.name);
  }
  if (!aligned_to(d_q_offsets, 4) || !aligned_to(d_k_offsets, 4) || !aligned_to(d_lse, 4))
    return fail(ctx, KB_ERR_ALIGNMENT, "%s: offsets or d_lse are not aligned to their element type", where);
  DeviceGuard g(ctx->device);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  KB_TRY(prepare_prompt(ctx));
  CUtensorMap map_q, map_k, map_v;
  KB_TRY(encode_heads(ctx, &map_q, q, q_tokens, q_heads, dim, dtype, 128));
  KB_TRY(encode_heads(ctx, &map_k, k, std::max<uint64_t>(k_tokens, 1), kv_heads, dim, dtype, kPromptKeys));
  KB_TRY(encode_heads(ctx, &map_v, v, std::max<uint64_t>(k_tokens, 1), kv_heads, dim, dtype, kPromptKeys));
  PromptParams p = {};
  p.q_offsets = d_q_offsets;
  p.k_offsets = d_k_offsets;
  p.sequences = sequences;
  p.q_tokens = (uint32_t)q_tokens;
  p.k_tokens = (uint32_t)k_tokens;
  p.hq = q_heads;
  p.group = q_heads / kv_heads;
  p.dim = dim;
  p.pair = p.group % 2 == 0;
  p.causal = causal;
  p.vec_out = aligned16(d_out) && out_row % 8 == 0 && out_head % 8 == 0;
  p.phase_keys = prompt_phase_keys(k_tokens, kv_heads, dim);
  p.scale_log2 = scale_log2;
  p.v = v.p;
  p.v_row = v.row;
  p.v_head = v.head;
  p.out = d_out;
  p.o_row = out_row;
  p.o_head = out_head;
  p.lse = d_lse;
  p.status = ctx->d_status;
  p.next = ctx->d_status + 40;
  // the lengths are the device's: room for every sequence's last, partial piece
  auto items = [&](uint64_t rows, uint64_t units) { return (d_q_offsets ? q_tokens / rows + sequences : (q_tokens + rows - 1) / rows) * units; };
  uint64_t grid = p.pair ? items(128, q_heads / 2) : items(256, q_heads);
  p.second = p.pair ? 0 : 128;
  // Fewer items than SMs: one tile each, whose steps are shorter with nobody beside them (1000 tokens of 32 heads on 8 25 us, in
  // twos 30; 1152, 144 items, 28 and 30; 128 behind 8192 cached ones 97 and 131; 4096 of 8 heads on 2 54 and 72); with more, two tiles keep the
  // tensor cores busier (1280 tokens, 160 items: 32 us, one by one 45; 1500 40 and 51).  By the tensors' sizes, of which lengths on the device may use less.
  if (grid <= (uint64_t)ctx->sm_count) {
    p.pair = false;
    p.second = kPromptNoSecond;
    grid = items(128, q_heads);
  }
  if (grid > 0x7FFFFFFFull) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 tiles", where);
  const unsigned int n = (unsigned int)std::min<uint64_t>(grid, ctx->sm_count);
  if (dim <= 64)
    return dtype == KB_F16 ? launch_prompt<KB_F16, 64>(ctx, map_q, map_k, map_v, p, n, st) : launch_prompt<KB_BF16, 64>(ctx, map_q, map_k, map_v, p, n, st);
  return dtype == KB_F16 ? launch_prompt<KB_F16, 128>(ctx, map_q, map_k, map_v, p, n, st) : launch_prompt<KB_BF16, 128>(ctx, map_q, map_k, map_v, p, n, st);
}

extern "C" kb_status kb_attention_paged_reserve(kb_ctx* ctx, void* stream) {
  TraceRange trace("kb_attention_paged_reserve");
  if (!ctx) return KB_ERR_INVALID_ARG;
  DeviceGuard g(ctx->device);
  KB_TRY(prepare_paged(ctx));
  return ensure_paged(ctx, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" kb_status kb_attention_paged(kb_ctx* ctx, const void* d_q, uint64_t q_row, uint64_t q_head, uint32_t q_heads,
                                        const kb_paged_cache* cache, uint32_t kv_heads, uint32_t dim, kb_dtype dtype,
                                        const int32_t* d_table, uint64_t table_row, uint32_t max_pages,
                                        const int32_t* d_lengths, uint32_t sequences, float scale, void* d_out,
                                        uint64_t out_row, uint64_t out_head, float* d_lse, void* stream) {
  TraceRange trace("kb_attention_paged");
  if (!ctx) return KB_ERR_INVALID_ARG;
  const char* where = "kb_attention_paged";
  if (dtype != KB_F16 && dtype != KB_BF16) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dtype %d is not fp16 or bf16", where, (int)dtype);
  KB_TRY(check_sizes(ctx, where, q_heads, kv_heads, dim, KB_ATTENTION_MAX_DIM));
  if (dim % 8 != 0) return fail(ctx, KB_ERR_UNSUPPORTED, "%s: dim %u is not a multiple of 8", where, dim);
  const float scale_log2 = (float)(scale * kLog2e);
  if (!(scale > 0.0f) || !std::isfinite(scale_log2)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: scale must be > 0 and at most 2^127", where);
  if (sequences > KB_OPS_MAX_DIM) return fail(ctx, KB_ERR_INVALID_ARG, "%s: more than 2^30 sequences", where);
  if (!cache) return fail(ctx, KB_ERR_INVALID_ARG, "%s: cache is NULL", where);
  if (sequences == 0) return KB_OK;
  Heads q{"d_q", d_q, q_row, q_head};
  KB_TRY(check_heads(ctx, where, q, 2));
  KB_TRY(check_out(ctx, where, {"d_out", d_out, out_row, out_head}, sequences, q_heads, dim, 2));
  KB_TRY(check_cache(ctx, where, *cache, 2));
  settle(q, sequences, q_heads, dim);
  if (!heads_aligned(q.p, q.row, q.head, 2) || !heads_aligned(cache->d_k, cache->k_row, cache->k_head, 2) || cache->k_page % 8 != 0 ||
      !heads_aligned(cache->d_v, cache->v_row, cache->v_head, 2) || cache->v_page % 8 != 0)
    return fail(ctx, KB_ERR_ALIGNMENT, "%s: queries and cache need 16-byte aligned pointers and strides", where);
  for (const auto& [n, a, b] : {std::tuple<uint64_t, uint64_t, uint64_t>{kv_heads, cache->k_head, cache->v_head}, {cache->page_size, cache->k_row, cache->v_row},
                                {cache->pages, cache->k_page, cache->v_page}})
    if (n > 1 && (a == 0 || b == 0 || a >= kMaxStride / 2 || b >= kMaxStride / 2))
      return fail(ctx, KB_ERR_INVALID_ARG, "%s: a stride of the cache is 0 or beyond 2^39 elements", where);
  if (!d_lengths || (!d_table && max_pages)) return fail(ctx, KB_ERR_INVALID_ARG, "%s: d_table or d_lengths is NULL", where);
  if (!aligned_to(d_table, 4) || !aligned_to(d_lengths, 4) || !aligned_to(d_lse, 4))
    return fail(ctx, KB_ERR_ALIGNMENT, "%s: d_table, d_lengths or d_lse is not aligned to its element type", where);
  if (sequences > 1 && (table_row < max_pages || table_row > kMaxStride))
    return fail(ctx, KB_ERR_INVALID_ARG, "%s: table_row %llu is less than max_pages %u, or beyond 2^40", where, (unsigned long long)table_row, max_pages);
  if ((uint64_t)max_pages * cache->page_size > 0x7FFFFFFFull) return fail(ctx, KB_ERR_INVALID_ARG, "%s: max_pages * page_size is beyond 2^31 - 1", where);
  DeviceGuard g(ctx->device);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  KB_TRY(prepare_paged(ctx));
  KB_TRY(ensure_paged(ctx, st));
  const PagedSpace space(ctx);
  PagedParams p = {};
  p.q = q.p;
  p.q_row = q.row;
  p.q_head = q.head;
  p.pages = cache->pages;
  p.page_size = cache->page_size;
  p.page_shift = 32;
  for (uint32_t i = 0; i < 31; ++i)
    if (p.page_size == 1u << i) p.page_shift = i;
  p.box = 16;
  while (p.page_size % p.box) p.box /= 2;
  // one copy brings all of 16 keys where their pieces of 64 elements follow one another as the kernel wants them
  const uint32_t whole = p.box == 16 && dim % 64 == 0 ? dim / 64 : 1;
  p.copies = (dim + 63) / 64 / whole;
  p.max_pages = max_pages;
  p.table = d_table;
  p.table_row = table_row;
  p.lengths = d_lengths;
  p.sequences = sequences;
  p.hkv = kv_heads;
  p.group = q_heads / kv_heads;
  p.chunks = p.group > 8 ? (p.group + 15) / 16 : 1;
  p.dim = dim;
  p.scale_log2 = scale_log2;
  p.out = d_out;
  p.o_row = out_row;
  p.o_head = out_head;
  p.lse = d_lse;
  p.q_heads = q_heads;
  p.vec_out = aligned_to(d_out, 8) && out_row % 4 == 0 && out_head % 4 == 0;
  p.part = reinterpret_cast<float*>(ctx->paged_ws + space.part);
  p.part_rl = reinterpret_cast<float*>(ctx->paged_ws + space.rl);
  p.arrived = reinterpret_cast<unsigned int*>(ctx->paged_ws + space.arrived);
  p.status = ctx->d_status;
  CUtensorMap map_k, map_v;
  KB_TRY(encode_cache(ctx, &map_k, cache->d_k, cache->k_page, cache->k_row, cache->k_head, *cache, kv_heads, dim, dtype, p.box, whole));
  KB_TRY(encode_cache(ctx, &map_v, cache->d_v, cache->v_page, cache->v_row, cache->v_head, *cache, kv_heads, dim, dtype, p.box, whole));
  return dtype == KB_F16 ? launch_paged<KB_F16>(ctx, map_k, map_v, p, st) : launch_paged<KB_BF16>(ctx, map_k, map_v, p, st);
}
