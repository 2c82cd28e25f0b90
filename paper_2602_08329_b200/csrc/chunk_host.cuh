// C entry point of the attention of many new tokens: checks and launch.  Included by prhs.cu (uses its context and helpers).
#pragma once
#include "chunk_attn.cuh"

namespace {

constexpr int kCARegsAtLaunch = 168;      // what the kernel's register split (2 x 216 + 72 per thread of a warpgroup) is made from

cudaError_t chunk_set_attributes(bool* fits) {
  *fits = true;
  for (const void* k : {(const void*)chunk_attn_kernel<false, false, false>, (const void*)chunk_attn_kernel<false, true, false>,
                        (const void*)chunk_attn_kernel<true, false, false>, (const void*)chunk_attn_kernel<true, true, false>,
                        (const void*)chunk_attn_kernel<false, false, true>, (const void*)chunk_attn_kernel<false, true, true>,
                        (const void*)chunk_attn_kernel<true, false, true>, (const void*)chunk_attn_kernel<true, true, true>}) {
    cudaFuncAttributes a;
    cudaError_t e = cudaFuncGetAttributes(&a, k);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kCASmemBytes);
    if (e != cudaSuccess) return e;
    // a warpgroup that asks for registers the block was not launched with would wait for good
    if (a.numRegs < kCARegsAtLaunch) *fits = false;
  }
  return cudaSuccess;
}

// Rounds that a cache of the context's largest size can ask for (see chunk_attn.cuh): the workspace has room for their pieces.
int chunk_rounds(const prhs_config& cfg) {
  const long long tiles = (long long)cfg.max_batch * cfg.num_kv_heads * ((cfg.max_context + kCATile - 1) / kCATile);
  return (int)std::min<long long>(kCAMaxRounds, (tiles + kCARoundTiles - 1) / kCARoundTiles);
}

// The workspace: for as many rounds as there is memory for (fewer read more of a long cache from DRAM).  Without any the
// context serves all other calls.
cudaError_t chunk_alloc(prhs_ctx* c) {
  for (int rounds = chunk_rounds(c->cfg); rounds > 0; rounds /= 2) {
    const size_t runs = (size_t)rounds * c->sm_count;
    cudaError_t e = dev_alloc(&c->chunk_part, 2 * runs * kCASlotFloats);
    if (e == cudaSuccess) {
      e = dev_alloc(&c->chunk_tickets, runs);
      if (e == cudaSuccess) {
        c->chunk_rounds = rounds;
        return cudaMemset(c->chunk_tickets, 0, runs * sizeof(unsigned int));
      }
      cudaFree(c->chunk_part);
      c->chunk_part = nullptr;
    }
    if (e != cudaErrorMemoryAllocation) return e;
    cudaGetLastError();
  }
  return cudaSuccess;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

// bf16, 128-byte swizzle, zeros out of bounds; strides in bytes, of the dimensions after the first.
bool encode_bf16(prhs_ctx* c, CUtensorMap* tm, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const cuuint32_t ones[3] = {1u, 1u, 1u};
  return reinterpret_cast<EncodeTiledFn>(c->encode_tiled)(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, ones,
                                                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

extern "C" {

prhs_status prhs_chunk_attn(prhs_ctx* ctx, const void* q, const int32_t* row_start, int32_t num_rows, const prhs_kv_view* kv,
                            const prhs_chunk_mask* mask, int32_t batch, void* out, float* out_lse, void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  if (num_rows != 0 && (!q || !out)) return fail(ctx, PRHS_ERR_INVALID_ARG, "NULL pointer");
  if (((uintptr_t)q | (uintptr_t)out) % 16) return fail(ctx, PRHS_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  ChunkParams p;
  int max_t;
  prhs_status rc = check_view(ctx, kv, batch, &p.kv, &max_t);
  if (rc == PRHS_OK) rc = check_table(ctx, kv, max_t);
  if (rc == PRHS_OK) rc = check_device(ctx);
  if (rc != PRHS_OK) return rc;
  if (num_rows < 0 || (!row_start && num_rows != batch))
    return fail(ctx, PRHS_ERR_INVALID_ARG, "num_rows must not be negative, and is the batch where row_start is NULL");
  const int hq = ctx->cfg.num_q_heads, hkv = ctx->cfg.num_kv_heads;
  const uintptr_t bytes = (uintptr_t)num_rows * hq * kRowBytes;
  if (!apart(q, bytes, out, bytes)) return fail(ctx, PRHS_ERR_INVALID_ARG, "q and out overlap");
  p.sinks = p.window = 0;
  p.psaw_c = 0.0;
  if (mask) {
    if (mask->sinks < 0 || mask->window < 0 || mask->psaw_layer_start < 0)
      return fail(ctx, PRHS_ERR_INVALID_ARG, "mask: negative sinks, window or psaw_layer_start");
    if (mask->psaw_layer_start > 0) {
      if (!(mask->psaw_phi > 0.f && mask->psaw_phi < 1.f && mask->psaw_alpha >= 0.f && std::isfinite(mask->psaw_alpha)) || mask->layer < 0)
        return fail(ctx, PRHS_ERR_INVALID_ARG, "mask: the sliding window needs 0 < phi < 1, alpha >= 0, layer >= 0");
      if (mask->layer >= ctx->cfg.num_layers) return fail(ctx, PRHS_ERR_CAPACITY, "mask: layer beyond num_layers");
      prhs_schedule s{};
      s.psaw_phi = mask->psaw_phi;
      s.psaw_alpha = mask->psaw_alpha;
      s.psaw_layer_start = mask->psaw_layer_start;
      p.psaw_c = psaw_factor(ctx, &s, mask->layer);
    }
    p.sinks = mask->sinks;
    p.window = mask->window;
  }
  if (!ctx->encode_tiled) return fail(ctx, PRHS_ERR_UNSUPPORTED, "chunk attention: the driver offers no tensor-map encoder");
  if (ctx->cfg.flags & PRHS_CFG_NO_CHUNK_ATTN) return fail(ctx, PRHS_ERR_UNSUPPORTED, "chunk attention: the context was created with PRHS_CFG_NO_CHUNK_ATTN");
  if (!ctx->chunk_tickets) return fail(ctx, PRHS_ERR_OOM, "chunk attention: prhs_create had no memory for its workspace");
  if (!ctx->chunk_fits) return fail(ctx, PRHS_ERR_UNSUPPORTED, "chunk attention: built with fewer registers than its warps share out");
  if (num_rows == 0) return PRHS_OK;
  const bool paged = kv->page_table != nullptr;
  const unsigned long long rows = (unsigned long long)((paged ? kv->num_pages : batch) - 1) * (unsigned long long)(kv->stride_outer >> 7) +
                                  (unsigned long long)(hkv - 1) * (unsigned long long)(kv->stride_head >> 7) +
                                  (unsigned long long)(paged ? kBlockRows : max_t);
  if (rows >= (1ull << 31) - kCATile) return fail(ctx, PRHS_ERR_UNSUPPORTED, "chunk attention: a cache of 2^31 rows or more");
  p.group = ctx->gq;
  // Few tokens: at most 64 / G rows per sequence on average (padding counts), for then an item of 64 rows holds all new tokens of a sequence.
  // Both kernels on both sides, us, 8 KV heads of 4, 16 sequences of n new tokens: at 4096 positions n = 1, 8, 16, 17, 32: few 71, 74, 86,
  // 146, 158, general 76, 77, 81, 81, 81; at 16384 n = 1, 8, 16, 17: 222, 225, 254, 460 against 230, 232, 243, 245; one sequence of 2047,
  // n = 1, 4, 16: 27, 27, 30 against 31, 31, 32.  From n = 12 on it is the weights' second part that is paid for.
  // The average does not see a long part among single tokens, whose items are then 64 rows too: 63 single tokens and one part of 256 or 900 at
  // 4096 positions take 360 and 520 us against 269 and 312 in the general kernel, at 16384 positions 1144 and 1695 against 1000 and
  // 1233; with the part alone at 65536 positions 3365 against 1342.  The host does not know the rows of a sequence; a caller
  // who does makes two calls.
  const bool few = num_rows <= (long long)batch * (kCATile / 2 / ctx->gq);
  p.tokens = (few ? kCATile / 2 : kCATile) / ctx->gq;
  alignas(64) CUtensorMap tm_q, tm_k, tm_v;
  const cuuint64_t qdim[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)hq, (cuuint64_t)num_rows}, qstr[2] = {(cuuint64_t)kRowBytes, (cuuint64_t)hq * kRowBytes};
  const cuuint32_t qbox[3] = {64u, (cuuint32_t)p.group, (cuuint32_t)p.tokens};
  const cuuint64_t kdim[2] = {(cuuint64_t)kHeadDim, (cuuint64_t)rows}, kstr[1] = {(cuuint64_t)kRowBytes};
  const cuuint32_t kbox[2] = {64u, paged ? (cuuint32_t)kBlockRows : (cuuint32_t)kCATile};
  if (!encode_bf16(ctx, &tm_q, q, 3, qdim, qstr, qbox) || !encode_bf16(ctx, &tm_k, kv->k, 2, kdim, kstr, kbox) ||
      !encode_bf16(ctx, &tm_v, kv->v, 2, kdim, kstr, kbox))
    return fail(ctx, PRHS_ERR_CUDA, "chunk attention: a tensor map could not be encoded");
  p.row_start = row_start;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.out_lse = out_lse;
  p.max_rounds = ctx->chunk_rounds;
  p.partials = ctx->chunk_part;
  p.tickets = ctx->chunk_tickets;
  p.flags = ctx->flags;
  p.num_rows = num_rows;
  p.batch = batch;
  p.num_q_heads = hq;
  p.num_kv_heads = hkv;
  p.max_len = max_t;
  p.oob_row = (unsigned int)rows;
  cudaStream_t st = as_stream(stream);
  {
    LaunchScope ls(ctx, PRHS_KIND_ATTN_DENSE, st);
    auto launch = [&](auto kernel) { kernel<<<ctx->sm_count, kCAThreads, kCASmemBytes, st>>>(tm_q, tm_k, tm_v, p); };
    const bool masks = p.window > 0 || p.psaw_c > 0.0;
    if (few && masks) launch(paged ? chunk_attn_kernel<true, true, true> : chunk_attn_kernel<false, true, true>);
    else if (few) launch(paged ? chunk_attn_kernel<true, false, true> : chunk_attn_kernel<false, false, true>);
    else if (masks) launch(paged ? chunk_attn_kernel<true, true, false> : chunk_attn_kernel<false, true, false>);
    else launch(paged ? chunk_attn_kernel<true, false, false> : chunk_attn_kernel<false, false, false>);
  }
  PRHS_CUDA(ctx, cudaGetLastError());
  return PRHS_OK;
}

}  // extern "C"
