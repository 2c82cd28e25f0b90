// C entry points of the 8-bit KV cache: checks and launches.  Included by prhs.cu (uses its context and helpers).
#pragma once
#include "bytekv.cuh"

namespace {

// The calling thread's current device must be the context's: its workspaces and every launch live there.
prhs_status check_device(prhs_ctx* c) {
  int dev = -1;
  PRHS_CUDA(c, cudaGetDevice(&dev));
  if (dev != c->device) return fail(c, PRHS_ERR_INVALID_ARG, "the current device is not the one the context was created on");
  return PRHS_OK;
}

// q [batch][Hq][128] in, out of the same shape: 16-byte aligned and apart (a CTA writes its result while others still
// read their queries).
prhs_status check_q_out(prhs_ctx* c, const void* q, const void* out, int batch) {
  if (!q || !out) return fail(c, PRHS_ERR_INVALID_ARG, "NULL pointer");
  if (((uintptr_t)q | (uintptr_t)out) % 16) return fail(c, PRHS_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  const uintptr_t bytes = (uintptr_t)std::max(batch, 0) * c->cfg.num_q_heads * kRowBytes;
  if ((uintptr_t)q < (uintptr_t)out + bytes && (uintptr_t)out < (uintptr_t)q + bytes)
    return fail(c, PRHS_ERR_INVALID_ARG, "q and out overlap");
  return PRHS_OK;
}

cudaError_t bytekv_set_attributes() {
  const struct { const void* kernel; int bytes; } all[] = {
      {(const void*)bytekv_attn_kernel<kE4M3, false, false>, Shape8<false, false>::kSmemBytes},
      {(const void*)bytekv_attn_kernel<kE4M3, false, true>, Shape8<false, true>::kSmemBytes},
      {(const void*)bytekv_attn_kernel<kE4M3, true, false>, Shape8<true, false>::kSmemBytes},
      {(const void*)bytekv_attn_kernel<kE5M2, false, false>, Shape8<false, false>::kSmemBytes},
      {(const void*)bytekv_attn_kernel<kE5M2, false, true>, Shape8<false, true>::kSmemBytes},
      {(const void*)bytekv_attn_kernel<kE5M2, true, false>, Shape8<true, false>::kSmemBytes}};
  for (const auto& k : all) {
    const cudaError_t e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, k.bytes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

prhs_status check_bytekv(prhs_ctx* ctx, const prhs_bytekv_view* kv, int batch, ByteKvDev* out, int* max_t) {
  if (!kv || !kv->k || !kv->v || !kv->k_scale || !kv->v_scale || !kv->k_tail || !kv->v_tail || !kv->seq_lens)
    return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv view: NULL pointer");
  if (kv->format != PRHS_BYTEKV_E4M3 && kv->format != PRHS_BYTEKV_E5M2) return fail(ctx, PRHS_ERR_UNSUPPORTED, "bytekv view: unknown format");
  if (batch < 1) return fail(ctx, PRHS_ERR_INVALID_ARG, "batch must be >= 1");
  if (batch > ctx->cfg.max_batch) return fail(ctx, PRHS_ERR_CAPACITY, "batch exceeds max_batch");
  if (((uintptr_t)kv->k | (uintptr_t)kv->v | (uintptr_t)kv->k_tail | (uintptr_t)kv->v_tail) % 16 ||
      ((uintptr_t)kv->k_scale | (uintptr_t)kv->v_scale) % 4)
    return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv view: codes and tails must be 16-byte aligned, scales 4-byte aligned");
  if (kv->stride_outer <= 0 || kv->stride_head <= 0 || (kv->stride_outer % kRow8Bytes) || (kv->stride_head % kRow8Bytes))
    return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv view: code strides must be positive multiples of 128");
  if (kv->scale_stride_outer <= 0 || kv->scale_stride_head <= 0)
    return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv view: scale strides must be positive");
  const bool paged = kv->page_table != nullptr;
  if (paged != (ctx->cfg.page_size == 16))
    return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv view: page table does not match the configured page_size");
  if (paged && (kv->page_table_stride < 1 || kv->num_pages < 1))
    return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv view: bad page table stride or pool size");
  if (kv->max_seq_len < 0) return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv view: negative max_seq_len");
  const int mt = kv->max_seq_len > 0 ? kv->max_seq_len : ctx->cfg.max_context;
  if (mt > ctx->cfg.max_context) return fail(ctx, PRHS_ERR_CAPACITY, "max_seq_len exceeds max_context");
  if (paged && (long long)kv->page_table_stride * kBlockRows < mt)
    return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv view: the page table's rows are shorter than max_seq_len");
  out->k = static_cast<const uint8_t*>(kv->k);
  out->v = static_cast<const uint8_t*>(kv->v);
  out->k_scale = kv->k_scale;
  out->v_scale = kv->v_scale;
  out->k_tail = static_cast<const __nv_bfloat16*>(kv->k_tail);
  out->v_tail = static_cast<const __nv_bfloat16*>(kv->v_tail);
  out->stride_outer = kv->stride_outer;
  out->stride_head = kv->stride_head;
  out->scale_stride_outer = kv->scale_stride_outer;
  out->scale_stride_head = kv->scale_stride_head;
  out->page_table = kv->page_table;
  out->page_table_stride = kv->page_table_stride;
  out->seq_lens = kv->seq_lens;
  out->num_pages = kv->num_pages;
  *max_t = mt;
  return check_device(ctx);
}

prhs_status launch_bytekv_attn(prhs_ctx* c, const void* q, const ByteKvDev& kv, int format, const int* idx, const int* count, int idx_stride,
                            int max_count, int max_t, int batch, void* out, float* out_lse, cudaStream_t st) {
  ByteKvAttnParams p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.kv = kv;
  p.idx = idx;
  p.count = count;
  p.idx_stride = idx_stride;
  p.batch = batch;
  p.num_q_heads = c->cfg.num_q_heads;
  p.group_size = c->gq;
  p.partials = c->stream_part;
  p.max_len = max_t;
  p.tickets = c->tickets;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.out_lse = out_lse;
  p.flags = c->flags;
  // how the units are dealt (see bytekv.cuh), and to how many CTAs: one per resident slot, fewer where the items
  // (k8MinRun per CTA, k8ShortRun where that still leaves one CTA per SM) would not fill them.  max_count: positions
  // of a sequence or entries of a list at most.
  const int slots = (idx ? Shape8<true, false>::kCtasPerSm : Shape8<false, false>::kCtasPerSm) * c->sm_count;
  const int min_run = idx ? k8MinRun<true> : k8MinRun<false>;
  const long long units = (long long)batch * (idx ? c->cfg.num_q_heads : c->cfg.num_kv_heads);
  const long long unit_max = std::max(1, (max_count + (idx ? kBlockRows - 1 : 0)) / kBlockRows);       // items of a unit
  if (units * unit_max >= (1ll << 30))
    return fail(c, PRHS_ERR_UNSUPPORTED, "units times their largest length above 2^34: pass a smaller max_seq_len or idx_stride");
  p.deal = !idx ? kRuns : 2 * units <= slots ? kParts : kWhole;
  p.sm_count = c->sm_count;
  const long long few = std::min<long long>(c->sm_count, units * ((unit_max + k8ShortRun - 1) / k8ShortRun));
  const long long full = std::max(few, units * ((unit_max + min_run - 1) / min_run)) +
                         (p.deal != kWhole && units < slots && unit_max > k8ShortRun ? units : 0);      // rounding of parts
  const int ctas = (int)(p.deal == kWhole ? units : std::min<long long>(slots, full));
  const dim3 grid(ctas);
  {
    LaunchScope ls(c, idx ? PRHS_KIND_ATTN_SPARSE : PRHS_KIND_ATTN_DENSE, st);
    const bool e4 = format == PRHS_BYTEKV_E4M3;
    auto launch = [&](auto kernel, int threads, int smem) { kernel<<<grid, threads, smem, st>>>(p); };
    using List = Shape8<true, false>;
    using Narrow = Shape8<false, false>;
    using Wide = Shape8<false, true>;
    if (idx) launch(e4 ? bytekv_attn_kernel<kE4M3, true, false> : bytekv_attn_kernel<kE5M2, true, false>, List::kThreads, List::kSmemBytes);
    else if (c->gq > 8) launch(e4 ? bytekv_attn_kernel<kE4M3, false, true> : bytekv_attn_kernel<kE5M2, false, true>, Wide::kThreads, Wide::kSmemBytes);
    else launch(e4 ? bytekv_attn_kernel<kE4M3, false, false> : bytekv_attn_kernel<kE5M2, false, false>, Narrow::kThreads, Narrow::kSmemBytes);
  }
  PRHS_CUDA(c, cudaGetLastError());
  return PRHS_OK;
}

}  // namespace

extern "C" {

prhs_status prhs_bytekv_append(prhs_ctx* ctx, const prhs_bytekv_view* kv, const void* new_k, const void* new_v, int64_t stride_seq,
                            int64_t stride_head, int64_t stride_row, const int32_t* new_lens, int32_t max_new, int32_t batch,
                            void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  if (!new_k || !new_v || !new_lens) return fail(ctx, PRHS_ERR_INVALID_ARG, "NULL pointer");
  if (((uintptr_t)new_k | (uintptr_t)new_v) % 16 || stride_seq < 0 || stride_head < 0 || stride_row < 0 || (stride_seq % 8) ||
      (stride_head % 8) || (stride_row % 8))
    return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv append: rows must be 16-byte aligned (base, and strides multiples of 8 elements)");
  ByteKvDev dv;
  int max_t;
  prhs_status rc = check_bytekv(ctx, kv, batch, &dv, &max_t);
  if (rc != PRHS_OK) return rc;
  if (max_new < 1) return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv append: max_new must be >= 1");
  if (max_new > max_t) return fail(ctx, PRHS_ERR_CAPACITY, "bytekv append: max_new exceeds max_seq_len");
  if (ctx->cfg.num_kv_heads > 65535 || batch > 65535) return fail(ctx, PRHS_ERR_UNSUPPORTED, "bytekv append: more than 65535 heads or sequences");
  cudaStream_t st = as_stream(stream);
  ByteKvAppendParams p;
  p.kv = dv;
  p.new_k = static_cast<const __nv_bfloat16*>(new_k);
  p.new_v = static_cast<const __nv_bfloat16*>(new_v);
  p.new_stride_seq = stride_seq;
  p.new_stride_head = stride_head;
  p.new_stride_row = stride_row;
  p.new_lens = new_lens;
  p.max_new = max_new;
  p.max_len = max_t;
  p.batch = batch;
  p.num_kv_heads = ctx->cfg.num_kv_heads;
  p.flags = ctx->flags;
  // blocks a sequence can touch: its rows may start anywhere in a block
  const int blocks = max_new == 1 ? 1 : (max_new + 2 * (kBlockRows - 1)) / kBlockRows;
  const int pairs = std::min(blocks, 4);                       // warp pairs (keys, values) per CTA
  const dim3 grid((blocks + pairs - 1) / pairs, ctx->cfg.num_kv_heads, batch);
  {
    LaunchScope ls(ctx, PRHS_KIND_MISC, st);
    if (kv->format == PRHS_BYTEKV_E4M3) bytekv_append_kernel<kE4M3><<<grid, 64 * pairs, 0, st>>>(p);
    else bytekv_append_kernel<kE5M2><<<grid, 64 * pairs, 0, st>>>(p);
  }
  PRHS_CUDA(ctx, cudaGetLastError());
  return PRHS_OK;
}

prhs_status prhs_bytekv_decode_attn(prhs_ctx* ctx, const void* q, const prhs_bytekv_view* kv, int32_t batch, void* out, float* out_lse,
                                 void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  ByteKvDev dv;
  int max_t;
  prhs_status rc = check_q_out(ctx, q, out, batch);
  if (rc == PRHS_OK) rc = check_bytekv(ctx, kv, batch, &dv, &max_t);
  if (rc != PRHS_OK) return rc;
  return launch_bytekv_attn(ctx, q, dv, kv->format, nullptr, nullptr, 0, max_t, max_t, batch, out, out_lse, as_stream(stream));
}

prhs_status prhs_bytekv_sparse_decode_attn(prhs_ctx* ctx, const void* q, const prhs_bytekv_view* kv, const int32_t* idx,
                                        const int32_t* count, int32_t idx_stride, int32_t batch, void* out, float* out_lse,
                                        void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  if (!idx || !count) return fail(ctx, PRHS_ERR_INVALID_ARG, "NULL pointer");
  if (idx_stride < 1) return fail(ctx, PRHS_ERR_INVALID_ARG, "idx_stride must be >= 1");
  if (idx_stride > (1 << 30)) return fail(ctx, PRHS_ERR_UNSUPPORTED, "idx_stride above 2^30");
  ByteKvDev dv;
  int max_t;
  prhs_status rc = check_q_out(ctx, q, out, batch);
  if (rc == PRHS_OK) rc = check_bytekv(ctx, kv, batch, &dv, &max_t);
  if (rc != PRHS_OK) return rc;
  return launch_bytekv_attn(ctx, q, dv, kv->format, idx, count, idx_stride, idx_stride, max_t, batch, out, out_lse, as_stream(stream));
}

}  // extern "C"
