// C entry points of the calls that bring new tokens into a cache, and of the read-back: checks and launches.  Included by
// prhs.cu (uses its context and helpers).
#pragma once
#include "tokens.cuh"

namespace {

// The bytes that rows x heads of 128 values span from their base.
uintptr_t rows_bytes(long long rows, long long heads, long long stride_row, long long stride_head) {
  return rows < 1 ? 0 : (uintptr_t)((rows - 1) * stride_row + (heads - 1) * stride_head + kHeadDim) * 2;
}
bool apart(const void* a, uintptr_t a_bytes, const void* b, uintptr_t b_bytes) {
  return (uintptr_t)a + a_bytes <= (uintptr_t)b || (uintptr_t)b + b_bytes <= (uintptr_t)a;
}

prhs_status check_tokens(prhs_ctx* c, const prhs_token_rows* rows, const prhs_qk_prep* prep, int batch, const void* q_out, TokenRowsDev* in,
                         PrepDev* pd) {
  if (!rows || !prep || (rows->num_rows != 0 && (!rows->q || !rows->k || !rows->v || !q_out))) return fail(c, PRHS_ERR_INVALID_ARG, "new tokens: NULL pointer");
  const int hq = c->cfg.num_q_heads, hkv = c->cfg.num_kv_heads;
  const int64_t strides[] = {rows->q_stride_row, rows->q_stride_head, rows->k_stride_row, rows->k_stride_head, rows->v_stride_row, rows->v_stride_head};
  for (int64_t s : strides)
    if (s < 0 || s % 8) return fail(c, PRHS_ERR_INVALID_ARG, "new tokens: strides must be multiples of 8 elements, not negative");
  if (((uintptr_t)rows->q | (uintptr_t)rows->k | (uintptr_t)rows->v | (uintptr_t)q_out) % 16)
    return fail(c, PRHS_ERR_INVALID_ARG, "new tokens: q, k, v and q_out must be 16-byte aligned");
  if (batch < 1) return fail(c, PRHS_ERR_INVALID_ARG, "batch must be >= 1");
  if (rows->num_rows < 0 || (!rows->row_start && rows->num_rows != batch))
    return fail(c, PRHS_ERR_INVALID_ARG, "new tokens: num_rows must not be negative, and is the batch where row_start is NULL");
  if (rows->positions && rows->positions_stride < rows->num_rows)
    return fail(c, PRHS_ERR_INVALID_ARG, "new tokens: positions_stride below num_rows");
  const uintptr_t out_bytes = rows_bytes(rows->num_rows, hq, (long long)hq * kHeadDim, kHeadDim);
  if (!apart(q_out, out_bytes, rows->q, rows_bytes(rows->num_rows, hq, rows->q_stride_row, rows->q_stride_head)) ||
      !apart(q_out, out_bytes, rows->k, rows_bytes(rows->num_rows, hkv, rows->k_stride_row, rows->k_stride_head)) ||
      !apart(q_out, out_bytes, rows->v, rows_bytes(rows->num_rows, hkv, rows->v_stride_row, rows->v_stride_head)))
    return fail(c, PRHS_ERR_INVALID_ARG, "new tokens: q_out overlaps the rows that come in");
  if (prep->flags & ~(PRHS_PREP_NORM | PRHS_PREP_ADJACENT)) return fail(c, PRHS_ERR_INVALID_ARG, "prep: unknown flag");
  if (prep->rot_dim < 0 || prep->rot_dim > kHeadDim || (prep->rot_dim & 1)) return fail(c, PRHS_ERR_INVALID_ARG, "prep: rot_dim must be even, 0 .. 128");
  if (prep->rot_dim && !prep->inv_freq) return fail(c, PRHS_ERR_INVALID_ARG, "prep: inv_freq is NULL");
  if (prep->num_axes < 1 || prep->num_axes > PRHS_MAX_AXES) return fail(c, PRHS_ERR_INVALID_ARG, "prep: num_axes must be 1 .. 4");
  for (int f = 0; f < prep->rot_dim / 2; ++f)
    if (prep->axis_of[f] >= prep->num_axes) return fail(c, PRHS_ERR_INVALID_ARG, "prep: axis_of names an axis beyond num_axes");
  if ((prep->flags & PRHS_PREP_NORM) ? !(prep->eps >= 0.f && std::isfinite(prep->eps)) : (prep->q_weight || prep->k_weight))
    return fail(c, PRHS_ERR_INVALID_ARG, "prep: eps must be finite and not negative; weights go with PRHS_PREP_NORM");
  if (((uintptr_t)prep->q_weight | (uintptr_t)prep->k_weight) % 16) return fail(c, PRHS_ERR_INVALID_ARG, "prep: weights must be 16-byte aligned");
  in->q = static_cast<const __nv_bfloat16*>(rows->q);
  in->k = static_cast<const __nv_bfloat16*>(rows->k);
  in->v = static_cast<const __nv_bfloat16*>(rows->v);
  in->q_row = rows->q_stride_row;
  in->q_head = rows->q_stride_head;
  in->k_row = rows->k_stride_row;
  in->k_head = rows->k_stride_head;
  in->v_row = rows->v_stride_row;
  in->v_head = rows->v_stride_head;
  in->row_start = rows->row_start;
  in->positions = rows->positions;
  in->positions_stride = rows->positions_stride;
  in->num_rows = rows->num_rows;
  in->batch = batch;
  in->num_q_heads = hq;
  in->num_kv_heads = hkv;
  pd->q_weight = prep->q_weight;
  pd->k_weight = prep->k_weight;
  pd->inv_freq = prep->inv_freq;
  pd->eps = prep->eps;
  pd->rot_scale = prep->rot_scale;
  pd->rot = prep->rot_dim;
  pd->norm = (prep->flags & PRHS_PREP_NORM) ? 1 : 0;
  memcpy(pd->axis_of, prep->axis_of, sizeof(pd->axis_of));
  return PRHS_OK;
}

cudaError_t tokens_set_attributes() {
  const struct { const void* kernel; int bytes; } all[] = {
      {(const void*)bytekv_qkv_append_kernel<kE4M3, kRotHalves>, kQkv8SmemBytes<kRotHalves>},
      {(const void*)bytekv_qkv_append_kernel<kE4M3, kRotAdjacent>, kQkv8SmemBytes<kRotAdjacent>},
      {(const void*)bytekv_qkv_append_kernel<kE4M3, kRotPartial>, kQkv8SmemBytes<kRotPartial>},
      {(const void*)bytekv_qkv_append_kernel<kE5M2, kRotHalves>, kQkv8SmemBytes<kRotHalves>},
      {(const void*)bytekv_qkv_append_kernel<kE5M2, kRotAdjacent>, kQkv8SmemBytes<kRotAdjacent>},
      {(const void*)bytekv_qkv_append_kernel<kE5M2, kRotPartial>, kQkv8SmemBytes<kRotPartial>}};
  for (const auto& k : all) {
    const cudaError_t e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, k.bytes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

int rot_kind(const prhs_qk_prep* prep) {
  if (prep->rot_dim == 0 || (prep->flags & PRHS_PREP_ADJACENT)) return kRotAdjacent;
  return prep->rot_dim == kHeadDim ? kRotHalves : kRotPartial;
}

// A page-table row must hold every position that max_seq_len allows: the kernels index it by length alone.
prhs_status check_table(prhs_ctx* c, const prhs_kv_view* kv, int max_t) {
  if (kv->page_table && (long long)kv->page_table_stride * kBlockRows < max_t)
    return fail(c, PRHS_ERR_INVALID_ARG, "kv view: the page table's rows are shorter than max_seq_len");
  return PRHS_OK;
}

}  // namespace

extern "C" {

prhs_status prhs_qkv_append(prhs_ctx* ctx, const prhs_token_rows* rows, const prhs_qk_prep* prep, const prhs_kv_view* kv, int32_t batch,
                            void* q_out, void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  QkvAppendParams p;
  int max_t;
  prhs_status rc = check_tokens(ctx, rows, prep, batch, q_out, &p.rows, &p.prep);
  if (rc == PRHS_OK) rc = check_view(ctx, kv, batch, &p.kv, &max_t);
  if (rc == PRHS_OK) rc = check_table(ctx, kv, max_t);
  if (rc == PRHS_OK) rc = check_device(ctx);
  if (rc != PRHS_OK) return rc;
  if (rows->num_rows == 0) return PRHS_OK;
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.max_len = max_t;
  p.flags = ctx->flags;
  // eight rows to a CTA, so that what it looks up first is little beside what it moves; fewer, and their heads over several CTAs,
  // where that leaves SMs without work
  const int heads = ctx->cfg.num_q_heads + 2 * ctx->cfg.num_kv_heads, groups = (heads + 3) / 4, want = 3 * ctx->sm_count;
  if (heads > kQkvMaxHeads) return fail(ctx, PRHS_ERR_UNSUPPORTED, "new tokens: more than 512 heads of queries, keys and values");
  p.cta_rows = std::max(1, std::min(kQkvRows, rows->num_rows / want));
  const int ctas = (rows->num_rows + p.cta_rows - 1) / p.cta_rows;
  const dim3 grid(ctas, std::max(1, std::min({want / ctas, (p.cta_rows * groups + kQkvWarps - 1) / kQkvWarps, 65535})));
  cudaStream_t st = as_stream(stream);
  {
    LaunchScope ls(ctx, PRHS_KIND_MISC, st);
    auto launch = [&](auto kernel) { kernel<<<grid, 32 * kQkvWarps, heads * sizeof(HeadPlace), st>>>(p); };
    switch (rot_kind(prep)) {
      case kRotHalves: launch(qkv_append_kernel<kRotHalves>); break;
      case kRotAdjacent: launch(qkv_append_kernel<kRotAdjacent>); break;
      default: launch(qkv_append_kernel<kRotPartial>);
    }
  }
  PRHS_CUDA(ctx, cudaGetLastError());
  return PRHS_OK;
}

prhs_status prhs_bytekv_qkv_append(prhs_ctx* ctx, const prhs_token_rows* rows, const prhs_qk_prep* prep, const prhs_bytekv_view* kv,
                                   int32_t batch, void* q_out, void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  ByteKvQkvParams p;
  int max_t;
  prhs_status rc = check_tokens(ctx, rows, prep, batch, q_out, &p.rows, &p.prep);
  if (rc == PRHS_OK) rc = check_bytekv(ctx, kv, batch, &p.kv, &max_t);
  if (rc != PRHS_OK) return rc;
  if (rows->num_rows == 0) return PRHS_OK;
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.max_len = max_t;
  p.flags = ctx->flags;
  // blocks that n tokens touch: at most n, and at most n / 16 + 2
  const long long n = rows->num_rows, blocks = std::min<long long>(n, n / kBlockRows + 2ll * batch);
  // a block's heads over several CTAs where blocks are few
  const int tasks = std::max(2 * ctx->cfg.num_kv_heads, (ctx->cfg.num_q_heads + 3) / 4);
  const long long by = std::min<long long>((tasks + kQkv8Warps - 1) / kQkv8Warps, std::max<long long>(1, 4ll * ctx->sm_count / blocks));
  cudaStream_t st = as_stream(stream);
  {
    LaunchScope ls(ctx, PRHS_KIND_MISC, st);
    const dim3 grid((unsigned)blocks, (unsigned)by);
    auto launch = [&](auto kernel, int smem) { kernel<<<grid, 32 * kQkv8Warps, smem, st>>>(p); };
    const int rot = rot_kind(prep);
    if (kv->format == PRHS_BYTEKV_E4M3) {
      if (rot == kRotHalves) launch(bytekv_qkv_append_kernel<kE4M3, kRotHalves>, kQkv8SmemBytes<kRotHalves>);
      else if (rot == kRotAdjacent) launch(bytekv_qkv_append_kernel<kE4M3, kRotAdjacent>, kQkv8SmemBytes<kRotAdjacent>);
      else launch(bytekv_qkv_append_kernel<kE4M3, kRotPartial>, kQkv8SmemBytes<kRotPartial>);
    } else {
      if (rot == kRotHalves) launch(bytekv_qkv_append_kernel<kE5M2, kRotHalves>, kQkv8SmemBytes<kRotHalves>);
      else if (rot == kRotAdjacent) launch(bytekv_qkv_append_kernel<kE5M2, kRotAdjacent>, kQkv8SmemBytes<kRotAdjacent>);
      else launch(bytekv_qkv_append_kernel<kE5M2, kRotPartial>, kQkv8SmemBytes<kRotPartial>);
    }
  }
  PRHS_CUDA(ctx, cudaGetLastError());
  return PRHS_OK;
}

prhs_status prhs_bytekv_read(prhs_ctx* ctx, const prhs_bytekv_view* kv, const prhs_kv_view* out, const int32_t* first, int32_t max_new,
                             int32_t batch, void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  ByteKvReadParams p;
  int max_t, out_t;
  prhs_status rc = check_bytekv(ctx, kv, batch, &p.kv, &max_t);
  if (rc == PRHS_OK) rc = check_view(ctx, out, batch, &p.out, &out_t);
  if (rc == PRHS_OK) rc = check_table(ctx, out, out_t);
  if (rc != PRHS_OK) return rc;
  if (out_t < max_t) return fail(ctx, PRHS_ERR_CAPACITY, "bytekv read: max_seq_len of the bf16 cache below that of the 8-bit cache");
  if (max_new < 0) return fail(ctx, PRHS_ERR_INVALID_ARG, "bytekv read: negative max_new");
  if (max_new > max_t) return fail(ctx, PRHS_ERR_CAPACITY, "bytekv read: max_new exceeds max_seq_len");
  if (ctx->cfg.num_kv_heads > 65535 || batch > 65535) return fail(ctx, PRHS_ERR_UNSUPPORTED, "bytekv read: more than 65535 heads or sequences");
  p.first = first;
  p.max_new = max_new ? max_new : max_t;
  p.max_len = max_t;
  p.num_kv_heads = ctx->cfg.num_kv_heads;
  p.flags = ctx->flags;
  const int blocks = p.max_new == 1 ? 1 : (p.max_new + 2 * (kBlockRows - 1)) / kBlockRows;
  const int pairs = std::min(blocks, 4);
  const dim3 grid((blocks + pairs - 1) / pairs, ctx->cfg.num_kv_heads, batch);
  cudaStream_t st = as_stream(stream);
  {
    LaunchScope ls(ctx, PRHS_KIND_MISC, st);
    if (kv->format == PRHS_BYTEKV_E4M3) bytekv_read_kernel<kE4M3><<<grid, 64 * pairs, 0, st>>>(p);
    else bytekv_read_kernel<kE5M2><<<grid, 64 * pairs, 0, st>>>(p);
  }
  PRHS_CUDA(ctx, cudaGetLastError());
  return PRHS_OK;
}

}  // extern "C"
