// C entry points of the block-selected attention: checks and launches.  Included by prhs.cu after bytekv_host.cuh.
#pragma once
#include "block_sparse.cuh"

namespace {

constexpr int kMaxBlocks = kMaxContext / kBlockRows;

cudaError_t block_set_attributes() {
  const struct { const void* kernel; int bytes; } all[] = {{(const void*)block_attn_kernel<4, false, false>, kTSmemBytes},
                                                           {(const void*)block_attn_kernel<4, true, false>, kTSmemBytes},
                                                           {(const void*)block_attn_kernel<4, false, true>, kTSmemBytes},
                                                           {(const void*)block_attn_kernel<8, false, false>, kTSmemBytes},
                                                           {(const void*)block_attn_kernel<8, true, false>, kTSmemBytes},
                                                           {(const void*)block_attn_kernel<8, false, true>, kTSmemBytes},
                                                           {(const void*)block_attn_kernel<16, false, false>, kTSmemBytes},
                                                           {(const void*)block_attn_kernel<16, true, false>, kTSmemBytes},
                                                           {(const void*)block_attn_kernel<16, false, true>, kTSmemBytes},
                                                           {(const void*)block_score_kernel<false>, kScoreSmemBytes},
                                                           {(const void*)block_score_kernel<true>, kScoreSmemBytes}};
  for (const auto& k : all) {
    const cudaError_t e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, k.bytes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

prhs_status check_bounds(prhs_ctx* ctx, const prhs_block_bounds_view* bv, BoundsDev* out) {
  if (!bv || !bv->codes || !bv->scale) return fail(ctx, PRHS_ERR_INVALID_ARG, "block bounds: NULL pointer");
  if ((uintptr_t)bv->codes % 16 || (uintptr_t)bv->scale % 4)
    return fail(ctx, PRHS_ERR_INVALID_ARG, "block bounds: codes must be 16-byte aligned, scales 4-byte aligned");
  if (bv->stride_outer <= 0 || bv->stride_head <= 0) return fail(ctx, PRHS_ERR_INVALID_ARG, "block bounds: strides must be positive");
  if (bv->stride_outer > 0x7fffffffll || bv->stride_head > 0x7fffffffll)
    return fail(ctx, PRHS_ERR_UNSUPPORTED, "block bounds: strides above 2^31 blocks");
  out->codes = bv->codes;
  out->scale = bv->scale;
  out->stride_outer = bv->stride_outer;
  out->stride_head = bv->stride_head;
  return PRHS_OK;
}

// The view as for the other calls, and what these kernels need on top: page-table rows that cover max_seq_len.
prhs_status check_block_view(prhs_ctx* ctx, const prhs_kv_view* kv, int batch, KvDev* dv, int* max_t) {
  prhs_status rc = check_view(ctx, kv, batch, dv, max_t);
  if (rc != PRHS_OK) return rc;
  if (kv->page_table && (long long)kv->page_table_stride * kBlockRows < *max_t)
    return fail(ctx, PRHS_ERR_INVALID_ARG, "kv view: the page table's rows are shorter than max_seq_len");
  return check_device(ctx);
}

prhs_status check_block_sched(prhs_ctx* ctx, const prhs_block_schedule* s, int blocks_stride, int max_t) {
  if (!s) return fail(ctx, PRHS_ERR_INVALID_ARG, "block schedule: NULL");
  if (s->top_blocks < 0 || s->sink_blocks < 0 || s->recent_blocks < 0)
    return fail(ctx, PRHS_ERR_INVALID_ARG, "block schedule: negative budget");
  if (s->top_blocks > kMaxBlocks || s->sink_blocks > kMaxBlocks || s->recent_blocks > kMaxBlocks)
    return fail(ctx, PRHS_ERR_CAPACITY, "block schedule: budget above the largest context");
  if (s->flags & ~PRHS_GROUP_SETS) return fail(ctx, PRHS_ERR_INVALID_ARG, "block schedule: unknown flag");
  const int most = std::min(s->top_blocks + s->sink_blocks + s->recent_blocks, (max_t + kBlockRows - 1) / kBlockRows);
  if (blocks_stride < std::max(most, 1)) return fail(ctx, PRHS_ERR_CAPACITY, "blocks_stride below the budget's blocks");
  return PRHS_OK;
}

bool block_shared(const prhs_ctx* c, uint32_t flags) { return (flags & PRHS_GROUP_SETS) && c->gq > 1; }

// Launch of a kernel that calls step_wait(): beside the end of the kernel before it in the stream (programmatic
// dependent launch), or in plain stream order.
template <typename P>
cudaError_t launch_ordered(void (*kernel)(P), dim3 grid, int threads, size_t smem, cudaStream_t st, const P& p, int overlap) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = overlap;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}
template <typename P>
cudaError_t launch_after(void (*kernel)(P), dim3 grid, int threads, size_t smem, cudaStream_t st, const P& p) {
  return launch_ordered(kernel, grid, threads, smem, st, p, 1);
}
prhs_status launch_block_topk(prhs_ctx* c, const void* q, const KvDev& kv, const BoundsDev& bd, const prhs_block_schedule* s,
                              int max_t, int batch, int32_t* out_blocks, int stride, int32_t* out_count, bool select, cudaStream_t st) {
  const bool shared = block_shared(c, s->flags);
  BlockScoreParams sp;
  sp.q = static_cast<const __nv_bfloat16*>(q);
  sp.kv = kv;
  sp.bd = bd;
  sp.bounds_outer = (int)bd.stride_outer;
  sp.bounds_head = (int)bd.stride_head;
  sp.scores = c->scores;
  sp.ld = c->ld;
  sp.batch = batch;
  sp.num_q_heads = c->cfg.num_q_heads;
  sp.group_size = c->gq;
  sp.group_max = shared ? 1 : 0;
  sp.max_len = max_t;
  sp.flags = c->flags;
  // one wave of CTAs, none with less than one round of its four warps
  const int blocks = (max_t + kBlockRows - 1) / kBlockRows;
  const long long groups = (long long)batch * c->cfg.num_kv_heads * ((blocks + kScoreRound - 1) / kScoreRound);
  if (groups >= (1ll << 30)) return fail(c, PRHS_ERR_UNSUPPORTED, "batch * heads * max_seq_len above 2^38: pass a smaller max_seq_len");
  const int ctas = (int)std::min<long long>(kScoreCtasPerSm * c->sm_count, (groups + kScoreWarps - 1) / kScoreWarps);
  {
    LaunchScope ls(c, PRHS_KIND_SCORE, st);
    if (c->gq > 8) block_score_kernel<true><<<ctas, kScoreWarps * 32, kScoreSmemBytes, st>>>(sp);
    else block_score_kernel<false><<<ctas, kScoreWarps * 32, kScoreSmemBytes, st>>>(sp);
  }
  PRHS_CUDA(c, cudaGetLastError());
  if (!select) return PRHS_OK;
  BlockSelectParams p;
  p.scores = c->scores;
  p.ld = c->ld;
  p.num_q_heads = c->cfg.num_q_heads;
  p.heads_per_unit = shared ? c->gq : 1;
  p.units_per_seq = c->cfg.num_q_heads / p.heads_per_unit;
  p.seq_lens = kv.seq_lens;
  p.top = s->top_blocks;
  p.sink = s->sink_blocks;
  p.recent = s->recent_blocks;
  p.out_blocks = out_blocks;
  p.stride = stride;
  p.out_count = out_count;
  p.max_len = max_t;
  {
    LaunchScope ls(c, PRHS_KIND_SELECT, st);
    const dim3 grid(batch * p.units_per_seq);
    cudaError_t e;
    if (blocks <= 4 * kBSThreads) e = launch_after(block_select_kernel<4>, grid, kBSThreads, 0, st, p);
    else if (blocks <= 8 * kBSThreads) e = launch_after(block_select_kernel<8>, grid, kBSThreads, 0, st, p);
    else if (blocks <= 16 * kBSThreads) e = launch_after(block_select_kernel<16>, grid, kBSThreads, 0, st, p);
    else if (blocks <= 32 * kBSThreads) e = launch_after(block_select_kernel<32>, grid, kBSThreads, 0, st, p);
    else e = launch_after(block_select_kernel<0>, grid, kBSThreads, 0, st, p);
    PRHS_CUDA(c, e);
  }
  return PRHS_OK;
}

// Splits of a list of blocks.  In cycles, as measured: a warp works one block off in about 900; 8 KB take 2.4 of the HBM
// stream; of the smaller of the two a quarter stays visible; a CTA's start and end cost about 3000, a merge of parts
// 3000, and 1500 for every batch of parts of every four heads (finish_unit).  us per step with 1, 2, 4, 8, 16 splits:
//   32 lists of 19 blocks (one user)      9.7 11.8 12.0 12.4 15.3     128 sets of 137 for 4 heads  52.4 53.6
//   32 lists of 73                       20.0 19.3 17.6 16.4 20.4     64 sets                      38.2 33.6 33.4 37.8
//   64 lists of 73                       22.9 22.0 20.3 24.4 31.4     32 sets                      32.4 27.0 23.2 21.5 26.0
//   256 lists of 73                      60 72                        8 sets                       28.7 23.6 19.5 17.8 17.0
// Or a warp per unit (0 splits): no start and end for every four warps, where units are many and lists short; at least one such
// CTA per SM, and a tenth to gain, since the last of these longer CTAs leave the SMs unevenly used.  us, splits and warps:
//   608 lists of 11 blocks  26.6 23.2    1856  70.8 65.1    512  20.3 22.1    1024 lists of 19  35.1 26.7    3840  117 101
//   768 lists of 73         88.4 91.2    1856  195 206
int block_splits(const prhs_ctx* c, int units, int blocks, int heads) {
  const int slots = 2 * c->sm_count;
  const int merged = 16 * std::max(1, kTWarps / heads), rounds = (heads + kTWarps - 1) / kTWarps;     // a merge: parts at a time, heads
  const double stream = 2.4 * units * blocks;
  auto cost_of = [&](long long ctas, int per_warp) {
    const double waves = (double)((ctas + slots - 1) / slots), work = waves * per_warp * 900.0;
    return std::max(work, stream) + 0.25 * std::min(work, stream) + waves * 3000.0;
  };
  int best = 1;
  double best_cost = 1e30;
  for (int s = 1; s <= kMaxSplits; ++s) {
    const int per_warp = (blocks + s * kTWarps - 1) / (s * kTWarps);
    const double cost = cost_of((long long)units * s, per_warp) + (s > 1 ? 3000.0 + 1500.0 * rounds * ((s + merged - 1) / merged) : 0.0);
    if (cost < best_cost * 0.999) { best_cost = cost; best = s; }
    if (per_warp == 1) break;
  }
  const int own = (units + kTWarps - 1) / kTWarps;
  return own >= c->sm_count && cost_of(own, blocks) < 0.92 * best_cost ? 0 : best;
}

struct BlockPlan {
  int splits;      // 0: a warp per unit
  bool select;     // the attention kernel selects for itself (kSelect in block_sparse.cuh has both sides)
};
BlockPlan block_plan(const prhs_ctx* c, int batch, uint32_t flags, int stride, int max_t, const prhs_block_schedule* step) {
  const int heads = block_shared(c, flags) ? c->gq : 1, units = batch * (c->cfg.num_q_heads / heads);
  const int blocks = std::max(1, (max_t + kBlockRows - 1) / kBlockRows);
  // a unit's blocks at most; a step knows more than the width of the table
  const int listed = step ? std::min(stride, step->sink_blocks + step->top_blocks + step->recent_blocks) : stride;
  BlockPlan plan;
  // (a grid has at most 65535 sequences, and as many units of one, on its own axes; a warp per unit needs neither)
  const bool axes = batch <= 65535 && units / batch <= 65535;
  plan.splits = axes ? block_splits(c, units, std::min(listed, blocks), heads) : 0;
  plan.select = step && plan.splits > 0 && blocks <= kSelectKeys * kTThreads && step->top_blocks <= kSelectTop;
  return plan;
}

prhs_status launch_block_attn(prhs_ctx* c, const void* q, const KvDev& kv, const int32_t* blocks, const int32_t* count, int stride,
                              uint32_t flags, int max_t, int batch, void* out, float* out_lse, const BlockPlan& plan, const prhs_block_schedule* step,
                              const BoundsDev* bd, cudaStream_t st) {
  const bool shared = block_shared(c, flags);
  BlockAttnParams p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.kv = kv;
  p.blocks = blocks;
  p.count = count;
  p.stride = stride;
  p.heads_per_unit = shared ? c->gq : 1;
  p.units_per_seq = c->cfg.num_q_heads / p.heads_per_unit;
  p.num_q_heads = c->cfg.num_q_heads;
  p.group_size = c->gq;
  p.splits = std::max(plan.splits, 1);
  p.units = batch * p.units_per_seq;
  p.max_len = max_t;
  p.fixed = step ? 1 : 0;
  p.sink = step ? step->sink_blocks : 0;
  p.recent = step ? step->recent_blocks : 0;
  p.top = step ? step->top_blocks : 0;
  p.bd = bd ? *bd : BoundsDev{};
  p.scores = c->scores;
  p.ld = c->ld;
  p.out_blocks = const_cast<int32_t*>(blocks);
  p.out_count = const_cast<int32_t*>(count);
  p.partials = c->partials;
  p.tickets = c->tickets;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.out_lse = out_lse;
  p.flags = c->flags;
  {
    LaunchScope ls(c, PRHS_KIND_ATTN_SPARSE, st);
    // `step`: the lists are this step's, from the kernel before; a caller's own may come from any kernel (ordinary launch)
    const bool own = plan.splits == 0;
    const dim3 grid = own ? dim3((p.units + kTWarps - 1) / kTWarps) : dim3(p.splits, p.units_per_seq, batch);
    auto form = [&](auto heads) {
      constexpr int kHeads = decltype(heads)::value;
      return own ? block_attn_kernel<kHeads, false, true> : plan.select ? block_attn_kernel<kHeads, true, false> : block_attn_kernel<kHeads, false, false>;
    };
    const auto kernel = p.heads_per_unit > 8 ? form(SlotC<16>{}) : p.heads_per_unit > 4 ? form(SlotC<8>{}) : form(SlotC<4>{});
    const cudaError_t e = launch_ordered(kernel, grid, kTThreads, kTSmemBytes, st, p, step ? 1 : 0);
    PRHS_CUDA(c, e);
  }
  return PRHS_OK;
}

}  // namespace

extern "C" {

prhs_status prhs_block_bounds(prhs_ctx* ctx, const prhs_kv_view* kv, const prhs_block_bounds_view* bounds, const int32_t* first,
                              int32_t max_new, int32_t batch, void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  KvDev dv;
  BoundsDev bd;
  int max_t;
  prhs_status rc = check_block_view(ctx, kv, batch, &dv, &max_t);
  if (rc == PRHS_OK) rc = check_bounds(ctx, bounds, &bd);
  if (rc != PRHS_OK) return rc;
  if (max_new < 0) return fail(ctx, PRHS_ERR_INVALID_ARG, "block bounds: negative max_new");
  const int most = (first && max_new > 0) ? std::min(max_new, max_t) : max_t;
  cudaStream_t st = as_stream(stream);
  BoundsParams p;
  p.kv = dv;
  p.bd = bd;
  p.first = first;
  p.max_new = most;
  p.max_len = max_t;
  p.flags = ctx->flags;
  if (ctx->cfg.num_kv_heads > 65535 || batch > 65535) return fail(ctx, PRHS_ERR_UNSUPPORTED, "block bounds: more than 65535 heads or sequences");
  // blocks a sequence can touch: its new positions may start anywhere in a block
  const int blocks = most == 1 ? 1 : std::min((most + 2 * (kBlockRows - 1)) / kBlockRows, (max_t + kBlockRows - 1) / kBlockRows);
  const int warps = std::min(blocks, 8);
  {
    LaunchScope ls(ctx, PRHS_KIND_MISC, st);
    block_bounds_kernel<<<dim3((blocks + warps - 1) / warps, ctx->cfg.num_kv_heads, batch), 32 * warps, 0, st>>>(p);
  }
  PRHS_CUDA(ctx, cudaGetLastError());
  return PRHS_OK;
}

prhs_status prhs_block_topk(prhs_ctx* ctx, const void* q, const prhs_kv_view* kv, const prhs_block_bounds_view* bounds,
                            const prhs_block_schedule* sched, int32_t batch, int32_t* out_blocks, int32_t blocks_stride,
                            int32_t* out_count, void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  if (!q || !out_blocks || !out_count) return fail(ctx, PRHS_ERR_INVALID_ARG, "NULL pointer");
  if ((uintptr_t)q % 16) return fail(ctx, PRHS_ERR_INVALID_ARG, "q must be 16-byte aligned");
  KvDev dv;
  BoundsDev bd;
  int max_t;
  prhs_status rc = check_block_view(ctx, kv, batch, &dv, &max_t);
  if (rc == PRHS_OK) rc = check_bounds(ctx, bounds, &bd);
  if (rc == PRHS_OK) rc = check_block_sched(ctx, sched, blocks_stride, max_t);
  if (rc != PRHS_OK) return rc;
  return launch_block_topk(ctx, q, dv, bd, sched, max_t, batch, out_blocks, blocks_stride, out_count, true, as_stream(stream));
}

prhs_status prhs_block_decode_attn(prhs_ctx* ctx, const void* q, const prhs_kv_view* kv, const int32_t* blocks, const int32_t* count,
                                   int32_t blocks_stride, uint32_t flags, int32_t batch, void* out, float* out_lse, void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  if (!blocks || !count) return fail(ctx, PRHS_ERR_INVALID_ARG, "NULL pointer");
  if (blocks_stride < 1 || blocks_stride > 3 * kMaxBlocks) return fail(ctx, PRHS_ERR_INVALID_ARG, "blocks_stride out of range");
  if (flags & ~PRHS_GROUP_SETS) return fail(ctx, PRHS_ERR_INVALID_ARG, "block attention: unknown flag");
  KvDev dv;
  int max_t;
  prhs_status rc = check_q_out(ctx, q, out, batch);
  if (rc == PRHS_OK) rc = check_block_view(ctx, kv, batch, &dv, &max_t);
  if (rc != PRHS_OK) return rc;
  return launch_block_attn(ctx, q, dv, blocks, count, blocks_stride, flags, max_t, batch, out, out_lse,
                           block_plan(ctx, batch, flags, blocks_stride, max_t, nullptr), nullptr, nullptr, as_stream(stream));
}

prhs_status prhs_block_decode_step(prhs_ctx* ctx, const void* q, const prhs_kv_view* kv, const prhs_block_bounds_view* bounds,
                                   const prhs_block_schedule* sched, int32_t batch, void* out, float* out_lse, int32_t* out_blocks,
                                   int32_t blocks_stride, int32_t* out_count, void* stream) {
  if (!ctx) return PRHS_ERR_INVALID_ARG;
  if (!out_blocks || !out_count) return fail(ctx, PRHS_ERR_INVALID_ARG, "NULL pointer");
  KvDev dv;
  BoundsDev bd;
  int max_t;
  prhs_status rc = check_q_out(ctx, q, out, batch);
  if (rc == PRHS_OK) rc = check_block_view(ctx, kv, batch, &dv, &max_t);
  if (rc == PRHS_OK) rc = check_bounds(ctx, bounds, &bd);
  if (rc == PRHS_OK) rc = check_block_sched(ctx, sched, blocks_stride, max_t);
  if (rc != PRHS_OK) return rc;
  if (sched->recent_blocks < 1)
    return fail(ctx, PRHS_ERR_INVALID_ARG, "block step: recent_blocks must be >= 1 (the last block is attended over, not scored)");
  const BlockPlan plan = block_plan(ctx, batch, sched->flags, blocks_stride, max_t, sched);
  rc = launch_block_topk(ctx, q, dv, bd, sched, max_t, batch, out_blocks, blocks_stride, out_count, !plan.select, as_stream(stream));
  if (rc != PRHS_OK) return rc;
  return launch_block_attn(ctx, q, dv, out_blocks, out_count, blocks_stride, sched->flags, max_t, batch, out, out_lse, plan, sched, &bd,
                           as_stream(stream));
}

}  // extern "C"
