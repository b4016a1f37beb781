// eb_route: top-k softmax gating (Section 2.1) and per-micro-batch workload vectors (Section 2.3).
//
// One warp per token, a block per chunk of at most 32 tokens of one micro-batch (eb_route.cuh).  Loads are integer counts:
// gathered per block in shared memory, then added with integer atomics in global memory (order independent, hence
// deterministic); a clearing kernel zeroes the rows of the micro-batches being routed first.  What bounds many tokens over few
// experts is those atomics, all on the same few words: added token by token, 16 x 4096 tokens to one of 8 experts took 64 us
// and 1 x 4096 to 6 of 64 19; per chunk 22 and 11.
#include "eb_route.cuh"
#include "eb_scores.cuh"

namespace {

// The chunk's counts, gathered in s_hist, to the loads.  s_load [D] is clear.
__device__ __forceinline__ void add_loads(const ModelParams& mp, int j, const int* s_hist, int* s_load, int32_t* __restrict__ mb_load, int32_t* __restrict__ mb_cnt) {
  const int tid = threadIdx.x;
  if (tid < mp.E && s_hist[tid] > 0) {
    atomicAdd(&mb_cnt[j * mp.E + tid], s_hist[tid]);
    atomicAdd(&s_load[mp.e2d[tid]], s_hist[tid]);
  }
  __syncthreads();
  if (tid < mp.D && s_load[tid] > 0) atomicAdd(&mb_load[j * mp.D + tid], s_load[tid]);
}

template <int PL>
__global__ void __launch_bounds__(kChunkThreads, PL <= 2 ? 2 : 1)
route_kernel(ModelParams mp, BatchParams bp, uint32_t route_mask, const float* __restrict__ logits,
             int32_t* __restrict__ topk_idx, float* __restrict__ topk_w, int32_t* __restrict__ mb_load,
             int32_t* __restrict__ mb_cnt) {
  EB_GRID_DEP_SYNC();
  __shared__ int s_hist[EB_MAX_E], s_load[EB_MAX_D];
  const int c = blockIdx.x, j = mb_of_chunk(bp, c), lane = threadIdx.x & 31;
  if (!((route_mask >> j) & 1u)) return;
  if (threadIdx.x < mp.D) s_load[threadIdx.x] = 0;
  route_chunk(mp, bp, c, j, true, topk_idx, s_hist, [&](int t) { return route_token<PL>(mp, t, lane, logits, topk_idx, topk_w); });
  add_loads(mp, j, s_hist, s_load, mb_load, mb_cnt);
}

// The same by scores, groups and a bias (eb_scores.cuh); Z: float or bf16.
template <int PL, typename Z>
__global__ void __launch_bounds__(kChunkThreads, 1)
route_scored_kernel(ModelParams mp, BatchParams bp, RouterParams rp, uint32_t route_mask, const Z* __restrict__ logits, int64_t stride,
                    int32_t* __restrict__ topk_idx, float* __restrict__ topk_w, int32_t* __restrict__ mb_load, int32_t* __restrict__ mb_cnt) {
  EB_GRID_DEP_SYNC();
  __shared__ int s_hist[EB_MAX_E], s_load[EB_MAX_D];
  const int c = blockIdx.x, j = mb_of_chunk(bp, c), lane = threadIdx.x & 31;
  if (!((route_mask >> j) & 1u)) return;
  if (threadIdx.x < mp.D) s_load[threadIdx.x] = 0;
  route_chunk(mp, bp, c, j, true, topk_idx, s_hist, [&](int t) { return route_scored<PL>(mp, rp, t, bp.layer[j], lane, logits + t * stride, topk_idx, topk_w); });
  add_loads(mp, j, s_hist, s_load, mb_load, mb_cnt);
}

__global__ void route_clear_kernel(ModelParams mp, BatchParams bp, uint32_t route_mask, int32_t* mb_load,
                                   int32_t* mb_cnt) {
  EB_GRID_DEP_SYNC();
  int i = blockIdx.x * blockDim.x + threadIdx.x;
  int per = mp.E + mp.D;
  if (i >= bp.n_mb * per) return;
  int j = i / per, r = i % per;
  if (!((route_mask >> j) & 1u)) return;
  if (r < mp.E) mb_cnt[j * mp.E + r] = 0;
  else mb_load[j * mp.D + (r - mp.E)] = 0;
}

}  // namespace

bool ebi_router_ok(const eb_config& g, const eb_router* r, RouterParams* out, const char** why) {
  *why = nullptr;
  if (!r) *why = "null router";
  else if (r->score != EB_SCORE_SOFTMAX && r->score != EB_SCORE_SIGMOID) *why = "unknown score function";
  else if (r->n_group < 1 || r->n_group > EB_MAX_ROUTER_GROUPS || g.E % r->n_group) *why = "n_group must divide E and be at most EB_MAX_ROUTER_GROUPS";
  else if (r->topk_group < 1 || r->topk_group > r->n_group) *why = "topk_group out of range";
  else if (r->group_top != 1 && r->group_top != 2) *why = "group_top must be 1 or 2";
  else if ((int64_t)r->topk_group * (g.E / r->n_group) < g.K) *why = "the groups kept hold fewer than K experts";
  else if (!(r->scale > 0.f) || !(r->scale <= 3.4e38f)) *why = "scale must be positive and finite";
  else if (reinterpret_cast<uintptr_t>(r->bias) & 3u) *why = "bias not 4-byte aligned";
  if (*why) return false;
  *out = RouterParams{r->score == EB_SCORE_SIGMOID, r->n_group, r->topk_group, r->group_top, r->scale, r->bias};
  return true;
}

// Clears the counts and routes.  kind 0: softmax top-k on f32 logits, rows one behind the other; 1, 2: by the router, f32 or bf16 logits.
static eb_status route_run(eb_ctx* c, void* stream, const eb_batch* batch, uint32_t route_mask, int kind, const RouterParams& rp, const void* logits,
                           int64_t stride, int32_t* topk_idx, float* topk_w, int32_t* mb_load, int32_t* mb_cnt) {
  BatchParams bp;
  eb_status s = ebi_make_batch(c, batch, &bp);
  if (s != EB_OK) return s;
  if (!logits || !topk_idx || !topk_w || !mb_load || !mb_cnt) return ebi_fail(c, EB_ERR_INVALID_ARG, "null pointer");
  if (bp.n_mb < 32 && (route_mask >> bp.n_mb) != 0) return ebi_fail(c, EB_ERR_INVALID_ARG, "route_mask beyond n_mb");
  if (bp.n_mb == 0 || route_mask == 0) return EB_OK;
  cudaStream_t st = (cudaStream_t)stream;
  KernelTimer timer(c, EBK_ROUTE, st);
  int n = bp.n_mb * (c->cfg.E + c->cfg.D);
  EB_LAUNCH(c, "route", ebi_launch(route_clear_kernel, dim3((n + 255) / 256), dim3(256), 0, st, c->mp, bp, route_mask, mb_load, mb_cnt));
  if (bp.n_chunks > 0) {
    const bool few = c->cfg.E <= 64;
    const dim3 grid(bp.n_chunks), block(kChunkThreads);
    if (kind == 0)
      EB_LAUNCH(c, "route", ebi_launch(few ? route_kernel<2> : route_kernel<kMaxPerLane>, grid, block, 0, st, c->mp, bp, route_mask,
                                       (const float*)logits, topk_idx, topk_w, mb_load, mb_cnt));
    else if (kind == 1)
      EB_LAUNCH(c, "route", ebi_launch(few ? route_scored_kernel<2, float> : route_scored_kernel<kMaxPerLane, float>, grid, block, 0, st, c->mp, bp, rp,
                                       route_mask, (const float*)logits, stride, topk_idx, topk_w, mb_load, mb_cnt));
    else
      EB_LAUNCH(c, "route", ebi_launch(few ? route_scored_kernel<2, bf16> : route_scored_kernel<kMaxPerLane, bf16>, grid, block, 0, st, c->mp, bp, rp,
                                       route_mask, (const bf16*)logits, stride, topk_idx, topk_w, mb_load, mb_cnt));
  }
  EB_LAUNCH_CHECK(c, "route");
  return EB_OK;
}

extern "C" eb_status eb_route(eb_ctx* c, void* stream, const eb_batch* batch, uint32_t route_mask,
                              const float* logits, int32_t* topk_idx, float* topk_w, int32_t* mb_load,
                              int32_t* mb_cnt) {
  if (!c) return EB_ERR_INVALID_ARG;
  return route_run(c, stream, batch, route_mask, c->scored ? 1 : 0, c->router, logits, c->cfg.E, topk_idx, topk_w, mb_load, mb_cnt);
}

extern "C" eb_status eb_route_scored(eb_ctx* c, void* stream, const eb_batch* batch, uint32_t route_mask, const eb_router* router,
                                     const void* logits, eb_type type, int64_t row_stride, int32_t* topk_idx, float* topk_w,
                                     int32_t* mb_load, int32_t* mb_cnt) {
  if (!c) return EB_ERR_INVALID_ARG;
  RouterParams rp;
  const char* why;
  if (!ebi_router_ok(c->cfg, router, &rp, &why)) return ebi_fail(c, EB_ERR_INVALID_ARG, why);
  if (type != EB_TYPE_F32 && type != EB_TYPE_BF16) return ebi_fail(c, EB_ERR_UNSUPPORTED, "logits must be f32 or bf16");
  if (row_stride < c->cfg.E) return ebi_fail(c, EB_ERR_INVALID_ARG, "row_stride smaller than E");
  if (reinterpret_cast<uintptr_t>(logits) & (type == EB_TYPE_F32 ? 3u : 1u)) return ebi_fail(c, EB_ERR_INVALID_ARG, "logits not aligned to their type");
  return route_run(c, stream, batch, route_mask, type == EB_TYPE_F32 ? 1 : 2, rp, logits, row_stride, topk_idx, topk_w, mb_load, mb_cnt);
}

extern "C" eb_status eb_set_router(eb_ctx* c, const eb_router* router) {
  if (!c) return EB_ERR_INVALID_ARG;
  RouterParams rp = {};
  const char* why;
  if (router && !ebi_router_ok(c->cfg, router, &rp, &why)) return ebi_fail(c, EB_ERR_INVALID_ARG, why);
  c->router = rp;
  c->scored = router != nullptr;
  return EB_OK;
}
