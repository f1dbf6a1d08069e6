// evict.hip - C ABI (include/still.h) of the scores of a paged cache's entries and of
// the eviction by them, for pages of every type.
#include "paged_host.hpp"
#include "evict.hpp"

namespace still {

// C8: keys of 8 bits, with scales ks.
template <bool C8>
static still_status paged_score_call(const still_paged_cache* cache, const float* ks, const still_paged_seqs* seqs,
                                     const still_paged_attend_config* cfg, const void* q, const double* q_positions,
                                     const float* lse, const int32_t* known, float* scores, void* stream) {
  still_status s = check_attend(cache, cfg);
  if (s != STILL_OK || (s = check_seqs(cache, seqs)) != STILL_OK) return s;
  const long esize = cache->mode == STILL_MODE_FP32 ? 4 : 2;
  const long q_row = (long)cache->n_kv_heads * cfg->group * cache->head_dim;
  if (cfg->q_stride < 0 || cfg->q_stride * esize % 16)
    return fail(STILL_E_SHAPE, "q_stride must be >= 0 and a multiple of 16 bytes");
  if ((s = check_ptr(cache->k, "cache k", true)) != STILL_OK || (s = check_ptr(cache->beta, "cache beta", false)) != STILL_OK ||
      (s = check_theta(cfg->rope_theta, q_positions)) != STILL_OK || (s = check_ptr(q, "q", true)) != STILL_OK ||
      (s = check_ptr(scores, "scores", true)) != STILL_OK)
    return s;
  if (!lse || ((uintptr_t)lse & 3u)) return fail(STILL_E_INVAL, "lse is NULL or not 4-byte aligned");
  if ((uintptr_t)known & 3u) return fail(STILL_E_INVAL, "known is not 4-byte aligned");
  PagedScoreArgs a;
  a.c = paged_args(cache, seqs);
  a.c.ks = const_cast<float*>(ks);
  a.q = (const char*)q;
  a.q_ts = (cfg->q_stride ? cfg->q_stride : q_row) * esize;
  a.lse = lse;
  a.known = known;
  a.scores = scores;
  a.qpos = cfg->rope_theta > 0.0 ? q_positions : nullptr;
  a.log2_theta = cfg->rope_theta > 0.0 ? std::log2(cfg->rope_theta) : 0.0;
  a.group = cfg->group;
  a.nq = cfg->n_queries;
  a.causal = cfg->causal;
  a.scale = cfg->scale != 0.f ? cfg->scale : 1.f / std::sqrt((float)cache->head_dim);
  hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  TIMED(STILL_K_ATTEND);
  const long pairs = (long)cache->n_kv_heads * seqs->n_seqs, cap = (long)seqs->max_pages * cache->page_size;
  const long z = std::min((cap + SCORE_CHUNK - 1) / SCORE_CHUNK, std::max(1L, 8192 / pairs));
  paged_dispatch(cache, [&](auto it, auto d) {
    using IT = decltype(it);
    using CT = std::conditional_t<C8, e4m3, IT>;
    constexpr int D = decltype(d)::value;
    const dim3 grid(cache->n_kv_heads, seqs->n_seqs, z);
    const bool rot = a.qpos != nullptr;
    auto launch = [&](auto rp) {
      using TL = ScoreTile<IT, D, decltype(rp)::value, CT>;
      hipLaunchKernelGGL((paged_score_kernel<IT, D, decltype(rp)::value, CT>), grid, dim3(256), TL::lds_bytes(rot, cfg->n_queries),
                         st, a);
    };
    const int R = cfg->group * cfg->n_queries;
    if (R <= 4) launch(std::integral_constant<int, 4>());
    else if (R <= 8) launch(std::integral_constant<int, 8>());
    else if (R <= 16) launch(std::integral_constant<int, 16>());
    else launch(std::integral_constant<int, 32>());
  });
  HIP_TRY(hipGetLastError());
  return STILL_OK;
}

static still_status check_evict(const still_paged_cache* cache, const still_paged_seqs* seqs, const still_paged_evict_config* cfg) {
  still_status s;
  if ((s = check_cache(cache)) != STILL_OK || (s = check_seqs(cache, seqs)) != STILL_OK) return s;
  if (!cfg) return fail(STILL_E_INVAL, "paged evict config is NULL");
  if (cfg->keep < 1 || cfg->first < 0 || cfg->recent < 0 || (long)cfg->first + cfg->recent > cfg->keep)
    return fail(STILL_E_SHAPE, "keep %d must be >= 1 and hold first %d and recent %d", cfg->keep, cfg->first, cfg->recent);
  if (cfg->keep > 1 << 30) return fail(STILL_E_UNSUPPORTED, "keep above 2^30, more than a table holds");
  if (cfg->shared != 0 && cfg->shared != 1) return fail(STILL_E_INVAL, "shared must be 0 or 1");
  return STILL_OK;
}

// The workspace: keys of lists that are formed ahead, and counts of their parts; none where
// a list's workgroup forms its own: where it holds them all (16384 keys; those of all heads
// together from 8192 on take longer to sum), and where there are lists for a quarter of the chip.
// us formed there / ahead (and a launch more, about 1.5): one sequence for all 8 heads of 9000
// entries 19 / 15, 64 such sequences 21 / 17; by head, 8 lists of 12000 entries 14 / 16, 64 of them
// 15 / 17, 8 of 20000 36 / 22, of 65536 70 / 32, 64 of them 71 / 39.
struct EvictPlan {
  long lists, kstride = 0;
  int kblocks = 0, kpart = 0;
  size_t total = 0;
};
static EvictPlan evict_plan(const still_paged_cache* c, const still_paged_seqs* q, const still_paged_evict_config* f) {
  EvictPlan p;
  const long cap = (long)q->max_pages * c->page_size;
  p.lists = (long)q->n_seqs * (f->shared ? 1 : c->n_kv_heads);
  if (cap <= (f->shared ? 8192 : 16384) || p.lists > 64 || p.lists * cap > 1L << 24) return p;
  p.kstride = cap;
  p.kpart = (int)rup((cap + 63) / 64, 4096);   // 64 parts at most
  p.kblocks = (int)((cap + p.kpart - 1) / p.kpart);
  p.total = p.lists * (cap * sizeof(uint32_t) + p.kblocks * SELECT_BINS * sizeof(int));
  return p;
}

// ks, vs: scales of pages of 8 bits, else NULL.
static still_status paged_evict_call(const still_paged_cache* cache, float* ks, float* vs, const still_paged_seqs* seqs,
                                     const still_paged_evict_config* cfg, float* scores, int32_t* kept, int32_t* new_lens,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  still_status s = check_evict(cache, seqs, cfg);
  if (s != STILL_OK) return s;
  if ((s = check_pages(cache)) != STILL_OK || (s = check_ptr(scores, "scores", true)) != STILL_OK) return s;
  if (!kept || !new_lens || ((uintptr_t)kept & 3u) || ((uintptr_t)new_lens & 3u))
    return fail(STILL_E_INVAL, "kept or new_lens is NULL or not 4-byte aligned");
  const EvictPlan plan = evict_plan(cache, seqs, cfg);
  const size_t need = plan.total;
  if (need && !workspace) return fail(STILL_E_WORKSPACE, "workspace is NULL");
  if (need && (s = check_ptr(workspace, "workspace", true)) != STILL_OK) return s;
  if (workspace_bytes < need) return fail(STILL_E_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes, need);
  PagedEvictArgs a;
  a.c = paged_args(cache, seqs);
  a.c.ks = ks;
  a.c.vs = vs;
  a.scores = scores;
  a.kept = kept;
  a.new_lens = new_lens;
  a.keep = cfg->keep;
  a.first = cfg->first;
  a.recent = cfg->recent;
  a.shared = cfg->shared;
  hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  TIMED(STILL_K_OTHER);
  const long cap = (long)seqs->max_pages * cache->page_size;
  const int H = cache->n_kv_heads, n_seqs = seqs->n_seqs;
  const int per_seq = cfg->shared ? 1 : H;
  const dim3 grid_of(per_seq, n_seqs);
  a.keys = (uint32_t*)workspace;
  a.kstride = plan.kstride;
  a.bins = (int*)(a.keys + plan.lists * plan.kstride);
  a.kblocks = plan.kblocks;
  a.kpart = plan.kpart;
  if (a.kstride) {
    hipLaunchKernelGGL(paged_keys_kernel, dim3(a.kblocks, per_seq, n_seqs), dim3(1024), 0, st, a);
    hipLaunchKernelGGL((paged_select_kernel<1024, 16, true>), grid_of, dim3(1024), 0, st, a);
  // us by 256 / 512 / 1024 threads: 512 lists of 1500 8.8 / 12.0 / 23, of 3000 19 / 13 / 24; 256 of
  // 6000 22 / 12 / 13
  } else if (cap <= 2048) {
    hipLaunchKernelGGL((paged_select_kernel<256, 8, false>), grid_of, dim3(256), 0, st, a);
  } else if (cap <= 8192) {
    hipLaunchKernelGGL((paged_select_kernel<512, 16, false>), grid_of, dim3(512), 0, st, a);
  } else {
    hipLaunchKernelGGL((paged_select_kernel<1024, 16, false>), grid_of, dim3(1024), 0, st, a);
  }
  HIP_TRY(hipGetLastError());
  // Workgroups of 1024 threads, and of 16 and 32 bits column pieces of their own, where there are
  // few lists: us of 8-bit moves to 1024 entries by 1024 / 256 threads, 8 lists 9 / 17, 64 11 / 20, 128
  // 19 / 24, 512 - / 62; of bf16 (four pieces / one) 64 lists 22 / 34, 128 43 / 41, 512 210 / 110; 8 lists
  // to 4096 in 1 / 2 / 4 / 8 pieces 51 / 29 / 22 / 26.
  const bool few = (long)H * n_seqs <= (ks ? 128 : 64);
  const int pieces = ks || !few ? 1 : 4;
  const dim3 grid(H, n_seqs, 2 * pieces + 1), threads(few ? 1024 : 256);
  auto move = [&](auto rowb, auto c8) {
    hipLaunchKernelGGL((paged_move_kernel<decltype(rowb)::value, decltype(c8)::value>), grid, threads, 0, st, a, pieces);
  };
  using No = std::false_type;
  using Yes = std::true_type;
  const int rowb = cache->head_dim * (ks ? 1 : cache->mode == STILL_MODE_FP32 ? 4 : 2);
  if (ks) {
    switch (rowb) {
      case 64: move(std::integral_constant<int, 64>(), Yes()); break;
      case 128: move(std::integral_constant<int, 128>(), Yes()); break;
      default: move(std::integral_constant<int, 256>(), Yes());
    }
  } else {
    switch (rowb) {
      case 128: move(std::integral_constant<int, 128>(), No()); break;
      case 256: move(std::integral_constant<int, 256>(), No()); break;
      case 512: move(std::integral_constant<int, 512>(), No()); break;
      default: move(std::integral_constant<int, 1024>(), No());
    }
  }
  HIP_TRY(hipGetLastError());
  return STILL_OK;
}

}  // namespace still

using namespace still;

extern "C" {

still_status still_paged_score(const still_paged_cache* cache, const still_paged_seqs* seqs,
                               const still_paged_attend_config* cfg, const void* q, const double* q_positions,
                               const float* lse, const int32_t* known, float* scores, void* stream) {
  return paged_score_call<false>(cache, nullptr, seqs, cfg, q, q_positions, lse, known, scores, stream);
}

still_status still_paged8_score(const still_paged8_cache* cache, const still_paged_seqs* seqs,
                                const still_paged_attend_config* cfg, const void* q, const double* q_positions,
                                const float* lse, const int32_t* known, float* scores, void* stream) {
  if (!cache) return fail(STILL_E_INVAL, "paged cache is NULL");
  const still_paged_cache c = plain_view(cache);
  still_status s;
  if ((s = check_attend(&c, cfg)) != STILL_OK || (s = check_ptr(cache->k_scale, "cache k_scale", true)) != STILL_OK) return s;
  return paged_score_call<true>(&c, cache->k_scale, seqs, cfg, q, q_positions, lse, known, scores, stream);
}

still_status still_paged_evict(const still_paged_cache* cache, const still_paged_seqs* seqs,
                               const still_paged_evict_config* cfg, float* scores, int32_t* kept, int32_t* new_lens,
                               void* workspace, size_t workspace_bytes, void* stream) {
  return paged_evict_call(cache, nullptr, nullptr, seqs, cfg, scores, kept, new_lens, workspace, workspace_bytes, stream);
}

size_t still_paged_evict_workspace_size(const still_paged_cache* cache, const still_paged_seqs* seqs,
                                        const still_paged_evict_config* cfg) {
  const std::string keep = g_last_error;
  if (check_evict(cache, seqs, cfg) != STILL_OK) {
    g_last_error = keep;
    return 0;
  }
  return evict_plan(cache, seqs, cfg).total;
}

still_status still_paged8_evict(const still_paged8_cache* cache, const still_paged_seqs* seqs,
                                const still_paged_evict_config* cfg, float* scores, int32_t* kept, int32_t* new_lens,
                                void* workspace, size_t workspace_bytes, void* stream) {
  if (!cache) return fail(STILL_E_INVAL, "paged cache is NULL");
  const still_paged_cache c = plain_view(cache);
  still_status s;
  if ((s = check_cache(&c)) != STILL_OK || (s = check_ptr(cache->k_scale, "cache k_scale", true)) != STILL_OK ||
      (s = check_ptr(cache->v_scale, "cache v_scale", true)) != STILL_OK)
    return s;
  return paged_evict_call(&c, cache->k_scale, cache->v_scale, seqs, cfg, scores, kept, new_lens, workspace,
                          workspace_bytes, stream);
}

}  // extern "C"
