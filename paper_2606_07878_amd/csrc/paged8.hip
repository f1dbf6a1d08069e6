// paged8.hip - C ABI (include/still.h) of the paged cache in 8 bits: append, gather
// and attention.
#include "paged_host.hpp"
#include "paged8.hpp"

namespace still {

static still_status check_scales(const still_paged8_cache* c) {
  still_status s;
  if ((s = check_ptr(c->k_scale, "cache k_scale", true)) != STILL_OK) return s;
  return check_ptr(c->v_scale, "cache v_scale", true);
}

static PagedArgs paged8_args(const still_paged8_cache* c, const still_paged_cache* plain, const still_paged_seqs* q) {
  PagedArgs a = paged_args(plain, q);
  a.ks = c->k_scale;
  a.vs = c->v_scale;
  return a;
}

}  // namespace still

using namespace still;

extern "C" {

still_status still_paged8_append(const still_paged8_cache* cache, const still_paged_seqs* seqs,
                                 const still_paged_tokens* t, void* stream) {
  if (!cache) return fail(STILL_E_INVAL, "paged cache is NULL");
  const still_paged_cache c = plain_view(cache);
  still_status s;
  if ((s = check_cache(&c)) != STILL_OK || (s = check_seqs(&c, seqs)) != STILL_OK ||
      (s = check_tokens(&c, seqs, t)) != STILL_OK || (s = check_scales(cache)) != STILL_OK || t->n_tokens == 0)
    return s;
  Append8Args a;
  a.t = append_args(paged8_args(cache, &c, seqs), &c, seqs, t);
  hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  TIMED(STILL_K_OTHER);
  paged_dispatch(&c, [&](auto it, auto d) {
    using IT = decltype(it);
    constexpr int D = decltype(d)::value;
    // Tokens of a workgroup, 1 or 16: one that is alone leads by itself; of longer runs one in
    // 16 does, and where they are few it does not matter that the others start for nothing.
    // us at 1 / 16, width 128, runs that start at any slot: 256 of 4 tokens 16 / 23, of 8 34 / 15, of 16 77 / 12; 64 of
    // 4 6 / 23; 4 of 8 5 / 14, of 64 8 / 11.  The host knows the mean run only: one of 2000 beside 255 sequences without
    // tokens, whose mean is 7.8, takes the first form, 47 / 12 (of width 256 75 / 19), beside 255 of one token each, whose
    // mean is 8.8, the second, 32 / 46 (47 / 56).
    // Heads of a workgroup: a wave's 2 units of two heads one after the other, or of four,
    // which share the angles.  us at 2 / 4 / 8: one token of 8 heads 4.5 / 5.3 / 6.6, 64 tokens
    // 5.0 / 5.9 / 7.8, 256 of width 256 9.6 / 7.2 / 8.9, 7k in 13 prompts (with two waves per SIMD) 46 / 37 / 42.
    auto launch = [&](auto tg) {
      constexpr int TG = decltype(tg)::value;
      const PagedGrid g(((unsigned)t->n_tokens + TG - 1) / TG);
      a.heads = std::min(c.n_kv_heads, TG == 1 && (long)t->n_tokens * c.n_kv_heads <= 1024 ? 2 : 4);
      hipLaunchKernelGGL((paged8_append_kernel<IT, D, TG>), dim3(g.x, (c.n_kv_heads + a.heads - 1) / a.heads, g.more),
                         dim3(256), 0, st, a);
    };
    if (t->n_tokens <= 256 || t->n_tokens / seqs->n_seqs < 8) launch(std::integral_constant<int, 1>());
    else launch(std::integral_constant<int, 16>());
  });
  HIP_TRY(hipGetLastError());
  return STILL_OK;
}

still_status still_paged8_gather(const still_paged8_cache* cache, const still_paged_seqs* seqs, int32_t seq,
                                 int32_t start, int32_t n, void* K, void* V, float* beta, void* stream) {
  if (!cache) return fail(STILL_E_INVAL, "paged cache is NULL");
  const still_paged_cache c = plain_view(cache);
  still_status s;
  if ((s = check_cache(&c)) != STILL_OK || (s = check_seqs(&c, seqs)) != STILL_OK ||
      (s = check_range(&c, seqs, seq, start, n, K, V, beta)) != STILL_OK || (s = check_scales(cache)) != STILL_OK || n == 0)
    return s;
  PagedGatherArgs a;
  a.c = paged8_args(cache, &c, seqs);
  a.K = (char*)K;
  a.V = (char*)V;
  a.beta = beta;
  a.seq = seq;
  a.start = start;
  a.n = n;
  hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  TIMED(STILL_K_OTHER);
  paged_dispatch(&c, [&](auto it, auto d) {
    const PagedGrid g(((unsigned)n + PAGED_GATHER_ROWS - 1) / PAGED_GATHER_ROWS);
    hipLaunchKernelGGL((paged8_gather_kernel<decltype(it), decltype(d)::value>), dim3(g.x, a.c.H, g.more), dim3(256), 0, st, a);
  });
  HIP_TRY(hipGetLastError());
  return STILL_OK;
}

size_t still_paged8_attend_workspace_size(const still_paged8_cache* cache, const still_paged_attend_config* cfg) {
  if (!cache) return 0;
  const still_paged_cache c = plain_view(cache);
  const std::string keep = g_last_error;
  if (check_attend(&c, cfg) != STILL_OK) {
    g_last_error = keep;
    return 0;
  }
  return paged_plan(&c, cfg, true).total;
}

still_status still_paged8_attend(const still_paged8_cache* cache, const still_paged_seqs* seqs,
                                 const still_paged_attend_config* cfg, const void* q, const double* q_positions,
                                 void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!cache) return fail(STILL_E_INVAL, "paged cache is NULL");
  const still_paged_cache c = plain_view(cache);
  still_status s;
  if ((s = check_attend(&c, cfg)) != STILL_OK || (s = check_scales(cache)) != STILL_OK) return s;
  return paged_attend_call<true>(&c, cache->k_scale, cache->v_scale, seqs, cfg, q, q_positions, out, lse, workspace,
                                 workspace_bytes, stream);
}

}  // extern "C"
