// paged.hip - C ABI (include/still.h) of the paged cache: append, gather and
// attention through the kernels in paged.hpp.
#include "paged_host.hpp"

using namespace still;

extern "C" {

still_status still_paged_append(const still_paged_cache* cache, const still_paged_seqs* seqs,
                                const still_paged_tokens* t, void* stream) {
  still_status s;
  if ((s = check_cache(cache)) != STILL_OK || (s = check_seqs(cache, seqs)) != STILL_OK ||
      (s = check_tokens(cache, seqs, t)) != STILL_OK || t->n_tokens == 0)
    return s;
  const PagedAppendArgs a = append_args(paged_args(cache, seqs), cache, seqs, t);
  hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  TIMED(STILL_K_OTHER);
  paged_dispatch(cache, [&](auto it, auto d) {
    using IT = decltype(it);
    const PagedGrid g(((unsigned)t->n_tokens + PAGED_APPEND_TPB - 1) / PAGED_APPEND_TPB);
    hipLaunchKernelGGL((paged_append_kernel<IT, decltype(d)::value>), dim3(g.x, g.more), dim3(256), 0, st, a);
  });
  HIP_TRY(hipGetLastError());
  return STILL_OK;
}

still_status still_paged_gather(const still_paged_cache* cache, const still_paged_seqs* seqs, int32_t seq,
                                int32_t start, int32_t n, void* K, void* V, float* beta, void* stream) {
  still_status s;
  if ((s = check_cache(cache)) != STILL_OK || (s = check_seqs(cache, seqs)) != STILL_OK ||
      (s = check_range(cache, seqs, seq, start, n, K, V, beta)) != STILL_OK || n == 0)
    return s;
  PagedGatherArgs a;
  a.c = paged_args(cache, seqs);
  a.K = (char*)K;
  a.V = (char*)V;
  a.beta = beta;
  a.seq = seq;
  a.start = start;
  a.n = n;
  hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  TIMED(STILL_K_OTHER);
  paged_dispatch(cache, [&](auto it, auto d) {
    using IT = decltype(it);
    const PagedGrid g(((unsigned)n + PAGED_GATHER_ROWS - 1) / PAGED_GATHER_ROWS);
    hipLaunchKernelGGL((paged_gather_kernel<IT, decltype(d)::value>), dim3(g.x, a.c.H, g.more), dim3(256), 0, st, a);
  });
  HIP_TRY(hipGetLastError());
  return STILL_OK;
}

size_t still_paged_attend_workspace_size(const still_paged_cache* cache, const still_paged_attend_config* cfg) {
  const std::string keep = g_last_error;
  if (check_attend(cache, cfg) != STILL_OK) {
    g_last_error = keep;
    return 0;
  }
  return paged_plan(cache, cfg, false).total;
}

still_status still_paged_attend(const still_paged_cache* cache, const still_paged_seqs* seqs,
                                const still_paged_attend_config* cfg, const void* q, const double* q_positions,
                                void* out, void* workspace, size_t workspace_bytes, void* stream) {
  return paged_attend_call<false>(cache, nullptr, nullptr, seqs, cfg, q, q_positions, out, nullptr, workspace,
                                  workspace_bytes, stream);
}

still_status still_paged_attend_lse(const still_paged_cache* cache, const still_paged_seqs* seqs,
                                    const still_paged_attend_config* cfg, const void* q, const double* q_positions,
                                    void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return paged_attend_call<false>(cache, nullptr, nullptr, seqs, cfg, q, q_positions, out, lse, workspace,
                                  workspace_bytes, stream);
}

}  // extern "C"
