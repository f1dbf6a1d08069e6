// paged_host.hpp - what the calls on paged caches share on the host: argument
// validation, the choice of an attention kernel, its workspace and its launches.
#pragma once
#include "host.hpp"
#include "paged.hpp"

namespace still {

inline still_status check_cache(const still_paged_cache* c) {
  if (!c) return fail(STILL_E_INVAL, "paged cache is NULL");
  if (c->mode != STILL_MODE_BF16 && c->mode != STILL_MODE_FP32) return fail(STILL_E_DTYPE, "unknown mode %d", c->mode);
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return fail(STILL_E_UNSUPPORTED, "paged head_dim %d not in {64, 128, 256}", c->head_dim);
  if (c->n_kv_heads < 1 || c->n_pages < 1) return fail(STILL_E_SHAPE, "paged n_kv_heads and n_pages must be >= 1");
  if (c->n_kv_heads > 65535) return fail(STILL_E_UNSUPPORTED, "n_kv_heads above 65535");
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return fail(STILL_E_UNSUPPORTED, "page_size %d is no power of two from 16 to 4096", c->page_size);
  return STILL_OK;
}

// The dimensions, pointers and rows' type of a cache in 8 bits, which the checks of the
// others cover.
inline still_paged_cache plain_view(const still_paged8_cache* c) {
  return {c->n_kv_heads, c->head_dim, c->page_size, c->n_pages, c->mode, c->k, c->v, c->beta};
}

inline still_status check_pages(const still_paged_cache* c) {
  still_status s;
  if ((s = check_ptr(c->k, "cache k", true)) != STILL_OK || (s = check_ptr(c->v, "cache v", true)) != STILL_OK) return s;
  return check_ptr(c->beta, "cache beta", false);
}

inline still_status check_seqs(const still_paged_cache* c, const still_paged_seqs* q) {
  if (!q) return fail(STILL_E_INVAL, "paged sequences are NULL");
  if (q->n_seqs < 1 || q->max_pages < 1) return fail(STILL_E_SHAPE, "n_seqs and max_pages must be >= 1");
  if (q->n_seqs > 65535) return fail(STILL_E_UNSUPPORTED, "n_seqs above 65535");
  if ((long)q->max_pages * c->page_size > (1L << 30))
    return fail(STILL_E_UNSUPPORTED, "max_pages * page_size above 2^30");
  if ((long)q->n_seqs * q->max_pages * c->page_size > (1L << 34))
    return fail(STILL_E_UNSUPPORTED, "n_seqs * max_pages * page_size above 2^34");
  if (q->table_stride < q->max_pages) return fail(STILL_E_SHAPE, "table_stride %d below max_pages %d", q->table_stride,
                                                  q->max_pages);
  if (!q->table || !q->lens || ((uintptr_t)q->table & 3u) || ((uintptr_t)q->lens & 3u))
    return fail(STILL_E_INVAL, "table or lens is NULL or not 4-byte aligned");
  return STILL_OK;
}

inline PagedArgs paged_args(const still_paged_cache* c, const still_paged_seqs* q) {
  PagedArgs a;
  a.k = (char*)c->k;
  a.v = (char*)c->v;
  a.ks = a.vs = nullptr;
  a.beta = c->beta;
  a.table = q->table;
  a.lens = q->lens;
  a.H = c->n_kv_heads;
  a.lp = __builtin_ctz((unsigned)c->page_size);
  a.n_pages = c->n_pages;
  a.n_seqs = q->n_seqs;
  a.max_pages = q->max_pages;
  a.tstride = q->table_stride;
  return a;
}

inline still_status check_theta(double theta, const double* positions) {
  if (!(theta >= 0.0) || !std::isfinite(theta)) return fail(STILL_E_INVAL, "rope_theta must be finite and >= 0");
  if (theta > 0.0 && (!positions || ((uintptr_t)positions & 7u)))
    return fail(STILL_E_INVAL, "rope_theta > 0 needs 8-byte aligned positions");
  return STILL_OK;
}

// Blocks of 256 threads along a grid's first dimension, and the rest of them along another:
// a dimension of 2^32 threads and more is cut to 32 bits without an error.
constexpr unsigned PAGED_GRID_X = 1u << 23;
struct PagedGrid {
  unsigned x, more;
  explicit PagedGrid(unsigned blocks) : x(std::min(blocks, PAGED_GRID_X)), more((blocks + PAGED_GRID_X - 1) / PAGED_GRID_X) {}
};

// f(IT(), head_dim constant) for the cache's element type and head width
template <class F>
inline void paged_dispatch(const still_paged_cache* c, F f) {
  auto width = [&](auto it) {
    switch (c->head_dim) {
      case 64: f(it, std::integral_constant<int, 64>()); break;
      case 128: f(it, std::integral_constant<int, 128>()); break;
      default: f(it, std::integral_constant<int, 256>()); break;
    }
  };
  if (c->mode == STILL_MODE_FP32) width(float());
  else width(bf16());
}

inline still_status check_attend(const still_paged_cache* c, const still_paged_attend_config* f) {
  still_status s = check_cache(c);
  if (s != STILL_OK) return s;
  if (!f) return fail(STILL_E_INVAL, "paged attend config is NULL");
  if (f->group < 1 || f->n_queries < 1) return fail(STILL_E_SHAPE, "group and n_queries must be >= 1");
  if ((long)f->group * f->n_queries > ATTEND_MAX_ROWS)
    return fail(STILL_E_UNSUPPORTED, "group * n_queries = %ld exceeds %d", (long)f->group * f->n_queries,
                ATTEND_MAX_ROWS);
  if (f->causal != 0 && f->causal != 1) return fail(STILL_E_INVAL, "causal must be 0 or 1");
  if (!std::isfinite(f->scale) || f->scale < 0.f) return fail(STILL_E_INVAL, "scale must be finite and >= 0");
  if (!(f->rope_theta >= 0.0) || !std::isfinite(f->rope_theta)) return fail(STILL_E_INVAL, "rope_theta must be >= 0");
  return STILL_OK;
}

// Who takes a sequence (and KV head).  Where its table is short one workgroup or
// one wave takes all of it: one launch instead of two (9.3 us of host time instead
// of 11.4), nothing joined, but one CU's rate of reading, or one wave's, for the
// longest one.  The host knows the table's capacity only, so a table as wide as the
// longest context takes parts, and streaming loads, while its sequences are short.  us in
// a graph, bf16 of width 128, 8 heads unless said.
// Team or parts (capacity 1024, the line), one sequence of 32 entries 4.9 / 8.3, 256
// 6.2 / 10.3, 512 8.9 / 10.3, 719 10.9 / 10.3, 1024 13.5 / 10.3; width 64, 719 7.6 /
// 9.7, 1024 9.1 / 9.7; width 256 (512, the line) 256 9.2 / 12.5, 512 13.4 / 12.5; fp32
// of width 64 256 6.2 / 9.6, 1024 13.5 / 9.6; 32 rows 256 8.0 / 14.1, 1024 15.9 / 15.4.
// 64 sequences (the line) of 1000 41 / 48; 70 of 1 to 1024, spread over their
// logarithm, 19.2 / 19.3.  So on the card parts are the faster ones for a few sequences of
// more than 700 entries; most tables of this width hold shorter ones, and outside a graph
// the second launch takes up to 2 us of that back.
// Wave or team: 30 sequences (below the line) of 30 entries 4.2 / 5.1, 128 6.5 / 5.8, 512
// 16.9 / 12.8; 40 (above) of 30 4.4 / 7.9, 128 6.7 / 9.3, 512 17.2 / 20.0; width 256, 40
// of 128 11.4 / 12.6; fp32 of width 64, 40 of 30 4.3 / 4.9, 256 15.7 / 11.5; 32 rows, 40 of
// 30 9.3 / 7.4, 256 19.1 / 14.1, rotated 12.7 / 14.7 and 25.1 / 21.6.
// Wave or parts: 256 sequences of 30 7.5 / 22.9, 256 41.8 / 54.8; 32 rows, 30 18.3 / 62;
// 70 of 1 to 1024 29.8 / 19.3, which is why waves take capacities to 512 only.
// Streaming loads where the call may read more than the memory-side cache holds (256
// MB): us with ordinary / streaming loads, one sequence of 131136 99 / 89, 64 of up to
// 16384 108 / 98, 5 of up to 20011 and 32 rows (410 MB) 48.8 / 47.6; below it the entries
// may still be there from the step before: 4 sequences of up to 9000 (147 MB) 23.6 / 25.8.
// 8 bits take the same lines.  us at widths 64, 128, 256 (4 rows unless said).  Team / parts (capacity
// 1024): one sequence of 256 4.8, 5.8, 7.3 / 9.6, 10.0, 11.4; 719 7.5, 8.9, 13.5 / 11.1, 10.2, 11.9; 1024 8.7,
// 10.2, 16.9 / 11.1, 10.2, 11.9; 32 rows of 719 11.6, 15.0, 21.5 / 12.3, 12.4, 17.2; 64 of 1000 15.6, 24.2, 45.5 /
// 23.3, 29.3, 49.0; 70 of 1 to 1024 10.9, 13.9, 20.8 / 19.4, 18.7, 24.3: parts are the faster ones for a few
// sequences of more than 512 of width 256, or of 32 rows, only.  Wave / team (capacity 512): 40 sequences
// of 30 4.1, 4.9, 6.5 / 5.4, 6.4, 6.3, of 128 6.7, 8.1, 11.1 / 5.8, 7.1, 8.3, of 512 17, 23, 32 / 8.8, 13.6, 19.9; 256 of
// 30 5.4, 6.9, 11.9 / 15.7, 19.6, 22.2, of 256 16.7, 24.9, 44 / 21.3, 31.5, 49; wave / parts 256 of 30 5.4, 6.9, 11.9 /
// 27, 23, 31.  Ordinary / streaming loads, one sequence of 131136 (134, 269, 537 MB) 37, 51, 111 / 36, 55, 96; 64 of
// 16000 (1.0, 2.1, 4.2 GB) 228, 357, 702 / 222, 353, 615; 4 of up to 9000 13.5, 12.4, 14.5 / 13.5, 13.0, 15.3.
enum PagedKernel { PAGED_PARTS, PAGED_STREAM, PAGED_TEAM, PAGED_WAVE };
inline PagedKernel paged_kernel(const still_paged_cache* c, const still_paged_seqs* q, int esize) {
  const long cap = (long)q->max_pages * c->page_size, pairs = (long)q->n_seqs * c->n_kv_heads;
  const PagedKernel parts = 2 * pairs * cap * c->head_dim * esize > (256L << 20) ? PAGED_STREAM : PAGED_PARTS;
  if (cap > 1024 || cap * c->head_dim * esize > 256 * 1024) return parts;
  if (cap <= 512) return pairs <= 256 ? PAGED_TEAM : PAGED_WAVE;
  return pairs <= 512 ? PAGED_TEAM : parts;
}

struct PagedPlan {
  int G;
  size_t opart, mpart, lpart, total;   // offsets behind the plan, bytes
};

inline PagedPlan paged_plan(const still_paged_cache* c, const still_paged_attend_config* f, bool eight) {
  PagedPlan p;
  // workgroups per KV head: as many as are resident at once
  p.G = std::max(1, 256 * paged_resident(eight ? 1 : c->mode == STILL_MODE_FP32 ? 4 : 2, c->head_dim, f->group * f->n_queries <= 16 ? 1 : 2) / c->n_kv_heads);
  const size_t slots = p.G == 1 ? 0 : (size_t)c->n_kv_heads * p.G * 2 * f->group * f->n_queries;   // one part: no joins
  p.opart = (size_t)rup(p.G * (long)sizeof(int4), 256);
  p.mpart = p.opart + slots * c->head_dim * sizeof(float);
  p.lpart = p.mpart + (size_t)rup((long)(slots * sizeof(float)), 256);
  p.total = p.lpart + (size_t)rup((long)(slots * sizeof(float)), 256) + 256;   // + alignment slack
  return p;
}

// Rows to append: what is wrong with them, or where they are.
inline still_status check_tokens(const still_paged_cache* cache, const still_paged_seqs* seqs, const still_paged_tokens* t) {
  still_status s;
  if (!t) return fail(STILL_E_INVAL, "tokens are NULL");
  if (t->n_tokens < 0) return fail(STILL_E_SHAPE, "n_tokens must be >= 0");
  if (!t->offsets && t->n_tokens % seqs->n_seqs)
    return fail(STILL_E_SHAPE, "%d tokens do not divide over %d sequences and no offsets are given", t->n_tokens,
                seqs->n_seqs);
  if ((uintptr_t)t->offsets & 3u) return fail(STILL_E_INVAL, "offsets are not 4-byte aligned");
  const long esize = cache->mode == STILL_MODE_FP32 ? 4 : 2;
  for (int64_t x : {t->k_token_stride, t->k_head_stride, t->v_token_stride, t->v_head_stride})
    if (x * esize % 16) return fail(STILL_E_SHAPE, "row strides must be multiples of 16 bytes");
  if (t->beta && !cache->beta) return fail(STILL_E_INVAL, "beta given to a cache without beta");
  if ((uintptr_t)t->beta & 3u) return fail(STILL_E_INVAL, "beta is not 4-byte aligned");
  if ((s = check_pages(cache)) != STILL_OK || t->n_tokens == 0) return s;
  if ((s = check_theta(t->rope_theta, t->positions)) != STILL_OK) return s;
  if ((s = check_ptr(t->k, "k", true)) != STILL_OK) return s;
  return check_ptr(t->v, "v", true);
}

inline PagedAppendArgs append_args(const PagedArgs& c, const still_paged_cache* cache, const still_paged_seqs* seqs,
                                   const still_paged_tokens* t) {
  const long esize = cache->mode == STILL_MODE_FP32 ? 4 : 2;
  PagedAppendArgs a;
  a.c = c;
  a.k = (const char*)t->k;
  a.v = (const char*)t->v;
  a.k_ts = t->k_token_stride * esize;
  a.k_hs = t->k_head_stride * esize;
  a.v_ts = t->v_token_stride * esize;
  a.v_hs = t->v_head_stride * esize;
  a.nbeta = t->beta;
  a.b_ts = t->beta_token_stride;
  a.b_hs = t->beta_head_stride;
  a.offsets = t->offsets;
  a.pos = t->rope_theta > 0.0 ? t->positions : nullptr;
  a.log2_theta = t->rope_theta > 0.0 ? std::log2(t->rope_theta) : 0.0;
  a.n_tokens = t->n_tokens;
  a.per_seq = t->n_tokens / seqs->n_seqs;
  return a;
}

inline still_status check_range(const still_paged_cache* cache, const still_paged_seqs* seqs, int32_t seq, int32_t start,
                                int32_t n, const void* K, const void* V, const float* beta) {
  still_status s;
  if (seq < 0 || seq >= seqs->n_seqs) return fail(STILL_E_SHAPE, "sequence %d outside [0, %d)", seq, seqs->n_seqs);
  if (start < 0 || n < 0 || (long)start + n > (long)seqs->max_pages * cache->page_size)
    return fail(STILL_E_SHAPE, "entries [%d, %ld) outside [0, %ld)", start, (long)start + n,
                (long)seqs->max_pages * cache->page_size);
  if (beta && !cache->beta) return fail(STILL_E_INVAL, "beta asked of a cache without beta");
  if ((uintptr_t)beta & 3u) return fail(STILL_E_INVAL, "beta is not 4-byte aligned");
  if ((s = check_pages(cache)) != STILL_OK || n == 0) return s;
  if ((s = check_ptr(K, "K", true)) != STILL_OK) return s;
  return check_ptr(V, "V", true);
}

// C8: entries of 8 bits, with scales ks and vs.
template <bool C8>
still_status paged_attend_call(const still_paged_cache* cache, const float* ks, const float* vs, const still_paged_seqs* seqs,
                               const still_paged_attend_config* cfg, const void* q, const double* q_positions, void* out,
                               float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  still_status s = check_attend(cache, cfg);
  if (s != STILL_OK || (s = check_seqs(cache, seqs)) != STILL_OK) return s;
  const long esize = cache->mode == STILL_MODE_FP32 ? 4 : 2;
  const long q_row = (long)cache->n_kv_heads * cfg->group * cache->head_dim;
  if (cfg->q_stride < 0 || cfg->q_stride * esize % 16)
    return fail(STILL_E_SHAPE, "q_stride must be >= 0 and a multiple of 16 bytes");
  if ((s = check_pages(cache)) != STILL_OK || (s = check_theta(cfg->rope_theta, q_positions)) != STILL_OK ||
      (s = check_ptr(q, "q", true)) != STILL_OK || (s = check_ptr(out, "out", true)) != STILL_OK)
    return s;
  if ((uintptr_t)lse & 3u) return fail(STILL_E_INVAL, "lse is not 4-byte aligned");
  if (!workspace) return fail(STILL_E_WORKSPACE, "workspace is NULL");
  const PagedPlan p = paged_plan(cache, cfg, C8);
  if (workspace_bytes < p.total)
    return fail(STILL_E_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes, p.total);
  char* ws = (char*)(((uintptr_t)workspace + 255) & ~(uintptr_t)255);
  PagedAttendArgs a;
  a.c = paged_args(cache, seqs);
  a.c.ks = const_cast<float*>(ks);
  a.c.vs = const_cast<float*>(vs);
  a.lse = lse;
  a.q = (const char*)q;
  a.q_ts = (cfg->q_stride ? cfg->q_stride : q_row) * esize;
  a.out = (char*)out;
  a.qpos = cfg->rope_theta > 0.0 ? q_positions : nullptr;
  a.log2_theta = cfg->rope_theta > 0.0 ? std::log2(cfg->rope_theta) : 0.0;
  a.group = cfg->group;
  a.nq = cfg->n_queries;
  a.nq_inv = (1 << 16) / cfg->n_queries + 1;
  a.causal = cfg->causal;
  a.scale = cfg->scale != 0.f ? cfg->scale : 1.f / std::sqrt((float)cache->head_dim);
  a.G = p.G;
  a.by_seq = seqs->n_seqs <= p.G;
  a.plan = (int4*)ws;
  a.opart = (float*)(ws + p.opart);
  a.mpart = (float*)(ws + p.mpart);
  a.lpart = (float*)(ws + p.lpart);
  hipStream_t st = (hipStream_t)stream;
  (void)hipGetLastError();
  TIMED(STILL_K_ATTEND);
  const int R = cfg->group * cfg->n_queries;
  paged_dispatch(cache, [&](auto it, auto d) {
    using IT = decltype(it);
    using CT = std::conditional_t<C8, e4m3, IT>;
    constexpr int D = decltype(d)::value;
    auto launch = [&](auto nr, auto sw) {
      constexpr int NR = decltype(nr)::value, SW = decltype(sw)::value;
      using TL = PagedTile<IT, D, NR, SW, CT>;
      hipLaunchKernelGGL((paged_attend_kernel<IT, D, NR, SW, CT>), dim3(a.c.H, SW > 0 ? a.c.n_seqs : a.G), dim3(64 * TL::NW),
                         (paged_lds_bytes<TL, sizeof(CT), D, NR, SW>(R, a.nq, a.qpos != nullptr)), st, a);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Parts = std::integral_constant<int, 0>;
    using Stream = std::integral_constant<int, -1>;
    switch (paged_kernel(cache, seqs, sizeof(CT))) {
      case PAGED_TEAM:
        if (R <= 16) launch(One(), std::integral_constant<int, paged_team(D, 1)>());
        else launch(Two(), std::integral_constant<int, paged_team(D, 2)>());
        return;
      case PAGED_WAVE:
        if (R <= 16) launch(One(), One());
        else launch(Two(), One());
        return;
      case PAGED_STREAM:
        if (R <= 16) launch(One(), Stream());
        else launch(Two(), Stream());
        break;
      default:
        if (R <= 16) launch(One(), Parts());
        else launch(Two(), Parts());
    }
    if (a.G > 1) {
      // wide blocks where a few of them may read hundreds of parts each: one sequence of
      // 400000 entries of one head 58 us with 256 threads, 50 with 1024; of 256 entries of
      // 8 heads 10.0 with 256, 11.2 with 1024
      const dim3 joins(R, a.c.H, std::min(a.c.n_seqs, a.G));
      const bool wide = a.G > 128 && ((long)a.c.max_pages << a.c.lp) > 128 * 128 && (long)joins.x * joins.y * joins.z <= 512;
      hipLaunchKernelGGL((paged_merge_kernel<IT, D>), joins, dim3(wide ? PAGED_MERGE_THREADS : 256), 0, st, a);
    }
  });
  HIP_TRY(hipGetLastError());
  return STILL_OK;
}

}  // namespace still
