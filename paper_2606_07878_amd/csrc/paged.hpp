// paged.hpp - kernels of the paged cache: appending rotated keys and values to
// a sequence's pages, reading a range of it back as dense rows, and attention
// of its newest tokens over it.
//
// Pages are [n_pages][H][P][d] (P entries of a head contiguous), P a power of
// two from 16 up; entry j of sequence s is slot j % P of page table[s][j / P].
// Page numbers and lengths are read on the device and may hold anything: every
// address below is formed from a page number checked against n_pages.
#pragma once
#include "common.hpp"
#include "consumer.hpp"

namespace still {

struct PagedArgs {
  char* k;              // pages
  char* v;
  float* beta;          // [n_pages][H][P] or NULL
  const int* table;
  const int* lens;
  int H, lp, n_pages;   // P = 1 << lp
  int n_seqs, max_pages;
  long tstride;         // table entries between sequences
};

__device__ __forceinline__ long paged_cap(const PagedArgs& a) { return (long)a.max_pages << a.lp; }
__device__ __forceinline__ int paged_len(const PagedArgs& a, int s) {
  return (int)min((long)max(a.lens[s], 0), paged_cap(a));
}
// page of entry j (0 <= j < cap) of sequence s; -1: absent
__device__ __forceinline__ int paged_page(const PagedArgs& a, int s, long j) {
  const int p = a.table[s * a.tstride + (j >> a.lp)];
  return (unsigned)p < (unsigned)a.n_pages ? p : -1;
}
// row (in rows of d elements) of entry j's head h in page p
__device__ __forceinline__ long paged_row(const PagedArgs& a, int p, int h, long j) {
  return (((long)p * a.H + h) << a.lp) + (j & ((1 << a.lp) - 1));
}

// ---------------------------------------------------------------------------
// Append.  A block takes TPB tokens with all their heads, so that a token's
// angles (fp64: positions reach 1e5 and more) are formed once.  A work item is
// a pair of 16-byte pieces d/2 apart, the two members of the rotated pairs.
// Moves 2 x 2 H d values per token; nothing else matters but the launch.
// ---------------------------------------------------------------------------
struct PagedAppendArgs {
  PagedArgs c;
  const char *k, *v;                                // rows
  long k_ts, k_hs, v_ts, v_hs;                      // bytes
  const float* nbeta;                               // or NULL
  long b_ts, b_hs;                                  // elements
  const int* offsets;                               // [n_seqs + 1] or NULL
  const double* pos;                                // NULL: no rotation
  double log2_theta;
  int n_tokens, per_seq;                            // per_seq: tokens per sequence without offsets
};

constexpr int PAGED_APPEND_TPB = 4;

// entry and sequence of token i; false: skipped
__device__ __forceinline__ bool paged_target(const PagedAppendArgs& a, int i, int& s, long& j) {
  long end;
  if (a.offsets) {
    int lo = 0, hi = a.c.n_seqs;   // offsets[lo] <= i < offsets[hi] once both ends are known to hold it
    if (i < a.offsets[0] || i >= a.offsets[hi]) return false;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.offsets[mid] <= i) lo = mid;
      else hi = mid;
    }
    s = lo;
    end = a.offsets[lo + 1];
  } else {
    s = i / a.per_seq;
    end = (long)(s + 1) * a.per_seq;
  }
  j = (long)a.c.lens[s] - end + i;
  return j >= 0 && j < paged_cap(a.c);
}

template <class IT, int D, int TPB>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int HP = D * (int)sizeof(IT) / 32, EPP = 16 / (int)sizeof(IT), HD = D / 2;
  __shared__ float2 cs[TPB][HD];
  __shared__ int page[TPB], slot[TPB];
  const int tid = threadIdx.x;
  const long t0 = (long)blockIdx.x * TPB;
  if (tid < TPB) {
    int p = -1, s;
    long j = 0;
    if (t0 + tid < a.n_tokens && paged_target(a, (int)(t0 + tid), s, j)) p = paged_page(a.c, s, j);
    page[tid] = p;
    slot[tid] = (int)(j & ((1 << a.c.lp) - 1));
  }
  if (a.pos) {
    for (int e = tid; e < TPB * HD; e += 256) {
      const int t = e / HD, i = e % HD;
      if (t0 + t < a.n_tokens) cs[t][i] = rope_cs(a.pos[t0 + t], exp2(a.log2_theta * (-2.0 * i / D)));
    }
  }
  __syncthreads();
  const int H = a.c.H, items = TPB * H * 2 * HP;
  for (int it = tid; it < items; it += 256) {
    const int p = it % HP, kv = it / HP & 1, r = it / (2 * HP), h = r / TPB, t = r % TPB;
    if (page[t] < 0) continue;
    const char* src = kv ? a.v + (t0 + t) * a.v_ts + h * a.v_hs : a.k + (t0 + t) * a.k_ts + h * a.k_hs;
    u32x4 x0 = ((const u32x4*)src)[p], x1 = ((const u32x4*)src)[p + HP];
    if (!kv && a.pos) {
      float f0[EPP], f1[EPP];
      unpack16<IT>(x0, f0);
      unpack16<IT>(x1, f1);
      IT y0[EPP], y1[EPP];
#pragma unroll
      for (int e = 0; e < EPP; ++e) {
        const float2 c = cs[t][p * EPP + e];
        y0[e] = from_f32<IT>(f0[e] * c.x - f1[e] * c.y);
        y1[e] = from_f32<IT>(f1[e] * c.x + f0[e] * c.y);
      }
      __builtin_memcpy(&x0, y0, 16);
      __builtin_memcpy(&x1, y1, 16);
    }
    u32x4* dst = (u32x4*)((kv ? a.c.v : a.c.k) + ((((long)page[t] * H + h) << a.c.lp) + slot[t]) * (D * (long)sizeof(IT)));
    dst[p] = x0;
    dst[p + HP] = x1;
  }
  if (a.c.beta)
    for (int it = tid; it < TPB * H; it += 256) {
      const int h = it / TPB, t = it % TPB;
      if (page[t] >= 0)
        a.c.beta[(((long)page[t] * H + h) << a.c.lp) + slot[t]] =
            a.nbeta ? a.nbeta[(t0 + t) * a.b_ts + h * a.b_hs] : 0.f;
    }
}

// ---------------------------------------------------------------------------
// Gather: block (x, h) copies PAGED_GATHER_ROWS entries of head h, a thread
// 16-byte pieces of keys and values.  Bound by the copy.
// ---------------------------------------------------------------------------
struct PagedGatherArgs {
  PagedArgs c;
  char *K, *V;
  float* beta;   // or NULL
  int seq, start, n;
};

constexpr int PAGED_GATHER_ROWS = 64;

template <class IT, int D>
__global__ __launch_bounds__(256) void paged_gather_kernel(PagedGatherArgs a) {
  constexpr int PPR = D * (int)sizeof(IT) / 16;
  const int tid = threadIdx.x, h = blockIdx.y, len = paged_len(a.c, a.seq);
  const long i0 = (long)blockIdx.x * PAGED_GATHER_ROWS;
  for (int it = tid; it < PAGED_GATHER_ROWS * PPR; it += 256) {
    const long i = i0 + it / PPR, j = a.start + i;
    const int p = it % PPR;
    if (i >= a.n) break;
    const int page = j < len ? paged_page(a.c, a.seq, j) : -1;
    u32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
    if (page >= 0) {
      const long at = paged_row(a.c, page, h, j) * PPR + p;
      x = ((const u32x4*)a.c.k)[at];
      y = ((const u32x4*)a.c.v)[at];
    }
    const long to = ((long)h * a.n + i) * PPR + p;
    ((u32x4*)a.K)[to] = x;
    ((u32x4*)a.V)[to] = y;
  }
  if (a.beta && tid < PAGED_GATHER_ROWS && i0 + tid < a.n) {
    const long i = i0 + tid, j = a.start + i;
    const int page = j < len ? paged_page(a.c, a.seq, j) : -1;
    a.beta[(long)h * a.n + i] = page >= 0 ? a.c.beta[paged_row(a.c, page, h, j)] : 0.f;
  }
}

// ---------------------------------------------------------------------------
// Attention: a workgroup of 4 waves per (KV head, sequence).  Wave w takes
// entries w, w + 4, ...; a lane holds D / 64 features of every query row's
// running sum.  The waves' sums are joined in LDS.
// ---------------------------------------------------------------------------
struct PagedAttendArgs {
  PagedArgs c;
  const char* q;       // tokens of [H * group][d]
  long q_ts;           // bytes
  char* out;
  const double* qpos;  // NULL: q as given
  double log2_theta;
  int group, nq, causal;
  float scale;
};

constexpr int PAGED_WAVES = 4;

template <class IT, int D, int RB>
__global__ __launch_bounds__(64 * PAGED_WAVES) void paged_attend_kernel(PagedAttendArgs a) {
  constexpr int FPL = D / 64;
  __shared__ float qs[RB][D];
  __shared__ float acc[RB][D];
  __shared__ float wm[PAGED_WAVES][RB], wl[PAGED_WAVES][RB];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int h = blockIdx.x, s = blockIdx.y, R = a.group * a.nq, Hq = a.c.H * a.group;
  const int len = paged_len(a.c, s);
  // row g * nq + i: query i of head h * group + g
  for (int e = tid; e < R * D; e += 64 * PAGED_WAVES) {
    const int r = e / D, x = e % D, g = r / a.nq, i = r % a.nq;
    const IT* q = (const IT*)(a.q + ((long)s * a.nq + i) * a.q_ts) + (long)(h * a.group + g) * D;
    float f = to_f32(q[x]);
    if (a.qpos) {
      const int j = x % (D / 2);
      const float2 c = rope_cs(a.qpos[(long)s * a.nq + i], exp2(a.log2_theta * (-2.0 * j / D)));
      f = x < D / 2 ? f * c.x - to_f32(q[x + D / 2]) * c.y : f * c.x + to_f32(q[x - D / 2]) * c.y;
    }
    qs[r][x] = f;
    acc[r][x] = 0.f;
  }
  __syncthreads();
  float m[RB], l[RB], o[RB][FPL];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int u = 0; u < FPL; ++u) o[r][u] = 0.f;
  }
  for (int j = w; j < len; j += PAGED_WAVES) {
    const int page = paged_page(a.c, s, j);
    if (page < 0) continue;
    const long at = paged_row(a.c, page, h, j);
    float kf[FPL], vf[FPL];
#pragma unroll
    for (int u = 0; u < FPL; ++u) {
      kf[u] = to_f32(((const IT*)a.c.k)[at * D + u * 64 + lane]);
      vf[u] = to_f32(((const IT*)a.c.v)[at * D + u * 64 + lane]);
    }
    const float bias = a.c.beta ? a.c.beta[at] : 0.f;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      if (r >= R) continue;
      float d = 0.f;
#pragma unroll
      for (int u = 0; u < FPL; ++u) d += qs[r][u * 64 + lane] * kf[u];
      d = group_sum<64>(d);
      const int last = a.causal ? len - a.nq + r % a.nq : len - 1;
      if (j > last) continue;
      const float x = d * a.scale + bias, mn = fmaxf(m[r], x);
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float al = expf(m[r] - ref), p = expf(x - ref);
      m[r] = mn;
      l[r] = l[r] * al + p;
#pragma unroll
      for (int u = 0; u < FPL; ++u) o[r][u] = o[r][u] * al + p * vf[u];
    }
  }
#pragma unroll
  for (int r = 0; r < RB; ++r)
    if (lane == 0) {
      wm[w][r] = m[r];
      wl[w][r] = l[r];
    }
  __syncthreads();
  for (int x = 0; x < PAGED_WAVES; ++x) {
    if (w == x) {
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        float M = wm[0][r];
#pragma unroll
        for (int y = 1; y < PAGED_WAVES; ++y) M = fmaxf(M, wm[y][r]);
        const float sc = expf(m[r] - (M == -INFINITY ? 0.f : M));
#pragma unroll
        for (int u = 0; u < FPL; ++u)
          if (r < R) acc[r][u * 64 + lane] += o[r][u] * sc;
      }
    }
    __syncthreads();
  }
  for (int e = tid; e < R * D; e += 64 * PAGED_WAVES) {
    const int r = e / D, x = e % D, g = r / a.nq, i = r % a.nq;
    float M = -INFINITY, L = 0.f;
    for (int y = 0; y < PAGED_WAVES; ++y) M = fmaxf(M, wm[y][r]);
    for (int y = 0; y < PAGED_WAVES; ++y) L += expf(wm[y][r] - (M == -INFINITY ? 0.f : M)) * wl[y][r];
    const float f = L == 0.f ? 0.f : acc[r][x] / L;   // (a NaN stays one)
    ((IT*)a.out)[(((long)s * a.nq + i) * Hq + h * a.group + g) * D + x] = from_f32<IT>(f);
  }
}

}  // namespace still
