// paged.hpp - kernels of the paged cache: appending rotated keys and values to
// a sequence's pages, reading a range of it back as dense rows, and attention
// of its newest tokens over it.
//
// Pages are [n_pages][H][P][d] (P entries of a head contiguous), P a power of
// two from 16 up; entry j of sequence s is slot j % P of page table[s][j / P].
// Page numbers and lengths are read on the device and may hold anything: every
// address below is formed from a page number checked against n_pages.
#pragma once
#include <algorithm>

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

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A uniform element through the scalar cache, whose loads are not counted with
// the vector loads: waiting for one waits for no row in flight.
template <class T>
__device__ __forceinline__ T scalar_load(const T* p, long i) {
  return ((const __attribute__((address_space(4))) T*)(uintptr_t)p)[i];
}

// ---------------------------------------------------------------------------
// Append.  A block takes four tokens with all their heads, so that a token's
// angles (fp64: positions reach 1e5 and more) are formed once; wave w finds token
// w's page while the rows are on their way, which it does not depend on.  A work
// item is a pair of 16-byte pieces d/2 apart, the two members of the rotated
// pairs.
// Moves 2 x 2 H d values per token; nothing else matters but the launch and the
// chain offsets -> length -> page.  The stores stream past the L2, which has nothing
// to gain from rows that the next kernels read once if at all: 6977 tokens of 8
// heads of width 256 (114 MB) 29.5 -> 21.5 us, 8192 of width 128 13.5 -> 11.9.
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

constexpr int PAGED_APPEND_TPB = 4;   // tokens per block, one per wave

// Sequence of token i: the last one whose first token is at or before i.  64-fold
// search by a wave; `probe` is the first step's offset of this lane.
__device__ __forceinline__ int paged_seq_of(const int* offsets, int n_seqs, int i, int probe) {
  int lo = 0, hi = n_seqs;
  for (bool first = true; hi - lo > 1; first = false) {
    const int step = (hi - lo + 63) / 64, x = lo + ((threadIdx.x & 63) + 1) * step;
    const int o = first ? probe : x < hi ? offsets[x] : 0;
    lo += step * __popcll(__ballot(x < hi && o <= i));
    hi = min(hi, lo + step);
  }
  return lo;
}

template <class IT, int D>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int TPB = PAGED_APPEND_TPB, HP = D * (int)sizeof(IT) / 32, EPP = 16 / (int)sizeof(IT), HD = D / 2;
  constexpr int U = HP >= 16 ? 4 : 2;   // items of a thread in flight
  __shared__ float2 cs[TPB][HD];
  __shared__ int page[TPB], slot[TPB];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const long t0 = ((long)blockIdx.y * gridDim.x + blockIdx.x) * TPB;
  if (t0 >= a.n_tokens) return;
  const int left = (int)min((long)TPB, a.n_tokens - t0);   // tokens of this block
  // the first step of the search, and a position per thread's first angle, ahead of the rows
  const int n_seqs = a.c.n_seqs, x0 = (lane + 1) * ((n_seqs + 63) / 64);
  const int probe = a.offsets && x0 < n_seqs ? a.offsets[x0] : 0;
  double pos[(TPB * HD + 255) / 256];   // of the thread's angles (256 / HD tokens apart, all of pair tid % HD)
#pragma unroll
  for (int k = 0; k < (TPB * HD + 255) / 256; ++k) pos[k] = a.pos ? a.pos[t0 + min((k * 256 + tid) / HD, left - 1)] : 0.0;
  __builtin_amdgcn_sched_barrier(0);
  const int H = a.c.H, items = TPB * H * 2 * HP;
  u32x4 x[U][2];
  auto load = [&](int b) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int it = b + k * 256 + tid, p = it % HP, kv = it / HP & 1, r = it / (2 * HP), h = min(r / TPB, H - 1);
      const long t = t0 + min(r % TPB, left - 1);
      const u32x4* src = (const u32x4*)(kv ? a.v + t * a.v_ts + h * a.v_hs : a.k + t * a.k_ts + h * a.k_hs);
      if (b + k * 256 < items) {
        x[k][0] = src[p];
        x[k][1] = src[p + HP];
      }
    }
  };
  load(0);
  __builtin_amdgcn_sched_barrier(0);
  {  // this wave's token: its entry's page and slot
    const int i = (int)t0 + w;
    int pg = -1;
    long j = -1;
    if (w < left) {
      int s;
      long end;
      if (a.offsets) {
        s = uniform(paged_seq_of(a.offsets, n_seqs, i, probe));
        end = scalar_load(a.offsets, s + 1);
        if (i < scalar_load(a.offsets, s) || i >= end) end = -1;   // before the first or behind the last
      } else {
        s = i / a.per_seq;
        end = (long)(s + 1) * a.per_seq;
      }
      if (end >= 0) j = scalar_load(a.c.lens, s) - end + i;
      if (j >= 0 && j < paged_cap(a.c)) {
        const int p = scalar_load(a.c.table, s * a.c.tstride + (j >> a.c.lp));
        if ((unsigned)p < (unsigned)a.c.n_pages) pg = p;
      }
    }
    if (lane == 0) {
      page[w] = pg;
      slot[w] = (int)(j & ((1 << a.c.lp) - 1));
    }
  }
  if (a.pos) {
    const double inv = exp2(a.log2_theta * (-2.0 * (tid % HD) / D));
#pragma unroll
    for (int k = 0; k < (TPB * HD + 255) / 256; ++k)
      if ((k * 256 + tid) / HD < left) cs[(k * 256 + tid) / HD][tid % HD] = rope_cs(pos[k], inv);
  }
  __syncthreads();
  for (int b = 0; b < items; b += U * 256) {
    if (b) load(b);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int it = b + k * 256 + tid, p = it % HP, kv = it / HP & 1, r = it / (2 * HP), h = r / TPB, t = r % TPB;
      if (it >= items || t >= left || page[t] < 0) continue;
      if (!kv && a.pos) {
        float f0[EPP], f1[EPP];
        unpack16<IT>(x[k][0], f0);
        unpack16<IT>(x[k][1], f1);
        IT y0[EPP], y1[EPP];
#pragma unroll
        for (int e = 0; e < EPP; ++e) {
          const float2 c = cs[t][p * EPP + e];
          y0[e] = from_f32<IT>(f0[e] * c.x - f1[e] * c.y);
          y1[e] = from_f32<IT>(f1[e] * c.x + f0[e] * c.y);
        }
        __builtin_memcpy(&x[k][0], y0, 16);
        __builtin_memcpy(&x[k][1], y1, 16);
      }
      u32x4* dst = (u32x4*)((kv ? a.c.v : a.c.k) + ((((long)page[t] * H + h) << a.c.lp) + slot[t]) * (D * (long)sizeof(IT)));
      __builtin_nontemporal_store(x[k][0], dst + p);
      __builtin_nontemporal_store(x[k][1], dst + p + HP);
    }
  }
  if (a.c.beta)
    for (int it = tid; it < TPB * H; it += 256) {
      const int h = it / TPB, t = it % TPB;
      if (t < left && page[t] >= 0)
        a.c.beta[(((long)page[t] * H + h) << a.c.lp) + slot[t]] =
            a.nbeta ? a.nbeta[(t0 + t) * a.b_ts + h * a.b_hs] : 0.f;
    }
}

// ---------------------------------------------------------------------------
// Gather: block (x, h, z) copies PAGED_GATHER_ROWS entries of head h, a thread
// 16-byte pieces of keys and values.  Bound by the copy: 65536 entries of 8 heads of
// width 256 (1.07 GB) 201 us, 5.3 TB/s, with streaming stores, 206 with ordinary ones.
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
  const long i0 = ((long)blockIdx.z * gridDim.x + blockIdx.x) * PAGED_GATHER_ROWS;
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
    __builtin_nontemporal_store(x, (u32x4*)a.K + to);
    __builtin_nontemporal_store(y, (u32x4*)a.V + to);
  }
  if (a.beta && tid < PAGED_GATHER_ROWS && i0 + tid < a.n) {
    const long i = i0 + tid, j = a.start + i;
    const int page = j < len ? paged_page(a.c, a.seq, j) : -1;
    a.beta[(long)h * a.n + i] = page >= 0 ? a.c.beta[paged_row(a.c, page, h, j)] : 0.f;
  }
}

// ---------------------------------------------------------------------------
// Attention.  The entries of all sequences, cut into chunks of CH, form one line
// per KV head (a sequence counts PAGED_PAD chunks more, for what its rows cost
// beside its entries); G workgroups per head take equal contiguous parts of it,
// so that ragged lengths load the chip evenly and the host needs to know none
// of them.  A part may hold the end of one sequence, several whole ones and the
// start of another.  A sequence that lies in one part is finished there; the
// others leave partial sums (at most two per workgroup: the sequence it
// continues and the one it starts), joined by paged_merge_kernel.
//
// Within a part, wave w of 4 takes chunks w, w + 4, ... of the part's, whichever
// sequence they belong to, so that its loads run on from one sequence into the
// next; the waves' sums are added where a sequence ends.
//   S^T[entry][row]: entries are the matrix rows, query rows the columns, so a
//   lane owns query row l = lane % 16 and its running maximum and sum stay in
//   the lane.  Lane group lg = lane / 16 of entry l reads 16-byte pieces
//   4 i + lg of its key: the pairing of contraction indices is free, so pieces
//   feed the product as loaded, against the same pieces of the query row.
//   O^T[feature][row]: register j of tile kt of S^T holds entry 16 kt + 4 lg + j.
//   Lane l reads pieces l, 16 + l, ... of its lane group's entries, so a load
//   reads whole runs of value rows; output tile e holds feature e of every
//   lane's.
//   bf16: the lane's 8 entries are the 8 contraction indices of one
//   v_mfma_f32_16x16x32_bf16; the 16-bit transposition is v_perm in the lane.
//   Weights and rotated queries go in as three bf16 parts, all their 24 bits.  Two
//   parts would round each by 2^-17: 45.0 us instead of 48.0 for 8 causal rows of 5
//   sequences, 87 instead of 97 for 16 sequences of width 64 and 32 rows, no difference
//   above 1 % to 16 rows.  fp32: one v_mfma_f32_16x16x4_f32 per entry.
// Keys of the next chunk are loaded once the logits have used this one's, values
// once P.V has; page numbers are read two chunks ahead, before the keys of the
// next one, so that they are there with them (loads return in order).  A tile is
// read through a buffer descriptor of its valid rows: the others read as zeros
// and cost nothing, so the loop has no branch around a load and every wait counts only
// the loads behind it.
//
// SW: workgroup (h, s) of SW waves takes all of sequence s; nothing is joined.
//
// Bound by the entries' bytes: one sequence of 131136 entries of 8 heads of width 128
// (537 MB) 83 us, 6.5 TB/s, joined in 4.6; 48 of 1024 to 9216 of width 256 (1.48 GB)
// 230 us, 6.5 TB/s (a plain read reaches 7.1); with 32 rows 166 MB in 42 us, 3.9 TB/s:
// 372 registers leave one wave per SIMD, whose first and last chunks nothing hides.
// ---------------------------------------------------------------------------
struct PagedAttendArgs {
  PagedArgs c;
  const char* q;       // tokens of [H * group][d]
  long q_ts;           // bytes
  char* out;
  const double* qpos;  // NULL: q as given
  double log2_theta;
  int group, nq, causal;
  int nq_inv;          // 2^16 / nq + 1: r / nq = r nq_inv >> 16 for the rows r < 32
  float scale;
  int G;               // workgroups per KV head
  int by_seq;          // plan entries are per sequence (n_seqs <= G), else per workgroup
  int4* plan;          // (sequence in several parts or -1, its first and its last workgroup, 0)
  float* opart;        // [H][G][2][R][D]
  float* mpart;        // [H][G][2][R]
  float* lpart;
};

constexpr int PAGED_ROUND = 256;         // sequences whose lengths a wave holds at a time, four per lane
// Chunks that a sequence counts beside its own.  us at 0 / 2 / 4 / 6 / 8: 64 sequences
// of 5 to 16384 entries 113.5 / 101.5 / 96.7 / 96.1 / 97.0, 300 of 20 to 900 73.0 / 65.3 /
// 64.9 / 66.0 / 66.0, 48 of 1024 to 9216 of width 256 238 / 239 / 239 / 241 / 243, 5 of
// 1500 to 20011 with 32 rows 50.8 / 49.0 / 47.7 / 47.5 / 47.6: flat from 4 on.
constexpr int PAGED_PAD = 6;
constexpr float PAGED_SLACK = 6.f;       // weights reach e^6 before they are scaled back
constexpr float LOG2E = 1.4426950408889634f, LOG2E_REST = (float)(1.4426950408889634 - (double)LOG2E), LN2 = 0.6931471805599453f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Parts of the line: waves per workgroup, workgroups resident on a CU, and
// 16-entry tiles per chunk: 128 KB of keys and values in flight per CU (of width 64
// half of that: its rate is the same, and short sequences take less).
constexpr int paged_waves(int esize, int D, int NR) { return NR == 2 && D <= 128 && esize == 4 ? 8 : 4; }
constexpr int paged_resident(int D, int NR) { return NR == 1 && D <= 128 ? 2 : 1; }
constexpr int paged_tiles(int esize, int D, int NR) {
  return (NR == 1 && D == 64 ? 64 : 128) * 1024 / (paged_waves(esize, D, NR) * paged_resident(D, NR) * 32 * D * esize);
}
// Whole sequences: waves per workgroup (two per SIMD, or as the registers allow).
constexpr int paged_team(int D, int NR) { return NR == 1 && D <= 128 ? 8 : 4; }

// SW: waves of a workgroup that takes a whole sequence; 0: parts of the line; -1:
// parts, the entries' loads streaming past the caches.
template <class IT, int D, int NR, int SW>
struct PagedTile {
  static constexpr bool B16 = sizeof(IT) == 2;
  static constexpr int NW = SW > 0 ? SW : paged_waves(sizeof(IT), D, NR);
  static constexpr int PER_SIMD = SW == 1 ? (D <= 128 ? 2 : 1) : NW * (SW > 0 ? 1 : paged_resident(D, NR)) / 4;
  static constexpr int NKT = SW > 0 ? (B16 ? 2 : 1) : paged_tiles(sizeof(IT), D, NR);   // 16-entry tiles per chunk
  static constexpr int CH = 16 * NKT;
  static constexpr int AUX = SW < 0 ? 2 : 0;            // cache policy of the entries' loads: 2 non-temporal
  static constexpr int ROWB = D * (int)sizeof(IT);
  static constexpr int NP = ROWB / 64;                  // 16-byte pieces of a key per lane
  static constexpr int FPT = D / 16, VB = FPT * (int)sizeof(IT);
  static constexpr int PB = VB < 16 ? VB : 16, EPV = PB / (int)sizeof(IT);   // bytes and features of a piece of a value row
  static constexpr int QROW = ROWB + 16;                // query rows in LDS (padded: 16 rows at one piece)
  static constexpr int OROW = D + 4;
  static constexpr int QPART = 16 * NR * QROW;
};

// Dynamic LDS: the query rows (rotated bf16 ones in three parts), behind them the
// waves' sums [waves][R][OROW] or, before there are any, the queries' angles
// [nq][D / 2].  The sums take the rows' place where both do not fit 160 KB, and in
// workgroups of one wave, many of which share a CU.
constexpr bool paged_alias(int D, int NR, int SW) { return SW == 1 || D * NR > 256; }
template <class TL>
inline __host__ __device__ int paged_q_bytes(bool rot) { return (TL::B16 && rot ? 3 : 1) * TL::QPART; }
template <class TL, int D, int NR, int SW>
inline size_t paged_lds_bytes(int R, int nq, bool rot) {
  const size_t q = paged_q_bytes<TL>(rot), o = (size_t)TL::NW * R * TL::OROW * sizeof(float);
  const size_t angles = rot ? (size_t)nq * D / 2 * sizeof(float2) : 0;
  return paged_alias(D, NR, SW) ? std::max(q + angles, o) : q + std::max(angles, o);
}

// x as the sum of three bf16: each takes the leading 8 bits of what the ones before
// leave, 24 in all, and the remainders are exact, so nothing of an fp32 value is lost.
// (Cut instead of rounded: a mask and a subtraction each, words packed by v_perm.)
__device__ __forceinline__ void bf16_parts(const float (&x)[8], bf16x8 (&p)[3]) {
  float r[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) r[k] = x[k];
#pragma unroll
  for (int part = 0; part < 3; ++part) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __builtin_amdgcn_perm(__float_as_uint(r[2 * k + 1]), __float_as_uint(r[2 * k]), 0x07060302u);
    p[part] = __builtin_bit_cast(bf16x8, w);
    if (part < 2)
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] -= __uint_as_float(__float_as_uint(r[k]) & 0xffff0000u);
  }
}

// e^x = 2^y (1 + e ln 2), y = x log2(e) rounded and e what that left; zero below
// 2^-126.  2^y alone is off by 1.25 |x| 2^-24 of itself, at most 2^-25 of the largest
// weight: far below a bf16 output's step, so bf16 leaves e out (with it, 8 causal rows of
// 5 sequences 50.0 us instead of 48.0).
template <class IT>
__device__ __forceinline__ float exp_of(float x) {
  const float y = x * LOG2E, p = __builtin_amdgcn_exp2f(y);
  if (sizeof(IT) == 2) return p;
  const float e = fmaf(x, LOG2E_REST, fmaf(x, LOG2E, -y));
  return y < -126.f ? 0.f : fmaf(p, e * LN2, p);   // (x = -inf: y is, e a NaN; a NaN stays one)
}

// maximum over lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float groups_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// inclusive sum over the wave's lanes up to this one
__device__ __forceinline__ int lanes_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);   // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // last lane of the row before, into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // lane 31 into rows 2 and 3
  return x;
}

// Lane k of a wave holds values 4 k .. 4 k + 3 of a list: value i (uniform), and
// the last one at or below v in a rising list that starts at or below it.
__device__ __forceinline__ int list_get(const int (&x)[4], int i) {
  const int l = i >> 2, k = i & 3;
  const int a = __builtin_amdgcn_readlane(x[0], l), b = __builtin_amdgcn_readlane(x[1], l);
  const int c = __builtin_amdgcn_readlane(x[2], l), d = __builtin_amdgcn_readlane(x[3], l);
  const int ab = k & 1 ? b : a, cd = k & 1 ? d : c;
  return k & 2 ? cd : ab;
}
__device__ __forceinline__ int list_find(const int (&x)[4], int v) {
  const int l = max(__popcll(__ballot(x[0] <= v)) - 1, 0);
  int i = 4 * l;
#pragma unroll
  for (int k = 1; k < 4; ++k) i += __builtin_amdgcn_readlane(x[k], l) <= v;
  return i;
}

// N pieces of PB bytes (8 or 16) of a buffer from byte off, 16 PB apart, as words
template <int PB, int N, int AUX>
__device__ __forceinline__ void buffer_pieces(__amdgpu_buffer_rsrc_t r, int off, uint32_t (&w)[N * PB / 4]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (PB == 8) {
      const u32x2 u = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off + 16 * PB * i, 0, AUX));
      w[2 * i] = u.x;
      w[2 * i + 1] = u.y;
    } else {
      const u32x4 u = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * PB * i, 0, AUX));
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * i + e] = u[e];
    }
  }
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t paged_rows(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000);
}

template <class IT, int D, int NR, int SW>
__global__ __launch_bounds__((64 * PagedTile<IT, D, NR, SW>::NW), (PagedTile<IT, D, NR, SW>::PER_SIMD))
void paged_attend_kernel(PagedAttendArgs a) {
  using TL = PagedTile<IT, D, NR, SW>;
  constexpr bool SINGLE = SW > 0;
  constexpr int NKT = TL::NKT, CH = TL::CH, NP = TL::NP, FPT = TL::FPT, VB = TL::VB, ROWB = TL::ROWB, NW = TL::NW;
  constexpr int QROW = TL::QROW, OROW = TL::OROW, NT = 64 * NW, HD = D / 2;
  constexpr bool ALIAS = paged_alias(D, NR, SW);
  extern __shared__ float4 paged_smem[];
  char* qs = (char*)paged_smem;                  // [16 NR][QROW], rotated bf16 rows: three parts of that
  __shared__ float wm[NW][16 * NR], wl[NW][16 * NR];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const int l = lane & 15, lg = lane >> 4;
  const int h = blockIdx.x, g = SINGLE ? 0 : blockIdx.y, R = a.group * a.nq, Hq = a.c.H * a.group;
  const int n_seqs = a.c.n_seqs, pad = n_seqs > 1 ? PAGED_PAD : 0;
  const bool rot = a.qpos != nullptr;
  float* osum = (float*)(qs + (ALIAS ? 0 : paged_q_bytes<TL>(rot)));   // [NW][R][OROW]
  float2* cs = (float2*)(qs + paged_q_bytes<TL>(rot));   // [nq][D / 2] (cos, sin) of the queries, where the sums come later
  const int koff = l * ROWB + lg * 16, voff = 4 * lg * ROWB + l * TL::PB;
  auto head_of = [&](int r) { return r * a.nq_inv >> 16; };   // of the group; the query is r - nq * that
  auto out_row = [&](int s, int r) {
    const int hr = head_of(r);
    return (((long)s * a.nq + r - hr * a.nq) * Hq + h * a.group + hr) * D;
  };

  // ---- a sequence's query rows, row g * nq + i query i of head h * group + g: a
  // thread's pairs of 16-byte pieces D / 2 apart, the members of the rotated pairs
  constexpr int HP = ROWB / 32, EPP = 16 / (int)sizeof(IT), QI = (16 * NR * HP + NT - 1) / NT;
  u32x4 qr[QI][2];
  // a thread's angles belong to one pair where the threads are a multiple of the pairs
  const double inv_freq = rot ? exp2(a.log2_theta * (-2.0 * (tid % HD) / D)) : 0.0;
  auto load_q = [&](int s) {
#pragma unroll
    for (int k = 0; k < QI; ++k) {
      const int e = k * NT + tid, r = min(e / HP, R - 1), hr = head_of(r);   // (rows past R repeat the last one)
      const u32x4* q = (const u32x4*)(a.q + ((long)s * a.nq + r - hr * a.nq) * a.q_ts + (h * a.group + hr) * ROWB);
      qr[k][0] = q[e % HP];
      qr[k][1] = q[e % HP + HP];
    }
  };
  auto stage_q = [&](int s) {   // rotated, in LDS; ends with a barrier
    if (rot) {
      for (int e = tid; e < a.nq * HD; e += NT)
        cs[e] = rope_cs(a.qpos[(long)s * a.nq + e / HD],
                        NT % HD == 0 ? inv_freq : exp2(a.log2_theta * (-2.0 * (e % HD) / D)));
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < QI; ++k) {
      const int e = k * NT + tid, r = e / HP, j = e % HP * EPP;
      if (16 * NR * HP % NT && r >= 16 * NR) break;
      if (rot) {
        const int i = min(r, R - 1);
        const float2* c = cs + (i - head_of(i) * a.nq) * HD + j;
        float x0[EPP], x1[EPP];
        unpack16<IT>(qr[k][0], x0);
        unpack16<IT>(qr[k][1], x1);
#pragma unroll
        for (int u = 0; u < EPP; ++u) {
          const float y = x0[u] * c[u].x - x1[u] * c[u].y;
          x1[u] = x1[u] * c[u].x + x0[u] * c[u].y;
          x0[u] = y;
        }
        if constexpr (TL::B16) {
          bf16x8 p0[3], p1[3];
          bf16_parts(x0, p0);
          bf16_parts(x1, p1);
          qr[k][0] = __builtin_bit_cast(u32x4, p0[0]);
          qr[k][1] = __builtin_bit_cast(u32x4, p1[0]);
#pragma unroll
          for (int part = 1; part < 3; ++part) {
            *(bf16x8*)(qs + part * TL::QPART + r * QROW + 16 * (e % HP)) = p0[part];
            *(bf16x8*)(qs + part * TL::QPART + r * QROW + 16 * (e % HP + HP)) = p1[part];
          }
        } else {
          qr[k][0] = u32x4{__float_as_uint(x0[0]), __float_as_uint(x0[1]), __float_as_uint(x0[2]), __float_as_uint(x0[3])};
          qr[k][1] = u32x4{__float_as_uint(x1[0]), __float_as_uint(x1[1]), __float_as_uint(x1[2]), __float_as_uint(x1[3])};
        }
      }
      *(u32x4*)(qs + r * QROW + 16 * (e % HP)) = qr[k][0];
      *(u32x4*)(qs + r * QROW + 16 * (e % HP + HP)) = qr[k][1];
    }
    __syncthreads();
  };

  // ---- this workgroup's part of the line
  const int cap = (int)paged_cap(a.c);
  int lens[4];    // of the round's sequences, four per lane
  auto load_lens = [&](int base) {
    const auto r = paged_rows(a.c.lens + base, 4 * min(PAGED_ROUND, n_seqs - base));   // (past them: zeros)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      lens[k] = min(max((int)__builtin_amdgcn_raw_buffer_load_b32(r, 16 * lane + 4 * k, 0, 0), 0), cap);
  };
  auto chunks = [&](int len) { return (len + CH - 1) / CH; };
  // workgroups with a part, the chunks (with pads) of one, how many take one more, this part's cuts
  int active = 0, share = 0, more = 0, v0 = 0, v1 = 0;
  auto cuts = [&](int T, int some) {        // of the sums over all sequences
    // a workgroup takes a chunk per wave, but not two short sequences, before another one starts
    active = min(a.G, max((T + NW - 1) / NW, some));
    if (g < active) {
      share = (T + pad * some) / active;
      more = T + pad * some - share * active;
      v0 = g * share + min(g, more);
      v1 = v0 + share + (g < more);
    }
  };
  if (!SINGLE && n_seqs > PAGED_ROUND) {
    int n = 0, some = 0;
    for (int base = 0; base < n_seqs; base += PAGED_ROUND) {
      load_lens(base);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        n += chunks(lens[k]);
        some += lens[k] > 0;
      }
    }
    cuts(__builtin_amdgcn_readlane(lanes_scan(n), 63), __builtin_amdgcn_readlane(lanes_scan(some), 63));
  }
  int4 goes_on = make_int4(-1, 0, 0, 0);
  int line = 0, padded = 0;   // chunks in front of the round, without and with pads
  for (int base = SINGLE ? blockIdx.y : 0; base < n_seqs; base += PAGED_ROUND) {
    const int cnt = SINGLE ? 1 : min(PAGED_ROUND, n_seqs - base);
    int first[4], padded_first[4], lo, hi;   // of the round's sequences on the line; the part's chunks in the round
    struct Chunk {
      int i, c, len;    // sequence of the round (none: PAGED_ROUND), chunk in it, its length
      int p[NKT];       // page numbers of its tiles, as read
    };
    auto load_pages = [&](Chunk& k, int i, int c) {   // of chunk c of sequence i (past its end: some page number)
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
        k.p[kt] = a.c.table[(base + i) * a.c.tstride + min((c * CH + 16 * kt) >> a.c.lp, a.c.max_pages - 1)];
    };
    Chunk cur_chunk, nxt;
    if constexpr (SINGLE) {   // rows, page numbers and length are on their way together
      load_q(base);
      load_pages(cur_chunk, 0, w);
      load_pages(nxt, 0, w + NW);
      __builtin_amdgcn_sched_barrier(0);
      lens[0] = min(max(scalar_load(a.c.lens, base), 0), cap);
      lo = 0;
      hi = chunks(lens[0]);
    } else {
      load_lens(base);
      int n = 0, some = 0, before = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        n += chunks(lens[k]);
        const unsigned long full = __ballot(lens[k] > 0);
        some += __popcll(full);
        before += __popcll(full & ((1UL << lane) - 1));
      }
      const int incl = lanes_scan(n), total = __builtin_amdgcn_readlane(incl, 63);
      if (n_seqs <= PAGED_ROUND) cuts(total, some);
      int f = line + incl - n, v = padded + incl - n + pad * before;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        first[k] = f;
        padded_first[k] = v;
        f += chunks(lens[k]);
        v += chunks(lens[k]) + (lens[k] > 0 ? pad : 0);
      }
      const int line_end = line + total, padded_end = padded + total + pad * some;
      auto cut = [&](int v) {   // the first chunk at or behind place v of the line with pads
        const int i = list_find(padded_first, v);
        const int c = list_get(first, i) + max(0, v - list_get(padded_first, i) - pad);
        return v <= padded ? line : v >= padded_end ? line_end : c;
      };
      lo = cut(v0);
      hi = cut(v1);
      line = line_end;
      padded = padded_end;
    }
    auto len_of = [&](int i) { return SINGLE ? lens[0] : list_get(lens, i); };
    // rows of sequences without entries
    for (int k = SINGLE ? 0 : g; k < cnt; k += SINGLE ? 1 : a.G)
      if (len_of(k) == 0) {
        for (int e = tid; e < R * (ROWB / 16); e += NT) {
          const u32x4 z = {0, 0, 0, 0};
          ((u32x4*)(a.out + out_row(base + k, e / (ROWB / 16)) * (long)sizeof(IT)))[e % (ROWB / 16)] = z;
        }
        if (!SINGLE && h == 0 && tid == 0 && a.by_seq) a.plan[base + k] = make_int4(-1, 0, 0, 0);
      }
    // ---- the stream of this wave's chunks
    auto locate = [&](Chunk& k, int u) {   // chunk u of the line: the last sequence that starts at or before it
      const int i = SINGLE ? 0 : min(list_find(first, u), cnt - 1);
      const bool there = u < hi;
      k.i = there ? i : PAGED_ROUND;
      k.len = there ? len_of(i) : 0;
      k.c = SINGLE ? u : max(u - list_get(first, i), 0);
      return i;
    };
    auto lookup = [&](int u) {
      Chunk k;
      const int i = locate(k, u);
      load_pages(k, i, k.c);
      return k;
    };
    struct Tiles {
      int i, c;
      int nv[NKT];      // valid entries of each tile
      long row[NKT];    // rows of the pages in front of the tile
    };
    auto resolve = [&](const Chunk& k) {
      Tiles t;
      t.i = k.i;
      t.c = k.c;
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const int j = k.c * CH + 16 * kt, p = uniform(k.p[kt]);
        const bool ok = j < k.len && (unsigned)p < (unsigned)a.c.n_pages;
        t.nv[kt] = ok ? min(16, k.len - j) : 0;
        t.row[kt] = (((long)(ok ? p : 0) * a.c.H + h) << a.c.lp) + (ok ? j & ((1 << a.c.lp) - 1) : 0);
      }
      return t;
    };
    u32x4 kp[NKT][NP];
    f32x4 bias[NKT];
    uint32_t vr[NKT * 4][VB / 4];
    // (the offsets are opaque to the compiler, which would keep every sum of one with
    // a constant in a register of its own instead of in the load)
    auto load_k = [&](const Tiles& k) {
      int off = koff, boff = 16 * lg;
      asm volatile("" : "+v"(off), "+v"(boff));
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const auto r = paged_rows(a.c.k + k.row[kt] * ROWB, k.nv[kt] * ROWB);
#pragma unroll
        for (int i = 0; i < NP; ++i)
          kp[kt][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 64 * i, 0, TL::AUX));
        bias[kt] = __builtin_bit_cast(
            f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       paged_rows(a.c.beta + k.row[kt], a.c.beta && k.nv[kt] > 0 ? 16 * 4 : 0), boff, 0, 0));
      }
    };
    auto load_v = [&](const Tiles& k) {
      int off = voff;
      asm volatile("" : "+v"(off));
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const auto r = paged_rows(a.c.v + k.row[kt] * ROWB, k.nv[kt] * ROWB);
#pragma unroll
        for (int j = 0; j < 4; ++j) buffer_pieces<TL::PB, VB / TL::PB, TL::AUX>(r, off + j * ROWB, vr[kt * 4 + j]);
      }
    };
    if (lo < hi) {
      int u = lo + w, i = SINGLE ? 0 : list_find(first, lo), at = lo;
      if constexpr (SINGLE) {
        locate(cur_chunk, u);
        locate(nxt, u + NW);
      } else {
        load_q(base + i);
        cur_chunk = lookup(u);
        nxt = lookup(u + NW);
      }
      Tiles cur = resolve(cur_chunk);
      load_k(cur);
      __builtin_amdgcn_sched_barrier(0);   // (loads stay in this order: their waits count the ones behind)
      load_v(cur);
      __builtin_amdgcn_sched_barrier(0);
      while (true) {   // the part's sequences that have entries
        const int len = len_of(i), s0 = SINGLE ? 0 : list_get(first, i), s1 = s0 + chunks(len);
        const int s = base + i, end = min(s1, hi);
        stage_q(s);
        f32x4 o[NR][FPT];
        float m[NR], ls[NR];
        int lim[NR];   // last entry that this lane's row sees
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
          m[rt] = -INFINITY;
          ls[rt] = 0.f;
          lim[rt] = a.causal ? len - a.nq + 16 * rt + l - head_of(16 * rt + l) * a.nq : len - 1;
#pragma unroll
          for (int e = 0; e < FPT; ++e) o[rt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int open = a.causal ? len - a.nq : len - 1;   // every row sees the entries up to this one
        while (cur.i == i) {
          u += NW;
          const Chunk third = lookup(u + NW);
          __builtin_amdgcn_sched_barrier(0);
          // ---- logits
          f32x4 x[NR][NKT];
#pragma unroll
          for (int rt = 0; rt < NR; ++rt)
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt) x[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) {
              const u32x4 qv = *(const u32x4*)(qs + (16 * rt + l) * QROW + 64 * p + 16 * lg);
#pragma unroll
              for (int kt = 0; kt < NKT; ++kt) {
                if constexpr (TL::B16) {
                  x[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                      __builtin_bit_cast(bf16x8, kp[kt][p]), __builtin_bit_cast(bf16x8, qv), x[rt][kt], 0, 0, 0);
                } else {
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    x[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kp[kt][p][e]),
                                                                     __uint_as_float(qv[e]), x[rt][kt], 0, 0, 0);
                }
              }
            }
          if (TL::B16 && rot) {
#pragma unroll
            for (int part = 1; part < 3; ++part)
#pragma unroll
              for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int rt = 0; rt < NR; ++rt) {
                  const u32x4 qv = *(const u32x4*)(qs + part * TL::QPART + (16 * rt + l) * QROW + 64 * p + 16 * lg);
#pragma unroll
                  for (int kt = 0; kt < NKT; ++kt)
                    x[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8, kp[kt][p]), __builtin_bit_cast(bf16x8, qv), x[rt][kt], 0, 0, 0);
                }
          }
          f32x4 bc[NKT];
#pragma unroll
          for (int kt = 0; kt < NKT; ++kt) bc[kt] = bias[kt];
          const Tiles next = resolve(nxt);
          load_k(next);
          __builtin_amdgcn_sched_barrier(0);
          // ---- online softmax of this lane's rows over its entries.  The sums stay
          // relative to m, a logit of the row, until one exceeds it by PAGED_SLACK.
          bool full = cur.c * CH + CH - 1 <= open;
#pragma unroll
          for (int kt = 0; kt < NKT; ++kt) full = full && cur.nv[kt] == 16;
          float cm[NR];
          bool grows = false;
#pragma unroll
          for (int rt = 0; rt < NR; ++rt) {
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
              for (int j = 0; j < 4; ++j) x[rt][kt][j] = fmaf(x[rt][kt][j], a.scale, bc[kt][j]);
            if (!full) {
#pragma unroll
              for (int kt = 0; kt < NKT; ++kt) {
                const int seen = min(cur.nv[kt], lim[rt] - (cur.c * CH + 16 * kt) + 1) - 4 * lg;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[rt][kt][j] = j < seen ? x[rt][kt][j] : -INFINITY;
              }
            }
            cm[rt] = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
              for (int j = 0; j < 4; ++j) cm[rt] = fmaxf(cm[rt], x[rt][kt][j]);
            cm[rt] = groups_max(cm[rt]);
            grows = grows || cm[rt] > m[rt] + PAGED_SLACK;
          }
          if (__any(grows)) {
#pragma unroll
            for (int rt = 0; rt < NR; ++rt) {
              const float mn = fmaxf(m[rt], cm[rt]);
              const float al = exp_of<IT>(m[rt] - (mn == -INFINITY ? 0.f : mn));
              m[rt] = mn;
              ls[rt] *= al;
#pragma unroll
              for (int e = 0; e < FPT; ++e) o[rt][e] *= al;
            }
          }
#pragma unroll
          for (int rt = 0; rt < NR; ++rt) {
            const float ref = m[rt] == -INFINITY ? 0.f : m[rt];
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                x[rt][kt][j] = exp_of<IT>(x[rt][kt][j] - ref);
                ls[rt] += x[rt][kt][j];   // (this lane's entries; its lane groups are added at the end)
              }
          }
          // ---- P.V
          if constexpr (TL::B16) {
#pragma unroll
            for (int k2 = 0; k2 < NKT; k2 += 2) {
              bf16x8 pp[NR][3];
#pragma unroll
              for (int rt = 0; rt < NR; ++rt) {
                const f32x4 &a0 = x[rt][k2], &a1 = x[rt][k2 + 1];
                const float p[8] = {a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
                bf16_parts(p, pp[rt]);
              }
#pragma unroll
              for (int e = 0; e < FPT; e += 2) {   // an even and an odd feature of one word
                u32x4 t0, t1;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const uint32_t a0 = vr[4 * k2 + 2 * k][e >> 1], a1 = vr[4 * k2 + 2 * k + 1][e >> 1];
                  t0[k] = __builtin_amdgcn_perm(a1, a0, 0x05040100u);
                  t1[k] = __builtin_amdgcn_perm(a1, a0, 0x07060302u);
                }
                const bf16x8 w0 = __builtin_bit_cast(bf16x8, t0), w1 = __builtin_bit_cast(bf16x8, t1);
#pragma unroll
                for (int rt = 0; rt < NR; ++rt)
#pragma unroll
                  for (int part = 0; part < 3; ++part) {
                    o[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w0, pp[rt][part], o[rt][e], 0, 0, 0);
                    o[rt][e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w1, pp[rt][part], o[rt][e + 1], 0, 0, 0);
                  }
              }
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4 * NKT; ++k)
#pragma unroll
              for (int e = 0; e < FPT; ++e)
#pragma unroll
                for (int rt = 0; rt < NR; ++rt)
                  o[rt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[k][e]), x[rt][k >> 2][k & 3],
                                                                  o[rt][e], 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
          load_v(next);
          __builtin_amdgcn_sched_barrier(0);
          cur = next;
          nxt = third;
        }
        // ---- the waves' sums into LDS, then added, the next rows on their way
        const bool last = SINGLE || end == hi;
        const int ni = last ? i : list_find(first, end);
        if (!last) load_q(base + ni);
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
          ls[rt] += __shfl_xor(ls[rt], 16);
          ls[rt] += __shfl_xor(ls[rt], 32);
        }
        if (ALIAS) __syncthreads();   // every wave has read the query rows
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
          const int r = 16 * rt + l;
          if (lg == 0) {
            wm[w][r] = m[rt];
            wl[w][r] = ls[rt];
          }
          if (r < R) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float* dst = osum + (w * R + r) * OROW + (4 * lg + j) * TL::EPV;
#pragma unroll
              for (int e = 0; e < FPT; e += 4)
                *(float4*)(dst + e / TL::EPV * 16 * TL::EPV + e % TL::EPV) = make_float4(o[rt][e][j], o[rt][e + 1][j], o[rt][e + 2][j], o[rt][e + 3][j]);
            }
          }
        }
        __syncthreads();   // (also: every wave has read the query rows)
        const bool starts = at == s0, whole = SINGLE || (starts && end == s1);
        const long slot = ((long)h * a.G + g) * 2 + (starts ? 1 : 0);
        for (int e = tid; e < R * (D / 4); e += NT) {
          const int r = e / (D / 4), x = e % (D / 4) * 4;
          float M = wm[0][r];
#pragma unroll
          for (int k = 1; k < NW; ++k) M = fmaxf(M, wm[k][r]);
          const float ref = M == -INFINITY ? 0.f : M;
          float L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < NW; ++k) {
            const float sc = exp_of<IT>(wm[k][r] - ref);
            const float4 y = *(const float4*)(osum + (k * R + r) * OROW + x);
            L += sc * wl[k][r];
            acc[0] += sc * y.x;
            acc[1] += sc * y.y;
            acc[2] += sc * y.z;
            acc[3] += sc * y.w;
          }
          if (whole) {
            const float inv = L == 0.f ? 0.f : 1.f / L;   // a row that sees nothing; a NaN stays one
            IT* dst = (IT*)a.out + out_row(s, r) + x;
#pragma unroll
            for (int k = 0; k < 4; ++k) dst[k] = from_f32<IT>(acc[k] * inv);
          } else {
            *(float4*)(a.opart + (slot * R + r) * D + x) = make_float4(acc[0], acc[1], acc[2], acc[3]);
            if (x == 0) {
              a.mpart[slot * R + r] = M;
              a.lpart[slot * R + r] = L;
            }
          }
        }
        if (!SINGLE && starts) {
          const int v = list_get(padded_first, i) + pad + s1 - s0;   // behind its last chunk
          // the workgroup of place v - 1
          const int to = v <= more * (share + 1) ? (v - 1) / (share + 1) : more + (v - 1 - more * (share + 1)) / share;
          const int4 p = whole ? make_int4(-1, 0, 0, 0) : make_int4(s, g, to, 0);
          if (a.by_seq) {
            if (h == 0 && tid == 0) a.plan[s] = p;
          } else if (!whole) {
            goes_on = p;
          }
        }
        if (last) break;
        i = ni;
        at = end;
        if (ALIAS || rot) __syncthreads();   // the sums have been read before the next sequence's rows or angles
      }
    }
    if (SINGLE) break;
    __syncthreads();   // the last sequence's sums have been read
  }
  if (!SINGLE && h == 0 && tid == 0 && !a.by_seq) a.plan[g] = goes_on;
}

// Joins the partial sums of the sequences that lie in several parts: block
// (r, h, k) row r of plan entry k.  Groups of D / 4 lanes take every NG-th part:
// many where few blocks read many parts each.
constexpr int PAGED_MERGE_THREADS = 1024;   // at most, 256 at least

template <class IT, int D>
__global__ __launch_bounds__(PAGED_MERGE_THREADS) void paged_merge_kernel(PagedAttendArgs a) {
  constexpr int LPR = D / 4, MAX = PAGED_MERGE_THREADS / LPR;
  __shared__ float4 acc[MAX][LPR];
  __shared__ float sum[MAX], top[MAX];
  const int NG = blockDim.x / LPR;
  const int r = blockIdx.x, h = blockIdx.y, R = a.group * a.nq, Hq = a.c.H * a.group;
  const int4 p = a.plan[blockIdx.z];
  if (p.x < 0) return;
  const int x = threadIdx.x % LPR, k = threadIdx.x / LPR, n = p.z - p.y + 1;
  // part 0: the start, slot 1 of its workgroup; part i: slot 0 of the i-th one behind it
  auto at = [&](int i) { return (((long)h * a.G + p.y + i) * 2 + (i == 0 ? 1 : 0)) * R + r; };
  float M = -INFINITY, L = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = k; i < n; i += NG) {
    const float m = a.mpart[at(i)], l = a.lpart[at(i)];
    const float4 v = *(const float4*)(a.opart + at(i) * D + 4 * x);
    const float mn = fmaxf(M, m), ref = mn == -INFINITY ? 0.f : mn;
    const float so = exp_of<IT>(M - ref), sn = exp_of<IT>(m - ref);
    M = mn;
    L = L * so + l * sn;
    y[0] = y[0] * so + v.x * sn;
    y[1] = y[1] * so + v.y * sn;
    y[2] = y[2] * so + v.z * sn;
    y[3] = y[3] * so + v.w * sn;
  }
  acc[k][x] = make_float4(y[0], y[1], y[2], y[3]);
  if (x == 0) {
    sum[k] = L;
    top[k] = M;
  }
  __syncthreads();
  if (k == 0) {
    float S = 0.f, z[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < NG; ++i) M = fmaxf(M, top[i]);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll 4
    for (int i = 0; i < NG; ++i) {
      const float4 v = acc[i][x];
      const float sc = exp_of<IT>(top[i] - ref);
      S += sum[i] * sc;
      z[0] += v.x * sc;
      z[1] += v.y * sc;
      z[2] += v.z * sc;
      z[3] += v.w * sc;
    }
    const float inv = S == 0.f ? 0.f : 1.f / S;
    IT* dst = (IT*)a.out + (((long)p.x * a.nq + r % a.nq) * Hq + h * a.group + r / a.nq) * D + 4 * x;
#pragma unroll
    for (int u = 0; u < 4; ++u) dst[u] = from_f32<IT>(z[u] * inv);
  }
}

}  // namespace still
