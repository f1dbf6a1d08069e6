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
// Attention.  The entries of all sequences, cut into chunks of CH, form one line
// per KV head; G workgroups per head take equal contiguous parts of it, so that
// ragged lengths load the chip evenly and the host needs to know none of them.
// A part may hold the end of one sequence, several whole ones and the start of
// another.  A sequence that lies in one part is finished there; the others
// leave partial sums (at most two per workgroup: the sequence it continues and
// the one it starts), joined by paged_merge_kernel.
//
// Within a part, wave w of 4 takes chunks w, w + 4, ... of a sequence.
//   S^T[entry][row]: entries are the matrix rows, query rows the columns, so a
//   lane owns query row l = lane % 16 and its running maximum and sum stay in
//   the lane.  Lane group lg = lane / 16 of entry l reads 16-byte pieces
//   4 i + lg of its key: the pairing of contraction indices is free, so pieces
//   feed the product as loaded, against the same pieces of the query row.
//   O^T[feature][row]: register j of tile kt of S^T holds entry 16 kt + 4 lg + j.
//   Lane l reads features [l D / 16, ..) of its lane group's entries, so value
//   rows are read whole too, and output tile e holds features e, D / 16 + e, ...
//   bf16: the lane's 8 entries are the 8 contraction indices of one
//   v_mfma_f32_16x16x32_bf16; the 16-bit transposition is v_perm in the lane.
//   Weights (and rotated queries) go in as two bf16 parts, hi + lo, 16 bits of
//   mantissa: one part alone would round each by 2^-9.  fp32: one
//   v_mfma_f32_16x16x4_f32 per entry.
// Keys of the next chunk are loaded once the logits have used this one's, values
// once P.V has: 32 bytes d of each wave are in flight throughout.
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
  int G;               // workgroups per KV head
  int2* plan;          // [G]: (sequence that starts in workgroup g and goes on, its last workgroup), or (-1, 0)
  float* opart;        // [H][G][2][R][D]
  float* mpart;        // [H][G][2][R]
  float* lpart;
};

constexpr int PAGED_WAVES = 4;
constexpr float LOG2E = 1.4426950408889634f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <class IT, int D>
struct PagedTile {
  static constexpr bool B16 = sizeof(IT) == 2;
  static constexpr int NKT = B16 ? 2 : 1;               // 16-entry tiles per chunk
  static constexpr int CH = 16 * NKT;
  static constexpr int ROWB = D * (int)sizeof(IT);
  static constexpr int NP = ROWB / 64;                  // 16-byte pieces of a key per lane
  static constexpr int FPT = D / 16, VB = FPT * (int)sizeof(IT);
  static constexpr int QROW = ROWB + 16;                // query rows in LDS (padded: 16 rows at one piece)
  static constexpr int OROW = D + 4;
};

// entries per chunk, for the host
inline int paged_chunk(bool fp32) { return fp32 ? PagedTile<float, 64>::CH : PagedTile<bf16, 64>::CH; }

// dynamic LDS: the query rows (bf16: two parts), later the waves' sums [4][R][OROW]
template <class IT, int D>
inline size_t paged_lds_bytes(int R) {
  using TL = PagedTile<IT, D>;
  const size_t q = (size_t)(R <= 16 ? 16 : 32) * TL::QROW * (TL::B16 ? 2 : 1);
  return std::max(q, (size_t)PAGED_WAVES * R * TL::OROW * sizeof(float));
}

// fast base-2 exponential (results below 2^-126 are zero)
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long uniform(long x) {
  return (long)(((unsigned long)(unsigned)uniform((int)(x >> 32)) << 32) | (unsigned)uniform((int)x));
}

// This workgroup's part [c0, c1) of the T chunks: the sequence s that holds c0
// and that sequence's first chunk.  The lengths are scanned by the block.
struct PagedPart {
  long T, c0, c1, at;   // at: first chunk of sequence s
  int s, active;        // active: workgroups per head that have a part
};

template <int CH>
__device__ __forceinline__ PagedPart paged_part(const PagedArgs& a, int g, int G) {
  __shared__ long wsum[PAGED_WAVES];
  __shared__ long found_at;
  __shared__ int found;
  constexpr int NT = 64 * PAGED_WAVES;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  auto chunks = [&](int s) -> long { return s < a.n_seqs ? (paged_len(a, s) + CH - 1) / CH : 0; };
  long mine = 0;
  for (int s = tid; s < a.n_seqs; s += NT) mine += chunks(s);
  long sum = mine;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
  if (lane == 0) wsum[w] = sum;
  __syncthreads();
  PagedPart p;
  p.T = 0;
#pragma unroll
  for (int i = 0; i < PAGED_WAVES; ++i) p.T += wsum[i];
  p.T = uniform(p.T);
  // a workgroup takes four chunks (one per wave) before another one starts
  p.active = (int)min((long)G, (p.T + PAGED_WAVES - 1) / PAGED_WAVES);
  p.c0 = p.c1 = p.at = 0;
  p.s = 0;
  if (g >= p.active) return p;
  p.c0 = g * p.T / p.active;
  p.c1 = (g + 1) * p.T / p.active;
  long before = 0;   // chunks of the sequences before this round's
  for (int base = 0; base < a.n_seqs; base += NT) {
    __syncthreads();   // wsum of the round before has been read
    const long n = base == 0 && a.n_seqs <= NT ? mine : chunks(base + tid);
    long incl = n;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const long x = __shfl_up(incl, off);
      if (lane >= off) incl += x;
    }
    if (lane == 63) wsum[w] = incl;
    __syncthreads();
    long first = before + incl - n, total = 0;
#pragma unroll
    for (int i = 0; i < PAGED_WAVES; ++i) {
      if (i < w) first += wsum[i];
      total += wsum[i];
    }
    if (first <= p.c0 && p.c0 < first + n) {   // one thread of one round
      found = base + tid;
      found_at = first;
    }
    before += total;
    if (before > p.c0) break;
  }
  __syncthreads();
  p.s = uniform(found);
  p.at = uniform(found_at);
  return p;
}

template <class IT, int D, int NR>
__global__ __launch_bounds__(64 * PAGED_WAVES, D * NR <= 128 ? 2 : 1) void paged_attend_kernel(PagedAttendArgs a) {
  using TL = PagedTile<IT, D>;
  constexpr int NKT = TL::NKT, CH = TL::CH, NP = TL::NP, FPT = TL::FPT, VB = TL::VB, ROWB = TL::ROWB;
  constexpr int QROW = TL::QROW, OROW = TL::OROW, NT = 64 * PAGED_WAVES, HD = D / 2;
  extern __shared__ float4 paged_smem[];
  char* qs = (char*)paged_smem;                  // [16 NR][QROW], bf16: the same again for the low parts
  char* ql = qs + 16 * NR * QROW;
  float* osum = (float*)paged_smem;              // [4][R][OROW]
  __shared__ float wm[PAGED_WAVES][16 * NR], wl[PAGED_WAVES][16 * NR];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const int l = lane & 15, lg = lane >> 4;
  const int h = blockIdx.x, g = blockIdx.y, R = a.group * a.nq, Hq = a.c.H * a.group;
  const bool rot = a.qpos != nullptr;
  // rows of sequences without entries
  for (int s = g; s < a.c.n_seqs; s += a.G)
    if (a.c.lens[s] <= 0)
      for (int e = tid; e < R * (ROWB / 16); e += NT) {
        const int r = e / (ROWB / 16), x = e % (ROWB / 16);
        const u32x4 z = {0, 0, 0, 0};
        ((u32x4*)(a.out + (((long)s * a.nq + r % a.nq) * Hq + h * a.group + r / a.nq) * ROWB))[x] = z;
      }
  const PagedPart part = paged_part<CH>(a.c, g, a.G);
  int2 goes_on = make_int2(-1, 0);
  long at = part.at, left = part.c1 - part.c0;
  int f0 = (int)(part.c0 - part.at);
  const int koff = l * ROWB + lg * 16, voff = 4 * lg * ROWB + l * VB;
  for (int s = part.s; left > 0 && s < a.c.n_seqs; ++s, f0 = 0) {
    const int len = uniform(paged_len(a.c, s)), ns = (len + CH - 1) / CH;
    const int f1 = (int)min((long)ns, f0 + left);
    left -= f1 - f0;
    at += ns;
    if (f0 >= f1) continue;
    // ---- chunks: where their 16-entry tiles lie, how many entries of each count
    struct Chunk {
      long row[NKT];
      int nv[NKT];
    };
    auto lookup = [&](int c) {
      Chunk k;
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const long j = (long)c * CH + 16 * kt;
        const int p = uniform(j < len ? paged_page(a.c, s, j) : -1);
        k.nv[kt] = p < 0 ? 0 : min(16, (int)(len - j));
        k.row[kt] = (((long)max(p, 0) * a.c.H + h) << a.c.lp) + (p < 0 ? 0 : j & ((1 << a.c.lp) - 1));
      }
      return k;
    };
    u32x4 kp[NKT][NP];
    float4 bias[NKT];
    uint32_t vr[NKT * 4][VB / 4];
    auto load_k = [&](const Chunk& k) {
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const char* base = a.c.k + k.row[kt] * ROWB;
#pragma unroll
        for (int i = 0; i < NP; ++i) kp[kt][i] = *(const u32x4*)(base + koff + 64 * i);
        bias[kt] = a.c.beta ? *(const float4*)(a.c.beta + k.row[kt] + 4 * lg) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    };
    auto load_v = [&](const Chunk& k) {
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const char* base = a.c.v + k.row[kt] * ROWB;
#pragma unroll
        for (int j = 0; j < 4; ++j) load_words<VB>(base + voff + j * ROWB, vr[kt * 4 + j]);
      }
    };
    Chunk cur = lookup(min(f0 + w, f1 - 1));
    load_k(cur);
    load_v(cur);
    // ---- query rows into LDS: row g * nq + i is query i of head h * group + g
    for (int e = tid; e < 16 * NR * HD; e += NT) {
      const int r = e / HD, j = e % HD;
      float x0 = 0.f, x1 = 0.f;
      if (r < R) {
        const long t = (long)s * a.nq + r % a.nq;
        const IT* q = (const IT*)(a.q + t * a.q_ts) + (long)(h * a.group + r / a.nq) * D;
        x0 = to_f32(q[j]);
        x1 = to_f32(q[j + HD]);
        if (rot) {
          const float2 cs = rope_cs(a.qpos[t], exp2(a.log2_theta * (-2.0 * j / D)));
          const float y0 = x0 * cs.x - x1 * cs.y;
          x1 = x1 * cs.x + x0 * cs.y;
          x0 = y0;
        }
      }
      if constexpr (TL::B16) {
        const __bf16 h0 = (__bf16)x0, h1 = (__bf16)x1;
        ((__bf16*)(qs + r * QROW))[j] = h0;
        ((__bf16*)(qs + r * QROW))[j + HD] = h1;
        if (rot) {
          ((__bf16*)(ql + r * QROW))[j] = (__bf16)(x0 - (float)h0);
          ((__bf16*)(ql + r * QROW))[j + HD] = (__bf16)(x1 - (float)h1);
        }
      } else {
        ((float*)(qs + r * QROW))[j] = x0;
        ((float*)(qs + r * QROW))[j + HD] = x1;
      }
    }
    __syncthreads();
    f32x4 o[NR][FPT];
    float m[NR], ls[NR];
    int lim[NR];   // last entry that this lane's row sees
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
      m[rt] = -INFINITY;
      ls[rt] = 0.f;
      lim[rt] = a.causal ? len - a.nq + (16 * rt + l) % a.nq : len - 1;
#pragma unroll
      for (int e = 0; e < FPT; ++e) o[rt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int open = a.causal ? len - a.nq : len - 1;   // entries up to this one are seen by every row
    for (int c = f0 + w; c < f1; c += PAGED_WAVES) {
      const bool more = c + PAGED_WAVES < f1;
      Chunk nxt;
      if (more) nxt = lookup(c + PAGED_WAVES);
      // ---- logits
      f32x4 x[NR][NKT];
#pragma unroll
      for (int rt = 0; rt < NR; ++rt)
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) x[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
          const int qoff = (16 * rt + l) * QROW + 64 * i + 16 * lg;
          const u32x4 qv = *(const u32x4*)(qs + qoff);
#pragma unroll
          for (int kt = 0; kt < NKT; ++kt) {
            if constexpr (TL::B16) {
              x[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kp[kt][i]),
                                                                  __builtin_bit_cast(bf16x8, qv), x[rt][kt], 0, 0, 0);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                x[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kp[kt][i][e]), __uint_as_float(qv[e]),
                                                                 x[rt][kt], 0, 0, 0);
            }
          }
          if (TL::B16 && rot) {
            const u32x4 qw = *(const u32x4*)(ql + qoff);
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
              x[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kp[kt][i]),
                                                                  __builtin_bit_cast(bf16x8, qw), x[rt][kt], 0, 0, 0);
          }
        }
      float4 bc[NKT];
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) bc[kt] = bias[kt];
      if (more) load_k(nxt);
      // ---- online softmax of this lane's rows over its entries
      bool full = c * CH + CH - 1 <= open;
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) full = full && cur.nv[kt] == 16;
      if (!full) {   // values that no row sees may be anything: zeros in their place
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < VB / 4; ++e) vr[kt * 4 + j][e] = 4 * lg + j < cur.nv[kt] ? vr[kt * 4 + j][e] : 0u;
      }
#pragma unroll
      for (int rt = 0; rt < NR; ++rt) {
        float cm = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
          const float bv[4] = {bc[kt].x, bc[kt].y, bc[kt].z, bc[kt].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) x[rt][kt][j] = fmaf(x[rt][kt][j], a.scale, bv[j]);
          if (!full) {
            const int seen = min(cur.nv[kt], lim[rt] - (c * CH + 16 * kt) + 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[rt][kt][j] = 4 * lg + j < seen ? x[rt][kt][j] : -INFINITY;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) cm = fmaxf(cm, x[rt][kt][j]);
        }
        cm = fmaxf(cm, __shfl_xor(cm, 16));
        cm = fmaxf(cm, __shfl_xor(cm, 32));
        const float mn = fmaxf(m[rt], cm), ref = mn == -INFINITY ? 0.f : mn;
        const float al = exp_of(m[rt] - ref);
        m[rt] = mn;
        float cs = 0.f;
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[rt][kt][j] = exp_of(x[rt][kt][j] - ref);
            cs += x[rt][kt][j];
          }
        ls[rt] = ls[rt] * al + cs;   // (this lane's entries; its lane groups are added at the end)
#pragma unroll
        for (int e = 0; e < FPT; ++e) o[rt][e] *= al;
      }
      // ---- P.V
      if constexpr (TL::B16) {
        bf16x8 ph[NR], pl[NR];
#pragma unroll
        for (int rt = 0; rt < NR; ++rt)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float p = x[rt][k >> 2][k & 3];
            ph[rt][k] = (__bf16)p;
            pl[rt][k] = (__bf16)(p - (float)ph[rt][k]);
          }
#pragma unroll
        for (int e = 0; e < FPT; ++e) {
          u32x4 t;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            t[k] = __builtin_amdgcn_perm(vr[2 * k + 1][e >> 1], vr[2 * k][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
          const bf16x8 vt = __builtin_bit_cast(bf16x8, t);
#pragma unroll
          for (int rt = 0; rt < NR; ++rt) {
            o[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, ph[rt], o[rt][e], 0, 0, 0);
            o[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pl[rt], o[rt][e], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < FPT; ++e)
#pragma unroll
            for (int rt = 0; rt < NR; ++rt)
              o[rt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[j][e]), x[rt][0][j], o[rt][e], 0, 0, 0);
      }
      if (more) {
        load_v(nxt);
        cur = nxt;
      }
    }
    // ---- the waves' sums into LDS, then added
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
      ls[rt] += __shfl_xor(ls[rt], 16);
      ls[rt] += __shfl_xor(ls[rt], 32);
    }
    __syncthreads();   // every wave has read the query rows
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
          float* dst = osum + (w * R + r) * OROW + (4 * lg + j) * FPT;
#pragma unroll
          for (int e = 0; e < FPT; e += 4)
            *(float4*)(dst + e) = make_float4(o[rt][e][j], o[rt][e + 1][j], o[rt][e + 2][j], o[rt][e + 3][j]);
        }
      }
    }
    __syncthreads();
    const bool whole = f0 == 0 && f1 == ns;
    const long slot = ((long)h * a.G + g) * 2 + (f0 == 0 ? 1 : 0);
    for (int e = tid; e < R * (D / 4); e += NT) {
      const int r = e / (D / 4), x = e % (D / 4) * 4;
      float M = wm[0][r];
#pragma unroll
      for (int i = 1; i < PAGED_WAVES; ++i) M = fmaxf(M, wm[i][r]);
      const float ref = M == -INFINITY ? 0.f : M;
      float L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < PAGED_WAVES; ++i) {
        const float sc = exp_of(wm[i][r] - ref);
        const float4 y = *(const float4*)(osum + (i * R + r) * OROW + x);
        L += sc * wl[i][r];
        acc[0] += sc * y.x;
        acc[1] += sc * y.y;
        acc[2] += sc * y.z;
        acc[3] += sc * y.w;
      }
      if (whole) {
        const float inv = L == 0.f ? 0.f : 1.f / L;   // a row that sees nothing; a NaN stays one
        IT* dst = (IT*)a.out + (((long)s * a.nq + r % a.nq) * Hq + h * a.group + r / a.nq) * D + x;
#pragma unroll
        for (int u = 0; u < 4; ++u) dst[u] = from_f32<IT>(acc[u] * inv);
      } else {
        *(float4*)(a.opart + (slot * R + r) * D + x) = make_float4(acc[0], acc[1], acc[2], acc[3]);
        if (x == 0) {
          a.mpart[slot * R + r] = M;
          a.lpart[slot * R + r] = L;
        }
      }
    }
    if (f0 == 0 && f1 < ns) goes_on = make_int2(s, (int)((at * part.active - 1) / part.T));
    __syncthreads();   // the sums have been read before the next sequence's query rows
  }
  if (h == 0 && tid == 0) a.plan[g] = goes_on;
}

// Joins the partial sums of the sequences that lie in several parts: block
// (x, h, g) those of the sequence that starts in workgroup g, rows x, x + gridDim.x, ...
template <class IT, int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttendArgs a) {
  constexpr int LPR = D / 4, NG = 256 / LPR;   // lanes per row, groups of parts
  __shared__ float4 acc[NG][LPR];
  __shared__ float sum[NG];
  const int h = blockIdx.y, g = blockIdx.z, R = a.group * a.nq, Hq = a.c.H * a.group;
  const int2 p = a.plan[g];
  if (p.x < 0) return;
  const int x = threadIdx.x % LPR, k = threadIdx.x / LPR, n = p.y - g + 1;
  // part 0: the start, slot 1 of workgroup g; part i: slot 0 of workgroup g + i
  auto slot = [&](int i) { return ((long)h * a.G + g + i) * 2 + (i == 0 ? 1 : 0); };
  for (int r = blockIdx.x; r < R; r += gridDim.x) {
    float M = -INFINITY;
    for (int i = 0; i < n; ++i) M = fmaxf(M, a.mpart[slot(i) * R + r]);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = k; i < n; i += NG) {
      const long at = slot(i) * R + r;
      const float sc = exp_of(a.mpart[at] - ref);
      const float4 v = *(const float4*)(a.opart + at * D + 4 * x);
      L += sc * a.lpart[at];
      y[0] += sc * v.x;
      y[1] += sc * v.y;
      y[2] += sc * v.z;
      y[3] += sc * v.w;
    }
    acc[k][x] = make_float4(y[0], y[1], y[2], y[3]);
    if (x == 0) sum[k] = L;
    __syncthreads();
    if (k == 0) {
      float S = 0.f, z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const float4 v = acc[i][x];
        S += sum[i];
        z[0] += v.x;
        z[1] += v.y;
        z[2] += v.z;
        z[3] += v.w;
      }
      const float inv = S == 0.f ? 0.f : 1.f / S;
      IT* dst = (IT*)a.out + (((long)p.x * a.nq + r % a.nq) * Hq + h * a.group + r / a.nq) * D + 4 * x;
#pragma unroll
      for (int u = 0; u < 4; ++u) dst[u] = from_f32<IT>(z[u] * inv);
    }
    __syncthreads();
  }
}

}  // namespace still
