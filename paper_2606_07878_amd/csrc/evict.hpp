// evict.hpp - kernels that keep track of what a paged cache's entries are worth and
// drop the others: the attention weights of the newest rows added to the entries'
// scores, the choice of the entries to keep, and their move to the front, in the pages.
#pragma once
#include "paged.hpp"
#include "paged8.hpp"

namespace still {

// ---------------------------------------------------------------------------
// Scores: w[j] = sum over the rows r of KV head h of e^(scale q_r . k_j + beta_j - lse_r).
// With the rows' lse from the attention before it the keys are read once more and
// nothing has to be joined: block (h, s, z) takes the chunks z, z + gridDim.z, ... of
// SCORE_CHUNK entries of sequence s, a wave NKT 16-entry tiles of one at a time.
// S^T[entry][row] as in paged_attend_kernel (16 entries by 16 rows): lane group lg holds
// entries 4 lg + j, lane l of it row l.  Where a KV head has 4 or 8 rows (a decode
// step) the logits of 4 or 2 tiles are put next to each other in the 16 lanes, so that the
// exponentials, of which there are more than products, are formed for rows that exist (4 rows
// over 64 sequences of 5 to 16384 entries of 8 heads in 8 bits 69 -> 46 us).
// Bound by the keys where sequences are long: 65536 entries of 8 heads of width 128, 4 rows: in 8
// bits (67 MB) 16 us, 4.2 TB/s, bf16 31; 32 rows 33.  A workgroup's start takes about 5 us beside:
// 64 sequences of 2000 (131 MB) 31, of 5 to 16384 43 (with chunks of 512 46, of 256 48).  More
// workgroups for a long sequence do not help: 65536 entries of bf16 and 32 rows 33.5, with chunks of
// 512 31.9, of 256 33.2; 4 rows 30.5, 29.4, 30.6; 8 bits and 4 rows 16.0, 15.4, 17.8, 32 rows 23.6, 25.4, 30.1.
// ---------------------------------------------------------------------------
struct PagedScoreArgs {
  PagedArgs c;         // (v is not read)
  const char* q;       // tokens of [H * group][d]
  long q_ts;           // bytes
  const float* lse;    // [tokens][H * group]
  const int* known;    // [n_seqs] or NULL
  float* scores;       // [n_pages][H][P]
  const double* qpos;
  double log2_theta;
  int group, nq, causal;
  float scale;
};

constexpr int SCORE_CHUNK = 1024;   // entries of a workgroup at a time

// RP: rows that fit a tile's lanes (4, 8, 16; 32: two tiles of rows).
template <class IT, int D, int RP, class CT>
struct ScoreTile {
  static constexpr bool C8 = sizeof(CT) == 1, B16 = C8 || sizeof(IT) == 2;
  static constexpr int ROWB = D * (int)sizeof(CT), NP = ROWB / 64, NR = RP == 32 ? 2 : 1;
  static constexpr int NKT = std::max(1, std::min(4, 512 / ROWB));   // tiles of a wave at a time: 8 KB of keys
  static constexpr int PK = std::min(NKT, RP < 16 ? 16 / RP : 1);    // of them side by side
  static constexpr int QROW = D * (B16 ? 2 : 4) + 16, QPART = 16 * NR * QROW;
  static __host__ __device__ bool split(bool rot) { return B16 && (rot || sizeof(IT) == 4); }
  static __host__ __device__ int lds_bytes(bool rot, int nq) {
    return (split(rot) ? 3 : 1) * QPART + (rot ? nq * D / 2 * (int)sizeof(float2) : 0);
  }
};

// sum over the lanes of a group of RP
template <int RP>
__device__ __forceinline__ float rows_sum(float x) {
  auto add = [](float x, auto c) { return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(c)::value, 0xF, 0xF, true)); };
  x = add(x, std::integral_constant<int, 0xB1>());                 // lanes 1 0 3 2, 2 3 0 1, then those of the
  x = add(x, std::integral_constant<int, 0x4E>());                 // other half of 8 and of 16
  if (RP >= 8) x = add(x, std::integral_constant<int, 0x141>());
  if (RP >= 16) x = add(x, std::integral_constant<int, 0x140>());
  return x;
}

template <class IT, int D, int RP, class CT>
__global__ __launch_bounds__(256) void paged_score_kernel(PagedScoreArgs a) {
  using TL = ScoreTile<IT, D, RP, CT>;
  constexpr bool C8 = TL::C8;
  constexpr int NKT = TL::NKT, NP = TL::NP, NR = TL::NR, ROWB = TL::ROWB, QROW = TL::QROW, HD = D / 2, STEP = 16 * NKT;
  constexpr int PK = TL::PK, G = NKT / PK, LR = RP < 16 ? RP : 16;   // groups of PK tiles; lanes of a tile
  extern __shared__ float4 score_smem[];
  char* qs = (char*)score_smem;                  // [16 NR][QROW], where split three parts of that
  float2* cs = (float2*)(qs + (TL::split(a.qpos != nullptr) ? 3 : 1) * TL::QPART);   // [nq][D / 2]
  __shared__ float row_lse[16 * NR];             // plus infinity: a row that takes no part
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), l = lane & 15, lg = lane >> 4;
  const int h = blockIdx.x, s = blockIdx.y, R = a.group * a.nq, Hq = a.c.H * a.group;
  const int len = paged_len(a.c, s);
  if ((long)blockIdx.z * SCORE_CHUNK >= len) return;
  const int known = a.known ? a.known[s] : len;
  const bool rot = a.qpos != nullptr;
  // ---- this wave's units of STEP entries, in rising order.  A lane looks after one tile of
  // each group: its page, its bias and scores.
  constexpr int UPC = SCORE_CHUNK / (4 * STEP);   // units of a chunk
  const int mine = min(l / LR, PK - 1);
  auto start_of = [&](int v) { return ((long)blockIdx.z + (long)(v / UPC) * gridDim.z) * SCORE_CHUNK + (v % UPC * 4 + w) * STEP; };
  struct Unit {
    long j0;
    int p[G];
  };
  auto lookup = [&](int v) {
    Unit u;
    u.j0 = start_of(v);
#pragma unroll
    for (int g = 0; g < G; ++g)
      u.p[g] = a.c.table[s * a.c.tstride + min((u.j0 + 16 * (g * PK + mine)) >> a.c.lp, (long)a.c.max_pages - 1)];
    return u;
  };
  u32x4 kp[NKT][NP];
  f32x4 bias[G], old[G];
  float ks[G];
  int nv[G];        // valid entries of the lane's tile
  float* to[G];     // their scores
  auto load = [&](const Unit& u) {
    auto rows_of = [&](long j, int p, bool& ok) {   // row of the pages in front of the tile at entry j
      ok = j < len && (unsigned)p < (unsigned)a.c.n_pages;
      return (((long)(ok ? p : 0) * a.c.H + h) << a.c.lp) + (ok ? (int)j & ((1 << a.c.lp) - 1) : 0);
    };
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int t = 0; t < PK; ++t) {
        const int kt = g * PK + t;
        bool ok;
        const long j = u.j0 + 16 * kt, row = rows_of(j, __builtin_amdgcn_readlane(u.p[g], t * LR), ok);
        const auto r = paged_rows(a.c.k + row * ROWB, ok ? (int)min(16L, len - j) * ROWB : 0);
#pragma unroll
        for (int i = 0; i < NP; ++i)
          kp[kt][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, l * ROWB + lg * 16 + 64 * i, 0, 0));
      }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      bool ok;
      const long j = u.j0 + 16 * (g * PK + mine), row = rows_of(j, u.p[g], ok);   // (not ok: of a page that is there)
      nv[g] = ok ? (int)min(16L, len - j) : 0;
      to[g] = a.scores + row + 4 * lg;
      old[g] = *(const f32x4*)to[g];
      bias[g] = a.c.beta ? *(const f32x4*)(a.c.beta + row + 4 * lg) : f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (C8) ks[g] = a.c.ks[row / PAGED_BLOCK];
    }
  };
  Unit cur = lookup(0);
  if (rot) {   // (cos, sin) of the queries' angles
    for (int e = tid; e < a.nq * HD; e += 256)
      cs[e] = rope_cs(a.qpos[(long)s * a.nq + e / HD], exp2(a.log2_theta * (-2.0 * (e % HD) / D)));
    __syncthreads();
  }
  load(cur);
  // ---- the query rows into LDS: row g * nq + i is query i of head h * group + g
  constexpr int EPI = TL::B16 ? 8 : 4, NV = EPI * (int)sizeof(IT) / 16, HP = HD / EPI;
  for (int e = tid; e < 16 * NR * HP; e += 256) {
    const int r = e / HP, p = e % HP, i = min(r, R - 1), g = i / a.nq;
    const long token = (long)s * a.nq + i - g * a.nq;
    const u32x4* src = (const u32x4*)(a.q + token * a.q_ts + (long)(h * a.group + g) * D * sizeof(IT));
    u32x4 y[2][NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      y[0][u] = src[p * NV + u];
      y[1][u] = src[(p + HP) * NV + u];
    }
    if (TL::split(rot) || rot) {
      float x0[EPI], x1[EPI];
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        unpack16<IT>(y[0][u], *(float(*)[EPI / NV])(x0 + u * (EPI / NV)));
        unpack16<IT>(y[1][u], *(float(*)[EPI / NV])(x1 + u * (EPI / NV)));
      }
      if (rot) {
        const float2* turn = cs + (i - g * a.nq) * HD + p * EPI;
#pragma unroll
        for (int u = 0; u < EPI; ++u) {
          const float2 c = turn[u];
          const float z = x0[u] * c.x - x1[u] * c.y;
          x1[u] = x1[u] * c.x + x0[u] * c.y;
          x0[u] = z;
        }
      }
      if constexpr (TL::B16) {
        bf16x8 p0[3], p1[3];
        bf16_parts(x0, p0);
        bf16_parts(x1, p1);
#pragma unroll
        for (int part = 0; part < 3; ++part) {
          *(bf16x8*)(qs + part * TL::QPART + r * QROW + 16 * p) = p0[part];
          *(bf16x8*)(qs + part * TL::QPART + r * QROW + 16 * (p + HP)) = p1[part];
        }
        continue;
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          y[0][0][u] = __float_as_uint(x0[u]);
          y[1][0][u] = __float_as_uint(x1[u]);
        }
      }
    }
    *(u32x4*)(qs + r * QROW + 16 * p) = y[0][0];
    *(u32x4*)(qs + r * QROW + 16 * (p + HP)) = y[1][0];
  }
  for (int r = tid; r < 16 * NR; r += 256) {
    const int g = min(r, R - 1) / a.nq;
    const float x = a.lse[((long)s * a.nq + min(r, R - 1) - g * a.nq) * Hq + h * a.group + g];
    row_lse[r] = r < R && x != -INFINITY ? x : INFINITY;
  }
  __syncthreads();
  float ref[NR];
  int lim[NR];   // last entry that this lane's row sees
#pragma unroll
  for (int rt = 0; rt < NR; ++rt) {
    const int r = 16 * rt + l % LR;
    ref[rt] = row_lse[r];
    lim[rt] = ref[rt] == INFINITY ? -1 : a.causal ? len - a.nq + r % a.nq : len - 1;
  }
  const bool writes = l % LR == 0 && l / LR < PK;
  for (int v = 0; cur.j0 < len; ++v) {
    const int j0 = (int)cur.j0;
    const Unit next = lookup(v + 1);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 x[NR][NKT];
#pragma unroll
    for (int rt = 0; rt < NR; ++rt)
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) x[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto product = [&](int part, const u32x4 (&kv)[NKT], int at) {
#pragma unroll
      for (int rt = 0; rt < NR; ++rt) {
        const u32x4 qv = *(const u32x4*)(qs + part * TL::QPART + (16 * rt + l) * QROW + at);
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
          if constexpr (TL::B16) {
            x[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kv[kt]),
                                                                __builtin_bit_cast(bf16x8, qv), x[rt][kt], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              x[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kv[kt][e]), __uint_as_float(qv[e]),
                                                               x[rt][kt], 0, 0, 0);
          }
        }
      }
    };
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int half = 0; half < (C8 ? 2 : 1); ++half) {
        u32x4 kv[NKT];
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
          kv[kt] = kp[kt][p];
          if constexpr (C8) {
            const uint32_t w0 = kp[kt][p][2 * half], w1 = kp[kt][p][2 * half + 1];
            kv[kt] = u32x4{e4m3_pair<false>(w0), e4m3_pair<true>(w0), e4m3_pair<false>(w1), e4m3_pair<true>(w1)};
          }
        }
        const int at = C8 ? 128 * p + 32 * lg + 16 * half : 64 * p + 16 * lg;
        product(0, kv, at);
        if (TL::split(rot)) {
          product(1, kv, at);
          product(2, kv, at);
        }
      }
    // the next unit's keys are on their way while this one's weights are summed
    f32x4 bc[G], oc[G];
    float sc[G], *dst[G];
    int n[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      bc[g] = bias[g];
      oc[g] = old[g];
      sc[g] = C8 ? a.scale * ks[g] : a.scale;
      n[g] = nv[g];
      dst[g] = to[g];
    }
    load(next);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int j1 = j0 + 16 * (g * PK + mine) + 4 * lg;   // the lane's first entry
      f32x4 sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum[j] = 0.f;
#pragma unroll
        for (int rt = 0; rt < NR; ++rt) {
          uint32_t y = __float_as_uint(x[rt][g * PK][j]);
          if constexpr (RP == 4) {   // lanes 0 .. 3 of a tile to those from 4, 8 and 12 on
            if constexpr (PK >= 2) y = __builtin_amdgcn_update_dpp(y, __float_as_uint(x[rt][g * PK + 1][j]), 0x114, 0xF, 0x2, false);
            if constexpr (PK >= 4) {
              y = __builtin_amdgcn_update_dpp(y, __float_as_uint(x[rt][g * PK + 2][j]), 0x118, 0xF, 0x4, false);
              y = __builtin_amdgcn_update_dpp(y, __float_as_uint(x[rt][g * PK + 3][j]), 0x11C, 0xF, 0x8, false);
            }
          }
          if constexpr (RP == 8 && PK == 2) y = __builtin_amdgcn_update_dpp(y, __float_as_uint(x[rt][g * PK + 1][j]), 0x118, 0xF, 0xC, false);
          const float e = exp_of<float>(fmaf(__uint_as_float(y), sc[g], bc[g][j]) - ref[rt]);
          sum[j] += j1 + j <= lim[rt] ? e : 0.f;   // (whatever an entry holds that the row does not see)
        }
        sum[j] = rows_sum<LR>(sum[j]);
        if (j1 + j < known) sum[j] += oc[g][j];
      }
      if (writes) {
        if (n[g] == 16) {
          *(f32x4*)dst[g] = sum;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (4 * lg + j < n[g]) dst[g][j] = sum[j];
        }
      }
    }
    cur = next;
  }
}

// ---------------------------------------------------------------------------
// Choice of the entries to keep.  Block (g, s): head g of sequence s, or all heads
// together (their scores added in 64 bits, rounded to 32).  Of n > keep entries the
// first and the recent ones stay and the m largest scores between them: the m-th
// largest key is found 11, 11 and 10 bits at a time by counting, then the entries
// above it, and those equal to it until there are enough, are listed in order.
// T threads hold up to K keys each; a list that is longer is read again for every step.  That
// costs less than keys of 65536 entries in registers: code for 64 of them, run once, waits for
// its instructions (34 us with 64 a thread, 27 with 16, 29 with 8).
// Long lists' counts are kept four times over (lane mod 4): most scores share a few
// exponents, and a count that many lanes raise at once takes them one by one.
// ---------------------------------------------------------------------------
struct PagedEvictArgs {
  PagedArgs c;
  float* scores;        // [n_pages][H][P]
  int* kept;            // [n_seqs][shared ? 1 : H][keep]
  int* new_lens;
  int keep, first, recent, shared;
  uint32_t* keys;       // [lists][kstride] or NULL
  long kstride;
  int* bins;            // [lists][kblocks][SELECT_BINS]: how many keys of each part start with these bits
  int kblocks, kpart;   // a list's parts, entries of one (a multiple of 4096)
};
constexpr int SELECT_BINS = 2048;

// the order of numbers as that of whole ones; NaN as minus infinity, -0 as 0
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t b = __float_as_uint(x != x ? -INFINITY : x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Few long lists: their keys by the whole chip first, four entries a thread, 0 for those that
// are not chosen from; and the first counting step, part by part.
__global__ __launch_bounds__(1024) void paged_keys_kernel(PagedEvictArgs a) {
  __shared__ int count[4 * SELECT_BINS];
  const int g = blockIdx.y, s = blockIdx.z, n = paged_len(a.c, s), tid = threadIdx.x;
  const long j0 = (long)blockIdx.x * a.kpart, j1 = min((long)n, j0 + a.kpart), list = (long)s * gridDim.y + g;
  if (n <= a.keep || j0 >= n) return;
  for (int i = tid; i < SELECT_BINS; i += 1024) ((int4*)count)[i] = make_int4(0, 0, 0, 0);
  __syncthreads();
  for (long j = j0 + 4 * tid; j < j1; j += 4096) {
    const int p = paged_page(a.c, s, j);
    f32x4 x = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (p >= 0 && !a.shared) x = *(const f32x4*)(a.scores + paged_row(a.c, p, g, j));
    if (p >= 0 && a.shared) {
      double sum[4] = {};
#pragma unroll 8
      for (int h = 0; h < a.c.H; ++h) {
        const f32x4 y = *(const f32x4*)(a.scores + paged_row(a.c, p, h, j));
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += y[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (float)sum[i];
    }
    u32x4 k;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      k[i] = j + i >= a.first && j + i < n - a.recent ? score_key(x[i]) : 0;
      if (k[i]) atomicAdd(&count[(k[i] >> 21) * 4 + tid % 4], 1);
    }
    *(u32x4*)(a.keys + list * a.kstride + j) = k;
  }
  __syncthreads();
  int* out = a.bins + (list * a.kblocks + blockIdx.x) * SELECT_BINS;
  for (int i = tid; i < SELECT_BINS; i += 1024) {
    const int4 x = ((const int4*)count)[i];
    out[i] = x.x + x.y + x.z + x.w;
  }
}

// DENSE: keys and first counts of paged_keys_kernel; keys that share the first bits found are
// put aside in the second step, so that the third one looks at them alone.
constexpr int SELECT_ASIDE = 8192;
template <int T, int K, bool DENSE>
__global__ __launch_bounds__(T) void paged_select_kernel(PagedEvictArgs a) {
  constexpr int BINS = SELECT_BINS, W = T / 64, PER = BINS / T, CP = T == 1024 ? 4 : 1;
  __shared__ int hist[BINS * CP], part[W], part_eq[W], found[4];
  __shared__ uint32_t aside[DENSE ? SELECT_ASIDE : 1];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), g = blockIdx.x, s = blockIdx.y;
  const int n = paged_len(a.c, s);
  int* kept = a.kept + ((long)s * gridDim.x + g) * a.keep;
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += T) kept[i] = i < n ? i : -1;
    return;
  }
  const int m = a.keep - a.first - a.recent;
  for (int i = tid; i < a.first; i += T) kept[i] = i;
  for (int i = tid; i < a.recent; i += T) kept[a.first + m + i] = n - a.recent + i;
  if (m == 0) return;
  const int lo = DENSE ? 0 : a.first, hi = DENSE ? n : n - a.recent;
  // a round: `steps` keys of every thread, those of a wave next to each other
  const int steps = min(K, (hi - lo + T - 1) / T), span = steps * T;
  uint32_t key[K];              // (of no entry: 0, below every key)
  auto entry = [&](int base, int k) { return base + (w * steps + k) * 64 + lane; };
  auto load = [&](int base) {
    if constexpr (DENSE) {
      // (behind the last key: zeros; a list's keys are 64 MB at most)
      const auto r = paged_rows(a.keys + ((long)s * gridDim.x + g) * a.kstride, hi * 4);
      const int off = ((int)base + w * steps * 64 + lane) * 4;
#pragma unroll
      for (int k0 = 0; k0 < K; k0 += 8) {
        if (k0 < steps) {
#pragma unroll
          for (int k = k0; k < k0 + 8; ++k) key[k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_raw_buffer_load_b32(r, off, k * 256, 0));
        }
#pragma unroll
        for (int k = k0; k < k0 + 8; ++k) key[k] = k < steps ? key[k] : 0;
      }
      return;
    }
    constexpr int B = K < 8 ? K : 8;   // at a time
#pragma unroll
    for (int k0 = 0; k0 < (DENSE ? 0 : K); k0 += B) {
      if (k0 >= steps) {
#pragma unroll
        for (int k = k0; k < k0 + B; ++k) key[k] = 0;
        continue;
      }
      int page[B];
      auto at = [&](int k) { return min(entry(base, k0 + k), hi - 1); };
#pragma unroll
      for (int k = 0; k < B; ++k) page[k] = a.c.table[s * a.c.tstride + (at(k) >> a.c.lp)];
      auto row = [&](int k, int h) {
        const bool ok = (unsigned)page[k] < (unsigned)a.c.n_pages;
        return paged_row(a.c, ok ? page[k] : 0, h, at(k));
      };
      float x[B];
      if (!a.shared) {
#pragma unroll
        for (int k = 0; k < B; ++k) x[k] = a.scores[row(k, g)];
      } else {
        double sum[B] = {};
        for (int h = 0; h < a.c.H; ++h)
#pragma unroll
          for (int k = 0; k < B; ++k) sum[k] += a.scores[row(k, h)];
#pragma unroll
        for (int k = 0; k < B; ++k) x[k] = (float)sum[k];
      }
#pragma unroll
      for (int k = 0; k < B; ++k) {
        const bool ok = (unsigned)page[k] < (unsigned)a.c.n_pages;
        key[k0 + k] = k0 + k < steps && entry(base, k0 + k) < hi ? score_key(ok ? x[k] : -INFINITY) : 0;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // f(k) for the keys held; those from `steps` on are 0
  auto each = [&](auto f) {
    constexpr int B = K < 16 ? K : 16;
#pragma unroll
    for (int k0 = 0; k0 < K; k0 += B)
      if (k0 < steps)
#pragma unroll
        for (int k = k0; k < k0 + B; ++k) f(k);
  };
  load(lo);
  const bool once = hi - lo <= span;
  auto in_front = [&](const int* x) {   // the sum of the waves' numbers in front of this one, and of all
    const int v = lane < W ? x[lane] : 0, incl = lanes_scan(v);
    return make_int2(__builtin_amdgcn_readlane(incl - v, w), __builtin_amdgcn_readlane(incl, 63));
  };
  uint32_t top = 0, mask = 0;   // the bits of the m-th largest key that are known
  int left = m;                 // its rank among the keys that have them
  bool all = false;             // that is the last one of them
  int cand = 0;                 // how many they are
  for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift - 10) {
    const int bins = shift ? 2048 : 1024;
    const bool given = DENSE && shift == 21, few = DENSE && cand <= SELECT_ASIDE;
    if (!given) {
      for (int i = tid; i < BINS * CP / 4; i += T) ((int4*)hist)[i] = make_int4(0, 0, 0, 0);
      if (tid == 0) found[3] = 0;
      __syncthreads();
      auto raise = [&](uint32_t k) { atomicAdd(&hist[(k >> shift & (bins - 1)) * CP + lane % CP], 1); };
      if (few && shift == 0) {
        for (int i = tid; i < cand; i += T)
          if (((aside[i] ^ top) & mask) == 0) raise(aside[i]);
      } else {
        for (long base = lo; base < hi; base += span) {
          if (!once && (base != lo || shift != 21)) load(base);
          each([&](int k) {   // (the known bits of a key of no entry are not those of `top`, once there are any)
            if (shift == 21 ? key[k] != 0 : ((key[k] ^ top) & mask) == 0) {
              raise(key[k]);
              if (few) {   // (in any order: they are only counted)
                const int at = atomicAdd(&found[3], 1);
                if (at < SELECT_ASIDE) aside[at] = key[k];
              }
            }
          });
        }
      }
      __syncthreads();
    }
    // thread t holds bins BINS - 1 - (PER t + i), so that sums run from the largest key down
    int c[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = BINS - 1 - (PER * tid + i);
      if (given) {
        c[i] = 0;
        const int* parts = a.bins + ((long)s * gridDim.x + g) * a.kblocks * BINS + b;
#pragma unroll 8
        for (int k = 0; k < (n + a.kpart - 1) / a.kpart; ++k) c[i] += parts[k * BINS];
      } else if constexpr (CP == 4) {
        const int4 x = ((const int4*)hist)[b];
        c[i] = x.x + x.y + x.z + x.w;
      } else {
        c[i] = hist[b];
      }
      sum += c[i];
    }
    const int incl = lanes_scan(sum);
    if (lane == 63) part[w] = incl;
    __syncthreads();
    int before = incl - sum + in_front(part).x;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (before < left && left <= before + c[i]) {   // (one thread's)
        found[0] = BINS - 1 - (PER * tid + i);
        found[1] = left - before;
        found[2] = left == before + c[i];
        if (shift == 21) found[3] = c[i];
      }
      before += c[i];
    }
    __syncthreads();
    top |= (uint32_t)found[0] << shift;
    mask |= (uint32_t)(bins - 1) << shift;
    left = found[1];
    all = found[2];
    if (shift == 21) cand = found[3];
    __syncthreads();
  }
  if (all) {   // every key equal to the m-th stays too
    top -= 1;  // (keys of entries are above 0)
    left = 0;
  }
  // ---- the list, wave by wave: how many keys each has above `top` and equal to it, then which.
  // (They are m, unless scores or workspace change meanwhile, which must not write past the list.)
  int more = 0, same = 0;       // in front of the round
  for (long base = lo; base < hi; base += span) {
    if (!once) load(base);
    int x = 0, y = 0;
    each([&](int k) { x += __popcll(__ballot(key[k] > top)); });
    if (left) each([&](int k) { y += __popcll(__ballot(key[k] == top)); });
    __syncthreads();            // the counts before have been read
    if (lane == 0) {
      part[w] = x;
      part_eq[w] = y;
    }
    __syncthreads();
    const int2 a0 = in_front(part), e0 = in_front(part_eq);
    int over = more + a0.x, eq = same + e0.x;
    more += a0.y;
    same += e0.y;
    auto lanes_below = [](unsigned long x) { return (int)__builtin_amdgcn_mbcnt_hi(x >> 32, __builtin_amdgcn_mbcnt_lo((uint32_t)x, 0)); };
    int* to = kept + a.first;
    if (left == 0) {
      each([&](int k) {
        const unsigned long o = __ballot(key[k] > top);
        const int at = over + lanes_below(o);
        if (key[k] > top && at < m) to[at] = entry((int)base, k);
        over += __popcll(o);
      });
      continue;
    }
    each([&](int k) {
      const unsigned long o = __ballot(key[k] > top), e = __ballot(key[k] == top);
      const int r = eq + lanes_below(e);
      const int at = over + lanes_below(o) + min(r, left);
      if ((key[k] > top || (key[k] == top && r < left)) && at < m) to[at] = entry((int)base, k);
      over += __popcll(o);
      eq += __popcll(e);
    });
  }
}

// ---------------------------------------------------------------------------
// The move.  Entry i of the kept list goes to place i, in the pages themselves: as
// kept[i] >= i and the list rises, a place is read only by entries in front of its own,
// so a workgroup that takes the entries in order, a chunk loaded as a whole before any
// of it is stored, needs no other memory.  Block (h, s, z): z counts the keys' and the
// values' column pieces (of 8 bits one each, for their scales), the last z the scores
// and bias.  In 8 bits a block of 16 places takes the largest scale of its new entries
// (E4M3_LEAST where they were all absent), and their codes are rescaled to it.
// 512 lists of 1088 entries to 1024, 8 bits of width 128 (272 MB) 62 us, 4.5 TB/s; 8 lists of 65536 to
// 4096, bf16 (34 MB) 22: two chunks one after the other, each three loads deep.
// ---------------------------------------------------------------------------
constexpr int EVICT_U = 8;   // 16-byte pieces of a thread in flight

template <int ROWB, bool C8>
__global__ __launch_bounds__(1024) void paged_move_kernel(PagedEvictArgs a, int pieces) {
  const int tid = threadIdx.x, T = blockDim.x, lane = tid & 63, w = tid >> 6, h = blockIdx.x, s = blockIdx.y, z = blockIdx.z;
  const int* kept = a.kept + ((long)s * (a.shared ? 1 : a.c.H) + (a.shared ? 0 : h)) * a.keep;
  if (z == 2 * pieces && h == 0 && tid == 0) a.new_lens[s] = min(paged_len(a.c, s), a.keep);
  if (kept[a.keep - 1] < 0) return;   // all of fewer entries stay
  constexpr int U = EVICT_U;
  const bool rows = z < 2 * pieces;
  // keys, values: a wave takes U * rpw entries in a row, rpw at a time; scores: U * 64
  const int kv = z / pieces, lpr = rows ? ROWB / 16 / pieces : 1, rpw = 64 / lpr, c = z % pieces * lpr + lane % lpr;
  char* pages = kv ? a.c.v : a.c.k;
  float* scales = kv ? a.c.vs : a.c.ks;
  const int chunk = (T >> 6) * U * rpw;
  auto entry = [&](int i0, int u) { return i0 + (w * U + u) * rpw + lane / lpr; };
  long from[U], to[U];                // rows of the pages that entry and place are, or -1
  auto find = [&](int i0) {
    int j[U], pf[U], pt[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      j[u] = entry(i0, u) < a.keep ? kept[entry(i0, u)] : -1;
      if (j[u] >= paged_cap(a.c)) j[u] = -1;   // (no entry: the list was written to meanwhile)
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      pf[u] = j[u] < 0 ? -1 : paged_page(a.c, s, j[u]);
      pt[u] = j[u] < 0 ? -1 : paged_page(a.c, s, entry(i0, u));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      from[u] = pf[u] < 0 ? -1 : paged_row(a.c, pf[u], h, j[u]);
      to[u] = pt[u] < 0 ? -1 : paged_row(a.c, pt[u], h, entry(i0, u));
    }
  };
  auto moves = [&](int i0) {          // (kept[i] == i: and so for every entry before it)
    const int last = min(i0 + chunk, a.keep) - 1;
    return kept[last] != last;
  };
  int i0 = 0;
  while (i0 < a.keep && !moves(i0)) i0 += chunk;
  if (i0 < a.keep) find(i0);
  for (; i0 < a.keep; i0 += chunk) {
    long at[U];
    if (!rows) {
      float x[U], b[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x[u] = from[u] < 0 ? 0.f : a.scores[from[u]];
        b[u] = from[u] < 0 || !a.c.beta ? 0.f : a.c.beta[from[u]];
        at[u] = to[u];
      }
      if (i0 + chunk < a.keep) find(i0 + chunk);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at[u] >= 0) {
          a.scores[at[u]] = x[u];
          if (a.c.beta) a.c.beta[at[u]] = b[u];
        }
      continue;
    }
    u32x4 x[U];
    float sc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = from[u] < 0 ? u32x4{0, 0, 0, 0} : __builtin_nontemporal_load((const u32x4*)(pages + from[u] * ROWB) + c);
      if (C8) sc[u] = from[u] < 0 ? 0.f : scales[from[u] / PAGED_BLOCK];
      at[u] = to[u];
    }
    if (i0 + chunk < a.keep) find(i0 + chunk);   // (places and list are not what this chunk writes)
    if constexpr (C8) {   // a block's largest scale: over its lanes, then over its steps
      constexpr int LPR = ROWB / 16, RPW = 64 / LPR, SPB = std::max(1, PAGED_BLOCK / RPW);   // steps of a block
#pragma unroll
      for (int u0 = 0; u0 < U; u0 += SPB) {
        float top = E4M3_LEAST;   // (of a block whose entries were all absent, too)
#pragma unroll
        for (int u = u0; u < u0 + SPB; ++u) {
          float t = sc[u];
#pragma unroll
          for (int d = LPR; d < LPR * std::min(PAGED_BLOCK, RPW); d <<= 1) t = fmaxf(t, __shfl_xor(t, d));
          top = fmaxf(top, t);
        }
        const float inv = 1.f / top;
#pragma unroll
        for (int u = u0; u < u0 + SPB; ++u) {
          const float ratio = sc[u] * inv;
          if (sc[u] != top)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float f[4];
              e4m3_floats(x[u][k], f);
              x[u][k] = e4m3_codes(f[0] * ratio, f[1] * ratio, f[2] * ratio, f[3] * ratio);
            }
          sc[u] = top;
        }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at[u] >= 0) {
        __builtin_nontemporal_store(x[u], (u32x4*)(pages + at[u] * ROWB) + c);
        if (C8 && lane % lpr == 0 && (at[u] & (PAGED_BLOCK - 1)) == 0) scales[at[u] / PAGED_BLOCK] = sc[u];
      }
  }
}

}  // namespace still
