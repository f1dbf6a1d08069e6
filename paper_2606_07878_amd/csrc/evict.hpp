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
// S^T[entry][row] as in paged_attend_kernel (16 entries by 16 rows), so a lane holds row
// l = lane % 16 of entries 4 lg + j, and the sum over the rows is one over 16 lanes.
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

constexpr int SCORE_CHUNK = 512;   // entries of a workgroup at a time

template <class IT, int D, int NR, class CT>
struct ScoreTile {
  static constexpr bool C8 = sizeof(CT) == 1, B16 = C8 || sizeof(IT) == 2;
  static constexpr int ROWB = D * (int)sizeof(CT), NP = ROWB / 64;
  static constexpr int NKT = std::max(1, std::min(8, 1024 / ROWB));   // tiles of a wave at a time: 16 KB of keys
  static constexpr int QROW = D * (B16 ? 2 : 4) + 16, QPART = 16 * NR * QROW;
  static __host__ __device__ bool split(bool rot) { return B16 && (rot || sizeof(IT) == 4); }
  static __host__ __device__ int lds_bytes(bool rot) { return (split(rot) ? 3 : 1) * QPART; }
};

template <class IT, int D, int NR, class CT>
__global__ __launch_bounds__(256) void paged_score_kernel(PagedScoreArgs a) {
  using TL = ScoreTile<IT, D, NR, CT>;
  constexpr bool C8 = TL::C8;
  constexpr int NKT = TL::NKT, NP = TL::NP, ROWB = TL::ROWB, QROW = TL::QROW, HD = D / 2, STEP = 16 * NKT;
  extern __shared__ float4 score_smem[];
  char* qs = (char*)score_smem;                  // [16 NR][QROW], where split three parts of that
  __shared__ float row_lse[16 * NR];             // plus infinity: a row that takes no part
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), l = lane & 15, lg = lane >> 4;
  const int h = blockIdx.x, s = blockIdx.y, R = a.group * a.nq, Hq = a.c.H * a.group;
  const int len = paged_len(a.c, s);
  if ((long)blockIdx.z * SCORE_CHUNK >= len) return;
  const int known = a.known ? a.known[s] : len;
  const bool rot = a.qpos != nullptr;
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
        const double pos = a.qpos[token];
#pragma unroll
        for (int u = 0; u < EPI; ++u) {
          const float2 c = rope_cs(pos, exp2(a.log2_theta * (-2.0 * (p * EPI + u) / D)));
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
    const int r = 16 * rt + l;
    ref[rt] = row_lse[r];
    lim[rt] = ref[rt] == INFINITY ? -1 : a.causal ? len - a.nq + r % a.nq : len - 1;
  }
  for (long z = (long)blockIdx.z * SCORE_CHUNK; z < len; z += (long)gridDim.z * SCORE_CHUNK)
    for (int j0 = (int)z + w * STEP; j0 < min((long)len, z + SCORE_CHUNK); j0 += 4 * STEP) {
      int nv[NKT];      // valid entries of each tile
      long row[NKT];    // rows of the pages in front of it
      u32x4 kp[NKT][NP];
      f32x4 bias[NKT], old[NKT];
      float ks[C8 ? NKT : 1];
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const int j = j0 + 16 * kt;
        const int p = uniform(a.c.table[s * a.c.tstride + min(j >> a.c.lp, a.c.max_pages - 1)]);
        const bool ok = j < len && (unsigned)p < (unsigned)a.c.n_pages;
        nv[kt] = ok ? min(16, len - j) : 0;
        row[kt] = (((long)(ok ? p : 0) * a.c.H + h) << a.c.lp) + (ok ? j & ((1 << a.c.lp) - 1) : 0);
      }
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const auto r = paged_rows(a.c.k + row[kt] * ROWB, nv[kt] * ROWB);
#pragma unroll
        for (int i = 0; i < NP; ++i)
          kp[kt][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, l * ROWB + lg * 16 + 64 * i, 0, 0));
        const int few = nv[kt] > 0 ? 64 : 0;
        bias[kt] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                 paged_rows(a.c.beta + row[kt], a.c.beta ? few : 0), 16 * lg, 0, 0));
        old[kt] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(paged_rows(a.scores + row[kt], few), 16 * lg, 0, 0));
        if constexpr (C8)
          ks[kt] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(
                                                 paged_rows(a.c.ks + row[kt] / PAGED_BLOCK, nv[kt] > 0 ? 4 : 0), 0, 0, 0));
      }
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
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        if (nv[kt] == 0) continue;
        const float sc = C8 ? a.scale * ks[C8 ? kt : 0] : a.scale;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int at = j0 + 16 * kt + 4 * lg + j;
#pragma unroll
          for (int rt = 0; rt < NR; ++rt) {
            const float y = exp_of<float>(fmaf(x[rt][kt][j], sc, bias[kt][j]) - ref[rt]);
            sum[j] += at <= lim[rt] ? y : 0.f;
          }
          sum[j] += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(sum[j]), 0x128, 0xF, 0xF, true));   // row_ror 8, 4, 2, 1
          sum[j] += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(sum[j]), 0x124, 0xF, 0xF, true));
          sum[j] += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(sum[j]), 0x122, 0xF, 0xF, true));
          sum[j] += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(sum[j]), 0x121, 0xF, 0xF, true));
          if (at < known) sum[j] += old[kt][j];
        }
        if (l == 0) {
          float* to = a.scores + row[kt] + 4 * lg;
          if (nv[kt] == 16) {
            *(f32x4*)to = sum;
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (4 * lg + j < nv[kt]) to[j] = sum[j];
          }
        }
      }
    }
}

// ---------------------------------------------------------------------------
// Choice of the entries to keep.  Block (g, s): head g of sequence s, or all heads
// together (their scores added in 64 bits, rounded to 32).  Of n > keep entries the
// first and the recent ones stay and the m largest scores between them: the m-th
// largest key is found 11, 11 and 10 bits at a time by counting, then every wave lists
// its part of the entries in order, those equal to that key until there are enough.
// ---------------------------------------------------------------------------
struct PagedEvictArgs {
  PagedArgs c;
  float* scores;        // [n_pages][H][P]
  int* kept;            // [n_seqs][shared ? 1 : H][keep]
  int* new_lens;
  int keep, first, recent, shared;
};

// the order of numbers as that of whole ones; NaN as minus infinity, -0 as 0
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t b = __float_as_uint(x != x ? -INFINITY : x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int T>
__global__ __launch_bounds__(T) void paged_select_kernel(PagedEvictArgs a) {
  constexpr int BINS = 2048, W = T / 64, PER = BINS / T;
  __shared__ int hist[BINS], part[W], part_eq[W], found[2];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), g = blockIdx.x, s = blockIdx.y;
  const int n = paged_len(a.c, s);
  int* kept = a.kept + ((long)s * gridDim.x + g) * a.keep;
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += T) kept[i] = i < n ? i : -1;
    return;
  }
  const int lo = a.first, hi = n - a.recent, m = a.keep - a.first - a.recent;   // lo + m < hi
  auto key = [&](int j) {
    const int p = paged_page(a.c, s, j);
    if (p < 0) return score_key(-INFINITY);
    if (!a.shared) return score_key(a.scores[paged_row(a.c, p, g, j)]);
    double x = 0.0;
    for (int h = 0; h < a.c.H; ++h) x += a.scores[paged_row(a.c, p, h, j)];
    return score_key((float)x);
  };
  uint32_t top = 0, mask = 0;   // the bits of the m-th largest key that are known
  int left = m;                 // its rank among the keys that have them
  for (int shift = 21; m > 0 && shift >= 0; shift = shift == 21 ? 10 : shift - 10) {
    const int bins = shift ? 2048 : 1024;
    for (int i = tid; i < BINS; i += T) hist[i] = 0;
    __syncthreads();
    for (int j = lo + tid; j < hi; j += T) {
      const uint32_t k = key(j);
      if ((k & mask) == top) atomicAdd(&hist[k >> shift & (bins - 1)], 1);
    }
    __syncthreads();
    // thread t holds bins BINS - 1 - (PER t + i), so that sums run from the largest key down
    int c[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += c[i] = hist[BINS - 1 - (PER * tid + i)];
    const int incl = lanes_scan(sum);
    if (lane == 63) part[w] = incl;
    __syncthreads();
    int before = incl - sum;
    for (int i = 0; i < w; ++i) before += part[i];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (before < left && left <= before + c[i]) {   // (one thread's)
        found[0] = BINS - 1 - (PER * tid + i);
        found[1] = left - before;
      }
      before += c[i];
    }
    __syncthreads();
    top |= (uint32_t)found[0] << shift;
    mask |= (uint32_t)(bins - 1) << shift;
    left = found[1];
    __syncthreads();
  }
  for (int i = tid; i < a.first; i += T) kept[i] = i;
  for (int i = tid; i < a.recent; i += T) kept[a.first + m + i] = hi + i;
  if (m == 0) return;
  // ---- every wave's part of the entries: how many it takes, then which
  const int each = ((hi - lo + W - 1) / W + 63) / 64 * 64, j0 = lo + w * each, j1 = min(hi, j0 + each);
  int more = 0, equal = 0;
  for (int j = j0; j < j1; j += 64) {
    const uint32_t k = j + lane < j1 ? key(j + lane) : 0;
    more += __popcll(__ballot(k > top));
    equal += __popcll(__ballot(k == top));
  }
  if (lane == 0) {
    part[w] = more;
    part_eq[w] = equal;
  }
  __syncthreads();
  more = equal = 0;
  for (int i = 0; i < w; ++i) {
    more += part[i];
    equal += part_eq[i];
  }
  for (int j = j0; j < j1; j += 64) {
    const uint32_t k = j + lane < j1 ? key(j + lane) : 0;
    const unsigned long over = __ballot(k > top), same = __ballot(k == top), below = (1UL << lane) - 1;
    const int e = equal + __popcll(same & below);
    if (k > top || (k == top && e < left)) kept[a.first + more + __popcll(over & below) + min(e, left)] = j + lane;
    more += __popcll(over);
    equal += __popcll(same);
  }
}

// ---------------------------------------------------------------------------
// The move.  Entry i of the kept list goes to place i, in the pages themselves: as
// kept[i] >= i and the list rises, a place is read only by entries in front of its own,
// so a workgroup that takes the entries in order, a chunk loaded as a whole before any
// of it is stored, needs no other memory.  Block (h, s, z): z counts the keys' and the
// values' column pieces (of 8 bits one each, for their scales), the last z the scores
// and bias.  In 8 bits a block of 16 places takes the largest scale of its new entries,
// and their codes are rescaled to it.
// ---------------------------------------------------------------------------
constexpr int EVICT_U = 8;   // 16-byte pieces of a thread in flight

template <int ROWB, bool C8>
__global__ __launch_bounds__(1024) void paged_move_kernel(PagedEvictArgs a, int pieces) {
  const int tid = threadIdx.x, T = blockDim.x, lane = tid & 63, w = tid >> 6, h = blockIdx.x, s = blockIdx.y, z = blockIdx.z;
  const int* kept = a.kept + ((long)s * (a.shared ? 1 : a.c.H) + (a.shared ? 0 : h)) * a.keep;
  if (z == 2 * pieces && h == 0 && tid == 0) a.new_lens[s] = min(paged_len(a.c, s), a.keep);
  if (kept[a.keep - 1] < 0) return;   // all of fewer entries stay
  constexpr int U = EVICT_U;
  if (z == 2 * pieces) {
    for (int i0 = 0; i0 < a.keep; i0 += U * T) {
      const int last = min(i0 + U * T, a.keep) - 1;
      if (kept[last] == last) continue;   // (and so every one before it)
      float x[U], b[U];
      int to[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * T + tid, j = i < a.keep ? kept[i] : -1, from = j < 0 ? -1 : paged_page(a.c, s, j);
        to[u] = j < 0 ? -1 : paged_page(a.c, s, i);
        const long row = paged_row(a.c, max(from, 0), h, max(j, 0));
        x[u] = from < 0 ? 0.f : a.scores[row];
        b[u] = from < 0 || !a.c.beta ? 0.f : a.c.beta[row];
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (to[u] >= 0) {
          const long row = paged_row(a.c, to[u], h, i0 + u * T + tid);
          a.scores[row] = x[u];
          if (a.c.beta) a.c.beta[row] = b[u];
        }
    }
    return;
  }
  // a wave takes U * RPW entries in a row, RPW at a time
  const int kv = z / pieces, lpr = ROWB / 16 / pieces, rpw = 64 / lpr, c = z % pieces * lpr + lane % lpr;
  char* pages = kv ? a.c.v : a.c.k;
  float* scales = kv ? a.c.vs : a.c.ks;
  const int chunk = (T >> 6) * U * rpw;
  for (int i0 = 0; i0 < a.keep; i0 += chunk) {
    const int last = min(i0 + chunk, a.keep) - 1;
    if (kept[last] == last) continue;
    u32x4 x[U];
    float sc[U];
    int to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + (w * U + u) * rpw + lane / lpr, j = i < a.keep ? kept[i] : -1;
      const int from = j < 0 ? -1 : paged_page(a.c, s, j);
      to[u] = j < 0 ? -1 : paged_page(a.c, s, i);
      const long row = paged_row(a.c, max(from, 0), h, max(j, 0));
      x[u] = from < 0 ? u32x4{0, 0, 0, 0} : ((const u32x4*)(pages + row * ROWB))[c];
      if (C8) sc[u] = from < 0 ? 0.f : scales[row / PAGED_BLOCK];
    }
    if constexpr (C8) {   // a block's largest scale: over its lanes, then over its steps
      constexpr int LPR = ROWB / 16, RPW = 64 / LPR, SPB = std::max(1, PAGED_BLOCK / RPW);   // steps of a block
#pragma unroll
      for (int u0 = 0; u0 < U; u0 += SPB) {
        float top = 0.f;
#pragma unroll
        for (int u = u0; u < u0 + SPB; ++u) {
          float t = sc[u];
#pragma unroll
          for (int d = LPR; d < LPR * std::min(PAGED_BLOCK, RPW); d <<= 1) t = fmaxf(t, __shfl_xor(t, d));
          top = fmaxf(top, t);
        }
        const float inv = top > 0.f ? 1.f / top : 0.f;
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
      if (to[u] >= 0) {
        const int i = i0 + (w * U + u) * rpw + lane / lpr;
        const long row = paged_row(a.c, to[u], h, i);
        ((u32x4*)(pages + row * ROWB))[c] = x[u];
        if (C8 && lane % lpr == 0 && (i & (PAGED_BLOCK - 1)) == 0) scales[row / PAGED_BLOCK] = sc[u];
      }
  }
}

}  // namespace still
