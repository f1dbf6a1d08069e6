// paged8.hpp - append and gather of the paged cache in 8 bits (attention over it
// is paged_attend_kernel).
//
// Pages hold e4m3 codes [n_pages][H][P][d]; blocks of 16 entries of a head share a
// float scale [n_pages][H][P / 16], and an entry stands for its code times that.  The
// append makes scales that are powers of two: rescaling a block's codes when it grows
// is then exact but for what falls below the smallest code, so a block rounds its
// entries once, and a code times its scale is a bf16 number.
#pragma once
#include "paged.hpp"

namespace still {

constexpr float E4M3_LEAST = 0x1p-100f;   // the smallest scale: no product of a code with it is a subnormal float

// The smallest power of two whose 448-fold (the largest code) reaches top, at least
// E4M3_LEAST.  With top = m 2^e, 1 <= m < 2, and 448 = 1.75 2^8 it is 2^(e - 8), twice that
// where m > 1.75.
__device__ __forceinline__ float e4m3_scale(float top) {
  const uint32_t b = __float_as_uint(top);
  const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u);
  return __uint_as_float((uint32_t)max(e, 127 - 100) << 23);
}

// Four floats of up to 448 as codes, rounded to nearest even; NaN as NaN.
__device__ __forceinline__ uint32_t e4m3_codes(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ void e4m3_floats(uint32_t w, float (&f)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  f[0] = lo[0];
  f[1] = lo[1];
  f[2] = hi[0];
  f[3] = hi[1];
}

// (cos, sin) of pos * inv in 64 bits: quarter turns taken off in two parts, then the
// Taylor polynomials on [-pi/4, pi/4], whose first left-out terms are 5e-17 and 2e-18.
// A key's rounding to 32 bits, and with it its block's scale, must not depend on the
// order of a sum: in 32 bits one block in 5 million would get another scale than
// the exact key asks for, which doubles its rounding errors.
__device__ __forceinline__ double2 rope_cs64(double pos, double inv) {
  const double ang = pos * inv;
  const double q = rint(ang * 0.63661977236758134);
  double r = fma(-q, 1.5707963267948966, ang);
  r = fma(-q, 6.123233995736766e-17, r);
  const double y = r * r;
  double s = -1. / 1307674368000., c = 1. / 20922789888000.;
  s = fma(s, y, 1. / 6227020800.);
  s = fma(s, y, -1. / 39916800.);
  s = fma(s, y, 1. / 362880.);
  s = fma(s, y, -1. / 5040.);
  s = fma(s, y, 1. / 120.);
  s = fma(s, y, -1. / 6.);
  s = fma(s * y, r, r);
  c = fma(c, y, -1. / 87178291200.);
  c = fma(c, y, 1. / 479001600.);
  c = fma(c, y, -1. / 3628800.);
  c = fma(c, y, 1. / 40320.);
  c = fma(c, y, -1. / 720.);
  c = fma(c, y, 1. / 24.);
  c = fma(c, y, -0.5);
  c = fma(c, y, 1.);
  const int k = (int)(q - 4.0 * floor(q * 0.25));
  const double a = k & 1 ? s : c, b = k & 1 ? c : s;
  return make_double2((k + 1) & 2 ? -a : a, k & 2 ? -b : b);
}

// ---------------------------------------------------------------------------
// Append.  A workgroup takes TG tokens in a row; those of them with which a block of
// entries begins in this call (the first token of a sequence, and each at a slot
// divisible by 16) lead, and the workgroup writes their blocks, one after the other, a
// wave a (head, key or value) at a time: its rows' largest magnitude decides the
// scale, so no two waves share a block.  A lane holds 8 values and the 8 that are
// rotated with them, d/2 further on.
// Reads the rows, writes a byte a value: 6977 tokens of 8 heads of width 256 (86 MB) 30 us, 2.9
// TB/s, 22 without rotation; the largest number of a block is known only once all of it is in
// registers, which leaves three waves per SIMD at that width, with three registers of 168 spilled to 16 bytes
// of scratch.  A single token costs the chain
// offsets -> length -> page -> old scale, 4.4 us.
// ---------------------------------------------------------------------------
struct Append8Args {
  PagedAppendArgs t;
  int heads;             // of a workgroup
};

template <class IT, int D, int TG>
__global__ __launch_bounds__(256, 3) void paged8_append_kernel(Append8Args p) {
  constexpr int HD = D / 2, IPR = HD / 8, RPS = 64 / IPR, ST = PAGED_BLOCK / RPS, NV = sizeof(IT) / 2;
  const PagedAppendArgs& a = p.t;
  __shared__ double2 cs[PAGED_BLOCK][HD];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const long t0 = ((long)blockIdx.z * gridDim.x + blockIdx.x) * TG;
  if (t0 >= a.n_tokens) return;
  const int h0 = blockIdx.y * p.heads, h1 = min(a.c.H, h0 + p.heads);
  // ---- lane t < TG: its token's entry j, and how many entries it leads
  long j = -1;
  int count = 0, page = -1;
  {
    const bool mine = lane < TG && t0 + lane < a.n_tokens;
    const int i = mine ? (int)t0 + lane : 0, n_seqs = a.c.n_seqs;
    int s = 0;
    long start = 0, end = -1;
    if (a.offsets) {
      const int x0 = (lane + 1) * ((n_seqs + 63) / 64);
      const int from = uniform(paged_seq_of(a.offsets, n_seqs, (int)t0, x0 < n_seqs ? a.offsets[x0] : 0));
      s = from;
      // sequences that start behind the first token, 64 at a time: a token is as many further on as
      // start up to it, in whichever 64.  (Tokens and offsets may be as many as an int counts: that
      // there are no more sequences is known from n_seqs alone.)
      for (int next = from + 1; next < n_seqs; next += 64) {
        const bool there = next + lane < n_seqs;
        const int o = there ? a.offsets[next + lane] : 0;
#pragma unroll
        for (int t = 0; t < TG; ++t) {
          const int n = __popcll(__ballot(there && o <= (int)t0 + t));
          if (lane == t) s += n;
        }
        if (next + 64 <= n_seqs && __builtin_amdgcn_readlane(o, 63) > (int)t0 + (TG - 1)) break;
      }
      if (mine) {
        start = a.offsets[s];
        end = a.offsets[s + 1];
        if (i < start || i >= end) end = -1;   // before the first or behind the last
      }
    } else if (mine) {
      s = i / a.per_seq;
      start = (long)s * a.per_seq;
      end = start + a.per_seq;
    }
    if (mine && end >= 0) {
      j = a.c.lens[s] - end + i;
      if (j >= 0 && j < paged_cap(a.c) && (j % PAGED_BLOCK == 0 || i == max(start, 0L))) {
        page = paged_page(a.c, s, j);
        if (page >= 0)
          count = (int)min(min((long)PAGED_BLOCK - j % PAGED_BLOCK, min(end, (long)a.n_tokens) - i), paged_cap(a.c) - j);
      }
    }
  }
  const double inv_freq = a.pos ? exp2(a.log2_theta * (-2.0 * (tid % HD) / D)) : 0.0;   // of this thread's angles
  unsigned long leaders = __ballot(count > 0);
  while (leaders) {
    const int t = __builtin_ctzll(leaders);
    leaders &= leaders - 1;
    const int n = __builtin_amdgcn_readlane(count, t), pg = __builtin_amdgcn_readlane(page, t);
    const int slot = __builtin_amdgcn_readlane((int)(j & ((1 << a.c.lp) - 1)), t), old = slot % PAGED_BLOCK;
    const long first = t0 + t;
    if (a.pos) {
      __syncthreads();   // the block before has been rotated
      for (int e = tid; e < n * HD; e += 256)
        cs[e / HD][e % HD] = rope_cs64(a.pos[first + e / HD], inv_freq);
      __syncthreads();
    }
    for (int u = 2 * h0 + w; u < 2 * h1; u += 4) {
      const int h = u >> 1, kv = u & 1;
      const long row = (((long)pg * a.c.H + h) << a.c.lp) + slot;
      float* scale = (kv ? a.c.vs : a.c.ks) + row / PAGED_BLOCK;
      const float before = old ? *scale : 0.f;
      const int r0 = lane / IPR, c = lane % IPR;
      float x[ST][16];
#pragma unroll
      for (int k = 0; k < ST; ++k) {
        const int r = k * RPS + r0;
        const u32x4* src = (const u32x4*)(kv ? a.v + (first + min(r, n - 1)) * a.v_ts + h * a.v_hs
                                             : a.k + (first + min(r, n - 1)) * a.k_ts + h * a.k_hs);
        u32x4 y[2][NV];
        if (k * RPS < n) {
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            y[0][v] = src[c * NV + v];
            y[1][v] = src[(IPR + c) * NV + v];
          }
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int v = 0; v < NV; ++v)
              unpack16<IT>(y[half][v], *(float(*)[16 / sizeof(IT)])(x[k] + 8 * half + v * (16 / sizeof(IT))));
        }
      }
      if (!kv && a.pos)
#pragma unroll
        for (int k = 0; k < ST; ++k) {
          const int r = min(k * RPS + r0, n - 1);
          if (k * RPS < n)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const double2 z = cs[r][c * 8 + e];
              const double x0 = x[k][e], x1 = x[k][8 + e];
              x[k][e] = (float)(x0 * z.x - x1 * z.y);
              x[k][8 + e] = (float)(x1 * z.x + x0 * z.y);
            }
        }
      auto largest = [&] {   // (a maximum leaves NaN out)
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < ST; ++k)
          if (k * RPS + r0 < n)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[k][e]));
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        return top;
      };
      float top = largest();
      if (uniform(__float_as_uint(top)) == 0x7f800000u) {   // infinities are held as NaN
#pragma unroll
        for (int k = 0; k < ST; ++k)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[k][e] = fabsf(x[k][e]) < INFINITY ? x[k][e] : NAN;
        top = largest();
      }
      const float need = e4m3_scale(top);
      const float now = old && !(need > before) ? before : need, inv = 1.f / now;
      char* codes = (kv ? a.c.v : a.c.k) + row * D;
      if (old && need > before) {   // the entries before them, in the new scale
        const float ratio = before * inv;
        for (int e = lane; e < old * (D / 16); e += 64) {
          u32x4* at = (u32x4*)(codes - old * D) + e;
          u32x4 y = *at;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float f[4];
            e4m3_floats(y[i], f);
            y[i] = e4m3_codes(f[0] * ratio, f[1] * ratio, f[2] * ratio, f[3] * ratio);
          }
          *at = y;
        }
      }
      if (lane == 0) *scale = now;
#pragma unroll
      for (int k = 0; k < ST; ++k) {
        const int r = k * RPS + r0;
        if (r < n) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float* f = x[k] + 8 * half;
            u32x2 y;
            y.x = e4m3_codes(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
            y.y = e4m3_codes(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
            __builtin_nontemporal_store(y, (u32x2*)(codes + r * D + half * HD + c * 8));
          }
        }
      }
    }
    if (a.c.beta)
      for (int e = tid; e < n * (h1 - h0); e += 256) {
        const int h = h0 + e / n, r = e % n;
        a.c.beta[(((long)pg * a.c.H + h) << a.c.lp) + slot + r] =
            a.nbeta ? a.nbeta[(first + r) * a.b_ts + h * a.b_hs] : 0.f;
      }
  }
}

// ---------------------------------------------------------------------------
// Gather: block (x, h, z) reads PAGED_GATHER_ROWS entries of head h, a thread the codes
// of 16 bytes of a row given out, keys and values.  Bound by the copy: 65536 entries of 8 heads
// of width 256 (806 MB) 151 us, 5.3 TB/s.
// ---------------------------------------------------------------------------
template <class IT, int D>
__global__ __launch_bounds__(256) void paged8_gather_kernel(PagedGatherArgs a) {
  constexpr int EPP = 16 / (int)sizeof(IT), PPR = D / EPP;
  const int tid = threadIdx.x, h = blockIdx.y, len = paged_len(a.c, a.seq);
  const long i0 = ((long)blockIdx.z * gridDim.x + blockIdx.x) * PAGED_GATHER_ROWS;
  for (int it = tid; it < PAGED_GATHER_ROWS * PPR; it += 256) {
    const long i = i0 + it / PPR, j = a.start + i;
    const int p = it % PPR;
    if (i >= a.n) break;
    const int page = j < len ? paged_page(a.c, a.seq, j) : -1;
    uint32_t x[EPP / 4] = {}, y[EPP / 4] = {};
    float sx = 0.f, sy = 0.f;
    if (page >= 0) {
      const long row = paged_row(a.c, page, h, j);
      __builtin_memcpy(x, a.c.k + row * D + p * EPP, EPP);
      __builtin_memcpy(y, a.c.v + row * D + p * EPP, EPP);
      sx = a.c.ks[row / PAGED_BLOCK];
      sy = a.c.vs[row / PAGED_BLOCK];
    }
    u32x4 out[2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      IT f[EPP];
#pragma unroll
      for (int e = 0; e < EPP; e += 4) {
        float g[4];
        e4m3_floats(kv ? y[e / 4] : x[e / 4], g);
#pragma unroll
        for (int u = 0; u < 4; ++u) f[e + u] = from_f32<IT>(g[u] * (kv ? sy : sx));
      }
      __builtin_memcpy(&out[kv], f, 16);
    }
    const long to = ((long)h * a.n + i) * PPR + p;
    __builtin_nontemporal_store(out[0], (u32x4*)a.K + to);
    __builtin_nontemporal_store(out[1], (u32x4*)a.V + to);
  }
  if (a.beta && tid < PAGED_GATHER_ROWS && i0 + tid < a.n) {
    const long i = i0 + tid, j = a.start + i;
    const int page = j < len ? paged_page(a.c, a.seq, j) : -1;
    a.beta[(long)h * a.n + i] = page >= 0 ? a.c.beta[paged_row(a.c, page, h, j)] : 0.f;
  }
}

}  // namespace still
