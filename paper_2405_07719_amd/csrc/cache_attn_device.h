// What the kernels of attention over the 8-bit cache share (device side).
#pragma once
#include <math.h>

#include "serve_internal.h"

namespace usp {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// eight codes as the operand of a product
__device__ inline bf16x8 widened(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// an exponent byte as the scale that it stands for
__device__ inline float scale_of(uint32_t x) { return __int_as_float((int)x << 23); }

// 0x80 in each byte that is a NaN code
__device__ inline uint32_t nan_codes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// bytes of a word whose first `n` (any number) stay
__device__ inline uint32_t first_bytes(int n) { return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : 0xffffffffu >> (32 - 8 * n); }

__device__ inline float natural_lse(float m, float l) { return l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.693147180559945309f; }

// The steps of all requests' units, laid one behind the other and cut into shares.  I: as in CacheUnits.
template <int THREADS, typename I>
struct Shares {
  typedef CacheUnits<I> Units;
  I before[THREADS + 1];           // steps of the requests before a thread's first one
  I part[THREADS / 64];
  CacheRequest first[THREADS];     // each thread's first request

  // By all threads of a workgroup: the steps in all.  Each thread counts `n / THREADS` requests in a row.
  __device__ I count(const CacheAttnArgs& a, int rows_per_tile) {
    const int tid = threadIdx.x, lane = tid & 63, n = a.n_seqs, per = (n + THREADS - 1) / THREADS;
    I sum = 0;
    for (int i = tid * per; i < (tid + 1) * per && i < n; ++i) {
      const CacheRequest r = Units::read(a, i);
      if (i == tid * per) first[tid] = r;
      sum += Units(a, r, rows_per_tile).per_head * a.hk;
    }
    I upto = sum, all = 0;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const I x = __shfl_up(upto, d);
      if (lane >= d) upto += x;
    }
    if (lane == 63) part[tid >> 6] = upto;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < tid >> 6) upto += part[w];
      all += part[w];
    }
    before[tid + 1] = upto;
    if (tid == 0) before[0] = 0;
    __syncthreads();
    return all;
  }

  // Where share `i` of `n` begins.
  __device__ static I cut(I all, int i, int n) {
    const I q = all / n, r = all - q * n;          // (r * i stays small)
    return q * i + r * i / n;
  }

  __device__ Units units(const CacheAttnArgs& a, int seq, int rows_per_tile) const {
    return a.n_seqs <= THREADS ? Units(a, first[seq], rows_per_tile) : Units(a, seq, rows_per_tile);
  }

  struct Where { int seq; I start; };      // a request, and its first step
  __device__ __forceinline__ Where find(const CacheAttnArgs& a, int rows_per_tile, I pos) const {
    // The last thread whose first request begins at pos or before, by 64 samples and then between two of them.
    constexpr int kEach = THREADS / 64;
    const int lane = threadIdx.x & 63, per = (a.n_seqs + THREADS - 1) / THREADS;
    int t = (63 - __builtin_clzll(__ballot(before[lane * kEach] <= pos))) * kEach;
    t += 63 - __builtin_clzll(__ballot(lane < kEach && before[t + (lane & (kEach - 1))] <= pos));
    t = __builtin_amdgcn_readfirstlane(t);
    Where w = {t * per, before[t]};
    for (; per > 1 && w.seq < a.n_seqs; ++w.seq) {
      const I steps = units(a, w.seq, rows_per_tile).per_head * a.hk;
      if (pos < w.start + steps) break;
      w.start += steps;
    }
    return w;
  }

  // The first step of the unit that step `pos` is of (the last step of all and one: itself).
  __device__ __forceinline__ I unit_start(const CacheAttnArgs& a, int rows_per_tile, I pos, I all) const {
    if (pos >= all) return all;
    const Where w = find(a, rows_per_tile, pos);
    return pos - units(a, w.seq, rows_per_tile).locate(pos - w.start).step;
  }

  // The pieces of units that steps [pos, stop) are, one after the other: visit(units, seq, place, end step, whole unit's steps).
  template <class Visit>
  __device__ __forceinline__ void walk(const CacheAttnArgs& a, int rows_per_tile, I pos, I stop, Visit visit) const {
    if (pos >= stop) return;
    Where w = find(a, rows_per_tile, pos);
    while (pos < stop && w.seq < a.n_seqs) {
      const Units u = units(a, w.seq, rows_per_tile);
      const I steps = u.per_head * a.hk;
      if (pos >= w.start + steps) {
        w.start += steps;
        ++w.seq;
        continue;
      }
      const typename Units::Place at = u.locate(pos - w.start);
      const int of = u.steps(at.tile), end = stop - pos < of - at.step ? at.step + (int)(stop - pos) : of;
      visit(u, w.seq, at.head, at.tile, at.step, end, of);
      pos += end - at.step;
    }
  }
};

}  // namespace
}  // namespace usp
