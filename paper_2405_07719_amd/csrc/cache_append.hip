// K and V rows into the pages of the 8-bit cache.
//
// HBM-bound: the values are read once, a third of their bytes or less are written.  A wave has one page, one KV head and one of
// K and V: the rows of a page stand together in `slots`, so the wave that finds a row whose predecessor lies in another page
// owns that page, its exponent byte and the tiles of V that the rows share with older tokens; nobody else writes there, and
// no atomics or second pass over the cache are needed.  It walks the page in tiles of 16 tokens: the maximum over all of them,
// then (again from the caches, or still in registers where there is one tile) the codes.
//
// Measured: K and V of 38 thousand rows of 12 prompts, as columns of a QKV product (8 heads of 128, 234 MB) 61 us, 3.9 TB/s: rows
// come in pieces of 256 bytes, 12 KB apart, and the last round of pages is a part of one (9900 pages for 3072 waves at a time);
// more waves with fewer registers were no faster (65 us).  One row for each of 64 requests 6.5 us: latency.
//
// A power of two as scale makes both steps exact but for the one rounding to e4m3: value * 2^-e is exact, and codes whose page
// needs a larger exponent later are halved exactly, as long as they stay normal (2^-6 and more).
#include <float.h>

#include "serve_internal.h"

namespace usp {
namespace {

constexpr int kThreads = 256;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline float power_of_two(int e) { return __int_as_float((e + 127) << 23); }

// what a value counts towards the page's maximum: NaN and infinities nothing
__device__ inline float magnitude_of(float x) {
  const float y = fabsf(x);
  return y <= FLT_MAX ? y : 0.0f;
}

// x / 2^e as the conversion takes it where values may be infinite or beyond the largest code: NaN for NaN and infinities
__device__ inline float held(float x, float inv) {
  const float y = x * inv, z = fabsf(y) > 448.0f ? copysignf(448.0f, y) : y;
  return fabsf(x) <= FLT_MAX ? z : __int_as_float(0x7fc00000);
}

__device__ inline uint32_t codes4(float a, float b, float c, float d) {
  int x = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, x, true);
}

// four codes at another exponent
__device__ inline uint32_t recoded(uint32_t x, float by) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  return codes4(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
}
__device__ inline u32x4 recoded(u32x4 x, float by) {
  return u32x4{recoded(x[0], by), recoded(x[1], by), recoded(x[2], by), recoded(x[3], by)};
}

// The smallest e with most <= 448 * 2^e = 1.75 * 2^(8 + e).
__device__ inline int exponent_for(float most) {
  const uint32_t bits = (uint32_t)__float_as_int(most);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000);
  return e < kCacheMinExp ? kCacheMinExp : e > kCacheMaxExp ? kCacheMaxExp : e;
}

// Two neighbouring elements as they were loaded, and as numbers.
template <typename T> struct Two;
template <> struct Two<__bf16> {
  typedef uint32_t raw;
  static __device__ f32x2 values(raw x) { return f32x2{__int_as_float((int)(x << 16)), __int_as_float((int)(x & 0xffff0000u))}; }
};
template <> struct Two<float> {
  typedef u32x2 raw;
  static __device__ f32x2 values(raw x) { return f32x2{__int_as_float((int)x[0]), __int_as_float((int)x[1])}; }
};

// One page and head of K (V_TILES false) or V.  x: the head's elements in the row of the first token; `n` tokens from place
// `old` on; codes: the page's codes of the head.
// PAST_CACHES: values are read nontemporally.
template <typename T, int HS, bool V_TILES, bool PAST_CACHES>
struct Page {
  // K: eight elements of a row to a lane; V: two columns to a lane, of 16 tokens (hs 128) or 8 (hs 64)
  static constexpr int kPer = V_TILES ? 2 : 8, kPairs = kPer / 2, kLanesPerRow = HS / kPer, kGroups = 64 / kLanesPerRow,
                       kTokens = 16 / kGroups;
  // Tiles whose values are all on their way, and stay in registers, at once: the 64 tokens of an ordinary page.
  static constexpr int kTiles = 4;
  typedef typename Two<T>::raw Raw;
  const T* x;
  int64_t stride;
  uint8_t* codes;
  int lane, old, n;

  __device__ int place(int tile, int i) const {      // of a lane's i-th token
    const int group = lane / kLanesPerRow;
    return tile * 16 + (V_TILES ? group * kTokens + i : i * kGroups + group);
  }
  __device__ bool given(int p) const { return p >= old && p < old + n; }
  __device__ int column() const { return lane % kLanesPerRow * kPer; }

  // A lane's elements of a tile.  Places that are not given read one that is: a load under a condition would be waited for
  // where it stands, one after the other.
  __device__ void load(int tile, Raw (&v)[kTokens][kPairs]) const {
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      int p = place(tile, i) - old;
      p = p < 0 ? 0 : p < n ? p : n - 1;
      const T* const from = x + p * stride + column();
      if constexpr (V_TILES) {
        v[i][0] = PAST_CACHES ? __builtin_nontemporal_load((const Raw*)from) : *(const Raw*)from;
      } else {
#pragma unroll
        for (int w = 0; w < (int)sizeof(T) / 2; ++w)
          ((u32x4*)v[i])[w] = PAST_CACHES ? __builtin_nontemporal_load((const u32x4*)from + w) : ((const u32x4*)from)[w];
      }
    }
  }

  // largest magnitude, infinity among them (a place that is not given repeats one that is)
  __device__ static float most(const Raw (&v)[kTokens][kPairs]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kTokens; ++i)
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const f32x2 y = Two<T>::values(v[i][j]);
        m = fmaxf(m, fmaxf(fabsf(y[0]), fabsf(y[1])));
      }
    return m;
  }
  __device__ static float most_finite(const Raw (&v)[kTokens][kPairs]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kTokens; ++i)
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const f32x2 y = Two<T>::values(v[i][j]);
        m = fmaxf(m, fmaxf(magnitude_of(y[0]), magnitude_of(y[1])));
      }
    return m;
  }

  // `odd`: infinities or values beyond the largest code may be among them; `by`: what codes of older tokens are multiplied
  // by (1: nothing)
  __device__ void store(int tile, const Raw (&v)[kTokens][kPairs], float inv, bool odd, float by) const {
    const auto code = [&](float y) { return odd ? held(y, inv) : y * inv; };
    if constexpr (!V_TILES) {
#pragma unroll
      for (int i = 0; i < kTokens; ++i) {
        const int p = place(tile, i);
        f32x2 y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[j] = Two<T>::values(v[i][j]);
          y[j] = f32x2{code(y[j][0]), code(y[j][1])};
        }
        if (given(p))
          *(u32x2*)(codes + p * HS + column()) = u32x2{codes4(y[0][0], y[0][1], y[1][0], y[1][1]), codes4(y[2][0], y[2][1], y[3][0], y[3][1])};
      }
    } else {
      const int first = place(tile, 0);
      const bool all = first >= old && first + kTokens <= old + n, none = first + kTokens <= old || first >= old + n;
      // (a group of lanes none of whose tokens are given still has older ones to round again)
      if (none && (by == 1.0f || first >= old)) return;
      uint32_t c[2][kTokens / 4];
#pragma unroll
      for (int w = 0; w < kTokens / 4; ++w) {
        f32x2 y[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          y[b] = Two<T>::values(v[4 * w + b][0]);
          y[b] = f32x2{code(y[b][0]), code(y[b][1])};
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) c[j][w] = codes4(y[0][j], y[1][j], y[2][j], y[3][j]);
      }
      uint32_t* const at = (uint32_t*)(codes + tile * 16 * HS + column() * 16 + first % 16);
      if (!all) {
#pragma unroll
        for (int w = 0; w < kTokens / 4; ++w) {
          uint32_t keep = 0, older = 0;                 // bytes that stay; bytes of older tokens
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int p = first + 4 * w + b;
            if (!given(p)) keep |= 0xffu << (8 * b);
            if (p < old) older |= 0xffu << (8 * b);
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t was = at[4 * j + w];
            if (by != 1.0f) was = (recoded(was, by) & older) | (was & ~older);
            c[j][w] = (c[j][w] & ~keep) | (was & keep);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if constexpr (kTokens == 16) *(u32x4*)(at + 4 * j) = u32x4{c[j][0], c[j][1], c[j][2], c[j][3]};
        else *(u32x2*)(at + 4 * j) = u32x2{c[j][0], c[j][1]};
      }
    }
  }

  __device__ void write(uint8_t* scale) const {
    const int t0 = old / 16, tiles = (old + n - 1) / 16 - t0 + 1;
    const int was = old ? (int)*scale - 127 : kCacheMinExp;
    Raw v[kTiles][kTokens][kPairs];
    // the first tiles last, so that they are in registers when their codes are formed
    float m = 0.0f, finite = 0.0f;
    bool infinite = false;
    for (int round = 0; round < 2; ++round) {
      for (int t = tiles > kTiles ? kTiles : 0; ; t = 0) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          if (t + i < tiles && (round == 0 || tiles > kTiles)) load(t0 + t + i, v[i]);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          if (t + i < tiles) {
            if (round == 0) m = fmaxf(m, most(v[i]));
            else finite = fmaxf(finite, most_finite(v[i]));
          }
        if (t == 0) break;
      }
      if (round == 0) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
        infinite = m > FLT_MAX;
        if (!infinite) break;
      }
    }
    if (infinite) {
      m = finite;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    }
    int e = exponent_for(m);
    const int floor = was < kCacheMinExp ? kCacheMinExp : was > kCacheMaxExp ? kCacheMaxExp : was;
    e = old && floor > e ? floor : e;
    const float inv = power_of_two(-e);
    const bool odd = infinite || m * inv > 448.0f;
    const int less = floor - e;
    const float by = old && less < 0 ? power_of_two(less < -126 ? -126 : less) : 1.0f;
    if (by != 1.0f) {      // older tokens: rows of K, whole tiles of V (the tile that the first new token shares comes below)
      const int chunks = (V_TILES ? t0 * 16 : old) * HS / 16;
      for (int i = lane; i < chunks; i += 64) ((u32x4*)codes)[i] = recoded(((u32x4*)codes)[i], by);
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
      if (i < tiles) store(t0 + i, v[i], inv, odd, by);
    if (tiles > kTiles) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
        if (kTiles + i < tiles) load(t0 + kTiles + i, v[i]);
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
        if (kTiles + i < tiles) store(t0 + kTiles + i, v[i], inv, odd, 1.0f);
    }
    if (lane == 0) *scale = (uint8_t)(e + 127);
  }
};

template <typename T, int HS, bool PAST_CACHES>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(CacheAppendArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int tensor = (int)(item & 1);
  const int64_t rest = item >> 1, win = rest / a.hk;
  const int head = (int)(rest - win * a.hk), page = 1 << a.page_shift;
  const int64_t row0 = (a.first_window + win) * a.window;
  if (win >= a.windows || row0 >= a.rows) return;
  const auto number_of = [&](int slot) { return slot >= 0 && slot < a.slots_end ? slot >> a.page_shift : -1; };
  bool leads = false;
  if (lane < a.window && row0 + lane < a.rows) {
    const int number = number_of(a.slots[row0 + lane]);
    leads = number >= 0 && (row0 + lane == 0 || number != number_of(a.slots[row0 + lane - 1]));
  }
  for (uint64_t left = __ballot(leads); left; left &= left - 1) {
    int64_t row = row0 + __builtin_ctzll(left);
    int slot = a.slots[row];
    const int number = slot >> a.page_shift;
    const int64_t place = (int64_t)number * a.hk + head;
    for (bool again = false;; again = true) {        // stretches of ascending places within the page, mostly one
      int n = 0;
      const int old = slot & (page - 1);
      for (;;) {
        const int i = n + lane;
        const bool follows = old + i < page && row + i < a.rows && a.slots[row + i] == slot + i;
        const uint64_t ends = ~__ballot(follows);
        if (ends) {
          n += __builtin_ctzll(ends);
          break;
        }
        n += 64;
      }
      if (again) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");      // the stretch before wrote to this page
      const T* const x = (const T*)a.x[tensor] + row * a.stride[tensor] + head * HS;
      uint8_t* const codes = a.codes[tensor] + place * page * HS;
      if (tensor) Page<T, HS, true, PAST_CACHES>{x, a.stride[1], codes, lane, old, n}.write(a.scale[1] + place);
      else Page<T, HS, false, PAST_CACHES>{x, a.stride[0], codes, lane, old, n}.write(a.scale[0] + place);
      row += n;
      if (row >= a.rows) break;
      slot = a.slots[row];
      if (number_of(slot) != number) break;
    }
  }
}

template <typename T>
void launch(const CacheAppendArgs& a, unsigned grid, bool past_caches, hipStream_t stream) {
  const auto go = [&](auto kernel) { kernel<<<dim3(grid), kThreads, 0, stream>>>(a); };
  if (a.hs == 128) past_caches ? go(cache_append_kernel<T, 128, true>) : go(cache_append_kernel<T, 128, false>);
  else past_caches ? go(cache_append_kernel<T, 64, true>) : go(cache_append_kernel<T, 64, false>);
}

}  // namespace

int launch_cache_append(const CacheAppendArgs& args, int dtype, hipStream_t stream) {
  CacheAppendArgs a = args;
  // Rows in which a wave looks for pages that begin there.  More rows than there can be requests are stretches of several
  // tokens: 38 thousand rows of 12 prompts take 67 us with 64 rows to a wave, 75 with 32 and 218 with 8, most of whose waves find
  // nothing.  One token of each request is a page to a row: then a wave would have to write one page after the other.
  const bool many = a.rows > USP_CACHE_MAX_REQUESTS;
  a.window = many ? 64 : a.rows > 2048 ? 8 : 1;
  // (several launches where one would have 2^32 threads or more)
  const int64_t windows = (a.rows + a.window - 1) / a.window, most = max_workgroups(kThreads) * (kThreads / 64) / (2 * a.hk);
  for (a.first_window = 0; a.first_window < windows; a.first_window += most) {
    a.windows = windows - a.first_window < most ? windows - a.first_window : most;
    const unsigned grid = (unsigned)((a.windows * a.hk * 2 + kThreads / 64 - 1) / (kThreads / 64));
    // A long prompt's rows, read once, go past the caches (66 -> 61 us for the same rows); a few are in them still (64 rows: 6.4
    // us, past the caches 6.9).
    if (dtype == USP_BF16) launch<__bf16>(a, grid, many, stream);
    else launch<float>(a, grid, many, stream);
  }
  return launch_status();
}

}  // namespace usp
