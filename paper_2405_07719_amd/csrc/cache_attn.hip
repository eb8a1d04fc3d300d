// Attention over the 8-bit cache: rows of ragged requests against their cached tokens.
//
// A unit is one request, KV head and tile of RT = 16 R rows (tokens x query heads of the KV head, so the query heads that
// share K and V share one read of them); its keys are walked in steps of 64.  All steps of all units, laid one behind the
// other, are cut evenly among the waves of the launch, whatever the lengths: every wave works out from the lengths, which
// stand on the device, where its share begins.  A unit that lies within one wave's share is finished there; one that is cut
// leaves partial results (maximum, sum, unnormalised output), of which a wave has two at most - the end of a unit that
// began before its share, and the beginning of one that goes on behind it - and a second launch joins them, in the order
// of the keys.
//
// The products are those of S^T = K Q^T and O^T = V^T P^T, so that a lane holds one row's scores and its output elements
// all along: row c = lane % 16, keys and elements by g = lane / 16.  Row 4 g' + r of the t-th 16-key product of a step
// is key 16 g' + 4 t + r, which gives lane group g the 16 keys of one block of the cache: its P is, as it stands, the
// operand of the second product, whose V operand is 16 bytes of one column of a V tile.  Nothing goes through LDS.
#include <math.h>

#include "serve_internal.h"

namespace usp {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kStep = kCacheStep;
typedef CacheUnits Units;

// What a wave leaves for the joining launch: `first`: 0, or its share begins inside a unit, which goes on behind it (1) or
// ends in it (2); seq >= 0: its share ends inside the unit (seq, head, tile), which begins in it.
struct Left { int first, seq, head, tile; };

struct Plan {
  CacheAttnArgs a;
  int waves;          // that have a share, at most; places in `left`
  Left* left;
  float* partial;     // [waves][2][RT][hs + 2]: per row m, l, then O
  int rows_per_tile;
};

__device__ inline float group_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float group_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// eight codes as the operand of a product
__device__ inline bf16x8 widened(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 0x80 in each byte that is a NaN code
__device__ inline uint32_t nan_codes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// bytes of a word whose first `n` (any number) stay
__device__ inline uint32_t first_bytes(int n) { return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : 0xffffffffu >> (32 - 8 * n); }

template <int HS, int R>
struct Walk {
  static constexpr int RT = 16 * R, KI = HS / 32, ET = HS / 16, KV16 = HS / 64;     // KV16: 16-byte reads of a K row's quarter
  const Plan& p;
  int lane, c, g;

  // a step's codes and scales
  u32x4 k[4][KV16], v[ET];
  float ks, vs;
  int number_k, number_v;       // pages of the blocks that the lane reads of K and of V; -1: none

  __device__ explicit Walk(const Plan& plan, int l) : p(plan), lane(l), c(l & 15), g(l >> 4) {}

  __device__ void find(const int32_t* row, int step, int vis) {
    number_k = cache_page(p.a, row, step * 4 + (c >> 2), vis);
    number_v = cache_page(p.a, row, step * 4 + g, vis);
  }
  __device__ void load_k(int step, int head) {
    const int inside = ((step * 4 + (c >> 2)) * 16) & ((1 << p.a.page_shift) - 1);
    const int64_t place = (int64_t)number_k * p.a.hk + head;
    const uint8_t* const at = p.a.k_codes + ((place << p.a.page_shift) + inside + (c & 3)) * HS + g * (HS / 4);
    ks = 1.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < KV16; ++i) k[t][i] = u32x4{0, 0, 0, 0};
    if (number_k >= 0) {
      ks = __int_as_float((int)p.a.k_scale[place] << 23);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < KV16; ++i) k[t][i] = *(const u32x4*)(at + t * 4 * HS + i * 16);
    }
  }
  __device__ void load_v(int step, int head) {
    const int inside = ((step * 4 + g) * 16) & ((1 << p.a.page_shift) - 1);
    const int64_t place = (int64_t)number_v * p.a.hk + head;
    const uint8_t* const at = p.a.v_codes + ((place << p.a.page_shift) + inside) * HS + c * 16;
    vs = 1.0f;
#pragma unroll
    for (int e = 0; e < ET; ++e) v[e] = u32x4{0, 0, 0, 0};
    if (number_v >= 0) {
      vs = __int_as_float((int)p.a.v_scale[place] << 23);
#pragma unroll
      for (int e = 0; e < ET; ++e) v[e] = *(const u32x4*)(at + e * 256);
    }
  }

  // Steps [s0, s1) of a unit of `steps` ones: results to o and lse if these are all, else to partial result `slot`.
  __device__ void unit(const Units& u, int seq, int head, int tile, int s0, int s1, bool whole, float* slot) {
    const CacheAttnArgs& a = p.a;
    const int32_t* const row = a.block_table + (int64_t)seq * a.max_pages;
    const int rows = u.rows(a, tile, RT);
    // keys that the tile's first and last rows see
    const int64_t row_first = (int64_t)tile * RT;
    const int vis = u.seen_by((row_first + rows - 1) / a.group), vis_first = u.seen_by(row_first / a.group);
    int limit[R];
    bf16x8 q[R][KI];
    f32x4 o[R][ET];
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int at = r * 16 + c, token = (int)((row_first + at) / a.group), h = (int)(row_first + at - (int64_t)token * a.group);
      limit[r] = at < rows ? u.seen_by(token) : vis;
      m[r] = -INFINITY;
      l[r] = 0.0f;
      const __bf16* const from = (const __bf16*)a.q + (int64_t)(u.cu + token) * a.q_stride + (head * a.group + h) * HS + g * (HS / 4);
#pragma unroll
      for (int i = 0; i < KI; ++i)
        q[r][i] = at < rows ? *(const bf16x8*)(from + i * 8) : bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < ET; ++e) o[r][e] = f32x4{0, 0, 0, 0};
    }
    const int end = (vis + kStep - 1) / kStep < s1 ? (vis + kStep - 1) / kStep : s1;
    if (s0 < end) {
      find(row, s0, vis);
      load_k(s0, head);
      load_v(s0, head);
    }
    for (int s = s0; s < end; ++s) {
      const bool more = s + 1 < end;
      const bool valid = number_v >= 0;               // of the block whose 16 keys the lane's scores are
      if (more) find(row, s + 1, vis);
      // S^T = K Q^T
      f32x4 x[R][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int r = 0; r < R; ++r) x[r][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < KI; ++i) {
          const bf16x8 w = widened(k[t][i / 2][i % 2 * 2], k[t][i / 2][i % 2 * 2 + 1], ks);
#pragma unroll
          for (int r = 0; r < R; ++r) x[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, q[r][i], x[r][t], 0, 0, 0);
        }
      }
      if (more) load_k(s + 1, head);
      const int key0 = s * kStep + g * 16;            // the lane's first key
      const bool masked = (s + 1) * kStep > vis_first || __ballot(!valid);
      if (masked) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!valid || key0 + 4 * t + e >= limit[r]) x[r][t][e] = -INFINITY;
      }
      bf16x8 pr[R][2];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = x[r][0][0];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, x[r][t][e]);
        top = group_max(top) * a.scale_log2e;
        const float now = fmaxf(m[r], top), use = now == -INFINITY ? 0.0f : now;
        const float alpha = exp2f(m[r] - use);
        m[r] = now;
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[r][t][e] = __builtin_amdgcn_exp2f(x[r][t][e] * a.scale_log2e - use);
            sum += x[r][t][e];
          }
        l[r] = l[r] * alpha + sum;
        if (__ballot(alpha != 1.0f)) {
#pragma unroll
          for (int e = 0; e < ET; ++e) o[r][e] *= alpha;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) pr[r][j][e] = (__bf16)x[r][2 * j + e / 4][e % 4];
      }
      // what stands behind the last key counts as zero, whatever it is
      if ((s + 1) * kStep > vis) {
#pragma unroll
        for (int e = 0; e < ET; ++e)
#pragma unroll
          for (int w = 0; w < 4; ++w) v[e][w] &= first_bytes(vis - key0 - 4 * w);
      }
      // NaN in a value that some rows of the tile see and others do not: 0 times it would be NaN for those.  Counted apart,
      // with another product, and taken as zero in the one that counts.
      if (vis_first < vis && (s + 1) * kStep > vis_first) {
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < ET; ++e)
#pragma unroll
          for (int w = 0; w < 4; ++w) any |= nan_codes(v[e][w]);
        if (__ballot(any != 0)) {
#pragma unroll
          for (int e = 0; e < ET; ++e) {
            bf16x8 is[2];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t n = nan_codes(v[e][w]);
#pragma unroll
              for (int b = 0; b < 4; ++b) is[w / 2][w % 2 * 4 + b] = (__bf16)((n >> (8 * b + 7)) & 1 ? 1.0f : 0.0f);
              v[e][w] &= ~((n >> 7) * 0xffu);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
              f32x4 count = {0, 0, 0, 0};
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                bf16x8 sees;
#pragma unroll
                for (int b = 0; b < 8; ++b) sees[b] = (__bf16)(valid && key0 + 8 * j + b < limit[r] ? 1.0f : 0.0f);
                count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is[j], sees, count, 0, 0, 0);
              }
#pragma unroll
              for (int b = 0; b < 4; ++b)
                if (count[b] > 0.0f) o[r][e][b] = NAN;
            }
          }
        }
      }
      // O^T += V^T P^T
#pragma unroll
      for (int e = 0; e < ET; ++e)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x8 w = widened(v[e][2 * j], v[e][2 * j + 1], vs);
#pragma unroll
          for (int r = 0; r < R; ++r) o[r][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, pr[r][j], o[r][e], 0, 0, 0);
        }
      if (more) load_v(s + 1, head);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      l[r] = group_sum(l[r]);
      const int at = r * 16 + c;
      if (at >= rows) continue;
      if (whole) {
        const int token = (int)((row_first + at) / a.group), h = head * a.group + (int)(row_first + at - (int64_t)token * a.group);
        const float inv = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
        const int64_t to = ((int64_t)(u.cu + token) * (a.hk * a.group) + h) * HS + g * 4;
#pragma unroll
        for (int e = 0; e < ET; ++e) {
          const f32x4 y = o[r][e] * inv;
          if (a.o_dtype == USP_BF16) *(bf16x4*)((__bf16*)a.o + to + e * 16) = __builtin_convertvector(y, bf16x4);
          else *(f32x4*)((float*)a.o + to + e * 16) = y;
        }
        if (g == 0) a.lse[(int64_t)h * a.total_q + u.cu + token] = l[r] == 0.0f ? -INFINITY : (m[r] + log2f(l[r])) * 0.693147180559945309f;
      } else {
        float* const to = slot + (int64_t)at * (HS + 2);
        if (g == 0) *(f32x2*)to = f32x2{m[r], l[r]};
#pragma unroll
        for (int e = 0; e < ET; ++e) {
          *(f32x2*)(to + 2 + e * 16 + g * 4) = f32x2{o[r][e][0], o[r][e][1]};
          *(f32x2*)(to + 4 + e * 16 + g * 4) = f32x2{o[r][e][2], o[r][e][3]};
        }
      }
    }
  }
};

template <int HS, int R>
__global__ __launch_bounds__(kThreads, R == 4 ? 1 : 2) void cache_attn_kernel(Plan p) {
  __shared__ int64_t before[kThreads + 1];       // steps of the requests before a thread's first one
  __shared__ int64_t part[kThreads / 64];
  const CacheAttnArgs& a = p.a;
  constexpr int RT = 16 * R;
  const int tid = threadIdx.x, lane = tid & 63, n = a.n_seqs;
  const int per = (n + kThreads - 1) / kThreads;
  int64_t sum = 0;
  for (int i = tid * per; i < (tid + 1) * per && i < n; ++i) sum += Units(a, i, RT).per_head * a.hk;
  int64_t upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 63) part[tid >> 6] = upto;
  __syncthreads();
  int64_t all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < tid >> 6) upto += part[w];
    all += part[w];
  }
  before[tid + 1] = upto;
  if (tid == 0) before[0] = 0;
  __syncthreads();

  const int wave = __builtin_amdgcn_readfirstlane((tid >> 6) * (int)gridDim.x + (int)blockIdx.x);
  const int shares = all < p.waves ? (int)all : p.waves;
  Left left = {0, -1, 0, 0};
  if (wave < shares) {
    int64_t pos = all * wave / shares;
    const int64_t stop = all * (wave + 1) / shares;
    float* const slots = p.partial + (int64_t)wave * 2 * RT * (HS + 2);
    int lo = 0, hi = kThreads;                   // the last thread whose first request begins at pos or before
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (before[mid] <= pos) lo = mid;
      else hi = mid;
    }
    int64_t start = before[lo];                  // where request `seq` begins
    int seq = __builtin_amdgcn_readfirstlane(lo * per);
    Walk<HS, R> walk(p, lane);
    while (pos < stop && seq < n) {
      const Units u(a, seq, RT);
      const int64_t steps = u.per_head * a.hk;
      if (pos >= start + steps) {
        start += steps;
        ++seq;
        continue;
      }
      const CacheUnits::Place at = u.locate(pos - start);
      const int head = at.head, tile = at.tile, s0 = at.step, of = u.steps(tile);
      const int s1 = stop - pos < of - s0 ? s0 + (int)(stop - pos) : of;
      const bool begins = s0 == 0, ends = s1 == of;
      walk.unit(u, seq, head, tile, s0, s1, begins && ends, slots + (begins ? RT * (HS + 2) : 0));
      if (!begins) left.first = ends ? 2 : 1;
      else if (!ends) left.seq = seq, left.head = head, left.tile = tile;
      pos += s1 - s0;
    }
  }
  if (lane == 0 && wave < p.waves) p.left[wave] = left;
}

// Joins the partial results of one unit: the beginning that wave w left, then what the waves behind it left up to the unit's end.
template <int HS, int R>
__global__ __launch_bounds__(kThreads) void cache_attn_join_kernel(Plan p) {
  constexpr int RT = 16 * R, kSlot = RT * (HS + 2);
  const CacheAttnArgs& a = p.a;
  const int w = blockIdx.x;
  const Left mine = p.left[w];
  if (mine.seq < 0) return;
  const Units u(a, mine.seq, RT);
  const int rows = u.rows(a, mine.tile, RT);
  int last = w + 1;
  while (last < p.waves - 1 && p.left[last].first == 1) ++last;
  for (int i = threadIdx.x; i < rows * HS; i += kThreads) {
    const int row = i / HS, e = i - row * HS;
    const float* at = p.partial + (int64_t)(2 * w + 1) * kSlot + row * (HS + 2);
    float m = at[0], l = at[1], o = at[2 + e];
    for (int x = w + 1; x <= last; ++x) {
      at = p.partial + (int64_t)(2 * x) * kSlot + row * (HS + 2);
      const float mx = at[0], lx = at[1], ox = at[2 + e];
      const float top = fmaxf(m, mx), use = top == -INFINITY ? 0.0f : top;
      const float keep = exp2f(m - use), add = exp2f(mx - use);
      l = l * keep + lx * add;
      o = o * keep + ox * add;
      m = top;
    }
    const int64_t row_in = (int64_t)mine.tile * RT + row;
    const int token = (int)(row_in / a.group), h = mine.head * a.group + (int)(row_in - (int64_t)token * a.group);
    const float y = l == 0.0f ? 0.0f : o / l;
    const int64_t to = ((int64_t)(u.cu + token) * (a.hk * a.group) + h) * HS + e;
    if (a.o_dtype == USP_BF16) ((__bf16*)a.o)[to] = (__bf16)y;
    else ((float*)a.o)[to] = y;
    if (e == 0) a.lse[(int64_t)h * a.total_q + u.cu + token] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.693147180559945309f;
  }
}

int tiles_of_16(int group, int max_q) {
  const int64_t rows = (int64_t)group * (max_q < 1 ? 1 : max_q);
  return rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
}
int waves_for(int r) { return r == 4 ? kPlanCUs * 4 : kPlanCUs * 8; }

template <int HS, int R>
void launch(const Plan& p, hipStream_t stream) {
  cache_attn_kernel<HS, R><<<dim3(p.waves / (kThreads / 64)), kThreads, 0, stream>>>(p);
  cache_attn_join_kernel<HS, R><<<dim3(p.waves), kThreads, 0, stream>>>(p);
}

}  // namespace

size_t cache_attn_workspace(int group, int hs, int max_q) {
  const int r = tiles_of_16(group, max_q);
  return (size_t)waves_for(r) * (sizeof(Left) + (size_t)2 * 16 * r * (hs + 2) * sizeof(float));
}

int launch_cache_attn(const CacheAttnArgs& a, int max_q, hipStream_t stream) {
  const int r = tiles_of_16(a.group, max_q);
  Plan p = {a, waves_for(r), (Left*)a.workspace, nullptr, 16 * r};
  p.partial = (float*)(p.left + p.waves);
  if (a.hs == 128) {
    if (r == 1) launch<128, 1>(p, stream);
    else if (r == 2) launch<128, 2>(p, stream);
    else launch<128, 4>(p, stream);
  } else {
    if (r == 1) launch<64, 1>(p, stream);
    else if (r == 2) launch<64, 2>(p, stream);
    else launch<64, 4>(p, stream);
  }
  return launch_status();
}

}  // namespace usp
