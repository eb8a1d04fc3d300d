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
#include "cache_attn_device.h"

namespace usp {
namespace {

constexpr int kThreads = 256, kStep = kCacheStep;
typedef CacheUnits Units;

__device__ inline float group_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float group_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

template <int HS, int R>
struct Walk {
  static constexpr int RT = 16 * R, KI = HS / 32, ET = HS / 16, KV16 = HS / 64;     // KV16: 16-byte reads of a K row's quarter
  const CachePlan& p;
  int lane, c, g;

  // a step's codes and scales
  u32x4 k[4][KV16], v[ET];
  uint32_t ks, vs;
  int number_k, number_v;       // pages of the blocks that the lane reads of K and of V; -1: none

  __device__ explicit Walk(const CachePlan& plan, int l) : p(plan), lane(l), c(l & 15), g(l >> 4) {}

  // (Neither lookups nor loads stand under a condition, where each would be waited for before the next: a block behind the last
  // one that counts is looked up as that one, and a page that is not there reads page 0.)
  __device__ void find(const int32_t* row, int step, int vis) {
    const int bk = step * 4 + (c >> 2), bv = step * 4 + g;
    const int nk = row[cache_entry(bk, vis, p.a.page_shift)], nv = row[cache_entry(bv, vis, p.a.page_shift)];
    number_k = cache_counts(bk, vis, nk, p.a.pages) ? nk : -1;
    number_v = cache_counts(bv, vis, nv, p.a.pages) ? nv : -1;
  }
  __device__ void load_k(int step, int head) {
    const int inside = ((step * 4 + (c >> 2)) * 16) & ((1 << p.a.page_shift) - 1);
    const int64_t place = (int64_t)(number_k < 0 ? 0 : number_k) * p.a.hk + head;
    const uint8_t* const at = p.a.k_codes + ((place << p.a.page_shift) + inside + (c & 3)) * HS + g * (HS / 4);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < KV16; ++i) k[t][i] = *(const u32x4*)(at + t * 4 * HS + i * 16);
    ks = p.a.k_scale[place];
  }
  __device__ void load_v(int step, int head) {
    const int inside = ((step * 4 + g) * 16) & ((1 << p.a.page_shift) - 1);
    const int64_t place = (int64_t)(number_v < 0 ? 0 : number_v) * p.a.hk + head;
    const uint8_t* const at = p.a.v_codes + ((place << p.a.page_shift) + inside) * HS + c * 16;
#pragma unroll
    for (int e = 0; e < ET; ++e) v[e] = *(const u32x4*)(at + e * 256);
    vs = p.a.v_scale[place];
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
      const float scale_k = scale_of(ks);
      // S^T = K Q^T
      f32x4 x[R][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int r = 0; r < R; ++r) x[r][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < KI; ++i) {
          const bf16x8 w = widened(k[t][i / 2][i % 2 * 2], k[t][i / 2][i % 2 * 2 + 1], scale_k);
#pragma unroll
          for (int r = 0; r < R; ++r) x[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, q[r][i], x[r][t], 0, 0, 0);
        }
      }
      if (more) load_k(s + 1, head);
      const int key0 = s * kStep + g * 16;            // the lane's first key
      const bool missing = __ballot(!valid) != 0, masked = (s + 1) * kStep > vis_first || missing;
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
      // what stands behind the last key, or in a page that is not there, counts as zero, whatever it is
      if ((s + 1) * kStep > vis || missing) {
        const int left = valid ? vis - key0 : 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t stay = first_bytes(left - 4 * w);
#pragma unroll
          for (int e = 0; e < ET; ++e) v[e][w] &= stay;
        }
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
      const float scale_v = valid ? scale_of(vs) : 1.0f;      // (0 times the NaN of a page in no use would be NaN)
#pragma unroll
      for (int e = 0; e < ET; ++e)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x8 w = widened(v[e][2 * j], v[e][2 * j + 1], scale_v);
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
        if (g == 0) a.lse[(int64_t)h * a.total_q + u.cu + token] = natural_lse(m[r], l[r]);
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
__global__ __launch_bounds__(kThreads, 2) void cache_attn_kernel(CachePlan p) {
  __shared__ Shares<kThreads> shares;
  constexpr int RT = 16 * R;
  const int64_t all = shares.count(p.a, RT);
  const int wave = __builtin_amdgcn_readfirstlane(((int)threadIdx.x >> 6) * (int)gridDim.x + (int)blockIdx.x);
  const int workers = all < p.workers ? (int)all : p.workers;
  CacheLeft left = {0, -1, 0, 0};
  if (wave < workers) {
    Walk<HS, R> walk(p, threadIdx.x & 63);
    float* const slots = p.partial + (int64_t)wave * 2 * RT * (HS + 2);
    shares.walk(p.a, RT, all * wave / workers, all * (wave + 1) / workers,
                [&](const CacheUnits& u, int seq, const CacheUnits::Place& at, int end, int of) __attribute__((always_inline)) {
                  const bool begins = at.step == 0, ends = end == of;
                  walk.unit(u, seq, at.head, at.tile, at.step, end, begins && ends, slots + (begins ? RT * (HS + 2) : 0));
                  if (!begins) left.first = ends ? 2 : 1;
                  else if (!ends) left.seq = seq, left.head = at.head, left.tile = at.tile;
                });
  }
  if ((threadIdx.x & 63) == 0 && wave < p.workers) p.left[wave] = left;
}

// Joins the partial results of one unit: the beginning that worker w left, then what the workers behind it left up to the unit's
// end.  blockIdx.y: which of the unit's rows.
template <int HS>
__global__ __launch_bounds__(kThreads) void cache_attn_join_kernel(CachePlan p, int rows_per_tile) {
  const int64_t slot = (int64_t)rows_per_tile * (HS + 2);
  const CacheAttnArgs& a = p.a;
  const int w = blockIdx.x;
  const CacheLeft mine = p.left[w];
  if (mine.seq < 0) return;
  const CacheUnits u(a, mine.seq, rows_per_tile);
  const int rows = u.rows(a, mine.tile, rows_per_tile);
  int last = w + 1;
  while (last < p.workers - 1 && p.left[last].first == 1) ++last;
  for (int i = blockIdx.y * kThreads + threadIdx.x; i < rows * HS; i += kThreads * gridDim.y) {
    const int row = i / HS, e = i - row * HS;
    const float* at = p.partial + (2 * (int64_t)w + 1) * slot + row * (HS + 2);
    float m = at[0], l = at[1], o = at[2 + e];
    for (int x = w + 1; x <= last; ++x) {
      at = p.partial + 2 * (int64_t)x * slot + row * (HS + 2);
      const float mx = at[0], lx = at[1], ox = at[2 + e];
      const float top = fmaxf(m, mx), use = top == -INFINITY ? 0.0f : top;
      const float keep = exp2f(m - use), add = exp2f(mx - use);
      l = l * keep + lx * add;
      o = o * keep + ox * add;
      m = top;
    }
    const int64_t row_in = (int64_t)mine.tile * rows_per_tile + row;
    const int token = (int)(row_in / a.group), h = mine.head * a.group + (int)(row_in - (int64_t)token * a.group);
    const float y = l == 0.0f ? 0.0f : o / l;
    const int64_t to = ((int64_t)(u.cu + token) * (a.hk * a.group) + h) * HS + e;
    if (a.o_dtype == USP_BF16) ((__bf16*)a.o)[to] = (__bf16)y;
    else ((float*)a.o)[to] = y;
    if (e == 0) a.lse[(int64_t)h * a.total_q + u.cu + token] = natural_lse(m, l);
  }
}

// Up to 16 rows of a request fit one product of the kernel that has a wave to itself; more go to the kernel for many rows.
bool few_rows(int group, int max_q) { return (int64_t)group * (max_q < 1 ? 1 : max_q) <= 16; }
int rows_of(bool few) { return few ? 16 : kCacheRowsTile; }
int workers_of(bool few) { return few ? kPlanCUs * 8 : kPlanCUs; }

}  // namespace

size_t cache_attn_workspace(int group, int hs, int max_q) {
  const bool few = few_rows(group, max_q);
  return (size_t)workers_of(few) * (sizeof(CacheLeft) + (size_t)2 * rows_of(few) * (hs + 2) * sizeof(float));
}

int launch_cache_attn(const CacheAttnArgs& a, int max_q, hipStream_t stream) {
  const bool few = few_rows(a.group, max_q);
  CachePlan p = {a, workers_of(few), (CacheLeft*)a.workspace, nullptr};
  p.partial = (float*)(p.left + p.workers);
  if (few) {
    const dim3 grid(p.workers / (kThreads / 64));
    if (a.hs == 128) cache_attn_kernel<128, 1><<<grid, kThreads, 0, stream>>>(p);
    else cache_attn_kernel<64, 1><<<grid, kThreads, 0, stream>>>(p);
  } else {
    const int st = launch_cache_attn_rows(p, stream);
    if (st != USP_OK) return st;
  }
  const dim3 grid(p.workers, few ? 1 : 8);
  if (a.hs == 128) cache_attn_join_kernel<128><<<grid, kThreads, 0, stream>>>(p, rows_of(few));
  else cache_attn_join_kernel<64><<<grid, kThreads, 0, stream>>>(p, rows_of(few));
  return launch_status();
}

}  // namespace usp
