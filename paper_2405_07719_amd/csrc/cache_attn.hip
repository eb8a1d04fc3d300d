// Attention over the 8-bit cache: rows of ragged requests against their cached tokens.
//
// A unit is one request, KV head and tile of 16 rows (tokens x query heads of the KV head, so the query heads that share K and
// V share one read of them); its keys are walked in steps of 64.  All steps of all units, laid one behind the other, are cut
// evenly among one workgroup per CU, and a workgroup's share among its eight waves, whatever the lengths: every workgroup works
// out from the lengths, which stand on the device, where its share begins.  A unit that lies within one wave's share is finished
// there.  The waves that share one put their results (maximum, sum, unnormalised output) into LDS, where all threads
// add them up, each for a row and four columns, in the order of the keys.  Units cut between
// workgroups leave partial results to a joining launch, two to a workgroup at most: the end of a unit that began before its share,
// and the beginning of one that goes on behind it.
//
// The products are those of S^T = K Q^T and O^T = V^T P^T, so that a lane holds one row's scores and its output elements
// all along: row c = lane % 16, keys and elements by g = lane / 16.  Row 4 g' + r of the t-th 16-key product of a step
// is key 16 g' + 4 t + r, which gives lane group g the 16 keys of one block of the cache: its P is, as it stands, the
// operand of the second product, whose V operand is 16 bytes of one column of a V tile.  Codes go from memory to registers to
// the matrix cores, not through LDS.
//
// HBM-bound where there is much to read: 64 requests of 256 to 32768 tokens (8 KV heads of 128, 907 MB) 156 us, 5.8 TB/s, one of
// 212993 tokens (436 MB) 83 us, 5.3 TB/s with both launches; a large copy by the library reaches 4.9.  A wave has the codes of one step in
// flight, 16 KB, and a CU eight waves.  Short caches are bound by latency: one request of 1003 tokens 8.0 us and 4.5 us for
// the joining launch (lengths, pages, codes, two products, partial results: one after the other).  12 waves to a CU at head size
// 64 were no faster (27.7 against 26.4 us for 20 requests of up to 6007 tokens).
#include "cache_attn_device.h"

namespace usp {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64, kStep = kCacheStep, kTile = 16, kJoinThreads = 256;

__device__ inline float group_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float group_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// ONCE: codes are read by one tile of rows alone, and so past the caches.
template <int HS, bool ONCE>
struct Walk {
  static constexpr int KI = HS / 32, ET = HS / 16, KV16 = HS / 64;     // KV16: 16-byte reads of a K row's quarter
  // A partial result in LDS: m and l of each row, then O, rows 16 bytes further apart than in memory (banks).
  static constexpr int kLdsRow = HS + 4, kLdsSlot = kTile * (kLdsRow + 2);
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
  __device__ static u32x4 read(const u32x4* p) { return ONCE ? __builtin_nontemporal_load(p) : *p; }
  __device__ void load_k(int step, int head) {
    const int inside = ((step * 4 + (c >> 2)) * 16) & ((1 << p.a.page_shift) - 1);
    const int64_t place = (int64_t)(number_k < 0 ? 0 : number_k) * p.a.hk + head;
    const uint8_t* const at = p.a.k_codes + ((place << p.a.page_shift) + inside + (c & 3)) * HS + g * (HS / 4);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < KV16; ++i) k[t][i] = read((const u32x4*)(at + t * 4 * HS + i * 16));
    ks = p.a.k_scale[place];
  }
  __device__ void load_v(int step, int head) {
    const int inside = ((step * 4 + g) * 16) & ((1 << p.a.page_shift) - 1);
    const int64_t place = (int64_t)(number_v < 0 ? 0 : number_v) * p.a.hk + head;
    const uint8_t* const at = p.a.v_codes + ((place << p.a.page_shift) + inside) * HS + c * 16;
#pragma unroll
    for (int e = 0; e < ET; ++e) v[e] = read((const u32x4*)(at + e * 256));
    vs = p.a.v_scale[place];
  }

  // the unit that is walked, or was last
  bf16x8 q[KI];
  f32x4 o[ET];
  float m, l;                  // l: the lane's part of the row's sum
  int rows, token, hq;         // rows of the tile; the lane's row: its token (of all) and query head

  // Steps [s0, s1) of a unit.
  template <typename Units>
  __device__ __forceinline__ void unit(const Units& u, int seq, int head, int tile, int s0, int s1) {
    const CacheAttnArgs& a = p.a;
    const int32_t* const row = a.block_table + (int64_t)seq * a.max_pages;
    rows = u.rows(a, tile, kTile);
    // keys that the tile's first and last rows see
    const uint32_t row_first = (uint32_t)tile * kTile, group = (uint32_t)a.group;
    const int vis = u.seen_by((row_first + rows - 1) / group), vis_first = u.seen_by(row_first / group);
    const int in = (int)((row_first + c) / group), limit = c < rows ? u.seen_by(in) : vis;
    token = u.cu + in;
    hq = head * a.group + (int)(row_first + c - (uint32_t)in * group);
    m = -INFINITY;
    l = 0.0f;
    const __bf16* const from = (const __bf16*)a.q + (int64_t)token * a.q_stride + hq * HS + g * (HS / 4);
#pragma unroll
    for (int i = 0; i < KI; ++i) q[i] = c < rows ? *(const bf16x8*)(from + i * 8) : bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < ET; ++e) o[e] = f32x4{0, 0, 0, 0};
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
      f32x4 x[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        x[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < KI; ++i)
          x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(k[t][i / 2][i % 2 * 2], k[t][i / 2][i % 2 * 2 + 1], scale_k), q[i], x[t], 0, 0, 0);
      }
      if (more) load_k(s + 1, head);
      const int key0 = s * kStep + g * 16;            // the lane's first key
      const bool missing = __ballot(!valid) != 0, cut = (s + 1) * kStep > vis_first;
      if (cut || missing) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!valid || key0 + 4 * t + e >= limit) x[t][e] = -INFINITY;
      }
      float top = x[0][0];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, x[t][e]);
      top = group_max(top) * a.scale_log2e;
      const float now = fmaxf(m, top), use = now == -INFINITY ? 0.0f : now, alpha = exp2f(m - use);
      m = now;
      float sum = 0.0f;
      bf16x8 pr[2];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = __builtin_amdgcn_exp2f(x[t][e] * a.scale_log2e - use);
          sum += w;
          pr[t / 2][t % 2 * 4 + e] = (__bf16)w;       // (bf16 is what the matrix cores take: half a step is 2^-8 of a weight)
        }
      l = l * alpha + sum;
      if (__ballot(alpha != 1.0f)) {
#pragma unroll
        for (int e = 0; e < ET; ++e) o[e] *= alpha;
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
      if (cut && vis_first < vis) {
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < ET; ++e)
#pragma unroll
          for (int w = 0; w < 4; ++w) any |= nan_codes(v[e][w]);
        if (__builtin_expect(__ballot(any != 0) != 0, 0)) {
          bf16x8 sees[2];
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int b = 0; b < 8; ++b) sees[j][b] = (__bf16)(valid && key0 + 8 * j + b < limit ? 1.0f : 0.0f);
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
            f32x4 count = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 2; ++j) count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is[j], sees[j], count, 0, 0, 0);
#pragma unroll
            for (int b = 0; b < 4; ++b)
              if (count[b] > 0.0f) o[e][b] = NAN;
          }
        }
      }
      // O^T += V^T P^T
      const float scale_v = valid ? scale_of(vs) : 1.0f;      // (0 times the NaN of a page in no use would be NaN)
#pragma unroll
      for (int e = 0; e < ET; ++e)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(v[e][2 * j], v[e][2 * j + 1], scale_v), pr[j], o[e], 0, 0, 0);
      if (more) load_v(s + 1, head);
    }
    l = group_sum(l);
  }

  __device__ void write() const {
    if (c >= rows) return;
    const CacheAttnArgs& a = p.a;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t to = ((int64_t)token * (a.hk * a.group) + hq) * HS + g * 4;
#pragma unroll
    for (int e = 0; e < ET; ++e) {
      const f32x4 y = o[e] * inv;
      if (a.o_dtype == USP_BF16) *(bf16x4*)((__bf16*)a.o + to + e * 16) = __builtin_convertvector(y, bf16x4);
      else *(f32x4*)((float*)a.o + to + e * 16) = y;
    }
    if (g == 0) a.lse[(int64_t)hq * a.total_q + token] = natural_lse(m, l);
  }
  __device__ void put(float* slot) const {
    if (c >= rows) return;
    if (g == 0) ((f32x2*)slot)[c] = f32x2{m, l};
#pragma unroll
    for (int e = 0; e < ET; ++e) *(f32x4*)(slot + 2 * kTile + c * kLdsRow + e * 16 + g * 4) = o[e];
  }
};

// Two partial results of a row as one.
struct Sum {
  float m, l;
  f32x4 o;
  __device__ void add(float m2, float l2, f32x4 o2) {
    const float top = fmaxf(m, m2), use = top == -INFINITY ? 0.0f : top, keep = exp2f(m - use), take = exp2f(m2 - use);
    m = top;
    l = l * keep + l2 * take;
    o = o * keep + o2 * take;
  }
  // row `row` of a unit's request and KV head, columns e .. e + 3
  template <int HS>
  __device__ void write(const CacheAttnArgs& a, const CacheLeft& unit, uint32_t row, int e) const {
    const int in = (int)(row / (uint32_t)a.group), hq = unit.head * a.group + (int)(row - (uint32_t)in * a.group), token = unit.cu + in;
    const f32x4 y = o * (l == 0.0f ? 0.0f : 1.0f / l);
    const int64_t to = ((int64_t)token * (a.hk * a.group) + hq) * HS + e;
    if (a.o_dtype == USP_BF16) *(bf16x4*)((__bf16*)a.o + to) = __builtin_convertvector(y, bf16x4);
    else *(f32x4*)((float*)a.o + to) = y;
    if (e == 0) a.lse[(int64_t)hq * a.total_q + token] = natural_lse(m, l);
  }
};

template <int HS, typename I> struct Lds {
  alignas(16) float slot[2 * kWaves][Walk<HS, true>::kLdsSlot];     // of each wave: the end of a unit, the beginning of one
  int first[kWaves];                                          // as in CacheLeft, of a wave's share
  CacheLeft end[kWaves];
  Shares<kThreads, I> shares;
};

template <int HS, bool ONCE, typename I>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_kernel(CachePlan p) {
  extern __shared__ __attribute__((aligned(16))) char dynamic[];
  Lds<HS, I>& lds = *(Lds<HS, I>*)dynamic;
  const Shares<kThreads, I>& shares = lds.shares;
  const I all = lds.shares.count(p.a, kTile);
  const int share = (int)blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int workers = all < p.workers ? (int)all : p.workers;
  I pos = share < workers ? shares.cut(all, share, workers) : all, stop = share < workers ? shares.cut(all, share + 1, workers) : all;
  if (p.whole) {
    pos = shares.unit_start(p.a, kTile, pos, all);
    stop = shares.unit_start(p.a, kTile, stop, all);
  }
  // (rounded up: the first wave has a step wherever the workgroup has one)
  const I n = stop - pos, mine = pos + n / kWaves * wave + (n % kWaves * wave + kWaves - 1) / kWaves,
          next = pos + n / kWaves * (wave + 1) + (n % kWaves * (wave + 1) + kWaves - 1) / kWaves;
  Walk<HS, ONCE> walk(p, threadIdx.x & 63);
  int first = 0, end_rows = 0, end_head = 0, end_tile = 0, end_cu = 0;
  shares.walk(p.a, kTile, mine, next, [&](const CacheUnits<I>& u, int seq, int head, int tile, int s0, int s1, int of) __attribute__((always_inline)) {
    const bool begins = s0 == 0, ends = s1 == of;
    walk.unit(u, seq, head, tile, s0, s1);
    if (begins && ends) {
      walk.write();
    } else {
      walk.put(lds.slot[2 * wave + begins]);
      if (begins) end_rows = walk.rows, end_head = head, end_tile = tile, end_cu = u.cu;
      else first = ends ? 2 : 1;
    }
  });
  // A wave without steps lets the unit that goes on around it pass (it has no partial result: 3).
  if ((threadIdx.x & 63) == 0) {
    lds.first[wave] = mine < next ? first : 3;
    lds.end[wave] = CacheLeft{0, end_rows, end_head, end_tile, end_cu};
  }
  __syncthreads();
  // Units that waves share, each from the wave that has its beginning, or from the first wave, where the unit began in a workgroup
  // before.
  constexpr int kTeam = HS / 4;
  const int row = threadIdx.x / kTeam, e = threadIdx.x % kTeam * 4;
  int left_first = 0, left_end = -1;      // what the workgroup leaves: the second as the wave that has it
  float* const slots = p.partial + share * 2 * CachePlan::slot(kTile, HS);
  for (int w = 0; w < kWaves; ++w) {
    const int f = lds.first[w];
    for (int begins = w ? 1 : 0; begins < 2; ++begins) {
      if (begins ? lds.end[w].rows == 0 : f != 1 && f != 2) continue;
      bool ended = !begins && f == 2;
      Sum sum = {-INFINITY, 0.0f, {0, 0, 0, 0}};
      for (int x = w; ; ++x) {
        if (x > w) {
          if (ended || x == kWaves) break;
          if (lds.first[x] == 3) continue;
          ended = lds.first[x] == 2;
        }
        const float* const slot = lds.slot[2 * x + (x == w ? begins : 0)];
        const f32x2 ml = ((const f32x2*)slot)[row & (kTile - 1)];
        const f32x4 o = *(const f32x4*)(slot + 2 * kTile + (row & (kTile - 1)) * Walk<HS, ONCE>::kLdsRow + e);
        if (x == w) sum = Sum{ml[0], ml[1], o};
        else sum.add(ml[0], ml[1], o);
      }
      if (begins && ended) {
        const CacheLeft& unit = lds.end[w];
        if (row < unit.rows) sum.template write<HS>(p.a, unit, (uint32_t)unit.tile * kTile + row, e);
      } else {
        float* const to = slots + (begins ? CachePlan::slot(kTile, HS) : 0);
        if (row < kTile) {
          if (e == 0) ((f32x2*)to)[row] = f32x2{sum.m, sum.l};
          *(f32x4*)(to + 2 * kTile + row * HS + e) = sum.o;
        }
        if (begins) left_end = w;
        else left_first = ended ? 2 : 1;
      }
    }
  }
  if (!p.whole && threadIdx.x == 0) {
    const CacheLeft& end = lds.end[left_end < 0 ? 0 : left_end];
    p.left[share] = CacheLeft{left_first, left_end < 0 ? 0 : end.rows, end.head, end.tile, end.cu};
  }
}

// Joins the partial results of units that workgroups share: of each the beginning that worker w left, then what the workers behind
// it left up to the unit's end.  A team of HS / 4 threads adds up parts of a row, four columns to a thread, in the order of the
// keys; several teams have a row between them, the more the fewer rows there are, so that a few long units are joined by the
// whole chip too.
template <int HS>
__global__ __launch_bounds__(kJoinThreads) void cache_attn_join_kernel(CachePlan p, int rows_per_tile) {
  constexpr int kTeam = HS / 4, kTeams = kJoinThreads / kTeam, kWorkers = kPlanCUs;
  static_assert(kWorkers == kJoinThreads, "a thread to each worker");
  __shared__ f32x4 sums[kTeams][kTeam];
  __shared__ f32x2 mls[kTeams];
  __shared__ CacheLeft left[kWorkers];
  __shared__ int leaders[kWorkers], counts[kJoinThreads / 64];
  const CacheAttnArgs& a = p.a;
  const int64_t slot = CachePlan::slot(rows_per_tile, HS);
  const int tid = threadIdx.x, lane = tid & 63, team = tid / kTeam, e = tid % kTeam * 4;
  left[tid] = p.left[tid];
  const uint64_t mine = __ballot(left[tid].rows > 0);
  if (lane == 0) counts[tid >> 6] = __builtin_popcountll(mine);
  __syncthreads();
  int units = 0, at = __builtin_popcountll(mine & ((1ull << lane) - 1));
  for (int w = 0; w < kJoinThreads / 64; ++w) {
    if (w < tid >> 6) at += counts[w];
    units += counts[w];
  }
  if (left[tid].rows > 0) leaders[at] = tid;
  __syncthreads();
  int together = 1;                                  // rows that a workgroup has at a time
  while (together < kTeams && units * rows_per_tile > together * (int)gridDim.x) together *= 2;
  const int share = kTeams / together, items = rows_per_tile / together;
  for (int item = blockIdx.x; item < units * items; item += gridDim.x) {
    const int w = leaders[item / items], first_row = item % items * together;
    const CacheLeft unit = left[w];
    if (first_row >= unit.rows) continue;
    int parts = 1;                                   // parts 1 .. parts - 1 are those of workers w + 1 ...
    for (;;) {
      const int x = w + parts + lane;
      const uint64_t on = __ballot(x < kWorkers && left[x & (kWorkers - 1)].first == 1);
      if (on != ~0ull) {
        parts += __builtin_ctzll(~on);
        break;
      }
      parts += 64;
    }
    parts += w + parts < kWorkers;                   // the one in which it ends
    const int row = first_row + team / share, from = team % share;
    const bool real = row < unit.rows;
    // (teams behind one another have parts behind one another)
    const int begin = parts * from / share, stop = real ? parts * (from + 1) / share : begin;
    Sum sum = {-INFINITY, 0.0f, {0, 0, 0, 0}};
#pragma unroll 4
    for (int x = begin; x < stop; ++x) {
      const float* const part = p.partial + (x ? 2 * (int64_t)(w + x) : 2 * (int64_t)w + 1) * slot;
      const f32x2 ml = ((const f32x2*)part)[row];
      sum.add(ml[0], ml[1], *(const f32x4*)(part + 2 * rows_per_tile + row * HS + e));
    }
    if (share > 1) {
      __syncthreads();                               // (the item before has been read)
      sums[team][tid % kTeam] = sum.o;
      if (e == 0) mls[team] = f32x2{sum.m, sum.l};
      __syncthreads();
      if (from == 0)
        for (int t = team + 1; t < team + share; ++t) sum.add(mls[t][0], mls[t][1], sums[t][tid % kTeam]);
    }
    if (real && from == 0) sum.template write<HS>(a, unit, (uint32_t)unit.tile * rows_per_tile + row, e);
  }
}

// Requests of few rows go to the kernel that gives each wave units of its own, which reads the cache again for every 16 rows; the
// one for many rows has a request's rows up to 256 at once, but a step of it takes as long for one as for all.  Measured with 8
// KV heads of 128, here / there: 64 requests of 256 to 32768 tokens, 16 rows 156 us, 32 rows 295 / 393, 64 rows 547 / 404; 64
// of 100 to 4000 tokens, 32 rows 63 / 134, 64 rows 94 / 141; one of 32768 tokens, 32 rows 28 / 38, 64 rows 38 / 40.  So 32 rows, and
// 64 where the table has room for 8192 tokens at most.
bool few_rows(int group, int max_q, int64_t most_tokens) {
  return (int64_t)group * (max_q < 1 ? 1 : max_q) <= (most_tokens <= 8192 ? 64 : 32);
}
int rows_of(bool few) { return few ? kTile : kCacheRowsTile; }

template <int HS, bool ONCE, typename I>
int launch_few(const CachePlan& p, hipStream_t stream) {
  static LdsLimitRaised raised;
  if (!raise_dynamic_lds_limit((const void*)cache_attn_kernel<HS, ONCE, I>, sizeof(Lds<HS, I>), raised)) return USP_ERR_LAUNCH;
  cache_attn_kernel<HS, ONCE, I><<<dim3(p.workers), kThreads, sizeof(Lds<HS, I>), stream>>>(p);
  return USP_OK;
}
template <int HS, bool ONCE>
int launch_few(const CachePlan& p, hipStream_t stream) {
  const CacheAttnArgs& a = p.a;
  // steps that there can be: tiles, each of the steps of a full table and of one more for each tile before it
  const double tiles = (double)a.total_q * a.group / kTile + a.n_seqs, steps = (double)((int64_t)a.max_pages << a.page_shift) / kStep + 2 + tiles;
  return tiles * steps * a.hk < 2e9 ? launch_few<HS, ONCE, int32_t>(p, stream) : launch_few<HS, ONCE, int64_t>(p, stream);
}

}  // namespace

size_t cache_attn_workspace(int group, int hs, int max_q) {
  const bool few = few_rows(group, max_q, INT64_MAX);
  return kPlanCUs * (sizeof(CacheLeft) + 2 * CachePlan::slot(rows_of(few), hs) * sizeof(float));
}

int launch_cache_attn(const CacheAttnArgs& a, int max_q, hipStream_t stream) {
  const int64_t most_tokens = (int64_t)a.max_pages << a.page_shift;
  const bool few = few_rows(a.group, max_q, most_tokens);
  CachePlan p = {a, kPlanCUs, (CacheLeft*)a.workspace, nullptr, 0};
  p.partial = (float*)(p.left + p.workers);
  // Rows of the table that hold 4096 tokens at most, and a unit and more for every CU: a wave has eight steps of a unit at most, and
  // the joining launch would cost more than cutting units between workgroups gains.
  p.whole = few && most_tokens <= 4096 && (int64_t)a.n_seqs * a.hk >= kPlanCUs;
  // Tiles of one request walk the same codes: where there are several, the caches are to keep them (64 requests of 100 to 4000
  // tokens, 32 rows: 63 us, past the caches 78); one tile reads them once (64 requests of up to 32768, 16 rows: 170, so 156).
  const bool once = (int64_t)a.group * max_q <= kTile;
  const int st = !few ? launch_cache_attn_rows(p, stream)
                 : a.hs == 128 ? (once ? launch_few<128, true>(p, stream) : launch_few<128, false>(p, stream))
                               : (once ? launch_few<64, true>(p, stream) : launch_few<64, false>(p, stream));
  if (st != USP_OK) return st;
  if (!p.whole) {
    const dim3 grid(kPlanCUs * 4);
    if (a.hs == 128) cache_attn_join_kernel<128><<<grid, kJoinThreads, 0, stream>>>(p, rows_of(few));
    else cache_attn_join_kernel<64><<<grid, kJoinThreads, 0, stream>>>(p, rows_of(few));
  }
  return launch_status();
}

}  // namespace usp
