// Attention over the 8-bit cache for many rows of a request (pieces of prompts): bound by the matrix cores.
//
// A unit is one request, KV head and tile of 256 rows (tokens x query heads of the KV head); the steps of all units, laid one
// behind the other, are cut evenly among one workgroup per CU, and units that are cut leave partial results for the joining
// launch (see cache_attn.hip).  A workgroup is 8 waves of 32 rows, two to a SIMD.  Codes are widened to bf16 once per
// workgroup, on their way into LDS, not once per wave: K as rows, V as the tiles lie, transposed, both with strides that keep
// 16-byte reads free of bank conflicts (HS * 2 + 16 and 144 bytes: an odd number of 16-byte pieces).
//
// S^T = K Q^T and O^T = V^T P^T, so that a lane holds one row (lane % 32) and every product's operand is what the one before
// leaves: of 16 tokens of V the lanes below 32 need 0-3 and 8-11, the others 4-7 and 12-15, which is the order in which they
// are written to LDS.
//
// Step s puts the codes of K three steps ahead and of V two steps ahead, which came during the step before, into LDS and asks for
// those behind them; then, side by side, the scores of step s + 1 and the products with V of step s (matrix cores), the
// exponentials of step s and the maxima of step s + 1 (vector ALU).  K and V have four buffers each, so that only every
// second step ends with a barrier (two buffers and a barrier at every step: 1 % slower with full tiles, 3 to 5 % with a few rows).
//
// Measured: 4096 rows of 32 heads over 49152 tokens (3.16 TFLOP) 2.8 ms, 1.11 to 1.15 PFLOP/s, matrix cores busy 55 % of the
// cycles; a library product of 8192 x 8192 matrices reaches 1.11, of 16384 1.37.  Without the exponentials, or without bringing
// codes to LDS, a step takes 8 to 9 % less: what is left is the two waves of a SIMD waiting for LDS operands and for each other.
#include "cache_attn_device.h"

namespace usp {
namespace {

constexpr int kThreads = 512, kStep = kCacheStep, kRows = 32, kLeastSteps = 4, kBuffers = 4;

template <int HS> constexpr int k_stride() { return HS * 2 + 16; }
constexpr int kVStride = kStep * 2 + 16;
template <int HS> constexpr int k_bytes() { return kStep * k_stride<HS>(); }
template <int HS> constexpr int v_bytes() { return HS * kVStride; }
// Beside K and V, for each buffer: which of a step's 16-token blocks have no page (a byte each), whether a wave brought
// NaN values (a byte each), and where they are (16 bits for each column and block).
struct Marks { uint8_t missing[4], unused[4], nan[kThreads / 64]; };
template <int HS> struct Lds {
  alignas(16) char k[kBuffers][k_bytes<HS>()];
  alignas(16) char v[kBuffers][v_bytes<HS>()];
  alignas(16) Marks marks[kBuffers];
  alignas(8) uint16_t nan[kBuffers][HS][4];
  Shares<kThreads, int64_t> shares;
};

template <int HS>
struct RowsWalk {
  static constexpr int KS = HS / 16, EB = HS / 32;
  // A wave brings 16-byte pieces of one 16-token block of a step, which lies in one piece of memory: hs 128 of K and V, hs 64 of
  // one of the two.
  static constexpr bool kBoth = HS == 128;
  static constexpr int kPieces = HS;          // of a block
  const CacheAttnArgs& a;
  Lds<HS>& lds;
  const int tid, wave, c, h;                  // c: the lane's row of the wave's 32, h: which half of the wave
  const int block, piece;

  __device__ RowsWalk(const CacheAttnArgs& args, Lds<HS>& shared)
      : a(args), lds(shared), tid(threadIdx.x), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), c(threadIdx.x & 31), h((threadIdx.x >> 5) & 1),
        block(kBoth ? wave >> 1 : wave & 3), piece(threadIdx.x % kPieces) {}

  __device__ bool brings_k() const { return kBoth || wave < 4; }
  __device__ bool brings_v() const { return kBoth || wave >= 4; }

  // The wave's block of a step: where its page's scales and its own codes are, of K as of V, and how many of its tokens count.
  // (A page that is not there reads page 0, unconditionally: a load under a condition would be waited for where it stands.)
  struct Block { int64_t place, codes; int left; };
  // (The number stays in a vector register until it is looked at, a step later: what is asked for before it would have to arrive
  // first.)
  __device__ int number(const int32_t* row, int step, int vis) const { return row[cache_entry(step * 4 + block, vis, a.page_shift)]; }
  __device__ Block found(int looked_up, int step, int vis, int head) const {
    const int number = __builtin_amdgcn_readfirstlane(looked_up);
    const bool counts = cache_counts(step * 4 + block, vis, number, a.pages);
    const int inside = (step * kStep + block * 16) & ((1 << a.page_shift) - 1);
    const int64_t place = (int64_t)(counts ? number : 0) * a.hk + head;
    return Block{place, ((place << a.page_shift) + inside) * HS, counts ? vis - step * kStep - block * 16 : 0};
  }
  struct Piece { u32x4 codes; uint32_t scale; };
  __device__ Piece load(const uint8_t* codes, const uint8_t* scales, const Block& b) const {
    return Piece{*(const u32x4*)(codes + b.codes + piece * 16), scales[b.place]};
  }

  __device__ void put_k(const Piece& x, int buffer) const {
    const float scale = scale_of(x.scale);
    const int key = block * 16 + piece / (HS / 16), at = piece % (HS / 16) * 32;
    bf16x8* const to = (bf16x8*)(lds.k[buffer] + key * k_stride<HS>() + at);
    to[0] = widened(x.codes[0], x.codes[1], scale);
    to[1] = widened(x.codes[2], x.codes[3], scale);
  }
  // `left`: how many of the block's tokens count.  What stands behind them counts as zero, whatever it is; NaN, too, which is
  // kept apart: 0 times it would be NaN for rows that do not see it.  `marked`: the wave's marks in a buffer are not those of
  // 16 tokens without NaN, which the kernel begins with.
  __device__ void put_v(const Piece& x, int buffer, int left, int& marked) const {
    const float scale = left > 0 ? scale_of(x.scale) : 1.0f;      // (0 times the NaN of a page in no use would be NaN)
    u32x4 y = x.codes;
    if (left < 16) {
#pragma unroll
      for (int w = 0; w < 4; ++w) y[w] &= first_bytes(left - 4 * w);
    }
    const uint32_t any = nan_codes(y[0]) | nan_codes(y[1]) | nan_codes(y[2]) | nan_codes(y[3]);
    const bool some = __ballot(any != 0) != 0, mark = some || left <= 0;
    if (__builtin_expect(mark || (marked >> buffer & 1), 0)) {
      uint32_t where = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t n = nan_codes(y[w]) >> 7;
        where |= ((n | n >> 7 | n >> 14 | n >> 21) & 15) << (4 * w);
        y[w] &= ~(n * 0xff);
      }
      lds.nan[buffer][piece][block] = (uint16_t)where;
      if ((tid & 63) == 0) {
        lds.marks[buffer].nan[wave] = some;
        lds.marks[buffer].missing[block] = left <= 0;
      }
      marked = (marked & ~(1 << buffer)) | mark << buffer;
    }
    bf16x8* const to = (bf16x8*)(lds.v[buffer] + piece * kVStride + block * 32);
    to[0] = widened(y[0], y[2], scale);
    to[1] = widened(y[1], y[3], scale);
  }
  // Marks of all buffers as put_v expects to find them.
  __device__ void clear_marks() const {
    if (tid < (int)(sizeof(lds.marks) / 4)) ((uint32_t*)lds.marks)[tid] = 0;
    for (int i = tid; i < (int)(sizeof(lds.nan) / 4); i += kThreads) ((uint32_t*)lds.nan)[i] = 0;
  }

  __device__ bf16x8 k_operand(int buffer, int kb, int ks) const {
    return *(const bf16x8*)(lds.k[buffer] + (kb * 32 + c) * k_stride<HS>() + ks * 32 + h * 16);
  }
  __device__ bf16x8 v_operand(int buffer, int eb, int j) const {
    return *(const bf16x8*)(lds.v[buffer] + (eb * 32 + c) * kVStride + j * 32 + h * 16);
  }

  // state of a unit's walk
  bf16x8 q[KS];
  f32x16 o[EB];
  float m, l;
  int marked = 0;
  int limit, vis_wave, vis_first;      // keys that the lane's row sees; that the wave's last and first rows see

  __device__ __forceinline__ void scores(int buffer, f32x16 (&x)[2]) const {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 y = {};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(buffer, kb, ks), q[ks], y, 0, 0, 0);
      x[kb] = y;
    }
  }

  // Operands of group n of a step's products: the scores of step s + 1, then the products with V of step s.
  static constexpr int kGroups = KS + 2 * EB;
  __device__ __forceinline__ void operands(int s, int n, bf16x8 (&f)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      f[i] = n < KS ? k_operand((s + 1) % kBuffers, i, n) : v_operand(s % kBuffers, (n - KS) % (EB / 2) * 2 + i, (n - KS) / (EB / 2));
  }
  // How many of a step's 32 weights are formed before group n.
  static constexpr int weights_before(int n) { return n <= KS ? 24 * n / KS : n - KS >= EB ? 32 : 24 + 8 * (n - KS) / EB; }

  // The vector work and products of step s, whose scores are x, and the scores of step s + 1 into y (behind the last step: of
  // what the buffer holds, for nobody).  top: the largest of the lane's scores, then of the next step's, none of them masked.
  __device__ __forceinline__ void compute(int s, u32x4 marks, f32x16 (&x)[2], f32x16 (&y)[2], float& top) {
    const uint32_t missing = __builtin_amdgcn_readfirstlane(marks[0]), nan = __builtin_amdgcn_readfirstlane(marks[2] | marks[3]);
    const bool cut = (s + 1) * kStep > vis_first;
    if (cut || missing) {
      top = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int in = kb * 32 + 8 * (i / 4) + 4 * h + i % 4;
          if (s * kStep + in >= limit || (missing >> (in / 16 * 8) & 1)) x[kb][i] = -INFINITY;
          top = fmaxf(top, x[kb][i]);
        }
    }
    bf16x8 f[3][2];
    operands(s, 0, f[0]);
    operands(s, 1, f[1]);
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_int(top), __float_as_int(top), false, false);
    top = fmaxf(__int_as_float(both[0]), __int_as_float(both[1])) * a.scale_log2e;
    // The value that is subtracted need not be the maximum: it moves where a row's grows by more than 2^8.
    if (__ballot(top > m + 8.0f)) {
      const float now = fmaxf(m, top), use = now == -INFINITY ? 0.0f : now, alpha = exp2f(m - use);
      m = now;
      l *= alpha;
#pragma unroll
      for (int eb = 0; eb < EB; ++eb) o[eb] *= alpha;
    }
    const float use = m == -INFINITY ? 0.0f : m;
    bf16x8 p[4];
    float sum = 0.0f;
    // Two products to a group, whose operands are on their way from LDS since two groups before; the groups are kept apart, or
    // the compiler would read every operand just ahead of its product.  24 of the exponentials stand beside the scores, the last
    // 8 and the next step's maxima beside the products with V.
#pragma unroll
    for (int n = 0; n < kGroups; ++n) {
      if (n + 2 < kGroups) operands(s, n + 2, f[(n + 2) % 3]);
      if (n < KS) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
          y[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % 3][kb], q[n], n ? y[kb] : f32x16{}, 0, 0, 0);
      } else {
        const int j = (n - KS) / (EB / 2), eb = (n - KS) % (EB / 2) * 2;
#pragma unroll
        for (int i = 0; i < 2; ++i) o[eb + i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % 3][i], p[j], o[eb + i], 0, 0, 0);
      }
#pragma unroll
      for (int i = weights_before(n); i < weights_before(n + 1); ++i) {
        const float w = __builtin_amdgcn_exp2f(x[i / 16][i % 16] * a.scale_log2e - use);
        sum += w;
        p[i / 8][i % 8] = (__bf16)w;
      }
      asm volatile("" : "+v"(sum));      // (or the additions would sink to the end, all weights waiting for them in registers)
      if (n == KS + EB) top = y[0][0];
      if (n >= KS + EB) {
        constexpr int kEach = 32 / EB;
#pragma unroll
        for (int i = (n - KS - EB) * kEach; i < (n - KS - EB + 1) * kEach; ++i) top = fmaxf(top, y[i / 16][i % 16]);
        asm volatile("" : "+v"(top));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    l += sum;
    if (__builtin_expect(nan != 0, 0)) {      // rows that see a NaN value are NaN in its column
      uint64_t seen = 0;
      for (int b = 0; b < 4; ++b) {
        const int n = limit - s * kStep - 16 * b;
        if (!(missing >> (8 * b) & 1)) seen |= (uint64_t)(n >= 16 ? 0xffff : n <= 0 ? 0 : (1 << n) - 1) << (16 * b);
      }
#pragma unroll
      for (int eb = 0; eb < EB; ++eb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (*(const uint64_t*)lds.nan[s % kBuffers][eb * 32 + 8 * (i / 4) + 4 * h + i % 4] & seen) o[eb][i] = NAN;
    }
  }

  // Steps [s0, s1) of a unit: results to o and lse if these are all, else to the partial result `slot`.
  __device__ __forceinline__ void unit(const CacheUnits<>& u, int seq, int head, int tile, int s0, int s1, bool whole, float* slot) {
    const int32_t* const row = a.block_table + (int64_t)seq * a.max_pages;
    const int rows = u.rows(a, tile, kCacheRowsTile);
    const uint32_t row_first = (uint32_t)tile * kCacheRowsTile, group = (uint32_t)a.group;
    const int vis = u.seen_by((row_first + rows - 1) / group);
    const int end = (vis + kStep - 1) / kStep < s1 ? (vis + kStep - 1) / kStep : s1;
    const int mine = wave * kRows + c, wave_rows = rows - wave * kRows < kRows ? rows - wave * kRows : kRows;
    const uint32_t row_wave = row_first + wave * kRows;
    const int token = (int)((row_first + mine) / group), hq = head * a.group + (int)(row_first + mine - (uint32_t)token * group);
    vis_wave = wave_rows > 0 ? __builtin_amdgcn_readfirstlane(u.seen_by((row_wave + wave_rows - 1) / group)) : 0;
    vis_first = wave_rows > 0 ? __builtin_amdgcn_readfirstlane(u.seen_by(row_wave / group)) : 0;
    limit = mine < rows ? u.seen_by(token) : vis_wave;
    m = -INFINITY;
    l = 0.0f;
    const __bf16* const from = (const __bf16*)a.q + (int64_t)(u.cu + token) * a.q_stride + hq * HS + h * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = mine < rows ? *(const bf16x8*)(from + ks * 16) : bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int eb = 0; eb < EB; ++eb) o[eb] = f32x16{};
    if (s0 < end) {
      const auto at_most = [&](int s) { return s < end ? s : end - 1; };
      const auto block_of = [&](int s) { return found(number(row, at_most(s), vis), at_most(s), vis, head); };
      const Block b0 = block_of(s0), b1 = block_of(s0 + 1), b2 = block_of(s0 + 2);
      Block bk = block_of(s0 + 4), bv = block_of(s0 + 3);      // of the codes that are asked for next
      int ahead = number(row, at_most(s0 + 5), vis), left;     // left: tokens of the V block that is on its way
      Piece kk = {}, vv = {};
      {
        Piece k0 = {}, k1 = {}, k2 = {}, v0 = {}, v1 = {};
        if (brings_k()) {
          k0 = load(a.k_codes, a.k_scale, b0);
          k1 = load(a.k_codes, a.k_scale, b1);
          k2 = load(a.k_codes, a.k_scale, b2);
          kk = load(a.k_codes, a.k_scale, bv);
        }
        if (brings_v()) {
          v0 = load(a.v_codes, a.v_scale, b0);
          v1 = load(a.v_codes, a.v_scale, b1);
          vv = load(a.v_codes, a.v_scale, b2);
        }
        left = b2.left;
        __syncthreads();                            // the unit before has been read
        if (brings_k()) {
          put_k(k0, s0 % kBuffers);
          put_k(k1, (s0 + 1) % kBuffers);
          put_k(k2, (s0 + 2) % kBuffers);
        }
        if (brings_v()) {
          put_v(v0, s0 % kBuffers, b0.left, marked);
          put_v(v1, (s0 + 1) % kBuffers, b1.left, marked);
        }
      }
      __syncthreads();
      f32x16 x[2], y[2];
      scores(s0 % kBuffers, x);
      __syncthreads();                              // (the first step's scores have been formed: its K makes room in the second step)
      float top = x[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[kb][i]);
      int s = s0;
      const auto step = [&](f32x16 (&now)[2], f32x16 (&next)[2]) __attribute__((always_inline)) {
        const u32x4 marks = *(const u32x4*)&lds.marks[s % kBuffers];
        if (brings_k()) put_k(kk, (s + 3) % kBuffers);
        if (brings_v()) put_v(vv, (s + 2) % kBuffers, left, marked);
        if (brings_k()) kk = load(a.k_codes, a.k_scale, bk);
        if (brings_v()) vv = load(a.v_codes, a.v_scale, bv);
        left = bv.left;
        bv = bk;
        bk = found(ahead, at_most(s + 5), vis, head);
        ahead = number(row, at_most(s + 6), vis);
        if (s * kStep < vis_wave) compute(s, marks, now, next, top);
        return ++s < end;
      };
      // Two steps from s on read K of s + 1 and s + 2 and V of s and s + 1, and write K of s + 3 and s + 4 and V of s + 2 and s + 3: other
      // buffers, of four each.
      while (step(x, y) && step(y, x)) __syncthreads();
    }
    l += __shfl_xor(l, 32);
    if (mine >= rows) return;
    if (whole) {
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const int64_t to = ((int64_t)(u.cu + token) * (a.hk * a.group) + hq) * HS + h * 4;
#pragma unroll
      for (int eb = 0; eb < EB; ++eb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 w = f32x4{o[eb][4 * i], o[eb][4 * i + 1], o[eb][4 * i + 2], o[eb][4 * i + 3]} * inv;
          if (a.o_dtype == USP_BF16) *(bf16x4*)((__bf16*)a.o + to + eb * 32 + i * 8) = __builtin_convertvector(w, bf16x4);
          else *(f32x4*)((float*)a.o + to + eb * 32 + i * 8) = w;
        }
      if (h == 0) a.lse[(int64_t)hq * a.total_q + u.cu + token] = natural_lse(m, l);
    } else {
      if (h == 0) ((f32x2*)slot)[mine] = f32x2{m, l};
      float* const to = slot + 2 * kCacheRowsTile + mine * HS + h * 4;
#pragma unroll
      for (int eb = 0; eb < EB; ++eb)
#pragma unroll
        for (int i = 0; i < 4; ++i) *(f32x4*)(to + eb * 32 + i * 8) = f32x4{o[eb][4 * i], o[eb][4 * i + 1], o[eb][4 * i + 2], o[eb][4 * i + 3]};
    }
  }
};

template <int HS>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_rows_kernel(CachePlan p) {
  extern __shared__ __attribute__((aligned(16))) char dynamic[];
  Lds<HS>& shared = *(Lds<HS>*)dynamic;
  const Shares<kThreads, int64_t>& shares = shared.shares;
  const int64_t all = shared.shares.count(p.a, kCacheRowsTile);
  // The workgroups of an XCD (blockIdx % 8) have shares that follow on one another: mostly of one KV head.
  const int n = (int)gridDim.x, share = n % 8 ? (int)blockIdx.x : (int)(blockIdx.x % 8) * (n / 8) + (int)blockIdx.x / 8;
  // (a share of fewer steps would cost less than the partial results that it leaves: 256 rows are the bytes of eight steps)
  const int64_t most = (all + kLeastSteps - 1) / kLeastSteps;
  const int workers = most < n ? (int)most : n;
  int first = 0, end_rows = 0, end_head = 0, end_tile = 0, end_cu = 0;      // as in CacheLeft
  if (share < workers) {
    RowsWalk<HS> walk(p.a, shared);
    walk.clear_marks();                             // (a barrier stands before the first use)
    float* const slots = p.partial + share * 2 * CachePlan::slot(kCacheRowsTile, HS);
    shares.walk(p.a, kCacheRowsTile, shares.cut(all, share, workers), shares.cut(all, share + 1, workers),
                [&](const CacheUnits<>& u, int seq, int head, int tile, int s0, int end, int of) __attribute__((always_inline)) {
                  const bool begins = s0 == 0, ends = end == of;
                  walk.unit(u, seq, head, tile, s0, end, begins && ends, slots + (begins ? CachePlan::slot(kCacheRowsTile, HS) : 0));
                  if (!begins) first = ends ? 2 : 1;
                  else if (!ends) end_rows = u.rows(p.a, tile, kCacheRowsTile), end_head = head, end_tile = tile, end_cu = u.cu;
                });
  }
  if (threadIdx.x == 0) p.left[share] = CacheLeft{first, end_rows, end_head, end_tile, end_cu};
}

template <int HS>
int launch(const CachePlan& p, hipStream_t stream) {
  static LdsLimitRaised raised;
  if (!raise_dynamic_lds_limit((const void*)cache_attn_rows_kernel<HS>, sizeof(Lds<HS>), raised)) return USP_ERR_LAUNCH;
  cache_attn_rows_kernel<HS><<<dim3(p.workers), kThreads, sizeof(Lds<HS>), stream>>>(p);
  return USP_OK;
}

}  // namespace

int launch_cache_attn_rows(const CachePlan& p, hipStream_t stream) { return p.a.hs == 128 ? launch<128>(p, stream) : launch<64>(p, stream); }

}  // namespace usp
