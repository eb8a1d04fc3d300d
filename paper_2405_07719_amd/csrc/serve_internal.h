// What the entry points of rotary positions and of the 8-bit cache share with their kernels (not part of the ABI).
#pragma once
#include "usp_internal.h"

namespace usp {

// A rotation as the kernel takes it: frequencies in turns (2 pi) per position.
struct RopeArgs {
  double turns[64];
  const void* x[2];            // Q and K: rows of heads[t] heads, stride[t] elements apart
  void* y[2];
  int64_t stride[2], out_stride[2];
  int heads[2];
  const int32_t* positions;    // one per row; nullptr: the rows are shards of ranks, positions by Algorithm 2
  int64_t rows;
  int hs, rotary_dim, pairs, in_place;
  float magnitude, sign;
  // shards: rows [rank][bs][per_shard], the first of rank0
  int64_t per_shard, ring_block, half_chunk;   // half_chunk: rows of a zigzag chunk; 0: contiguous blocks
  int bs, rank0, ulysses, ring;
};
int launch_rope(const RopeArgs& a, int dtype, hipStream_t stream);

struct CacheExtendArgs {
  const int32_t *cu_new, *len_before, *free_pages;
  int32_t *block_table, *len_after, *slots, *positions, *taken;
  int64_t total_new, pages, n_free;
  int n_seqs, max_pages, page_shift;
};
int launch_cache_extend(const CacheExtendArgs& a, hipStream_t stream);

// Exponents of a page's scale: with the smallest, 2^-9 (the least code) times it is still a normal bf16 and fp32 number; with
// the largest, the sum of 2^23 values of 448 times it, with weights of up to 2^8, is still finite (attention divides by the sum of its
// weights at the end).
constexpr int kCacheMinExp = -117, kCacheMaxExp = 88;

struct CacheAppendArgs {
  const void* x[2];            // K, V
  uint8_t* codes[2];
  uint8_t* scale[2];
  int64_t stride[2];
  const int32_t* slots;
  int64_t rows, slots_end;     // pages * page
  int64_t first_window, windows;   // of a launch
  int page_shift, hk, hs, window;  // window: rows in which a wave looks for pages that begin there
};
int launch_cache_append(const CacheAppendArgs& a, int dtype, hipStream_t stream);

struct CacheAttnArgs {
  const uint8_t *k_codes, *v_codes, *k_scale, *v_scale;
  const void* q;
  const int32_t *cu_q, *kv_len, *block_table;
  void* o;
  float* lse;
  void* workspace;
  int64_t pages, q_stride, total_q;
  int page_shift, hk, hs, group, max_pages, n_seqs, causal, o_dtype;
  float scale_log2e;
};

// Keys of one step of a unit's walk.
constexpr int kCacheStep = 64;

struct CacheRequest { int cu, nq, len; };      // first row, rows, keys

// One request's units (KV head, tile of rows) and how many steps each is taken to have: tiles of a causal request see more keys
// one after the other.  (Exact for a single tile, else up to a step too many; a tile that is at its end early is done early.)
// I: what holds sums of steps; 32 bits where they cannot be more (divisions of 64 bits are long).
template <typename I = int64_t>
struct CacheUnits {
  int cu, nq, len, tiles, base, each, causal;
  I per_head;   // steps of one KV head's tiles
  typedef CacheRequest Request;
  __host__ __device__ static Request read(const CacheAttnArgs& a, int i) {
    const int total = (int)a.total_q;
    int c0 = a.cu_q[i], c1 = a.cu_q[i + 1];
    c0 = c0 < 0 ? 0 : c0 > total ? total : c0;
    c1 = c1 < c0 ? c0 : c1 > total ? total : c1;
    const int64_t most = INT32_MAX & ~127, all = (int64_t)a.max_pages << a.page_shift, room = all < most ? all : most;   // (the end of the last step fits)
    const int x = a.kv_len[i];
    return Request{c0, c1 - c0, x < 0 ? 0 : x > room ? (int)room : x};
  }
  __host__ __device__ CacheUnits(const CacheAttnArgs& a, const Request& r, int rows_per_tile) : cu(r.cu), nq(r.nq), len(r.len), causal(a.causal) {
    tiles = (int)(((int64_t)nq * a.group + rows_per_tile - 1) / rows_per_tile);
    each = 0;
    base = len ? (len - 1) / kCacheStep + 1 : 1;
    if (causal && tiles > 1) {
      each = ((rows_per_tile + a.group - 1) / a.group + kCacheStep - 1) / kCacheStep;
      base = len > nq ? (len - nq - 1) / kCacheStep + 1 : 0;
    }
    per_head = upto(tiles);
  }
  __host__ __device__ CacheUnits(const CacheAttnArgs& a, int i, int rows_per_tile) : CacheUnits(a, read(a, i), rows_per_tile) {}
  // steps of tiles 0 .. j - 1, and of tile j
  __host__ __device__ I upto(int j) const { return (I)j * base + (I)each * (I)((int64_t)j * (j + 1) / 2); }
  __host__ __device__ int steps(int j) const { return base + each * (j + 1); }
  // keys that a token sees
  __host__ __device__ int seen_by(int64_t token) const {
    const int64_t x = causal ? len - (int64_t)nq + token + 1 : len;
    return x < 0 ? 0 : (int)x;
  }
  // rows of a tile
  __host__ __device__ int rows(const CacheAttnArgs& a, int tile, int rows_per_tile) const {
    const int64_t left = (int64_t)nq * a.group - (int64_t)tile * rows_per_tile;
    return left < rows_per_tile ? (int)left : rows_per_tile;
  }
  // the unit and its step at `pos` of the request's steps (head after head, tile after tile)
  struct Place { int head, tile, step; };
  __host__ __device__ Place locate(I pos) const {
    const int head = (int)(pos / per_head);
    const I in_head = pos - head * per_head;
    int tile = 0, above = tiles;
    while (above - tile > 1) {
      const int mid = (tile + above) / 2;
      if (upto(mid) <= in_head) tile = mid;
      else above = mid;
    }
    return Place{head, tile, (int)(in_head - upto(tile))};
  }
};

// Where the page number of 16-key block b stands in a request's row of the table, of which the first `vis` keys count, vis >= 1;
// blocks behind the last that counts are looked up as that one, so that the lookup needs no condition.
__host__ __device__ inline int cache_entry(int b, int vis, int page_shift) {
  const int last = (vis - 1) / 16;
  return (b < last ? b : last) >> (page_shift - 4);
}
// Whether block b counts and `number` is a page of the cache.
__host__ __device__ inline bool cache_counts(int b, int vis, int number, int64_t pages) {
  return (int64_t)b * 16 < vis && number >= 0 && number < pages;
}

// What a worker (a wave, or a workgroup) leaves for the joining launch: `first`: 0, or its share begins inside a unit, which goes
// on behind it (1) or ends in it (2); rows > 0: its share ends inside a unit of so many rows, which begins in it: (KV head, tile) of
// the request whose first row is cu.
struct CacheLeft { int first, rows, head, tile, cu; };

struct CachePlan {
  CacheAttnArgs a;
  int workers;         // shares, at most
  CacheLeft* left;     // [workers]
  // [workers][2] partial results, [0]: of the unit that began before the share, [1]: of the one that goes on behind it.  Each: m and
  // l of every row of a tile, then O.
  float* partial;
  int whole;           // shares end with units: there are no partial results
  __host__ __device__ static int64_t slot(int rows_per_tile, int hs) { return (int64_t)rows_per_tile * (hs + 2); }
};

constexpr int kCacheRowsTile = 256;      // rows of a unit of the kernel for many rows
int launch_cache_attn_rows(const CachePlan& p, hipStream_t stream);
int launch_cache_attn(const CacheAttnArgs& a, int max_q, hipStream_t stream);
size_t cache_attn_workspace(int group, int hs, int max_q);

}  // namespace usp
