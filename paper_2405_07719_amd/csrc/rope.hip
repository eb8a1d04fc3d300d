// Rotary positions of Q and K in one launch, forward and backward (the transpose: the angle negated).
//
// HBM-bound: each element is read once and written once.  A thread holds E = 8 (bf16) or 4 (fp32) pairs of one row's
// frequencies: it forms their sines and cosines once, in registers, and turns the same places of several heads with them, so
// there is no table of angles to read.  The angle is position * frequency in turns in 64 bits, of which the nearest quarter
// turn is taken off there: a 32-bit angle of position 2^18 is off by up to 2^-7 radians already.  What is left lies within an eighth of a
// turn, where Taylor's polynomials of x^9 and x^10 are exact to 2e-9.
//
// Measured: Q and K of a training rank (8192 rows of 32 + 8 heads of 128, bf16, 168 MB) 33 us, 5.1 TB/s; a copy of as many
// bytes by the library takes 34.5.  Values are read nontemporally, which makes 37 us 33; written so, too, 34, and interleaved
// pairs in fp32, whose lines two stores share, 44 instead of 35.  Eight rows: 4.0 us on the GPU (latency: arguments, positions, values, one after the other), 5.9 us a call.
#include "serve_internal.h"

namespace usp {
namespace {

constexpr int kThreads = 256;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Vec;
template <> struct Vec<__bf16> { typedef bf16x8 type; static constexpr int E = 8; typedef f32x8 wide; };
template <> struct Vec<float> { typedef f32x4 type; static constexpr int E = 4; typedef f32x4 wide; };

// sine and cosine of `turns` turns
__device__ inline void sine_cosine(double turns, float* s, float* c) {
  const double quarters = 4.0 * (turns - rint(turns)), n = rint(quarters);     // n in -2 .. 2
  const float x = (float)(quarters - n) * 1.57079632679489662f, z = x * x;
  const float sx = x * (1.0f + z * (-1.0f / 6 + z * (1.0f / 120 + z * (-1.0f / 5040 + z * (1.0f / 362880)))));
  const float cx = 1.0f + z * (-0.5f + z * (1.0f / 24 + z * (-1.0f / 720 + z * (1.0f / 40320 + z * (-1.0f / 3628800)))));
  const int quadrant = (int)n & 3;
  const float a = quadrant & 1 ? cx : sx, b = quadrant & 1 ? sx : cx;
  *s = quadrant & 2 ? -a : a;
  *c = (quadrant + 1) & 2 ? -b : b;
}

// 2^log_groups threads share a row's heads.
template <typename T, int HS>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int log_groups, int64_t first_row) {
  typedef typename Vec<T>::type V;
  typedef typename Vec<T>::wide W;
  constexpr int E = Vec<T>::E, kUnits = HS / (2 * E);      // threads that hold one head of one row
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x, unit = id % kUnits, rest = id / kUnits;
  double turns_of[E];                                      // (ahead of all that waits for the other arguments)
#pragma unroll
  for (int e = 0; e < E; ++e) turns_of[e] = a.turns[unit * E + e];
  const int group = (int)(rest & ((1u << log_groups) - 1)), head_groups = 1 << log_groups;
  const int64_t row = first_row + (rest >> log_groups);
  if (row >= a.rows) return;
  const bool turns = (int)unit * 2 * E < a.rotary_dim;
  if (!turns && a.in_place) return;
  int64_t pos;
  if (a.positions) {
    pos = a.positions[row];
  } else {
    const int64_t shard = row / a.per_shard, i = row - shard * a.per_shard;
    const int rank = a.rank0 + (int)(shard / a.bs), r = rank / a.ulysses, u = rank - r * a.ulysses;
    const int64_t j = u * a.per_shard + i;                 // place in the ring rank's block
    pos = !a.half_chunk ? r * a.ring_block + j
                        : j < a.half_chunk ? r * a.half_chunk + j : (2 * a.ring - 1 - r) * a.half_chunk + j - a.half_chunk;
  }
  float s[E], c[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    sine_cosine((double)pos * turns_of[e], &s[e], &c[e]);
    s[e] *= a.sign * a.magnitude;
    c[e] *= a.magnitude;
  }
  // the first of each pair begins at element e0, the second (or the next E elements) at e1
  const bool halves = turns && !a.pairs;
  const int e0 = (int)unit * (halves ? E : 2 * E), e1 = halves ? e0 + a.rotary_dim / 2 : e0 + E;
  const int heads = a.heads[0] + a.heads[1];
#pragma unroll 2
  for (int h = group; h < heads; h += head_groups) {
    const int t = h >= a.heads[0], ht = t ? h - a.heads[0] : h;
    const T* x = (const T*)a.x[t] + row * a.stride[t] + ht * HS;
    T* y = (T*)a.y[t] + row * a.out_stride[t] + ht * HS;
    V va = __builtin_nontemporal_load((const V*)(x + e0)), vb = __builtin_nontemporal_load((const V*)(x + e1));
    if (turns) {
      const W fa = __builtin_convertvector(va, W), fb = __builtin_convertvector(vb, W);
      W ga, gb;
      if (halves) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          ga[e] = fa[e] * c[e] - fb[e] * s[e];
          gb[e] = fa[e] * s[e] + fb[e] * c[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          ga[2 * e] = fa[2 * e] * c[e] - fa[2 * e + 1] * s[e];
          ga[2 * e + 1] = fa[2 * e] * s[e] + fa[2 * e + 1] * c[e];
          gb[2 * e] = fb[2 * e] * c[E / 2 + e] - fb[2 * e + 1] * s[E / 2 + e];
          gb[2 * e + 1] = fb[2 * e] * s[E / 2 + e] + fb[2 * e + 1] * c[E / 2 + e];
        }
      }
      va = __builtin_convertvector(ga, V);
      vb = __builtin_convertvector(gb, V);
    }
    *(V*)(y + e0) = va;
    *(V*)(y + e1) = vb;
  }
}

}  // namespace

template <typename T>
static void launch(const RopeArgs& a, int log_groups, int64_t first, unsigned grid, hipStream_t stream) {
  if (a.hs == 128) rope_kernel<T, 128><<<dim3(grid), kThreads, 0, stream>>>(a, log_groups, first);
  else rope_kernel<T, 64><<<dim3(grid), kThreads, 0, stream>>>(a, log_groups, first);
}

int launch_rope(const RopeArgs& a, int dtype, hipStream_t stream) {
  const int heads = a.heads[0] + a.heads[1], units = a.hs / (dtype == USP_BF16 ? 16 : 8);
  // One thread per row, unit and head while that fills the chip once over; then more heads to a thread, which forms its
  // angles once for all of them.  Powers of two, so that a thread's place takes shifts: with divisions the training rank's
  // rows took 41 us.
  int log_groups = 0;
  while (2 << log_groups <= heads && a.rows * units << log_groups < (int64_t)kPlanCUs * 2048) ++log_groups;
  // (several launches where one would have 2^32 threads or more)
  const int64_t most = max_workgroups(kThreads) * kThreads / units >> log_groups;
  for (int64_t first = 0; first < a.rows; first += most) {
    const int64_t rows = a.rows - first < most ? a.rows - first : most;
    const unsigned grid = (unsigned)(((rows * units << log_groups) + kThreads - 1) / kThreads);
    if (dtype == USP_BF16) launch<__bf16>(a, log_groups, first, grid, stream);
    else launch<float>(a, log_groups, first, grid, stream);
  }
  return launch_status();
}

}  // namespace usp
