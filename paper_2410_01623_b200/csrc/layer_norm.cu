// Layer norm, forward and backward, with the form without mean and bias (RMS).
//
//   y = (x - mu) s g + b,   mu = mean(x) (RMS: 0),   s = 1 / sqrt(mean((x - mu)^2) + eps)
//   with h = (x - mu) s, q = dy g:   dx = s (q - mean(q) - h mean(q h))   (RMS: without mean(q))
//   dg = sum over rows of dy h,   db = sum over rows of dy
//
// A group of 4 to 1024 threads takes a row, each thread 16 elements of it: fetched once, into shared memory, where only this thread
// reads them (in the backward pass with mean or of more than 8192 columns twice: there are no registers to keep them in); the next rows
// are on their way meanwhile, where there is room.  Gain and bias lie in shared memory in the order in which
// the threads read them.  Statistics are fp32, the variance from the differences to the mean.  In the backward pass a
// thread has the same columns in every row of its group, so that dg and db grow in its registers; the groups of a block are added in shared memory, the
// blocks in a second launch, always in the same order.
//
// Rows that do not start on 16-byte boundaries (odd widths) are read and written in the same aligned 16 bytes: a group
// takes only rows that begin equally far behind such a boundary.
#include <math.h>

#include <algorithm>

#include "rows.cuh"
#include "tc_ptx.cuh"

namespace fira {
namespace {

constexpr int LN_THREADS = 256;             // of a block, where a row takes no more
constexpr int LN_EACH = 16;                 // elements of a row that a thread has
constexpr int LN_MAX_HIDDEN = 1024 * LN_EACH;
constexpr int LN_SMS = 148;

// The threads of a row, and this thread's place.
struct Group {
  int threads, id, rank, count;             // id of count groups in the block
  unsigned mask;                            // its lanes, where it is a part of a warp
  __device__ __forceinline__ explicit Group(int per_row) : threads(per_row), id(threadIdx.x / per_row), rank(threadIdx.x % per_row), count(blockDim.x / per_row),
    mask(per_row >= 32 ? 0xffffffffu : ((1u << per_row) - 1) << (threadIdx.x & 31 & ~(per_row - 1))) {}
};

// (LN_THREADS is four groups of two warps at most.)
__device__ __forceinline__ void group_barrier(const Group& g) {
  if (g.count == 1) __syncthreads();
  else if (g.id == 0) asm volatile("bar.sync 1, %0;" :: "r"(g.threads) : "memory");
  else if (g.id == 1) asm volatile("bar.sync 2, %0;" :: "r"(g.threads) : "memory");
  else if (g.id == 2) asm volatile("bar.sync 3, %0;" :: "r"(g.threads) : "memory");
  else asm volatile("bar.sync 4, %0;" :: "r"(g.threads) : "memory");
}

// Sums over the group of one or two values of each thread.  Calls use the two buffers in turn, so that one barrier is enough.
// PART: the group is a part of a warp (the others of the warp may be elsewhere).
template <int VALUES, bool PART>
__device__ __forceinline__ float2 group_sum(float2 v, const Group& g, float2 (*red)[32], int& turn) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    if (PART && o >= g.threads) continue;
    v.x += __shfl_xor_sync(PART ? g.mask : 0xffffffffu, v.x, o);
    if (VALUES == 2) v.y += __shfl_xor_sync(PART ? g.mask : 0xffffffffu, v.y, o);
  }
  if (PART || g.threads == 32) return v;
  const int lane = threadIdx.x & 31, warps = g.threads >> 5, first = g.id * warps;
  if (lane == 0) red[turn][threadIdx.x >> 5] = v;
  group_barrier(g);
  v = lane < warps ? red[turn][first + lane] : make_float2(0.f, 0.f);
  turn ^= 1;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    if (VALUES == 2) v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  return v;
}

// How a thread's pieces of a row (N elements each, 16 bytes) lie in memory.
// ALIGNED: rows are whole 16-byte units on 16-byte boundaries.
// SHIFTED: a row begins `shift` elements behind such a boundary; the pieces are those of memory, and the first and the
//   last may lie partly outside the row: all 16 aligned bytes are fetched, of which one at least is the row's, and the others
//   dropped.  (All rows of a group, in all tensors, have the same shift, so that a piece has the same columns in all of them.)
// SINGLE: one element per thread in turn, for rows of one tensor that begin otherwise than those of another.
enum Mode { SINGLE, SHIFTED, ALIGNED };

template <typename T, Mode MODE>
struct Cols {
  static constexpr int N = rows::PER16<T>, PIECES = LN_EACH / N;
  static constexpr unsigned FULL = (1u << N) - 1;
  int rank, threads, hidden, shift;
  unsigned bits;                            // bit p N + e: that element is one of the row
  __device__ __forceinline__ int at(int p, int e) const { return MODE == SINGLE ? (p * N + e) * threads + rank : (p * threads + rank) * N + e - shift; }
  __device__ __forceinline__ bool in(int p, int e) const { return bits >> (p * N + e) & 1; }
  __device__ __forceinline__ bool any(int p) const { return (bits >> (p * N) & FULL) != 0; }
  __device__ __forceinline__ bool whole(int p) const { return MODE == ALIGNED ? any(p) : MODE == SHIFTED && (bits >> (p * N) & FULL) == FULL; }
  __device__ __forceinline__ Cols(const Group& g, int width, int begins) : rank(g.rank), threads(g.threads), hidden(width), shift(begins), bits(0) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int e = 0; e < N; ++e) bits |= (at(p, e) >= 0 && at(p, e) < hidden ? 1u : 0u) << (p * N + e);
  }
  // A row on its way to slots of this thread, one per piece and `apart` apart (zeros where a piece is none of the row).
  __device__ __forceinline__ void fetch(const T* row, uint4* slot, int apart) const {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      if (MODE != SINGLE) {
        if (any(p))
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"((unsigned)__cvta_generic_to_shared(slot + p * apart)), "l"(row + at(p, 0)) : "memory");
      } else {
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        T* v = reinterpret_cast<T*>(&u);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (in(p, e)) v[e] = row[at(p, e)];
        slot[p * apart] = u;
      }
    }
  }
  // Once a row is there: zeros where its ends' pieces are not the row's.
  __device__ __forceinline__ void trim(uint4* slot, int apart) const {
    if constexpr (MODE == SHIFTED) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        if (!any(p) || whole(p)) continue;
        unsigned* w = reinterpret_cast<unsigned*>(slot + p * apart);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[k] &= sizeof(T) == 4 ? 0u - (bits >> (p * N + k) & 1) : ((0u - (bits >> (p * N + 2 * k) & 1)) & 0xffffu) | (0u - (bits >> (p * N + 2 * k + 1) & 1)) << 16;
      }
    }
  }
  __device__ __forceinline__ void store(T* row, int p, const float2 (&v)[N / 2]) const {
    const uint4 u = rows::pack<T>(v);
    if (whole(p)) {
      *reinterpret_cast<uint4*>(row + at(p, 0)) = u;
    } else if (MODE != ALIGNED) {
      const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (in(p, e)) {
          if constexpr (sizeof(T) == 4) reinterpret_cast<unsigned*>(row)[at(p, e)] = w[e];
          else reinterpret_cast<unsigned short*>(row)[at(p, e)] = (unsigned short)(w[e / 2] >> (e & 1) * 16);
        }
    }
  }
  // Gains or biases, of either type, into shared memory: four elements of every thread of the group after one another.
  __device__ __forceinline__ void keep(const void* q, int bf16, float* to) const {
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          v[k] = !q || !in(p, e + k) ? 0.f : bf16 ? to_float(static_cast<const __nv_bfloat16*>(q)[at(p, e + k)]) : static_cast<const float*>(q)[at(p, e + k)];
        reinterpret_cast<float4*>(to)[(p * N + e) / 4 * threads + rank] = make_float4(v[0], v[1], v[2], v[3]);
      }
  }
  __device__ __forceinline__ void kept(const float* from, int p, float2 (&v)[N / 2]) const {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      const float4 u = reinterpret_cast<const float4*>(from)[(p * N + e) / 4 * threads + rank];
      v[e / 2] = make_float2(u.x, u.y); v[e / 2 + 1] = make_float2(u.z, u.w);
    }
  }
};
// Elements from the 16-byte boundary in front of a row to the row.
template <typename T>
__device__ __forceinline__ int shift_of(const T* row) { return (int)(((uintptr_t)row & 15) / sizeof(T)); }

// Rows on their way to shared memory, the one that is worked on among them: as many as there is room for.
template <typename T, bool LONG, bool RMS>
constexpr int NORM_STAGES = !LONG && RMS && sizeof(T) == 2 ? 3 : !LONG || RMS || sizeof(T) == 2 ? 2 : 1;
template <typename T, bool LONG, bool RMS>
constexpr size_t NORM_SMEM = (RMS ? 1 : 2) * LN_EACH * sizeof(float) + NORM_STAGES<T, LONG, RMS> * LN_EACH * sizeof(T);     // per thread
template <typename T, int THREADS>
constexpr int GRAD_STAGES = THREADS == 1024 ? (sizeof(T) == 2 ? 2 : 1) : THREADS == 512 ? (sizeof(T) == 2 ? 4 : 2) : (sizeof(T) == 2 ? 3 : 2);
template <typename T, int THREADS>
constexpr size_t GRAD_SMEM = (size_t)LN_EACH * sizeof(float) + 2 * GRAD_STAGES<T, THREADS> * LN_EACH * sizeof(T);

// Blocks of the backward pass on an SM (where rows take LN_THREADS threads at most): three where 80 registers nearly suffice (56 bytes of a
// thread spilled; 65536 rows of 512, bf16, without mean: 45 us), two of more registers elsewhere (of 256, fp32: 62 us with three, 43 with two).
template <typename T, Mode MODE, bool RMS, int THREADS>
constexpr int GRAD_RESIDENT = THREADS > LN_THREADS ? 1 : RMS && MODE == ALIGNED && sizeof(T) == 2 ? 3 : 2;

// SIZE: rows of a part of a warp, of up to LN_THREADS threads, of more.
enum Size { PART, SOME, BIG };

template <typename T, Mode MODE, Size SIZE, bool RMS>
__global__ void __launch_bounds__(SIZE == BIG ? 1024 : LN_THREADS, SIZE == BIG ? 1 : 4)
k_layer_norm(const T* x, long long ld_x, long long nrows, int hidden, int per_row, const void* gain, const void* bias, int param_bf16, float eps,
             T* y, long long ld_y, float* __restrict__ mean, float* __restrict__ rstd) {
  using C = Cols<T, MODE>;
  constexpr int N = C::N, PIECES = C::PIECES, STAGES = NORM_STAGES<T, SIZE == BIG, RMS>;
  static_assert((SIZE == BIG ? 1024 : LN_THREADS) * NORM_SMEM<T, SIZE == BIG, RMS> + 2048 <= 227 * 1024, "shared memory of a block");
  extern __shared__ float4 kept4[];         // gains of every group, then (not RMS) biases, then the rows on their way
  __shared__ float2 red[2][32];
  const Group g(per_row);
  const long long stride = (long long)gridDim.x * g.count;
  long long row = (long long)blockIdx.x * g.count + g.id;
  if (row >= nrows) return;                 // a whole group: its barrier is its own
  const C cols(g, hidden, MODE == SHIFTED ? shift_of(x + row * ld_x) : 0);
  const int apart = blockDim.x;             // (a thread reads what it fetched or wrote: no barriers here)
  uint4* ring = reinterpret_cast<uint4*>(kept4 + (RMS ? 1 : 2) * blockDim.x * (LN_EACH / 4)) + threadIdx.x;
  if (MODE != SINGLE) {
#pragma unroll
    for (int k = 0; k < STAGES * PIECES; ++k) ring[k * apart] = make_uint4(0u, 0u, 0u, 0u);
  }
  auto fetch = [&](long long r, int stage) {
    if (r < nrows) cols.fetch(x + r * ld_x, ring + stage * PIECES * apart, apart);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int k = 0; k + 1 < STAGES; ++k) fetch(row + k * stride, k);
  float* gains = reinterpret_cast<float*>(kept4) + g.id * per_row * LN_EACH;
  float* biases = gains + blockDim.x * LN_EACH;
  cols.keep(gain, param_bf16, gains);
  if (!RMS) cols.keep(bias, param_bf16, biases);
  const float inv = 1.f / (float)hidden;
  int turn = 0, stage = 0;
  for (;;) {
    fetch(row + (STAGES - 1) * stride, stage == 0 ? STAGES - 1 : stage - 1);
    asm volatile("cp.async.wait_group %0;" :: "n"(STAGES - 1) : "memory");
    uint4* slots = ring + stage * PIECES * apart;
    cols.trim(slots, apart);
    float2 v[PIECES][N / 2], s = make_float2(0.f, 0.f);
    float mu = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) rows::unpack<T>(slots[p * apart], v[p]);
    if (!RMS) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int e = 0; e < N / 2; ++e) s = rows::add2(s, v[p][e]);
      mu = group_sum<1, SIZE == PART>(make_float2(s.x + s.y, 0.f), g, red, turn).x * inv;
      s = make_float2(0.f, 0.f);
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
#pragma unroll
        for (int e = 0; e < N / 2; ++e) v[p][e] = rows::add2(v[p][e], rows::both(-mu));
        if (!cols.whole(p)) {               // what lies outside the row is no part of the variance
#pragma unroll
          for (int e = 0; e < N / 2; ++e) {
            if (!cols.in(p, 2 * e)) v[p][e].x = 0.f;
            if (!cols.in(p, 2 * e + 1)) v[p][e].y = 0.f;
          }
        }
      }
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int e = 0; e < N / 2; ++e) s = rows::fma2(v[p][e], v[p][e], s);
    const float rs = 1.f / sqrtf(group_sum<1, SIZE == PART>(make_float2(s.x + s.y, 0.f), g, red, turn).x * inv + eps);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      float2 w[N / 2], b[N / 2];
      cols.kept(gains, p, w);
      if (!RMS) cols.kept(biases, p, b);
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        const float2 h = rows::mul2(v[p][e], rows::both(rs));
        v[p][e] = RMS ? rows::mul2(h, w[e]) : rows::fma2(h, w[e], b[e]);
      }
      cols.store(y + row * ld_y, p, v[p]);
    }
    if (g.rank == 0) {
      rstd[row] = rs;
      if (!RMS) mean[row] = mu;
    }
    row += stride;
    if (row >= nrows) return;
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
}

// parts: per block the sums of dy h, then (want_bias) those of dy, `hidden` floats each.
template <typename T, Mode MODE, int THREADS, bool PARTS, bool RMS>
__global__ void __launch_bounds__(THREADS, (GRAD_RESIDENT<T, MODE, RMS, THREADS>))
k_layer_norm_grad(const T* dy, long long ld_dy, const T* x, long long ld_x, long long nrows, int hidden, int per_row, const void* gain,
                  int param_bf16, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, long long ld_dx,
                  float* __restrict__ parts, int want_bias) {
  using C = Cols<T, MODE>;
  constexpr int N = C::N, PIECES = C::PIECES, STAGES = GRAD_STAGES<T, THREADS>;
  constexpr bool KEEP = RMS && THREADS < 1024;        // h and q stay in registers while the sums are made: where there are registers
  static_assert(THREADS * GRAD_SMEM<T, THREADS> + 2048 <= 227 * 1024, "shared memory of a block");
  extern __shared__ float4 kept4[];         // gains of every group; then sums of the groups; behind them the rows on their way
  __shared__ float2 red[2][32];
  ptx::grid_launch_next();
  const Group g(per_row);
  const long long stride = (long long)gridDim.x * g.count;
  long long row = (long long)blockIdx.x * g.count + g.id;
  if (PARTS && MODE == SHIFTED) {           // the groups of a warp eight rows apart: they begin alike, and have the same columns
    const int groups = 32 / g.threads;
    const long long warp = (long long)blockIdx.x * (THREADS / 32) + threadIdx.x / 32;
    row = (warp / 8 * groups + g.id % groups) * 8 + warp % 8;
  }
  const C cols(g, hidden, MODE == SHIFTED ? shift_of(x + row * ld_x) : 0);
  float2 dg[PIECES][N / 2], db[PIECES][N / 2];
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int e = 0; e < N / 2; ++e) dg[p][e] = db[p][e] = make_float2(0.f, 0.f);
  if (row < nrows) {
    const int apart = blockDim.x;           // (a thread reads what it fetched or wrote: no barriers here)
    uint4* ring = reinterpret_cast<uint4*>(kept4 + blockDim.x * (LN_EACH / 4)) + threadIdx.x;
    if (MODE != SINGLE) {
#pragma unroll
      for (int k = 0; k < STAGES * 2 * PIECES; ++k) ring[k * apart] = make_uint4(0u, 0u, 0u, 0u);
    }
    auto fetch = [&](long long r, int stage) {
      if (r < nrows) {
        cols.fetch(x + r * ld_x, ring + (stage * 2) * PIECES * apart, apart);
        cols.fetch(dy + r * ld_dy, ring + (stage * 2 + 1) * PIECES * apart, apart);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k + 1 < STAGES; ++k) fetch(row + k * stride, k);
    float rs = rstd[row], mu = RMS ? 0.f : mean[row];
    float* gains = reinterpret_cast<float*>(kept4) + g.id * per_row * LN_EACH;
    cols.keep(gain, param_bf16, gains);
    const float inv = 1.f / (float)hidden;
    int turn = 0, stage = 0;
    for (;;) {
      const bool more = row + stride < nrows;
      float next_rs = 0.f, next_mu = 0.f;
      if (more) {
        next_rs = rstd[row + stride];
        if (!RMS) next_mu = mean[row + stride];
      }
      fetch(row + (STAGES - 1) * stride, stage == 0 ? STAGES - 1 : stage - 1);
      asm volatile("cp.async.wait_group %0;" :: "n"(STAGES - 1) : "memory");
      uint4* rx = ring + (stage * 2) * PIECES * apart;
      uint4* ry = ring + (stage * 2 + 1) * PIECES * apart;
      cols.trim(rx, apart);
      cols.trim(ry, apart);
      float2 h[PIECES][N / 2], q[PIECES][N / 2], along2 = make_float2(0.f, 0.f), level2 = make_float2(0.f, 0.f);
      // h, q and dy of piece p
      auto terms = [&](int p, float2 (&hp)[N / 2], float2 (&qp)[N / 2], float2 (&d)[N / 2]) {
        float2 w[N / 2];
        rows::unpack<T>(rx[p * apart], hp);
        rows::unpack<T>(ry[p * apart], d);
        cols.kept(gains, p, w);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          hp[e] = rows::mul2(RMS ? hp[e] : rows::add2(hp[e], rows::both(-mu)), rows::both(rs));
          qp[e] = rows::mul2(d[e], w[e]);
        }
      };
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        float2 d[N / 2];
        terms(p, h[p], q[p], d);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          along2 = rows::fma2(q[p][e], h[p][e], along2);
          dg[p][e] = rows::fma2(d[e], h[p][e], dg[p][e]);
          if (!RMS) { level2 = rows::add2(level2, q[p][e]); db[p][e] = rows::add2(db[p][e], d[e]); }
        }
        if (!KEEP) asm volatile("" ::: "memory");     // one piece after the other: registers
      }
      const float2 s = group_sum<RMS ? 1 : 2, PARTS>(make_float2(along2.x + along2.y, level2.x + level2.y), g, red, turn);
      const float2 along = rows::both(-s.x * inv), level = rows::both(-s.y * inv);
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        if (!KEEP) { float2 d[N / 2]; terms(p, h[p], q[p], d); }
#pragma unroll
        for (int e = 0; e < N / 2; ++e)
          h[p][e] = rows::mul2(rows::both(rs), rows::fma2(h[p][e], along, RMS ? q[p][e] : rows::add2(q[p][e], level)));
        cols.store(dx + row * ld_dx, p, h[p]);
        if (!KEEP) asm volatile("" ::: "memory");
      }
      if (!more) break;
      row += stride;
      rs = next_rs; mu = next_mu;
      stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
  }
  // Groups of a warp (which have the same columns) by shuffles, then the groups, or the warps, one after another.
  int turns = g.count, turn = g.id;
  if (PARTS) {
    __syncwarp();
#pragma unroll
    for (int o = 4; o < 32; o *= 2) {
      if (o < g.threads) continue;
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          dg[p][e].x += __shfl_xor_sync(0xffffffffu, dg[p][e].x, o); dg[p][e].y += __shfl_xor_sync(0xffffffffu, dg[p][e].y, o);
          if (!RMS) { db[p][e].x += __shfl_xor_sync(0xffffffffu, db[p][e].x, o); db[p][e].y += __shfl_xor_sync(0xffffffffu, db[p][e].y, o); }
        }
    }
    turns = blockDim.x / 32;
    turn = (threadIdx.x & 31) < g.threads ? (int)(threadIdx.x / 32) : -1;
  }
  float* sums = reinterpret_cast<float*>(kept4);      // [2 or 1][hidden]: where there are groups, no more than the gains took
  if (turns > 1) __syncthreads();
  float* out = parts + (long long)blockIdx.x * hidden * (want_bias ? 2 : 1);
  for (int k = 0; k < turns; ++k) {
    if (turn == k) {
      float* to = k + 1 < turns ? sums : out;
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          if (!cols.in(p, e)) continue;
          const int c = cols.at(p, e);
          const float u = e & 1 ? dg[p][e / 2].y : dg[p][e / 2].x;
          to[c] = k > 0 ? u + sums[c] : u;
          if (want_bias) {
            const float v = e & 1 ? db[p][e / 2].y : db[p][e / 2].x;
            to[hidden + c] = k > 0 ? v + sums[hidden + c] : v;
          }
        }
    }
    if (turns > 1) __syncthreads();
  }
}

// Adds the blocks' sums: 32 columns per block, the blocks' rows dealt to 32 warps.
__global__ void __launch_bounds__(1024)
k_layer_norm_params(const float* parts, int nparts, int width, int hidden, void* dgain, void* dbias, int bf16, int accumulate) {
  __shared__ float part[32][33];
  ptx::grid_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;     // of width = hidden, or 2 hidden with the bias behind the gain
  float s = 0.f;
  if (c < width) {
#pragma unroll 8
    for (int r = warp; r < nparts; r += 32) s += parts[(long long)r * width + c];
  }
  part[warp][lane] = s;
  __syncthreads();
  s = part[lane][warp];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const int col = blockIdx.x * 32 + warp;
  if (lane == 0 && col < width) {
    void* out = col < hidden ? dgain : dbias;
    const int at = col < hidden ? col : col - hidden;
    if (bf16) {
      __nv_bfloat16* q = static_cast<__nv_bfloat16*>(out) + at;
      *q = __float2bfloat16_rn(accumulate ? to_float(*q) + s : s);
    } else {
      float* q = static_cast<float*>(out) + at;
      *q = accumulate ? *q + s : s;
    }
  }
}

// How a call's rows are taken; a shifted row takes up to a piece more.
struct RowPlan {
  int per_row = 0, threads = 0, groups = 0;
  Mode mode = SINGLE;
  Size size = SOME;
};
RowPlan rows_of(long long hidden, size_t bytes, Mode mode) {
  RowPlan p;
  const long long extent = hidden + (mode == SHIFTED ? 16 / (long long)bytes - 1 : 0);
  if (extent > LN_MAX_HIDDEN) return rows_of(hidden, bytes, SINGLE);
  p.mode = mode;
  p.per_row = 4;
  while ((long long)p.per_row * LN_EACH < extent) p.per_row *= 2;
  p.threads = std::max(LN_THREADS, p.per_row);
  p.groups = p.threads / p.per_row;
  p.size = p.per_row < 32 ? PART : p.per_row > LN_THREADS ? BIG : SOME;
  return p;
}
// All groups get one row at most, or a number of groups that is a multiple of 8: then the rows of a group begin equally
// far behind a 16-byte boundary, whatever their pitch.
long long blocks_for(const RowPlan& p, long long nrows, long long most, long long rows_each) {
  const long long all = std::max<long long>(1, (nrows + p.groups - 1) / p.groups);
  const long long some = std::min(most, (nrows + rows_each * p.groups - 1) / (rows_each * p.groups));
  return std::min(all, std::max<long long>(8, (some + 7) / 8 * 8));
}
// Blocks of the backward pass: as many as are resident at once, and four rows at least for a group, since each block
// writes its sums of dg and db.
int grad_blocks(const RowPlan& p, long long nrows, bool rms, size_t bytes) {
  const int resident = p.size == BIG ? 1 : rms && p.mode == ALIGNED && bytes == 2 ? GRAD_RESIDENT<__nv_bfloat16, ALIGNED, true, LN_THREADS> : GRAD_RESIDENT<float, SINGLE, false, LN_THREADS>;
  return (int)blocks_for(p, nrows, resident * LN_SMS / 8 * 8, 4);
}

template <typename T, Mode MODE, Size SIZE, bool RMS>
cudaError_t run_forward(const RowPlan& p, const void* x, long long ld_x, long long nrows, int hidden, const void* gain, const void* bias, int param_bf16,
                        float eps, void* y, long long ld_y, float* mean, float* rstd, cudaStream_t st) {
  const size_t smem = p.threads * NORM_SMEM<T, SIZE == BIG, RMS>;
  const cudaError_t e = cudaFuncSetAttribute(k_layer_norm<T, MODE, SIZE, RMS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)((SIZE == BIG ? 1024 : LN_THREADS) * NORM_SMEM<T, SIZE == BIG, RMS>));
  if (e != cudaSuccess) return e;
  // four times as many blocks as are resident, since SMs far from the memory take longer (32768 rows of 4096, bf16: 100 us
  // with four blocks per SM in all, 89 with 16, 96 with 32)
  const unsigned blocks = (unsigned)blocks_for(p, nrows, (SIZE == BIG ? 4 : 16) * LN_SMS, 1);
  k_layer_norm<T, MODE, SIZE, RMS><<<blocks, p.threads, smem, st>>>((const T*)x, ld_x, nrows, hidden, p.per_row, gain, bias, param_bf16, eps, (T*)y, ld_y, mean, rstd);
  return cudaGetLastError();
}
template <typename T, Mode MODE, int THREADS, bool PARTS, bool RMS>
cudaError_t run_backward_of(const RowPlan& p, const void* dy, long long ld_dy, const void* x, long long ld_x, long long nrows, int hidden, const void* gain,
                            int param_bf16, const float* mean, const float* rstd, void* dx, long long ld_dx, float* parts, int want_bias, cudaStream_t st) {
  const cudaError_t e = cudaFuncSetAttribute(k_layer_norm_grad<T, MODE, THREADS, PARTS, RMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(THREADS * GRAD_SMEM<T, THREADS>));
  if (e != cudaSuccess) return e;
  k_layer_norm_grad<T, MODE, THREADS, PARTS, RMS><<<grad_blocks(p, nrows, RMS, sizeof(T)), p.threads, p.threads * GRAD_SMEM<T, THREADS>, st>>>(
      (const T*)dy, ld_dy, (const T*)x, ld_x, nrows, hidden, p.per_row, gain, param_bf16, mean, rstd, (T*)dx, ld_dx, parts, want_bias);
  return cudaGetLastError();
}
template <typename T, Mode MODE, Size SIZE, bool RMS, typename... A>
cudaError_t run_backward(const RowPlan& p, A... a) {
  if constexpr (SIZE != BIG) return run_backward_of<T, MODE, LN_THREADS, SIZE == PART, RMS>(p, a...);
  else return p.per_row == 512 ? run_backward_of<T, MODE, 512, false, RMS>(p, a...) : run_backward_of<T, MODE, 1024, false, RMS>(p, a...);
}

fira_status check_norm(const std::string& who, int64_t rows, int64_t hidden, fira_dtype dtype, fira_dtype param_dtype) {
  if (rows < 0 || rows > (1ll << 40) || hidden <= 0) { set_error(who + ": need 0 <= rows <= 2^40 and hidden > 0"); return FIRA_ERR_INVALID_ARG; }
  if (hidden > LN_MAX_HIDDEN) { set_error(who + ": rows of more than 16384 elements"); return FIRA_ERR_UNSUPPORTED; }
  if ((dtype != FIRA_F32 && dtype != FIRA_BF16) || (param_dtype != FIRA_F32 && param_dtype != FIRA_BF16)) { set_error(who + ": unknown dtype"); return FIRA_ERR_INVALID_ARG; }
  return FIRA_OK;
}
bool off(const void* p, size_t size) { return !p || ((uintptr_t)p & (size - 1)); }
bool bad_ld(int64_t& ld, int64_t hidden) {
  if (ld == 0) ld = hidden;
  return ld < hidden || ld > (1ll << 32);
}

// Whether rows of the two tensors begin equally far behind a 16-byte boundary, all of them.
bool alike(const void* a, long long ld_a, const void* b, long long ld_b, size_t size) {
  return (((uintptr_t)a ^ (uintptr_t)b) & 15) == 0 && ((ld_a - ld_b) * (long long)size) % 16 == 0;
}
Mode mode_of(const void* a, long long ld, long long hidden, size_t size, bool all_alike) {
  return !all_alike ? SINGLE : rows::aligned16(a, ld, hidden, size) ? ALIGNED : SHIFTED;
}

#define LN_DISPATCH_MODE(CALL, T, M)                                                                                    \
  do {                                                                                                                  \
    if (p.size == BIG) { if (rms) CALL(T, M, BIG, true); else CALL(T, M, BIG, false); }                                 \
    else if (p.size == PART) { if (rms) CALL(T, M, PART, true); else CALL(T, M, PART, false); }                         \
    else { if (rms) CALL(T, M, SOME, true); else CALL(T, M, SOME, false); }                                             \
  } while (0)
#define LN_DISPATCH_TYPE(CALL, T)                                                                                       \
  do {                                                                                                                  \
    if (p.mode == ALIGNED) LN_DISPATCH_MODE(CALL, T, ALIGNED);                                                          \
    else if (p.mode == SHIFTED) LN_DISPATCH_MODE(CALL, T, SHIFTED);                                                     \
    else LN_DISPATCH_MODE(CALL, T, SINGLE);                                                                             \
  } while (0)
#define LN_DISPATCH(CALL)                                                                                               \
  do {                                                                                                                  \
    if (dtype == FIRA_BF16) LN_DISPATCH_TYPE(CALL, __nv_bfloat16);                                                      \
    else LN_DISPATCH_TYPE(CALL, float);                                                                                 \
  } while (0)

}  // namespace
}  // namespace fira

using namespace fira;

extern "C" fira_status fira_layer_norm(const void* x_dev, int64_t ld_x, fira_dtype dtype, int64_t nrows, int64_t hidden,
                                       const void* gain_dev, const void* bias_dev, fira_dtype param_dtype, float eps, void* y_dev,
                                       int64_t ld_y, float* mean_dev, float* rstd_dev, void* cuda_stream) {
  return guarded([&]() -> fira_status {
    const std::string who("fira_layer_norm");
    const fira_status bad = check_norm(who, nrows, hidden, dtype, param_dtype);
    if (bad != FIRA_OK) return bad;
    if (bad_ld(ld_x, hidden) || bad_ld(ld_y, hidden)) { set_error(who + ": ld below the width, or above 2^32"); return FIRA_ERR_INVALID_ARG; }
    if (!(eps >= 0.f) || isinf(eps)) { set_error(who + ": eps must be >= 0"); return FIRA_ERR_INVALID_ARG; }
    const bool rms = mean_dev == nullptr;
    if (rms && bias_dev) { set_error(who + ": the form without mean has no bias"); return FIRA_ERR_INVALID_ARG; }
    if (nrows == 0) return FIRA_OK;
    const size_t es = dtype == FIRA_BF16 ? 2 : 4, ps = param_dtype == FIRA_BF16 ? 2 : 4;
    if (off(x_dev, es) || off(y_dev, es) || off(gain_dev, ps) || (bias_dev && off(bias_dev, ps)) || off(rstd_dev, 4) || (!rms && off(mean_dev, 4))) {
      set_error(who + ": pointers must be non-null and aligned to their elements"); return FIRA_ERR_INVALID_ARG;
    }
    const RowPlan p = rows_of(hidden, es, mode_of(x_dev, ld_x, hidden, es, alike(x_dev, ld_x, y_dev, ld_y, es)));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
#define LN_FORWARD(T, W, B, R) e = run_forward<T, W, B, R>(p, x_dev, ld_x, nrows, (int)hidden, gain_dev, bias_dev, param_dtype == FIRA_BF16, eps, y_dev, ld_y, mean_dev, rstd_dev, st)
    LN_DISPATCH(LN_FORWARD);
#undef LN_FORWARD
    if (e != cudaSuccess) { set_error(who + ": " + cudaGetErrorString(e)); return FIRA_ERR_CUDA; }
    return FIRA_OK;
  });
}

extern "C" size_t fira_layer_norm_grad_work_bytes(int64_t nrows, int64_t hidden, fira_dtype dtype) {
  if (nrows < 0 || hidden <= 0 || hidden > LN_MAX_HIDDEN) return 0;
  const size_t es = dtype == FIRA_BF16 ? 2 : 4;
  int blocks = 0;                           // however the rows will begin
  for (const Mode mode : {SINGLE, SHIFTED, ALIGNED})
    for (const bool rms : {false, true}) blocks = std::max(blocks, grad_blocks(rows_of(hidden, es, mode), nrows, rms, es));
  return align_up((size_t)blocks * 2 * hidden * sizeof(float));
}

extern "C" fira_status fira_layer_norm_grad(const void* dY_dev, int64_t ld_dy, const void* x_dev, int64_t ld_x, fira_dtype dtype,
                                            int64_t nrows, int64_t hidden, const void* gain_dev, fira_dtype param_dtype,
                                            const float* mean_dev, const float* rstd_dev, void* dX_dev, int64_t ld_dx,
                                            void* dgain_dev, void* dbias_dev, fira_dtype grad_dtype, int32_t accumulate,
                                            void* work_dev, size_t work_bytes, void* cuda_stream) {
  return guarded([&]() -> fira_status {
    const std::string who("fira_layer_norm_grad");
    const fira_status bad = check_norm(who, nrows, hidden, dtype, param_dtype);
    if (bad != FIRA_OK) return bad;
    if (grad_dtype != FIRA_F32 && grad_dtype != FIRA_BF16) { set_error(who + ": unknown dtype"); return FIRA_ERR_INVALID_ARG; }
    if (bad_ld(ld_dy, hidden) || bad_ld(ld_x, hidden) || bad_ld(ld_dx, hidden)) { set_error(who + ": ld below the width, or above 2^32"); return FIRA_ERR_INVALID_ARG; }
    const bool rms = mean_dev == nullptr;
    if (rms && dbias_dev) { set_error(who + ": the form without mean has no bias"); return FIRA_ERR_INVALID_ARG; }
    const size_t es = dtype == FIRA_BF16 ? 2 : 4, ps = param_dtype == FIRA_BF16 ? 2 : 4, gs = grad_dtype == FIRA_BF16 ? 2 : 4;
    if (off(dgain_dev, gs) || (dbias_dev && off(dbias_dev, gs)) || off(work_dev, 256) ||
        (nrows > 0 && (off(dY_dev, es) || off(x_dev, es) || off(dX_dev, es) || off(gain_dev, ps) || off(rstd_dev, 4) || (!rms && off(mean_dev, 4))))) {
      set_error(who + ": pointers must be non-null and aligned to their elements (work: 256 bytes)"); return FIRA_ERR_INVALID_ARG;
    }
    const size_t need = fira_layer_norm_grad_work_bytes(nrows, hidden, dtype);
    if (work_bytes < need) {
      set_error(who + ": workspace too small: " + std::to_string(work_bytes) + " bytes, " + std::to_string(need) + " needed");
      return FIRA_ERR_WORKSPACE_TOO_SMALL;
    }
    const RowPlan p = rows_of(hidden, es, mode_of(x_dev, ld_x, hidden, es, alike(dY_dev, ld_dy, x_dev, ld_x, es) && alike(dY_dev, ld_dy, dX_dev, ld_dx, es)));
    const int want_bias = dbias_dev != nullptr;
    float* parts = static_cast<float*>(work_dev);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
#define LN_BACKWARD(T, W, B, R) e = run_backward<T, W, B, R>(p, dY_dev, ld_dy, x_dev, ld_x, nrows, (int)hidden, gain_dev, param_dtype == FIRA_BF16, mean_dev, rstd_dev, dX_dev, ld_dx, parts, want_bias, st)
    LN_DISPATCH(LN_BACKWARD);
#undef LN_BACKWARD
    const int width = (int)hidden * (want_bias ? 2 : 1);
    if (e == cudaSuccess)
      e = launch_chained(k_layer_norm_params, dim3((width + 31) / 32), 1024, 0, st, true, 1, (const float*)parts, grad_blocks(p, nrows, rms, es), width,
                         (int)hidden, dgain_dev, dbias_dev, grad_dtype == FIRA_BF16 ? 1 : 0, accumulate != 0 ? 1 : 0);
    if (e != cudaSuccess) { set_error(who + ": " + cudaGetErrorString(e)); return FIRA_ERR_CUDA; }
    return FIRA_OK;
  });
}
