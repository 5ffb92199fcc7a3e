// Layer norm, forward and backward, with the form without mean and bias (RMS).
//
//   y = (x - mu) s g + b,   mu = mean(x) (RMS: 0),   s = 1 / sqrt(mean((x - mu)^2) + eps)
//   with h = (x - mu) s, q = dy g:   dx = s (q - mean(q) - h mean(q h))   (RMS: without mean(q))
//   dg = sum over rows of dy h,   db = sum over rows of dy
//
// A group of 32 to 1024 threads takes a row, each thread PIECES pieces of 16 bytes of it, which stay in registers
// (as they were read) from the load to the store; the next row is on its way meanwhile.  Statistics are fp32, the
// variance from the differences to the mean.  In the backward pass a thread has the same columns in every row of its
// group, so that dg and db grow in its registers; the groups of a block are added in shared memory, the blocks in a second
// launch, always in the same order.
#include <math.h>

#include <algorithm>

#include "rows.cuh"
#include "tc_ptx.cuh"

namespace fira {
namespace {

constexpr int LN_THREADS = 256;             // of a block, where a row takes no more
constexpr int LN_MAX_HIDDEN = 16384;
constexpr int LN_SMS = 148;

// The threads of a row, and this thread's place.
struct Group {
  int threads, id, rank, count;             // id of count groups in the block
  __device__ __forceinline__ explicit Group(int per_row) : threads(per_row), id(threadIdx.x / per_row), rank(threadIdx.x % per_row), count(blockDim.x / per_row) {}
};

// (LN_THREADS is four groups of two warps at most.)
__device__ __forceinline__ void group_barrier(const Group& g) {
  if (g.count == 1) __syncthreads();
  else if (g.id == 0) asm volatile("bar.sync 1, %0;" :: "r"(g.threads) : "memory");
  else if (g.id == 1) asm volatile("bar.sync 2, %0;" :: "r"(g.threads) : "memory");
  else if (g.id == 2) asm volatile("bar.sync 3, %0;" :: "r"(g.threads) : "memory");
  else asm volatile("bar.sync 4, %0;" :: "r"(g.threads) : "memory");
}

// Sums over the group of two values of each thread.  Calls use the two buffers in turn, so that one barrier is enough.
__device__ __forceinline__ float2 group_sum(float2 v, const Group& g, float2 (*red)[32], int& turn) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if (g.threads == 32) return v;
  const int lane = threadIdx.x & 31, warps = g.threads >> 5, first = g.id * warps;
  if (lane == 0) red[turn][threadIdx.x >> 5] = v;
  group_barrier(g);
  v = lane < warps ? red[turn][first + lane] : make_float2(0.f, 0.f);
  turn ^= 1;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  return v;
}

// The pieces of a row that a thread has: N elements each, next to one another where rows are read in 16-byte accesses,
// one per thread in turn otherwise.
template <typename T, bool VECTOR, int PIECES>
struct Cols {
  static constexpr int N = rows::PER16<T>;
  int rank, threads, hidden;
  __device__ __forceinline__ int at(int p, int e) const { return VECTOR ? (p * threads + rank) * N + e : (p * N + e) * threads + rank; }
  __device__ __forceinline__ bool in(int p, int e) const { return at(p, VECTOR ? 0 : e) < hidden; }
  __device__ __forceinline__ void load(const T* row, uint4 (&r)[PIECES]) const {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      r[p] = make_uint4(0u, 0u, 0u, 0u);
      if (VECTOR) {
        if (in(p, 0)) r[p] = *reinterpret_cast<const uint4*>(row + at(p, 0));
      } else {
        T* v = reinterpret_cast<T*>(&r[p]);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (in(p, e)) v[e] = row[at(p, e)];
      }
    }
  }
  __device__ __forceinline__ void store(T* row, int p, const float (&v)[N]) const {
    if (VECTOR) {
      if (in(p, 0)) rows::store_vec<T, N>(row + at(p, 0), v);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (in(p, e)) row[at(p, e)] = from_float<T>(v[e]);
    }
  }
  // Gains and biases, of either type.
  __device__ __forceinline__ void params(const void* q, int bf16, float (&v)[PIECES][N]) const {
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int e = 0; e < N; ++e)
        v[p][e] = !q || !in(p, e) ? 0.f : bf16 ? to_float(static_cast<const __nv_bfloat16*>(q)[at(p, e)]) : static_cast<const float*>(q)[at(p, e)];
  }
};

template <typename T, bool VECTOR, int PIECES, bool RMS>
__global__ void __launch_bounds__(PIECES > 2 && sizeof(T) == 4 ? 1024 : 512)
k_layer_norm(const T* x, long long ld_x, long long nrows, int hidden, int per_row, const void* gain, const void* bias, int param_bf16, float eps,
             T* y, long long ld_y, float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int N = rows::PER16<T>;
  __shared__ float2 red[2][32];
  const Group g(per_row);
  const Cols<T, VECTOR, PIECES> cols{g.rank, per_row, hidden};
  const long long stride = (long long)gridDim.x * g.count;
  long long row = (long long)blockIdx.x * g.count + g.id;
  if (row >= nrows) return;                 // a whole group: its barrier is its own
  uint4 raw[PIECES], next[PIECES];
  cols.load(x + row * ld_x, raw);
  float w[PIECES][N], b[PIECES][N];
  cols.params(gain, param_bf16, w);
  cols.params(bias, param_bf16, b);
  const float inv = 1.f / (float)hidden;
  int turn = 0;
  for (;;) {
    const bool more = row + stride < nrows;
    if (more) cols.load(x + (row + stride) * ld_x, next);
    float mu = 0.f;
    float2 s = make_float2(0.f, 0.f);
    if (!RMS) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        float v[N];
        rows::unpack<T>(raw[p], v);
#pragma unroll
        for (int e = 0; e < N; ++e) s.x += v[e];
      }
      mu = group_sum(s, g, red, turn).x * inv;
      s.x = 0.f;
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      float v[N];
      rows::unpack<T>(raw[p], v);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (RMS) s.x = fmaf(v[e], v[e], s.x);
        else if (cols.in(p, e)) s.x = fmaf(v[e] - mu, v[e] - mu, s.x);
    }
    const float rs = 1.f / sqrtf(group_sum(s, g, red, turn).x * inv + eps);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      float v[N];
      rows::unpack<T>(raw[p], v);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = RMS ? v[e] * rs * w[p][e] : fmaf((v[e] - mu) * rs, w[p][e], b[p][e]);
      cols.store(y + row * ld_y, p, v);
    }
    if (g.rank == 0) {
      rstd[row] = rs;
      if (!RMS) mean[row] = mu;
    }
    if (!more) return;
    row += stride;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) raw[p] = next[p];
  }
}

// parts: per block the sums of dy h, then those of dy, `hidden` floats each.
template <typename T, bool VECTOR, int PIECES, bool RMS>
__global__ void __launch_bounds__(PIECES > 2 && sizeof(T) == 4 ? 1024 : 512)
k_layer_norm_grad(const T* dy, long long ld_dy, const T* x, long long ld_x, long long nrows, int hidden, int per_row, const void* gain,
                  int param_bf16, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, long long ld_dx,
                  float* __restrict__ parts, int want_bias) {
  constexpr int N = rows::PER16<T>;
  extern __shared__ float sums[];           // [2 or 1][hidden]
  __shared__ float2 red[2][32];
  ptx::grid_launch_next();
  const Group g(per_row);
  const Cols<T, VECTOR, PIECES> cols{g.rank, per_row, hidden};
  const long long stride = (long long)gridDim.x * g.count;
  long long row = (long long)blockIdx.x * g.count + g.id;
  float w[PIECES][N], dg[PIECES][N], db[PIECES][N];
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int e = 0; e < N; ++e) dg[p][e] = db[p][e] = 0.f;
  if (row < nrows) {
    uint4 rx[PIECES], ry[PIECES], nx[PIECES], ny[PIECES];
    cols.load(x + row * ld_x, rx);
    cols.load(dy + row * ld_dy, ry);
    float rs = rstd[row], mu = RMS ? 0.f : mean[row];
    cols.params(gain, param_bf16, w);
    const float inv = 1.f / (float)hidden;
    int turn = 0;
    for (;;) {
      const bool more = row + stride < nrows;
      float next_rs = 0.f, next_mu = 0.f;
      if (more) {
        cols.load(x + (row + stride) * ld_x, nx);
        cols.load(dy + (row + stride) * ld_dy, ny);
        next_rs = rstd[row + stride];
        if (!RMS) next_mu = mean[row + stride];
      }
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        float a[N], d[N];
        rows::unpack<T>(rx[p], a);
        rows::unpack<T>(ry[p], d);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float h = RMS ? a[e] * rs : (a[e] - mu) * rs, q = d[e] * w[p][e];
          s.x = fmaf(q, h, s.x);
          if (!RMS) s.y += q;
          dg[p][e] = fmaf(d[e], h, dg[p][e]);
          if (!RMS) db[p][e] += d[e];
        }
      }
      s = group_sum(s, g, red, turn);
      const float along = s.x * inv, level = s.y * inv;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        float a[N], d[N];
        rows::unpack<T>(rx[p], a);
        rows::unpack<T>(ry[p], d);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float h = RMS ? a[e] * rs : (a[e] - mu) * rs, q = d[e] * w[p][e];
          a[e] = rs * fmaf(-h, along, RMS ? q : q - level);
        }
        cols.store(dx + row * ld_dx, p, a);
      }
      if (!more) break;
      row += stride;
      rs = next_rs; mu = next_mu;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) { rx[p] = nx[p]; ry[p] = ny[p]; }
    }
  }
  // the groups one after another
  for (int k = 0; k < g.count; ++k) {
    if (g.id == k) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          if (!cols.in(p, e)) continue;
          const int c = cols.at(p, e);
          float u = dg[p][e], v = db[p][e];
          if (k > 0) { u += sums[c]; if (want_bias) v += sums[hidden + c]; }
          if (k + 1 < g.count) {
            sums[c] = u;
            if (want_bias) sums[hidden + c] = v;
          } else {
            float* out = parts + (long long)blockIdx.x * hidden * (want_bias ? 2 : 1);
            out[c] = u;
            if (want_bias) out[hidden + c] = v;
          }
        }
    }
    if (g.count > 1) __syncthreads();
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
#pragma unroll 4
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

// Threads of a row: as few as hold it at two pieces each, at least a warp; beyond 512 of them, four pieces each.
int threads_per_row(long long hidden, int dtype) {
  const int n = dtype == FIRA_BF16 ? 8 : 4;
  int t = 32;
  while (t < 512 && (long long)t * 2 * n < hidden) t *= 2;
  return (long long)t * 4 * n < hidden ? 1024 : t;
}
bool four_pieces(long long hidden, int dtype) { return hidden > 512 * 2 * (dtype == FIRA_BF16 ? 8 : 4); }
int block_threads(int per_row) { return std::max(LN_THREADS, per_row); }
// Blocks of the backward pass: each writes its sums of dg and db once, so a group has eight rows at least before
// there are more.
int grad_blocks(long long nrows, int per_row) {
  const long long groups = block_threads(per_row) / per_row;
  const long long most = per_row > 512 ? LN_SMS : per_row > 256 ? 2 * LN_SMS : 3 * LN_SMS;
  return (int)std::max<long long>(1, std::min(most, (nrows + 8 * groups - 1) / (8 * groups)));
}

template <typename T, bool VECTOR, int PIECES, bool RMS>
void run_forward(const void* x, long long ld_x, long long nrows, int hidden, int per_row, const void* gain, const void* bias, int param_bf16, float eps,
                 void* y, long long ld_y, float* mean, float* rstd, cudaStream_t st) {
  const int threads = block_threads(per_row), groups = threads / per_row;
  const unsigned blocks = (unsigned)std::min<long long>((nrows + groups - 1) / groups, LN_SMS * 6);
  k_layer_norm<T, VECTOR, PIECES, RMS><<<blocks, threads, 0, st>>>((const T*)x, ld_x, nrows, hidden, per_row, gain, bias, param_bf16, eps, (T*)y, ld_y, mean, rstd);
}
template <typename T, bool VECTOR, int PIECES, bool RMS>
cudaError_t run_backward(const void* dy, long long ld_dy, const void* x, long long ld_x, long long nrows, int hidden, int per_row, const void* gain,
                         int param_bf16, const float* mean, const float* rstd, void* dx, long long ld_dx, float* parts, int want_bias, cudaStream_t st) {
  const int threads = block_threads(per_row), groups = threads / per_row;
  const size_t smem = groups > 1 ? (size_t)hidden * (want_bias ? 2 : 1) * sizeof(float) : 0;
  k_layer_norm_grad<T, VECTOR, PIECES, RMS><<<grad_blocks(nrows, per_row), threads, smem, st>>>(
      (const T*)dy, ld_dy, (const T*)x, ld_x, nrows, hidden, per_row, gain, param_bf16, mean, rstd, (T*)dx, ld_dx, parts, want_bias);
  return cudaGetLastError();
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

#define LN_DISPATCH_PIECES(CALL, T, P)                                                                                  \
  do {                                                                                                                  \
    if (vector) { if (rms) CALL(T, true, P, true); else CALL(T, true, P, false); }                                      \
    else        { if (rms) CALL(T, false, P, true); else CALL(T, false, P, false); }                                    \
  } while (0)
#define LN_DISPATCH(CALL)                                                                                               \
  do {                                                                                                                  \
    const bool four = four_pieces(hidden, dtype);                                                                       \
    if (dtype == FIRA_BF16) { if (four) LN_DISPATCH_PIECES(CALL, __nv_bfloat16, 4); else LN_DISPATCH_PIECES(CALL, __nv_bfloat16, 2); } \
    else { if (four) LN_DISPATCH_PIECES(CALL, float, 4); else LN_DISPATCH_PIECES(CALL, float, 2); }                     \
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
    const bool vector = rows::aligned16(x_dev, ld_x, hidden, es) && rows::aligned16(y_dev, ld_y, hidden, es);
    const int per_row = threads_per_row(hidden, dtype);
    cudaStream_t st = (cudaStream_t)cuda_stream;
#define LN_FORWARD(T, V, P, R) run_forward<T, V, P, R>(x_dev, ld_x, nrows, (int)hidden, per_row, gain_dev, bias_dev, param_dtype == FIRA_BF16, eps, y_dev, ld_y, mean_dev, rstd_dev, st)
    LN_DISPATCH(LN_FORWARD);
#undef LN_FORWARD
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { set_error(who + ": " + cudaGetErrorString(e)); return FIRA_ERR_CUDA; }
    return FIRA_OK;
  });
}

extern "C" size_t fira_layer_norm_grad_work_bytes(int64_t nrows, int64_t hidden, fira_dtype dtype) {
  if (nrows < 0 || hidden <= 0 || hidden > LN_MAX_HIDDEN) return 0;
  return align_up((size_t)grad_blocks(nrows, threads_per_row(hidden, dtype)) * 2 * hidden * sizeof(float));
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
    const bool vector = rows::aligned16(dY_dev, ld_dy, hidden, es) && rows::aligned16(x_dev, ld_x, hidden, es) && rows::aligned16(dX_dev, ld_dx, hidden, es);
    const int per_row = threads_per_row(hidden, dtype), want_bias = dbias_dev != nullptr;
    float* parts = static_cast<float*>(work_dev);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
#define LN_BACKWARD(T, V, P, R) e = run_backward<T, V, P, R>(dY_dev, ld_dy, x_dev, ld_x, nrows, (int)hidden, per_row, gain_dev, param_dtype == FIRA_BF16, mean_dev, rstd_dev, dX_dev, ld_dx, parts, want_bias, st)
    LN_DISPATCH(LN_BACKWARD);
#undef LN_BACKWARD
    const int width = (int)hidden * (want_bias ? 2 : 1);
    if (e == cudaSuccess)
      e = launch_chained(k_layer_norm_params, dim3((width + 31) / 32), 1024, 0, st, true, 1, (const float*)parts, grad_blocks(nrows, per_row), width,
                         (int)hidden, dgain_dev, dbias_dev, grad_dtype == FIRA_BF16 ? 1 : 0, accumulate != 0 ? 1 : 0);
    if (e != cudaSuccess) { set_error(who + ": " + cudaGetErrorString(e)); return FIRA_ERR_CUDA; }
    return FIRA_OK;
  });
}
