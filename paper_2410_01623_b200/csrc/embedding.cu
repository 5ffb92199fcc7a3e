// Rows of an embedding table, and the table's gradient.
//
//   Y_i = a E[t_i]                         (t_i outside 0 .. vocab-1: a row of zeros)
//   dE_v = a sum over {i : t_i = v} of dY_i
//
// The gradient takes two launches.  k_token_order sorts the positions by token: each block owns a range of tokens and
// reads all tokens of the batch (they stay in L2: 148 blocks x 512 KB at 131072 tokens), counts those below its range,
// which is where its own positions begin in the sorted order, and those of each row of its range, and then stores
// its positions.  No block waits for another, and the order is the same in every call.
// k_table_grad sums: a warp takes T sorted positions and a slice of columns, whole rows of the table where a row has
// at most T positions (the warp in whose range it begins does all of it).  A row with more, as words at the top of a
// Zipf law have, is cut at the multiples of T; the parts are stored, and the warp that comes last, by a counter, adds them
// in their order.  Rows without a token are zeroed by warps of the same launch.  Sums are fp32, rounded once.
#include <math.h>

#include <algorithm>

#include "rows.cuh"
#include "tc_ptx.cuh"

namespace fira {
namespace {

constexpr int EM_THREADS = 256;
constexpr int EM_WARPS = EM_THREADS / 32;
constexpr int EM_SMS = 148;

// ------------------------------------------------------------------------------------------------ lookup
constexpr int LK_ROWS = 4;                 // rows of a warp in flight

template <typename TOK>
__device__ __forceinline__ int token_at(const TOK* tokens, long long i, int vocab) {
  const long long t = (long long)tokens[i];
  return t >= 0 && t < vocab ? (int)t : -1;
}

// A warp takes LK_ROWS positions and a slice of the columns.
template <typename T, typename TOK, bool VECTOR>
__global__ void __launch_bounds__(EM_THREADS)
k_embedding(const T* __restrict__ table, long long ld, const TOK* __restrict__ tokens, long long n, int vocab, int hidden, int slices,
            float scale, T* __restrict__ out, long long ld_out) {
  constexpr int N = rows::PER16<T>;
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * EM_WARPS + (threadIdx.x >> 5);
  const long long i0 = unit / slices * LK_ROWS;
  const int col0 = (int)(unit % slices) * 32 * N;
  if (i0 >= n) return;
  int t[LK_ROWS];
#pragma unroll
  for (int u = 0; u < LK_ROWS; ++u) t[u] = i0 + u < n ? token_at(tokens, i0 + u, vocab) : -1;
  if (VECTOR) {
    const int col = col0 + lane * N;
    if (col >= hidden) return;
    float v[LK_ROWS][N];
#pragma unroll
    for (int u = 0; u < LK_ROWS; ++u) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[u][e] = 0.f;
      if (t[u] >= 0) rows::load_vec<T, N>(table + (long long)t[u] * ld + col, v[u]);
    }
#pragma unroll
    for (int u = 0; u < LK_ROWS; ++u) {
      if (i0 + u >= n) break;
#pragma unroll
      for (int e = 0; e < N; ++e) v[u][e] *= scale;
      rows::store_vec<T, N>(out + (i0 + u) * ld_out + col, v[u]);
    }
  } else {
#pragma unroll
    for (int u = 0; u < LK_ROWS; ++u) {
      if (i0 + u >= n) break;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int col = col0 + e * 32 + lane;
        if (col < hidden) out[(i0 + u) * ld_out + col] = from_float<T>(t[u] >= 0 ? scale * to_float<T>(table[(long long)t[u] * ld + col]) : 0.f);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ order of the tokens
constexpr int ORD_THREADS = 1024;
constexpr int ORD_WARPS = ORD_THREADS / 32;
constexpr int ORD_MAX_ROWS = 1024;          // rows of a block's range: a thread each, and 128 KB of counts
constexpr int ORD_STEP = 128;               // tokens of a warp's step: four per lane

// Four tokens from position i on (-1 behind the end and where a token is none of the table's).
template <typename TOK, bool VECTOR>
__device__ __forceinline__ void load_tokens(const TOK* __restrict__ tokens, int i, int n, int vocab, int (&t)[4]) {
  long long x[4] = {-1, -1, -1, -1};
  if (VECTOR && i + 4 <= n) {
    if constexpr (sizeof(TOK) == 4) {
      const int4 u = *reinterpret_cast<const int4*>(tokens + i);
      x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
    } else {
      const longlong2 a = reinterpret_cast<const longlong2*>(tokens + i)[0], b = reinterpret_cast<const longlong2*>(tokens + i)[1];
      x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) if (i + j < n) x[j] = (long long)tokens[i + j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) t[j] = x[j] >= 0 && x[j] < vocab ? (int)x[j] : -1;
}

__device__ __forceinline__ unsigned warp_inclusive(unsigned x) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) >= o) x += y;
  }
  return x;
}

// order: (position, token) sorted by token; start[v]: where row v begins, start[vocab]: tokens of the table in the batch.
// Among equal tokens the order goes by warp (a stretch of positions each), step, place in the lane's four, lane.
template <typename TOK, bool VECTOR>
__global__ void __launch_bounds__(ORD_THREADS)
k_token_order(const TOK* __restrict__ tokens, int n, int vocab, int range, int2* __restrict__ order, int* __restrict__ start,
              unsigned* __restrict__ counters, long long ncounters) {
  extern __shared__ unsigned cnt[];         // [ORD_WARPS][range]
  __shared__ unsigned below_s[ORD_WARPS], sum_s[ORD_WARPS];
  ptx::grid_launch_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int v0 = blockIdx.x * range;        // (grid: ceil(vocab / range) blocks, so v0 < vocab)
  const unsigned here = (unsigned)min(range, vocab - v0);
  for (long long i = (long long)blockIdx.x * ORD_THREADS + threadIdx.x; i < ncounters; i += (long long)gridDim.x * ORD_THREADS) counters[i] = 0;
  for (int i = threadIdx.x; i < ORD_WARPS * range; i += ORD_THREADS) cnt[i] = 0;
  __syncthreads();
  unsigned* mine = cnt + warp * range;
  const int steps = (n + ORD_STEP - 1) / ORD_STEP, per_warp = (steps + ORD_WARPS - 1) / ORD_WARPS;
  const int s0 = min(steps, warp * per_warp), s1 = min(steps, s0 + per_warp);
  unsigned below = 0;
#pragma unroll 4
  for (int s = s0; s < s1; ++s) {
    int t[4];
    load_tokens<TOK, VECTOR>(tokens, s * ORD_STEP + lane * 4, n, vocab, t);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      below += (unsigned)t[j] < (unsigned)v0;
      const unsigned r = (unsigned)t[j] - (unsigned)v0;
      if (r < here) atomicAdd(&mine[r], 1u);
    }
  }
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) below_s[warp] = below;
  __syncthreads();
  below = __reduce_add_sync(0xffffffffu, below_s[lane]);
  const unsigned r = threadIdx.x;
  unsigned total = 0;
  if (r < here)
    for (int w = 0; w < ORD_WARPS; ++w) {
      const unsigned c = cnt[w * range + r];
      cnt[w * range + r] = total;
      total += c;
    }
  const unsigned inclusive = warp_inclusive(total);
  if (lane == 31) sum_s[warp] = inclusive;
  __syncthreads();
  const unsigned sums = warp_inclusive(sum_s[lane]);
  const unsigned in_front = __shfl_sync(0xffffffffu, sums, max(warp - 1, 0));
  const unsigned front = below + (warp ? in_front : 0u) + inclusive - total;
  if (r < here) {
    start[v0 + r] = (int)front;
    if (v0 + (int)r == vocab - 1) start[vocab] = (int)(front + total);
    for (int w = 0; w < ORD_WARPS; ++w) cnt[w * range + r] += front;
  }
  __syncthreads();
#pragma unroll 2
  for (int s = s0; s < s1; ++s) {
    int t[4];
    const int i = s * ORD_STEP + lane * 4;
    load_tokens<TOK, VECTOR>(tokens, i, n, vocab, t);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned k = (unsigned)t[j] - (unsigned)v0;
      const bool in = k < here;
      if (__any_sync(0xffffffffu, in)) {
        const unsigned same = __match_any_sync(0xffffffffu, in ? k : 0x80000000u | lane);
        const unsigned at = in ? mine[k] : 0u;
        __syncwarp();
        if (in) {
          order[at + __popc(same & ((1u << lane) - 1))] = make_int2(i + j, t[j]);
          if (lane == __ffs(same) - 1) mine[k] = at + __popc(same);
        }
        __syncwarp();
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ sums of the rows
constexpr int TG_UNROLL = 8;                // rows of dY in flight
constexpr int TG_ZERO_ROWS = 16;            // rows that a warp looks over for tokens

struct TablePlan {
  int range, blocks;                        // k_token_order
  int T;                                    // sorted positions of a warp
  long long chunks;
  int slices;
  size_t off_start, off_counters, off_parts, bytes;
};

template <typename TI, typename TO, bool VECTOR>
struct Slice {
  static constexpr int N = rows::PER16<TI>;
  int col0, lane, hidden;
  struct alignas(16) Piece { TI v[N]; };                // as it was read: 16 bytes, converted where it is added
  __device__ __forceinline__ void load(const TI* row, Piece& p) const {
    if (VECTOR) {
      if (col0 + lane * N < hidden) *reinterpret_cast<uint4*>(&p) = *reinterpret_cast<const uint4*>(row + col0 + lane * N);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int c = col0 + e * 32 + lane;
        if (c < hidden) p.v[e] = row[c];
      }
    }
  }
  __device__ __forceinline__ void add(const Piece& p, float (&sum)[N]) const {
    float v[N];
    rows::unpack<TI>(*reinterpret_cast<const uint4*>(&p), v);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] += v[e];
  }
  __device__ __forceinline__ void store(TO* row, float (&v)[N], float scale, bool add) const {
    if (VECTOR) {
      if (col0 + lane * N >= hidden) return;
      TO* p = row + col0 + lane * N;
      if constexpr (N * sizeof(TO) % 16 == 0) {
        float old[N];
        if (add) rows::load_vec<TO, N>(p, old);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = add ? fmaf(scale, v[e], old[e]) : scale * v[e];
        rows::store_vec<TO, N>(p, v);
      } else {                              // fp32 rows into bf16: 8 bytes
        static_assert(N == 4 && sizeof(TO) == 2, "");
        uint2* q = reinterpret_cast<uint2*>(p);
        float old[4] = {0.f, 0.f, 0.f, 0.f};
        if (add) {
          const uint2 u = *q;
          old[0] = __uint_as_float(u.x << 16); old[1] = __uint_as_float(u.x & 0xffff0000u);
          old[2] = __uint_as_float(u.y << 16); old[3] = __uint_as_float(u.y & 0xffff0000u);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = add ? fmaf(scale, v[e], old[e]) : scale * v[e];
        const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
        *q = make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int c = col0 + e * 32 + lane;
        if (c < hidden) row[c] = from_float<TO>(add ? fmaf(scale, v[e], to_float<TO>(row[c])) : scale * v[e]);
      }
    }
  }
  // A part of a long row: 32 N floats, of which a lane keeps its own.
  __device__ __forceinline__ void store_part(float* p, const float (&v)[N]) const {
#pragma unroll
    for (int e = 0; e < N; e += 4) __stcg(reinterpret_cast<float4*>(p + e * 32) + lane, make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]));
  }
  __device__ __forceinline__ void add_part(const float* p, float (&v)[N]) const {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      const float4 u = __ldcg(reinterpret_cast<const float4*>(p + e * 32) + lane);
      v[e] += u.x; v[e + 1] += u.y; v[e + 2] += u.z; v[e + 3] += u.w;
    }
  }
};

template <typename TI, typename TO, bool VECTOR>
__global__ void __launch_bounds__(EM_THREADS)
k_table_grad(const int2* order, const int* start, unsigned* counters, float* parts,
             const TI* __restrict__ dY, long long ld, int vocab, int hidden, int T, long long chunks, int slices, float scale, int add,
             TO* __restrict__ G, long long ldg) {
  constexpr int N = rows::PER16<TI>;
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * EM_WARPS + (threadIdx.x >> 5);
  ptx::grid_wait();
  if (unit >= chunks * slices) {            // rows that no token names
    const long long first = (unit - chunks * slices) * TG_ZERO_ROWS;
    if (add || first >= vocab) return;     // (the last block has warps to spare)
    const int here = (int)min((long long)TG_ZERO_ROWS, vocab - first);
    const int s = lane <= here ? start[first + lane] : 0;
    const int next = __shfl_down_sync(0xffffffffu, s, 1);     // (by all lanes)
    const unsigned empty = __ballot_sync(0xffffffffu, lane < here && s == next);
    for (int k = 0; k < here; ++k) {
      if (!(empty >> k & 1)) continue;
      TO* row = G + (first + k) * ldg;
      if (VECTOR) {
        const int bytes = hidden * (int)sizeof(TO);     // a multiple of 8
        for (int b = lane * 8; b < bytes; b += 256) *reinterpret_cast<uint2*>(reinterpret_cast<char*>(row) + b) = make_uint2(0u, 0u);
      } else {
        for (int c = lane; c < hidden; c += 32) row[c] = from_float<TO>(0.f);
      }
    }
    return;
  }
  const long long chunk = unit / slices;
  const int slice = (int)(unit % slices);
  const int n = start[vocab];
  const long long p0 = chunk * T;
  if (p0 >= n) return;
  const int a0 = (int)p0, p1 = (int)min(p0 + T, (long long)n);
  const int v_first = order[a0].y, v_last = order[p1 - 1].y;
  const int first_s = start[v_first], first_e = start[v_first + 1], last_s = start[v_last], last_e = start[v_last + 1];
  const bool first_long = first_e - first_s > T, last_long = last_e - last_s > T;
  const int a = !first_long && first_s < a0 ? first_e : a0, b = last_long ? p1 : last_e;
  if (a >= b) return;
  Slice<TI, TO, VECTOR> at;
  at.col0 = slice * 32 * N; at.lane = lane; at.hidden = hidden;

  float sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
  // Row v is done, or this warp's part of it.
  auto flush = [&](int v) {
    if (!((first_long && v == v_first) || (last_long && v == v_last))) {
      at.store(G + v * ldg, sum, scale, add);
    } else {
      const int s = v == v_first ? first_s : last_s, e = v == v_first ? first_e : last_e;
      const long long c0 = s / T, c1 = (e - 1) / T;
      // two long rows may meet in a chunk: the one that begins there has the second place
      auto part = [&](long long c) { return parts + ((2 * c + (c == c0 ? 1 : 0)) * slices + slice) * (32 * N); };
      at.store_part(part(chunk), sum);
      __threadfence();
      __syncwarp();
      unsigned before = 0;
      if (lane == 0) before = atomicAdd(&counters[c0 * slices + slice], 1u);
      before = __shfl_sync(0xffffffffu, before, 0);
      if (before == (unsigned)(c1 - c0)) {  // all parts are there
        __threadfence();
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] = 0.f;
#pragma unroll 4
        for (long long c = c0; c <= c1; ++c) at.add_part(part(c), sum);
        at.store(G + v * ldg, sum, scale, add);
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.f;
  };
  int current = order[a].y;
  for (int q = a; q < b; q += 32) {
    const int2 entry = q + lane < b ? order[q + lane] : make_int2(0, 0);
    const int m = min(32, b - q);
    for (int k = 0; k < m; k += TG_UNROLL) {
      typename Slice<TI, TO, VECTOR>::Piece v[TG_UNROLL];
#pragma unroll
      for (int u = 0; u < TG_UNROLL; ++u) {
        *reinterpret_cast<uint4*>(&v[u]) = make_uint4(0u, 0u, 0u, 0u);
        const int i = __shfl_sync(0xffffffffu, entry.x, (k + u) & 31);
        if (k + u < m) at.load(dY + (long long)i * ld, v[u]);
      }
#pragma unroll
      for (int u = 0; u < TG_UNROLL; ++u) {
        const int t = __shfl_sync(0xffffffffu, entry.y, (k + u) & 31);
        if (k + u < m) {
          if (t != current) { flush(current); current = t; }
          at.add(v[u], sum);
        }
      }
    }
  }
  flush(current);
}

// The grid and the sections of the workspace of a gradient.
TablePlan plan_for(long long n, long long vocab, long long hidden, bool f32) {
  TablePlan p;
  p.range = (int)std::min<long long>(ORD_MAX_ROWS, std::max<long long>(32, (vocab + EM_SMS - 1) / EM_SMS));
  p.blocks = (int)((vocab + p.range - 1) / p.range);
  const long long width = 32 * (f32 ? 4 : 8);
  p.slices = (int)((hidden + width - 1) / width);
  // Few positions: short stretches, so that all SMs have warps enough; many: long ones, whose parts of long rows weigh little.
  p.T = 16;
  while (p.T < 128 && (n / (2 * p.T)) * p.slices >= EM_SMS * 32) p.T *= 2;
  p.chunks = (n + p.T - 1) / p.T;
  size_t at = align_up((size_t)n * sizeof(int2));
  p.off_start = at; at += align_up((size_t)(vocab + 1) * sizeof(int));
  p.off_counters = at; at += align_up((size_t)p.chunks * p.slices * sizeof(unsigned));
  p.off_parts = at; at += (size_t)p.chunks * 2 * p.slices * width * sizeof(float);
  p.bytes = align_up(std::max<size_t>(at, 256));
  return p;
}

constexpr long long EM_MAX_TOKENS = 1ll << 30, EM_MAX_VOCAB = 1ll << 30, EM_MAX_HIDDEN = 1ll << 24;

fira_status check_sizes(const std::string& who, int64_t count, int64_t vocab, int64_t hidden, int32_t token_bits) {
  if (count < 0 || vocab <= 0 || hidden <= 0 || count > EM_MAX_TOKENS || vocab > EM_MAX_VOCAB || hidden > EM_MAX_HIDDEN) {
    set_error(who + ": need 0 <= count <= 2^30, 1 <= vocab <= 2^30, 1 <= hidden <= 2^24"); return FIRA_ERR_INVALID_ARG;
  }
  if (token_bits != 32 && token_bits != 64) { set_error(who + ": tokens are of 32 or 64 bits"); return FIRA_ERR_INVALID_ARG; }
  return FIRA_OK;
}

template <typename T, typename TOK>
void run_lookup(const void* table, long long ld, const void* tokens, long long n, int vocab, int hidden, float scale, void* out, long long ld_out,
                cudaStream_t st) {
  const int width = 32 * rows::PER16<T>, slices = (hidden + width - 1) / width;
  const long long units = (n + LK_ROWS - 1) / LK_ROWS * slices;
  const unsigned blocks = (unsigned)((units + EM_WARPS - 1) / EM_WARPS);
  if (rows::aligned16(table, ld, hidden, sizeof(T)) && rows::aligned16(out, ld_out, hidden, sizeof(T)))
    k_embedding<T, TOK, true><<<blocks, EM_THREADS, 0, st>>>((const T*)table, ld, (const TOK*)tokens, n, vocab, hidden, slices, scale, (T*)out, ld_out);
  else
    k_embedding<T, TOK, false><<<blocks, EM_THREADS, 0, st>>>((const T*)table, ld, (const TOK*)tokens, n, vocab, hidden, slices, scale, (T*)out, ld_out);
}

// The counts of a block's range are above the default limit of shared memory: a setting per device and kernel.
template <typename TOK, bool VECTOR>
cudaError_t run_order(const TablePlan& p, const void* tokens, int n, int vocab, char* work, cudaStream_t st) {
  const size_t smem = (size_t)ORD_WARPS * p.range * sizeof(unsigned);
  if (smem > 48 * 1024 - 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_token_order<TOK, VECTOR>, cudaFuncAttributeMaxDynamicSharedMemorySize, ORD_WARPS * ORD_MAX_ROWS * 4);
    if (e != cudaSuccess) return e;
  }
  k_token_order<TOK, VECTOR><<<p.blocks, ORD_THREADS, smem, st>>>((const TOK*)tokens, n, vocab, p.range, (int2*)work, (int*)(work + p.off_start),
                                                                  (unsigned*)(work + p.off_counters), p.chunks * p.slices);
  return cudaGetLastError();
}

template <typename TI, typename TO>
cudaError_t run_grad(const TablePlan& p, const void* dY, long long ld, int vocab, int hidden, float scale, int add, void* G, long long ldg, char* work,
                     bool vector, cudaStream_t st) {
  const long long units = p.chunks * p.slices + (add ? 0 : (vocab + TG_ZERO_ROWS - 1) / TG_ZERO_ROWS);
  if (units == 0) return cudaSuccess;
  const dim3 grid((unsigned)((units + EM_WARPS - 1) / EM_WARPS));
  return launch_chained(vector ? k_table_grad<TI, TO, true> : k_table_grad<TI, TO, false>, grid, EM_THREADS, 0, st, true, 1, (const int2*)work,
                        (const int*)(work + p.off_start), (unsigned*)(work + p.off_counters), (float*)(work + p.off_parts), (const TI*)dY, ld,
                        vocab, hidden, p.T, p.chunks, p.slices, scale, add, (TO*)G, ldg);
}

}  // namespace
}  // namespace fira

using namespace fira;

extern "C" fira_status fira_embedding(const void* table_dev, int64_t vocab, int64_t hidden, int64_t ld, fira_dtype dtype,
                                      const void* tokens_dev, int32_t token_bits, int64_t count, float scale, void* out_dev,
                                      int64_t ld_out, void* cuda_stream) {
  return guarded([&]() -> fira_status {
    const fira_status bad = check_sizes("fira_embedding", count, vocab, hidden, token_bits);
    if (bad != FIRA_OK) return bad;
    if (dtype != FIRA_F32 && dtype != FIRA_BF16) { set_error("fira_embedding: unknown dtype"); return FIRA_ERR_INVALID_ARG; }
    if (ld == 0) ld = hidden;
    if (ld_out == 0) ld_out = hidden;
    if (ld < hidden || ld_out < hidden || ld > (1ll << 32) || ld_out > (1ll << 32)) { set_error("fira_embedding: ld below the width, or above 2^32"); return FIRA_ERR_INVALID_ARG; }
    if (count == 0) return FIRA_OK;
    const size_t es = dtype == FIRA_BF16 ? 2 : 4;
    if (!table_dev || !tokens_dev || !out_dev || (((uintptr_t)table_dev | (uintptr_t)out_dev) & (es - 1)) || ((uintptr_t)tokens_dev & (token_bits / 8 - 1))) {
      set_error("fira_embedding: pointers must be non-null and aligned to their elements"); return FIRA_ERR_INVALID_ARG;
    }
    const long long width = 32 * (16 / (long long)es);
    if ((count + LK_ROWS - 1) / LK_ROWS * ((hidden + width - 1) / width) > 0x7fffffffll * EM_WARPS) { set_error("fira_embedding: too many elements in one call"); return FIRA_ERR_INVALID_ARG; }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == FIRA_BF16) {
      if (token_bits == 32) run_lookup<__nv_bfloat16, int>(table_dev, ld, tokens_dev, count, (int)vocab, (int)hidden, scale, out_dev, ld_out, st);
      else run_lookup<__nv_bfloat16, long long>(table_dev, ld, tokens_dev, count, (int)vocab, (int)hidden, scale, out_dev, ld_out, st);
    } else {
      if (token_bits == 32) run_lookup<float, int>(table_dev, ld, tokens_dev, count, (int)vocab, (int)hidden, scale, out_dev, ld_out, st);
      else run_lookup<float, long long>(table_dev, ld, tokens_dev, count, (int)vocab, (int)hidden, scale, out_dev, ld_out, st);
    }
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { set_error(std::string("fira_embedding: ") + cudaGetErrorString(e)); return FIRA_ERR_CUDA; }
    return FIRA_OK;
  });
}

extern "C" size_t fira_embedding_grad_work_bytes(int64_t count, int64_t vocab, int64_t hidden, fira_dtype dtype) {
  if (count < 0 || vocab <= 0 || hidden <= 0 || count > EM_MAX_TOKENS || vocab > EM_MAX_VOCAB || hidden > EM_MAX_HIDDEN) return 0;
  return plan_for(count, vocab, hidden, dtype == FIRA_F32).bytes;
}

extern "C" fira_status fira_embedding_grad(const void* tokens_dev, int32_t token_bits, int64_t count, const void* dY_dev, int64_t ld,
                                           fira_dtype dtype, int64_t vocab, int64_t hidden, float scale, void* G_dev, int64_t ldg,
                                           fira_dtype grad_dtype, int32_t accumulate, void* work_dev, size_t work_bytes,
                                           void* cuda_stream) {
  return guarded([&]() -> fira_status {
    const std::string who("fira_embedding_grad");
    const fira_status bad = check_sizes(who, count, vocab, hidden, token_bits);
    if (bad != FIRA_OK) return bad;
    if ((dtype != FIRA_F32 && dtype != FIRA_BF16) || (grad_dtype != FIRA_F32 && grad_dtype != FIRA_BF16)) { set_error(who + ": unknown dtype"); return FIRA_ERR_INVALID_ARG; }
    if (ld == 0) ld = hidden;
    if (ldg == 0) ldg = hidden;
    if (ld < hidden || ldg < hidden || ld > (1ll << 32) || ldg > (1ll << 32)) { set_error(who + ": ld below the width, or above 2^32"); return FIRA_ERR_INVALID_ARG; }
    const size_t es = dtype == FIRA_BF16 ? 2 : 4, gs = grad_dtype == FIRA_BF16 ? 2 : 4;
    if (!G_dev || ((uintptr_t)G_dev & (gs - 1)) || !work_dev || ((uintptr_t)work_dev & 255) ||
        (count > 0 && (!tokens_dev || !dY_dev || ((uintptr_t)dY_dev & (es - 1)) || ((uintptr_t)tokens_dev & (token_bits / 8 - 1))))) {
      set_error(who + ": pointers must be non-null and aligned to their elements (work: 256 bytes)"); return FIRA_ERR_INVALID_ARG;
    }
    const TablePlan p = plan_for(count, vocab, hidden, dtype == FIRA_F32);
    if (work_bytes < p.bytes) {
      set_error(who + ": workspace too small: " + std::to_string(work_bytes) + " bytes, " + std::to_string(p.bytes) + " needed");
      return FIRA_ERR_WORKSPACE_TOO_SMALL;
    }
    if (p.chunks * p.slices > 0x3fffffffll * EM_WARPS) { set_error(who + ": too many elements in one call"); return FIRA_ERR_INVALID_ARG; }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    char* work = static_cast<char*>(work_dev);
    const int n = (int)count, v = (int)vocab, h = (int)hidden;
    const bool token_vector = ((uintptr_t)tokens_dev & 15) == 0;
    cudaError_t e;
    if (token_bits == 32) e = token_vector ? run_order<int, true>(p, tokens_dev, n, v, work, st) : run_order<int, false>(p, tokens_dev, n, v, work, st);
    else e = token_vector ? run_order<long long, true>(p, tokens_dev, n, v, work, st) : run_order<long long, false>(p, tokens_dev, n, v, work, st);
    // a lane's piece of dY is 16 bytes; of G it is 8, 16 or 32
    const bool vector = rows::aligned16(dY_dev, ld, hidden, es) && (ldg * (long long)gs) % 16 == 0 && ((uintptr_t)G_dev & 15) == 0;
    if (e == cudaSuccess) {
      if (dtype == FIRA_BF16)
        e = grad_dtype == FIRA_BF16 ? run_grad<__nv_bfloat16, __nv_bfloat16>(p, dY_dev, ld, v, h, scale, accumulate != 0, G_dev, ldg, work, vector, st)
                                    : run_grad<__nv_bfloat16, float>(p, dY_dev, ld, v, h, scale, accumulate != 0, G_dev, ldg, work, vector, st);
      else
        e = grad_dtype == FIRA_BF16 ? run_grad<float, __nv_bfloat16>(p, dY_dev, ld, v, h, scale, accumulate != 0, G_dev, ldg, work, vector, st)
                                    : run_grad<float, float>(p, dY_dev, ld, v, h, scale, accumulate != 0, G_dev, ldg, work, vector, st);
    }
    if (e != cudaSuccess) { set_error(who + ": " + cudaGetErrorString(e)); return FIRA_ERR_CUDA; }
    return FIRA_OK;
  });
}
