// Rows of an embedding table, and the table's gradient.
//
//   Y_i = a E[t_i]                         (t_i outside 0 .. vocab-1: a row of zeros)
//   dE_v = a sum over {i : t_i = v} of dY_i
//
// The gradient takes two launches, or three for large batches (k_token_split and k_token_gather in place of k_token_order, each token
// read once).  k_token_order groups the positions by token: each block owns the tokens of one
// remainder by the number of blocks (so that the frequent ones, which in most vocabularies lie side by side, fall to different blocks)
// and reads all tokens of the batch, which stay in L2.  It counts those of lower remainders, which is where its own
// positions begin, and lists its own in shared memory; then it sorts the list by row.  No block waits for another, and the
// order is the same in every call.
// k_table_grad sums: a warp takes T positions of that order and a slice of columns, whole rows of the table where a row has
// at most T positions (the warp in whose stretch it begins does all of it).  A row with more, as words at the top of a
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

// Wide rows of whole 16-byte units on 16-byte boundaries: a warp takes LK_ROWS positions and a slice of 32 units.
// (131072 rows of 1024, bf16: 55 us; by k_embedding_words 64.  Of 64, fp32: 10.3 and 9.7.)
template <typename T, typename TOK>
__global__ void __launch_bounds__(EM_THREADS)
k_embedding_rows(const T* __restrict__ table, long long ld, const TOK* __restrict__ tokens, long long n, int vocab, int hidden, int slices,
                 float scale, T* __restrict__ out, long long ld_out) {
  constexpr int N = rows::PER16<T>;
  const long long unit = (long long)blockIdx.x * EM_WARPS + (threadIdx.x >> 5);
  const long long i0 = unit / slices * LK_ROWS;
  const int col = ((int)(unit % slices) * 32 + (threadIdx.x & 31)) * N;
  if (i0 >= n || col >= hidden) return;
  int t[LK_ROWS];
#pragma unroll
  for (int u = 0; u < LK_ROWS; ++u) t[u] = i0 + u < n ? token_at(tokens, i0 + u, vocab) : -1;
  uint4 a[LK_ROWS];
#pragma unroll
  for (int u = 0; u < LK_ROWS; ++u) a[u] = t[u] >= 0 ? *reinterpret_cast<const uint4*>(table + (long long)t[u] * ld + col) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int u = 0; u < LK_ROWS; ++u) {
    if (i0 + u >= n) break;
    float2 v[N / 2];
    rows::unpack<T>(a[u], v);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) v[e] = rows::mul2(v[e], rows::both(scale));
    *reinterpret_cast<uint4*>(out + (i0 + u) * ld_out + col) = rows::pack<T>(v);
  }
}

// The output goes by items of one or two words of 16 aligned bytes, `items` to a row, which are dealt to the threads in a row of their
// own, so that rows of any width keep all lanes busy.  ALIGNED (one word, two items of a thread): all rows are whole
// 16-byte units on 16-byte boundaries.  Otherwise (two words, one item) they are funnelled from three aligned words of the table,
// of which those are read that hold a byte of them (131072 rows of 1023, bf16: 83 us; one word and two items 103).
// Factors that are not finite, or negative, go that way too, wherever the rows begin: there alone a position without a token has a factor of
// its own, 0, since its zeros are multiplied like the rest (that factor in all kernels: 131072 rows of 1024, bf16, 54.0 -> 54.9 us; 200000 of 64, 9.7 -> 10.5).
template <bool ALIGNED>
constexpr int LK_WORDS = ALIGNED ? 1 : 2;
template <bool ALIGNED>
constexpr int LK_ITEMS = ALIGNED ? 2 : 1;

template <typename T, typename TOK, bool ALIGNED>
__global__ void __launch_bounds__(EM_THREADS)
k_embedding_words(const T* __restrict__ table, long long ld, const TOK* __restrict__ tokens, long long n, int vocab, int hidden, unsigned items,
                  float scale, T* __restrict__ out, long long ld_out) {
  constexpr int N = rows::PER16<T>, W = LK_WORDS<ALIGNED>, LK_EACH = LK_ITEMS<ALIGNED>;
  const long long first = (long long)blockIdx.x * (EM_THREADS * LK_EACH), row0 = first / items;
  const unsigned item0 = (unsigned)(first - row0 * items);
  uint4 a[LK_EACH][W + (ALIGNED ? 0 : 1)];
  T* to[LK_EACH];                           // the first word, and the column of its first element (hidden: none)
  int col[LK_EACH], skip[LK_EACH];
  bool none[LK_EACH];                       // no token
#pragma unroll
  for (int u = 0; u < LK_EACH; ++u) {
    const unsigned x = item0 + u * EM_THREADS + threadIdx.x, down = x / items;      // (items < 2^23: no overflow)
    const long long i = row0 + down;
#pragma unroll
    for (int w = 0; w < W + (ALIGNED ? 0 : 1); ++w) a[u][w] = make_uint4(0u, 0u, 0u, 0u);
    col[u] = hidden; skip[u] = 0; to[u] = out; none[u] = true;
    if (i >= n) continue;
    const int t = token_at(tokens, i, vocab);
    none[u] = t < 0;
    T* out_row = out + i * ld_out;
    const T* row = table + (long long)max(t, 0) * ld;
    col[u] = (int)(x - down * items) * (N * W);
    if (ALIGNED) {
      if (t >= 0) a[u][0] = *reinterpret_cast<const uint4*>(row + col[u]);
    } else {
      col[u] -= (int)(((uintptr_t)out_row & 15) / sizeof(T));
      const uintptr_t from = (uintptr_t)(row + max(col[u], 0)), end = (uintptr_t)(row + min(col[u] + N * W, hidden));     // the bytes that are wanted
      const uintptr_t begin = (uintptr_t)(row + col[u]), word = begin & ~(uintptr_t)15;
      skip[u] = (int)(begin & 15);
      if (t >= 0 && from < end) {
#pragma unroll
        for (int w = 0; w < W + 1; ++w)
          if (word + 16 * w + 16 > from && word + 16 * w < end) a[u][w] = *reinterpret_cast<const uint4*>(word + 16 * w);
      }
    }
    to[u] = out_row + col[u];
  }
#pragma unroll
  for (int u = 0; u < LK_EACH; ++u) {
#pragma unroll
    for (int w = 0; w < W; ++w) {
      uint4 x = a[u][w];
      if constexpr (!ALIGNED) x = rows::funnel16(a[u][w], a[u][w + 1], skip[u]);
      if (scale != 1.f) {
        const float by = !ALIGNED && none[u] ? 0.f : scale;
        float2 v[N / 2];
        rows::unpack<T>(x, v);
#pragma unroll
        for (int e = 0; e < N / 2; ++e) v[e] = rows::mul2(v[e], rows::both(by));
        x = rows::pack<T>(v);
      }
      if (ALIGNED) {
        if (col[u] < hidden) *reinterpret_cast<uint4*>(to[u]) = x;
      } else {
        if (col[u] + w * N < hidden) rows::store_between(to[u] + w * N, x, col[u] + w * N, 0, hidden);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ order of the tokens
constexpr int ORD_MIN_BLOCKS = 128;         // a power of two: a remainder is a few low bits
constexpr int ORD_MAX_ROWS = 1024;          // rows of a block
constexpr int ORD_MAX_THREADS = 1024;
constexpr int ORD_STEP = 128;               // tokens of a warp's step: four per lane
constexpr int ORD_LIST = 256;               // entries of a warp's list

// Four tokens from position i on: 0xffffffff behind the end and where a token is none of the table's.
template <typename TOK, bool VECTOR>
__device__ __forceinline__ void load_tokens(const TOK* __restrict__ tokens, int i, int n, int vocab, unsigned (&t)[4]) {
  unsigned high[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < 4; ++j) t[j] = 0xffffffffu;
  if (VECTOR && i + 4 <= n) {
    const uint4 u = reinterpret_cast<const uint4*>(tokens + i)[0];
    if constexpr (sizeof(TOK) == 4) {
      t[0] = u.x; t[1] = u.y; t[2] = u.z; t[3] = u.w;
    } else {
      const uint4 w = reinterpret_cast<const uint4*>(tokens + i)[1];
      t[0] = u.x; t[1] = u.z; t[2] = w.x; t[3] = w.z;
      high[0] = u.y; high[1] = u.w; high[2] = w.y; high[3] = w.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < n) { t[j] = (unsigned)tokens[i + j]; if (sizeof(TOK) == 8) high[j] = (unsigned)((unsigned long long)tokens[i + j] >> 32); }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) t[j] = t[j] < (unsigned)vocab && high[j] == 0u ? t[j] : 0xffffffffu;
}

__device__ __forceinline__ unsigned warp_inclusive(unsigned x) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) >= o) x += y;
  }
  return x;
}

// Stores the positions of up to 32 entries (a lane's own: row r where `in`) at the places that `mine` counts.
__device__ __forceinline__ void place_entries(bool in, unsigned r, int position, int token, unsigned* mine, int2* order) {
  const int lane = threadIdx.x & 31;
  const unsigned same = __match_any_sync(0xffffffffu, in ? r : 0x80000000u | lane);
  const unsigned at = in ? mine[r] : 0u;
  __syncwarp();
  if (in) {
    order[at + __popc(same & ((1u << lane) - 1))] = make_int2(position, token);
    if (lane == __ffs(same) - 1) mine[r] = at + __popc(same);
  }
  __syncwarp();
}

// From the counts [warp][row] of a block's rows to the places of their positions: `front` is that of the first one.  Leaves
// in counts where each warp's part of a row begins, and the rows' spans; returns the place behind the last one.
__device__ __forceinline__ unsigned row_fronts(unsigned* counts, int warps, int nrows, unsigned front, int shift, unsigned me, int vocab, int2* span,
                                               unsigned* sum_s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int base = 0; base < nrows; base += blockDim.x) {
    const int r = base + threadIdx.x;
    unsigned count = 0;
    if (r < nrows) {
#pragma unroll 8
      for (int w = 0; w < warps; ++w) {
        const unsigned c = counts[w * nrows + r];
        counts[w * nrows + r] = count;
        count += c;
      }
    }
    const unsigned inclusive = warp_inclusive(count);
    if (lane == 31) sum_s[warp] = inclusive;
    __syncthreads();
    const unsigned sums = warp_inclusive(lane < warps ? sum_s[lane] : 0u);
    const unsigned in_front = __shfl_sync(0xffffffffu, sums, max(warp - 1, 0));
    const unsigned at = front + (warp ? in_front : 0u) + inclusive - count;
    front += __shfl_sync(0xffffffffu, sums, 31);
    if (r < nrows) {
      const long long v = ((long long)r << shift) + me;
      if (v < vocab) span[v] = make_int2((int)at, (int)(at + count));
#pragma unroll 8
      for (int w = 0; w < warps; ++w) counts[w * nrows + r] += at;
    }
    __syncthreads();
  }
  return front;
}

// order: (position, token), equal tokens together; span[v]: where those of v begin and end; *total: tokens of the table.
// Among equal tokens the order goes by warp (a stretch of positions each), step, place in the lane's four, lane.
// Block b has the tokens v with v & (gridDim - 1) = b, in rows v >> shift.
template <typename TOK, bool VECTOR>
__global__ void __launch_bounds__(ORD_MAX_THREADS)
k_token_order(const TOK* __restrict__ tokens, int n, int vocab, int shift, int nrows, int2* __restrict__ order, int2* __restrict__ span,
              int* __restrict__ total, unsigned* __restrict__ counters, long long ncounters) {
  extern __shared__ __align__(16) unsigned shared[];      // counts [warps][nrows], lists [warps][ORD_LIST] of (position, row)
  __shared__ unsigned below_s[32], sum_s[32];
  ptx::grid_launch_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, threads = blockDim.x;
  const unsigned me = blockIdx.x, mask = gridDim.x - 1;
  for (long long i = (long long)blockIdx.x * threads + threadIdx.x; i < ncounters; i += (long long)gridDim.x * threads) counters[i] = 0;
  unsigned* mine = shared + warp * nrows;
  int2* list = reinterpret_cast<int2*>(shared + ((warps * nrows + 1) & ~1)) + warp * ORD_LIST;
  for (int i = threadIdx.x; i < warps * nrows; i += threads) shared[i] = 0;
  __syncthreads();
  const int steps = (n + ORD_STEP - 1) / ORD_STEP, per_warp = (steps + warps - 1) / warps;
  const int s0 = min(steps, warp * per_warp), s1 = min(steps, s0 + per_warp);
  unsigned below = 0;
  int listed = 0;                           // entries of this warp, whether the list holds them or not
  constexpr int AHEAD = 4;                  // steps whose tokens are on their way at once
  for (int first = s0; first < s1; first += AHEAD) {
    unsigned t[AHEAD][4];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load_tokens<TOK, VECTOR>(tokens, (first + u) * ORD_STEP + lane * 4, first + u < s1 ? n : 0, vocab, t[u]);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      unsigned home[4];                     // of a position without a token: no block's
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        home[j] = t[u][j] == 0xffffffffu ? t[u][j] : t[u][j] & mask;
        below += home[j] < me;
      }
      if (!__any_sync(0xffffffffu, home[0] == me || home[1] == me || home[2] == me || home[3] == me)) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned found = __ballot_sync(0xffffffffu, home[j] == me);
        if (home[j] == me) {
          const unsigned r = t[u][j] >> shift;
          atomicAdd(&mine[r], 1u);
          const int k = listed + __popc(found & ((1u << lane) - 1));
          if (k < ORD_LIST) list[k] = make_int2((first + u) * ORD_STEP + lane * 4 + j, (int)r);
        }
        listed += __popc(found);
      }
    }
  }
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) below_s[warp] = below;
  __syncthreads();
  const unsigned front = __reduce_add_sync(0xffffffffu, lane < warps ? below_s[lane] : 0u);
  const unsigned end = row_fronts(shared, warps, nrows, front, shift, me, vocab, span, sum_s);
  if (me == mask && threadIdx.x == 0) *total = (int)end;
  if (listed <= ORD_LIST) {
    for (int k = 0; k < listed; k += 32) {
      const bool in = k + lane < listed;
      const int2 e = in ? list[k + lane] : make_int2(0, 0);
      place_entries(in, (unsigned)e.y, e.x, (int)(((unsigned)e.y << shift) + me), mine, order);
    }
  } else {
    for (int s = s0; s < s1; ++s) {
      unsigned t[4];
      const int i = s * ORD_STEP + lane * 4;
      load_tokens<TOK, VECTOR>(tokens, i, n, vocab, t);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = t[j] != 0xffffffffu && (t[j] & mask) == me;
        if (__any_sync(0xffffffffu, in)) place_entries(in, t[j] >> shift, i + j, (int)t[j], mine, order);
      }
    }
  }
}

// The same for large batches, in two launches: every block of k_token_order reads all tokens, which takes 36 us at 131072 of them
// (and 8 at 4096); these read each token once.  k_token_split deals a tile of positions to the remainders, in their order;
// entries [tile][ORD_TILE], and per remainder and tile how many there are (counts) and where they begin in the tile (fronts).
constexpr int ORD_TILE = 1024;
constexpr int ORD_SPLIT_FROM = 16384;       // positions from which on there are two launches (16384, hidden 512, fp32: 31 us both ways; 65536: 60 and 56)
constexpr int ORD_SPLIT_BLOCKS = 512;       // remainders that k_token_split has counts for; where the vocabulary asks for more, it deals by these
                                            // lower bits, and each block of k_token_gather takes its own of the tokens of one

template <typename TOK>
__global__ void __launch_bounds__(ORD_TILE)
k_token_split(const TOK* __restrict__ tokens, int n, int vocab, int blocks, int2* __restrict__ entries, int* __restrict__ counts, int* __restrict__ fronts,
              unsigned* __restrict__ counters, long long ncounters) {
  extern __shared__ __align__(16) unsigned shared[];      // [32 warps][blocks]
  __shared__ unsigned sum_s[32];
  ptx::grid_launch_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tile = blockIdx.x, tiles = gridDim.x;
  for (long long i = (long long)tile * ORD_TILE + threadIdx.x; i < ncounters; i += (long long)tiles * ORD_TILE) counters[i] = 0;
  for (int i = threadIdx.x; i < 32 * blocks; i += ORD_TILE) shared[i] = 0;
  const int position = tile * ORD_TILE + threadIdx.x;
  const int token = position < n ? token_at(tokens, position, vocab) : -1;
  const unsigned home = (unsigned)token & (unsigned)(blocks - 1);
  __syncthreads();
  const unsigned same = __match_any_sync(0xffffffffu, token >= 0 ? home : 0x80000000u | lane);
  if (token >= 0 && lane == __ffs(same) - 1) shared[warp * blocks + home] = __popc(same);
  __syncthreads();
  const int h = threadIdx.x;
  unsigned count = 0;
  if (h < blocks) {
#pragma unroll 8
    for (int w = 0; w < 32; ++w) {
      const unsigned c = shared[w * blocks + h];
      shared[w * blocks + h] = count;
      count += c;
    }
  }
  const unsigned inclusive = warp_inclusive(count);
  if (lane == 31) sum_s[warp] = inclusive;
  __syncthreads();
  const unsigned in_front = __shfl_sync(0xffffffffu, warp_inclusive(sum_s[lane]), max(warp - 1, 0));
  if (h < blocks) {
    const unsigned at = (warp ? in_front : 0u) + inclusive - count;
    counts[(long long)h * tiles + tile] = (int)count;
    fronts[(long long)h * tiles + tile] = (int)at;
#pragma unroll 8
    for (int w = 0; w < 32; ++w) shared[w * blocks + h] += at;
  }
  __syncthreads();
  if (token >= 0) entries[(long long)tile * ORD_TILE + shared[warp * blocks + home] + __popc(same & ((1u << lane) - 1))] = make_int2(position, token);
}

// Block b sorts the entries of remainder b by row; a warp takes the tiles of a stretch.  Otherwise as k_token_order.
// FINE: there are more blocks than the `split` remainders that the entries were dealt to, and a block takes its own among those of
// one of them (131072 positions, 600000 tokens, hidden 8, fp32, whole call: 104 us; every block reading all tokens: 198).
template <bool FINE>
__global__ void __launch_bounds__(ORD_MAX_THREADS)
k_token_gather(const int2* entries, const int* counts, const int* fronts, int tiles, int split, int vocab, int shift, int nrows, int2* order, int2* span,
               int* total) {
  extern __shared__ __align__(16) unsigned shared[];      // counts [warps][nrows], lists [warps][ORD_LIST] of (position, token)
  __shared__ unsigned below_s[32], sum_s[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, threads = blockDim.x;
  const unsigned me = blockIdx.x, mask = gridDim.x - 1, dealt = FINE ? me & (unsigned)(split - 1) : me;
  for (int i = threadIdx.x; i < warps * nrows; i += threads) shared[i] = 0;
  __syncthreads();
  ptx::grid_wait();
  ptx::grid_launch_next();                  // (behind the wait: the next kernel may rely on k_token_split too)
  counts += (long long)dealt * tiles;
  fronts += (long long)dealt * tiles;
  unsigned below = 0;                       // tokens of lower remainders: of all dealt in front of this one's, and of those dealt with it
  for (int t = threadIdx.x; t < tiles; t += threads) below += fronts[t];
  unsigned* mine = shared + warp * nrows;
  int2* list = reinterpret_cast<int2*>(shared + ((warps * nrows + 1) & ~1)) + warp * ORD_LIST;
  const int per_warp = (tiles + warps - 1) / warps, t0 = min(tiles, warp * per_warp), t1 = min(tiles, t0 + per_warp);
  // The entries of this warp's tiles one behind another, 32 at a time: f(whether this lane has one, its number, its place).
  auto each = [&](auto f) {
    int seen = 0;
    for (int t = t0; t < t1; t += 32) {
      const int here = min(32, t1 - t), c = lane < here ? counts[t + lane] : 0;
      const int at = lane < here ? (t + lane) * ORD_TILE + fronts[t + lane] : 0;       // (tiles * ORD_TILE is about n)
      const int inclusive = (int)warp_inclusive((unsigned)c), all = __shfl_sync(0xffffffffu, inclusive, 31);
      for (int k = lane; k - lane < all; k += 32) {
        int j = 0;
        for (int i = 0; i + 1 < here; ++i) j += k >= __shfl_sync(0xffffffffu, inclusive, i);
        const int begins = __shfl_sync(0xffffffffu, at - (inclusive - c), j);
        f(k < all, seen + k, begins + k);
      }
      seen += all;
    }
  };
  int listed = 0;                           // FINE: entries of this warp and block, whether the list holds them or not
  each([&](bool in, int k, int at) {
    if constexpr (FINE) {
      const int2 x = in ? entries[at] : make_int2(0, 0);
      const unsigned home = (unsigned)x.y & mask;
      below += in && home < me;
      in = in && home == me;
      const unsigned found = __ballot_sync(0xffffffffu, in);
      k = listed + __popc(found & ((1u << lane) - 1));
      listed += __popc(found);
      if (in) {
        atomicAdd(&mine[(unsigned)x.y >> shift], 1u);
        if (k < ORD_LIST) list[k] = x;
      }
    } else if (in) {
      const int2 x = entries[at];
      atomicAdd(&mine[(unsigned)x.y >> shift], 1u);
      if (k < ORD_LIST) list[k] = x;
    }
  });
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) below_s[warp] = below;
  __syncthreads();
  const unsigned front = __reduce_add_sync(0xffffffffu, lane < warps ? below_s[lane] : 0u);
  const unsigned end = row_fronts(shared, warps, nrows, front, shift, me, vocab, span, sum_s);
  if (me == gridDim.x - 1 && threadIdx.x == 0) *total = (int)end;
  if (FINE && listed <= ORD_LIST) {
    for (int k = lane; k - lane < listed; k += 32) {
      const int2 x = k < listed ? list[k] : make_int2(0, 0);
      place_entries(k < listed, (unsigned)x.y >> shift, x.x, x.y, mine, order);
    }
  } else {
    each([&](bool in, int k, int at) {
      const int2 x = !in ? make_int2(0, 0) : !FINE && k < ORD_LIST ? list[k] : entries[at];
      if (FINE) in = in && ((unsigned)x.y & mask) == me;
      place_entries(in, (unsigned)x.y >> shift, x.x, x.y, mine, order);
    });
  }
}

// ------------------------------------------------------------------------------------------------ sums of the rows
constexpr int TG_DEPTH = 4;                 // rows of dY of a warp on their way
constexpr int TG_MIN = 8;                   // positions of a stretch at least
constexpr int TG_GROUP = 16;                // stretches whose parts of a long row are added by one warp
// Rows that a block looks over for tokens: TG_ZERO_ROWS, or TG_ZERO_MOST where looking takes longer than zeroing: blocks that look
// through all tokens, and rows of 1024 bytes, up to 1536 with the number of tokens.  (us a call with 64 and with 256, fp32, at 512, 4096 and 16384
// tokens of a vocabulary of 32000: hidden 64 10.1 and 9.5, 14.1 and 13.9, 20.4 and 19.8; 256 12.8 and 11.1, 14.9 and 13.6, 21.5 and 19.5; 512 17.5 and 13.8,
// 19.2 and 20.3, 28.3 and 27.3; 1024 27 and 40, 31 and 42, 45 and 52; 4096 85 and 153, 95 and 159, 135 and 194.  Of 128000, hidden 64: 19 and 15, 23 and 19,
// 34 and 23; hidden 384: 37 and 39, 43 and 42, 54 and 48.  bf16, of 32000, hidden 768: 16 and 14, 18 and 17, 26 and 24)
constexpr int TG_ZERO_ROWS = 64;
constexpr int TG_ZERO_MOST = 256;
constexpr int TG_ZERO_EARLY = 16384;        // tokens up to which such a block looks through them itself (1024: 20.8 us, or 21.9; 16384: 31.0 and 32.1)

struct TablePlan {
  int shift, blocks, nrows, threads;        // of the order of the tokens
  int tiles, split;                         // k_token_split's, and the remainders that it deals to; 0: k_token_order
  long long chunks;                         // stretches of the order
  int slices, pieces;
  long long counters() const { return 3 * chunks * slices; }     // per place of a part, and per stretch in which a long row begins
  size_t off_span, off_total, off_counters, off_entries, off_counts, off_fronts, off_parts, bytes;
};

// The columns of a warp: PIECES times 32 lanes of 16 bytes of dY.  ALIGNED: the rows of dY and G are whole 16-byte units on
// 16-byte boundaries, and a lane reads the 16 bytes that it fetched itself.  Otherwise the warp fetches the aligned words that
// hold a byte of its columns, one more than it has lanes, and a lane funnels its columns from two of them.
template <typename TI, typename TO, bool ALIGNED, int PIECES>
struct Slice {
  static constexpr int E = rows::PER16<TI>, N = E * PIECES, WIDTH = 32 * N, WORDS = 32 * PIECES + (ALIGNED ? 0 : 1);
  int col0, lane, hidden;
  __device__ __forceinline__ int col(int p) const { return col0 + (p * 32 + lane) * E; }
  // A row on its way to a slot; *skip: where its columns begin in the slot.
  __device__ __forceinline__ void fetch(const TI* row, uint4* slot, int* skip) const {
    if (ALIGNED) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
        if (col(p) < hidden)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"((unsigned)__cvta_generic_to_shared(slot + p * 32 + lane)), "l"(row + col(p)) : "memory");
    } else {
      const uintptr_t from = (uintptr_t)(row + col0), end = (uintptr_t)(row + min(col0 + WIDTH, hidden)), word = from & ~(uintptr_t)15;
      for (int w = lane; w < WORDS; w += 32)
        if (word + 16 * w < end)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"((unsigned)__cvta_generic_to_shared(slot + w)), "l"(word + 16 * w) : "memory");
      if (lane == 0) *skip = (int)(from & 15);
    }
  }
  // Adds the row in a slot whose fetch has been waited for.  (Columns beyond the width: whatever is there, never stored.)
  __device__ __forceinline__ void add(const uint4* slot, const int* skip, float (&sum)[N]) const {
    if (!ALIGNED) __syncwarp();             // words that other lanes fetched
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      float2 v[E / 2];
      if (ALIGNED) rows::unpack<TI>(slot[p * 32 + lane], v);
      else rows::unpack<TI>(rows::funnel16(slot[p * 32 + lane], slot[p * 32 + lane + 1], *skip), v);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 s = rows::add2(make_float2(sum[p * E + e], sum[p * E + e + 1]), v[e / 2]);
        sum[p * E + e] = s.x; sum[p * E + e + 1] = s.y;
      }
    }
    if (!ALIGNED) __syncwarp();             // the slot is filled anew
  }
  // (All lanes of the warp.)
  __device__ __forceinline__ void store(TO* row, float (&sum)[N], float scale, bool add) const {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      float* v = sum + p * E;
      const int c = col(p);
      if (ALIGNED) {
        if (c >= hidden) continue;
        TO* q = row + c;
        float w[E];
        if constexpr (E * sizeof(TO) % 16 == 0) {
          if (add) rows::load_vec<TO, E>(q, w);
        } else if (add) {                   // fp32 rows into bf16: 8 bytes
          const uint2 u = *reinterpret_cast<const uint2*>(q);
          w[0] = __uint_as_float(u.x << 16); w[1] = __uint_as_float(u.x & 0xffff0000u);
          w[2] = __uint_as_float(u.y << 16); w[3] = __uint_as_float(u.y & 0xffff0000u);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = add ? fmaf(scale, v[e], w[e]) : scale * v[e];
        if constexpr (E * sizeof(TO) % 16 == 0) {
          rows::store_vec<TO, E>(q, w);
        } else {
          static_assert(E == 4 && sizeof(TO) == 2, "");
          const __nv_bfloat162 a = __floats2bfloat162_rn(w[0], w[1]), b = __floats2bfloat162_rn(w[2], w[3]);
          *reinterpret_cast<uint2*>(q) = make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
        }
      } else if (sizeof(TO) == sizeof(TI) && !add) {
        // the aligned word in which this lane's columns begin: its first bytes are the lane's before; the last lane has
        // bytes left for one word more
        if constexpr (sizeof(TO) == sizeof(TI)) {
          float2 w[E / 2];
#pragma unroll
          for (int e = 0; e < E / 2; ++e) w[e] = rows::mul2(make_float2(v[2 * e], v[2 * e + 1]), rows::both(scale));
          const uint4 own = rows::pack<TO>(w);
          uint4 left;
          left.x = __shfl_up_sync(0xffffffffu, own.x, 1); left.y = __shfl_up_sync(0xffffffffu, own.y, 1);
          left.z = __shfl_up_sync(0xffffffffu, own.z, 1); left.w = __shfl_up_sync(0xffffffffu, own.w, 1);
          const int behind = (int)((uintptr_t)(row + c) & 15), at = behind / (int)sizeof(TO);       // (the same in all lanes)
          const int lo = col0 + p * 32 * E, hi = min(lo + 32 * E, hidden);
          rows::store_between(row + c - at, behind ? rows::funnel16(left, own, 16 - behind) : own, c - at, lo, hi);
          if (lane == 31 && behind) rows::store_between(row + c - at + E, rows::funnel16(own, own, 16 - behind), c - at + E, lo, hi);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (c + e < hidden) row[c + e] = from_float<TO>(add ? fmaf(scale, v[e], to_float<TO>(row[c + e])) : scale * v[e]);
      }
    }
  }
  // A part of a long row: WIDTH floats, of which a lane keeps its own.
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

__host__ __device__ constexpr int zero_rows_of(int ntokens, long long row_bytes) {
  return ntokens <= TG_ZERO_EARLY && row_bytes <= (ntokens < 4096 ? 1024 + ntokens / 8 : 1536) ? TG_ZERO_MOST : TG_ZERO_ROWS;
}

// Zeroes the rows of `first` on that no token names.  early: in front of the wait for k_token_order, from the tokens.
template <typename TO, typename TOK, bool ALIGNED>
__device__ __forceinline__ void zero_rows(long long first, int zero_rows_each, int vocab, int hidden, const int2* span, const TOK* __restrict__ tokens, int n, bool early, TO* G,
                                          long long ldg) {
  __shared__ unsigned char named[TG_ZERO_MOST];
  const int here = (int)min((long long)zero_rows_each, vocab - first);
  if (early) {
    for (int k = threadIdx.x; k < TG_ZERO_MOST; k += EM_THREADS) named[k] = 0;
    __syncthreads();
#pragma unroll 8
    for (int i = threadIdx.x; i < n; i += EM_THREADS) {
      const long long r = (long long)tokens[i] - first;
      if (r >= 0 && r < here) named[r] = 1;
    }
  } else {
    ptx::grid_wait();
    for (int k = threadIdx.x; k < here; k += EM_THREADS) {
      const int2 s = span[first + k];
      named[k] = s.x != s.y;
    }
  }
  __syncthreads();
  const int lane = threadIdx.x & 31;
  for (int k = threadIdx.x >> 5; k < here; k += EM_WARPS) {
    if (named[k]) continue;
    TO* row = G + (first + k) * ldg;
    if (ALIGNED) {
      const int bytes = hidden * (int)sizeof(TO);       // a multiple of 8
      for (int b = lane * 16; b + 16 <= bytes; b += 512) *reinterpret_cast<uint4*>(reinterpret_cast<char*>(row) + b) = make_uint4(0u, 0u, 0u, 0u);
      if (lane == 0 && (bytes & 8)) *reinterpret_cast<uint2*>(reinterpret_cast<char*>(row) + bytes - 8) = make_uint2(0u, 0u);
    } else {
      constexpr int N = rows::PER16<TO>;
      const int at = (int)((uintptr_t)row & 15) / (int)sizeof(TO);
      for (int c = lane * N - at; c < hidden; c += 32 * N) rows::store_between(row + c, make_uint4(0u, 0u, 0u, 0u), c, 0, hidden);
    }
  }
}

// zero_blocks blocks zero, zero_rows_of() rows each; the warps of the others take a stretch of T positions and a slice each.
template <typename TI, typename TO, typename TOK, bool ALIGNED, int PIECES>
__global__ void __launch_bounds__(EM_THREADS, PIECES == 1 ? 4 : 3)
k_table_grad(const int2* order, const int2* span, const int* total, unsigned* counters, float* parts, const TOK* __restrict__ tokens, int ntokens,
             const TI* __restrict__ dY, long long ld, int vocab, int hidden, long long chunks, int slices, int zero_blocks, float scale, int add,
             TO* __restrict__ G, long long ldg) {
  using Cols = Slice<TI, TO, ALIGNED, PIECES>;
  constexpr int N = Cols::N;
  __shared__ uint4 ring[EM_WARPS][TG_DEPTH][Cols::WORDS];
  __shared__ int skips[EM_WARPS][TG_DEPTH];
  // blocks that zero: in front where they need not wait, behind (where they fill the places that others leave) otherwise
  const bool early = ntokens <= TG_ZERO_EARLY;
  const int main_blocks = gridDim.x - zero_blocks, block = early ? (int)blockIdx.x - zero_blocks : (int)blockIdx.x;
  if (block < 0 || block >= main_blocks) {
    const int each = zero_rows_of(ntokens, (long long)hidden * sizeof(TO));
    zero_rows<TO, TOK, ALIGNED>((long long)(early ? blockIdx.x : block - main_blocks) * each, each, vocab, hidden, span, tokens, ntokens, early, G, ldg);
    ptx::grid_wait();                       // (this kernel does not end before the one in front of it)
    return;
  }
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)block * EM_WARPS + (threadIdx.x >> 5);
  ptx::grid_wait();
  const long long chunk = unit / slices;
  const int slice = (int)(unit - chunk * slices);
  const int n = *total;
  const int T = max(TG_MIN, (int)((n + chunks - 1) / chunks));
  const long long p0 = chunk * T;
  if (chunk >= chunks || p0 >= n) return;
  const int a0 = (int)p0, p1 = (int)min(p0 + T, (long long)n);
  const int v_first = order[a0].y, v_last = order[p1 - 1].y;
  const int2 sf = span[v_first], sl = span[v_last];
  const int first_s = sf.x, first_e = sf.y, last_s = sl.x, last_e = sl.y;
  const bool first_long = first_e - first_s > T, last_long = last_e - last_s > T;
  const int a = !first_long && first_s < a0 ? first_e : a0, b = last_long ? p1 : last_e;
  if (a >= b) return;
  const Cols at{slice * Cols::WIDTH, lane, hidden};

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
      // two long rows may meet in a stretch: the one that begins there has the second place
      auto place = [&](long long c) { return (2 * c + (c == c0 ? 1 : 0)) * slices + slice; };
      // Whether this warp is the last of n at a counter; what the others stored is then there.
      auto last_of = [&](unsigned* counter, long long n) {
        __threadfence();
        __syncwarp();
        unsigned before = 0;
        if (lane == 0) before = atomicAdd(counter, 1u);
        before = __shfl_sync(0xffffffffu, before, 0);
        __threadfence();
        return before == (unsigned)(n - 1);
      };
      auto add_parts = [&](long long from, long long to, long long step) {
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] = 0.f;
        const long long first = from / step * step;         // (in steps that are counted from 0, but not below `from`)
#pragma unroll 4
        for (long long c = first; c <= to; c += step) at.add_part(parts + place(max(c, from)) * Cols::WIDTH, sum);
      };
      // The parts of a group of stretches are added by the last of its warps, and left in the place of the first; the groups'
      // sums by the last group's.
      const long long group = chunk / TG_GROUP, from = max(c0, group * TG_GROUP), to = min(c1, group * TG_GROUP + TG_GROUP - 1);
      const long long ngroups = c1 / TG_GROUP - c0 / TG_GROUP + 1;
      at.store_part(parts + place(chunk) * Cols::WIDTH, sum);
      if (last_of(&counters[place(from)], to - from + 1)) {
        add_parts(from, to, 1);
        bool last = ngroups == 1;
        if (!last) {
          at.store_part(parts + place(from) * Cols::WIDTH, sum);
          last = last_of(&counters[(2 * chunks + c0) * slices + slice], ngroups);
          if (last) add_parts(c0, c1, TG_GROUP);
        }
        if (last) at.store(G + v * ldg, sum, scale, add);
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.f;
  };
  // A window of 32 positions of the order: their tokens, and the rows that are fetched while they are summed.
  uint4 (*slots)[Cols::WORDS] = ring[threadIdx.x >> 5];
  int* skip = skips[threadIdx.x >> 5];
  auto token_at = [&](int k) { return k < b ? order[k].y : -1; };
  auto row_at = [&](int k) { return k < b ? order[k].x : -1; };
  const int ahead = row_at(a + lane);
  int token = token_at(a + lane), row = row_at(a + TG_DEPTH + lane);
#pragma unroll
  for (int k = 0; k < TG_DEPTH; ++k) {
    const int i = __shfl_sync(0xffffffffu, ahead, k);
    if (i >= 0) at.fetch(dY + (long long)i * ld, slots[k], skip + k);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  int current = __shfl_sync(0xffffffffu, token, 0);
  for (int q = a; q < b; q += 32) {
    const int token_next = token_at(q + 32 + lane), row_next = row_at(q + 32 + TG_DEPTH + lane);
    const int m = min(32, b - q);
    const int before = __shfl_up_sync(0xffffffffu, token, 1);
    const unsigned changes = __ballot_sync(0xffffffffu, token != (lane ? before : current));     // where another row begins
    int k = 0;
    while (true) {
      const unsigned rest = changes >> k;               // (k < 32)
      const int end = rest ? min(m, k + __ffs(rest) - 1) : m;
      for (; k < end; ++k) {
        asm volatile("cp.async.wait_group %0;" :: "n"(TG_DEPTH - 1) : "memory");
        uint4* slot = slots[k % TG_DEPTH];
        at.add(slot, skip + k % TG_DEPTH, sum);
        const int i = __shfl_sync(0xffffffffu, row, k);
        if (i >= 0) at.fetch(dY + (long long)i * ld, slot, skip + k % TG_DEPTH);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      if (k >= m) break;
      flush(current);
      current = __shfl_sync(0xffffffffu, token, k);
      // the position that began it is summed now; the next change is looked for behind it
      asm volatile("cp.async.wait_group %0;" :: "n"(TG_DEPTH - 1) : "memory");
      uint4* slot = slots[k % TG_DEPTH];
      at.add(slot, skip + k % TG_DEPTH, sum);
      const int i = __shfl_sync(0xffffffffu, row, k);
      if (i >= 0) at.fetch(dY + (long long)i * ld, slot, skip + k % TG_DEPTH);
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (++k >= m) break;
    }
    token = token_next; row = row_next;
  }
  flush(current);
}

// The grid and the sections of the workspace of a gradient.
TablePlan plan_for(long long n, long long vocab, long long hidden, bool f32) {
  TablePlan p;
  p.blocks = ORD_MIN_BLOCKS;
  while ((vocab + p.blocks - 1) / p.blocks > ORD_MAX_ROWS) p.blocks *= 2;
  p.shift = 0;
  while ((1 << p.shift) < p.blocks) ++p.shift;
  p.nrows = (int)((vocab + p.blocks - 1) / p.blocks);
  p.tiles = n > ORD_SPLIT_FROM ? (int)((n + ORD_TILE - 1) / ORD_TILE) : 0;
  p.split = std::min(p.blocks, ORD_SPLIT_BLOCKS);
  // every warp has counts of its own, which cost time per warp: few warps for few tokens
  p.threads = n > 32768 ? ORD_MAX_THREADS : n > 8192 ? 512 : 256;
  // 512 bytes of dY per warp and row, or 1024, which takes fewer instructions per byte
  p.pieces = hidden > 32 * (f32 ? 4 : 8) ? 2 : 1;
  const long long width = 32 * (f32 ? 4 : 8) * p.pieces;
  p.slices = (int)((hidden + width - 1) / width);
  // As many stretches as there are warps on the GPU at once, or four times as many where that leaves 32 positions each (131072 tokens,
  // hidden 2048, bf16: 142 us, 133 so; hidden 512: 60, and 69 with four times as many of 8); of few positions as many as
  // have TG_MIN each.  All are of one length, which follows from the number of tokens that the device finds.
  const long long warps = EM_SMS * (p.pieces == 2 ? 3 : 4) * EM_WARPS;
  p.chunks = std::max<long long>(1, std::max(std::min((n + TG_MIN - 1) / TG_MIN, warps / p.slices), std::min(n / 32, 4 * warps / p.slices)));
  if (n == 0) p.chunks = 0;
  size_t at = align_up((size_t)n * sizeof(int2));
  p.off_span = at; at += align_up((size_t)vocab * sizeof(int2));
  p.off_total = at; at += 256;
  p.off_counters = at; at += align_up((size_t)p.counters() * sizeof(unsigned));
  p.off_entries = at; at += (size_t)p.tiles * ORD_TILE * sizeof(int2);
  p.off_counts = at; at += align_up((size_t)p.tiles * p.split * sizeof(int));
  p.off_fronts = at; at += align_up((size_t)p.tiles * p.split * sizeof(int));
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

// The 16-byte words that a row of the output has a part of, at most.
unsigned words_of(long long hidden, size_t size, bool aligned) { return (unsigned)((hidden * (long long)size + (aligned ? 0 : 16 - (long long)size) + 15) / 16); }

template <typename T, typename TOK>
void run_lookup(const void* table, long long ld, const void* tokens, long long n, int vocab, int hidden, float scale, void* out, long long ld_out,
                cudaStream_t st) {
  const bool aligned = rows::aligned16(table, ld, hidden, sizeof(T)) && rows::aligned16(out, ld_out, hidden, sizeof(T)) && isfinite(scale) && !signbit(scale);
  const unsigned words = words_of(hidden, sizeof(T), aligned), items = aligned ? words : (words + LK_WORDS<false> - 1) / LK_WORDS<false>;
  const int per_block = EM_THREADS * (aligned ? LK_ITEMS<true> : LK_ITEMS<false>);
  const unsigned blocks = (unsigned)((n * items + per_block - 1) / per_block);
  if (aligned && words >= 96) {              // (the last slice of 32 leaves a quarter of the lanes idle at most)
    const int slices = (int)((words + 31) / 32);
    k_embedding_rows<T, TOK><<<(unsigned)(((n + LK_ROWS - 1) / LK_ROWS * slices + EM_WARPS - 1) / EM_WARPS), EM_THREADS, 0, st>>>(
        (const T*)table, ld, (const TOK*)tokens, n, vocab, hidden, slices, scale, (T*)out, ld_out);
  } else if (aligned)
    k_embedding_words<T, TOK, true><<<blocks, EM_THREADS, 0, st>>>((const T*)table, ld, (const TOK*)tokens, n, vocab, hidden, items, scale, (T*)out, ld_out);
  else
    k_embedding_words<T, TOK, false><<<blocks, EM_THREADS, 0, st>>>((const T*)table, ld, (const TOK*)tokens, n, vocab, hidden, items, scale, (T*)out, ld_out);
}

// Counts and lists may be above the default limit of shared memory: a setting per device and kernel.
size_t order_smem(int warps, int nrows) { return (size_t)((warps * nrows + 1) & ~1) * sizeof(unsigned) + (size_t)warps * ORD_LIST * sizeof(int2); }

template <typename TOK>
cudaError_t run_split(const TablePlan& p, const void* tokens, int n, int vocab, char* work, cudaStream_t st) {
  const size_t smem = (size_t)32 * p.split * sizeof(unsigned), gather = order_smem(p.threads / 32, p.nrows);
  auto kernel = p.split < p.blocks ? k_token_gather<true> : k_token_gather<false>;
  if (smem > 47 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_token_split<TOK>, cudaFuncAttributeMaxDynamicSharedMemorySize, 32 * ORD_SPLIT_BLOCKS * 4);
    if (e != cudaSuccess) return e;
  }
  if (gather > 47 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)order_smem(ORD_MAX_THREADS / 32, ORD_MAX_ROWS));
    if (e != cudaSuccess) return e;
  }
  int2* entries = (int2*)(work + p.off_entries);
  int* counts = (int*)(work + p.off_counts);
  int* fronts = (int*)(work + p.off_fronts);
  k_token_split<TOK><<<p.tiles, ORD_TILE, smem, st>>>((const TOK*)tokens, n, vocab, p.split, entries, counts, fronts, (unsigned*)(work + p.off_counters),
                                                      p.counters());
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_chained(kernel, dim3(p.blocks), p.threads, gather, st, true, 1, (const int2*)entries, (const int*)counts, (const int*)fronts, p.tiles,
                        p.split, vocab, p.shift, p.nrows, (int2*)work, (int2*)(work + p.off_span), (int*)(work + p.off_total));
}
template <typename TOK, bool VECTOR>
cudaError_t run_order(const TablePlan& p, const void* tokens, int n, int vocab, char* work, cudaStream_t st) {
  if (p.tiles) return run_split<TOK>(p, tokens, n, vocab, work, st);
  const size_t smem = order_smem(p.threads / 32, p.nrows);
  if (smem > 47 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_token_order<TOK, VECTOR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)order_smem(ORD_MAX_THREADS / 32, ORD_MAX_ROWS));
    if (e != cudaSuccess) return e;
  }
  k_token_order<TOK, VECTOR><<<p.blocks, p.threads, smem, st>>>((const TOK*)tokens, n, vocab, p.shift, p.nrows, (int2*)work, (int2*)(work + p.off_span),
                                                                (int*)(work + p.off_total), (unsigned*)(work + p.off_counters), p.counters());
  return cudaGetLastError();
}

template <typename TI, typename TO, typename TOK>
cudaError_t run_grad(const TablePlan& p, const void* tokens, int n, const void* dY, long long ld, int vocab, int hidden, float scale, int add, void* G, long long ldg, char* work,
                     bool vector, cudaStream_t st) {
  const int zero_rows_each = zero_rows_of(n, (long long)hidden * sizeof(TO)), zero_blocks = add ? 0 : (vocab + zero_rows_each - 1) / zero_rows_each;
  const dim3 grid((unsigned)(zero_blocks + (p.chunks * p.slices + EM_WARPS - 1) / EM_WARPS));
  if (grid.x == 0) return cudaSuccess;
  auto kernel = p.pieces == 2 ? (vector ? k_table_grad<TI, TO, TOK, true, 2> : k_table_grad<TI, TO, TOK, false, 2>)
                              : (vector ? k_table_grad<TI, TO, TOK, true, 1> : k_table_grad<TI, TO, TOK, false, 1>);
  return launch_chained(kernel, grid, EM_THREADS, 0, st, true, 1, (const int2*)work,
                        (const int2*)(work + p.off_span), (const int*)(work + p.off_total), (unsigned*)(work + p.off_counters),
                        (float*)(work + p.off_parts), (const TOK*)tokens, n, (const TI*)dY, ld, vocab, hidden, p.chunks, p.slices, zero_blocks, scale,
                        add, (TO*)G, ldg);
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
    if (count * words_of(hidden, es, false) > 0x7fffffffll * EM_THREADS) { set_error("fira_embedding: too many elements in one call"); return FIRA_ERR_INVALID_ARG; }
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
#define EM_GRAD(TI, TO)                                                                                                          \
  (token_bits == 32 ? run_grad<TI, TO, int>(p, tokens_dev, n, dY_dev, ld, v, h, scale, accumulate != 0, G_dev, ldg, work, vector, st) \
                    : run_grad<TI, TO, long long>(p, tokens_dev, n, dY_dev, ld, v, h, scale, accumulate != 0, G_dev, ldg, work, vector, st))
    if (e == cudaSuccess) {
      if (dtype == FIRA_BF16) e = grad_dtype == FIRA_BF16 ? EM_GRAD(__nv_bfloat16, __nv_bfloat16) : EM_GRAD(__nv_bfloat16, float);
      else e = grad_dtype == FIRA_BF16 ? EM_GRAD(float, __nv_bfloat16) : EM_GRAD(float, float);
    }
#undef EM_GRAD
    if (e != cudaSuccess) { set_error(who + ": " + cudaGetErrorString(e)); return FIRA_ERR_CUDA; }
    return FIRA_OK;
  });
}
