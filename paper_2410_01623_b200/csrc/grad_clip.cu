// The norm over a list of gradients, and clipping by it.
//
//   N = sqrt(sum_i ||G_i||^2),  s = max_norm / max(N, max_norm),  out_i = s G_i
//
// Two kernels over a list of tensors whose table travels in the kernel arguments (nothing is allocated, nothing of
// it outlives the call).  k_grad_squares leaves one sum of squares per block; k_grad_scale adds those up in a fixed
// order in every block (they are a few KB), so that no third launch lies between, and scales.  The same call gives the same sums: no
// atomics.  (Which elements are a thread's depends on the tensors' and outputs' places between 16-byte boundaries.)
//
// A thread squares 32 elements into one fp32 sum and adds that to a double.  Where the fp32 sum says nothing (it left
// the range in which neither an overflow nor what underflowed matters) the elements, still in registers, are squared
// again in double: the norm holds over the whole range of the types.
#include <math.h>

#include <algorithm>

#include "rows.cuh"
#include "tc_ptx.cuh"

namespace fira {
namespace {

constexpr int GC_THREADS = 256;
constexpr int GC_CHUNK = 8;                       // elements of a chunk: 16 bytes of bf16, 32 of fp32
constexpr int GC_UNROLL = 4;                      // chunks of a thread in flight
constexpr int GC_TILE = GC_THREADS * GC_UNROLL;   // chunks of a tile (8192 elements)
constexpr int GC_SMS = 148;
constexpr int GC_BLOCKS = GC_SMS * 4;             // blocks of the sums, all resident: tiles are dealt to them in turn
constexpr int GC_SCALE_BLOCKS = GC_SMS * 32;      // of the scaling: eight times as many as are resident, since SMs far from the
                                                  // memory take longer (2.7 GB of bf16: 925 us with 4 per SM, 831 so, as long as a copy)
constexpr int GC_MANY = 480, GC_FEW = 48;         // tensors of a launch: 31 KB of kernel arguments, or 3.1 KB
// Bytes of a list that the sums leave in L2 for the scaling (232 MB of fp32: 110 -> 104 us; 1440 bf16 tensors of 60000, three launches with
// 48 MB each 156 us, with 48 in all 147).  In place with a factor of 1 nothing reads them again, and they stay: the optimizer step that
// follows takes the same time (350 us to 1.35 ms, both types), ten passes over another 80 MB that L2 would hold up to 209 us instead of 176.
constexpr long long GC_KEPT = 48ll << 20;

// One tensor.  A flat one is one row; rows of a pitched one start on their own.
struct GradEntry {
  const void* g;
  void* o;
  long long ld, out_ld;     // of a pitched tensor, elements
  long long n;              // elements of a row
  long long chunks;         // of the whole tensor
  int tile_start;           // tiles of the tensors in front of it
  unsigned char bf16, out_bf16;
  unsigned char single;     // a chunk is one element: where G and out do not begin alike
  unsigned char pitched : 1;
  unsigned char shift : 7;  // elements from a 16-byte boundary to the first one of a row, alike in G and out and in all rows
  long long whole;          // tiles from the first on that end within the tensor (the others go chunk by chunk)
};
// A tile of GC_TILE whole chunks in a row: not the first one of a tensor that begins between two boundaries.
__device__ __forceinline__ bool is_whole(const GradEntry& t, int tile) {
  const int i = tile - t.tile_start;
  return i < t.whole && (i > 0 || t.shift == 0);
}

template <int CAP>
struct GradTable {
  GradEntry t[CAP];
  int count, tiles;
};

// The tensor of a tile: the last one (q, most often) or found by halving.  (One by one, lists of hundreds of small
// tensors took 28 us for the norm alone: each look at the table is a miss of the constant cache.)
__device__ __forceinline__ int find_tensor(const GradEntry* t, int count, int q, int tile) {
  int lo = 0, hi = count;                   // t[lo].tile_start <= tile, and t[hi]'s is not
  if (tile >= t[q].tile_start) {
    if (q + 1 == count || tile < t[q + 1].tile_start) return q;
    lo = q + 1;
  } else {
    hi = q;
  }
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t[mid].tile_start <= tile) lo = mid; else hi = mid;
  }
  return lo;
}

// Where chunk c of the tensor starts in G and in out, and how many elements it has.
struct Place { long long at, out_at; int len; };
__device__ __forceinline__ Place place(const GradEntry& t, long long c, long long row0, unsigned col0, unsigned local) {
  const int w = t.single ? 1 : GC_CHUNK;
  long long col, row = 0;
  if (!t.pitched) {
    col = c * w - t.shift;
  } else {
    const unsigned per_row = (unsigned)((t.n + t.shift + w - 1) / w);
    const unsigned x = col0 + local, down = x / per_row;      // col0 < per_row < 2^31, local < 2^11: no overflow
    col = (long long)(x - down * per_row) * w - t.shift;
    row = row0 + down;
  }
  const long long from = col < 0 ? 0 : col, to = col + w < t.n ? col + w : t.n;
  Place p;
  p.at = row * t.ld + from;
  p.out_at = row * t.out_ld + from;
  p.len = (int)(to - from);
  return p;
}

__device__ __forceinline__ void load_chunk(const GradEntry& t, const Place& p, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  if (p.len == 8) {
    if (t.bf16) {
      rows::load_vec<__nv_bfloat16, 8>(static_cast<const __nv_bfloat16*>(t.g) + p.at, v);
    } else {
      rows::load_vec<float, 8>(static_cast<const float*>(t.g) + p.at, v);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < p.len) v[e] = t.bf16 ? to_float(static_cast<const __nv_bfloat16*>(t.g)[p.at + e]) : static_cast<const float*>(t.g)[p.at + e];
  }
}

__device__ __forceinline__ void store_chunk(const GradEntry& t, const Place& p, const float (&v)[8]) {
  if (p.len == 8) {
    if (t.out_bf16) rows::store_vec<__nv_bfloat16, 8>(static_cast<__nv_bfloat16*>(t.o) + p.out_at, v);
    else rows::store_vec<float, 8>(static_cast<float*>(t.o) + p.out_at, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < p.len) {
        if (t.out_bf16) static_cast<__nv_bfloat16*>(t.o)[p.out_at + e] = __float2bfloat16_rn(v[e]);
        else static_cast<float*>(t.o)[p.out_at + e] = v[e];
      }
  }
}

// L2 policies.  What is read once makes room for what the scaling reads again, after which that is to go first too.
__device__ __forceinline__ uint64_t policy(bool first) {
  uint64_t p;
  if (first) asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  else asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint4 load16(const void* p, uint64_t pol) {
  uint4 u;
  asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.b32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p), "l"(pol));
  return u;
}
__device__ __forceinline__ void store16(void* p, const uint4& u, uint64_t pol) {
  asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1, %2, %3, %4}, %5;" :: "l"(p), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w), "l"(pol) : "memory");
}
__device__ __forceinline__ void store8(void* p, unsigned x, unsigned y, uint64_t pol) {
  asm volatile("st.global.L2::cache_hint.v2.b32 [%0], {%1, %2}, %3;" :: "l"(p), "r"(x), "r"(y), "l"(pol) : "memory");
}
__device__ __forceinline__ unsigned pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&h);
}

// The chunks of this thread in a tile.
struct Tile {
  int q;                       // tensor
  long long first, row0;       // first chunk; for a pitched tensor its row and column
  unsigned col0;
};
__device__ __forceinline__ Tile open_tile(const GradEntry* t, int q, int tile) {
  Tile x;
  x.q = q;
  x.first = (long long)(tile - t[q].tile_start) * GC_TILE;
  x.row0 = 0; x.col0 = 0;
  if (t[q].pitched) {
    const int w = t[q].single ? 1 : GC_CHUNK;
    const long long per_row = (t[q].n + t[q].shift + w - 1) / w;
    x.row0 = x.first / per_row;
    x.col0 = (unsigned)(x.first - x.row0 * per_row);
  }
  return x;
}

__device__ __forceinline__ void load_tile(const GradEntry* tab, const Tile& x, Place (&p)[GC_UNROLL], float (&v)[GC_UNROLL][8]) {
  const GradEntry& t = tab[x.q];
#pragma unroll
  for (int u = 0; u < GC_UNROLL; ++u) {
    const unsigned local = u * GC_THREADS + threadIdx.x;
    const long long c = x.first + local;
    if (c < t.chunks) {
      p[u] = place(t, c, x.row0, x.col0, local);
    } else {
      p[u].at = p[u].out_at = 0; p[u].len = 0;
    }
    load_chunk(t, p[u], v[u]);
  }
}

// Whole tiles: 16 bytes per thread and load, W of them (4: bf16, 8: fp32).
template <int W>
__device__ __forceinline__ void load_whole(const GradEntry& t, long long first, uint64_t pol, uint4 (&u)[W]) {
  const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(t.g) - t.shift * (W == 8 ? 4 : 2)) + first * (W / GC_UNROLL) + threadIdx.x;
#pragma unroll
  for (int i = 0; i < W; ++i) u[i] = load16(p + i * GC_THREADS, pol);
}
template <int W>
__device__ __forceinline__ void unpack_whole(const uint4& u, float* v) {
  if constexpr (W == 8) rows::unpack<float>(u, v);
  else rows::unpack<__nv_bfloat16>(u, v);
}
constexpr int GC_ELEMS = GC_UNROLL * GC_CHUNK;     // of a thread in a tile

// The sum of the squares of a thread's elements of a tile.
__device__ __forceinline__ double squares(const float (&v)[GC_ELEMS]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < GC_ELEMS; ++e) s = fmaf(v[e], v[e], s);
  if (s >= 0x1p-80f && s <= 0x1p126f) return (double)s;      // what underflowed is below 32 * 2^-126, the rounding below 32 * 2^-24 of s
  bool any = false;
#pragma unroll
  for (int e = 0; e < GC_ELEMS; ++e) any |= v[e] != 0.f;
  double d = 0.0;
  if (any) {
#pragma unroll
    for (int e = 0; e < GC_ELEMS; ++e) d = fma((double)v[e], (double)v[e], d);
  }
  return d;
}
template <int W>
__device__ __forceinline__ double whole_squares(const GradEntry& t, long long first, uint64_t pol) {
  uint4 u[W];
  load_whole<W>(t, first, pol, u);
  float v[GC_ELEMS];
#pragma unroll
  for (int i = 0; i < W; ++i) unpack_whole<W>(u[i], v + i * (GC_ELEMS / W));
  return squares(v);
}
template <int W, bool OUT_BF16>
__device__ __forceinline__ void whole_scale(const GradEntry& t, long long first, float scale, uint64_t pol) {
  uint4 u[W];
  load_whole<W>(t, first, pol, u);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    constexpr int N = GC_ELEMS / W;
    float v[N];
    unpack_whole<W>(u[i], v);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] *= scale;
    // the 16 bytes that were read, seen as elements of the tensor
    const long long at = (first * (W / GC_UNROLL) + i * GC_THREADS + threadIdx.x) * N - t.shift;
    if constexpr (OUT_BF16) {
      __nv_bfloat16* q = static_cast<__nv_bfloat16*>(t.o) + at;
      if constexpr (N == 8) store16(q, make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])), pol);
      else store8(q, pack2(v[0], v[1]), pack2(v[2], v[3]), pol);
    } else {
      float* q = static_cast<float*>(t.o) + at;
#pragma unroll
      for (int e = 0; e < N; e += 4)
        store16(q + e, make_uint4(__float_as_uint(v[e]), __float_as_uint(v[e + 1]), __float_as_uint(v[e + 2]), __float_as_uint(v[e + 3])), pol);
    }
  }
}

__device__ __forceinline__ double block_sum(double s, double* smem) {
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = s;
  __syncthreads();
  double r = 0.0;
#pragma unroll
  for (int w = 0; w < GC_THREADS / 32; ++w) r += smem[w];
  return r;
}

template <int CAP>
__global__ void __launch_bounds__(GC_THREADS, 4)
k_grad_squares(const __grid_constant__ GradTable<CAP> tab, double* __restrict__ sums, int kept) {
  __shared__ double red[GC_THREADS / 32];
  ptx::grid_launch_next();     // its blocks take the places that ours leave, and wait for the last of ours
  const uint64_t once = policy(true), again = policy(false);
  double total = 0.0;
  int q = 0;
  for (int tile = blockIdx.x; tile < tab.tiles; tile += gridDim.x) {
    q = find_tensor(tab.t, tab.count, q, tile);
    const GradEntry& t = tab.t[q];
    if (is_whole(t, tile)) {
      const uint64_t pol = tile >= kept ? again : once;
      const long long first = (long long)(tile - t.tile_start) * GC_TILE;
      total += t.bf16 ? whole_squares<4>(t, first, pol) : whole_squares<8>(t, first, pol);
    } else {
      Place p[GC_UNROLL];
      float v[GC_UNROLL][8];
      load_tile(tab.t, open_tile(tab.t, q, tile), p, v);
      total += squares(reinterpret_cast<const float (&)[GC_ELEMS]>(v));
    }
  }
  const double r = block_sum(total, red);
  if (threadIdx.x == 0) sums[blockIdx.x] = r;
}

// The norm from the sums of all blocks, in an order that their number alone fixes.
__device__ __forceinline__ double norm_of(const double* sums, int nsums, double* red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < nsums; i += GC_THREADS) s += sums[i];
  return sqrt(block_sum(s, red));
}

__global__ void __launch_bounds__(GC_THREADS)
k_grad_norm(const double* sums, int nsums, float* norm_out) {
  __shared__ double red[GC_THREADS / 32];
  ptx::grid_wait();
  const double norm = norm_of(sums, nsums, red);
  if (threadIdx.x == 0) *norm_out = (float)norm;
}

template <int CAP>
__global__ void __launch_bounds__(GC_THREADS, 4)
k_grad_scale(const __grid_constant__ GradTable<CAP> tab, const double* sums, int nsums, float max_norm, float* norm_out, float* scale_out,
             int in_place) {
  __shared__ double red[GC_THREADS / 32];
  ptx::grid_wait();
  const double norm = norm_of(sums, nsums, red);
  const bool finite = norm <= 1.7976931348623157e308;
  const float scale = finite && norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
  if (blockIdx.x == 0 && threadIdx.x == 0) { *norm_out = (float)norm; *scale_out = scale; }
  if (in_place && scale == 1.f) return;
  const uint64_t once = policy(true);
  int q = tab.count - 1;
  // from the end: what the sums read last is what the L2 still holds
  for (int tile = tab.tiles - 1 - (int)blockIdx.x; tile >= 0; tile -= gridDim.x) {
    q = find_tensor(tab.t, tab.count, q, tile);
    const GradEntry& t = tab.t[q];
    if (is_whole(t, tile)) {
      const long long first = (long long)(tile - t.tile_start) * GC_TILE;
      if (t.bf16) {
        if (t.out_bf16) whole_scale<4, true>(t, first, scale, once);
        else whole_scale<4, false>(t, first, scale, once);
      } else {
        if (t.out_bf16) whole_scale<8, true>(t, first, scale, once);
        else whole_scale<8, false>(t, first, scale, once);
      }
    } else {
      Place p[GC_UNROLL];
      float v[GC_UNROLL][8];
      load_tile(tab.t, open_tile(tab.t, q, tile), p, v);
#pragma unroll
      for (int u = 0; u < GC_UNROLL; ++u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] *= scale;
        if (p[u].len) store_chunk(t, p[u], v[u]);
      }
    }
  }
}

int launches_for(int count) { return (count + GC_MANY - 1) / GC_MANY; }

fira_status check_list(const char* who, int32_t count, const fira_grad_desc* descs, const void* const* G_dev, void* const* out_dev) {
  const std::string name(who);
  if (count <= 0 || !descs || !G_dev) { set_error(name + ": null argument or empty list"); return FIRA_ERR_INVALID_ARG; }
  auto refuse = [&](int i, const char* why) { set_error(name + ": tensor " + std::to_string(i) + ": " + why); return FIRA_ERR_INVALID_ARG; };
  for (int base = 0; base < count; base += GC_MANY) {
    long long tiles = 0;
    for (int i = base; i < std::min(count, base + GC_MANY); ++i) {
      const fira_grad_desc& d = descs[i];
      if (d.rows < 0 || d.cols < 0) return refuse(i, "negative size");
      if (d.rows > 1 && ((d.ld != 0 && d.ld < d.cols) || (out_dev && d.out_ld != 0 && d.out_ld < d.cols))) return refuse(i, "ld below the width");
      if ((d.dtype != FIRA_F32 && d.dtype != FIRA_BF16) || (out_dev && d.out_dtype != FIRA_F32 && d.out_dtype != FIRA_BF16)) return refuse(i, "unknown dtype");
      if (d.rows == 0 || d.cols == 0) continue;
      const long long pitch = std::max<long long>({d.cols, d.rows > 1 ? d.ld : 0, d.rows > 1 && out_dev ? d.out_ld : 0});
      if (d.rows > (1ll << 40) || d.cols > (1ll << 40) || d.rows > (1ll << 42) / pitch || (d.rows > 1 && d.cols >= (1ll << 31) - GC_TILE)) return refuse(i, "too large");
      const size_t es = d.dtype == FIRA_BF16 ? 2 : 4, os = d.out_dtype == FIRA_BF16 ? 2 : 4;
      if (!G_dev[i] || ((uintptr_t)G_dev[i] & (es - 1)) || (out_dev && (!out_dev[i] || ((uintptr_t)out_dev[i] & (os - 1)))))
        return refuse(i, "pointers must be non-null and aligned to their elements");
      // every element a chunk of its own is the most that a tensor takes
      tiles += (d.rows * d.cols + GC_TILE - 1) / GC_TILE;
    }
    if (tiles > 0x7fff0000ll) { set_error(name + ": too many elements in one call"); return FIRA_ERR_INVALID_ARG; }
  }
  return FIRA_OK;
}

// No tensor may be written twice or over another one's input, and one written over its own keeps its type and layout.
fira_status check_outputs(int32_t count, const fira_grad_desc* descs, const void* const* G_dev, void* const* out_dev) {
  if (count <= 0 || !descs || !G_dev) return FIRA_OK;      // said by check_list
  std::vector<const void*> written;
  written.reserve(count);
  for (int i = 0; i < count; ++i) {
    const fira_grad_desc& d = descs[i];
    if (d.rows <= 0 || d.cols <= 0) continue;
    if (out_dev && out_dev[i] == G_dev[i] && (d.dtype != d.out_dtype || (d.rows > 1 && (d.ld ? d.ld : d.cols) != (d.out_ld ? d.out_ld : d.cols)))) {
      set_error("fira_clip_grads: tensor " + std::to_string(i) + ": in place needs the same type and ld"); return FIRA_ERR_INVALID_ARG;
    }
    written.push_back(out_dev ? out_dev[i] : G_dev[i]);
  }
  std::sort(written.begin(), written.end());
  if (std::adjacent_find(written.begin(), written.end()) != written.end()) {
    set_error("fira_clip_grads: a tensor is written twice"); return FIRA_ERR_INVALID_ARG;
  }
  for (int i = 0; out_dev && i < count; ++i) {
    const void* g = G_dev[i];
    if (descs[i].rows <= 0 || descs[i].cols <= 0 || out_dev[i] == g || g < written.front() || g > written.back()) continue;
    if (std::binary_search(written.begin(), written.end(), g)) {
      set_error("fira_clip_grads: tensor " + std::to_string(i) + " is the output of another one"); return FIRA_ERR_INVALID_ARG;
    }
  }
  return FIRA_OK;
}

template <int CAP>
void fill(GradTable<CAP>& tab, int base, int n, const fira_grad_desc* descs, const void* const* G_dev, void* const* out_dev) {
  long long tiles = 0;
  tab.count = 0;
  for (int i = base; i < base + n; ++i) {
    const fira_grad_desc& d = descs[i];
    if (d.rows == 0 || d.cols == 0) continue;
    const long long ld = d.rows == 1 || d.ld == 0 ? d.cols : d.ld;
    const long long out_ld = !out_dev ? ld : d.rows == 1 || d.out_ld == 0 ? d.cols : d.out_ld;
    const size_t es = d.dtype == FIRA_BF16 ? 2 : 4;
    GradEntry& t = tab.t[tab.count++];
    t.g = G_dev[i];
    t.o = out_dev ? out_dev[i] : const_cast<void*>(G_dev[i]);
    t.bf16 = d.dtype == FIRA_BF16;
    t.out_bf16 = out_dev ? d.out_dtype == FIRA_BF16 : t.bf16;
    const size_t os = t.out_bf16 ? 2 : 4;
    t.ld = ld; t.out_ld = out_ld;
    t.pitched = ld != d.cols || out_ld != d.cols;
    t.n = t.pitched ? d.cols : d.rows * d.cols;
    // elements behind a 16-byte boundary: bf16 has the longer way between two of them
    const size_t shift = t.out_bf16 ? ((uintptr_t)t.o & 15) / 2 : t.bf16 ? ((uintptr_t)t.g & 15) / 2 : ((uintptr_t)t.g & 15) / 4;
    t.single = (((uintptr_t)t.g - shift * es) & 15) != 0 || (((uintptr_t)t.o - shift * os) & 15) != 0 || (t.pitched && ((ld * es | out_ld * os) & 15) != 0);
    t.shift = t.single ? 0 : (unsigned char)shift;
    const long long w = t.single ? 1 : GC_CHUNK;
    t.chunks = (t.pitched ? d.rows : 1) * ((t.n + t.shift + w - 1) / w);
    t.whole = t.pitched || t.single ? 0 : (t.n + t.shift) / GC_CHUNK / GC_TILE;
    t.tile_start = (int)tiles;
    tiles += (t.chunks + GC_TILE - 1) / GC_TILE;
  }
  tab.tiles = (int)tiles;
}

// Bytes of the tensors from `from` on, as far as they matter: what is left of GC_KEPT for those in front of them.
long long kept_in_front_of(int32_t from, int32_t count, const fira_grad_desc* descs) {
  long long left = GC_KEPT;
  for (int32_t i = count; i-- > from && left > 0;) left -= descs[i].rows * descs[i].cols * (descs[i].dtype == FIRA_BF16 ? 2 : 4);
  return std::max(left, 0ll);
}

// The first tile from which on a launch's bytes fit what the L2 is expected to keep of them.
template <int CAP>
int kept_from(const GradTable<CAP>& tab, long long kept) {
  long long bytes = 0;
  for (int q = tab.count - 1; q >= 0; --q) {
    const long long per_tile = (long long)GC_TILE * (tab.t[q].single ? 1 : GC_CHUNK) * (tab.t[q].bf16 ? 2 : 4);
    const long long tiles = (q + 1 < tab.count ? tab.t[q + 1].tile_start : tab.tiles) - tab.t[q].tile_start;
    if (bytes + tiles * per_tile > kept) return tab.t[q].tile_start + (int)(tiles - (kept - bytes) / per_tile);
    bytes += tiles * per_tile;
  }
  return 0;
}

// out_dev null: in place.  scale_dev null: the norm alone.
template <int CAP>
cudaError_t run_list(int32_t count, const fira_grad_desc* descs, const void* const* G_dev, void* const* out_dev, float max_norm,
                     float* norm_dev, float* scale_dev, double* sums, cudaStream_t st) {
  GradTable<CAP> tab;
  int nsums = 0;
  for (int base = 0; base < count; base += CAP) {
    fill(tab, base, std::min(CAP, count - base), descs, G_dev, out_dev);
    const int blocks = std::max(1, std::min(GC_BLOCKS, tab.tiles));
    k_grad_squares<CAP><<<blocks, GC_THREADS, 0, st>>>(tab, sums + nsums, scale_dev ? kept_from(tab, kept_in_front_of(std::min(count, base + CAP), count, descs)) : tab.tiles);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    nsums += blocks;
  }
  if (!scale_dev) return launch_chained(k_grad_norm, dim3(1), GC_THREADS, 0, st, true, 1, (const double*)sums, nsums, norm_dev);
  bool chained = true;          // only behind the sums: a second part of a long list runs behind a kernel that lets it in at its end
  for (int base = (count - 1) / CAP * CAP; base >= 0; base -= CAP) {
    if (count > CAP) fill(tab, base, std::min(CAP, count - base), descs, G_dev, out_dev);
    const int blocks = std::max(1, std::min(GC_SCALE_BLOCKS, tab.tiles));
    const cudaError_t e = launch_chained(k_grad_scale<CAP>, dim3(blocks), GC_THREADS, 0, st, chained, 1, tab, (const double*)sums, nsums,
                                         max_norm, norm_dev, scale_dev, out_dev == nullptr ? 1 : 0);
    if (e != cudaSuccess) return e;
    chained = false;
  }
  return cudaSuccess;
}

fira_status run(const char* who, int32_t count, const fira_grad_desc* descs, const void* const* G_dev, void* const* out_dev, float max_norm,
                float* norm_dev, float* scale_dev, void* work_dev, size_t work_bytes, void* cuda_stream) {
  const fira_status bad = check_list(who, count, descs, G_dev, out_dev);
  if (bad != FIRA_OK) return bad;
  if (!norm_dev || !work_dev || ((uintptr_t)work_dev & 15) || ((uintptr_t)norm_dev & 3) || ((uintptr_t)scale_dev & 3)) {
    set_error(std::string(who) + ": norm, scale and work must be aligned device pointers (work: 16 bytes)"); return FIRA_ERR_INVALID_ARG;
  }
  if (work_bytes < fira_grad_work_bytes(count)) {
    set_error(std::string(who) + ": workspace too small: " + std::to_string(work_bytes) + " bytes, " + std::to_string(fira_grad_work_bytes(count)) + " needed");
    return FIRA_ERR_WORKSPACE_TOO_SMALL;
  }
  double* sums = static_cast<double*>(work_dev);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = count <= GC_FEW ? run_list<GC_FEW>(count, descs, G_dev, out_dev, max_norm, norm_dev, scale_dev, sums, st)
                                        : run_list<GC_MANY>(count, descs, G_dev, out_dev, max_norm, norm_dev, scale_dev, sums, st);
  if (e != cudaSuccess) { set_error(std::string(who) + ": " + cudaGetErrorString(e)); return FIRA_ERR_CUDA; }
  return FIRA_OK;
}

}  // namespace
}  // namespace fira

using namespace fira;

extern "C" size_t fira_grad_work_bytes(int32_t count) {
  return (size_t)std::max(1, launches_for(std::max(1, count))) * GC_BLOCKS * sizeof(double);
}

extern "C" fira_status fira_grad_norm(int32_t count, const fira_grad_desc* descs, const void* const* G_dev, float* norm_dev,
                                      void* work_dev, size_t work_bytes, void* cuda_stream) {
  return guarded([&] {
    return run("fira_grad_norm", count, descs, G_dev, nullptr, 1.f, norm_dev, nullptr, work_dev, work_bytes, cuda_stream);
  });
}

extern "C" fira_status fira_clip_grads(int32_t count, const fira_grad_desc* descs, const void* const* G_dev, void* const* out_dev,
                                       float max_norm, float* norm_dev, float* scale_dev, void* work_dev, size_t work_bytes,
                                       void* cuda_stream) {
  return guarded([&]() -> fira_status {
    if (!(max_norm > 0.f)) { set_error("fira_clip_grads: max_norm must be > 0"); return FIRA_ERR_INVALID_ARG; }
    if (!scale_dev) { set_error("fira_clip_grads: null argument or empty list"); return FIRA_ERR_INVALID_ARG; }
    const fira_status bad = check_outputs(count, descs, G_dev, out_dev);
    if (bad != FIRA_OK) return bad;
    return run("fira_clip_grads", count, descs, G_dev, out_dev, max_norm, norm_dev, scale_dev, work_dev, work_bytes, cuda_stream);
  });
}
