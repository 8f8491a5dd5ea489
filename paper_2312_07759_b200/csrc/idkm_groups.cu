// Hard assignment with a scale per group of weights: the 4-bit codes and scales one ships where a layer's rows or channels
// differ in size too much for one codebook.  A group of g consecutive weights of a row gets s = max|w| / max|c|, rounded to the
// type the scales are kept in, and every weight the codebook entry nearest to it over s:  q(w) = argmin_j |w - s c_j|.
//
// Arithmetic.  The codebook is sorted once per block; a weight descends a binary tree of the 15 midpoints with r = w / s, four
// steps of a subtraction each.  r is off by at most 2^-21 max|c| (1 / s to two units in the last place, one rounding of the
// difference, one of a midpoint, |r| <= 2 max|c| or beyond every midpoint), so a weight that passes no midpoint within GROUPS_MARGIN = 2^-20 max|c|
// has the nearest entry; any other, a few in 10^5, is compared with all entries in fp64, where the products s c_j are exact and
// ties go to the lowest index.  The result is that of the fp64 comparison for every weight.
//
// What bounds it: instructions, 37 a weight: 8192 x 8192 fp32 in groups of 128 take 103 us, 2.9 TB/s (49 a weight: 153).  Traffic
// (W in, half a byte a weight out) would allow 47.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include "idkm_types.cuh"
#include "../../include/idkm.h"

namespace {

using namespace idkm;

constexpr int GROUPS_BLOCK = 256;
constexpr int GROUPS_LANE = 8;                       // consecutive weights of a lane: its codes are one 32-bit word
constexpr int GROUPS_WARP = 32 * GROUPS_LANE;        // weights of a warp
constexpr float GROUPS_MARGIN = 9.5367431640625e-07f;   // 2^-20

struct GroupsParams {
  const void* W;
  long long rows, ldw;
  int cols;
  const void* C;
  int k;
  int group, n_groups;
  unsigned char* codes;
  long long pitch;
  void* scales;
  void* Wq;
  int vec_in, vec_out;   // rows of W, of Wq, start on 16-byte boundaries
};

struct GroupsTable {
  float c[16];          // the codebook as given; entries that are not finite, and those past k, are NaN
  float tree[16];       // midpoints of the sorted distinct entries, [0] unused: children of node i are 2 i and 2 i + 1
  unsigned long long at;   // the index of the entry at each place of the sorted order, 4 bits each
  float margin, c_max;
  int zero;             // the code of a weight that is 0: the entry nearest to 0
  int sorted;           // the codebook is in order, each entry once: places are codes
  int slow;             // entries so close, or so large or small, that every weight is compared in fp64
};

// Sorts the codebook by counting.  Called by the whole block.
template <class T>
__device__ void groups_table(GroupsTable& t, const void* C, int k) {
  const int tid = threadIdx.x;
  const float inf = __int_as_float(0x7f800000), nan = __int_as_float(0x7fc00000);
  if (tid < 16) {
    const float x = tid < k ? to_f32(reinterpret_cast<const T*>(C)[tid]) : nan;
    t.c[tid] = fabsf(x) < inf ? x : nan;
  }
  __syncthreads();
  if (tid < 32) {
    const float x = tid < 16 ? t.c[tid] : nan;
    bool kept = x == x;   // the first of equal entries
    int rank = 0;
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float y = t.c[j];
      if (y == y) most = fmaxf(most, fabsf(y));
      if (y == x && j < tid) kept = false;
    }
    const unsigned keepers = __ballot_sync(0xffffffffu, kept);
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if ((keepers >> j & 1u) && t.c[j] < x) ++rank;
    // place `rank` of the sorted order; the next larger kept entry
    float up = inf;
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if ((keepers >> j & 1u) && t.c[j] > x) up = fminf(up, t.c[j]);
    const float mid = up < inf ? 0.5f * x + 0.5f * up : inf;   // above the place; inf above the last one
    const bool close = kept && up < inf && !(up - x > 1e-12f * most);
    const int slow = __any_sync(0xffffffffu, close) || !(most > 8.6736174e-19f && most < 1.1529215e18f);   // 2^-60, 2^60
    unsigned lo = 0u, hi = 0u;
    if (kept) {
      if (rank < 8) lo = (unsigned)tid << (4 * rank);
      else hi = (unsigned)tid << (4 * (rank - 8));
    }
    lo = __reduce_or_sync(0xffffffffu, lo);
    hi = __reduce_or_sync(0xffffffffu, hi);
    if (tid < 16) t.tree[tid] = inf;
    // (a codebook symmetric about 0 has a midpoint there, and a pruned layer many weights on it)
    const unsigned size = kept ? __float_as_uint(x) & 0x7fffffffu : 0xffffffffu, least = __reduce_min_sync(0xffffffffu, size);
    const int zero = (int)__reduce_min_sync(0xffffffffu, kept && size == least ? (unsigned)tid : 31u) & 15;
    __syncwarp();
    // the midpoint above place p (0..14) is the node that separates p from p + 1: in-order position p of a tree of 15
    if (kept && rank < 15) {
      const int p = rank + 1, low = __ffs(p) - 1;          // p = odd * 2^low, at depth 3 - low
      t.tree[(1 << (3 - low)) + (p >> (low + 1))] = mid;
    }
    const int sorted = __all_sync(0xffffffffu, !kept || rank == tid);
    if (tid == 0) {
      t.sorted = sorted;
      t.at = (unsigned long long)hi << 32 | lo;
      t.margin = GROUPS_MARGIN * most;
      t.c_max = most;
      t.slow = slow;
      t.zero = zero;
    }
  }
  __syncthreads();
}

__device__ __noinline__ int groups_exact(const GroupsTable& t, float w, float s) {
  double best = 1.0 / 0.0;
  int at = 0;
  for (int j = 0; j < 16; ++j) {
    const double d = fabs((double)w - (double)s * (double)t.c[j]);
    if (d < best) {   // (a NaN is never nearer)
      best = d;
      at = j;
    }
  }
  return at;
}

// s = max|w| / max|c| as the scales' type holds it, and the factor to look weights up by (0: the group needs the exact form).
template <class T>
__device__ __forceinline__ T groups_scale(const GroupsTable& t, float most, float& s, float& inv) {
  const T held = from_f32<T>(t.c_max > 0.f ? __fdiv_rn(most, t.c_max) : 0.f);
  s = to_f32(held);
  inv = (!t.slow && s > 7.8886091e-31f && s < 1.2676506e30f) ? __fdividef(1.f, s) : 0.f;   // 2^-100, 2^100
  return held;
}

// The codes of a lane's eight weights.
__device__ __forceinline__ unsigned groups_codes(const GroupsTable& t, const float (&w)[GROUPS_LANE], float s, float inv) {
  // node 2 i + 1 where the weight lies above the midpoint of node i: the sign of midpoint - w / s, shifted in.  Leaves are 16 to
  // 31, 16 + the place.
  float near = __int_as_float(0x7f800000);
  unsigned node[GROUPS_LANE];
  const float back = -inv;
#pragma unroll
  for (int e = 0; e < GROUPS_LANE; ++e) node[e] = 1u;
#pragma unroll
  for (int level = 0; level < 4; ++level) {
    float d[GROUPS_LANE];
#pragma unroll
    for (int e = 0; e < GROUPS_LANE; ++e) {
      d[e] = __fmaf_rn(w[e], back, t.tree[node[e]]);   // (one rounding less than a product and a difference)
      node[e] = __funnelshift_l(__float_as_uint(d[e]), node[e], 1);
    }
#pragma unroll
    for (int e = 0; e < GROUPS_LANE; e += 2) asm("min.abs.f32 %0, %0, %1, %2;" : "+f"(near) : "f"(d[e]), "f"(d[e + 1]));
  }
  unsigned out = 0u;
  if (t.sorted) {
#pragma unroll
    for (int e = 0; e < GROUPS_LANE; ++e) out += node[e] << (4 * e);
    out -= 0x11111110u;   // 16 of every leaf
  } else {
#pragma unroll
    for (int e = 0; e < GROUPS_LANE; ++e) out |= ((unsigned)(t.at >> (4u * (node[e] & 15u))) & 15u) << (4 * e);
  }
  if (!(near > t.margin) || inv == 0.f) {   // one of them at least is close to a midpoint, or the group needs the exact form
    const bool finite = fabsf(s) < __int_as_float(0x7f800000);
#pragma unroll 1
    for (int e = 0; e < GROUPS_LANE; ++e) {
      const float x = e == 0 ? w[0] : e == 1 ? w[1] : e == 2 ? w[2] : e == 3 ? w[3] : e == 4 ? w[4] : e == 5 ? w[5] : e == 6 ? w[6] : w[7];
      out = (out & ~(15u << (4 * e))) | (unsigned)(!finite || s == 0.f ? 0 : x == 0.f ? t.zero : groups_exact(t, x, s)) << (4 * e);
    }
  }
  return out;
}

// Eight weights of a row from column c on; zeros past its end.
template <class TW>
__device__ __forceinline__ void groups_load(const TW* row, int c, int cols, int vec, float (&w)[GROUPS_LANE]) {
  if (vec && c + GROUPS_LANE <= cols) {
    constexpr int N = Vec16<TW>::N;
#pragma unroll
    for (int q = 0; q < GROUPS_LANE / N; ++q) {
      Vec16<TW> x;
      x.raw = __ldg(reinterpret_cast<const uint4*>(row + c) + q);
#pragma unroll
      for (int e = 0; e < N; ++e) w[q * N + e] = to_f32(x.e[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < GROUPS_LANE; ++e) w[e] = c + e < cols ? to_f32(row[c + e]) : 0.f;
  }
}

template <class TW>
__device__ __forceinline__ void groups_store_wq(const GroupsTable& t, TW* row, int c, int cols, int vec, unsigned codes, float s) {
  float q[GROUPS_LANE];
#pragma unroll
  for (int e = 0; e < GROUPS_LANE; ++e) q[e] = s * t.c[codes >> (4 * e) & 15u];
  if (vec && c + GROUPS_LANE <= cols) {
    constexpr int N = Vec16<TW>::N;
#pragma unroll
    for (int v = 0; v < GROUPS_LANE / N; ++v) {
      Vec16<TW> x;
#pragma unroll
      for (int e = 0; e < N; ++e) x.e[e] = from_f32<TW>(q[v * N + e]);
      reinterpret_cast<uint4*>(row + c)[v] = x.raw;
    }
  } else {
#pragma unroll
    for (int e = 0; e < GROUPS_LANE; ++e)
      if (c + e < cols) row[c + e] = from_f32<TW>(q[e]);
  }
}

// Codes of the weights past a row's end are 0.
__device__ __forceinline__ unsigned groups_keep(unsigned codes, int c, int cols) {
  return c + GROUPS_LANE <= cols ? codes : c >= cols ? 0u : codes & ((1u << (4 * (cols - c))) - 1u);
}

// The larger of two sizes (what it takes may have a sign); a NaN stays.
__device__ __forceinline__ float groups_larger(float a, float b) {
  float r;
  asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return fabsf(r);
}
__device__ __forceinline__ float groups_largest(const float (&w)[GROUPS_LANE]) {
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < GROUPS_LANE; e += 2) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(w[e]), "f"(w[e + 1]));
  return most;
}

// Groups of 32, 64, 128 or 256 weights: L = g / 8 neighbouring lanes share one.  A warp takes GROUPS_PIECES pieces of 256 weights of a
// row at a time, all of them asked for before the first is looked at.
constexpr int GROUPS_PIECES = 2;   // (1, 3, 4: 114, 104, 105 us where 2 take 103)
template <class TW>
struct GroupsRaw {   // a lane's eight weights as they lie in memory
  uint4 v[GROUPS_LANE / Vec16<TW>::N];
};
template <class TW>
__device__ __noinline__ GroupsRaw<TW> groups_edge(const TW* row, int c, int cols) {   // one by one; zeros past the row's end
  GroupsRaw<TW> r;
  constexpr int N = Vec16<TW>::N;
#pragma unroll
  for (int q = 0; q < GROUPS_LANE / N; ++q) {
    Vec16<TW> x;
#pragma unroll
    for (int e = 0; e < N; ++e) x.e[e] = c + q * N + e < cols ? row[c + q * N + e] : from_f32<TW>(0.f);
    r.v[q] = x.raw;
  }
  return r;
}
template <class TW, class T>
__global__ void __launch_bounds__(GROUPS_BLOCK, 4) idkm_groups_short(const __grid_constant__ GroupsParams p) {
  constexpr int N = Vec16<TW>::N, V = GROUPS_LANE / N;
  __shared__ GroupsTable t;
  const int lane = threadIdx.x & 31, L = p.group / GROUPS_LANE, shift = __ffs(p.group) - 1, cols = p.cols, span = GROUPS_PIECES * GROUPS_WARP;
  const unsigned per_row = (unsigned)((cols + span - 1) / span), n_warps = gridDim.x * (GROUPS_BLOCK / 32);
  // every n_warps-th span of a row, row by row
  const unsigned from = blockIdx.x * (GROUPS_BLOCK / 32) + (threadIdx.x >> 5), rows_on = n_warps / per_row, on = n_warps - rows_on * per_row;
  long long row = from / per_row;
  unsigned part = from - (unsigned)row * per_row;
  GroupsRaw<TW> raw[GROUPS_PIECES];
  auto fetch = [&](const TW* w, int c0) {
#pragma unroll
    for (int q = 0; q < GROUPS_PIECES; ++q) {
      const int c = c0 + q * GROUPS_WARP;
      const int whole = p.vec_in && c + GROUPS_LANE <= cols;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        raw[q].v[v] = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                     : "+r"(raw[q].v[v].x), "+r"(raw[q].v[v].y), "+r"(raw[q].v[v].z), "+r"(raw[q].v[v].w)
                     : "l"(w + c + v * N), "r"(whole));
      }
    }
    if (!p.vec_in || c0 + (GROUPS_PIECES - 1) * GROUPS_WARP + GROUPS_LANE > cols) {
#pragma unroll
      for (int q = 0; q < GROUPS_PIECES; ++q) {
        const int c = c0 + q * GROUPS_WARP;
        if (c < cols && (!p.vec_in || c + GROUPS_LANE > cols)) raw[q] = groups_edge(w, c, cols);
      }
    }
  };
  for (bool first = true;; first = false) {
    const int c0 = (int)part * span + lane * GROUPS_LANE;
    if (row < p.rows) fetch(reinterpret_cast<const TW*>(p.W) + row * p.ldw, c0);
    if (first) groups_table<T>(t, p.C, p.k);   // (all warps of the block, those without work too, while the first weights are on their way)
    if (row >= p.rows) break;
    unsigned char* to = p.codes + row * p.pitch;
    T* scales = reinterpret_cast<T*>(p.scales) + row * p.n_groups;
#pragma unroll
    for (int q = 0; q < GROUPS_PIECES; ++q) {
      const int c = c0 + q * GROUPS_WARP;
      if ((int)part * span + q * GROUPS_WARP >= cols) break;   // (the whole warp)
      float w[GROUPS_LANE];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        Vec16<TW> x;
        x.raw = raw[q].v[v];
#pragma unroll
        for (int e = 0; e < N; ++e) w[v * N + e] = to_f32(x.e[e]);
      }
      float most = groups_largest(w);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, most, o);
        if (o < L) most = groups_larger(most, other);
      }
      float s, inv;
      const T held = groups_scale<T>(t, most, s, inv);
      const unsigned codes = groups_keep(groups_codes(t, w, s, inv), c, cols);
      if (c < cols) {
        if ((lane & (L - 1)) == 0) scales[c >> shift] = held;
        if (p.Wq) groups_store_wq(t, reinterpret_cast<TW*>(p.Wq) + row * cols, c, cols, p.vec_out, codes, s);
      }
      if (c < 2 * (int)p.pitch) *reinterpret_cast<unsigned*>(to + c / 2) = codes;
    }
    row += rows_on;
    part += on;
    if (part >= per_row) {
      part -= per_row;
      ++row;
    }
  }
}

// Longer groups: a block each, which reads the group twice (the second time from L2).
template <class TW, class T>
__global__ void __launch_bounds__(GROUPS_BLOCK) idkm_groups_long(const __grid_constant__ GroupsParams p) {
  __shared__ GroupsTable t;
  __shared__ float part[GROUPS_BLOCK / 32];
  groups_table<T>(t, p.C, p.k);
  for (long long i = blockIdx.x; i < p.rows * p.n_groups; i += gridDim.x) {
    const long long row = i / p.n_groups;
    const int g = (int)(i - row * p.n_groups), begin = g * p.group;
    const int end = p.cols - begin < p.group ? p.cols : begin + p.group, end_codes = g + 1 == p.n_groups ? 2 * (int)p.pitch : end;
    const TW* wr = reinterpret_cast<const TW*>(p.W) + row * p.ldw;
    float most = 0.f;
    for (int c = begin + threadIdx.x * GROUPS_LANE; c < end; c += GROUPS_BLOCK * GROUPS_LANE) {
      float w[GROUPS_LANE];
      groups_load(wr, c, end, p.vec_in, w);
      most = groups_larger(most, groups_largest(w));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = groups_larger(most, __shfl_xor_sync(0xffffffffu, most, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = most;
    __syncthreads();
    most = 0.f;
#pragma unroll
    for (int q = 0; q < GROUPS_BLOCK / 32; ++q) most = groups_larger(most, part[q]);
    __syncthreads();
    float s, inv;
    const T held = groups_scale<T>(t, most, s, inv);
    if (threadIdx.x == 0) reinterpret_cast<T*>(p.scales)[i] = held;
    for (int c = begin + threadIdx.x * GROUPS_LANE; c < end_codes; c += GROUPS_BLOCK * GROUPS_LANE) {
      float w[GROUPS_LANE];
      groups_load(wr, c, end, p.vec_in, w);
      const unsigned codes = groups_keep(groups_codes(t, w, s, inv), c, end);
      if (p.Wq) groups_store_wq(t, reinterpret_cast<TW*>(p.Wq) + row * p.cols, c, end, p.vec_out, codes, s);
      *reinterpret_cast<unsigned*>(p.codes + row * p.pitch + c / 2) = codes;
    }
  }
}

}  // namespace

extern "C" int64_t idkm_group_codes_pitch(int64_t cols) { return cols < 1 ? 0 : (cols + 31) / 32 * 16; }

extern "C" int idkm_assign_groups(const void* W, int w_type, int64_t rows, int64_t cols, int64_t ldw, const void* C, int k, int type,
                                  int64_t group, unsigned char* codes_out, void* scales_out, void* Wq_out, void* cuda_stream) {
  if (!W || !C || !codes_out || !scales_out) return IDKM_ERR_NULL;
  if (k < 1 || k > 16 || !elem_known(w_type) || !elem_known(type)) return IDKM_ERR_UNSUPPORTED;
  if (rows < 1 || cols < 1 || ldw < cols || group < 1 || cols > INT32_MAX - 4096 || cols > (INT64_C(1) << 50) / rows) return IDKM_ERR_SHAPE;
  if (group < cols && group != 32 && group != 64 && group % 128 != 0) return IDKM_ERR_UNSUPPORTED;
  if (Wq_out == W || Wq_out == (void*)codes_out || Wq_out == scales_out) return IDKM_ERR_PARAM;
  const int wb = elem_bytes(w_type), tb = elem_bytes(type);
  if (((uintptr_t)W | (uintptr_t)Wq_out) % wb || ((uintptr_t)C | (uintptr_t)scales_out) % tb || (uintptr_t)codes_out % 16) return IDKM_ERR_ALIGN;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
    return IDKM_ERR_CUDA;
  GroupsParams p;
  p.W = W; p.rows = rows; p.cols = (int)cols; p.ldw = ldw; p.C = C; p.k = k;
  p.pitch = idkm_group_codes_pitch(cols);
  // one scale per row: a group that ends with the row (32 codes at a time are kept whole)
  p.group = (int)(group >= cols ? (cols <= 32 ? 32 : cols <= 64 ? 64 : (cols + 127) / 128 * 128) : group);
  p.n_groups = (int)((cols + p.group - 1) / p.group);
  p.codes = codes_out; p.scales = scales_out; p.Wq = Wq_out;
  p.vec_in = (uintptr_t)W % 16 == 0 && ldw * wb % 16 == 0;
  p.vec_out = (uintptr_t)Wq_out % 16 == 0 && cols * wb % 16 == 0;
  const bool shorter = p.group <= GROUPS_WARP && GROUPS_WARP % p.group == 0;
  const long long per_row = (cols + GROUPS_PIECES * GROUPS_WARP - 1) / (GROUPS_PIECES * GROUPS_WARP);
  const long long jobs = shorter ? (rows * per_row + GROUPS_BLOCK / 32 - 1) / (GROUPS_BLOCK / 32) : rows * p.n_groups, most = (long long)sms * (shorter ? 4 : 8);
  const int grid = (int)(jobs < most ? jobs : most);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  return with_type(w_type, [&](auto* w) {
    return with_type(type, [&](auto* c) {
      using TW = std::remove_pointer_t<decltype(w)>;
      using T = std::remove_pointer_t<decltype(c)>;
      if (shorter) idkm_groups_short<TW, T><<<grid, GROUPS_BLOCK, 0, st>>>(p);
      else idkm_groups_long<TW, T><<<grid, GROUPS_BLOCK, 0, st>>>(p);
      return cudaGetLastError() == cudaSuccess ? IDKM_OK : IDKM_ERR_CUDA;
    });
  });
}
