// Distillation from a teacher's top logits: the loss by which a quantised network is trained from the full-precision one, and
// its gradient with respect to the student's logits.  For a row z in R^V, teacher entries (i_j, t_j), temperature tau:
//   p_j = softmax_j(t_j / tau) over the entries with 0 <= i_j < V,   q_v = softmax_v(z_v / tau),
//   loss = tau^2 sum_j p_j (ln p_j - ln q_{i_j}),    dz_v = w tau (q_v - sum_{j: i_j = v} p_j).
// A row without entries (or whose t_j are all -inf) has loss 0 and gradient 0; p_j below 2^-126 of the largest is 0 in the loss.  As sum_j p_j = 1,
//   loss = tau^2 (sum_j p_j (t_j - z_{i_j}) / tau - L_t + L_z),   L_t, L_z the logarithms of the two normalisers.
//
// One pass over z.  A row is a cluster of as few blocks as hold it (8 vectors of 16 bytes a thread, up to 8 blocks); a thread sums
// e_v = exp((z_v - m) / tau), m its largest element, and keeps the e_v in registers.  Warps and blocks join (m, sum) and the teacher's
// part, which every block has whole but for the entries' products, for which it takes the entries of its own part of the row;
// blocks send theirs into the others' shared memory.  Then q_v = e_v exp((m - M) / tau) / S: an element costs one exponential, 2
// or 4 bytes in, as many out.  Entries' places are written again after the dense part.
// What bounds it: at 4096 x 32000 bf16 logits 111 us, 4.7 TB/s: the elements' instructions (about 6 each) and the chain of a row's
// two barriers and one exchange, behind which the next row's entries are prepared (8 us).  Measured when this took 124 us: 4 vectors
// a thread and twice the blocks 269 us (a row's bookkeeping is per warp), exponentials computed twice instead of kept, for three blocks
// of a multiprocessor instead of two, 147, one block of 512 threads instead of two of 256 131, warps' parts joined by every thread
// from shared memory instead of by lanes 136.  The gradient alone is streamed: 1021 x 100003 fp16 66 us, 6.2 TB/s, as fast as a copy.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <type_traits>
#include "idkm_per_device.h"
#include "idkm_types.cuh"
#include "../../include/idkm.h"

namespace {

using namespace idkm;

constexpr int DISTILL_MAX_CLUSTER = 8;
constexpr int DISTILL_POLLS = 1 << 19;   // (each waits for some time itself, 2 us: about a second)
constexpr float LOG2E = 1.4426950408889634f, LOG2E_LOW = (float)(1.4426950408889634 - (double)1.4426950408889634f);

struct DistillParams {
  const void* z;
  long long rows, vocab, ldz;
  const void* idx;
  int idx_bytes;
  const void* t;
  int t_type, top;
  float tau, c2, c2_low;   // log2(e) / tau, and what it lacks
  const float* weight;
  float* loss;
  float* stats;         // read by the gradient, written by the loss
  void* dz;
  long long lddz;
  int parts;            // blocks of a row
  int trips;            // times a block goes through its registers' worth of vectors
};

enum DistillMode { DISTILL_LOSS, DISTILL_GRAD, DISTILL_STEP };

__device__ __forceinline__ float distill_ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Sums of exp((x - m) c2) and of the teacher's products against the largest x, m.  An empty part is (-inf, 0, 0); a part with a
// NaN has one in its sum.
struct DistillPart {
  float m, s;        // student
  float tm, ts, ta;  // teacher: largest t, sum of exp((t - tm) / tau), sum of that times t - z over the block's own entries with z > -inf
  float tx;          // ... largest t of those with z = -inf
};

// exp((m - top) / tau), 0 where m is -inf (an empty part, whatever top is).
__device__ __forceinline__ float distill_scale(float m, float top, float c2) {
  return m == __int_as_float(0xff800000) ? 0.f : distill_ex2((m - top) * c2);
}

// A part that another scale multiplies: 0 stays 0 whatever the scale; NaN stays.
__device__ __forceinline__ float distill_scaled(float s, float f) { return s == 0.f ? 0.f : s * f; }

__device__ __forceinline__ float distill_warp_max(float x) {   // (NaN aside)
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float distill_warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Joins the warps' parts, lane i < WARPS holding that of warp i (other lanes an empty one): all lanes get the block's.
template <int WARPS>
__device__ __forceinline__ DistillPart distill_join(DistillPart a, float c2) {
  const float M = distill_warp_max(a.m), T = distill_warp_max(a.tm);
  const float g = distill_scale(a.tm, T, c2);
  a.s = distill_scaled(a.s, distill_scale(a.m, M, c2));
  a.ts = distill_scaled(a.ts, g);
  a.ta = g == 0.f ? 0.f : a.ta * g;   // (sums that overflowed next to the warp's largest t, too)
  a.tx = distill_warp_max(a.tx);
#pragma unroll
  for (int o = WARPS >> 1; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.ts += __shfl_xor_sync(0xffffffffu, a.ts, o);
    a.ta += __shfl_xor_sync(0xffffffffu, a.ta, o);
  }
  a.m = M;
  a.tm = T;
  a.s = __shfl_sync(0xffffffffu, a.s, 0);
  a.ts = __shfl_sync(0xffffffffu, a.ts, 0);
  a.ta = __shfl_sync(0xffffffffu, a.ta, 0);
  if (distill_scale(a.tx, T, c2) > 0.f) a.ta = __int_as_float(0x7f800000);   // (mass that is not 0 next to the row's largest)
  return a;
}

// Two floats at once.
__device__ __forceinline__ float2 distill_add(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 c, a, b;\n\tmov.b64 {%0, %1}, c;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 distill_mul(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 c, a, b;\n\tmov.b64 {%0, %1}, c;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}

// 16 bytes of a row as pairs, and their largest element (NaN aside).
__device__ __forceinline__ float2 distill_pair(const uint4& x, int i, float*) {
  return i == 0 ? make_float2(__uint_as_float(x.x), __uint_as_float(x.y)) : make_float2(__uint_as_float(x.z), __uint_as_float(x.w));
}
__device__ __forceinline__ unsigned distill_word(const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }
__device__ __forceinline__ float2 distill_pair(const uint4& x, int i, __nv_bfloat16*) {
  const unsigned w = distill_word(x, i);
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 distill_pair(const uint4& x, int i, __half*) {
  const unsigned w = distill_word(x, i);
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ float distill_top(const uint4& x, float*) {
  return fmaxf(fmaxf(__uint_as_float(x.x), __uint_as_float(x.y)), fmaxf(__uint_as_float(x.z), __uint_as_float(x.w)));
}
__device__ __forceinline__ float distill_top(const uint4& x, __nv_bfloat16*) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&x);
  const float2 t = __bfloat1622float2(__hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
  return fmaxf(t.x, t.y);
}
__device__ __forceinline__ float distill_top(const uint4& x, __half*) {
  const __half2* h = reinterpret_cast<const __half2*>(&x);
  const float2 t = __half22float2(__hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
  return fmaxf(t.x, t.y);
}
__device__ __forceinline__ uint4 distill_pack(const float2* v, float*) {
  return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
}
__device__ __forceinline__ uint4 distill_pack(const float2* v, __nv_bfloat16*) {
  uint4 r;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __float22bfloat162_rn(v[i]);
  return r;
}
__device__ __forceinline__ uint4 distill_pack(const float2* v, __half*) {
  uint4 r;
  __half2* h = reinterpret_cast<__half2*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __float22half2_rn(v[i]);
  return r;
}

// Vectors that reach past a row's ends, element by element; -inf for what is not the row's.  `first`: the row's index of the
// vector's first element, which is below 0 where the row does not begin on a 16-byte boundary.  (Not inlined: the compiler
// would run these loads, predicated off, for every vector -- 41 instructions an element instead of about 9.)
template <class T>
__device__ __noinline__ uint4 distill_load_edge(const T* z, int first, int vocab) {
  constexpr int N = Vec16<T>::N;
  Vec16<T> x;
#pragma unroll
  for (int e = 0; e < N; ++e) x.e[e] = first + e >= 0 && first + e < vocab ? z[first + e] : from_f32<T>(__int_as_float(0xff800000));
  return x.raw;
}
template <class T>
__device__ __noinline__ void distill_store_edge(T* dz, int first, int vocab, uint4 v) {
  constexpr int N = Vec16<T>::N;
  Vec16<T> x;
  x.raw = v;
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (first + e >= 0 && first + e < vocab) dz[first + e] = x.e[e];
}

// A row's geometry on 16-byte boundaries: vector v holds the elements [v N - lead, (v + 1) N - lead); those in [full0, full1) lie
// whole in the row, the first and the last may not.
template <class T>
struct DistillGrid {
  static constexpr int N = Vec16<T>::N;
  const T* z;
  int lead, vectors, full0, full1;
  __device__ __forceinline__ DistillGrid(const DistillParams& p, long long row) {
    z = reinterpret_cast<const T*>(p.z) + row * p.ldz;
    lead = (int)(((uintptr_t)z & 15u) / sizeof(T));
    vectors = ((int)p.vocab + lead + N - 1) / N;
    full0 = lead ? 1 : 0;
    full1 = ((int)p.vocab + lead) / N;
  }
  __device__ __forceinline__ const uint4* at(int v) const { return reinterpret_cast<const uint4*>(z - lead) + v; }
  __device__ __forceinline__ bool edge(int v) const { return v < vectors && (v < full0 || v >= full1); }
  __device__ __forceinline__ int first(int v) const { return v * N - lead; }
};

// An entry of the teacher as it lies in memory.  (Nothing is computed from it before the turn it is used in: the first use
// would wait for the load.)
struct DistillRaw {
  uint2 v;
  unsigned t;
};
__device__ __forceinline__ DistillRaw distill_raw(const DistillParams& p, long long row, int j) {
  DistillRaw r;
  r.v = make_uint2(0xffffffffu, 0xffffffffu);
  r.t = 0u;
  if (j < p.top && row < p.rows) {
    const long long i = row * p.top + j;
    if (p.idx_bytes == 8) r.v = __ldg(reinterpret_cast<const uint2*>(p.idx) + i);
    else r.v.x = __ldg(reinterpret_cast<const unsigned*>(p.idx) + i);
    if (p.t_type == ELEM_F32) r.t = __ldg(reinterpret_cast<const unsigned*>(p.t) + i);
    else r.t = __ldg(reinterpret_cast<const unsigned short*>(p.t) + i);
  }
  return r;
}
// Its index, -1 where it does not count, and its logit, -inf there.
__device__ __forceinline__ void distill_entry(const DistillParams& p, const DistillRaw& r, int& at, float& t) {
  const int high = p.idx_bytes == 8 ? (int)r.v.y : (int)r.v.x >> 31;
  const bool counts = high == 0 && r.v.x < (unsigned)p.vocab;
  at = counts ? (int)r.v.x : -1;
  t = p.t_type == ELEM_F32 ? __uint_as_float(r.t) : p.t_type == ELEM_BF16 ? __uint_as_float(r.t << 16) : __half2float(__ushort_as_half((unsigned short)r.t));
  t = counts ? t : __int_as_float(0xff800000);
}

// Whether an index is among a block's entries twice: a table with open addressing in shared memory, at most a quarter full.
constexpr int DISTILL_TABLE = 4 * IDKM_DISTILL_MAX_TOP;
__device__ __forceinline__ int distill_enter(int* table, int at, int* twice) {   // the place it got
  unsigned h = ((unsigned)at * 2654435761u) >> 22;
  static_assert(DISTILL_TABLE == 1 << 10, "ten bits of the product");
  while (true) {   // (ends: there are more places than entries)
    const int old = atomicCAS(table + h, -1, at);
    if (old == at) {
      *twice = 1;
      return -1;
    }
    if (old == -1) return (int)h;
    h = (h + 1) % DISTILL_TABLE;
  }
}

// The sum of the probabilities exp((t - tm) / tau) / ts of the entries at place `at`, entry j's; -1 where one before j is at the
// same place (the first of them writes).
__device__ __noinline__ float distill_taken(const int* s_at, const float* s_t, int top, int at, int j, float tm, float inv_ts, float c2) {
  float taken = 0.f;
  for (int i = 0; i < top; ++i)
    if (s_at[i] == at) {
      if (i < j) return -1.f;
      taken += distill_ex2((s_t[i] - tm) * c2) * inv_ts;
    }
  return taken;
}

template <class T>
__device__ __forceinline__ unsigned distill_lowest() {   // -inf, as often as a word holds it
  return sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;
}

// The loss, and with STEP the gradient.  Blocks stay: a cluster takes every n-th row, and while it works on one the vectors
// of the next are on their way into shared memory, every thread fetching what it will read itself, and the entries of the next and
// the one after into registers.  LONG: rows of more vectors than the cluster's threads hold, taken in trips.
template <class T, int BLOCK, int NV, int MODE, bool LONG>
__global__ void __launch_bounds__(BLOCK, 512 / BLOCK) idkm_distill_rows(const __grid_constant__ DistillParams p) {
  constexpr int N = Vec16<T>::N, H = N / 2, WARPS = BLOCK / 32;
  T* const type = nullptr;
  static_assert(BLOCK >= IDKM_DISTILL_MAX_TOP, "an entry a thread");
  const float none = __int_as_float(0xff800000);
  extern __shared__ uint4 slots[];                              // [NV][BLOCK]
  __shared__ __align__(16) int s_at[2][IDKM_DISTILL_MAX_TOP];   // the entries' indices and logits, by turns: a row's are written
  __shared__ float s_t[2][IDKM_DISTILL_MAX_TOP];                // while slower threads read the last one's
  __shared__ int s_table[MODE == DISTILL_STEP ? DISTILL_TABLE : 1], s_twice[2];
  __shared__ DistillPart s_warp[2][WARPS];
  __shared__ __align__(16) float4 s_part[2][DISTILL_MAX_CLUSTER];   // (m, s, ta) of the cluster's blocks
  __shared__ __align__(8) unsigned long long s_bar[2];              // complete when those of a row are there
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, parts = p.parts, part = blockIdx.x % (unsigned)parts;
  const long long n_clusters = gridDim.x / (unsigned)parts;
  long long row = blockIdx.x / (unsigned)parts;
  const float c2 = p.c2;
  const int trips = LONG ? p.trips : 1, v0 = part * NV * BLOCK * trips;
  const uint32_t slot = (uint32_t)__cvta_generic_to_shared(slots + tid);

  // this thread's vectors of a trip: v + q BLOCK, whole ones for q < n (but for the first, if the row begins inside it)
  auto vector = [&](int trip) { return v0 + trip * NV * BLOCK + tid; };
  auto whole = [&](const DistillGrid<T>& g, int v) {
    const int end = min(g.full1, v0 + NV * BLOCK * trips), n = (end - v + BLOCK - 1) / BLOCK;
    return end <= v ? 0 : n;
  };
  auto fetch = [&](long long r, int trip) {
    const DistillGrid<T> g(p, r);
    const int v = vector(trip), n = whole(g, v);
    const uint4* from = g.at(v);
#pragma unroll
    for (int q = 0; q < NV; ++q)
      if (q < n && (q > 0 || v >= g.full0))
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot + q * BLOCK * 16), "l"(from + q * BLOCK) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (row < p.rows) fetch(row, 0);
  int at, at1;   // the entries of this row and of the next; those of the row after as they come
  float t, t1, w = 1.f, w1 = 1.f;
  DistillRaw raw;
  T own = from_f32<T>(0.f), own1 = own;   // the student's logits at the entries' places, if this block's part of the row holds them
  auto has = [&](const DistillGrid<T>& g, int place) {
    const int v = (place + g.lead) / N;
    return place >= 0 && v >= v0 && v < v0 + NV * BLOCK * trips;
  };
  {
    const DistillRaw r0 = distill_raw(p, row, tid);
    raw = distill_raw(p, row + n_clusters, tid);
    distill_entry(p, r0, at, t);
    if (row < p.rows) {
      const DistillGrid<T> g(p, row);
      if (has(g, at)) own = g.z[at];
      if (MODE == DISTILL_STEP && p.weight) w = p.weight[row];
    }
  }
  if (MODE == DISTILL_STEP) {
    for (int i = tid; i < DISTILL_TABLE; i += BLOCK) s_table[i] = -1;
    if (tid < 2) s_twice[tid] = 0;
    __syncthreads();
  }
  const uint32_t bar = (uint32_t)__cvta_generic_to_shared(s_bar);
  uint32_t there = 0, there_bar = 0, phase = 0;
  bool lost = false;   // a wait ran out (it does not: a cluster's blocks run together); later ones do not wait, nothing more is sent
  if (parts > 1) {
    if (tid == 0) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar + 8) : "memory");
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // (every block of the cluster runs, its barriers are ready)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const int peer = tid < parts ? tid : 0;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(&s_part[0][part])), "r"(peer));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there_bar) : "r"(bar), "r"(peer));
  }
  for (int turn = 0; row < p.rows; row += n_clusters, turn ^= 1) {
    const DistillGrid<T> g(p, row);
    const long long next = row + n_clusters;
    const bool mine = has(g, at);
    int entered = -1;
    if (tid < p.top) {
      s_at[turn][tid] = at;
      s_t[turn][tid] = t;
      if (MODE == DISTILL_STEP && mine) entered = distill_enter(s_table, at, s_twice + turn);
    }

    uint4 x[NV];
    float2 e[LONG || MODE == DISTILL_LOSS ? 1 : NV * H];
    auto read = [&](int trip) {   // what fetch() brought
      const int v = vector(trip), n = whole(g, v);
      if (n >= NV && v >= g.full0) {
#pragma unroll
        for (int q = 0; q < NV; ++q) x[q] = slots[q * BLOCK + tid];
        return;
      }
      const unsigned low = distill_lowest<T>();
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        x[q] = make_uint4(low, low, low, low);
        if (q < n && (q > 0 || v >= g.full0)) x[q] = slots[q * BLOCK + tid];
      }
      if (v < g.full0 || (g.vectors > g.full1 && g.full1 >= v && (g.full1 - v) % BLOCK == 0)) {   // (a thread at either end of the row)
#pragma unroll
        for (int q = 0; q < NV; ++q)
          if (g.edge(v + q * BLOCK) && v + q * BLOCK < v0 + NV * BLOCK * trips) x[q] = distill_load_edge(g.z, g.first(v + q * BLOCK), (int)p.vocab);
      }
    };
    float m = none, sum = 0.f;
    for (int trip = 0; trip < trips; ++trip) {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      read(trip);
      float top = m;
#pragma unroll
      for (int q = 0; q < NV; ++q) top = fmaxf(top, distill_top(x[q], type));
      if (LONG) sum = distill_scaled(sum, distill_scale(m, top, c2));
      m = top;
      const float from = top == none ? 0.f : -top;
      float2 acc = make_float2(0.f, 0.f);
#pragma unroll
      for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const float2 d = distill_mul(distill_add(distill_pair(x[q], i, type), make_float2(from, from)), make_float2(c2, c2));
          const float2 y = make_float2(distill_ex2(d.x), distill_ex2(d.y));
          acc = distill_add(acc, y);
          if constexpr (!LONG && MODE == DISTILL_STEP) e[q * H + i] = y;
        }
      sum += acc.x + acc.y;
      if (LONG && trip + 1 < trips) fetch(row, trip + 1);   // (what was in the slots has been used)
      else if (next < p.rows) fetch(next, 0);
    }
    // the warp's: the largest first, then one scale a thread
    DistillPart a;
    a.m = distill_warp_max(m);
    a.s = distill_warp_sum(distill_scaled(sum, distill_scale(m, a.m, c2)));
    a.tm = none;
    a.ts = a.ta = 0.f;
    a.tx = none;
    if (warp * 32 < p.top) {
      a.tm = distill_warp_max(t);
      const float u = t == none ? 0.f : distill_ex2((t - a.tm) * c2);
      a.ts = distill_warp_sum(u);
      const float z = to_f32(own);
      a.ta = distill_warp_sum(mine && t != none && z != none ? u * (t - z) : 0.f);
      a.tx = distill_warp_max(mine && z == none ? t : none);
    }
    if (lane == 0) s_warp[turn][warp] = a;
    __syncthreads();
    const DistillPart empty = {none, 0.f, none, 0.f, 0.f, none};
    a = distill_join<WARPS>(lane < WARPS ? s_warp[turn][lane] : empty, c2);
    if (parts > 1 && warp == 0 && !lost) {
      // (the next row's parts go to the other turn's places; those of the row after are sent once every block has sent the next
      // row's, and so has read these.  Sent with their arrival: a cluster barrier would wait for this thread's stores to dz too)
      if (tid == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar + 8 * turn), "r"(16 * parts) : "memory");
      if (tid < parts)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                     ::"r"(there + turn * (uint32_t)sizeof(s_part[0])), "f"(a.m), "f"(a.s), "f"(a.ta), "f"(0.f), "r"(there_bar + 8 * turn) : "memory");
    }
    const bool some = !(a.tm == none && a.ts == 0.f);
    float taken = -1.f;
    if (MODE == DISTILL_STEP && mine) {   // (the table and the other turn's flag are emptied for the next row, whose entries come after the second barrier)
      if (some) {
        const float inv = __fdividef(1.f, a.ts);
        taken = s_twice[turn] ? distill_taken(s_at[turn], s_t[turn], p.top, at, tid, a.tm, inv, c2) : distill_ex2((t - a.tm) * c2) * inv;
      }
      if (entered >= 0) s_table[entered] = -1;
    }
    if (MODE == DISTILL_STEP && tid == 0) s_twice[turn ^ 1] = 0;
    // while the parts are on their way: the next row's entries, the one after asked for
    if (next < p.rows) {
      if (warp * 32 < p.top) {
        distill_entry(p, raw, at1, t1);
        raw = distill_raw(p, next + n_clusters, tid);
        const DistillGrid<T> g1(p, next);
        if (has(g1, at1)) own1 = g1.z[at1];
      } else {
        at1 = -1;
        t1 = none;
      }
      if (MODE == DISTILL_STEP && p.weight) w1 = p.weight[next];
    }
    if (parts > 1) {
      bool ok = lost;
      for (int i = 0; i < DISTILL_POLLS && !ok; ++i) {
        unsigned done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done)
                     : "r"(bar + 8 * turn), "r"(phase >> turn & 1u)
                     : "memory");
        ok = done != 0;
      }
      lost |= !ok;
      phase ^= 1u << turn;
      // (every block holds the teacher's sums whole: only the products add up)
      float M = none;
      for (int q = 0; q < parts; ++q) M = fmaxf(M, s_part[turn][q].x);
      a.s = a.ta = 0.f;
      for (int q = 0; q < parts; ++q) {
        const float4 b = s_part[turn][q];
        a.s += distill_scaled(b.y, distill_scale(b.x, M, c2));
        a.ta += b.z;
      }
      a.m = M;
      if (lost) a.s = __int_as_float(0x7fc00000);
      if (next >= p.rows) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    }
    if (MODE == DISTILL_STEP) {
      const float wt = p.tau * w, scale = __fdividef(wt, a.s), f = LONG ? scale : distill_scale(m, a.m, c2) * scale;
      T* dz = reinterpret_cast<T*>(p.dz) + row * p.lddz;
      const bool same = (((uintptr_t)dz ^ (uintptr_t)g.z) & 15u) == 0;   // vectors of dz lie as those of z do
      for (int trip = 0; trip < trips; ++trip) {
        const int v = vector(trip), n = whole(g, v);
        if constexpr (LONG) {
          const unsigned low = distill_lowest<T>();
#pragma unroll
          for (int q = 0; q < NV; ++q) {
            x[q] = make_uint4(low, low, low, low);
            if (q < n && (q > 0 || v >= g.full0)) x[q] = g.at(v)[q * BLOCK];
            else if (g.edge(v + q * BLOCK) && v + q * BLOCK < v0 + NV * BLOCK * trips) x[q] = distill_load_edge(g.z, g.first(v + q * BLOCK), (int)p.vocab);
          }
        }
        auto gradient = [&](int q) {
          float2 y[H];
#pragma unroll
          for (int i = 0; i < H; ++i) {
            if constexpr (LONG) {
              const float2 d = distill_mul(distill_add(distill_pair(x[q], i, type), make_float2(-a.m, -a.m)), make_float2(c2, c2));
              y[i] = make_float2(distill_ex2(d.x), distill_ex2(d.y));
            } else y[i] = e[q * H + i];
            y[i] = distill_mul(y[i], make_float2(f, f));
          }
          return distill_pack(y, type);
        };
        uint4* to = reinterpret_cast<uint4*>(dz - g.lead) + v;
        if (some && same && n >= NV && v >= g.full0) {
#pragma unroll
          for (int q = 0; q < NV; ++q) to[q * BLOCK] = gradient(q);
        } else {
#pragma unroll
          for (int q = 0; q < NV; ++q) {
            const uint4 out = some ? gradient(q) : make_uint4(0u, 0u, 0u, 0u);   // (0 whatever the logits are, NaN among them)
            if (same && q < n && (q > 0 || v >= g.full0)) to[q * BLOCK] = out;
            else if (v + q * BLOCK < min(g.vectors, v0 + NV * BLOCK * trips)) distill_store_edge(dz, g.first(v + q * BLOCK), (int)p.vocab, out);
          }
        }
      }
      __syncthreads();   // the dense part of every thread is written
      if (!(taken == -1.f)) dz[at] = from_f32<T>(distill_ex2((to_f32(own) - a.m) * c2) * scale - wt * taken);
    }
    if (part == 0 && tid == BLOCK - 1) {
      // tau^2 (sum p (t - z) / tau - L_t + L_z), L = (largest) / tau + ln(sum)
      const float ls = logf(a.s), lt = logf(a.ts);
      const double d = (double)(a.ta / a.ts) + ((double)a.m - (double)a.tm);
      p.loss[row] = some ? (float)((double)p.tau * d + (double)p.tau * p.tau * ((double)ls - (double)lt)) : 0.f;
      if (p.stats) {
        p.stats[2 * row] = a.m / p.tau + ls;
        p.stats[2 * row + 1] = some ? a.tm / p.tau + lt : none;
      }
    }
    at = at1; t = t1; own = own1; w = w1;
  }
  // (no block leaves while another, whose wait for it may have run out, can still send it something)
  if (parts > 1) asm volatile("barrier.cluster.wait;" ::: "memory");
}

// The gradient alone, from the normalisers that the loss left: a block takes NV vectors a thread of one row.
constexpr int DISTILL_GRAD_BLOCK = 256;
template <class T, int NV>
__global__ void __launch_bounds__(DISTILL_GRAD_BLOCK) idkm_distill_grad(const __grid_constant__ DistillParams p) {
  constexpr int N = Vec16<T>::N, H = N / 2, BLOCK = DISTILL_GRAD_BLOCK;
  T* const type = nullptr;
  const float none = __int_as_float(0xff800000);
  __shared__ __align__(16) int s_at[IDKM_DISTILL_MAX_TOP];
  __shared__ float s_t[IDKM_DISTILL_MAX_TOP];
  __shared__ int s_table[DISTILL_TABLE], s_twice;
  const int tid = threadIdx.x, part = blockIdx.x % (unsigned)p.parts;
  const long long row = blockIdx.x / (unsigned)p.parts;
  const DistillGrid<T> g(p, row);
  const int v0 = part * NV * BLOCK, v = v0 + tid, end = min(g.full1, v0 + NV * BLOCK);
  const DistillRaw raw = distill_raw(p, row, tid);
  uint4 x[NV];
  const unsigned low = distill_lowest<T>();
#pragma unroll
  for (int q = 0; q < NV; ++q) {   // (all of them asked for before the first is looked at)
    x[q] = make_uint4(low, low, low, low);
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "+r"(x[q].x), "+r"(x[q].y), "+r"(x[q].z), "+r"(x[q].w)
                 : "l"(g.at(v) + q * BLOCK), "r"((int)(v + q * BLOCK < end && v + q * BLOCK >= g.full0))
                 : "memory");
  }
  int at;
  float t, own = 0.f;
  distill_entry(p, raw, at, t);
  const float lse_t = p.stats[2 * row + 1], L = p.stats[2 * row], w = p.tau * (p.weight ? p.weight[row] : 1.f);
  const int place = (at + g.lead) / N;
  const bool mine = at >= 0 && place >= v0 && place < v0 + NV * BLOCK, some = lse_t != none;
  if (mine) own = to_f32(g.z[at]);
  for (int i = tid; i < DISTILL_TABLE; i += BLOCK) s_table[i] = -1;
  if (tid == 0) s_twice = 0;
  if (tid < p.top) {
    s_at[tid] = at;
    s_t[tid] = t;
  }
  __syncthreads();
  if (mine) distill_enter(s_table, at, &s_twice);
  __syncthreads();   // (every thread has read its entry's place: what follows may write it)
  // x = z / tau - L in units of log2, for fp32 with the low parts of log2(e) / tau and of L log2(e), which have either sign: where x is
  // -inf already (z is, or leaves the range) they are left out
  const float lh = L * LOG2E, ll = __fmaf_rn(L, LOG2E_LOW, __fmaf_rn(L, LOG2E, -lh));
  auto q_of = [&](float z) {
    float y = __fmaf_rn(z, p.c2, -lh);
    if (sizeof(T) == 4) y = y == none ? y : y + __fmaf_rn(z, p.c2_low, -ll);
    return w * distill_ex2(y > 0.f ? 0.f : y);   // (q <= 1, also where the rounding of a huge L says otherwise)
  };
  // (the teacher's probabilities are exp(t / tau - lse_t): as exp((t - tm) / tau) with tm = lse_t tau)
  float taken = -1.f;
  if (mine && some) taken = s_twice ? distill_taken(s_at, s_t, p.top, at, tid, lse_t * p.tau, 1.f, p.c2) : distill_ex2((t - lse_t * p.tau) * p.c2);
  T* dz = reinterpret_cast<T*>(p.dz) + row * p.lddz;
  const bool same = (((uintptr_t)dz ^ (uintptr_t)g.z) & 15u) == 0;
  uint4* to = reinterpret_cast<uint4*>(dz - g.lead) + v;
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    const int u = v + q * BLOCK;
    if (u >= min(g.vectors, v0 + NV * BLOCK)) break;
    const bool edge = g.edge(u);
    if (edge) x[q] = distill_load_edge(g.z, g.first(u), (int)p.vocab);
    float2 y[H];
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const float2 d = distill_pair(x[q], i, type);
      y[i] = make_float2(q_of(d.x), q_of(d.y));
    }
    uint4 out = distill_pack(y, type);
    if (!some) out = make_uint4(0u, 0u, 0u, 0u);
    if (same && !edge) to[q * BLOCK] = out;
    else distill_store_edge(dz, g.first(u), (int)p.vocab, out);
  }
  __syncthreads();   // the dense part of every thread is written
  if (!(taken == -1.f)) dz[at] = from_f32<T>(q_of(own) - w * taken);
}

template <class T, int BLOCK, int NV, int MODE, bool LONG>
cudaError_t distill_rows(const DistillParams& p, int sms, cudaStream_t st) {
  const int smem = NV * BLOCK * 16;
  if (smem > 32 * 1024) {
    static PerDevice limit;
    const cudaError_t rc = allow_smem(limit, idkm_distill_rows<T, BLOCK, NV, MODE, LONG>, smem);
    if (rc != cudaSuccess) return rc;
  }
  const long long resident = (long long)sms * (BLOCK == 512 ? 1 : NV <= 2 ? 6 : NV <= 4 ? 3 : 2) / p.parts;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.rows < resident ? p.rows : resident) * p.parts));
  cfg.blockDim = dim3(BLOCK);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.parts > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, idkm_distill_rows<T, BLOCK, NV, MODE, LONG>, p);
}

template <class T, int MODE>
cudaError_t distill_rows(const DistillParams& p, int block, int nv, int sms, cudaStream_t st) {
  if (p.trips > 1) return distill_rows<T, 512, 8, MODE, true>(p, sms, st);
  if (block == 512) {
    if (nv <= 4) return distill_rows<T, 512, 4, MODE, false>(p, sms, st);
    return distill_rows<T, 512, 8, MODE, false>(p, sms, st);
  }
  switch (nv) {
    case 1: return distill_rows<T, 256, 1, MODE, false>(p, sms, st);
    case 2: return distill_rows<T, 256, 2, MODE, false>(p, sms, st);
    case 3: return distill_rows<T, 256, 3, MODE, false>(p, sms, st);
    case 4: return distill_rows<T, 256, 4, MODE, false>(p, sms, st);
    case 5: return distill_rows<T, 256, 5, MODE, false>(p, sms, st);
    case 6: return distill_rows<T, 256, 6, MODE, false>(p, sms, st);
    case 7: return distill_rows<T, 256, 7, MODE, false>(p, sms, st);
    default: return distill_rows<T, 256, 8, MODE, false>(p, sms, st);
  }
}

template <class T>
cudaError_t distill_grad(const DistillParams& p, int nv, cudaStream_t st) {
  const unsigned grid = (unsigned)(p.rows * p.parts);
  switch (nv) {
    case 1: idkm_distill_grad<T, 1><<<grid, DISTILL_GRAD_BLOCK, 0, st>>>(p); break;
    case 2: idkm_distill_grad<T, 2><<<grid, DISTILL_GRAD_BLOCK, 0, st>>>(p); break;
    case 4: idkm_distill_grad<T, 4><<<grid, DISTILL_GRAD_BLOCK, 0, st>>>(p); break;
    default: idkm_distill_grad<T, 8><<<grid, DISTILL_GRAD_BLOCK, 0, st>>>(p); break;
  }
  return cudaGetLastError();
}

int distill(DistillParams p, int type, void* cuda_stream) {
  if (!p.z || !p.idx || !p.t) return IDKM_ERR_NULL;
  if (!elem_known(type) || !elem_known(p.t_type) || (p.idx_bytes != 4 && p.idx_bytes != 8) || p.top < 1 || p.top > IDKM_DISTILL_MAX_TOP)
    return IDKM_ERR_UNSUPPORTED;
  if (p.rows < 1 || p.vocab < 1 || p.ldz < p.vocab || (p.dz && p.lddz < p.vocab) || p.vocab > (INT64_C(1) << 30) || p.vocab > (INT64_C(1) << 50) / p.rows) return IDKM_ERR_SHAPE;
  if (!(p.tau > 0.f) || !(p.tau < 3.0e38f)) return IDKM_ERR_PARAM;
  const double c = 1.4426950408889634 / (double)p.tau;
  if (!(c < 3.0e38)) return IDKM_ERR_PARAM;   // (tau below the normal range)
  p.c2 = (float)c;
  p.c2_low = (float)(c - (double)p.c2);
  if (p.dz == p.z && p.lddz != p.ldz) return IDKM_ERR_PARAM;
  const int b = elem_bytes(type);
  if (((uintptr_t)p.z | (uintptr_t)p.dz) % b || (uintptr_t)p.idx % p.idx_bytes || (uintptr_t)p.t % elem_bytes(p.t_type) ||
      ((uintptr_t)p.loss | (uintptr_t)p.stats | (uintptr_t)p.weight) % 4)
    return IDKM_ERR_ALIGN;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
    return IDKM_ERR_CUDA;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const int mode = !p.loss ? DISTILL_GRAD : p.dz ? DISTILL_STEP : DISTILL_LOSS;
  // 16-byte vectors of a row (one more where it begins between boundaries), `block` of them a register of every thread
  const long long vectors = (p.vocab * b + 15) / 16 + (((uintptr_t)p.z | (uintptr_t)(p.rows > 1 ? p.ldz * b : 0)) & 15u ? 1 : 0);
  int block = 256, nv;
  p.trips = 1;
  if (mode == DISTILL_GRAD) {
    const long long regs = (vectors + DISTILL_GRAD_BLOCK - 1) / DISTILL_GRAD_BLOCK;
    nv = regs >= 8 ? 8 : regs > 2 ? 4 : (int)regs;
    while (nv > 1 && p.rows * ((regs + nv - 1) / nv) < sms * 2) nv /= 2;   // few rows: a block for each multiprocessor
    p.parts = (int)((regs + nv - 1) / nv);
  } else {
    long long regs = (vectors + block - 1) / block, parts = (regs + 7) / 8;
    if (parts > DISTILL_MAX_CLUSTER) {
      block = 512;
      regs = (vectors + block - 1) / block;
      parts = (regs + 7) / 8;
      if (parts > DISTILL_MAX_CLUSTER) parts = DISTILL_MAX_CLUSTER;
    }
    // few rows: more blocks for each, as long as there are multiprocessors without one
    while (parts < regs && parts < DISTILL_MAX_CLUSTER && p.rows * parts < sms) ++parts;
    const long long per = (regs + parts - 1) / parts;
    p.trips = (int)((per + 7) / 8);
    nv = p.trips > 1 ? 8 : block == 512 ? (per <= 4 ? 4 : 8) : (int)per;
    p.parts = (int)((regs + (long long)nv * p.trips - 1) / ((long long)nv * p.trips));
  }
  // (a grid has at most 2^31 - 1 blocks)
  const long long at_once = (long long)INT32_MAX / p.parts;
  const DistillParams all = p;
  for (long long r = 0; r < all.rows; r += at_once) {
    p.rows = all.rows - r < at_once ? all.rows - r : at_once;
    p.z = (const char*)all.z + r * all.ldz * b;
    p.idx = (const char*)all.idx + r * all.top * all.idx_bytes;
    p.t = (const char*)all.t + r * all.top * elem_bytes(all.t_type);
    p.weight = all.weight ? all.weight + r : nullptr;
    p.loss = all.loss ? all.loss + r : nullptr;
    p.stats = all.stats ? all.stats + 2 * r : nullptr;
    p.dz = all.dz ? (char*)all.dz + r * all.lddz * b : nullptr;
    const cudaError_t rc = (cudaError_t)with_type(type, [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      return (int)(mode == DISTILL_GRAD ? distill_grad<T>(p, nv, st)
                   : mode == DISTILL_STEP ? distill_rows<T, DISTILL_STEP>(p, block, nv, sms, st) : distill_rows<T, DISTILL_LOSS>(p, block, nv, sms, st));
    });
    if (rc != cudaSuccess) {
      (void)cudaGetLastError();
      return IDKM_ERR_CUDA;
    }
  }
  return IDKM_OK;
}

}  // namespace

extern "C" int idkm_distill_forward(const void* z, int type, int64_t rows, int64_t vocab, int64_t ldz, const void* idx, int idx_bytes, const void* t,
                                    int t_type, int top, float tau, float* loss_out, float* stats_out, void* cuda_stream) {
  if (!loss_out) return IDKM_ERR_NULL;
  return distill(DistillParams{z, rows, vocab, ldz, idx, idx_bytes, t, t_type, top, tau, 0.f, 0.f, nullptr, loss_out, stats_out, nullptr, 0}, type, cuda_stream);
}

extern "C" int idkm_distill_backward(const void* z, int type, int64_t rows, int64_t vocab, int64_t ldz, const void* idx, int idx_bytes, const void* t,
                                     int t_type, int top, float tau, const float* stats, const float* weight, void* dz_out, int64_t lddz,
                                     void* cuda_stream) {
  if (!stats || !dz_out) return IDKM_ERR_NULL;
  return distill(DistillParams{z, rows, vocab, ldz, idx, idx_bytes, t, t_type, top, tau, 0.f, 0.f, weight, nullptr, const_cast<float*>(stats), dz_out, lddz},
                 type, cuda_stream);
}

extern "C" int idkm_distill_step(const void* z, int type, int64_t rows, int64_t vocab, int64_t ldz, const void* idx, int idx_bytes, const void* t,
                                 int t_type, int top, float tau, const float* weight, float* loss_out, void* dz_out, int64_t lddz,
                                 void* cuda_stream) {
  if (!loss_out || !dz_out) return IDKM_ERR_NULL;
  return distill(DistillParams{z, rows, vocab, ldz, idx, idx_bytes, t, t_type, top, tau, 0.f, 0.f, weight, loss_out, nullptr, dz_out, lddz}, type, cuda_stream);
}
