// Distillation from a teacher's top logits: the loss by which a quantised network is trained from the full-precision one, and
// its gradient with respect to the student's logits.  For a row z in R^V, teacher entries (i_j, t_j), temperature tau:
//   p_j = softmax_j(t_j / tau) over the entries with 0 <= i_j < V,   q_v = softmax_v(z_v / tau),
//   loss = tau^2 sum_j p_j (ln p_j - ln q_{i_j}),    dz_v = w tau (q_v - sum_{j: i_j = v} p_j).
// A row without entries (or whose t_j are all -inf) has loss 0 and gradient 0.  As sum_j p_j = 1,
//   loss = tau^2 (sum_j p_j (t_j - z_{i_j}) / tau - L_t + L_z),   L_t, L_z the logarithms of the two normalisers.
//
// One pass over z.  A row is a cluster of up to 8 blocks; a thread keeps its few 16-byte vectors of the row in registers, their
// largest element m and e_v = exp((z_v - m) / tau).  Threads, warps and blocks then join (m, sum of e) and the teacher's part, which
// every block has whole but for the entries' products, for which it takes the entries of its own part of the row; blocks
// write theirs into the shared memory of the others, one cluster barrier.  Then q_v = e_v exp((m - M) / tau) / S, so an element
// costs one exponential, 2 or 4 bytes in and as many out.  Entries' places are written again after the dense part.
// What bounds it: traffic.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <type_traits>
#include "idkm_types.cuh"
#include "../../include/idkm.h"

namespace {

using namespace idkm;

constexpr int DISTILL_BLOCK = 256;
constexpr int DISTILL_MAX_CLUSTER = 8;
constexpr float LOG2E = 1.4426950408889634f;

struct DistillParams {
  const void* z;
  long long rows, vocab, ldz;
  const void* idx;
  int idx_bytes;
  const void* t;
  int t_type, top;
  float tau;
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

__device__ __forceinline__ float distill_teacher(const DistillParams& p, long long i) {
  if (p.t_type == ELEM_F32) return __ldg(reinterpret_cast<const float*>(p.t) + i);
  if (p.t_type == ELEM_BF16) return to_f32(__ldg(reinterpret_cast<const __nv_bfloat16*>(p.t) + i));
  return to_f32(__ldg(reinterpret_cast<const __half*>(p.t) + i));
}

// Sums of exp((x - m) c2) and of the teacher's products against the largest x, m.  An empty part is (-inf, 0, 0); a part with a
// NaN has one in its sum.
struct DistillPart {
  float m, s;        // student
  float tm, ts, ta;  // teacher: largest t, sum of exp((t - tm) / tau), sum of that times t - z over the block's own entries
};

// exp((m - top) / tau), 0 where m is -inf (an empty part, whatever top is).
__device__ __forceinline__ float distill_scale(float m, float top, float c2) {
  return m == __int_as_float(0xff800000) ? 0.f : distill_ex2((m - top) * c2);
}

// A part that another scale multiplies: 0 stays 0 whatever the scale; NaN stays.
__device__ __forceinline__ float distill_scaled(float s, float f) { return s == 0.f ? 0.f : s * f; }

__device__ __forceinline__ void distill_join(DistillPart& a, const DistillPart& b, float c2) {
  const float top = fmaxf(a.m, b.m), fa = distill_scale(a.m, top, c2), fb = distill_scale(b.m, top, c2);
  a.s = distill_scaled(a.s, fa) + distill_scaled(b.s, fb);
  a.m = top;
  const float tt = fmaxf(a.tm, b.tm), ga = distill_scale(a.tm, tt, c2), gb = distill_scale(b.tm, tt, c2);
  a.ts = distill_scaled(a.ts, ga) + distill_scaled(b.ts, gb);
  // (the teacher's mass, however small, on a logit of -inf: infinite, whatever the scale)
  const float inf = __int_as_float(0x7f800000);
  a.ta = a.ta == inf || b.ta == inf ? inf : distill_scaled(a.ta, ga) + distill_scaled(b.ta, gb);
  a.tm = tt;
}

__device__ __forceinline__ float distill_warp_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float distill_warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// The elements of one 16-byte vector of a row; -inf where it reaches past the row's ends.  `first`: the row's index of its first
// element, which is below 0 where the row does not begin on a 16-byte boundary.
template <class T>
__device__ __forceinline__ Vec16<T> distill_load(const T* z, long long first, long long vocab) {
  constexpr int N = Vec16<T>::N;
  Vec16<T> x;
  if (first >= 0 && first + N <= vocab) x.raw = *reinterpret_cast<const uint4*>(z + first);
  else {
#pragma unroll
    for (int e = 0; e < N; ++e) x.e[e] = first + e >= 0 && first + e < vocab ? z[first + e] : from_f32<T>(__int_as_float(0xff800000));
  }
  return x;
}

template <class T>
__device__ __forceinline__ void distill_store(T* dz, long long first, long long vocab, bool whole, const float* v) {
  constexpr int N = Vec16<T>::N;
  if (whole && first >= 0 && first + N <= vocab) {
    Vec16<T> x;
#pragma unroll
    for (int e = 0; e < N; ++e) x.e[e] = from_f32<T>(v[e]);
    *reinterpret_cast<uint4*>(dz + first) = x.raw;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (first + e >= 0 && first + e < vocab) dz[first + e] = from_f32<T>(v[e]);
  }
}

template <class T, int NV, int MODE>
__global__ void __launch_bounds__(DISTILL_BLOCK) idkm_distill(const DistillParams p) {
  constexpr int N = Vec16<T>::N, WARPS = DISTILL_BLOCK / 32;
  static_assert(DISTILL_BLOCK >= IDKM_DISTILL_MAX_TOP, "an entry a thread");
  const float none = __int_as_float(0xff800000);
  __shared__ __align__(16) int s_at[IDKM_DISTILL_MAX_TOP];   // the entries' indices, -1 where they do not count
  __shared__ float s_p[IDKM_DISTILL_MAX_TOP];                // their probabilities
  __shared__ DistillPart s_warp[WARPS], s_part[DISTILL_MAX_CLUSTER];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.x / (unsigned)p.parts;
  const int part = (int)(blockIdx.x - (unsigned)row * (unsigned)p.parts);
  if (MODE != DISTILL_GRAD && p.parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (this block runs)
  const T* z = reinterpret_cast<const T*>(p.z) + row * p.ldz;
  const float c2 = LOG2E / p.tau;
  // vectors on 16-byte boundaries: the first may begin before the row; block `part` takes vectors [v0, v1)
  const int lead = (int)(((uintptr_t)z & 15u) / sizeof(T));
  const int vectors = (int)((p.vocab + lead + N - 1) / N), share = NV * DISTILL_BLOCK * p.trips;
  const int v0 = part * share, v1 = min(v0 + share, vectors);
  auto first_of = [&](int v) { return (long long)v * N - lead; };

  int at = -1;
  float tt = none;
  if (tid < p.top) {
    const long long i = row * p.top + tid;
    const long long v = p.idx_bytes == 8 ? __ldg(reinterpret_cast<const long long*>(p.idx) + i) : (long long)__ldg(reinterpret_cast<const int*>(p.idx) + i);
    if (v >= 0 && v < p.vocab) {
      at = (int)v;
      tt = distill_teacher(p, i);
    }
    s_at[tid] = at;
  }
  Vec16<T> x[NV];
  float e[NV * N];
  auto load = [&](int trip) {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int v = v0 + (trip * NV + q) * DISTILL_BLOCK + tid;
      x[q] = distill_load(z, v < v1 ? first_of(v) : (long long)p.vocab, p.vocab);
    }
  };
  const bool mine = at >= 0 && (at + lead) / N >= v0 && (at + lead) / N < v1;   // this block's part of the row holds the entry
  load(0);
  const float own = mine ? to_f32(z[at]) : 0.f;   // (read before anything is written: dz may be z)

  float m = none, lse_t;   // the thread's largest element; ln of the teacher's normaliser
  float M = 0.f, factor = 0.f;
  if (MODE == DISTILL_GRAD) {
    lse_t = p.stats[2 * row + 1];
    __syncthreads();   // (every thread has read its entry's place: what follows may write it)
  } else {
    DistillPart a;
    float sum = 0.f;
    for (int trip = 0; trip < p.trips; ++trip) {
      if (trip) load(trip);
      float top = none;
#pragma unroll
      for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, to_f32(x[q].e[i]));
      top = fmaxf(top, m);
      const float from = top == none ? 0.f : top;
      sum = distill_scaled(sum, distill_scale(m, top, c2));
      m = top;
#pragma unroll
      for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          e[q * N + i] = distill_ex2((to_f32(x[q].e[i]) - from) * c2);
          sum += e[q * N + i];
        }
    }
    // the warp's: the largest first, then one scale a thread
    a.m = distill_warp_max(m);
    a.s = distill_warp_sum(distill_scaled(sum, distill_scale(m, a.m, c2)));
    a.tm = none;
    a.ts = a.ta = 0.f;
    if (warp * 32 < p.top) {
      a.tm = distill_warp_max(tt);
      const float w = tt == none ? 0.f : distill_ex2((tt - a.tm) * c2);
      a.ts = distill_warp_sum(w);
      const float term = own == none ? -none : w * (tt - own);
      a.ta = distill_warp_sum(mine && tt != none ? term : 0.f);
    }
    if (lane == 0) s_warp[warp] = a;
    __syncthreads();
    a = s_warp[0];
#pragma unroll
    for (int q = 1; q < WARPS; ++q) distill_join(a, s_warp[q], c2);
    if (p.parts > 1) {
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // (every block of the cluster runs: its memory may be written)
      if (tid < p.parts) {
        uint32_t there;
        const uint32_t here = (uint32_t)__cvta_generic_to_shared(&s_part[part]);
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(tid));
        const float v[5] = {a.m, a.s, a.tm, a.ts, a.ta};
#pragma unroll
        for (int q = 0; q < 5; ++q) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there + 4 * q), "f"(v[q]) : "memory");
      }
      __syncwarp();
      asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      // (every block holds the teacher's sums whole: only the products add up)
      a = s_part[0];
      for (int q = 1; q < p.parts; ++q) {
        DistillPart b = s_part[q];
        b.ts = 0.f;
        distill_join(a, b, c2);
      }
    }
    M = a.m;
    lse_t = a.tm == none && a.ts == 0.f ? none : a.tm / p.tau + logf(a.ts);
    if (part == 0 && tid == 0) {
      const double lz = (double)a.m / p.tau + (double)logf(a.s), lt = (double)a.tm / p.tau + (double)logf(a.ts);
      p.loss[row] = lse_t == none ? 0.f : (float)((double)p.tau * p.tau * ((double)a.ta / (double)a.ts / p.tau - lt + lz));
      if (p.stats) {
        p.stats[2 * row] = (float)lz;
        p.stats[2 * row + 1] = lse_t;
      }
    }
    factor = 1.f / a.s;
  }
  if (MODE == DISTILL_LOSS) return;

  const bool some = lse_t != none;
  const float w = p.tau * (p.weight ? p.weight[row] : 1.f);
  T* dz = reinterpret_cast<T*>(p.dz) + row * p.lddz;
  const bool whole = (((uintptr_t)dz ^ (uintptr_t)z) & 15u) == 0;
  if (tid < p.top) s_p[tid] = tt == none ? 0.f : expf(tt / p.tau - lse_t);
  if (MODE == DISTILL_GRAD) {
    // x = z / tau - L_z in units of log2, the low parts of 1 / tau and L_z with it
    const double c = 1.4426950408889634 / (double)p.tau, l = (double)p.stats[2 * row] * 1.4426950408889634;
    const float ch = (float)c, cl = (float)(c - (double)ch), lh = (float)l, ll = (float)(l - (double)lh);
    auto q_of = [&](float v) {
      const float y = sizeof(T) == 4 ? __fmaf_rn(v, ch, -lh) + __fmaf_rn(v, cl, -ll) : __fmaf_rn(v, ch, -lh);
      return some ? w * distill_ex2(y > 0.f ? 0.f : y) : 0.f;   // (q <= 1, also where the rounding of a huge L_z says otherwise)
    };
    for (int trip = 0; trip < p.trips; ++trip) {
      if (trip) load(trip);
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        const int v = v0 + (trip * NV + q) * DISTILL_BLOCK + tid;
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = q_of(to_f32(x[q].e[i]));
        if (v < v1) distill_store(dz, first_of(v), p.vocab, whole, y);
      }
    }
    factor = q_of(own);
  } else {
    const float scale = factor * w;
    for (int trip = 0; trip < p.trips; ++trip) {
      float f = distill_scale(m, M, c2) * scale;
      if (p.trips > 1) {   // (the registers hold the last trip only)
        load(trip);
        f = scale;
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
          for (int i = 0; i < N; ++i) e[q * N + i] = distill_ex2((to_f32(x[q].e[i]) - M) * c2);
      }
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        const int v = v0 + (trip * NV + q) * DISTILL_BLOCK + tid;
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = some ? e[q * N + i] * f : 0.f;
        if (v < v1) distill_store(dz, first_of(v), p.vocab, whole, y);
      }
    }
    factor = distill_ex2((own - M) * c2) * scale;
  }
  __syncthreads();   // the dense part of every thread is written, the entries' probabilities are there
  if (mine && some) {
    float taken = 0.f;
    bool again = false;
    int j = 0;
    for (; j + 4 <= p.top; j += 4) {
      const int4 o = *reinterpret_cast<const int4*>(s_at + j);
      if (o.x == at) { taken += s_p[j]; again |= j < tid; }
      if (o.y == at) { taken += s_p[j + 1]; again |= j + 1 < tid; }
      if (o.z == at) { taken += s_p[j + 2]; again |= j + 2 < tid; }
      if (o.w == at) { taken += s_p[j + 3]; again |= j + 3 < tid; }
    }
    for (; j < p.top; ++j)
      if (s_at[j] == at) { taken += s_p[j]; again |= j < tid; }
    if (!again) dz[at] = from_f32<T>(factor - w * taken);   // (the first of equal indices writes)
  }
}

template <class T, int MODE>
cudaError_t distill_launch(const DistillParams& given, int nv, cudaStream_t st) {
  const DistillParams p = given;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.rows * p.parts));
  cfg.blockDim = dim3(DISTILL_BLOCK);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = MODE != DISTILL_GRAD && p.parts > 1 ? 1 : 0;
  switch (nv) {
    case 1: return cudaLaunchKernelEx(&cfg, idkm_distill<T, 1, MODE>, p);
    case 2: return cudaLaunchKernelEx(&cfg, idkm_distill<T, 2, MODE>, p);
    case 3: return cudaLaunchKernelEx(&cfg, idkm_distill<T, 3, MODE>, p);
    case 4: return cudaLaunchKernelEx(&cfg, idkm_distill<T, 4, MODE>, p);
    case 6: return cudaLaunchKernelEx(&cfg, idkm_distill<T, 6, MODE>, p);
    default: return cudaLaunchKernelEx(&cfg, idkm_distill<T, 8, MODE>, p);
  }
}

int distill(DistillParams p, int type, void* cuda_stream) {
  if (!p.z || !p.idx || !p.t) return IDKM_ERR_NULL;
  if (!elem_known(type) || !elem_known(p.t_type) || (p.idx_bytes != 4 && p.idx_bytes != 8) || p.top < 1 || p.top > IDKM_DISTILL_MAX_TOP)
    return IDKM_ERR_UNSUPPORTED;
  if (p.rows < 1 || p.vocab < 1 || p.ldz < p.vocab || (p.dz && p.lddz < p.vocab) || p.vocab > (INT64_C(1) << 30) || p.vocab > (INT64_C(1) << 50) / p.rows) return IDKM_ERR_SHAPE;
  if (!(p.tau > 0.f) || !(p.tau < 3.0e38f)) return IDKM_ERR_PARAM;
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
  // 16-byte vectors of a row (one more where it begins between boundaries), DISTILL_BLOCK of them a register of every thread
  const long long vectors = (p.vocab * b + 15) / 16 + (((uintptr_t)p.z | (uintptr_t)(p.rows > 1 ? p.ldz * b : 0)) & 15u ? 1 : 0);
  const long long regs = (vectors + DISTILL_BLOCK - 1) / DISTILL_BLOCK;
  const int most = b == 4 ? 8 : mode == DISTILL_GRAD ? 4 : 6;
  long long parts = (regs + most - 1) / most;
  if (mode != DISTILL_GRAD && parts > DISTILL_MAX_CLUSTER) parts = DISTILL_MAX_CLUSTER;
  // few rows: more blocks for each, as long as there are multiprocessors without one
  while (parts < regs && parts < DISTILL_MAX_CLUSTER && p.rows * parts < sms) ++parts;
  const long long per = (regs + parts - 1) / parts;   // registers of a thread, in trips of at most 8
  const int trips = (int)((per + 7) / 8);
  const int need = (int)((per + trips - 1) / trips), nv = need == 5 ? 6 : need == 7 ? 8 : need;
  p.parts = (int)((regs + (long long)nv * trips - 1) / ((long long)nv * trips));
  p.trips = trips;
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
      return (int)(mode == DISTILL_GRAD ? distill_launch<T, DISTILL_GRAD>(p, nv, st) : mode == DISTILL_STEP ? distill_launch<T, DISTILL_STEP>(p, nv, st) : distill_launch<T, DISTILL_LOSS>(p, nv, st));
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
  return distill(DistillParams{z, rows, vocab, ldz, idx, idx_bytes, t, t_type, top, tau, nullptr, loss_out, stats_out, nullptr, 0}, type, cuda_stream);
}

extern "C" int idkm_distill_backward(const void* z, int type, int64_t rows, int64_t vocab, int64_t ldz, const void* idx, int idx_bytes, const void* t,
                                     int t_type, int top, float tau, const float* stats, const float* weight, void* dz_out, int64_t lddz,
                                     void* cuda_stream) {
  if (!stats || !dz_out) return IDKM_ERR_NULL;
  return distill(DistillParams{z, rows, vocab, ldz, idx, idx_bytes, t, t_type, top, tau, weight, nullptr, const_cast<float*>(stats), dz_out, lddz},
                 type, cuda_stream);
}

extern "C" int idkm_distill_step(const void* z, int type, int64_t rows, int64_t vocab, int64_t ldz, const void* idx, int idx_bytes, const void* t,
                                 int t_type, int top, float tau, const float* weight, float* loss_out, void* dz_out, int64_t lddz,
                                 void* cuda_stream) {
  if (!loss_out || !dz_out) return IDKM_ERR_NULL;
  return distill(DistillParams{z, rows, vocab, ldz, idx, idx_bytes, t, t_type, top, tau, weight, loss_out, nullptr, dz_out, lddz}, type, cuda_stream);
}
