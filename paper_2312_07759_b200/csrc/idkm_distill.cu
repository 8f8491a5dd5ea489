// Distillation from a teacher's top logits: the loss by which a quantised network is trained from the full-precision one, and
// its gradient with respect to the student's logits.  For a row z in R^V, teacher entries (i_j, t_j), temperature tau:
//   p_j = softmax_j(t_j / tau) over the entries with 0 <= i_j < V,   q_v = softmax_v(z_v / tau),
//   loss = tau^2 sum_j p_j (ln p_j - ln q_{i_j}),    dz_v = w tau (q_v - sum_{j: i_j = v} p_j).
// A row without entries (or whose t_j are all -inf) has loss 0 and gradient 0.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include "idkm_types.cuh"
#include "../../include/idkm.h"

namespace {

using namespace idkm;

constexpr int DISTILL_BLOCK = 512;

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
};

struct DistillRow {
  long long at[IDKM_DISTILL_MAX_TOP];   // index of an entry, -1 where it does not count
  float t[IDKM_DISTILL_MAX_TOP];        // t_j / tau, then p_j
  float lse_t;
};

__device__ __forceinline__ float distill_teacher(const DistillParams& p, long long i) {
  if (p.t_type == ELEM_F32) return reinterpret_cast<const float*>(p.t)[i];
  if (p.t_type == ELEM_BF16) return to_f32(reinterpret_cast<const __nv_bfloat16*>(p.t)[i]);
  return to_f32(reinterpret_cast<const __half*>(p.t)[i]);
}

// (max, sum of exp(x - max)) of two parts; an empty part is (-inf, 0), one with a NaN has a NaN for its sum.
__device__ __forceinline__ void distill_join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  s = (s == 0.f ? 0.f : s * expf(m - top)) + (s2 == 0.f ? 0.f : s2 * expf(m2 - top));
  m = top;
}

// Reads a row's entries and normalises the teacher's part.  Called by the whole block.
__device__ void distill_entries(const DistillParams& p, long long row, DistillRow& r, const float* stats) {
  const float none = __int_as_float(0xff800000);
  for (int j = threadIdx.x; j < p.top; j += blockDim.x) {
    const long long i = row * p.top + j;
    const long long v = p.idx_bytes == 8 ? reinterpret_cast<const long long*>(p.idx)[i] : (long long)reinterpret_cast<const int*>(p.idx)[i];
    const bool fine = v >= 0 && v < p.vocab;
    r.at[j] = fine ? v : -1;
    r.t[j] = fine ? __fdiv_rn(distill_teacher(p, i), p.tau) : none;
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    float lse;
    if (stats) lse = stats[2 * row + 1];
    else {
      float m = none, s = 0.f;
      for (int j = threadIdx.x; j < p.top; j += 32) m = fmaxf(m, r.t[j]);
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      for (int j = threadIdx.x; j < p.top; j += 32) s += r.t[j] == none ? 0.f : expf(r.t[j] - m);   // (NaN stays)
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      lse = m == none && s == 0.f ? none : m + logf(s);
    }
    if (threadIdx.x == 0) r.lse_t = lse;
  }
  __syncthreads();
}

template <class T>
__global__ void __launch_bounds__(DISTILL_BLOCK) idkm_distill_rows(const DistillParams p) {
  __shared__ DistillRow r;
  __shared__ float part_m[DISTILL_BLOCK / 32], part_s[DISTILL_BLOCK / 32];
  const float none = __int_as_float(0xff800000);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* z = reinterpret_cast<const T*>(p.z) + row * p.ldz;
    const bool known = p.loss == nullptr;   // the gradient alone: the normalisers are given
    distill_entries(p, row, r, known ? p.stats : nullptr);
    float lse;
    if (known) lse = p.stats[2 * row];
    else {
      float m = none, s = 0.f;
      for (long long v = tid; v < p.vocab; v += DISTILL_BLOCK) {
        const float x = __fdiv_rn(to_f32(z[v]), p.tau);
        distill_join(m, s, x, x == none ? 0.f : 1.f);
      }
      for (int o = 16; o > 0; o >>= 1) distill_join(m, s, __shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o));
      if (lane == 0) { part_m[warp] = m; part_s[warp] = s; }
      __syncthreads();
      m = none; s = 0.f;
      for (int q = 0; q < DISTILL_BLOCK / 32; ++q) distill_join(m, s, part_m[q], part_s[q]);
      lse = m + logf(s);
      if (warp == 0) {
        double sum = 0.0;
        for (int j = lane; j < p.top; j += 32) {
          const float lp = r.t[j] - r.lse_t, pj = r.t[j] == none || r.lse_t == none ? 0.f : expf(lp);
          if (!(pj <= 0.f)) sum += (double)pj * ((double)lp - ((double)__fdiv_rn(to_f32(z[r.at[j]]), p.tau) - (double)lse));
        }
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) {
          p.loss[row] = (float)((double)p.tau * p.tau * sum);
          if (p.stats) { p.stats[2 * row] = lse; p.stats[2 * row + 1] = r.lse_t; }
        }
      }
    }
    if (p.dz) {
      T* dz = reinterpret_cast<T*>(p.dz) + row * p.lddz;
      const float w = p.tau * (p.weight ? p.weight[row] : 1.f);
      const bool some = r.lse_t != none;
      __syncthreads();
      // an entry's own value of z, before the row is overwritten (dz may be z)
      float own = 0.f, taken = 0.f;
      bool first = false;
      if (tid < p.top && r.at[tid] >= 0 && some) {
        first = true;
        own = __fdiv_rn(to_f32(z[r.at[tid]]), p.tau);
        for (int j = 0; j < p.top; ++j)
          if (r.at[j] == r.at[tid]) {
            if (j < tid) first = false;
            taken += r.t[j] == none ? 0.f : expf(r.t[j] - r.lse_t);
          }
      }
      __syncthreads();
      for (long long v = tid; v < p.vocab; v += DISTILL_BLOCK) dz[v] = from_f32<T>(some ? w * expf(__fdiv_rn(to_f32(z[v]), p.tau) - lse) : 0.f);
      __syncthreads();
      if (first) dz[r.at[tid]] = from_f32<T>(w * (expf(own - lse) - taken));
    }
    __syncthreads();
  }
}

int distill(const DistillParams& p, int type, void* cuda_stream) {
  if (!p.z || !p.idx || !p.t) return IDKM_ERR_NULL;
  if (!elem_known(type) || !elem_known(p.t_type) || (p.idx_bytes != 4 && p.idx_bytes != 8) || p.top < 1 || p.top > IDKM_DISTILL_MAX_TOP)
    return IDKM_ERR_UNSUPPORTED;
  if (p.rows < 1 || p.vocab < 1 || p.ldz < p.vocab || (p.dz && p.lddz < p.vocab) || p.vocab > (INT64_C(1) << 50) / p.rows) return IDKM_ERR_SHAPE;
  if (!(p.tau > 0.f) || !(p.tau < 3.0e38f)) return IDKM_ERR_PARAM;
  if (p.dz == p.z && p.lddz != p.ldz) return IDKM_ERR_PARAM;
  const int b = elem_bytes(type);
  if (((uintptr_t)p.z | (uintptr_t)p.dz) % b || (uintptr_t)p.idx % p.idx_bytes || (uintptr_t)p.t % elem_bytes(p.t_type) ||
      ((uintptr_t)p.loss | (uintptr_t)p.stats | (uintptr_t)p.weight) % 4)
    return IDKM_ERR_ALIGN;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
    return IDKM_ERR_CUDA;
  const int grid = (int)(p.rows < (long long)sms * 4 ? p.rows : (long long)sms * 4);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  return with_type(type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    idkm_distill_rows<T><<<grid, DISTILL_BLOCK, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? IDKM_OK : IDKM_ERR_CUDA;
  });
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
