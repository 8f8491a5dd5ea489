// Products with 4-bit weights and group scales: Y[m][n] = sum_k s[n][k / g] C[code[n][k]] X[m][k].
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include "idkm_types.cuh"
#include "../../include/idkm.h"

namespace {

using namespace idkm;

struct CodesParams {
  const void* X;
  long long tokens, ldx;
  const unsigned char* codes;
  long long rows, cols, pitch;
  const void* C;
  int k;
  const void* scales;
  long long group, n_groups;
  void* Y;
  long long ldy;
  int vec_x;   // rows of X start on 16-byte boundaries
};

constexpr int ROWS_BLOCK = 256;
constexpr int ROWS_LANE = 8;   // consecutive weights of a lane: one word of codes

// A warp takes a row of W and TOK rows of X; every lane looks its eight weights up and adds their products, the group's scale
// multiplies the sum of the eight.
template <class T, int TOK>
__global__ void __launch_bounds__(ROWS_BLOCK) idkm_codes_rows(const CodesParams p) {
  __shared__ float lut[16];
  if (threadIdx.x < 16) lut[threadIdx.x] = threadIdx.x < p.k ? to_f32(reinterpret_cast<const T*>(p.C)[threadIdx.x]) : 0.f;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const long long m0 = (long long)blockIdx.y * TOK;
  const T* X = reinterpret_cast<const T*>(p.X) + m0 * p.ldx;
  const int n_tok = (int)min((long long)TOK, p.tokens - m0);
  for (long long n = (long long)blockIdx.x * (ROWS_BLOCK / 32) + (threadIdx.x >> 5); n < p.rows; n += (long long)gridDim.x * (ROWS_BLOCK / 32)) {
    const unsigned char* row = p.codes + n * p.pitch;
    float acc[TOK];
#pragma unroll
    for (int m = 0; m < TOK; ++m) acc[m] = 0.f;
    for (long long c = lane * ROWS_LANE; c < p.cols; c += 32 * ROWS_LANE) {
      const unsigned word = __ldg(reinterpret_cast<const unsigned*>(row + c / 2));
      const float s = p.scales ? to_f32(reinterpret_cast<const T*>(p.scales)[n * p.n_groups + c / p.group]) : 1.f;
      float w[ROWS_LANE];
#pragma unroll
      for (int e = 0; e < ROWS_LANE; ++e) w[e] = lut[word >> (4 * e) & 15u];
#pragma unroll
      for (int m = 0; m < TOK; ++m) {
        if (m >= n_tok) continue;
        const T* x = X + m * p.ldx + c;
        float xs[ROWS_LANE];
        if (p.vec_x && c + ROWS_LANE <= p.cols) {
          constexpr int N = Vec16<T>::N;
#pragma unroll
          for (int q = 0; q < ROWS_LANE / N; ++q) {
            Vec16<T> v;
            v.raw = __ldg(reinterpret_cast<const uint4*>(x) + q);
#pragma unroll
            for (int e = 0; e < N; ++e) xs[q * N + e] = to_f32(v.e[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < ROWS_LANE; ++e) xs[e] = c + e < p.cols ? to_f32(x[e]) : 0.f;
        }
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < ROWS_LANE; ++e) sum = fmaf(w[e], xs[e], sum);
        acc[m] = fmaf(s, sum, acc[m]);
      }
    }
#pragma unroll
    for (int m = 0; m < TOK; ++m) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[m] += __shfl_xor_sync(0xffffffffu, acc[m], o);
      if (lane == 0 && m < n_tok) reinterpret_cast<T*>(p.Y)[(m0 + m) * p.ldy + n] = from_f32<T>(acc[m]);
    }
  }
}

}  // namespace

extern "C" int idkm_matmul_codes(const void* X, int type, int64_t tokens, int64_t ldx, const unsigned char* codes, int64_t rows, int64_t cols,
                                 int64_t pitch, const void* C, int k, const void* scales, int64_t group, void* Y, int64_t ldy,
                                 void* cuda_stream) {
  if (!X || !codes || !C || !Y) return IDKM_ERR_NULL;
  if (k < 1 || k > 16 || !elem_known(type)) return IDKM_ERR_UNSUPPORTED;
  if (tokens < 1 || rows < 1 || cols < 1 || ldx < cols || ldy < rows || pitch < (cols + 31) / 32 * 16 || (scales && group < 1) ||
      cols > (INT64_C(1) << 50) / rows || tokens > (INT64_C(1) << 31))
    return IDKM_ERR_SHAPE;
  if (scales && group < cols && group != 32 && group != 64 && group % 128 != 0) return IDKM_ERR_UNSUPPORTED;
  if (Y == X || Y == C || Y == (const void*)codes || Y == scales) return IDKM_ERR_PARAM;
  const int tb = elem_bytes(type);
  if (((uintptr_t)X | (uintptr_t)C | (uintptr_t)scales | (uintptr_t)Y) % tb || ((uintptr_t)codes | (uintptr_t)pitch) % 16) return IDKM_ERR_ALIGN;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
    return IDKM_ERR_CUDA;
  CodesParams p;
  p.X = X; p.tokens = tokens; p.ldx = ldx; p.codes = codes; p.rows = rows; p.cols = cols; p.pitch = pitch; p.C = C; p.k = k;
  p.scales = scales;
  p.group = !scales || group >= cols ? (cols + 127) / 128 * 128 : group;
  p.n_groups = (cols + p.group - 1) / p.group;
  p.Y = Y; p.ldy = ldy;
  p.vec_x = (uintptr_t)X % 16 == 0 && ldx * tb % 16 == 0;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const long long blocks = (rows + ROWS_BLOCK / 32 - 1) / (ROWS_BLOCK / 32);
  return with_type(type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    constexpr int TOK = 4;
    const long long tiles = (tokens + TOK - 1) / TOK;
    for (long long at = 0; at < tiles; at += 65535) {   // (a grid's second dimension)
      CodesParams q = p;
      q.X = reinterpret_cast<const T*>(X) + at * TOK * ldx;
      q.Y = reinterpret_cast<T*>(Y) + at * TOK * ldy;
      q.tokens = tokens - at * TOK;
      const dim3 grid((unsigned)(blocks < (long long)sms * 8 ? blocks : (long long)sms * 8), (unsigned)(tiles - at < 65535 ? tiles - at : 65535));
      if (tokens == 1) idkm_codes_rows<T, 1><<<grid, ROWS_BLOCK, 0, st>>>(q);
      else idkm_codes_rows<T, TOK><<<grid, ROWS_BLOCK, 0, st>>>(q);
      if (cudaGetLastError() != cudaSuccess) return IDKM_ERR_CUDA;
    }
    return IDKM_OK;
  });
}
