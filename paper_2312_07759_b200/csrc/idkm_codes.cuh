// What the kernels of products with 4-bit codes share.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>
#include "idkm_types.cuh"

namespace idkm {

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
  int missing;   // 16-bit X: the copy of codes that is left out (a test's; below 0: none)
};

// Products for many rows of 16-bit X, on the tensor cores (idkm_codes_prompt.cu).
struct PromptPlan {
  int hn, split;   // half the rows of X of a tile; pairs of blocks that share its columns
  long long ns;    // what it takes, about
};
PromptPlan codes_prompt_plan(const CodesParams& p, int sms);
cudaError_t codes_prompt(const CodesParams& p, int type, const PromptPlan& plan, int sms, cudaStream_t st);

__device__ __forceinline__ float code_scale(unsigned short u, __nv_bfloat16*) { return __uint_as_float((unsigned)u << 16); }
__device__ __forceinline__ float code_scale(unsigned short u, __half*) { return __half2float(__ushort_as_half(u)); }

// Eight 16-bit elements that begin `off` bytes (an even number) into the first of two words of memory; zeros from the `left`-th on.
__device__ __forceinline__ uint4 code_align8(const uint4& a, const uint4& b, unsigned off, int left) {
  unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (off) {
    if (off & 8u) { w[0] = w[2]; w[1] = w[3]; w[2] = w[4]; w[3] = w[5]; w[4] = w[6]; w[5] = w[7]; }
    if (off & 4u) { w[0] = w[1]; w[1] = w[2]; w[2] = w[3]; w[3] = w[4]; w[4] = w[5]; }
    if (off & 2u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
  }
  if (left < 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= left >= 2 * i + 2 ? ~0u : left == 2 * i + 1 ? 0xffffu : 0u;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// The 16-byte word of memory at `word` and the next one, each where it is wanted, zeros elsewhere; nothing branches, so that what
// is asked for next does not wait.
__device__ __forceinline__ void code_ask(uint4& a, uint4& b, uintptr_t word, int first, int second) {
  a = b = make_uint4(0u, 0u, 0u, 0u);
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %9, 0;\n\tsetp.ne.b32 q, %10, 0;\n\t@p ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%8];\n\t"
               "@q ld.global.nc.v4.u32 {%4, %5, %6, %7}, [%8+16];\n\t}"
               : "+r"(a.x), "+r"(a.y), "+r"(a.z), "+r"(a.w), "+r"(b.x), "+r"(b.y), "+r"(b.z), "+r"(b.w) : "l"(word), "r"(first), "r"(second));
}

constexpr int CODE_POLLS = 1 << 19;   // (each waits for some time itself, 2 us: about a second)
__device__ __forceinline__ bool code_wait(unsigned bar, unsigned parity) {
  for (int i = 0; i < CODE_POLLS; ++i) {
    unsigned done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (done) return true;
  }
  return false;
}
__device__ __forceinline__ void code_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

}  // namespace idkm
