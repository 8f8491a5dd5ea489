// Products with 4-bit weights and group scales for many rows of 16-bit X (a prompt, a large batch), on the tensor cores.
//
// A block computes tiles of 128 rows of W by N = 2 HN rows of X, W's codes taken apart on the way: a thread of the looking-up
// warps has a row of W, turns 128 of its codes into 64 pairs of codebook entries (a table of the 256 pairs with a copy for every
// lane, as for few rows of X) and stores them into tensor memory, where tcgen05.mma takes its first operand from: codes never
// become weights in shared memory, whose bandwidth the second operand, X, needs.  The scale of a group multiplies its fp32 sum, in
// registers: two accumulators of HN columns take turns, and while the tensor cores work on one, the threads that keep the
// sums (a row of W and HN rows of X each) add the other's, times the row's scale, to theirs.  So every product is that of the
// codebook's own values, as for few rows; a scale multiplied into the operand would be rounded to 8 bits with it.
//
// Roles (16 warps): 0-7 sums, 8-11 lookups, 12 issues the products, 13 the copies (TMA; X whose rows do not start on 16 bytes is
// copied by warps 13-15).  Every wait is bounded; if one runs out, the block's results are NaN.
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <type_traits>
#include "idkm_codes.cuh"
#include "idkm_per_device.h"
#include "../../include/idkm.h"

namespace idkm {
namespace {

constexpr int PR_M = 128, PR_BLOCK = 512, PR_K = 128;   // rows of W of a tile, threads, columns of a chunk (one buffer of the first operand)
constexpr int PR_XS = 4, PR_CS = 2;                     // stages of X (64 columns), of codes (256 columns)
constexpr int PR_TABLE = 32 * 1024, PR_CODES = PR_M * 128;

template <int HN>
struct PrCfg {
  static constexpr int N = 2 * HN, X_STAGE = N * 128;
  static constexpr int OFF_CODES = PR_TABLE, OFF_X = OFF_CODES + PR_CS * PR_CODES, BYTES = OFF_X + PR_XS * X_STAGE;
  static constexpr int SMEM = BYTES + PR_TABLE;   // (the table lies on a multiple of its size)
  static constexpr int A0 = N, COLS = N + 128 <= 256 ? 256 : 512;   // columns of tensor memory: accumulators, then two buffers of 64
};

__device__ __forceinline__ unsigned pr_smem(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }

// K-major operand of rows of 128 bytes, swizzled by 128: 8 rows are 1024 bytes.
__device__ __forceinline__ unsigned long long pr_desc(unsigned addr) {
  return (unsigned long long)((addr >> 4) & 0x3fffu) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

__device__ __forceinline__ void pr_store32(unsigned addr, const unsigned (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
      "%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]),
      "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
__device__ __forceinline__ void pr_load16(unsigned addr, unsigned (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
}
// what has been asked for has arrived; r depends on it
__device__ __forceinline__ void pr_arrived(unsigned (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void pr_commit(unsigned bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pr_tma(unsigned to, const CUtensorMap* map, int x, int y, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void pr_expect(unsigned bar, int bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// A place in a ring of buffers: which one, and the parity of its next completion.
template <int S>
struct PrRing {
  int at = 0;
  unsigned parity = 0;
  __device__ __forceinline__ void next() {
    if (++at == S) {
      at = 0;
      parity ^= 1u;
    }
  }
};

// SEGS: groups of a chunk (1 where groups are longer), whose sums are taken one by one.
template <class T, int HN, int SEGS, bool TMA>
__global__ void __launch_bounds__(PR_BLOCK, 1) idkm_codes_prompt(const __grid_constant__ CodesParams p, const __grid_constant__ CUtensorMap map_codes,
                                                                 const __grid_constant__ CUtensorMap map_x) {
  using Cfg = PrCfg<HN>;
  constexpr int STEPS = 8 / SEGS;   // products of 16 columns of a segment
  T* const type = nullptr;
  extern __shared__ __align__(16) unsigned char pr_raw[];
  __shared__ __align__(8) unsigned long long s_bar[2 * PR_XS + 2 * PR_CS + 8];
  __shared__ unsigned s_tmem;
  const unsigned raw = pr_smem(pr_raw), base = (raw + PR_TABLE - 1) & ~(unsigned)(PR_TABLE - 1);
  unsigned char* const mem = pr_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned bars = pr_smem(s_bar);
  const unsigned x_full = bars, x_empty = x_full + 8 * PR_XS, c_full = x_empty + 8 * PR_XS, c_empty = c_full + 8 * PR_CS;
  const unsigned a_full = c_empty + 8 * PR_CS, a_empty = a_full + 16, d_full = a_empty + 16, d_empty = d_full + 16;
  if (tid == 0) {
    for (int i = 0; i < PR_XS; ++i) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(x_full + 8 * i), "r"(TMA ? 1 : 96) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(x_empty + 8 * i) : "memory");
    }
    for (int i = 0; i < PR_CS; ++i) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(c_full + 8 * i) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 4;" ::"r"(c_empty + 8 * i) : "memory");
    }
    for (int i = 0; i < 2; ++i) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 4;" ::"r"(a_full + 8 * i) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(a_empty + 8 * i) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(d_full + 8 * i) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 4;" ::"r"(d_empty + 8 * i) : "memory");
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(pr_smem(&s_tmem)), "r"(Cfg::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid < 256) {   // the pairs of codebook entries, one for every lane
    const unsigned short* c = reinterpret_cast<const unsigned short*>(p.C);
    const unsigned lo = (tid & 15) < p.k ? __ldg(c + (tid & 15)) : 0u, hi = (tid >> 4) < p.k ? __ldg(c + (tid >> 4)) : 0u, both = lo | hi << 16;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(base + tid * 128 + ((q + lane) & 7) * 16), "r"(both) : "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned tmem = *reinterpret_cast<volatile unsigned*>(&s_tmem);

  const int n_chunks = (int)((p.cols + PR_K - 1) / PR_K);
  const long long tiles_x = (p.tokens + Cfg::N - 1) / Cfg::N, tiles = tiles_x * ((p.rows + PR_M - 1) / PR_M);
  bool ok = true;

  if (warp < 8) {   // ---- the sums
    asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
    const int h = warp >> 2, quad = warp & 3;
    const unsigned from = tmem + ((unsigned)(quad * 32) << 16) + (unsigned)(h * HN);
    const int per = SEGS > 1 ? 1 : (int)(p.group / PR_K);   // chunks of a group
    unsigned parity = 0;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
      const long long row = tile / tiles_x * PR_M + quad * 32 + lane, tok0 = tile % tiles_x * Cfg::N + h * HN;
      const unsigned short* s_row = p.scales && row < p.rows ? reinterpret_cast<const unsigned short*>(p.scales) + row * p.n_groups : nullptr;
      float acc[HN];
#pragma unroll
      for (int i = 0; i < HN; ++i) acc[i] = 0.f;
      int g = 0, left = per;   // the group, and chunks of it that are left
      unsigned short next = s_row ? __ldg(s_row) : (unsigned short)0;
#pragma unroll 1
      for (int seg = 0; seg < n_chunks * SEGS; ++seg) {
        const float s = p.scales ? code_scale(next, type) : 1.f;
        if (SEGS > 1 || --left == 0) {
          left = per;
          ++g;
          next = 0;   // (groups past the last one: columns past the last one, 0)
          if (s_row && g < p.n_groups) next = __ldg(s_row + g);
        }
        if (ok) ok = code_wait(d_full + 8 * h, parity);
        parity ^= 1u;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        unsigned r0[16], r1[16];
        auto add = [&](const unsigned (&r)[16], int at) {
#pragma unroll
          for (int i = 0; i < 16; i += 2)
            asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%0, %1};\n\tfma.rn.f32x2 c, a, b, c;\n\tmov.b64 {%0, %1}, c;\n\t}"
                : "+f"(acc[at + i]), "+f"(acc[at + i + 1]) : "r"(r[i]), "r"(r[i + 1]), "f"(s));
        };
        pr_load16(from, r0);
#pragma unroll
        for (int at = 0; at < HN; at += 32) {
          pr_arrived(r0);
          if (at + 16 < HN) pr_load16(from + at + 16, r1);
          else {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) code_arrive(d_empty + 8 * h);
          }
          add(r0, at);
          if (at + 16 < HN) {
            pr_arrived(r1);
            if (at + 32 < HN) pr_load16(from + at + 32, r0);
            else {
              asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
              __syncwarp();
              if (lane == 0) code_arrive(d_empty + 8 * h);
            }
            add(r1, at + 16);
          }
        }
      }
      if (row < p.rows) {
        T* y = reinterpret_cast<T*>(p.Y) + row;
#pragma unroll
        for (int i = 0; i < HN; ++i)
          if (tok0 + i < p.tokens) y[(tok0 + i) * p.ldy] = from_f32<T>(ok ? acc[i] : __int_as_float(0x7fc00000));
      }
    }
  } else if (warp < 12) {   // ---- the lookups
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    const int quad = warp & 3, r = quad * 32 + lane;
    unsigned mine;   // (there after the barrier only)
    asm volatile("or.b32 %0, %1, %2;" : "=r"(mine) : "r"(base), "r"((unsigned)lane * 4u) : "memory");
    const unsigned my_codes = base + Cfg::OFF_CODES + (unsigned)r * 128u;
    const unsigned to = tmem + ((unsigned)(quad * 32) << 16) + (unsigned)Cfg::A0;
    PrRing<PR_CS> cr;
    PrRing<2> ar;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
#pragma unroll 1
      for (int c = 0; c < n_chunks; ++c) {
        if (ok && (c & 1) == 0) ok = code_wait(c_full + 8 * cr.at, cr.parity);
        if (ok) ok = code_wait(a_empty + 8 * ar.at, ar.parity ^ 1u);
        ok = __all_sync(0xffffffffu, ok);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          unsigned v[32];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const unsigned piece = (unsigned)((c & 1) * 4 + half * 2 + j);
            unsigned w[4];
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                         : "r"(my_codes + cr.at * PR_CODES + ((piece ^ (unsigned)(r & 7)) << 4)) : "memory");
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const unsigned o[4] = {w[q] << 7, w[q] >> 1, w[q] >> 9, w[q] >> 17};
#pragma unroll
              for (int i = 0; i < 4; ++i) asm("ld.shared.u32 %0, [%1];" : "=r"(v[j * 16 + q * 4 + i]) : "r"((o[i] & 0x7f80u) | mine));
            }
          }
          pr_store32(to + (unsigned)(ar.at * 64 + half * 32), v);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          code_arrive(a_full + 8 * ar.at);
          if ((c & 1) || c + 1 == n_chunks) code_arrive(c_empty + 8 * cr.at);
        }
        if ((c & 1) || c + 1 == n_chunks) cr.next();
        ar.next();
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 12) {   // ---- the products
      if (lane == 0) {
        const unsigned kind = std::is_same<T, __half>::value ? 0u : 1u;
        const unsigned idesc = (1u << 4) | (kind << 7) | (kind << 10) | ((unsigned)(HN >> 3) << 17) | ((unsigned)(PR_M >> 4) << 24);
        PrRing<PR_XS> xr;
        PrRing<2> ar;
        unsigned d_turn = 1;   // (both accumulators are free at first)
        for (long long tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
#pragma unroll 1
          for (int c = 0; c < n_chunks && ok; ++c) {
            ok = code_wait(a_full + 8 * ar.at, ar.parity);
            const int x0 = xr.at;
            ok = ok && code_wait(x_full + 8 * xr.at, xr.parity);
            xr.next();
            const int x1 = xr.at;
            ok = ok && code_wait(x_full + 8 * xr.at, xr.parity);
            xr.next();
#pragma unroll
            for (int seg = 0; seg < SEGS; ++seg) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                ok = ok && code_wait(d_empty + 8 * h, d_turn);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                  const int k16 = seg * STEPS + i;
                  const unsigned long long b = pr_desc(base + Cfg::OFF_X + (k16 < 4 ? x0 : x1) * Cfg::X_STAGE + h * HN * 128 + (k16 & 3) * 32);
                  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                               ::"r"(tmem + (unsigned)(h * HN)), "r"(tmem + (unsigned)(Cfg::A0 + ar.at * 64 + k16 * 8)), "l"(b), "r"(idesc), "r"(i > 0 ? 1u : 0u)
                               : "memory");
                }
                pr_commit(d_full + 8 * h);
              }
              d_turn ^= 1u;
            }
            if (ok) {
              pr_commit(a_empty + 8 * ar.at);
              pr_commit(x_empty + 8 * x0);
              pr_commit(x_empty + 8 * x1);
            }
            ar.next();
          }
        }
      }
    } else {   // ---- the copies
      PrRing<PR_XS> xr;
      PrRing<PR_CS> cr;
      bool x_filled = false, c_filled = false;   // every stage has been filled once
      for (long long tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
        const long long row0 = tile / tiles_x * PR_M, tok0 = tile % tiles_x * Cfg::N;
#pragma unroll 1
        for (int c = 0; c < n_chunks && ok; ++c) {
          if (warp == 13 && lane == 0 && (c & 1) == 0) {
            if (c_filled) ok = code_wait(c_empty + 8 * cr.at, cr.parity ^ 1u);
            if (ok) {
              pr_expect(c_full + 8 * cr.at, PR_CODES);
              pr_tma(base + Cfg::OFF_CODES + cr.at * PR_CODES, &map_codes, c * (PR_K / 2), (int)row0, c_full + 8 * cr.at);
              cr.next();
              if (cr.at == 0) c_filled = true;
            }
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const unsigned at = base + Cfg::OFF_X + xr.at * Cfg::X_STAGE;
            if (TMA) {
              if (warp == 13 && lane == 0) {
                if (x_filled && ok) ok = code_wait(x_empty + 8 * xr.at, xr.parity ^ 1u);
                if (ok) {
                  pr_expect(x_full + 8 * xr.at, Cfg::X_STAGE);
                  pr_tma(at, &map_x, c * PR_K + j * 64, (int)tok0, x_full + 8 * xr.at);
                }
              }
            } else {
              if (x_filled && ok) ok = code_wait(x_empty + 8 * xr.at, xr.parity ^ 1u);
              for (int i = tid - 13 * 32; i < Cfg::N * 8; i += 96) {
                const int m = i >> 3, v = i & 7;
                uint4 x = make_uint4(0u, 0u, 0u, 0u);
                if (tok0 + m < p.tokens) x = code_load8(reinterpret_cast<const T*>(p.X) + (tok0 + m) * p.ldx, c * PR_K + j * 64 + v * 8, p.cols);
                *reinterpret_cast<uint4*>(mem + Cfg::OFF_X + xr.at * Cfg::X_STAGE + m * 128 + ((v ^ (m & 7)) << 4)) = x;
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              code_arrive(x_full + 8 * xr.at);
            }
            xr.next();
            if (xr.at == 0) x_filled = true;
          }
        }
      }
      // nothing is left under way when the block ends: every stage that was filled has been waited for by those who read it, unless
      // they gave up
      if (warp == 13 && lane == 0 && !ok) {
        for (int i = 0; i < 2 * PR_CS; ++i) code_wait(c_full + 8 * (i % PR_CS), (unsigned)(i / PR_CS));
        for (int i = 0; i < 2 * PR_XS; ++i) code_wait(x_full + 8 * (i % PR_XS), (unsigned)(i / PR_XS));
      }
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Cfg::COLS));
}

typedef CUresult (*PrEncode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
PrEncode pr_encode() {
  static const PrEncode f = [] {
    void* q = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &q, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      q = nullptr;
    return reinterpret_cast<PrEncode>(q);
  }();
  return f;
}
// A matrix of `rows` rows of `inner` elements, `pitch` bytes apart, read by boxes of 128 bytes by `box` rows, swizzled; zeros outside.
bool pr_map(CUtensorMap& m, CUtensorMapDataType type, int bytes, const void* at, long long inner, long long rows, long long pitch, int box) {
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
  const cuuint32_t boxes[2] = {(cuuint32_t)(128 / bytes), (cuuint32_t)box}, steps[2] = {1, 1};
  return pr_encode()(&m, type, 2, const_cast<void*>(at), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int HN, int SEGS, bool TMA>
cudaError_t pr_launch(const CodesParams& p, int sms, cudaStream_t st) {
  using Cfg = PrCfg<HN>;
  CUtensorMap codes, x = {};
  if (!pr_map(codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.codes, (p.cols + 31) / 32 * 16, p.rows, p.pitch, PR_M)) return cudaErrorInvalidValue;
  if (TMA && !pr_map(x, std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.X, p.cols, p.tokens,
                     p.ldx * 2, Cfg::N))
    return cudaErrorInvalidValue;
  static PerDevice limit;
  const cudaError_t rc = allow_smem(limit, idkm_codes_prompt<T, HN, SEGS, TMA>, Cfg::SMEM);
  if (rc != cudaSuccess) return rc;
  const long long tiles = (p.rows + PR_M - 1) / PR_M * ((p.tokens + Cfg::N - 1) / Cfg::N);
  idkm_codes_prompt<T, HN, SEGS, TMA><<<(int)(tiles < sms ? tiles : sms), PR_BLOCK, Cfg::SMEM, st>>>(p, codes, x);
  return cudaGetLastError();
}

template <class T, int HN>
cudaError_t pr_launch(const CodesParams& p, int sms, cudaStream_t st) {
  const int segs = !p.scales || p.group >= 128 ? 1 : (int)(128 / p.group);
  if (p.vec_x) return segs == 1 ? pr_launch<T, HN, 1, true>(p, sms, st) : segs == 2 ? pr_launch<T, HN, 2, true>(p, sms, st) : pr_launch<T, HN, 4, true>(p, sms, st);
  return segs == 1 ? pr_launch<T, HN, 1, false>(p, sms, st) : segs == 2 ? pr_launch<T, HN, 2, false>(p, sms, st) : pr_launch<T, HN, 4, false>(p, sms, st);
}

}  // namespace

cudaError_t codes_prompt(const CodesParams& p, int type, int sms, cudaStream_t st) {
  if (!pr_encode()) return cudaErrorNotSupported;
  if (p.rows > INT32_MAX - PR_M || p.cols > INT32_MAX - 512 || p.tokens > INT32_MAX - 256) return cudaErrorInvalidValue;
  // rows of X of a tile: those whose waves of tiles cost least; a chunk costs its products, 4 cycles a row of X, but at least the
  // lookups (420)
  const long long tiles_w = (p.rows + PR_M - 1) / PR_M;
  int best = 128;
  long long least = INT64_MAX;
  for (int hn = 16; hn <= 128; hn *= 2) {
    const long long tiles = tiles_w * ((p.tokens + 2 * hn - 1) / (2 * hn)), cost = (tiles + sms - 1) / sms * (8 * hn > 420 ? 8 * hn : 420);
    if (cost < least || (cost == least && hn <= best)) {
      least = cost;
      best = hn;
    }
  }
  auto run = [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return best == 16 ? pr_launch<T, 16>(p, sms, st) : best == 32 ? pr_launch<T, 32>(p, sms, st) : best == 64 ? pr_launch<T, 64>(p, sms, st) : pr_launch<T, 128>(p, sms, st);
  };
  return type == ELEM_BF16 ? run((__nv_bfloat16*)nullptr) : run((__half*)nullptr);
}

}  // namespace idkm
