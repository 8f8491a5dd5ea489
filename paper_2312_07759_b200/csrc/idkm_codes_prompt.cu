// Products with 4-bit weights and group scales for many rows of 16-bit X (a prompt, a large batch), on the tensor cores.
//
// A pair of blocks (a cluster) computes tiles of 256 rows of W, 128 a block, by N = 2 HN rows of X, of which either block holds
// half (tcgen05 with cta_group::2: a block's X serves the other's rows of W too, so X comes from L2 and through shared memory once
// for 256 rows).  W's codes are taken apart on the way: a thread of the looking-up warps has a row of W, turns 128 of its codes into
// 64 pairs of codebook entries (a table of the 256 pairs with a copy for every lane, as for few rows of X) and stores them into tensor
// memory, where tcgen05.mma takes its first operand from: codes never become weights in shared memory.  The scale of a group
// multiplies its fp32 sum, in registers: three accumulators of HN columns take turns (with two, the
// products wait for the sums), and while the tensor cores work on one, the threads that keep the
// sums (a row of W and HN / 2 rows of X each) add another's, times the row's scale, to theirs.  So every product
// is that of the codebook's own values, as for few rows; a scale multiplied into the operand would be rounded to 8 bits with it.
//
// Roles (24 warps a block): 0-15 sums, 16-19 lookups, 20 issues the products (the first block's, for both), 21 and 22 the copies
// (TMA; X whose rows do not start on 16 bytes is copied by warps 21-23).  What the issuing thread waits for -- X, lookups, accumulators
// that have been added -- is counted in the first block's barriers, by both; what it frees it tells both.  Every wait is
// bounded.  Whoever's wait runs out hands nothing over any more, so that the waits for it run out too, those of the sums last, and the
// pair's results are NaN.
//
// Where there are fewer tiles than pairs of blocks, 2 or 4 pairs of a cluster share a tile's columns; their sums meet in the first one's
// shared memory, in a fixed order (32 rows of X through 8192 x 28672: 129 us -> 71 with 2 pairs; 40 through 535 x 11392: 54 -> 22 with 4).
//
// What bounds it: the sums, whose loads from tensor memory compete with the products' own accumulators for it (without them 198 us
// of 237, groups of 128), then the products.
// Measured, 2048 rows through 8192 x 8192 bf16: 237 us, 1160 TFLOP/s, 0.70 of a plain library product's rate in a burst.
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <atomic>
#include <type_traits>
#include "idkm_codes.cuh"
#include "idkm_per_device.h"
#include "../../include/idkm.h"

namespace idkm {
namespace {

constexpr int PR_M = 128, PR_BLOCK = 768, PR_K = 128;   // rows of W of a tile, threads, columns of a chunk (one buffer of the first operand)
constexpr int PR_XS = 6, PR_CS = 3, PR_DS = 3;          // stages of X (64 columns), of codes (256 columns), accumulators
constexpr int PR_ASK = 2;                               // words of X that a thread has under way where TMA cannot copy it
constexpr int PR_SPLIT = 4;                             // pairs of blocks that share a tile's columns, at most
// shared memory: the codes before the table, which lies on a multiple of 64 KB (an address is put together by bytes), X after it
constexpr int PR_TABLE = 64 * 1024, PR_CODES = PR_M * 128, PR_FRONT = PR_TABLE - 1024;   // (shared memory starts at 1 KB or above)

template <int HN>
struct PrCfg {
  static constexpr int N = 2 * HN, X_HALF = HN / 2 * 128, X_STAGE = 2 * X_HALF;   // a block's rows of X for either accumulator
  static constexpr int SMEM = PR_FRONT + PR_TABLE + PR_XS * X_STAGE;
  static_assert(SMEM + 1024 + 256 <= 228 * 1024 && PR_CS * PR_CODES + 8192 <= PR_TABLE, "the X stages after the table, the codes' before");
  static_assert(1024 * HN <= PR_TABLE + PR_XS * X_STAGE, "the sums of a block fit there");
  static constexpr int A0 = PR_DS * HN, COLS = A0 + 128 <= 256 ? 256 : 512;   // columns of tensor memory: accumulators, then two buffers of 64
};

__device__ __forceinline__ unsigned pr_smem(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }

// A product of 16 columns, both blocks' 128 rows by HN rows of X.  b: 16-byte words to the second operand, K-major rows of 128
// bytes, swizzled by 128, 8 rows 1024 bytes.
__device__ __forceinline__ void pr_mma(unsigned d, unsigned a, unsigned b, unsigned idesc, unsigned accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 x, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], x, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"((int)(64u | (1u << 14) | (2u << 29)))
      : "memory");
}

__device__ __forceinline__ void pr_store16(unsigned addr, const unsigned (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(v[0]), "r"(v[1]),
      "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]),
      "r"(v[14]), "r"(v[15])
      : "memory");
}
template <int W>   // 8 or 16
__device__ __forceinline__ void pr_load(unsigned addr, unsigned (&r)[W]) {
  if constexpr (W == 16)
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
  else
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr)
                 : "memory");
}
// what has been asked for has arrived; r depends on it
template <int W>
__device__ __forceinline__ void pr_arrived(unsigned (&r)[W]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < W; ++i) asm volatile("" : "+r"(r[i]));
}
// to the barrier of either block of the pair, once the products issued so far are done
__device__ __forceinline__ void pr_commit(unsigned bar, unsigned short pair) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(pair) : "memory");
}
__device__ __forceinline__ void pr_tma(unsigned to, const CUtensorMap* map, int x, int y, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// the same, telling the first block's barrier
__device__ __forceinline__ void pr_tma_pair(unsigned to, const CUtensorMap* map, int x, int y, unsigned first_bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(first_bar) : "memory");
}
// an address of a block of the cluster
__device__ __forceinline__ unsigned pr_there(unsigned at, unsigned block) {
  unsigned r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(block));
  return r;
}
// all threads of the cluster
__device__ __forceinline__ void pr_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// (What is handed over lies in tensor memory, and the fence before orders it: nothing written to memory has to be waited for.)
__device__ __forceinline__ void pr_arrive_first(unsigned first_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(first_bar) : "memory");
}
__device__ __forceinline__ void pr_arrive_first_written(unsigned first_bar) {   // ... where it does
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(first_bar) : "memory");
}
__device__ __forceinline__ bool pr_wait_both(unsigned bar, unsigned parity) {   // for what both blocks count
  for (int i = 0; i < CODE_POLLS; ++i) {
    unsigned done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (done) return true;
  }
  return false;
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
  // Waits for what each buffer was last begun with (a buffer that was never begun with: not at all).
  __device__ __forceinline__ void drain(unsigned full) const {
#pragma unroll 1
    for (int i = 0; i < S; ++i) code_wait(full + 8 * i, i < at ? parity : parity ^ 1u);
  }
};

// SEGS: groups of a chunk (1 where groups are longer), whose sums are taken one by one.
template <class T, int HN, int SEGS, bool TMA>
__global__ void __launch_bounds__(PR_BLOCK, 1) idkm_codes_prompt(const __grid_constant__ CodesParams p, const __grid_constant__ CUtensorMap map_codes,
                                                                 const __grid_constant__ CUtensorMap map_x, int split) {
  using Cfg = PrCfg<HN>;
  constexpr int STEPS = 8 / SEGS;   // products of 16 columns of a segment
  T* const type = nullptr;
  extern __shared__ __align__(16) unsigned char pr_raw[];
  __shared__ __align__(8) unsigned long long s_bar[2 * PR_XS + 2 * PR_CS + 4 + 2 * PR_DS + 1];
  __shared__ unsigned s_tmem;
  const unsigned raw = pr_smem(pr_raw), base = (raw + PR_TABLE - 1) & ~(unsigned)(PR_TABLE - 1);
  // (codes and X on multiples of 1024, which the swizzle goes by)
  const unsigned codes0 = base - PR_CS * PR_CODES, x0_at = base + PR_TABLE;
  unsigned char* const mem_x = pr_raw + (x0_at - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x & 1;
  const int pair = (int)(blockIdx.x % (unsigned)(2 * split)) >> 1;   // of the cluster
  const unsigned first = 2u * (unsigned)pair;
  const unsigned bars = pr_smem(s_bar);
  const unsigned x_full = bars, x_empty = x_full + 8 * PR_XS, c_full = x_empty + 8 * PR_XS, c_empty = c_full + 8 * PR_CS;
  const unsigned a_full = c_empty + 8 * PR_CS, a_empty = a_full + 16, d_full = a_empty + 16, d_empty = d_full + 8 * PR_DS, all_done = d_empty + 8 * PR_DS;
  if (tid == 0) {
    for (int i = 0; i < PR_XS; ++i) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(x_full + 8 * i), "r"(TMA ? 1 : 6) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(x_empty + 8 * i) : "memory");
    }
    for (int i = 0; i < PR_CS; ++i) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(c_full + 8 * i) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 4;" ::"r"(c_empty + 8 * i) : "memory");
    }
    for (int i = 0; i < 2; ++i) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 8;" ::"r"(a_full + 8 * i) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(a_empty + 8 * i) : "memory");
    }
    for (int i = 0; i < PR_DS; ++i) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(d_full + 8 * i) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 16;" ::"r"(d_empty + 8 * i) : "memory");
    }
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(all_done) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 20) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(pr_smem(&s_tmem)), "r"(Cfg::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (tid < 256) {   // the pairs of codebook entries, one for every lane
    const unsigned short* c = reinterpret_cast<const unsigned short*>(p.C);
    const unsigned lo = (tid & 15) < p.k ? __ldg(c + (tid & 15)) : 0u, hi = (tid >> 4) < p.k ? __ldg(c + (tid >> 4)) : 0u, both = lo | hi << 16;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(base + tid * 256 + ((q + lane) & 7) * 16), "r"(both) : "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  pr_meet();   // (all blocks run, their barriers are ready)
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned tmem = *reinterpret_cast<volatile unsigned*>(&s_tmem);

  // this pair's chunks: from chunk0 on (an even one, codes are copied by two)
  const int all_chunks = (int)((p.cols + PR_K - 1) / PR_K), share = ((all_chunks + 1) / 2 + split - 1) / split * 2, chunk0 = min(pair * share, all_chunks);
  const int n_chunks = min(share, all_chunks - chunk0);
  const long long tiles_x = (p.tokens + Cfg::N - 1) / Cfg::N, tiles = tiles_x * ((p.rows + 2 * PR_M - 1) / (2 * PR_M));
  const long long tile0 = blockIdx.x / (unsigned)(2 * split), tile_on = gridDim.x / (unsigned)(2 * split);
  bool ok = true;

  if (warp < 16) {   // ---- the sums
    asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
    constexpr int HC = HN / 2;   // columns of a thread
    const int h = warp >> 3, part = warp >> 2 & 1, quad = warp & 3;
    const unsigned from0 = tmem + ((unsigned)(quad * 32) << 16) + (unsigned)(part * HC);
    const int per = SEGS > 1 ? 1 : (int)(p.group / PR_K);   // chunks of a group
    const unsigned d_added = pr_there(d_empty, first);
    int buffer = h;        // every second accumulation is this half's, the accumulators take turns
    unsigned parity = 0;
    for (long long tile = tile0; tile < tiles; tile += tile_on) {
      const long long row = (tile / tiles_x * 2 + rank) * PR_M + quad * 32 + lane, tok0 = tile % tiles_x * Cfg::N + h * HN + part * HC;
      const unsigned short* s_row = p.scales && row < p.rows ? reinterpret_cast<const unsigned short*>(p.scales) + row * p.n_groups : nullptr;
      float acc[HC];
#pragma unroll
      for (int i = 0; i < HC; ++i) acc[i] = 0.f;
      int g = SEGS > 1 ? chunk0 * SEGS : chunk0 / per, left = SEGS > 1 ? per : per - (chunk0 - g * per);   // the group, and chunks of it that are left
      unsigned short next = s_row && g < p.n_groups ? __ldg(s_row + g) : (unsigned short)0;
#pragma unroll 1
      for (int seg = 0; seg < n_chunks * SEGS; ++seg) {
        const float s = p.scales ? code_scale(next, type) : 1.f;
        if (SEGS > 1 || --left == 0) {
          left = per;
          ++g;
          next = 0;   // (groups past the last one: columns past the last one, 0)
          if (s_row && g < p.n_groups) next = __ldg(s_row + g);
        }
        if (ok) ok = code_wait(d_full + 8 * buffer, parity);
        const unsigned from = from0 + (unsigned)(buffer * HN), added = d_added + 8 * buffer;
        buffer += 2;
        if (buffer >= PR_DS) {
          buffer -= PR_DS;
          parity ^= 1u;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        constexpr int W = HC < 16 ? 8 : 16;
        unsigned r0[W], r1[W];
        auto add = [&](const unsigned (&r)[W], int at) {
#pragma unroll
          for (int i = 0; i < W; i += 2)
            asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%0, %1};\n\tfma.rn.f32x2 c, a, b, c;\n\tmov.b64 {%0, %1}, c;\n\t}"
                : "+f"(acc[at + i]), "+f"(acc[at + i + 1]) : "r"(r[i]), "r"(r[i + 1]), "f"(s));
        };
        auto taken = [&] {   // everything has arrived: the accumulator is free
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) pr_arrive_first(added);
        };
#pragma unroll
        for (int at = 0; at < HC; at += 2 * W) {
          pr_load(from + at, r0);
          if (at + W < HC) pr_load(from + at + W, r1);
          pr_arrived(r0);
          if (at + W < HC) pr_arrived(r1);
          if (at + 2 * W >= HC) taken();
          add(r0, at);
          if (at + W < HC) add(r1, at + W);
        }
      }
      // the pairs' sums: a half of the pairs sends, through the table's memory and that of X behind it, the other half adds
      for (int step = 1; step < split; step *= 2) {
        __syncwarp();
        pr_meet();   // (the table and X are not needed any more, what was sent before has been read)
        if (pair % (2 * step) == step) {
          const unsigned there = pr_there(base, (unsigned)(2 * (pair - step) + rank)) + (unsigned)tid * 4u;
#pragma unroll
          for (int i = 0; i < HC; ++i)
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there + (unsigned)i * 2048u), "f"(ok ? acc[i] : __int_as_float(0x7fc00000)) : "memory");
        }
        pr_meet();
        if (pair % (2 * step) == 0) {
#pragma unroll
          for (int i = 0; i < HC; ++i) {
            float v;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(base + (unsigned)tid * 4u + (unsigned)i * 2048u) : "memory");
            acc[i] += v;
          }
        }
      }
      if (row < p.rows && pair == 0) {
        T* y = reinterpret_cast<T*>(p.Y) + row;
#pragma unroll
        for (int i = 0; i < HC; ++i)
          if (tok0 + i < p.tokens) y[(tok0 + i) * p.ldy] = from_f32<T>(ok ? acc[i] : __int_as_float(0x7fc00000));
      }
    }
  } else if (warp < 20) {   // ---- the lookups
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    const int quad = warp & 3, r = quad * 32 + lane;
    unsigned mine;   // (there after the barrier only)
    asm volatile("or.b32 %0, %1, %2;" : "=r"(mine) : "r"(base), "r"((unsigned)lane * 4u) : "memory");
    const unsigned my_codes = codes0 + (unsigned)r * 128u;
    const unsigned to = tmem + ((unsigned)(quad * 32) << 16) + (unsigned)Cfg::A0;
    const unsigned a_there = pr_there(a_full, first);
    PrRing<PR_CS> cr;
    PrRing<2> ar;
    for (long long tile = tile0; tile < tiles && ok; tile += tile_on) {
#pragma unroll 1
      for (int c = 0; c < n_chunks; ++c) {
        if ((c & 1) == 0) ok = code_wait(c_full + 8 * cr.at, cr.parity);
        unsigned w[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[j][0]), "=r"(w[j][1]), "=r"(w[j][2]), "=r"(w[j][3])
                       : "r"(my_codes + cr.at * PR_CODES + ((((unsigned)(c & 1) * 4u + (unsigned)j) ^ (unsigned)(r & 7)) << 4)) : "memory");
        if (ok) ok = code_wait(a_empty + 8 * ar.at, ar.parity ^ 1u);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;   // (the buffer may be in use, the codes may not be there: no products of them)
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          unsigned v[16];
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i)   // (the lane's byte, byte i of the codes, the table's two)
              asm("ld.shared.u32 %0, [%1];" : "=r"(v[q * 4 + i]) : "r"(__byte_perm(mine, w[j][q], 0x3240u + 0x10u * (unsigned)i)));
          pr_store16(to + (unsigned)(ar.at * 64 + j * 16), v);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          pr_arrive_first(a_there + 8 * ar.at);
          if ((c & 1) || c + 1 == n_chunks) code_arrive(c_empty + 8 * cr.at);
        }
        if ((c & 1) || c + 1 == n_chunks) cr.next();
        ar.next();
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 20) {   // ---- the products
      if (rank == 0) {
        // The whole warp goes round, so that what the products are given is known to be the same for all lanes; one lane issues.
        // (One lane going round alone issued a product every 105 cycles, 64 are enough.)
        unsigned chosen;
        asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(chosen));
        const unsigned kind = std::is_same<T, __half>::value ? 0u : 1u;
        const unsigned idesc = (1u << 4) | (kind << 7) | (kind << 10) | ((unsigned)(HN >> 3) << 17) | ((unsigned)(2 * PR_M >> 4) << 24);
        const unsigned d0 = __shfl_sync(0xffffffffu, tmem, 0), x_base = (x0_at >> 4) | (1u << 16);
        const unsigned short both = (unsigned short)(3u << first);
        PrRing<PR_XS> xr;
        PrRing<2> ar;
        PrRing<PR_DS> dr;
        for (long long tile = tile0; tile < tiles && ok; tile += tile_on) {
#pragma unroll 1
          for (int c = 0; c < n_chunks && ok; ++c) {
            ok = pr_wait_both(a_full + 8 * ar.at, ar.parity);
            const int x0 = xr.at;
            ok = ok && pr_wait_both(x_full + 8 * xr.at, xr.parity);
            xr.next();
            const int x1 = xr.at;
            ok = ok && pr_wait_both(x_full + 8 * xr.at, xr.parity);
            xr.next();
            const unsigned b0 = x_base + (unsigned)x0 * (Cfg::X_STAGE / 16), b1 = x_base + (unsigned)x1 * (Cfg::X_STAGE / 16), a0 = d0 + (unsigned)(Cfg::A0 + ar.at * 64);
#pragma unroll
            for (int seg = 0; seg < SEGS; ++seg) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                ok = ok && pr_wait_both(d_empty + 8 * dr.at, dr.parity ^ 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (chosen) {
#pragma unroll
                  for (int i = 0; i < STEPS; ++i) {
                    const int k16 = seg * STEPS + i;
                    pr_mma(d0 + (unsigned)(dr.at * HN), a0 + (unsigned)(k16 * 8), (k16 < 4 ? b0 : b1) + (unsigned)(h * (Cfg::X_HALF / 16) + (k16 & 3) * 2), idesc, i > 0);
                  }
                  pr_commit(d_full + 8 * dr.at, both);
                  if (seg + 1 == SEGS && h == 1) {
                    pr_commit(a_empty + 8 * ar.at, both);
                    pr_commit(x_empty + 8 * x0, both);
                    pr_commit(x_empty + 8 * x1, both);
                  }
                }
                __syncwarp();
                dr.next();
              }
            }
            ar.next();
          }
        }
        // (products under way, of which none is when the block ends, also where a wait ran out)
        if (chosen) pr_commit(all_done, (unsigned short)(1u << first));
        code_wait(all_done, 0u);
      }
    } else if (!TMA || warp == 21 || warp == 22) {   // ---- the copies: with TMA X by one thread, the codes, which are further ahead, by another
      PrRing<PR_XS> xr;
      PrRing<PR_CS> cr;
      bool x_filled = false, c_filled = false;   // every stage has been filled once
      const unsigned x_there = pr_there(x_full, first);
      for (long long tile = tile0; tile < tiles && ok; tile += tile_on) {
        const long long row0 = (tile / tiles_x * 2 + rank) * PR_M, tok0 = tile % tiles_x * Cfg::N;
#pragma unroll 1
        for (int c = 0; c < n_chunks && ok; ++c) {
          if (warp == (TMA ? 22 : 21) && lane == 0 && (c & 1) == 0) {
            if (c_filled) ok = code_wait(c_empty + 8 * cr.at, cr.parity ^ 1u);
            if (ok) {
              if (c / 2 != p.missing) {
                pr_expect(c_full + 8 * cr.at, PR_CODES);
                pr_tma(codes0 + cr.at * PR_CODES, &map_codes, (chunk0 + c) * (PR_K / 2), (int)row0, c_full + 8 * cr.at);
              }
              cr.next();
              if (cr.at == 0) c_filled = true;
            }
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const unsigned at = x0_at + xr.at * Cfg::X_STAGE;
            if (TMA) {
              if (warp == 21 && lane == 0) {
                if (x_filled) ok = code_wait(x_empty + 8 * xr.at, xr.parity ^ 1u);
                if (ok) {
                  if (rank == 0) pr_expect(x_full + 8 * xr.at, 2 * Cfg::X_STAGE);   // (of both blocks)
#pragma unroll
                  for (int h = 0; h < 2; ++h)
                    pr_tma_pair(at + h * Cfg::X_HALF, &map_x, (chunk0 + c) * PR_K + j * 64, (int)tok0 + h * HN + rank * (HN / 2), x_there + 8 * xr.at);
                }
              }
            } else {
              if (x_filled && ok) ok = code_wait(x_empty + 8 * xr.at, xr.parity ^ 1u);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;   // (the stage may be in use)
              // (what PR_ASK words need is asked for before the first is looked at)
              for (int i0 = tid - 21 * 32; i0 < HN * 8; i0 += 96 * PR_ASK) {
                uint4 a[PR_ASK], b[PR_ASK];
                const int k = (chunk0 + c) * PR_K + j * 64 + (i0 & 7) * 8;   // (96 is a multiple of 8: of all of them)
                auto row_of = [&](int i) {
                  const int m = i >> 3, h = m >= HN / 2;   // (halves are whole groups of 8 rows: the swizzle is that of the row in either)
                  return tok0 + h * HN + rank * (HN / 2) + (m - h * (HN / 2));
                };
#pragma unroll
                for (int u = 0; u < PR_ASK; ++u) {
                  const int i = i0 + u * 96;
                  const long long tok = row_of(i);
                  const uintptr_t row = (uintptr_t)(reinterpret_cast<const T*>(p.X) + tok * p.ldx), at = row + 2ll * k, end = row + 2 * p.cols, word = at & ~(uintptr_t)15;
                  const int one = i < HN * 8 && tok < p.tokens && at < end, two = one && (at & 15) && word + 16 < end;
                  code_ask(a[u], b[u], word, one, two);
                }
#pragma unroll
                for (int u = 0; u < PR_ASK; ++u) {
                  const int i = i0 + u * 96, m = i >> 3;
                  if (i >= HN * 8) break;
                  const unsigned off = (unsigned)((uintptr_t)(reinterpret_cast<const T*>(p.X) + row_of(i) * p.ldx) & 15u);   // (columns by eights: the row's)
                  *reinterpret_cast<uint4*>(mem_x + xr.at * Cfg::X_STAGE + m * 128 + (((i & 7) ^ (m & 7)) << 4)) = code_align8(a[u], b[u], off, (int)p.cols - k);
                }
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) pr_arrive_first_written(x_there + 8 * xr.at);
            }
            if (!ok) break;
            xr.next();
            if (xr.at == 0) x_filled = true;
          }
        }
      }
      // nothing is left under way when the block ends, whoever gave up (what X the second block asked for the first one's barrier counts)
      if (lane == 0) {
        if (warp == (TMA ? 22 : 21)) cr.drain(c_full);
        if (TMA && warp == 21 && rank == 0) xr.drain(x_full);
      }
    }
  }
  __syncwarp();
  if (warp >= 16)
    for (int step = 1; step < split; step *= 2) {   // (where the sums meet)
      pr_meet();
      pr_meet();
    }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  pr_meet();   // (no block leaves while another may still tell it something)
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 20) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Cfg::COLS));
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

void pr_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&attr)[1], long long clusters, int split, int smem, cudaStream_t st) {
  cfg.gridDim = dim3((unsigned)(2 * split * clusters));
  cfg.blockDim = dim3(PR_BLOCK);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)(2 * split);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
}
// Clusters of `split` pairs that run at once on the current device (on a B200 74, 33 and 15 of 1, 2 and 4 pairs: fewer than its
// multiprocessors would make, as a cluster stays within a part of them).  Asked for once a device; a block has a multiprocessor in every variant.
int pr_clusters(int split) {
  static std::atomic<int> known[64][PR_SPLIT + 1];   // (0: not asked for yet)
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  const bool keep = dev >= 0 && dev < 64;
  int n = keep ? known[dev][split].load(std::memory_order_relaxed) : 0;
  if (n > 0) return n;
  static PerDevice limit;
  if (allow_smem(limit, idkm_codes_prompt<__nv_bfloat16, 16, 1, true>, PrCfg<16>::SMEM) != cudaSuccess) return 0;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  pr_config(cfg, attr, 1, split, PrCfg<16>::SMEM, nullptr);
  if (cudaOccupancyMaxActiveClusters(&n, idkm_codes_prompt<__nv_bfloat16, 16, 1, true>, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();
    return 0;
  }
  if (keep) known[dev][split].store(n, std::memory_order_relaxed);
  return n;
}

template <class T, int HN, int SEGS, bool TMA>
cudaError_t pr_launch(const CodesParams& p, int split, int sms, cudaStream_t st) {
  using Cfg = PrCfg<HN>;
  CUtensorMap codes, x = {};
  if (!pr_map(codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.codes, (p.cols + 31) / 32 * 16, p.rows, p.pitch, PR_M)) return cudaErrorInvalidValue;
  if (TMA && !pr_map(x, std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.X, p.cols, p.tokens,
                     p.ldx * 2, HN / 2))
    return cudaErrorInvalidValue;
  static PerDevice limit;
  const cudaError_t rc = allow_smem(limit, idkm_codes_prompt<T, HN, SEGS, TMA>, Cfg::SMEM);
  if (rc != cudaSuccess) return rc;
  const long long tiles = (p.rows + 2 * PR_M - 1) / (2 * PR_M) * ((p.tokens + Cfg::N - 1) / Cfg::N), pairs = sms / 2;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  pr_config(cfg, attr, split > 1 || tiles < pairs ? tiles : pairs, split, Cfg::SMEM, st);   // (shared columns: a tile for every cluster)
  return cudaLaunchKernelEx(&cfg, idkm_codes_prompt<T, HN, SEGS, TMA>, p, codes, x, split);
}

template <class T, int HN>
cudaError_t pr_launch(const CodesParams& p, int split, int sms, cudaStream_t st) {
  const int segs = !p.scales || p.group >= 128 ? 1 : (int)(128 / p.group);
  if (p.vec_x) return segs == 1 ? pr_launch<T, HN, 1, true>(p, split, sms, st) : segs == 2 ? pr_launch<T, HN, 2, true>(p, split, sms, st) : pr_launch<T, HN, 4, true>(p, split, sms, st);
  return segs == 1 ? pr_launch<T, HN, 1, false>(p, split, sms, st) : segs == 2 ? pr_launch<T, HN, 2, false>(p, split, sms, st) : pr_launch<T, HN, 4, false>(p, split, sms, st);
}

}  // namespace

PromptPlan codes_prompt_plan(const CodesParams& p, int sms) {
  // rows of X of a tile: those whose waves of tiles cost least.  A chunk of 128 columns took 0.63, 0.66, 0.76 and 0.92 us at HN =
  // 16, 32, 64 and 128 (2048 rows through 8192 x 8192: 1120, 594, 342 and 237 us in all), about 1200 + 5 HN halves of a nanosecond.
  // Where there are few tiles, the pairs of a cluster share a tile's columns; sums that meet cost about 1000 + 20 HN ns a step.
  const long long tiles_w = (p.rows + 2 * PR_M - 1) / (2 * PR_M), pairs = sms / 2, chunks = (p.cols + PR_K - 1) / PR_K;
  PromptPlan plan = {128, 1, INT64_MAX};
  for (int hn = 16; hn <= 128; hn *= 2)
    for (int s = 1, steps = 0; s <= PR_SPLIT; s *= 2, ++steps) {
      const long long tiles = tiles_w * ((p.tokens + 2 * hn - 1) / (2 * hn));
      if (s > 1 && (tiles * s > pairs || chunks < 4 * s || tiles > pr_clusters(s))) break;
      const long long cost = (s > 1 ? 1 : (tiles + pairs - 1) / pairs) * ((chunks + s - 1) / s) * (1200 + 5 * hn) + steps * (2000 + 40 * hn);
      if (cost < plan.ns) plan = {hn, s, cost};
    }
  // (groups of 64 and 32: 17 rows through 4096 x 14336 39 and 52 us, 14 through 535 x 11392 22 and 39)
  const int segments = !p.scales || p.group >= 128 ? 10 : p.group == 64 ? 14 : 18;
  plan.ns = plan.ns / 20 * segments;
  return plan;
}

cudaError_t codes_prompt(const CodesParams& p, int type, const PromptPlan& plan, int sms, cudaStream_t st) {
  if (!pr_encode()) return cudaErrorNotSupported;
  auto run = [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return plan.hn == 16 ? pr_launch<T, 16>(p, plan.split, sms, st) : plan.hn == 32 ? pr_launch<T, 32>(p, plan.split, sms, st) : plan.hn == 64 ? pr_launch<T, 64>(p, plan.split, sms, st) : pr_launch<T, 128>(p, plan.split, sms, st);
  };
  return type == ELEM_BF16 ? run((__nv_bfloat16*)nullptr) : run((__half*)nullptr);
}

}  // namespace idkm
