// Products with 4-bit weights and group scales: Y[m][n] = sum_k s[n][k / g] C[code[n][k]] X[m][k], for few rows of X.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <atomic>
#include <type_traits>
#include "idkm_per_device.h"
#include "idkm_codes.cuh"
#include "../../include/idkm.h"

namespace {

using namespace idkm;

constexpr int ROWS_BLOCK = 256, ROWS_WARPS = ROWS_BLOCK / 32;
constexpr int ROWS_LANE = 8;   // consecutive weights of a lane: one word of codes
constexpr int ROWS_OF = 4;     // rows of W of a warp

// Full precision.  A warp takes four rows of W and TOK rows of X, so that what it loads of
// X serves four rows; every lane looks eight weights of each row up and adds their products, the group's scale multiplies the
// sum of the eight.  `split` warps of a block share the columns of the same rows, where there are few rows; their sums meet in shared
// memory in the order of the warps.
// What bounds it: a warp has few turns, each with loads, 32 lookups and 32 TOK multiply-adds behind one another; 5 rows through 4096 x
// 4608 take 18 us (a row of W a warp, columns not shared: 33), 5.2 T multiply-adds a second of 37.
template <int TOK>
__global__ void __launch_bounds__(ROWS_BLOCK) idkm_codes_rows(const __grid_constant__ CodesParams p, int split) {
  __shared__ float lut[16];
  __shared__ float part[ROWS_WARPS][ROWS_OF * TOK];
  if (threadIdx.x < 16) lut[threadIdx.x] = threadIdx.x < p.k ? reinterpret_cast<const float*>(p.C)[threadIdx.x] : 0.f;
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp % split, sets = ROWS_WARPS / split;
  const long long m0 = (long long)blockIdx.y * TOK;
  const float* X = reinterpret_cast<const float*>(p.X) + m0 * p.ldx;
  const int n_tok = (int)min((long long)TOK, p.tokens - m0);
  const long long quads = (p.rows + ROWS_OF - 1) / ROWS_OF;
  for (long long first = (long long)blockIdx.x * sets; first < quads; first += (long long)gridDim.x * sets) {
    const long long n0 = (first + warp / split) * ROWS_OF;
    float acc[ROWS_OF][TOK];
#pragma unroll
    for (int r = 0; r < ROWS_OF; ++r)
#pragma unroll
      for (int m = 0; m < TOK; ++m) acc[r][m] = 0.f;
    if (n0 < p.rows) {
      const int rows = (int)min((long long)ROWS_OF, p.rows - n0);
      const unsigned char* codes = p.codes + n0 * p.pitch;
      const float* scales = p.scales ? reinterpret_cast<const float*>(p.scales) + n0 * p.n_groups : nullptr;
      const int cols = (int)p.cols, group = (int)p.group, on = split * 32 * ROWS_LANE;
      unsigned word[ROWS_OF], next[ROWS_OF];
      const unsigned char* row_at[ROWS_OF];
#pragma unroll
      for (int r = 0; r < ROWS_OF; ++r) row_at[r] = codes + (r < rows ? r : 0) * p.pitch;
      auto fetch = [&](unsigned (&to)[ROWS_OF], int c) {   // (rows past the last one: the first's)
#pragma unroll
        for (int r = 0; r < ROWS_OF; ++r) {
          to[r] = 0u;
          if (c < cols) to[r] = __ldg(reinterpret_cast<const unsigned*>(row_at[r] + c / 2));
        }
      };
      int c = (mine * 32 + lane) * ROWS_LANE;
      fetch(word, c);
      for (; c < cols; c += on) {
        fetch(next, c + on);
        const bool whole = p.vec_x && c + ROWS_LANE <= cols;
        // X is asked for before anything is looked at; rows past the last one count for nothing
        float xs[TOK][ROWS_LANE];
        if (whole) {
          float4 v[TOK][ROWS_LANE / 4];
          const float* x = X + c;
#pragma unroll
          for (int m = 0; m < TOK; ++m) {
#pragma unroll
            for (int q = 0; q < ROWS_LANE / 4; ++q) v[m][q] = __ldg(reinterpret_cast<const float4*>(x) + q);
            if (m + 1 < n_tok) x += p.ldx;   // (rows past the last one: the last)
          }
#pragma unroll
          for (int m = 0; m < TOK; ++m)
#pragma unroll
            for (int q = 0; q < ROWS_LANE / 4; ++q) {
              xs[m][4 * q] = v[m][q].x;
              xs[m][4 * q + 1] = v[m][q].y;
              xs[m][4 * q + 2] = v[m][q].z;
              xs[m][4 * q + 3] = v[m][q].w;
            }
        } else {
#pragma unroll
          for (int m = 0; m < TOK; ++m)
#pragma unroll
            for (int e = 0; e < ROWS_LANE; ++e) xs[m][e] = c + e < cols ? X[(m < n_tok ? m : 0) * p.ldx + c + e] : 0.f;
        }
        const int g = scales ? c / group : 0;
        float s[ROWS_OF];
#pragma unroll
        for (int r = 0; r < ROWS_OF; ++r) s[r] = scales ? scales[(r < rows ? r : 0) * p.n_groups + g] : 1.f;
#pragma unroll
        for (int r = 0; r < ROWS_OF; ++r) {
          float w[ROWS_LANE];
#pragma unroll
          for (int e = 0; e < ROWS_LANE; ++e) w[e] = lut[word[r] >> (4 * e) & 15u];
#pragma unroll
          for (int m = 0; m < TOK; ++m) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < ROWS_LANE; ++e) sum = fmaf(w[e], xs[m][e], sum);
            acc[r][m] = fmaf(s[r], sum, acc[r][m]);
          }
          word[r] = next[r];
        }
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS_OF; ++r)
#pragma unroll
      for (int m = 0; m < TOK; ++m) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc[r][m] += __shfl_xor_sync(0xffffffffu, acc[r][m], o);
        if (lane == 0) part[warp][r * TOK + m] = acc[r][m];
      }
    __syncthreads();
    for (int i = threadIdx.x; i < sets * ROWS_OF * TOK; i += ROWS_BLOCK) {
      const int set = i / (ROWS_OF * TOK), o = i % (ROWS_OF * TOK);
      const long long n = (first + set) * ROWS_OF + o / TOK;
      float v = 0.f;
      for (int q = 0; q < split; ++q) v += part[set * split + q][o];
      if (n < p.rows && o % TOK < n_tok) reinterpret_cast<float*>(p.Y)[(m0 + o % TOK) * p.ldy + n] = v;
    }
    __syncthreads();
  }
}

// ---- a few rows of X in 16-bit types ------------------------------------------------------------------------------------
// A pair of codes, one byte, is looked up in a table of the 256 pairs of codebook entries, and the pairs are the operands of matrix
// products over 16 rows of W: no conversion, no multiplication of single weights, and the sums of all columns in fp32.
//
// Which column of X a product's k-th place holds is free as long as both operands agree, so a thread takes 32 neighbouring codes
// of two rows as they lie in memory (16 bytes each): the four threads that share a row cover 128 columns, a "strip".  The table
// has a copy for every lane (a word of each of the 32 banks), so that 32 lanes look 32 different pairs up in one cycle: 64
// weights a cycle of a multiprocessor at most, 9 TB/s of codes, above what memory delivers.  Its rows are 256 bytes apart and it lies on a
// multiple of 64 KB, so that an address is four bytes put together by one instruction: two of the table's, the pair, the lane's.
// (Rows of 128 bytes, a shift and a mask a pair, took 11 % longer.)
// What bounds it: one row through 28672 x 8192 takes 36.3 us, 3.3 TB/s, 22 weights a cycle; a loop of lookups and products alone reaches
// 56.  Nothing is saturated (shared memory 64 % of the active cycles, issue slots 54 %, DRAM 40 %): four warps a scheduler wait for
// their own chains, 7.9 cycles an instruction (1.7 of fixed latency, 1.5 for a place in shared memory's queue, 0.9 for its answers, 0.4
// for codes), and the tiles, dealt whole, are 13 a block where 12.1 would be even.
//
// The scale multiplies the group's fp32 sum.  Where a strip has Q = 2 or 4 groups, the threads of a row exchange words first (a
// transposition by shuffles), so that all four work on one group at a time.
//
// Where X does not fit into shared memory, its columns are taken slab by slab: the block goes through a round of its tiles with each
// and keeps their sums, in fp32, until the last (through 8192 x 28672 bf16: 1, 4, 8 rows 43, 60, 77 us; by the lanes of full precision 90,
// 138, 297).
//
// One block a multiprocessor takes its share of the tiles of 16 rows, a batch of tiles at a time.  The batch's chunks of two strips,
// one after another, go to its 16 warps in turn, so that the block reads pieces of rows that lie together.  A warp of its own has
// them copied into shared memory, 16 chunks a stage, two or three stages ahead (loads into registers two steps ahead were
// waited for wherever the loop branches: 41 to 52 us).  The warps' sums of a batch meet in shared memory (in the halves of the table's
// rows that are free) in a fixed order, its scales come while the batch before is worked on, X lies there in the order the
// threads read it.
constexpr int FEW_WARPS = 16, FEW_BLOCK = 32 * FEW_WARPS, FEW_ROWS = 16, FEW_TOKENS = 16;
constexpr int FEW_ASK = 4;   // words of X that a thread has under way at the start
constexpr int FEW_STRIPS = 2, FEW_CHUNK = 128 * FEW_STRIPS;
constexpr int FEW_PITCH = FEW_WARPS * (FEW_CHUNK / 2) + 64, FEW_STAGE = FEW_ROWS * FEW_PITCH;   // (two rows' 64 bytes in different banks)
constexpr int FEW_TABLE = 64 * 1024, FEW_SMEM = 227 * 1024 - 256, FEW_TILES = 8;   // tiles of a batch, at most (the first batch's scales are waited for)
constexpr int FEW_SLAB = 255;          // chunks of a slab, at most
constexpr int FEW_KEPT = 16 * 1024;    // bytes of the sums that are kept from slab to slab, at most
constexpr int FEW_BEFORE = FEW_TABLE - 1024, FEW_AFTER = FEW_SMEM - FEW_BEFORE - FEW_TABLE;     // shared memory starts at 1 KB

__device__ __forceinline__ void few_mma(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1, __nv_bfloat16*) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void few_mma(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1, __half*) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Words w[q] of threads t = 0..3 of a quad: Q = 4: thread t gets word t of thread q's; Q = 2: of the threads with q / 2 = t / 2 words
// 2 (t % 2) and 2 (t % 2) + 1 -- so that w[q] of the whole quad belongs to group q Q / 4 of the chunk.
template <int Q>
__device__ __forceinline__ void few_exchange(uint4& w, int tig) {
  if constexpr (Q >= 2) {   // halves between threads t and t ^ 2
    const bool up = tig & 2;
    const unsigned a = __shfl_xor_sync(0xffffffffu, up ? w.x : w.z, 2), b = __shfl_xor_sync(0xffffffffu, up ? w.y : w.w, 2);
    if (up) { w.x = a; w.y = b; }
    else { w.z = a; w.w = b; }
  }
  if constexpr (Q == 4) {   // words between threads t and t ^ 1
    const bool up = tig & 1;
    const unsigned a = __shfl_xor_sync(0xffffffffu, up ? w.x : w.y, 1), b = __shfl_xor_sync(0xffffffffu, up ? w.z : w.w, 1);
    if (up) { w.x = a; w.z = b; }
    else { w.y = a; w.w = b; }
  }
}
// The columns, by eights within a chunk, that w[q] of thread t then stands for.
template <int Q>
__host__ __device__ __forceinline__ constexpr int few_column(int q, int t) {
  // word j of thread s stands for eight 4 s + j
  return Q == 1 ? 4 * t + q : Q == 2 ? 4 * ((q & 2) + (t & 1)) + (t & 2) + (q & 1) : 4 * q + t;
}

// How a product is taken: tiles of a batch, stages of codes, words of a row's scales in shared memory (odd: a bank a row), bytes of
// a row of X there (two rows' 64 bytes in different banks).
struct FewPlan {
  int slab, tiles, stages, scale_words, xs;   // chunks of a slab, all but the last one's
  int round;                     // tiles of a round, whose sums are kept from slab to slab; all of a block's where there is one slab
  int per_block, extra;          // tiles of every block, blocks that have one more
  int words;            // that a row's scales of a slab may touch
  unsigned scale_inv;   // i * scale_inv >> 32 is i over those
  unsigned x_words;     // i * x_words >> 32 is i over the 16-byte words of a row of X
  int per;              // strips of a group, where groups have whole strips
  unsigned per_group;   // strip * per_group >> 20 is the group of a strip (strips below 2^10, a group's below 2^9; for longer ones 0)
  __host__ __device__ int scale_bytes() const { return 2 * tiles * FEW_ROWS * scale_words * 4; }   // of two batches
  int kept;                      // bytes of the sums that are kept
  int awaited;                   // bytes that every copy is waited for beyond its own: 0 (16 in a test of waits that run out)
};

// The i-th 16 of the sums that meet, in the free halves of the table's rows.
__device__ __forceinline__ float* few_sums(unsigned char* table, int i) { return reinterpret_cast<float*>(table + (i >> 1) * 256 + 128 + (i & 1) * 64); }

// PARTS: the columns come in more than one slab (the loops below are one turn each otherwise).
template <class T, int Q, int NT, bool SCALED, bool PARTS>
__global__ void __launch_bounds__(FEW_BLOCK + 32, 1) idkm_codes_few(const __grid_constant__ CodesParams p, const __grid_constant__ FewPlan f) {
  T* const type = nullptr;
  extern __shared__ __align__(16) unsigned char few_raw[];
  __shared__ __align__(8) unsigned long long s_bar[2][4];   // a stage's codes are there; all warps have read them
  const unsigned raw = (unsigned)__cvta_generic_to_shared(few_raw), table = (raw + FEW_TABLE - 1) & ~(unsigned)(FEW_TABLE - 1);
  const unsigned stage0 = table + FEW_TABLE, full = (unsigned)__cvta_generic_to_shared(s_bar), empty = full + 32;
  unsigned char* const at_table = few_raw + (table - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const int all_chunks = (int)((p.cols + FEW_CHUNK - 1) / FEW_CHUNK), tokens = (int)p.tokens;
  const T* const X = reinterpret_cast<const T*>(p.X);
  const int slab = PARTS ? f.slab : all_chunks;
  const int front = f.scale_bytes() + (PARTS ? f.kept : 0);
  const int before = min(((int)(table - raw) - front) / f.xs, tokens);   // rows of X that lie before the table
  auto row_of = [&](int m) { return m < before ? few_raw + front + m * f.xs : at_table + FEW_TABLE + f.stages * FEW_STAGE + (m - before) * f.xs; };
  const int code_bytes = (int)((p.cols + 31) / 32) * 16;
  const int n_groups = (int)p.n_groups;
  const int tile0 = (int)blockIdx.x * f.per_block + min((int)blockIdx.x, f.extra), tile1 = tile0 + f.per_block + ((int)blockIdx.x < f.extra ? 1 : 0);

  if (warp == FEW_WARPS) {   // the copies: a lane a row
    if (lane < 2 * f.stages)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"((lane & 1 ? empty : full) + 8 * (lane >> 1)), "r"(lane & 1 ? FEW_WARPS : FEW_ROWS) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    asm volatile("bar.arrive 2, %0;" ::"n"(FEW_BLOCK + 32) : "memory");   // (the barriers are ready)
    if (lane < FEW_ROWS) {
      int stage = 0, turn = 0;
      bool filled = false, ok = true;   // every stage has been filled once; no wait has run out
      for (int round = tile0; round < tile1 && ok; round += f.round) {
        const int end = PARTS ? min(round + f.round, tile1) : tile1;
        for (int chunk0 = 0; chunk0 < all_chunks && ok; chunk0 += slab) {
          const int chunks = PARTS ? min(slab, all_chunks - chunk0) : all_chunks;
          for (int batch = round; batch < end && ok; batch += f.tiles) {
            const int steps = min(f.tiles, end - batch) * chunks;
            int tile = batch, chunk = 0;
            for (int s = 0; s < steps; s += FEW_WARPS) {
              const unsigned bar = full + 8 * stage;
              if (filled && !(ok = code_wait(empty + 8 * stage, (turn & 1) ^ 1))) break;
              unsigned to = stage0 + stage * FEW_STAGE + lane * FEW_PITCH;
              for (int left = min(FEW_WARPS, steps - s); left > 0;) {
                const int n = min(left, chunks - chunk);
                const long long row = (long long)tile * FEW_ROWS + lane;
                const int at = (chunk0 + chunk) * (FEW_CHUNK / 2), bytes = min(n * (FEW_CHUNK / 2), code_bytes - at);
                if (row < p.rows) {   // (what is not copied is what was there: codes of rows or columns past the last count for nothing)
                  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes + f.awaited) : "memory");
                  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                               ::"r"(to), "l"(p.codes + row * p.pitch + at), "r"(bytes), "r"(bar) : "memory");
                }
                to += n * (FEW_CHUNK / 2);
                left -= n;
                chunk += n;
                if (chunk == chunks) {
                  chunk = 0;
                  ++tile;
                }
              }
              code_arrive(bar);
              if (++stage == f.stages) {
                stage = 0;
                turn ^= 1;
                filled = true;
              }
            }
          }
          if (!PARTS) break;
        }
        if (!PARTS) break;
      }
      // (no copy is under way when the block ends, also where the others gave up waiting for one)
      for (int i = 0; i < f.stages; ++i) code_wait(full + 8 * i, i < stage ? turn : turn ^ 1);
    }
    return;
  }

  // scales of a batch, by words; a row's may begin in the middle of one.  (A word that holds one byte of them lies in their pages.)
  auto copy_scales = [&](int batch, int end, int g0, int n, int turn) {   // groups g0 to g0 + n
    const long long r0 = (long long)batch * FEW_ROWS;
    const int rows = (int)min((long long)(min(batch + f.tiles, end) - batch) * FEW_ROWS, p.rows - r0);
    const unsigned to = raw + (unsigned)(turn * (f.scale_bytes() / 2));
    const uintptr_t from = (uintptr_t)p.scales + 2 * (r0 * p.n_groups + g0);
    for (int i = tid; i < rows * f.words; i += FEW_BLOCK) {
      const int r = (int)__umulhi((unsigned)i, f.scale_inv), w = i - r * f.words;
      const uintptr_t at = from + 2 * (unsigned)(r * n_groups), word = (at & ~(uintptr_t)3) + 4 * w;
      if (word < at + 2 * n) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + (unsigned)(r * f.scale_words + w) * 4u), "l"(word) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // The codebook, and X by 16-byte words, whatever its rows' alignment: the one or two words of memory that hold eight elements (one
  // that holds a byte of the row lies in its pages).  All that a thread loads it asks for before it looks at the first.
  const unsigned short* c = reinterpret_cast<const unsigned short*>(p.C);
  unsigned lo = 0u, hi = 0u;
  if (tid < 256) {
    if ((tid & 15) < p.k) lo = __ldg(c + (tid & 15));
    if ((tid >> 4) < p.k) hi = __ldg(c + (tid >> 4));
  }
  const int words = slab * (FEW_CHUNK / 8), n_words = tokens * words;
  auto column_of = [&](int v) { return (v >> 4) * 128 + 8 * few_column<Q>((v >> 2) & 3, v & 3); };   // place 4 q + t of a strip: for word q of thread t
  auto ask = [&](int i, int col0, uint4& a, uint4& b) {
    const int m = (int)__umulhi((unsigned)i, f.x_words), k = column_of(i - m * words);   // (columns in bytes pass 32 bits)
    const uintptr_t row = (uintptr_t)(X + m * p.ldx), at = row + 2ll * col0 + 2 * k, end = row + 2 * p.cols;
    const uintptr_t word = at & ~(uintptr_t)15;
    const int first = i < n_words && at < end, second = first && (at & 15) && word + 16 < end;
    code_ask(a, b, word, first, second);
  };
  auto place = [&](int i, int col0, const uint4& a, const uint4& b) {
    if (i >= n_words) return;
    const int m = (int)__umulhi((unsigned)i, f.x_words), v = i - m * words;
    const unsigned off = (unsigned)((uintptr_t)(X + m * p.ldx) & 15u);   // (columns by eights: the row's)
    *reinterpret_cast<uint4*>(row_of(m) + v * 16) = code_align8(a, b, off, (int)p.cols - col0 - column_of(v));
  };
  auto load_slab = [&](int col0, auto meanwhile) {
    uint4 a[FEW_ASK], b[FEW_ASK];
#pragma unroll
    for (int u = 0; u < FEW_ASK; ++u) ask(tid + u * FEW_BLOCK, col0, a[u], b[u]);
    meanwhile();
    for (int i0 = tid;;) {
#pragma unroll
      for (int u = 0; u < FEW_ASK; ++u) place(i0 + u * FEW_BLOCK, col0, a[u], b[u]);
      i0 += FEW_ASK * FEW_BLOCK;
      if (i0 >= n_words) break;
#pragma unroll
      for (int u = 0; u < FEW_ASK; ++u) ask(i0 + u * FEW_BLOCK, col0, a[u], b[u]);
    }
  };
  auto meet = [] { asm volatile("bar.sync 1, %0;" ::"n"(FEW_BLOCK) : "memory"); };

  // (a value that is there after the barrier only: the lookups, which may be moved about, stay behind it)
  unsigned mine;
  asm volatile("or.b32 %0, %1, %2;" : "=r"(mine) : "r"(table), "r"((unsigned)lane * 4u) : "memory");
  // this thread's row of X; threads of columns that X has no row for keep their zeros
  const unsigned char* x_row[NT];
  bool x_there[NT];
  uint4 x[2][NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    x_there[n] = n * 8 + gid < tokens;
    x_row[n] = row_of(min(n * 8 + gid, tokens - 1)) + tig * 16;
    x[0][n] = x[1][n] = make_uint4(0u, 0u, 0u, 0u);
  }
  const unsigned my_codes = stage0 + gid * FEW_PITCH + warp * (FEW_CHUNK / 2) + tig * 16;
  int stage = 0, stage_turn = 0, turn = 0;
  bool lost = false;   // a wait ran out (none does: the copies wait for nothing but these warps); later ones do not wait, nothing is handed back
  float tot[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) tot[n][i] = 0.f;
  bool first = true;
  for (int round = tile0; round < tile1; round += f.round) {
    const int end = PARTS ? min(round + f.round, tile1) : tile1;
    for (int chunk0 = 0; chunk0 < all_chunks; chunk0 += slab) {
      const int chunks = PARTS ? min(slab, all_chunks - chunk0) : all_chunks, parts = min(chunks, FEW_WARPS), batch_sums = f.tiles * parts * tokens;
      // the slab's groups; where they have whole strips, the first of its strips is the phase-th of one
      const int strip0 = chunk0 * FEW_STRIPS;
      int g0 = 0, n_slab = n_groups, phase = 0;
      if (PARTS) {
        g0 = Q > 1 ? strip0 * Q : strip0 / f.per;
        phase = Q > 1 ? 0 : strip0 - g0 * f.per;
        n_slab = min(n_groups - g0, Q > 1 ? chunks * FEW_STRIPS * Q : (phase + chunks * FEW_STRIPS - 1) / f.per + 1);
      }
      auto first_scale = [&](int strip) {
        if (Q > 1) return strip * Q;
        strip += phase;
        return (int)((unsigned)strip * f.per_group >> 20) + (PARTS && f.per_group == 0 && strip >= f.per);
      };
      {
        load_slab(chunk0 * FEW_CHUNK, [&] {   // (the first batch's scales come meanwhile)
          if (SCALED) copy_scales(round, end, g0, n_slab, turn);
        });
        if ((!PARTS || first) && tid < 256) {
          const unsigned both = lo | hi << 16;
#pragma unroll
          for (int q = 0; q < 8; ++q)   // (lanes at different places of their rows: in different banks)
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(table + tid * 256 + ((q + lane) & 7) * 16), "r"(both) : "memory");
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (!PARTS || first) asm volatile("bar.sync 2, %0;" ::"n"(FEW_BLOCK + 32) : "memory");
        else meet();
        first = false;
      }
      for (int batch = round; batch < end; batch += f.tiles, turn ^= 1) {
        if (SCALED) copy_scales(batch + f.tiles, end, g0, n_slab, turn ^ 1);
        const int n_batch = min(f.tiles, end - batch), steps = n_batch * chunks;
        int tile = warp / chunks, chunk = warp % chunks;   // of the batch
        for (int s = 0; s < steps; s += FEW_WARPS) {
          if (!lost) lost = !code_wait(full + 8 * stage, stage_turn);
          uint4 w[FEW_STRIPS][2];
#pragma unroll
          for (int u = 0; u < FEW_STRIPS; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[u][h].x), "=r"(w[u][h].y), "=r"(w[u][h].z), "=r"(w[u][h].w)
                           : "r"(my_codes + stage * FEW_STAGE + h * 8 * FEW_PITCH + u * 64));
          if (s + warp < steps) {
            float acc[NT][4];
            if (SCALED) {
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
            }
            const int x_at = chunk * (2 * FEW_CHUNK);
            unsigned scale_of[2];   // the scales of this thread's rows
            if (SCALED) {
              const int r = tile * FEW_ROWS + gid;
              const unsigned odd = ((unsigned)((uintptr_t)p.scales >> 1) + ((unsigned)r & (unsigned)n_groups) + (unsigned)g0) & 1u;   // (16 and 8 rows on: the same)
              scale_of[0] = raw + (unsigned)(turn * (f.scale_bytes() / 2) + r * f.scale_words * 4) + 2 * odd;
              scale_of[1] = scale_of[0] + 8 * f.scale_words * 4;
            }
#pragma unroll
            for (int u = 0; u < FEW_STRIPS; ++u) {
#pragma unroll
              for (int h = 0; h < 2; ++h) few_exchange<Q>(w[u][h], tig);
#pragma unroll
              for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
                  if (x_there[n]) x[q & 1][n] = *reinterpret_cast<const uint4*>(x_row[n] + x_at + u * 256 + q * 64);
                const unsigned w0 = q == 0 ? w[u][0].x : q == 1 ? w[u][0].y : q == 2 ? w[u][0].z : w[u][0].w;
                const unsigned w1 = q == 0 ? w[u][1].x : q == 1 ? w[u][1].y : q == 2 ? w[u][1].z : w[u][1].w;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  unsigned a[4];
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    // (the lane's byte, byte 2 j + i / 2 of the codes, the table's two)
                    const unsigned at = __byte_perm(mine, i & 1 ? w1 : w0, 0x3240u + 0x10u * (unsigned)(2 * j + i / 2));
                    asm("ld.shared.u32 %0, [%1];" : "=r"(a[i]) : "r"(at));
                  }
#pragma unroll
                  for (int n = 0; n < NT; ++n) few_mma(SCALED ? acc[n] : tot[n], a, j ? x[q & 1][n].z : x[q & 1][n].x, j ? x[q & 1][n].w : x[q & 1][n].y, type);
                }
                if (SCALED && (q + 1) % (4 / Q) == 0) {   // a group, or a strip, is done
                  const int g = first_scale(chunk * FEW_STRIPS + u) + (Q > 1 ? q * Q / 4 : 0);
                  float sc[2];
#pragma unroll
                  for (int h = 0; h < 2; ++h) {   // (past the last group only where the codes are past the last column too)
                    unsigned short v = 0;
                    if (g < n_slab) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(scale_of[h] + 2 * g));
                    sc[h] = code_scale(v, type);
                  }
#pragma unroll
                  for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                      tot[n][i] = fmaf(sc[i / 2], acc[n][i], tot[n][i]);
                      acc[n][i] = 0.f;
                    }
                }
              }
            }
            const int here = tile, part = chunks < FEW_WARPS ? chunk : warp;
            chunk += FEW_WARPS;
            while (chunk >= chunks) {
              chunk -= chunks;
              ++tile;
            }
            if (tile != here) {   // the warp's part of the tile is done
              if (lost) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                  for (int i = 0; i < 4; ++i) tot[n][i] = __int_as_float(0x7fc00000);
              }
              const int base = turn * batch_sums + (here * parts + part) * tokens + 2 * tig;
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                if (n * 8 + 2 * tig < tokens) {
                  float* to = few_sums(at_table, base + n * 8) + gid;
                  to[0] = tot[n][0];
                  to[8] = tot[n][2];
                }
                if (n * 8 + 2 * tig + 1 < tokens) {
                  float* to = few_sums(at_table, base + n * 8 + 1) + gid;
                  to[0] = tot[n][1];
                  to[8] = tot[n][3];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) tot[n][i] = 0.f;
              }
            }
          }
          // (the codes have been used, so they have been read)
          __syncwarp();
          if (lane == 0 && !lost) code_arrive(empty + 8 * stage);   // (a stage whose codes may be still to come is not filled again)
          if (++stage == f.stages) {
            stage = 0;
            stage_turn ^= 1;
          }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        meet();   // the batch is done, the next one's scales are there
        const int n = n_batch * FEW_ROWS;
        for (int o = tid; o < n * tokens; o += FEW_BLOCK) {
          const int m = o / n, r = o - m * n;
          const int base = turn * batch_sums + (r / FEW_ROWS) * parts * tokens + m;
          float v = 0.f;
          for (int i = 0; i < parts; ++i) v += few_sums(at_table, base + i * tokens)[r % FEW_ROWS];
          float* const kept = reinterpret_cast<float*>(few_raw + f.scale_bytes()) + (batch - round) * FEW_ROWS * tokens + o;   // (this thread's alone)
          if (PARTS && chunk0 > 0) v = *kept + v;
          const long long row = (long long)batch * FEW_ROWS + r;
          if (PARTS && chunk0 + chunks < all_chunks) *kept = v;
          else if (row < p.rows) reinterpret_cast<T*>(p.Y)[m * p.ldy + row] = from_f32<T>(v);
        }
      }
      if (!PARTS) break;
    }
    if (!PARTS) break;
  }
}

// The plan of a product: X of a slab and two batches' scales in shared memory before the table and after it, the stages after it, the
// batches' sums in the table's free halves.  One slab where all of X fits, with three stages or two; otherwise as few as there can be.
inline FewPlan few_plan(const CodesParams& p, int tiles_of_block) {
  FewPlan f = {};
  const int tokens = (int)p.tokens, chunks = (int)((p.cols + FEW_CHUNK - 1) / FEW_CHUNK);
  if (p.group >= 128) {
    f.per = (int)(p.group / 128);
    f.per_group = f.per >= 512 ? 0u : (unsigned)(((1 << 20) + f.per - 1) / f.per);
  }
  for (int slabs = (chunks + FEW_SLAB - 1) / FEW_SLAB;; ++slabs) {
    f.slab = (chunks + slabs - 1) / slabs;
    f.xs = f.slab * (2 * FEW_CHUNK) + 64;
    f.x_words = (unsigned)((0x100000000ull + f.slab * (FEW_CHUNK / 8) - 1) / (f.slab * (FEW_CHUNK / 8)));
    long long groups = p.n_groups;   // that a slab touches at most
    if (slabs > 1) groups = p.group < 128 ? f.slab * (FEW_CHUNK / p.group) : (f.slab * FEW_STRIPS - 1) / f.per + 2;
    if (groups > p.n_groups) groups = p.n_groups;
    f.words = groups > 1 ? (int)(groups / 2 + 1) : 2;
    f.scale_inv = (unsigned)((0x100000000ull + f.words - 1) / f.words);
    f.scale_words = p.scales ? (int)(groups / 2 + 1) | 1 : 0;
    const int parts = f.slab < FEW_WARPS ? f.slab : FEW_WARPS;
    for (f.stages = 3; f.stages >= 2; --f.stages)
      for (f.tiles = FEW_TILES; f.tiles >= 1; f.tiles /= 2) {
        if (2 * f.tiles * parts * FEW_ROWS * tokens * 4 > FEW_TABLE / 2) continue;
        f.round = tiles_of_block;
        f.kept = 0;
        if (slabs > 1) {
          const int most = FEW_KEPT / (FEW_ROWS * tokens * 4) / f.tiles * f.tiles;
          if (most < f.round) f.round = most;
          f.kept = f.round * FEW_ROWS * tokens * 4;
        }
        const int left = FEW_BEFORE - 1024 - f.scale_bytes() - f.kept;   // (shared memory starts at up to 2 KB)
        const int after = FEW_AFTER - f.stages * FEW_STAGE;
        if (left >= 0 && after >= 0 && left / f.xs + after / f.xs >= tokens) return f;
      }
  }
}

template <class T, int Q, int NT, bool SCALED, bool PARTS>
cudaError_t few_launch(const CodesParams& p, const FewPlan& f, int blocks, cudaStream_t st) {
  static PerDevice limit;
  const cudaError_t rc = allow_smem(limit, idkm_codes_few<T, Q, NT, SCALED, PARTS>, FEW_SMEM);
  if (rc != cudaSuccess) return rc;
  idkm_codes_few<T, Q, NT, SCALED, PARTS><<<blocks, FEW_BLOCK + 32, FEW_SMEM, st>>>(p, f);
  return cudaGetLastError();
}

template <class T, int Q, bool SCALED>
cudaError_t few_launch(const CodesParams& p, int sms, cudaStream_t st) {
  const int tiles = (int)((p.rows + FEW_ROWS - 1) / FEW_ROWS), blocks = tiles < sms ? tiles : sms;
  FewPlan f = few_plan(p, (tiles + blocks - 1) / blocks);
  f.awaited = p.missing < 0 ? 0 : 16;
  f.per_block = tiles / blocks;
  f.extra = tiles % blocks;
  const bool parts = f.kept > 0;
  if (p.tokens > 8) {
    // X in parts is slow for so many rows (the parts are short, a batch is a tile): about 350 ns a tile of rows and a chunk.  The tensor cores
    // of pairs of blocks take less for large W: 16 rows through 8192 x 28672, groups of 128, 143 us and 71; 9 through 4096 x 14336, groups of
    // 64, 33 and 52; 14 through 535 x 11392, groups of 32, 28 and 39.
    if (parts) {
      const PromptPlan plan = codes_prompt_plan(p, sms);
      if (plan.ns < 350ll * ((tiles + blocks - 1) / blocks) * ((p.cols + FEW_CHUNK - 1) / FEW_CHUNK))
        return codes_prompt(p, std::is_same<T, __half>::value ? ELEM_F16 : ELEM_BF16, plan, sms, st);
      return few_launch<T, Q, 2, SCALED, true>(p, f, blocks, st);
    }
    return few_launch<T, Q, 2, SCALED, false>(p, f, blocks, st);
  }
  return parts ? few_launch<T, Q, 1, SCALED, true>(p, f, blocks, st) : few_launch<T, Q, 1, SCALED, false>(p, f, blocks, st);
}

template <class T>
cudaError_t few_launch(const CodesParams& p, int sms, cudaStream_t st) {
  return !p.scales ? few_launch<T, 1, false>(p, sms, st) : p.group == 32 ? few_launch<T, 4, true>(p, sms, st)
         : p.group == 64 ? few_launch<T, 2, true>(p, sms, st) : few_launch<T, 1, true>(p, sms, st);
}

cudaError_t rows_launch(const CodesParams& p, int sms, cudaStream_t st) {
  const int TOK = p.tokens < 8 ? (int)p.tokens : 8;
  const long long tiles = (p.tokens + TOK - 1) / TOK, quads = (p.rows + ROWS_OF - 1) / ROWS_OF;
  // warps that share rows: until 16 a multiprocessor have work, as long as each has 256 columns
  int split = 1;
  while (split < ROWS_WARPS && quads * (tiles < 65535 ? tiles : 65535) * split < (long long)sms * 16 && p.cols > 256ll * split) split *= 2;
  const long long blocks = (quads + ROWS_WARPS / split - 1) / (ROWS_WARPS / split);
  for (long long at = 0; at < tiles; at += 65535) {   // (a grid's second dimension)
    CodesParams q = p;
    q.X = reinterpret_cast<const float*>(p.X) + at * TOK * p.ldx;
    q.Y = reinterpret_cast<float*>(p.Y) + at * TOK * p.ldy;
    q.tokens = p.tokens - at * TOK;
    const dim3 grid((unsigned)(blocks < (long long)sms * 8 ? blocks : (long long)sms * 8), (unsigned)(tiles - at < 65535 ? tiles - at : 65535));
    switch (TOK) {
      case 1: idkm_codes_rows<1><<<grid, ROWS_BLOCK, 0, st>>>(q, split); break;
      case 2: idkm_codes_rows<2><<<grid, ROWS_BLOCK, 0, st>>>(q, split); break;
      case 3: idkm_codes_rows<3><<<grid, ROWS_BLOCK, 0, st>>>(q, split); break;
      case 4: idkm_codes_rows<4><<<grid, ROWS_BLOCK, 0, st>>>(q, split); break;
      case 5: idkm_codes_rows<5><<<grid, ROWS_BLOCK, 0, st>>>(q, split); break;
      case 6: idkm_codes_rows<6><<<grid, ROWS_BLOCK, 0, st>>>(q, split); break;
      case 7: idkm_codes_rows<7><<<grid, ROWS_BLOCK, 0, st>>>(q, split); break;
      default: idkm_codes_rows<8><<<grid, ROWS_BLOCK, 0, st>>>(q, split); break;
    }
    const cudaError_t rc = cudaGetLastError();
    if (rc != cudaSuccess) return rc;
  }
  return cudaSuccess;
}

std::atomic<int> hook_missing_copy{0};   // idkm_set_codes_test_hooks; 0 at rest

}  // namespace

extern "C" int idkm_set_codes_test_hooks(int missing_copy) {
  if (missing_copy < 0 || missing_copy > (1 << 24)) return IDKM_ERR_PARAM;
  hook_missing_copy.store(missing_copy, std::memory_order_relaxed);
  return IDKM_OK;
}

extern "C" int idkm_matmul_codes(const void* X, int type, int64_t tokens, int64_t ldx, const unsigned char* codes, int64_t rows, int64_t cols,
                                 int64_t pitch, const void* C, int k, const void* scales, int64_t group, void* Y, int64_t ldy,
                                 void* cuda_stream) {
  if (!X || !codes || !C || !Y) return IDKM_ERR_NULL;
  if (k < 1 || k > 16 || !elem_known(type)) return IDKM_ERR_UNSUPPORTED;
  constexpr int64_t most = INT32_MAX - 4096;   // (indexes of a row, and of a step past the last)
  if (tokens < 1 || rows < 1 || cols < 1 || ldx < cols || ldy < rows || pitch < (cols + 31) / 32 * 16 || (scales && group < 1) ||
      cols > (INT64_C(1) << 50) / rows || rows > most || cols > most || tokens > most)
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
  p.missing = hook_missing_copy.load(std::memory_order_relaxed) - 1;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (type == ELEM_F32) return rows_launch(p, sms, st) == cudaSuccess ? IDKM_OK : IDKM_ERR_CUDA;
  const bool few = tokens <= FEW_TOKENS;
  const cudaError_t rc = !few ? codes_prompt(p, type, codes_prompt_plan(p, sms), sms, st) : type == ELEM_BF16 ? few_launch<__nv_bfloat16>(p, sms, st) : few_launch<__half>(p, sms, st);
  return rc == cudaSuccess ? IDKM_OK : IDKM_ERR_CUDA;
}
