// Linear layers in 8-bit integers: out[m, n] = sx[m] sw[n] sum_k xq[m, k] q[n, k], with a scale a token (sx = max |x| / 127, xq = x / sx
// rounded to the nearest integer) and a scale an output channel.  Products and sums are exact in int32; out is made of the sum and the two scales in fp32.
//
// The weights are the A operand of tcgen05.mma (kind::i8, 128 channels an instruction) and the tokens the B operand (16 to 256 of them),
// so that few tokens waste no rows of an instruction: a decode step reads the weights once at HBM's rate, a prompt keeps the tensor cores busy.  Both
// operands lie in memory as the instruction wants them in shared memory: atoms of 8 rows x 128 bytes in the 128-byte swizzle (16-byte chunk c
// of row r at chunk c ^ (r & 7)), padded with zeros to whole atoms.  So a stage of the ring is two plain bulk copies, of one run of memory each,
// with no tensor map and no edge cases:
//   weights  [N / 128 tiles][K / 128 blocks][128 rows x 128 bytes], laid out once;  scales [N]
//   tokens   [K / 128 blocks][M / 8 groups][8 rows x 128 bytes], written by the quantisation;  scales [M]
// A CTA (one an SM): warp 0 copies, warp 1 issues the instructions into one of two accumulators in tensor memory, warps 2 to 9 scale and
// store the other one.  Four forms, by what bounds the call (plan_for), and a kernel of its own for one token of a small layer
// (i8_one_token_kernel):
//   kShare    few tiles: the CTAs of a cluster share a tile's K and add their integers through distributed shared memory (any order gives
//             the same bits)
//   kRowsEven up to 128 tokens, many channels: the weights' bytes decide.  Every CTA takes the same number of channels, in groups of 8 wherever they
//             lie (an atom is one run of memory), for all tokens; whole tiles dealt to 148 SMs leave some with one more than the others.
//             (151,936 x 2048, 48 tokens to fp32: 60.5 us, 5.6 TB/s; 75 with whole tiles)
//   kTiles    tiles of 128 channels and up to 256 tokens one after the other
//   kPairs    many tiles: two CTAs share a tile of 256 channels and up to 256 tokens (cta_group::2), each fetching its channels and half of the tokens:
//             a third less to fetch, and six stages where four fit (4096 tokens, 16,384 x 4096, bf16: 191 us with the quantisation, 2.9 POP/s; 204
//             as kTiles)
#include <cuda.h>

#include "jp_common.cuh"
#include "jp_internal.h"

namespace jp {
namespace {

constexpr int kRows = 128;                    // channels of a tile
constexpr int kBlock = 128;                   // k of a stage: one row of the swizzle
constexpr int kTileBytes = kRows * kBlock;
constexpr int kResultWarps = 8;               // two for each quarter of tensor memory's lanes, half of the tokens each
constexpr int kThreads = 64 + 32 * kResultWarps;
constexpr int kMaxStages = 12;
constexpr int kRingBytes = 200 * 1024;
constexpr long long kSpin = 4000000000ll;     // clock cycles after which a wait gives up

struct Control {                              // behind the ring in shared memory
  unsigned long long full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
  float sx[kResultWarps][256];
  uint32_t tmem;
  int abort;
};
constexpr int kSharedBytes = 1024 + kRingBytes + (int)sizeof(Control);
static_assert(kSharedBytes <= 232448, "beyond the 227 KB a CTA can have");

__device__ __forceinline__ uint32_t s32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(unsigned long long* b, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(s32(b)), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(unsigned long long* b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(s32(b)) : "memory"); }
__device__ __forceinline__ void bar_expect(unsigned long long* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(s32(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(unsigned long long* b, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 1000;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(s32(b)), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __noinline__ bool bar_wait(unsigned long long* b, uint32_t parity, volatile int* abort) {      // false: gave up, or another role did
  long long t0 = 0;
  for (uint32_t i = 0;; ++i) {
    if (bar_try(b, parity)) return true;
    if ((i & 63u) == 0u) {
      if (*abort) return false;
      const long long now = clock64();
      if (i == 0u) t0 = now;
      else if (now - t0 > kSpin) { *abort = 1; return false; }
    }
  }
}
__device__ __forceinline__ void copy(void* to, const void* from, uint32_t bytes, unsigned long long* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(s32(to)), "l"(from), "r"(bytes), "r"(s32(bar)) : "memory");
}
// Shared-memory descriptor of a K-major operand in the 128-byte swizzle: address / 16, 1024 bytes between groups of 8 rows, version 1.
__device__ __forceinline__ uint64_t operand(uint32_t address) {
  return (uint64_t)((address & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(s32(bar)) : "memory");
}
// The same for a pair of CTAs: copies that are counted on the even CTA's barrier (bit 24 of a shared::cluster address is the CTA's rank), instructions
// over both CTAs' shared and tensor memory, and arrivals on the same barrier of both.
__device__ __forceinline__ void copy_pair(uint32_t to, const CUtensorMap* map, int row, unsigned long long* bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map), "r"(0), "r"(row),
               "r"(s32(bar) & 0xFEFFFFFFu) : "memory");
}
__device__ __forceinline__ void mma_i8_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit_pair(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(s32(bar)), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void arrive_even(unsigned long long* bar) {
  asm volatile("{\n\t.reg .b32 ra;\n\tmapa.shared::cluster.u32 ra, %0, 0;\n\tmbarrier.arrive.shared::cluster.b64 _, [ra];\n\t}" ::"r"(s32(bar)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory"); }
// 16 columns of a warp's lanes: the load, and the wait for loads before their registers are used
__device__ __forceinline__ void tmem_ld16(uint32_t addr, int (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                 "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr) : "memory");
}
__device__ __forceinline__ int tmem_ld1(uint32_t addr) {      // one column, waited for
  int v;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void tmem_wait(int (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) asm volatile("" : "+r"(r[i]));
}

template <bool BF16> __device__ __forceinline__ void put(void* out, int64_t i, float v) {
  if constexpr (BF16) ((__nv_bfloat16*)out)[i] = __float2bfloat16_rn(v);
  else ((float*)out)[i] = v;
}

// r sx sw: by the product of the scales, where that is a normal number (or one of them is 0, infinite or NaN, and so the result what it has to be); where
// it is not, the result may be all the same, and is made in 64 bits.
// least_sx, most_sx: the smallest and the largest of the tokens' scales, those that are 0, infinite or NaN left out
__device__ __forceinline__ bool product_is_normal(float least_sx, float most_sx, float sw) {
  const float a = fabsf(sw), inf = __int_as_float(0x7f800000);
  return a == 0.f || !(a < inf) || (a * least_sx >= 0x1p-126f && a * most_sx < inf);
}
__device__ __forceinline__ bool counts_as_scale(float sx) { return sx > 0.f && sx < __int_as_float(0x7f800000); }
__device__ __noinline__ float scaled(int r, float sx, float sw) {
  return !counts_as_scale(sx) || product_is_normal(sx, sx, sw) ? (float)r * (sx * sw) : (float)((double)r * ((double)sx * (double)sw));
}

enum Form { kShare, kRowsEven, kTiles, kPairs };

// (Compiled as if for 448 threads, so that one takes 128 registers: a block then starts, and fetches weights, beside the quantisation's last ones.  With
// 147 of them 300 tokens of 4096 x 4096 take 18.9 us instead of 18.3.  Not the pairs, which have many more tokens to quantise: 4096 x 4096 x 16,384 190.4
// us with 128 registers for 188 before, 194.5 with 149 for 193 on another GPU.)
template <bool BF16, int FORM>
__global__ void __launch_bounds__(FORM == kPairs ? kThreads : 448, 1) i8_linear_kernel(I8Args A, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x) {
  constexpr bool SPLIT = FORM == kShare, PAIR = FORM == kPairs;
  extern __shared__ unsigned char raw[];
  unsigned char* const ring = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  Control& sm = *(Control*)(ring + kRingBytes);
  uint32_t rank = 0;
  if (SPLIT || PAIR) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int TN = A.tokens_tile, stages = A.stages, ranks = SPLIT ? A.split : PAIR ? 2 : 1;
  const uint32_t stage_bytes = kTileBytes + (uint32_t)(PAIR ? TN / 2 : TN) * kBlock;
  const int k0 = SPLIT ? (int)(A.kblocks * rank / ranks) : 0, k1 = SPLIT ? (int)(A.kblocks * (rank + 1) / ranks) : (int)A.kblocks;
  // tiles of this CTA: first, first + step .. below end (kShare: one), and the channels of them that are its own
  int64_t first = blockIdx.x / ranks, step = gridDim.x / ranks, end = A.tiles, row0 = 0, row1 = A.N;
  if (FORM == kRowsEven) {
    const int64_t groups = (A.N + 7) / 8;
    row0 = groups * blockIdx.x / gridDim.x * 8;
    row1 = groups * (blockIdx.x + 1) / gridDim.x * 8;
    first = row0 / kRows;
    step = 1;
    end = (row1 + kRows - 1) / kRows;
  }

  if (tid == 0) {
    for (int s = 0; s < stages; ++s) { bar_init(&sm.full[s], 1); bar_init(&sm.empty[s], 1); }
    for (int b = 0; b < 2; ++b) { bar_init(&sm.acc_full[b], 1); bar_init(&sm.acc_empty[b], PAIR ? 2 * kResultWarps : kResultWarps); }
    sm.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(s32(&sm.tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(s32(&sm.tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
  }
  __syncthreads();
  if (PAIR) cluster_sync();                    // the partner's barriers exist before anything is sent to them
  fence_after();
  const uint32_t tmem = *(volatile uint32_t*)&sm.tmem;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  if (warp == 0) {
    // ---- copies of the next stage of both operands, tile after tile
    if (PAIR) {
      if (lane == 0) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        uint32_t n = 0, s = 0, use = 0;
        bool ok = true;
        for (int64_t tile = first; tile < end && ok; tile += step) {
          // (channels behind the last tile and tokens behind the last group read zeros, or tokens that are not stored)
          const int w_row = (int)((tile / A.tiles_m * 2 + rank) * A.kblocks * kRows), x_row = (int)(tile % A.tiles_m * TN + rank * (TN / 2));
          for (int kb = 0; kb < (int)A.kblocks; ++kb, ++n) {
            if (!bar_wait(&sm.empty[s], (use & 1u) ^ 1u, &sm.abort)) { ok = false; break; }
            if (rank == 0) bar_expect(&sm.full[s], 2u * stage_bytes);
            copy_pair(s32(ring) + s * stage_bytes, &map_w, w_row + kb * kRows, &sm.full[s]);
            copy_pair(s32(ring) + s * stage_bytes + kTileBytes, &map_x, x_row + kb * (int)A.padded_m, &sm.full[s]);
            if (++s == (uint32_t)stages) s = 0, ++use;
          }
        }
        if (!ok) {                             // as below; the even CTA's barriers count both CTAs' copies
          if (A.status) atomicExch(A.status, (int)JP_ERR_TIMEOUT);
          for (uint32_t i = n < (uint32_t)stages ? 0 : n - stages; rank == 0 && i < n; ++i) {
            const long long t0 = clock64();
            while (!bar_try(&sm.full[i % stages], (i / stages) & 1u))
              if (clock64() - t0 > kSpin) break;
          }
        }
      }
    } else if (lane == 0) {
      // The weights do not depend on the quantisation in front of this kernel: with A.early their first stages are fetched before it is done.
      uint32_t armed = 0;
      bool ok = true, waited = false;
      // what the copies of a tile's stages have in common
      const uint8_t* weights = nullptr;
      const uint8_t* xq = nullptr;
      uint32_t w_bytes = 0, w_at = 0, x_bytes = 0;
      const int64_t x_step = A.padded_m / 8 * 1024;
      auto enter = [&](int64_t tile) {
        const int64_t m0 = tile % A.tiles_m * TN, rows = A.padded_m - m0 < TN ? A.padded_m - m0 : TN, n = tile / A.tiles_m;
        uint32_t from = 0, to = kRows;         // channels of the tile
        if (FORM == kRowsEven) {
          from = n * kRows < row0 ? (uint32_t)(row0 - n * kRows) : 0u;
          to = (n + 1) * kRows > row1 ? (uint32_t)(row1 - n * kRows) : (uint32_t)kRows;
        }
        w_at = from * kBlock;
        w_bytes = (to - from) * kBlock;
        x_bytes = (uint32_t)rows * kBlock;
        weights = A.weights + (n * A.kblocks + k0) * kTileBytes + w_at;
        xq = A.xq + k0 * x_step + m0 / 8 * 1024;
      };
      auto arm = [&](int kb, uint32_t s) {
        bar_expect(&sm.full[s], w_bytes + x_bytes);
        copy(ring + s * stage_bytes + w_at, weights + (int64_t)(kb - k0) * kTileBytes, w_bytes, &sm.full[s]);
      };
      auto tokens = [&](int kb, uint32_t s) { copy(ring + s * stage_bytes + kTileBytes, xq + (kb - k0) * x_step, x_bytes, &sm.full[s]); };
      if (A.early && first < end) {
        const int n = k1 - k0 < stages ? k1 - k0 : stages;
        enter(first);
        for (int i = 0; i < n; ++i) arm(k0 + i, i);
        asm volatile("griddepcontrol.wait;" ::: "memory");
        waited = true;
        for (int i = 0; i < n; ++i) tokens(k0 + i, i);
        armed = n;
      }
      if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
      uint32_t n = 0, s = 0, use = 0;          // stages passed; the place of the next one, and how often it was used
      for (int64_t tile = first; tile < end && ok; tile += step) {
        enter(tile);
        for (int kb = k0; kb < k1; ++kb, ++n) {
          if (n >= armed) {
            if (!bar_wait(&sm.empty[s], (use & 1u) ^ 1u, &sm.abort)) { ok = false; break; }
            arm(kb, s);
            tokens(kb, s);
          }
          if (++s == (uint32_t)stages) s = 0, ++use;
        }
      }
      if (!ok) {                               // leave no copy in flight: wait (bounded) for the last one of every stage
        if (A.status) atomicExch(A.status, (int)JP_ERR_TIMEOUT);
        for (uint32_t i = n < (uint32_t)stages ? 0 : n - stages; i < n; ++i) {
          const long long t0 = clock64();
          while (!bar_try(&sm.full[i % stages], (i / stages) & 1u))
            if (clock64() - t0 > kSpin) break;
        }
      }
    }
  } else if (warp == 1) {
    // ---- instructions: 32 k each, four a stage
    if (lane == 0 && (!PAIR || rank == 0)) {
      // int32 accumulator, signed 8-bit operands, both K-major, TN columns, 128 rows (256 of a pair)
      const uint32_t shape = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TN >> 3) << 17) | ((uint32_t)((PAIR ? 2 * kRows : kRows) >> 4) << 24);
      uint32_t s = 0, phase = 0;
      bool ok = true;
      int t = 0;
      for (int64_t tile = first; tile < end && ok; tile += step, ++t) {
        const uint32_t buf = t & 1, use = t >> 1;
        if (!bar_wait(&sm.acc_empty[buf], (use & 1u) ^ 1u, &sm.abort)) { ok = false; break; }
        fence_after();
        for (int kb = k0; kb < k1; ++kb) {
          if (!bar_wait(&sm.full[s], phase, &sm.abort)) { ok = false; break; }
          fence_after();
          const uint32_t at = s32(ring) + s * stage_bytes;
          const uint64_t a = operand(at), b = operand(at + kTileBytes);
#pragma unroll
          for (int q = 0; q < kBlock / 32; ++q) {    // 32 bytes further inside the swizzled row: start address + 2
            if (PAIR) mma_i8_pair(tmem + buf * 256, a + q * 2, b + q * 2, shape, kb != k0 || q != 0);
            else mma_i8(tmem + buf * 256, a + q * 2, b + q * 2, shape, kb != k0 || q != 0);
          }
          if (PAIR) commit_pair(&sm.empty[s]);
          else commit(&sm.empty[s]);
          if (++s == (uint32_t)stages) s = 0, phase ^= 1u;
        }
        if (ok) {
          if (PAIR) commit_pair(&sm.acc_full[buf]);
          else commit(&sm.acc_full[buf]);
        }
      }
      if (!ok && A.status) atomicExch(A.status, (int)JP_ERR_TIMEOUT);
    }
  } else {
    // ---- results: a thread has one channel, columns are tokens
    const int q = warp & 3, w = warp - 2;      // the quarter of tensor memory's lanes this warp may read
    const int row = q * 32 + lane;
    constexpr int ES = BF16 ? 2 : 4;
    // pairs of channels in one word, where words are aligned: two lanes swap halves of two tokens, and each stores one of them
    const bool words = BF16 && ((uintptr_t)A.out & 3) == 0 && A.ld_out % 2 == 0 && A.N % 2 == 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int t = 0;
    for (int64_t tile = first; tile < end; tile += step, ++t) {
      const uint32_t buf = t & 1, use = t >> 1;
      const int64_t m0 = tile % A.tiles_m * TN, n = (PAIR ? tile / A.tiles_m * 2 + rank : tile / A.tiles_m) * kRows + row;
      const int cols = (int)(A.M - m0 < TN ? A.M - m0 : TN), half = (cols + 31) / 32 * 16, c_first = w < 4 ? 0 : half, c_end = w < 4 ? (half < cols ? half : cols) : cols;
      const bool mine = FORM == kRowsEven ? n >= row0 && n < row1 && n < A.N : n < A.N;
      const float sw = mine ? A.weight_scales[n] : 0.f;
      bool normal = true;                      // of all products of these scales (one answer a warp: a test an element costs a sixth of a prompt's time)
      if (!SPLIT) {
        uint32_t least = 0x7f800000u, most = 0u;
        __syncwarp();
        for (int c = c_first + lane; c < c_end; c += 32) {
          const float sx = __ldcg(A.token_scales + m0 + c);
          sm.sx[w][c] = sx;
          if (counts_as_scale(sx)) least = min(least, __float_as_uint(sx)), most = max(most, __float_as_uint(sx));
        }
        least = __reduce_min_sync(0xffffffffu, least);
        most = __reduce_max_sync(0xffffffffu, most);
        normal = __all_sync(0xffffffffu, product_is_normal(__uint_as_float(least), __uint_as_float(most), sw));
      }
      if (!bar_wait(&sm.acc_full[buf], use & 1u, &sm.abort)) {
        if (lane == 0 && A.status) atomicExch(A.status, (int)JP_ERR_TIMEOUT);
        break;
      }
      fence_after();
      const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + buf * 256;
      char* out = (char*)A.out + ((m0 + c_first) * A.ld_out + n) * ES;
      const int64_t ld = A.ld_out * ES;
      for (int c = c_first; !normal && c < c_end; ++c) {
        const float v = scaled(tmem_ld1(from + c), sm.sx[w][c], sw);
        if (mine) put<BF16>(out, 0, v);
        out += ld;
      }
      int r[2][16];
      if (normal && c_first < c_end) tmem_ld16(from + c_first, r[0]);
#pragma unroll 1
      for (int c0 = c_first; normal && c0 < c_end; c0 += 32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {          // (the next 16 columns are under way while these are stored)
          const int c = c0 + 16 * h;
          if (c >= c_end) break;
          tmem_wait(r[h]);
          if (c + 16 < c_end) tmem_ld16(from + c + 16, r[h ^ 1]);
          if (SPLIT) {                         // (the ring is free: all of its stages have been read)
#pragma unroll
            for (int j = 0; j < 16; ++j) ((int*)ring)[(c + j) * kRows + row] = r[h][j];
          } else if (words) {
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
              const float a = (float)r[h][j] * (sm.sx[w][c + j] * sw), b = (float)r[h][j + 1] * (sm.sx[w][c + j + 1] * sw);
              const float other = __shfl_xor_sync(0xffffffffu, (lane & 1) ? a : b, 1);
              const __nv_bfloat162 v = (lane & 1) ? __floats2bfloat162_rn(other, b) : __floats2bfloat162_rn(a, other);
              if (mine && c + j + (lane & 1) < c_end) *(uint32_t*)(out + ((lane & 1) ? ld - 2 : 0)) = *(const uint32_t*)&v;
              out += 2 * ld;
            }
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              if (mine && c + j < c_end) put<BF16>(out, 0, (float)r[h][j] * (sm.sx[w][c + j] * sw));
              out += ld;
            }
          }
        }
      }
      fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) arrive_even(&sm.acc_empty[buf]);
        else bar_arrive(&sm.acc_empty[buf]);
      }
    }
  }
  if (SPLIT) {                                 // the ranks' sums of every rank-th token
    __syncwarp();
    cluster_sync();
    const int64_t tile = first;
    if (warp >= 2 && !*(volatile int*)&sm.abort) {
      const int row = (warp & 3) * 32 + lane;
      const int64_t m0 = tile % A.tiles_m * TN, n = tile / A.tiles_m * kRows + row;
      const int cols = (int)(A.M - m0 < TN ? A.M - m0 : TN);
      if (n < A.N) {
        const float sw = A.weight_scales[n];
        const auto sum_of = [&](int c) {
          int sum = 0;
          for (int r = 0; r < ranks; ++r) {
            uint32_t from;
            int v;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(s32((int*)ring + c * kRows + row)), "r"(r));
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
            sum += v;
          }
          return sum;
        };
        bool normal = true;
        for (int c = rank * 2 + (warp - 2) / 4; c < cols; c += ranks * 2) {
          const int sum = sum_of(c);
          const float sx = __ldcg(A.token_scales + m0 + c), p = sx * sw;
          normal &= (fabsf(p) >= 0x1p-126f && fabsf(p) < __int_as_float(0x7f800000)) || sx == 0.f;
          put<BF16>(A.out, (m0 + c) * A.ld_out + n, (float)sum * p);
        }
        if (!normal)                           // once more, rather than a branch at each element
          for (int c = rank * 2 + (warp - 2) / 4; c < cols; c += ranks * 2) put<BF16>(A.out, (m0 + c) * A.ld_out + n, scaled(sum_of(c), __ldcg(A.token_scales + m0 + c), sw));
      }
    }
    __syncwarp();
    cluster_sync();                            // nobody leaves while its sums are read
  }
  fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();                    // neither CTA leaves while the other may still use its memory
  if (warp == 1 && PAIR) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  } else if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// ---- layouts ------------------------------------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(256) i8_pack_kernel(I8PackArgs A) {
  const int64_t chunks = A.tiles_n * A.kblocks * (kTileBytes / 16);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
    const int row = (int)(i / 8 % kRows), at = (int)(i % 8);
    const int64_t kb = i / (kTileBytes / 16) % A.kblocks, n = i / (kTileBytes / 16) / A.kblocks * kRows + row;
    const int64_t k0 = kb * kBlock + (at ^ (row & 7)) * 16;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (n < A.N)
      for (int e = 0; e < 16; ++e)
        if (k0 + e < A.K) w[e / 4] |= (uint32_t)(uint8_t)A.q[n * A.ld_q + k0 + e] << (8 * (e & 3));
    ((uint4*)A.packed)[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  float* scales = (float*)((char*)A.packed + A.tiles_n * A.kblocks * kTileBytes);
  for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < A.tiles_n * kRows; n += (int64_t)gridDim.x * 256) scales[n] = n < A.N ? A.scales[n] : 0.f;
}

// Quantisation of a token's row: q = 127 x / max |x| rounded to the nearest integer, halves to the even one, as exact arithmetic has it.  x
// and the maximum have 8 significant bits, so 127 x and (2 q + 1) max / 2 are exact in fp32, and 127 x / max is either a half or at least 1/512 (of numbers up
// to 254) away from one: the product with a rounded reciprocal (off by 2^-15 at most) picks the right integer, or one of the two of a
// half, and the remainder of the product tells a half.  max is scaled to 1 .. 2 first, by a power of two, so that nothing overflows or leaves the normal numbers.
constexpr int kQuantThreads = 256;

struct Chunk { uint4 a, b; };                  // 16 bf16
__device__ __forceinline__ Chunk load_chunk(const I8QuantArgs& A, const char* row, int64_t k0) {
  Chunk c{make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
  if (A.vectors && k0 + 16 <= A.K) {
    c.a = ((const uint4*)(row + k0 * 2))[0];
    c.b = ((const uint4*)(row + k0 * 2))[1];
  } else if (k0 < A.K) {
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t lo = k0 + 2 * e < A.K ? ((const uint16_t*)row)[k0 + 2 * e] : 0u, hi = k0 + 2 * e + 1 < A.K ? ((const uint16_t*)row)[k0 + 2 * e + 1] : 0u;
      w[e] = lo | hi << 16;
    }
    c.a = make_uint4(w[0], w[1], w[2], w[3]);
    c.b = make_uint4(w[4], w[5], w[6], w[7]);
  }
  return c;
}
__device__ __forceinline__ uint32_t word_of(const Chunk& c, int i) {
  return i == 0 ? c.a.x : i == 1 ? c.a.y : i == 2 ? c.a.z : i == 3 ? c.a.w : i == 4 ? c.b.x : i == 5 ? c.b.y : i == 6 ? c.b.z : c.b.w;
}
// The largest magnitude, as the bits of a bf16: ordered like integers, infinity and NaN above all numbers.
__device__ __forceinline__ uint32_t largest(const Chunk& c, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = __vmaxu2(m, word_of(c, i) & 0x7fff7fffu);
  return m;
}
__device__ __forceinline__ int quantized(float x, float scale, float m, float inv) {
  const float xs = x * scale, x127 = xs * 127.f;
  const float n = rintf(x127 * inv);
  const float rest = fmaf(-n, m, x127);        // exact wherever it matters
  int q = (int)n;
  if (fabsf(rest) * 2.f == m && (q & 1)) q += rest > 0.f ? 1 : -1;
  return q;
}
__device__ __forceinline__ uint4 quantized_chunk(const Chunk& c, float scale, float m, float inv) {
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[i] = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t w = word_of(c, (4 * i + e) / 2);
      o[i] |= ((uint32_t)quantized(__uint_as_float((e & 1) ? w & 0xffff0000u : w << 16), scale, m, inv) & 0xffu) << (8 * e);
    }
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// What a token's largest magnitude (the bits of a bf16) makes of it.
struct TokenScale {
  float most, scale, scaled, inv;
  bool usable;
  __device__ __forceinline__ explicit TokenScale(uint32_t top) {
    most = __uint_as_float(top << 16);
    // a power of two that takes the largest magnitude to 1 .. 2 (subnormal ones come out below 1, still with all of their bits)
    const uint32_t exponent = top >> 7;
    scale = exponent == 0u ? __uint_as_float(253u << 23) : exponent == 254u ? __uint_as_float(1u << 22) : __uint_as_float((254u - exponent) << 23);
    scaled = most * scale;
    inv = scaled > 0.f ? 1.f / scaled : 0.f;
    usable = exponent < 255u;                  // else a NaN or an infinity: the token's outputs are NaN
  }
  __device__ __forceinline__ float step() const { return usable ? most / 127.f : __uint_as_float(0x7fc00000u); }
};

// kHeld: chunks of 16 a thread keeps between the maximum and the rounding; a row's others are read again.  (One, for rows of up to 4096, leaves
// room for eight blocks an SM: 4096 x 4096 25 us with four.)
template <int kHeld> __global__ void __launch_bounds__(kQuantThreads, kHeld == 1 ? 8 : 3) i8_quantize_kernel(I8QuantArgs A) {
  __shared__ uint32_t sh[kQuantThreads / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t m = blockIdx.x, chunks = A.kblocks * (kBlock / 16);
  const char* row = (const char*)A.x + m * A.ld_x * 2;
  Chunk held[kHeld];
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int64_t c = (int64_t)i * blockDim.x + threadIdx.x;
    held[i] = load_chunk(A, row, c < chunks ? c * 16 : A.K);
    top = largest(held[i], top);
  }
  for (int64_t c = (int64_t)kHeld * blockDim.x + threadIdx.x; c < chunks; c += blockDim.x) top = largest(load_chunk(A, row, c * 16), top);
  top = (top & 0xffffu) > top >> 16 ? top & 0xffffu : top >> 16;
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = top;
  __syncthreads();
  for (int w = 0; w < (int)blockDim.x / 32; ++w) top = sh[w] > top ? sh[w] : top;
  const TokenScale t(top);
  const float scale = t.scale, scaled = t.scaled, inv = t.inv;
  const bool usable = t.usable;
  char* out = (char*)A.tokens + (m / 8) * 1024 + (m & 7) * 128;
  auto place = [&](int64_t c) { return (uint4*)(out + c / 8 * (A.padded_m / 8) * 1024 + (((int)(c & 7) ^ (int)(m & 7)) * 16)); };
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int64_t c = (int64_t)i * blockDim.x + threadIdx.x;
    if (c < chunks) *place(c) = usable ? quantized_chunk(held[i], scale, scaled, inv) : none;
  }
  for (int64_t c = (int64_t)kHeld * blockDim.x + threadIdx.x; c < chunks; c += blockDim.x)
    *place(c) = usable ? quantized_chunk(load_chunk(A, row, c * 16), scale, scaled, inv) : none;
  if (threadIdx.x == 0)
    ((float*)((char*)A.tokens + A.padded_m * A.kblocks * kBlock))[m] = t.step();
}

// One token of a small layer, in one launch: a CTA quantises the token by itself into shared memory (it is short, so that this costs less than a
// kernel in front) and takes 8 channels, its warps a part of K each; four products an instruction (dp4a), as a tensor-core tile would be 1/128 full.
// Latency bounds such a call.
constexpr int kOneBatch = 4;                   // 1 KB lines of weights a warp has on the way at once
constexpr int64_t kOneK = 16384, kOneWeights = 48 << 20;
template <bool BF16> __global__ void __launch_bounds__(256) i8_one_token_kernel(I8QuantArgs X, I8Args A) {
  extern __shared__ uint4 xs[];                // [K / 16]
  __shared__ uint32_t top;
  __shared__ int sums[8][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, kblocks = (int)A.kblocks, chunks = kblocks * (kBlock / 16);
  if (threadIdx.x == 0) top = 0u;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __syncthreads();
  const int64_t group = blockIdx.x;            // of 8 channels: 1024 contiguous bytes of a block of K
  const uint4* const w = (const uint4*)(A.weights + group / 16 * A.kblocks * kTileBytes + group % 16 * 1024) + lane;
  uint4 held[kOneBatch][2];                    // chunks lane and lane + 32 of the line: channels lane / 8 and 4 + lane / 8
  const auto load = [&](int kb) {
#pragma unroll
    for (int i = 0; i < kOneBatch; ++i) {
      const bool has = kb + 8 * i < kblocks;
      const uint4* const from = w + (int64_t)(kb + 8 * i) * (kTileBytes / 16);
      held[i][0] = has ? __ldg(from) : make_uint4(0u, 0u, 0u, 0u);
      held[i][1] = has ? __ldg(from + 32) : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  load(warp);
  uint32_t t = 0u;
  for (int c = threadIdx.x; c < chunks; c += 256) t = largest(load_chunk(X, (const char*)X.x, c * 16), t);
  t = (t & 0xffffu) > t >> 16 ? t & 0xffffu : t >> 16;
  t = __reduce_max_sync(0xffffffffu, t);
  if (lane == 0) atomicMax(&top, t);           // (integers: any order)
  __syncthreads();
  const TokenScale token(top);
  for (int c = threadIdx.x; c < chunks; c += 256)
    xs[c] = token.usable ? quantized_chunk(load_chunk(X, (const char*)X.x, c * 16), token.scale, token.scaled, token.inv) : make_uint4(0u, 0u, 0u, 0u);
  __syncthreads();
  int acc[2] = {0, 0};
  const int at[2] = {(lane & 7) ^ (lane >> 3), (lane & 7) ^ (4 + (lane >> 3))};          // where in the row's 128 bytes the chunks belong
  for (int kb = warp; kb < kblocks; kb += 8 * kOneBatch) {
    if (kb != warp) load(kb);
#pragma unroll
    for (int i = 0; i < kOneBatch; ++i)
      if (kb + 8 * i < kblocks)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 p = xs[(kb + 8 * i) * 8 + at[h]], q = held[i][h];
          acc[h] = __dp4a((int)q.x, (int)p.x, __dp4a((int)q.y, (int)p.y, __dp4a((int)q.z, (int)p.z, __dp4a((int)q.w, (int)p.w, acc[h]))));
        }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) acc[h] += __shfl_xor_sync(0xffffffffu, acc[h], o);
    if ((lane & 7) == 0) sums[warp][4 * h + (lane >> 3)] = acc[h];
  }
  __syncthreads();
  const int64_t n = group * 8 + threadIdx.x;
  if (threadIdx.x < 8 && n < A.N) {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += sums[i][threadIdx.x];
    const float sx = token.step(), sw = A.weight_scales[n], p = sx * sw;
    put<BF16>(A.out, n, fabsf(p) >= 0x1p-126f && fabsf(p) < __int_as_float(0x7f800000) ? (float)sum * p : scaled(sum, sx, sw));
  }
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Tokens a tile takes and CTAs that share a tile's K.  A tile of c tokens takes about c + 64 (its instructions, and the copy of its channels
// beside them); the least rounds over the SMs times that, of the token counts that share M evenly.
struct Plan { Form form; int tokens, split; int64_t tiles_m; };
Plan plan_for(int64_t M, int64_t N, int64_t kblocks, int sms) {
  const int64_t tiles_n = (N + kRows - 1) / kRows, least = (M + 255) / 256;
  Plan p{};
  p.split = 1;
  if (M <= 128 && tiles_n > sms) {
    p.form = kRowsEven;
    p.tokens = (int)up(M, 16);
    p.tiles_m = 1;
    return p;
  }
  double best = 0;
  for (int64_t tm = least; tm <= least * 3 && tm <= (M + 15) / 16; ++tm) {
    const int64_t c = up((M + tm - 1) / tm, 16), rounds = (tiles_n * tm + sms - 1) / sms;
    const double cost = (double)rounds * (double)(c + 64);
    if (p.tokens == 0 || cost < best) best = cost, p.tokens = (int)c, p.tiles_m = (M + c - 1) / c;
  }
  // pairs of CTAs where they have two rounds of tiles at least
  const int64_t pairs = (tiles_n + 1) / 2 * least;
  if (M > 128 && pairs >= sms && N * kblocks < (int64_t)1 << 30 && up(M, 8) * kblocks < (int64_t)1 << 30) {
    p.form = kPairs;
    p.tokens = (int)up((M + least - 1) / least, 32);
    p.tiles_m = (M + p.tokens - 1) / p.tokens;
    return p;
  }
  const int64_t tiles = tiles_n * p.tiles_m;
  while (p.split < 8 && tiles * p.split * 2 <= sms && kblocks >= p.split * 2) p.split *= 2;
  p.form = p.split > 1 ? kShare : kTiles;
  return p;
}

}  // namespace

size_t i8_packed_bytes(int64_t N, int64_t K) {
  const int64_t tiles = (N + kRows - 1) / kRows;
  return (size_t)(tiles * ((K + kBlock - 1) / kBlock) * kTileBytes + tiles * kRows * 4);
}
size_t i8_token_bytes(int64_t M, int64_t K) { return (size_t)(up(M, 8) * up(K, kBlock) + up(M, 8) * 4); }

cudaError_t launch_i8_pack(I8PackArgs a, cudaStream_t s, int sms) {
  a.tiles_n = (a.N + kRows - 1) / kRows;
  a.kblocks = (a.K + kBlock - 1) / kBlock;
  const int64_t need = (a.tiles_n * a.kblocks * (kTileBytes / 16) + 255) / 256, most = (int64_t)sms * 8;
  i8_pack_kernel<<<(unsigned)(need < most ? need : most), 256, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_i8_quantize(I8QuantArgs a, cudaStream_t s) {
  a.padded_m = up(a.M, 8);
  a.kblocks = (a.K + kBlock - 1) / kBlock;
  a.vectors = ((uintptr_t)a.x & 15) == 0 && a.ld_x % 8 == 0;
  const int64_t threads = up(a.kblocks * (kBlock / 16), 32);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.M);
  cfg.blockDim = dim3((unsigned)(threads < kQuantThreads ? threads : kQuantThreads));
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, threads <= kQuantThreads ? i8_quantize_kernel<1> : i8_quantize_kernel<4>, a);
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
  static EncodeTiled fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found);
    return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? (EncodeTiled)f : nullptr;
  }();
  return fn;
}
// Rows of 128 bytes as they lie (they are swizzled already), fetched `box` at a time; rows behind the last one read zeros.
static bool map_rows(CUtensorMap* map, const void* base, int64_t rows, uint32_t box) {
  const cuuint64_t dims[2] = {(cuuint64_t)kBlock, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)kBlock};
  const cuuint32_t boxes[2] = {(cuuint32_t)kBlock, box}, steps[2] = {1, 1};
  return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BF16, int FORM> static cudaError_t launch_linear(const I8Args& a, cudaStream_t s, int sms) {
  const cudaError_t e = allow_shared_memory<i8_linear_kernel<BF16, FORM>>(kSharedBytes);
  if (e != cudaSuccess) return e;
  CUtensorMap map_w{}, map_x{};
  if (FORM == kPairs) {
    if (!encode_tiled()) return cudaErrorNotSupported;
    const int64_t tiles_n = (a.N + kRows - 1) / kRows;
    if (!map_rows(&map_w, a.weights, tiles_n * a.kblocks * kRows, kRows) || !map_rows(&map_x, a.xq, a.kblocks * a.padded_m, (uint32_t)a.tokens_tile / 2))
      return cudaErrorInvalidValue;
  }
  cudaLaunchConfig_t cfg{};
  const int64_t pairs = a.tiles < sms / 2 ? a.tiles : sms / 2;
  cfg.gridDim = dim3((unsigned)(FORM == kShare ? a.tiles * a.split : FORM == kPairs ? 2 * pairs : FORM == kRowsEven || a.tiles > sms ? sms : a.tiles));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSharedBytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = FORM == kPairs ? 2u : (unsigned)a.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = FORM == kShare || FORM == kPairs ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, i8_linear_kernel<BF16, FORM>, a, map_w, map_x);
}

// Measured in us, one token to bf16, N x K (two launches with the kernels above in brackets): 512 x 512 2.3 (5.0), 2048 x 2048 3.3 (9.9), 9472 x 4096
// 10.8 (13.1), 11,008 x 4096 12.4 (15.4), 2048 x 16,384 12.0 (20.8); more weights or channels: 9472 x 8192 17.8 (18.2), 18,944 x 2048 13.6 (11.7),
// 40,960 x 1024 23.6 (15.9), 151,936 x 2048 90 (56), where every CTA's own quantisation adds up.
bool i8_one_token(int64_t M, int64_t N, int64_t K, int sms) { return M == 1 && K <= kOneK && N <= 80 * (int64_t)sms && N * K <= kOneWeights; }

cudaError_t launch_i8_one_token(I8QuantArgs x, I8Args a, const void* packed, bool out_bf16, cudaStream_t s) {
  a.kblocks = (x.K + kBlock - 1) / kBlock;
  x.vectors = ((uintptr_t)x.x & 15) == 0;
  a.weights = (const uint8_t*)packed;
  a.weight_scales = (const float*)((const char*)packed + (a.N + kRows - 1) / kRows * a.kblocks * kTileBytes);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((a.N + 7) / 8));
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = (size_t)(a.kblocks * kBlock);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return out_bf16 ? cudaLaunchKernelEx(&cfg, i8_one_token_kernel<true>, x, a) : cudaLaunchKernelEx(&cfg, i8_one_token_kernel<false>, x, a);
}

cudaError_t launch_i8_linear(I8Args a, const void* packed, const void* tokens, int64_t K, bool out_bf16, cudaStream_t s, int sms) {
  a.kblocks = (K + kBlock - 1) / kBlock;
  a.padded_m = up(a.M, 8);
  const Plan p = plan_for(a.M, a.N, a.kblocks, sms);
  const int64_t tiles_n = (a.N + kRows - 1) / kRows;
  a.tokens_tile = p.tokens;
  a.tiles_m = p.tiles_m;
  a.tiles = (p.form == kPairs ? (tiles_n + 1) / 2 : tiles_n) * p.tiles_m;
  a.split = p.split;
  const int fit = kRingBytes / (kTileBytes + (p.form == kPairs ? p.tokens / 2 : p.tokens) * kBlock);
  a.stages = fit < kMaxStages ? fit : kMaxStages;
  a.weights = (const uint8_t*)packed;
  a.weight_scales = (const float*)((const char*)packed + tiles_n * a.kblocks * kTileBytes);
  a.xq = (const uint8_t*)tokens;
  a.token_scales = (const float*)((const char*)tokens + a.padded_m * a.kblocks * kBlock);
  if (p.form == kShare) return out_bf16 ? launch_linear<true, kShare>(a, s, sms) : launch_linear<false, kShare>(a, s, sms);
  if (p.form == kRowsEven) return out_bf16 ? launch_linear<true, kRowsEven>(a, s, sms) : launch_linear<false, kRowsEven>(a, s, sms);
  if (p.form == kPairs) return out_bf16 ? launch_linear<true, kPairs>(a, s, sms) : launch_linear<false, kPairs>(a, s, sms);
  return out_bf16 ? launch_linear<true, kTiles>(a, s, sms) : launch_linear<false, kTiles>(a, s, sms);
}

}  // namespace jp
