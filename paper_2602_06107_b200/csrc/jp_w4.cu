// Linear layer with 4-bit weights and group scales for a few tokens:
//   out[m, n] = sum_k x[m, k] (q[n, k] - z[n, k / group]) s[n, k / group]
//
// The weights are read once, half a byte each, and bound the call by HBM: at 6.5 TB/s an SM gets about 46 weights a
// clock.  The products go through mma.sync m16n8k16 with 16 rows of weights as A and 8 tokens as B: q - z is a small
// integer, exact in bf16, so a group's sum is exact products added in fp32, and the group's scale multiplies that
// fp32 sum.  (tcgen05 would need the 16-bit weights written to shared memory or TMEM first, 92 of the 128 bytes a
// clock that shared memory moves, and a TMEM read per group for the scales; with 1 to 32 tokens its rate is of no use.)
//
// Weights are laid out once (pack_kernel) in the order the MMA's A fragments want them: tiles of 16 rows, blocks of 128 columns, per
// block 8 steps of k = 16.  Which of a group's columns make a step is free as long as A and B agree: two steps take 32 columns, lane t of
// a row's four 8 t .. 8 t + 7, so that a lane's x of two steps are 16 bytes of memory.  A lane's 8 weights of a step are one 32-bit word
// whose nibbles j and j + 4 are the two halves of fragment register j: four masks, one shift and four packed multiply-adds (scaled2) make
// the fragment.  A block is 1024 bytes of words, then one 32-bit word per (row, group): the scale as fp32 with its low 4 bits replaced by
// z (scales come in bf16 or fp16: those bits are zero).  Blocks of a tile follow one another, tiles too: what a warp reads is one
// contiguous run of memory, or a few.
//
// Work split: a CTA takes a contiguous run of tiles, and its 16 warps take equal contiguous runs of the CTA's blocks,
// whatever the tile boundaries.  So every size keeps all warps busy to within one block; a tile that two or more warps share is
// summed in shared memory in the warps' order (deterministic).  x is staged in shared memory once per CTA in B-fragment order.
#include <cuda_fp16.h>

#include <atomic>

#include "jp_common.cuh"
#include "jp_internal.h"

namespace jp {
namespace {

constexpr int kTileRows = 16;
constexpr int kBlockK = 128;
constexpr int kWarps = 16;
constexpr int kDepth = 3;
constexpr int kSharedBytes = 232448;  // of one block
// A warp takes a unit at a time and has three of them in flight (four: below, 30.8 and 63.5 us).  A unit is two blocks where there are
// enough (less to do per block around the products): two of one tile, or for many tiles the same block of two tiles, which then share what
// is read of x (weights from HBM at full clocks: 151,936 x 2048 and one token, one block 34.6 us, two of a tile 32.1, of two tiles 30.3; x
// 4096 and eight, 72.2, 65.0, 60.9; at 11008 x 4096 pairs of tiles come out uneven, 10.6 us, two blocks of one tile 9.5).  Above eight
// tokens the products take longer than either saves.
// What the ring and the warps' parts of shared tiles leave is for x.
__host__ __device__ constexpr int block_bytes(int groups) { return 1024 + kTileRows * 4 * groups; }
__host__ __device__ constexpr int part_bytes(int tiles, int nt) { return kWarps * tiles * nt * 32 * 16; }
__host__ __device__ constexpr int ring_bytes(int blocks, int groups) { return kWarps * kDepth * blocks * block_bytes(groups); }
constexpr int x_bytes(int nt, int tiles, int unit, int groups) {
  return kSharedBytes - ring_bytes(tiles * unit, groups) - part_bytes(tiles, nt);
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// d = a b: the first step of a group
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// Bits 0 .. 7 of a bf16 are the number bits 2^-133, over the subnormals and the first normal binade alike.  So a nibble that is
// masked out in place, at bits 0 or 4 of each half, is q 2^-133 or q 2^-129, and one fused multiply-add by 2^127 with -z / 64 or
// -z / 4 makes it (q - z) / 64 or / 4, exactly: no shift, no exponent to set.  (The
// finished sum takes the 64 or the 4 back: a large scale would leave fp32 by it.)
constexpr uint32_t k2To127 = 0x7f007f00u, kMinus2To127 = 0xff00ff00u;
__device__ __forceinline__ uint32_t scaled2(uint32_t bits, uint32_t minus_z) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(bits), "r"(k2To127), "r"(minus_z));
  return d;
}
__device__ __forceinline__ uint32_t minus_scaled2(uint32_t bits) {      // -z / 64 (z at bits 0) or -z / 4 (at bits 4)
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(bits), "r"(kMinus2To127), "r"(0u));
  return d;
}

__device__ __forceinline__ void copy16(void* smem, const void* global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(global) : "memory");
}

template <int NT>
__device__ __forceinline__ void store_tile(const W4Args& A, const float (&acc)[NT][4], int64_t tile, int lane) {
  const int64_t n = tile * kTileRows + (lane >> 2);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t row = n + (e >> 1) * 8;
      const int m = t * 8 + (lane & 3) * 2 + (e & 1);
      if (m < A.M && row < A.N) {
        const float sum = acc[t][e] * (e < 2 ? 64.f : 4.f);
        if (A.out_bf16) ((__nv_bfloat16*)A.out)[m * A.ld_out + row] = __float2bfloat16_rn(sum);
        else ((float*)A.out)[m * A.ld_out + row] = sum;
      }
    }
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 16 bytes at this place in the shared memory of another CTA of the cluster
__device__ __forceinline__ float4 load_cluster(const float4* p, int cta) {
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(cta));
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}

// SPLIT: the CTAs of a cluster share a run of tiles and take a part of the columns each; the tiles' sums stay in shared memory, and
// at the end every CTA adds those of some tiles, in the cluster's order.
template <int NT, int GROUPS, int TILES, int UNIT, bool SPLIT>
__global__ void __launch_bounds__(kWarps * 32, 1) w4_kernel(W4Args A) {
  static_assert(TILES == 1 || UNIT == 1, "a unit is blocks of one tile, or a block of two");
  static_assert(!SPLIT || TILES * UNIT == 1, "units of one block");
  constexpr int kBlock = block_bytes(GROUPS), kBytes = UNIT * TILES * kBlock;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  char* ring = smem + warp * kDepth * kBytes;
  float4* parts = (float4*)(smem + ring_bytes(TILES * UNIT, GROUPS));                 // [warp][TILES][NT][lane]: of a tile that an earlier warp begins
  const int row_blocks = (int)A.kblocks;
  const int64_t runs = TILES == 1 ? A.tiles : (A.tiles + 1) / 2;        // (below, a tile is a pair of them)
  const int ctas = SPLIT ? A.split : 1, rank = SPLIT ? blockIdx.x % ctas : 0;
  const int64_t run = blockIdx.x / ctas, all_runs = gridDim.x / ctas;
  const int64_t tile0 = runs * run / all_runs, tile1 = runs * (run + 1) / all_runs;
  const int kb0 = SPLIT ? row_blocks * rank / ctas : 0, kblocks = SPLIT ? row_blocks * (rank + 1) / ctas - kb0 : row_blocks;       // this CTA's
  float4* sums = (float4*)(smem + ring_bytes(TILES * UNIT, GROUPS) + part_bytes(TILES, NT));     // (SPLIT) [tile][NT][lane]
  uint4* xs = (uint4*)sums + (SPLIT ? (tile1 - tile0) * NT * 32 : 0);        // [block][step pair][token][lane % 4]
  const int tile_units = kblocks / UNIT;
  const int64_t blocks = (tile1 - tile0) * tile_units;      // (units)
  const int64_t b0 = blocks * warp / kWarps, b1 = blocks * (warp + 1) / kWarps;
  const int count = (int)(b1 - b0);
  const char* src;
  int in_kb = 0;                                            // (SPLIT, pairs) block of the next unit to load, and where the second tile's is
  int64_t in_tile = 0, second = 0;
  if constexpr (SPLIT) {
    in_kb = (int)(b0 % kblocks);
    src = (const char*)A.packed + ((tile0 + b0 / kblocks) * row_blocks + kb0 + in_kb) * kBlock + lane * 16;
  } else if constexpr (TILES == 1) {
    src = (const char*)A.packed + (tile0 * tile_units + b0) * kBytes + lane * 16;
  } else {
    in_tile = tile0 + b0 / tile_units;
    in_kb = (int)(b0 % tile_units);
    src = (const char*)A.packed + (in_tile * 2 * kblocks + in_kb) * kBlock + lane * 16;
    second = 2 * in_tile + 1 < A.tiles ? (int64_t)kblocks * kBlock : 0;        // (the last pair may have one tile: its rows come twice)
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");                // launched as a programmatic dependent of whatever is before it
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int issued = 0, slot_in = 0, slot_out = 0;
  auto fetch = [&]() {
    if (issued < count) {
      if constexpr (TILES == 1) {
#pragma unroll
        for (int c = 0; c < kBytes; c += 512)
          if (c + 512 <= kBytes || lane * 16 < kBytes - c) copy16(ring + slot_in + c + lane * 16, src + c);
        src += kBytes;
        if (SPLIT && ++in_kb == kblocks) {
          in_kb = 0;
          src += (int64_t)(row_blocks - kblocks) * kBlock;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int c = 0; c < kBlock; c += 512)
            if (c + 512 <= kBlock || lane * 16 < kBlock - c)
              copy16(ring + slot_in + j * kBlock + c + lane * 16, src + (j ? second : 0) + c);
        src += kBlock;
        if (++in_kb == kblocks) {
          in_kb = 0;
          src += (int64_t)kblocks * kBlock;
          second = 2 * ++in_tile + 1 < A.tiles ? (int64_t)kblocks * kBlock : 0;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ++issued;
    slot_in = slot_in == (kDepth - 1) * kBytes ? 0 : slot_in + kBytes;
  };
  fetch();
  fetch();
  // x in B-fragment order: unit (block, step pair, token, t) of 16 bytes is columns 128 block + 32 pair + 8 t and the next seven.
  // Asynchronous copies and little code: in the smallest calls fetching instructions is part of the time (the loops unrolled by eight
  // cost 4 us).
  const uintptr_t starts = (uintptr_t)A.x | (uintptr_t)(A.M > 1 ? A.ld_x * 2 : 0);
  if ((starts & 15) == 0) {                                 // a lane takes units, a warp eight step pairs of one token to one of eight
    const int some = A.M > 4 ? 3 : A.M > 2 ? 2 : A.M - 1, r = lane >> 2, pairs = 8 >> some;
    for (int sp = warp * pairs + (r >> some); sp < 4 * kblocks; sp += kWarps * pairs) {
      const int k = kb0 * kBlockK + sp * 32 + (lane & 3) * 8, bytes = k < A.K ? (A.K - k < 8 ? (int)(A.K - k) * 2 : 16) : 0;        // the rest is zeros
      const uint16_t* xr = (const uint16_t*)A.x + (bytes ? k : 0);
      uint4* to = xs + sp * A.M * 4 + (lane & 3);
#pragma unroll 1
      for (int m = r & ((1 << some) - 1); m < A.M; m += 8)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to + m * 4)),
                     "l"(xr + m * A.ld_x), "r"(bytes) : "memory");
    }
  } else {                                                  // a lane takes two columns, a warp half a block's, token after token
    for (int half = warp; half < 2 * kblocks; half += kWarps) {
      const int k = kb0 * kBlockK + half * 64 + lane * 2;
      const int valid = k + 1 < A.K ? 4 : k < A.K ? 2 : 0;  // bytes; the rest is filled with zeros
      const uint16_t* xr = (const uint16_t*)A.x + (valid ? k : 0);
      uint32_t* to = (uint32_t*)(xs + (half * 2 + (lane >> 4)) * A.M * 4) + (lane & 15);
      if ((starts & 3) == 0) {
#pragma unroll 1
        for (int m = 0; m < A.M; ++m, xr += A.ld_x, to += 16)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(xr), "r"(valid) : "memory");
      } else if (A.M > 4) {             // rows that start on odd elements, eight tokens together (15 x 84091 x 3347: 53 us by four, 45)
#pragma unroll 1
        for (int m = 0; m < A.M; m += 8) {
          uint32_t lo[8], hi[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint16_t* const from = xr + (m + i < A.M ? (m + i) * A.ld_x : 0);
            lo[i] = valid ? __ldg(from) : 0u;
            hi[i] = valid == 4 ? __ldg(from + 1) : 0u;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (m + i < A.M) to[(m + i) * 16] = lo[i] | hi[i] << 16;
        }
      } else {
#pragma unroll 4
        for (int m = 0; m < A.M; ++m)
          to[m * 16] = (valid ? __ldg(xr + m * A.ld_x) : 0u) | (valid == 4 ? (uint32_t)__ldg(xr + m * A.ld_x + 1) << 16 : 0u);
      }
    }
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
  for (int j = 2; j < kDepth; ++j) fetch();
  asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 2) : "memory");
  __syncthreads();

  float acc[TILES][NT][4];
#pragma unroll
  for (int j = 0; j < TILES; ++j)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][t][e] = 0.f;
  auto keep_part = [&]() {
#pragma unroll
    for (int j = 0; j < TILES; ++j)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        parts[((warp * TILES + j) * NT + t) * 32 + lane] = make_float4(acc[j][t][0], acc[j][t][1], acc[j][t][2], acc[j][t][3]);
  };
  int64_t tile = b0 / tile_units;                   // within the CTA's run
  auto put_tile = [&]() {
#pragma unroll
    for (int j = 0; j < TILES; ++j) {
      if constexpr (SPLIT) {
#pragma unroll
        for (int t = 0; t < NT; ++t) sums[(tile * NT + t) * 32 + lane] = make_float4(acc[j][t][0], acc[j][t][1], acc[j][t][2], acc[j][t][3]);
      } else {
        store_tile<NT>(A, acc[j], (tile0 + tile) * TILES + j, lane);
      }
    }
  };
  int kb = (int)(b0 - tile * tile_units);
  bool whole = kb == 0;                             // this warp has the tile from its first block on
  const int row = lane >> 2;
  // (a column of B makes the same column of the result alone: places without a token take the last token's, and are not stored)
  const uint4* xt[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) xt[t] = xs + min(t * 8 + row, A.M - 1) * 4 + (lane & 3);
  const int x_pair = A.M * 4;
  int x_at = kb * UNIT * 4 * x_pair;
  for (int b = 0; b < count; ++b) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
    __syncwarp();
#pragma unroll
    for (int u = 0; u < UNIT; ++u) {
      uint32_t sw[TILES][2][GROUPS];
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        const char* const words = ring + slot_out + (u + j) * kBlock + 1024;
        if constexpr (GROUPS == 1) {
          sw[j][0][0] = ((const uint32_t*)words)[row];
          sw[j][1][0] = ((const uint32_t*)words)[row + 8];
        } else if constexpr (GROUPS == 2) {
          *(uint2*)sw[j][0] = ((const uint2*)words)[row];
          *(uint2*)sw[j][1] = ((const uint2*)words)[row + 8];
        } else {
          *(uint4*)sw[j][0] = ((const uint4*)words)[row];
          *(uint4*)sw[j][1] = ((const uint4*)words)[row + 8];
        }
      }
      float part[TILES][NT][4];
      uint32_t z0[TILES], z1[TILES];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint4 v[TILES];
#pragma unroll
        for (int j = 0; j < TILES; ++j) v[j] = ((const uint4*)(ring + slot_out + (u + j) * kBlock))[half * 32 + lane];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const int pair = half * 2 + p;
          uint4 f[NT];
#pragma unroll
          for (int t = 0; t < NT; ++t) f[t] = xt[t][x_at + (u * 4 + pair) * x_pair];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int step = pair * 2 + h, grp = step * GROUPS / 8;
            const bool first = step % (8 / GROUPS) == 0;
#pragma unroll
            for (int j = 0; j < TILES; ++j) {
              if (first) {
                z0[j] = minus_scaled2((sw[j][0][grp] & 15u) * 0x00010001u);
                z1[j] = minus_scaled2((sw[j][1][grp] & 15u) * 0x00100010u);
              }
              const uint32_t w = p == 0 ? (h == 0 ? v[j].x : v[j].y) : (h == 0 ? v[j].z : v[j].w);
              uint32_t a[4];
              const uint32_t w8 = w >> 8;
              a[0] = scaled2(w & 0x000f000fu, z0[j]);
              a[1] = scaled2(w & 0x00f000f0u, z1[j]);
              a[2] = scaled2(w8 & 0x000f000fu, z0[j]);
              a[3] = scaled2(w8 & 0x00f000f0u, z1[j]);
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                if (first) mma_bf16_first(part[j][t], a, h == 0 ? f[t].x : f[t].z, h == 0 ? f[t].y : f[t].w);
                else mma_bf16(part[j][t], a, h == 0 ? f[t].x : f[t].z, h == 0 ? f[t].y : f[t].w);
              }
              if ((step + 1) % (8 / GROUPS) == 0) {
                const float s0 = __uint_as_float(sw[j][0][grp] & ~15u), s1 = __uint_as_float(sw[j][1][grp] & ~15u);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                  acc[j][t][0] = fmaf(part[j][t][0], s0, acc[j][t][0]);
                  acc[j][t][1] = fmaf(part[j][t][1], s0, acc[j][t][1]);
                  acc[j][t][2] = fmaf(part[j][t][2], s1, acc[j][t][2]);
                  acc[j][t][3] = fmaf(part[j][t][3], s1, acc[j][t][3]);
                }
              }
            }
          }
        }
      }
    }
    __syncwarp();                                   // (every lane has read the scales: the place may be filled again)
    fetch();
    slot_out = slot_out == (kDepth - 1) * kBytes ? 0 : slot_out + kBytes;
    x_at += UNIT * 4 * x_pair;
    if (++kb == tile_units) {
      if (whole) {
        put_tile();
      } else {
        keep_part();
      }
#pragma unroll
      for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][t][e] = 0.f;
      kb = 0;
      x_at = 0;
      ++tile;
      whole = true;
    }
  }
  // A tile that is not finished: its first warp keeps its part and adds those of the warps after it, in their order.
  const bool open = count > 0 && kb != 0;
  if (open && !whole) keep_part();
  __syncthreads();
  if (open && whole) {
    const int64_t end = (tile + 1) * tile_units;
    for (int o = warp + 1; o < kWarps; ++o) {
      const int64_t o0 = blocks * o / kWarps, o1 = blocks * (o + 1) / kWarps;
      if (o0 >= end) break;
      if (o1 == o0) continue;
#pragma unroll
      for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float4 v = parts[((o * TILES + j) * NT + t) * 32 + lane];
          acc[j][t][0] += v.x; acc[j][t][1] += v.y; acc[j][t][2] += v.z; acc[j][t][3] += v.w;
        }
    }
    put_tile();
  }
  if constexpr (SPLIT) {
    cluster_sync();
    for (int64_t i = rank + (int64_t)warp * ctas; i < tile1 - tile0; i += (int64_t)kWarps * ctas) {
      float sum[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[t][e] = 0.f;
      for (int o = 0; o < ctas; ++o)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float4 v = load_cluster(sums + (i * NT + t) * 32 + lane, o);
          sum[t][0] += v.x; sum[t][1] += v.y; sum[t][2] += v.z; sum[t][3] += v.w;
        }
      store_tile<NT>(A, sum, tile0 + i, lane);
    }
    cluster_sync();                                 // (no CTA leaves while its sums are read)
  }
}

// One thread per 32-bit word of a block: a lane's 8 weights of one step, or one (row, group) scale word.
__global__ void __launch_bounds__(256) w4_pack_kernel(W4PackArgs A) {
  const int groups = kBlockK / A.group, words = 256 + kTileRows * groups;
  const int64_t total = A.tiles * A.kblocks * words;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t block = i / words;
    const int w = (int)(i - block * words);
    const int64_t tile = block / A.kblocks, k0 = (block - tile * A.kblocks) * kBlockK;
    auto zero_of = [&](int64_t n, int64_t k) -> uint32_t {
      return A.zeros && n < A.N && k < A.K ? A.zeros[n * A.ld_zeros + k / A.group] & 15u : 8u;
    };
    uint32_t v = 0;
    if (w < 256) {
      const int half = w >> 7, lane = (w >> 2) & 31, step = half * 4 + (w & 3);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t n = tile * kTileRows + (lane >> 2) + (j & 1) * 8;
        const int64_t k = k0 + (step >> 1) * 32 + (lane & 3) * 8 + (step & 1) * 4 + (j >> 1) * 2;
        const uint32_t z = zero_of(n, k);                 // past the end: q = z, which contributes nothing
        const uint32_t byte = n < A.N && k < A.K ? A.q[n * A.ld_q + k / 2] : z | z << 4;
        v |= (byte & 15u) << (4 * j);
        v |= (k + 1 < A.K ? byte >> 4 : z) << (16 + 4 * j);
      }
    } else {
      const int row = (w - 256) / groups;
      const int64_t n = tile * kTileRows + row, k = k0 + (int64_t)((w - 256) - row * groups) * A.group;
      float s = 0.f;
      if (n < A.N && k < A.K) {
        const int64_t at = n * A.ld_scales + k / A.group;
        s = A.scales_bf16 ? __uint_as_float((uint32_t)((const uint16_t*)A.scales)[at] << 16)
                          : __half2float(((const __half*)A.scales)[at]);
      }
      v = (__float_as_uint(s) & ~15u) | zero_of(n, k);
    }
    ((uint32_t*)A.packed)[i] = v;
  }
}

// Clusters of `split` CTAs that are resident at once, or fewer (a cluster is within one of the groups that the SMs form, and each of these
// has some left over: 74, 33 and 15 of 2, 4 and 8), and the shared memory a CTA needs for its part of x and its run's sums.
int split_runs(int64_t tiles, int split, int sms) {
  const int64_t most = sms > 6 * split ? (sms - 5 * (split - 1)) / split : 1;
  return (int)(tiles < most ? tiles : most);
}
int64_t split_bytes(int64_t tiles, int64_t kblocks, int64_t M, int nt, int split, int sms) {
  const int runs = split_runs(tiles, split, sms);
  return (tiles + runs - 1) / runs * nt * 512 + (kblocks + split - 1) / split * kBlockK * 2 * M;
}
constexpr int kMaxSplit = 8;
constexpr int token_groups(int64_t M) { return M <= 8 ? 1 : M <= 16 ? 2 : 4; }      // of eight, that the products take
// CTAs that share the columns of a tile, 1: none.  Two or more where the tokens' x does not fit beside the ring (it would take a launch
// for each part of the tokens, each reading the weights again), as few as fit with the run's sums (30 tokens, 9217 x 8192: 51 us in
// launches, 29 in clusters of eight); and where tiles are few, so that more SMs work (28 tokens, 109 x 6274: 26 us, 7.8; one token,
// 256 x 8192: 5.3, 4.1).
int split_of(int64_t tiles, int64_t kblocks, int groups, int64_t M, int sms) {
  const int nt = token_groups(M);
  const int64_t room = x_bytes(nt, 1, 1, groups);
  const bool fits = M * kblocks * kBlockK * 2 <= room;
  int best = 1;
  for (int split = 2; split <= kMaxSplit && split <= kblocks; split *= 2) {
    if (split_bytes(tiles, kblocks, M, nt, split, sms) > room) continue;
    if (fits && !(tiles * split * 2 <= sms && kblocks >= 8 * split)) break;
    best = split;
    if (!fits) break;
  }
  return best;
}

template <int NT, int GROUPS, int TILES, int UNIT, bool SPLIT = false>
cudaError_t run(const W4Args& a, cudaStream_t s, int sms, int device) {
  static std::atomic<bool> ready[64];               // per device: the kernel may use this much shared memory
  if (device < 0 || device >= 64 || !ready[device].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(w4_kernel<NT, GROUPS, TILES, UNIT, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
    if (e != cudaSuccess) return e;
    if (device >= 0 && device < 64) ready[device].store(true, std::memory_order_release);
  }
  const int64_t runs = (a.tiles + TILES - 1) / TILES;
  int bytes, grid;
  if constexpr (SPLIT) {
    grid = split_runs(a.tiles, a.split, sms) * a.split;
    bytes = kSharedBytes - x_bytes(NT, 1, 1, GROUPS) + (int)split_bytes(a.tiles, a.kblocks, a.M, NT, a.split, sms);
  } else {
    grid = (int)(runs < sms ? runs : sms);
    bytes = ring_bytes(TILES * UNIT, GROUPS) + part_bytes(TILES, NT) + (int)a.kblocks * kBlockK * 2 * a.M;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // set up while the kernel before it ends: 0.5 us a call
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = SPLIT ? a.split : 1;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = SPLIT ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, w4_kernel<NT, GROUPS, TILES, UNIT, SPLIT>, a);
}

template <int NT, int GROUPS>
cudaError_t run_unit(const W4Args& a, cudaStream_t s, int sms, int device) {
  const int64_t grid = a.tiles < sms ? a.tiles : sms, x = a.kblocks * kBlockK * 2 * a.M;
  if (a.split > 1) return run<NT, GROUPS, 1, 1, true>(a, s, sms, device);
  if constexpr (NT == 1) {
    if (a.tiles >= 8 * sms && x <= x_bytes(1, 2, 1, GROUPS)) return run<1, GROUPS, 2, 1>(a, s, sms, device);
    // (with fewer units than these half of the warps would be idle)
    if (a.kblocks % 2 == 0 && a.tiles * a.kblocks >= 4 * kWarps * grid && x <= x_bytes(1, 1, 2, GROUPS))
      return run<1, GROUPS, 1, 2>(a, s, sms, device);
  }
  return run<NT, GROUPS, 1, 1>(a, s, sms, device);
}

template <int NT>
cudaError_t run_groups(const W4Args& a, int group, cudaStream_t s, int sms, int device) {
  if (group == 128) return run_unit<NT, 1>(a, s, sms, device);
  if (group == 64) return run_unit<NT, 2>(a, s, sms, device);
  return run_unit<NT, 4>(a, s, sms, device);
}

// Blocks of 128 columns a row has in the layout: an even number (the last one zeros) for weights large enough to be taken by two.
int64_t blocks_of(int64_t N, int64_t K) {
  const int64_t n = (K + kBlockK - 1) / kBlockK, tiles = (N + kTileRows - 1) / kTileRows;
  return n >= 8 && tiles * n >= 8192 ? (n + 1) / 2 * 2 : n;
}

}  // namespace

size_t w4_packed_bytes(int64_t N, int64_t K, int group) {
  const int64_t tiles = (N + kTileRows - 1) / kTileRows;
  return (size_t)(tiles * blocks_of(N, K)) * (size_t)block_bytes(kBlockK / group);
}

cudaError_t launch_w4_pack(W4PackArgs a, cudaStream_t s, int sms) {
  a.tiles = (a.N + kTileRows - 1) / kTileRows;
  a.kblocks = blocks_of(a.N, a.K);
  w4_pack_kernel<<<sms * 8, 256, 0, s>>>(a);
  return cudaGetLastError();
}

// Tokens of one launch, of M that are left (32 at most).  As few launches as shared memory allows, since each reads all weights: x of a
// launch is in one block or in the clusters that share the columns (one token always fits).  The launches are even, or all but the last
// whole groups of eight tokens where that makes fewer groups, which is what the products take (23 tokens, 26375 x 7955: 15 and 8 72 us, 12
// and 11 79; 32 tokens, 4096 x 14336: 16 and 16 28 us, 26 and 6 37).
int w4_tokens_per_launch(int64_t N, int64_t K, int group, int64_t M, int sms) {
  const int groups = kBlockK / group;
  const int64_t tiles = (N + kTileRows - 1) / kTileRows, kblocks = blocks_of(N, K);
  auto fits = [&](int64_t m) {
    return m * kblocks * kBlockK * 2 <= x_bytes(token_groups(m), 1, 1, groups) || split_of(tiles, kblocks, groups, m, sms) > 1;
  };
  int64_t m = M < kW4MaxTokens ? M : kW4MaxTokens;
  while (m > 1 && !fits(m)) --m;
  const int64_t launches = (M + m - 1) / m, even = (M + launches - 1) / launches, whole = (even + 7) / 8 * 8 < m ? (even + 7) / 8 * 8 : m;
  auto products = [&](int64_t each) { return (launches - 1) * token_groups(each) + token_groups(M - (launches - 1) * each); };
  return (int)(products(whole) < products(even) ? whole : even);
}

cudaError_t launch_w4(W4Args a, int group, cudaStream_t s, int sms, int device) {
  a.tiles = (a.N + kTileRows - 1) / kTileRows;
  a.kblocks = blocks_of(a.N, a.K);
  a.split = split_of(a.tiles, a.kblocks, kBlockK / group, a.M, sms);
  static_assert(kW4MaxK * 2 <= x_bytes(1, 1, 1, 4), "one token fits");
  if (a.M <= 8) return run_groups<1>(a, group, s, sms, device);
  if (a.M <= 16) return run_groups<2>(a, group, s, sms, device);
  return run_groups<4>(a, group, s, sms, device);
}

}  // namespace jp
