// Linear layer with 4-bit weights and group scales for a few tokens:
//   out[m, n] = sum_k x[m, k] (q[n, k] - z[n, k / group]) s[n, k / group]
//
// The weights are read once, half a byte each, and bound the call by HBM: at 6.5 TB/s an SM gets about 46 weights a
// clock.  The products go through mma.sync m16n8k16 with 16 rows of weights as A and 8 tokens as B: q - z is a small
// integer, exact in bf16, so a group's sum is exact products added in fp32, and the group's scale multiplies that
// fp32 sum.  (tcgen05 would need the 16-bit weights written to shared memory or TMEM first, 92 of the 128 bytes a
// clock that shared memory moves, and a TMEM read per group for the scales; with 1 to 32 tokens its rate is of no use.)
//
// Weights are laid out once (pack_kernel) in the order the MMA's A fragments want them: tiles of 16 rows, blocks of 128
// columns, per block 8 steps of k = 16.  A lane's 8 weights of a step are one 32-bit word whose nibbles j and j + 4 are the
// two halves of fragment register j, so (word >> 4j) & 0x000f000f | 0x43004300 is that register plus 128 (bf16 128 + q), and
// one packed subtraction of 128 + z gives the exact value.  A block is 1024 bytes of words, then one 32-bit word per
// (row, group): the scale as fp32 with its low 4 bits replaced by z (scales come in bf16 or fp16: those bits are zero).
// Blocks of a tile follow one another, tiles too: what a warp reads is one contiguous run of memory.
//
// Work split: a CTA takes a contiguous run of tiles, and its 16 warps take equal contiguous runs of the CTA's blocks,
// whatever the tile boundaries.  So every size keeps all warps busy to within one block; a tile that two or more warps share is
// summed in shared memory in the warps' order (deterministic).  x is staged in shared memory once per CTA in B-fragment order.
#include <cuda_fp16.h>

#include "jp_common.cuh"
#include "jp_internal.h"

namespace jp {
namespace {

constexpr int kTileRows = 16;
constexpr int kBlockK = 128;
constexpr int kWarps = 16;
constexpr int kDepth = 4;             // blocks a warp has in flight
constexpr int kXBytes = 128 * 1024;   // shared memory for x

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// (w >> shift) & 0x000f000f | 0x43004300, minus 128 + z in both halves: two exact bf16 integers
__device__ __forceinline__ uint32_t dequant2(uint32_t w, int shift, uint32_t z128) {
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(r) : "r"(w >> shift));
  const __nv_bfloat162 d = __hsub2(*(const __nv_bfloat162*)&r, *(const __nv_bfloat162*)&z128);
  return *(const uint32_t*)&d;
}

template <int GROUPS> struct ScaleWords;      // a row's scale words of one block
template <> struct ScaleWords<1> { uint32_t w[1]; };
template <> struct alignas(8) ScaleWords<2> { uint32_t w[2]; };
template <> struct alignas(16) ScaleWords<4> { uint32_t w[4]; };

template <int GROUPS>
struct Block {
  uint4 q[2];
  ScaleWords<GROUPS> s[2];                    // rows lane / 4 and lane / 4 + 8
};

template <int GROUPS>
__device__ __forceinline__ void load_block(Block<GROUPS>& b, const char* p, int lane) {
  b.q[0] = ldg_stream((const uint4*)p + lane);
  b.q[1] = ldg_stream((const uint4*)p + 32 + lane);
  const ScaleWords<GROUPS>* s = (const ScaleWords<GROUPS>*)(p + 1024);
  b.s[0] = s[lane >> 2];
  b.s[1] = s[(lane >> 2) + 8];
}

template <int NT, int GROUPS>
__device__ __forceinline__ void store_tile(const W4Args& A, const float (&acc)[NT][4], int64_t tile, int lane) {
  const int64_t n = tile * kTileRows + (lane >> 2);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t row = n + (e >> 1) * 8;
      const int m = t * 8 + (lane & 3) * 2 + (e & 1);
      if (m < A.M && row < A.N) {
        if (A.out_bf16) ((__nv_bfloat16*)A.out)[m * A.ld_out + row] = __float2bfloat16_rn(acc[t][e]);
        else ((float*)A.out)[m * A.ld_out + row] = acc[t][e];
      }
    }
}

template <int NT, int GROUPS>
__global__ void __launch_bounds__(kWarps * 32, 1) w4_kernel(W4Args A) {
  constexpr int kBytes = 1024 + kTileRows * 4 * GROUPS;
  extern __shared__ __align__(16) char smem[];
  float4* slots = (float4*)smem;                                        // [warp][head, tail][NT][lane]
  uint4* xs = (uint4*)(smem + kWarps * 2 * NT * 32 * 16);               // [block][step pair][token][lane % 4]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t tile0 = A.tiles * blockIdx.x / gridDim.x, tile1 = A.tiles * (blockIdx.x + 1) / gridDim.x;
  const int64_t blocks = (tile1 - tile0) * A.kblocks;
  const int64_t b0 = blocks * warp / kWarps, b1 = blocks * (warp + 1) / kWarps;
  const char* base = (const char*)A.packed + tile0 * A.kblocks * kBytes;
  Block<GROUPS> ring[kDepth];
#pragma unroll
  for (int j = 0; j < kDepth; ++j)
    if (b0 + j < b1) load_block(ring[j], base + (b0 + j) * kBytes, lane);

  // x in B-fragment order: word w of unit (block, step pair, token, t) is columns 128 block + 32 pair + 16 (w / 2)
  // + 8 (w % 2) + 2 t and the next
  const int units = (int)A.kblocks * 4 * A.M * 4;
  for (int u = tid; u < units; u += kWarps * 32) {
    const int t = u & 3, m = (u >> 2) % A.M, pair = (u >> 2) / A.M;
    const uint16_t* xr = (const uint16_t*)A.x + (int64_t)m * A.ld_x;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t k = (int64_t)pair * 32 + (i >> 1) * 16 + (i & 1) * 8 + t * 2;
      const uint32_t lo = k < A.K ? xr[k] : 0, hi = k + 1 < A.K ? xr[k + 1] : 0;
      w[i] = lo | hi << 16;
    }
    xs[u] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __syncthreads();

  float acc[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[t][e] = 0.f;
  int64_t tile = b0 / A.kblocks;                    // within the CTA's run
  int kb = (int)(b0 - tile * A.kblocks);
  bool whole = kb == 0;                             // this warp has the tile from its first block on
  for (int64_t b = b0; b < b1; b += kDepth) {
#pragma unroll
    for (int j = 0; j < kDepth; ++j) {
      if (b + j < b1) {
        const uint4* xb = xs + (int64_t)kb * 16 * A.M;
        float part[NT][4];
#pragma unroll
        for (int step = 0; step < 8; ++step) {
          const int grp = step * GROUPS / 8;
          if (step % (8 / GROUPS) == 0) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) part[t][e] = 0.f;
          }
          const uint32_t z0 = (ring[j].s[0].w[grp] & 15u) * 0x00010001u | 0x43004300u;
          const uint32_t z1 = (ring[j].s[1].w[grp] & 15u) * 0x00010001u | 0x43004300u;
          const uint4& v = ring[j].q[step >> 2];
          const uint32_t w = (step & 3) == 0 ? v.x : (step & 3) == 1 ? v.y : (step & 3) == 2 ? v.z : v.w;
          uint32_t a[4];
          a[0] = dequant2(w, 0, z0);
          a[1] = dequant2(w, 4, z1);
          a[2] = dequant2(w, 8, z0);
          a[3] = dequant2(w, 12, z1);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const int m = t * 8 + (lane >> 2);
            uint2 f = make_uint2(0u, 0u);
            if (m < A.M) f = ((const uint2*)(xb + ((step >> 1) * A.M + m) * 4 + (lane & 3)))[step & 1];
            mma_bf16(part[t], a, f.x, f.y);
          }
          if ((step + 1) % (8 / GROUPS) == 0) {
            const float s0 = __uint_as_float(ring[j].s[0].w[grp] & ~15u), s1 = __uint_as_float(ring[j].s[1].w[grp] & ~15u);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              acc[t][0] = fmaf(part[t][0], s0, acc[t][0]);
              acc[t][1] = fmaf(part[t][1], s0, acc[t][1]);
              acc[t][2] = fmaf(part[t][2], s1, acc[t][2]);
              acc[t][3] = fmaf(part[t][3], s1, acc[t][3]);
            }
          }
        }
        if (b + j + kDepth < b1) load_block(ring[j], base + (b + j + kDepth) * kBytes, lane);
        ++kb;
        const bool tile_end = kb == A.kblocks;
        if (tile_end || b + j + 1 == b1) {
          if (tile_end && whole) {
            store_tile<NT, GROUPS>(A, acc, tile0 + tile, lane);
          } else {
            // slot 0: the part of a tile that an earlier warp began; slot 1: of one that this warp begins
            float4* s = slots + ((warp * 2 + (whole ? 1 : 0)) * NT) * 32 + lane;
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t * 32] = make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
          }
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] = 0.f;
          if (tile_end) { kb = 0; ++tile; whole = true; }
        }
      }
    }
  }
  __syncthreads();
  // The warp that has a shared tile's first block adds the parts of the warps after it.
  if (b1 > b0) {
    const int64_t last = (b1 - 1) / A.kblocks, end = (last + 1) * A.kblocks;
    if (b1 < end && last * A.kblocks >= b0) {
      float sum[NT][4];
      const float4* s = slots + ((warp * 2 + 1) * NT) * 32 + lane;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float4 v = s[t * 32];
        sum[t][0] = v.x; sum[t][1] = v.y; sum[t][2] = v.z; sum[t][3] = v.w;
      }
      for (int o = warp + 1; o < kWarps; ++o) {
        const int64_t o0 = blocks * o / kWarps, o1 = blocks * (o + 1) / kWarps;
        if (o0 >= end) break;
        if (o1 == o0) continue;
        const float4* q = slots + ((o * 2) * NT) * 32 + lane;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float4 v = q[t * 32];
          sum[t][0] += v.x; sum[t][1] += v.y; sum[t][2] += v.z; sum[t][3] += v.w;
        }
      }
      store_tile<NT, GROUPS>(A, sum, tile0 + last, lane);
    }
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
        const int64_t k = k0 + step * 16 + (j >> 1) * 8 + (lane & 3) * 2;
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

template <int NT, int GROUPS>
cudaError_t run(const W4Args& a, cudaStream_t s, int sms) {
  const int bytes = kWarps * 2 * NT * 32 * 16 + (int)a.kblocks * 4 * a.M * 4 * 16;
  cudaError_t e = cudaFuncSetAttribute(w4_kernel<NT, GROUPS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       kWarps * 2 * NT * 32 * 16 + kXBytes);
  if (e != cudaSuccess) return e;
  const int grid = (int)(a.tiles < sms ? a.tiles : sms);
  w4_kernel<NT, GROUPS><<<grid, kWarps * 32, bytes, s>>>(a);
  return cudaGetLastError();
}

template <int NT>
cudaError_t run_groups(const W4Args& a, int group, cudaStream_t s, int sms) {
  if (group == 128) return run<NT, 1>(a, s, sms);
  if (group == 64) return run<NT, 2>(a, s, sms);
  return run<NT, 4>(a, s, sms);
}

}  // namespace

size_t w4_packed_bytes(int64_t N, int64_t K, int group) {
  const int64_t tiles = (N + kTileRows - 1) / kTileRows, kblocks = (K + kBlockK - 1) / kBlockK;
  return (size_t)(tiles * kblocks) * (size_t)(1024 + kTileRows * 4 * (kBlockK / group));
}

cudaError_t launch_w4_pack(W4PackArgs a, cudaStream_t s, int sms) {
  a.tiles = (a.N + kTileRows - 1) / kTileRows;
  a.kblocks = (a.K + kBlockK - 1) / kBlockK;
  w4_pack_kernel<<<sms * 8, 256, 0, s>>>(a);
  return cudaGetLastError();
}

// Tokens of one launch: as many as shared memory holds of x.
int w4_tokens_per_launch(int64_t K) {
  const int64_t kblocks = (K + kBlockK - 1) / kBlockK;
  const int64_t m = kXBytes / (kblocks * kBlockK * 2);
  return (int)(m < kW4MaxTokens ? m : kW4MaxTokens);
}

cudaError_t launch_w4(W4Args a, int group, cudaStream_t s, int sms) {
  a.tiles = (a.N + kTileRows - 1) / kTileRows;
  a.kblocks = (a.K + kBlockK - 1) / kBlockK;
  if (a.M <= 8) return run_groups<1>(a, group, s, sms);
  if (a.M <= 16) return run_groups<2>(a, group, s, sms);
  return run_groups<4>(a, group, s, sms);
}

}  // namespace jp
