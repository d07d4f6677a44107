// The norms before and after a block of a model, fused with its gate and the residual stream: forward and backward over rows [T, H].
//
//   u = (x - mu1) r1 w1 + b1  (the norm behind the block; u = x without w1),   s = residual + a gt[t] gc[h] u  (rounded to its type),
//   y = (s - mu2) r2 w2 + b2  (the norm in front of the next block, of s as stored: what the backward reads);  mu = 0 for RMS norm
//   gs = ds + r2 (g2 - mean g2 - xhat2 mean(g2 xhat2)), g2 = dy w2;   dresidual = gs
//   du = a gt gc gs;   dx = r1 (g1 - mean g1 - xhat1 mean(g1 xhat1)), g1 = du w1
//   dgc = sum_t a gt u gs,  dgt = sum_h a gc u gs,  dw1 = sum_t du xhat1,  db1 = sum_t du,  dw2 = sum_t dy xhat2,  db2 = sum_t dy
//
// Bound by HBM: forward reads x and the residual and writes s and y, backward reads dy, ds, s and x and writes dresidual and dx, each
// once.  A row stays in the registers of one block of threads through all of its sums; the next row is fetched meanwhile.  A thread owns
// fixed columns, so the sums over rows add up in its registers; blocks leave a line each in the workspace, which a second kernel
// adds in a fixed order: no atomics, the same bits every time.
#include "jp_common.cuh"
#include "jp_internal.h"

namespace jp {
namespace {

constexpr int kMaxWarps = 32;

__device__ __forceinline__ float param(const void* p, int64_t i, bool bf16) {
  return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16) : ((const float*)p)[i];
}

// W consecutive elements: a 16-byte vector, or one element where rows do not start on 16 bytes.
template <int DT, int W> struct Item;
template <int DT> struct Item<DT, Vec<DT>::N> {
  uint4 v;
  __device__ __forceinline__ void load(const void* p) {
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  }
  __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ float get(int e) const { return Vec<DT>::get(v, e); }
  __device__ __forceinline__ void set(const float* f) {     // rounds
    if constexpr (DT == JP_BF16) {
      uint32_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
        o[e] = *(const uint32_t*)&h;
      }
      v = make_uint4(o[0], o[1], o[2], o[3]);
    } else {
      v = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
  }
  __device__ __forceinline__ void store(void* p) const { stg_stream((uint4*)p, v); }
};
template <int DT> struct Item<DT, 1> {
  uint32_t v;                                               // as fp32
  __device__ __forceinline__ void load(const void* p) {
    if constexpr (DT == JP_BF16) v = (uint32_t)(*(const volatile uint16_t*)p) << 16;
    else v = *(const volatile uint32_t*)p;
  }
  __device__ __forceinline__ void zero() { v = 0u; }
  __device__ __forceinline__ float get(int) const { return __uint_as_float(v); }
  __device__ __forceinline__ void set(const float* f) {
    v = DT == JP_BF16 ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(f[0])) << 16 : __float_as_uint(f[0]);
  }
  __device__ __forceinline__ void store(void* p) const {
    if constexpr (DT == JP_BF16) *(uint16_t*)p = (uint16_t)(v >> 16);
    else *(uint32_t*)p = v;
  }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// N sums over the block, in all of its threads.  `slot` alternates between uses, so that one barrier each is enough.
template <int N> __device__ __forceinline__ void block_sums(float (&v)[N], float (*sh)[3][kMaxWarps], int& slot) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
  if (blockDim.x == 32) return;
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  float (*part)[kMaxWarps] = sh[slot];
  slot ^= 1;
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) part[i][threadIdx.x >> 5] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < warps ? part[i][lane] : 0.f);
}

template <int W> __device__ __forceinline__ int64_t column(int i) { return (int64_t)(threadIdx.x + i * (int)blockDim.x) * W; }

// W parameters from column c on (through L1: every row reads them again), 1 or 0 where there are none
template <int W> __device__ __forceinline__ void params(const void* p, int64_t c, bool bf16, float none, float* f) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < W; ++e) f[e] = none;
  } else if constexpr (W == 1) {
    f[0] = param(p, c, bf16);
  } else if (bf16) {
    if constexpr (W == 8) {
      const uint4 v = __ldg((const uint4*)((const uint16_t*)p + c));
#pragma unroll
      for (int e = 0; e < W; ++e) f[e] = Vec<JP_BF16>::get(v, e);
    } else {
      const uint2 v = __ldg((const uint2*)((const uint16_t*)p + c));
      f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
      f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int q = 0; q < W; q += 4) {
      const float4 v = __ldg((const float4*)((const float*)p + c + q));
      f[q] = v.x; f[q + 1] = v.y; f[q + 2] = v.z; f[q + 3] = v.w;
    }
  }
}

// Mean (0 for RMS norm) and 1 / sqrt(mean of squares + eps) of a row held in registers; squares are taken of x - mu.
template <int DT, int W, int NV>
__device__ __forceinline__ void row_stats(const BlockArgs& A, const Item<DT, W> (&x)[NV], float (*sh)[3][kMaxWarps], int& slot, float& mean, float& rstd) {
  const float inv_h = 1.f / (float)A.H;
  mean = 0.f;
  if (!A.rms) {
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < W; ++e) s[0] += x[i].get(e);      // (0 past the end)
    block_sums<1>(s, sh, slot);
    mean = s[0] * inv_h;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (column<W>(i) < A.H) {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const float d = x[i].get(e) - mean;
        q[0] = fmaf(d, d, q[0]);
      }
    }
  block_sums<1>(q, sh, slot);
  rstd = 1.f / sqrtf(q[0] * inv_h + A.eps);
}

template <int DT, int W, int NV>
__global__ void __launch_bounds__(1024) block_fwd_kernel(BlockArgs A) {
  constexpr int ES = Vec<DT>::ESIZE;
  using It = Item<DT, W>;
  __shared__ float sh[2][3][kMaxWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int slot = 0;
  It nx[NV], nr[NV];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      nx[i].zero();
      nr[i].zero();
      if (row < A.T && c < A.H) {
        nx[i].load((const char*)A.x + (row * A.ld_x + c) * ES);
        nr[i].load((const char*)A.residual + (row * A.ld_residual + c) * ES);
      }
    }
  };
  fetch(blockIdx.x);
  for (int64_t row = blockIdx.x; row < A.T; row += gridDim.x) {
    It x[NV], s[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = nx[i];
      s[i] = nr[i];
    }
    fetch(row + gridDim.x);
    float scale = A.scale;
    if (A.token_gate) scale *= A.token_gate[row];
    float m1 = 0.f, r1 = 1.f, m2, r2;
    if (A.post_weight) {
      row_stats<DT, W, NV>(A, x, sh, slot, m1, r1);
      if (threadIdx.x == 0) {
        if (A.out_post_mean) A.out_post_mean[row] = m1;
        if (A.out_post_rstd) A.out_post_rstd[row] = r1;
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      if (c < A.H) {
        float w[W], b[W], g[W], o[W];
        params<W>(A.post_weight, c, A.param_bf16, 1.f, w);
        params<W>(A.post_bias, c, A.param_bf16, 0.f, b);
        params<W>(A.gate, c, A.param_bf16, 1.f, g);
#pragma unroll
        for (int e = 0; e < W; ++e) o[e] = fmaf(fmaf((x[i].get(e) - m1) * r1, w[e], b[e]), scale * g[e], s[i].get(e));
        s[i].set(o);
        s[i].store((char*)A.sum + (row * A.ld_sum + c) * ES);
      }
    }
    row_stats<DT, W, NV>(A, s, sh, slot, m2, r2);
    if (threadIdx.x == 0) {
      if (A.out_mean) A.out_mean[row] = m2;
      if (A.out_rstd) A.out_rstd[row] = r2;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      if (c < A.H) {
        float w[W], b[W], o[W];
        params<W>(A.weight, c, A.param_bf16, 1.f, w);
        params<W>(A.bias, c, A.param_bf16, 0.f, b);
#pragma unroll
        for (int e = 0; e < W; ++e) o[e] = fmaf((s[i].get(e) - m2) * r2, w[e], b[e]);
        It y;
        y.set(o);
        y.store((char*)A.y + (row * A.ld_y + c) * ES);
      }
    }
  }
}

// Any width: the rows are read again for each of their sums (from L2).
template <int DT>
__global__ void __launch_bounds__(1024) block_fwd_wide_kernel(BlockArgs A) {
  constexpr int ES = Vec<DT>::ESIZE;
  using It = Item<DT, 1>;
  __shared__ float sh[2][3][kMaxWarps];
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  auto at = [&](const void* p, int64_t i) { It t; t.load((const char*)p + i * ES); return t.get(0); };
  auto stats = [&](const void* p, int64_t first, float& mean, float& rstd) {
    mean = 0.f;
    if (!A.rms) {
      float s[1] = {0.f};
      for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) s[0] += at(p, first + c);
      block_sums<1>(s, sh, slot);
      mean = s[0] * inv_h;
    }
    float q[1] = {0.f};
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float d = at(p, first + c) - mean;
      q[0] = fmaf(d, d, q[0]);
    }
    block_sums<1>(q, sh, slot);
    rstd = 1.f / sqrtf(q[0] * inv_h + A.eps);
  };
  for (int64_t row = blockIdx.x; row < A.T; row += gridDim.x) {
    float scale = A.scale, m1 = 0.f, r1 = 1.f, m2, r2;
    if (A.token_gate) scale *= A.token_gate[row];
    if (A.post_weight) {
      stats(A.x, row * A.ld_x, m1, r1);
      if (threadIdx.x == 0) {
        if (A.out_post_mean) A.out_post_mean[row] = m1;
        if (A.out_post_rstd) A.out_post_rstd[row] = r1;
      }
    }
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      float w, b, g;
      params<1>(A.post_weight, c, A.param_bf16, 1.f, &w);
      params<1>(A.post_bias, c, A.param_bf16, 0.f, &b);
      params<1>(A.gate, c, A.param_bf16, 1.f, &g);
      const float o = fmaf(fmaf((at(A.x, row * A.ld_x + c) - m1) * r1, w, b), scale * g, at(A.residual, row * A.ld_residual + c));
      It s;
      s.set(&o);
      s.store((char*)A.sum + (row * A.ld_sum + c) * ES);
    }
    stats(A.sum, row * A.ld_sum, m2, r2);                   // (each thread reads what it wrote itself)
    if (threadIdx.x == 0) {
      if (A.out_mean) A.out_mean[row] = m2;
      if (A.out_rstd) A.out_rstd[row] = r2;
    }
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      float w, b;
      params<1>(A.weight, c, A.param_bf16, 1.f, &w);
      params<1>(A.bias, c, A.param_bf16, 0.f, &b);
      const float o = fmaf((at(A.sum, row * A.ld_sum + c) - m2) * r2, w, b);
      It y;
      y.set(&o);
      y.store((char*)A.y + (row * A.ld_y + c) * ES);
    }
  }
}

// Sums over rows: dw2, then db2 (BIAS), dw1 (POST), db1 (POST and BIAS), dgate (GATE), each a line of H.
__host__ __device__ constexpr int n_sums(bool post, bool gate, bool bias) { return 1 + bias + post + (post && bias) + gate; }
constexpr int kMaxSums = 5;

template <int DT, int W, int NV, bool POST, bool GATE, bool BIAS>
__global__ void __launch_bounds__(512) block_bwd_kernel(BlockArgs A) {
  constexpr int ES = Vec<DT>::ESIZE, N = n_sums(POST, GATE, BIAS);
  constexpr int B2 = 1, W1 = 1 + BIAS, B1 = W1 + 1, G = W1 + POST + (POST && BIAS);
  using It = Item<DT, W>;
  __shared__ float sh[2][3][kMaxWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  const bool use_x = POST || GATE || A.token_gate;
  float acc[N][NV][W];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < W; ++e) acc[n][i][e] = 0.f;
  It ndy[NV], nds[NV], ns[NV], nx[NV];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      ndy[i].zero(); nds[i].zero(); ns[i].zero(); nx[i].zero();
      if (row < A.T && c < A.H) {
        ndy[i].load((const char*)A.dy + (row * A.ld_dy + c) * ES);
        if (A.dsum) nds[i].load((const char*)A.dsum + (row * A.ld_dsum + c) * ES);
        ns[i].load((const char*)A.sum + (row * A.ld_sum + c) * ES);
        if (use_x) nx[i].load((const char*)A.x + (row * A.ld_x + c) * ES);
      }
    }
  };
  fetch(blockIdx.x);
  for (int64_t row = blockIdx.x; row < A.T; row += gridDim.x) {
    It dy[NV], ds[NV], s[NV], x[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      dy[i] = ndy[i]; ds[i] = nds[i]; s[i] = ns[i]; x[i] = nx[i];
    }
    const float m2 = A.rms ? 0.f : A.mean[row], r2 = A.rstd[row];
    const float m1 = POST && !A.rms ? A.post_mean[row] : 0.f, r1 = POST ? A.post_rstd[row] : 1.f;
    const float gt = A.token_gate ? A.token_gate[row] : 1.f;
    fetch(row + gridDim.x);
    float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      if (c < A.H) {
        float w[W];
        params<W>(A.weight, c, A.param_bf16, 1.f, w);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float d = dy[i].get(e), xh = (s[i].get(e) - m2) * r2, g = d * w[e];
          v[0] += g;
          v[1] = fmaf(g, xh, v[1]);
          acc[0][i][e] = fmaf(d, xh, acc[0][i][e]);
          if (BIAS) acc[B2][i][e] += d;
        }
      }
    }
    block_sums<3>(v, sh, slot);
    const float a1 = A.rms ? 0.f : v[0] * inv_h, a2 = v[1] * inv_h;
    float gs[NV][W], t[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      if (c < A.H) {
        float w2[W], w1[W], b1[W], gc[W];
        params<W>(A.weight, c, A.param_bf16, 1.f, w2);
        params<W>(POST ? A.post_weight : nullptr, c, A.param_bf16, 1.f, w1);
        params<W>(POST ? A.post_bias : nullptr, c, A.param_bf16, 0.f, b1);
        params<W>(GATE ? A.gate : nullptr, c, A.param_bf16, 1.f, gc);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float xh2 = (s[i].get(e) - m2) * r2;
          const float g = fmaf(r2, fmaf(-xh2, a2, fmaf(dy[i].get(e), w2[e], -a1)), ds[i].get(e));
          const float xh1 = (x[i].get(e) - m1) * r1, u = POST ? fmaf(xh1, w1[e], b1[e]) : x[i].get(e);
          const float gu = A.scale * g * u, du = A.scale * gt * gc[e] * g;
          gs[i][e] = g;
          if (GATE) acc[G][i][e] = fmaf(gt, gu, acc[G][i][e]);
          t[2] = fmaf(gc[e], gu, t[2]);
          if (POST) {
            const float g1 = du * w1[e];
            t[0] += g1;
            t[1] = fmaf(g1, xh1, t[1]);
            acc[W1][i][e] = fmaf(du, xh1, acc[W1][i][e]);
            if (BIAS) acc[B1][i][e] += du;
          }
        }
        It o;
        o.set(gs[i]);
        o.store((char*)A.dresidual + (row * A.ld_dresidual + c) * ES);
      }
    }
    if (POST || A.token_gate) block_sums<3>(t, sh, slot);
    if (A.token_gate && threadIdx.x == 0) A.dtoken_gate[row] = t[2];
    const float c1 = A.rms ? 0.f : t[0] * inv_h, c2 = t[1] * inv_h;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      if (c < A.H) {
        float w1[W], gc[W], o[W];
        params<W>(POST ? A.post_weight : nullptr, c, A.param_bf16, 1.f, w1);
        params<W>(GATE ? A.gate : nullptr, c, A.param_bf16, 1.f, gc);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float du = A.scale * gt * gc[e] * gs[i][e];
          o[e] = POST ? r1 * fmaf(-(x[i].get(e) - m1) * r1, c2, fmaf(du, w1[e], -c1)) : du;
        }
        It d;
        d.set(o);
        d.store((char*)A.dx + (row * A.ld_dx + c) * ES);
      }
    }
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // the kernel that adds the lines may set up
  float* line = A.partial + (int64_t)blockIdx.x * N * A.H;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (column<W>(i) < A.H) {
#pragma unroll
        for (int e = 0; e < W; ++e) line[n * A.H + column<W>(i) + e] = acc[n][i][e];
      }
}

// Any width: rows are read again for each sum, and the sums over rows stay in the block's line of the workspace (each thread its columns).
template <int DT>
__global__ void __launch_bounds__(1024) block_bwd_wide_kernel(BlockArgs A, int n_lines) {
  constexpr int ES = Vec<DT>::ESIZE;
  using It = Item<DT, 1>;
  __shared__ float sh[2][3][kMaxWarps];
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  const bool post = A.post_weight != nullptr, use_x = post || A.gate || A.token_gate, bias = A.with_bias;
  float* line = A.partial + (int64_t)blockIdx.x * n_lines * A.H;
  float* const l_w2 = line, * const l_b2 = line + A.H, * const l_w1 = line + (1 + bias) * A.H, * const l_b1 = l_w1 + A.H,
       * const l_g = line + (1 + bias + post + (post && bias)) * A.H;
  for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x)
    for (int n = 0; n < n_lines; ++n) line[n * A.H + c] = 0.f;
  auto at = [&](const void* p, int64_t i) { It t; t.load((const char*)p + i * ES); return t.get(0); };
  for (int64_t row = blockIdx.x; row < A.T; row += gridDim.x) {
    const float m2 = A.rms ? 0.f : A.mean[row], r2 = A.rstd[row];
    const float m1 = post && !A.rms ? A.post_mean[row] : 0.f, r1 = post ? A.post_rstd[row] : 1.f;
    const float gt = A.token_gate ? A.token_gate[row] : 1.f;
    float v[3] = {0.f, 0.f, 0.f}, t[3] = {0.f, 0.f, 0.f};
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float d = at(A.dy, row * A.ld_dy + c), xh = (at(A.sum, row * A.ld_sum + c) - m2) * r2, g = d * param(A.weight, c, A.param_bf16);
      v[0] += g;
      v[1] = fmaf(g, xh, v[1]);
      l_w2[c] = fmaf(d, xh, l_w2[c]);
      if (bias) l_b2[c] += d;
    }
    block_sums<3>(v, sh, slot);
    const float a1 = A.rms ? 0.f : v[0] * inv_h, a2 = v[1] * inv_h;
    // gs of a column; dresidual and dx may lie where dy, dsum, x or sum do, so both are written in the last pass only
    auto gs_at = [&](int64_t c) {
      const float xh = (at(A.sum, row * A.ld_sum + c) - m2) * r2;
      return fmaf(r2, fmaf(-xh, a2, fmaf(at(A.dy, row * A.ld_dy + c), param(A.weight, c, A.param_bf16), -a1)),
                  A.dsum ? at(A.dsum, row * A.ld_dsum + c) : 0.f);
    };
    if (use_x) {
      for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
        const float g = gs_at(c), xv = at(A.x, row * A.ld_x + c), xh1 = (xv - m1) * r1;
        float w1, b1, gc;
        params<1>(A.post_weight, c, A.param_bf16, 1.f, &w1);
        params<1>(A.post_bias, c, A.param_bf16, 0.f, &b1);
        params<1>(A.gate, c, A.param_bf16, 1.f, &gc);
        const float u = post ? fmaf(xh1, w1, b1) : xv, gu = A.scale * g * u, du = A.scale * gt * gc * g;
        if (A.gate) l_g[c] = fmaf(gt, gu, l_g[c]);
        t[2] = fmaf(gc, gu, t[2]);
        if (post) {
          t[0] += du * w1;
          t[1] = fmaf(du * w1, xh1, t[1]);
          l_w1[c] = fmaf(du, xh1, l_w1[c]);
          if (bias) l_b1[c] += du;
        }
      }
      block_sums<3>(t, sh, slot);
      if (A.token_gate && threadIdx.x == 0) A.dtoken_gate[row] = t[2];
    }
    const float c1 = A.rms ? 0.f : t[0] * inv_h, c2 = t[1] * inv_h;
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float g = gs_at(c);
      float w1, gc;
      params<1>(A.post_weight, c, A.param_bf16, 1.f, &w1);
      params<1>(A.gate, c, A.param_bf16, 1.f, &gc);
      const float du = A.scale * gt * gc * g;
      const float o = post ? r1 * fmaf(-(at(A.x, row * A.ld_x + c) - m1) * r1, c2, fmaf(du, w1, -c1)) : du;
      It d;
      d.set(&g);
      d.store((char*)A.dresidual + (row * A.ld_dresidual + c) * ES);
      d.set(&o);
      d.store((char*)A.dx + (row * A.ld_dx + c) * ES);
    }
  }
}

struct Outputs { float* p[kMaxSums]; };

// Column sums of the blocks' lines, in a fixed order: 32 threads a column, each every 32nd line, then their sums.
__global__ void __launch_bounds__(1024) block_lines_kernel(const float* partial, int64_t lines, int64_t H, int n, Outputs out) {
  __shared__ float sh[32][33];
  const int which = blockIdx.y;
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float s = 0.f;
  if (c < H) {
    const float* p = partial + ((int64_t)threadIdx.y * n + which) * H + c;
#pragma unroll 8
    for (int64_t g = threadIdx.y; g < lines; g += 32, p += 32 * n * H) s += *p;
  }
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  const float v = warp_sum(sh[threadIdx.x][threadIdx.y]);   // warp y has column y of the block
  const int64_t o = (int64_t)blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && o < H) out.p[which][o] = v;
}

// Threads a row (a block) and accesses a thread.
struct Plan {
  int w;          // elements an access: a 16-byte vector, or 1
  int nv;         // accesses a thread; 0: the kernels for any width
  int threads;
};

bool vectors(const BlockArgs& a, bool backward) {
  const int64_t es = a.dtype == JP_BF16 ? 2 : 4;
  uintptr_t bits = (uintptr_t)a.x | (uintptr_t)a.sum | (uintptr_t)a.post_weight | (uintptr_t)a.post_bias | (uintptr_t)a.gate | (uintptr_t)a.weight | (uintptr_t)a.bias;
  int64_t pitch = (a.x ? a.ld_x : 0) | a.ld_sum;
  if (backward) {
    bits |= (uintptr_t)a.dy | (uintptr_t)a.dsum | (uintptr_t)a.dx | (uintptr_t)a.dresidual;
    pitch |= a.ld_dy | (a.dsum ? a.ld_dsum : 0) | a.ld_dx | a.ld_dresidual;
  } else {
    bits |= (uintptr_t)a.residual | (uintptr_t)a.y;
    pitch |= a.ld_residual | a.ld_y;
  }
  return a.H * es % 16 == 0 && pitch * es % 16 == 0 && (bits & 15) == 0;
}

Plan plan_for(int64_t H, int dtype, bool vec, bool backward) {
  Plan p{};
  const int vw = dtype == JP_BF16 ? 8 : 4, most = backward ? 512 : 1024;
  p.w = vec ? vw : 1;
  const int64_t n = (H + p.w - 1) / p.w;
  p.nv = 0;
  if (vec) {
    for (int nv = 1; nv <= 16 / vw; nv *= 2)
      if (n <= (int64_t)nv * most) { p.nv = nv; break; }
  } else {
    p.nv = n <= 8 * most ? 8 : n <= 16 * most ? 16 : 0;
  }
  if (p.nv == 0) return {1, 0, 1024};
  p.threads = (int)(((n + p.nv - 1) / p.nv + 31) / 32 * 32);
  return p;
}

// Blocks: what an SM holds of 1024 threads (backward 512), at most 16 of them; fewer where rows are.
int grid_for(int64_t T, const Plan& p, int sms, bool backward) {
  int per = (backward && p.nv ? 512 : 1024) / p.threads;
  per = per > 16 ? 16 : per;
  const int64_t cap = (int64_t)sms * per;
  return (int)(T < cap ? T : cap);
}

template <class... P, class... Q>
cudaError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, cudaStream_t s, Q... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int DT> cudaError_t forward(const BlockArgs& a, cudaStream_t s, int sms) {
  constexpr int VW = Vec<DT>::N;
  const Plan p = plan_for(a.H, a.dtype, vectors(a, false), false);
  const dim3 g(grid_for(a.T, p, sms, false)), b(p.threads);
  if (p.nv == 0) {
    block_fwd_wide_kernel<DT><<<g, b, 0, s>>>(a);
    return cudaGetLastError();
  }
  if (p.w == 1) return p.nv == 8 ? launch(block_fwd_kernel<DT, 1, 8>, g, b, s, a) : launch(block_fwd_kernel<DT, 1, 16>, g, b, s, a);
  if (p.nv == 1) return launch(block_fwd_kernel<DT, VW, 1>, g, b, s, a);
  if (p.nv == 2) return launch(block_fwd_kernel<DT, VW, 2>, g, b, s, a);
  if constexpr (DT == JP_F32) return launch(block_fwd_kernel<DT, VW, 4>, g, b, s, a);
  return cudaErrorInvalidConfiguration;
}

template <int DT, bool POST, bool GATE, bool BIAS> cudaError_t backward(const BlockArgs& a, const Plan& p, dim3 g, cudaStream_t s) {
  constexpr int VW = Vec<DT>::N;
  const dim3 b(p.threads);
  if (p.w == 1) return p.nv == 8 ? launch(block_bwd_kernel<DT, 1, 8, POST, GATE, BIAS>, g, b, s, a) : launch(block_bwd_kernel<DT, 1, 16, POST, GATE, BIAS>, g, b, s, a);
  if (p.nv == 1) return launch(block_bwd_kernel<DT, VW, 1, POST, GATE, BIAS>, g, b, s, a);
  if (p.nv == 2) return launch(block_bwd_kernel<DT, VW, 2, POST, GATE, BIAS>, g, b, s, a);
  if constexpr (DT == JP_F32) return launch(block_bwd_kernel<DT, VW, 4, POST, GATE, BIAS>, g, b, s, a);
  return cudaErrorInvalidConfiguration;
}
template <int DT, bool POST, bool GATE> cudaError_t backward(const BlockArgs& a, const Plan& p, dim3 g, cudaStream_t s) {
  return a.with_bias ? backward<DT, POST, GATE, true>(a, p, g, s) : backward<DT, POST, GATE, false>(a, p, g, s);
}
template <int DT> cudaError_t backward(const BlockArgs& a, const Plan& p, dim3 g, int n_lines, cudaStream_t s) {
  if (p.nv == 0) {
    block_bwd_wide_kernel<DT><<<g, p.threads, 0, s>>>(a, n_lines);
    return cudaGetLastError();
  }
  if (a.post_weight) return a.gate ? backward<DT, true, true>(a, p, g, s) : backward<DT, true, false>(a, p, g, s);
  return a.gate ? backward<DT, false, true>(a, p, g, s) : backward<DT, false, false>(a, p, g, s);
}

}  // namespace

cudaError_t launch_block_forward(const BlockArgs& a, cudaStream_t s, int sms) {
  return a.dtype == JP_BF16 ? forward<JP_BF16>(a, s, sms) : forward<JP_F32>(a, s, sms);
}

// The lines a backward call can need, whatever the alignment of its pointers.
size_t block_workspace_bytes(int64_t T, int64_t H, int dtype, int sms) {
  int most = 0;
  for (const bool vec : {false, true}) {
    const int g = grid_for(T, plan_for(H, dtype, vec, true), sms, true);
    most = g > most ? g : most;
  }
  return (size_t)most * kMaxSums * (size_t)H * sizeof(float);
}

cudaError_t launch_block_backward(const BlockArgs& a, cudaStream_t s, int sms) {
  const Plan p = plan_for(a.H, a.dtype, vectors(a, true), true);
  const int grid = grid_for(a.T, p, sms, true);
  const bool post = a.post_weight != nullptr, gate = a.gate != nullptr;
  const int n = n_sums(post, gate, a.with_bias);
  const cudaError_t e = a.dtype == JP_BF16 ? backward<JP_BF16>(a, p, dim3(grid), n, s) : backward<JP_F32>(a, p, dim3(grid), n, s);
  if (e != cudaSuccess) return e;
  Outputs out{};
  int k = 0;
  out.p[k++] = a.dweight;
  if (a.with_bias) out.p[k++] = a.dbias;
  if (post) out.p[k++] = a.dpost_weight;
  if (post && a.with_bias) out.p[k++] = a.dpost_bias;
  if (gate) out.p[k++] = a.dgate;
  return launch(block_lines_kernel, dim3((unsigned)((a.H + 31) / 32), n), dim3(32, 32), s, (const float*)a.partial, (int64_t)grid, a.H, n, out);
}

}  // namespace jp
