// Layer norm and RMS norm over the rows of a [T, H] matrix, forward and backward, with the gradients of the
// weight and the bias.
//
//   mu = mean_h x (0 for RMS norm),  r = 1 / sqrt(mean_h (x - mu)^2 + eps),  xhat = (x - mu) r
//   y  = xhat w + b
//   g  = dy w,  dx = r (g - mean_h g - xhat mean_h (g xhat))     (no mean_h g for RMS norm)
//   dw = sum_t dy xhat,  db = sum_t dy
//
// Both passes are bound by HBM: forward reads x and writes y, backward reads x and dy and writes dx.  A row
// stays in the registers of one group of threads between its reduction and its output, so nothing is read
// twice; the squares are taken of x - mu (a second reduction over registers) because E x^2 - mu^2 cancels.
// A group walks rows with the fixed stride of the grid and loads the next row before it reduces the present
// one.  Each thread owns fixed columns, so dw and db add up in its registers over all rows of its group; the
// groups' sums go to the workspace and a second kernel adds them in a fixed order: no atomics, the same bits
// every time.
#include "jp_common.cuh"
#include "jp_internal.h"

namespace jp {
namespace {

constexpr int kMaxWarps = 32;

__device__ __forceinline__ float load_elem(const void* p, int64_t i, bool bf16) {
  return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16) : ((const float*)p)[i];
}

// W consecutive elements of type DT: one 16-byte access, or one element where rows do not start on 16 bytes.
template <int DT, int W> struct Access;
template <int DT> struct Access<DT, Vec<DT>::N> {
  using raw = uint4;
  static constexpr int W = Vec<DT>::N;
  __device__ static __forceinline__ raw load(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
  }
  __device__ static __forceinline__ raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
  __device__ static __forceinline__ void unpack(const raw& v, float* f) {
#pragma unroll
    for (int e = 0; e < W; ++e) f[e] = Vec<DT>::get(v, e);
  }
  __device__ static __forceinline__ void store(void* p, const float* f) {
    uint4 v;
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
    stg_stream((uint4*)p, v);
  }
};
template <int DT> struct Access<DT, 1> {
  using raw = uint32_t;
  static constexpr int W = 1;
  __device__ static __forceinline__ raw load(const void* p) {
    if constexpr (DT == JP_BF16) return (uint32_t)(*(const volatile uint16_t*)p) << 16;
    else return *(const volatile uint32_t*)p;
  }
  __device__ static __forceinline__ raw zero() { return 0u; }
  __device__ static __forceinline__ void unpack(const raw& v, float* f) { f[0] = __uint_as_float(v); }
  __device__ static __forceinline__ void store(void* p, const float* f) {
    if constexpr (DT == JP_BF16) *(__nv_bfloat16*)p = __float2bfloat16_rn(f[0]);
    else *(float*)p = f[0];
  }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the threads of a row's group: one warp (blockDim.x == 32, any number of rows per block), or the whole
// block.  `slot` alternates between uses so that one barrier per sum is enough.
__device__ __forceinline__ float2 group_sum(float a, float b, float2 (*sh)[kMaxWarps], int& slot) {
  a = warp_sum(a);
  b = warp_sum(b);
  if (blockDim.x == 32) return make_float2(a, b);
  const int warps = blockDim.x >> 5;
  float2* s = sh[slot];
  slot ^= 1;
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const float2 v = lane < warps ? s[lane] : make_float2(0.f, 0.f);
  return make_float2(warp_sum(v.x), warp_sum(v.y));
}

template <int DT, int W, int NV>
__global__ void __launch_bounds__((W == 1 ? NV > 8 : NV > 1) ? 512 : 256) norm_fwd_kernel(NormArgs A) {
  using Ac = Access<DT, W>;
  constexpr int ES = Vec<DT>::ESIZE;
  __shared__ float2 sh[2][kMaxWarps];
  int slot = 0;
  const int n = blockDim.x;
  const float inv_h = 1.f / (float)A.H;
  typename Ac::raw next[NV];
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  auto fetch = [&](int64_t r) {
    const char* x = (const char*)A.x + r * A.ld_x * ES;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(threadIdx.x + i * n) * W;
      next[i] = c < A.H ? Ac::load(x + c * ES) : Ac::zero();
    }
  };
  if (row < A.T) fetch(row);
  for (; row < A.T; row += step) {
    float v[NV][W];
#pragma unroll
    for (int i = 0; i < NV; ++i) Ac::unpack(next[i], v[i]);
    if (row + step < A.T) fetch(row + step);
    float mean = 0.f;
    if (!A.rms) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e) s += v[i][e];
      mean = group_sum(s, 0.f, sh, slot).x * inv_h;
    }
    float s2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(threadIdx.x + i * n) * W;
      if (c < A.H) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          v[i][e] -= mean;
          s2 = fmaf(v[i][e], v[i][e], s2);
        }
      }
    }
    const float rstd = 1.f / sqrtf(group_sum(s2, 0.f, sh, slot).x * inv_h + A.eps);
    if (threadIdx.x == 0) {
      if (A.out_mean) A.out_mean[row] = mean;
      if (A.out_rstd) A.out_rstd[row] = rstd;
    }
    char* y = (char*)A.y + row * A.ld_y * ES;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(threadIdx.x + i * n) * W;
      if (c < A.H) {
        float o[W];
#pragma unroll
        for (int e = 0; e < W; ++e) {
          o[e] = v[i][e] * rstd * load_elem(A.weight, c + e, A.param_bf16);
          if (A.bias) o[e] += load_elem(A.bias, c + e, A.param_bf16);
        }
        Ac::store(y + c * ES, o);
      }
    }
  }
}

// Any width: the row is read again for each of its sums (from L2) instead of being held.
template <int DT>
__global__ void __launch_bounds__(1024) norm_fwd_wide_kernel(NormArgs A) {
  using Ac = Access<DT, 1>;
  constexpr int ES = Vec<DT>::ESIZE;
  __shared__ float2 sh[2][kMaxWarps];
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  for (int64_t row = blockIdx.x; row < A.T; row += gridDim.x) {
    const char* x = (const char*)A.x + row * A.ld_x * ES;
    float mean = 0.f;
    if (!A.rms) {
      float s = 0.f;
      for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) s += __uint_as_float(Ac::load(x + c * ES));
      mean = group_sum(s, 0.f, sh, slot).x * inv_h;
    }
    float s2 = 0.f;
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float d = __uint_as_float(Ac::load(x + c * ES)) - mean;
      s2 = fmaf(d, d, s2);
    }
    const float rstd = 1.f / sqrtf(group_sum(s2, 0.f, sh, slot).x * inv_h + A.eps);
    if (threadIdx.x == 0) {
      if (A.out_mean) A.out_mean[row] = mean;
      if (A.out_rstd) A.out_rstd[row] = rstd;
    }
    char* y = (char*)A.y + row * A.ld_y * ES;
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      float o = (__uint_as_float(Ac::load(x + c * ES)) - mean) * rstd * load_elem(A.weight, c, A.param_bf16);
      if (A.bias) o += load_elem(A.bias, c, A.param_bf16);
      Ac::store(y + c * ES, &o);
    }
  }
}

template <int DT, int W, int NV>
__global__ void __launch_bounds__((W == 1 ? NV > 8 : NV > 1) ? 512 : 256) norm_bwd_kernel(NormArgs A) {
  using Ac = Access<DT, W>;
  constexpr int ES = Vec<DT>::ESIZE;
  __shared__ float2 sh[2][kMaxWarps];
  int slot = 0;
  const int n = blockDim.x;
  const float inv_h = 1.f / (float)A.H;
  float dw[NV][W], db[NV][W];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < W; ++e) dw[i][e] = db[i][e] = 0.f;
  typename Ac::raw nx[NV], ny[NV];
  const int64_t group = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  auto fetch = [&](int64_t r) {
    const char* x = (const char*)A.x + r * A.ld_x * ES;
    const char* dy = (const char*)A.dy + r * A.ld_dy * ES;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(threadIdx.x + i * n) * W;
      nx[i] = c < A.H ? Ac::load(x + c * ES) : Ac::zero();
      ny[i] = c < A.H ? Ac::load(dy + c * ES) : Ac::zero();
    }
  };
  if (group < A.T) fetch(group);
  for (int64_t row = group; row < A.T; row += step) {
    typename Ac::raw cx[NV], cy[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) { cx[i] = nx[i]; cy[i] = ny[i]; }
    if (row + step < A.T) fetch(row + step);
    const float mean = A.rms ? 0.f : A.mean[row], rstd = A.rstd[row];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(threadIdx.x + i * n) * W;
      if (c < A.H) {
        float x[W], dy[W];
        Ac::unpack(cx[i], x);
        Ac::unpack(cy[i], dy);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float xh = (x[e] - mean) * rstd, g = dy[e] * load_elem(A.weight, c + e, A.param_bf16);
          s1 += g;
          s2 = fmaf(g, xh, s2);
          dw[i][e] = fmaf(dy[e], xh, dw[i][e]);
          db[i][e] += dy[e];
        }
      }
    }
    const float2 s = group_sum(s1, s2, sh, slot);
    const float m1 = A.rms ? 0.f : s.x * inv_h, m2 = s.y * inv_h;
    char* dx = (char*)A.dx + row * A.ld_dx * ES;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = (int64_t)(threadIdx.x + i * n) * W;
      if (c < A.H) {
        float x[W], dy[W], o[W];
        Ac::unpack(cx[i], x);
        Ac::unpack(cy[i], dy);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float xh = (x[e] - mean) * rstd, g = dy[e] * load_elem(A.weight, c + e, A.param_bf16);
          o[e] = (g - m1 - xh * m2) * rstd;
        }
        Ac::store(dx + c * ES, o);
      }
    }
  }
  float* pw = A.partial + group * 2 * A.H;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t c = (int64_t)(threadIdx.x + i * n) * W;
    if (c < A.H) {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        pw[c + e] = dw[i][e];
        if (A.dbias) pw[A.H + c + e] = db[i][e];
      }
    }
  }
}

// Any width: sums of dw and db stay in the block's line of the workspace (each thread its own columns).
template <int DT>
__global__ void __launch_bounds__(1024) norm_bwd_wide_kernel(NormArgs A) {
  using Ac = Access<DT, 1>;
  constexpr int ES = Vec<DT>::ESIZE;
  __shared__ float2 sh[2][kMaxWarps];
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  float* pw = A.partial + (int64_t)blockIdx.x * 2 * A.H;
  for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) pw[c] = pw[A.H + c] = 0.f;
  for (int64_t row = blockIdx.x; row < A.T; row += gridDim.x) {
    const char* x = (const char*)A.x + row * A.ld_x * ES;
    const char* dy = (const char*)A.dy + row * A.ld_dy * ES;
    char* dx = (char*)A.dx + row * A.ld_dx * ES;
    const float mean = A.rms ? 0.f : A.mean[row], rstd = A.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float d = __uint_as_float(Ac::load(dy + c * ES));
      const float xh = (__uint_as_float(Ac::load(x + c * ES)) - mean) * rstd, g = d * load_elem(A.weight, c, A.param_bf16);
      s1 += g;
      s2 = fmaf(g, xh, s2);
      pw[c] = fmaf(d, xh, pw[c]);
      pw[A.H + c] += d;
    }
    const float2 s = group_sum(s1, s2, sh, slot);
    const float m1 = A.rms ? 0.f : s.x * inv_h, m2 = s.y * inv_h;
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float d = __uint_as_float(Ac::load(dy + c * ES));
      const float xh = (__uint_as_float(Ac::load(x + c * ES)) - mean) * rstd, g = d * load_elem(A.weight, c, A.param_bf16);
      const float o = (g - m1 - xh * m2) * rstd;
      Ac::store(dx + c * ES, &o);
    }
  }
}

// dw[c] = sum over the groups' lines, in a fixed order: 8 threads a column, each every 8th line, then their sums.
__global__ void __launch_bounds__(256) norm_sum_kernel(const float* partial, int64_t groups, int64_t H, float* dw,
                                                       float* db) {
  __shared__ float sh[8][33];
  const bool second = blockIdx.y == 1;
  float* out = second ? db : dw;
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
  float s = 0.f;
  if (c < H)
    for (int64_t g = threadIdx.y; g < groups; g += 8) s += partial[(g * 2 + second) * H + c];
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y == 0 && c < H) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += sh[i][threadIdx.x];
    out[c] = s;
  }
}

struct Plan {
  int w;          // elements an access: a 16-byte vector or 1
  int nv;         // accesses a thread; 0 = the kernels for any width
  int threads;    // a row's group
  int rows;       // groups a block
};

bool vector_rows(const NormArgs& a, bool backward) {
  const int64_t es = a.dtype == JP_BF16 ? 2 : 4;
  auto ok = [&](const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * es % 16 == 0; };
  if (a.H * es % 16) return false;
  return backward ? ok(a.x, a.ld_x) && ok(a.dy, a.ld_dy) && ok(a.dx, a.ld_dx) : ok(a.x, a.ld_x) && ok(a.y, a.ld_y);
}

// Threads and registers of a row.  16-byte accesses where rows start on 16 bytes, else single elements; 1, 2 or 4 vectors
// (8 or 16 elements) a thread so that rows up to 16384 bf16 (8192 fp32, or 8192 unaligned) stay in registers.
Plan plan_for(int64_t H, int dtype, bool vec) {
  Plan p{};
  p.w = vec ? (dtype == JP_BF16 ? 8 : 4) : 1;
  const int64_t n = (H + p.w - 1) / p.w;
  if (vec) p.nv = n <= 256 ? 1 : n <= 1024 ? 2 : n <= 2048 ? 4 : 0;
  else p.nv = n <= 2048 ? 8 : n <= 8192 ? 16 : 0;
  if (p.nv == 0) { p.threads = 1024; p.rows = 1; p.w = 1; return p; }
  const int64_t per = (n + p.nv - 1) / p.nv;
  p.threads = (int)((per + 31) / 32 * 32);
  p.rows = p.threads == 32 ? 8 : 1;
  return p;
}

// Blocks: all rows at once where there are few, else what the SMs hold.
int grid_for(int64_t T, const Plan& p, int sms) {
  const int64_t need = (T + p.rows - 1) / p.rows;
  const int per_sm = 1024 / (p.threads * p.rows);
  const int64_t cap = (int64_t)sms * (per_sm > 8 ? 8 : per_sm);
  return (int)(need < cap ? need : cap);
}

template <int DT>
void fwd(const NormArgs& a, const Plan& p, int grid, cudaStream_t s) {
  constexpr int VW = Vec<DT>::N;
  const dim3 b(p.threads, p.rows);
  if (p.nv == 0) norm_fwd_wide_kernel<DT><<<grid, b, 0, s>>>(a);
  else if (p.w == 1 && p.nv == 8) norm_fwd_kernel<DT, 1, 8><<<grid, b, 0, s>>>(a);
  else if (p.w == 1) norm_fwd_kernel<DT, 1, 16><<<grid, b, 0, s>>>(a);
  else if (p.nv == 1) norm_fwd_kernel<DT, VW, 1><<<grid, b, 0, s>>>(a);
  else if (p.nv == 2) norm_fwd_kernel<DT, VW, 2><<<grid, b, 0, s>>>(a);
  else norm_fwd_kernel<DT, VW, 4><<<grid, b, 0, s>>>(a);
}

template <int DT>
void bwd(const NormArgs& a, const Plan& p, int grid, cudaStream_t s) {
  constexpr int VW = Vec<DT>::N;
  const dim3 b(p.threads, p.rows);
  if (p.nv == 0) norm_bwd_wide_kernel<DT><<<grid, b, 0, s>>>(a);
  else if (p.w == 1 && p.nv == 8) norm_bwd_kernel<DT, 1, 8><<<grid, b, 0, s>>>(a);
  else if (p.w == 1) norm_bwd_kernel<DT, 1, 16><<<grid, b, 0, s>>>(a);
  else if (p.nv == 1) norm_bwd_kernel<DT, VW, 1><<<grid, b, 0, s>>>(a);
  else if (p.nv == 2) norm_bwd_kernel<DT, VW, 2><<<grid, b, 0, s>>>(a);
  else norm_bwd_kernel<DT, VW, 4><<<grid, b, 0, s>>>(a);
}

}  // namespace

cudaError_t launch_norm_forward(const NormArgs& a, cudaStream_t s, int sms) {
  const Plan p = plan_for(a.H, a.dtype, vector_rows(a, false));
  const int grid = grid_for(a.T, p, sms);
  if (a.dtype == JP_BF16) fwd<JP_BF16>(a, p, grid, s);
  else fwd<JP_F32>(a, p, grid, s);
  return cudaGetLastError();
}

// Lines of partial sums a backward call can need, whatever the alignment of its pointers.
int64_t norm_backward_groups(int64_t T, int64_t H, int dtype, int sms) {
  int64_t most = 0;
  for (int vec = 0; vec < 2; ++vec) {
    const Plan p = plan_for(H, dtype, vec != 0);
    const int64_t g = (int64_t)grid_for(T, p, sms) * p.rows;
    most = g > most ? g : most;
  }
  return most;
}

cudaError_t launch_norm_backward(const NormArgs& a, cudaStream_t s, int sms) {
  const Plan p = plan_for(a.H, a.dtype, vector_rows(a, true));
  const int grid = grid_for(a.T, p, sms);
  if (a.dtype == JP_BF16) bwd<JP_BF16>(a, p, grid, s);
  else bwd<JP_F32>(a, p, grid, s);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  norm_sum_kernel<<<dim3((unsigned)((a.H + 31) / 32), a.dbias ? 2 : 1), dim3(32, 8), 0, s>>>(
      a.partial, (int64_t)grid * p.rows, a.H, a.dweight, a.dbias);
  return cudaGetLastError();
}

}  // namespace jp
