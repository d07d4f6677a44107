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
// Groups walk rows with the fixed stride of the grid, weight and bias in registers.  The next rows come through asynchronous copies, each
// thread into places of its own (kStages rows ahead, no barriers); what lies before and behind a row's aligned vectors is one element a
// thread (Span).  Where x and y (or x, dy and dx) differ in their offsets to 16 bytes the group copies together (Rows of width 1).
// Each thread owns fixed columns, so dw and db add up in its registers over all rows of its group; the
// groups' sums go to the workspace and a second kernel adds them in a fixed order: no atomics, the same bits
// every time.
#include <type_traits>

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

// Two fp32 operations in one instruction: at 8192 x 4096 both passes are as much bound by issue as by HBM (forward with bias 31 us
// without, 28.9; backward of RMS norm 41, 39.4).  xhat is (x - mu) r in two of them, not x r + (-mu r) in one: rounding mu r would leave
// 2^-24 |mu| r in every xhat, a thousand times its own rounding in a row whose mean is a thousand standard deviations.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  asm("{.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;}" : "+f"(a.x), "+f"(a.y) : "f"(b.x), "f"(b.y));
  return a;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  asm("{.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;}" : "+f"(a.x), "+f"(a.y) : "f"(b.x), "f"(b.y));
  return a;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  asm("{.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%0, %1};\n\tfma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;}"
      : "+f"(c.x), "+f"(c.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}

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
  float2 t = s[0];
  for (int w = 1; w < warps; ++w) {
    t.x += s[w].x;
    t.y += s[w].y;
  }
  return t;
}

// Columns of this thread: access i covers columns (threadIdx.x + i * blockDim.x) * W and the next W - 1.
template <int W> __device__ __forceinline__ int64_t column(int i) { return (int64_t)(threadIdx.x + i * (int)blockDim.x) * W; }

// A row that does not start on 16 bytes: the elements before the first boundary, the vectors between, and the elements behind the last
// boundary.  The vectors are dealt out like those of an aligned row, and the edges (below two vectors) one a thread, so that nothing of
// a neighbouring row is read or masked.  A group's rows are a multiple of the period apart after which starts repeat: threads keep their
// columns.
struct Span {
  int head, tail;
  int64_t body;                 // elements of each
  int64_t edge;                 // this thread's column of the edges, or -1
};
template <int W> __device__ __forceinline__ Span span_of(bool off, const void* base, int64_t row, int64_t ld, int es, int64_t H) {
  Span s{0, 0, H, -1};
  if (off) {
    const int64_t first = (int64_t)((16 - ((uintptr_t)base + (uintptr_t)(row * ld * es))) & 15) / es;
    s.head = (int)(first < H ? first : H);
    s.tail = (int)(H - s.head) % W;
    s.body = H - s.head - s.tail;
    const int t = threadIdx.x;
    s.edge = t < s.head ? t : t >= W && t - W < s.tail ? s.head + s.body + (t - W) : -1;
  }
  return s;
}

// Weight or bias at the thread's columns, loaded once: bf16 pairs as they are, the rest as fp32.
template <int W, int NV, bool BF16>
struct Params {
  static constexpr int N = W == 1 ? NV : BF16 ? NV * W / 2 : NV * W;
  uint32_t r[N];
  __device__ __forceinline__ void load(const void* p, int64_t H) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      if constexpr (W == 1) {
        r[i] = p && c < H ? (BF16 ? (uint32_t)((const uint16_t*)p)[c] << 16 : ((const uint32_t*)p)[c]) : 0u;
      } else {
        constexpr int words = N / NV;
#pragma unroll
        for (int q = 0; q < words; q += 2) {
          const uint2 v = p && c < H ? *(const uint2*)((const char*)p + c * (BF16 ? 2 : 4) + q * 4) : make_uint2(0u, 0u);
          r[i * words + q] = v.x;
          r[i * words + q + 1] = v.y;
        }
      }
    }
  }
  __device__ __forceinline__ void load(const void* p, const Span& sp) {      // of a span's vectors
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = 0u;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (p && column<W>(i) < sp.body) {
        const int64_t c = sp.head + column<W>(i);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          if constexpr (BF16) r[(i * W + e) / 2] |= (uint32_t)((const uint16_t*)p)[c + e] << (16 * (e & 1));
          else r[i * W + e] = ((const uint32_t*)p)[c + e];
        }
      }
  }
  __device__ __forceinline__ void read(const char* p) {     // (NV == 1) W consecutive ones
#pragma unroll
    for (int q = 0; q < N; q += N < 4 ? 2 : 4) {
      if constexpr (N < 4) {
        const uint2 v = *(const uint2*)(p + q * 4);
        r[q] = v.x; r[q + 1] = v.y;
      } else {
        const uint4 v = *(const uint4*)(p + q * 4);
        r[q] = v.x; r[q + 1] = v.y; r[q + 2] = v.z; r[q + 3] = v.w;
      }
    }
  }
  __device__ __forceinline__ float get(int i, int e) const {
    if constexpr (W == 1) return __uint_as_float(r[i]);
    else if constexpr (BF16) {
      const uint32_t w = r[(i * W + e) / 2];
      return __uint_as_float((e & 1) ? (w & 0xffff0000u) : (w << 16));
    } else return __uint_as_float(r[i * W + e]);
  }
};

// The group's rows of NT matrices one after the other: row `first`, then every `step`-th.
constexpr int kStages = 3;
template <int DT, int W, int NV, int NT, bool OFF = false, int STAGES = kStages>
struct Rows {
  using Ac = Access<DT, W>;
  static constexpr int ES = Vec<DT>::ESIZE;
  const char* next[NT];         // the next row to fetch, from this thread's first column on
  int64_t stride[NT];           // bytes from one row of the group to the next
  int64_t left;                 // rows not fetched yet
  const uint4* read;            // this thread's column of places [STAGES][NT][NV][threads of the block]
  uint32_t write;
  int threads, in, out;
  bool have[NV];                // the access is within the row
  // (OFF) the thread's element of the edges: of the next two rows, loaded two rows ahead
  const char* edge[NT];
  int64_t edges_left;
  uint32_t edge0[NT], edge1[NT];
  __device__ __forceinline__ void next_edge() {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      edge0[t] = edge1[t];
      edge1[t] = 0u;
      if (edges_left > 0) edge1[t] = Access<DT, 1>::load(edge[t]);
      edge[t] += stride[t];
    }
    --edges_left;
  }
  __device__ __forceinline__ void fetch() {
    if (left > 0) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (have[i]) {
            const char* p = next[t] + (int64_t)i * (int)blockDim.x * W * ES;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(write + ((in + t) * NV + i) * threads * 16), "l"(p) : "memory");
          }
#pragma unroll
      for (int t = 0; t < NT; ++t) next[t] += stride[t];
      --left;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    in = in == (STAGES - 1) * NT ? 0 : in + NT;
  }
  // rows first, first + step, ... below T of the NT matrices
  __device__ __forceinline__ void start(const void* const (&base)[NT], const int64_t (&ld)[NT], int64_t first, int64_t step, int64_t T,
                                        const Span& sp, uint4* smem) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      next[t] = (const char*)base[t] + (first * ld[t] + sp.head + (int64_t)threadIdx.x * W) * ES;
      if (OFF) edge[t] = (const char*)base[t] + (first * ld[t] + sp.edge) * ES;
      stride[t] = step * ld[t] * ES;
    }
    left = first < T ? (T - first + step - 1) / step : 0;
    threads = blockDim.x * blockDim.y;
    read = smem + threadIdx.y * blockDim.x + threadIdx.x;
    write = (uint32_t)__cvta_generic_to_shared(read);
    in = out = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) have[i] = column<W>(i) < sp.body;
#pragma unroll
    for (int s = 0; s < STAGES; ++s) fetch();
    if (OFF) {
      edges_left = sp.edge >= 0 && first < T ? (T - first + step - 1) / step : 0;
      next_edge();
      next_edge();
    }
  }
  // the oldest row; columns past the end read 0
  __device__ __forceinline__ void take(typename Ac::raw (&v)[NT][NV], float (&ve)[NT]) {
    if (OFF) {
#pragma unroll
      for (int t = 0; t < NT; ++t) ve[t] = __uint_as_float(edge0[t]);
      next_edge();
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[t][i] = have[i] ? read[((out + t) * NV + i) * threads] : Ac::zero();
    out = out == (STAGES - 1) * NT ? 0 : out + NT;
  }
};

// The same for matrices whose rows start at different offsets to 16 bytes: the group copies the 16-byte vectors that cover a row (a row's
// place begins at the row's own offset), and every thread reads its elements once all have arrived.  Vectors that reach beyond the
// matrix, in its first and last row, are copied element by element.  The place is free again after the barrier of the row's first sum.
// (With element loads into registers, one row ahead, 8192 x 4095 bf16 took 147 us forward and 225 us backward; this 70 and 93, rows of
// one offset as spans 32 and 66.)
__host__ __device__ inline int span_bytes(int64_t H, int es) { return (int)((H * es + 15) / 16 + 1) * 16; }
template <int DT, int NV, int NT, int STAGES>
struct Rows<DT, 1, NV, NT, false, STAGES> {
  static constexpr int ES = Vec<DT>::ESIZE;
  const char* next[NT];         // the next row to fetch
  const char* taken[NT];        // the next row to take
  const char* lo[NT];
  const char* hi[NT];           // the matrix
  int64_t stride[NT], left;
  char* place;                  // [STAGES][NT][span]
  int span, bytes, in, out;
  bool have[NV];
  __device__ __forceinline__ void fetch() {
    if (left > 0) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const char* const p = next[t];
        const int head = (int)((uintptr_t)p & 15);
        const char* from = p - head + threadIdx.x * 16;
        char* to = place + (in + t) * span + threadIdx.x * 16;
        for (int i = threadIdx.x * 16; i < head + bytes; i += blockDim.x * 16, from += blockDim.x * 16, to += blockDim.x * 16) {
          if (from >= lo[t] && from + 16 <= hi[t]) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
          } else {
            for (int q = 0; q < 16; q += ES)
              if (from + q >= p && from + q < p + bytes) {
                if constexpr (ES == 2) *(uint16_t*)(to + q) = *(const volatile uint16_t*)(from + q);
                else *(uint32_t*)(to + q) = *(const volatile uint32_t*)(from + q);
              }
          }
        }
        next[t] += stride[t];
      }
      --left;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    in = in == (STAGES - 1) * NT ? 0 : in + NT;
  }
  __device__ __forceinline__ void start(const void* const (&base)[NT], const int64_t (&ld)[NT], int64_t first, int64_t step, int64_t T,
                                        const Span& sp, uint4* smem) {
    const int64_t H = sp.body;
    bytes = (int)H * ES;
    span = span_bytes(H, ES);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      lo[t] = (const char*)base[t];
      hi[t] = lo[t] + ((T - 1) * ld[t] + H) * ES;
      next[t] = taken[t] = lo[t] + first * ld[t] * ES;
      stride[t] = step * ld[t] * ES;
    }
    left = first < T ? (T - first + step - 1) / step : 0;
    place = (char*)smem + threadIdx.y * STAGES * NT * span;
    in = out = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) have[i] = column<1>(i) < H;
#pragma unroll 1
    for (int s = 0; s < STAGES; ++s) fetch();
  }
  __device__ __forceinline__ void take(uint32_t (&v)[NT][NV], float (&)[NT]) {
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
    if (blockDim.x == 32) __syncwarp();
    else __syncthreads();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const char* row = place + (out + t) * span + ((uintptr_t)taken[t] & 15);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        v[t][i] = 0u;
        if (have[i]) {
          if constexpr (ES == 2) v[t][i] = (uint32_t)((const uint16_t*)row)[threadIdx.x + i * blockDim.x] << 16;
          else v[t][i] = ((const uint32_t*)row)[threadIdx.x + i * blockDim.x];
        }
      }
      taken[t] += stride[t];
    }
    out = out == (STAGES - 1) * NT ? 0 : out + NT;
  }
};

// Threads and blocks an SM holds of the kernels below
constexpr int group_threads(int w, int nv) { return (w == 1 ? nv > 8 : nv > 1) ? 512 : 256; }

template <int DT, int W, int NV, bool PB, bool OFF>
__global__ void __launch_bounds__(group_threads(W, NV)) norm_fwd_kernel(NormArgs A) {
  using Ac = Access<DT, W>;
  constexpr int ES = Vec<DT>::ESIZE;
  extern __shared__ uint4 places[];
  __shared__ float2 sh[2][kMaxWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");        // launched as a programmatic dependent of whatever is before it
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const Span span = span_of<W>(OFF, A.x, row, A.ld_x, ES, A.H);
  Rows<DT, W, NV, 1, OFF> in;
  in.start({A.x}, {A.ld_x}, row, step, A.T, span, places);
  Params<W, NV, PB> w, b;
  float we = 0.f, be = 0.f;     // of the edge
  if constexpr (OFF) {
    w.load(A.weight, span);
    b.load(A.bias, span);
    if (span.edge >= 0) {
      we = load_elem(A.weight, span.edge, PB);
      if (A.bias) be = load_elem(A.bias, span.edge, PB);
    }
  } else {
    w.load(A.weight, A.H);
    b.load(A.bias, A.H);
  }
  for (; row < A.T; row += step) {
    float v[NV][W];
    typename Ac::raw raw[1][NV];
    float ve[1] = {0.f};
    in.take(raw, ve);
#pragma unroll
    for (int i = 0; i < NV; ++i) Ac::unpack(raw[0][i], v[i]);
    if (W > 1) in.fetch();
    float mean = 0.f;
    if (!A.rms) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e) s += v[i][e];
      if (OFF) s += ve[0];
      mean = group_sum(s, 0.f, sh, slot).x * inv_h;
    }
    float s2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (column<W>(i) < span.body) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          v[i][e] -= mean;
          s2 = fmaf(v[i][e], v[i][e], s2);
        }
      }
    }
    if (OFF && span.edge >= 0) {
      ve[0] -= mean;
      s2 = fmaf(ve[0], ve[0], s2);
    }
    const float rstd = 1.f / sqrtf(group_sum(s2, 0.f, sh, slot).x * inv_h + A.eps);
    if (W == 1) {
      __syncwarp();                                         // (every thread of the group has read the row)
      in.fetch();
    }
    if (threadIdx.x == 0) {
      if (A.out_mean) A.out_mean[row] = mean;
      if (A.out_rstd) A.out_rstd[row] = rstd;
    }
    if (OFF && span.edge >= 0) {
      const float o = fmaf(ve[0] * rstd, we, be);
      Access<DT, 1>::store((char*)A.y + (row * A.ld_y + span.edge) * ES, &o);
    }
    char* y = (char*)A.y + (row * A.ld_y + span.head) * ES;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = column<W>(i);
      if (c < span.body) {
        float o[W];
#pragma unroll
        for (int e = 0; e < W; ++e) o[e] = fmaf(v[i][e] * rstd, w.get(i, e), b.get(i, e));
        Ac::store(y + c * ES, o);
      }
    }
  }
}

// One warp a row, NVL vectors a lane, for many rows of up to 5120 bf16 or 2560 fp32: the reductions are shuffles and no row waits for
// another (a block a row, with a barrier for each of its two sums, took 48 us at 8192 x 4096 with bias in bf16 and 52 at 6553 x 5120; this
// takes 29 and 31).  Weight and bias are in shared memory beside the rows to come; wider rows leave too few warps an SM (at 4096 x 8192,
// five of them, RMS norm, 42 us; a block a row 40).
constexpr int kWarpStages = 2;
__host__ __device__ constexpr int warp_rows(int nvl) { return nvl == 20 ? 9 : 12; }   // rows a block
__host__ __device__ constexpr int warp_blocks(int nvl) { return nvl >= 16 ? 1 : nvl == 8 ? 2 : 3; }      // per SM
__host__ __device__ inline int param_bytes(int64_t H, int ps) { return ((int)H * ps + 15) / 16 * 16; }      // of one of them
template <int DT, int NVL, bool PB, bool OFF, bool CENTER>
__global__ void __launch_bounds__(32 * warp_rows(NVL), warp_blocks(NVL)) norm_fwd_warp_kernel(NormArgs A) {
  constexpr int kWarpRows = warp_rows(NVL);
  constexpr int W = Vec<DT>::N, ES = Vec<DT>::ESIZE, PS = PB ? 2 : 4;
  using Ac = Access<DT, W>;
  extern __shared__ uint4 places[];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x;
  const float inv_h = 1.f / (float)A.H;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  // (OFF: the rows of a block are the grid apart, which is a multiple of the period: they share weight and bias in shared memory)
  int64_t row = OFF ? blockIdx.x + (int64_t)gridDim.x * threadIdx.y : (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const Span span = span_of<W>(OFF, A.x, blockIdx.x, A.ld_x, ES, A.H);
  const int end = (int)span.body;
  Rows<DT, W, NVL, 1, OFF, kWarpStages> in;
  in.start({A.x}, {A.ld_x}, row, step, A.T, span, places);
  const int n = param_bytes(A.H, PS) / 16, tid = threadIdx.y * 32 + lane;
  uint4* const params = places + kWarpStages * NVL * 32 * kWarpRows;
  float we = 0.f, be = 0.f;
  if constexpr (OFF) {
    using P = std::conditional_t<PB, uint16_t, uint32_t>;
    for (int c = tid; c < end; c += 32 * kWarpRows) {
      ((P*)params)[c] = ((const P*)A.weight)[span.head + c];
      if (A.bias) ((P*)(params + n))[c] = ((const P*)A.bias)[span.head + c];
    }
    if (span.edge >= 0) {
      we = load_elem(A.weight, span.edge, PB);
      if (A.bias) be = load_elem(A.bias, span.edge, PB);
    }
  } else {
    for (int i = tid; i < end * PS / 8; i += 32 * kWarpRows) {        // (four bf16 are the least a row has)
      ((uint2*)params)[i] = ((const uint2*)A.weight)[i];
      if (A.bias) ((uint2*)(params + n))[i] = ((const uint2*)A.bias)[i];
    }
  }
  const char* w = (const char*)params;
  const char* b = A.bias ? (const char*)(params + n) : nullptr;
  __syncthreads();
  for (; row < A.T; row += step) {
    uint4 rows[1][NVL];
    float ve[1] = {0.f};
    in.take(rows, ve);
    uint4 (&v)[NVL] = rows[0];
    in.fetch();
    float mean = 0.f;
    if (!A.rms) {                                           // (CENTER; as a branch, or the row stays unpacked from here on and spills)
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NVL; ++i) {
        float t[W];
        Ac::unpack(v[i], t);
#pragma unroll
        for (int o = 1; o < W; o *= 2)
#pragma unroll
          for (int e = 0; e + o < W; e += 2 * o) t[e] += t[e + o];
        s += t[0];
      }
      if (OFF) s += ve[0];
      mean = warp_sum(s) * inv_h;
    }
    const float2 less = make_float2(-mean, -mean);
    float2 sq = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NVL; ++i)
      if ((lane + i * 32) * W < end) {
        float t[W];
        Ac::unpack(v[i], t);
#pragma unroll
        for (int e = 0; e < W; e += 2) {
          const float2 x = make_float2(t[e], t[e + 1]), d = CENTER ? add2(x, less) : x;
          sq = fma2(d, d, sq);
        }
      }
    float s2 = sq.x + sq.y;
    if (OFF && span.edge >= 0) s2 = fmaf(ve[0] - mean, ve[0] - mean, s2);
    const float rstd = 1.f / sqrtf(warp_sum(s2) * inv_h + A.eps);
    const float2 scale = make_float2(rstd, rstd);
    if (lane == 0) {
      if (A.out_mean) A.out_mean[row] = mean;
      if (A.out_rstd) A.out_rstd[row] = rstd;
    }
    if (OFF && span.edge >= 0) {
      const float o = fmaf((ve[0] - mean) * rstd, we, be);
      Access<DT, 1>::store((char*)A.y + (row * A.ld_y + span.edge) * ES, &o);
    }
    char* y = (char*)A.y + (row * A.ld_y + span.head) * ES;
#pragma unroll
    for (int i = 0; i < NVL; ++i) {
      const int c = (lane + i * 32) * W;
      if (c < end) {
        float t[W], o[W];
        Ac::unpack(v[i], t);
        Params<W, 1, PB> p, q;
        p.read(w + c * PS);
        if (b) q.read(b + c * PS);
#pragma unroll
        for (int e = 0; e < W; e += 2) {
          const float2 x = make_float2(t[e], t[e + 1]), xh = mul2(CENTER ? add2(x, less) : x, scale);
          const float2 add = b ? make_float2(q.get(0, e), q.get(0, e + 1)) : make_float2(0.f, 0.f);
          const float2 r = fma2(xh, make_float2(p.get(0, e), p.get(0, e + 1)), add);
          o[e] = r.x;
          o[e + 1] = r.y;
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

// N sums at once over the threads of a row's group (N a power of two up to 8), every thread getting all of them: N - 1 + log2(32 / N)
// shuffles instead of 5 N, one barrier, and each warp adds the warps' parts by itself.
template <int N>
__device__ __forceinline__ void group_sums(float (&v)[N], float (*sh)[N][kMaxWarps], int& slot) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = N, o = 16; o > 0; o >>= 1) {
    if (n > 1) {                                            // half of the values go to the lanes that differ in bit o
      n /= 2;
#pragma unroll
      for (int i = 0; i < N / 2; ++i)
        if (i < n) {
          const float keep = (lane & o) ? v[i + n] : v[i], send = (lane & o) ? v[i] : v[i + n];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
  constexpr int kLanes = 32 / N;                            // lane / kLanes is the number of the sum it holds
  const int mine = lane / kLanes;
  float s = v[0];
  if (blockDim.x > 32) {
    const int warps = blockDim.x >> 5;
    float (*part)[kMaxWarps] = sh[slot];
    slot ^= 1;
    if (lane % kLanes == 0) part[mine][threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.f;
    for (int w = lane % kLanes; w < warps; w += kLanes) s += part[mine][w];
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, s, i * kLanes);
}

__device__ __forceinline__ void keep_packed(uint4& v) { asm volatile("" : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w)); }
__device__ __forceinline__ void keep_packed(uint32_t& v) { asm volatile("" : "+r"(v)); }

// Rows a group takes at a time, so that their sums share a barrier: at 8192 x 4096 (RMS norm, bf16) two take three quarters of
// the time of one; four do not fit the registers (1.2 times), but for 4 fp32 a thread (16000 x 768: two 37 us, four 28).  With their edges
// rows of 2 x 8 bf16 a thread fit one at a time (8192 x 4095: two 89 us, one 66), and so do those of a layer norm with the bias's
// gradient (sums: 8192 x 4096, two 58.6 us, one 51.9).
__host__ __device__ constexpr int bwd_rows(int w, int nv, bool off, bool sums) {
  return w == 1 || nv == 4 || ((off || sums) && w == 8 && nv == 2) ? 1 : w == 4 && nv == 1 ? 4 : 2;
}

template <int DT, int W, int NV, bool PB, bool BIAS, bool OFF, bool CENTER>
__global__ void __launch_bounds__(512) norm_bwd_kernel(NormArgs A) {
  using Ac = Access<DT, W>;
  constexpr int ES = Vec<DT>::ESIZE, R = bwd_rows(W, NV, OFF, BIAS && CENTER);
  extern __shared__ uint4 places[];
  __shared__ float sh[2][2 * R][kMaxWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  float dw[NV][W], db[BIAS ? NV : 1][W];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < W; ++e) {
      dw[i][e] = 0.f;
      if (BIAS) db[i][e] = 0.f;
    }
  const int64_t group = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const Span span = span_of<W>(OFF, A.x, group, A.ld_x, ES, A.H);
  Rows<DT, W, NV, 2, OFF, W == 1 ? kStages : 2 * R> in;
  in.start({A.x, A.dy}, {A.ld_x, A.ld_dy}, group, step, A.T, span, places);
  float w[NV][W];
  const float we = OFF && span.edge >= 0 ? load_elem(A.weight, span.edge, PB) : 0.f;
  float dwe = 0.f, dbe = 0.f;   // of the edge
  {
    Params<W, NV, PB> p;
    if constexpr (OFF) p.load(A.weight, span);
    else p.load(A.weight, A.H);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < W; ++e) w[i][e] = p.get(i, e);
  }
  char* out = (char*)A.dx + (group * A.ld_dx + span.head + (int64_t)threadIdx.x * W) * ES;
  const int64_t out_edge = (span.edge - span.head - (int64_t)threadIdx.x * W) * ES;
  const int64_t out_stride = step * A.ld_dx * ES;
  float mean_next[R], rstd_next[R];
  auto fetch_stats = [&](int64_t row) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool have = row + r * step < A.T;
      mean_next[r] = CENTER && have ? A.mean[row + r * step] : 0.f;
      rstd_next[r] = have ? A.rstd[row + r * step] : 0.f;
    }
  };
  fetch_stats(group);
  for (int64_t row = group; row < A.T; row += R * step) {
    typename Ac::raw raw[R][2][NV];
    float mean[R], rstd[R], s[2 * R], edge[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] = mean_next[r];
      rstd[r] = rstd_next[r];
      edge[r][0] = edge[r][1] = 0.f;
      in.take(raw[r], edge[r]);
      if (r > 0 && row + r * step >= A.T) {                 // past the last row: 0, and so is everything below
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[r][0][i] = raw[r][1][i] = Ac::zero();
        edge[r][0] = edge[r][1] = 0.f;
      }
      if (W > 1) in.fetch();
    }
    fetch_stats(row + R * step);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float2 s1v = make_float2(0.f, 0.f), s2v = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float x[W], dy[W];
        Ac::unpack(raw[r][0][i], x);
        Ac::unpack(raw[r][1][i], dy);                       // (0 past the end, and so is everything below)
        if constexpr (W > 1) {
#pragma unroll
          for (int e = 0; e < W; e += 2) {
            const float2 d = make_float2(dy[e], dy[e + 1]);
            const float2 xe = make_float2(x[e], x[e + 1]);
            const float2 xh = mul2(CENTER ? add2(xe, make_float2(-mean[r], -mean[r])) : xe, make_float2(rstd[r], rstd[r]));
            const float2 g = mul2(d, make_float2(w[i][e], w[i][e + 1]));
            s1v = add2(s1v, g);
            s2v = fma2(g, xh, s2v);
            const float2 dwe2 = fma2(d, xh, make_float2(dw[i][e], dw[i][e + 1]));
            dw[i][e] = dwe2.x;
            dw[i][e + 1] = dwe2.y;
            if (BIAS) {
              const float2 dbe2 = add2(make_float2(db[i][e], db[i][e + 1]), d);
              db[i][e] = dbe2.x;
              db[i][e + 1] = dbe2.y;
            }
          }
        } else {
          const float xh = (CENTER ? x[0] - mean[r] : x[0]) * rstd[r], g = dy[0] * w[i][0];
          s1v.x += g;
          s2v.x = fmaf(g, xh, s2v.x);
          dw[i][0] = fmaf(dy[0], xh, dw[i][0]);
          if (BIAS) db[i][0] += dy[0];
        }
      }
      float s1 = s1v.x + s1v.y, s2 = s2v.x + s2v.y;
      if (OFF) {
        const float xh = (CENTER ? edge[r][0] - mean[r] : edge[r][0]) * rstd[r], g = edge[r][1] * we;
        s1 += g;
        s2 = fmaf(g, xh, s2);
        dwe = fmaf(edge[r][1], xh, dwe);
        dbe += edge[r][1];
      }
      s[2 * r] = s1;
      s[2 * r + 1] = s2;
    }
    group_sums<2 * R>(s, sh, slot);
    if (W == 1) {
      __syncwarp();                                         // (every thread of the group has read the rows)
      in.fetch();
    }
    // (unpacked again below instead of being kept over the sums: as fp32 a row takes twice the registers)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        keep_packed(raw[r][0][i]);
        keep_packed(raw[r][1][i]);
      }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r * step >= A.T) break;
      // dx = r (g - m1 - xhat m2) = r g + ((x - mu) c1 + c0)
      const float m1 = CENTER ? s[2 * r] * inv_h : 0.f, m2 = s[2 * r + 1] * inv_h;
      const float c1 = -rstd[r] * (rstd[r] * m2), c0 = -rstd[r] * m1;      // (r r alone may leave fp32: tiny rows, eps 0)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (in.have[i]) {
          float x[W], dy[W], o[W];
          Ac::unpack(raw[r][0][i], x);
          Ac::unpack(raw[r][1][i], dy);
#pragma unroll
          for (int e = 0; e < W; e += 2) {
            if constexpr (W > 1) {
              const float2 g = mul2(make_float2(dy[e], dy[e + 1]), make_float2(w[i][e], w[i][e + 1]));
              const float2 xe = make_float2(x[e], x[e + 1]);
              const float2 rest = fma2(CENTER ? add2(xe, make_float2(-mean[r], -mean[r])) : xe, make_float2(c1, c1), make_float2(c0, c0));
              const float2 d = fma2(g, make_float2(rstd[r], rstd[r]), rest);
              o[e] = d.x;
              o[e + 1] = d.y;
            } else {
              o[e] = fmaf(dy[e] * w[i][e], rstd[r], fmaf(CENTER ? x[e] - mean[r] : x[e], c1, c0));
            }
          }
          Ac::store(out + (int64_t)i * (int)blockDim.x * W * ES, o);
        }
      }
      if (OFF && span.edge >= 0) {
        const float o = fmaf(edge[r][1] * we, rstd[r], fmaf(CENTER ? edge[r][0] - mean[r] : edge[r][0], c1, c0));
        Access<DT, 1>::store(out + out_edge, &o);
      }
      out += out_stride;
    }
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // the kernel that adds the lines may set up
  constexpr int kPer = BIAS ? 2 : 1;
  if constexpr (W == 1 ? NV <= 8 : NV == 1)                 // (only these have rows of one warp)
  if (blockDim.y > 1) {     // short rows: the block's groups are added first, in their order (30000 x 63 bf16: 29 -> 18 us)
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    float* all = (float*)places;                            // [groups][kPer][H]: less than the rows took
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t c = span.head + column<W>(i);
      if (column<W>(i) < span.body) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          all[threadIdx.y * kPer * A.H + c + e] = dw[i][e];
          if (BIAS) all[(threadIdx.y * kPer + 1) * A.H + c + e] = db[i][e];
        }
      }
    }
    if (OFF && span.edge >= 0) {
      all[threadIdx.y * kPer * A.H + span.edge] = dwe;
      if (BIAS) all[(threadIdx.y * kPer + 1) * A.H + span.edge] = dbe;
    }
    __syncthreads();
    float* line = A.partial + (int64_t)blockIdx.x * kPer * A.H;
    for (int c = threadIdx.y * 32 + threadIdx.x; c < kPer * (int)A.H; c += 32 * blockDim.y) {
      float t = all[c];
      for (int y = 1; y < blockDim.y; ++y) t += all[y * kPer * (int)A.H + c];
      line[c] = t;
    }
    return;
  }
  float* pw = A.partial + group * kPer * A.H;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t c = span.head + column<W>(i);
    if (column<W>(i) < span.body) {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        pw[c + e] = dw[i][e];
        if (BIAS) pw[A.H + c + e] = db[i][e];
      }
    }
  }
  if (OFF && span.edge >= 0) {
    pw[span.edge] = dwe;
    if (BIAS) pw[A.H + span.edge] = dbe;
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
  const int per_group = A.dbias ? 2 : 1;
  float* pw = A.partial + (int64_t)blockIdx.x * per_group * A.H;
  for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {             // (the thread that adds to a place empties it: no barrier)
    pw[c] = 0.f;
    if (A.dbias) pw[A.H + c] = 0.f;
  }
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
      if (A.dbias) pw[A.H + c] += d;
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

// dw[c] = sum over the groups' lines, in a fixed order: 32 threads a column, each every 32nd line, then their sums.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* partial, int64_t groups, int64_t H, int per_group,
                                                        float* dw, float* db) {
  __shared__ float sh[32][33];
  const int which = blockIdx.y;
  float* out = which ? db : dw;
  const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float s = 0.f;
  if (c < H) {
    const float* p = partial + ((int64_t)threadIdx.y * per_group + which) * H + c;
#pragma unroll 8
    for (int64_t g = threadIdx.y; g < groups; g += 32, p += 32 * per_group * H) s += *p;
  }
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  const float v = warp_sum(sh[threadIdx.x][threadIdx.y]);   // warp y has column y of the block
  const int64_t o = (int64_t)blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && o < H) out[o] = v;
}

struct Plan {
  int w;          // elements an access: a 16-byte vector or 1
  int nv;         // accesses a thread; 0 = the kernels for any width
  int threads;    // a row's group
  int rows;       // groups a block
};

enum RowKind { kAligned, kSpans, kElements };        // rows on 16 bytes; all matrices' rows at the same offsets to 16 bytes; neither
struct RowsAt { RowKind kind; int period; };          // rows after which the offsets repeat
RowsAt rows_at(const NormArgs& a, bool backward) {
  const int64_t es = a.dtype == JP_BF16 ? 2 : 4;
  const void* p[3] = {a.x, backward ? a.dx : a.y, backward ? a.dy : a.x};
  const int64_t ld[3] = {a.ld_x, backward ? a.ld_dx : a.ld_y, backward ? a.ld_dy : a.ld_x};
  bool aligned = a.H * es % 16 == 0 && ((uintptr_t)a.weight & 15) == 0 && ((uintptr_t)a.bias & 15) == 0;
  for (int i = 0; i < 3; ++i) {
    if ((((uintptr_t)p[i] ^ (uintptr_t)p[0]) & 15) != 0 || (ld[i] - ld[0]) * es % 16 != 0) return {kElements, 1};
    aligned = aligned && ((uintptr_t)p[i] & 15) == 0 && ld[i] * es % 16 == 0;
  }
  int period = 1;
  while (a.ld_x * es * period % 16 != 0) period *= 2;
  return {aligned ? kAligned : kSpans, period};
}

// Threads and registers of a row.  16-byte accesses, or single elements where the matrices' rows differ in their offsets; 1, 2 or 4
// vectors (2, 8 or 16 elements) a thread so that rows up to 16384 bf16 (8192 fp32, or 8192 single elements) stay in registers; the sums
// of a backward pass take as much again, so 8192 there (and two aligned vectors from 192 on: 12000 x 2048 bf16 46 us with
// one, 42; of 12000 x 2047, where two take one row at a time, 48 with one, 53).
Plan plan_for(int64_t H, int dtype, RowKind kind, bool backward) {
  Plan p{};
  const int vw = dtype == JP_BF16 ? 8 : 4;
  p.w = kind == kElements ? 1 : vw;
  const int64_t n = (H + p.w - 1) / p.w;
  if (p.w > 1) p.nv = n <= (backward && kind == kAligned ? 192 : 256) ? 1 : n <= 1024 ? 2 : n <= (backward ? 8192 / p.w : 2048) ? 4 : 0;
  else p.nv = n <= 64 ? 2 : n <= 2048 ? 8 : n <= 8192 ? 16 : 0;
  if (p.nv == 0) { p.threads = 1024; p.rows = 1; p.w = 1; return p; }
  const int64_t per = (n + p.nv - 1) / p.nv;
  p.threads = (int)((per + 31) / 32 * 32);
  p.rows = p.threads == 32 ? 8 : 1;
  return p;
}

// Blocks: all rows at once where there are few, else what the registers of an SM hold: 512 threads of a backward pass and of 16 elements
// a thread, 768 of 8 single elements, 1024 of the rest; a multiple of the period.
int grid_for(int64_t T, const Plan& p, int sms, bool backward, int period) {
  const int64_t need = (T + p.rows - 1) / p.rows;
  const int per_sm = (p.w == 1 && p.nv == 2 ? 1024 : backward || p.nv == 16 ? 512 : p.w == 1 ? 768 : 1024) / (p.threads * p.rows);
  const int64_t cap = (int64_t)sms * (per_sm > 8 ? 8 : per_sm < 1 ? 1 : per_sm);
  if (need <= cap) return (int)need;
  if (p.rows % period == 0) return (int)cap;
  return (int)(cap < period ? period : cap / period * period);
}

// The limit of dynamic shared memory belongs to the kernel on the device, for all contexts and threads: every call sets it to the same
// amount, whatever its width, so that none lowers it under another between its setting and its launch.
constexpr int kSharedBytes = 232448 - 2048;                 // of one block, less the static part of the widest kernel
static_assert(kWarpStages * 16 * 32 * warp_rows(16) * 16 + 2 * 4096 * 4 <= kSharedBytes && kWarpStages * 20 * 32 * warp_rows(20) * 16 + 2 * 5120 * 4 <= kSharedBytes, "");
template <auto kernel>
cudaError_t launch(const NormArgs& a, dim3 grid, dim3 block, int smem, cudaStream_t s) {
  if (smem > 47 * 1024) {                                   // (with the static part beyond what a kernel has without asking)
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int DT, bool PB, int NVL>
cudaError_t fwd_warp(const NormArgs& a, const RowsAt& at, cudaStream_t s, int sms) {
  constexpr int kWarpRows = warp_rows(NVL);
  const int64_t most = (int64_t)sms * warp_blocks(NVL), cap = most < at.period ? at.period : most / at.period * at.period;
  const bool off = at.kind == kSpans;
  const int64_t need = off ? cap : (a.T + kWarpRows - 1) / kWarpRows;
  const int smem = kWarpStages * NVL * 32 * kWarpRows * 16 +
                   param_bytes(a.H, PB ? 2 : 4) * (a.bias ? 2 : 1);
  const dim3 g((unsigned)(need < cap ? need : cap)), b(32, kWarpRows);
  if (a.rms) return off ? launch<norm_fwd_warp_kernel<DT, NVL, PB, true, false>>(a, g, b, smem, s) : launch<norm_fwd_warp_kernel<DT, NVL, PB, false, false>>(a, g, b, smem, s);
  return off ? launch<norm_fwd_warp_kernel<DT, NVL, PB, true, true>>(a, g, b, smem, s) : launch<norm_fwd_warp_kernel<DT, NVL, PB, false, true>>(a, g, b, smem, s);
}

template <int DT, bool PB>
cudaError_t fwd(const NormArgs& a, cudaStream_t s, int sms) {
  constexpr int VW = Vec<DT>::N;
  const RowsAt at = rows_at(a, false);
  const RowKind kind = at.kind == kSpans && a.H <= 64 ? kElements : at.kind;
  // a warp a row where every SM gets its blocks full of rows; with fewer rows a block a row is done sooner
  const int64_t n = (a.H + VW - 1) / VW;
  if (at.kind != kElements && a.T >= (int64_t)sms * 12 && n > 64 && n <= 640) {
    if (n <= 128) return fwd_warp<DT, PB, 4>(a, at, s, sms);
    if (n <= 256) return fwd_warp<DT, PB, 8>(a, at, s, sms);
    if (n <= 512) return fwd_warp<DT, PB, 16>(a, at, s, sms);
    return fwd_warp<DT, PB, 20>(a, at, s, sms);
  }
  // (short rows: vectors would leave most lanes idle, 14 us at 30,000 x 63 bf16 against 11)
  const Plan p = plan_for(a.H, a.dtype, kind, false);
  const int grid = grid_for(a.T, p, sms, false, at.period);
  const dim3 b(p.threads, p.rows);
  const int smem = kStages * p.rows * (p.w > 1 ? p.nv * p.threads * 16 : span_bytes(a.H, Vec<DT>::ESIZE));
  if (p.nv == 0) { norm_fwd_wide_kernel<DT><<<grid, b, 0, s>>>(a); return cudaGetLastError(); }
  if (p.w == 1)
    return p.nv == 2   ? launch<norm_fwd_kernel<DT, 1, 2, PB, false>>(a, grid, b, smem, s)
           : p.nv == 8 ? launch<norm_fwd_kernel<DT, 1, 8, PB, false>>(a, grid, b, smem, s)
                       : launch<norm_fwd_kernel<DT, 1, 16, PB, false>>(a, grid, b, smem, s);
  if (kind == kSpans)
    return p.nv == 1   ? launch<norm_fwd_kernel<DT, VW, 1, PB, true>>(a, grid, b, smem, s)
           : p.nv == 2 ? launch<norm_fwd_kernel<DT, VW, 2, PB, true>>(a, grid, b, smem, s)
                       : launch<norm_fwd_kernel<DT, VW, 4, PB, true>>(a, grid, b, smem, s);
  if (p.nv == 1) return launch<norm_fwd_kernel<DT, VW, 1, PB, false>>(a, grid, b, smem, s);
  if (p.nv == 2) return launch<norm_fwd_kernel<DT, VW, 2, PB, false>>(a, grid, b, smem, s);
  return launch<norm_fwd_kernel<DT, VW, 4, PB, false>>(a, grid, b, smem, s);
}

template <int DT, bool PB, bool BIAS, bool CENTER>
cudaError_t bwd(const NormArgs& a, const Plan& p, bool off, int grid, cudaStream_t s) {
  constexpr int VW = Vec<DT>::N;
  const dim3 b(p.threads, p.rows);
  const int smem = 2 * p.rows * (p.w > 1 ? 2 * bwd_rows(p.w, p.nv, off, BIAS && CENTER) * p.nv * p.threads * 16 : kStages * span_bytes(a.H, Vec<DT>::ESIZE));
  if (p.nv == 0) { norm_bwd_wide_kernel<DT><<<grid, b, 0, s>>>(a); return cudaGetLastError(); }
  if (p.w == 1)
    return p.nv == 2   ? launch<norm_bwd_kernel<DT, 1, 2, PB, BIAS, false, CENTER>>(a, grid, b, smem, s)
           : p.nv == 8 ? launch<norm_bwd_kernel<DT, 1, 8, PB, BIAS, false, CENTER>>(a, grid, b, smem, s)
                       : launch<norm_bwd_kernel<DT, 1, 16, PB, BIAS, false, CENTER>>(a, grid, b, smem, s);
  if (off) {
    if (p.nv == 1) return launch<norm_bwd_kernel<DT, VW, 1, PB, BIAS, true, CENTER>>(a, grid, b, smem, s);
    if (p.nv == 2) return launch<norm_bwd_kernel<DT, VW, 2, PB, BIAS, true, CENTER>>(a, grid, b, smem, s);
    if constexpr (DT == JP_F32) return launch<norm_bwd_kernel<DT, VW, 4, PB, BIAS, true, CENTER>>(a, grid, b, smem, s);
    return cudaErrorInvalidConfiguration;
  }
  if (p.nv == 1) return launch<norm_bwd_kernel<DT, VW, 1, PB, BIAS, false, CENTER>>(a, grid, b, smem, s);
  if (p.nv == 2) return launch<norm_bwd_kernel<DT, VW, 2, PB, BIAS, false, CENTER>>(a, grid, b, smem, s);
  if constexpr (DT == JP_F32) return launch<norm_bwd_kernel<DT, VW, 4, PB, BIAS, false, CENTER>>(a, grid, b, smem, s);
  return cudaErrorInvalidConfiguration;
}

template <int DT, bool PB>
cudaError_t bwd(const NormArgs& a, const Plan& p, bool off, int grid, cudaStream_t s) {
  if (a.rms) return a.dbias ? bwd<DT, PB, true, false>(a, p, off, grid, s) : bwd<DT, PB, false, false>(a, p, off, grid, s);
  return a.dbias ? bwd<DT, PB, true, true>(a, p, off, grid, s) : bwd<DT, PB, false, true>(a, p, off, grid, s);
}

}  // namespace

cudaError_t launch_norm_forward(const NormArgs& a, cudaStream_t s, int sms) {
  if (a.dtype == JP_BF16) return a.param_bf16 ? fwd<JP_BF16, true>(a, s, sms) : fwd<JP_BF16, false>(a, s, sms);
  return a.param_bf16 ? fwd<JP_F32, true>(a, s, sms) : fwd<JP_F32, false>(a, s, sms);
}

// Lines of partial sums a backward call can need, whatever the alignment of its pointers.
int64_t norm_backward_groups(int64_t T, int64_t H, int dtype, int sms) {
  int64_t most = 0;
  for (const RowKind kind : {kAligned, kSpans, kElements})
    for (const int period : {1, 8}) {
      const int64_t g = grid_for(T, plan_for(H, dtype, kind, true), sms, true, period);
      most = g > most ? g : most;
    }
  return most;
}

cudaError_t launch_norm_backward(const NormArgs& a, cudaStream_t s, int sms) {
  const RowsAt at = rows_at(a, true);
  const Plan p = plan_for(a.H, a.dtype, at.kind, true);
  const int grid = grid_for(a.T, p, sms, true, at.period);
  const bool off = at.kind == kSpans;
  cudaError_t e;
  if (a.dtype == JP_BF16) e = a.param_bf16 ? bwd<JP_BF16, true>(a, p, off, grid, s) : bwd<JP_BF16, false>(a, p, off, grid, s);
  else e = a.param_bf16 ? bwd<JP_F32, true>(a, p, off, grid, s) : bwd<JP_F32, false>(a, p, off, grid, s);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((a.H + 31) / 32), a.dbias ? 2 : 1);
  cfg.blockDim = dim3(32, 32);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, norm_sum_kernel, (const float*)a.partial, (int64_t)grid, a.H, a.dbias ? 2 : 1, a.dweight, a.dbias);
}

}  // namespace jp
