// The norms before and after a block of a model, fused with its gate and the residual stream: forward and backward over rows [T, H].
//
//   u = (x - mu1) r1 w1 + b1  (the norm behind the block; u = x without w1),   s = residual + a gt[t] gc[h] u  (rounded to its type),
//   y = (s - mu2) r2 w2 + b2  (the norm in front of the next block, of s as stored: what the backward reads);  mu = 0 for RMS norm
//   gs = ds + r2 (g2 - mean g2 - xhat2 mean(g2 xhat2)), g2 = dy w2;   dresidual = gs
//   du = a gt gc gs;   dx = r1 (g1 - mean g1 - xhat1 mean(g1 xhat1)), g1 = du w1
//   dgc = sum_t a gt u gs,  dgt = sum_h a gc u gs,  dw1 = sum_t du xhat1,  db1 = sum_t du,  dw2 = sum_t dy xhat2,  db2 = sum_t dy
//
// Bound by HBM: forward reads x and the residual and writes s and y, backward reads dy, ds, s and x and writes dresidual and dx, each
// once.  A row belongs to one group of threads through all of its sums, 8 elements a thread, so that the parameters of a thread's columns
// stay in registers; the next rows come through asynchronous copies into shared memory meanwhile.  Two rows at a time share their sums'
// barriers.  The sums over rows add up in registers too, and there are fewer of them than gradients: with Q1 = sum_t gt gs xhat1 and
// Q0 = sum_t gt gs,  dw1 = a gc Q1,  db1 = a gc Q0,  dgc = a (w1 Q1 + b1 Q0),  and dgt is what dx's sum has anyway.  The groups of a block add
// theirs in their order, the blocks leave a line each in the workspace, which a second kernel adds in a fixed order: no atomics, the
// same bits every time.
// A thread reads what it copied itself, 16 bytes at a time, no barrier for the data.  Rows that start anywhere, all matrices at the same offset to
// 16 bytes (packed ones of odd width): the vectors that cover the row; what belongs to other rows is masked in the first one and cut from the
// last one's copy, and a group's rows are a multiple of the period apart after which offsets repeat, so a thread keeps its columns.  Matrices at
// different offsets: the group copies the covering vectors together and reads elements.
// Measured, 8192 rows of bf16, RMS norms with gate: forward 4096 columns 48 us (5.6 TB/s), 4095 97 us; backward 4096 82 us (4.9 TB/s), 4095 145 us;
// with layer norms, biases and a gate a token, forward 82 and 204 us, backward 127 and 248 us.
#include "jp_common.cuh"
#include "jp_internal.h"
#include "jp_pairs.cuh"

namespace jp {
namespace {

constexpr int kMaxWarps = 32;
constexpr int kMaxValues = 6;                  // sums that share a barrier

__device__ __forceinline__ float param(const void* p, int64_t i, bool bf16) {
  return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16) : ((const float*)p)[i];
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Groups are the rows of threadIdx.x; a warp that is a group of its own needs no barrier.  SOLE: the block is one group (barriers by number
// would reserve all 16 of them, and an SM has 64).
template <bool SOLE> __device__ __forceinline__ void group_sync() {
  if (blockDim.x == 32) __syncwarp();
  else if (SOLE) __syncthreads();
  else asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.y + 1), "r"(blockDim.x) : "memory");
}

// N sums over the group, in all of its threads, at once: at each step of a warp's sum half of the values go to the other half of the lanes
// (N - 1 + log2(32 / N) shuffles for N a power of two, instead of 5 N), and so when each warp adds the warps' sums.  `slot` alternates
// between uses, so that one barrier each is enough.
template <bool SOLE, int N> __device__ __forceinline__ void group_sums(float (&v)[N], float (*sh)[kMaxValues][kMaxWarps], int& slot) {
  constexpr int M = N == 1 ? 1 : N == 2 ? 2 : N <= 4 ? 4 : 8, kLanes = 32 / M;      // lanes a value has
  const int lane = threadIdx.x & 31;
  float t[M];
#pragma unroll
  for (int i = 0; i < M; ++i) t[i] = i < N ? v[i] : 0.f;
#pragma unroll
  for (int n = M, o = 16; o > 0; o >>= 1) {
    if (n > 1) {
      n /= 2;
#pragma unroll
      for (int i = 0; i < M / 2; ++i)
        if (i < n) {
          const float keep = (lane & o) ? t[i + n] : t[i], send = (lane & o) ? t[i] : t[i + n];
          t[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
    } else {
      t[0] += __shfl_xor_sync(0xffffffffu, t[0], o);
    }
  }
  float s = t[0];                                           // of value lane / kLanes
  if (blockDim.x > 32) {
    const int warps = blockDim.x >> 5, first = threadIdx.y * warps, mine = lane / kLanes;
    float (*part)[kMaxWarps] = sh[slot];
    slot ^= 1;
    if (lane % kLanes == 0 && mine < N) part[mine][first + (threadIdx.x >> 5)] = s;
    group_sync<SOLE>();
    s = 0.f;
    if (mine < N)
      for (int w = lane % kLanes; w < warps; w += kLanes) s += part[mine][first + w];
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, s, i * kLanes);
}

// Shared memory by its own addresses (32 bits, no generic loads).
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
template <int ES> __device__ __forceinline__ uint32_t lds_one(uint32_t at) {
  uint32_t v;
  if constexpr (ES == 2) {
    uint16_t h;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at) : "memory");
    v = h;
  } else {
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  }
  return v;
}
template <int ES> __device__ __forceinline__ void sts_one(uint32_t at, const char* from) {
  if constexpr (ES == 2) asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(*(const volatile uint16_t*)from) : "memory");
  else asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(*(const volatile uint32_t*)from) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const char* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const char* from, int bytes) {      // zeros behind the first `bytes`, which alone are read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const char* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}

enum Kind { kAligned, kShared, kElements };                 // rows on 16 bytes; all matrices' rows at the same offsets to 16 bytes; neither

// What a thread has of a row: NU units.  A unit is a 16-byte vector, or (kElements) two elements a group's width apart.
template <int DT, int KIND> struct Unit {
  static constexpr bool VEC = KIND != kElements;
  static constexpr int W = VEC ? Vec<DT>::N : 1;            // consecutive elements
  static constexpr int E = VEC ? W : 2, P = E / 2;          // elements and pairs of a unit
  static constexpr int ES = Vec<DT>::ESIZE;
  int H;                                                    // (widths that fit the registers: far below 31 bits)
  int first;                                                // column of the first unit (kShared: of its vector, from -W + 1 on)
  unsigned have, part;                                      // bits: some of the unit's columns are in the row; not all of them
  // `row`: where a row of the group starts
  template <int NU> __device__ __forceinline__ void start(const void* row, int64_t H_) {
    H = (int)H_;
    first = VEC ? (int)threadIdx.x * W - (KIND == kShared ? (int)((uintptr_t)row & 15) / ES : 0) : threadIdx.x;
    have = part = 0u;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      int n = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) n += inside(column(u, e));
      have |= (n > 0 ? 1u : 0u) << u;
      part |= (n > 0 && n < E ? 1u : 0u) << u;
    }
  }
  __device__ __forceinline__ int column(int u, int e) const { return VEC ? first + u * (int)blockDim.x * W + e : first + (2 * u + e) * (int)blockDim.x; }
  __device__ __forceinline__ bool inside(int c) const { return (unsigned)c < (unsigned)H; }
  __device__ __forceinline__ bool inside(int u, int e) const { return KIND == kAligned ? (have >> u & 1u) != 0u : inside(column(u, e)); }
  // a unit in its type
  struct Raw { uint32_t w[VEC ? 4 : ES == 2 ? 1 : 2]; };
  __device__ static __forceinline__ void unpack(const Raw& r, float2 (&f)[P]) {
    if constexpr (ES == 2) {
#pragma unroll
      for (int p = 0; p < P; ++p) f[p] = make_float2(__uint_as_float(r.w[p] << 16), __uint_as_float(r.w[p] & 0xffff0000u));
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p) f[p] = make_float2(__uint_as_float(r.w[2 * p]), __uint_as_float(r.w[2 * p + 1]));
    }
  }
  // (unpacked again behind a sum instead of being kept over it: as fp32 a row takes twice the registers)
  __device__ static __forceinline__ void keep(Raw& r) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Raw) / 4); ++i) asm volatile("" : "+r"(r.w[i]));
  }
  __device__ static __forceinline__ Raw pack(const float2 (&f)[P]) {      // rounds
    Raw r;
    if constexpr (ES == 2) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[p].x, f[p].y);
        r.w[p] = *(const uint32_t*)&h;
      }
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p) r.w[2 * p] = __float_as_uint(f[p].x), r.w[2 * p + 1] = __float_as_uint(f[p].y);
    }
    return r;
  }
  // kShared: the row's first vector, in the places `at` of NT matrices: what belongs to the row before reads 0 from here on
  template <int NT> __device__ __forceinline__ void mask(uint32_t at, int place) const {
    uint4 v[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) v[t] = lds16(at + t * place);
    uint32_t keep[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) keep[i] = (first + 2 * i >= 0 ? 0xffffu : 0u) | (first + 2 * i + 1 >= 0 ? 0xffff0000u : 0u);
#pragma unroll
    for (int t = 0; t < NT; ++t)
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at + t * place), "r"(v[t].x & keep[0]), "r"(v[t].y & keep[1]), "r"(v[t].z & keep[2]), "r"(v[t].w & keep[3]) : "memory");
  }
  // `at`: the thread's first unit of the row
  __device__ __forceinline__ void store(char* at, int u, const Raw& r) const {
    if constexpr (VEC) {
      at += u * (int)blockDim.x * 16;
      if (KIND == kShared && (part >> u & 1u)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool lo = inside(u, ES == 2 ? 2 * i : i), hi = ES == 2 ? inside(u, 2 * i + 1) : lo;
          if (lo && hi) ((uint32_t*)at)[i] = r.w[i];
          else if (lo || hi) ((uint16_t*)at)[2 * i + hi] = (uint16_t)(r.w[i] >> (hi ? 16 : 0));
        }
      } else if (have >> u & 1u) {
        stg_stream((uint4*)at, make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (inside(u, e)) {
          char* const to = at + (2 * u + e) * (int)blockDim.x * ES;
          if constexpr (ES == 2) *(uint16_t*)to = (uint16_t)(r.w[0] >> (16 * e));
          else *(uint32_t*)to = r.w[e];
        }
    }
  }
  // parameters at the unit's columns; `none` where there are none, 0 outside the row
  __device__ __forceinline__ void params(const void* p, int u, bool bf16, float none, float2 (&f)[P]) const {
    const char* const at = (const char*)p + (int64_t)column(u, 0) * (bf16 ? 2 : 4);
    const int next = (VEC ? 1 : (int)blockDim.x) * (bf16 ? 2 : 4);
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = inside(u, e) ? none : 0.f;
    if (p) {
      if (bf16) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (inside(u, e)) v[e] = __uint_as_float((uint32_t)*(const uint16_t*)(at + e * next) << 16);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (inside(u, e)) v[e] = *(const float*)(at + e * next);
      }
    }
#pragma unroll
    for (int q = 0; q < P; ++q) f[q] = make_float2(v[2 * q], v[2 * q + 1]);
  }
};

// Bytes of a row's place in shared memory: the vectors of all threads, or the vectors that cover a row wherever it starts.
inline int place_bytes(bool vec, int threads, int units, int64_t H, int es) {
  return vec ? threads * units * 16 : (int)((H * es + 15) / 16 + 1) * 16;
}

// Where column `column` of a row is.  (From the row's number each time: the pitches lie in the constant bank, and pointers that move along would
// take registers, which the sums over rows need.)
template <int ES> __device__ __forceinline__ char* row_at(const void* base, int64_t ld, unsigned row, int column) {
  return (char*)base + ((int64_t)((uint64_t)row * (uint32_t)ld) + column) * ES;
}

// The matrices that the forward and the backward read.
struct ForwardIn {
  static constexpr int N = 2;
  __device__ static __forceinline__ const void* base(const BlockArgs& A, int t) { return t == 0 ? A.x : A.residual; }
  __device__ static __forceinline__ int64_t ld(const BlockArgs& A, int t) { return t == 0 ? A.ld_x : A.ld_residual; }
};
struct BackwardIn {
  static constexpr int N = 4;
  __device__ static __forceinline__ const void* base(const BlockArgs& A, int t) { return t == 0 ? A.dy : t == 1 ? A.sum : t == 2 ? A.dsum : A.x; }
  __device__ static __forceinline__ int64_t ld(const BlockArgs& A, int t) { return t == 0 ? A.ld_dy : t == 1 ? A.ld_sum : t == 2 ? A.ld_dsum : A.ld_x; }
};

// The group's rows of the matrices IN: row `first`, then every `step`-th, STAGES of them under way.
template <int DT, int KIND, int NU, class IN, int STAGES, bool SOLE> struct Ring {
  using Un = Unit<DT, KIND>;
  static constexpr int ES = Vec<DT>::ESIZE, NT = IN::N;
  static constexpr bool VEC = Un::VEC;
  const BlockArgs& A;
  unsigned next, step;                                      // the next row to fetch (below 2^32: T, and so step, are below 2^31)
  uint32_t mem, in, out, end;                               // places (VEC: the thread's own): all, to fill, the oldest row's
  int place;
  unsigned there;                                           // bits: there is such a matrix
  __device__ __forceinline__ Ring(const BlockArgs& A_) : A(A_) {}
  // kElements: 16 bytes of a row's covering vectors; in the rows whose vectors may reach beyond the matrix (`edge`), those that lie in part outside
  // the row element by element
  __device__ __forceinline__ void copy(uint32_t to, const char* from, const char* row, int bytes, bool edge) const {
    if (edge && (from < row || from + 16 > row + bytes)) {
#pragma unroll 1
      for (int q = 0; q < 16; q += ES)
        if (from + q >= row && from + q < row + bytes) sts_one<ES>(to + q, from + q);
    } else {
      copy16(to, from);
    }
  }
  // kShared: the row's first vector, which begins in front of the row.  fp32: the row's words of it (the others are never written); bf16: all of it,
  // to be masked, but for a row that it could reach beyond the matrix of, its elements.  `bytes`: up to the row's end
  __device__ __forceinline__ void copy_first(const Un& un, uint32_t to, const char* from, int bytes) const {
    if (ES == 2 && next >= A.edge_rows) {
      copy16(to, from, bytes);
    } else {
#pragma unroll
      for (int q = 0; q < 16; q += ES)
        if (q >= -un.first * ES && q < bytes) {
          if (ES == 4) copy4(to + q, from + q);
          else sts_one<ES>(to + q, from + q);
        }
    }
  }
  __device__ __forceinline__ void fetch(const Un& un) {
    if (next < (unsigned)A.T) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
        if (there >> t & 1u) {
          const uint32_t to = in + t * place;
          if constexpr (VEC) {
            const char* const at = row_at<ES>(IN::base(A, t), IN::ld(A, t), next, un.first);
#pragma unroll
            for (int u = 0; u < NU; ++u)
              if (un.have >> u & 1u) {
                const char* const from = at + u * (int)blockDim.x * 16;
                const int left = (un.H - un.column(u, 0)) * ES, bytes = left < 16 ? left : 16;
                if (KIND != kShared) copy16(to + u * blockDim.x * 16, from);
                else if (u == 0 && un.first < 0) copy_first(un, to, from, bytes);
                else copy16(to + u * blockDim.x * 16, from, bytes);
              }
          } else {
            const char* const row = row_at<ES>(IN::base(A, t), IN::ld(A, t), next, 0);
            const int skip = (int)((uintptr_t)row & 15), bytes = un.H * ES;
            const bool edge = next < A.edge_rows || next + A.edge_rows >= (unsigned)A.T;
            for (int i = threadIdx.x * 16; i < skip + bytes; i += blockDim.x * 16) copy(to + i, row - skip + i, row, bytes, edge);
          }
        }
      next += step;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    in += NT * place;
    if (in == end) in = mem;
  }
  __device__ __forceinline__ void start(const Un& un, unsigned there_, unsigned first, unsigned step_, const void* mem_, int place_) {
    place = place_;
    mem = (uint32_t)__cvta_generic_to_shared(mem_) + (VEC ? threadIdx.x * 16 : 0);
    in = out = mem;
    end = mem + STAGES * NT * place;
    there = there_;
    next = first;
    step = step_;
    if constexpr (VEC) {                                    // what is never fetched reads 0
      if (un.have != (1u << NU) - 1u || un.first < 0 || there != (1u << NT) - 1u || (int64_t)first + (int64_t)(STAGES - 1) * step >= A.T)
        for (uint32_t at = mem; at != end; at += place)
#pragma unroll
          for (int u = 0; u < NU; ++u)
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at + u * blockDim.x * 16), "r"(0u) : "memory");
    }
#pragma unroll 1
    for (int s = 0; s < STAGES; ++s) fetch(un);
  }
  template <int R> __device__ __forceinline__ void wait(const Un& un) {   // for the oldest R rows
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - R) : "memory");
    if (!VEC) group_sync<SOLE>();
    if (KIND == kShared && ES == 2 && un.first < 0) {        // (a place is the thread's own)
#pragma unroll
      for (int r = 0; r < R; ++r) un.template mask<NT>(row(r), place);
    }
  }
  __device__ __forceinline__ uint32_t row(int r) const {      // the r-th oldest row's places
    const uint32_t at = out + r * NT * place;
    return r > 0 && at >= end ? at - STAGES * NT * place : at;
  }
  // unit u of matrix t of a row, whose places are `at` (kElements: a place begins at its row's offset to 16)
  __device__ __forceinline__ typename Un::Raw get(const Un& un, uint32_t at, int t, int u, unsigned number) const {
    typename Un::Raw w;
    if constexpr (VEC) {
      const uint4 v = lds16(at + t * place + u * blockDim.x * 16);
      w.w[0] = v.x; w.w[1] = v.y; w.w[2] = v.z; w.w[3] = v.w;
    } else {
#pragma unroll
      for (int i = 0; i < (int)(sizeof(w) / 4); ++i) w.w[i] = 0u;
      if (there >> t & 1u) {
        const uint32_t from = at + t * place + ((unsigned)(uintptr_t)row_at<ES>(IN::base(A, t), IN::ld(A, t), number, 0) & 15u) + threadIdx.x * ES;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (un.inside(u, e)) {
            const uint32_t v = lds_one<ES>(from + (2 * u + e) * blockDim.x * ES);
            if constexpr (ES == 2) w.w[0] |= v << (16 * e);
            else w.w[e] = v;
          }
      }
    }
    return w;
  }
  template <int R> __device__ __forceinline__ void done(const Un& un) {   // the oldest R rows' places are free
    if (!VEC) group_sync<SOLE>();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      out += NT * place;
      if (out == end) out = mem;
      fetch(un);
    }
  }
};

// x - mu of a unit's pair p where there are columns, 0 outside the row
template <class Un> __device__ __forceinline__ float2 centred(const Un& un, float2 x, float mu, int u, int p) {
  const float2 d = add2(x, make_float2(-mu, -mu));
  if (Un::VEC && !(un.part >> u & 1u)) return (un.have >> u & 1u) ? d : make_float2(0.f, 0.f);
  return make_float2(un.inside(u, 2 * p) ? d.x : 0.f, un.inside(u, 2 * p + 1) ? d.y : 0.f);
}

// Mean (0 for RMS norm) and 1 / sqrt(mean of squares + eps) of R rows; squares are taken of x - mu.  get(r, u, f): unit u of row r.
template <class Un, int NU, int R, bool FULL, class Get>
__device__ __forceinline__ void row_stats(const BlockArgs& A, const Un& un, Get get, float (*sh)[kMaxValues][kMaxWarps], int& slot, float (&mean)[R], float (&rstd)[R]) {
  const float inv_h = 1.f / (float)A.H;
  const bool center = FULL && !A.rms;
  float v[R];
#pragma unroll
  for (int r = 0; r < R; ++r) mean[r] = 0.f;
  if (center) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float2 t = make_float2(0.f, 0.f);
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        float2 x[Un::P];
        get(r, u, x);                                       // (0 past the end)
#pragma unroll
        for (int p = 0; p < Un::P; ++p) t = add2(t, x[p]);
      }
      v[r] = t.x + t.y;
    }
    group_sums<true, R>(v, sh, slot);
#pragma unroll
    for (int r = 0; r < R; ++r) mean[r] = v[r] * inv_h;
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float2 t = make_float2(0.f, 0.f);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      float2 x[Un::P];
      get(r, u, x);
#pragma unroll
      for (int p = 0; p < Un::P; ++p) {
        if (center) x[p] = centred(un, x[p], mean[r], u, p);
        t = fma2(x[p], x[p], t);
      }
    }
    v[r] = t.x + t.y;
  }
  group_sums<true, R>(v, sh, slot);
#pragma unroll
  for (int r = 0; r < R; ++r) rstd[r] = rsqrtf(v[r] * inv_h + A.eps);     // (2 units in the last place at most)
}

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// R rows at a time.  FULL: layer norm, biases, a gate a token; without it those instructions and registers are left out.  (64 registers, whatever the block:
// an SM has 1024 threads of it.)
template <int DT, int KIND, int NU, int R, int STAGES, bool FULL>
__global__ void __launch_bounds__(1024, 1) block_fwd_kernel(const __grid_constant__ BlockArgs A, int place) {
  using Un = Unit<DT, KIND>;
  constexpr int ES = Vec<DT>::ESIZE, P = Un::P;
  extern __shared__ uint4 places[];
  __shared__ float sh[2][kMaxValues][kMaxWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");        // launched as a programmatic dependent of whatever is before it
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int slot = 0;
  const unsigned step = gridDim.x;
  const bool center = FULL && !A.rms, post = A.post_weight != nullptr;
  Un un;
  un.template start<NU>(row_at<ES>(A.x, A.ld_x, blockIdx.x, 0), A.H);
  Ring<DT, KIND, NU, ForwardIn, STAGES, true> in(A);
  in.start(un, 3u, blockIdx.x, step, places, place);
  // s = residual + gt (xhat1 fw + fb),  y = xhat2 w2 + b2
  float2 fw[NU][P], fb[FULL ? NU : 1][P], w2[NU][P], b2[FULL ? NU : 1][P];
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    float2 g[P];
    un.params(A.post_weight, u, A.param_bf16, 1.f, fw[u]);
    un.params(A.gate, u, A.param_bf16, 1.f, g);
    un.params(A.weight, u, A.param_bf16, 1.f, w2[u]);
#pragma unroll
    for (int p = 0; p < P; ++p) g[p] = mul2(g[p], both(A.scale));
    if (FULL) {
      un.params(A.post_bias, u, A.param_bf16, 0.f, fb[u]);
      un.params(A.bias, u, A.param_bf16, 0.f, b2[u]);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
      fw[u][p] = mul2(fw[u][p], g[p]);
      if (FULL) fb[u][p] = mul2(fb[u][p], g[p]);
    }
  }
  for (unsigned row = blockIdx.x; row < (unsigned)A.T; row += R * step) {
    float m1[R], r1[R], m2[R], r2[R];
    in.template wait<R>(un);
    typename Un::Raw rx[R][NU], s[R][NU];                   // s: the residual, then the sum
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t at = in.row(r);
#pragma unroll
      for (int u = 0; u < NU; ++u) rx[r][u] = in.get(un, at, 0, u, row + r * step);
#pragma unroll
      for (int u = 0; u < NU; ++u) s[r][u] = in.get(un, at, 1, u, row + r * step);
    }
    in.template done<R>(un);
    if (post) {
      row_stats<Un, NU, R, FULL>(A, un, [&](int r, int u, float2 (&f)[P]) { Un::unpack(rx[r][u], f); }, sh, slot, m1, r1);
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) m1[r] = 0.f, r1[r] = 1.f;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const unsigned t = row + r * step;
      if (r > 0 && t >= (unsigned)A.T) break;
      char* const to = row_at<ES>(A.sum, A.ld_sum, t, un.first);
      const float gt = FULL && A.token_gate ? A.token_gate[t] : 1.f;
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        float2 x[P], o[P];
        Un::unpack(rx[r][u], x);
        Un::unpack(s[r][u], o);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if (center) x[p] = add2(x[p], both(-m1[r]));
          x[p] = mul2(x[p], both(r1[r]));
          o[p] = FULL ? fma2(fma2(x[p], fw[u][p], fb[u][p]), both(gt), o[p]) : fma2(x[p], fw[u][p], o[p]);
        }
        s[r][u] = Un::pack(o);
        un.store(to, u, s[r][u]);
      }
      if (threadIdx.x == 0 && post) {
        if (A.out_post_mean) A.out_post_mean[t] = m1[r];
        if (A.out_post_rstd) A.out_post_rstd[t] = r1[r];
      }
    }
    row_stats<Un, NU, R, FULL>(A, un, [&](int r, int u, float2 (&f)[P]) { Un::unpack(s[r][u], f); }, sh, slot, m2, r2);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const unsigned t = row + r * step;
      if (r > 0 && t >= (unsigned)A.T) break;
      char* const to = row_at<ES>(A.y, A.ld_y, t, un.first);
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        float2 x[P];
        Un::unpack(s[r][u], x);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if (center) x[p] = add2(x[p], both(-m2[r]));
          x[p] = mul2(x[p], both(r2[r]));
          x[p] = FULL ? fma2(x[p], w2[u][p], b2[u][p]) : mul2(x[p], w2[u][p]);
        }
        un.store(to, u, Un::pack(x));
      }
      if (threadIdx.x == 0) {
        if (A.out_mean) A.out_mean[t] = m2[r];
        if (A.out_rstd) A.out_rstd[t] = r2[r];
      }
    }
  }
}

// One element, for rows of any width.
template <int DT> __device__ __forceinline__ float element(const void* p, int64_t i) {
  if constexpr (DT == JP_BF16) return __uint_as_float((uint32_t)((const volatile uint16_t*)p)[i] << 16);
  else return ((const volatile float*)p)[i];
}
template <int DT> __device__ __forceinline__ void put(void* p, int64_t i, float v) {
  if constexpr (DT == JP_BF16) ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v);
  else ((float*)p)[i] = v;
}
__device__ __forceinline__ float param_or(const void* p, int64_t i, bool bf16, float none) { return p ? param(p, i, bf16) : none; }

// Any width: the rows are read again for each of their sums (from L2).
template <int DT>
__global__ void __launch_bounds__(1024) block_fwd_wide_kernel(BlockArgs A) {
  __shared__ float sh[2][kMaxValues][kMaxWarps];
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  auto at = [](const void* p, int64_t i) { return element<DT>(p, i); };
  auto stats = [&](const void* p, int64_t first, float& mean, float& rstd) {
    mean = 0.f;
    if (!A.rms) {
      float s[1] = {0.f};
      for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) s[0] += at(p, first + c);
      group_sums<true, 1>(s, sh, slot);
      mean = s[0] * inv_h;
    }
    float q[1] = {0.f};
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float d = at(p, first + c) - mean;
      q[0] = fmaf(d, d, q[0]);
    }
    group_sums<true, 1>(q, sh, slot);
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
      w = param_or(A.post_weight, c, A.param_bf16, 1.f);
      b = param_or(A.post_bias, c, A.param_bf16, 0.f);
      g = param_or(A.gate, c, A.param_bf16, 1.f);
      const float o = fmaf(fmaf((at(A.x, row * A.ld_x + c) - m1) * r1, w, b), scale * g, at(A.residual, row * A.ld_residual + c));
      put<DT>(A.sum, row * A.ld_sum + c, o);
    }
    stats(A.sum, row * A.ld_sum, m2, r2);                   // (each thread reads what it wrote itself)
    if (threadIdx.x == 0) {
      if (A.out_mean) A.out_mean[row] = m2;
      if (A.out_rstd) A.out_rstd[row] = r2;
    }
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      float w, b;
      w = param_or(A.weight, c, A.param_bf16, 1.f);
      b = param_or(A.bias, c, A.param_bf16, 0.f);
      const float o = fmaf((at(A.sum, row * A.ld_sum + c) - m2) * r2, w, b);
      put<DT>(A.y, row * A.ld_y + c, o);
    }
  }
}

// Lines of sums over rows: dw2, Q1 and, with FULL, db2 and Q0.
constexpr int kMaxSums = 4;

template <int DT, int KIND, int NU, int R, int STAGES, bool POST, bool FULL, int THREADS>
__global__ void __launch_bounds__(THREADS) block_bwd_kernel(const __grid_constant__ BlockArgs A, int place) {
  using Un = Unit<DT, KIND>;
  constexpr int ES = Vec<DT>::ESIZE, P = Un::P, N = FULL ? 4 : 2, V1 = FULL ? 2 * R : R, V2 = FULL ? 3 * R : R;
  // Where they fit the registers, a row's values are held as they were stored from its first sum on and its places are free at once; else
  // they are read again behind each sum.
  constexpr bool HOLD = KIND == kAligned && !FULL && NU * Un::E == 8 && THREADS == 512;     // (8192 x 4096 in 96 registers: 362 us instead of 82)
  constexpr int HR = HOLD ? R : 1, HU = HOLD ? NU : 1;
  static_assert(V2 <= kMaxValues, "");
  extern __shared__ uint4 places[];
  __shared__ float sh[2][kMaxValues][kMaxWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  const bool token = FULL && A.token_gate != nullptr, center = FULL && !A.rms, use_x = POST || A.gate || token;
  float2 acc[N][NU][P];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int p = 0; p < P; ++p) acc[n][u][p] = both(0.f);
  const unsigned first = blockIdx.x * blockDim.y + threadIdx.y, step = gridDim.x * blockDim.y;
  Un un;
  un.template start<NU>(row_at<ES>(A.dy, A.ld_dy, first, 0), A.H);
  Ring<DT, KIND, NU, BackwardIn, STAGES, false> in(A);
  in.start(un, 3u | (A.dsum ? 4u : 0u) | (use_x ? 8u : 0u), first, step, (char*)places + threadIdx.y * STAGES * 4 * place, place);
  float2 w2[NU][P], fw[NU][P], fb[FULL ? NU : 1][P];        // fw = a gc w1, fb = a gc b1
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    float2 g[P];
    un.params(A.weight, u, A.param_bf16, 1.f, w2[u]);
    un.params(POST ? A.post_weight : nullptr, u, A.param_bf16, 1.f, fw[u]);
    un.params(A.gate, u, A.param_bf16, 1.f, g);
    if (FULL) un.params(A.post_bias, u, A.param_bf16, 0.f, fb[u]);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      g[p] = mul2(g[p], both(A.scale));
      fw[u][p] = mul2(fw[u][p], g[p]);
      if (FULL) fb[u][p] = mul2(fb[u][p], g[p]);
    }
  }
  // the rows' scalars, fetched a turn ahead (a row behind the last one reads 0 throughout)
  float next[R][5];
  auto scalars = [&](unsigned row) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const unsigned at = row + r * step;
      const bool have = at < (unsigned)A.T;
      next[r][0] = POST && center && have ? A.post_mean[at] : 0.f;
      next[r][1] = !POST ? 1.f : have ? A.post_rstd[at] : 0.f;
      next[r][2] = center && have ? A.mean[at] : 0.f;
      next[r][3] = have ? A.rstd[at] : 0.f;
      next[r][4] = token && have ? A.token_gate[at] : have ? 1.f : 0.f;
    }
  };
  scalars(first);
  for (unsigned row = first; row < (unsigned)A.T; row += R * step) {
    float m1[R], r1[R], m2[R], r2[R], gt[R], v[V1], t[V2];
#pragma unroll
    for (int r = 0; r < R; ++r) m1[r] = next[r][0], r1[r] = next[r][1], m2[r] = next[r][2], r2[r] = next[r][3], gt[r] = next[r][4];
    scalars(row + R * step);
    in.template wait<R>(un);
    typename Un::Raw held[4][HR][HU];
    if constexpr (HOLD) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int t = 0; t < 4; ++t) held[t][r][u] = in.get(un, in.row(r), t, u, row + r * step);
      in.template done<R>(un);
    }
    auto read = [&](int t, int r, int u, float2 (&f)[P]) {  // unit u of dy, sum, dsum or x
      if constexpr (HOLD) Un::unpack(held[t][r][u], f);
      else Un::unpack(in.get(un, in.row(r), t, u, row + r * step), f);
    };
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float2 v1 = both(0.f), v2 = v1;
      if (r == 0 || row + r * step < (unsigned)A.T) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          float2 d[P], s[P];
          read(0, r, u, d);
          read(1, r, u, s);
#pragma unroll
          for (int p = 0; p < P; ++p) {
            if (center) s[p] = add2(s[p], both(-m2[r]));
            const float2 xh = mul2(s[p], both(r2[r])), g = mul2(d[p], w2[u][p]);
            if (center) v1 = add2(v1, g);
            v2 = fma2(g, xh, v2);
            acc[0][u][p] = fma2(d[p], xh, acc[0][u][p]);
            if (FULL) acc[2][u][p] = add2(acc[2][u][p], d[p]);
          }
        }
      }
      v[r] = v2.x + v2.y;
      if (FULL) v[R + r] = v1.x + v1.y;
    }
    group_sums<false, V1>(v, sh, slot);
    if constexpr (HOLD) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < NU; ++u) Un::keep(held[0][r][u]), Un::keep(held[1][r][u]);
    }
    // gs = r2 (dy w2 - a1 - xhat2 a2) + ds
    float2 gs[R][NU][P];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const unsigned at = row + r * step;
      char* const to = row_at<ES>(A.dresidual, A.ld_dresidual, at, un.first);
      const float a1 = center ? v[V1 - R + r] * inv_h : 0.f, k2 = -r2[r] * (r2[r] * (v[r] * inv_h));      // (r r alone may leave fp32)
      float2 t0 = both(0.f), t1 = t0, tb = t0;
      if (r == 0 || at < (unsigned)A.T) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          float2 d[P], s[P], e[P], x[P];
          read(0, r, u, d);
          read(1, r, u, s);
          read(2, r, u, e);
          read(3, r, u, x);
#pragma unroll
          for (int p = 0; p < P; ++p) {
            if (center) s[p] = add2(s[p], both(-m2[r]));
            float2 g = mul2(d[p], w2[u][p]);
            if (center) g = add2(g, both(-a1));
            g = fma2(g, both(r2[r]), fma2(s[p], both(k2), e[p]));
            gs[r][u][p] = g;
            if (center) x[p] = add2(x[p], both(-m1[r]));
            const float2 xh = POST ? mul2(x[p], both(r1[r])) : x[p], g1 = mul2(g, fw[u][p]), gg = FULL ? mul2(g, both(gt[r])) : g;
            t1 = fma2(g1, xh, t1);
            acc[1][u][p] = fma2(gg, xh, acc[1][u][p]);
            if (FULL) {
              t0 = add2(t0, g1);
              tb = fma2(g, fb[u][p], tb);
              acc[3][u][p] = add2(acc[3][u][p], gg);
            }
          }
          un.store(to, u, Un::pack(gs[r][u]));
        }
      }
      t[r] = t1.x + t1.y;
      if (FULL) {
        t[R + r] = t0.x + t0.y;
        t[2 * R + r] = tb.x + tb.y;
      }
    }
    if (POST || token) group_sums<false, V2>(t, sh, slot);
    if constexpr (HOLD) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < NU; ++u) Un::keep(held[3][r][u]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const unsigned at = row + r * step;
      if (r > 0 && at >= (unsigned)A.T) break;
      char* const to = row_at<ES>(A.dx, A.ld_dx, at, un.first);
      if (token && threadIdx.x == 0) A.dtoken_gate[at] = t[r] + t[V2 - R + r];
      // dx = r1 (gt g1 - c1 - xhat1 c2)
      const float c0 = center ? -r1[r] * (gt[r] * (t[V2 > R ? R + r : r] * inv_h)) : 0.f, c2 = -r1[r] * (r1[r] * (gt[r] * (t[r] * inv_h))), rg = r1[r] * gt[r];
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        float2 o[P], x[P];
        if (POST) read(3, r, u, x);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          o[p] = mul2(gs[r][u][p], fw[u][p]);
          if (POST) {
            if (center) x[p] = add2(x[p], both(-m1[r]));
            o[p] = fma2(o[p], both(rg), fma2(x[p], both(c2), both(c0)));
          } else if (FULL) {
            o[p] = mul2(o[p], both(gt[r]));
          }
        }
        un.store(to, u, Un::pack(o));
      }
    }
    if constexpr (!HOLD) in.template done<R>(un);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // the kernel that adds the lines may set up
  // the block's groups one after the other, in shared memory; the last one writes the block's line
  float* const all = (float*)places;                        // [N][H]
  for (int g = 0; g < (int)blockDim.y; ++g) {
    __syncthreads();
    if ((int)threadIdx.y == g) {
      float* to = g + 1 == (int)blockDim.y ? A.partial + (int64_t)blockIdx.x * N * A.H : all;
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int p = 0; p < P; ++p)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const int c = n * un.H + un.column(u, 2 * p + half);
              if (un.inside(u, 2 * p + half)) {
                float sum = half ? acc[n][u][p].y : acc[n][u][p].x;
                if (g > 0) sum += all[c];
                to[c] = sum;
              }
            }
    }
  }
}

// Any width: rows are read again for each sum, and the sums over rows stay in the block's line of the workspace (each thread its columns).
template <int DT>
__global__ void __launch_bounds__(1024) block_bwd_wide_kernel(BlockArgs A) {
  __shared__ float sh[2][kMaxValues][kMaxWarps];
  int slot = 0;
  const float inv_h = 1.f / (float)A.H;
  const bool post = A.post_weight != nullptr, use_x = post || A.gate || A.token_gate;
  float* const line = A.partial + (int64_t)blockIdx.x * kMaxSums * A.H;
  for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x)
    for (int n = 0; n < kMaxSums; ++n) line[n * A.H + c] = 0.f;
  auto at = [](const void* p, int64_t i) { return element<DT>(p, i); };
  for (int64_t row = blockIdx.x; row < A.T; row += gridDim.x) {
    const float m2 = A.rms ? 0.f : A.mean[row], r2 = A.rstd[row];
    const float m1 = post && !A.rms ? A.post_mean[row] : 0.f, r1 = post ? A.post_rstd[row] : 1.f;
    const float gt = A.token_gate ? A.token_gate[row] : 1.f;
    float v[2] = {0.f, 0.f}, t[3] = {0.f, 0.f, 0.f};
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float d = at(A.dy, row * A.ld_dy + c), xh = (at(A.sum, row * A.ld_sum + c) - m2) * r2, g = d * param(A.weight, c, A.param_bf16);
      v[0] += g;
      v[1] = fmaf(g, xh, v[1]);
      line[c] = fmaf(d, xh, line[c]);
      line[2 * A.H + c] += d;
    }
    group_sums<true, 2>(v, sh, slot);
    const float a1 = A.rms ? 0.f : v[0] * inv_h, a2 = v[1] * inv_h;
    // gs of a column; dresidual and dx may lie where dy, dsum, x or sum do, so both are written in the last pass only
    auto gs_at = [&](int64_t c) {
      const float xh = (at(A.sum, row * A.ld_sum + c) - m2) * r2;
      return fmaf(r2, fmaf(-xh, a2, fmaf(at(A.dy, row * A.ld_dy + c), param(A.weight, c, A.param_bf16), -a1)),
                  A.dsum ? at(A.dsum, row * A.ld_dsum + c) : 0.f);
    };
    auto factor = [&](int64_t c) { return A.scale * param_or(A.gate, c, A.param_bf16, 1.f); };
    if (use_x) {
      for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
        const float g = gs_at(c), xh = (at(A.x, row * A.ld_x + c) - m1) * r1, f = factor(c);
        const float g1 = g * f * param_or(A.post_weight, c, A.param_bf16, 1.f);
        t[0] += g1;
        t[1] = fmaf(g1, xh, t[1]);
        t[2] = fmaf(g, f * param_or(A.post_bias, c, A.param_bf16, 0.f), t[2]);
        line[A.H + c] = fmaf(g * gt, xh, line[A.H + c]);
        line[3 * A.H + c] += g * gt;
      }
      group_sums<true, 3>(t, sh, slot);
      if (A.token_gate && threadIdx.x == 0) A.dtoken_gate[row] = t[1] + t[2];
    }
    const float c1 = A.rms ? 0.f : gt * (t[0] * inv_h), c2 = gt * (t[1] * inv_h);
    for (int64_t c = threadIdx.x; c < A.H; c += blockDim.x) {
      const float g = gs_at(c), g1 = gt * g * factor(c);
      const float o = post ? r1 * (fmaf(g1, param(A.post_weight, c, A.param_bf16), -c1) - (at(A.x, row * A.ld_x + c) - m1) * r1 * c2) : g1;
      put<DT>(A.dresidual, row * A.ld_dresidual + c, g);
      put<DT>(A.dx, row * A.ld_dx + c, o);
    }
  }
}

// Column sums of the blocks' lines in a fixed order, 32 threads a column, each every 32nd line, then their sums; and the gradients that
// are made of them.  Blocks with y = 0: of dw2 and db2; y = 1: of Q1 and Q0.
__global__ void __launch_bounds__(1024) block_lines_kernel(BlockArgs A, int lines, int n) {
  __shared__ float sh[2][32][33];
  const int which = blockIdx.y;
  const int64_t H = A.H, c = (int64_t)blockIdx.x * 32 + threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float a = 0.f, b = 0.f;
  if (c < H) {
    const float* p = A.partial + ((int64_t)threadIdx.y * n + which) * H + c;
#pragma unroll 8
    for (int g = threadIdx.y; g < lines; g += 32, p += 32 * n * H) {
      a += p[0];
      if (n > 2) b += p[2 * H];
    }
  }
  sh[0][threadIdx.y][threadIdx.x] = a;
  sh[1][threadIdx.y][threadIdx.x] = b;
  __syncthreads();
  a = warp_sum(sh[0][threadIdx.x][threadIdx.y]);            // warp y has column y of the block
  b = warp_sum(sh[1][threadIdx.x][threadIdx.y]);
  const int64_t o = (int64_t)blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x != 0 || o >= H) return;
  if (which == 0) {
    A.dweight[o] = a;
    if (A.with_bias) A.dbias[o] = b;
  } else {
    const float f = A.scale * param_or(A.gate, o, A.param_bf16, 1.f);
    if (A.post_weight) {
      A.dpost_weight[o] = f * a;
      if (A.with_bias) A.dpost_bias[o] = f * b;
    }
    if (A.gate) A.dgate[o] = A.scale * (param_or(A.post_weight, o, A.param_bf16, 1.f) * a + param_or(A.post_bias, o, A.param_bf16, 0.f) * b);
  }
}

// Threads a row (a group), rows at a time and under way, groups a block.
struct Plan {
  Kind kind;
  int period;              // rows after which offsets to 16 bytes repeat
  bool twice;              // 16 elements a thread instead of 8
  int rows, stages;        // rows 0: the kernels for any width
  int threads, groups, place, smem;
};

void kind_of(const BlockArgs& a, bool backward, Plan* p) {
  const int64_t es = a.dtype == JP_BF16 ? 2 : 4;
  const void* at[6] = {a.sum, a.x, backward ? a.dy : a.residual, backward ? a.dsum : a.y, a.dx, a.dresidual};
  const int64_t ld[6] = {a.ld_sum, a.ld_x, backward ? a.ld_dy : a.ld_residual, backward ? a.ld_dsum : a.ld_y, a.ld_dx, a.ld_dresidual};
  p->kind = a.H * es % 16 == 0 ? kAligned : kShared;
  for (int i = 0; i < 6; ++i) {
    if (!at[i]) continue;
    if ((((uintptr_t)at[i] ^ (uintptr_t)a.sum) & 15) != 0 || (ld[i] - a.ld_sum) * es % 16 != 0) { p->kind = kElements; break; }
    if (((uintptr_t)at[i] & 15) != 0 || ld[i] * es % 16 != 0) p->kind = kShared;
  }
  p->period = 1;
  while (p->kind == kShared && a.ld_sum * es * p->period % 16 != 0) p->period *= 2;
}

constexpr int kSharedBytes = 225 * 1024;      // of an SM, for rows
constexpr int stages_of(int rows, bool twice, int dt) { return rows == 2 ? 6 : twice && dt == JP_F32 ? 1 : 3; }

// Threads a block may have: usual, or most where it has one group more of 8 elements a thread then (one instead of none, two instead of one)
Plan plan_for(const BlockArgs& a, bool backward, bool one_row, int matrices, int usual, int most, int sms) {
  const int dtype = a.dtype, es = dtype == JP_BF16 ? 2 : 4, w = 16 / es;
  const int64_t T = a.T;
  Plan p{};
  kind_of(a, backward, &p);
  const bool vec = p.kind != kElements;
  const int64_t H = p.kind == kShared ? (a.H + 2 * w - 2) / w * w : a.H;     // the columns that covering vectors have
  for (const int each : {8, 16}) {
    p.twice = each == 16;
    const int64_t threads = ((H + each - 1) / each + 31) / 32 * 32;
    if (threads > (p.twice ? usual : most)) continue;
    p.threads = (int)threads;
    p.groups = usual / p.threads;
    if (p.groups < 2 && !p.twice && most / p.threads > p.groups) p.groups = most / p.threads;
    p.place = place_bytes(vec, p.threads, (p.twice ? 2 : 1) * es / 2, H, es);
    // two rows at a time where every group has several and their places fit
    for (p.rows = p.twice || one_row || T < 4 * (int64_t)sms * p.groups ? 1 : 2; p.rows >= 1; --p.rows) {
      p.stages = stages_of(p.rows, p.twice, dtype);
      p.smem = p.stages * matrices * p.place;
      if ((int64_t)p.smem * p.groups <= kSharedBytes) return p;
      if (p.rows == 1) {
        p.groups = kSharedBytes / p.smem;
        if (p.groups > 0) return p;
      }
    }
  }
  p.rows = 0;
  return p;
}

// Blocks: one for each group's rows, or what fits the GPU; then a multiple of the period.
int grid_for(int64_t T, const Plan& p, int groups_a_block, int64_t most) {
  const int64_t each = (int64_t)groups_a_block * p.rows, need = (T + each - 1) / each;
  if (need <= most && T <= need * groups_a_block) return (int)need;
  int64_t g = need < most ? need : most;
  while (g > 1 && g * groups_a_block % p.period != 0) --g;
  return g * groups_a_block % p.period == 0 ? (int)g : p.period;
}

template <auto kernel, class... Q> cudaError_t launch(dim3 grid, dim3 block, int smem, cudaStream_t s, Q... args) {
  if (smem > 0) {
    const cudaError_t e = allow_shared_memory<kernel>(kSharedBytes);
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
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Forward: a block a group, 1024 threads an SM, or what an SM's memory holds of such blocks with what each has beside its rows' places (64 threads: 15).
constexpr int kSmBytes = 228 * 1024, kOwnBytes = 1024 + 2 * kMaxValues * kMaxWarps * (int)sizeof(float);
template <int DT, bool FULL> cudaError_t forward(const BlockArgs& a, cudaStream_t s, int sms) {
  const Plan p = plan_for(a, false, false, 2, 1024, 1024, sms);
  if (p.rows == 0) {
    block_fwd_wide_kernel<DT><<<(unsigned)(a.T < sms ? a.T : sms), 1024, 0, s>>>(a);
    return cudaGetLastError();
  }
  const int fit = kSmBytes / (p.smem + kOwnBytes), most = p.groups < 24 ? p.groups : 24;
  const dim3 g((unsigned)grid_for(a.T, p, 1, (int64_t)sms * (fit < most ? fit : most))), b(p.threads);
  constexpr int V = DT == JP_BF16 ? 1 : 2, E = 4;
#define JP_FORWARD(KIND, NU, R, TWICE) launch<block_fwd_kernel<DT, KIND, NU, R, stages_of(R, TWICE, DT), FULL>>(g, b, p.smem, s, a, p.place)
  if (p.twice) return p.kind == kAligned ? JP_FORWARD(kAligned, 2 * V, 1, true) : p.kind == kShared ? JP_FORWARD(kShared, 2 * V, 1, true) : JP_FORWARD(kElements, 2 * E, 1, true);
  if (p.rows == 2) return p.kind == kAligned ? JP_FORWARD(kAligned, V, 2, false) : p.kind == kShared ? JP_FORWARD(kShared, V, 2, false) : JP_FORWARD(kElements, E, 2, false);
  return p.kind == kAligned ? JP_FORWARD(kAligned, V, 1, false) : p.kind == kShared ? JP_FORWARD(kShared, V, 1, false) : JP_FORWARD(kElements, E, 1, false);
#undef JP_FORWARD
}

// Backward: the groups of an SM in one block, of 512 threads, or of 640 with 96 registers each where that makes room for a row more (bf16, 8192 rows:
// 4095 columns 184 us with 16 elements a thread, 144 with 640 threads; 2047 107 and 74, 2560 68 and 57; with gates and layer norms 4095 358 and
// 254, 2560 106 and 98; not for a third row: 24,496 x 1283 fp32 222 and 236).
template <int DT, bool POST, bool FULL> cudaError_t backward(const BlockArgs& a, const Plan& p, dim3 g, cudaStream_t s) {
  constexpr int V = DT == JP_BF16 ? 1 : 2, E = 4;
  const dim3 b(p.threads, p.groups);
  const int sums = p.groups > 1 ? (FULL ? 4 : 2) * (int)a.H * 4 : 0, rows = p.smem * p.groups, smem = rows > sums ? rows : sums;
#define JP_BACKWARD(THREADS, KIND, NU, R, TWICE) launch<block_bwd_kernel<DT, KIND, NU, R, stages_of(R, TWICE, DT), POST, FULL, THREADS>>(g, b, smem, s, a, p.place)
#define JP_KINDS(THREADS, VECTORS, ELEMENTS, R, TWICE) (p.kind == kAligned ? JP_BACKWARD(THREADS, kAligned, VECTORS, R, TWICE) : p.kind == kShared ? JP_BACKWARD(THREADS, kShared, VECTORS, R, TWICE) \
                                                                                             : JP_BACKWARD(THREADS, kElements, ELEMENTS, R, TWICE))
  if (p.twice) return JP_KINDS(512, 2 * V, 2 * E, 1, true);
  const bool many = p.threads * p.groups > 512;
  if constexpr (!FULL && DT == JP_BF16)
    if (many && p.rows == 2) return JP_KINDS(640, V, E, 2, false);
  if constexpr (!FULL || DT == JP_F32)
    if (p.rows == 2) return JP_KINDS(512, V, E, 2, false);      // (with 640 threads in fp32 their places do not fit)
  return many ? JP_KINDS(640, V, E, 1, false) : JP_KINDS(512, V, E, 1, false);
#undef JP_KINDS
#undef JP_BACKWARD
}
template <int DT> cudaError_t backward(const BlockArgs& a, const Plan& p, int grid, bool full, cudaStream_t s) {
  if (p.rows == 0) {
    block_bwd_wide_kernel<DT><<<grid, 1024, 0, s>>>(a);
    return cudaGetLastError();
  }
  const dim3 g(grid);
  if (a.post_weight) return full ? backward<DT, true, true>(a, p, g, s) : backward<DT, true, false>(a, p, g, s);
  return full ? backward<DT, false, true>(a, p, g, s) : backward<DT, false, false>(a, p, g, s);
}

bool full(const BlockArgs& a, bool backward) { return !a.rms || a.token_gate || a.post_bias || (backward ? a.with_bias : a.bias != nullptr); }

}  // namespace

static uint32_t edge_rows(const BlockArgs& a, bool backward) {
  const int64_t es = a.dtype == JP_BF16 ? 2 : 4, ld[4] = {a.ld_x, a.ld_sum, backward ? a.ld_dy : a.ld_residual, backward ? a.ld_dsum : a.ld_sum};
  uint32_t n = 1;
  for (int64_t v : ld) n = rows_near_an_end(v * es) > n ? rows_near_an_end(v * es) : n;
  return n;
}

cudaError_t launch_block_forward(BlockArgs a, cudaStream_t s, int sms) {
  a.edge_rows = edge_rows(a, false);
  if (a.dtype == JP_BF16) return full(a, false) ? forward<JP_BF16, true>(a, s, sms) : forward<JP_BF16, false>(a, s, sms);
  return full(a, false) ? forward<JP_F32, true>(a, s, sms) : forward<JP_F32, false>(a, s, sms);
}

// At most a line a block and SM, whatever the kernel.
size_t block_workspace_bytes(int64_t T, int64_t H, int, int sms) { return (size_t)(T < sms ? T : sms) * kMaxSums * (size_t)H * sizeof(float); }

cudaError_t launch_block_backward(BlockArgs a, cudaStream_t s, int sms) {
  a.edge_rows = edge_rows(a, true);
  const Plan p = plan_for(a, true, a.dtype == JP_BF16 && full(a, true), 4, 512, 640, sms);      // (8192 x 4096 layer norms with gates: one row at a time 127 us, two 130)
  const int grid = p.rows ? grid_for(a.T, p, p.groups, sms) : (int)(a.T < sms ? a.T : sms), n = p.rows == 0 || full(a, true) ? 4 : 2;
  const cudaError_t e = a.dtype == JP_BF16 ? backward<JP_BF16>(a, p, grid, n == 4, s) : backward<JP_F32>(a, p, grid, n == 4, s);
  if (e != cudaSuccess) return e;
  const unsigned y = a.post_weight || a.gate ? 2 : 1;
  return launch<block_lines_kernel>(dim3((unsigned)((a.H + 31) / 32), y), dim3(32, 32), 0, s, a, grid, n);
}

}  // namespace jp
