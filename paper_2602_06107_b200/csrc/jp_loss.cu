// Losses of one model over its logits [T, V], with the gradient of the logits: the clipped policy loss with a KL term, and the preference
// loss of pairs of sequences.  For row t with sampled token x, temperature tau and p = softmax(z / tau):
//
//   lp = z_x / tau - log sum_v exp(z_v / tau),   dL/dz_v = k (1[v = x] - p_v) / tau,   k = dL/dlp
//   policy      r = exp(lp - lp_old), d = lp_ref - lp:  L = sum_t c_t (max(-A r, -A clip(r)) + beta (exp(d) - d - 1)),
//               k = c (-A r [unclipped branch] + beta (1 - exp(d)))
//   preference  S = sum or mean of a sequence's lp, h = beta ((S - R)_chosen - (S - R)_rejected) - margin:
//               L = mean over pairs of -(1 - e) log sigma(h) - e log sigma(-h),  k = +-(beta / P) (e sigma(h) - (1 - e) sigma(-h))
//
// Bound by HBM.  The policy loss has a row's k as soon as the row's sum is known, so sum and gradient are one launch, and the row stays in
// shared memory in between, spread over the blocks of a cluster: HBM and L2 see one read and one write.  The preference loss needs both
// sequences of a pair first: a pass for the sums, one for the gradients, each a stream through a ring of places.  Each thread copies its own
// vectors (asynchronously, no barriers) and fetches the next row's into a place as soon as it has read it for the last time; several blocks
// an SM (four of 256 threads where 13 vectors a thread hold a row, or two of 512 where eight small ones cannot), so that some load and store while
// others wait for their sum.
// One warp makes a row's scalars of the warps' sums.  Rows that no cluster can hold are read twice.
// Measured, bf16, V = 151,936: policy loss, 4096 rows of which some are masked, 2.2 GB, 444 us (5.0 TB/s; with two blocks of 512 threads 483 instead
// of 450, with five of 192 474); preference loss, six pairs of sequences, 3.5 GB in three passes, 642 us (5.5 TB/s).  Vectors are counted in
// 32 bits: their addresses in 64 cost 1 to 3 %.
// Sums of exponentials are fp32 (in 2^x of z log2(e) / tau, relative to a running maximum): a thread adds a vector's 8 (bf16) or 4 (fp32) terms as a tree
// and the result to its sum, one addition a vector, each off by 2^-24 of the sum so far.  That is V / (8 or 4) / (threads of the blocks that share a
// row) of them: at most 14 where a row stays in shared memory; in a stream with a block a row (more rows than SMs) 37 for 151,936 in bf16, 489 for 1,000,000
// in fp32; in rows that no cluster can hold an eighth of that.  So a row's sum is off by half that number times 2^-24 in this, relatively.  The row's
// scalars are fp64: the clip is a decision, and exp(d) - d - 1 cancels.
#include <atomic>

#include "jp_common.cuh"
#include "jp_internal.h"
#include "jp_pairs.cuh"

namespace jp {
namespace {

constexpr int kMostThreads = 512;             // of a block; an SM has 1024, whatever the block
constexpr int kMaxCluster = 8;
constexpr int kUnroll = 4;
constexpr float kFloor = -1.0e38f;            // below any row's maximum (in units of log2) that counts as one

enum Mode { kPolicy, kPolicyNoGrad, kPrefSums, kPrefGrad };

__device__ __forceinline__ uint4 ld_row(const uint4* p) {   // (not the read-only path: the gradient may take the logits' place)
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
template <int DT> __device__ __forceinline__ uint4 pack(const float* f) {
  if constexpr (DT == JP_BF16) {
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
      o[e] = *(const uint32_t*)&h;
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
  } else {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
}
template <int DT> __device__ __forceinline__ void store_one(void* row, int64_t i, float f) {
  if constexpr (DT == JP_BF16) ((__nv_bfloat16*)row)[i] = __float2bfloat16_rn(f);
  else ((float*)row)[i] = f;
}

// (Whole lines of 128 bytes, so that the places behind it start on one: 16 bytes off 32, every copy's line is split, which costs 4 to 8 %.)
struct alignas(128) Shared {
  float2 warp[2][kMostThreads / 32];              // by the parity of the row's number, like what follows
  float2 part[2][kMaxCluster];                // of the cluster's blocks
  unsigned long long arrived[2];              // barriers that count the parts' bytes
  float top, k_over_s, coef;
  int count[kMostThreads / 32];
  long long lost_row, lost_count;             // the row whose exchange gave up (-1: none did), and its number among the block's
};
constexpr long long kSpin = 4000000000ll;     // clock cycles after which a wait gives up

// (maximum, sum) over a warp
__device__ __forceinline__ float2 warp_merge(float2 v) {
  float m = v.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float s = v.y * ex2_approx(v.x - m);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return make_float2(m, s);
}

__device__ __forceinline__ bool parts_are_here(uint32_t bar, uint32_t phase) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, 1000;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(phase) : "memory");
  return ok != 0u;
}

// By all threads of a cluster's blocks, before the first exchange.
__device__ __forceinline__ void exchange_start(Shared& sh) {
  if (threadIdx.x < 2) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"((uint32_t)__cvta_generic_to_shared(&sh.arrived[threadIdx.x])) : "memory");
  if (threadIdx.x == 0) sh.lost_row = -1;
  if (threadIdx.x == 0) asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// By one warp: the row's (maximum, sum) over the block's warps, then over the cluster's blocks, each of which sends its part to every other one's
// shared memory (and gets the same total: the parts are merged in the same order).  A wait that gives up returns a sum below 0, and so does every row
// of this block behind it: its barrier's phase is open still, and the others no longer hear of this block and give up in their turn.
__device__ __forceinline__ float2 row_total(Shared& sh, int rank, int ranks, int64_t count, int64_t row, long long limit = kSpin) {
  const int p = (int)(count & 1), lane = threadIdx.x & 31;
  float2 v = warp_merge(lane < (int)blockDim.x / 32 ? sh.warp[p][lane] : make_float2(kFloor, 0.f));
  if (ranks == 1) return v;
  if (sh.lost_row >= 0) return make_float2(0.f, -1.f);
  const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&sh.arrived[p]), at = (uint32_t)__cvta_generic_to_shared(&sh.part[p][rank]);
  if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(ranks * 8) : "memory");
  if (lane < ranks) {
    uint32_t to, theirs;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(at), "r"(lane));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(theirs) : "r"(bar), "r"(lane));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(to), "f"(v.x), "f"(v.y), "r"(theirs) : "memory");
  }
  const uint32_t phase = (uint32_t)(count >> 1) & 1u;
  bool here = false;
  long long t0 = 0;
  for (uint32_t i = 0; !here; ++i) {
    here = parts_are_here(bar, phase);
    if (!here && (i & 63u) == 0u) {
      const long long now = clock64();
      if (i == 0u) t0 = now;
      else if (now - t0 > limit) break;
    }
  }
  if (__any_sync(0xffffffffu, !here)) {       // (for all lanes alike)
    if (lane == 0) sh.lost_row = row, sh.lost_count = count;
    __syncwarp();
    return make_float2(0.f, -1.f);
  }
  v = warp_merge(lane < ranks ? sh.part[p][lane] : make_float2(kFloor, 0.f));
  return v;
}

// By all threads of a cluster's blocks, behind the last exchange.  A block leaves at once: it has all parts of its last row, so nothing is on its way
// to it.  Not so one that gave up, and its shared memory has to stay until the others send no more: it waits until their threads have come here, then
// (with a limit) for what they sent last, and long enough that their stores have arrived too.  True in that case, for its first warp.
// (Arrivals that release those stores instead would cost every call 0.2 us.)
__device__ __forceinline__ bool exchange_end(Shared& sh) {
  asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  if (threadIdx.x >= 32 || sh.lost_row < 0) return false;
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&sh.arrived[sh.lost_count & 1]), phase = (uint32_t)(sh.lost_count >> 1) & 1u;
  const long long t0 = clock64();
  while (!parts_are_here(bar, phase) && clock64() - t0 < 1000000ll) {}
  while (clock64() - t0 < 200000ll) {}
  return true;
}

// The largest of a vector's values (NaN aside)
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
  uint32_t m;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  return m;
}
template <int DT> __device__ __forceinline__ float largest(uint4 v) {
  if constexpr (DT == JP_BF16) {
    const uint32_t m = max_pair(max_pair(v.x, v.y), max_pair(v.z, v.w));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  } else {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
}
// Values 2 q and 2 q + 1
template <int DT> __device__ __forceinline__ float2 value_pair(uint4 v, int q) {
  if constexpr (DT == JP_BF16) {
    const uint32_t w = q == 0 ? v.x : q == 1 ? v.y : q == 2 ? v.z : v.w;
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  } else {
    return q == 0 ? make_float2(__uint_as_float(v.x), __uint_as_float(v.y)) : make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
  }
}
// A vector's part of the running (maximum, sum); exponents and sums two at a time.
template <int DT> __device__ __forceinline__ void add_vector(uint4 v, float c, float& m, float& s) {
  constexpr int W = Vec<DT>::N;
  const float top = largest<DT>(v) * c;
  if (top > m) {
    s *= ex2_approx(m - top);
    m = top;
  }
  float2 e[W / 2];
#pragma unroll
  for (int q = 0; q < W / 2; ++q) {
    const float2 y = fma2(value_pair<DT>(v, q), make_float2(c, c), make_float2(-m, -m));
    e[q] = make_float2(ex2_approx(y.x), ex2_approx(y.y));
  }
#pragma unroll
  for (int o = 1; o < W / 2; o *= 2)
#pragma unroll
    for (int q = 0; q + o < W / 2; q += 2 * o) e[q] = add2(e[q], e[q + o]);
  s += e[0].x + e[0].y;
}
// The row's last elements, less than a vector
template <int DT> __device__ __forceinline__ void add_tail(const char* z, int64_t i, float c, float& m, float& s) {
  const float v = Vec<DT>::load_scalar(z, i), top = fmaxf(v * c, m);
  s = s * ex2_approx(m - top) + ex2_approx(fmaf(v, c, -top));
  m = top;
}
// Gradient of a vector: coef 1[v = x] - k 2^(z c - m), k = coef / s; `hit`: it holds the token.  (The token's place is written once more: as an index into
// the vector it would go through local memory.)
template <int DT> __device__ __forceinline__ void put_gradient(char* to, uint4 v, float c, float m, float k, float coef, bool hit, int x) {
  constexpr int W = Vec<DT>::N;
  auto at = [&](int q) {
    const float2 y = fma2(value_pair<DT>(v, q), make_float2(c, c), make_float2(-m, -m));
    return mul2(make_float2(ex2_approx(y.x), ex2_approx(y.y)), make_float2(-k, -k));
  };
  float g[W];
#pragma unroll
  for (int q = 0; q < W / 2; ++q) {
    const float2 t = at(q);
    g[2 * q] = t.x;
    g[2 * q + 1] = t.y;
  }
  stg_stream((uint4*)to, pack<DT>(g));
  if (hit) {
    const float2 t = at(x % W / 2);
    store_one<DT>(to, x % W, coef + ((x & 1) ? t.y : t.x));
  }
}

// A block's part of a row straight from memory, kUnroll vectors of a thread at a time.
template <int DT> __device__ __forceinline__ float2 row_sums(const char* z, int64_t v0, int64_t v1, float c) {
  float m = kFloor, s = 0.f;
  for (int64_t i0 = v0; i0 < v1; i0 += (int)blockDim.x * kUnroll) {
    uint4 v[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int64_t i = i0 + j * (int)blockDim.x + threadIdx.x;
      v[j] = i < v1 ? ld_row((const uint4*)z + i) : Vec<DT>::neg_inf();
    }
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) add_vector<DT>(v[j], c, m, s);
  }
  return make_float2(m, s);
}
template <int DT> __device__ __forceinline__ void row_gradient(const char* z, char* dz, int64_t v0, int64_t v1, float c, float m, float k, float coef, int64_t x) {
  for (int64_t i0 = v0; i0 < v1; i0 += (int)blockDim.x * kUnroll) {
    uint4 v[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int64_t i = i0 + j * (int)blockDim.x + threadIdx.x;
      if (i < v1) v[j] = ld_row((const uint4*)z + i);
    }
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int64_t i = i0 + j * (int)blockDim.x + threadIdx.x;
      if (i < v1) put_gradient<DT>(dz + i * 16, v[j], c, m, k, coef, i == x / Vec<DT>::N, (int)x);
    }
  }
}
template <int DT> __device__ __forceinline__ void tail_gradient(const char* z, char* dz, int64_t t, float c, float m, float k, float coef, int64_t x) {
  store_one<DT>(dz, t, (t == x ? coef : 0.f) - k * ex2_approx(fmaf(Vec<DT>::load_scalar(z, t), c, -m)));
}

template <int DT> __device__ __forceinline__ void row_zeros(char* dz, int64_t v0, int64_t v1, int64_t tail0, int64_t V) {
  for (int64_t i = v0 + threadIdx.x; i < v1; i += (int)blockDim.x) stg_stream((uint4*)dz + i, make_uint4(0u, 0u, 0u, 0u));
  if (tail0 + threadIdx.x < V) store_one<DT>(dz, tail0 + threadIdx.x, 0.f);
}

// Rows that take part: every block counts them by itself.
__device__ __forceinline__ double inverse_count(Shared& sh, const uint8_t* mask, int64_t T, int64_t n_valid) {
  if (n_valid > 0) return 1.0 / (double)n_valid;
  if (!mask) return 1.0 / (double)T;
  int n = 0;
  const int64_t head = (16 - ((uintptr_t)mask & 15)) & 15;
  const int64_t first = head < T ? head : T, vecs = (T - first) / 16;
  const uint4* m = (const uint4*)(mask + first);
  for (int64_t i = threadIdx.x; i < vecs; i += (int)blockDim.x) {
    const uint4 v = m[i];
    n += __popc(__vcmpne4(v.x, 0u) & 0x01010101u) + __popc(__vcmpne4(v.y, 0u) & 0x01010101u) +
         __popc(__vcmpne4(v.z, 0u) & 0x01010101u) + __popc(__vcmpne4(v.w, 0u) & 0x01010101u);
  }
  if ((int64_t)threadIdx.x < first) n += mask[threadIdx.x] != 0;
  if (first + vecs * 16 + threadIdx.x < T) n += mask[first + vecs * 16 + threadIdx.x] != 0;
  n = __reduce_add_sync(0xffffffffu, n);
  if ((threadIdx.x & 31) == 0) sh.count[threadIdx.x >> 5] = n;
  __syncthreads();
  int64_t all = 0;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) all += sh.count[w];
  return all > 0 ? 1.0 / (double)all : 0.0;
}

// Until at most n groups of copies are under way; n is a constant where it is called (the instruction takes no other).
__device__ __forceinline__ void wait_copies(int n) {
  switch (n) {
#define JP_WAIT(N) case N: asm volatile("cp.async.wait_group " #N ";" ::: "memory"); break;
    JP_WAIT(1) JP_WAIT(2) JP_WAIT(3) JP_WAIT(4) JP_WAIT(5) JP_WAIT(6) JP_WAIT(7) JP_WAIT(8) JP_WAIT(9) JP_WAIT(10) JP_WAIT(11) JP_WAIT(12) JP_WAIT(13)
#undef JP_WAIT
    default: asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// A row's inputs beside its logits, read before its sum: their time covers the loads (and nobody has written the row yet).
struct RowInputs { float zx, adv, old, ref, weight; };

// What becomes of a row's (maximum, sum), by one warp: two of its lanes take the two exponentials at the same time.
template <int MODE>
__device__ __forceinline__ void row_scalars(const LossArgs& A, Shared& sh, int64_t row, bool writes, float2 t, const RowInputs& in, double inv_n) {
  const int lane = threadIdx.x & 31;
  const double none = __longlong_as_double(0x7ff8000000000000ll);
  if (t.y < 0.f) {                            // the blocks' parts did not arrive: NaN in the loss and in the gradient
    if (lane == 0) {
      sh.coef = sh.k_over_s = (float)none;
      if (MODE == kPrefSums) {
        if (writes) A.row_lp[row] = none, A.row_used[row] = 1, A.row_sum[row] = t;
      } else if (writes) {
        A.term[row] = A.kl_term[row] = none;
      }
    }
    return;
  }
  // in log2 first: c is log2(e) / tau in fp32, and so are m and the exponents behind the sum; c_to_nat takes its rounding back
  const double lp = ((double)in.zx * (double)A.c - (double)t.x - log2((double)t.y)) * A.c_to_nat;
  const bool usable = t.x > kFloor && t.x < 3.4e38f && t.y < 3.4e38f;        // (NaN and infinities end in the sum)
  if (MODE == kPrefSums) {
    const bool fine = usable && lp > -3.0e38;
    if (writes && lane == 0) {
      A.row_lp[row] = fine ? lp : 0.0;
      A.row_used[row] = fine;
      A.row_sum[row] = t;
      if (A.out_logp) A.out_logp[row] = fine ? (float)lp : 0.f;
      if (A.out_state) A.out_state[row] = fine ? 1 : 3;
    }
    return;
  }
  const double d = (double)in.ref - lp, e = exp(lane == 1 ? d : lp - (double)in.old);
  const double r = usable ? __shfl_sync(0xffffffffu, e, 0) : none, e1 = __shfl_sync(0xffffffffu, e, 1) - 1.0;
  const double a = in.adv, plain = -a * r;
  double loss = plain, slope = plain, kl = 0.0;
  bool live = true;
  if (A.clip) {
    const double clipped = -a * fmin(fmax(r, 1.0 - (double)A.eps_lo), 1.0 + (double)A.eps_hi);
    live = !(plain < clipped);
    if (!live) loss = clipped, slope = 0.0;
  }
  if (A.logp_ref) {
    // e - 1 is off by 2^-53, of which d^2 / 2 next to 0 would be nothing: there, the series, off by 2^-48 of itself at most, and never below 0
    const bool near = fabs(d) < 0x1p-10;
    kl = near ? d * d * fma(d, fma(d, fma(d, 1.0 / 120, 1.0 / 24), 1.0 / 6), 0.5) : e1 - d;
    slope -= (double)A.kl_coef * (near ? kl + d : e1);
  }
  const double wt = (double)in.weight * inv_n;
  const float co = (float)(wt * slope * A.grad_scale);
  const bool fine = isfinite(wt * loss) && isfinite((float)kl) && isfinite(co) && !isnan(r);
  if (lane == 0) {
    sh.coef = fine ? co : 0.f;
    sh.k_over_s = fine ? co / t.y : 0.f;
    if (writes) {
      if (A.out_logp) A.out_logp[row] = fine ? (float)lp : 0.f;
      if (A.out_kl) A.out_kl[row] = fine ? (float)kl : 0.f;
      if (A.out_state) A.out_state[row] = fine ? (live ? 1 : 2) : 3;
      A.term[row] = fine ? wt * loss : 0.0;
      A.kl_term[row] = fine ? wt * kl : 0.0;
    }
  }
}

// A row that takes no part: what is written of it beside its gradient.
template <int MODE> __device__ __forceinline__ void row_without(const LossArgs& A, int64_t row) {
  if (MODE == kPrefGrad) return;
  if (A.out_logp) A.out_logp[row] = 0.f;
  if (A.out_state) A.out_state[row] = 0;
  if (MODE == kPrefSums) {
    A.row_lp[row] = 0.0;
    A.row_used[row] = 0;
  } else {
    if (A.out_kl) A.out_kl[row] = 0.f;
    A.term[row] = 0.0;
    A.kl_term[row] = 0.0;
  }
}

// kPolicy: NV vectors a thread hold a block's part of a row; NV = 0: any row, straight from memory, twice.
// The others: a ring of NV vectors a thread; rows of any length, in whole turns of the ring.
template <int DT, int MODE, int NV, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) loss_rows_kernel(LossArgs A) {
  extern __shared__ uint4 places[];           // [NV][threads]: each thread its own
  __shared__ Shared sh;
  constexpr int W = Vec<DT>::N, ES = Vec<DT>::ESIZE;
  constexpr bool STREAM = MODE != kPolicy, GRAD = MODE == kPolicy || MODE == kPrefGrad;
  const int ranks = A.cluster, rank = blockIdx.x % ranks, clusters = gridDim.x / ranks;
  if (ranks > 1) exchange_start(sh);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t vecs = A.V / W, each = (vecs + ranks - 1) / ranks;
  const int64_t v0 = each * rank < vecs ? each * rank : vecs, v1 = v0 + each < vecs ? v0 + each : vecs;
  const int64_t tail0 = rank == ranks - 1 ? vecs * W : A.V;       // the last block has what is left behind the vectors
  const int mine = (int)(v1 - v0) - (int)threadIdx.x;             // vector i is there if i * kThreads < mine (a row has less than 2^29)
  const int turns = NV > 0 ? (int)((v1 - v0 + NV * kThreads - 1) / (NV * kThreads > 0 ? NV * kThreads : 1)) : 0;       // of the ring, a row
  const uint32_t place = (uint32_t)__cvta_generic_to_shared(places) + threadIdx.x * 16;
  const int64_t first = (v0 + threadIdx.x) * 16;                  // bytes from a row's start to the thread's first vector
  int64_t lo = 0, hi = A.T;
  if (MODE == kPrefSums) {
    lo = A.seq_start[0];
    hi = A.seq_start[2 * A.P];
  }
  // the n-th row of all; gradients of pairs from the last row on: the end of the logits is what L2 still has from their sums
  auto nth = [&](int64_t n) { return MODE == kPrefGrad ? A.T - 1 - n : n; };
  // the token of the n-th row, -1 if it takes no part
  auto token_of = [&](int64_t n) {
    if (n >= A.T) return -1;
    const int64_t row = nth(n);
    int32_t x = A.tokens[row];
    if (MODE == kPrefGrad) return A.row_coef[row] != 0.f ? x : -1;
    if (A.mask != nullptr && A.mask[row] == 0) x = -1;
    if (MODE == kPrefSums && (row < lo || row >= hi)) x = -1;
    return x < A.V ? x : -1;
  };
  // where the thread's first vector of the n-th row is, and `mine` of it (0 behind the last row)
  auto source = [&](int64_t n) { return (const char*)A.z + (n < A.T ? nth(n) : 0) * A.ld * ES + first; };
  auto mine_of = [&](int64_t n) { return n < A.T ? mine : 0; };
  // vector i of a row, or an empty group of copies
  auto fetch = [&](const char* row, int have, int slot, int i) {
    if (i * kThreads < have)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(place + slot * kThreads * 16), "l"(row + (int64_t)i * (kThreads * 16)) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // `next`: the next of this cluster's rows that takes part, with its token; `ahead`: the token of the row behind it, read a row's time before
  // it is needed
  int64_t n = blockIdx.x / ranks, next = n;
  int32_t token, ahead = token_of(next);
  auto advance = [&]() {
    while (ahead < 0 && next < A.T) {
      next += clusters;
      ahead = token_of(next);
    }
    if (next > A.T) next = A.T;
    token = ahead;
    ahead = token_of(next + clusters);
  };
  advance();
#pragma unroll
  for (int i = 0; i < NV; ++i) fetch(source(next), mine_of(next), i, i);
  const double inv_n = MODE == kPolicy || MODE == kPolicyNoGrad ? inverse_count(sh, A.mask, A.T, A.n_valid) : 0.0;
  for (int64_t count = 0;; ++count) {
    for (; n < next; n += clusters) {         // rows that take no part
      if (threadIdx.x == 0 && rank == 0) row_without<MODE>(A, nth(n));
      if (GRAD) row_zeros<DT>((char*)A.dz + nth(n) * A.ld_d * ES, v0, v1, tail0, A.V);
    }
    if (next >= A.T) break;
    const int64_t row = nth(next), x = token;
    next += clusters;
    advance();
    const char* z = (const char*)A.z + row * A.ld * ES;
    char* dz = (char*)A.dz + row * A.ld_d * ES;
    const char* const next_row = source(next);
    const int next_mine = mine_of(next);
    float m = 0.f, k = 0.f, coef = 0.f;
    if (MODE == kPrefGrad) {
      coef = A.row_coef[row];
      const float2 r = A.row_sum[row];
      m = r.x;
      k = coef / r.y;
    } else {
      RowInputs in{0.f, 0.f, 0.f, 0.f, 1.f};
      if (threadIdx.x < 32) {
        in.zx = Vec<DT>::load_scalar(z, x);
        if (MODE != kPrefSums) {
          in.adv = A.advantages[row];
          in.old = A.logp_old[row];
          if (A.logp_ref) in.ref = A.logp_ref[row];
          if (A.token_weight) in.weight = A.token_weight[row];
        }
      }
      float top = kFloor, sum = 0.f;
      if constexpr (NV == 0) {
        const float2 t = row_sums<DT>(z, v0, v1, A.c);
        top = t.x;
        sum = t.y;
      } else {
        for (int turn = 0; turn < (STREAM ? turns : 1); ++turn) {
#pragma unroll
          for (int u = 0; u < NV; ++u) {
            const int i = turn * NV + u;
            wait_copies(STREAM ? NV - 1 : NV - 1 - u);
            uint4 v;
            const bool have = i * kThreads < mine;
            if (have) v = lds16(place + u * kThreads * 16);
            if (STREAM) {
              if (turn + 1 < turns) fetch(z + first, mine, u, i + NV);
              else fetch(next_row, next_mine, u, u);
            }
            if (have) add_vector<DT>(v, A.c, top, sum);
          }
        }
      }
      if (tail0 + threadIdx.x < A.V) add_tail<DT>(z, tail0 + threadIdx.x, A.c, top, sum);
      const float2 t = warp_merge(make_float2(top, sum));
      if ((threadIdx.x & 31) == 0) sh.warp[count & 1][threadIdx.x >> 5] = t;
      __syncthreads();
      if (threadIdx.x < 32) {                 // (without a gradient the others go on with the next row)
        // the token's logit has arrived before the other blocks hear of this one: they may write the gradient over it
        if (MODE == kPolicy) asm volatile("{.reg .f32 t;\n\tmov.f32 t, %0;}" ::"f"(in.zx) : "memory");
        const float2 all = row_total(sh, rank, ranks, count, row);
        if (MODE == kPolicy && threadIdx.x == 0) sh.top = all.x;
        row_scalars<MODE>(A, sh, row, rank == 0, all, in, inv_n);
      }
      if (MODE == kPolicy) {
        __syncthreads();
        m = sh.top;
        coef = sh.coef;
        k = sh.k_over_s;
      }
    }
    if (GRAD) {
      if constexpr (NV == 0) {
        if (coef != 0.f) row_gradient<DT>(z, dz, v0, v1, A.c, m, k, coef, x);
        else row_zeros<DT>(dz, v0, v1, A.V, A.V);
      } else {
        const int token_at = (int)(x / W - v0) - (int)threadIdx.x;
        for (int turn = 0; turn < (STREAM ? turns : 1); ++turn) {
#pragma unroll
          for (int u = 0; u < NV; ++u) {
            const int i = turn * NV + u;
            if (STREAM) wait_copies(NV - 1);
            uint4 v;
            const bool have = i * kThreads < mine;
            if (have) v = lds16(place + u * kThreads * 16);
            if (STREAM && turn + 1 < turns) fetch(z + first, mine, u, i + NV);
            else fetch(next_row, next_mine, u, u);
            if (have) {
              char* const to = dz + first + (int64_t)i * (kThreads * 16);
              if (coef != 0.f) put_gradient<DT>(to, v, A.c, m, k, coef, i * kThreads == token_at, (int)x);
              else stg_stream((uint4*)to, make_uint4(0u, 0u, 0u, 0u));
            }
          }
        }
      }
      if (tail0 + threadIdx.x < A.V) {
        if (coef != 0.f) tail_gradient<DT>(z, dz, tail0 + threadIdx.x, A.c, m, k, coef, x);
        else store_one<DT>(dz, tail0 + threadIdx.x, 0.f);
      }
    }
    n += clusters;
  }
  // a block that gave up: NaN in the loss, whatever the row's first block made of it
  if (MODE != kPrefGrad && ranks > 1 && exchange_end(sh) && threadIdx.x == 0) {
    const double none = __longlong_as_double(0x7ff8000000000000ll);
    if (MODE == kPrefSums) A.row_lp[sh.lost_row] = none, A.row_used[sh.lost_row] = 1;
    else A.term[sh.lost_row] = none;
  }
}

// Two blocks, the second of which sends its part only after the first one has given up: the part has to find the first one's memory, and both end.
__global__ void __launch_bounds__(64) exchange_selftest_kernel(long long limit, int32_t* status) {
  __shared__ Shared sh;
  const int rank = blockIdx.x;
  exchange_start(sh);
  if (threadIdx.x < 32) {
    if (threadIdx.x < 2) sh.warp[0][threadIdx.x] = make_float2(3.f + rank, 1.f);
    __syncwarp();
    const long long t0 = clock64(), late = limit / 4 * 5 + 4000000ll;
    while (rank == 1 && clock64() - t0 < late) {}
    const float2 t = row_total(sh, rank, 2, 0, 0, limit);
    if (threadIdx.x == 0 && (rank == 0 ? t.y >= 0.f : t.x != 4.f || t.y != 3.f)) atomicExch(status, (int)JP_ERR_CUDA);
  }
  if (exchange_end(sh) && threadIdx.x == 0 && (sh.part[0][1].x != 4.f || sh.part[0][1].y != 2.f)) atomicExch(status, (int)JP_ERR_CUDA);
}

__device__ __forceinline__ double warp_add(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over a block of 1024 threads in a fixed order, in thread 0.
__device__ __forceinline__ double block_add(double v, double* sh) {
  v = warp_add(v);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = threadIdx.x < 32 ? sh[threadIdx.x] : 0.0;
  if (threadIdx.x < 32) v = warp_add(v);
  __syncthreads();
  return v;
}

__global__ void __launch_bounds__(1024) policy_sum_kernel(LossArgs A) {
  __shared__ double sh[32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  double a = 0.0, b = 0.0;
  for (int64_t i = threadIdx.x; i < A.T; i += 1024) {
    a += A.term[i];
    b += A.kl_term[i];
  }
  a = block_add(a, sh);
  b = block_add(b, sh);
  if (threadIdx.x == 0) {
    A.out_loss[0] = (float)(a + (double)A.kl_coef * b);
    A.out_loss[1] = (float)a;
    A.out_loss[2] = (float)b;
  }
}

// The pairs, by one block: a warp a sequence's sum, a thread a pair's loss and slope, then every row's coefficient.
__global__ void __launch_bounds__(1024) preference_pairs_kernel(LossArgs A) {
  __shared__ double sh[32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31;
  for (int64_t s = threadIdx.x >> 5; s < 2 * A.P; s += 32) {
    int64_t a = A.seq_start[s], b = A.seq_start[s + 1];
    a = a < 0 ? 0 : a;
    b = b > A.T ? A.T : b;
    double sum = 0.0, n = 0.0;
    for (int64_t i = a + lane; i < b; i += 32) {
      sum += A.row_lp[i];
      n += A.row_used[i] ? 1.0 : 0.0;
    }
    sum = warp_add(sum);
    n = warp_add(n);
    if (lane == 0) {
      const double per = A.average ? (n > 0.0 ? 1.0 / n : 0.0) : 1.0;
      A.seq_sum[s] = sum * per;
      A.seq_per[s] = per;
    }
  }
  __syncthreads();
  double loss = 0.0;
  for (int64_t p = threadIdx.x; p < A.P; p += 1024) {
    double gap = A.seq_sum[2 * p] - A.seq_sum[2 * p + 1];
    if (A.ref_logp) gap -= (double)A.ref_logp[2 * p] - (double)A.ref_logp[2 * p + 1];
    const double h = (double)A.beta * gap - (double)A.margin, e = A.label_smoothing;
    const double up = log1p(exp(-fabs(h)));
    // (a side without weight adds nothing, also where h is infinite)
    loss += (e < 1.0 ? (1.0 - e) * (up + fmax(-h, 0.0)) : 0.0) + (e > 0.0 ? e * (up + fmax(h, 0.0)) : 0.0);
    // (sigma of either sign without taking 1 - sigma, which would lose the small one)
    const double small = exp(-fabs(h)) / (1.0 + exp(-fabs(h))), large = 1.0 / (1.0 + exp(-fabs(h)));
    const double slope = (double)A.beta * A.grad_scale / (double)A.P * (e * (h > 0.0 ? large : small) - (1.0 - e) * (h > 0.0 ? small : large));
    if (A.out_margin) A.out_margin[p] = (float)h;
    for (int side = 0; side < 2; ++side) {
      const int64_t s = 2 * p + side;
      if (A.out_seq_logp) A.out_seq_logp[s] = (float)A.seq_sum[s];
      A.seq_per[s] *= side ? -slope : slope;
    }
  }
  loss = block_add(loss, sh);                 // (and a barrier: seq_per is read below)
  if (threadIdx.x == 0) A.out_loss[0] = (float)(loss / (double)(A.P > 0 ? A.P : 1));
  if (!A.dz) return;
  for (int64_t i = threadIdx.x; i < A.T; i += 1024) {
    float coef = 0.f;
    if (A.row_used[i]) {                      // the sequence of the row: the last one that starts at or before it
      int64_t lo = 0, hi = 2 * A.P;
      while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (A.seq_start[mid] <= i) lo = mid;
        else hi = mid;
      }
      coef = (float)A.seq_per[lo];
    }
    A.row_coef[i] = isfinite(coef) ? coef : 0.f;
  }
}

constexpr int kMostVectors = 14;              // a thread: of blocks of 512 threads two fit an SM (112 KB each), of 256 threads three

template <class K>
cudaError_t launch(K kernel, const LossArgs& a, unsigned grid, unsigned threads, int cluster, int smem, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

// Clusters of c blocks that the GPU holds at once (fewer than its SMs' threads would, where c does not divide what shares their memory, or the memory of a
// block does not go so often into an SM's); asked once for each kernel, size and device, since the answer is always the same.
template <auto kernel, int kThreads> int clusters_at_once(int c, int smem, int sms) {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices][kMaxCluster + 1];
  int device = 0, n = 0;
  const bool keep = cudaGetDevice(&device) == cudaSuccess && device < kDevices;
  if (keep && (n = known[device][c].load(std::memory_order_relaxed)) > 0) return n;
  cudaError_t e;
  if (c == 1) {
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kThreads, smem);
    n *= sms;
  } else {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(sms * (1024 / kThreads) / c * c));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = c;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
  }
  if (e != cudaSuccess || n < 1) {
    cudaGetLastError();
    return sms * (1024 / kThreads) / c;
  }
  if (keep) known[device][c].store(n, std::memory_order_relaxed);
  return n;
}

template <int NV, int kThreads, int DT, int MODE> cudaError_t rows_of(const LossArgs& a, cudaStream_t s, int sms) {
  constexpr auto kernel = loss_rows_kernel<DT, MODE, NV, kThreads>;
  constexpr int smem = NV * kThreads * 16;
  if (smem > 0) {
    const cudaError_t e = allow_shared_memory<kernel>(smem);
    if (e != cudaSuccess) return e;
  }
  const int64_t most = clusters_at_once<kernel, kThreads>(a.cluster, smem, sms), clusters = most < a.T ? most : a.T;
  return launch(kernel, a, (unsigned)(clusters * a.cluster), kThreads, a.cluster, smem, s);
}

// Blocks that share a row: enough that all SMs have work where rows are few, and `most` vectors a thread (0: any number) hold it; not more than
// leave every thread a vector.
int cluster_for(int64_t T, int64_t vecs, int threads, int most, int sms) {
  int c = 1;
  while (c < kMaxCluster && (T * c * 2 <= (int64_t)sms * (1024 / threads) || (most > 0 && vecs > (int64_t)c * threads * most)) && vecs >= 2 * c * threads) c *= 2;
  return c;
}

template <int DT, int MODE, int kThreads> cudaError_t resident(LossArgs a, int64_t vecs, cudaStream_t s, int sms) {
  const int64_t per = (vecs + a.cluster - 1) / a.cluster;
  if constexpr (kThreads == 256) {            // (blocks of 512 start where those end)
    if (per <= 1 * kThreads) return rows_of<1, kThreads, DT, MODE>(a, s, sms);
    if (per <= 2 * kThreads) return rows_of<2, kThreads, DT, MODE>(a, s, sms);
    if (per <= 4 * kThreads) return rows_of<4, kThreads, DT, MODE>(a, s, sms);
    if (per <= 7 * kThreads) return rows_of<7, kThreads, DT, MODE>(a, s, sms);
  }
  if (per <= 10 * kThreads) return rows_of<10, kThreads, DT, MODE>(a, s, sms);
  // With 13 vectors four blocks of 256 threads fit an SM (bf16, us, three in brackets: 4096 x 24,000 83 (87), 4096 x 100,277 345 (397), 2048 x 200,064 337
  // (397); fp32 2048 x 50,257 150 (177)); three are better for fp32 rows of one block (8192 x 12,000 136, four 143),
  // and for what 14 vectors hold and 13 do not (bf16 4096 x 28,000 98, as two blocks of 7 vectors 106; 4096 x 56,000 192 and 211).
  if constexpr (kThreads == 256)
    if (per <= 13 * kThreads && (DT == JP_BF16 || a.cluster > 1)) return rows_of<13, kThreads, DT, MODE>(a, s, sms);
  return rows_of<kMostVectors, kThreads, DT, MODE>(a, s, sms);
}

template <int DT, int MODE> cudaError_t rows(LossArgs a, cudaStream_t s, int sms) {
  const int64_t vecs = (a.V + Vec<DT>::N - 1) / Vec<DT>::N;
  // Many short rows: a row's latency (barriers, its scalars) decides, so more of them at a time in smaller blocks, where four rows an SM are not
  // all of them.  bf16, us, with blocks of 256 and 512 threads in brackets: policy loss 65,536 x 1000 144 (242), 65,536 x 2000 173 (264), 30,000 x
  // 5003 151 (190); preference loss, 64 pairs of up to 512 rows, V = 1000 151 (449), 32 of 256, V = 5003 97 (161).
  const bool narrow = a.T > (int64_t)sms * 4;
  a.cluster = 1;
  if constexpr (MODE != kPolicy) {
    if (narrow && vecs <= 64 * 4) return rows_of<2, 64, DT, MODE>(a, s, sms);
    if (narrow && vecs <= 128 * 8) return rows_of<8, 128, DT, MODE>(a, s, sms);
    a.cluster = cluster_for(a.T, vecs, 512, 0, sms);
    return vecs <= (int64_t)a.cluster * 2 * 512 ? rows_of<2, 512, DT, MODE>(a, s, sms) : rows_of<8, 512, DT, MODE>(a, s, sms);
  } else {
    if (narrow && vecs <= 64 * 2) return rows_of<2, 64, DT, MODE>(a, s, sms);
    if (narrow && vecs <= 64 * 4) return rows_of<4, 64, DT, MODE>(a, s, sms);
    if (narrow && vecs <= 128 * 7) return rows_of<7, 128, DT, MODE>(a, s, sms);
    // four rows' blocks an SM (three with 14 vectors a thread) where eight blocks of 256 threads hold a row, two where it takes eight of 512
    if (vecs <= (int64_t)kMaxCluster * 256 * kMostVectors) {
      a.cluster = cluster_for(a.T, vecs, 256, kMostVectors, sms);
      return resident<DT, MODE, 256>(a, vecs, s, sms);
    }
    a.cluster = kMaxCluster;
    if (vecs <= (int64_t)kMaxCluster * 512 * kMostVectors) return resident<DT, MODE, 512>(a, vecs, s, sms);
    return rows_of<0, 512, DT, MODE>(a, s, sms);
  }
}
template <int MODE> cudaError_t rows(const LossArgs& a, cudaStream_t s, int sms) {
  return a.dtype == JP_BF16 ? rows<JP_BF16, MODE>(a, s, sms) : rows<JP_F32, MODE>(a, s, sms);
}

}  // namespace

cudaError_t launch_exchange_selftest(long long limit_cycles, int32_t* status, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(64);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 2;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, exchange_selftest_kernel, limit_cycles, status);
}

namespace {
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
}  // namespace

size_t policy_workspace_bytes(int64_t T) { return 2 * up256((size_t)T * 8); }

cudaError_t launch_policy(LossArgs a, void* workspace, cudaStream_t s, int sms) {
  a.term = (double*)workspace;
  a.kl_term = (double*)((char*)workspace + up256((size_t)a.T * 8));
  const cudaError_t e = a.dz ? rows<kPolicy>(a, s, sms) : rows<kPolicyNoGrad>(a, s, sms);
  return e != cudaSuccess ? e : launch(policy_sum_kernel, a, 1, 1024, 1, 0, s);
}

size_t preference_workspace_bytes(int64_t T, int64_t P) {
  return 2 * up256((size_t)T * 8) + up256((size_t)T * 4) + up256((size_t)T) + 2 * up256((size_t)P * 16);
}

cudaError_t launch_preference(LossArgs a, void* workspace, cudaStream_t s, int sms, int* n_launch) {
  char* w = (char*)workspace;
  auto take = [&](size_t n) { char* p = w; w += up256(n); return p; };
  a.row_lp = (double*)take((size_t)a.T * 8);
  a.row_sum = (float2*)take((size_t)a.T * 8);
  a.row_coef = (float*)take((size_t)a.T * 4);
  a.row_used = (uint8_t*)take((size_t)a.T);
  a.seq_sum = (double*)take((size_t)a.P * 16);
  a.seq_per = (double*)take((size_t)a.P * 16);
  *n_launch = 0;
  cudaError_t e = rows<kPrefSums>(a, s, sms);
  if (e == cudaSuccess) { *n_launch = 1; e = launch(preference_pairs_kernel, a, 1, 1024, 1, 0, s); }
  if (e == cudaSuccess) { *n_launch = 2; if (a.dz) e = rows<kPrefGrad>(a, s, sms); }
  if (e == cudaSuccess && a.dz) *n_launch = 3;
  return e;
}

}  // namespace jp
