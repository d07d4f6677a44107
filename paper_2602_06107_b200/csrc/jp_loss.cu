// Losses of one model over its logits [T, V], with the gradient of the logits: the clipped policy loss with a KL term, and the preference
// loss of pairs of sequences.  For row t with sampled token x, temperature tau and p = softmax(z / tau):
//
//   lp = z_x / tau - log sum_v exp(z_v / tau),   dL/dz_v = k (1[v = x] - p_v) / tau,   k = dL/dlp
//   policy      r = exp(lp - lp_old), d = lp_ref - lp:  L = sum_t c_t (max(-A r, -A clip(r)) + beta (exp(d) - d - 1)),
//               k = c (-A r [unclipped branch] + beta (1 - exp(d)))
//   preference  S = sum or mean of a sequence's lp, h = beta ((S - R)_chosen - (S - R)_rejected) - margin:
//               L = mean over pairs of -(1 - e) log sigma(h) - e log sigma(-h),  k = +-(beta / P) (e sigma(h) - (1 - e) sigma(-h))
//
// Bound by HBM.  The policy loss has a row's k as soon as the row's sum is known, so sum and gradient are one launch: the row is read
// twice, the second time from L2, and HBM sees one read and one write.  The preference loss needs both sequences of a pair first: a pass
// for the sums, one for the gradients.  A row is shared by the blocks of a cluster; their (maximum, sum) pairs meet in shared memory.
// Sums of exponentials are fp32 of at most a few hundred terms a thread (in 2^x of z log2(e) / tau, relative to a running maximum), the row's
// scalars fp64: the clip is a decision, and exp(d) - d - 1 cancels.
#include "jp_common.cuh"
#include "jp_internal.h"

namespace jp {
namespace {

constexpr int kThreads = 512;
constexpr int kBlocksPerSm = 2;
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

// (maximum, sum of 2^(y - maximum)) of two parts
__device__ __forceinline__ float2 merge(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  return make_float2(m, a.y * ex2_approx(a.x - m) + b.y * ex2_approx(b.x - m));
}

struct Shared {
  float2 warp[kThreads / 32];
  float2 part[2][kMaxCluster];                // of the cluster's blocks, by the parity of the row's number
  float k_over_s, coef;
  int count[kThreads / 32];
  double inv_n;
};

// The row's (maximum, sum) in all threads of all blocks of the cluster.
__device__ __forceinline__ float2 cluster_total(Shared& sh, float2 v, int rank, int ranks, int& parity) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = merge(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
  if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5] = v;
  __syncthreads();
  v = sh.warp[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) v = merge(v, sh.warp[w]);
  if (ranks == 1) return v;
  if ((int)threadIdx.x < ranks) {             // to the place of this block in every block of the cluster
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(&sh.part[parity][rank])), "r"((uint32_t)threadIdx.x));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(v.x), "f"(v.y) : "memory");
  }
  // (the places of the next row are others, and nobody is two rows ahead: one barrier a row)
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
  v = sh.part[parity][0];
  for (int r = 1; r < ranks; ++r) v = merge(v, sh.part[parity][r]);
  parity ^= 1;
  return v;
}

template <int DT> __device__ __forceinline__ float2 row_sums(const char* z, int64_t v0, int64_t v1, int64_t tail0, int64_t V, float c) {
  constexpr int W = Vec<DT>::N;
  float m = kFloor, s = 0.f;
  for (int64_t i0 = v0; i0 < v1; i0 += kThreads * kUnroll) {
    uint4 v[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int64_t i = i0 + j * kThreads + threadIdx.x;
      v[j] = i < v1 ? ld_row((const uint4*)z + i) : Vec<DT>::neg_inf();
    }
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const float top = Vec<DT>::vmax(v[j]) * c;
      if (top > m) {
        s *= ex2_approx(m - top);
        m = top;
      }
      float e[W];
#pragma unroll
      for (int q = 0; q < W; ++q) e[q] = ex2_approx(fmaf(Vec<DT>::get(v[j], q), c, -m));
#pragma unroll
      for (int o = 1; o < W; o *= 2)
#pragma unroll
        for (int q = 0; q + o < W; q += 2 * o) e[q] += e[q + o];
      s += e[0];
    }
  }
  if (tail0 + threadIdx.x < V) {              // the row's last elements, less than a vector
    const float y = Vec<DT>::load_scalar(z, tail0 + threadIdx.x) * c, top = fmaxf(y, m);
    s = s * ex2_approx(m - top) + ex2_approx(fmaf(Vec<DT>::load_scalar(z, tail0 + threadIdx.x), c, -top));
    m = top;
  }
  return make_float2(m, s);
}

// Gradient of the block's part of a row: coef (1[v = x] - p_v), p_v = 2^(z c - m) / s, k = coef / s.
template <int DT> __device__ __forceinline__ void row_gradient(const char* z, char* dz, int64_t v0, int64_t v1, int64_t tail0, int64_t V, float c,
                                                               float m, float k, float coef, int64_t x) {
  constexpr int W = Vec<DT>::N;
  for (int64_t i0 = v0; i0 < v1; i0 += kThreads * kUnroll) {
    uint4 v[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int64_t i = i0 + j * kThreads + threadIdx.x;
      if (i < v1) v[j] = ld_row((const uint4*)z + i);
    }
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      const int64_t i = i0 + j * kThreads + threadIdx.x;
      if (i < v1) {
        float g[W];
#pragma unroll
        for (int q = 0; q < W; ++q) {
          g[q] = -k * ex2_approx(fmaf(Vec<DT>::get(v[j], q), c, -m));
          if (i * W + q == x) g[q] += coef;
        }
        stg_stream((uint4*)dz + i, pack<DT>(g));
      }
    }
  }
  const int64_t t = tail0 + threadIdx.x;
  if (t < V) store_one<DT>(dz, t, (t == x ? coef : 0.f) - k * ex2_approx(fmaf(Vec<DT>::load_scalar(z, t), c, -m)));
}

template <int DT> __device__ __forceinline__ void row_zeros(char* dz, int64_t v0, int64_t v1, int64_t tail0, int64_t V) {
  for (int64_t i = v0 + threadIdx.x; i < v1; i += kThreads) stg_stream((uint4*)dz + i, make_uint4(0u, 0u, 0u, 0u));
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
  for (int64_t i = threadIdx.x; i < vecs; i += kThreads) {
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
  for (int w = 0; w < kThreads / 32; ++w) all += sh.count[w];
  return all > 0 ? 1.0 / (double)all : 0.0;
}

template <int DT, int MODE>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) loss_rows_kernel(LossArgs A) {
  __shared__ Shared sh;
  constexpr int W = Vec<DT>::N, ES = Vec<DT>::ESIZE;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int ranks = A.cluster, rank = blockIdx.x % ranks, clusters = gridDim.x / ranks;
  const int64_t vecs = A.V / W, each = (vecs + ranks - 1) / ranks;
  const int64_t v0 = each * rank < vecs ? each * rank : vecs, v1 = v0 + each < vecs ? v0 + each : vecs;
  const int64_t tail0 = rank == ranks - 1 ? vecs * W : A.V;       // the last block has what is left behind the vectors
  const double inv_n = MODE == kPolicy || MODE == kPolicyNoGrad ? inverse_count(sh, A.mask, A.T, A.n_valid) : 0.0;
  int parity = 0;
  for (int64_t n = blockIdx.x / ranks; n < A.T; n += clusters) {
    // (gradients of pairs from the last row on: the end of the logits is what L2 still has from their sums)
    const int64_t row = MODE == kPrefGrad ? A.T - 1 - n : n;
    const char* z = (const char*)A.z + row * A.ld * ES;
    char* dz = (char*)A.dz + row * A.ld_d * ES;
    const int64_t x = A.tokens[row];
    bool on = (A.mask == nullptr || A.mask[row] != 0) && x >= 0 && x < A.V;
    float m = 0.f, k = 0.f, coef = 0.f;
    if (MODE == kPrefGrad) {
      coef = A.row_coef[row];
      if (coef != 0.f) {
        const float2 r = A.row_sum[row];
        m = r.x;
        k = coef / r.y;
      }
    } else {
      if (MODE == kPrefSums) on = on && row >= A.seq_start[0] && row < A.seq_start[2 * A.P];
      if (!on) {
        if (threadIdx.x == 0 && rank == 0) {
          if (A.out_logp) A.out_logp[row] = 0.f;
          if (A.out_state) A.out_state[row] = 0;
          if (MODE == kPrefSums) A.row_lp[row] = 0.0, A.row_used[row] = 0;
          else {
            if (A.out_kl) A.out_kl[row] = 0.f;
            A.term[row] = 0.0;
            A.kl_term[row] = 0.0;
          }
        }
      } else {
        float zx = 0.f, adv = 0.f, old = 0.f, ref = 0.f, weight = 1.f;
        if (threadIdx.x == 0) {               // (read before the sums: their time covers the loads; nobody has written the row yet)
          zx = Vec<DT>::load_scalar(z, x);
          if (MODE != kPrefSums) {
            adv = A.advantages[row];
            old = A.logp_old[row];
            if (A.logp_ref) ref = A.logp_ref[row];
            if (A.token_weight) weight = A.token_weight[row];
          }
        }
        const float2 t = cluster_total(sh, row_sums<DT>(z, v0, v1, tail0, A.V, A.c), rank, ranks, parity);
        m = t.x;
        if (threadIdx.x == 0) {
          // in log2 first: c is log2(e) / tau in fp32, and so are m and the exponents behind the sum; c_to_nat takes its rounding back
          const double lp = ((double)zx * (double)A.c - (double)t.x - log2((double)t.y)) * A.c_to_nat;
          const bool usable = t.x > kFloor && t.x < 3.4e38f && t.y < 3.4e38f;        // (NaN and infinities end in the sum)
          const double none = __longlong_as_double(0x7ff8000000000000ll);
          if (MODE == kPrefSums) {
            const bool fine = usable && lp > -3.0e38;
            if (rank == 0) {
              A.row_lp[row] = fine ? lp : 0.0;
              A.row_used[row] = fine;
              A.row_sum[row] = t;
              if (A.out_logp) A.out_logp[row] = fine ? (float)lp : 0.f;
              if (A.out_state) A.out_state[row] = fine ? 1 : 3;
            }
          } else {
            const double a = adv, r = usable ? exp(lp - (double)old) : none, plain = -a * r;
            double loss = plain, slope = plain, kl = 0.0;
            bool live = true;
            if (A.clip) {
              const double clipped = -a * fmin(fmax(r, 1.0 - (double)A.eps_lo), 1.0 + (double)A.eps_hi);
              live = !(plain < clipped);
              if (!live) loss = clipped, slope = 0.0;
            }
            if (A.logp_ref) {
              const double d = (double)ref - lp, e1 = expm1(d);
              kl = e1 - d;
              slope -= (double)A.kl_coef * e1;
            }
            const double wt = (double)weight * inv_n;
            const float co = (float)(wt * slope * A.grad_scale);
            const bool fine = isfinite(wt * loss) && isfinite((float)kl) && isfinite(co) && !isnan(r);
            sh.coef = fine ? co : 0.f;
            sh.k_over_s = fine ? co / t.y : 0.f;
            if (rank == 0) {
              if (A.out_logp) A.out_logp[row] = fine ? (float)lp : 0.f;
              if (A.out_kl) A.out_kl[row] = fine ? (float)kl : 0.f;
              if (A.out_state) A.out_state[row] = fine ? (live ? 1 : 2) : 3;
              A.term[row] = fine ? wt * loss : 0.0;
              A.kl_term[row] = fine ? wt * kl : 0.0;
            }
          }
        }
        if (MODE == kPolicy) {
          __syncthreads();
          coef = sh.coef;
          k = sh.k_over_s;
        }
      }
    }
    if (MODE == kPolicy || MODE == kPrefGrad) {
      if (coef != 0.f) row_gradient<DT>(z, dz, v0, v1, tail0, A.V, A.c, m, k, coef, x);
      else row_zeros<DT>(dz, v0, v1, tail0, A.V);
    }
    if (MODE != kPrefGrad && on) __syncthreads();           // (the next row writes what this one reads of sh)
  }
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
    loss += (1.0 - e) * (up + fmax(-h, 0.0)) + e * (up + fmax(h, 0.0));
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

template <class K>
cudaError_t launch(K kernel, const LossArgs& a, unsigned grid, unsigned threads, int cluster, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
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

template <int MODE> cudaError_t rows(LossArgs a, cudaStream_t s, int sms) {
  // Blocks that share a row: enough that all SMs have work where rows are few, and that the rows in flight (48 MB of logits) stay in L2
  // until they are read again; not more than leave every thread a vector.
  const int64_t bytes = a.V * (a.dtype == JP_BF16 ? 2 : 4), blocks = (int64_t)sms * kBlocksPerSm;
  int c = 1;
  while (c < kMaxCluster && (a.T * c * 2 <= blocks || blocks / c * bytes > (48 << 20)) && bytes / (2 * c) >= 8 * 1024) c *= 2;
  a.cluster = c;
  const int64_t clusters = blocks / c < a.T ? blocks / c : a.T;
  if (a.dtype == JP_BF16) return launch(loss_rows_kernel<JP_BF16, MODE>, a, (unsigned)(clusters * c), kThreads, c, s);
  return launch(loss_rows_kernel<JP_F32, MODE>, a, (unsigned)(clusters * c), kThreads, c, s);
}

}  // namespace

namespace {
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
}  // namespace

size_t policy_workspace_bytes(int64_t T) { return 2 * up256((size_t)T * 8); }

cudaError_t launch_policy(LossArgs a, void* workspace, cudaStream_t s, int sms) {
  a.term = (double*)workspace;
  a.kl_term = (double*)((char*)workspace + up256((size_t)a.T * 8));
  const cudaError_t e = a.dz ? rows<kPolicy>(a, s, sms) : rows<kPolicyNoGrad>(a, s, sms);
  return e != cudaSuccess ? e : launch(policy_sum_kernel, a, 1, 1024, 1, s);
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
  if (e == cudaSuccess) { *n_launch = 1; e = launch(preference_pairs_kernel, a, 1, 1024, 1, s); }
  if (e == cudaSuccess) { *n_launch = 2; if (a.dz) e = rows<kPrefGrad>(a, s, sms); }
  if (e == cudaSuccess && a.dz) *n_launch = 3;
  return e;
}

}  // namespace jp
