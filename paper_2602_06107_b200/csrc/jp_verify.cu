// Verification of drafted tokens against the target model (speculative decoding) from given random numbers.
//
// Sequence b has n drafted tokens x_0 .. x_{n-1}, target logits for positions 0 .. n and draft logits for 0 .. n-1 (or none:
// the draft put all its mass on x_i).  With p_i, q_i the softmaxes at the sequence's temperature:
//   draft i is accepted while u_i < p_i(x_i) / q_i(x_i);
//   at the first rejection, position m, the next token is drawn from max(p_m - q_m, 0) / S;
//   with all n accepted (m = n) it is drawn from p_n.
// The draw is the first v with cumulative mass > u S.  At temperature 0 drafts must equal the target's argmax.
//
// Bound by HBM: (2 n + 1) rows of the vocabulary are read once, one pair of rows a sequence once more.
//
// verify_rows_kernel sums 2^(z c - R) over slices of rows (c = log2 e / temperature).  The reference R needs to be neither the
// maximum nor known in advance: fp32 has 2^+-126 of room, so R is taken from the row's first elements, the same for every
// slice, and a slice whose sum leaves 2^-60 .. 2^120 is done again from its own maximum.  So the loop has no running maximum: one
// unpack, two FMAs (c as a sum of two floats: |z c| reaches 100 and 2^-24 of that would show in the log-probabilities), one ex2 and
// one add an element; eight terms are added in fp32, the rest in fp64.
//
// verify_draw_kernel takes the decisions of a sequence (again in every block: cheaper than a launch of its own) and then the
// masses of the row to draw from, by segments.  Which token a draw hits depends on sums over the vocabulary next to a
// border, so this pass is fp64: 2^x from a table of 16 entries (one wavefront of shared memory whatever the indices) and a
// polynomial of degree 5 (Tang's table-driven scheme), about 12 fp64 operations an element.  The row sums of the first pass are good to
// 1e-7 only, so they serve to decide the sign of p - q; per segment sum p and sum q over p > q are kept apart, beside the
// full sums, and the last block of a sequence to finish scales them with the exact normalisers.  A decision closer than
// 2e-5 to its random number takes its two row sums again in fp64.
#include "jp_common.cuh"
#include "jp_internal.h"

namespace jp {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr double kLog2eD = 1.4426950408889634074;
constexpr double kLn2D = 0.69314718055994530942;

struct RowPart {           // sum over a slice of 2^((z - ref) c) = s.  The difference of logits is taken first: rows of the type's lowest
                           // value are legal, and z c alone would lose the rest
  double ref, s;
  float max;               // greedy rows: largest logit of the slice and its lowest index
  int32_t idx;
  double pad;
};
struct SegPart {           // of one warp's segment of the row to draw from, relative to the first pass's normalisers
  double p, q;             // sums over v with p(v) > q(v)
  double p_all, q_all;
};

struct Scale {             // c = log2(e) / temperature as hi + lo, lo > 0 (so that -inf stays -inf)
  float hi, lo;
  double c;
};
__device__ __forceinline__ Scale scale_of(float t) {
  Scale s;
  s.c = kLog2eD / (double)t;
  s.hi = __double2float_rz(s.c);
  if ((double)s.hi >= s.c) s.hi = __uint_as_float(__float_as_uint(s.hi) - 1u);
  s.lo = (float)(s.c - (double)s.hi);
  return s;
}
// 0: greedy, 1: an ordinary temperature, -1: not one
__device__ __forceinline__ int temperature_kind(float t) { return t == 0.f ? 0 : (t >= 1e-4f && t <= 1e4f) ? 1 : -1; }

// 16-byte vector i of a row; the last one may be short and is filled up with -inf.
template <int DT>
__device__ __forceinline__ uint4 row_vec(const char* row, int64_t i, int64_t V) {
  constexpr int W = Vec<DT>::N;
  if ((i + 1) * W <= V) return ldg_stream((const uint4*)row + i);
  uint4 v = Vec<DT>::neg_inf();
  for (int e = 0; e < W; ++e)
    if (i * W + e < V) Vec<DT>::set(v, e, Vec<DT>::load_scalar(row, i * W + e));
  return v;
}

__device__ __forceinline__ double warp_sum_d(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ double block_sum_d(double v, double* sh) {
  v = warp_sum_d(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s += sh[w];
  return s;
}

// Sum of v over the threads before this one, and over all of them.
__device__ __forceinline__ double block_scan_d(double v, double* sh, double* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  __syncthreads();
  if (lane == 31) sh[warp] = incl;
  __syncthreads();
  double base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w == warp) base = sum;
    sum += sh[w];
  }
  *total = sum;
  const double before = __shfl_up_sync(0xffffffffu, incl, 1);
  return base + (lane ? before : 0.0);
}

// 2^x for x <= 1000, to about 2e-13; 0 below -1000 (and for -inf).  NaN stays NaN.
__device__ __forceinline__ double exp2_table(double x, const double* tab) {
  constexpr double kMagic = 422212465065984.0;            // 1.5 * 2^48: adding it leaves round(16 x) in the low word
  const double m = x + kMagic;
  const int k = __double2loint(m);
  const double r = x - (m - kMagic);                      // |r| <= 1/32
  double y = 0.0013333558146428443423;                    // ln2^5 / 120
  y = fma(y, r, 0.0096181291076284771619);
  y = fma(y, r, 0.055504108664821579953);
  y = fma(y, r, 0.24022650695910071233);
  y = fma(y, r, 0.69314718055994530942);
  y = fma(y, r, 1.0);
  y *= tab[k & 15];
  const double z = __hiloint2double(__double2hiint(y) + ((k >> 4) << 20), __double2loint(y));
  return x < -1000.0 ? 0.0 : z;
}

// A row's sum of 2^((z - ref) c) in fp64 by the whole block, with its own maximum as reference.
template <int DT>
__device__ RowPart exact_slice(const char* row, int64_t i0, int64_t i1, int64_t V, double c, const double* tab,
                               double* sh) {
  constexpr int W = Vec<DT>::N;
  float m = JP_NEG_INF;
  bool nan = false;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kThreads) {
    const uint4 v = row_vec<DT>(row, i, V);
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const float z = Vec<DT>::get(v, e);
      m = fmaxf(m, z);
      nan |= z != z;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = (double)m;
  nan = __syncthreads_or(nan);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) m = fmaxf(m, (float)sh[w]);
  double s = 0;
  const bool ok = !nan && m > JP_NEG_INF && m < __int_as_float(0x7f800000);
  if (ok)
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kThreads) {
      const uint4 v = row_vec<DT>(row, i, V);
#pragma unroll
      for (int e = 0; e < W; ++e) s += exp2_table(((double)Vec<DT>::get(v, e) - (double)m) * c, tab);
    }
  s = block_sum_d(s, sh);
  RowPart r{};
  r.ref = ok ? (double)m : 0.0;
  r.s = ok ? s : (nan || m > 0.f ? __longlong_as_double(0x7ff8000000000000ll) : 0.0);
  return r;
}

__device__ __forceinline__ void fill_table(double* tab) {
  if (threadIdx.x < 16) tab[threadIdx.x] = exp2((double)threadIdx.x / 16.0);
  __syncthreads();
}

template <int DT>
__global__ void __launch_bounds__(kThreads) verify_rows_kernel(VerifyArgs A) {
  constexpr int W = Vec<DT>::N;
  constexpr int kUnroll = 4;
  __shared__ double sh[kWarps];
  __shared__ double tab[16];
  __shared__ unsigned long long s_key[kWarps];
  const int64_t unit = blockIdx.x, line = unit / A.splits;
  const int split = (int)(unit - line * A.splits);
  const int64_t b = line / A.rows_per_seq;
  const int j = (int)(line - b * A.rows_per_seq);
  if (j == 0 && split == 0 && threadIdx.x == 0) A.ticket[b] = 0;
  int n = A.n_draft ? A.n_draft[b] : A.N;
  n = n < 0 ? 0 : (n > A.N ? A.N : n);
  const float temp = A.temperature ? A.temperature[b] : 1.f;
  const int kind = temperature_kind(temp);
  const bool is_draft = j > A.N;
  // rows nobody needs: past the drafts, of a sequence without a usable temperature, draft rows of a greedy one
  if (kind < 0 || (is_draft ? (j - A.N - 1 >= n || kind == 0) : j > n)) return;
  const char* row = is_draft ? (const char*)A.draft + (b * A.seq_draft + (int64_t)(j - A.N - 1) * A.ld_draft) * Vec<DT>::ESIZE
                             : (const char*)A.target + (b * A.seq_target + (int64_t)j * A.ld_target) * Vec<DT>::ESIZE;
  const int64_t nv = (A.V + W - 1) / W;
  const int64_t i0 = nv * split / A.splits, i1 = nv * (split + 1) / A.splits;
  const Scale sc = scale_of(kind == 0 ? 1.f : temp);
  const uint4 first = row_vec<DT>(row, 0, A.V);
  float zref = Vec<DT>::vmax(first);
  // Beyond 1e6, z times what hi + lo leave of c would count; with 0 such a slice leaves the range below and is taken exactly.
  if (!(fabsf(zref * sc.hi) < 1e6f)) zref = 0.f;
  const float ref = zref * sc.hi;

  double s = 0;
  auto add = [&](const uint4& v) {
    float t[W];
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const float z = Vec<DT>::get(v, e);
      t[e] = ex2_approx(fmaf(z, sc.lo, fmaf(z, sc.hi, -ref)));
    }
#pragma unroll
    for (int o = 1; o < W; o *= 2)
#pragma unroll
      for (int e = 0; e + o < W; e += 2 * o) t[e] += t[e + o];
    s += (double)t[0];
  };
  unsigned long long key = 0;
  int64_t i = i0 + threadIdx.x;
  const int64_t full = (A.V / W) < i1 ? A.V / W : i1;      // vectors with all their elements
  for (; i + (kUnroll - 1) * kThreads < full; i += kUnroll * kThreads) {
    uint4 v[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) v[k] = ldg_stream((const uint4*)row + i + k * kThreads);
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) add(v[k]);
  }
  for (; i < i1; i += kThreads) add(row_vec<DT>(row, i, A.V));
  s = block_sum_d(s, sh);
  RowPart part{};
  part.ref = (double)zref;
  part.s = s * exp2((double)ref - (double)zref * sc.c);     // (what the rounding of ref took)
  if (!(s > 0x1p-60 && s < 0x1p120)) {
    fill_table(tab);
    part = exact_slice<DT>(row, i0, i1, A.V, sc.c, tab, sh);
  }
  if (kind == 0) {                                          // greedy: where the slice's maximum is (read again, from L2)
    for (int64_t k = i0 + threadIdx.x; k < i1; k += kThreads) {
      const uint4 v = row_vec<DT>(row, k, A.V);
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (k * W + e < A.V) {
          const unsigned long long c = make_key(Vec<DT>::get(v, e), (uint32_t)(k * W + e));
          key = c > key ? c : key;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long c = __shfl_xor_sync(0xffffffffu, key, o);
      key = c > key ? c : key;
    }
    if ((threadIdx.x & 31) == 0) s_key[threadIdx.x >> 5] = key;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) key = s_key[w] > key ? s_key[w] : key;
    part.max = key_value(key);
    part.idx = (int32_t)key_index(key);
  }
  if (threadIdx.x == 0) ((RowPart*)A.parts)[unit] = part;
}

// One row's log2 of its sum of 2^((z - row_ref) c), by one warp, from the slices' parts in a fixed order; NaN for a row that has none.
__device__ __forceinline__ double row_lse2(const RowPart* p, int splits, double c, int lane, double* row_ref, int* at) {
  double ref = -1e300, s = 0;                                // (logits are above -1e39)
  bool bad = false;
  unsigned long long key = 0;
  for (int i = lane; i < splits; i += 32) {
    const RowPart r = p[i];
    bad |= r.s != r.s;
    if (r.s > 0) ref = r.ref > ref ? r.ref : ref;
    const unsigned long long k = make_key(r.max, (uint32_t)r.idx);
    key = k > key ? k : key;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const double v = __shfl_xor_sync(0xffffffffu, ref, o);
    ref = v > ref ? v : ref;
    const unsigned long long k = __shfl_xor_sync(0xffffffffu, key, o);
    key = k > key ? k : key;
  }
  for (int i = lane; i < splits; i += 32) {
    const RowPart r = p[i];
    if (r.s > 0) s += r.ref == ref ? r.s : r.s * exp2((r.ref - ref) * c);
  }
  s = warp_sum_d(s);
  bad = __any_sync(0xffffffffu, bad);
  *row_ref = ref;
  *at = (int)key_index(key);
  return bad || !(s > 0) ? __longlong_as_double(0x7ff8000000000000ll) : log2(s);
}

template <int DT>
__global__ void __launch_bounds__(kThreads) verify_draw_kernel(VerifyArgs A) {
  constexpr int W = Vec<DT>::N, ES = Vec<DT>::ESIZE;
  __shared__ double tab[16], sh[kWarps];
  __shared__ double s_lse[2 * kVerifyMaxDraft + 1];         // target rows 0 .. N, then draft rows: log2 of the sum ...
  __shared__ double s_ref[2 * kVerifyMaxDraft + 1];         // ... relative to this logit
  __shared__ int s_arg[kVerifyMaxDraft + 1];
  __shared__ double s_ratio[kVerifyMaxDraft];
  __shared__ int s_near, s_m, s_last, s_pick;
  __shared__ double s_best;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t b = blockIdx.y;
  const int split = blockIdx.x;
  const int N = A.N;
  int n = A.n_draft ? A.n_draft[b] : N;
  n = n < 0 ? 0 : (n > N ? N : n);
  const float temp = A.temperature ? A.temperature[b] : 1.f;
  const int kind = temperature_kind(temp);
  const Scale sc = scale_of(kind == 1 ? temp : 1.f);
  const bool with_q = A.draft != nullptr && kind == 1;
  const char* target = (const char*)A.target + b * A.seq_target * ES;
  const char* draft = (const char*)A.draft + (A.draft ? b * A.seq_draft * ES : 0);
  const int32_t* tokens = A.tokens + b * N;
  const double kNan = __longlong_as_double(0x7ff8000000000000ll);
  fill_table(tab);

  // the rows' normalisers
  const int rows = kind < 0 ? 0 : n + 1 + (with_q ? n : 0);
  for (int r = warp; r < rows; r += kWarps) {
    const int j = r <= n ? r : N + 1 + (r - n - 1);
    double ref;
    int at;
    const double l = row_lse2((const RowPart*)A.parts + (b * A.rows_per_seq + j) * A.splits, A.splits, sc.c, lane, &ref, &at);
    if (lane == 0) {
      s_lse[j] = l;
      s_ref[j] = ref;
      if (r <= n) s_arg[r] = at;
    }
  }
  __syncthreads();

  // decisions: lane i has draft i (N <= 32)
  if (warp == 0) {
    double ratio = 0;
    bool near = false;
    if (kind >= 0 && lane < n) {
      const int x = tokens[lane];
      const double lt = s_lse[lane];
      const float u = A.u_accept[b * N + lane];
      if (x >= 0 && x < A.V && lt == lt) {
        if (kind == 0) {
          ratio = x == s_arg[lane] ? 1.0 : 0.0;
        } else {
          const double p = ((double)Vec<DT>::load_scalar(target + lane * A.ld_target * ES, x) - s_ref[lane]) * sc.c - lt;
          double d = p;
          if (with_q)
            d -= ((double)Vec<DT>::load_scalar(draft + lane * A.ld_draft * ES, x) - s_ref[N + 1 + lane]) * sc.c - s_lse[N + 1 + lane];
          ratio = p > -1e300 && d == d ? exp2(d) : 0.0;
          near = fabs(ratio - (double)u) <= 2e-5 * ratio && ratio > 0 && ratio < 1e300;
        }
      }
    }
    if (lane < n) s_ratio[lane] = ratio;
    const bool no = lane < n && !near && !((double)(lane < n ? A.u_accept[b * N + lane] : 0.f) < ratio);
    const unsigned stop = __ballot_sync(0xffffffffu, no);
    const unsigned before = stop ? (stop & (0u - stop)) - 1u : 0xffffffffu;     // drafts in front of the first clear rejection
    const unsigned nb = __ballot_sync(0xffffffffu, near) & before;
    if (lane == 0) s_near = (int)nb;
  }
  __syncthreads();
  for (unsigned todo = (unsigned)s_near; todo; todo &= todo - 1) {              // (the same in every thread)
    const int i = __ffs(todo) - 1;
    const RowPart t = exact_slice<DT>(target + i * A.ld_target * ES, 0, (A.V + W - 1) / W, A.V, sc.c, tab, sh);
    RowPart q{};
    if (with_q) q = exact_slice<DT>(draft + i * A.ld_draft * ES, 0, (A.V + W - 1) / W, A.V, sc.c, tab, sh);
    if (tid == 0) {
      const int x = tokens[i];
      double d = ((double)Vec<DT>::load_scalar(target + i * A.ld_target * ES, x) - t.ref) * sc.c - log2(t.s);
      if (with_q) d -= ((double)Vec<DT>::load_scalar(draft + i * A.ld_draft * ES, x) - q.ref) * sc.c - log2(q.s);
      s_ratio[i] = exp2(d);
    }
  }
  __syncthreads();
  if (warp == 0) {
    const bool no = lane < n && !((double)A.u_accept[b * N + lane] < s_ratio[lane]);
    const unsigned stop = __ballot_sync(0xffffffffu, no);
    const int m = stop ? __ffs(stop) - 1 : n;
    if (lane == 0) s_m = kind < 0 ? 0 : m;
  }
  __syncthreads();
  const int m = s_m;
  const bool rejected = m < n;
  const double lt = kind < 0 ? kNan : s_lse[m];
  const double lq = rejected && with_q ? s_lse[N + 1 + m] : 0.0;
  const double rt = kind < 0 ? 0.0 : s_ref[m], rq = rejected && with_q ? s_ref[N + 1 + m] : 0.0;
  const bool use_q = rejected && with_q;
  const bool usable = lt == lt && lq == lq;                 // else the row to draw from is bad: token -1
  if (split == 0) {
    if (tid == 0) A.out_n_accepted[b] = m;
    for (int i = tid; i <= N; i += kThreads) {
      int32_t tok = -1;
      float lp = 0.f;
      if (i < m || (i == m && kind == 0 && usable)) {
        tok = i < m ? tokens[i] : s_arg[m];
        lp = (float)((((double)Vec<DT>::load_scalar(target + i * A.ld_target * ES, tok) - s_ref[i]) * sc.c - s_lse[i]) * kLn2D);
      }
      if (i != m || kind == 0 || !usable) {                 // (else the last block of the sequence writes it)
        A.out_tokens[b * (N + 1) + i] = tok;
        if (A.out_logp) A.out_logp[b * (N + 1) + i] = lp;
      }
      if (i < N && A.out_accept_prob)
        A.out_accept_prob[b * N + i] = i <= m && i < n && kind >= 0 ? (float)fmin(s_ratio[i], 1.0) : 0.f;
    }
  }
  if (kind != 1 || !usable) return;

  // masses of the row to draw from: this block's slice, a contiguous run of vectors a warp
  const char* zt = target + m * A.ld_target * ES;
  const char* zq = draft + (use_q ? m * A.ld_draft * ES : 0);
  const int skip = rejected && !with_q ? tokens[m] : -1;    // a draft without logits had all its mass there
  const int64_t nv = (A.V + W - 1) / W;
  const int segs = A.draw_splits * kWarps;
  auto seg_first = [&](int g) { return nv * g / segs; };
  SegPart part{};
  {
    const int g = split * kWarps + warp;
    const int64_t i1 = seg_first(g + 1);
    for (int64_t i = seg_first(g) + lane; i < i1; i += 32) {
      const uint4 vt = row_vec<DT>(zt, i, A.V);
      const uint4 vq = use_q ? row_vec<DT>(zq, i, A.V) : vt;
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const double p = exp2_table(fma((double)Vec<DT>::get(vt, e) - rt, sc.c, -lt), tab);
        part.p_all += p;
        if (use_q) {
          const double q = exp2_table(fma((double)Vec<DT>::get(vq, e) - rq, sc.c, -lq), tab);
          part.q_all += q;
          if (p > q) { part.p += p; part.q += q; }
        } else if (i * W + e != skip) {
          part.p += p;
        }
      }
    }
    part.p = warp_sum_d(part.p);
    part.q = warp_sum_d(part.q);
    part.p_all = warp_sum_d(part.p_all);
    part.q_all = warp_sum_d(part.q_all);
    if (lane == 0) {
      ((SegPart*)A.segs)[b * segs + g] = part;
      __threadfence();
    }
  }
  __syncthreads();
  if (tid == 0) s_last = atomicAdd(&A.ticket[b], 1) == A.draw_splits - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();

  // last block of the sequence: exact normalisers, the segment that the draw falls into, the element in it
  const volatile double* sp = (const volatile double*)((SegPart*)A.segs + b * segs);
  double P = 0, Q = 0;
  for (int g = tid; g < segs; g += kThreads) { P += sp[g * 4 + 2]; Q += sp[g * 4 + 3]; }
  P = block_sum_d(P, sh);
  Q = block_sum_d(Q, sh);
  const double a = 1.0 / P, c = use_q ? 1.0 / Q : 0.0;
  bool whole = false;                                       // no mass left above zero: draw from p itself
  auto seg_mass = [&](int g) {
    const double v = whole ? sp[g * 4 + 2] * a : sp[g * 4] * a - sp[g * 4 + 1] * c;
    return v > 0 ? v : 0.0;
  };
  // every thread has a contiguous run of segments; exclusive sums over the threads in order
  const int per = (segs + kThreads - 1) / kThreads;
  double mine = 0, total = 0, before = 0;
  for (int round = 0; round < 2; ++round) {
    mine = 0;
    for (int k = 0; k < per; ++k)
      if (tid * per + k < segs) mine += seg_mass(tid * per + k);
    before = block_scan_d(mine, sh, &total);
    if (total > 0) break;
    whole = true;
  }
  const float u = A.u_sample[b];
  const double want = u > 0.f ? (double)u * total : 0.0;
  if (tid == 0) s_pick = -1;
  __syncthreads();
  {
    double acc = before;
    for (int k = 0; k < per; ++k) {
      const int g = tid * per + k;
      if (g >= segs) break;
      const double w = seg_mass(g);
      // the draw falls here; a draw beyond the end (u >= 1, rounding) takes the last segment with mass
      if (w > 0 && acc <= want) atomicMax(&s_pick, g);
      acc += w;
    }
  }
  __syncthreads();
  const int g = s_pick < 0 ? 0 : s_pick;
  if (tid == g / per) {                                     // the sum before it, in the order of the search
    double acc = before;
    for (int k = tid * per; k < g; ++k) acc += seg_mass(k);
    s_best = acc;
  }
  __syncthreads();
  const double base = s_best;
  const int64_t e0 = seg_first(g) * W, e1 = seg_first(g + 1) * W < A.V ? seg_first(g + 1) * W : A.V;
  const int64_t each = (e1 - e0 + kThreads - 1) / kThreads;
  const int64_t f0 = e0 + each * tid, f1 = f0 + each < e1 ? f0 + each : e1;
  auto mass = [&](int64_t v) {
    const double p = exp2_table(fma((double)Vec<DT>::load_scalar(zt, v) - rt, sc.c, -lt), tab) * a;
    if (whole) return p;
    if (!use_q) return v == skip ? 0.0 : p;
    const double q = exp2_table(fma((double)Vec<DT>::load_scalar(zq, v) - rq, sc.c, -lq), tab) * c;
    return p > q ? p - q : 0.0;
  };
  mine = 0;
  for (int64_t v = f0; v < f1; ++v) mine += mass(v);
  if (tid == 0) s_pick = -1;
  before = base + block_scan_d(mine, sh, &total);           // (its barriers also order s_pick)
  {
    double acc = before;
    int pick = -1;
    for (int64_t v = f0; v < f1; ++v) {
      const double w = mass(v);
      if (w > 0 && acc <= want) pick = (int)(v - e0);       // the last with acc <= want is the first whose end is beyond it
      acc += w;
    }
    if (pick >= 0) atomicMax(&s_pick, pick);
  }
  __syncthreads();
  if (tid == 0) {
    const int64_t v = e0 + (s_pick < 0 ? 0 : s_pick);
    A.out_tokens[b * (N + 1) + m] = (int32_t)v;
    if (A.out_logp)
      A.out_logp[b * (N + 1) + m] = (float)((((double)Vec<DT>::load_scalar(zt, v) - rt) * sc.c - lt - log2(P)) * kLn2D);
  }
}

}  // namespace

VerifyPlan verify_plan(int64_t B, int N, int64_t V, int dtype, bool with_draft, int sms) {
  VerifyPlan p{};
  p.rows_per_seq = N + 1 + (with_draft ? N : 0);
  const int64_t nv = (V + (dtype == JP_BF16 ? 7 : 3)) / (dtype == JP_BF16 ? 8 : 4);
  const int64_t lines = B * p.rows_per_seq;
  auto pick = [&](int64_t want, int64_t most) { return (int)(want < 1 ? 1 : want > most ? (most < 1 ? 1 : most) : want); };
  p.splits = pick((sms * 16 + lines - 1) / lines, (nv + 511) / 512);
  p.draw_splits = pick((sms * 4 + B - 1) / B, (nv + 255) / 256);
  if (p.draw_splits > 64) p.draw_splits = 64;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  p.parts_off = up((size_t)B * 4);
  p.segs_off = p.parts_off + up((size_t)lines * p.splits * sizeof(RowPart));
  p.bytes = p.segs_off + up((size_t)B * p.draw_splits * kWarps * sizeof(SegPart));
  return p;
}

cudaError_t launch_verify(VerifyArgs a, int dtype, cudaStream_t s) {
  const dim3 g1((unsigned)(a.B * a.rows_per_seq * a.splits)), g2((unsigned)a.draw_splits, (unsigned)a.B);
  if (dtype == JP_BF16) verify_rows_kernel<JP_BF16><<<g1, kThreads, 0, s>>>(a);
  else verify_rows_kernel<JP_F32><<<g1, kThreads, 0, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  if (dtype == JP_BF16) verify_draw_kernel<JP_BF16><<<g2, kThreads, 0, s>>>(a);
  else verify_draw_kernel<JP_F32><<<g2, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace jp
