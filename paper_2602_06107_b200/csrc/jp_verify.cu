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
// verify_rows_kernel sums 2^((z - R) c) over slices of rows (c = log2 e / temperature).  The reference R need not be the maximum: fp32
// has 2^+-126 of room.  So it is the largest of the slice's first 8 KB, and the loop has no running maximum: one unpack, one
// FMA, one ex2 and one add an element; 16 terms (fp32 input: 8) are added in fp32, the rest in fp64.  Terms that reach
// 256 together (a peak outside the sample: exponents of 8 and more are rounded by more than 2^-22) are taken again in fp64, and a slice
// whose sum leaves 2^-60 .. 2^60 from its own maximum.
//
// verify_draw_kernel takes the decisions of a sequence (again in every block: cheaper than a launch of its own) and then the
// masses of the row to draw from, by segments.  Which token a draw hits depends on sums over the vocabulary next to a
// border, so this pass is fp64: 2^x from a table of 32 entries and a polynomial of degree 4 (Tang's table-driven scheme), about 10 fp64
// operations an element.  The row sums of the first pass are good to 1e-7, in the worst case to 3e-6, so they serve to decide the sign of p - q; per segment
// sum p and sum q over p > q are kept apart, beside the full sums, and the last block of a sequence to finish scales them with the
// exact normalisers (and, for rows so nearly equal that the sign matters, takes the segments again with these).  A decision closer
// than kNear (2e-5) to its random number takes its two row sums again in fp64.
#include "jp_common.cuh"
#include "jp_internal.h"

namespace jp {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kDrawBlocks = 2;       // blocks of the draw per SM (three get 80 registers a thread and were 5 % slower)
constexpr unsigned kAll = 0xffffffffu;
constexpr double kNear = 2e-5;       // decisions closer to their random number than this have their sums taken again in fp64
constexpr double kLog2eD = 1.4426950408889634074;
constexpr double kLn2D = 0.69314718055994530942;
// Logits below ref + kFloor / c have probability 0 (ref: the row's reference, 2^-60 to 2^66 of its sum).  The sums take them as
// 2^kClamp instead, which is one operation an element: 2^31 of them stay below 2^kTiny, what has a probability above it.
constexpr double kFloor = -840.0, kTiny = 0x1p-850, kClamp = -900.0;

__constant__ double kPow2[32] = {    // 2^(j / 32)
    1.0, 1.0218971486541166, 1.0442737824274138, 1.0671404006768237,
    1.0905077326652577, 1.1143867425958924, 1.1387886347566916, 1.1637248587775775,
    1.189207115002721, 1.215247359980469, 1.241857812073484, 1.2690509571917332,
    1.2968395546510096, 1.3252366431597413, 1.3542555469368927, 1.383909881963832,
    1.4142135623730951, 1.4451808069770467, 1.4768261459394993, 1.5091644275934228,
    1.5422108254079407, 1.5759808451078865, 1.6104903319492543, 1.645755478153965,
    1.681792830507429, 1.718619298122478, 1.7562521603732995, 1.7947090750031072,
    1.8340080864093424, 1.8741676341103, 1.9152065613971474, 1.9571441241754002};

struct RowPart {           // sum over a slice of 2^((z - ref) c) = s.  The difference of logits is taken first: rows of the type's lowest
  double s;                // value are legal, and z c alone would lose the rest
  float ref;               // a logit (greedy rows: the slice's largest, at idx)
  int32_t idx;
};
struct SegPart {           // of one warp's segment of the row to draw from, normalised by the first pass's sums
  double p, q;             // sums over v with p(v) > q(v)
  double p_all, q_all;
};

__device__ __forceinline__ double log2e_over(float t) { return t == 1.f ? kLog2eD : kLog2eD / (double)t; }
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
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
__device__ __forceinline__ float warp_max_f(float v) {      // (NaN comes out as the largest or smallest: callers test for it apart)
  return order_bits_f32(__reduce_max_sync(kAll, f32_order_bits(v)));
}
__device__ __forceinline__ double block_sum_d(double v, double* sh) {
  v = warp_sum_d(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  static_assert(kWarps == 8, "pairs below");
  return ((sh[0] + sh[1]) + (sh[2] + sh[3])) + ((sh[4] + sh[5]) + (sh[6] + sh[7]));
}
__device__ __forceinline__ float block_max_f(float v, float* sh) {
  v = warp_max_f(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) v = fmaxf(v, sh[w]);
  return v;
}
// Sum of v over the threads before this one, and over all of them.
__device__ __forceinline__ double block_scan_d(double v, double* sh, double* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double u = __shfl_up_sync(kAll, incl, o);
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
  const double before = __shfl_up_sync(kAll, incl, 1);
  return base + (lane ? before : 0.0);
}

// 2^x times what tab is scaled by, |x| <= 1000, to about 2e-12 relative.  tab[j] is scale 2^(j / 32) with j << 15 taken from its
// high word, so that adding k << 15 for k = round(32 x) gives scale 2^(k / 32) in one addition.
// Constants whose low word is 0 are part of an instruction; the two that need all their bits come in registers (c1 = ln 2,
// c2 = ln^2 2 / 2), since the compiler would otherwise move them there again for every element.
__device__ __forceinline__ double exp2_table(double x, const double* tab, double c1, double c2) {
  constexpr double kMagic = 211106232532992.0;            // 1.5 * 2^47: adding it leaves k in the low word
  const double m = x + kMagic;
  const int k = __double2loint(m);
  const double t = tab[k & 31];
  const double r = x - (m - kMagic);                      // |r| <= 1/64; terms of exp(r ln 2) up to r^4
  double y = 0.009618125855922699;                        // ln^4 2 / 24 and ln^3 2 / 6 to 2^-21: r^3 makes 1e-13 of that
  y = fma(y, r, 0.05550411343574524);
  y = fma(y, r, c2);
  y = fma(y, r, c1);
  y = fma(y, r, 1.0);
  return y * __hiloint2double(__double2hiint(t) + (k << 15), __double2loint(t));
}
constexpr double kLn2Square = 0.24022650695910071233;     // ln^2 2 / 2
__device__ __forceinline__ double exp2_clamped(double x, const double* tab) {     // 0 below -1000, 2^1000 above
  return x < -1000.0 ? 0.0 : exp2_table(x < 1000.0 ? x : 1000.0, tab, kLn2D, kLn2Square);
}
__device__ __forceinline__ double table_entry(int j, double scale) {
  const double t = kPow2[j] * scale;
  return __hiloint2double(__double2hiint(t) - (j << 15), __double2loint(t));
}
__device__ __forceinline__ void fill_table(double* tab) {
  if (threadIdx.x < 32) tab[threadIdx.x] = table_entry(threadIdx.x, 1.0);
}

// A slice's sum in fp64 by the whole block, with its own maximum as reference.
template <int DT>
__device__ __noinline__ RowPart exact_slice(const char* row, int64_t i0, int64_t i1, int64_t V, double c,
                                            const double* tab, double* sh) {
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
  m = block_max_f(m, (float*)sh);
  nan = __syncthreads_or(nan);
  const bool ok = !nan && m > JP_NEG_INF && m < __int_as_float(0x7f800000);
  double s = 0;
  if (ok)
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kThreads) {
      const uint4 v = row_vec<DT>(row, i, V);
#pragma unroll
      for (int e = 0; e < W; ++e) s += exp2_clamped(((double)Vec<DT>::get(v, e) - (double)m) * c, tab);
    }
  s = block_sum_d(s, sh);
  RowPart r;
  r.ref = ok ? m : 0.f;
  r.idx = 0;
  r.s = ok ? s : (nan || m > 0.f ? __longlong_as_double(0x7ff8000000000000ll) : 0.0);
  return r;
}

// The terms of two vectors in fp64; infinity where they leave the range.
template <int DT>
__device__ __noinline__ double exact_terms(uint4 v0, uint4 v1, float zref, double c, const double* tab) {
  constexpr int W = Vec<DT>::N;
  double s = 0;
#pragma unroll
  for (int e = 0; e < 2 * W; ++e) {
    const double x = ((double)Vec<DT>::get(e < W ? v0 : v1, e % W) - (double)zref) * c;
    s += x > 60.0 ? __longlong_as_double(0x7ff0000000000000ll) : exp2_clamped(x, tab);
  }
  return s;
}

constexpr int kGroup = 2;       // vectors a thread takes at a time
constexpr int kGroups = 3;      // groups in flight: 24 KB a block (more were no faster)
template <int DT> __device__ __forceinline__ uint4 neg_inf() { return Vec<DT>::neg_inf(); }

// A thread's vectors p[tid], p[tid + kThreads], ... below n through its own places in shared memory, kGroups groups ahead (asynchronous
// copies: with loads into registers a block's 64 KB would be four round trips to HBM).  No thread reads another's places: no barriers.
struct RowStream {
  const uint4* p;
  uint4* place;                 // [kGroups * kGroup][kThreads], this thread's column
  int n, issue, take, slot_in, slot_out;
  __device__ __forceinline__ void fetch() {
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const int i = issue + k * kThreads;
      if (i < n)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(place + (slot_in + k) * kThreads)),
                     "l"(p + i) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    issue += kGroup * kThreads;
    slot_in = slot_in == (kGroups - 1) * kGroup ? 0 : slot_in + kGroup;
  }
  __device__ __forceinline__ void start(const uint4* from, uint4* smem, int count) {
    p = from;
    place = smem + threadIdx.x;
    n = count;
    issue = take = threadIdx.x;
    slot_in = slot_out = 0;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) fetch();
  }
  __device__ __forceinline__ void next(uint4 (&v)[kGroup], const uint4& none) {      // the oldest group, and another one on its way
    asm volatile("cp.async.wait_group %0;" ::"n"(kGroups - 1) : "memory");
#pragma unroll
    for (int k = 0; k < kGroup; ++k) v[k] = take + k * kThreads < n ? place[(slot_out + k) * kThreads] : none;
    take += kGroup * kThreads;
    slot_out = slot_out == (kGroups - 1) * kGroup ? 0 : slot_out + kGroup;
    fetch();
  }
};

// A thread's share of a slice: sum of 2^(z cf - zref cf) and, for greedy rows, its largest logit and that one's vector.
struct RowSums {
  double fast, exact;
  float best;
  int best_i;
};
template <int DT, bool GREEDY>
struct RowLoop {
  static constexpr int W = Vec<DT>::N;
  float cf, ref;
  float zref;
  double c;
  const double* tab;
  RowSums r;
  __device__ __forceinline__ void two(const uint4& v0, const uint4& v1, int i0, int i1) {
    float t[4];
#pragma unroll
    for (int e = 0; e < 2 * W; ++e) {
      const float x = ex2_approx(fmaf(Vec<DT>::get(e < W ? v0 : v1, e % W), cf, -ref));
      t[e & 3] = e < 4 ? x : t[e & 3] + x;
    }
    t[0] = (t[0] + t[1]) + (t[2] + t[3]);
    if (t[0] > 256.f) r.exact += exact_terms<DT>(v0, v1, zref, c, tab);    // rare: logits well above the sample that gave the reference
    else r.fast += (double)t[0];
    if (GREEDY) {
      const float m0 = Vec<DT>::vmax(v0), m1 = Vec<DT>::vmax(v1);
      if (m0 > r.best) { r.best = m0; r.best_i = i0; }
      if (m1 > r.best) { r.best = m1; r.best_i = i1; }
    }
  }
  // The thread's vectors: group 0 in v; later ones come through its places in shared memory.
  __device__ __forceinline__ void run(uint4 (&v)[kGroup], RowStream& in, int n, const uint4& last, int last_i) {
    for (int i = threadIdx.x;;) {
#pragma unroll
      for (int k = 0; k < kGroup; k += 2) two(v[k], v[k + 1], i + k * kThreads, i + (k + 1) * kThreads);
      i += kGroup * kThreads;
      if (i - (int)threadIdx.x >= n) break;
      in.next(v, neg_inf<DT>());
    }
    if (last_i >= 0) two(last, neg_inf<DT>(), last_i, last_i);          // the row's short last vector
  }
};

template <int DT>
__global__ void __launch_bounds__(kThreads, 4) verify_rows_kernel(VerifyArgs A) {
  constexpr int W = Vec<DT>::N;
  extern __shared__ uint4 places[];
  __shared__ double sh[kWarps];
  __shared__ double tab[32];
  __shared__ unsigned long long s_key[kWarps];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // the second pass may set up; it waits for this grid's end itself
  const int split = blockIdx.x, j = blockIdx.y;
  const int64_t b = blockIdx.z;
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
  const int64_t i0 = (int64_t)split * A.split_vecs, i1 = i0 + A.split_vecs < nv ? i0 + A.split_vecs : nv;
  const int64_t full = (A.V / W) < i1 ? A.V / W : i1;      // vectors with all their elements end here
  const int n_vec = (int)(full - i0);                       // (a row is below 2^31 elements)
  RowStream in;
  in.start((const uint4*)row + i0, places, n_vec);
  const int last_i = full < i1 && threadIdx.x == 0 ? n_vec : -1;
  uint4 last = Vec<DT>::neg_inf();
  if (last_i >= 0) last = row_vec<DT>(row, i0 + n_vec, A.V);
  fill_table(tab);
  uint4 v[kGroup];
  in.next(v, neg_inf<DT>());
  const double c = log2e_over(kind == 0 ? 1.f : temp);
  const float cf = (float)c;
  float zref = fmaxf(Vec<DT>::vmax(last), Vec<DT>::vmax2(v[0], v[1]));
  zref = block_max_f(zref, (float*)sh);
  if (!(fabsf(zref) < 1e30f)) zref = 0.f;                   // (such a slice leaves the range below and is taken exactly)
  const float ref = zref * cf;
  RowSums r{0.0, 0.0, JP_NEG_INF, 0};
  if (kind == 0) {
    RowLoop<DT, true> loop{cf, ref, zref, c, tab, r};
    loop.run(v, in, n_vec, last, last_i);
    r = loop.r;
  } else {
    RowLoop<DT, false> loop{cf, ref, zref, c, tab, r};
    loop.run(v, in, n_vec, last, last_i);
    r = loop.r;
  }
  RowPart part;
  part.ref = zref;
  part.idx = 0;
  // relative to zref (ref is rounded).  An exponent x that counts is off by half its step and by what cf lacks of c, 2^-25 |x|: 1.1e-6 of its
  // term where the sample gave a reference (of a slice's 2^15 terms those below 2^-20 hardly count).  Where the whole sample was masked, zref is 0 and
  // all that counts may lie near 2^-60: 2^-19 and 60 2^-25, times ln 2, 2.6e-6.  Two rows of that stay well within the 2e-5 of kNear.
  part.s = block_sum_d(r.fast * exp2_clamped((double)ref - (double)zref * (double)cf, tab) + r.exact, sh);
  if (!(part.s > 0x1p-60 && part.s < 0x1p60)) part = exact_slice<DT>(row, i0, i1, A.V, c, tab, sh);
  if (kind == 0) {                                          // greedy: the slice's largest logit becomes its reference
    unsigned long long key = 0;
    if (r.best > JP_NEG_INF) {
      const uint4 u = row_vec<DT>(row, i0 + r.best_i, A.V);
#pragma unroll
      for (int e = W - 1; e >= 0; --e)
        if (Vec<DT>::get(u, e) == r.best) key = make_key(r.best, (uint32_t)((i0 + r.best_i) * W + e));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long k = __shfl_xor_sync(kAll, key, o);
      key = k > key ? k : key;
    }
    if ((threadIdx.x & 31) == 0) s_key[threadIdx.x >> 5] = key;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) key = s_key[w] > key ? s_key[w] : key;
    if (part.s > 0) {
      const float m = key_value(key);
      part.s *= exp2_clamped(((double)part.ref - (double)m) * c, tab);
      part.ref = m;
      part.idx = (int32_t)key_index(key);
    }
  }
  if (threadIdx.x == 0) ((RowPart*)A.parts)[(b * A.rows_per_seq + j) * A.splits + split] = part;
}

// One row's sum of 2^((z - row_ref) c), by one warp, from the slices' parts in a fixed order; 0 for a row that has none or is not
// finite.
__device__ __forceinline__ double row_sum(const RowPart* p, int splits, double c, const double* tab, int lane,
                                          float* row_ref, int* at) {
  RowPart r[kVerifyMaxSplits / 32];
  float ref = JP_NEG_INF;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < kVerifyMaxSplits / 32; ++k) {
    r[k].s = 0;
    r[k].ref = JP_NEG_INF;
    r[k].idx = 0;
    if (lane + 32 * k < splits) {
      const int4 w = __ldcg((const int4*)(p + lane + 32 * k));
      r[k].s = __hiloint2double(w.y, w.x);
      r[k].ref = __int_as_float(w.z);
      r[k].idx = w.w;
      bad |= r[k].s != r[k].s;
      if (r[k].s > 0) ref = fmaxf(ref, r[k].ref);
    }
  }
  ref = warp_max_f(ref);
  double s = 0;
  uint32_t idx = 0x7fffffffu;
#pragma unroll
  for (int k = 0; k < kVerifyMaxSplits / 32; ++k)
    if (r[k].s > 0) {
      s += r[k].s * exp2_clamped(((double)r[k].ref - (double)ref) * c, tab);
      if (r[k].ref == ref) idx = min(idx, (uint32_t)r[k].idx);
    }
  s = warp_sum_d(s);
  *row_ref = ref;
  *at = (int)__reduce_min_sync(kAll, idx);
  return __any_sync(kAll, bad) ? 0.0 : s;
}

// One of the two rows to draw from: element z has probability 2^((z - ref) c) over the row's sum, whose reciprocal is in the table.
struct DrawRow {
  const char* z;
  double c, ref, off;        // off = -ref c
  double c1, c2;             // of exp2_table
  float cut;                 // smaller logits count as this one: 2^kClamp
  const double* tab;
  // FAR: references so large that off would lose too much, and that cut may be the reference itself
  template <bool FAR>
  __device__ __forceinline__ double prob(float v) const {
    if (FAR) {
      const double y = exp2_table(((double)v - ref) * c, tab, c1, c2);
      return v < cut ? 0.0 : y;
    }
    return exp2_table(fma((double)fmaxf(v, cut), c, off), tab, c1, c2);
  }
};

// Sums of the segments first, first + step, ... (count of them) of seg_vecs vectors each (a multiple of 32), by one warp, into
// out[segment].
template <int DT, bool Q, bool FAR>
__device__ __forceinline__ void segments(const DrawRow& T, const DrawRow& D, int64_t skip, int first, int step, int count,
                                         int64_t seg_vecs, int64_t nv, int64_t V, SegPart* out) {
  constexpr int W = Vec<DT>::N;
  const int lane = threadIdx.x & 31;
  const int steps = (int)seg_vecs / 32, full = (int)(V / W);
  const int skip_vec = skip >= 0 ? (int)(skip / W) : -1;
  // Two vectors are in flight while one is computed.  (They move through registers: a loop unrolled by three does not fit the
  // instruction cache and ran a quarter slower.)
  uint4 t0, t1, q0, q1;
  int in_left = count, in_step = 0, at_vec = first * (int)seg_vecs + lane;         // the next vector to load
  auto fetch = [&](uint4& vt, uint4& vq) {
    vt = vq = Vec<DT>::neg_inf();
    if (in_left > 0) {
      if (at_vec < full) {
        vt = ldg_stream((const uint4*)T.z + at_vec);
        if (Q) vq = ldg_stream((const uint4*)D.z + at_vec);
      } else if (at_vec < (int)nv) {
        vt = row_vec<DT>(T.z, at_vec, V);
        if (Q) vq = row_vec<DT>(D.z, at_vec, V);
      }
      if (!Q && at_vec == skip_vec) Vec<DT>::set(vt, (int)(skip - (int64_t)skip_vec * W), JP_NEG_INF);
      at_vec += 32;
      if (++in_step == steps) {
        in_step = 0;
        --in_left;
        at_vec += (step - 1) * (int)seg_vecs;
      }
    }
  };
  fetch(t0, q0);
  fetch(t1, q1);
  for (int at = 0; at < count; ++at) {
    SegPart s{};
#pragma unroll 1
    for (int k = 0; k < steps; ++k) {
      const uint4 vt = t0, vq = q0;
      t0 = t1;
      q0 = q1;
      fetch(t1, q1);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const double p = T.prob<FAR>(Vec<DT>::get(vt, e));
        if (Q) {
          const double q = D.prob<FAR>(Vec<DT>::get(vq, e));
          s.p_all += p;
          s.q_all += q;
          if (p > q) { s.p += p; s.q += q; }
        } else {
          s.p += p;
        }
      }
    }
    s.p = warp_sum_d(s.p);
    if (Q) {
      s.q = warp_sum_d(s.q);
      s.p_all = warp_sum_d(s.p_all);
      s.q_all = warp_sum_d(s.q_all);
    }
    if (lane == 0) out[first + at * step] = s;
  }
}

// A draw from max(p - q, 0) takes its segments again where that sums to less than kApart times what the first pass's sums are off by
// (eta).  For entries whose log (p / q) spreads over s, the whole is about 0.4 s and those of the wrong sign are off by 0.2 eta^2 / s
// together: 1e-7 of the whole at this border.
constexpr double kApart = 1e3;
// All segments again by one block, with p and q in their exact normalisation.
template <int DT>
__device__ __noinline__ void segments_again(DrawRow T, DrawRow D, bool far, int segs, int64_t seg_vecs, int64_t nv, int64_t V, SegPart* out) {
  const int warp = threadIdx.x >> 5, count = warp < segs ? (segs - warp + kWarps - 1) / kWarps : 0;
  if (far) segments<DT, true, true>(T, D, -1, warp, kWarps, count, seg_vecs, nv, V, out);
  else segments<DT, true, false>(T, D, -1, warp, kWarps, count, seg_vecs, nv, V, out);
}

// Of all threads' (place, sum before it), the one with the largest place; place -1: none.
struct Pick { int place; double before; };
__device__ __forceinline__ Pick block_last(int place, double before, Pick* sh) {
  const int best = __reduce_max_sync(kAll, place);
  __syncthreads();
  if (place == best && (best >= 0 || (threadIdx.x & 31) == 0)) sh[threadIdx.x >> 5] = Pick{place, before};
  __syncthreads();
  Pick p = sh[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w)
    if (sh[w].place > p.place) p = sh[w];
  return p;
}

template <int DT>
__global__ void __launch_bounds__(kThreads, kDrawBlocks) verify_draw_kernel(VerifyArgs A) {
  constexpr int W = Vec<DT>::N, ES = Vec<DT>::ESIZE;
  __shared__ double tab[32], tab_t[32], tab_q[32], sh[kWarps];
  __shared__ Pick s_pick[kWarps];
  __shared__ double s_sum[2 * kVerifyMaxDraft + 1];         // target rows 0 .. N, then draft rows: sum of exponentials,
  __shared__ double s_inv[2 * kVerifyMaxDraft + 1];         // its reciprocal ...
  __shared__ float s_ref[2 * kVerifyMaxDraft + 1];          // ... relative to this logit
  __shared__ int s_arg[kVerifyMaxDraft + 1];
  __shared__ double s_ratio[kVerifyMaxDraft];
  __shared__ float s_zt[kVerifyMaxDraft], s_zd[kVerifyMaxDraft], s_u[kVerifyMaxDraft];
  __shared__ int s_tok[kVerifyMaxDraft];
  __shared__ int s_near, s_m, s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t b = blockIdx.y;
  const int split = blockIdx.x;
  const int N = A.N;
  int n = A.n_draft ? A.n_draft[b] : N;
  n = n < 0 ? 0 : (n > N ? N : n);
  const float temp = A.temperature ? A.temperature[b] : 1.f;
  const int kind = temperature_kind(temp);
  const double c = log2e_over(kind == 1 ? temp : 1.f);
  const bool with_q = A.draft != nullptr && kind == 1;
  const char* target = (const char*)A.target + b * A.seq_target * ES;
  const char* draft = (const char*)A.draft + (A.draft ? b * A.seq_draft * ES : 0);
  fill_table(tab);
  if (tid < n) {                                            // what does not come from the first pass, while that may still run
    const int x = A.tokens[b * N + tid];
    const bool in = x >= 0 && x < A.V;
    s_tok[tid] = x;
    s_u[tid] = A.u_accept[b * N + tid];
    s_zt[tid] = in ? Vec<DT>::load_scalar(target + tid * A.ld_target * ES, x) : JP_NEG_INF;
    s_zd[tid] = in && with_q ? Vec<DT>::load_scalar(draft + tid * A.ld_draft * ES, x) : 0.f;
  }
  const float u_sample = A.u_sample[b];
  if (tid == 0) s_last = 0;
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");

  // the rows' sums
  const int rows = kind < 0 ? 0 : n + 1 + (with_q ? n : 0);
  for (int r = warp; r < rows; r += kWarps) {
    const int j = r <= n ? r : N + 1 + (r - n - 1);
    float ref;
    int at;
    const double s = row_sum((const RowPart*)A.parts + (b * A.rows_per_seq + j) * A.splits, A.splits, c, tab, lane, &ref, &at);
    if (lane == 0) {
      s_sum[j] = s;
      s_inv[j] = 1.0 / s;
      s_ref[j] = ref;
      if (r <= n) s_arg[r] = at;
    }
  }
  __syncthreads();

  // decisions: lane i has draft i (N <= 32)
  if (warp == 0) {
    double ratio = 0;
    bool near = false;
    if (kind >= 0 && lane < n && s_sum[lane] > 0) {
      if (kind == 0) {
        ratio = s_tok[lane] == s_arg[lane] ? 1.0 : 0.0;
      } else if (s_zt[lane] > JP_NEG_INF) {
        double d = ((double)s_zt[lane] - (double)s_ref[lane]) * c, scale = s_inv[lane];
        bool ok = d >= kFloor;                              // (a token masked by the type's lowest value is not emitted)
        if (with_q) {
          const double sq = s_sum[N + 1 + lane];
          ok = ok && sq > 0;
          d -= ((double)s_zd[lane] - (double)s_ref[N + 1 + lane]) * c;
          scale *= sq;
        }
        ratio = ok ? exp2_clamped(d, tab) * scale : 0.0;
        near = ok && fabs(ratio - (double)s_u[lane]) <= kNear * ratio && ratio > 0;
      }
    }
    if (lane < n) s_ratio[lane] = ratio;
    const bool yes = lane < n && (double)s_u[lane < n ? lane : 0] < ratio;
    const unsigned stop = __ballot_sync(kAll, lane < n && !near && !yes);
    const unsigned before = stop ? (stop & (0u - stop)) - 1u : kAll;            // drafts in front of the first clear rejection
    const unsigned nb = __ballot_sync(kAll, near) & before;
    if (lane == 0) {
      s_near = (int)nb;
      s_m = stop ? __ffs(stop) - 1 : n;
    }
  }
  __syncthreads();
  if (s_near) {
    for (unsigned todo = (unsigned)s_near; todo; todo &= todo - 1) {            // (the same in every thread)
      const int i = __ffs(todo) - 1;
      const int64_t nv = (A.V + W - 1) / W;
      const RowPart t = exact_slice<DT>(target + i * A.ld_target * ES, 0, nv, A.V, c, tab, sh);
      double d = ((double)s_zt[i] - (double)t.ref) * c, over = t.s;
      if (with_q) {
        const RowPart q = exact_slice<DT>(draft + i * A.ld_draft * ES, 0, nv, A.V, c, tab, sh);
        d -= ((double)s_zd[i] - (double)q.ref) * c;
        over /= q.s;
      }
      if (tid == 0) s_ratio[i] = exp2(d) / over;
    }
    __syncthreads();
    if (warp == 0) {
      const unsigned stop = __ballot_sync(kAll, lane < n && !((double)s_u[lane < n ? lane : 0] < s_ratio[lane < n ? lane : 0]));
      if (lane == 0) s_m = stop ? __ffs(stop) - 1 : n;
    }
    __syncthreads();
  }
  const int m = kind < 0 ? 0 : s_m;
  const bool rejected = m < n;
  const bool use_q = rejected && with_q;
  const double sum_t = kind < 0 ? 0.0 : s_sum[m], sum_q = use_q ? s_sum[N + 1 + m] : 1.0;
  const bool usable = sum_t > 0 && sum_q > 0;               // else the row to draw from is bad: token -1
  if (split == 0) {
    if (tid == 0) A.out_n_accepted[b] = m;
    for (int i = tid; i <= N; i += kThreads) {
      int32_t tok = -1;
      float lp = 0.f;
      if (i < m || (i == m && kind == 0 && usable)) {
        tok = i < m ? s_tok[i] : s_arg[m];
        const float z = i < m ? s_zt[i] : Vec<DT>::load_scalar(target + i * A.ld_target * ES, tok);
        if (A.out_logp) lp = (float)((((double)z - (double)s_ref[i]) * c - log2(s_sum[i])) * kLn2D);
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
  double c1 = kLn2D, c2 = kLn2Square;
  asm volatile("" : "+d"(c1), "+d"(c2));                    // (values to keep in registers, not constants)
  auto row_of = [&](const char* z, int r, double* table) {
    DrawRow d;
    d.z = z;
    d.c = c;
    d.ref = (double)s_ref[r];
    d.off = -d.ref * c;
    d.cut = __double2float_ru(d.ref + kClamp / c);
    d.c1 = c1;
    d.c2 = c2;
    d.tab = table;
    if (tid < 32) table[tid] = table_entry(tid, s_inv[r]);
    return d;
  };
  const DrawRow T = row_of(target + m * A.ld_target * ES, m, tab_t);
  const DrawRow D = use_q ? row_of(draft + m * A.ld_draft * ES, N + 1 + m, tab_q) : T;
  const bool far = !(fabs(T.off) < 0x1p20 && fabs(D.off) < 0x1p20);
  const int64_t skip = rejected && !with_q ? s_tok[m] : -1; // a draft without logits had all its mass there
  __syncthreads();
  const int64_t nv = (A.V + W - 1) / W;
  const int segs = A.n_segs;
  SegPart* parts = (SegPart*)A.segs + b * segs;
  {
    const int g0 = split * A.block_segs, g1 = g0 + A.block_segs < segs ? g0 + A.block_segs : segs;
    const int first = g0 + warp, count = first < g1 ? (g1 - first + kWarps - 1) / kWarps : 0;
    if (far) {
      if (use_q) segments<DT, true, true>(T, D, skip, first, kWarps, count, A.seg_vecs, nv, A.V, parts);
      else segments<DT, false, true>(T, D, skip, first, kWarps, count, A.seg_vecs, nv, A.V, parts);
    } else {
      if (use_q) segments<DT, true, false>(T, D, skip, first, kWarps, count, A.seg_vecs, nv, A.V, parts);
      else segments<DT, false, false>(T, D, skip, first, kWarps, count, A.seg_vecs, nv, A.V, parts);
    }
    if (lane == 0) {
      int before;
      asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(&A.ticket[b]) : "memory");
      if (before == A.draw_splits * kWarps - 1) s_last = 1;
    }
  }
  __syncthreads();
  if (!s_last) return;                                      // (the block whose warp came last has every other segment's sums in sight)

  // last block of the sequence: exact normalisers, the segment that the draw falls into, the element in it.  Every thread has a
  // contiguous run of at most kPer segments.
  const double2* sp = (const double2*)parts;
  const int per = (segs + kThreads - 1) / kThreads;
  constexpr int kPer = kVerifyMaxSegs / kThreads;
  double mass_of[kPer], q_of[kPer], all_of[kPer];
  const double tiny = kTiny * s_inv[m];
  double a = 1.0, cq = 0.0, P = 1.0, mine, total, before;
  for (bool again = false;; again = true) {
    double pa = 0, qa = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      mass_of[k] = q_of[k] = all_of[k] = 0;
      const int g = tid * per + k;
      if (k < per && g < segs) {
        const double2 w = __ldcg(sp + 2 * g), v = __ldcg(sp + 2 * g + 1);
        mass_of[k] = w.x;
        q_of[k] = w.y;
        all_of[k] = v.x;
        pa += v.x;
        qa += v.y;
      }
    }
    double apart = 0;
    if (again) {
      a = cq = 1.0;
    } else if (use_q) {
      P = block_sum_d(pa, sh);
      const double Q = block_sum_d(qa, sh);
      a = 1.0 / P;
      cq = 1.0 / Q;
      apart = fabs(P - Q);
    }
    mine = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      mass_of[k] = mass_of[k] * a - q_of[k] * cq;
      if (!(mass_of[k] > tiny)) mass_of[k] = 0;
      mine += mass_of[k];
    }
    before = block_scan_d(mine, sh, &total);
    // Where p / q lies between 1 and P / Q the first pass's sums had the sign of p - q wrong, and such an entry counts with up to
    // |P / Q - 1| p (1e-7 p and less) more or less than it should.  Two nearly equal rows, where that may count, are taken
    // again with the sums known now.
    if (!(apart * kApart > total)) break;
    if (tid < 32) {
      tab_t[tid] = table_entry(tid, s_inv[m] * a);
      tab_q[tid] = table_entry(tid, s_inv[N + 1 + m] * cq);
    }
    __syncthreads();
    segments_again<DT>(T, D, far, segs, A.seg_vecs, nv, A.V, parts);
    __syncthreads();
  }
  const bool whole = use_q && !(total > 0);                 // nothing left above zero: draw from p itself
  if (whole) {
    mine = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      mass_of[k] = all_of[k] * a > tiny ? all_of[k] * a : 0;
      mine += mass_of[k];
    }
    before = block_scan_d(mine, sh, &total);
  }
  int64_t token = skip;                                     // (without draft logits: p itself is 1 there)
  if (total > 0) {
    // the draw falls into the last segment with mass whose sum before it is within u S; beyond the end (u >= 1, rounding) that
    // is the last segment with mass
    const double want = u_sample > 0.f ? (double)u_sample * total : 0.0;
    Pick pick{-1, 0.0};
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (mass_of[k] > 0 && before <= want) pick = Pick{tid * per + k, before};
      before += mass_of[k];
    }
    Pick seg = block_last(pick.place, pick.before, s_pick);
    if (seg.place < 0) seg = Pick{0, 0.0};                  // (cannot be: the first segment with mass has nothing before it)
    const int64_t e0 = seg.place * A.seg_vecs * W, e1 = e0 + A.seg_vecs * W < A.V ? e0 + A.seg_vecs * W : A.V;
    const int64_t each = (A.seg_vecs * W + kThreads - 1) / kThreads;
    const int64_t f0 = e0 + each * tid, f1 = f0 + each < e1 ? f0 + each : e1;
    const double floor_t = T.ref + kFloor / c, floor_q = D.ref + kFloor / c;
    auto mass = [&](int64_t v) {
      const float zt = Vec<DT>::load_scalar(T.z, v);
      const double p = (double)zt < floor_t || v == skip ? 0.0 : (far ? T.prob<true>(zt) : T.prob<false>(zt)) * a;
      if (whole || !use_q) return p;
      const float zq = Vec<DT>::load_scalar(D.z, v);
      const double q = (double)zq < floor_q ? 0.0 : (far ? D.prob<true>(zq) : D.prob<false>(zq)) * cq;
      return p > q ? p - q : 0.0;
    };
    constexpr int kKeep = 4;                                // a thread's first elements are kept for the second walk
    double keep[kKeep];
    mine = 0;
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
      keep[k] = f0 + k < f1 ? mass(f0 + k) : 0.0;
      mine += keep[k];
    }
    for (int64_t v = f0 + kKeep; v < f1; ++v) mine += mass(v);
    before = seg.before + block_scan_d(mine, sh, &total);
    pick = Pick{-1, 0.0};
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
      if (keep[k] > 0 && before <= want) pick = Pick{(int)(f0 + k - e0), 0.0};
      before += keep[k];
    }
    for (int64_t v = f0 + kKeep; v < f1 && before <= want; ++v) {
      const double w = mass(v);
      if (w > 0) pick = Pick{(int)(v - e0), 0.0};
      before += w;
    }
    const Pick at = block_last(pick.place, 0.0, s_pick);
    token = e0 + (at.place < 0 ? 0 : at.place);
  }
  if (tid == 0) {
    const bool have = token >= 0 && token < A.V;
    A.out_tokens[b * (N + 1) + m] = have ? (int32_t)token : -1;
    if (A.out_logp)
      A.out_logp[b * (N + 1) + m] =
          have ? (float)((((double)Vec<DT>::load_scalar(T.z, token) - T.ref) * c - log2(sum_t * P)) * kLn2D) : 0.f;
  }
}

}  // namespace

VerifyPlan verify_plan(int64_t B, int N, int64_t V, int dtype, bool with_draft, int sms) {
  VerifyPlan p{};
  p.rows_per_seq = N + 1 + (with_draft ? N : 0);
  const int64_t nv = (V + (dtype == JP_BF16 ? 7 : 3)) / (dtype == JP_BF16 ? 8 : 4);
  const int64_t lines = B * p.rows_per_seq;
  auto pick = [&](int64_t want, int64_t most) { return (int)(want < 1 ? 1 : want > most ? (most < 1 ? 1 : most) : want); };
  // Slices of the row pass: 64 KB where there are rows enough to fill the SMs several times over, down to 8 KB where there are few.
  int want = pick((sms * 10 + lines - 1) / lines, (nv + 511) / 512);
  const int coarse = pick((nv + 4095) / 4096, kVerifyMaxSplits);
  want = want < coarse ? coarse : (want > kVerifyMaxSplits ? kVerifyMaxSplits : want);
  p.split_vecs = (nv + want - 1) / want;
  p.splits = (int)((nv + p.split_vecs - 1) / p.split_vecs);
  // Segments of the draw: short ones where there are few sequences, longer ones (fewer reductions) where they fill the SMs; blocks:
  // one wave of kDrawBlocks per SM.
  const int64_t warps = (int64_t)sms * kDrawBlocks * kWarps;
  p.seg_vecs = B * ((nv + 127) / 128) >= 2 * warps ? 128 : B * ((nv + 63) / 64) >= warps ? 64 : 32;
  if (p.seg_vecs * kVerifyMaxSegs < nv) p.seg_vecs = ((nv + kVerifyMaxSegs - 1) / kVerifyMaxSegs + 31) / 32 * 32;
  p.n_segs = (int)((nv + p.seg_vecs - 1) / p.seg_vecs);
  p.draw_splits = pick(sms * kDrawBlocks / B, (p.n_segs + kWarps - 1) / kWarps);
  p.block_segs = (p.n_segs + p.draw_splits - 1) / p.draw_splits;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  p.parts_off = up((size_t)B * 4);
  p.segs_off = p.parts_off + up((size_t)lines * p.splits * sizeof(RowPart));
  p.bytes = p.segs_off + up((size_t)B * p.n_segs * sizeof(SegPart));
  return p;
}

cudaError_t launch_verify(VerifyArgs a, int dtype, cudaStream_t s) {
  const dim3 g1((unsigned)a.splits, (unsigned)a.rows_per_seq, (unsigned)a.B), g2((unsigned)a.draw_splits, (unsigned)a.B);
  constexpr int kPlaces = kGroups * kGroup * kThreads * 16;
  auto* rows = dtype == JP_BF16 ? verify_rows_kernel<JP_BF16> : verify_rows_kernel<JP_F32>;
  rows<<<g1, kThreads, kPlaces, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = g2;
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;      // may set up while the row pass runs
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return dtype == JP_BF16 ? cudaLaunchKernelEx(&cfg, verify_draw_kernel<JP_BF16>, a)
                          : cudaLaunchKernelEx(&cfg, verify_draw_kernel<JP_F32>, a);
}

}  // namespace jp
