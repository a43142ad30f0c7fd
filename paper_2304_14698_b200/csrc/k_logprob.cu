// Rows of logits as categorical distributions: the log probability of a given choice, the entropy and the best
// alternatives (xrl_logprob), and the gradient of the first two with respect to the logits (xrl_logprob_grad).
//
// A row's support is what its mask leaves and what is above -infinity; with m its largest logit, s the scale,
//   l = ln sum_j exp(s (x_j - m)),   ln p_j = s (x_j - m) - l,   H = -sum_j p_j ln p_j,
//   dx_j = s [ dlogp (1[j = t] - p_j) - dH p_j (ln p_j + H) ]          (0 outside the support).
// Both are bound by HBM: the forward pass reads every logit once, the gradient reads and writes each once.
#include <cuda.h>

#include "xrl_internal.cuh"

namespace xrl {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -INFINITY;
constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kMostTop = 32;             // alternatives: one lane of a warp each
// What -infinity becomes in the gradient, where p = 2^((x - m) c - l) is 0 for it and a product with it finite.  (A bf16
// number, 0xF149.)
constexpr float kFloor = -9.953287e29f;
// The sums of a row are taken relative to r = c m rounded, which all terms share: as long as |c m| is at most 2^24 that is
// off by 1 at most and cancels.  Logits below -2^23 / c count as that (their share is 0 all the same: a row whose largest
// is below -2^22 / c, or above 2^24 / c, is done again by careful_row).
constexpr float kLowest = -8388608.f, kLow = -4194304.f, kHigh = 16777216.f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {     // a number that is none stays one
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// two fp32 numbers in one register pair, and the instructions that take both at once
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(f32x2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {         // numbers that are none are passed over
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <typename T> __device__ __forceinline__ float load1(const T* p) { return to_float(__ldg(p)); }
template <> __device__ __forceinline__ float load1<bf16>(const bf16* p) {
  return bf16_bits_to_float(__ldg(reinterpret_cast<const uint16_t*>(p)));
}

struct RowArgs {
  const void* x;
  int64_t x_stride;
  const int32_t* token;
  const uint8_t* mask;
  int64_t mask_stride;
  int64_t rows;
  int32_t vocab;
  float scale;
};

// The sums of part of a row relative to the exponent r (in powers of two): s = sum 2^(c x - r), t = sum of the same
// times (c x - r); m is the largest x.  r = c m rounded: all terms share it, so its rounding cancels.
struct Sums {
  float m, r, s, t;
};
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
  Sums o;
  o.m = fmaxf(a.m, b.m);
  o.r = fmaxf(a.r, b.r);
  const float da = a.r - o.r, db = b.r - o.r, ea = ex2(da), eb = ex2(db);
  o.s = a.s * ea + b.s * eb;
  o.t = fmaf(da, a.s, a.t) * ea + fmaf(db, b.s, b.t) * eb;
  return o;
}
__device__ __forceinline__ Sums join_warp(Sums v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    Sums o;
    o.m = __shfl_xor_sync(kAll, v.m, d);
    o.r = __shfl_xor_sync(kAll, v.r, d);
    o.s = __shfl_xor_sync(kAll, v.s, d);
    o.t = __shfl_xor_sync(kAll, v.t, d);
    v = join(v, o);
  }
  return v;
}

// ---- the best k of a set, one per lane, best first; ties go to the lower index ---------------------------------
struct Best {
  float v = kNegInf;
  int32_t i = INT32_MAX;
};
__device__ __forceinline__ bool better(float v, int32_t i, float w, int32_t j) { return v > w || (v == w && i < j); }
// every lane offers one entry (v = -infinity: none); `last` is the list's k-th entry
__device__ __forceinline__ void offer(Best& mine, Best& last, float v, int32_t i, int k, int lane) {
  while (true) {
    const unsigned some = __ballot_sync(kAll, v > kNegInf && better(v, i, last.v, last.i));
    if (!some) return;
    const int from = __ffs(some) - 1;
    const float cv = __shfl_sync(kAll, v, from);
    const int32_t ci = __shfl_sync(kAll, i, from);
    if (lane == from) v = kNegInf;
    const int at = __popc(__ballot_sync(kAll, better(mine.v, mine.i, cv, ci)));
    const float uv = __shfl_up_sync(kAll, mine.v, 1);
    const int32_t ui = __shfl_up_sync(kAll, mine.i, 1);
    if (lane > at) { mine.v = uv; mine.i = ui; }
    if (lane == at) { mine.v = cv; mine.i = ci; }
    last.v = __shfl_sync(kAll, mine.v, k - 1);
    last.i = __shfl_sync(kAll, mine.i, k - 1);
  }
}

// ---- a row's results from its sums ------------------------------------------------------------------------------
struct RowOut {
  float *logp, *entropy, *norm;
  int32_t* top_token;
  float* top_logp;
  int top;
};
struct RowNorm {
  float m, l;                            // largest logit, ln sum exp(s (x - m))
};
// from sums relative to r (careful: relative to c m itself)
__device__ __forceinline__ RowNorm norm_of(const Sums& v, float c) {
  return {v.m, kLn2 * (log2f(v.s) - fmaf(v.m, c, -v.r))};
}
__device__ __forceinline__ float entropy_of(const Sums& v) {
  const float h = kLn2 * (log2f(v.s) - v.t / v.s);
  return h < 0.f ? 0.f : h;              // a rounding below 0, where one entry has all the probability
}
__device__ __forceinline__ float logp_of(float x, const RowNorm& n, float scale) {
  return x > kNegInf || x != x ? fmaf(scale, x - n.m, -n.l) : kNegInf;
}
template <typename T>
__device__ __forceinline__ void write_row(const RowArgs& a, const RowOut& o, int64_t row, const RowNorm& n, float entropy) {
  if (o.norm) *reinterpret_cast<float2*>(o.norm + 2 * row) = make_float2(n.m, n.l);
  if (o.entropy) o.entropy[row] = entropy;
  if (o.logp) {
    const int32_t t = a.token[row];
    float lp = 0.f;
    if (t < -1 || t >= a.vocab) {
      lp = NAN;
    } else if (t >= 0) {
      float x = load1(static_cast<const T*>(a.x) + row * a.x_stride + t);
      if (a.mask && !a.mask[row * a.mask_stride + t]) x = kNegInf;
      lp = logp_of(x, n, a.scale);
    }
    o.logp[row] = lp;
  }
}
__device__ __forceinline__ void write_top(const RowArgs& a, const RowOut& o, int64_t row, const RowNorm& n, const Best& b,
                                          int lane) {
  if (lane < o.top) {
    const bool some = b.v > kNegInf;
    o.top_token[row * o.top + lane] = some ? b.i : -1;
    o.top_logp[row * o.top + lane] = some ? logp_of(b.v, n, a.scale) : kNegInf;
  }
}

// ---- short rows: a warp per row, the row in registers -----------------------------------------------------------
template <typename T, int E, bool MASK>
__global__ void __launch_bounds__(128) k_logprob_warp(RowArgs a, RowOut o) {
  enter();
  const int lane = threadIdx.x & 31;
  const float c = a.scale * kLog2e;
  for (int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 5); row < a.rows; row += int64_t(gridDim.x) * 4) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = e * 32 + lane;
      v[e] = j < a.vocab ? load1(x + j) : kNegInf;
      if (MASK && j < a.vocab && !__ldg(a.mask + row * a.mask_stride + j)) v[e] = kNegInf;
    }
    float m = kNegInf;
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, d));
    const float base = m > kNegInf ? m : 0.f;
    Sums q = {m, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = (v[e] - base) * c, p = ex2(d);
      q.s += p;
      q.t = p > 0.f || p != p ? fmaf(p, d, q.t) : q.t;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      q.s += __shfl_xor_sync(kAll, q.s, d);
      q.t += __shfl_xor_sync(kAll, q.t, d);
    }
    const bool empty = q.s == 0.f;
    const RowNorm n = {m, empty ? kNegInf : kLn2 * log2f(q.s)};
    if (lane == 0) write_row<T>(a, o, row, n, empty ? 0.f : entropy_of(q));
    if (o.top) {
      Best mine, last;
#pragma unroll
      for (int e = 0; e < E; ++e) offer(mine, last, v[e], e * 32 + lane, o.top, lane);
      write_top(a, o, row, n, mine, lane);
    }
  }
}

// ---- long rows: a CTA, or a cluster of them, per row ------------------------------------------------------------
// 16 bytes of a row as they lie in memory, entries without their mask byte at -infinity
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
  static __device__ __forceinline__ void drop(uint4& v, uint32_t m0, uint32_t) {
    if (!(m0 & 0xFFu)) v.x = 0xFF800000u;
    if (!(m0 & 0xFF00u)) v.y = 0xFF800000u;
    if (!(m0 & 0xFF0000u)) v.z = 0xFF800000u;
    if (!(m0 & 0xFF000000u)) v.w = 0xFF800000u;
  }
};
template <> struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
  static __device__ __forceinline__ uint32_t drop2(uint32_t v, uint32_t m, uint32_t lo, uint32_t hi) {
    if (!(m & lo)) v = (v & 0xFFFF0000u) | 0xFF80u;
    if (!(m & hi)) v = (v & 0xFFFFu) | 0xFF800000u;
    return v;
  }
  static __device__ __forceinline__ void drop(uint4& v, uint32_t m0, uint32_t m1) {
    v.x = drop2(v.x, m0, 0xFFu, 0xFF00u);
    v.y = drop2(v.y, m0, 0xFF0000u, 0xFF000000u);
    v.z = drop2(v.z, m1, 0xFFu, 0xFF00u);
    v.w = drop2(v.w, m1, 0xFF0000u, 0xFF000000u);
  }
};
// N mask bytes from any address: the aligned words that hold them (each holds one of them at least)
template <int N>
__device__ __forceinline__ void mask_words(const uint8_t* p, uint32_t& m0, uint32_t& m1) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  const uint32_t* w = reinterpret_cast<const uint32_t*>(at & ~uintptr_t(3));
  const uint32_t off = uint32_t(at & 3) * 8;
  const uint32_t w0 = __ldg(w), w1 = N == 8 || off ? __ldg(w + 1) : 0u;
  m0 = __funnelshift_r(w0, w1, off);
  m1 = 0;
  if (N == 8) m1 = __funnelshift_r(w1, off ? __ldg(w + 2) : 0u, off);
}
__device__ __forceinline__ uint4 load_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// A row as `head` single entries up to the first 16-byte boundary, `vecs` whole vectors, and the rest
template <typename T> struct Row {
  const T* x;
  const uint8_t* mask;
  int head, vecs, tail, vocab;
  __device__ __forceinline__ Row(const RowArgs& a, int64_t row, bool masked) {
    constexpr int N = Vec<T>::N;
    x = static_cast<const T*>(a.x) + row * a.x_stride;
    mask = masked ? a.mask + row * a.mask_stride : nullptr;
    vocab = a.vocab;
    head = int((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / int(sizeof(T));
    if (head > vocab) head = vocab;
    vecs = (vocab - head) / N;
    tail = vocab - head - vecs * N;
  }
  __device__ __forceinline__ float at(int j) const {
    const float v = load1(x + j);
    return mask && !__ldg(mask + j) ? kNegInf : v;
  }
  // the entries outside whole vectors: at most 2 (N - 1) of them, number i of 0..15
  __device__ __forceinline__ int edge(int i) const {
    return i < head ? i : i - head < tail ? vocab - tail + (i - head) : -1;
  }
  template <bool MASK> __device__ __forceinline__ uint4 vec(int j) const {
    constexpr int N = Vec<T>::N;
    uint4 v = load_stream(x + head + size_t(j) * N);
    if (MASK) {
      uint32_t m0, m1;
      mask_words<N>(mask + head + size_t(j) * N, m0, m1);
      Vec<T>::drop(v, m0, m1);
    }
    return v;
  }
};
__device__ __forceinline__ uint32_t key_of(float v) {          // unsigned order = order of the floats
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float float_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

// A row whose logits are too far from 0 for the above: largest first, then the sums of differences.
template <typename T, int THREADS>
__device__ __noinline__ void careful_row(const RowArgs& a, bool masked, int64_t row, float* red, Sums& out) {
  const Row<T> r(a, row, masked);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float c = a.scale * kLog2e;
  float m = kNegInf;
  for (int j = threadIdx.x; j < r.vocab; j += THREADS) m = fmaxf(m, r.at(j));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, d));
  __syncthreads();
  if (lane == 0) red[warp] = m;
  __syncthreads();
  for (int w = 0; w < THREADS / 32; ++w) m = fmaxf(m, red[w]);
  const float base = m > kNegInf ? m : 0.f;
  float s = 0.f, t = 0.f;
  for (int j = threadIdx.x; j < r.vocab; j += THREADS) {
    const float d = (r.at(j) - base) * c, p = ex2(d);
    s += p;
    if (p > 0.f || p != p) t = fmaf(p, d, t);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    s += __shfl_xor_sync(kAll, s, d);
    t += __shfl_xor_sync(kAll, t, d);
  }
  __syncthreads();
  if (lane == 0) { red[warp] = s; red[32 + warp] = t; }
  __syncthreads();
  s = t = 0.f;
  for (int w = 0; w < THREADS / 32; ++w) { s += red[w]; t += red[32 + w]; }
  out = {m, 0.f, s, t};
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive_wait() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote(const void* p, uint32_t rank) {     // the same address in another CTA of the cluster
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(uint32_t(__cvta_generic_to_shared(p))), "r"(rank));
  return r;
}
__device__ __forceinline__ float remote_f(uint32_t at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ int32_t remote_i(uint32_t at) {
  int32_t v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

// The logits of U vectors for the arithmetic, none below `floor`: N pairs of fp32 numbers; and the largest of them as they were
template <int U>
__device__ __forceinline__ float spread(const uint4 (&v)[U], f32x2 (&f)[U * 4], float floor, const bf16*) {
  const uint32_t f2 = pack_bf16x2(floor, floor);
  const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
  uint32_t m = w[0];
#pragma unroll
  for (int i = 1; i < U * 4; ++i) m = max_bf16x2(m, w[i]);
#pragma unroll
  for (int i = 0; i < U * 4; ++i) {
    const uint32_t x = max_nan_bf16x2(w[i], f2);
    f[i] = pair(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
  }
  return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
}
template <int U>
__device__ __forceinline__ float spread(const uint4 (&v)[U], f32x2 (&f)[U * 2], float floor, const float*) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
  float m = __uint_as_float(w[0]);
#pragma unroll
  for (int i = 1; i < U * 4; ++i) m = fmaxf(m, __uint_as_float(w[i]));
#pragma unroll
  for (int i = 0; i < U * 2; ++i)
    f[i] = pair(max_nan(__uint_as_float(w[2 * i]), floor), max_nan(__uint_as_float(w[2 * i + 1]), floor));
  return m;
}
// adds them to a thread's sums
template <typename T, int U>
__device__ __forceinline__ void add_chunk(Sums& q, const uint4 (&v)[U], float c, float floor) {
  constexpr int P = U * Vec<T>::N / 2;
  f32x2 f[P];
  const float m = fmaxf(q.m, spread<U>(v, f, floor, static_cast<const T*>(nullptr)));
  const float r = fmaxf(m, floor) * c, d = q.r - r, e = ex2(d);
  const f32x2 cc = pair(c, c), rr = pair(-r, -r);
  f32x2 s[2] = {pair(q.s * e, 0.f), 0ull}, t[2] = {pair(fmaf(d, q.s, q.t) * e, 0.f), 0ull};
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const f32x2 y = fma2(f[i], cc, rr);
    float y0, y1;
    unpair(y, y0, y1);
    const f32x2 p = pair(ex2(y0), ex2(y1));
    s[i & 1] = add2(s[i & 1], p);
    t[i & 1] = fma2(p, y, t[i & 1]);
  }
  float a, b;
  unpair(add2(s[0], s[1]), a, b);
  q.s = a + b;
  unpair(add2(t[0], t[1]), a, b);
  q.t = a + b;
  q.m = m;
  q.r = r;
}

// ---- the best k of a CTA's part of a row -----------------------------------------------------------------------
// Candidates in shared memory: the k best of n <= THREADS, by counting for each how many are better
template <int THREADS> struct Candidates {
  float v[THREADS];
  int32_t i[THREADS];
  float best_v[kMostTop];
  int32_t best_i[kMostTop];
  int n;
};
template <int THREADS> __device__ __forceinline__ void rank_candidates(Candidates<THREADS>& s, int n, int k) {
  if (threadIdx.x < kMostTop) { s.best_v[threadIdx.x] = kNegInf; s.best_i[threadIdx.x] = INT32_MAX; }
  __syncthreads();
  if (int(threadIdx.x) < n) {
    const float v = s.v[threadIdx.x];
    const int32_t i = s.i[threadIdx.x];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += better(s.v[j], s.i[j], v, i) ? 1 : 0;
    if (rank < k && v > kNegInf) { s.best_v[rank] = v; s.best_i[rank] = i; }
  }
  __syncthreads();
}

// A thread's largest logit (thread_max) is known.  At least k threads hold one of `bound` or more, so the k best are no
// less; few other logits are, and only the threads whose largest is that high have any.  Their vectors are read again, spread
// over the lanes of their warp, and what reaches the bound is ranked.  Where that is more than one entry per thread of
// the CTA (equal logits everywhere, or fewer than k threads with any) each warp keeps a sorted list of its whole part instead.
template <typename T, int THREADS, bool MASK>
__device__ __forceinline__ void best_of_part(const Row<T>& r, int v0, int v1, bool edges, float thread_max, float part_max, int k,
                                             Candidates<THREADS>& s, uint32_t* red) {
  constexpr int N = Vec<T>::N, U = 4, W = THREADS / 32, GROUP = THREADS / 32;
  static_assert(GROUP <= 32, "32 groups of threads");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t mine = key_of(thread_max);
  uint32_t g = mine;
#pragma unroll
  for (int d = 1; d < GROUP; d <<= 1) g = max(g, __shfl_xor_sync(kAll, g, d));
  if (threadIdx.x % GROUP == 0) red[threadIdx.x / GROUP] = g;
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  // 32 groups, each with a thread at `lo` or above
  uint32_t lo = __reduce_min_sync(kAll, red[lane]), hi = key_of(part_max);
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    const int cnt = __syncthreads_count(mine >= mid);
    if (cnt >= k) {
      lo = mid;
      if (cnt <= k + k / 2) break;
    } else {
      hi = mid - 1;
    }
  }
  const float bound = float_of(lo);
  const unsigned flags = __ballot_sync(kAll, thread_max > kNegInf && mine >= lo);
  const int iters = (v1 - v0 + THREADS - 1) / THREADS, items = __popc(flags) * iters;
  auto put = [&](float v, int32_t i) {
    if (v >= bound && v > kNegInf) {
      const int at = atomicAdd(&s.n, 1);
      if (at < THREADS) { s.v[at] = v; s.i[at] = i; }
    }
  };
  for (int i = lane; i < items; i += 32) {
    const int j = v0 + warp * 32 + __fns(flags, 0, i / iters + 1) + (i % iters) * THREADS;
    if (j < v1) {
      const uint4 v = r.template vec<MASK>(j);
      float f[N];
      unpack(v, f);
#pragma unroll
      for (int e = 0; e < N; ++e) put(f[e], r.head + j * N + e);
    }
  }
  if (edges && threadIdx.x < 16) {
    const int j = r.edge(threadIdx.x);
    if (j >= 0) put(r.at(j), j);
  }
  __syncthreads();
  int n = s.n;
  if (n > THREADS) {
    Best mine_b, last;
    for (int j0 = v0 + warp * 32; j0 < v1; j0 += U * THREADS) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = j0 + u * THREADS + lane;
        v[u] = j < v1 ? r.template vec<MASK>(j) : Vec<T>::none();
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[N];
        unpack(v[u], f);
#pragma unroll
        for (int i = 0; i < N; ++i) offer(mine_b, last, f[i], r.head + (j0 + u * THREADS + lane) * N + i, k, lane);
      }
    }
    if (edges && warp == 0) {
      const int j = lane < 16 ? r.edge(lane) : -1;
      offer(mine_b, last, j >= 0 ? r.at(j) : kNegInf, j, k, lane);
    }
    s.v[threadIdx.x] = mine_b.v;
    s.i[threadIdx.x] = mine_b.i;
    __syncthreads();
    n = THREADS;
  }
  rank_candidates<THREADS>(s, n, k);
}

template <typename T, int THREADS, bool MASK, bool TOP>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_logprob_cta(RowArgs a, RowOut o, int parts) {
  enter();
  constexpr int U = 4, W = THREADS / 32;
  __shared__ Sums s_sums[W];
  __shared__ float s_red[64];
  __shared__ Candidates<TOP ? THREADS : 32> s_best;
  __shared__ Sums s_part;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = int64_t(blockIdx.x) / parts;
  const int part = parts > 1 ? int(cluster_rank()) : 0;
  const Row<T> r(a, row, MASK);
  const float c = a.scale * kLog2e;
  const int v0 = int(int64_t(r.vecs) * part / parts), v1 = int(int64_t(r.vecs) * (part + 1) / parts);
  // (as a bf16 number, which it is for both types; rounded, it is within 2^-9 of itself)
  const float floor = to_float(bf16(kLowest / c));
  const Sums zero = {kNegInf, floor * c, 0.f, 0.f};

  Sums q = zero;
  for (int j = v0 + threadIdx.x; j < v1; j += U * THREADS) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = j + u * THREADS < v1 ? r.template vec<MASK>(j + u * THREADS) : Vec<T>::none();
    add_chunk<T, U>(q, v, c, floor);
  }
  const float thread_max = q.m;          // (of its whole vectors)
  if (part == 0 && threadIdx.x < 16) {
    const int j = r.edge(threadIdx.x);
    if (j >= 0) {
      const float x = r.at(j), z = max_nan(x, floor), e = fmaxf(x, floor) * c, y = fmaf(z, c, -e), p = ex2(y);
      q = join(q, Sums{fmaxf(x, kNegInf), e, p, p * y});
    }
  }
  q = join_warp(q);
  if (lane == 0) s_sums[warp] = q;
  __syncthreads();
  q = lane < W ? s_sums[lane] : zero;
  q = join_warp(q);

  if (TOP) best_of_part<T, TOP ? THREADS : 32, MASK>(r, v0, v1, part == 0, thread_max, q.m, o.top, s_best, reinterpret_cast<uint32_t*>(s_red));
  if (parts > 1) {
    if (threadIdx.x == 0) s_part = q;
    cluster_arrive_wait();
    if (part == 0) {
      if (lane > 0 && lane < parts) {
        const uint32_t at = remote(&s_part, lane);
        q = {remote_f(at), remote_f(at + 4), remote_f(at + 8), remote_f(at + 12)};
      } else if (lane >= parts) {
        q = zero;
      }
      q = join_warp(q);
      if (TOP) {
        const int p = threadIdx.x / kMostTop, e = threadIdx.x % kMostTop;
        float v = kNegInf;
        int32_t i = INT32_MAX;
        if (p < parts) {
          v = remote_f(remote(&s_best.best_v[e], p));
          i = remote_i(remote(&s_best.best_i[e], p));
        }
        s_best.v[threadIdx.x] = v;
        s_best.i[threadIdx.x] = i;
      }
    }
    cluster_arrive_wait();               // nobody leaves, and nothing is written again, while it is read
    if (part != 0) return;
    if (TOP) rank_candidates(s_best, parts * kMostTop, o.top);
  }
  RowNorm n;
  float entropy;
  if (q.m > kNegInf && q.m < INFINITY && !(q.m * c > kLow && q.m * c < kHigh)) {
    Sums z;
    careful_row<T, THREADS>(a, MASK, row, s_red, z);
    n = {z.m, kLn2 * log2f(z.s)};
    entropy = entropy_of(z);
  } else if (q.m > kNegInf || q.s != q.s) {
    n = norm_of(q, c);
    if (q.s != q.s) n.l = NAN;
    entropy = entropy_of(q);
  } else {
    n = {kNegInf, kNegInf};
    entropy = 0.f;
  }
  if (threadIdx.x == 0) write_row<T>(a, o, row, n, entropy);
  if (TOP && warp == 0) write_top(a, o, row, n, Best{s_best.best_v[lane], s_best.best_i[lane]}, lane);
}

// ---- gradient ---------------------------------------------------------------------------------------------------
struct GradArgs {
  const float *norm, *dlogp, *entropy, *dentropy;
  void* grad;
  int64_t grad_stride;
};
// One entry as the formula says it; what the fast form below leaves out
struct RowGrad {
  float m, c, l2, dl, dh, ent;           // l2: l in powers of two; dl, dh times the scale
  int32_t t;
  __device__ __forceinline__ float operator()(float x, int j) const {
    const float y = fmaf(x - m, c, -l2), p = ex2(y);
    const float g = fmaf(dl, (j == t ? 1.f : 0.f) - p, p > 0.f || p != p ? -dh * p * fmaf(kLn2, y, ent) : 0.f);
    return x > kNegInf || x != x ? g : 0.f;
  }
};
template <typename T> __device__ __forceinline__ uint4 round_pairs(const f32x2* g);
template <> __device__ __forceinline__ uint4 round_pairs<bf16>(const f32x2* g) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpair(g[i], f[2 * i], f[2 * i + 1]);
  return pack(f);
}
template <> __device__ __forceinline__ uint4 round_pairs<float>(const f32x2* g) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) unpair(g[i], f[2 * i], f[2 * i + 1]);
  return pack(f);
}
// A warp takes 32 x U vectors of a row at a time.  With p = 2^y the entry is p (A + B y), plus dl at the token:
// A = -(dl + dh H), B = -dh ln 2.  -infinity becomes kFloor first, for which p is 0; rows where that does not do (a norm
// or gradients that are not finite, logits all below the floor) go entry by entry.
template <typename T, bool MASK>
__global__ void __launch_bounds__(256) k_logprob_grad(RowArgs a, GradArgs g, int segs) {
  enter();
  constexpr int N = Vec<T>::N, U = 4, P = N / 2;
  const int lane = threadIdx.x & 31;
  const int64_t items = a.rows * segs, step = int64_t(gridDim.x) * 8;
  for (int64_t item = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5); item < items; item += step) {
    const int64_t row = items <= INT32_MAX ? int64_t(uint32_t(item) / uint32_t(segs)) : item / segs;
    const int seg = int(item - row * segs);
    const Row<T> r(a, row, MASK);
    const int j0 = seg * 32 * U + lane;
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = j0 + u * 32 < r.vecs ? r.template vec<MASK>(j0 + u * 32) : Vec<T>::none();
    T* out = static_cast<T*>(g.grad) + row * g.grad_stride;
    RowGrad f;
    const float2 n = __ldg(reinterpret_cast<const float2*>(g.norm) + row);
    f.t = a.token ? __ldg(a.token + row) : -1;
    f.m = n.x;
    f.c = a.scale * kLog2e;
    f.l2 = n.y * kLog2e;
    f.dl = f.t == -1 || !g.dlogp ? 0.f : f.t < -1 || f.t >= a.vocab ? NAN : a.scale * __ldg(g.dlogp + row);
    f.dh = g.dentropy ? a.scale * __ldg(g.dentropy + row) : 0.f;
    f.ent = g.dentropy ? __ldg(g.entropy + row) : 0.f;
    const bool whole = ((reinterpret_cast<uintptr_t>(out + r.head)) & 15) == 0;
    const float A = -fmaf(f.dh, f.ent, f.dl), B = -f.dh * kLn2;
    // (every product of the fast form is finite then)
    const bool fast = f.m > kFloor && fabsf(A) + fabsf(B) * fmaf(fabsf(f.m) - kFloor, f.c, fabsf(f.l2)) < INFINITY;
    if (fast) {
      const f32x2 mm = pair(-f.m, -f.m), cc = pair(f.c, f.c), ll = pair(-f.l2, -f.l2), aa = pair(A, A), bb = pair(B, B);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (j0 + u * 32 >= r.vecs) break;
        const int j = r.head + (j0 + u * 32) * N;
        f32x2 x[P];
        const uint4 one[1] = {v[u]};
        spread<1>(one, x, kFloor, static_cast<const T*>(nullptr));
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const f32x2 y = fma2(add2(x[i], mm), cc, ll);
          float y0, y1;
          unpair(y, y0, y1);
          x[i] = mul2(pair(ex2(y0), ex2(y1)), fma2(y, bb, aa));
        }
        if (uint32_t(f.t - j) < uint32_t(N)) {           // (a token outside the support has no share)
          float z[N];
          unpack(v[u], z);
          bool kept = false;
#pragma unroll
          for (int i = 0; i < N; ++i) kept |= f.t - j == i && z[i] > kNegInf;
#pragma unroll
          for (int i = 0; i < P; ++i) {
            float lo, hi;
            unpair(x[i], lo, hi);
            x[i] = pair(f.t - j == 2 * i && kept ? lo + f.dl : lo, f.t - j == 2 * i + 1 && kept ? hi + f.dl : hi);
          }
        }
        const uint4 w = round_pairs<T>(x);
        if (whole) {
          *reinterpret_cast<uint4*>(out + j) = w;
        } else {
          const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
          for (int i = 0; i < N; ++i) out[j + i] = e[i];
        }
      }
    } else {
#pragma unroll 1
      for (int u = 0; u < U; ++u) {
        if (j0 + u * 32 >= r.vecs) break;
        const int j = r.head + (j0 + u * 32) * N;
        float x[N];
        unpack(r.template vec<MASK>(j0 + u * 32), x);
#pragma unroll
        for (int i = 0; i < N; ++i) out[j + i] = T(f(x[i], j + i));
      }
    }
    if (seg == 0 && lane < 16) {
      const int j = r.edge(lane);
      if (j >= 0) {
        const float x = r.at(j);
        float d = f(x, j);
        if (fast) {                      // the same roundings as in a whole vector
          const float y = fmaf(max_nan(x, kFloor) - f.m, f.c, -f.l2);
          d = ex2(y) * fmaf(y, B, A);
          if (j == f.t && x > kNegInf) d += f.dl;
        }
        out[j] = T(d);
      }
    }
  }
}

template <typename K, typename... A>
void launch_cluster(K kernel, unsigned grid, unsigned threads, unsigned cluster, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = threads;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  cudaLaunchKernelEx(&cfg, kernel, args...);
}

#ifndef LP_THREADS
#define LP_THREADS 512
#endif
constexpr int kThreads = LP_THREADS;
template <typename T, bool MASK, int THREADS>
void launch_cta(const RowArgs& a, const RowOut& o, int parts, cudaStream_t st) {
  const unsigned grid = unsigned(a.rows * parts);
  if (o.top) launch_cluster(k_logprob_cta<T, THREADS, MASK, true>, grid, THREADS, parts, st, a, o, parts);
  else launch_cluster(k_logprob_cta<T, THREADS, MASK, false>, grid, THREADS, parts, st, a, o, parts);
}
template <typename T, bool MASK>
void launch_rows(const RowArgs& a, const RowOut& o, cudaStream_t st) {
  if (a.vocab <= 1024) {
    const int64_t ctas = (a.rows + 3) / 4;
    const unsigned grid = unsigned(ctas < (int64_t(1) << 30) ? ctas : int64_t(1) << 30);
    if (a.vocab <= 128) launch(k_logprob_warp<T, 4, MASK>, grid, 128, 0, st, a, o);
    else if (a.vocab <= 256) launch(k_logprob_warp<T, 8, MASK>, grid, 128, 0, st, a, o);
    else if (a.vocab <= 512) launch(k_logprob_warp<T, 16, MASK>, grid, 128, 0, st, a, o);
    else launch(k_logprob_warp<T, 32, MASK>, grid, 128, 0, st, a, o);
    return;
  }
  int parts = 1;
  while (parts < 8 && a.rows * parts * 2 <= 2 * kNumSMs && a.vocab / (parts * 2) >= 4096) parts *= 2;
  launch_cta<T, MASK, kThreads>(a, o, parts, st);
}
template <typename T, bool MASK>
void launch_grad(const RowArgs& a, const GradArgs& g, cudaStream_t st) {
  const int segs = a.vocab / Vec<T>::N / (32 * 4) + 1;
  const int64_t ctas = (a.rows * segs + 7) / 8;
  const unsigned grid = unsigned(ctas < (int64_t(1) << 30) ? ctas : int64_t(1) << 30);
  launch(k_logprob_grad<T, MASK>, grid, 256, 0, st, a, g, segs);
}

}  // namespace

int launch_logprob(int dtype, int64_t rows, int32_t vocab, const void* logits, int64_t row_stride, const int32_t* token,
                   const uint8_t* mask, int64_t mask_stride, float scale, int32_t num_top, float* logp, float* entropy,
                   float* norm, int32_t* top_token, float* top_logp, cudaStream_t st) {
  if (rows <= 0) return 0;
  const RowArgs a = {logits, row_stride, token, mask, mask_stride, rows, vocab, scale};
  const RowOut o = {logp, entropy, norm, top_token, top_logp, num_top};
  if (dtype == XRL_BF16) mask ? launch_rows<bf16, true>(a, o, st) : launch_rows<bf16, false>(a, o, st);
  else mask ? launch_rows<float, true>(a, o, st) : launch_rows<float, false>(a, o, st);
  return 1;
}

int launch_logprob_grad(int dtype, int64_t rows, int32_t vocab, const void* logits, int64_t row_stride, const int32_t* token,
                        const uint8_t* mask, int64_t mask_stride, float scale, const float* norm, const float* dlogp,
                        const float* entropy, const float* dentropy, void* grad, int64_t grad_stride, cudaStream_t st) {
  if (rows <= 0) return 0;
  const RowArgs a = {logits, row_stride, token, mask, mask_stride, rows, vocab, scale};
  const GradArgs g = {norm, dlogp, entropy, dentropy, grad, grad_stride};
  if (dtype == XRL_BF16) mask ? launch_grad<bf16, true>(a, g, st) : launch_grad<bf16, false>(a, g, st);
  else mask ? launch_grad<float, true>(a, g, st) : launch_grad<float, false>(a, g, st);
  return 1;
}

}  // namespace xrl
