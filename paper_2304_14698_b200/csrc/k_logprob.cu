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
__device__ __forceinline__ uint32_t key_of(float v) {          // unsigned order = order of the floats
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float float_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
__device__ __forceinline__ float max_warp(float v) { return float_of(__reduce_max_sync(kAll, key_of(v))); }      // no NaN
__device__ __forceinline__ Sums join_warp(const Sums& v) {
  Sums o;
  o.m = max_warp(v.m);
  o.r = max_warp(v.r);
  const float d = v.r - o.r, e = ex2(d);
  o.s = v.s * e;
  o.t = fmaf(d, v.s, v.t) * e;
#pragma unroll
  for (int d2 = 16; d2 > 0; d2 >>= 1) {
    o.s += __shfl_xor_sync(kAll, o.s, d2);
    o.t += __shfl_xor_sync(kAll, o.t, d2);
  }
  return o;
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
// The row's token and its logit, asked for before the row is walked
struct Given {
  int32_t t = -1;
  float x = kNegInf;
};
template <typename T> __device__ __forceinline__ Given given_of(const RowArgs& a, int64_t row) {
  Given g;
  if (a.token) {
    g.t = __ldg(a.token + row);
    if (g.t >= 0 && g.t < a.vocab) {
      g.x = load1(static_cast<const T*>(a.x) + row * a.x_stride + g.t);
      if (a.mask && !__ldg(a.mask + row * a.mask_stride + g.t)) g.x = kNegInf;
    }
  }
  return g;
}
__device__ __forceinline__ void write_row(const RowArgs& a, const RowOut& o, int64_t row, const Given& g, const RowNorm& n,
                                          float entropy) {
  if (o.norm) *reinterpret_cast<float2*>(o.norm + 2 * row) = make_float2(n.m, n.l);
  if (o.entropy) o.entropy[row] = entropy;
  if (o.logp) o.logp[row] = g.t == -1 ? 0.f : g.t < -1 || g.t >= a.vocab ? NAN : logp_of(g.x, n, a.scale);
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
    Given given;
    if (lane == 0) given = given_of<T>(a, row);
    float v[E];
    uint8_t left[MASK ? E : 1];
    const uint8_t* mask = MASK ? a.mask + row * a.mask_stride : nullptr;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = e * 32 + lane;
      v[e] = j < a.vocab ? load1(x + j) : kNegInf;
      if (MASK) left[e] = j < a.vocab ? __ldg(mask + j) : uint8_t(0);
    }
    if (MASK) {                          // (after all loads)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = left[e] ? v[e] : kNegInf;
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
    if (lane == 0) write_row(a, o, row, given, n, empty ? 0.f : entropy_of(q));
    if (o.top) {                         // the best of the lanes' best is taken out, `top` times; of equals the lowest index
      Best mine;
      for (int k = 0; k < o.top; ++k) {
        float best = kNegInf;
        int at = 0;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (v[e] > best) { best = v[e]; at = e; }
        const uint32_t key = key_of(best), most = __reduce_max_sync(kAll, key);
        if (most == key_of(kNegInf)) break;
        const unsigned i = __reduce_min_sync(kAll, key == most ? unsigned(at * 32 + lane) : kAll);
        const float taken = __shfl_sync(kAll, best, i & 31);
        if (lane == k) { mine.v = taken; mine.i = int32_t(i); }
        if (lane == int(i & 31))
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (e == at) v[e] = kNegInf;
      }
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
// ---- a thread's own copies ahead: what it will read, on its way to its own places in shared memory ------------------
// cp.async needs neither registers nor, as no thread reads another's places, barriers.
template <int BYTES> __device__ __forceinline__ void copy_ahead(uint32_t dst, const void* src) {
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// DEPTH groups of U vectors per thread, each with the words of its mask
template <typename T, int THREADS, int U> struct Ahead {
  static constexpr int DEPTH = 3, N = Vec<T>::N, WORDS = N / 4 + 1;
  static constexpr int VEC_BYTES = THREADS * 16, WORD_BYTES = THREADS * 4;
  static constexpr int GROUP_BYTES = U * (VEC_BYTES + WORDS * WORD_BYTES);
  static constexpr int BYTES = DEPTH * GROUP_BYTES;
  uint32_t base;                         // of the thread
  __device__ __forceinline__ explicit Ahead(const void* smem)
      : base(static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + threadIdx.x * 16) {}
  __device__ __forceinline__ uint32_t vec_at(int group, int u) const { return base + group * GROUP_BYTES + u * VEC_BYTES; }
  __device__ __forceinline__ uint32_t word_at(int group, int u, int w) const {
    return base - threadIdx.x * 12 + group * GROUP_BYTES + U * VEC_BYTES + (u * WORDS + w) * WORD_BYTES;
  }
  __device__ __forceinline__ void ask(int group, int u, const T* x, const uint8_t* mask) const {
    copy_ahead<16>(vec_at(group, u), x);
    const uintptr_t at = reinterpret_cast<uintptr_t>(mask);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(at & ~uintptr_t(3));
#pragma unroll
    for (int i = 0; i < WORDS; ++i)
      if (i + 1 < WORDS || (at & 3)) copy_ahead<4>(word_at(group, u, i), w + i);
  }
  __device__ __forceinline__ uint4 take(int group, int u, const uint8_t* mask) const {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(vec_at(group, u)) : "memory");
    const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(mask) & 3) * 8;
    uint32_t w[3] = {0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < WORDS; ++i)
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i]) : "r"(word_at(group, u, i)) : "memory");
    // (the last word is whatever lay there where nothing was asked for; no bit of it is used then)
    Vec<T>::drop(v, __funnelshift_r(w[0], w[1], off), N == 8 ? __funnelshift_r(w[1], w[2], off) : 0u);
    return v;
  }
};
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
// A row whose logits are too far from 0 for the above: largest first, then the sums of differences.  One entry per thread and
// load, and of a cluster one CTA for the whole row (8,192 x 32,000 bf16 487 us in place of 83, 16 x 128,000 61 in place of 6): such rows
// are rare, and the kernel that all others run keeps its registers.
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
__device__ __forceinline__ uint64_t remote_u64(uint32_t at) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
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
// adds them to a thread's sums; the largest of them
template <typename T, int U>
__device__ __forceinline__ float add_chunk(Sums& q, const uint4 (&v)[U], float c, float floor) {
  constexpr int P = U * Vec<T>::N / 2;
  f32x2 f[P];
  const float here = spread<U>(v, f, floor, static_cast<const T*>(nullptr)), m = fmaxf(q.m, here);
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
  return here;
}

// ---- the best k of a CTA's part of a row -----------------------------------------------------------------------
// An entry as one whole number: by value first, the lower index then; 0 is none
__device__ __forceinline__ uint64_t rank_key(float v, int32_t i) { return uint64_t(key_of(v)) << 32 | uint32_t(~i); }
__device__ __forceinline__ Best best_of(uint64_t key) {
  Best b;
  if (key) { b.v = float_of(uint32_t(key >> 32)); b.i = int32_t(~uint32_t(key)); }
  return b;
}
constexpr int kSlots = 8;                // stretches of a thread's vectors
// Candidates in shared memory: the k best of n <= THREADS, by counting for each how many are better
template <int THREADS> struct Candidates {
  uint64_t key[THREADS], best[kMostTop];
  float largest[kSlots][THREADS];        // of each stretch of each thread's vectors
  uint8_t again[kSlots * THREADS];       // of each warp: lane and stretch (times 32) of what is walked again
  int n;
};
template <int THREADS> __device__ __forceinline__ void rank_candidates(Candidates<THREADS>& s, int n, int k) {
  if (threadIdx.x < kMostTop) s.best[threadIdx.x] = 0;
  if (int(threadIdx.x) >= n) s.key[threadIdx.x] = 0;
  __syncthreads();
  if (int(threadIdx.x) < n) {
    const uint64_t mine = s.key[threadIdx.x];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; j += 2) {
      const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(&s.key[j]);
      rank += (two.x > mine ? 1 : 0) + (two.y > mine ? 1 : 0);
    }
    if (rank < k && mine) s.best[rank] = mine;
  }
  __syncthreads();
}

// A thread's largest logit (thread_max) is known, and that of each of up to eight stretches of its vectors, `stretch` vectors
// long.  At least k threads hold one of `bound` or more, so the k best are no less; few other logits are, and only the
// stretches whose largest is that high have any.  Their vectors are read again, spread over the lanes of their warp, and what
// reaches the bound is ranked.  Where that is more than one entry per thread of the CTA (equal logits everywhere, or fewer than
// k threads with any) each warp keeps a sorted list of its whole part instead.
template <typename T, int THREADS, bool MASK>
__device__ __forceinline__ void best_of_part(const Row<T>& r, int v0, int v1, bool edges, float thread_max, float part_max, int stretches, int stretch, int k,
                                             Candidates<THREADS>& s, uint32_t* red) {
  constexpr int N = Vec<T>::N, U = 4, GROUP = THREADS / 32;
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
  uint8_t* again = s.again + warp * 32 * kSlots;
  int items = 0;
  if (__any_sync(kAll, thread_max > kNegInf && mine >= lo)) {
    for (int i = 0; i < stretches; ++i) {
      const float most = s.largest[i][threadIdx.x];
      const bool some = most > kNegInf && most >= bound;
      const unsigned flags = __ballot_sync(kAll, some);
      if (some) again[items + __popc(flags & ((1u << lane) - 1))] = uint8_t(i * 32 + lane);
      items += __popc(flags);
    }
    items *= stretch;
    __syncwarp();
  }
  auto put = [&](float v, int32_t i) {
    if (v >= bound && v > kNegInf) {
      const int at = atomicAdd(&s.n, 1);
      if (at < THREADS) s.key[at] = rank_key(v, i);
    }
  };
  for (int i = lane; i < items; i += 32) {
    const int which = i / stretch, at = again[which];
    const int j = v0 + warp * 32 + (at & 31) + ((at >> 5) * stretch + i - which * stretch) * THREADS;
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
    s.key[threadIdx.x] = mine_b.v > kNegInf ? rank_key(mine_b.v, mine_b.i) : 0;
    __syncthreads();
    n = THREADS;
  }
  rank_candidates<THREADS>(s, n, k);
}

// A CTA takes a row (parts > 1: a cluster does, each CTA a part of it).  What hides the loads is other CTAs' arithmetic:
// copies into shared memory ahead of it, by CTAs that stay for many rows, came to 115 us where this takes 92 (8,192 x 32,000 bf16).
template <typename T, int THREADS, int U, int CTAS, bool MASK, bool TOP>
__global__ void __launch_bounds__(THREADS, CTAS) k_logprob_cta(RowArgs a, RowOut o, int log_parts) {
  enter();
  constexpr int W = THREADS / 32, GROUP = U * THREADS;
  __shared__ Sums s_sums[W];
  __shared__ float s_red[64];
  __shared__ __align__(16) Candidates<TOP ? THREADS : 32> s_best;
  __shared__ Sums s_part;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int parts = 1 << log_parts, part = parts > 1 ? int(cluster_rank()) : 0;
  // part p of a row's vectors starts here (below 2^29 vectors and 8 parts: 32 bits)
  auto start_of = [&](int vecs, int p) { return int((uint32_t(vecs) * uint32_t(p)) >> log_parts); };
  const float c = a.scale * kLog2e;
  // (as a bf16 number, which it is for both types; rounded, it is within 2^-9 of itself)
  const float floor = to_float(bf16(kLowest / c));
  const Sums zero = {kNegInf, floor * c, 0.f, 0.f};

  const int64_t row = blockIdx.x >> log_parts;
  const Row<T> r(a, row, MASK);
  Given given;
  if (threadIdx.x == 0 && part == 0) given = given_of<T>(a, row);
  const int v0 = start_of(r.vecs, part), v1 = start_of(r.vecs, part + 1);
  Sums q = zero;
  int j = v0 + threadIdx.x;              // the thread's next vector
  // the largest of a stretch of `rounds` of the loop
  const int rounds = TOP ? max((v1 - v0 + kSlots * GROUP - 1) / (kSlots * GROUP), 1) : 1;
  float most = kNegInf;
  int round = 0, slot = 0;
  for (int left = v1 - v0; left > 0; left -= GROUP, j += GROUP) {
    float here = kNegInf;
    if (left >= GROUP) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = r.template vec<MASK>(j + u * THREADS);
      here = add_chunk<T, U>(q, v, c, floor);
    } else if (2 * left > GROUP) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = j + u * THREADS < v1 ? r.template vec<MASK>(j + u * THREADS) : Vec<T>::none();
      here = add_chunk<T, U>(q, v, c, floor);
    } else {
#pragma unroll 1
      for (int u = 0; u < U; ++u) {
        if (j + u * THREADS - lane >= v1) break;         // no vector for the whole warp
        const uint4 v[1] = {j + u * THREADS < v1 ? r.template vec<MASK>(j + u * THREADS) : Vec<T>::none()};
        here = fmaxf(here, add_chunk<T, 1>(q, v, c, floor));
      }
    }
    if (TOP) {
      most = fmaxf(most, here);
      if (++round == rounds) {
        s_best.largest[slot++][threadIdx.x] = most;
        most = kNegInf;
        round = 0;
      }
    }
  }
  if (TOP && round) s_best.largest[slot++][threadIdx.x] = most;
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
  float largest = max_warp(q.m);
  if (TOP) best_of_part<T, TOP ? THREADS : 32, MASK>(r, v0, v1, part == 0, thread_max, largest, slot,
                                                         min(rounds * U, (v1 - v0 + THREADS - 1) / THREADS), o.top, s_best, reinterpret_cast<uint32_t*>(s_red));
  if (parts > 1 || warp == 0) q = join_warp(q);
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
      largest = max_warp(q.m);
      q = join_warp(q);
      if (TOP) {
        const int p = threadIdx.x / o.top, e = threadIdx.x - p * o.top;
        s_best.key[threadIdx.x] = p < parts ? remote_u64(remote(&s_best.best[e], p)) : 0;
      }
    }
    cluster_arrive_wait();               // nobody leaves, and nothing is written again, while it is read
    if (part != 0) return;
    if (TOP) rank_candidates(s_best, parts * o.top, o.top);
  }
  if (largest > kNegInf && largest < INFINITY && !(largest * c > kLow && largest * c < kHigh)) {       // (all threads agree)
    careful_row<T, THREADS>(a, MASK, row, s_red, q);
    if (warp == 0) {
      const RowNorm n = {q.m, kLn2 * log2f(q.s)};
      if (lane == 0) write_row(a, o, row, given, n, entropy_of(q));
      if (TOP) write_top(a, o, row, n, best_of(s_best.best[lane]), lane);
    }
  } else if (warp == 0) {
    RowNorm n = {kNegInf, kNegInf};
    float entropy = 0.f;
    if (largest > kNegInf || q.s != q.s) {
      n = norm_of(q, c);
      if (q.s != q.s) n.l = NAN;
      entropy = entropy_of(q);
    }
    if (lane == 0) write_row(a, o, row, given, n, entropy);
    if (TOP) write_top(a, o, row, n, best_of(s_best.best[lane]), lane);
  }
}

// ---- gradient ---------------------------------------------------------------------------------------------------
struct GradArgs {
  const float *norm, *dlogp, *entropy, *dentropy;
  void* grad;
  int64_t grad_stride;
};
// What a row's entries share, as it lies in memory and as it is used.  With p = 2^y, y = (x - m) c - l2, an entry is
// p (A + B y), plus dl at the token: A = -(dl + dh H), B = -dh ln 2.  -infinity becomes kFloor first, for which p is 0; rows
// where that does not do (a norm or gradients that are not finite, logits all below the floor) go entry by entry.
struct RowInputs {
  float2 norm = {0.f, 0.f};
  int32_t t = -1;
  float dlogp = 0.f, dentropy = 0.f, entropy = 0.f;
};
__device__ __forceinline__ RowInputs inputs_of(const RowArgs& a, const GradArgs& g, int64_t row) {
  RowInputs r;
  r.norm = __ldg(reinterpret_cast<const float2*>(g.norm) + row);
  if (a.token) r.t = __ldg(a.token + row);
  if (g.dlogp) r.dlogp = __ldg(g.dlogp + row);
  if (g.dentropy) { r.dentropy = __ldg(g.dentropy + row); r.entropy = __ldg(g.entropy + row); }
  return r;
}
struct RowGrad {
  float m, c, l2, dl, dh, ent, A, B;     // l2: l in powers of two; dl, dh times the scale
  int32_t t;
  bool fast;
  __device__ __forceinline__ RowGrad(const RowArgs& a, const RowInputs& r) {
    t = r.t;
    m = r.norm.x;
    c = a.scale * kLog2e;
    l2 = r.norm.y * kLog2e;
    dl = t == -1 ? 0.f : t < -1 || t >= a.vocab ? NAN : a.scale * r.dlogp;
    dh = a.scale * r.dentropy;
    ent = r.entropy;
    A = -fmaf(dh, ent, dl);
    B = -dh * kLn2;
    // (every product of the fast form is finite then)
    fast = m > kFloor && fabsf(A) + fabsf(B) * fmaf(fabsf(m) - kFloor, c, fabsf(l2)) < INFINITY;
  }
  // one entry; of a fast row with the roundings of a whole vector
  __device__ __forceinline__ float operator()(float x, int j) const {
    if (fast) {
      const float y = fmaf(max_nan(x, kFloor) - m, c, -l2), d = ex2(y) * fmaf(y, B, A);
      return j == t && x > kNegInf ? d + dl : d;
    }
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
// the gradient of a vector's entries j ... j + N - 1
template <typename T>
__device__ __forceinline__ void grad_vector(const RowGrad& f, const uint4& v, int j, T* out, bool whole) {
  constexpr int N = Vec<T>::N, P = N / 2;
  uint4 w;
  if (f.fast) {
    const f32x2 mm = pair(-f.m, -f.m), cc = pair(f.c, f.c), ll = pair(-f.l2, -f.l2), aa = pair(f.A, f.A), bb = pair(f.B, f.B);
    f32x2 x[P];
    const uint4 one[1] = {v};
    spread<1>(one, x, kFloor, static_cast<const T*>(nullptr));
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const f32x2 y = fma2(add2(x[i], mm), cc, ll);
      float y0, y1;
      unpair(y, y0, y1);
      x[i] = mul2(pair(ex2(y0), ex2(y1)), fma2(y, bb, aa));
    }
    if (uint32_t(f.t - j) < uint32_t(N)) {               // (a token outside the support has no share)
      float z[N];
      unpack(v, z);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float lo, hi;
        unpair(x[i], lo, hi);
        x[i] = pair(f.t - j == 2 * i && z[2 * i] > kNegInf ? lo + f.dl : lo,
                    f.t - j == 2 * i + 1 && z[2 * i + 1] > kNegInf ? hi + f.dl : hi);
      }
    }
    w = round_pairs<T>(x);
  } else {
    float z[N];
    unpack(v, z);
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = f(z[i], j + i);
    w = pack(z);
  }
  if (whole) {
    *reinterpret_cast<uint4*>(out + j) = w;
  } else {
    const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
    for (int i = 0; i < N; ++i) out[j + i] = e[i];
  }
}
template <typename T>
__device__ __forceinline__ void grad_edges(const RowGrad& f, const Row<T>& r, T* out, int i) {
  const int j = i < 16 ? r.edge(i) : -1;
  if (j >= 0) out[j] = T(f(r.at(j), j));
}
template <typename T> __device__ __forceinline__ bool aligned16(const T* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Short rows: a warp takes 32 x U vectors of a row at a time.
template <typename T, bool MASK>
__global__ void __launch_bounds__(256) k_logprob_grad(RowArgs a, GradArgs g, int segs) {
  enter();
  constexpr int N = Vec<T>::N, U = 4;
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
    const RowGrad f(a, inputs_of(a, g, row));
    const bool whole = aligned16(out + r.head);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * 32 < r.vecs) grad_vector(f, v[u], r.head + (j0 + u * 32) * N, out, whole);
    if (seg == 0) grad_edges(f, r, out, lane);
  }
}

// Long rows: a CTA takes THREADS x U vectors of one.
template <typename T, int THREADS, int U, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) k_logprob_grad_cta(RowArgs a, GradArgs g, int pieces) {
  enter();
  constexpr int N = Vec<T>::N;
  const int64_t row = int64_t(blockIdx.x / uint32_t(pieces));
  const int v0 = int(blockIdx.x - uint32_t(row) * uint32_t(pieces)) * U * THREADS, j0 = v0 + int(threadIdx.x);
  const Row<T> r(a, row, false);
  const RowInputs in = inputs_of(a, g, row);
  uint4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) v[u] = j0 + u * THREADS < r.vecs ? r.template vec<false>(j0 + u * THREADS) : Vec<T>::none();
  T* out = static_cast<T*>(g.grad) + row * g.grad_stride;
  const RowGrad f(a, in);
  const bool whole = aligned16(out + r.head);
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (j0 + u * THREADS < r.vecs) grad_vector(f, v[u], r.head + (j0 + u * THREADS) * N, out, whole);
  if (v0 == 0) grad_edges(f, r, out, threadIdx.x);
}

// Long masked rows: resident CTAs take pieces of rows in turn, each `piece` vectors, copied ahead across pieces with their
// mask bytes; what a row shares is asked for a piece ahead too.
template <typename T, int THREADS, int U>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_logprob_grad_rows(RowArgs a, GradArgs g, int pieces, int piece) {
  using A = Ahead<T, THREADS, U>;
  enter();
  constexpr int N = Vec<T>::N, GROUP = U * THREADS;
  extern __shared__ __align__(16) uint8_t s_ahead[];
  const A ahead(s_ahead);
  const int64_t units = a.rows * pieces;
  auto split = [&](int64_t unit, int64_t& row, int& at) {
    row = units <= INT32_MAX ? int64_t(uint32_t(unit) / uint32_t(pieces)) : unit / pieces;
    at = int(unit - row * pieces) * piece;
  };
  int64_t p_unit = blockIdx.x;
  int p_group = 0, p_left = 0;
  const T* p_x = nullptr;
  const uint8_t* p_mask = nullptr;
  auto p_start = [&]() {
    p_left = 0;
    if (p_unit >= units) return;
    int64_t row;
    int v0;
    split(p_unit, row, v0);
    const Row<T> r(a, row, true);
    p_left = min(r.vecs - v0, piece);
    const int64_t at = r.head + (int64_t(v0) + threadIdx.x) * N;
    p_x = r.x + at;
    p_mask = r.mask + at;
  };
  auto ask = [&]() {
    if (p_left >= GROUP) {
#pragma unroll
      for (int u = 0; u < U; ++u) ahead.ask(p_group, u, p_x + u * THREADS * N, p_mask + u * THREADS * N);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u * THREADS + int(threadIdx.x) < p_left) ahead.ask(p_group, u, p_x + u * THREADS * N, p_mask + u * THREADS * N);
    }
    copies_end_group();
    p_group = p_group + 1 < A::DEPTH ? p_group + 1 : 0;
    p_x += GROUP * N;
    p_mask += GROUP * N;
    p_left -= GROUP;
    if (p_left <= 0) {
      p_unit += gridDim.x;
      p_start();
    }
  };
  p_start();
#pragma unroll
  for (int d = 0; d < A::DEPTH - 1; ++d) ask();
  int group = 0;
  RowInputs next;
  int64_t row = 0;
  int v0 = 0;
  if (int64_t(blockIdx.x) < units) {
    split(blockIdx.x, row, v0);
    next = inputs_of(a, g, row);
  }
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const RowGrad f(a, next);
    split(unit, row, v0);
    const Row<T> r(a, row, true);
    T* out = static_cast<T*>(g.grad) + row * g.grad_stride;
    const bool whole = aligned16(out + r.head);
    if (unit + gridDim.x < units) {
      int64_t then;
      int at;
      split(unit + gridDim.x, then, at);
      next = inputs_of(a, g, then);
    }
    if (v0 == 0) grad_edges(f, r, out, threadIdx.x);
    int left = min(r.vecs - v0, piece), j = r.head + (v0 + int(threadIdx.x)) * N;
    const uint8_t* mask = r.mask + j;
    do {
      ask();
      copies_wait<A::DEPTH - 1>();
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u * THREADS + int(threadIdx.x) < left)
          grad_vector(f, ahead.take(group, u, mask + u * THREADS * N), j + u * THREADS * N, out, whole);
      group = group + 1 < A::DEPTH ? group + 1 : 0;
      j += GROUP * N;
      mask += GROUP * N;
      left -= GROUP;
    } while (left > 0);
  }
  copies_wait<0>();
}

template <typename K, typename... A>
void launch_cluster(K kernel, unsigned grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.dynamicSmemBytes = smem;
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

template <typename T, int THREADS, int U, int CTAS, bool MASK, bool TOP>
void launch_cta(const RowArgs& a, const RowOut& o, int log_parts, cudaStream_t st) {
  launch_cluster(k_logprob_cta<T, THREADS, U, CTAS, MASK, TOP>, unsigned(a.rows << log_parts), THREADS, 0, 1 << log_parts, st, a, o,
                 log_parts);
}
// Threads, vectors a thread has in flight, CTAs an SM holds; rows of so many 16-byte vectors.  Measured in us, 200 MB of logits where
// no rows are given (bf16 / fp32):
// - without alternatives: 64 by four 61 / 53 at 300 vectors, 48 / 43 at 600, 47 / 42 at 4,000; 64 by eight 72 / 59, 51 / 47 and 42 / 37,
//   at 1,500 38 / 34; 128 by eight 38 / 35 at 4,000, 37 / 34 at 3,000, at 1,500 51 / 48.  With masks 64 by four 67 / 54 at 600,
//   60 / 48 at 1,500, 73 / 60 at 4,000; 128 by four 72 / 62, 61 / 53 and 63 / 53; 128 by eight 66 / 57 at 4,000, at 6,500 60 / 45
//   where 128 by four takes 64 / 53.
// - with 20 alternatives, whose search is a CTA's: 64 by four 89 / 79 at 600, 57 / 52 at 1,500, 59 / 55 at 2,200; 128 by four 105 / 94,
//   61 / 54 and 56 / 53; 256 by four 188 / 168, 101 / 89 and 78 / 69.  20 are the most that 64 threads take: with 32 more logits reach
//   their bound than there are threads (600: 330 / 215, 128 by four 123 / 108).
// - 256 threads for long rows: with masks and 5 alternatives at 9,000 vectors 99 / 80 for 2,200 rows, 133 / 111 for 3,000, 128 by four
//   101 / 86 and 132 / 118; at 12,500 94 / 74 for 1,500 rows and 171 / 138 for 3,000, 128 by four 105 / 98 and 177 / 160.  Without masks
//   they lose up to 12,000 vectors (6,500: fp32 1,000 rows 24 -> 28, 3,000 64 -> 73; 9,000: bf16 5,000 rows 131 -> 147) but
//   where rows are few (fp32 400 rows of 9,000 24 -> 17, of 6,500 18 -> 15); behind that they lose 2 to 9 % with 5 alternatives and win as
//   much with 20 (fp32 12,500, 2,200 rows: 82 -> 84, 94 -> 89).
// - masked searches in bf16 keep their registers by nine CTAs of 128 in place of ten: 5 alternatives at 3,000 74 -> 71, at 4,000
//   78 -> 71, at 6,500 77 -> 68; below 1,000 vectors the tenth is worth more (32 alternatives at 160 475 -> 413, at 600 172 -> 160).
template <typename T, bool MASK, bool TOP>
void launch_long(const RowArgs& a, const RowOut& o, cudaStream_t st) {
  const int vecs = a.vocab / Vec<T>::N;
  int log_parts = 0;                     // few rows: clusters, no CTA with less than 4,096 entries
  while (log_parts < 3 && a.rows << (log_parts + 1) <= 2 * kNumSMs && a.vocab >> (log_parts + 1) >= 4096) ++log_parts;
  if (log_parts == 3) return launch_cta<T, 256, 4, 4, MASK, TOP>(a, o, 3, st);
  if (a.rows << log_parts <= 2 * kNumSMs) return launch_cta<T, 512, 4, 2, MASK, TOP>(a, o, log_parts, st);
  if constexpr (TOP) {
    if (vecs < 2048 && o.top <= 20) return launch_cta<T, 64, 4, 20, MASK, TOP>(a, o, 0, st);
    if (vecs >= 6000 && (MASK || vecs >= 12000 || a.rows <= 4 * kNumSMs)) return launch_cta<T, 256, 4, 4, MASK, TOP>(a, o, 0, st);
    if constexpr (MASK && Vec<T>::N == 8) {
      if (vecs >= 1000) return launch_cta<T, 128, 4, 9, MASK, TOP>(a, o, 0, st);
    }
    launch_cta<T, 128, 4, 10, MASK, TOP>(a, o, 0, st);
  } else {
    if (vecs < (MASK ? 2000 : 512)) return launch_cta<T, 64, 4, 20, MASK, TOP>(a, o, 0, st);
    if (vecs >= (MASK ? 6000 : 3000)) return launch_cta<T, 128, 8, 7, MASK, TOP>(a, o, 0, st);
    if constexpr (MASK) launch_cta<T, 128, 4, 10, MASK, TOP>(a, o, 0, st);
    else launch_cta<T, 64, 8, 14, MASK, TOP>(a, o, 0, st);
  }
}
template <typename T, bool MASK>
bool launch_rows(const RowArgs& a, const RowOut& o, cudaStream_t st) {
  if (a.vocab > 1024) {
    o.top ? launch_long<T, MASK, true>(a, o, st) : launch_long<T, MASK, false>(a, o, st);
    return true;
  }
  // What a warp takes out of registers one by one soon costs more than a CTA's search (us, 16 and 16,384 rows of 1,000 fp32, 5
  // alternatives 4.1 and 29, by CTAs 4.1 and 35; 20: 8.6 and 81, 5.8 and 45)
  if (o.top > 8 && a.vocab > 512) {
    if (o.top <= 20) launch_cta<T, 64, 4, 20, MASK, true>(a, o, 0, st);
    else launch_cta<T, 128, 4, 10, MASK, true>(a, o, 0, st);
    return true;
  }
  const int64_t ctas = (a.rows + 3) / 4;
  const unsigned grid = unsigned(ctas < (int64_t(1) << 30) ? ctas : int64_t(1) << 30);
  if (a.vocab <= 128) launch(k_logprob_warp<T, 4, MASK>, grid, 128, 0, st, a, o);
  else if (a.vocab <= 256) launch(k_logprob_warp<T, 8, MASK>, grid, 128, 0, st, a, o);
  else if (a.vocab <= 512) launch(k_logprob_warp<T, 16, MASK>, grid, 128, 0, st, a, o);
  else launch(k_logprob_warp<T, 32, MASK>, grid, 128, 0, st, a, o);
  return true;
}
// In us, 8,192 x 32,000 bf16: a CTA per piece 157 without a mask, 256 with one; resident CTAs with copies ahead 200 and 232.
template <typename T, bool MASK>
bool launch_grad(const RowArgs& a, const GradArgs& g, cudaStream_t st) {
  const int vecs = a.vocab / Vec<T>::N;
  if (vecs >= 512) {                     // (shorter rows leave much of a CTA idle)
    if constexpr (MASK) {
      constexpr int THREADS = 256, U = 2, SMEM = Ahead<T, THREADS, U>::BYTES;
      static bool done[64] = {};
      if (!ensure_dynamic_smem(k_logprob_grad_rows<T, THREADS, U>, SMEM, done)) return false;
      const int piece = 2 * U * THREADS, pieces = (vecs + piece - 1) / piece;
      const int64_t units = a.rows * pieces, most = int64_t(kNumSMs) * (1024 / THREADS);
      launch(k_logprob_grad_rows<T, THREADS, U>, unsigned(units < most ? units : most), THREADS, SMEM, st, a, g, pieces, piece);
      return true;
    } else {
      constexpr int THREADS = 128, U = 4;
      const int pieces = (vecs + THREADS * U - 1) / (THREADS * U);
      if (a.rows * pieces <= INT32_MAX) {
        launch(k_logprob_grad_cta<T, THREADS, U, 10>, unsigned(a.rows * pieces), THREADS, 0, st, a, g, pieces);
        return true;
      }
    }
  }
  const int segs = vecs / (32 * 4) + 1;
  const int64_t ctas = (a.rows * segs + 7) / 8;
  const unsigned grid = unsigned(ctas < (int64_t(1) << 30) ? ctas : int64_t(1) << 30);
  launch(k_logprob_grad<T, MASK>, grid, 256, 0, st, a, g, segs);
  return true;
}

}  // namespace

bool launch_logprob(int dtype, int64_t rows, int32_t vocab, const void* logits, int64_t row_stride, const int32_t* token,
                   const uint8_t* mask, int64_t mask_stride, float scale, int32_t num_top, float* logp, float* entropy,
                   float* norm, int32_t* top_token, float* top_logp, cudaStream_t st) {
  if (rows <= 0) return true;
  const RowArgs a = {logits, row_stride, token, mask, mask_stride, rows, vocab, scale};
  const RowOut o = {logp, entropy, norm, top_token, top_logp, num_top};
  if (dtype == XRL_BF16) return mask ? launch_rows<bf16, true>(a, o, st) : launch_rows<bf16, false>(a, o, st);
  return mask ? launch_rows<float, true>(a, o, st) : launch_rows<float, false>(a, o, st);
}

bool launch_logprob_grad(int dtype, int64_t rows, int32_t vocab, const void* logits, int64_t row_stride, const int32_t* token,
                        const uint8_t* mask, int64_t mask_stride, float scale, const float* norm, const float* dlogp,
                        const float* entropy, const float* dentropy, void* grad, int64_t grad_stride, cudaStream_t st) {
  if (rows <= 0) return true;
  const RowArgs a = {logits, row_stride, token, mask, mask_stride, rows, vocab, scale};
  const GradArgs g = {norm, dlogp, entropy, dentropy, grad, grad_stride};
  if (dtype == XRL_BF16) return mask ? launch_grad<bf16, true>(a, g, st) : launch_grad<bf16, false>(a, g, st);
  return mask ? launch_grad<float, true>(a, g, st) : launch_grad<float, false>(a, g, st);
}

}  // namespace xrl
