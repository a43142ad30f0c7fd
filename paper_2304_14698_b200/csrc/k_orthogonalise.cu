// Newton-Schulz orthogonalisation of update matrices (xrl_orthogonalise), on the 5th-generation tensor cores:
//   X_0 = G / (||G||_F + eps);   A = X X^T (the smaller side),  B = b A + c A^2,  X <- a X + B X;   `steps` times.
//
// Operands are fp16, scaled by powers of two: X has entries of 1 / sqrt(rows cols) in the mean and none above 1.2, A and B
// none above 3, so 2^k with k <= 14 keeps all of them inside fp16's range with 11 bits each.  X travels as the sum of two
// fp16 numbers, hi + lo (22 bits).  What is rounded to one fp16 number where it meets another matrix would cost the most on
// the diagonals of A and B, whose entries outweigh all others: D_A and D_B are held apart in fp32, and with A = D_A + F
//   B_ij = b F_ij + c ((d_i + d_j) F_ij + (F F)_ij),   X' = (a + D_B) X + (B - D_B) X
// only the small rest goes through the tensor cores.  (2-norm error of five steps before the result's rounding, matrices of
// 64 to 4,096: 1e-4 to 1.3e-3, 2 to 7 times less than with the diagonals inside; rounding to bf16 is 1.7e-3.)  bf16 updates
// take one product of hi parts; fp32 ones add hi lo and lo hi, which leaves 2^-22 of an entry.
// A and B are symmetric: only tiles on and above the diagonal are computed, and stored twice.
//
// Bound by the tensor cores for large matrices; by the chain of 3 * steps launches for small ones.
// Every wait on an mbarrier is bounded; on expiry the kernel records XRL_ERR_TIMEOUT, lets its copies in flight land, frees
// its tensor memory and returns.
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

#include "xrl_umma.cuh"

namespace xrl {

using namespace umma;

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;     // the quintic's coefficients
constexpr float kGramScale = 16384.f;    // of F and of B's rest
constexpr int kNormBlocks = 64;          // partial sums of squares per matrix, at most
constexpr int kPad = 64;                 // row strides of the workspace's matrices are multiples of this

struct Half2 { __half *hi, *lo; };

// ---- norm and first X --------------------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256)
k_ns_norm(const T* __restrict__ g, int64_t ld, int64_t batch_stride, int rows, int cols, double* partial, int32_t* status) {
  enter();
  __shared__ double red[8];
  const T* m = g + blockIdx.y * batch_stride;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *status = XRL_OK;
  double s = 0.0;
  for (int r = blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += gridDim.x * 8)
    for (int c = threadIdx.x & 31; c < cols; c += 32) {
      const double v = to_float(m[r * ld + c]);
      s += v * v;
    }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) s += red[w];
    partial[blockIdx.y * gridDim.x + blockIdx.x] = s;
  }
}

__device__ __forceinline__ void split(float v, __half& hi, __half& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));
}

template <typename T>
__global__ void __launch_bounds__(256)
k_ns_start(const T* __restrict__ g, int64_t ld, int64_t batch_stride, int rows, int cols, const double* partial, int nparts,
           double eps, float scale, Half2 x, int64_t ldx) {
  enter();
  __shared__ double s_inv;
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int i = 0; i < nparts; ++i) s += partial[blockIdx.y * nparts + i];
    s_inv = double(scale) / (sqrt(s) + eps);
  }
  __syncthreads();
  const double inv = s_inv;
  const T* m = g + blockIdx.y * batch_stride;
  const int64_t base = blockIdx.y * int64_t(rows) * ldx;
  for (int r = blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += gridDim.x * 8)
    for (int c = threadIdx.x & 31; c < cols; c += 32) {
      __half hi, lo;
      split(float(double(to_float(m[r * ld + c])) * inv), hi, lo);
      x.hi[base + r * ldx + c] = hi;
      x.lo[base + r * ldx + c] = lo;
    }
}

// ---- the products ------------------------------------------------------------------------------------------------
enum Mode { GRAM, POLY, APPLY };
struct NsArgs {
  int m, n, k;                           // of the product
  int tiles_n, tiles;                    // per matrix; symmetric products: tiles on and above the diagonal
  int total;                             // tiles of all matrices
  float descale;                         // accumulator -> value
  Half2 in;                              // POLY: F; APPLY: X (the product's shape)
  int64_t ld_in;
  float in_unscale;
  const float* diag_in;                  // [batch x small side]
  Half2 out;
  int64_t ld_out;
  float out_scale;
  float* diag_out;
  void* user;                            // APPLY: the caller's matrices in place of `out`
  int64_t user_ld, user_batch;
  int32_t* status;
};

constexpr int kTile = 128, kStep = 64;   // rows per CTA, reduction per stage
constexpr int kOperand = kTile * kStep * 2;
constexpr int kEpiWarps = 8, kThreads = 64 + 32 * kEpiWarps;

// CHUNK: stages whose products stay in one accumulator.  The tensor cores cut the sum after each instruction instead of
// rounding it, which shrinks a sum of n instructions by about n / 4 units in its last place (fp32, 32 x 8,192 in one
// accumulator: 4e-5 of the update).  fp32 updates therefore add the accumulators of 128 entries of the reduction in registers,
// and issue the small products of a stage first, onto a small sum.
template <int NPROD> struct Cfg {
  static constexpr int CHUNK = NPROD == 1 ? 1 << 30 : 2;
  static constexpr int STAGE = kOperand * (NPROD == 1 ? 2 : 4);
  static constexpr int STAGES = NPROD == 1 ? 6 : 3;
  static constexpr int OFF_BAR = STAGES * STAGE;
  static constexpr int OFF_TMEM = OFF_BAR + 8 * (2 * STAGES + 4);
  static constexpr int SMEM_BYTES = OFF_TMEM + 16;
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// MN-major, 128-byte swizzle: 64 entries of the outer index by 8 of the reduction in 1,024 bytes, 64 x 64 chunks 8 KB apart
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr) {
  return uint64_t((addr & 0x3FFFFu) >> 4) | (uint64_t(8192 >> 4) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) |
         (uint64_t(2) << 61);
}
template <bool MN> __device__ __forceinline__ uint64_t operand_desc(uint32_t addr, int k) {
  return MN ? smem_desc_mn(addr + k * 2048) : smem_desc(addr + k * 32);
}
template <bool MN>
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* map, int outer, int k, int z, uint32_t bar) {
  if (MN) {
    tma_load_3d(dst, map, outer, k, z, bar);
    tma_load_3d(dst + kOperand / 2, map, outer + 64, k, z, bar);
  } else {
    tma_load_3d(dst, map, k, outer, z, bar);
  }
}

struct Tile { int z, i, j; };            // matrix, tile row, tile column
template <bool SYM> __device__ __forceinline__ Tile tile_of(const NsArgs& a, int t) {
  Tile r;
  r.z = t / a.tiles;
  t -= r.z * a.tiles;
  if (SYM) {                             // column by column of the upper triangle: column j holds j + 1 tiles
    int j = int((sqrtf(8.f * float(t) + 1.f) - 1.f) * 0.5f);
    while ((j + 1) * (j + 2) / 2 <= t) ++j;
    while (j * (j + 1) / 2 > t) --j;
    r.j = j;
    r.i = t - j * (j + 1) / 2;
  } else {
    r.i = t / a.tiles_n;
    r.j = t - r.i * a.tiles_n;
  }
  return r;
}

__device__ __forceinline__ uint32_t pack_half2(__half a, __half b) {
  return uint32_t(__half_as_ushort(a)) | (uint32_t(__half_as_ushort(b)) << 16);
}
__device__ __forceinline__ void load32(const __half* p, uint32_t (&r)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 v = *reinterpret_cast<const uint4*>(p + 8 * i);
    r[4 * i] = v.x; r[4 * i + 1] = v.y; r[4 * i + 2] = v.z; r[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ float half_of(const uint32_t (&r)[16], int i) {
  return __half2float(__ushort_as_half(uint16_t(i & 1 ? r[i >> 1] >> 16 : r[i >> 1] & 0xFFFFu)));
}
__device__ __forceinline__ void store_row(__half* p, const uint32_t (&r)[16]) {
  store32(p, r[0], r[1], r[2], r[3], r[4], r[5], r[6], r[7]);
  store32(p + 16, r[8], r[9], r[10], r[11], r[12], r[13], r[14], r[15]);
}

template <typename T> __device__ __forceinline__ void store_user(T* p, const float (&v)[32], int count) {
  constexpr int N = VecOf<T>::N;
  if (count == 32 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < 32; i += N) {
      float f[N];
#pragma unroll
      for (int t = 0; t < N; ++t) f[t] = v[i + t];
      store_vec(p + i, f);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i < count) p[i] = T(v[i]);
  }
}

// 32 columns of a row of the result, from the accumulator
template <int MODE, bool TALL, int NPROD>
__device__ __forceinline__ void finish(const NsArgs& a, const Tile& t, int row, int col, const float* v) {
  const int small = TALL ? a.n : a.m;                    // (symmetric products: both)
  if (MODE == APPLY) {
    if (row >= a.m || col >= a.n) return;
    const int64_t at = (int64_t(t.z) * a.m + row) * a.ld_in + col;
    uint32_t hi[16], lo[16];
    load32(a.in.hi + at, hi);
    load32(a.in.lo + at, lo);
    float f[32];
    const float* d = a.diag_in + int64_t(t.z) * small;
    const float dr = TALL ? 0.f : kA + d[row];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float w = TALL ? kA + (col + i < small ? __ldg(d + col + i) : 0.f) : dr;
      f[i] = fmaf(w, (half_of(hi, i) + half_of(lo, i)) * a.in_unscale, v[i] * a.descale);
    }
    if (a.user) {
      typedef typename std::conditional<NPROD == 1, bf16, float>::type T;
      store_user(static_cast<T*>(a.user) + t.z * a.user_batch + row * a.user_ld + col, f, a.n - col < 32 ? a.n - col : 32);
    } else {
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        __half h0, h1, l0, l1;
        split(f[i] * a.out_scale, h0, l0);
        split(f[i + 1] * a.out_scale, h1, l1);
        hi[i >> 1] = pack_half2(h0, h1);
        lo[i >> 1] = pack_half2(l0, l1);
      }
      const int64_t to = (int64_t(t.z) * a.m + row) * a.ld_out + col;
      store_row(a.out.hi + to, hi);
      store_row(a.out.lo + to, lo);
    }
    return;
  }
  if (col >= a.n || row >= a.m) return;
  float f[32];
  const float* d = a.diag_in + int64_t(t.z) * small;
  if (MODE == POLY) {
    const int64_t at = (int64_t(t.z) * a.m + row) * a.ld_in + col;
    uint32_t hi[16], lo[16];
    load32(a.in.hi + at, hi);
    load32(a.in.lo + at, lo);
    const float di = d[row];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float x = (half_of(hi, i) + half_of(lo, i)) * a.in_unscale, dj = col + i < a.n ? __ldg(d + col + i) : 0.f;
      const float s = v[i] * a.descale;
      f[i] = col + i == row ? fmaf(kB, di, kC * fmaf(di, di, s)) : fmaf(kB, x, kC * fmaf(di + dj, x, s));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = v[i] * a.descale;
  }
  const bool lo_too = MODE == GRAM || NPROD > 1;
  uint32_t hi[16], lo[16];
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    __half h0, h1, l0, l1;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (col + i + e == row) { a.diag_out[int64_t(t.z) * small + row] = f[i + e]; f[i + e] = 0.f; }
    split(f[i] * a.out_scale, h0, l0);
    split(f[i + 1] * a.out_scale, h1, l1);
    hi[i >> 1] = pack_half2(h0, h1);
    lo[i >> 1] = pack_half2(l0, l1);
  }
  const int64_t base = int64_t(t.z) * a.m * a.ld_out;
  store_row(a.out.hi + base + row * a.ld_out + col, hi);
  if (lo_too) store_row(a.out.lo + base + row * a.ld_out + col, lo);
  if (t.i != t.j) {                      // and below the diagonal: 32 lanes write 32 neighbours
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (col + i >= a.n) break;
      const int64_t to = base + (col + i) * a.ld_out + row;
      a.out.hi[to] = __ushort_as_half(uint16_t(i & 1 ? hi[i >> 1] >> 16 : hi[i >> 1]));
      if (lo_too) a.out.lo[to] = __ushort_as_half(uint16_t(i & 1 ? lo[i >> 1] >> 16 : lo[i >> 1]));
    }
  }
}

struct Maps { CUtensorMap a_hi, a_lo, b_hi, b_lo; };

template <int MODE, bool TALL, int NPROD>
__global__ void __launch_bounds__(kThreads, 1) k_ns_product(const __grid_constant__ Maps maps, const NsArgs a) {
  using C = Cfg<NPROD>;
  constexpr bool SYM = MODE != APPLY, A_MN = MODE == GRAM && TALL, B_MN = A_MN || (MODE == APPLY && !TALL);
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((base & 1023u) != 0) {
    if (threadIdx.x == 0) raise(a.status, XRL_ERR_UNSUPPORTED);
    return;
  }
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_TMEM);
  auto bar_full = [&](int s) { return base + C::OFF_BAR + 8u * s; };
  auto bar_empty = [&](int s) { return base + C::OFF_BAR + 8u * (C::STAGES + s); };
  auto bar_acc_full = [&](int b) { return base + C::OFF_BAR + 8u * (2 * C::STAGES + b); };
  auto bar_acc_empty = [&](int b) { return base + C::OFF_BAR + 8u * (2 * C::STAGES + 2 + b); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(bar_acc_full(b), 1); mbar_init(bar_acc_empty(b), kEpiWarps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(tmem_slot)), "r"(uint32_t(2 * kTile)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int ksteps = (a.k + kStep - 1) / kStep;
  enter();

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      fence_async_all();
      for (int tile = blockIdx.x; ok && tile < a.total; tile += gridDim.x) {
        const Tile t = tile_of<SYM>(a, tile);
        for (int k = 0; k < ksteps; ++k, ++it) {
          const int s = it % C::STAGES;
          const uint32_t round = it / C::STAGES;
          if (round > 0 && !mbar_wait(bar_empty(s), (round - 1) & 1)) { ok = false; break; }
          mbar_expect_tx(bar_full(s), C::STAGE);
          const uint32_t at = base + s * C::STAGE;
          load_operand<A_MN>(at, &maps.a_hi, t.i * kTile, k * kStep, t.z, bar_full(s));
          load_operand<B_MN>(at + kOperand, &maps.b_hi, t.j * kTile, k * kStep, t.z, bar_full(s));
          if (NPROD > 1) {
            load_operand<A_MN>(at + 2 * kOperand, &maps.a_lo, t.i * kTile, k * kStep, t.z, bar_full(s));
            load_operand<B_MN>(at + 3 * kOperand, &maps.b_lo, t.j * kTile, k * kStep, t.z, bar_full(s));
          }
        }
      }
      if (!ok) {
        raise(a.status, XRL_ERR_TIMEOUT);
        for (uint32_t j = it > uint32_t(C::STAGES) ? it - C::STAGES : 0; j < it; ++j)
          mbar_wait(bar_full(j % C::STAGES), (j / C::STAGES) & 1);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      // fp32 accumulators, fp16 x fp16, M = N = 128; bits 15 and 16: MN-major operands
      constexpr uint32_t idesc = (1u << 4) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | (uint32_t(kTile >> 3) << 17) |
                                 (uint32_t(kTile >> 4) << 24);
      uint32_t it = 0, lt = 0;
      bool ok = true;
      for (int tile = blockIdx.x; ok && tile < a.total; tile += gridDim.x) {
        for (int k0 = 0; ok && k0 < ksteps; k0 = k0 < ksteps - C::CHUNK ? k0 + C::CHUNK : ksteps, ++lt) {
          const int k1 = k0 < ksteps - C::CHUNK ? k0 + C::CHUNK : ksteps, buf = lt & 1;
          if (lt > 1 && !mbar_wait(bar_acc_empty(buf), ((lt >> 1) - 1) & 1)) { ok = false; break; }
          tc_fence_after();
          const uint32_t acc = tmem_base + uint32_t(buf * kTile);
          for (int k = k0; k < k1; ++k, ++it) {
            const int s = it % C::STAGES;
            if (!mbar_wait(bar_full(s), (it / C::STAGES) & 1)) { ok = false; break; }
            tc_fence_after();
            const uint32_t at = base + s * C::STAGE;
            if (NPROD > 1) {
#pragma unroll
              for (int kk = 0; kk < kStep / 16; ++kk) {
                tc_mma(acc, operand_desc<A_MN>(at, kk), operand_desc<B_MN>(at + 3 * kOperand, kk), idesc, k > k0 || kk ? 1u : 0u);
                tc_mma(acc, operand_desc<A_MN>(at + 2 * kOperand, kk), operand_desc<B_MN>(at + kOperand, kk), idesc, 1u);
              }
            }
#pragma unroll
            for (int kk = 0; kk < kStep / 16; ++kk)
              tc_mma(acc, operand_desc<A_MN>(at, kk), operand_desc<B_MN>(at + kOperand, kk), idesc,
                     NPROD > 1 || k > k0 || kk ? 1u : 0u);
            tc_commit(bar_empty(s));
          }
          if (ok) tc_commit(bar_acc_full(buf));
        }
      }
      if (!ok) raise(a.status, XRL_ERR_TIMEOUT);
    }
  } else {
    constexpr int COLS = kTile / 2;      // of a warp
    const int q = warp & 3, half = (warp - 2) >> 2;
    uint32_t lt = 0;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < a.total; tile += gridDim.x) {
      const Tile t = tile_of<SYM>(a, tile);
      const int row = t.i * kTile + q * 32 + lane, col = t.j * kTile + half * COLS;
      float sum[NPROD == 1 ? 1 : COLS];
      for (int k0 = 0; k0 < ksteps; k0 = k0 < ksteps - C::CHUNK ? k0 + C::CHUNK : ksteps, ++lt) {
        const int buf = lt & 1;
        uint32_t got = 1;
        if (lane == 0) {
          got = 0;                       // a whole tile is multiplied first: the limit of one wait, several times over
          for (int w = 0; w < 4 && !got; ++w) got = mbar_wait(bar_acc_full(buf), (lt >> 1) & 1) ? 1u : 0u;
          if (!got) raise(a.status, XRL_ERR_TIMEOUT);
        }
        ok = __shfl_sync(0xFFFFFFFFu, got, 0) != 0;
        if (!ok) break;
        tc_fence_after();
        const uint32_t taddr = tmem_base + (uint32_t(q * 32) << 16) + uint32_t(buf * kTile + half * COLS);
        if (NPROD == 1) {                // straight from the accumulator
#pragma unroll 1
          for (int c = 0; c < COLS; c += 32) {
            __syncwarp();
            uint32_t v[32];
            tc_ld32(taddr + c, v);
            tc_wait_ld();
            float f[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
            finish<MODE, TALL, NPROD>(a, t, row, col + c, f);
          }
        } else {
#pragma unroll
          for (int c = 0; c < COLS; c += 32) {
            uint32_t v[32];
            tc_ld32(taddr + c, v);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[NPROD == 1 ? 0 : c + i] = (k0 == 0 ? 0.f : sum[NPROD == 1 ? 0 : c + i]) + __uint_as_float(v[i]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_acc_empty(buf));
      }
      if (!ok) break;
      if (NPROD > 1) {
#pragma unroll
        for (int c = 0; c < COLS; c += 32) finish<MODE, TALL, NPROD>(a, t, row, col + c, sum + c);
      }
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(uint32_t(2 * kTile)) : "memory");
  }
}

// ---- host side ---------------------------------------------------------------------------------------------------
// fp16 matrices [batch][rows][cols] with rows ld entries apart, box of 64 columns by box_rows rows, 128-byte swizzle
bool make_map3(CUtensorMap* m, const void* ptr, int batch, int rows, int cols, int64_t ld, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {cuuint64_t(cols), cuuint64_t(rows), cuuint64_t(batch)};
  cuuint64_t strides[2] = {cuuint64_t(ld) * 2, cuuint64_t(ld) * 2 * cuuint64_t(rows)};
  cuuint32_t box[3] = {KCH, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// one operand's pair of maps: its outer index along the rows (K-major) or along the columns (MN-major)
bool make_operand(CUtensorMap* hi, CUtensorMap* lo, const Half2& p, int batch, int rows, int cols, int64_t ld, bool mn) {
  const uint32_t box = mn ? kStep : kTile;
  return make_map3(hi, p.hi, batch, rows, cols, ld, box) && make_map3(lo, p.lo, batch, rows, cols, ld, box);
}

template <int MODE, bool TALL, int NPROD>
bool launch_product(const Maps& maps, const NsArgs& a, cudaStream_t st) {
  static bool done[64] = {};
  if (!ensure_dynamic_smem(k_ns_product<MODE, TALL, NPROD>, Cfg<NPROD>::SMEM_BYTES, done)) return false;
  const unsigned grid = unsigned(a.total < kNumSMs ? a.total : kNumSMs);
  launch(k_ns_product<MODE, TALL, NPROD>, grid, kThreads, Cfg<NPROD>::SMEM_BYTES, st, maps, a);
  return true;
}

// the workspace's pieces
struct NsSpace {
  int32_t* status;
  double* partial;
  float *dA, *dB;
  Half2 x[2], f, b;
  int64_t ldx, ldm;
  size_t bytes;
};
NsSpace layout(void* ws, int batch, int rows, int cols) {
  NsSpace s;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t p = at;
    at += (bytes + 255) & ~size_t(255);
    return static_cast<char*>(ws) + p;
  };
  const int small = rows < cols ? rows : cols;
  s.ldx = (int64_t(cols) + kPad - 1) / kPad * kPad;
  s.ldm = (int64_t(small) + kPad - 1) / kPad * kPad;
  s.status = reinterpret_cast<int32_t*>(take(4));
  s.partial = reinterpret_cast<double*>(take(size_t(batch) * kNormBlocks * 8));
  s.dA = reinterpret_cast<float*>(take(size_t(batch) * small * 4));
  s.dB = reinterpret_cast<float*>(take(size_t(batch) * small * 4));
  const size_t xb = size_t(batch) * rows * s.ldx * 2, mb = size_t(batch) * small * s.ldm * 2;
  for (Half2* p : {&s.x[0], &s.x[1]}) {
    p->hi = reinterpret_cast<__half*>(take(xb));
    p->lo = reinterpret_cast<__half*>(take(xb));
  }
  for (Half2* p : {&s.f, &s.b}) {
    p->hi = reinterpret_cast<__half*>(take(mb));
    p->lo = reinterpret_cast<__half*>(take(mb));
  }
  s.bytes = at;
  return s;
}

template <typename T, int NPROD, bool TALL>
bool run_steps(int batch, int rows, int cols, const void* grad, int64_t ld, int64_t bs, int steps, double eps, void* out,
               int64_t out_ld, int64_t out_bs, const NsSpace& s, int32_t* status, cudaStream_t st) {
  const int small = TALL ? cols : rows, large = TALL ? rows : cols;
  int k = int(lround(0.5 * log2(double(rows) * double(cols))));
  if (k > 14) k = 14;
  const float xs = float(1 << k);
  const int rb = (rows + 7) / 8 < kNormBlocks ? (rows + 7) / 8 : kNormBlocks;
  launch(k_ns_norm<T>, dim3(rb, batch), 256, 0, st, static_cast<const T*>(grad), ld, bs, rows, cols, s.partial, status);
  launch(k_ns_start<T>, dim3((rows + 7) / 8, batch), 256, 0, st, static_cast<const T*>(grad), ld, bs, rows, cols, s.partial, rb,
         eps, xs, s.x[0], s.ldx);

  const int tm = (small + kTile - 1) / kTile, tl = (large + kTile - 1) / kTile;
  NsArgs sym = {};
  sym.m = sym.n = small;
  sym.tiles_n = tm;
  sym.tiles = tm * (tm + 1) / 2;
  sym.total = sym.tiles * batch;
  sym.ld_in = sym.ld_out = s.ldm;
  sym.out_scale = kGramScale;
  sym.in_unscale = 1.f / kGramScale;
  sym.diag_in = s.dA;
  sym.status = status;
  NsArgs gram = sym, poly = sym, apply = sym;
  gram.k = large;
  gram.descale = 1.f / (xs * xs);
  gram.out = s.f;
  gram.diag_out = s.dA;
  poly.k = small;
  poly.descale = 1.f / (kGramScale * kGramScale);
  poly.in = s.f;
  poly.out = s.b;
  poly.diag_out = s.dB;
  apply.m = rows;
  apply.n = cols;
  apply.k = small;
  apply.tiles_n = TALL ? tm : tl;
  apply.tiles = tm * tl;
  apply.total = apply.tiles * batch;
  apply.descale = 1.f / (kGramScale * xs);
  apply.ld_in = apply.ld_out = s.ldx;
  apply.in_unscale = 1.f / xs;
  apply.out_scale = xs;
  apply.diag_in = s.dB;

  Maps mg[2], mp, ma[2];
  bool ok = make_operand(&mp.a_hi, &mp.a_lo, s.f, batch, small, small, s.ldm, false);
  mp.b_hi = mp.a_hi;
  mp.b_lo = mp.a_lo;
  for (int i = 0; i < 2; ++i) {
    ok = ok && make_operand(&mg[i].a_hi, &mg[i].a_lo, s.x[i], batch, rows, cols, s.ldx, TALL);
    mg[i].b_hi = mg[i].a_hi;
    mg[i].b_lo = mg[i].a_lo;
    if (TALL) {
      ok = ok && make_operand(&ma[i].a_hi, &ma[i].a_lo, s.x[i], batch, rows, cols, s.ldx, false) &&
           make_operand(&ma[i].b_hi, &ma[i].b_lo, s.b, batch, small, small, s.ldm, false);
    } else {
      ok = ok && make_operand(&ma[i].a_hi, &ma[i].a_lo, s.b, batch, small, small, s.ldm, false) &&
           make_operand(&ma[i].b_hi, &ma[i].b_lo, s.x[i], batch, rows, cols, s.ldx, true);
    }
  }
  for (int i = 0; ok && i < steps; ++i) {
    apply.in = s.x[i & 1];
    apply.out = s.x[(i + 1) & 1];
    if (i == steps - 1) {
      apply.user = out;
      apply.user_ld = out_ld;
      apply.user_batch = out_bs;
    }
    ok = launch_product<GRAM, TALL, NPROD>(mg[i & 1], gram, st) && launch_product<POLY, false, NPROD>(mp, poly, st) &&
         launch_product<APPLY, TALL, NPROD>(ma[i & 1], apply, st);
  }
  return ok;
}

}  // namespace

size_t orthogonalise_workspace(int32_t batch, int32_t rows, int32_t cols) { return layout(nullptr, batch, rows, cols).bytes; }

bool launch_orthogonalise(int dtype, int32_t batch, int32_t rows, int32_t cols, const void* grad, int64_t ld, int64_t batch_stride,
                          int32_t steps, float eps, void* out, int64_t out_ld, int64_t out_batch_stride, void* workspace,
                          int32_t* status, cudaStream_t st) {
  const NsSpace s = layout(workspace, batch, rows, cols);
  if (!status) status = s.status;
  auto f = dtype == XRL_BF16 ? (rows > cols ? run_steps<bf16, 1, true> : run_steps<bf16, 1, false>)
                             : (rows > cols ? run_steps<float, 3, true> : run_steps<float, 3, false>);
  return f(batch, rows, cols, grad, ld, batch_stride, steps, double(eps), out, out_ld, out_batch_stride, s, status, st);
}

}  // namespace xrl
