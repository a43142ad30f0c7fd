// Newton-Schulz orthogonalisation of update matrices (xrl_orthogonalise), on the 5th-generation tensor cores:
//   X_0 = G / (||G||_F + eps);   A = X X^T (the smaller side),  B = b A + c A^2,  X <- a X + B X;   `steps` times.
//
// Operands are fp16, scaled by powers of two: X has entries of 1 / sqrt(rows cols) in the mean and none above 1.2, A and B
// none above 3, so 2^k with k <= 14 keeps all of them inside fp16's range with 11 bits each.  X travels as the sum of two
// fp16 numbers, hi + lo (22 bits).  What is rounded to one fp16 number where it meets another matrix would cost the most on
// the diagonals of A and B, whose entries outweigh all others: D_A and D_B are held apart in fp32, and with A = D_A + F
//   B_ij = b F_ij + c ((d_i + d_j) F_ij + (F F)_ij),   X' = (a + D_B) X + (B - D_B) X
// only the small rest goes through the tensor cores.  (2-norm error of five steps before the result's rounding, matrices of
// 64 to 4,096 with random entries: 1e-4 to 1.3e-3, 2 to 7 times less than with the diagonals inside; rounding to bf16 is 1.7e-3.
// Where entries have one size their roundings do not average out, and X's, F's and B's go into every product the same way: all
// ones, or signs of rank one, 1e-3 to 1.4e-2, 256 square 1.28e-2.)  bf16 updates take one product of hi parts; fp32 ones add
// hi lo and lo hi, which leaves 2^-22 of an entry.
// A and B are symmetric: only tiles on and above the diagonal are computed, and stored twice.
//
// Bound by the tensor cores for large matrices; by the chain of 3 * steps launches for small ones.
// Every wait on an mbarrier is bounded; on expiry the kernel records XRL_ERR_TIMEOUT, lets its copies in flight land, frees
// its tensor memory and returns.  The last product then writes NaN: all over when it finds the word set by a launch before
// it, else what a warp had to write whose wait ran out.  No caller takes such a result for an update.
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

#include "xrl_umma.cuh"

namespace xrl {

using namespace umma;

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;     // the quintic's coefficients
constexpr float kGramScale = 16384.f;    // of F and of B's rest
constexpr int kNormBlocks = 256;         // partial sums of squares per matrix, at most
constexpr int kPad = 64;                 // row strides of the workspace's matrices are multiples of this

struct Half2 { __half *hi, *lo; };

// ---- norm and first X --------------------------------------------------------------------------------------------
// eight entries of a row from column c on (0 beyond the last)
template <typename T>
__device__ __forceinline__ void load8(const T* row, int c, int cols, float (&f)[8]) {
  constexpr int N = VecOf<T>::N;
  if (c + 8 <= cols && (reinterpret_cast<uintptr_t>(row + c) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < 8; i += N) {
      float v[N];
      unpack(*reinterpret_cast<const uint4*>(row + c + i), v);
#pragma unroll
      for (int t = 0; t < N; ++t) f[i + t] = v[t];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c + i < cols ? to_float(row[c + i]) : 0.f;
  }
}

template <typename T>
__global__ void __launch_bounds__(256)
k_ns_norm(const T* g, int64_t ld, int64_t batch_stride, int rows, int cols, double* partial, int32_t* status) {
  enter();
  __shared__ double red[8];
  const T* m = g + blockIdx.y * batch_stride;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *status = XRL_OK;
  const int groups = (cols + 7) / 8;
  const int64_t pieces = int64_t(rows) * groups;
  double s = 0.0;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += int64_t(gridDim.x) * 256) {
    const int64_t r = i / groups;
    float f[8];
    load8(m + r * ld, int(i - r * groups) * 8, cols, f);
#pragma unroll
    for (int t = 0; t < 8; ++t) s = fma(double(f[t]), double(f[t]), s);
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

// two values as hi + lo
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(a, b);
  const float2 back = __half22float2(h);
  const __half2 l = __floats2half2_rn(a - back.x, b - back.y);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  lo = *reinterpret_cast<const uint32_t*>(&l);
}

template <typename T>
__global__ void __launch_bounds__(256)
k_ns_start(const T* g, int64_t ld, int64_t batch_stride, int rows, int cols, const double* partial, int nparts, double eps,
           float scale, Half2 x, int64_t ldx) {
  enter();
  __shared__ double s_inv;
  if (threadIdx.x < 32) {
    double s = 0.0;
    for (int i = threadIdx.x; i < nparts; i += 32) s += partial[blockIdx.y * nparts + i];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if (threadIdx.x == 0) s_inv = double(scale) / (sqrt(s) + eps);
  }
  __syncthreads();
  const double inv = s_inv;
  const T* m = g + blockIdx.y * batch_stride;
  const int64_t base = blockIdx.y * int64_t(rows) * ldx;
  const int groups = (cols + 7) / 8;
  const int64_t pieces = int64_t(rows) * groups;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += int64_t(gridDim.x) * 256) {
    const int64_t r = i / groups;
    const int c = int(i - r * groups) * 8;
    float f[8];
    load8(m + r * ld, c, cols, f);
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) split2(float(double(f[2 * t]) * inv), float(double(f[2 * t + 1]) * inv), hi[t], lo[t]);
    *reinterpret_cast<uint4*>(x.hi + base + r * ldx + c) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(x.lo + base + r * ldx + c) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

// ---- the products ------------------------------------------------------------------------------------------------
enum Mode { GRAM, POLY, APPLY };
struct NsArgs {
  int m, n, k;                           // of the product
  int tiles_n, tiles;                    // per matrix; symmetric products: tiles on and above the diagonal
  int total;                             // tiles of all matrices
  int parts;                             // CTAs that share a tile's reduction (SPLIT)
  float descale;                         // accumulator -> value
  float gain;                            // accumulator -> its share of the scaled result
  const float* diag_in;                  // [batch][diag_stride]
  float* diag_out;
  int64_t diag_stride;
  void* user;                            // APPLY: the caller's matrices in place of the next X
  int64_t user_ld, user_batch;
  float unscale;                         // scaled result -> the caller's
  int32_t* status;
};

constexpr int kRows = 128, kStep = 64;   // rows of the result per CTA, reduction per stage
constexpr int kEpiWarps = 16, kThreads = 64 + 32 * kEpiWarps;
constexpr int kBlockBytes = 32 * 32 * 2; // a 32 x 32 piece of an epilogue warp: rows of 64 bytes, 64-byte swizzle

// CTAS: of a tile.  A pair multiplies 256 rows by N columns with one instruction; each holds its 128 rows of the left operand
// and N / 2 of the right one, so a tile of 256 x 256 asks half of what four of 128 x 128 do of L2.
// CHUNK: stages whose products stay in one accumulator.  The tensor cores cut the sum after each instruction instead of
// rounding it, which shrinks a sum of n instructions by about n / 4 units in its last place (fp32, 32 x 8,192 in one
// accumulator: 4e-5 of the update).  fp32 updates therefore add the accumulators of 128 (pairs: 256) entries of the reduction in
// registers.  Errors against 64 bits, of 49 x 1,270, 256 and 512 square by 128 entries 5e-7, 6e-7 and 6e-7, by 256 1.0e-6, 1.2e-6
// and 1.1e-6 (five layers of 256 then 92 instead of 96 us), of 2,048 square by 256 1.2e-6, by 384 1.9e-6 (517 instead of 521 us);
// plain fp32 products have 1.3e-6, 1.8e-6, 2.4e-6 and 3.6e-6.
// APART: products with a lo part go to an accumulator of their own, so that one instruction multiplies a left hi part
// with both parts of the right operand (four layers of 512 135 -> 128 us); the pairs, whose right operand is split over two
// SMs, add them to the same one, a stage's small products first.
template <int CTAS, int COLS, int NPROD> struct Cfg {
  static constexpr int M = CTAS * kRows, N = COLS;
  static constexpr int SUB = M / N;                       // tiles side by side in a square of M x M
  static constexpr int CHUNK = NPROD == 1 ? 1 << 30 : CTAS == 1 ? 2 : 4;
  static constexpr bool APART = NPROD > 1 && CTAS == 1;
  static constexpr int ACC = APART ? 2 * N : N;           // columns of an accumulator
  static constexpr int B_ROWS = N / CTAS;
  static constexpr int A_BYTES = kRows * kStep * 2, B_BYTES = B_ROWS * kStep * 2;
  static constexpr int PARTS = NPROD == 1 ? 1 : 2;        // hi; hi and lo
  static constexpr int OFF_B = PARTS * A_BYTES;           // a stage: A hi, A lo, B hi, B lo
  static constexpr int STAGE = PARTS * (A_BYTES + B_BYTES);
  static constexpr int STAGE_BYTES = kEpiWarps * 2 * kBlockBytes;
  static constexpr int MOST = (227 * 1024 - STAGE_BYTES - 512) / STAGE;
  static constexpr int STAGES = MOST < 6 ? MOST : 6;
  static constexpr int OFF_BLOCKS = STAGES * STAGE;       // two pieces per epilogue warp: hi and lo
  static constexpr int OFF_BAR = OFF_BLOCKS + STAGE_BYTES;
  static constexpr int OFF_TMEM = OFF_BAR + 8 * (2 * STAGES + 4 + kEpiWarps);
  static constexpr int SMEM_BYTES = OFF_TMEM + 16;
  static constexpr int TMEM_COLS = 2 * ACC;
  static constexpr int WARP_COLS = N == 256 ? 64 : 32;    // of an epilogue warp
  static constexpr int WORKERS = 4 * (N / WARP_COLS);     // epilogue warps with something to do
  static_assert(SMEM_BYTES <= 227 * 1024 && M % N == 0 && WORKERS <= kEpiWarps, "shared memory of one SM, whole squares");
};

// of a pair, every copy reports to the first CTA's barrier (the same offset; bit 24 of a shared address tells the two apart)
template <int CTAS>
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if (CTAS == 1)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar & 0xFEFFFFFFu) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void mma(uint32_t acc, uint64_t da, uint64_t db, uint32_t idesc, uint32_t add) {
  if (CTAS == 1) {
    tc_mma(acc, da, db, idesc, add);
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(acc), "l"(da), "l"(db), "r"(idesc), "r"(add) : "memory");
  }
}
// arrives at the barrier, of a pair at both CTAs', when the products issued so far are done
template <int CTAS> __device__ __forceinline__ void commit(uint32_t bar) {
  if (CTAS == 1)
    tc_commit(bar);
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(uint16_t(3)) : "memory");
}
// arrives at the first CTA's barrier
template <int CTAS> __device__ __forceinline__ void arrive_first(uint32_t bar) {
  if (CTAS == 1) {
    mbar_arrive(bar);
  } else {
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.release.cluster.shared::cluster.b64 _, [a];\n\t}" ::"r"(bar) : "memory");
  }
}
__device__ __forceinline__ bool elected() {              // true in one lane of a converged warp
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
// the whole warp, with one answer
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity) {
  return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity));
}
template <int CTAS> __device__ __forceinline__ void tile_sync() {      // all threads of the CTA, of a pair of both
  if (CTAS == 1) __syncthreads();
  else asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// After a wait that ran out in seconds: copies in flight take microseconds
__device__ __forceinline__ void let_copies_land() {
  const unsigned long long t0 = now_ns();
  while (now_ns() - t0 < 5000000ull) {}
}
// MN-major, 128-byte swizzle: 64 entries of the outer index by 8 of the reduction in 1,024 bytes, 64 x 64 chunks 8 KB apart
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr) {
  return uint64_t((addr & 0x3FFFFu) >> 4) | (uint64_t(8192 >> 4) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) |
         (uint64_t(2) << 61);
}
template <bool MN> __device__ __forceinline__ uint64_t operand_desc(uint32_t addr, int k) {
  return MN ? smem_desc_mn(addr + k * 2048) : smem_desc(addr + k * 32);
}
template <int CTAS, bool MN, int ROWS>
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* map, int outer, int k, int z, uint32_t bar) {
  if (MN) {
    for (int c = 0; c < ROWS; c += 64) tma_load_3d<CTAS>(dst + c * 128, map, outer + c, k, z, bar);
  } else {
    tma_load_3d<CTAS>(dst, map, k, outer, z, bar);
  }
}

// A tile: matrix, first row and column; `turned`: symmetric products store it a second time below the diagonal
struct Tile { int z, row, col; bool turned; };
template <int M, int N, bool SYM> __device__ __forceinline__ Tile tile_of(const NsArgs& a, int t) {
  Tile r;
  r.z = t / a.tiles;
  t -= r.z * a.tiles;
  r.turned = false;
  if (SYM) {                             // squares of M x M, column by column of the upper triangle: column j holds j + 1
    const int sub = t % (M / N);
    t /= M / N;
    int j = int((sqrtf(8.f * float(t) + 1.f) - 1.f) * 0.5f);
    while ((j + 1) * (j + 2) / 2 <= t) ++j;
    while (j * (j + 1) / 2 > t) --j;
    const int i = t - j * (j + 1) / 2;
    r.row = i * M;
    r.col = j * M + sub * N;
    r.turned = i != j;
  } else {
    const int i = t / a.tiles_n;
    r.row = i * M;
    r.col = (t - i * a.tiles_n) * N;
  }
  return r;
}

__device__ __forceinline__ void tc_st16(uint32_t taddr, const float* r) {
  const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
        "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(taddr) : "memory");
}
// 16 rows by 32 columns: lane l has columns 8 c + 2 (l % 4) and the next one, of row l / 4 in r[4 c], r[4 c + 1] and of row
// l / 4 + 8 in the two after them - which is how ldmatrix and stmatrix hand out 8 x 8 blocks of 16-bit numbers
__device__ __forceinline__ void tc_ld_blocks(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <bool TURN> __device__ __forceinline__ void stmatrix4(uint32_t at, const uint32_t* r) {
  if (TURN)
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
  else
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ float2 floats_of(uint32_t hi, uint32_t lo) {
  const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi)), l = __half22float2(*reinterpret_cast<const __half2*>(&lo));
  return make_float2(h.x + l.x, h.y + l.y);
}
// 16 bytes `chunk` of row `row` of a piece
__device__ __forceinline__ uint32_t block_at(uint32_t piece, int row, int chunk) {
  return piece + row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4);
}

struct Maps { CUtensorMap a_hi, a_lo, b_hi, b_lo, in_hi, in_lo, out_hi, out_lo; };

// An epilogue warp's pieces of 32 x 32.  What a piece reads besides the accumulator (`in`: F or X) comes by TMA to where its
// result will be; the result goes through shared memory to the TMA unit, and its transpose after it.
struct Pieces {
  uint32_t hi, bar;                      // lo: kBlockBytes behind hi
  uint32_t turned;                       // where the transpose leaves from: a place of its own where half the warps are idle, or hi
  uint32_t phase = 0;
  int lane;
};
template <int MODE>
__device__ __forceinline__ void ask(const Maps& maps, const NsArgs& a, Pieces& w, int z, int row, int col) {
  if (MODE == GRAM || row >= a.m || col >= a.n) return;
  fence_async_smem();                    // behind what the warp itself read and wrote here
  __syncwarp();
  if (w.lane == 0) {
    tma_wait_read<0>();                  // the stores that left from here have been read
    mbar_expect_tx(w.bar, 2 * kBlockBytes);
    tma_load_3d<1>(w.hi, &maps.in_hi, col, row, z, w.bar);
    tma_load_3d<1>(w.hi + kBlockBytes, &maps.in_lo, col, row, z, w.bar);
  }
}
template <int MODE, bool TALL, int NPROD, bool APART>
__device__ __forceinline__ bool finish(const Maps& maps, const NsArgs& a, Pieces& w, const Tile& t, int row, int col,
                                       uint32_t taddr, int lo_cols) {
  if (row >= a.m || col >= a.n) return true;             // the whole warp
  const int lane = w.lane, r = lane >> 2, c = (lane & 3) * 2;
  const uint32_t lo_piece = w.hi + kBlockBytes;
  const float* d = a.diag_in + t.z * a.diag_stride;
  float dr[4];
  float2 dc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {                          // (beyond the matrix: the padding's, for entries that are clipped)
    dr[i] = MODE == POLY || (MODE == APPLY && !TALL) ? __ldg(d + row + 8 * i + r) : 0.f;
    dc[i] = MODE == POLY || (MODE == APPLY && TALL) ? __ldg(reinterpret_cast<const float2*>(d + col + 8 * i + c)) : make_float2(0.f, 0.f);
  }
  if (MODE != GRAM) {
    if (!wait_warp(w.bar, w.phase)) return false;
    w.phase ^= 1;
  } else {
    if (lane == 0) tma_wait_read<0>();
    __syncwarp();
  }
  constexpr bool LO = MODE != POLY || NPROD > 1;
  const bool user = MODE == APPLY && a.user;
  uint32_t hi[4][4], lo[4][4];                           // 8 x 8 blocks of the result
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t v[16];
    tc_ld_blocks(taddr + (uint32_t(h * 16) << 16), v);
    if (APART && lo_cols) {
      uint32_t u[16];
      tc_ld_blocks(taddr + lo_cols + (uint32_t(h * 16) << 16), u);
      tc_wait_ld();
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(u[i]));
    } else {
      tc_wait_ld();
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int rb = 2 * h + s;
      const uint32_t at = block_at(w.hi, rb * 8 + (lane & 7), lane >> 3);
      uint32_t xh[4], xl[4];
      if (MODE != GRAM) {
        ldmatrix4(at, xh);
        ldmatrix4(at + kBlockBytes, xl);
      }
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) {
        const float v0 = __uint_as_float(v[4 * cb + 2 * s]), v1 = __uint_as_float(v[4 * cb + 2 * s + 1]);
        float f0 = v0 * a.gain, f1 = v1 * a.gain;
        if (MODE != GRAM) {
          const float2 x = floats_of(xh[cb], xl[cb]);
          const float w0 = MODE == POLY ? fmaf(kC, dr[rb] + dc[cb].x, kB) : kA + (TALL ? dc[cb].x : dr[rb]);
          const float w1 = MODE == POLY ? fmaf(kC, dr[rb] + dc[cb].y, kB) : kA + (TALL ? dc[cb].y : dr[rb]);
          f0 = fmaf(w0, x.x, f0);
          f1 = fmaf(w1, x.y, f1);
        }
        if (MODE != APPLY && rb == cb && row == col && (r == c || r == c + 1)) {       // the diagonal, kept apart
          float q = (r == c ? v0 : v1) * a.descale;
          if (MODE == POLY) q = fmaf(kB, dr[rb], kC * fmaf(dr[rb], dr[rb], q));
          if (row + 8 * rb + r < a.m) a.diag_out[t.z * a.diag_stride + row + 8 * rb + r] = q;
          if (r == c) f0 = 0.f;
          else f1 = 0.f;
        }
        if (user) {
          f0 *= a.unscale;
          f1 *= a.unscale;
          if (NPROD == 1) {
            hi[rb][cb] = pack_bf16x2(f0, f1);
          } else {                                       // rows of 128 bytes over both pieces, after all of `in` is read
            hi[rb][cb] = __float_as_uint(f0);
            lo[rb][cb] = __float_as_uint(f1);
          }
        } else {
          split2(f0, f1, hi[rb][cb], lo[rb][cb]);
        }
      }
      if (!user) {
        stmatrix4<false>(at, hi[rb]);
        if (LO) stmatrix4<false>(at + kBlockBytes, lo[rb]);
      } else if (NPROD == 1) {
        stmatrix4<false>(at, hi[rb]);
      }
    }
  }
  if (user) {
    typedef typename std::conditional<NPROD == 1, bf16, float>::type T;
    constexpr int N = VecOf<T>::N, CHUNKS = 32 / N;      // 16-byte chunks of a row
    __syncwarp();
    if (NPROD > 1) {
#pragma unroll
      for (int rb = 0; rb < 4; ++rb)
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          const int y = rb * 8 + r, chunk = (cb * 8 + c) >> 2;
          asm volatile("st.shared.v2.b32 [%0], {%1, %2};"
                       ::"r"(w.hi + y * 128 + ((chunk ^ (y & 7)) << 4) + (c & 2) * 4), "r"(hi[rb][cb]), "r"(lo[rb][cb]) : "memory");
        }
      __syncwarp();
    }
    T* out = static_cast<T*>(a.user) + t.z * a.user_batch + col;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int y = (i * 32 + lane) / CHUNKS, chunk = lane % CHUNKS;
      const uint32_t at = NPROD == 1 ? block_at(w.hi, y, chunk) : w.hi + y * 128 + ((chunk ^ (y & 7)) << 4);
      uint4 q;
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(at) : "memory");
      if (row + y < a.m) {
        T* p = out + (row + y) * a.user_ld + chunk * N;
        const int left = a.n - col - chunk * N;
        if (left >= N && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
          *reinterpret_cast<uint4*>(p) = q;
        } else {
          const T* e = reinterpret_cast<const T*>(&q);
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (j < left) p[j] = e[j];
        }
      }
    }
    __syncwarp();
    return true;
  }
  fence_async_smem();
  __syncwarp();
  if (lane == 0) {
    tma_store_3d(&maps.out_hi, w.hi, col, row, t.z);
    if (LO) tma_store_3d(&maps.out_lo, lo_piece, col, row, t.z);
    tma_commit();
  }
  if (MODE != APPLY && t.turned) {                       // below the diagonal
    if (w.turned == w.hi) {
      if (lane == 0) tma_wait_read<0>();
      __syncwarp();
    }
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
      stmatrix4<true>(block_at(w.turned, lane, rb), hi[rb]);
      if (LO) stmatrix4<true>(block_at(w.turned + kBlockBytes, lane, rb), lo[rb]);
    }
    fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_3d(&maps.out_hi, w.turned, row, col, t.z);
      if (LO) tma_store_3d(&maps.out_lo, w.turned + kBlockBytes, row, col, t.z);
      tma_commit();
    }
  }
  return true;
}

// NaN for the caller in place of a piece of up to 32 rows and `cols` columns
template <typename T> __device__ __noinline__ void write_none(T* out, int64_t ld, int rows, int cols) {
  for (int y = 0; y < rows && y < 32; ++y)
    for (int x = threadIdx.x & 31; x < cols; x += 32) out[y * ld + x] = T(NAN);
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
}

// SPLIT: a cluster of up to eight CTAs shares a tile of a long reduction, a stretch of it each; the accumulators then meet
// through the cluster's shared memory, each CTA adding up (always in the same order) and finishing some of the tile's pieces.  For
// Gram matrices of few tiles.
template <int CTAS, int COLS, int MODE, bool TALL, int NPROD, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1) k_ns_product(const __grid_constant__ Maps maps, const NsArgs a) {
  using C = Cfg<CTAS, COLS, NPROD>;
  constexpr bool SYM = MODE != APPLY, A_MN = MODE == GRAM && TALL, B_MN = A_MN || (MODE == APPLY && !TALL);
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  const int warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x) >> 5, 0), lane = threadIdx.x & 31;
  constexpr int DUMP = (C::N + 4) * 4;   // bytes of a row of a tile in shared memory
  const int group = SPLIT ? a.parts : CTAS;
  const int rank = SPLIT ? 0 : int(blockIdx.x) % CTAS, part = SPLIT ? int(blockIdx.x) % group : 0;
  const int first = int(blockIdx.x) / group, step = int(gridDim.x) / group;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_TMEM);
  auto bar_full = [&](int s) { return base + C::OFF_BAR + 8u * s; };
  auto bar_empty = [&](int s) { return base + C::OFF_BAR + 8u * (C::STAGES + s); };
  auto bar_acc_full = [&](int b) { return base + C::OFF_BAR + 8u * (2 * C::STAGES + b); };
  auto bar_acc_empty = [&](int b) { return base + C::OFF_BAR + 8u * (2 * C::STAGES + 2 + b); };
  auto bar_in = [&](int w) { return base + C::OFF_BAR + 8u * (2 * C::STAGES + 4 + w); };
  if (threadIdx.x == 0) {
    prefetch_map(&maps.a_hi);
    prefetch_map(&maps.b_hi);
    if (NPROD > 1) { prefetch_map(&maps.a_lo); prefetch_map(&maps.b_lo); }
    if (MODE != GRAM) { prefetch_map(&maps.in_hi); prefetch_map(&maps.in_lo); }
    for (int w = 0; w < kEpiWarps; ++w) mbar_init(bar_in(w), 1);
    for (int s = 0; s < C::STAGES; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(bar_acc_full(b), 1); mbar_init(bar_acc_empty(b), CTAS * C::WORKERS); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 1) {
    if (CTAS == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                   ::"r"(smem_u32(tmem_slot)), "r"(uint32_t(C::TMEM_COLS)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                   ::"r"(smem_u32(tmem_slot)), "r"(uint32_t(C::TMEM_COLS)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncwarp();
  tile_sync<CTAS>();
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xFFFFFFFFu, *tmem_slot, 0);
  const int total = a.total;
  const bool sound = (base & 1023u) == 0;                // the swizzle's pattern starts on 1,024 bytes
  auto give_up = [&]() { raise(a.status, sound ? XRL_ERR_TIMEOUT : XRL_ERR_UNSUPPORTED); };
  const int all_ksteps = (a.k + kStep - 1) / kStep;
  const int kbegin = SPLIT ? all_ksteps * part / group : 0;
  const int ksteps = SPLIT ? all_ksteps * (part + 1) / group - kbegin : all_ksteps;
  enter();
  // Where SMs are free for the next product's CTAs, one to an SM (five layers of 256 96 -> 92 us on the device, 128 x 1,024 100 ->
  // 93).  Not the last one, behind which any kernel may come (scores of 2,000 x 32,000 behind five layers of 256 118.4 -> 117.2
  // together, gradient 134.6 -> 133.6, scores of 4,096 x 1,201 100.1 -> 100.8).
  if (gridDim.x * 2 <= kNumSMs && !(MODE == APPLY && a.user)) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // Both of the next roles run with the whole warp, one lane of which issues: what the loops carry is then the same for all
  // lanes and stays in uniform registers, where the instructions want it.  (Run by one lane alone, a product instruction cost
  // that lane some 115 cycles, and a 256 x 256 x 16 product takes 128: 4,096 square bf16 1,504 us.)
  if (warp == 0) {
    uint32_t it = 0;
    bool ok = sound;
    fence_async_all();
    for (int tile = first; ok && tile < total; tile += step) {
      const Tile t = tile_of<C::M, C::N, SYM>(a, tile);
      const int row = t.row + rank * kRows, col = t.col + rank * C::B_ROWS;
      for (int k = 0; k < ksteps; ++k, ++it) {
        const int s = it % C::STAGES;
        const uint32_t round = it / C::STAGES;
        if (round > 0 && !wait_warp(bar_empty(s), (round - 1) & 1)) { ok = false; break; }
        const uint32_t at = base + s * C::STAGE;
        if (elected()) {
          if (rank == 0) mbar_expect_tx(bar_full(s), CTAS * C::STAGE);
          load_operand<CTAS, A_MN, kRows>(at, &maps.a_hi, row, (kbegin + k) * kStep, t.z, bar_full(s));
          load_operand<CTAS, B_MN, C::B_ROWS>(at + C::OFF_B, &maps.b_hi, col, (kbegin + k) * kStep, t.z, bar_full(s));
          if (NPROD > 1) {
            load_operand<CTAS, A_MN, kRows>(at + C::A_BYTES, &maps.a_lo, row, (kbegin + k) * kStep, t.z, bar_full(s));
            load_operand<CTAS, B_MN, C::B_ROWS>(at + C::OFF_B + C::B_BYTES, &maps.b_lo, col, (kbegin + k) * kStep, t.z, bar_full(s));
          }
        }
        __syncwarp();
      }
    }
    if (!ok) {
      if (lane == 0) give_up();
      let_copies_land();
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // fp32 accumulators, fp16 x fp16; bits 15 and 16: MN-major operands
      constexpr uint32_t idesc = (1u << 4) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | (uint32_t(C::N >> 3) << 17) |
                                 (uint32_t(C::M >> 4) << 24);
      constexpr uint32_t idesc_both = idesc + (uint32_t(C::N >> 3) << 17);       // twice the columns
      // a descriptor's address counts 16 bytes from its lowest bit
      const uint64_t a0 = operand_desc<A_MN>(base, 0), b0 = operand_desc<B_MN>(base + C::OFF_B, 0);
      constexpr int A_K = (A_MN ? 2048 : 32) >> 4, B_K = (B_MN ? 2048 : 32) >> 4, A_LO = C::A_BYTES >> 4, B_LO = C::B_BYTES >> 4;
      uint32_t it = 0, lt = 0;
      bool ok = sound;
      for (int tile = first; ok && tile < total; tile += step) {
        for (int k0 = 0; ok && k0 < ksteps; k0 = k0 < ksteps - C::CHUNK ? k0 + C::CHUNK : ksteps, ++lt) {
          const int k1 = k0 < ksteps - C::CHUNK ? k0 + C::CHUNK : ksteps, buf = lt & 1;
          if (lt > 1 && !wait_warp(bar_acc_empty(buf), ((lt >> 1) - 1) & 1)) { ok = false; break; }
          tc_fence_after();
          const uint32_t acc = tmem_base + uint32_t(buf * C::ACC);
          for (int k = k0; k < k1; ++k, ++it) {
            const int s = it % C::STAGES;
            if (!wait_warp(bar_full(s), (it / C::STAGES) & 1)) { ok = false; break; }
            tc_fence_after();
            const uint64_t da = a0 + uint64_t(s * (C::STAGE >> 4)), db = b0 + uint64_t(s * (C::STAGE >> 4));
            if (elected()) {
              const uint32_t first = k > k0 ? 1u : 0u;
#pragma unroll
              for (int kk = 0; kk < kStep / 16; ++kk) {
                const uint64_t ak = da + kk * A_K, bk = db + kk * B_K;
                if (NPROD == 1) {
                  mma<CTAS>(acc, ak, bk, idesc, first | kk ? 1u : 0u);
                } else if (C::APART) {   // hi and lo of the right operand lie side by side, and so do the accumulator's halves
                  mma<CTAS>(acc, ak, bk, idesc_both, first | kk ? 1u : 0u);
                  mma<CTAS>(acc + C::N, ak + A_LO, bk, idesc, 1u);
                } else {
                  mma<CTAS>(acc, ak, bk + B_LO, idesc, first | kk ? 1u : 0u);
                  mma<CTAS>(acc, ak + A_LO, bk, idesc, 1u);
                }
              }
              if (NPROD > 1 && !C::APART) {
#pragma unroll
                for (int kk = 0; kk < kStep / 16; ++kk) mma<CTAS>(acc, da + kk * A_K, db + kk * B_K, idesc, 1u);
              }
              commit<CTAS>(bar_empty(s));
              if (k + 1 == k1) commit<CTAS>(bar_acc_full(buf));
            }
            __syncwarp();
          }
        }
      }
      if (!ok && lane == 0) give_up();
    }
  } else if (warp - 2 < C::WORKERS) {
    constexpr int WC = C::WARP_COLS;
    const int q = warp & 3, side = (warp - 2) >> 2;
    Pieces w;
    w.hi = base + C::OFF_BLOCKS + (warp - 2) * 2 * kBlockBytes;
    w.turned = w.hi + (2 * C::WORKERS <= kEpiWarps ? C::WORKERS * 2 * kBlockBytes : 0);
    w.bar = bar_in(warp - 2);
    w.lane = lane;
    uint32_t lt = 0;
    bool ok = sound;
    bool broken = false;                 // by an earlier launch (the whole warp with one answer)
    if (MODE == APPLY && a.user) broken = __any_sync(0xFFFFFFFFu, *static_cast<volatile int32_t*>(a.status) != XRL_OK);
    for (int tile = first; ok && tile < total; tile += step) {
      const Tile t = tile_of<C::M, C::N, SYM>(a, tile);
      const int row = t.row + rank * kRows + q * 32, col = t.col + side * WC;
      ask<MODE>(maps, a, w, t.z, row, col);
      float sum[NPROD == 1 ? 1 : WC];
      for (int k0 = 0; k0 < ksteps; ++lt) {
        const int k1 = k0 < ksteps - C::CHUNK ? k0 + C::CHUNK : ksteps, buf = lt & 1;
        ok = false;                      // a whole tile is multiplied first: the limit of one wait, several times over
        for (int i = 0; i < 4 && !ok; ++i) ok = wait_warp(bar_acc_full(buf), (lt >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        const uint32_t taddr = tmem_base + (uint32_t(q * 32) << 16) + uint32_t(buf * C::ACC + side * WC);
        if (NPROD > 1 && ksteps > C::CHUNK) {
          // the sums so far; with the last accumulator they go back into its place
          uint32_t v[NPROD == 1 ? 1 : WC], u[NPROD == 1 ? 1 : WC];
          if constexpr (NPROD > 1) {
            static_assert(WC == 32, "one load");
            tc_ld32(taddr, v);
            if (C::APART) tc_ld32(taddr + C::N, u);
            tc_wait_ld();
          }
          if (k1 < ksteps) {             // the accumulator is free before its values are added
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_first<CTAS>(bar_acc_empty(buf));
          }
#pragma unroll
          for (int i = 0; i < (NPROD == 1 ? 1 : WC); ++i) sum[i] = (k0 == 0 ? 0.f : sum[i]) + (C::APART ? __uint_as_float(v[i]) + __uint_as_float(u[i]) : __uint_as_float(v[i]));
          k0 = k1;
          if (k1 < ksteps) continue;
          if constexpr (NPROD > 1 && !SPLIT) {
#pragma unroll
            for (int c = 0; c < WC; c += 16) tc_st16(taddr + c, sum + c);
          }
          if (!SPLIT) asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        }
        if constexpr (SPLIT) {
          uint32_t v[32];
          if (NPROD > 1 && ksteps > C::CHUNK) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(sum[NPROD == 1 ? 0 : i]);
          } else {
            tc_ld32(taddr, v);
            if (C::APART) {
              uint32_t u[32];
              tc_ld32(taddr + C::N, u);
              tc_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(u[i]));
            } else {
              tc_wait_ld();
            }
          }
          uint8_t* to = smem + (q * 32 + lane) * DUMP + side * 128;      // where the stages were: all are multiplied
#pragma unroll
          for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(to + 4 * i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
#pragma unroll 1
          for (int c = 0; ok && c < WC; c += 32) {
            if (c) ask<MODE>(maps, a, w, t.z, row, col + c);
            __syncwarp();
            ok = finish<MODE, TALL, NPROD, C::APART>(maps, a, w, t, row, col + c, taddr + c, ksteps > C::CHUNK ? 0 : C::N);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_first<CTAS>(bar_acc_empty(buf));
        }
        k0 = k1;
      }
    }
    if (!ok) {
      if (lane == 0) give_up();
      let_copies_land();
    }
    if (MODE == APPLY && a.user && (broken || !ok)) {    // (what it has written of the result too)
      typedef typename std::conditional<NPROD == 1, bf16, float>::type T;
      __syncwarp();
      for (int tile = first; tile < total; tile += step) {
        const Tile t = tile_of<C::M, C::N, SYM>(a, tile);
        const int row = t.row + rank * kRows + q * 32, col = t.col + side * WC;
        write_none(static_cast<T*>(a.user) + t.z * a.user_batch + row * a.user_ld + col, a.user_ld, a.m - row, min(a.n - col, WC));
      }
    }
    if (lane == 0) tma_wait_read<0>();   // (the launch ends when what they write is there)
  }
  if constexpr (SPLIT) {
    __syncwarp();
    tile_sync<2>();
    const int share = C::WORKERS / group, worker = warp - 2;
    if (worker >= 0 && worker < share && first < total) {
      const Tile t = tile_of<C::M, C::N, SYM>(a, first);
      const int piece = part * share + worker, q = piece & 3, side = piece >> 2;
      const uint32_t from = base + (q * 32 + lane) * DUMP + side * 128;
      float sum[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) sum[i] = 0.f;
#pragma unroll 1
      for (int p = 0; p < group; ++p) {
        uint32_t at;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(from), "r"(p));
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          float x, y, z, w;
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(x), "=f"(y), "=f"(z), "=f"(w) : "r"(at + 4 * i) : "memory");
          sum[i] += x; sum[i + 1] += y; sum[i + 2] += z; sum[i + 3] += w;
        }
      }
      tc_fence_after();
      // as a place to turn rows into 8 x 8 blocks: 32 columns for each of the warps that share 32 lanes
      const uint32_t taddr = tmem_base + (uint32_t((warp & 3) * 32) << 16) + uint32_t(worker >> 2) * 32;
      tc_st16(taddr, sum);
      tc_st16(taddr + 16, sum + 16);
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      Pieces w;
      w.hi = base + C::OFF_BLOCKS + worker * 2 * kBlockBytes;
      w.turned = w.hi + share * 2 * kBlockBytes;         // (half the workers at most have a piece)
      w.bar = bar_in(worker);
      w.lane = lane;
      finish<MODE, TALL, NPROD, C::APART>(maps, a, w, t, t.row + q * 32, t.col + side * 32, taddr, 0);
      if (lane == 0) tma_wait_read<0>();
    }
    __syncwarp();
    tile_sync<2>();                      // nobody leaves while its accumulators are read
  }
  tc_fence_before();
  __syncwarp();
  tile_sync<CTAS>();
  if (warp == 1) {
    tc_fence_after();
    if (CTAS == 1)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(uint32_t(C::TMEM_COLS)) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(uint32_t(C::TMEM_COLS)) : "memory");
  }
}

// ---- host side ---------------------------------------------------------------------------------------------------
// fp16 matrices [batch][rows][cols] with rows ld entries apart, box of 64 columns by box_rows rows, 128-byte swizzle; or the
// epilogue's pieces of 32 x 32, 64-byte swizzle
bool make_map3(CUtensorMap* m, const void* ptr, int batch, int rows, int cols, int64_t ld, uint32_t box_rows, bool piece = false) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {cuuint64_t(cols), cuuint64_t(rows), cuuint64_t(batch)};
  cuuint64_t strides[2] = {cuuint64_t(ld) * 2, cuuint64_t(ld) * 2 * cuuint64_t(rows)};
  cuuint32_t box[3] = {cuuint32_t(piece ? 32 : KCH), box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, piece ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// fp16 operands as matrices of the workspace
struct Operand { Half2 p; int rows, cols; int64_t ld; };
// one operand's pair of maps: its outer index along the rows (K-major, `outer` of them a load) or along the columns (MN-major)
bool make_operand(CUtensorMap* hi, CUtensorMap* lo, const Operand& o, int batch, bool mn, int outer, bool both) {
  const uint32_t box = mn ? kStep : outer;
  return make_map3(hi, o.p.hi, batch, o.rows, o.cols, o.ld, box) && (!both || make_map3(lo, o.p.lo, batch, o.rows, o.cols, o.ld, box));
}

template <int CTAS, int COLS, int MODE, bool TALL, int NPROD, bool SPLIT = false>
bool launch_tiles(const Maps& maps, NsArgs a, int batch, cudaStream_t st, int parts = 1) {
  using C = Cfg<CTAS, COLS, NPROD>;
  static bool done[64] = {};
  if (!ensure_dynamic_smem(k_ns_product<CTAS, COLS, MODE, TALL, NPROD, SPLIT>, C::SMEM_BYTES, done)) return false;
  const int tm = (a.m + C::M - 1) / C::M;
  a.tiles_n = (a.n + C::N - 1) / C::N;
  a.tiles = MODE == APPLY ? tm * a.tiles_n : tm * (tm + 1) / 2 * C::SUB;
  a.total = a.tiles * batch;
  a.parts = parts;
  const int cluster = CTAS * parts, most = kNumSMs / cluster;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = unsigned((a.total < most ? a.total : most) * cluster);
  cfg.blockDim = kThreads;
  cfg.dynamicSmemBytes = C::SMEM_BYTES;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_ns_product<CTAS, COLS, MODE, TALL, NPROD, SPLIT>, maps, a) == cudaSuccess;
}

bool make_pieces(CUtensorMap* hi, CUtensorMap* lo, const Operand& o, int batch) {
  return make_map3(hi, o.p.hi, batch, o.rows, o.cols, o.ld, 32, true) && make_map3(lo, o.p.lo, batch, o.rows, o.cols, o.ld, 32, true);
}

// Tiles of a product: of 256 rows by a pair of CTAs where those keep most SMs busy (4,096 square bf16 1,491 us, with tiles of
// 128 x 128 1,990; but 1,001 square Gram matrices, 10 tiles of 256, by 72 of 128 x 64), else of 128 x 128 (one product), else of
// 128 x 64 (five layers of 256 161 us in 128 x 128 when that was written, 118 in 128 x 64)
template <int MODE, bool TALL, int NPROD>
bool launch_product(const Operand& left, const Operand& right, const Operand* in, const Operand& out, const NsArgs& a, int batch,
                    cudaStream_t st) {
  constexpr bool A_MN = MODE == GRAM && TALL, B_MN = A_MN || (MODE == APPLY && !TALL);
  constexpr int WIDE = NPROD == 1 ? 256 : 128;           // columns of a pair's tile
  auto tiles = [&](int m, int n) {
    const int64_t tm = (a.m + m - 1) / m, tn = (a.n + n - 1) / n;
    return (MODE == APPLY ? tm * tn : tm * (tm + 1) / 2 * (m / n)) * batch;
  };
  // (where a pair has less than two tiles of a short reduction to apply, smaller ones let one's epilogue run under the next one's
  // products: 5,000 x 800 225 -> 197 us, 800 x 5,000 220 -> 196, 600 x 8,000 250 -> 237, 4,100 x 1,001 207 -> 204, two of 2,048 x 1,024
  // 187 -> 184; but 2,048 square 233 -> 241, 2,800 460 to 505 -> 570, and 1,280 x 5,120 would still gain, 264 -> 258)
  const bool shallow = MODE == APPLY && NPROD == 1 && a.k <= 1024 && tiles(256, WIDE) < kNumSMs;
  const int kind = !shallow && tiles(256, WIDE) >= 60 && a.m > 128 && a.n > 128 ? 2
                   : NPROD == 1 && tiles(128, 128) >= 100 && a.n > 64 ? 1 : 0;
  // A long reduction of few tiles: one tile to a cluster, and shares that are worth the meeting, some 3 us: 12 stages of one
  // product or 5 of three (fp32 49 x 1,270 109 -> 100 us, bf16 4,100 x 1,001 228 -> 209; but fp32 256 x 512 in two 107 -> 111, bf16
  // 128 x 1,024 in four 70 -> 84).  Clusters of two, four and eight have room for 72, 32 and 16 on the GPU at a time (36 clusters of
  // four: 4,100 x 1,001 209 -> 306).  A stage of 128 columns takes 512 cycles, of 64 375; one product has either.
  const int stages = (a.k + kStep - 1) / kStep;
  auto shares = [&](int columns) {
    int p = 1;
    while (p < 8 && tiles(128, columns) <= (p == 1 ? 72 : p == 2 ? 32 : 16) && stages >= (NPROD == 1 ? 24 : 10) * p) p *= 2;
    return p;
  };
  const bool shared = MODE == GRAM && kind == 0;
  const int parts64 = shared ? shares(64) : 1, parts128 = shared && NPROD == 1 ? shares(128) : 1;
  const bool wide = parts128 > 1 && 512 * parts64 < 375 * parts128;
  const int outer = kind == 2 ? WIDE / 2 : kind == 1 || wide ? 128 : 64;
  Maps maps;
  if (!make_operand(&maps.a_hi, &maps.a_lo, left, batch, A_MN, kRows, NPROD > 1) ||
      !make_operand(&maps.b_hi, &maps.b_lo, right, batch, B_MN, outer, NPROD > 1) ||
      (in && !make_pieces(&maps.in_hi, &maps.in_lo, *in, batch)) || !make_pieces(&maps.out_hi, &maps.out_lo, out, batch))
    return false;
  if (kind == 2) return launch_tiles<2, WIDE, MODE, TALL, NPROD>(maps, a, batch, st);
  if (NPROD == 1 && kind == 1) return launch_tiles<1, NPROD == 1 ? 128 : 64, MODE, TALL, NPROD>(maps, a, batch, st);
  if constexpr (MODE == GRAM) {
    if constexpr (NPROD == 1) {
      if (wide) return launch_tiles<1, 128, MODE, TALL, NPROD, true>(maps, a, batch, st, parts128);
    }
    if (parts64 > 1) return launch_tiles<1, 64, MODE, TALL, NPROD, true>(maps, a, batch, st, parts64);
  }
  return launch_tiles<1, 64, MODE, TALL, NPROD>(maps, a, batch, st);
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
  s.dA = reinterpret_cast<float*>(take(size_t(batch) * s.ldm * 4));
  s.dB = reinterpret_cast<float*>(take(size_t(batch) * s.ldm * 4));
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
  const int64_t pieces = (int64_t(rows) * ((cols + 7) / 8) + 255) / 256;
  const int nb = int(pieces < kNormBlocks ? pieces : kNormBlocks), sb = int(pieces < 8 * kNumSMs ? pieces : 8 * kNumSMs);
  launch(k_ns_norm<T>, dim3(nb, batch), 256, 0, st, static_cast<const T*>(grad), ld, bs, rows, cols, s.partial, status);
  launch(k_ns_start<T>, dim3(sb, batch), 256, 0, st, static_cast<const T*>(grad), ld, bs, rows, cols, s.partial, nb, eps, xs,
         s.x[0], s.ldx);

  NsArgs gram = {};
  gram.m = gram.n = small;
  gram.k = large;
  gram.diag_stride = s.ldm;
  gram.descale = 1.f / (xs * xs);
  gram.gain = kGramScale / (xs * xs);
  gram.diag_in = s.dA;
  gram.diag_out = s.dA;
  gram.status = status;
  NsArgs poly = gram, apply = gram;
  poly.k = small;
  poly.descale = 1.f / (kGramScale * kGramScale);
  poly.gain = kC / kGramScale;
  poly.diag_out = s.dB;
  apply.m = rows;
  apply.n = cols;
  apply.k = small;
  apply.gain = 1.f / kGramScale;
  apply.unscale = 1.f / xs;
  apply.diag_in = s.dB;

  const Operand f = {s.f, small, small, s.ldm}, b = {s.b, small, small, s.ldm};
  for (int i = 0; i < steps; ++i) {
    const Operand x = {s.x[i & 1], rows, cols, s.ldx}, next = {s.x[(i + 1) & 1], rows, cols, s.ldx};
    if (i == steps - 1) {
      apply.user = out;
      apply.user_ld = out_ld;
      apply.user_batch = out_bs;
    }
    if (!launch_product<GRAM, TALL, NPROD>(x, x, nullptr, f, gram, batch, st) ||
        !launch_product<POLY, false, NPROD>(f, f, &f, b, poly, batch, st) ||
        !launch_product<APPLY, TALL, NPROD>(TALL ? x : b, TALL ? b : x, &x, next, apply, batch, st))
      return false;
  }
  return true;
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
