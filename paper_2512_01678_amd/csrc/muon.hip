// muon.hip -- updates orthogonalised by Newton-Schulz products, and the optimiser step that
// uses them.
//
// The update of a weight matrix is replaced by a near-orthogonal matrix with the same singular
// vectors.  With X (p x q, p <= q: transposed where rows > cols) scaled to |X|_F = 1, `steps` times
//   A = X X^T,  B = a + b A + c A A,  X <- B X,   a, b, c = 3.4445, -4.7750, 2.0315
// which applies the odd polynomial a t + b t^3 + c t^5 to every singular value.
//
// All products are C = P Q^T with both operands contiguous along the summed axis: X is kept in
// both orientations (X for X X^T; Y = X^T for Y' = Y B, B being symmetric), and the
// product that makes the next X writes both.  Only the tiles on and above the diagonal of A and B
// are computed; the others are their mirror images.
//
// Arithmetic: matrices here are bounded (singular values stay below 1.3), so a value v is held as
// two fp16 parts of v 2^s: hi the nearest fp16, lo the nearest fp16 of the rest.  Together they
// keep 22 bits and a sign, an error of at most 2^-23 relative, and a product is three matrix
// instructions, hi hi + hi lo + lo hi, accumulated in fp32 (lo lo is at most 2^-22 of the product
// and 2^-25 of it on average, which leaves the error of the whole at that of fp32 products): half
// of the six that the exact split into bf16 parts (bf16x6.h) takes at twice the speed of light.
// The scales (2^12 for X, 2^10 for A and B) keep hi of any element that matters out of fp16's
// subnormal range and the largest below 2^13.
#include <hip/hip_fp16.h>

#include <type_traits>

#include "internal.h"

namespace gcn {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kMats = 16;
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kScaleX = 4096.f;   // 2^12
constexpr float kScaleA = 1024.f;   // 2^10
constexpr float kGramScale = kScaleA / (kScaleX * kScaleX);
constexpr int kTile = 64;           // plane sizes are multiples of it
constexpr int kMaxPartials = 1024;
constexpr int64_t kMaxSum = 2048;    // columns summed in one fp32 accumulator of X X^T

// Kinds of launch.
enum { kSums, kPlanes, kGram, kJoin, kPoly, kUpdate, kKinds };

// One matrix.  Planes: hi, then lo.  Grouped by use in 64-byte lines: a kernel that follows another pays
// for every line of its arguments that it waits for.
struct alignas(64) Mat {
  _Float16* X;      // p x q
  _Float16* Y[2];   // q x p
  _Float16* A;      // p x p
  _Float16* B;      // p x p
  float* part;      // splits x tiles, where there are several splits
  int32_t pp, qp;   // short and long side, padded
  int32_t splits;   // X X^T: parts of the sum over q, of kchunk columns each
  int32_t kchunk;

  const float* g;   // gradient, or the matrix to orthogonalise
  float* m;         // momentum buffer, or NULL
  float* w;         // parameter, or NULL
  float* out;       // the orthogonalised matrix, or NULL
  int64_t ldg, ldo;
  int32_t rows, cols;
  float step;       // lr * scale
  int32_t n_partial;
  double* partial;  // sums of squares
  int32_t vec;      // g and m have rows without gaps, 16-byte aligned, a multiple of 4 elements
};

struct NsArgs {
  int32_t first[kKinds][kMats];  // first workgroup of each matrix in each kind of launch
  Mat mat[kMats];
  int32_t total[kKinds];
  int32_t count;
  float mu, omu, keep;  // momentum, 1 - momentum, 1 - lr * weight decay
  int32_t nesterov;
  int32_t last;         // the update writes the result instead of the planes
  int32_t flip;         // Y[flip] is read, Y[1 - flip] written
};

// The matrix that workgroup `block` of this kind of launch works on (unused places hold INT32_MAX).
__device__ __forceinline__ int find_mat(const NsArgs& a, int kind, int block) {
  int n = 0;
#pragma unroll
  for (int i = 1; i < kMats; ++i) n += block >= a.first[kind][i] ? 1 : 0;
  return n;
}

// A plane of R rows and K columns (multiples of 64) is stored in slabs of 8 columns, each R x 8 and
// contiguous: an operand of a matrix instruction (32 rows, 16 columns, 16 bytes a lane) is two runs of 512
// bytes in the order of the lanes, and what a workgroup reads falls on all channels of the L2, whatever
// the sizes (in row order, rows a power of two apart do not).
__device__ __forceinline__ int64_t place(int64_t R, int64_t r, int64_t k) { return ((k >> 3) * R + r) * 8 + (k & 7); }

__device__ __forceinline__ void split2(float v, _Float16& hi, _Float16& lo) {
  // v is one rounded value from here on: without this the compiler may fuse the product that makes it
  // with one conversion and not with the other, and near a tie hi and lo would belong to two values
  asm("" : "+v"(v));
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}

// The same of two values, as packed pairs, and back.
__device__ __forceinline__ void split_pair2(float a, float b, uint32_t& hi, uint32_t& lo) {
  asm("" : "+v"(a), "+v"(b));
  const f32x2 v = {a, b};
  const half2v h = __builtin_convertvector(v, half2v);
  const half2v r = __builtin_convertvector(v - __builtin_convertvector(h, f32x2), half2v);
  hi = __builtin_bit_cast(uint32_t, h);
  lo = __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ void split_quad(f32x4 v, u32x2& hi, u32x2& lo) {
  uint32_t h0, h1, l0, l1;
  split_pair2(v[0], v[1], h0, l0);
  split_pair2(v[2], v[3], h1, l1);
  hi = u32x2{h0, h1};
  lo = u32x2{l0, l1};
}
__device__ __forceinline__ void join_pair2(uint32_t hi, uint32_t lo, float& a, float& b) {
  const f32x2 h = __builtin_convertvector(__builtin_bit_cast(half2v, hi), f32x2);
  const f32x2 l = __builtin_convertvector(__builtin_bit_cast(half2v, lo), f32x2);
  a = h[0] + l[0];
  b = h[1] + l[1];
}
__device__ __forceinline__ half8 half8_of(u32x4 v) { return __builtin_bit_cast(half8, v); }

__device__ __forceinline__ float momentum_of(const NsArgs& a, float g, float m) { return a.mu * m + a.omu * g; }
// u: what is orthogonalised, from the gradient and the already updated momentum buffer.
__device__ __forceinline__ float update_of(const NsArgs& a, const Mat& t, float g, float m) {
  if (!t.m) return g;
  return a.nesterov ? a.omu * g + a.mu * m : m;
}

// Momentum, and the sum of squares of u in fp64 (an fp32 square overflows from 1.8e19 on and
// vanishes below 1e-23).
__global__ void __launch_bounds__(256) k_ns_sums(NsArgs a) {
  __shared__ double red[4];
  const int im = find_mat(a, kSums, blockIdx.x);
  const Mat& t = a.mat[im];
  const int b = blockIdx.x - a.first[kSums][im], tid = threadIdx.x;
  double s = 0.0;
  if (t.vec) {
    // rows without gaps, 16-byte aligned: four vectors a thread at a time
    const int64_t n4 = (int64_t)t.rows * t.cols / 4;
    const f32x4* g4 = reinterpret_cast<const f32x4*>(t.g);
    f32x4* m4 = reinterpret_cast<f32x4*>(t.m);
    for (int64_t i0 = (int64_t)b * 1024; i0 < n4; i0 += (int64_t)t.n_partial * 1024) {
      f32x4 g[4] = {}, m[4] = {};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i0 + k * 256 + tid < n4) g[k] = g4[i0 + k * 256 + tid];
      if (t.m) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i0 + k * 256 + tid < n4) m[k] = m4[i0 + k * 256 + tid];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int e = 0; e < 4; ++e) m[k][e] = momentum_of(a, g[k][e], m[k][e]);
          if (i0 + k * 256 + tid < n4) m4[i0 + k * 256 + tid] = m[k];
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double u = (double)update_of(a, t, g[k][e], m[k][e]);
          s += u * u;
        }
    }
  } else {
    int log = 0;
    while (log < 8 && (1 << log) < t.cols) ++log;
    const int tx = tid & ((1 << log) - 1), ty = tid >> log, ry = 256 >> log;
    for (int64_t r = (int64_t)b * ry + ty; r < t.rows; r += (int64_t)t.n_partial * ry)
      for (int64_t c0 = tx; c0 < t.cols; c0 += (int64_t)4 << log) {
        float g[4] = {}, m[4] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t c = c0 + ((int64_t)k << log);
          if (c < t.cols) {
            g[k] = t.g[r * t.ldg + c];
            if (t.m) m[k] = t.m[r * t.cols + c];
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t c = c0 + ((int64_t)k << log);
          if (t.m && c < t.cols) {
            m[k] = momentum_of(a, g[k], m[k]);
            t.m[r * t.cols + c] = m[k];
          }
          const double u = (double)update_of(a, t, g[k], m[k]);
          s += u * u;
        }
      }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) t.partial[b] = red[0] + red[1] + red[2] + red[3];
}

// 2^12 / |u|_F from the sum of squares: 0 where u = 0, NaN where it is not finite.
__device__ __forceinline__ double scale_of(double s) {
  return s > 0.0 ? (double)kScaleX / sqrt(s) : (s == s ? 0.0 : s);
}

// X = u / |u|_F (0 where u = 0) in both orientations, zero in the padding; a 64 x 64 tile of X
// per workgroup, turned through LDS.
__global__ void __launch_bounds__(256) k_ns_planes(NsArgs a) {
  __shared__ float tile[kTile][kTile + 1];
  __shared__ double red[4];
  const int im = find_mat(a, kPlanes, blockIdx.x);
  const Mat& t = a.mat[im];
  const int b = blockIdx.x - a.first[kPlanes][im];
  const int tid = threadIdx.x;
  const int nq = t.qp / kTile;
  const int i0 = (b / nq) * kTile, j0 = (b % nq) * kTile;  // place in X (p x q)
  const bool turned = t.rows > t.cols;                     // u is q x p
  const int r0 = turned ? j0 : i0, c0 = turned ? i0 : j0;  // place in u
  float g[16], m[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int64_t r = r0 + k * 4 + tid / kTile, c = c0 + tid % kTile;
    const bool in = r < t.rows && c < t.cols;
    g[k] = in ? t.g[r * t.ldg + c] : 0.f;
    m[k] = in && t.m ? t.m[r * t.cols + c] : 0.f;
  }
  double s = 0.0;
  for (int k = tid; k < t.n_partial; k += 256) s += t.partial[k];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  const double inv = scale_of(red[0] + red[1] + red[2] + red[3]);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int64_t r = r0 + k * 4 + tid / kTile, c = c0 + tid % kTile;
    const bool in = r < t.rows && c < t.cols;
    tile[k * 4 + tid / kTile][tid % kTile] = in ? (float)((double)update_of(a, t, g[k], m[k]) * inv) : 0.f;
  }
  __syncthreads();
  // 16 bytes (8 columns) a lane, 64 rows of a slab a wavefront
  const int64_t plane = (int64_t)t.pp * t.qp;
  const int x = tid % 64;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int y = (tid / 64 + 4 * k) * 8;
    half8 xh, xl, yh, yl;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u0 = tile[x][y + e], u1 = tile[y + e][x];
      _Float16 hi, lo;
      split2(turned ? u1 : u0, hi, lo);  // X(i0 + x, j0 + y + e)
      xh[e] = hi;
      xl[e] = lo;
      split2(turned ? u0 : u1, hi, lo);  // Y(j0 + x, i0 + y + e)
      yh[e] = hi;
      yl[e] = lo;
    }
    const int64_t ax = place(t.pp, i0 + x, j0 + y), ay = place(t.qp, j0 + x, i0 + y);
    *reinterpret_cast<half8*>(t.X + ax) = xh;
    *reinterpret_cast<half8*>(t.X + plane + ax) = xl;
    *reinterpret_cast<half8*>(t.Y[0] + ay) = yh;
    *reinterpret_cast<half8*>(t.Y[0] + plane + ay) = yl;
  }
}

// A 4 x 4 block turned between the four lanes of a quad: lane i gives column i (rows 0 .. 3) and gets
// row i (columns 0 .. 3), or the other way round.
__device__ __forceinline__ half4 turn4(half4 v) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  const u2 a = __builtin_bit_cast(u2, v);
  const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
  // pairs of columns: the even lane keeps rows 0 and 2, the odd one rows 1 and 3
  const uint32_t sel = odd ? 0x03020706u : 0x05040100u;
  const uint32_t x0 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a[0], 0xB1, 0xF, 0xF, false);
  const uint32_t x1 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a[1], 0xB1, 0xF, 0xF, false);
  const uint32_t p0 = __builtin_amdgcn_perm(x0, a[0], sel), p1 = __builtin_amdgcn_perm(x1, a[1], sel);
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(high ? p0 : p1), 0x4E, 0xF, 0xF, false);
  const u2 r = {high ? y : p0, high ? p1 : y};
  return __builtin_bit_cast(half4, r);
}

// A 32 x 32 sub-tile of the planes of S (R x K), zero outside: rows row + 8 q + 0 .. 3 of column col a lane.
// A lane reads four columns of one row.
struct SubTile {
  half4 hi[4], lo[4];
  template <bool WHOLE>  // all of it is inside
  __device__ __forceinline__ void load(const _Float16* S, int64_t R, int64_t K, int64_t row, int64_t col) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t r = row + 8 * q + threadIdx.x % 4, c = col - threadIdx.x % 4;
      hi[q] = lo[q] = half4{};
      if (WHOLE || (r < R && c < K)) {
        hi[q] = *reinterpret_cast<const half4*>(S + place(R, r, c));
        lo[q] = *reinterpret_cast<const half4*>(S + R * K + place(R, r, c));
      }
    }
  }
  // acc += f (hi + lo)
  __device__ __forceinline__ void add_to(f32x16& acc, float f) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const half4 h = turn4(hi[q]), l = turn4(lo[q]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[4 * q + e] += f * ((float)h[e] + (float)l[e]);
    }
  }
};

// Issue order of the instructions around it: READS LDS reads, WRITES LDS writes and LOADS loads spread
// over MATS matrix instructions, the reads over the first two thirds (the next ones need them).  A burst of
// LDS reads would leave the matrix core idle until the LDS has served all four wavefronts.
template <int MATS, int READS, int WRITES, int LOADS, int I = 0>
__device__ __forceinline__ void interleave() {
  __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
  constexpr int early = (2 * MATS + 2) / 3;
  constexpr int r = I < early ? (I + 1) * READS / early - I * READS / early : 0;
  constexpr int w = (I + 1) * WRITES / MATS - I * WRITES / MATS;
  constexpr int l = (I + 1) * LOADS / MATS - I * LOADS / MATS;
  if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
  if constexpr (w > 0) __builtin_amdgcn_sched_group_barrier(0x200, w, 0);
  if constexpr (l > 0) __builtin_amdgcn_sched_group_barrier(0x020, l, 0);
  if constexpr (I + 1 < MATS) interleave<MATS, READS, WRITES, LOADS, I + 1>();
}

// A tile of C = P Q^T over columns [k0, k1) (multiples of 64): rows r0 .. r0 + BM - 1 of P (which has
// `rows_p`; places past them re-read the last) and c0 .. of Q, hi and lo planes of rows x K elements.
// 2 x 2 wavefronts, each TM x TN sub-tiles of 32 x 32.  The sum starts from what acc holds.  Two LDS
// buffers, one barrier per BK columns, and DEPTH of them on their way through registers: what a
// kernel reads was written by the one before, mostly on another XCD, so it comes from beyond the L2,
// and the matrix work on BK columns is shorter than that.
template <int BM, int BN, int BK, int DEPTH>
struct Product {
  static constexpr int NT = 256;
  static constexpr int TM = BM / 64, TN = BN / 64;
  static constexpr int kBuf = 2 * (BM + BN) * BK;  // halves of one buffer: P hi, P lo, Q hi, Q lo
  static constexpr int kPerA = 2 * BM * BK / 8 / NT, kPerB = 2 * BN * BK / 8 / NT;  // 16-byte chunks per thread
  static_assert(BK == 32 && BM * 4 % NT == 0 && BN * 4 % NT == 0, "whole chunks per thread and plane");
  static_assert(DEPTH == 1 || DEPTH == 2, "slabs on their way");

  f32x16 acc[TM][TN];

  __device__ __forceinline__ void run(const _Float16* P, int64_t r0, int64_t rows_p, const _Float16* Q, int64_t c0,
                                      int64_t rows_q, int64_t K, int64_t k0, int64_t k1, _Float16* lds) {
    const int tid = threadIdx.x, wave = tid / 64, l = tid % 64;
    const int wm = wave & 1, wn = wave >> 1, h = l / 32, l32 = l % 32;
    // This thread's chunks of a plane's four slabs: bytes from the tile's first row in the first slab.
    constexpr int kHalfA = kPerA / 2, kHalfB = kPerB / 2;
    uint32_t off_a[kHalfA], off_b[kHalfB];
#pragma unroll
    for (int i = 0; i < kHalfA; ++i) {
      const int c = tid + i * NT, rr = c % BM;
      off_a[i] = (uint32_t)((r0 + rr < rows_p ? rr : (int)(rows_p - 1 - r0)) + c / BM * (int)rows_p) * 16;
    }
#pragma unroll
    for (int i = 0; i < kHalfB; ++i) {
      const int c = tid + i * NT, rr = c % BN;
      off_b[i] = (uint32_t)((c0 + rr < rows_q ? rr : (int)(rows_q - 1 - c0)) + c / BN * (int)rows_q) * 16;
    }
    const int64_t plane_p = 2 * rows_p * K, plane_q = 2 * rows_q * K;  // bytes
    const char* src_p = reinterpret_cast<const char*>(P + place(rows_p, r0, k0));
    const char* src_q = reinterpret_cast<const char*>(Q + place(rows_q, c0, k0));
    const int ns = (int)((k1 - k0) / BK);
    int loaded = 0;
    half8 ra[DEPTH][kPerA], rb[DEPTH][kPerB];
    auto load = [&](half8* a, half8* b) {
#pragma unroll
      for (int i = 0; i < kPerA; ++i)
        a[i] = *reinterpret_cast<const half8*>(src_p + (i < kHalfA ? 0 : plane_p) + off_a[i % kHalfA]);
#pragma unroll
      for (int i = 0; i < kPerB; ++i)
        b[i] = *reinterpret_cast<const half8*>(src_q + (i < kHalfB ? 0 : plane_q) + off_b[i % kHalfB]);
      // past the end the last slabs are loaded again (and never multiplied): every pass of the loop then
      // has the same loads in flight, so that a wait counts them instead of draining them
      if (++loaded < ns) {
        src_p += 4 * 16 * rows_p;
        src_q += 4 * 16 * rows_q;
      }
    };
    const int dst = tid * 8;
    auto store_one = [&](_Float16* buf, const half8* a, const half8* b, int i) {
      if (i < kPerA)
        *reinterpret_cast<half8*>(buf + dst + i * NT * 8) = a[i];
      else
        *reinterpret_cast<half8*>(buf + 2 * BM * BK + dst + (i - kPerA) * NT * 8) = b[i - kPerA];
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      load(ra[d], rb[d]);
      __builtin_amdgcn_sched_barrier(0);  // in this order: the loop's waits count on it
    }
#pragma unroll
    for (int i = 0; i < kPerA + kPerB; ++i) store_one(lds, ra[0], rb[0], i);
    __builtin_amdgcn_sched_barrier(0);
    load(ra[0], rb[0]);
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    constexpr int KK = BK / 16, kWrites = kPerA + kPerB, kPer = (kWrites + KK - 2) / (KK - 1);
    constexpr int kMats = 3 * TM * TN, kReads = 2 * (TM + TN);
    Frags f[2];
    f[0].read(lds, 0, wm, wn, h, l32);
    __builtin_amdgcn_sched_barrier(0);
    // The next fragments are on their way while these are multiplied, the next slab's writes go between
    // the matrix instructions, and the slab's last fragments are multiplied behind the barrier, while the
    // first of the next slab are read.  d = s % DEPTH.
    auto slab = [&](int s, auto dd) {
      constexpr int next = (decltype(dd)::value + 1) % DEPTH;  // the registers that hold slab s + 1
      const _Float16* cur = lds + (s & 1) * kBuf;
      _Float16* other = lds + ((s + 1) & 1) * kBuf;
#pragma unroll
      for (int kk = 0; kk + 1 < KK; ++kk) {
        f[(kk + 1) & 1].read(cur, kk + 1, wm, wn, h, l32);
        multiply(f[kk & 1]);
#pragma unroll
        for (int i = kk * kPer; i < (kk + 1) * kPer && i < kWrites; ++i) store_one(other, ra[next], rb[next], i);
        interleave<kMats, kReads, kPer, 0>();
        __builtin_amdgcn_sched_barrier(0);
      }
      __syncthreads();
      f[0].read(other, 0, wm, wn, h, l32);
      multiply(f[(KK - 1) & 1]);
      load(ra[next], rb[next]);
      interleave<kMats, kReads, 0, kWrites>();
      __builtin_amdgcn_sched_barrier(0);
    };
    // whole rounds of DEPTH (no way out in between: at a way out the waits would have to allow for
    // every order of the loads), then the rest
    int s0 = 0;
    for (; s0 + DEPTH <= ns; s0 += DEPTH) {
      slab(s0, std::integral_constant<int, 0>{});
      if constexpr (DEPTH > 1) slab(s0 + 1, std::integral_constant<int, 1>{});
    }
    if constexpr (DEPTH > 1)
      if (s0 < ns) slab(s0, std::integral_constant<int, 0>{});
  }

  struct Frags {
    half8 ah[TM], al[TM], bh[TN], bl[TN];
    __device__ __forceinline__ void read(const _Float16* la, int kk, int wm, int wn, int h, int l32) {
      const _Float16* lb = la + 2 * BM * BK;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int o = ((kk * 2 + h) * BM + (wm * TM + i) * 32 + l32) * 8;
        ah[i] = *reinterpret_cast<const half8*>(la + o);
        al[i] = *reinterpret_cast<const half8*>(la + BM * BK + o);
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int o = ((kk * 2 + h) * BN + (wn * TN + j) * 32 + l32) * 8;
        bh[j] = *reinterpret_cast<const half8*>(lb + o);
        bl[j] = *reinterpret_cast<const half8*>(lb + BN * BK + o);
      }
    }
  };
  __device__ __forceinline__ void multiply(const Frags& f) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.al[i], f.bh[j], acc[i][j], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.ah[i], f.bl[j], acc[i][j], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.ah[i], f.bh[j], acc[i][j], 0, 0, 0);
  }

  // Sub-tile (i, j) of this wavefront: its first row in the tile (a lane holds rows row + 8 q + 0 .. 3,
  // q = 0 .. 3) and this lane's column.
  static __device__ __forceinline__ int row_of(int i) {
    return ((threadIdx.x / 64 & 1) * TM + i) * 32 + 4 * (threadIdx.x % 64 / 32);
  }
  static __device__ __forceinline__ int col_of(int j) { return ((threadIdx.x / 128) * TN + j) * 32 + threadIdx.x % 32; }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  }
  // acc = f (hi + lo) of the matrix S (R x K planes) at this tile, before the sum.
  __device__ __forceinline__ void start(float f, const _Float16* S, int64_t R, int64_t K, int64_t r0, int64_t c0) {
    clear();
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        SubTile t;
        t.template load<false>(S, R, K, r0 + row_of(i), c0 + col_of(j));
        t.add_to(acc[i][j], f);
      }
  }

  // f(row, col, v): four consecutive rows row .. row + 3 of column col of the tile.
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          f(row_of(i) + 8 * q, col_of(j), v);
        }
  }
};

// A 64 x 64 tile whose sum is shared out over the wavefronts: each takes a quarter of the columns and
// computes the whole tile, 2 x 2 sub-tiles, from operands that it loads straight into registers, DEPTH
// slabs ahead; nothing goes through LDS until the four sums are joined, each wavefront taking one
// sub-tile.  Staged through LDS, a 64 x 64 tile reads 16 KB of it for 12 matrix instructions a wavefront
// instead of 8 KB of memory, with a barrier for each slab, and its latency is the longer one.
template <int DEPTH>
struct ProductK {
  static constexpr int TM = 1, TN = 1;
  static constexpr int kBuf = 4 * 3 * 64 * 16 * 2 / 2;  // halves; twice that: 4 x 3 sub-tiles of fp32
  f32x16 acc[1][1];

  static __device__ __forceinline__ int row_of(int) {
    return (threadIdx.x / 64 & 1) * 32 + 4 * (threadIdx.x % 64 / 32);
  }
  static __device__ __forceinline__ int col_of(int) { return threadIdx.x / 128 * 32 + threadIdx.x % 32; }

  // What the sum starts from is loaded behind the first operands and added at the end.
  const _Float16* from = nullptr;
  int64_t from_r, from_k;
  float factor;
  __device__ __forceinline__ void clear() {}
  __device__ __forceinline__ void start(float f, const _Float16* S, int64_t R, int64_t K, int64_t, int64_t) {
    from = S;
    from_r = R;
    from_k = K;
    factor = f;
  }

  struct Operands {
    half8 ph[2], pl[2], qh[2], ql[2];
  };

  __device__ __forceinline__ void run(const _Float16* P, int64_t r0, int64_t rows_p, const _Float16* Q, int64_t c0,
                                      int64_t rows_q, int64_t K, int64_t k0, int64_t k1, _Float16* lds) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64;
    const int n = (int)((k1 - k0) / 64);  // slabs of this wavefront
    const int64_t kw = k0 + (int64_t)wave * n * 16;
    const uint32_t off_p = (uint32_t)(l % 32 + l / 32 * (int)rows_p) * 16;
    const uint32_t off_q = (uint32_t)(l % 32 + l / 32 * (int)rows_q) * 16;
    const int64_t plane_p = 2 * rows_p * K, plane_q = 2 * rows_q * K;  // bytes
    const char* src_p = reinterpret_cast<const char*>(P + place(rows_p, r0, kw));
    const char* src_q = reinterpret_cast<const char*>(Q + place(rows_q, c0, kw));
    int loaded = 0;
    Operands o[DEPTH];
    auto load = [&](Operands& x) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x.ph[i] = *reinterpret_cast<const half8*>(src_p + off_p + i * 512);
        x.pl[i] = *reinterpret_cast<const half8*>(src_p + plane_p + off_p + i * 512);
        x.qh[i] = *reinterpret_cast<const half8*>(src_q + off_q + i * 512);
        x.ql[i] = *reinterpret_cast<const half8*>(src_q + plane_q + off_q + i * 512);
      }
      // past the end the last slab is loaded again (see Product)
      if (++loaded < n) {
        src_p += 32 * rows_p;
        src_q += 32 * rows_q;
      }
    };
    f32x16 sum[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[i][j][r] = 0.f;
    auto multiply = [&](const Operands& x) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x.pl[i], x.qh[j], sum[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x.ph[i], x.ql[j], sum[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x.ph[i], x.qh[j], sum[i][j], 0, 0, 0);
    };
#pragma unroll
    for (int d = 0; d + 1 < DEPTH; ++d) {
      load(o[d]);
      __builtin_amdgcn_sched_barrier(0);  // in this order: the loop's waits count on it
    }
    SubTile first;
    if (from) first.template load<true>(from, from_r, from_k, r0 + row_of(0), c0 + col_of(0));
    __builtin_amdgcn_sched_barrier(0);
    // the loads go between the matrix instructions: a burst of them would take the four wavefronts, which
    // keep step, longer to issue than the matrix work itself
    int s = 0;
    for (; s + DEPTH <= n; s += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        multiply(o[d]);
        load(o[(d + DEPTH - 1) % DEPTH]);
        interleave<12, 0, 0, 8>();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (s < n) {
      multiply(o[0]);
      load(o[DEPTH - 1]);
      interleave<12, 0, 0, 8>();
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int d = 1; d + 1 < DEPTH; ++d)
      if (s + d < n) multiply(o[d]);
    // sub-tile (i, j) belongs to wavefront i + 2 j: the others leave theirs in LDS, and it adds the four
    // in order
    f32x4* box = reinterpret_cast<f32x4*>(lds);
#pragma unroll
    for (int own = 0; own < 4; ++own)
      if (own != wave) {
        const int slot = own * 3 + (wave < own ? wave : wave - 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x16& t = sum[own & 1][own >> 1];
          box[(slot * 4 + q) * 64 + l] = f32x4{t[4 * q], t[4 * q + 1], t[4 * q + 2], t[4 * q + 3]};
        }
      }
    __syncthreads();
    // element by element: a choice between whole sub-tiles would put them in memory
    f32x16 mine;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float lo = wave & 1 ? sum[1][0][r] : sum[0][0][r], hi = wave & 1 ? sum[1][1][r] : sum[0][1][r];
      mine[r] = wave & 2 ? hi : lo;
    }
    f32x16 total;
#pragma unroll
    for (int r = 0; r < 16; ++r) total[r] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w == wave) {
#pragma unroll
        for (int r = 0; r < 16; ++r) total[r] += mine[r];
      } else {
        const int slot = wave * 3 + (w < wave ? w : w - 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 t = box[(slot * 4 + q) * 64 + l];
#pragma unroll
          for (int e = 0; e < 4; ++e) total[4 * q + e] += t[e];
        }
      }
    }
    if (from) first.add_to(total, factor);
    acc[0][0] = total;
  }

  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float v[4] = {acc[0][0][4 * q], acc[0][0][4 * q + 1], acc[0][0][4 * q + 2], acc[0][0][4 * q + 3]};
      f(row_of(0) + 8 * q, col_of(0), v);
    }
  }
};

// The product of a tile of side T.
template <int T>
struct ProductOf {
  using type = Product<T, T, 32, T == 128 ? 2 : 1>;
};
template <>
struct ProductOf<64> {
  using type = ProductK<4>;
};

// Four values down a column, rows row .. row + 3, into the planes of M (R x K), four columns of one row
// a lane, and turned into those of T (K x R), where a lane's own four are contiguous; T may be NULL.
__device__ __forceinline__ void write_planes(const float v[4], _Float16* M, _Float16* T, int64_t R, int64_t K,
                                             int64_t row, int64_t col) {
  half4 hi, lo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    _Float16 a, b;
    split2(v[e], a, b);
    hi[e] = a;
    lo[e] = b;
  }
  const int64_t m = place(R, row + threadIdx.x % 4, col - threadIdx.x % 4), plane = R * K;
  *reinterpret_cast<half4*>(M + m) = turn4(hi);
  *reinterpret_cast<half4*>(M + plane + m) = turn4(lo);
  if (T) {
    const int64_t t = place(K, col, row);
    *reinterpret_cast<half4*>(T + t) = hi;
    *reinterpret_cast<half4*>(T + plane + t) = lo;
  }
}

// Workgroups go to the 8 XCDs in turn, and each XCD has an L2 of its own, which starts empty (the kernel
// before wrote from all of them): a run of consecutive tiles to each, so that it reads few panels.
// Returns the unit that this workgroup takes, or total and more where there is none left.
__device__ __forceinline__ int xcd_unit(int total) {
  const int per = (total + 7) / 8;
  const int u = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  return (int)(blockIdx.x >> 3) < per ? u : total;
}

constexpr int kBand = 4;  // tile rows that are walked together, column by column

// Tile u of m x n tiles.
__device__ __forceinline__ void band_tile(int u, int m, int n, int& i, int& j) {
  const int band = u / (kBand * n);
  u -= band * kBand * n;
  const int h = m - band * kBand < kBand ? m - band * kBand : kBand;
  j = u / h;
  i = band * kBand + u - j * h;
}

// Tile u, i <= j, of the upper triangle of n x n tiles.
__device__ __forceinline__ void upper_tile(int u, int n, int& i, int& j) {
  int b = 0;  // first row of the band
  for (;; b += kBand) {
    const int h = n - b < kBand ? n - b : kBand;
    const int in_band = h * (h + 1) / 2 + h * (n - b - h);
    if (u < in_band || b + kBand >= n) break;
    u -= in_band;
  }
  const int h = n - b < kBand ? n - b : kBand;
  int c = 0;  // column from b on: 1, 2, .. h tiles, then h each
  while (c < h && u > c) u -= ++c;
  if (c < h) {
    i = b + u;
    j = b + c;
  } else {
    i = b + u % h;
    j = b + h + u / h;
  }
}

// One value (or four down a column) of A or B, and its mirror image where the tile is above the diagonal.
__device__ __forceinline__ void write_sym(const Mat& t, _Float16* out, const float v[4], int64_t row, int64_t col,
                                          bool diagonal) {
  // a tile on the diagonal is written as it was computed: its two halves may differ in the last bit
  write_planes(v, out, diagonal ? nullptr : out, t.pp, t.pp, row, col);
}

// A = X X^T (SQUARE = false; where the sum is split, this split's part of it), or B = a + b A + c A A.
template <int T, bool SQUARE>
__global__ void __launch_bounds__(256) k_ns_sym(NsArgs a) {
  using Prod = typename ProductOf<T>::type;
  __shared__ __attribute__((aligned(16))) _Float16 lds[2 * Prod::kBuf];
  const int kind = SQUARE ? kPoly : kGram;
  const int unit = xcd_unit(a.total[kind]);
  if (unit >= a.total[kind]) return;
  const int im = find_mat(a, kind, unit);
  const Mat& t = a.mat[im];
  const int n = (t.pp + T - 1) / T, b = unit - a.first[kind][im], tiles = n * (n + 1) / 2;
  int i, j;
  upper_tile(b % tiles, n, i, j);
  const int64_t r0 = (int64_t)i * T, c0 = (int64_t)j * T;
  Prod prod;
  if (SQUARE) {
    prod.start(kNsB / kNsC * kScaleA, t.A, t.pp, t.pp, r0, c0);
    prod.run(t.A, r0, t.pp, t.A, c0, t.pp, t.pp, 0, t.pp, lds);
  } else {
    prod.clear();
    const int64_t z = b / tiles, k0 = z * t.kchunk, k1 = k0 + t.kchunk < t.qp ? k0 + t.kchunk : t.qp;
    prod.run(t.X, r0, t.pp, t.X, c0, t.pp, t.qp, k0, k1, lds);
    if (t.splits > 1) {
      // as the registers hold it: k_ns_join reads it back with the same lanes
      f32x4* part = reinterpret_cast<f32x4*>(t.part) + ((int64_t)z * tiles + b % tiles) * (T * T / 4) + threadIdx.x;
#pragma unroll
      for (int u = 0; u < Prod::TM; ++u)
#pragma unroll
        for (int v = 0; v < Prod::TN; ++v)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            part[((u * Prod::TN + v) * 4 + q) * 256] = f32x4{prod.acc[u][v][4 * q], prod.acc[u][v][4 * q + 1],
                                                             prod.acc[u][v][4 * q + 2], prod.acc[u][v][4 * q + 3]};
      return;
    }
  }
  prod.each([&](int row, int col, const float acc[4]) {
    if (T > kTile && (r0 + row >= t.pp || c0 + col >= t.pp)) return;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = acc[e] * (SQUARE ? kNsC / kScaleA : kGramScale);
      if (SQUARE && i == j && row + e == col) v[e] += kNsA * kScaleA;
    }
    write_sym(t, SQUARE ? t.B : t.A, v, r0 + row, c0 + col, i == j);
  });
}

// A from the parts of a split sum, added in order; 64 x 64 of a tile (one sub-tile of each wavefront) a
// workgroup.
template <int T>
__global__ void __launch_bounds__(256) k_ns_join(NsArgs a) {
  using Prod = typename ProductOf<T>::type;
  constexpr int kSub = Prod::TM * Prod::TN;
  const int im = find_mat(a, kJoin, blockIdx.x);
  const Mat& t = a.mat[im];
  const int n = (t.pp + T - 1) / T, tiles = n * (n + 1) / 2;
  const int b = (blockIdx.x - a.first[kJoin][im]) / kSub, sub = (blockIdx.x - a.first[kJoin][im]) % kSub;
  int i, j;
  upper_tile(b, n, i, j);
  const f32x4* part = reinterpret_cast<const f32x4*>(t.part) + (int64_t)b * (T * T / 4) + sub * 4 * 256 + threadIdx.x;
  f32x4 v[4] = {};
  for (int z = 0; z < t.splits; ++z)
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += part[(int64_t)z * tiles * (T * T / 4) + q * 256];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float w[4] = {v[q][0] * kGramScale, v[q][1] * kGramScale, v[q][2] * kGramScale, v[q][3] * kGramScale};
    const int64_t row = (int64_t)i * T + Prod::row_of(sub / Prod::TN) + 8 * q, col = (int64_t)j * T + Prod::col_of(sub % Prod::TN);
    if (T == kTile || (row < t.pp && col < t.pp)) write_sym(t, t.A, w, row, col, i == j);
  }
}

// Y' = Y B, written in both orientations, or in the last step as the result.
template <int T>
__global__ void __launch_bounds__(256) k_ns_update(NsArgs a) {
  using Prod = typename ProductOf<T>::type;
  __shared__ __attribute__((aligned(16))) _Float16 lds[2 * Prod::kBuf];
  const int unit = xcd_unit(a.total[kUpdate]);
  if (unit >= a.total[kUpdate]) return;
  const int im = find_mat(a, kUpdate, unit);
  const Mat& t = a.mat[im];
  int ti, tj;
  band_tile(unit - a.first[kUpdate][im], (t.qp + T - 1) / T, (t.pp + T - 1) / T, ti, tj);
  const int64_t r0 = (int64_t)ti * T, c0 = (int64_t)tj * T;
  const _Float16* Y = t.Y[a.flip];
  Prod prod;
  const bool turned = t.rows > t.cols;
  // the result goes to out(q, p) of pitches (sq, sp)
  const int64_t nq = turned ? t.rows : t.cols, np = turned ? t.cols : t.rows;
  float* out = t.w ? t.w : t.out;
  const int64_t ldo = t.w ? t.cols : t.ldo, sq = turned ? ldo : 1, sp = turned ? 1 : ldo;
  // four consecutive q of a lane are one vector where the result's rows run along q and are aligned
  const bool vec = sq == 1 && ldo % 4 == 0 && nq % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0;
  auto weights = [&](int i, int j, float old[16]) {
    const int64_t q0 = r0 + Prod::row_of(i), p = c0 + Prod::col_of(j);
    if (vec) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f32x4 v{};
        if (q0 + 8 * e < nq && p < np) v = *reinterpret_cast<const f32x4*>(out + p * sp + q0 + 8 * e);
#pragma unroll
        for (int k = 0; k < 4; ++k) old[4 * e + k] = v[k];
      }
      return;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t q = q0 + 8 * (e / 4) + e % 4;
      old[e] = q < nq && p < np ? out[q * sq + p * sp] : 0.f;
    }
  };
  float old[16] = {};
  if (T == kTile && a.last && t.w) weights(0, 0, old);
  prod.clear();
  prod.run(Y, r0, t.qp, t.B, c0, t.pp, t.pp, 0, t.pp, lds);
  if (!a.last) {
    prod.each([&](int row, int col, const float acc[4]) {
      if (T > kTile && (r0 + row >= t.qp || c0 + col >= t.pp)) return;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[e] * (1.f / kScaleA);
      write_planes(v, t.Y[1 - a.flip], t.X, t.qp, t.pp, r0 + row, c0 + col);
    });
    return;
  }
  const float scale = (t.w ? -t.step : 1.f) / (kScaleA * kScaleX);
#pragma unroll
  for (int i = 0; i < Prod::TM; ++i)
#pragma unroll
    for (int j = 0; j < Prod::TN; ++j) {
      const int64_t q0 = r0 + Prod::row_of(i), p = c0 + Prod::col_of(j);
      if (T > kTile && t.w) weights(i, j, old);
      if (vec) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x4 v;
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = a.keep * old[4 * e + k] + prod.acc[i][j][4 * e + k] * scale;
          if (q0 + 8 * e < nq && p < np) *reinterpret_cast<f32x4*>(out + p * sp + q0 + 8 * e) = v;
        }
        continue;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t q = q0 + 8 * (e / 4) + e % 4;
        if (q < nq && p < np) out[q * sq + p * sp] = a.keep * old[e] + prod.acc[i][j][e] * scale;
      }
    }
}

// A whole matrix in one workgroup, all steps: p <= 32 PT and q <= 256 NS.  The strips of 32 rows of Y are
// dealt out to the 8 wavefronts, NS each, and stay in registers, as the matrix core leaves them: lane l
// holds column l % 32 of each 32 x 32 sub-tile, and in its two half8 rows 8 (j / 4) + 4 (l / 32) + j % 4
// and 16 more.  Y^T Y sums over the rows, in whatever order both operands agree on, so those registers
// are its operands as they are; only Y B needs a strip turned, through LDS.  What bounds it is the chain
// of short products and the barriers between them: 1.4 to 8 us a step where the launches above take 14 to 20
// (in all, 5 steps: 16 x 7 13 us instead of 82, 1,433 x 16 51 instead of 114, 60 x 700 75 instead of 108).
//
// Rows row .. row + 3 of column col of a symmetric matrix in LDS, as four columns of row col, and (both) where they
// belong too.
template <int P, int PITCH>
__device__ __forceinline__ void write_both(_Float16 (&m)[2][P][PITCH], u32x2 hi, u32x2 lo, int row, int col, bool both) {
  *reinterpret_cast<u32x2*>(&m[0][col][row]) = hi;
  *reinterpret_cast<u32x2*>(&m[1][col][row]) = lo;
  if (both) {
    const int e = threadIdx.x % 4;
    *reinterpret_cast<half4*>(&m[0][row + e][col - e]) = turn4(__builtin_bit_cast(half4, hi));
    *reinterpret_cast<half4*>(&m[1][row + e][col - e]) = turn4(__builtin_bit_cast(half4, lo));
  }
}

template <int PT, int NS>
__global__ void __launch_bounds__(512) k_ns_small(NsArgs a, int steps) {
  constexpr int W = 8, P = 32 * PT, kPitch = P + 8;
  constexpr int kTiles = PT * (PT + 1) / 2;
  // sums of Y^T Y by wavefront (fp32), and later the turned strips, share one place
  constexpr int kSumBytes = W * kTiles * 1024 * 4, kTurns = PT == 1 ? 2 : 1, kTurnBytes = W * kTurns * 2 * 32 * kPitch * 2;
  __shared__ __attribute__((aligned(16))) char box[kSumBytes > kTurnBytes ? kSumBytes : kTurnBytes];
  __shared__ __attribute__((aligned(16))) _Float16 la[2][P][kPitch];  // A: hi, lo
  __shared__ __attribute__((aligned(16))) _Float16 lb[2][P][kPitch];  // B
  __shared__ double red[W];
  const Mat& t = a.mat[blockIdx.x];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l = tid % 64, h = l / 32, l32 = l % 32;
  const bool turned = t.rows > t.cols;
  const int np = turned ? t.cols : t.rows, nq = turned ? t.rows : t.cols;
  // places in bytes, of 32 bits (small_form sees to it)
  const uint32_t sp = turned ? 4 : 4 * (uint32_t)t.ldg, sq = turned ? 4 * (uint32_t)t.ldg : 4;  // of g(q, p)
  const uint32_t mp = turned ? 4 : 4 * (uint32_t)t.cols, mq = turned ? 4 * (uint32_t)t.cols : 4;
  auto at = [](auto* base, uint32_t off) {
    using C = std::conditional_t<std::is_const_v<std::remove_pointer_t<decltype(base)>>, const char, char>;
    return reinterpret_cast<decltype(base)>(reinterpret_cast<C*>(base) + off);
  };
  const int strips = (nq + 31) / 32;

  // u, its sum of squares and the new momentum
  float u[NS][PT][16];
  double s = 0.0;
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int p = i * 32 + l32, q0 = (n * W + wave) * 32 + 4 * h;
      float g[16], m[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int q = q0 + 8 * (r / 4) + r % 4;
        const bool in = p < np && q < nq;
        g[r] = in ? *at(t.g, q * sq + p * sp) : 0.f;
        m[r] = in && t.m ? *at(t.m, q * mq + p * mp) : 0.f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int q = q0 + 8 * (r / 4) + r % 4;
        if (t.m) {
          m[r] = momentum_of(a, g[r], m[r]);
          if (p < np && q < nq) *at(t.m, q * mq + p * mp) = m[r];
        }
        u[n][i][r] = update_of(a, t, g[r], m[r]);
        s += (double)u[n][i][r] * (double)u[n][i][r];
      }
      // two sub-tiles' loads in flight: all of them would not fit the registers
      if ((n * PT + i) % 2 == 1) __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (l == 0) red[wave] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < W; ++w) s += red[w];
  const double inv = scale_of(s);
  // the lane's number afresh: places and conditions computed from it above would otherwise be kept, in
  // registers, until they are used again
  int l1 = l;
  asm volatile("" : "+v"(l1));
  // pairs of fp16: left as 16-bit values, the compiler would give each a register
  u32x4 yh[NS][PT][2], yl[NS][PT][2];
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int i = 0; i < PT; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const int p = i * 32 + l1 % 32, q = (n * W + wave) * 32 + 4 * (l1 / 32) + 8 * (r / 4) + r % 4;
        uint32_t hi, lo;
        split_pair2(p < np && q < nq ? (float)((double)u[n][i][r] * inv) : 0.f,
                    p < np && q + 1 < nq ? (float)((double)u[n][i][r + 1] * inv) : 0.f, hi, lo);
        yh[n][i][r / 8][r % 8 / 2] = hi;
        yl[n][i][r / 8][r % 8 / 2] = lo;
        if (r == 14) __builtin_amdgcn_sched_barrier(0);
      }

  for (int step = 0; step < steps; ++step) {
    // A = Y^T Y: this wavefront's strips, then the sum over the wavefronts.  The three kinds of part
    // products go to accumulators of their own where there is one sub-tile only (a chain on one would wait for itself).
    f32x4* sums = reinterpret_cast<f32x4*>(box);
    {
      constexpr int kAcc = PT == 1 ? 3 : kTiles;
      f32x16 acc[kAcc];
#pragma unroll
      for (int k = 0; k < kAcc; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[k][r] = 0.f;
#pragma unroll
      for (int n = 0; n < NS; ++n)
        if (n * W + wave < strips)
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int part = 0; part < 3; ++part)
#pragma unroll
              for (int i = 0; i < PT; ++i)
#pragma unroll
                for (int j = i; j < PT; ++j) {
                  const int k = PT == 1 ? part : i + j;  // (0, 0), (0, 1), (1, 1)
                  acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(half8_of(part == 0 ? yl[n][i][g] : yh[n][i][g]),
                                                                  half8_of(part == 1 ? yl[n][j][g] : yh[n][j][g]), acc[k],
                                                                  0, 0, 0);
                }
      if constexpr (PT == 1) acc[0] = acc[0] + acc[1] + acc[2];
#pragma unroll
      for (int k = 0; k < kTiles; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          sums[((k * W + wave) * 4 + q) * 64 + l] = f32x4{acc[k][4 * q], acc[k][4 * q + 1], acc[k][4 * q + 2], acc[k][4 * q + 3]};
    }
    __syncthreads();
    // four rows of a column a thread; A is symmetric: they are written as four columns of a row
#pragma unroll
    for (int v = 0; v < (kTiles * 256 + 511) / 512; ++v) {
      const int u4 = v * 512 + tid, k = u4 / 256, q = u4 / 64 % 4;
      if (kTiles * 256 % 512 == 0 || k < kTiles) {
        f32x4 x{};
#pragma unroll
        for (int w = 0; w < W; ++w) x += sums[(k * W + w) * 256 + u4 % 256];
        const int row = 32 * (k / 2) + 8 * q + 4 * h, col = 32 * ((k + 1) / 2) + l32;
        u32x2 hi, lo;
        split_quad(x * kGramScale, hi, lo);
        write_both(la, hi, lo, row, col, k == 1);
      }
    }
    __syncthreads();
    // B = a + b A + c A A, a sub-tile on or above the diagonal a wavefront
    if (wave < kTiles) {
      const int i = wave / 2, j = (wave + 1) / 2;
      half4 h4[4], l4[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        h4[q] = *reinterpret_cast<const half4*>(&la[0][j * 32 + l32][i * 32 + 8 * q + 4 * h]);
        l4[q] = *reinterpret_cast<const half4*>(&la[1][j * 32 + l32][i * 32 + 8 * q + 4 * h]);
      }
      f32x16 acc[3];
#pragma unroll
      for (int part = 0; part < 3; ++part)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[part][r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < 2 * PT; ++kk) {
        const half8 ah = *reinterpret_cast<const half8*>(&la[0][i * 32 + l32][kk * 16 + h * 8]);
        const half8 al = *reinterpret_cast<const half8*>(&la[1][i * 32 + l32][kk * 16 + h * 8]);
        const half8 bh = *reinterpret_cast<const half8*>(&la[0][j * 32 + l32][kk * 16 + h * 8]);
        const half8 bl = *reinterpret_cast<const half8*>(&la[1][j * 32 + l32][kk * 16 + h * 8]);
        acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, acc[0], 0, 0, 0);
        acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, acc[1], 0, 0, 0);
        acc[2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, acc[2], 0, 0, 0);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = kNsB * ((float)h4[q][e] + (float)l4[q][e]) +
                 (acc[0][4 * q + e] + acc[1][4 * q + e] + acc[2][4 * q + e]) * (kNsC / kScaleA);
          if (i == j && 8 * q + 4 * h + e == l32) v[e] += kNsA * kScaleA;
        }
        u32x2 hi, lo;
        split_quad(v, hi, lo);
        write_both(lb, hi, lo, i * 32 + 8 * q + 4 * h, j * 32 + l32, i != j);
      }
    }
    __syncthreads();
    // Y <- Y B, strip by strip; the turned strip lies in this wavefront's own place
    half8 bh[2 * PT][PT], bl[2 * PT][PT];
#pragma unroll
    for (int kk = 0; kk < 2 * PT; ++kk)
#pragma unroll
      for (int j = 0; j < PT; ++j) {
        bh[kk][j] = *reinterpret_cast<const half8*>(&lb[0][j * 32 + l32][kk * 16 + h * 8]);
        bl[kk][j] = *reinterpret_cast<const half8*>(&lb[1][j * 32 + l32][kk * 16 + h * 8]);
      }
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (n * W + wave < strips) {
        _Float16* turn = reinterpret_cast<_Float16*>(box) + (wave * kTurns + n % kTurns) * 2 * 32 * kPitch;
#pragma unroll
        for (int i = 0; i < PT; ++i)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            // lane 4 k + e holds rows 8 q4 + 4 h .. of column 4 k + e and gets row + e of columns 4 k ..
            const u32x2 vh = {yh[n][i][q4 / 2][q4 % 2 * 2], yh[n][i][q4 / 2][q4 % 2 * 2 + 1]};
            const u32x2 vl = {yl[n][i][q4 / 2][q4 % 2 * 2], yl[n][i][q4 / 2][q4 % 2 * 2 + 1]};
            const int row = 8 * q4 + 4 * h + l % 4, col = i * 32 + l32 / 4 * 4;
            *reinterpret_cast<half4*>(turn + row * kPitch + col) = turn4(__builtin_bit_cast(half4, vh));
            *reinterpret_cast<half4*>(turn + (32 + row) * kPitch + col) = turn4(__builtin_bit_cast(half4, vl));
          }
        __builtin_amdgcn_wave_barrier();
        f32x16 acc[PT];
#pragma unroll
        for (int j = 0; j < PT; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 2 * PT; ++kk) {
          const half8 ah = *reinterpret_cast<const half8*>(turn + l32 * kPitch + kk * 16 + h * 8);
          const half8 al = *reinterpret_cast<const half8*>(turn + (32 + l32) * kPitch + kk * 16 + h * 8);
#pragma unroll
          for (int j = 0; j < PT; ++j) {
            acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh[kk][j], acc[j], 0, 0, 0);
            acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl[kk][j], acc[j], 0, 0, 0);
            acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh[kk][j], acc[j], 0, 0, 0);
          }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < PT; ++j)
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            uint32_t hi, lo;
            split_pair2(acc[j][r] * (1.f / kScaleA), acc[j][r + 1] * (1.f / kScaleA), hi, lo);
            yh[n][j][r / 8][r % 8 / 2] = hi;
            yl[n][j][r / 8][r % 8 / 2] = lo;
          }
        if (n % kTurns == kTurns - 1) __builtin_amdgcn_sched_barrier(0);
      }
    __syncthreads();  // the turned strips are done with before the next sums
  }

  float* out = t.w ? t.w : t.out;
  const uint32_t ldo = 4 * (uint32_t)(t.w ? t.cols : t.ldo), oq = turned ? ldo : 4, op = turned ? 4 : ldo;
  const float scale = (t.w ? -t.step : 1.f) / kScaleX;
  int l2 = l;
  asm volatile("" : "+v"(l2));
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int p = i * 32 + l2 % 32, q0 = (n * W + wave) * 32 + 4 * (l2 / 32);
      float old[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int q = q0 + 8 * (r / 4) + r % 4;
        old[r] = t.w && p < np && q < nq ? *at(out, q * oq + p * op) : 0.f;
      }
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const int q = q0 + 8 * (r / 4) + r % 4;
        float v0, v1;
        join_pair2(yh[n][i][r / 8][r % 8 / 2], yl[n][i][r / 8][r % 8 / 2], v0, v1);
        if (p < np && q < nq) *at(out, q * oq + p * op) = a.keep * old[r] + scale * v0;
        if (p < np && q + 1 < nq) *at(out, (q + 1) * oq + p * op) = a.keep * old[r + 1] + scale * v1;
      }
      if ((n * PT + i) % 2 == 1) __builtin_amdgcn_sched_barrier(0);
    }
}

// Tile sides of the three products, for all matrices of a call.
struct Tiles {
  int gram, poly, update;
};

int64_t upper_tiles(int64_t pp, int tile) {
  const int64_t n = ceil_div(pp, tile);
  return n * (n + 1) / 2;
}

// The side that takes the least time: rounds of 256 workgroups, each of side^2, at the relative times per
// element that large products take with it (4,096^2: 7.5, 26.6 and 51 us per 1,024 columns of a tile of
// 64, 128 and 192: 1.32, 1.17 and 1 per element).  Small tiles fill the chip, large ones read less.
int tile_for(int64_t (*count)(const NsArgs&, int), const NsArgs& a) {
  int best = 64;
  double cost = 0;
  for (int tile : {64, 128, 192}) {
    const double rate = tile == 64 ? 1.32 : tile == 128 ? 1.17 : 1.0;
    const double c = (double)ceil_div(count(a, tile), 256) * tile * tile * rate;
    if (tile == 64 || c < cost) {
      cost = c;
      best = tile;
    }
  }
  return best;
}

int64_t count_sym(const NsArgs& a, int tile) {
  int64_t n = 0;
  for (int i = 0; i < a.count; ++i) n += upper_tiles(a.mat[i].pp, tile);
  return n;
}
int64_t count_update(const NsArgs& a, int tile) {
  int64_t n = 0;
  for (int i = 0; i < a.count; ++i) n += ceil_div(a.mat[i].pp, tile) * ceil_div(a.mat[i].qp, tile);
  return n;
}
Tiles pick_tiles(const NsArgs& a) {
  const int sym = tile_for(count_sym, a);
  return {sym, sym, tile_for(count_update, a)};
}

// Sizes, workgroup ranges and buffers of the matrices (empty ones are left out).
NsArgs plan(const NsTensor* t, int count, Arena& w, int64_t blocks[kKinds], Tiles* tiles) {
  NsArgs a{};
  for (int k = 0; k < kKinds; ++k) {
    blocks[k] = 0;
    for (int i = 0; i < kMats; ++i) a.first[k][i] = INT32_MAX;
  }
  for (int i = 0; i < count; ++i) {
    if (t[i].rows == 0 || t[i].cols == 0) continue;
    Mat& m = a.mat[a.count++];
    m.g = t[i].g;
    m.ldg = t[i].ldg;
    m.m = t[i].m;
    m.w = t[i].w;
    m.out = t[i].out;
    m.ldo = t[i].ldo;
    m.rows = (int32_t)t[i].rows;
    m.cols = (int32_t)t[i].cols;
    m.step = (float)t[i].step;
    m.pp = (int32_t)round_up(std::min(m.rows, m.cols), kTile);
    m.qp = (int32_t)round_up(std::max(m.rows, m.cols), kTile);
    m.vec = m.ldg == m.cols && ((int64_t)m.rows * m.cols) % 4 == 0 && aligned16(m.g) && (!m.m || aligned16(m.m));
    m.n_partial = (int32_t)std::min<int64_t>(kMaxPartials, ceil_div((int64_t)m.rows * m.cols, 4096));
  }
  *tiles = pick_tiles(a);
  // X X^T sums over the long side: split where the tiles do not fill the chip (at least 256 columns a
  // part), and where one accumulator would take more than kMaxSum columns.
  int64_t gram = 0;
  for (int i = 0; i < a.count; ++i) gram += upper_tiles(a.mat[i].pp, tiles->gram);
  for (int i = 0; i < a.count; ++i) {
    Mat& m = a.mat[i];
    const int64_t fill = std::max<int64_t>(1, 256 / gram), most = ceil_div(m.qp, 256);
    const int64_t splits = std::max(std::min(fill, most), ceil_div(m.qp, kMaxSum));
    m.kchunk = (int32_t)round_up(ceil_div(m.qp, splits), kTile);
    m.splits = (int32_t)ceil_div(m.qp, m.kchunk);
    const int64_t xy = 2 * (int64_t)m.pp * m.qp, ab = 2 * (int64_t)m.pp * m.pp;
    m.X = w.take<_Float16>(xy);
    m.Y[0] = w.take<_Float16>(xy);
    m.Y[1] = w.take<_Float16>(xy);
    m.A = w.take<_Float16>(ab);
    m.B = w.take<_Float16>(ab);
    m.partial = w.take<double>(m.n_partial);
    const int64_t ut = upper_tiles(m.pp, tiles->gram);
    if (m.splits > 1) m.part = w.take<float>(m.splits * ut * tiles->gram * tiles->gram);
    const int64_t n64 = m.pp / kTile, np = ceil_div(m.pp, tiles->update), nq = ceil_div(m.qp, tiles->update);
    int64_t need[kKinds];
    need[kSums] = m.n_partial;
    need[kPlanes] = n64 * (m.qp / kTile);
    need[kGram] = ut * m.splits;
    need[kJoin] = m.splits > 1 ? ut * (tiles->gram / 64) * (tiles->gram / 64) : 0;
    need[kPoly] = upper_tiles(m.pp, tiles->poly);
    need[kUpdate] = np * nq;
    for (int k = 0; k < kKinds; ++k) {
      a.first[k][i] = (int32_t)blocks[k];
      blocks[k] += need[k];
    }
  }
  for (int k = 0; k < kKinds; ++k) a.total[k] = (int32_t)blocks[k];
  return a;
}

unsigned xcd_grid(int64_t units) { return (unsigned)(8 * ceil_div(units, 8)); }

// The small form takes a call whose matrices all fit it: their sizes, and places in 32 bits.
bool small_form(const NsTensor* t, int count, int* pt, int* ns) {
  int64_t p = 0, q = 0;
  for (int i = 0; i < count; ++i) {
    if (t[i].rows == 0 || t[i].cols == 0) continue;
    p = std::max(p, std::min(t[i].rows, t[i].cols));
    q = std::max(q, std::max(t[i].rows, t[i].cols));
    if (std::max(t[i].ldg, t[i].ldo) > (1 << 18)) return false;
  }
  *pt = p <= 32 ? 1 : 2;
  *ns = q <= 256 ? 1 : q <= 512 ? 2 : q <= (p <= 32 ? 1024 : 768) ? (p <= 32 ? 4 : 3) : 6;
  return p <= 64 && q <= (*pt == 1 ? 1536 : 768);
}

void launch_small(int pt, int ns, const NsArgs& a, int steps, hipStream_t s) {
  const dim3 grid((unsigned)a.count), block(512);
  if (pt == 1) {
    if (ns == 1) hipLaunchKernelGGL((k_ns_small<1, 1>), grid, block, 0, s, a, steps);
    else if (ns == 2) hipLaunchKernelGGL((k_ns_small<1, 2>), grid, block, 0, s, a, steps);
    else if (ns == 4) hipLaunchKernelGGL((k_ns_small<1, 4>), grid, block, 0, s, a, steps);
    else hipLaunchKernelGGL((k_ns_small<1, 6>), grid, block, 0, s, a, steps);
  } else {
    if (ns == 1) hipLaunchKernelGGL((k_ns_small<2, 1>), grid, block, 0, s, a, steps);
    else if (ns == 2) hipLaunchKernelGGL((k_ns_small<2, 2>), grid, block, 0, s, a, steps);
    else hipLaunchKernelGGL((k_ns_small<2, 3>), grid, block, 0, s, a, steps);
  }
}

template <bool SQUARE>
void launch_sym(int tile, unsigned grid, const NsArgs& a, hipStream_t s) {
  if (tile == 192)
    hipLaunchKernelGGL((k_ns_sym<192, SQUARE>), dim3(grid), dim3(256), 0, s, a);
  else if (tile == 128)
    hipLaunchKernelGGL((k_ns_sym<128, SQUARE>), dim3(grid), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_ns_sym<64, SQUARE>), dim3(grid), dim3(256), 0, s, a);
}

void launch_join(int tile, unsigned grid, const NsArgs& a, hipStream_t s) {
  if (tile == 192)
    hipLaunchKernelGGL(k_ns_join<192>, dim3(grid), dim3(256), 0, s, a);
  else if (tile == 128)
    hipLaunchKernelGGL(k_ns_join<128>, dim3(grid), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(k_ns_join<64>, dim3(grid), dim3(256), 0, s, a);
}

void launch_update(int tile, unsigned grid, const NsArgs& a, hipStream_t s) {
  if (tile == 192)
    hipLaunchKernelGGL(k_ns_update<192>, dim3(grid), dim3(256), 0, s, a);
  else if (tile == 128)
    hipLaunchKernelGGL(k_ns_update<128>, dim3(grid), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(k_ns_update<64>, dim3(grid), dim3(256), 0, s, a);
}

}  // namespace

size_t newton_schulz_workspace(const NsTensor* t, int count) {
  Arena w;
  int64_t blocks[kKinds];
  Tiles tiles;
  int pt, ns;
  if (small_form(t, count, &pt, &ns)) return 0;
  plan(t, count, w, blocks, &tiles);
  return w.used;
}

gcn_status launch_newton_schulz(const NsTensor* t, int count, int32_t steps, double momentum, bool nesterov,
                                double keep, void* ws, hipStream_t s) {
  Arena w;
  w.base = static_cast<char*>(ws);
  int64_t blocks[kKinds];
  Tiles tiles;
  NsArgs a = plan(t, count, w, blocks, &tiles);
  if (a.count == 0) return GCN_OK;
  ProfScope prof("newton_schulz", a.mat[0].pp, a.mat[0].qp, 0, s);
  a.mu = (float)momentum;
  a.omu = (float)(1.0 - momentum);
  a.keep = (float)keep;
  a.nesterov = nesterov ? 1 : 0;
  int pt, ns;
  if (small_form(t, count, &pt, &ns)) {
    launch_small(pt, ns, a, steps, s);
    return check_launch("newton-schulz, one workgroup a matrix");
  }
  hipLaunchKernelGGL(k_ns_sums, dim3((unsigned)blocks[kSums]), dim3(256), 0, s, a);
  GCN_TRY(check_launch("newton-schulz norm"));
  hipLaunchKernelGGL(k_ns_planes, dim3((unsigned)blocks[kPlanes]), dim3(256), 0, s, a);
  GCN_TRY(check_launch("newton-schulz planes"));
  for (int k = 0; k < steps; ++k) {
    a.flip = k & 1;
    a.last = k == steps - 1;
    launch_sym<false>(tiles.gram, xcd_grid(blocks[kGram]), a, s);
    GCN_TRY(check_launch("newton-schulz X X^T"));
    if (blocks[kJoin] > 0) {
      launch_join(tiles.gram, (unsigned)blocks[kJoin], a, s);
      GCN_TRY(check_launch("newton-schulz join"));
    }
    launch_sym<true>(tiles.poly, xcd_grid(blocks[kPoly]), a, s);
    GCN_TRY(check_launch("newton-schulz polynomial"));
    launch_update(tiles.update, xcd_grid(blocks[kUpdate]), a, s);
    GCN_TRY(check_launch("newton-schulz update"));
  }
  return GCN_OK;
}

}  // namespace gcn
