// norm_device.h -- what the group norm's kernels share: places in a block, rows, activations and the sums
// over the fragments of a panel.
//
// Addresses: a row's base is the same for a whole wavefront and lives in scalar registers; a lane adds 32
// bits (its row among the ry that are read together, and its column).  With 64-bit places per lane, and the
// full-range expf and divide in the activation, the vector units and not the memory bounded these kernels
// (262,144 x 128 in 8,192 graphs, SiLU, in one pass, at the time: 115 us forward and 222 backward instead of 85 and 191).
#pragma once

#include "internal.h"

namespace gcn {

struct NormArgs {
  NormParams p;
  int32_t cg;       // channels per group
  int32_t tx_log;   // log2 of the lanes that share a row
  int32_t pw;       // columns per panel (blockIdx.y)
  int32_t n_panel;
  int32_t n_frag;   // (panel, group) overlaps: id panel + group
  int64_t rows;     // rows per block (one pass, backward: graphs)
  int64_t n_block;  // blocks
  int one;          // threads per graph of the one-pass form, or 0
  int32_t n_col;    // workgroups of a panel that add column sums in the backward's second pass
  bool joined;      // one graph of few pieces: pass 2 joins them itself
  float* part0;     // per piece and fragment: a value close to the mean, or sum of gamma d
  float* part1;     // squared distances from it, or sum of gamma d xh
  float* part2;     // forward: distances from it
  float* m1;        // per (graph, group)
  float* m2;
  float* col0;      // per block and column: sum of d
  float* col1;      // sum of d xh
};

// norm_one.hip
void launch_norm_one(const NormArgs& a, bool vec, hipStream_t s);
void launch_norm_grad_one(const NormArgs& a, bool vec, hipStream_t s);
// Rows that a thread of the one-pass forms has in registers at a time, by threads per graph: as many as leave
// 4 wavefronts to a SIMD.  Backward holds two matrices; 262,144 x 128 in 8,192 graphs, inputs that are not in
// the caches: 147 us with 2 rows, 135 with 4, 133 with 6, 164 with 8; forward 83 us with 16, 90 with 8.
constexpr int rows_fwd(int nt) { return nt == 64 ? 16 : 12; }
constexpr int rows_bwd() { return 6; }

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t seg_begin(const NormParams& p, int32_t s) {
  if (!p.seg_ptr) return 0;
  const int64_t v = p.seg_ptr[s];
  return v < 0 ? 0 : (v < p.n ? v : p.n);
}
__device__ __forceinline__ int64_t seg_end(const NormParams& p, int32_t s) {
  if (!p.seg_ptr) return p.n;
  const int64_t v = p.seg_ptr[s + 1];
  return v < 0 ? 0 : (v < p.n ? v : p.n);
}
// The last graph that begins at or before row r (0 if none does).
__device__ __forceinline__ int32_t seg_of(const NormParams& p, int64_t r) {
  if (!p.seg_ptr) return 0;
  int32_t lo = 0, hi = p.n_seg;  // seg_ptr[lo] <= r or lo == 0; seg_ptr[hi] > r or hi == n_seg
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (p.seg_ptr[mid] <= r) lo = mid; else hi = mid;
  }
  return lo;
}

// For a walk over the graphs from row r on that has met an empty one (s): past eight of them in a row the next
// is looked up, so that a batch of mostly empty graphs does not cost a step for each in every block.
__device__ __forceinline__ void skip_empty(const NormParams& p, int64_t r, int32_t& s, int& met) {
  if (++met < 8) return;
  met = 0;
  const int32_t next = seg_of(p, r);
  if (next > s + 1) s = next - 1;  // the walk's ++s
}

template <int V>
struct Vals {
  float v[V];
};
// V columns `off` bytes into the row (`left` = columns of the matrix from there on); a quad of an aligned
// row may take in columns behind the width, which are set to zero.
template <int V>
__device__ __forceinline__ Vals<V> load_raw(const float* row, uint32_t off) {
  const char* at = reinterpret_cast<const char*>(row) + off;
  Vals<V> r;
  if constexpr (V == 4) {
    const f32x4 q = *reinterpret_cast<const f32x4*>(at);
#pragma unroll
    for (int j = 0; j < 4; ++j) r.v[j] = q[j];
  } else {
    r.v[0] = *reinterpret_cast<const float*>(at);
  }
  return r;
}
template <int V>
__device__ __forceinline__ Vals<V> clip_cols(Vals<V> r, int32_t left) {
#pragma unroll
  for (int j = 1; j < V; ++j) r.v[j] = left > j ? r.v[j] : 0.f;
  return r;
}
template <int V>
__device__ __forceinline__ Vals<V> load_cols(const float* row, uint32_t off, int32_t left) {
  return clip_cols<V>(load_raw<V>(row, off), left);
}
// STREAM: past the caches.
template <int V, bool STREAM = false>
__device__ __forceinline__ void store_cols(float* row, uint32_t off, const Vals<V>& r, int32_t left) {
  char* at = reinterpret_cast<char*>(row) + off;
  if constexpr (V == 4) {
    if (left >= 4) {
      const f32x4 q = {r.v[0], r.v[1], r.v[2], r.v[3]};
      if constexpr (STREAM)
        __builtin_nontemporal_store(q, reinterpret_cast<f32x4*>(at));
      else
        *reinterpret_cast<f32x4*>(at) = q;
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < left) reinterpret_cast<float*>(at)[i] = r.v[i];
    }
  } else {
    *reinterpret_cast<float*>(at) = r.v[0];
  }
}

// Loads that only some lanes make, and uses of theirs under the same conditions: left to itself the compiler
// waits at each use, as if the one before had been skipped, and such a wait behind a store is a wait for the
// store (one counter has both).  This is the one wait for all of them.  The registers are set before such a
// load and its columns clipped at the use: anything done to them under the load's own condition would wait
// there for that load.  Together: 400,000 x 64 in 12,000 graphs, one channel a group, 58 us forward instead of 138.
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// f(r, x) of rows ty, ty + ry, .. < len of src, r the row less ty (the same for all lanes), four loads of
// 16 bytes or eight of 4 in flight (four of 4 take 82 us instead of 75 forward and 118 instead of 110 backward at
// 500,009 x 47); and the same with a second matrix.
template <int V, class F>
__device__ __forceinline__ void each_row(const float* src, int64_t ld, uint32_t off, int ty, int ry, int64_t len,
                                         int32_t left, F f) {
  constexpr int U = V == 1 ? 8 : 4;
  int64_t r = 0;
  for (; r + U * ry <= len; r += U * ry) {
    Vals<V> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load_cols<V>(src + (r + u * ry) * ld, off, left);
#pragma unroll
    for (int u = 0; u < U; ++u) f(r + u * ry, x[u]);
  }
  const int rest = (int)(len - r) - ty;
  Vals<V> x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    x[u] = Vals<V>{};
    if (u * ry < rest) x[u] = load_raw<V>(src + (r + u * ry) * ld, off);
  }
  loads_done();
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (u * ry < rest) {
      x[u] = clip_cols<V>(x[u], left);
      f(r + u * ry, x[u]);
    }
}
template <int V, class F>
__device__ __forceinline__ void each_row(const float* a, int64_t lda, uint32_t off_a, const float* b, int64_t ldb,
                                         uint32_t off_b, int ty, int ry, int64_t len, int32_t left, F f) {
  constexpr int U = V == 1 ? 8 : 4;
  int64_t r = 0;
  for (; r + U * ry <= len; r += U * ry) {
    Vals<V> x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = load_cols<V>(a + (r + u * ry) * lda, off_a, left);
      y[u] = load_cols<V>(b + (r + u * ry) * ldb, off_b, left);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) f(r + u * ry, x[u], y[u]);
  }
  const int rest = (int)(len - r) - ty;
  Vals<V> x[U], y[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    x[u] = y[u] = Vals<V>{};
    if (u * ry < rest) {
      x[u] = load_raw<V>(a + (r + u * ry) * lda, off_a);
      y[u] = load_raw<V>(b + (r + u * ry) * ldb, off_b);
    }
  }
  loads_done();
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (u * ry < rest) {
      x[u] = clip_cols<V>(x[u], left);
      y[u] = clip_cols<V>(y[u], left);
      f(r + u * ry, x[u], y[u]);
    }
}

// exp(-z) from the hardware's 2^x: the error of its argument, |z| 2^-24, only shows where the result is
// small beside the 1 it is added to, or, in z exp(z), relative to |z| times the result.
__device__ __forceinline__ float exp_neg(float z) { return __builtin_amdgcn_exp2f(z * -1.44269504f); }
template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == GCN_ACT_RELU) return z > 0.f ? z : (z == z ? 0.f : z);
  if constexpr (ACT == GCN_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + exp_neg(z));
  return z;
}
// act'(z) times dy; ReLU's derivative is 1[z > 0], as in the layers.  SiLU's is q (1 + z (1 - q)) with
// q = 1 / (1 + e), 1 - q = e q; below z = -80, where it is less than 1e-32, that of -80 is taken: e stays finite, and
// q, which no longer falls, is not multiplied by a z that does.
template <int ACT>
__device__ __forceinline__ float act_grad(float dy, float z) {
  if constexpr (ACT == GCN_ACT_RELU) return z > 0.f ? dy : 0.f;
  if constexpr (ACT == GCN_ACT_SILU) {
    z = z < -80.f ? -80.f : z;
    const float e = exp_neg(z), q = __builtin_amdgcn_rcpf(1.f + e);
    return dy * (q * (1.f + z * (e * q)));
  }
  return dy;
}

// This thread's place in a block: columns c0 .. c0 + V - 1, rows ty, ty + ry, ...
template <int V, int NT = kThreads>
struct Place {
  int tx, ty, ry, panel;
  int32_t p0, c0, left;  // first column of the panel, of the thread; columns left from c0 on
  int32_t gfirst, nf;    // first group of the panel, fragments in it
  __device__ __forceinline__ explicit Place(const NormArgs& a) {
    const int tid = threadIdx.x;
    tx = tid & ((1 << a.tx_log) - 1);
    ty = tid >> a.tx_log;
    ry = NT >> a.tx_log;
    panel = blockIdx.y;
    p0 = panel * a.pw;
    c0 = p0 + tx * V;
    left = a.p.c - c0;
    gfirst = p0 / a.cg;
    const int32_t last = (p0 + a.pw < a.p.c ? p0 + a.pw : a.p.c) - 1;
    nf = last / a.cg - gfirst + 1;
  }
  // Bytes from the first of the rows that are read together, of pitch ld.
  __device__ __forceinline__ uint32_t off(int64_t ld) const { return ((uint32_t)ty * (uint32_t)ld + (uint32_t)c0) * 4; }
};

// Groups, gamma and beta of the columns from c0 on.
template <int V>
__device__ __forceinline__ void affine(const NormArgs& a, int32_t c0, float* gamma, float* beta, int32_t* g) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int32_t c = c0 + j < a.p.c ? c0 + j : a.p.c - 1;
    g[j] = c / a.cg;
    gamma[j] = a.p.gamma ? a.p.gamma[c] : 1.f;
    beta[j] = a.p.beta ? a.p.beta[c] : 0.f;
  }
}

// Columns [lo, hi) of the panel that belong to its fragment f, counted from the panel's first.
__device__ __forceinline__ void frag_cols(const NormArgs& a, int32_t p0, int32_t gfirst, int f, int& lo, int& hi) {
  const int32_t g = gfirst + f;
  const int32_t b = g * a.cg, e = b + a.cg, pe = p0 + a.pw < a.p.c ? p0 + a.pw : a.p.c;
  lo = (b > p0 ? b : p0) - p0;
  hi = (e < pe ? e : pe) - p0;
}

// Sums over each fragment of K arrays red (ry rows of pw columns each) in a fixed order; emit(f, sums) on one
// lane each.  Lanes of a wavefront share a fragment: lc of them over its columns, the others over rows.
template <int NT, int K, class Emit>
__device__ __forceinline__ void frag_sums_of(const NormArgs& a, int32_t p0, int32_t gfirst, int nf, int ry,
                                             const float* const (&red)[K], Emit emit) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int w = a.cg < a.pw ? a.cg : a.pw;
  int lc = 1;
  while (lc < w && lc < 64) lc <<= 1;
  int lr = 1;
  while (lr < ry && lc * lr < 64) lr <<= 1;
  const int per = 64 / (lc * lr);  // fragments per wavefront at a time
  const int sub = lane & (lc * lr - 1);
  for (int f0 = wave * per; f0 < nf; f0 += (NT / 64) * per) {
    const int f = f0 + lane / (lc * lr);
    float v[K] = {};
    if (f < nf) {
      int lo, hi;
      frag_cols(a, p0, gfirst, f, lo, hi);
      for (int y = sub / lc; y < ry; y += lr)
        for (int c = lo + (sub & (lc - 1)); c < hi; c += lc)
#pragma unroll
          for (int k = 0; k < K; ++k) v[k] += red[k][y * a.pw + c];
    }
    for (int o = (lc * lr) >> 1; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o, 64);
    if (f < nf && sub == 0) emit(f, v);
  }
}
template <int NT = kThreads, class Emit>
__device__ __forceinline__ void frag_sums(const NormArgs& a, int32_t p0, int32_t gfirst, int nf, int ry,
                                          const float* red, Emit emit) {
  const float* const one[1] = {red};
  frag_sums_of<NT, 1>(a, p0, gfirst, nf, ry, one, [&](int f, const float* v) { emit(f, v[0]); });
}

// LDS of join_threads: a panel has at most 64 V columns.
template <int V>
struct JoinBox {
  float red0[kThreads * V], red1[kThreads * V];
  float mean[64 * V], rest[64 * V], dev[64 * V];
};

// The threads' values joined over `rows` rows: box.mean[f] is a value close to the mean of the panel's fragment f,
// box.rest[f] and box.dev[f] the sums of the distances and of the squared distances from it, for all threads behind the
// call.  A thread has cnt values, first among them, of mean first + md and squared deviations m2.  What is added up
// is distances, from a value of the fragment (that of its first column in the first row, which has values) and then
// from the mean that this gives: differences of values that are close are exact, so the size of the values costs no
// digits, the rounding of the mean to fp32 is known (rest), and a constant group has exactly its value.
template <int V, int NT>
__device__ __forceinline__ void join_threads(const NormArgs& a, const Place<V, NT>& t, float cnt, const float* first,
                                             const float* md, const float* m2, const int32_t* g, float rows,
                                             JoinBox<V>& box) {
  if (t.ty == 0)
#pragma unroll
    for (int j = 0; j < V; ++j) box.rest[t.tx * V + j] = first[j];
  __syncthreads();
  const int at = t.ty * a.pw + t.tx * V;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int32_t b = g[j] * a.cg;
    box.red0[at + j] = cnt * ((first[j] - box.rest[(b > t.p0 ? b : t.p0) - t.p0]) + md[j]);
  }
  __syncthreads();
  frag_sums<NT>(a, t.p0, t.gfirst, t.nf, t.ry, box.red0, [&](int f, float v) {
    int lo, hi;
    frag_cols(a, t.p0, t.gfirst, f, lo, hi);
    box.mean[f] = box.rest[lo] + v / (rows * (float)(hi - lo));
  });
  __syncthreads();
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float d = (first[j] - box.mean[g[j] - t.gfirst]) + md[j];
    box.red0[at + j] = cnt * d;
    box.red1[at + j] = m2[j] + cnt * d * d;
  }
  __syncthreads();
  const float* const both[2] = {box.red0, box.red1};
  frag_sums_of<NT, 2>(a, t.p0, t.gfirst, t.nf, t.ry, both, [&](int f, const float* v) {
    box.rest[f] = v[0];
    box.dev[f] = v[1];
  });
  __syncthreads();
}

// Count, first value, mean less that and squared deviations of this thread's rows among [r, r + len).
template <int V, int NT>
__device__ __forceinline__ float read_stats(const NormParams& p, const Place<V, NT>& t, int64_t r, int64_t len,
                                            float* first, float* md, float* m2) {
  Vals<V> k{}, sum{}, sq{};
  float cnt = 0.f;
  if (t.left > 0 && t.ty < len) {
    const float* src = p.X + r * p.ldx;
    const uint32_t off = t.off(p.ldx);
    k = load_cols<V>(src, off, t.left);
    cnt = (float)((len - t.ty + t.ry - 1) / t.ry);
    each_row<V>(src, p.ldx, off, t.ty, t.ry, len, t.left, [&](int64_t, const Vals<V>& x) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = x.v[j] - k.v[j];
        sum.v[j] += d;
        sq.v[j] += d * d;
      }
    });
  }
  const float inv = cnt > 0.f ? 1.f / cnt : 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    first[j] = k.v[j];
    md[j] = sum.v[j] * inv;
    m2[j] = sq.v[j] - sum.v[j] * md[j];
  }
  return cnt;
}

// Mean and 1 / sqrt(var + eps) of 1 / inv elements from what join_threads leaves of their group.
__device__ __forceinline__ void finish_stats(float center, float rest, float dev, double inv, double eps, float& mean,
                                             float& rstd) {
  const double e = (double)rest * inv, var = (double)dev * inv - e * e;
  mean = (float)((double)center + e);
  rstd = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps));
}

// The columns of a workgroup's panel: tot over its row lanes (red0, red1: as large as the workgroup).
template <int V, int NT>
__device__ __forceinline__ void write_columns(const NormArgs& a, const Place<V, NT>& t, const float* tot0,
                                              const float* tot1, float* red0, float* red1) {
  const NormParams& p = a.p;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int at = t.ty * a.pw + t.tx * V + j;
    red0[at] = tot0[j];
    red1[at] = tot1[j];
  }
  __syncthreads();
  // as many lanes a column as there are, up to a wavefront
  int lanes = 1;
  while (lanes < 64 && lanes < t.ry && lanes * 2 * a.pw <= NT) lanes <<= 1;
  const int sub = threadIdx.x & (lanes - 1);
  for (int at = 0; at < a.pw; at += NT / lanes) {
    const int c = at + threadIdx.x / lanes;
    const bool in = c < a.pw && t.p0 + c < p.c;
    float v0 = 0.f, v1 = 0.f;
    if (in)
      for (int y = sub; y < t.ry; y += lanes) {
        v0 += red0[y * a.pw + c];
        v1 += red1[y * a.pw + c];
      }
    for (int o = lanes >> 1; o > 0; o >>= 1) {
      v0 += __shfl_xor(v0, o, 64);
      v1 += __shfl_xor(v1, o, 64);
    }
    if (in && sub == 0) {
      a.col0[(int64_t)blockIdx.x * p.c + t.p0 + c] = v0;
      a.col1[(int64_t)blockIdx.x * p.c + t.p0 + c] = v1;
    }
  }
}

// xh and d of x and dy in their places.
template <int V, int ACT>
__device__ __forceinline__ void normalise(Vals<V>& x, Vals<V>& dy, const float* mean, const float* rstd,
                                          const float* gamma, const float* beta) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float xh = (x.v[j] - mean[j]) * rstd[j];
    dy.v[j] = act_grad<ACT>(dy.v[j], gamma[j] * xh + beta[j]);
    x.v[j] = xh;
  }
}

}  // namespace
}  // namespace gcn
