// norm.hip -- group norm with an activation over the nodes of each graph of a batch.
//
// H is n x c, one node per row (channels last).  A batch is consecutive row ranges, one
// per graph (seg_ptr); the channels are cut into `groups` equal groups.  With N the
// elements of one (graph, group):
//   mu = sum x / N, var = sum (x - mu)^2 / N, r = 1 / sqrt(var + eps)
//   xh = (x - mu) r, z = gamma xh + beta, y = act(z)
// and backward, with d = dy act'(z):
//   dbeta = sum_rows d, dgamma = sum_rows d xh
//   m1 = sum gamma d / N, m2 = sum gamma d xh / N (per graph and group)
//   dx = r (gamma d - m1 - xh m2)
//
// HBM bounds it: 8 n c bytes forward, 12 n c backward, where a (graph, group) fits on
// chip; otherwise the input is read twice.  The form here takes any lengths: the rows are
// cut into equal blocks whatever the graphs (so that one graph of millions of rows and
// thousands of short ones both fill the chip), and a block's part of a graph is a piece.
// Pass 1 writes partial statistics of every piece, a second kernel joins them per
// (graph, group), pass 2 applies them, taking the blocks in reverse order so that it starts
// on the rows that pass 1 left in cache.  Piece ids need no list: walking the blocks and
// the graphs in row order, each step moves to the next block or to the next graph, so
// block + graph is unique.
//
// Precision: a thread sums (x - k) and (x - k)^2 about k, its first value, in fp32 (a
// mean far from zero then costs no digits); threads and pieces are joined by their counts,
// means and squared deviations (Chan, Golub, LeVeque 1979), the means as distances from a value
// of the group, pieces in fp64.  The mean is rounded once, when it is written.
#include "norm_device.h"

namespace gcn {
namespace {

// Pass 1, forward: a value close to the mean, distances and squared distances from it, of every piece and
// fragment.
template <int V>
__global__ void __launch_bounds__(kThreads) k_norm_stats(NormArgs a) {
  __shared__ JoinBox<V> box;
  const NormParams& p = a.p;
  const Place<V> t(a);
  int32_t g[V];
#pragma unroll
  for (int j = 0; j < V; ++j) g[j] = (t.c0 + j < p.c ? t.c0 + j : p.c - 1) / a.cg;
  const int64_t r0 = (int64_t)blockIdx.x * a.rows;
  const int64_t r1 = r0 + a.rows < p.n ? r0 + a.rows : p.n;
  int64_t r = r0;
  int met = 0;
  for (int32_t s = seg_of(p, r0); s < p.n_seg && r < r1; ++s) {
    const int64_t b = seg_begin(p, s), e0 = seg_end(p, s);
    if (r < b) r = b;
    const int64_t e = e0 < r1 ? e0 : r1;
    if (e <= r) {
      skip_empty(p, r, s, met);
      continue;
    }
    met = 0;
    float first[V], md[V], m2[V];
    const float cnt = read_stats(p, t, r, e - r, first, md, m2);
    join_threads(a, t, cnt, first, md, m2, g, (float)(e - r), box);
    const int64_t piece = ((int64_t)blockIdx.x + s) * a.n_frag + t.panel + t.gfirst;
    for (int f = threadIdx.x; f < t.nf; f += kThreads) {
      a.part0[piece + f] = box.mean[f];
      a.part1[piece + f] = box.dev[f];
      a.part2[piece + f] = box.rest[f];
    }
    __syncthreads();
    r = e;
  }
}

// The pieces of graph s and group g joined in row order: every LT-th from `sub` on, then over the LT lanes.
// n: elements; forward ref + s0 / n is the mean and s1 / n - (s0 / n)^2 the variance, backward s0 and s1 are
// the sums.
struct Joined {
  double n, ref, s0, s1;
};
template <int LT, bool BWD>
__device__ __forceinline__ Joined join_pieces(const NormArgs& a, int32_t s, int32_t g, int sub) {
  const NormParams& p = a.p;
  const int64_t b = seg_begin(p, s), e = seg_end(p, s);
  const int32_t c0 = g * a.cg, c1 = c0 + a.cg;
  const int32_t q0 = c0 / a.pw, q1 = (c1 - 1) / a.pw;
  Joined v{};
  if (b < e) {
    const int64_t k0 = b / a.rows, k1 = (e - 1) / a.rows;
    if (!BWD) v.ref = (double)a.part0[(k0 + s) * a.n_frag + q0 + g];
#pragma unroll 4
    for (int64_t k = k0 + sub; k <= k1; k += LT) {
      const int64_t rb = k * a.rows > b ? k * a.rows : b;
      const int64_t re = (k + 1) * a.rows < e ? (k + 1) * a.rows : e;
      for (int32_t q = q0; q <= q1; ++q) {
        const int64_t at = (k + s) * a.n_frag + q + g;
        const int32_t lo = c0 > q * a.pw ? c0 : q * a.pw;
        const int32_t hi = c1 < (q + 1) * a.pw ? c1 : (q + 1) * a.pw;
        if (BWD) {
          v.s0 += (double)a.part0[at];
          v.s1 += (double)a.part1[at];
        } else {
          // about the first piece's value, in fp64
          const double m = (double)(re - rb) * (double)(hi - lo), d = (double)a.part0[at] - v.ref;
          const double rest = (double)a.part2[at];
          v.s0 += m * d + rest;
          v.s1 += (double)a.part1[at] + (m * d + 2.0 * rest) * d;
        }
      }
    }
    v.n = (double)(e - b) * (double)a.cg;
  }
  constexpr int kLanes = LT < 64 ? LT : 64;
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    v.s0 += __shfl_xor(v.s0, o, 64);
    v.s1 += __shfl_xor(v.s1, o, 64);
  }
  return v;
}
__device__ __forceinline__ void moments(const Joined& v, double eps, float& mean, float& rstd) {
  mean = rstd = 0.f;
  if (v.n > 0.0) {
    const double md = v.s0 / v.n, var = v.s1 / v.n - md * md;
    mean = (float)(v.ref + md);
    rstd = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps));
  }
}

// All (graph, group) pairs, LT lanes each (kThreads: a workgroup each).
template <int LT, bool BWD>
__global__ void __launch_bounds__(kThreads) k_norm_join(NormArgs a) {
  __shared__ double box[2][4];
  const NormParams& p = a.p;
  const int64_t task = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / LT;
  const int sub = threadIdx.x % LT;
  if (task >= (int64_t)p.n_seg * p.groups) return;
  Joined v = join_pieces<LT, BWD>(a, (int32_t)(task / p.groups), (int32_t)(task % p.groups), sub);
  if constexpr (LT > 64) {
    if (threadIdx.x % 64 == 0) {
      box[0][threadIdx.x / 64] = v.s0;
      box[1][threadIdx.x / 64] = v.s1;
    }
    __syncthreads();
    v.s0 = box[0][0] + box[0][1] + box[0][2] + box[0][3];
    v.s1 = box[1][0] + box[1][1] + box[1][2] + box[1][3];
  }
  if (sub != 0) return;
  if (BWD) {
    a.m1[task] = v.n > 0.0 ? (float)(v.s0 / v.n) : 0.f;
    a.m2[task] = v.n > 0.0 ? (float)(v.s1 / v.n) : 0.f;
  } else {
    moments(v, p.eps, p.mean[task], p.rstd[task]);
  }
}

// One graph of few pieces (a.joined): every workgroup joins its panel's groups itself, 16 lanes each, into
// v0 and v1 in LDS; the first block also writes them down.
template <bool BWD>
__device__ __forceinline__ void join_here(const NormArgs& a, int32_t gfirst, int nf, int64_t block, float* v0, float* v1) {
  const NormParams& p = a.p;
  for (int f0 = 0; f0 < nf; f0 += kThreads / 16) {
    const int f = f0 + threadIdx.x / 16;
    const Joined v = join_pieces<16, BWD>(a, 0, gfirst + (f < nf ? f : nf - 1), threadIdx.x % 16);
    if (f < nf && threadIdx.x % 16 == 0) {
      if (BWD) {
        v0[f] = (float)(v.s0 / v.n);
        v1[f] = (float)(v.s1 / v.n);
      } else {
        float mean, rstd;
        moments(v, p.eps, mean, rstd);
        v0[f] = mean;
        v1[f] = rstd;
        if (block == 0) {
          p.mean[gfirst + f] = mean;
          p.rstd[gfirst + f] = rstd;
        }
      }
    }
  }
  __syncthreads();
}

// Pass 2, forward.
template <int V, int ACT, bool STREAM>
__global__ void __launch_bounds__(kThreads) k_norm_apply(NormArgs a) {
  __shared__ float v0[kThreads * V];
  __shared__ float v1[kThreads * V];
  const NormParams& p = a.p;
  const Place<V> t(a);
  const int64_t block = gridDim.x - 1 - blockIdx.x;
  if (a.joined) join_here<false>(a, t.gfirst, t.nf, block, v0, v1);
  if (t.left <= 0) return;
  const int64_t r0 = block * a.rows;
  const int64_t r1 = r0 + a.rows < p.n ? r0 + a.rows : p.n;
  float gamma[V], beta[V];
  int32_t g[V];
  affine<V>(a, t.c0, gamma, beta, g);
  const uint32_t off_x = t.off(p.ldx), off_y = t.off(p.ldy);
  int64_t r = r0;
  int met = 0;
  for (int32_t s = seg_of(p, r0); s < p.n_seg && r < r1; ++s) {
    const int64_t b = seg_begin(p, s), e0 = seg_end(p, s);
    if (r < b) r = b;
    const int64_t e = e0 < r1 ? e0 : r1;
    if (e <= r) {
      skip_empty(p, r, s, met);
      continue;
    }
    met = 0;
    float mean[V], sc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      mean[j] = a.joined ? v0[g[j] - t.gfirst] : p.mean[(int64_t)s * p.groups + g[j]];
      sc[j] = a.joined ? v1[g[j] - t.gfirst] : p.rstd[(int64_t)s * p.groups + g[j]];
    }
    float* dst = p.Y + r * p.ldy;
    each_row<V>(p.X + r * p.ldx, p.ldx, off_x, t.ty, t.ry, e - r, t.left, [&](int64_t i, const Vals<V>& x) {
      Vals<V> y;
#pragma unroll
      for (int j = 0; j < V; ++j) y.v[j] = activate<ACT>(gamma[j] * ((x.v[j] - mean[j]) * sc[j]) + beta[j]);
      store_cols<V, STREAM>(dst + i * p.ldy, off_y, y, t.left);
    });
    r = e;
  }
}

// Pass 1, backward: sums of gamma d and gamma d xh of every piece and fragment, and of d and d xh of every
// block and column.
template <int V, int ACT>
__global__ void __launch_bounds__(kThreads) k_norm_grad_sums(NormArgs a) {
  __shared__ float red0[kThreads * V];
  __shared__ float red1[kThreads * V];
  const NormParams& p = a.p;
  const Place<V> t(a);
  const int64_t r0 = (int64_t)blockIdx.x * a.rows;
  const int64_t r1 = r0 + a.rows < p.n ? r0 + a.rows : p.n;
  float gamma[V], beta[V], tot0[V] = {}, tot1[V] = {};
  int32_t g[V];
  affine<V>(a, t.c0, gamma, beta, g);
  const uint32_t off_x = t.off(p.ldx), off_d = t.off(p.lddy);
  int64_t r = r0;
  int met = 0;
  for (int32_t s = seg_of(p, r0); s < p.n_seg && r < r1; ++s) {
    const int64_t b = seg_begin(p, s), e0 = seg_end(p, s);
    if (r < b) r = b;
    const int64_t e = e0 < r1 ? e0 : r1;
    if (e <= r) {
      skip_empty(p, r, s, met);
      continue;
    }
    met = 0;
    float s0[V], s1[V], mean[V], rstd[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      s0[j] = s1[j] = 0.f;
      mean[j] = p.mean[(int64_t)s * p.groups + g[j]];
      rstd[j] = p.rstd[(int64_t)s * p.groups + g[j]];
    }
    if (t.left > 0)
      each_row<V>(p.X + r * p.ldx, p.ldx, off_x, p.dY + r * p.lddy, p.lddy, off_d, t.ty, t.ry, e - r, t.left,
                  [&](int64_t, Vals<V>& x, Vals<V>& d) {
                    normalise<V, ACT>(x, d, mean, rstd, gamma, beta);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                      s0[j] += d.v[j];
                      s1[j] += d.v[j] * x.v[j];
                    }
                  });
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int at = t.ty * a.pw + t.tx * V + j;
      red0[at] = gamma[j] * s0[j];
      red1[at] = gamma[j] * s1[j];
      tot0[j] += s0[j];
      tot1[j] += s1[j];
    }
    __syncthreads();
    const int64_t piece = ((int64_t)blockIdx.x + s) * a.n_frag + t.panel + t.gfirst;
    frag_sums(a, t.p0, t.gfirst, t.nf, t.ry, red0, [&](int f, float v) { a.part0[piece + f] = v; });
    frag_sums(a, t.p0, t.gfirst, t.nf, t.ry, red1, [&](int f, float v) { a.part1[piece + f] = v; });
    __syncthreads();
    r = e;
  }
  write_columns(a, t, tot0, tot1, red0, red1);
}

// dbeta (which = 0) or dgamma of columns c0 .. c0 + 3: the blocks' column sums added in fp64 by NT / 4 lanes a
// column.
template <int NT>
__device__ __forceinline__ void sum_columns(const NormArgs& a, int32_t c0, int which, double (*part)[4]) {
  const NormParams& p = a.p;
  const int x = threadIdx.x % 4, y = threadIdx.x / 4;
  const int32_t c = c0 + x;
  const float* src = which == 0 ? a.col0 : a.col1;
  float* out = which == 0 ? p.dbeta : p.dgamma;
  if (!out) return;
  double v = 0.0;
  if (c < p.c) {
#pragma unroll 8
    for (int64_t k = y; k < a.n_block; k += NT / 4) v += (double)src[k * p.c + c];
  }
#pragma unroll
  for (int o = 4; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
  if (threadIdx.x % 64 < 4) part[threadIdx.x / 64][x] = v;
  __syncthreads();
  if (threadIdx.x < 4 && c < p.c) {
    v = 0.0;
    for (int k = 0; k < NT / 64; ++k) v += part[k][x];
    out[c] = (float)v;
  }
}

// Where there is no second pass: 4 columns a workgroup.
__global__ void __launch_bounds__(1024) k_norm_columns(NormArgs a) {
  __shared__ double part[16][4];
  sum_columns<1024>(a, blockIdx.x * 4, blockIdx.y, part);
}

// Pass 2, backward.  The first a.n_col workgroups of a panel add its column sums: hidden behind the others they
// cost nothing, in a launch of their own 5 to 10 us.
template <int V, int ACT, bool STREAM>
__global__ void __launch_bounds__(kThreads) k_norm_grad(NormArgs a) {
  __shared__ float v0[kThreads * V];
  __shared__ float v1[kThreads * V];
  __shared__ double part[kThreads / 64][4];
  const NormParams& p = a.p;
  const Place<V> t(a);
  if ((int)blockIdx.x < a.n_col) {
    sum_columns<kThreads>(a, t.p0 + (int)blockIdx.x / 2 * 4, blockIdx.x % 2, part);
    return;
  }
  const int64_t block = gridDim.x - 1 - blockIdx.x;
  if (a.joined) join_here<true>(a, t.gfirst, t.nf, block, v0, v1);
  if (t.left <= 0) return;
  const int64_t r0 = block * a.rows;
  const int64_t r1 = r0 + a.rows < p.n ? r0 + a.rows : p.n;
  float gamma[V], beta[V];
  int32_t g[V];
  affine<V>(a, t.c0, gamma, beta, g);
  const uint32_t off_x = t.off(p.ldx), off_d = t.off(p.lddy), off = t.off(p.lddx);
  int64_t r = r0;
  int met = 0;
  for (int32_t s = seg_of(p, r0); s < p.n_seg && r < r1; ++s) {
    const int64_t b = seg_begin(p, s), e0 = seg_end(p, s);
    if (r < b) r = b;
    const int64_t e = e0 < r1 ? e0 : r1;
    if (e <= r) {
      skip_empty(p, r, s, met);
      continue;
    }
    met = 0;
    float mean[V], rstd[V], m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int64_t at = (int64_t)s * p.groups + g[j];
      mean[j] = p.mean[at];
      rstd[j] = p.rstd[at];
      m1[j] = a.joined ? v0[g[j] - t.gfirst] : a.m1[at];
      m2[j] = a.joined ? v1[g[j] - t.gfirst] : a.m2[at];
    }
    float* dst = p.dX + r * p.lddx;
    each_row<V>(p.X + r * p.ldx, p.ldx, off_x, p.dY + r * p.lddy, p.lddy, off_d, t.ty, t.ry, e - r, t.left,
                [&](int64_t i, Vals<V>& x, Vals<V>& d) {
                  normalise<V, ACT>(x, d, mean, rstd, gamma, beta);
                  Vals<V> o;
#pragma unroll
                  for (int j = 0; j < V; ++j) o.v[j] = rstd[j] * (gamma[j] * d.v[j] - m1[j] - x.v[j] * m2[j]);
                  store_cols<V, STREAM>(dst + i * p.lddx, off, o, t.left);
                });
    r = e;
  }
}

bool rows_vec(const void* q, int64_t ld) { return aligned16(q) && ld % 4 == 0; }

// The layout of a call, its buffers carved from the workspace.  vec: 16-byte rows everywhere (the size query
// has no buffers to look at: it takes the larger of the two layouts).
NormArgs plan(const NormParams& p, bool bwd, bool vec, Arena& w) {
  NormArgs a{};
  a.p = p;
  a.cg = p.c / p.groups;
  const int v = vec ? 4 : 1;
  while (a.tx_log < 6 && (v << a.tx_log) < p.c) ++a.tx_log;
  a.pw = v << a.tx_log;
  a.n_panel = (int32_t)ceil_div(p.c, a.pw);
  a.n_frag = a.n_panel - 1 + p.groups;
  // One pass for batches of at least 256 graphs and panels of whole groups: a workgroup a graph, where graphs
  // on average fit its registers forward (longer ones are read twice, out of the caches; backward, with half
  // the registers for each matrix, few graphs have to be half as long) and the longest, which is the end of the
  // call, is at most 16 times that.  Forward a wavefront a graph, where they fit that and the others of the batch
  // hide the longest.  128 channels, SiLU, lengths spread exponentially, one input again and again, microseconds:
  //   graphs x mean rows   wavefronts   workgroups   two passes   backward   in two passes
  //        256 x 32            30           15           33          23           33
  //        256 x 96            82           29           31          50           35
  //       1024 x 32            32           18           45          31           48
  //       1024 x 96            93           36           59          66           70
  //       4096 x 32            44           47           89          68          109
  //       4096 x 64            89           62          112         133          161
  //       8192 x 32            76           86          144         136          196
  // (A launch takes less than 2^32 threads.)
  if (p.seg_ptr && p.max_seg >= 0 && p.n_seg < (1 << 24) && (int64_t)p.n_seg * a.n_panel >= 256 &&
      (a.n_panel == 1 || a.pw % a.cg == 0)) {
    const int lanes = a.cg / 4;
    const bool wave = !bwd && vec && (a.cg == 1 || a.cg == 2 || (a.cg % 4 == 0 && (lanes & (lanes - 1)) == 0));
    const int64_t fit1 = (int64_t)rows_fwd(64) * (64 >> a.tx_log);
    const int64_t fit = (int64_t)rows_fwd(kThreads) * (kThreads >> a.tx_log);
    const int64_t mean = p.n / p.n_seg;
    if (wave && mean <= fit1 && (p.max_seg <= 2 * fit1 || p.max_seg <= p.n / 256)) a.one = 64;
    else if (mean <= (bwd && p.n_seg < 512 ? fit / 2 : fit) && p.max_seg <= 16 * fit) a.one = kThreads;
  }
  // A few small graphs: a workgroup a graph and group, its panel being the group, where the longest fits its
  // registers (backward twice over) and it is little data, since such a panel may be less than a line of a row.
  // Microseconds, forward and backward, beside two passes: 2,708 x 16 in 4 groups 12 and 15 instead of 15 and 17
  // (much of it the caller's); 1,000 x 256 in 32 groups 12 and 14 instead of 20 and 20; 5,000 x 64 in 20 graphs 13 and
  // 17 instead of 25 and 27; but 3,000 x 1,024 in 256 groups 30 and 60 instead of 21 and 28.
  const int lanes = a.cg / v;
  const int64_t longest = p.seg_ptr ? p.max_seg : p.n;
  const int64_t most = (bwd ? rows_bwd() * 2 : rows_fwd(kThreads)) * kThreads;
  if (!a.one && p.n_seg > 0 && a.cg % v == 0 && (lanes & (lanes - 1)) == 0 && lanes <= 64 && longest >= 0 &&
      longest <= most / lanes && p.groups <= 65535 && (int64_t)p.n_seg * p.groups <= 4096 &&
      p.n <= ((int64_t)1 << 20) / p.c) {
    a.one = kThreads;
    for (a.tx_log = 0; 1 << a.tx_log < lanes;) ++a.tx_log;
    a.pw = a.cg;
    a.n_panel = p.groups;
  }
  if (a.one) {
    a.rows = ceil_div(p.n_seg, 1024);  // backward: graphs a workgroup, whose column sums are kept together
    a.n_block = ceil_div(p.n_seg, a.rows);
  } else {
    // about 8 workgroups a CU and at least four rows per thread; a single graph that 64 blocks of fewer rows
    // cover takes those, so few that pass 2 joins their pieces itself
    const int64_t ry = kThreads >> a.tx_log;
    a.rows = std::max<int64_t>(ceil_div(p.n * a.n_panel, 2048), 4 * ry);
    if (!p.seg_ptr && p.n <= 64 * a.rows) {
      a.rows = ceil_div(p.n, 64);
      a.joined = p.n > 0;
    }
    a.rows = std::max<int64_t>(round_up(a.rows, ry), ry);
    a.n_block = ceil_div(p.n, a.rows);
    const int64_t pieces = (a.n_block + p.n_seg) * a.n_frag;
    a.part0 = w.take<float>(pieces);
    a.part1 = w.take<float>(pieces);
    if (!bwd) a.part2 = w.take<float>(pieces);
  }
  if (bwd) {
    if (!a.one) {
      a.m1 = w.take<float>((int64_t)p.n_seg * p.groups);
      a.m2 = w.take<float>((int64_t)p.n_seg * p.groups);
    }
    a.col0 = w.take<float>(a.n_block * p.c);
    a.col1 = w.take<float>(a.n_block * p.c);
    if (a.one && a.n_block == 1) {  // the one block's sums are the result
      if (p.dbeta) a.col0 = p.dbeta;
      if (p.dgamma) a.col1 = p.dgamma;
    }
  }
  return a;
}

// Results that the 256 MB cache behind the L2s cannot hold are written past it, which leaves it to the input's
// second reading (2,449,029 x 256: 1,460 us forward instead of 1,540, 2,355 backward instead of 2,420).
bool streams(const NormArgs& a) { return a.p.n * a.p.c * 4 > ((int64_t)512 << 20); }

template <bool BWD>
void launch_join(const NormArgs& a, hipStream_t s) {
  const int64_t tasks = (int64_t)a.p.n_seg * a.p.groups;
  // few graphs: long lists of pieces, a workgroup each; many: 16 lanes each
  if (a.n_block > 16 * (int64_t)a.p.n_seg)
    hipLaunchKernelGGL((k_norm_join<kThreads, BWD>), dim3((unsigned)tasks), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_norm_join<16, BWD>), dim3((unsigned)ceil_div(tasks * 16, kThreads)), dim3(kThreads), 0, s, a);
}

template <int V, int ACT>
gcn_status run_fwd(const NormArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.n_block, (unsigned)a.n_panel);
  if (a.n_block > 0) {
    hipLaunchKernelGGL(k_norm_stats<V>, grid, dim3(kThreads), 0, s, a);
    GCN_TRY(check_launch("group norm statistics"));
  }
  if (!a.joined && (int64_t)a.p.n_seg * a.p.groups > 0) {
    launch_join<false>(a, s);
    GCN_TRY(check_launch("group norm join"));
  }
  if (a.n_block > 0) {
    if (streams(a))
      hipLaunchKernelGGL((k_norm_apply<V, ACT, true>), grid, dim3(kThreads), 0, s, a);
    else
      hipLaunchKernelGGL((k_norm_apply<V, ACT, false>), grid, dim3(kThreads), 0, s, a);
    GCN_TRY(check_launch("group norm apply"));
  }
  return GCN_OK;
}

template <int V, int ACT>
gcn_status run_bwd(NormArgs a, hipStream_t s) {
  const NormParams& p = a.p;
  const dim3 grid((unsigned)a.n_block, (unsigned)a.n_panel);
  if (a.one) {
    launch_norm_grad_one(a, V == 4, s);
    GCN_TRY(check_launch("group norm gradient"));
  } else if (a.n_block > 0) {
    hipLaunchKernelGGL((k_norm_grad_sums<V, ACT>), grid, dim3(kThreads), 0, s, a);
    GCN_TRY(check_launch("group norm gradient sums"));
  }
  const bool sums = p.dgamma || p.dbeta, second = !a.one && p.dX && a.n_block > 0 && p.n_seg > 0;
  if (!second) {
    if (sums && !(a.one && a.n_block == 1)) {
      hipLaunchKernelGGL(k_norm_columns, dim3((unsigned)ceil_div(p.c, 4), 2), dim3(1024), 0, s, a);
      GCN_TRY(check_launch("group norm column sums"));
    }
    return GCN_OK;
  }
  if (!a.joined) {
    launch_join<true>(a, s);
    GCN_TRY(check_launch("group norm gradient join"));
  }
  a.n_col = sums ? 2 * (int32_t)ceil_div(a.pw, 4) : 0;  // two outputs, four columns each
  const dim3 all((unsigned)(a.n_block + a.n_col), (unsigned)a.n_panel);
  if (streams(a))
    hipLaunchKernelGGL((k_norm_grad<V, ACT, true>), all, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_norm_grad<V, ACT, false>), all, dim3(kThreads), 0, s, a);
  return check_launch("group norm gradient");
}

template <int V>
gcn_status run(const NormArgs& a, bool bwd, hipStream_t s) {
  if (a.p.act == GCN_ACT_RELU) return bwd ? run_bwd<V, GCN_ACT_RELU>(a, s) : run_fwd<V, GCN_ACT_RELU>(a, s);
  if (a.p.act == GCN_ACT_SILU) return bwd ? run_bwd<V, GCN_ACT_SILU>(a, s) : run_fwd<V, GCN_ACT_SILU>(a, s);
  return bwd ? run_bwd<V, GCN_ACT_NONE>(a, s) : run_fwd<V, GCN_ACT_NONE>(a, s);
}

}  // namespace

size_t group_norm_workspace(const NormParams& p, bool bwd) {
  size_t most = 0;
  for (int v = 0; v < 2; ++v) {
    Arena w;
    plan(p, bwd, v != 0, w);
    most = std::max(most, w.used);
  }
  return most;
}

gcn_status launch_group_norm(const NormParams& p, void* ws, hipStream_t s) {
  ProfScope prof("group_norm_fwd", p.c, p.n, 0, s);
  const bool vec = rows_vec(p.X, p.ldx) && rows_vec(p.Y, p.ldy);
  Arena w;
  w.base = static_cast<char*>(ws);
  const NormArgs a = plan(p, false, vec, w);
  if (a.one) {
    launch_norm_one(a, vec, s);
    return check_launch("group norm");
  }
  return vec ? run<4>(a, false, s) : run<1>(a, false, s);
}

gcn_status launch_group_norm_bwd(const NormParams& p, void* ws, hipStream_t s) {
  ProfScope prof("group_norm_bwd", p.c, p.n, 0, s);
  const bool vec = rows_vec(p.X, p.ldx) && rows_vec(p.dY, p.lddy) && (!p.dX || rows_vec(p.dX, p.lddx));
  Arena w;
  w.base = static_cast<char*>(ws);
  const NormArgs a = plan(p, true, vec, w);
  return vec ? run<4>(a, true, s) : run<1>(a, true, s);
}

}  // namespace gcn
