// norm_one.hip -- the group norm in one pass over the data, for batches of graphs whose (graph, group) fits
// on chip: the statistics of a graph and its result, or its sums and gradients, come from one reading.
#include "norm_device.h"

namespace gcn {
namespace {

// A workgroup per graph and panel of whole groups.  rows_fwd rows a thread are in registers at a
// time; a graph of more of them is read again for the result.
template <int V, int ACT>
__global__ void __launch_bounds__(kThreads) k_norm_one(NormArgs a) {
  __shared__ JoinBox<V> box;
  constexpr int kRows = rows_fwd(kThreads);
  const NormParams& p = a.p;
  const int32_t s = blockIdx.x;
  const Place<V> t(a);
  float gamma[V], beta[V];
  int32_t g[V];
  affine<V>(a, t.c0, gamma, beta, g);
  const int64_t b = seg_begin(p, s), len = seg_end(p, s) - b;
  if (len <= 0) {
    for (int f = threadIdx.x; f < t.nf; f += kThreads) {
      p.mean[(int64_t)s * p.groups + t.gfirst + f] = 0.f;
      p.rstd[(int64_t)s * p.groups + t.gfirst + f] = 0.f;
    }
    return;
  }
  // rows in registers at a time; the last of them stay for the result, which takes the others in reverse
  const int held = kRows * t.ry;
  const bool live = t.left > 0 && t.ty < len;
  const float* src = p.X + b * p.ldx;
  const uint32_t off = t.off(p.ldx);
  Vals<V> x[kRows], first{};
  float sum[V] = {}, sq[V] = {};
  int64_t at = 0;
  auto load = [&]() {
    const float* row = src + at * p.ldx;
    const int mine = live ? (int)(len - at < held ? len - at : held) - t.ty : 0;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      x[k] = Vals<V>{};
      if (k * t.ry < mine) x[k] = load_raw<V>(row + (int64_t)k * t.ry * p.ldx, off);
    }
    loads_done();
    return mine;
  };
  int mine;
  for (;; at += held) {
    mine = load();
    if (at == 0 && live) first = clip_cols<V>(x[0], t.left);
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k * t.ry < mine) {
        const Vals<V> v = clip_cols<V>(x[k], t.left);  // here, so that no load is waited for on its own
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = v.v[j] - first.v[j];
          sum[j] += d;
          sq[j] += d * d;
        }
      }
    if (at + held >= len) break;
  }
  const float cnt = live ? (float)((len - t.ty + t.ry - 1) >> (8 - a.tx_log)) : 0.f, inv = live ? 1.f / cnt : 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    sum[j] *= inv;
    sq[j] -= sum[j] * (sum[j] * cnt);
  }
  join_threads(a, t, cnt, first.v, sum, sq, g, (float)len, box);
  const double share = 1.0 / ((double)len * (double)a.cg);
  for (int f = threadIdx.x; f < t.nf; f += kThreads) {
    finish_stats(box.mean[f], box.rest[f], box.dev[f], share, p.eps, box.mean[f], box.dev[f]);
    p.mean[(int64_t)s * p.groups + t.gfirst + f] = box.mean[f];
    p.rstd[(int64_t)s * p.groups + t.gfirst + f] = box.dev[f];
  }
  __syncthreads();
  if (t.left <= 0) return;
  float mean[V], sc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    mean[j] = box.mean[g[j] - t.gfirst];
    sc[j] = box.dev[g[j] - t.gfirst];
  }
  const uint32_t off_y = t.off(p.ldy);
  for (;;) {
    float* dst = p.Y + (b + at) * p.ldy;
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k * t.ry < mine) {
        Vals<V> y;
#pragma unroll
        for (int j = 0; j < V; ++j) y.v[j] = activate<ACT>(gamma[j] * ((x[k].v[j] - mean[j]) * sc[j]) + beta[j]);
        store_cols<V>(dst + (int64_t)k * t.ry * p.ldy, off_y, y, t.left);
      }
    if (at == 0) return;
    at -= held;
    mine = load();
  }
}

// Backward: a workgroup and one graph; x and dy of rows_bwd rows a thread are in registers at a time.
template <int V, int ACT>
__device__ __forceinline__ void norm_grad_one(const NormArgs& a, const Place<V>& t, int32_t s, const float* gamma,
                                              const float* beta, const int32_t* g, float* tot0, float* tot1, float* red0,
                                              float* red1, float* f0, float* f1) {
  constexpr int kRows = rows_bwd();
  const NormParams& p = a.p;
  const int64_t b = seg_begin(p, s), len = seg_end(p, s) - b;
  if (len <= 0) return;
  const float* sx = p.X + b * p.ldx;
  const float* sd = p.dY + b * p.lddy;
  const uint32_t off_x = t.off(p.ldx), off_d = t.off(p.lddy);
  // rows in registers at a time, normalised; the last of them stay for the result, which takes the others in
  // reverse
  const int held = kRows * t.ry;
  const bool live = t.left > 0 && t.ty < len;
  float s0[V], s1[V], mean[V], rstd[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    s0[j] = s1[j] = 0.f;
    mean[j] = p.mean[(int64_t)s * p.groups + g[j]];
    rstd[j] = p.rstd[(int64_t)s * p.groups + g[j]];
  }
  Vals<V> x[kRows], d[kRows];
  int64_t first = 0;
  auto load = [&]() {
    const float *rx = sx + first * p.ldx, *rd = sd + first * p.lddy;
    const int mine = live ? (int)(len - first < held ? len - first : held) - t.ty : 0;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      x[k] = d[k] = Vals<V>{};
      if (k * t.ry < mine) {
        x[k] = load_raw<V>(rx + (int64_t)k * t.ry * p.ldx, off_x);
        d[k] = load_raw<V>(rd + (int64_t)k * t.ry * p.lddy, off_d);
      }
    }
    loads_done();
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k * t.ry < mine) {
        x[k] = clip_cols<V>(x[k], t.left);
        d[k] = clip_cols<V>(d[k], t.left);
        normalise<V, ACT>(x[k], d[k], mean, rstd, gamma, beta);
      }
    return mine;
  };
  int mine;
  for (;; first += held) {
    mine = load();
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k * t.ry < mine)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          s0[j] += d[k].v[j];
          s1[j] += d[k].v[j] * x[k].v[j];
        }
    if (first + held >= len) break;
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int at = t.ty * a.pw + t.tx * V + j;
    red0[at] = gamma[j] * s0[j];
    red1[at] = gamma[j] * s1[j];
    tot0[j] += s0[j];
    tot1[j] += s1[j];
  }
  if (!p.dX) return;  // each thread writes its own places again: nothing to wait for
  __syncthreads();
  const float inv = 1.f / ((float)len * (float)a.cg);
  frag_sums(a, t.p0, t.gfirst, t.nf, t.ry, red0, [&](int f, float v) { f0[f] = v * inv; });
  frag_sums(a, t.p0, t.gfirst, t.nf, t.ry, red1, [&](int f, float v) { f1[f] = v * inv; });
  __syncthreads();
  if (t.left > 0) {
    float m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      m1[j] = f0[g[j] - t.gfirst];
      m2[j] = f1[g[j] - t.gfirst];
    }
    const uint32_t off = t.off(p.lddx);
    for (;;) {
      float* dst = p.dX + (b + first) * p.lddx;
#pragma unroll
      for (int k = 0; k < kRows; ++k)
        if (k * t.ry < mine) {
          Vals<V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) o.v[j] = rstd[j] * (gamma[j] * d[k].v[j] - m1[j] - x[k].v[j] * m2[j]);
          store_cols<V>(dst + (int64_t)k * t.ry * p.lddx, off, o, t.left);
        }
      if (first == 0) break;
      first -= held;
      mine = load();
    }
  }
  __syncthreads();  // f0 and f1 are read before the next graph's sums
}

// A workgroup takes a.rows consecutive graphs: their column sums leave it together.  4 wavefronts to a SIMD: one
// register more, and 262,144 x 128 in 8,192 graphs takes 160 us instead of 135.
template <int V, int ACT>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(4))) k_norm_grad_one(NormArgs a) {
  __shared__ float red0[kThreads * V];
  __shared__ float red1[kThreads * V];
  __shared__ float f0[kThreads * V];
  __shared__ float f1[kThreads * V];
  const Place<V> t(a);
  float gamma[V], beta[V], tot0[V] = {}, tot1[V] = {};
  int32_t g[V];
  affine<V>(a, t.c0, gamma, beta, g);
  for (int64_t s = (int64_t)blockIdx.x * a.rows; s < a.p.n_seg && s < (int64_t)(blockIdx.x + 1) * a.rows; ++s)
    norm_grad_one<V, ACT>(a, t, (int32_t)s, gamma, beta, g, tot0, tot1, red0, red1, f0, f1);
  write_columns(a, t, tot0, tot1, red0, red1);
}

// A wavefront per graph and panel: no LDS and no barrier, and its registers are free again when its graph is
// done, so that many graphs are under way on a CU at a time.  16-byte rows only; the lanes of a group are a
// power of two, or a lane holds SUB > 1 groups.
template <int SUB>
struct WavePlace {
  int tx, ty, ry, tx_lanes, group_lanes;
  int32_t c0, left, panel;
  __device__ __forceinline__ explicit WavePlace(const NormArgs& a) {
    const int lane = threadIdx.x & 63;
    tx_lanes = 1 << a.tx_log;
    tx = lane & (tx_lanes - 1);
    ty = lane >> a.tx_log;
    ry = 64 >> a.tx_log;
    panel = blockIdx.y;
    c0 = panel * a.pw + tx * 4;
    left = a.p.c - c0;
    group_lanes = SUB == 1 ? a.cg / 4 : 1;
  }
  __device__ __forceinline__ uint32_t off(int64_t ld) const { return ((uint32_t)ty * (uint32_t)ld + (uint32_t)c0) * 4; }
  // Sums of a lane's four values over their groups and all rows, at every lane.
  __device__ __forceinline__ void sums(float v[4]) const {
    if constexpr (SUB == 1) v[0] = v[1] = v[2] = v[3] = (v[0] + v[1]) + (v[2] + v[3]);
    if constexpr (SUB == 2) {
      v[0] = v[1] = v[0] + v[1];
      v[2] = v[3] = v[2] + v[3];
    }
#pragma unroll
    for (int k = 0; k < SUB; ++k) {
      float x = v[k * 4 / SUB];
      for (int o = 1; o < group_lanes; o <<= 1) x += __shfl_xor(x, o, 64);
      for (int o = tx_lanes; o < 64; o <<= 1) x += __shfl_xor(x, o, 64);
#pragma unroll
      for (int j = 0; j < 4 / SUB; ++j) v[k * 4 / SUB + j] = x;
    }
  }
};

template <int ACT, int SUB>
__global__ void __launch_bounds__(64) k_norm_wave(NormArgs a) {
  constexpr int kRows = rows_fwd(64);
  const NormParams& p = a.p;
  const WavePlace<SUB> t(a);
  const int64_t s = blockIdx.x;
  const int64_t b = seg_begin(p, (int32_t)s), end = seg_end(p, (int32_t)s);
  const int64_t len = end > b ? end - b : 0;
  float gamma[4], beta[4];
  int32_t g[4];
  affine<4>(a, t.c0, gamma, beta, g);
  const float* src = p.X + b * p.ldx;
  const uint32_t off = t.off(p.ldx);
  // rows in registers at a time; the last of them stay for the result, which takes the others in reverse
  const int held = kRows * t.ry;
  const bool live = t.left > 0 && t.ty < len;
  Vals<4> x[kRows], first{};
  float sum[4] = {}, sq[4] = {}, cnt = 0.f;
  int64_t at = 0;
  auto load = [&]() {
    const float* row = src + at * p.ldx;
    const int mine = live ? (int)(len - at < held ? len - at : held) - t.ty : 0;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      x[k] = Vals<4>{};
      if (k * t.ry < mine) x[k] = load_raw<4>(row + (int64_t)k * t.ry * p.ldx, off);
    }
    loads_done();
    return mine;
  };
  int mine;
  for (;; at += held) {
    mine = load();
    if (at == 0 && live) first = clip_cols<4>(x[0], t.left);
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k * t.ry < mine) {
        const Vals<4> v = clip_cols<4>(x[k], t.left);  // here, so that no load is waited for on its own
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float d = v.v[j] - first.v[j];
          sum[j] += d;
          sq[j] += d * d;
        }
      }
    if (at + held >= len) break;
  }
  if (live) cnt = (float)((len - t.ty + t.ry - 1) >> (6 - a.tx_log));
  // joined as in join_threads: distances from one value of the group, and then from the mean that this gives
  const float inv = cnt > 0.f ? 1.f / cnt : 0.f, all = 1.f / fmaxf((float)len * (float)a.cg, 1.f);
  float center[4], rest[4], dev[4];
#pragma unroll
  for (int k = 0; k < SUB; ++k) {
    const float v = __shfl(first.v[k * 4 / SUB], t.tx & ~(t.group_lanes - 1), 64);
#pragma unroll
    for (int j = 0; j < 4 / SUB; ++j) center[k * 4 / SUB + j] = v;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    sum[j] *= inv;
    rest[j] = cnt * ((first.v[j] - center[j]) + sum[j]);
  }
  t.sums(rest);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    center[j] += rest[j] * all;
    const float d = (first.v[j] - center[j]) + sum[j];
    rest[j] = cnt * d;
    dev[j] = sq[j] - sum[j] * (sum[j] * cnt) + cnt * d * d;
  }
  t.sums(rest);
  t.sums(dev);
  float fm[4], sc[4];
  const double share = 1.0 / ((double)len * (double)a.cg);
#pragma unroll
  for (int k = 0; k < SUB; ++k) {
    float m = 0.f, r = 0.f;
    if (len > 0) finish_stats(center[k * 4 / SUB], rest[k * 4 / SUB], dev[k * 4 / SUB], share, p.eps, m, r);
#pragma unroll
    for (int j = 0; j < 4 / SUB; ++j) {
      fm[k * 4 / SUB + j] = m;
      sc[k * 4 / SUB + j] = r;
    }
    // the first lane of the group in the first row
    if (t.left > k * 4 / SUB && t.ty == 0 && (t.tx & (t.group_lanes - 1)) == 0) {
      p.mean[s * p.groups + g[k * 4 / SUB]] = m;
      p.rstd[s * p.groups + g[k * 4 / SUB]] = r;
    }
  }
  const uint32_t off_y = t.off(p.ldy);
  for (;;) {
    float* dst = p.Y + (b + at) * p.ldy;
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k * t.ry < mine) {
        Vals<4> y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y.v[j] = activate<ACT>(gamma[j] * ((x[k].v[j] - fm[j]) * sc[j]) + beta[j]);
        store_cols<4>(dst + (int64_t)k * t.ry * p.ldy, off_y, y, t.left);
      }
    if (at == 0) return;
    at -= held;
    mine = load();
  }
}

template <int ACT>
void launch(NormArgs a, bool vec, hipStream_t s) {
  const dim3 grid((unsigned)a.p.n_seg, (unsigned)a.n_panel);
  if (a.one == 64) {
    if (a.cg == 1)
      hipLaunchKernelGGL((k_norm_wave<ACT, 4>), grid, dim3(64), 0, s, a);
    else if (a.cg == 2)
      hipLaunchKernelGGL((k_norm_wave<ACT, 2>), grid, dim3(64), 0, s, a);
    else
      hipLaunchKernelGGL((k_norm_wave<ACT, 1>), grid, dim3(64), 0, s, a);
    return;
  }
  if (vec)
    hipLaunchKernelGGL((k_norm_one<4, ACT>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_norm_one<1, ACT>), grid, dim3(kThreads), 0, s, a);
}

template <int ACT>
void launch_grad(const NormArgs& a, bool vec, hipStream_t s) {
  const dim3 grid((unsigned)a.n_block, (unsigned)a.n_panel);
  if (vec)
    hipLaunchKernelGGL((k_norm_grad_one<4, ACT>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_norm_grad_one<1, ACT>), grid, dim3(kThreads), 0, s, a);
}

}  // namespace

void launch_norm_one(const NormArgs& a, bool vec, hipStream_t s) {
  if (a.p.act == GCN_ACT_RELU) launch<GCN_ACT_RELU>(a, vec, s);
  else if (a.p.act == GCN_ACT_SILU) launch<GCN_ACT_SILU>(a, vec, s);
  else launch<GCN_ACT_NONE>(a, vec, s);
}
void launch_norm_grad_one(const NormArgs& a, bool vec, hipStream_t s) {
  if (a.p.act == GCN_ACT_RELU) launch_grad<GCN_ACT_RELU>(a, vec, s);
  else if (a.p.act == GCN_ACT_SILU) launch_grad<GCN_ACT_SILU>(a, vec, s);
  else launch_grad<GCN_ACT_NONE>(a, vec, s);
}

}  // namespace gcn
