// Group normalisation with the activation behind it, channels last, and its backward pass.
//
// With m = positions x channels of a group of an image:
//   mean = sum x / m,  r = 1 / sqrt(sum (x - mean)^2 / m + eps),  z = (x - mean) r scale + shift,  y = act(z)
//   dz = dy act'(z),  xhat = (x - mean) r,  dshift = sum dz,  dscale = sum dz xhat  (over images and positions)
//   dx = r (scale dz - (s1 + xhat s2) / m),  s1 = sum scale dz,  s2 = sum scale dz xhat  (over the group)
// Bound by HBM: x in and y out, or x and dy in and dx out.  A group's statistics need all of its values before the first is
// written, so where a workgroup can hold them in registers they are read once ("whole"); where it cannot, a first launch
// leaves statistics of chunks of positions and a second one reads the values again (from the memory-side cache, as far as they fit).
//
// Sums go channel by channel: a lane owns 16 bytes of channels at a fixed place of the pixel and walks positions, the rows of lanes
// are added through LDS in a fixed order, and groups are put together from their channels, whatever number of channels a group has.
// Variances are sums of squared distances from the mean of what is summed, joined by
// sum of those + sum of count x (mean - joint mean)^2, from lanes to channels to groups: no difference of large sums.
#include "dev_common.hpp"
#include "operators.hpp"

#include <algorithm>
#include <type_traits>

#include "../../include/sasgd.h"

namespace sasgd {

namespace {

template <typename T, int V> struct Raw;
template <> struct Raw<float, 4> { typedef float4 type; };
template <> struct Raw<bf16_t, 8> { typedef uint4 type; };
template <> struct Raw<float, 1> { typedef float type; };
template <> struct Raw<bf16_t, 1> { typedef bf16_t type; };

__device__ __forceinline__ void unpack(const float4& r, float (&f)[4]) { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
__device__ __forceinline__ void unpack(const uint4& r, float (&f)[8]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int k = 0; k < 4; k++) {
    f[2 * k] = __uint_as_float(w[k] << 16);
    f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(float r, float (&f)[1]) { f[0] = r; }
__device__ __forceinline__ void unpack(bf16_t r, float (&f)[1]) { f[0] = bf2f(r); }
__device__ __forceinline__ void pack(float4& r, const float (&f)[4]) { r = make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void pack(uint4& r, const float (&f)[8]) {
  r = make_uint4(pack2bf(f[0], f[1]), pack2bf(f[2], f[3]), pack2bf(f[4], f[5]), pack2bf(f[6], f[7]));
}
__device__ __forceinline__ void pack(float& r, const float (&f)[1]) { r = f[0]; }
__device__ __forceinline__ void pack(bf16_t& r, const float (&f)[1]) { r = f2bf(f[0]); }

// 1 / (1 + exp(-z)) by the hardware's exponential and reciprocal (1 ulp each)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }

template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == SASGD_ACT_RELU) return z <= 0.f ? 0.f : z;         // (NaN stays)
  if (ACT == SASGD_ACT_SILU) return z * sigmoid(z);
  return z;
}
// z from x - mean.  Behind a ReLU each operation is rounded by itself: forward and backward pass (and whoever computes z by the formula) agree
// on its sign.  Elsewhere r scale is one factor.
template <int ACT>
__device__ __forceinline__ float affine(float xc, float r, float scale, float slope, float shift) {
  if (ACT == SASGD_ACT_RELU) {
#pragma clang fp contract(off)
    return xc * r * scale + shift;
  }
  return fmaf(xc, slope, shift);
}
// dz = dy act'(z)
template <int ACT>
__device__ __forceinline__ float through(float d, float z) {
  if (ACT == SASGD_ACT_RELU) return z > 0.f ? d : 0.f;
  if (ACT == SASGD_ACT_SILU) {
    const float s = sigmoid(z);
    return d * fmaf(z, fmaf(-s, s, s), s);
  }
  return d;
}

__device__ __forceinline__ float param(const GroupNormArgs& A, uintptr_t at, int c) {
  return A.param_bf16 ? bf2f(((const bf16_t*)at)[c]) : ((const float*)at)[c];
}

constexpr int kLaneChannels = 64;    // channels of a group up to which one lane adds them

// Which image of a learner, and which slab of its channels or chunk of its positions, a workgroup works on.  Parts of one image are eight
// workgroups apart: they run on one XCD at about the same time, where narrow slabs share the lines of L2.
struct Place {
  int64_t image;
  int part;
};
__device__ __forceinline__ bool place_of(const GroupNormArgs& A, int parts, Place& p) {
  if (parts == 1) {
    p.image = blockIdx.x;
    p.part = 0;
    return true;
  }
  const uint32_t b = blockIdx.x, eighth = b >> 3, group = eighth / (uint32_t)parts;
  p.image = (int64_t)group * 8 + (b & 7);
  p.part = (int)(eighth - group * (uint32_t)parts);
  return p.image < A.s.images;
}

// Columns of lanes: lane t has vector `col` of a pixel in row `row` of the workgroup's lanes, and positions row, row + rows, ...
struct Lanes {
  int cols, rows, row, col;
  bool active;
};
__device__ __forceinline__ Lanes lanes_of(const GroupNormCols& c, int t) {
  Lanes l;
  l.cols = c.cols;
  l.rows = c.rows;
  l.row = c.by_cols(t);
  l.col = t - l.row * c.cols;
  l.active = l.row < c.rows;
  return l;
}

// Sum over the wavefront, in every lane: shifts within rows of 16 lanes, then rows to rows, without a trip through LDS.
__device__ __forceinline__ float wave_total(float v) {
#define STEP(ctrl, rows) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, true));
  STEP(0x111, 0xf) STEP(0x112, 0xf) STEP(0x114, 0xf) STEP(0x118, 0xf) STEP(0x142, 0xa) STEP(0x143, 0xc)
#undef STEP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sums over the rows of lanes, channel by channel (n = cols V of them), of K quantities at a time; lane (seg, c) adds the rows
// seg, seg + segs, ... of channel c, then the segments are added.  value(k, row, c): what to add; out[k stride + c].  red: K threads floats.
template <int K, typename F>
__device__ __forceinline__ void row_sums(const GroupNormCols& cols, int n, float* red, float* out, int stride, F value) {
  const int t = threadIdx.x, T = blockDim.x, segs = cols.segs;
  if (segs > 1) {
    const int seg = cols.by_n(t), c = t - seg * n;
    float s[K];
#pragma unroll
    for (int k = 0; k < K; k++) s[k] = 0.f;
    if (seg < segs)
      for (int r = seg; r < cols.rows; r += segs)
#pragma unroll
        for (int k = 0; k < K; k++) s[k] += value(k, r, c);
    int left = segs;
    if (cols.fold) {                                 // n is a power of two below 64: first within the wavefront
      for (int o = n; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < K; k++) s[k] += __shfl_xor(s[k], o, 64);
      left = T >> 6;
    }
    const bool mine = cols.fold ? (t & 63) < n : seg < segs;
    const int at = cols.fold ? (t >> 6) * n + c : t;
    if (mine)
#pragma unroll
      for (int k = 0; k < K; k++) red[k * T + at] = s[k];
    __syncthreads();
    if (t < n)
#pragma unroll
      for (int k = 0; k < K; k++) {
        float a = 0.f;
        for (int q = 0; q < left; q++) a += red[k * T + q * n + t];
        out[k * stride + t] = a;
      }
  } else {
    for (int c = t; c < n; c += T)
#pragma unroll
      for (int k = 0; k < K; k++) {
        float a = 0.f;
        for (int r = 0; r < cols.rows; r++) a += value(k, r, c);
        out[k * stride + c] = a;
      }
  }
  __syncthreads();
}

// Mean and sum of squared distances of every channel of `np` positions from what lanes have of them: lane sums `sum` of `count` values and
// squared distances `dev` from the lane's own mean.  mean[c], dev[c]; rows: 2 threads V floats, red: threads floats.
template <int V>
__device__ __forceinline__ void channel_moments(const float (&sum)[V], const float (&dev)[V], const GroupNormCols& cols, const Lanes& l, int np, float* rows,
                                                float* red, float* mean, float* m2) {
  const int n = cols.cols * V;
  float* rd = rows + cols.rows * n;
  if (l.active)
#pragma unroll
    for (int j = 0; j < V; j++) {
      rows[l.row * n + l.col * V + j] = sum[j];
      rd[l.row * n + l.col * V + j] = dev[j];
    }
  __syncthreads();
  row_sums<1>(cols, n, red, mean, 0, [&](int, int r, int c) { return rows[r * n + c]; });
  const float inv = 1.f / (float)np;
  for (int c = threadIdx.x; c < n; c += blockDim.x) mean[c] *= inv;
  __syncthreads();
  // a row has its share of the positions, the first ones one more
  const int each = np / cols.rows, more = np - each * cols.rows;
  const float one = each > 0 ? 1.f / (float)each : 0.f, plus = 1.f / (float)(each + 1);
  row_sums<1>(cols, n, red, m2, 0, [&](int, int r, int c) {
    const float count = (float)(each + (r < more)), off = rows[r * n + c] * (r < more ? plus : one) - mean[c];
    return rd[r * n + c] + (count > 0.f ? count * off * off : 0.f);
  });
}

// The workgroup's groups from the moments of their channels (mean[c], m2[c] of `np` values each): done(g, mean, sum of squared distances).  A lane a
// group, or a wavefront a group where they have many channels (320 channels in 32 groups by wavefronts: 4 us of a workgroup's 9).
template <typename F>
__device__ __forceinline__ void group_moments(const float* mean, const float* m2, int groups, int cpg, int np, F done) {
  const int t = threadIdx.x, T = blockDim.x;
  if (cpg <= kLaneChannels) {
    for (int g = t; g < groups; g += T) {
      float s = 0.f, d = 0.f, off = 0.f;
      for (int c = g * cpg; c < (g + 1) * cpg; c++) {
        s += mean[c];
        d += m2[c];
      }
      const float mu = s / (float)cpg;
      for (int c = g * cpg; c < (g + 1) * cpg; c++) off += (mean[c] - mu) * (mean[c] - mu);
      done(g, mu, d + (float)np * off);
    }
    return;
  }
  const int lane = t & 63;
  for (int g = t >> 6; g < groups; g += T >> 6) {
    float s = 0.f, d = 0.f, off = 0.f;
    for (int c = g * cpg + lane; c < (g + 1) * cpg; c += 64) {
      s += mean[c];
      d += m2[c];
    }
    const float mu = wave_total(s) / (float)cpg;
    for (int c = g * cpg + lane; c < (g + 1) * cpg; c += 64) off += (mean[c] - mu) * (mean[c] - mu);
    const float m = wave_total(d) + (float)np * wave_total(off);
    if (lane == 0) done(g, mu, m);
  }
}

template <typename T, int V>
__device__ __forceinline__ void add_moments(const typename Raw<T, V>::type& raw, const float (&first)[V], float (&s)[V], float (&q)[V]) {
  float f[V];
  unpack(raw, f);
#pragma unroll
  for (int j = 0; j < V; j++) {
    const float e = f[j] - first[j];
    s[j] += e;
    q[j] = fmaf(e, e, q[j]);
  }
}
// From sums of distances from the lane's first value to the sum and the squared distances from the lane's mean: the cancellation costs
// at most `count` roundings of the result, as no value is further from the mean than the root of count variances.
template <int V>
__device__ __forceinline__ void close_moments(const float (&first)[V], float (&s)[V], float (&q)[V], int count) {
  const float n = (float)count, inv = count > 0 ? 1.f / n : 0.f;
#pragma unroll
  for (int j = 0; j < V; j++) {
    q[j] = fmaxf(q[j] - s[j] * s[j] * inv, 0.f);
    s[j] = count > 0 ? fmaf(first[j], n, s[j]) : 0.f;
  }
}
__device__ __forceinline__ int count_of(const Lanes& l, int np) { return l.active && l.row < np ? (np - 1 - l.row) / l.rows + 1 : 0; }

// ------------------------------------------------------------------------------------------------ forward
// A workgroup holds a slab of an image.  LDS: rows [2 threads V], red [threads], mean [S], m2 [S], group [2 S / cpg]
template <typename T, int V, int NV, int ACT>
__global__ __launch_bounds__(V == 1 ? 1024 : 256, V == 1 ? 1 : 2) void group_norm_kernel(const GroupNormArgs A) {
  extern __shared__ float lds[];
  typedef typename Raw<T, V>::type raw_t;
  Place at;
  if (!place_of(A, A.plan.slabs, at)) return;
  const uintptr_t base = A.base[blockIdx.y], wts = A.wts[blockIdx.y];
  const int C = A.s.channels, cpg = A.cpg;
  const int c0 = at.part * A.plan.slab, S = min(A.plan.slab, C - c0), np = A.s.positions;
  const GroupNormCols cols = A.cols[at.part == A.plan.slabs - 1];
  const int t = threadIdx.x, threads = blockDim.x;
  float* rows = lds;
  float* red = rows + 2 * threads * V;
  float* mean = red + threads;
  float* m2 = mean + S;
  float* group = m2 + S;
  const Lanes l = lanes_of(cols, t);
  const int count = count_of(l, np), first_c = l.col * V;
  const T* x = (const T*)(base + A.x) + at.image * A.x_image + l.row * A.x_pixel + c0 + first_c;
  const int64_t step = l.rows * A.x_pixel;
  raw_t held[NV];
#pragma unroll
  for (int k = 0; k < NV; k++)
    if (k < count) held[k] = *(const raw_t*)(x + k * step);
  float sc[V], sh[V];
#pragma unroll
  for (int j = 0; j < V; j++) {
    sc[j] = A.has_scale && l.active ? param(A, wts + A.scale, c0 + first_c + j) : 1.f;
    sh[j] = A.has_shift && l.active ? param(A, wts + A.shift, c0 + first_c + j) : 0.f;
  }
  {
    float first[V], s[V], q[V];
#pragma unroll
    for (int j = 0; j < V; j++) first[j] = s[j] = q[j] = 0.f;
    if (count > 0) unpack(held[0], first);
#pragma unroll
    for (int k = 1; k < NV; k++)
      if (k < count) add_moments<T, V>(held[k], first, s, q);
    close_moments<V>(first, s, q, count);
    channel_moments<V>(s, q, cols, l, np, rows, red, mean, m2);
  }
  group_moments(mean, m2, A.by_cpg(S), cpg, np, [&](int g, float mu, float sq) {
    const float r = 1.f / sqrtf(sq / ((float)np * (float)cpg) + A.eps);
    group[2 * g] = mu;
    group[2 * g + 1] = r;
    if (A.has_stats) ((float2*)(base + A.stats))[at.image * A.s.groups + A.by_cpg(c0) + g] = make_float2(mu, r);
  });
  __syncthreads();
  if (count == 0) return;
  float mu[V], r[V], slope[V];
#pragma unroll
  for (int j = 0; j < V; j++) {
    const int g = A.by_cpg(first_c + j);
    mu[j] = group[2 * g];
    r[j] = group[2 * g + 1];
    slope[j] = r[j] * sc[j];
  }
  T* y = (T*)(base + A.y) + at.image * A.y_image + l.row * A.y_pixel + c0 + first_c;
  const int64_t ystep = l.rows * A.y_pixel;
#pragma unroll
  for (int k = 0; k < NV; k++)
    if (k < count) {
      float f[V];
      unpack(held[k], f);
#pragma unroll
      for (int j = 0; j < V; j++) f[j] = activate<ACT>(affine<ACT>(f[j] - mu[j], r[j], sc[j], slope[j], sh[j]));
      raw_t o;
      pack(o, f);
      *(raw_t*)(y + k * ystep) = o;
    }
}

// Images that no workgroup can hold, first launch: the moments of a chunk of positions.  LDS: rows, red, mean [C], m2 [C]
template <typename T, int V>
__global__ __launch_bounds__(256) void group_norm_chunk_kernel(const GroupNormArgs A) {
  extern __shared__ float lds[];
  typedef typename Raw<T, V>::type raw_t;
  Place at;
  if (!place_of(A, A.plan.chunks, at)) return;
  const uintptr_t base = A.base[blockIdx.y];
  const int C = A.s.channels, cpg = A.cpg, p0 = at.part * A.plan.chunk, np = min(A.plan.chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  float* rows = lds;
  float* red = rows + 2 * threads * V;
  float* mean = red + threads;
  float* m2 = mean + C;
  const T* x0 = (const T*)(base + A.x) + at.image * A.x_image + (int64_t)p0 * A.x_pixel;
  for (int c0 = 0; c0 < C; c0 += A.cols[0].cols * V) {      // (one turn up to `threads` vectors a pixel)
    const GroupNormCols cols = A.cols[c0 + A.cols[0].cols * V >= C];
    const Lanes l = lanes_of(cols, t);
    const int count = count_of(l, np);
    const T* x = x0 + l.row * A.x_pixel + c0 + l.col * V;
    const int64_t step = l.rows * A.x_pixel;
    float first[V], s[V], q[V];
#pragma unroll
    for (int j = 0; j < V; j++) first[j] = s[j] = q[j] = 0.f;
    if (count > 0) unpack(*(const raw_t*)x, first);
    int k = 1;
    constexpr int U = 8;
    for (; k + U <= count; k += U) {
      raw_t in[U];
#pragma unroll
      for (int i = 0; i < U; i++) in[i] = *(const raw_t*)(x + (k + i) * step);
#pragma unroll
      for (int i = 0; i < U; i++) add_moments<T, V>(in[i], first, s, q);
    }
    for (; k < count; k++) add_moments<T, V>(*(const raw_t*)(x + k * step), first, s, q);
    close_moments<V>(first, s, q, count);
    channel_moments<V>(s, q, cols, l, np, rows, red, mean + c0, m2 + c0);
  }
  float2* parts = (float2*)(base + A.parts) + (at.image * A.plan.chunks + at.part) * A.s.groups;
  group_moments(mean, m2, A.s.groups, cpg, np, [&](int g, float mu, float sq) { parts[g] = make_float2(mu, sq); });
}

// Second launch: the image's statistics from its chunks', then y.  LDS: group [2 groups]
template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void group_norm_apply_kernel(const GroupNormArgs A) {
  extern __shared__ float group[];
  typedef typename Raw<T, V>::type raw_t;
  Place at;
  if (!place_of(A, A.plan.chunks, at)) return;
  const uintptr_t base = A.base[blockIdx.y], wts = A.wts[blockIdx.y];
  const int C = A.s.channels, G = A.s.groups, chunk = A.plan.chunk, chunks = A.plan.chunks;
  const int p0 = at.part * chunk, np = min(chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  const float2* parts = (const float2*)(base + A.parts) + at.image * chunks * G;
  const float last = (float)(A.s.positions - (chunks - 1) * chunk), full = (float)chunk, total = (float)A.s.positions, cpg = (float)A.cpg;
  for (int i = t; i < G * A.spread; i += threads) {          // `spread` neighbouring lanes a group
    const int g = i / A.spread, first = i - g * A.spread;
    float s = 0.f, m2 = 0.f;
    for (int k = first; k < chunks; k += A.spread) s += parts[k * G + g].x * (k < chunks - 1 ? full : last);
    for (int o = 1; o < A.spread; o <<= 1) s += __shfl_xor(s, o, 64);
    const float mu = s / total;
    for (int k = first; k < chunks; k += A.spread) {
      const float2 p = parts[k * G + g];
      m2 += p.y + (k < chunks - 1 ? full : last) * cpg * (p.x - mu) * (p.x - mu);
    }
    for (int o = 1; o < A.spread; o <<= 1) m2 += __shfl_xor(m2, o, 64);
    if (first == 0) {
      const float r = 1.f / sqrtf(m2 / (total * cpg) + A.eps);
      group[2 * g] = mu;
      group[2 * g + 1] = r;
      if (A.has_stats && at.part == 0) ((float2*)(base + A.stats))[at.image * G + g] = make_float2(mu, r);
    }
  }
  __syncthreads();
  for (int c0 = 0; c0 < C; c0 += A.cols[0].cols * V) {
    const Lanes l = lanes_of(A.cols[c0 + A.cols[0].cols * V >= C], t);
    const int count = count_of(l, np), c = c0 + l.col * V;
    if (count == 0) continue;
    float mu[V], r[V], sc[V], sh[V], slope[V];
#pragma unroll
    for (int j = 0; j < V; j++) {
      const int g = A.by_cpg(c + j);
      mu[j] = group[2 * g];
      r[j] = group[2 * g + 1];
      sc[j] = A.has_scale ? param(A, wts + A.scale, c + j) : 1.f;
      sh[j] = A.has_shift ? param(A, wts + A.shift, c + j) : 0.f;
      slope[j] = r[j] * sc[j];
    }
    const T* x = (const T*)(base + A.x) + at.image * A.x_image + (int64_t)(p0 + l.row) * A.x_pixel + c;
    T* y = (T*)(base + A.y) + at.image * A.y_image + (int64_t)(p0 + l.row) * A.y_pixel + c;
    const int64_t step = l.rows * A.x_pixel, ystep = l.rows * A.y_pixel;
    auto one = [&](const raw_t& in, int k) {
      float f[V];
      unpack(in, f);
#pragma unroll
      for (int j = 0; j < V; j++) f[j] = activate<ACT>(affine<ACT>(f[j] - mu[j], r[j], sc[j], slope[j], sh[j]));
      raw_t o;
      pack(o, f);
      *(raw_t*)(y + k * ystep) = o;
    };
    constexpr int U = 4;
    int k = 0;
    for (; k + U <= count; k += U) {
      raw_t in[U];
#pragma unroll
      for (int i = 0; i < U; i++) in[i] = *(const raw_t*)(x + (k + i) * step);
#pragma unroll
      for (int i = 0; i < U; i++) one(in[i], k + i);
    }
    for (; k < count; k++) one(*(const raw_t*)(x + k * step), k);
  }
}

// ------------------------------------------------------------------------------------------------ backward
// dx = dz a + (x - mean) c + b with a = r scale, b = - r s1 / m, c = - r^2 s2 / m
template <int V>
struct GradientLane {
  float mu[V], r[V], sc[V], sh[V], slope[V];
};
template <int V>
__device__ __forceinline__ void load_lane(const GroupNormArgs& A, uintptr_t base, uintptr_t wts, int64_t image, int c, GradientLane<V>& p) {
  const float2* stats = (const float2*)(base + A.stats) + image * A.s.groups;
#pragma unroll
  for (int j = 0; j < V; j++) {
    const float2 st = stats[A.by_cpg(c + j)];
    p.mu[j] = st.x;
    p.r[j] = st.y;
    p.sc[j] = A.has_scale ? param(A, wts + A.scale, c + j) : 1.f;
    p.sh[j] = A.has_shift ? param(A, wts + A.shift, c + j) : 0.f;
    p.slope[j] = p.r[j] * p.sc[j];
  }
}

// dz of a vector, its sums and those of dz (x - mean) added to a and b; d becomes dz
template <int V, int ACT>
__device__ __forceinline__ void add_gradient(const float (&f)[V], float (&d)[V], const GradientLane<V>& p, float (&a)[V], float (&b)[V]) {
#pragma unroll
  for (int j = 0; j < V; j++) {
    const float xc = f[j] - p.mu[j];
    d[j] = through<ACT>(d[j], ACT == SASGD_ACT_NONE ? 0.f : affine<ACT>(xc, p.r[j], p.sc[j], p.slope[j], p.sh[j]));
    a[j] += d[j];
    b[j] = fmaf(d[j], xc, b[j]);
  }
}

// Channel sums of dz and dz xhat of the workgroup: out[c], out[stride + c].  rows: 2 threads V floats, red: 2 threads.
template <int V>
__device__ __forceinline__ void gradient_sums(const float (&a)[V], const float (&b)[V], const GradientLane<V>& p, const GroupNormCols& cols, const Lanes& l,
                                              float* rows, float* red, float* out, int stride) {
  const int n = cols.cols * V;
  float* rb = rows + cols.rows * n;
  if (l.active)
#pragma unroll
    for (int j = 0; j < V; j++) {
      rows[l.row * n + l.col * V + j] = a[j];
      rb[l.row * n + l.col * V + j] = b[j] * p.r[j];
    }
  __syncthreads();
  row_sums<2>(cols, n, red, out, stride, [&](int k, int r, int c) { return (k ? rb : rows)[r * n + c]; });
}

// s1 and s2 of the workgroup's groups from its channels' sums (the first is channel c0 of the image): done(g, s1, s2)
template <typename F>
__device__ __forceinline__ void group_gradient(const GroupNormArgs& A, uintptr_t wts, const float* sa, const float* sb, int c0, int groups, F done) {
  const int t = threadIdx.x, T = blockDim.x, cpg = A.cpg;
  if (cpg <= kLaneChannels) {
    for (int g = t; g < groups; g += T) {
      float s1 = 0.f, s2 = 0.f;
      for (int c = g * cpg; c < (g + 1) * cpg; c++) {
        const float w = A.has_scale ? param(A, wts + A.scale, c0 + c) : 1.f;
        s1 = fmaf(w, sa[c], s1);
        s2 = fmaf(w, sb[c], s2);
      }
      done(g, s1, s2);
    }
    return;
  }
  const int lane = t & 63;
  for (int g = t >> 6; g < groups; g += T >> 6) {
    float s1 = 0.f, s2 = 0.f;
    for (int c = g * cpg + lane; c < (g + 1) * cpg; c += 64) {
      const float w = A.has_scale ? param(A, wts + A.scale, c0 + c) : 1.f;
      s1 = fmaf(w, sa[c], s1);
      s2 = fmaf(w, sb[c], s2);
    }
    s1 = wave_total(s1);
    s2 = wave_total(s2);
    if (lane == 0) done(g, s1, s2);
  }
}

// What a lane keeps of dy between the sums and dx: dz.  Behind a ReLU or nothing that is dy or 0 and stays in its type, behind silu fp32.
template <typename T, int V, int ACT> struct Kept { typedef typename Raw<T, V>::type type; };
template <> struct Kept<bf16_t, 8, SASGD_ACT_SILU> { struct type { float f[8]; }; };
template <> struct Kept<bf16_t, 1, SASGD_ACT_SILU> { typedef float type; };
__device__ __forceinline__ void unpack(const Kept<bf16_t, 8, SASGD_ACT_SILU>::type& r, float (&f)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j++) f[j] = r.f[j];
}
__device__ __forceinline__ void keep(Kept<bf16_t, 8, SASGD_ACT_SILU>::type& r, const float (&f)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j++) r.f[j] = f[j];
}
__device__ __forceinline__ void keep(float4& r, const float (&f)[4]) { pack(r, f); }
__device__ __forceinline__ void keep(float& r, const float (&f)[1]) { r = f[0]; }
__device__ __forceinline__ void keep(bf16_t& r, const float (&f)[1]) { r = f2bf(f[0]); }
__device__ __forceinline__ void keep(uint4& r, const float (&f)[8]) {      // values that are bf16 already: their upper halves
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; k++) w[k] = __builtin_amdgcn_perm(__float_as_uint(f[2 * k + 1]), __float_as_uint(f[2 * k]), 0x07060302);
  r = make_uint4(w[0], w[1], w[2], w[3]);
}

// A workgroup holds a slab of x and dy.  LDS: rows [2 threads V], red [2 threads], sa [S], sb [S], group [2 S / cpg]
template <typename T, int V, int NV, int ACT>
__global__ __launch_bounds__(V == 1 ? 1024 : 256, V == 1 ? 1 : 2) void group_norm_gradient_kernel(const GroupNormArgs A) {
  extern __shared__ float lds[];
  typedef typename Raw<T, V>::type raw_t;
  Place at;
  if (!place_of(A, A.plan.slabs, at)) return;
  const uintptr_t base = A.base[blockIdx.y], wts = A.wts[blockIdx.y];
  const int C = A.s.channels;
  const int c0 = at.part * A.plan.slab, S = min(A.plan.slab, C - c0), np = A.s.positions;
  const GroupNormCols cols = A.cols[at.part == A.plan.slabs - 1];
  const int t = threadIdx.x, threads = blockDim.x;
  float* rows = lds;
  float* red = rows + 2 * threads * V;
  float* sums = red + 2 * threads;
  float* group = sums + 2 * S;
  const Lanes l = lanes_of(cols, t);
  const int count = count_of(l, np), first_c = l.col * V;
  const T* x = (const T*)(base + A.x) + at.image * A.x_image + l.row * A.x_pixel + c0 + first_c;
  const T* dy = (const T*)(base + A.dy) + at.image * A.y_image + l.row * A.y_pixel + c0 + first_c;
  const int64_t step = l.rows * A.x_pixel, ystep = l.rows * A.y_pixel;
  raw_t hx[NV];
  typename Kept<T, V, ACT>::type hz[NV];
  GradientLane<V> p;
  {
    raw_t hd[NV];
#pragma unroll
    for (int k = 0; k < NV; k++)
      if (k < count) {
        hx[k] = *(const raw_t*)(x + k * step);
        hd[k] = *(const raw_t*)(dy + k * ystep);
      }
    if (l.active) load_lane<V>(A, base, wts, at.image, c0 + first_c, p);
    float a[V], b[V];
#pragma unroll
    for (int j = 0; j < V; j++) a[j] = b[j] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++)
      if (k < count) {
        float f[V], d[V];
        unpack(hx[k], f);
        unpack(hd[k], d);
        add_gradient<V, ACT>(f, d, p, a, b);
        keep(hz[k], d);
      }
    gradient_sums<V>(a, b, p, cols, l, rows, red, sums, S);
  }
  {
    float2* out = (float2*)(base + A.sums) + at.image * C + c0;
    for (int c = t; c < S; c += threads) out[c] = make_float2(sums[S + c], sums[c]);
  }
  if (!A.has_dx) return;
  group_gradient(A, wts, sums, sums + S, c0, A.by_cpg(S), [&](int g, float s1, float s2) {
    group[2 * g] = s1;
    group[2 * g + 1] = s2;
  });
  __syncthreads();
  if (count == 0) return;
  const float inv = 1.f / ((float)np * (float)A.cpg);
  float b[V], c[V];
#pragma unroll
  for (int j = 0; j < V; j++) {
    const int g = A.by_cpg(first_c + j);
    b[j] = -p.r[j] * (group[2 * g] * inv);
    c[j] = -p.r[j] * p.r[j] * (group[2 * g + 1] * inv);
  }
  T* dx = (T*)(base + A.dx) + at.image * A.y_image + l.row * A.y_pixel + c0 + first_c;
#pragma unroll
  for (int k = 0; k < NV; k++)
    if (k < count) {
      float f[V], d[V];
      unpack(hx[k], f);
      unpack(hz[k], d);
#pragma unroll
      for (int j = 0; j < V; j++) {
        d[j] = fmaf(d[j], p.slope[j], fmaf(f[j] - p.mu[j], c[j], b[j]));
        if (A.mask && !(f[j] > 0.f)) d[j] = 0.f;
      }
      raw_t o;
      pack(o, d);
      *(raw_t*)(dx + k * ystep) = o;
    }
}

// Images that no workgroup can hold, first launch: sums of a chunk of positions.  LDS: rows, red [2 threads], sums [2 C]
template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void group_norm_gradient_chunk_kernel(const GroupNormArgs A) {
  extern __shared__ float lds[];
  typedef typename Raw<T, V>::type raw_t;
  Place at;
  if (!place_of(A, A.plan.chunks, at)) return;
  const uintptr_t base = A.base[blockIdx.y], wts = A.wts[blockIdx.y];
  const int C = A.s.channels, p0 = at.part * A.plan.chunk, np = min(A.plan.chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  float* rows = lds;
  float* red = rows + 2 * threads * V;
  float* sa = red + 2 * threads;
  float* sb = sa + C;
  for (int c0 = 0; c0 < C; c0 += A.cols[0].cols * V) {
    const GroupNormCols cols = A.cols[c0 + A.cols[0].cols * V >= C];
    const Lanes l = lanes_of(cols, t);
    const int count = count_of(l, np), c = c0 + l.col * V;
    const T* x = (const T*)(base + A.x) + at.image * A.x_image + (int64_t)(p0 + l.row) * A.x_pixel + c;
    const T* dy = (const T*)(base + A.dy) + at.image * A.y_image + (int64_t)(p0 + l.row) * A.y_pixel + c;
    const int64_t step = l.rows * A.x_pixel, ystep = l.rows * A.y_pixel;
    GradientLane<V> p;
    if (l.active) load_lane<V>(A, base, wts, at.image, c, p);
    float a[V], b[V];
#pragma unroll
    for (int j = 0; j < V; j++) a[j] = b[j] = 0.f;
    auto one = [&](const raw_t& ix, const raw_t& id) {
      float f[V], d[V];
      unpack(ix, f);
      unpack(id, d);
      add_gradient<V, ACT>(f, d, p, a, b);
    };
    constexpr int U = 4;
    int k = 0;
    for (; k + U <= count; k += U) {
      raw_t ix[U], id[U];
#pragma unroll
      for (int i = 0; i < U; i++) {
        ix[i] = *(const raw_t*)(x + (k + i) * step);
        id[i] = *(const raw_t*)(dy + (k + i) * ystep);
      }
#pragma unroll
      for (int i = 0; i < U; i++) one(ix[i], id[i]);
    }
    for (; k < count; k++) one(*(const raw_t*)(x + k * step), *(const raw_t*)(dy + k * ystep));
    gradient_sums<V>(a, b, p, cols, l, rows, red, sa + c0, C);
  }
  float2* out = (float2*)(base + A.sums) + (at.image * A.plan.chunks + at.part) * C;
  for (int c = t; c < C; c += threads) out[c] = make_float2(sb[c], sa[c]);
  if (!A.has_dx) return;
  float2* parts = (float2*)(base + A.parts) + (at.image * A.plan.chunks + at.part) * A.s.groups;
  group_gradient(A, wts, sa, sb, 0, A.s.groups, [&](int g, float s1, float s2) { parts[g] = make_float2(s1, s2); });
}

// Second launch: s1 and s2 of the image from its chunks', then dx.  LDS: group [2 groups]
template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void group_norm_gradient_apply_kernel(const GroupNormArgs A) {
  extern __shared__ float group[];
  typedef typename Raw<T, V>::type raw_t;
  Place at;
  if (!place_of(A, A.plan.chunks, at)) return;
  const uintptr_t base = A.base[blockIdx.y], wts = A.wts[blockIdx.y];
  const int C = A.s.channels, G = A.s.groups, chunks = A.plan.chunks;
  const int p0 = at.part * A.plan.chunk, np = min(A.plan.chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  const float2* parts = (const float2*)(base + A.parts) + at.image * chunks * G;
  const float inv = 1.f / ((float)A.s.positions * (float)A.cpg);
  for (int i = t; i < G * A.spread; i += threads) {
    const int g = i / A.spread, first = i - g * A.spread;
    float s1 = 0.f, s2 = 0.f;
    for (int k = first; k < chunks; k += A.spread) {
      s1 += parts[k * G + g].x;
      s2 += parts[k * G + g].y;
    }
    for (int o = 1; o < A.spread; o <<= 1) {
      s1 += __shfl_xor(s1, o, 64);
      s2 += __shfl_xor(s2, o, 64);
    }
    if (first == 0) {
      group[2 * g] = s1 * inv;
      group[2 * g + 1] = s2 * inv;
    }
  }
  __syncthreads();
  for (int c0 = 0; c0 < C; c0 += A.cols[0].cols * V) {
    const Lanes l = lanes_of(A.cols[c0 + A.cols[0].cols * V >= C], t);
    const int count = count_of(l, np), ch = c0 + l.col * V;
    if (count == 0) continue;
    GradientLane<V> p;
    load_lane<V>(A, base, wts, at.image, ch, p);
    float b[V], c[V];
#pragma unroll
    for (int j = 0; j < V; j++) {
      const int g = A.by_cpg(ch + j);
      b[j] = -p.r[j] * group[2 * g];
      c[j] = -p.r[j] * p.r[j] * group[2 * g + 1];
    }
    const T* x = (const T*)(base + A.x) + at.image * A.x_image + (int64_t)(p0 + l.row) * A.x_pixel + ch;
    const T* dy = (const T*)(base + A.dy) + at.image * A.y_image + (int64_t)(p0 + l.row) * A.y_pixel + ch;
    T* dx = (T*)(base + A.dx) + at.image * A.y_image + (int64_t)(p0 + l.row) * A.y_pixel + ch;
    const int64_t step = l.rows * A.x_pixel, ystep = l.rows * A.y_pixel;
    auto one = [&](const raw_t& ix, const raw_t& id, int k) {
      float f[V], d[V];
      unpack(ix, f);
      unpack(id, d);
#pragma unroll
      for (int j = 0; j < V; j++) {
        const float xc = f[j] - p.mu[j];
        const float dz = through<ACT>(d[j], ACT == SASGD_ACT_NONE ? 0.f : affine<ACT>(xc, p.r[j], p.sc[j], p.slope[j], p.sh[j]));
        d[j] = fmaf(dz, p.slope[j], fmaf(xc, c[j], b[j]));
        if (A.mask && !(f[j] > 0.f)) d[j] = 0.f;
      }
      raw_t o;
      pack(o, d);
      *(raw_t*)(dx + k * ystep) = o;
    };
    constexpr int U = 2;
    int k = 0;
    for (; k + U <= count; k += U) {
      raw_t ix[U], id[U];
#pragma unroll
      for (int i = 0; i < U; i++) {
        ix[i] = *(const raw_t*)(x + (k + i) * step);
        id[i] = *(const raw_t*)(dy + (k + i) * ystep);
      }
#pragma unroll
      for (int i = 0; i < U; i++) one(ix[i], id[i], k + i);
    }
    for (; k < count; k++) one(*(const raw_t*)(x + k * step), *(const raw_t*)(dy + k * ystep), k);
  }
}

// dscale, dshift: rows of channel sums [rows][C][2] added, 32 channels a workgroup and eight rows at a time.  Many rows in two launches: the first
// leaves a row per blockIdx.y (`per` rows each).
template <bool LAST>
__global__ __launch_bounds__(256) void group_norm_finish_kernel(const GroupNormArgs A, int64_t from, int64_t rows, int64_t per, int64_t to) {
  __shared__ float2 part[8][32];
  const int learner = blockIdx.z, ch = threadIdx.x & 31, seg = threadIdx.x >> 5, c = blockIdx.x * 32 + ch, C = A.s.channels;
  const int64_t r0 = blockIdx.y * per, r1 = r0 + per < rows ? r0 + per : rows;
  const float2* sums = (const float2*)(A.base[learner] + from);
  float a = 0.f, b = 0.f;
  if (c < C) {
#pragma unroll 8
    for (int64_t k = r0 + seg; k < r1; k += 8) {
      const float2 s = sums[k * C + c];
      a += s.x;
      b += s.y;
    }
  }
  part[seg][ch] = make_float2(a, b);
  __syncthreads();
  if (seg == 0 && c < C) {
    a = b = 0.f;
#pragma unroll
    for (int k = 0; k < 8; k++) {
      a += part[k][ch].x;
      b += part[k][ch].y;
    }
    if (!LAST) {
      ((float2*)(A.base[learner] + to))[(int64_t)blockIdx.y * C + c] = make_float2(a, b);
    } else {
      if (A.has_dscale) ((float*)(A.grads[learner] + A.dscale))[c] = a;
      if (A.has_dshift) ((float*)(A.grads[learner] + A.dshift))[c] = b;
    }
  }
}

constexpr int64_t kFinishRows = 128;               // rows of sums that one launch adds; more in two launches, of this many each

int64_t finish_splits(int64_t rows) { return rows <= kFinishRows ? 0 : std::min<int64_t>((rows + 63) / 64, kFinishRows); }

size_t lds_bytes(const GroupNormArgs& a, bool gradient) {
  const int S = a.plan.whole ? a.plan.slab : a.s.channels, T = a.plan.threads;
  return ((size_t)T * (2 * a.plan.vec + (gradient ? 2 : 1)) + 2 * S + (a.plan.whole ? 2 * (S / a.cpg) : 0)) * 4;
}

}  // namespace

constexpr int kHeldForward[] = {4, 8, 16, 24, 36}, kHeldBackward[] = {4, 8, 12, 16}, kHeldNarrow[] = {8, 24};

// Small images are held whole, in slabs of whole groups and whole vectors: the smallest that makes segments of 128 bytes a pixel, or 64 or 32
// where no more fit in, or all channels; smaller ones still where the launch would otherwise have fewer workgroups than the chip has places.
GroupNormPlan group_norm_plan(const GroupNormShape& s, bool wide, bool gradient, int learners) {
  GroupNormPlan p;
  const int size = s.bf16 ? 2 : 4, cpg = s.channels / s.groups;
  p.vec = wide ? 16 / size : 1;
  int unit = cpg;
  while (unit % p.vec != 0) unit += cpg;           // (ends: the channels are whole vectors)
  p.chunk = s.positions;
  p.chunks = 1;
  auto take = [&](int slab) {                      // does a workgroup hold it, and how
    const int cols = slab / p.vec;
    auto fits = [&](int threads, int held) {
      if (threads < cols || (int64_t)(threads / cols) * held < s.positions) return false;
      p.whole = true;
      p.slab = slab;
      p.slabs = (s.channels + slab - 1) / slab;
      p.threads = threads;
      p.held = held;
      return true;
    };
    if (slab > 1024) return false;                 // (LDS)
    if (!wide) {
      for (int held : kHeldNarrow)
        for (int threads : {256, 512, 1024})
          if (fits(threads, held)) return true;
      return false;
    }
    if (gradient) {
      for (int held : kHeldBackward)
        if (fits(256, held)) return true;
      return false;
    }
    for (int held : kHeldForward)
      if (fits(256, held)) return true;
    return false;
  };
  for (int bytes = 128; bytes >= 32; bytes /= 2) {
    int slab = std::min(s.channels, (bytes / size + unit - 1) / unit * unit);
    while (slab > unit && s.images * learners * ((s.channels + slab - 1) / slab) < 512) slab = std::max(unit, slab / 2 / unit * unit);
    if (take(slab)) return p;
  }
  p.whole = false;
  p.slab = s.channels;
  p.slabs = 1;
  p.threads = 256;
  p.held = 0;
  // chunks of 64 KiB, smaller ones where that makes fewer than 1 024 workgroups, at most 32 an image and at least 16 KiB
  const int64_t image = (int64_t)s.positions * s.channels * size, images = std::max<int64_t>(1, s.images * learners);
  int64_t chunks = std::max((image + 65535) / 65536, (1024 + images - 1) / images);
  chunks = std::min(std::min(chunks, image / 16384), (int64_t)32);
  chunks = std::max<int64_t>(1, chunks);
  p.chunk = (int)((s.positions + chunks - 1) / chunks);
  p.chunks = (s.positions + p.chunk - 1) / p.chunk;
  return p;
}

size_t group_norm_sums_at(const GroupNormShape& s, const GroupNormPlan& p) { return p.whole ? 0 : ((size_t)s.images * p.chunks * s.groups * 8 + 15) / 16 * 16; }
size_t group_norm_scratch_bytes(const GroupNormShape& s, const GroupNormPlan& p, bool gradient) {
  const int64_t rows = s.images * p.chunks;
  return group_norm_sums_at(s, p) + (gradient ? (size_t)(rows + finish_splits(rows)) * s.channels * 8 : 0);
}

static uint32_t workgroups(const GroupNormArgs& a) {
  const int parts = a.plan.whole ? a.plan.slabs : a.plan.chunks;
  return (uint32_t)(parts == 1 ? a.s.images : (a.s.images + 7) / 8 * 8 * parts);
}

// The columns of lanes: [0] of a full slab (or turn of channels), [1] of the last.
static void set_columns(GroupNormArgs& a) {
  const int V = a.plan.vec, all = (a.plan.whole ? a.plan.slab : a.s.channels) / V, most = std::min(all, a.plan.threads);
  const int last = a.plan.whole ? (a.s.channels - (a.plan.slabs - 1) * a.plan.slab) / V : all - (all - 1) / most * most;
  for (int k = 0; k < 2; k++) {
    GroupNormCols& c = a.cols[k];
    c.cols = k ? last : most;
    c.rows = a.plan.threads / c.cols;
    c.by_cols.set(c.cols);
    const int n = c.cols * V;
    c.segs = a.plan.threads / n;
    c.by_n.set(n);
    c.fold = n < 64 && (n & (n - 1)) == 0;
  }
  a.cpg = a.s.channels / a.s.groups;
  a.by_cpg.set(a.cpg);
  for (a.spread = 1; a.spread < 64 && a.spread * 2 <= a.plan.chunks && a.spread * 2 * a.s.groups <= a.plan.threads;) a.spread *= 2;
}

#define BY_ACTIVATION(launch)                                                  \
  (a.activation == SASGD_ACT_RELU ? launch(std::integral_constant<int, SASGD_ACT_RELU>()) \
   : a.activation == SASGD_ACT_SILU ? launch(std::integral_constant<int, SASGD_ACT_SILU>()) : launch(std::integral_constant<int, SASGD_ACT_NONE>()))

template <typename T, int V, int NV>
static void forward_held(const GroupNormArgs& a, dim3 grid, hipStream_t stream) {
  auto launch = [&](auto act) { group_norm_kernel<T, V, NV, decltype(act)::value><<<grid, a.plan.threads, lds_bytes(a, false), stream>>>(a); };
  BY_ACTIVATION(launch);
}
template <typename T, int V, int NV>
static void backward_held(const GroupNormArgs& a, dim3 grid, hipStream_t stream) {
  auto launch = [&](auto act) { group_norm_gradient_kernel<T, V, NV, decltype(act)::value><<<grid, a.plan.threads, lds_bytes(a, true), stream>>>(a); };
  BY_ACTIVATION(launch);
}

template <typename T, int V>
static hipError_t forward(const GroupNormArgs& a, hipStream_t stream) {
  const dim3 grid(workgroups(a), (uint32_t)a.learners);
  if (a.plan.whole) {
    if constexpr (V == 1) {
      if (a.plan.held == 8) forward_held<T, V, 8>(a, grid, stream);
      else forward_held<T, V, 24>(a, grid, stream);
    } else {
      switch (a.plan.held) {
        case 4: forward_held<T, V, 4>(a, grid, stream); break;
        case 8: forward_held<T, V, 8>(a, grid, stream); break;
        case 16: forward_held<T, V, 16>(a, grid, stream); break;
        case 24: forward_held<T, V, 24>(a, grid, stream); break;
        default: forward_held<T, V, 36>(a, grid, stream); break;
      }
    }
    return hipGetLastError();
  }
  group_norm_chunk_kernel<T, V><<<grid, a.plan.threads, lds_bytes(a, false), stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto launch = [&](auto act) { group_norm_apply_kernel<T, V, decltype(act)::value><<<grid, a.plan.threads, (size_t)a.s.groups * 8, stream>>>(a); };
  BY_ACTIVATION(launch);
  return hipGetLastError();
}

template <typename T, int V>
static hipError_t backward(const GroupNormArgs& a, hipStream_t stream) {
  const dim3 grid(workgroups(a), (uint32_t)a.learners);
  if (a.plan.whole) {
    if constexpr (V == 1) {
      if (a.plan.held == 8) backward_held<T, V, 8>(a, grid, stream);
      else backward_held<T, V, 24>(a, grid, stream);
    } else {
      switch (a.plan.held) {
        case 4: backward_held<T, V, 4>(a, grid, stream); break;
        case 8: backward_held<T, V, 8>(a, grid, stream); break;
        case 12: backward_held<T, V, 12>(a, grid, stream); break;
        default: backward_held<T, V, 16>(a, grid, stream); break;
      }
    }
    return hipGetLastError();
  }
  auto sums = [&](auto act) { group_norm_gradient_chunk_kernel<T, V, decltype(act)::value><<<grid, a.plan.threads, lds_bytes(a, true), stream>>>(a); };
  BY_ACTIVATION(sums);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.has_dx) return e;
  auto launch = [&](auto act) { group_norm_gradient_apply_kernel<T, V, decltype(act)::value><<<grid, a.plan.threads, (size_t)a.s.groups * 8, stream>>>(a); };
  BY_ACTIVATION(launch);
  return hipGetLastError();
}

hipError_t launch_group_norm(GroupNormArgs& a, hipStream_t stream) {
  if (a.s.images == 0) return hipSuccess;
  set_columns(a);
  if (a.s.bf16) return a.plan.vec == 8 ? forward<bf16_t, 8>(a, stream) : forward<bf16_t, 1>(a, stream);
  return a.plan.vec == 4 ? forward<float, 4>(a, stream) : forward<float, 1>(a, stream);
}

hipError_t launch_group_norm_gradient(GroupNormArgs& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.s.images > 0) {
    set_columns(a);
    if (a.s.bf16) e = a.plan.vec == 8 ? backward<bf16_t, 8>(a, stream) : backward<bf16_t, 1>(a, stream);
    else e = a.plan.vec == 4 ? backward<float, 4>(a, stream) : backward<float, 1>(a, stream);
  }
  if (e != hipSuccess || (!a.has_dscale && !a.has_dshift)) return e;
  const int64_t rows = a.s.images * a.plan.chunks, splits = finish_splits(rows);
  const uint32_t strips = (uint32_t)(a.s.channels + 31) / 32, learners = (uint32_t)a.learners;
  int64_t from = a.sums, left = rows;
  if (splits > 0) {
    const int64_t to = a.sums + rows * a.s.channels * 8, per = (rows + splits - 1) / splits;
    group_norm_finish_kernel<false><<<dim3(strips, (uint32_t)splits, learners), 256, 0, stream>>>(a, from, rows, per, to);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    from = to;
    left = splits;
  }
  group_norm_finish_kernel<true><<<dim3(strips, 1, learners), 256, 0, stream>>>(a, from, left, left, 0);
  return hipGetLastError();
}

}  // namespace sasgd
