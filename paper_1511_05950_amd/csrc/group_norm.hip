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
// The variance is the mean of squared distances from the channel's own mean over the values in registers, then
// sum of those + count x (channel mean - group mean)^2: no difference of large sums.
#include "dev_common.hpp"
#include "operators.hpp"

#include <algorithm>

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

template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == SASGD_ACT_RELU) return z <= 0.f ? 0.f : z;         // (NaN stays)
  if (ACT == SASGD_ACT_SILU) return z / (1.f + __expf(-z));
  return z;
}
// act'(z)
template <int ACT>
__device__ __forceinline__ float slope(float z) {
  if (ACT == SASGD_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (ACT == SASGD_ACT_SILU) {
    const float s = 1.f / (1.f + __expf(-z));
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}
// Each operation rounded by itself: forward and backward pass (and whoever computes z by the formula) agree on the sign of z.
__device__ __forceinline__ float hat(float x, float mean, float r) {
#pragma clang fp contract(off)
  return (x - mean) * r;
}
__device__ __forceinline__ float affine(float h, float scale, float shift) {
#pragma clang fp contract(off)
  return h * scale + shift;
}

__device__ __forceinline__ float param(const GroupNormArgs& A, uintptr_t at, int c) {
  return A.param_bf16 ? bf2f(((const bf16_t*)at)[c]) : ((const float*)at)[c];
}

// Where a workgroup is: which image of which learner, which slab or chunk.
struct Place {
  int learner;
  int64_t image;
  int part;
};
__device__ __forceinline__ Place place_of(const GroupNormArgs& A, int parts) {
  const uint32_t b = blockIdx.x, per = (uint32_t)A.s.images * (uint32_t)parts;
  Place p;
  p.learner = (int)(b / per);
  const uint32_t rest = b - p.learner * per;
  p.image = rest / (uint32_t)parts;
  p.part = (int)(rest - (uint32_t)p.image * (uint32_t)parts);
  return p;
}

// out[c] = sum over the workgroup's rows of lanes of what they have for channel c = col V + j, c < n.  red: blockDim.x V floats.
template <int V>
__device__ __forceinline__ void channel_sums(const float (&part)[V], float* red, float* out, int row, int col, bool active, int rows, int n) {
  const int t = threadIdx.x, T = blockDim.x;
  if (active)
#pragma unroll
    for (int j = 0; j < V; j++) red[row * n + col * V + j] = part[j];
  __syncthreads();
  const int segs = T / n;
  if (segs > 1) {
    const int seg = t / n, c = t - seg * n;
    float s = 0.f;
    if (seg < segs)
      for (int r = seg; r < rows; r += segs) s += red[r * n + c];
    __syncthreads();
    if (seg < segs) red[t] = s;
    __syncthreads();
    if (t < n) {
      s = 0.f;
      for (int k = 0; k < segs; k++) s += red[k * n + t];
      out[t] = s;
    }
  } else {
    for (int c = t; c < n; c += T) {
      float s = 0.f;
      for (int r = 0; r < rows; r++) s += red[r * n + c];
      out[c] = s;
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------------------------------------ forward
// LDS: red [threads V], mean [S], dev [S], group [2 S / channels of a group]
template <typename T, int V, int NV, int ACT, bool WHOLE>
__global__ __launch_bounds__(1024) void group_norm_kernel(const GroupNormArgs A) {
  extern __shared__ float lds[];
  typedef typename Raw<T, V>::type raw_t;
  const Place at = place_of(A, WHOLE ? A.plan.slabs : A.plan.chunks);
  const int C = A.s.channels, cpg = C / A.s.groups;
  const int c0 = WHOLE ? at.part * A.plan.slab : 0, S = WHOLE ? min(A.plan.slab, C - c0) : C;
  const int p0 = WHOLE ? 0 : at.part * A.plan.chunk, np = WHOLE ? A.s.positions : min(A.plan.chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  float* red = lds;
  float* mean = red + threads * V;
  float* dev = mean + S;
  float* group = dev + S;
  const T* x = (const T*)(A.base[at.learner] + A.x) + at.image * A.x_image + (int64_t)p0 * A.x_pixel + c0;
  const int all = S / V, most = min(all, threads);
  raw_t held[NV];
  int row = 0, col = 0;
  bool active = false;
  for (int q = 0; q < all; q += most) {            // (one turn where the workgroup writes)
    const int cols = min(most, all - q), rows = threads / cols;
    row = t / cols;
    col = t - row * cols;
    active = row < rows;
    const T* xq = x + (q + col) * V;
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; j++) sum[j] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++)
      if (active && row + k * rows < np) held[k] = *(const raw_t*)(xq + (int64_t)(row + k * rows) * A.x_pixel);
#pragma unroll
    for (int k = 0; k < NV; k++)
      if (active && row + k * rows < np) {
        float f[V];
        unpack(held[k], f);
#pragma unroll
        for (int j = 0; j < V; j++) sum[j] += f[j];
      }
    channel_sums<V>(sum, red, mean + q * V, row, col, active, rows, cols * V);
    const float inv = 1.f / (float)np;
    float mu[V];
#pragma unroll
    for (int j = 0; j < V; j++) {
      mu[j] = mean[(q + col) * V + j] * inv;
      sum[j] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < NV; k++)
      if (active && row + k * rows < np) {
        float f[V];
        unpack(held[k], f);
#pragma unroll
        for (int j = 0; j < V; j++) sum[j] += (f[j] - mu[j]) * (f[j] - mu[j]);
      }
    channel_sums<V>(sum, red, dev + q * V, row, col, active, rows, cols * V);
  }
  // groups from their channels, a wavefront a group
  const int lane = t & 63, gs = S / cpg;
  const float inv = 1.f / (float)np;
  for (int g = t >> 6; g < gs; g += threads >> 6) {
    float s = 0.f, d = 0.f;
    for (int c = lane; c < cpg; c += 64) {
      s += mean[g * cpg + c] * inv;
      d += dev[g * cpg + c];
    }
    const float mu = wave_sum(s) / (float)cpg;
    float off = 0.f;
    for (int c = lane; c < cpg; c += 64) {
      const float e = mean[g * cpg + c] * inv - mu;
      off += e * e;
    }
    const float m2 = wave_sum(d) + (float)np * wave_sum(off);
    if (lane == 0) {
      const int64_t gi = at.image * A.s.groups + c0 / cpg + g;
      if (WHOLE) {
        const float r = 1.f / sqrtf(m2 / ((float)np * (float)cpg) + A.eps);
        group[2 * g] = mu;
        group[2 * g + 1] = r;
        if (A.has_stats) ((float2*)(A.base[at.learner] + A.stats))[gi] = make_float2(mu, r);
      } else {
        ((float2*)(A.base[at.learner] + A.parts))[(at.image * A.plan.chunks + at.part) * A.s.groups + g] = make_float2(mu, m2);
      }
    }
  }
  if (!WHOLE) return;
  __syncthreads();
  if (!active) return;
  float mu[V], r[V], sc[V], sh[V];
#pragma unroll
  for (int j = 0; j < V; j++) {
    const int c = col * V + j, g = c / cpg;
    mu[j] = group[2 * g];
    r[j] = group[2 * g + 1];
    sc[j] = A.has_scale ? param(A, A.wts[at.learner] + A.scale, c0 + c) : 1.f;
    sh[j] = A.has_shift ? param(A, A.wts[at.learner] + A.shift, c0 + c) : 0.f;
  }
  const int rows = threads / all;
  T* y = (T*)(A.base[at.learner] + A.y) + at.image * A.y_image + c0 + col * V;
#pragma unroll
  for (int k = 0; k < NV; k++)
    if (row + k * rows < np) {
      float f[V];
      unpack(held[k], f);
#pragma unroll
      for (int j = 0; j < V; j++) f[j] = activate<ACT>(affine(hat(f[j], mu[j], r[j]), sc[j], sh[j]));
      raw_t o;
      pack(o, f);
      *(raw_t*)(y + (int64_t)(row + k * rows) * A.y_pixel) = o;
    }
}

// Second launch where an image is cut into chunks: statistics of the whole image from those of its chunks, then y.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void group_norm_apply_kernel(const GroupNormArgs A) {
  extern __shared__ float group[];                 // [groups][2]
  typedef typename Raw<T, V>::type raw_t;
  const Place at = place_of(A, A.plan.chunks);
  const int C = A.s.channels, G = A.s.groups, cpg = C / G, chunk = A.plan.chunk, chunks = A.plan.chunks;
  const int p0 = at.part * chunk, np = min(chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  const float2* parts = (const float2*)(A.base[at.learner] + A.parts) + at.image * chunks * G;
  for (int g = t; g < G; g += threads) {
    float s = 0.f, m2 = 0.f;
    for (int k = 0; k < chunks; k++) s += parts[k * G + g].x * (float)min(chunk, A.s.positions - k * chunk);
    const float mu = s / (float)A.s.positions;
    for (int k = 0; k < chunks; k++) {
      const float2 p = parts[k * G + g];
      m2 += p.y + (float)min(chunk, A.s.positions - k * chunk) * (float)cpg * (p.x - mu) * (p.x - mu);
    }
    const float r = 1.f / sqrtf(m2 / ((float)A.s.positions * (float)cpg) + A.eps);
    group[2 * g] = mu;
    group[2 * g + 1] = r;
    if (A.has_stats && at.part == 0) ((float2*)(A.base[at.learner] + A.stats))[at.image * G + g] = make_float2(mu, r);
  }
  __syncthreads();
  const T* x = (const T*)(A.base[at.learner] + A.x) + at.image * A.x_image + (int64_t)p0 * A.x_pixel;
  T* y = (T*)(A.base[at.learner] + A.y) + at.image * A.y_image + (int64_t)p0 * A.y_pixel;
  const int all = C / V, most = min(all, threads);
  for (int q = 0; q < all; q += most) {
    const int cols = min(most, all - q), rows = threads / cols, row = t / cols, col = q + t - row * cols;
    if (row >= rows) continue;
    float mu[V], r[V], sc[V], sh[V];
#pragma unroll
    for (int j = 0; j < V; j++) {
      const int c = col * V + j, g = c / cpg;
      mu[j] = group[2 * g];
      r[j] = group[2 * g + 1];
      sc[j] = A.has_scale ? param(A, A.wts[at.learner] + A.scale, c) : 1.f;
      sh[j] = A.has_shift ? param(A, A.wts[at.learner] + A.shift, c) : 0.f;
    }
#pragma unroll 4
    for (int p = row; p < np; p += rows) {
      const raw_t in = *(const raw_t*)(x + (int64_t)p * A.x_pixel + col * V);
      float f[V];
      unpack(in, f);
#pragma unroll
      for (int j = 0; j < V; j++) f[j] = activate<ACT>(affine(hat(f[j], mu[j], r[j]), sc[j], sh[j]));
      raw_t o;
      pack(o, f);
      *(raw_t*)(y + (int64_t)p * A.y_pixel + col * V) = o;
    }
  }
}

// ------------------------------------------------------------------------------------------------ backward
template <int V>
__device__ __forceinline__ void load_params(const GroupNormArgs& A, const Place& at, int c0, int cpg, float (&mu)[V], float (&r)[V], float (&sc)[V], float (&sh)[V]) {
  const float2* stats = (const float2*)(A.base[at.learner] + A.stats) + at.image * A.s.groups;
#pragma unroll
  for (int j = 0; j < V; j++) {
    const int c = c0 + j;
    const float2 st = stats[c / cpg];
    mu[j] = st.x;
    r[j] = st.y;
    sc[j] = A.has_scale ? param(A, A.wts[at.learner] + A.scale, c) : 1.f;
    sh[j] = A.has_shift ? param(A, A.wts[at.learner] + A.shift, c) : 0.f;
  }
}

// LDS: red [threads V], a [S] (sums of dz), b [S] (of dz xhat), group [2 S / channels of a group]
template <typename T, int V, int NV, int ACT, bool WHOLE>
__global__ __launch_bounds__(1024) void group_norm_gradient_kernel(const GroupNormArgs A) {
  extern __shared__ float lds[];
  typedef typename Raw<T, V>::type raw_t;
  const Place at = place_of(A, WHOLE ? A.plan.slabs : A.plan.chunks);
  const int C = A.s.channels, cpg = C / A.s.groups;
  const int c0 = WHOLE ? at.part * A.plan.slab : 0, S = WHOLE ? min(A.plan.slab, C - c0) : C;
  const int p0 = WHOLE ? 0 : at.part * A.plan.chunk, np = WHOLE ? A.s.positions : min(A.plan.chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  float* red = lds;
  float* sa = red + threads * V;
  float* sb = sa + S;
  float* group = sb + S;
  const T* x = (const T*)(A.base[at.learner] + A.x) + at.image * A.x_image + (int64_t)p0 * A.x_pixel + c0;
  const T* dy = (const T*)(A.base[at.learner] + A.dy) + at.image * A.y_image + (int64_t)p0 * A.y_pixel + c0;
  const int all = S / V, most = min(all, threads);
  raw_t hx[NV], hd[NV];
  float mu[V], r[V], sc[V], sh[V];
  int row = 0, col = 0;
  bool active = false;
  for (int q = 0; q < all; q += most) {            // (one turn where the workgroup writes dx)
    const int cols = min(most, all - q), rows = threads / cols;
    row = t / cols;
    col = t - row * cols;
    active = row < rows;
    const T* xq = x + (q + col) * V;
    const T* dq = dy + (q + col) * V;
    float a[V], b[V];
#pragma unroll
    for (int j = 0; j < V; j++) a[j] = b[j] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++)
      if (active && row + k * rows < np) {
        hx[k] = *(const raw_t*)(xq + (int64_t)(row + k * rows) * A.x_pixel);
        hd[k] = *(const raw_t*)(dq + (int64_t)(row + k * rows) * A.y_pixel);
      }
    load_params<V>(A, at, c0 + (q + col) * V, cpg, mu, r, sc, sh);
#pragma unroll
    for (int k = 0; k < NV; k++)
      if (active && row + k * rows < np) {
        float f[V], d[V];
        unpack(hx[k], f);
        unpack(hd[k], d);
#pragma unroll
        for (int j = 0; j < V; j++) {
          const float h = hat(f[j], mu[j], r[j]);
          const float dz = ACT == SASGD_ACT_NONE ? d[j] : d[j] * slope<ACT>(affine(h, sc[j], sh[j]));
          a[j] += dz;
          b[j] += dz * h;
        }
      }
    channel_sums<V>(a, red, sa + q * V, row, col, active, rows, cols * V);
    channel_sums<V>(b, red, sb + q * V, row, col, active, rows, cols * V);
  }
  {
    float2* out = (float2*)(A.base[at.learner] + A.sums) + (at.image * A.plan.chunks + (WHOLE ? 0 : at.part)) * C + c0;
    for (int c = t; c < S; c += threads) out[c] = make_float2(sb[c], sa[c]);
  }
  if (!A.has_dx) return;
  const int lane = t & 63, gs = S / cpg;
  for (int g = t >> 6; g < gs; g += threads >> 6) {
    float s1 = 0.f, s2 = 0.f;
    for (int c = lane; c < cpg; c += 64) {
      const float w = A.has_scale ? param(A, A.wts[at.learner] + A.scale, c0 + g * cpg + c) : 1.f;
      s1 += w * sa[g * cpg + c];
      s2 += w * sb[g * cpg + c];
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if (lane == 0) {
      if (WHOLE) {
        group[2 * g] = s1;
        group[2 * g + 1] = s2;
      } else {
        ((float2*)(A.base[at.learner] + A.parts))[(at.image * A.plan.chunks + at.part) * A.s.groups + g] = make_float2(s1, s2);
      }
    }
  }
  if (!WHOLE) return;
  __syncthreads();
  if (!active) return;
  const float inv = 1.f / ((float)np * (float)cpg);
  float s1[V], s2[V];
#pragma unroll
  for (int j = 0; j < V; j++) {
    const int g = (col * V + j) / cpg;
    s1[j] = group[2 * g] * inv;
    s2[j] = group[2 * g + 1] * inv;
  }
  const int rows = threads / all;
  T* dx = (T*)(A.base[at.learner] + A.dx) + at.image * A.y_image + c0 + col * V;
#pragma unroll
  for (int k = 0; k < NV; k++)
    if (row + k * rows < np) {
      float f[V], d[V];
      unpack(hx[k], f);
      unpack(hd[k], d);
#pragma unroll
      for (int j = 0; j < V; j++) {
        const float h = hat(f[j], mu[j], r[j]);
        const float dz = ACT == SASGD_ACT_NONE ? d[j] : d[j] * slope<ACT>(affine(h, sc[j], sh[j]));
        d[j] = r[j] * (sc[j] * dz - (s1[j] + h * s2[j]));
        if (A.mask && !(f[j] > 0.f)) d[j] = 0.f;
      }
      raw_t o;
      pack(o, d);
      *(raw_t*)(dx + (int64_t)(row + k * rows) * A.y_pixel) = o;
    }
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void group_norm_gradient_apply_kernel(const GroupNormArgs A) {
  extern __shared__ float group[];                 // [groups][2]
  typedef typename Raw<T, V>::type raw_t;
  const Place at = place_of(A, A.plan.chunks);
  const int C = A.s.channels, G = A.s.groups, cpg = C / G, chunk = A.plan.chunk, chunks = A.plan.chunks;
  const int p0 = at.part * chunk, np = min(chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  const float2* parts = (const float2*)(A.base[at.learner] + A.parts) + at.image * chunks * G;
  const float inv = 1.f / ((float)A.s.positions * (float)cpg);
  for (int g = t; g < G; g += threads) {
    float s1 = 0.f, s2 = 0.f;
    for (int k = 0; k < chunks; k++) {
      const float2 p = parts[k * G + g];
      s1 += p.x;
      s2 += p.y;
    }
    group[2 * g] = s1 * inv;
    group[2 * g + 1] = s2 * inv;
  }
  __syncthreads();
  const T* x = (const T*)(A.base[at.learner] + A.x) + at.image * A.x_image + (int64_t)p0 * A.x_pixel;
  const T* dy = (const T*)(A.base[at.learner] + A.dy) + at.image * A.y_image + (int64_t)p0 * A.y_pixel;
  T* dx = (T*)(A.base[at.learner] + A.dx) + at.image * A.y_image + (int64_t)p0 * A.y_pixel;
  const int all = C / V, most = min(all, threads);
  for (int q = 0; q < all; q += most) {
    const int cols = min(most, all - q), rows = threads / cols, row = t / cols, col = q + t - row * cols;
    if (row >= rows) continue;
    float mu[V], r[V], sc[V], sh[V], s1[V], s2[V];
    load_params<V>(A, at, col * V, cpg, mu, r, sc, sh);
#pragma unroll
    for (int j = 0; j < V; j++) {
      const int g = (col * V + j) / cpg;
      s1[j] = group[2 * g];
      s2[j] = group[2 * g + 1];
    }
#pragma unroll 2
    for (int p = row; p < np; p += rows) {
      const raw_t ix = *(const raw_t*)(x + (int64_t)p * A.x_pixel + col * V), id = *(const raw_t*)(dy + (int64_t)p * A.y_pixel + col * V);
      float f[V], d[V];
      unpack(ix, f);
      unpack(id, d);
#pragma unroll
      for (int j = 0; j < V; j++) {
        const float h = hat(f[j], mu[j], r[j]);
        const float dz = ACT == SASGD_ACT_NONE ? d[j] : d[j] * slope<ACT>(affine(h, sc[j], sh[j]));
        d[j] = r[j] * (sc[j] * dz - (s1[j] + h * s2[j]));
        if (A.mask && !(f[j] > 0.f)) d[j] = 0.f;
      }
      raw_t o;
      pack(o, d);
      *(raw_t*)(dx + (int64_t)p * A.y_pixel + col * V) = o;
    }
  }
}

// dscale, dshift: the rows of `sums` (a row per image and chunk) added, 32 channels a workgroup, 32 rows at a time.
__global__ __launch_bounds__(1024) void group_norm_finish_kernel(const GroupNormArgs A) {
  __shared__ float2 part[32][33];
  const int learner = blockIdx.y, ch = threadIdx.x & 31, seg = threadIdx.x >> 5, c = blockIdx.x * 32 + ch, C = A.s.channels;
  const int64_t rows = A.s.images * A.plan.chunks;
  const float2* sums = (const float2*)(A.base[learner] + A.sums);
  float a = 0.f, b = 0.f;
  if (c < C)
    for (int64_t k = seg; k < rows; k += 32) {
      const float2 s = sums[k * C + c];
      a += s.x;
      b += s.y;
    }
  part[seg][ch] = make_float2(a, b);
  __syncthreads();
  if (seg == 0 && c < C) {
    a = b = 0.f;
    for (int k = 0; k < 32; k++) {
      a += part[k][ch].x;
      b += part[k][ch].y;
    }
    if (A.has_dscale) ((float*)(A.grads[learner] + A.dscale))[c] = a;
    if (A.has_dshift) ((float*)(A.grads[learner] + A.dshift))[c] = b;
  }
}

size_t lds_bytes(const GroupNormArgs& a) {
  const int S = a.plan.whole ? a.plan.slab : a.s.channels, cpg = a.s.channels / a.s.groups;
  return ((size_t)a.plan.threads * a.plan.vec + 2 * S + (a.plan.whole ? 2 * (S / cpg) : 0)) * 4;
}

}  // namespace

// Small images are held whole: the smallest slab of whole groups and whole vectors that makes segments of 128 bytes a pixel (64 where 128 do
// not fit in), or all channels; smaller ones still where the launch would otherwise have fewer workgroups than the chip compute units.
GroupNormPlan group_norm_plan(const GroupNormShape& s, bool wide, bool gradient, int learners) {
  GroupNormPlan p;
  const int size = s.bf16 ? 2 : 4, cpg = s.channels / s.groups;
  p.vec = wide ? 16 / size : 1;
  const int small = wide ? 4 : 8, big = wide ? (gradient ? 8 : 16) : 32;
  int unit = cpg;
  while (unit % p.vec != 0) unit += cpg;           // (whole vectors: the channels are a multiple of them)
  p.whole = false;
  p.slab = s.channels;
  p.slabs = 1;
  for (int bytes = 128; bytes >= 64 && !p.whole; bytes /= 2) {
    int slab = std::min(s.channels, (bytes / size + unit - 1) / unit * unit);
    while (slab > unit && s.images * learners * ((s.channels + slab - 1) / slab) < 256) slab = std::max(unit, slab / 2 / unit * unit);
    if ((int64_t)slab / p.vec * s.positions > (int64_t)1024 * big || slab / p.vec > 1024 || slab > 2048) continue;     // (LDS)
    p.whole = true;
    p.slab = slab;
    p.slabs = (s.channels + slab - 1) / slab;
  }
  if (p.whole) {
    const int cols = p.slab / p.vec;
    auto fits = [&](int threads, int held) { return threads >= cols && (int64_t)(threads / cols) * held >= s.positions; };
    p.threads = 1024;
    p.held = big;
    for (int held : {small, big})
      for (int threads : {256, 512, 1024})
        if (fits(threads, held)) {
          p.threads = threads;
          p.held = held;
          p.chunk = s.positions;
          p.chunks = 1;
          return p;
        }
    p.whole = false;                               // lanes left over by the columns: it does not fit after all
    p.slab = s.channels;
    p.slabs = 1;
  }
  p.threads = 512;
  p.held = wide ? (gradient ? 4 : 4) : 8;
  const int cols = std::min(s.channels / p.vec, p.threads);
  p.chunk = std::min(s.positions, p.threads / cols * p.held);
  p.chunks = (s.positions + p.chunk - 1) / p.chunk;
  return p;
}

size_t group_norm_part_bytes(const GroupNormShape& s, const GroupNormPlan& p) { return p.whole ? 0 : (size_t)s.images * p.chunks * s.groups * 8; }
size_t group_norm_sum_bytes(const GroupNormShape& s, const GroupNormPlan& p) { return (size_t)s.images * p.chunks * s.channels * 8; }

#define BY_ACTIVATION(call)                                  \
  do {                                                       \
    if (a.activation == SASGD_ACT_RELU) call(SASGD_ACT_RELU); \
    else if (a.activation == SASGD_ACT_SILU) call(SASGD_ACT_SILU); \
    else call(SASGD_ACT_NONE);                               \
  } while (0)

template <typename T, int V, int SMALL, int BIG>
static hipError_t forward(const GroupNormArgs& a, hipStream_t stream) {
  const dim3 grid((uint32_t)(a.s.images * a.learners * (a.plan.whole ? a.plan.slabs : a.plan.chunks)));
  const size_t lds = lds_bytes(a);
#define WHOLE_SMALL(ACT) group_norm_kernel<T, V, SMALL, ACT, true><<<grid, a.plan.threads, lds, stream>>>(a)
#define WHOLE_BIG(ACT) group_norm_kernel<T, V, BIG, ACT, true><<<grid, a.plan.threads, lds, stream>>>(a)
#define APPLY(ACT) group_norm_apply_kernel<T, V, ACT><<<grid, 256, (size_t)a.s.groups * 8, stream>>>(a)
  if (a.plan.whole) {
    if (a.plan.held == SMALL) BY_ACTIVATION(WHOLE_SMALL);
    else BY_ACTIVATION(WHOLE_BIG);
    return hipGetLastError();
  }
  group_norm_kernel<T, V, SMALL, SASGD_ACT_NONE, false><<<grid, a.plan.threads, lds, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  BY_ACTIVATION(APPLY);
  return hipGetLastError();
#undef WHOLE_SMALL
#undef WHOLE_BIG
#undef APPLY
}

template <typename T, int V, int SMALL, int BIG>
static hipError_t backward(const GroupNormArgs& a, hipStream_t stream) {
  const dim3 grid((uint32_t)(a.s.images * a.learners * (a.plan.whole ? a.plan.slabs : a.plan.chunks)));
  const size_t lds = lds_bytes(a);
#define WHOLE_SMALL(ACT) group_norm_gradient_kernel<T, V, SMALL, ACT, true><<<grid, a.plan.threads, lds, stream>>>(a)
#define WHOLE_BIG(ACT) group_norm_gradient_kernel<T, V, BIG, ACT, true><<<grid, a.plan.threads, lds, stream>>>(a)
#define CHUNKS(ACT) group_norm_gradient_kernel<T, V, SMALL, ACT, false><<<grid, a.plan.threads, lds, stream>>>(a)
#define APPLY(ACT) group_norm_gradient_apply_kernel<T, V, ACT><<<grid, 256, (size_t)a.s.groups * 8, stream>>>(a)
  if (a.plan.whole) {
    if (a.plan.held == SMALL) BY_ACTIVATION(WHOLE_SMALL);
    else BY_ACTIVATION(WHOLE_BIG);
    return hipGetLastError();
  }
  BY_ACTIVATION(CHUNKS);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.has_dx) return e;
  BY_ACTIVATION(APPLY);
  return hipGetLastError();
#undef WHOLE_SMALL
#undef WHOLE_BIG
#undef CHUNKS
#undef APPLY
}

hipError_t launch_group_norm(const GroupNormArgs& a, hipStream_t stream) {
  if (a.s.images == 0) return hipSuccess;
  if (a.s.bf16) return a.plan.vec == 8 ? forward<bf16_t, 8, 4, 16>(a, stream) : forward<bf16_t, 1, 8, 32>(a, stream);
  return a.plan.vec == 4 ? forward<float, 4, 4, 16>(a, stream) : forward<float, 1, 8, 32>(a, stream);
}

hipError_t launch_group_norm_gradient(const GroupNormArgs& a, hipStream_t stream) {
  if (a.s.images > 0) {
    hipError_t e;
    if (a.s.bf16) e = a.plan.vec == 8 ? backward<bf16_t, 8, 4, 8>(a, stream) : backward<bf16_t, 1, 8, 32>(a, stream);
    else e = a.plan.vec == 4 ? backward<float, 4, 4, 8>(a, stream) : backward<float, 1, 8, 32>(a, stream);
    if (e != hipSuccess) return e;
  }
  if (!a.has_dscale && !a.has_dshift) return hipSuccess;
  group_norm_finish_kernel<<<dim3((uint32_t)(a.s.channels + 31) / 32, (uint32_t)a.learners), 1024, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace sasgd
