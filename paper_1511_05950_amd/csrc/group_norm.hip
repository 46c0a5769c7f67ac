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
// Sums go by units of neighbouring channels (one, two, or a lane's whole vector where a group is whole vectors; one in the backward pass, whose dscale
// and dshift want them): a lane owns 16 bytes of channels at a fixed place of the pixel and walks positions, the rows of lanes are added through LDS in a
// fixed order, and groups are put together from their units, whatever number of channels a group has.  Variances are sums of squared distances
// from the mean of what is summed, joined by sum of those + sum of count x (mean - joint mean)^2, from lanes to units to groups.  Two differences of sums are
// left: a lane's squares less its sum's (Moments, DotMoments), good to 32 bits or to 256 roundings of them, and that of an image's at most 64 chunks
// (group_norm_apply_kernel), of distances from the first one's mean, good to 64 times the few roundings of its sums.
//
// What bounds it now (MI355X; a copy of 160 MB runs at 5.36 TB/s, reading and writing, of 4 GiB at 4.74): bf16 2 304 x 32 x 32 x 32 gradient 104 us, 4.4 TB/s;
// 288 x 27 x 27 x 256 gradient 77 us, 4.2 TB/s: HBM, and the vector ALU between the phases of a workgroup.  288 x 54 x 54 x 96 forward 97 us (95 to 101 from run
// to run): 37 of statistics, 60 at the copy's rate; held in slabs of 24 channels by 256 lanes it was 106 (segments of 48 bytes of a line), in larger slabs by more lanes it
// has not been tried.  16 x 64 x 64 x 320 33 us: the second read, and both launches' ends.  4 x 32 x 32 x 32 fp32 6.5 us: a launch and the chain of its phases.
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

// Past the caches: what a call reads or writes for the last time.  (Segments of 48 bytes of a line that several workgroups share then take twice as long:
// group_norm_plan cuts channels at 64 bytes.  Through them and past them, bf16: 288 x 27 x 27 x 256 gradient 91 and 78 us, 2 304 x 32 x 32 x 32 120 and 105,
// 288 x 54 x 54 x 96 forward 114 and 94, 16 x 64 x 64 x 320 36 and 34.)
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ float4 load_once(const float4* p) {
  const f4 v = __builtin_nontemporal_load((const f4*)p);
  return make_float4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  const u4 v = __builtin_nontemporal_load((const u4*)p);
  return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ float load_once(const float* p) { return *p; }
__device__ __forceinline__ bf16_t load_once(const bf16_t* p) { return *p; }
__device__ __forceinline__ void store_once(float4* p, const float4& r) {
  const f4 v = {r.x, r.y, r.z, r.w};
  __builtin_nontemporal_store(v, (f4*)p);
}
__device__ __forceinline__ void store_once(uint4* p, const uint4& r) {
  const u4 v = {r.x, r.y, r.z, r.w};
  __builtin_nontemporal_store(v, (u4*)p);
}
__device__ __forceinline__ void store_once(float* p, float r) { *p = r; }
__device__ __forceinline__ void store_once(bf16_t* p, bf16_t r) { *p = r; }
// N vectors of a lane, `step` apart, those from `count` on left out.
template <bool ONCE, int N, typename R, typename T>
__device__ __forceinline__ void load_rows(R (&held)[N], const T* x, int64_t step, int count) {
#pragma unroll
  for (int k = 0; k < N; k++)
    if (k < count) held[k] = ONCE ? load_once((const R*)(x + k * step)) : *(const R*)(x + k * step);
}
template <bool ONCE, typename R>
__device__ __forceinline__ void store_row(R* p, const R& r) {
  if (ONCE) store_once(p, r);
  else *p = r;
}

template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == SASGD_ACT_RELU) return __builtin_elementwise_maximum(z, 0.f);       // (NaN stays)
  if (ACT == SASGD_ACT_SILU) return z * sigmoid(z);
  return z;
}
// z from x - mean.  Behind a ReLU each operation is rounded by itself, in both directions: the backward pass passes dy where the forward pass gave a positive
// output, and whoever computes z by the formula agrees on its sign.  Elsewhere r scale is one factor.
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

// Values of a group up to which one lane adds them, a wavefront above (by lanes and by wavefronts: 5 values of each of 32 groups, 16 x 32 x 32 x 320
// forward, 18 and 21 us; 64 of one, 256 x 4 x 4 x 512, 12 and 7; 43 of one, 30 x 23 x 20 x 43 gradient, 14 and 12).
constexpr int kLaneChannels = 8;

// Scales and shifts of the workgroup's channels, a lane a channel, to LDS: a lane has its eight from there instead of sixteen loads of its own (behind
// the next barrier).  Fetched in front of the values and written behind them: what waits for them does not wait for the values.
struct Params {
  uint32_t scale, shift;
  __device__ __forceinline__ void fetch(const GroupNormArgs& A, uintptr_t wts, int c) {
    const uintptr_t a = wts + A.scale, b = wts + A.shift;
    scale = shift = 0;
    if (A.has_scale) scale = A.param_bf16 ? ((const bf16_t*)a)[c] : ((const uint32_t*)a)[c];
    if (A.has_shift) shift = A.param_bf16 ? ((const bf16_t*)b)[c] : ((const uint32_t*)b)[c];
  }
  __device__ __forceinline__ void put(const GroupNormArgs& A, float* to_scale, float* to_shift) const {
    const int up = A.param_bf16 ? 16 : 0;
    *to_scale = A.has_scale ? __uint_as_float(scale << up) : 1.f;
    *to_shift = __uint_as_float(shift << up);
  }
};

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

// Sums of a vector's values go by units of V / U neighbouring channels: all of a group's, or as many as divide it (U = 1, V / 2 or V).
// Mean and sum of squared distances of every unit of `np` positions from what lanes have of them: lane sums `sum` and squared distances `dev` from the
// lane's own mean.  mean[c], dev[c]; rows: 2 threads U floats, red: threads floats.
template <int V, int U>
__device__ __forceinline__ void unit_moments(const float (&sum)[U], const float (&dev)[U], const GroupNormCols& cols, const Lanes& l, int np, float* rows,
                                             float* red, float* mean, float* m2) {
  const int n = cols.cols * U;
  float* rd = rows + cols.rows * n;
  if (l.active)
#pragma unroll
    for (int j = 0; j < U; j++) {
      rows[l.row * n + l.col * U + j] = sum[j];
      rd[l.row * n + l.col * U + j] = dev[j];
    }
  __syncthreads();
  row_sums<1>(cols, n, red, mean, 0, [&](int, int r, int c) { return rows[r * n + c]; });
  constexpr int kEach = V / U;
  const float inv = 1.f / (float)(np * kEach);
  for (int c = threadIdx.x; c < n; c += blockDim.x) mean[c] *= inv;
  __syncthreads();
  // a row has its share of the positions, the first ones one more
  const int each = np / cols.rows, more = np - each * cols.rows;
  const float one = each > 0 ? 1.f / (float)(each * kEach) : 0.f, plus = 1.f / (float)((each + 1) * kEach);
  row_sums<1>(cols, n, red, m2, 0, [&](int, int r, int c) {
    const float count = (float)((each + (r < more)) * kEach), off = rows[r * n + c] * (r < more ? plus : one) - mean[c];
    return rd[r * n + c] + (count > 0.f ? count * off * off : 0.f);
  });
}

// The workgroup's groups from the moments of their `cpg` units (mean[c], m2[c] of `np` values each): done(g, mean, sum of squared distances).  A lane a
// group, or a wavefront a group where they have many units.
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

// What a lane adds up of its positions, by units: start, add, (now and then) fold, close.  close gives sum and squared distances of the lane's mean of `count`
// positions; false: the squared distances are to be added up again from that mean.
//
// Where the values are not kept: sums and squares in 64 bits, of distances from the lane's first value.  A square of two fp32 numbers is exact there, and as the
// first value is one of them its square is at most the sum of squared distances: the difference cancels by at most the number n of values, and n^2 2^-53 of it is
// off, half an fp32 step for 16 384 values of a lane (4 096 x 4 096 pixels of four channels), however far the first one is from the rest.
template <typename T, int V, int U>
struct Moments {
  float first[U];
  double s[U], q[U];
  __device__ __forceinline__ void start(const typename Raw<T, V>::type& raw, bool any) {
    float f[V];
#pragma unroll
    for (int k = 0; k < U; k++) {
      first[k] = 0.f;
      s[k] = q[k] = 0.0;
    }
    if (!any) return;
    unpack(raw, f);
#pragma unroll
    for (int k = 0; k < U; k++) first[k] = f[k * (V / U)];
    if (U < V) add(raw);
  }
  __device__ __forceinline__ void add(const typename Raw<T, V>::type& raw) {
    float f[V];
    unpack(raw, f);
#pragma unroll
    for (int j = 0; j < V; j++) {
      const int k = j / (V / U);
      // (bf16 values 2^16 apart or less: exact in 32 bits)
      const double e = sizeof(T) == 2 ? (double)(f[j] - first[k]) : (double)f[j] - (double)first[k];
      s[k] += e;
      q[k] = fma(e, e, q[k]);
    }
  }
  __device__ __forceinline__ void fold() {}
  __device__ __forceinline__ bool close(int count, float (&sum)[U], float (&dev)[U]) {
    const double n = (double)count * (V / U), inv = count > 0 ? 1.0 / n : 0.0;
#pragma unroll
    for (int k = 0; k < U; k++) {
      dev[k] = (float)fmax(q[k] - s[k] * s[k] * inv, 0.0);
      sum[k] = count > 0 ? (float)fma((double)first[k], n, s[k]) : 0.f;
    }
    return true;
  }
};
// Where they are, in registers: sums in 32 bits (at most 144 values), then the distances in a second pass (the 64-bit operations take longer: 30 x 23 x 20 x 43
// fp32 9.2 us with them, 8.4 so).
template <typename T, int V, int U>
struct HeldMoments {
  float first[U], s[U];
  __device__ __forceinline__ void start(const typename Raw<T, V>::type& raw, bool any) {
    float f[V];
#pragma unroll
    for (int k = 0; k < U; k++) first[k] = s[k] = 0.f;
    if (!any) return;
    unpack(raw, f);
#pragma unroll
    for (int k = 0; k < U; k++) first[k] = f[k * (V / U)];
    if (U < V) add(raw);
  }
  __device__ __forceinline__ void add(const typename Raw<T, V>::type& raw) {
    float f[V];
    unpack(raw, f);
#pragma unroll
    for (int j = 0; j < V; j++) s[j / (V / U)] += f[j] - first[j / (V / U)];
  }
  __device__ __forceinline__ bool close(int count, float (&sum)[U], float (&dev)[U]) {
    const float n = (float)(count * (V / U));
#pragma unroll
    for (int k = 0; k < U; k++) {
      dev[k] = 0.f;
      sum[k] = count > 0 ? fmaf(first[k], n, s[k]) : 0.f;
    }
    return false;
  }
};
// bf16 in units of two channels and more: pairs by the dot product instructions, one instruction a value instead of four.  Distances from 0, so
// where a lane's values are far from 0 against their spread its squared distances are added up again from its mean.  Sums of kFold vectors in
// 32 bits, of more (LONG) in 64: a lane's squares are off by some kFold roundings, and what is left of them after the check by eight times that.  (The 64-bit
// sums' registers cost a lane of few vectors: 288 x 54 x 54 x 96 97 us without them, 101 with.)
constexpr int kFold = 32;
template <int U, bool LONG>
struct DotMoments {
  float s[4], q[4];
  double sum_[U], squares_[U];
  __device__ __forceinline__ void start(const uint4& raw, bool any) {
#pragma unroll
    for (int j = 0; j < 4; j++) s[j] = q[j] = 0.f;
#pragma unroll
    for (int k = 0; k < U; k++) sum_[k] = squares_[k] = 0.0;
    if (any) add(raw);
  }
  __device__ __forceinline__ void add(const uint4& raw) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    const bf2 ones = __builtin_bit_cast(bf2, 0x3f803f80u);
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const bf2 x = __builtin_bit_cast(bf2, w[k]);
      s[k] = __builtin_amdgcn_fdot2_f32_bf16(x, ones, s[k], false);
      q[k] = __builtin_amdgcn_fdot2_f32_bf16(x, x, q[k], false);
    }
  }
  __device__ __forceinline__ void fold() {         // behind every kFold vectors
#pragma unroll
    for (int j = 0; j < 4; j++) {
      sum_[j / (4 / U)] += s[j];
      squares_[j / (4 / U)] += q[j];
      s[j] = q[j] = 0.f;
    }
  }
  __device__ __forceinline__ bool close(int count, float (&sum)[U], float (&dev)[U]) {
    const bool folded = LONG && count > kFold;
    const float inv = count > 0 ? 1.f / ((float)count * (8 / U)) : 0.f;
    bool fine = true;
    if (folded) fold();
#pragma unroll
    for (int k = 0; k < U; k++) {
      float a = 0.f, b = 0.f;
#pragma unroll
      for (int j = k * (4 / U); j < (k + 1) * (4 / U); j++) {
        a += s[j];
        b += q[j];
      }
      if (folded) {
        a = (float)sum_[k];
        b = (float)squares_[k];
      }
      sum[k] = a;
      dev[k] = fmaxf(b - a * a * inv, 0.f);
      fine = fine && !(dev[k] < 0.125f * b);
    }
    return fine;
  }
};
template <typename T, int V, int U, bool HELD, bool LONG> using LaneMoments =
    std::conditional_t<(V == 8 && U < 8), DotMoments<U, LONG>, std::conditional_t<HELD, HeldMoments<T, V, U>, Moments<T, V, U>>>;
// Squared distances from the lane's means, once more.
template <typename T, int V, int U>
__device__ __forceinline__ void add_distances(const typename Raw<T, V>::type& raw, const float (&mean)[U], float (&dev)[U]) {
  float f[V];
  unpack(raw, f);
#pragma unroll
  for (int j = 0; j < V; j++) {
    const float e = f[j] - mean[j / (V / U)];
    dev[j / (V / U)] = fmaf(e, e, dev[j / (V / U)]);
  }
}
__device__ __forceinline__ int count_of(const Lanes& l, int np) { return l.active && l.row < np ? (np - 1 - l.row) / l.rows + 1 : 0; }

// ------------------------------------------------------------------------------------------------ forward
// A workgroup holds a slab of an image.  LDS: scale [S], shift [S], rows [2 threads U], red [threads], mean and m2 of the
// units, group [2 S / cpg]
template <typename T, int V, int U, int NV, int ACT, bool ONCE>
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
  float* scale = lds;
  float* rows = scale + 2 * S;
  float* red = rows + 2 * threads * U;
  float* mean = red + threads;
  float* m2 = mean + S / (V / U);
  float* group = m2 + S / (V / U);
  const Lanes l = lanes_of(cols, t);
  const int count = count_of(l, np), first_c = l.col * V;
  const T* x = (const T*)(base + A.x) + at.image * A.x_image + l.row * A.x_pixel + c0 + first_c;
  const int64_t step = l.rows * A.x_pixel;
  Params par;
  if (t < S) par.fetch(A, wts, c0 + t);
  raw_t held[NV];
  load_rows<ONCE>(held, x, step, count);
  for (int c = t; c < S; c += threads) {
    if (c != t) par.fetch(A, wts, c0 + c);
    par.put(A, scale + c, scale + S + c);
  }
  {
    LaneMoments<T, V, U, true, false> mom;
    float sum[U], dev[U];
    mom.start(held[0], count > 0);
#pragma unroll
    for (int k = 1; k < NV; k++)
      if (k < count) mom.add(held[k]);
    const float inv = 1.f / ((float)count * (V / U));
    if (!mom.close(count, sum, dev)) {
      float mu[U];
#pragma unroll
      for (int j = 0; j < U; j++) {
        mu[j] = sum[j] * inv;
        dev[j] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < NV; k++)
        if (k < count) add_distances<T, V, U>(held[k], mu, dev);
    }
    unit_moments<V, U>(sum, dev, cols, l, np, rows, red, mean, m2);
  }
  group_moments(mean, m2, A.by_cpg(S), cpg / (V / U), np * (V / U), [&](int g, float mu, float sq) {
    const float r = 1.f / sqrtf(sq / ((float)np * (float)cpg) + A.eps);
    group[2 * g] = mu;
    group[2 * g + 1] = r;
    if (A.has_stats) ((float2*)(base + A.stats))[at.image * A.s.groups + A.by_cpg(c0) + g] = make_float2(mu, r);
  });
  __syncthreads();
  if (count == 0) return;
  float mu[V], r[V], sc[V], sh[V], slope[V];
  if (V > 1) {                                       // (S is whole vectors: 16-byte places)
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      *(float4*)(sc + j) = *(const float4*)(scale + first_c + j);
      *(float4*)(sh + j) = *(const float4*)(scale + S + first_c + j);
    }
  } else {
    sc[0] = scale[first_c];
    sh[0] = scale[S + first_c];
  }
#pragma unroll
  for (int j = 0; j < V; j++) {
    const int g = A.by_cpg(first_c + (U == 1 ? 0 : j));
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
      store_row<ONCE>((raw_t*)(y + k * ystep), o);
    }
}

// Images that no workgroup can hold, first launch: the moments of a chunk of positions.  LDS: rows [2 threads U], red [threads], mean and m2 of the units
constexpr int kAhead = 8;            // loads of a lane on their way (288 x 54 x 54 x 96 forward with 4, 8, 16: 98, 94, 102 us)
static_assert(kFold % kAhead == 0, "sums are folded between loads");
template <typename T, int V, int U, bool LONG>
__global__ __launch_bounds__(256) void group_norm_chunk_kernel(const GroupNormArgs A) {
  extern __shared__ float lds[];
  typedef typename Raw<T, V>::type raw_t;
  Place at;
  if (!place_of(A, A.plan.chunks, at)) return;
  const uintptr_t base = A.base[blockIdx.y];
  const int C = A.s.channels, cpg = A.cpg, p0 = at.part * A.plan.chunk, np = min(A.plan.chunk, A.s.positions - p0);
  const int t = threadIdx.x, threads = blockDim.x;
  float* rows = lds;
  float* red = rows + 2 * threads * U;
  float* mean = red + threads;
  float* m2 = mean + C / (V / U);
  const T* x0 = (const T*)(base + A.x) + at.image * A.x_image + (int64_t)p0 * A.x_pixel;
  for (int c0 = 0; c0 < C; c0 += A.cols[0].cols * V) {      // (one turn up to `threads` vectors a pixel)
    const GroupNormCols cols = A.cols[c0 + A.cols[0].cols * V >= C];
    const Lanes l = lanes_of(cols, t);
    const int count = count_of(l, np);
    const T* x = x0 + l.row * A.x_pixel + c0 + l.col * V;
    const int64_t step = l.rows * A.x_pixel;
    LaneMoments<T, V, U, false, LONG> mom;
    float sum[U], dev[U];
    for (int k = 0; k < count || k == 0; k += kAhead) {
      raw_t in[kAhead];
      load_rows<false>(in, x + k * step, step, count - k);
      if (k == 0) mom.start(in[0], count > 0);
      else if (LONG && k % kFold == 0) mom.fold();
#pragma unroll
      for (int i = 0; i < kAhead; i++)
        if (k + i < count && k + i > 0) mom.add(in[i]);
    }
    if (!mom.close(count, sum, dev)) {
      // (read once more: 288 x 54 x 54 x 96 whose channels lie five deviations from 0 114 us instead of 97)
      float mu[U];
      double total[U];
#pragma unroll
      for (int j = 0; j < U; j++) {
        mu[j] = sum[j] / (float)(count * (V / U));
        dev[j] = 0.f;
        total[j] = 0.0;
      }
      for (int k = 0; k < count; k++) {
        add_distances<T, V, U>(*(const raw_t*)(x + k * step), mu, dev);
        if (LONG && k % kFold == kFold - 1)
#pragma unroll
          for (int j = 0; j < U; j++) {
            total[j] += dev[j];
            dev[j] = 0.f;
          }
      }
      if (LONG)
#pragma unroll
        for (int j = 0; j < U; j++) dev[j] = (float)(total[j] + dev[j]);
    }
    unit_moments<V, U>(sum, dev, cols, l, np, rows, red, mean + c0 / (V / U), m2 + c0 / (V / U));
  }
  float2* parts = (float2*)(base + A.parts) + (at.image * A.plan.chunks + at.part) * A.s.groups;
  group_moments(mean, m2, A.s.groups, cpg / (V / U), np * (V / U), [&](int g, float mu, float sq) { parts[g] = make_float2(mu, sq); });
}

// group[2 g], group[2 g + 1]: sums over the image's chunks of value(chunk, group), `spread` lanes a group (neighbouring lanes have neighbouring groups).
// LDS: group [2 groups], then [2 spread groups].
template <typename F>
__device__ __forceinline__ void chunk_sums(float* group, int G, int chunks, int spread, F value) {
  float2* part = (float2*)(group + 2 * G);
  const int t = threadIdx.x, T = blockDim.x;
  for (int i = t; i < G * spread; i += T) {
    const int s = i / G, g = i - s * G;
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int k = s; k < chunks; k += spread) {
      const float2 v = value(k, g);
      sum.x += v.x;
      sum.y += v.y;
    }
    part[i] = sum;
  }
  __syncthreads();
  for (int g = t; g < G; g += T) {
    float2 sum = part[g];
    for (int s = 1; s < spread; s++) {
      sum.x += part[s * G + g].x;
      sum.y += part[s * G + g].y;
    }
    group[2 * g] = sum.x;
    group[2 * g + 1] = sum.y;
  }
  __syncthreads();
}

// Second launch: the image's statistics from its chunks', then y.  LDS: see chunk_sums
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
  // the first values are on their way while the statistics are put together
  const T* xp = (const T*)(base + A.x) + at.image * A.x_image + (int64_t)p0 * A.x_pixel;
  raw_t in[kAhead];
  {
    const Lanes l = lanes_of(A.cols[A.cols[0].cols * V >= C], t);
    load_rows<true>(in, xp + l.row * A.x_pixel + l.col * V, l.rows * A.x_pixel, count_of(l, np));
  }
  const float2* parts = (const float2*)(base + A.parts) + at.image * chunks * G;
  const float last = (float)(A.s.positions - (chunks - 1) * chunk), full = (float)chunk, total = (float)A.s.positions, cpg = (float)A.cpg;
  // distances of the chunks' means from the first one's: sums of n d and of n d^2 + the chunks' own
  chunk_sums(group, G, chunks, A.spread, [&](int k, int g) {
    const float2 p = parts[k * G + g];
    const float n = (k < chunks - 1 ? full : last), d = p.x - parts[g].x;
    return make_float2(n * d, n * cpg * d * d + p.y);
  });
  for (int g = t; g < G; g += threads) {
    const float s = group[2 * g] / total, m2 = __builtin_elementwise_maximum(group[2 * g + 1] - total * cpg * s * s, 0.f);       // (NaN stays)
    const float mu = parts[g].x + s, r = 1.f / sqrtf(m2 / (total * cpg) + A.eps);
    group[2 * g] = mu;
    group[2 * g + 1] = r;
    if (A.has_stats && at.part == 0) ((float2*)(base + A.stats))[at.image * G + g] = make_float2(mu, r);
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
    const T* x = xp + l.row * A.x_pixel + c;
    T* y = (T*)(base + A.y) + at.image * A.y_image + (int64_t)(p0 + l.row) * A.y_pixel + c;
    const int64_t step = l.rows * A.x_pixel, ystep = l.rows * A.y_pixel;
    auto one = [&](const raw_t& in, int k) {
      float f[V];
      unpack(in, f);
#pragma unroll
      for (int j = 0; j < V; j++) f[j] = activate<ACT>(affine<ACT>(f[j] - mu[j], r[j], sc[j], slope[j], sh[j]));
      raw_t o;
      pack(o, f);
      store_once((raw_t*)(y + k * ystep), o);
    };
    for (int k = 0; k < count; k += kAhead) {
      if (k > 0 || c0 > 0) load_rows<true>(in, x + k * step, step, count - k);
#pragma unroll
      for (int i = 0; i < kAhead; i++)
        if (k + i < count) one(in[i], k + i);
    }
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

// The workgroup's channel sums (`n` channels: sa of dz, sb of dz xhat) to `out`, then times scale(c) in place, for the groups' s1 and s2.
template <typename F>
__device__ __forceinline__ void store_sums(float* sa, float* sb, int n, float2* out, F scale) {
  for (int c = threadIdx.x; c < n; c += blockDim.x) {
    const float w = scale(c);
    out[c] = make_float2(sb[c], sa[c]);
    sa[c] *= w;
    sb[c] *= w;
  }
  __syncthreads();
}
// s1 and s2 of the workgroup's groups from those: done(g, s1, s2)
template <typename F>
__device__ __forceinline__ void group_gradient(const float* sa, const float* sb, int cpg, int groups, F done) {
  const int t = threadIdx.x, T = blockDim.x;
  if (cpg <= kLaneChannels) {
    for (int g = t; g < groups; g += T) {
      float s1 = 0.f, s2 = 0.f;
      for (int c = g * cpg; c < (g + 1) * cpg; c++) {
        s1 += sa[c];
        s2 += sb[c];
      }
      done(g, s1, s2);
    }
    return;
  }
  const int lane = t & 63;
  for (int g = t >> 6; g < groups; g += T >> 6) {
    float s1 = 0.f, s2 = 0.f;
    for (int c = g * cpg + lane; c < (g + 1) * cpg; c += 64) {
      s1 += sa[c];
      s2 += sb[c];
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

// A workgroup holds a slab of x and dy.  LDS: scale [S], shift [S], rows [2 threads V], red [2 threads], sa [S], sb [S], group [2 S / cpg]
template <typename T, int V, int NV, int ACT, bool ONCE>
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
  float* scale = lds;
  float* rows = scale + 2 * S;
  float* red = rows + 2 * threads * V;
  float* sums = red + 2 * threads;
  float* group = sums + 2 * S;
  const Lanes l = lanes_of(cols, t);
  const int count = count_of(l, np), first_c = l.col * V;
  const T* x = (const T*)(base + A.x) + at.image * A.x_image + l.row * A.x_pixel + c0 + first_c;
  const T* dy = (const T*)(base + A.dy) + at.image * A.y_image + l.row * A.y_pixel + c0 + first_c;
  const int64_t step = l.rows * A.x_pixel, ystep = l.rows * A.y_pixel;
  const int gs = A.by_cpg(S);
  const float2* stats = (const float2*)(base + A.stats) + at.image * A.s.groups + A.by_cpg(c0);
  Params par;
  float2 stat = make_float2(0.f, 0.f);
  if (t < S) par.fetch(A, wts, c0 + t);
  if (t < gs) stat = stats[t];
  raw_t hx[NV];
  typename Kept<T, V, ACT>::type hz[NV];
  GradientLane<V> p;
  {
    raw_t hd[NV];
    load_rows<ONCE>(hx, x, step, count);
    load_rows<ONCE>(hd, dy, ystep, count);
    for (int c = t; c < S; c += threads) {
      if (c != t) par.fetch(A, wts, c0 + c);
      par.put(A, scale + c, scale + S + c);
    }
    for (int g = t; g < gs; g += threads) {
      if (g != t) stat = stats[g];
      group[2 * g] = stat.x;
      group[2 * g + 1] = stat.y;
    }
    __syncthreads();
    if (V > 1) {                                     // (S is whole vectors: 16-byte places)
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        *(float4*)(p.sc + j) = *(const float4*)(scale + first_c + j);
        *(float4*)(p.sh + j) = *(const float4*)(scale + S + first_c + j);
      }
    } else {
      p.sc[0] = scale[first_c];
      p.sh[0] = scale[S + first_c];
    }
#pragma unroll
    for (int j = 0; j < V; j++) {
      const int g = A.by_cpg(first_c + j);
      p.mu[j] = group[2 * g];
      p.r[j] = group[2 * g + 1];
      p.slope[j] = p.r[j] * p.sc[j];
    }
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
  store_sums(sums, sums + S, S, (float2*)(base + A.sums) + at.image * C + c0, [&](int c) { return scale[c]; });
  if (!A.has_dx) return;
  group_gradient(sums, sums + S, A.cpg, gs, [&](int g, float s1, float s2) {
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
      store_row<ONCE>((raw_t*)(dx + k * ystep), o);
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
    constexpr int kPairs = kAhead / 2;
    for (int k = 0; k < count; k += kPairs) {
      raw_t ix[kPairs], id[kPairs];
      load_rows<false>(ix, x + k * step, step, count - k);
      load_rows<false>(id, dy + k * ystep, ystep, count - k);
#pragma unroll
      for (int i = 0; i < kPairs; i++)
        if (k + i < count) one(ix[i], id[i]);
    }
    gradient_sums<V>(a, b, p, cols, l, rows, red, sa + c0, C);
  }
  store_sums(sa, sb, C, (float2*)(base + A.sums) + (at.image * A.plan.chunks + at.part) * C,
             [&](int c) { return A.has_scale ? param(A, wts + A.scale, c) : 1.f; });
  if (!A.has_dx) return;
  float2* parts = (float2*)(base + A.parts) + (at.image * A.plan.chunks + at.part) * A.s.groups;
  group_gradient(sa, sb, A.cpg, A.s.groups, [&](int g, float s1, float s2) { parts[g] = make_float2(s1, s2); });
}

// Second launch: s1 and s2 of the image from its chunks', then dx.  LDS: see chunk_sums
template <typename T, int V, int ACT>
__global__ __launch_bounds__(256) void group_norm_gradient_apply_kernel(const GroupNormArgs A) {
  extern __shared__ float group[];
  typedef typename Raw<T, V>::type raw_t;
  Place at;
  if (!place_of(A, A.plan.chunks, at)) return;
  const uintptr_t base = A.base[blockIdx.y], wts = A.wts[blockIdx.y];
  const int C = A.s.channels, G = A.s.groups, chunks = A.plan.chunks;
  const int p0 = at.part * A.plan.chunk, np = min(A.plan.chunk, A.s.positions - p0);
  const int t = threadIdx.x;
  // the first values are on their way while the sums are put together
  constexpr int kPairs = kAhead / 2;
  const T* xp = (const T*)(base + A.x) + at.image * A.x_image + (int64_t)p0 * A.x_pixel;
  const T* dp = (const T*)(base + A.dy) + at.image * A.y_image + (int64_t)p0 * A.y_pixel;
  raw_t ix[kPairs], id[kPairs];
  {
    const Lanes l = lanes_of(A.cols[A.cols[0].cols * V >= C], t);
    const int count = count_of(l, np);
    load_rows<true>(ix, xp + l.row * A.x_pixel + l.col * V, l.rows * A.x_pixel, count);
    load_rows<true>(id, dp + l.row * A.y_pixel + l.col * V, l.rows * A.y_pixel, count);
  }
  const float2* parts = (const float2*)(base + A.parts) + at.image * chunks * G;
  const float inv = 1.f / ((float)A.s.positions * (float)A.cpg);
  chunk_sums(group, G, chunks, A.spread, [&](int k, int g) { return parts[k * G + g]; });
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
      b[j] = -p.r[j] * (group[2 * g] * inv);
      c[j] = -p.r[j] * p.r[j] * (group[2 * g + 1] * inv);
    }
    const T* x = xp + l.row * A.x_pixel + ch;
    const T* dy = dp + l.row * A.y_pixel + ch;
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
      store_once((raw_t*)(dx + k * ystep), o);
    };
    for (int k = 0; k < count; k += kPairs) {
      if (k > 0 || c0 > 0) {
        load_rows<true>(ix, x + k * step, step, count - k);
        load_rows<true>(id, dy + k * ystep, ystep, count - k);
      }
#pragma unroll
      for (int i = 0; i < kPairs; i++)
        if (k + i < count) one(ix[i], id[i], k + i);
    }
  }
}

// dscale, dshift: rows of channel sums [rows][C][2] added, 32 channels a workgroup and 32 rows at a time.  Many rows in two launches: the first
// leaves a row per blockIdx.y (`per` rows each).  In one launch and in two, the whole gradient of n x 32 x 32 x 32: n = 256 20 and 23 us, 512 28 and 29,
// 2 304 111 and 105.
constexpr int64_t kFinishRows = 512;
template <bool LAST>
__global__ __launch_bounds__(1024) void group_norm_finish_kernel(const GroupNormArgs A, int64_t from, int64_t rows, int64_t per, int64_t to) {
  __shared__ float2 part[32][33];
  const int learner = blockIdx.z, ch = threadIdx.x & 31, seg = threadIdx.x >> 5, c = blockIdx.x * 32 + ch, C = A.s.channels;
  const int64_t r0 = blockIdx.y * per, r1 = r0 + per < rows ? r0 + per : rows;
  const float2* sums = (const float2*)(A.base[learner] + from);
  float a = 0.f, b = 0.f;
  if (c < C) {
#pragma unroll 8
    for (int64_t k = r0 + seg; k < r1; k += 32) {
      const float2 s = sums[k * C + c];
      a += s.x;
      b += s.y;
    }
  }
  part[seg][ch] = make_float2(a, b);
  __syncthreads();
  // a wavefront's halves take one channel each: its 32 rows
  const int row = threadIdx.x & 31, own = threadIdx.x >> 5;
  float2 s = part[row][own];
  for (int o = 16; o > 0; o >>= 1) {
    s.x += __shfl_xor(s.x, o, 64);
    s.y += __shfl_xor(s.y, o, 64);
  }
  const int to_c = blockIdx.x * 32 + own;
  if (row != 0 || to_c >= C) return;
  if (!LAST) {
    ((float2*)(A.base[learner] + to))[(int64_t)blockIdx.y * C + to_c] = s;
  } else {
    if (A.has_dscale) ((float*)(A.grads[learner] + A.dscale))[to_c] = s.x;
    if (A.has_dshift) ((float*)(A.grads[learner] + A.dshift))[to_c] = s.y;
  }
}

int64_t finish_splits(int64_t rows) { return rows <= kFinishRows ? 0 : std::min<int64_t>((rows + 127) / 128, kFinishRows); }

size_t lds_bytes(const GroupNormArgs& a, bool gradient) {
  const int S = a.plan.whole ? a.plan.slab : a.s.channels, T = a.plan.threads;
  return ((size_t)T * (2 * a.plan.vec + (gradient ? 2 : 1)) + 2 * S + (a.plan.whole ? 2 * (S / a.cpg) + 2 * S : 0)) * 4;
}

}  // namespace

constexpr int kHeldForward[] = {4, 8, 16, 24, 36}, kHeldBackward[] = {4, 8, 12, 16, 24}, kHeldNarrow[] = {8, 24};

// Small images are held whole, in slabs of whole groups and whole vectors: the smallest that makes segments of 128 bytes a pixel, or 64 where no more
// fit in, or all channels (288 x 27 x 27 x 256, bf16, in segments of 128 bytes, of 64, in chunks: gradient 78, 87, 111 us, forward 49, 61, 65).  Larger
// ones where there are kPlenty workgroups all the same (7 x 7 x 512, with and without: 4 096 images forward 73 and 102 us, gradient 119 and 213; 512 images
// 11 and 17, 27 and 36; with 2 048 for kPlenty 512 images stay without), smaller ones where the launch would have fewer workgroups than the chip has places.
// Workgroups that share lines go through the caches, and hold up to eight vectors a lane (20 x 20 x 320, held and in chunks: 64 images forward 12 and
// 21 us, 1 024 152 and 140; gradient 21 and 40, 199 and 251.  288 x 54 x 54 x 96, 36 vectors: 106 and 94).
constexpr int64_t kPlenty = 1024;
// Chunks (64 x 64 x 128 in rounds of 512 and 1 024 workgroups: 16 images forward 18 and 21 us, gradient 30 and 38, 32 images 23 and 25, 42 and 49;
// 288 x 54 x 54 x 96 forward 96 and 93.  128 x 128 x 320 in at most 64, 128 and 256: one image forward 50, 44, 56, gradient 75, 76, 90, 16 forward 90, 96, 100).
constexpr int64_t kRound = 512, kMostChunks = 64;

GroupNormPlan group_norm_plan(const GroupNormShape& s, bool wide, bool gradient, bool silu, int learners) {
  GroupNormPlan p;
  const int size = s.bf16 ? 2 : 4, cpg = s.channels / s.groups;
  p.vec = wide ? 16 / size : 1;
  p.once = true;
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
        if (held <= (silu && s.bf16 ? 16 : 24) && fits(256, held)) return true;
      return false;
    }
    for (int held : kHeldForward)
      if (fits(256, held)) return true;
    return false;
  };
  auto slabs = [&](int slab) { return s.images * learners * ((s.channels + slab - 1) / slab); };
  auto shares_lines = [&](int slab) { return slab < s.channels && ((slab * size) % 64 != 0 || (s.channels * size) % 64 != 0); };
  for (int bytes = 128; bytes >= 64; bytes /= 2) {
    int slab = std::min(s.channels, (bytes / size + unit - 1) / unit * unit);
    // many small images: larger slabs while there are workgroups enough and a lane holds no more than eight vectors
    while (slab < s.channels && slabs(slab * 2) >= kPlenty && (int64_t)std::min(slab * 2, s.channels) / p.vec * s.positions <= 256 * 8) slab = std::min(slab * 2, s.channels);
    while (slab > unit && slabs(slab) < 512) slab = std::max(unit, slab / 2 / unit * unit);
    if (!take(slab)) continue;
    p.once = !shares_lines(slab);
    if (p.once || p.held <= 8) return p;
  }
  p.whole = false;
  p.slab = s.channels;
  p.slabs = 1;
  p.threads = 256;
  p.held = 0;
  // chunks of about 64 KiB, and whole rounds of kRound workgroups of them
  const int64_t image = (int64_t)s.positions * s.channels * size, images = std::max<int64_t>(1, s.images * learners);
  const int64_t rounds = (images * ((image + 1023) / 1024) + kRound * 64 - 1) / (kRound * 64);
  int64_t chunks = std::min(std::min(kRound * rounds / images, image / 16384), kMostChunks);
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
static void set_columns(GroupNormArgs& a, int units) {       // units: of a vector, that sums go by
  const int V = a.plan.vec, all = (a.plan.whole ? a.plan.slab : a.s.channels) / V, most = std::min(all, a.plan.threads);
  const int last = a.plan.whole ? (a.s.channels - (a.plan.slabs - 1) * a.plan.slab) / V : all - (all - 1) / most * most;
  for (int k = 0; k < 2; k++) {
    GroupNormCols& c = a.cols[k];
    c.cols = k ? last : most;
    c.rows = a.plan.threads / c.cols;
    c.by_cols.set(c.cols);
    const int n = c.cols * units;
    c.segs = a.plan.threads / n;
    c.by_n.set(n);
    c.fold = n < 64 && (n & (n - 1)) == 0;
  }
  a.cpg = a.s.channels / a.s.groups;
  a.by_cpg.set(a.cpg);
  for (a.spread = 1; a.spread * 2 <= a.plan.chunks && a.spread * 2 * a.s.groups <= a.plan.threads;) a.spread *= 2;
}

#define BY_ACTIVATION(launch)                                                  \
  (a.activation == SASGD_ACT_RELU ? launch(std::integral_constant<int, SASGD_ACT_RELU>()) \
   : a.activation == SASGD_ACT_SILU ? launch(std::integral_constant<int, SASGD_ACT_SILU>()) : launch(std::integral_constant<int, SASGD_ACT_NONE>()))

template <typename T, int V, int U, int NV>
static void forward_held(const GroupNormArgs& a, dim3 grid, hipStream_t stream) {
  auto launch = [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    if constexpr (NV <= 8 && V > 1)
      if (!a.plan.once) return group_norm_kernel<T, V, U, NV, ACT, false><<<grid, a.plan.threads, lds_bytes(a, false), stream>>>(a);
    group_norm_kernel<T, V, U, NV, ACT, true><<<grid, a.plan.threads, lds_bytes(a, false), stream>>>(a);
  };
  BY_ACTIVATION(launch);
}
template <typename T, int V, int NV>
static void backward_held(const GroupNormArgs& a, dim3 grid, hipStream_t stream) {
  auto launch = [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    if constexpr (NV <= 8 && V > 1)
      if (!a.plan.once) return group_norm_gradient_kernel<T, V, NV, ACT, false><<<grid, a.plan.threads, lds_bytes(a, true), stream>>>(a);
    // (behind silu dz of bf16 is kept in 32 bits: up to 16 vectors, group_norm_plan)
    if constexpr (!(NV > 16 && ACT == SASGD_ACT_SILU && V == 8)) group_norm_gradient_kernel<T, V, NV, ACT, true><<<grid, a.plan.threads, lds_bytes(a, true), stream>>>(a);
  };
  BY_ACTIVATION(launch);
}

template <typename T, int V, int U>
static hipError_t forward(GroupNormArgs& a, hipStream_t stream) {
  set_columns(a, U);
  const dim3 grid(workgroups(a), (uint32_t)a.learners);
  if (a.plan.whole) {
    if constexpr (V == 1) {
      if (a.plan.held == 8) forward_held<T, V, U, 8>(a, grid, stream);
      else forward_held<T, V, U, 24>(a, grid, stream);
    } else {
      switch (a.plan.held) {
        case 4: forward_held<T, V, U, 4>(a, grid, stream); break;
        case 8: forward_held<T, V, U, 8>(a, grid, stream); break;
        case 16: forward_held<T, V, U, 16>(a, grid, stream); break;
        case 24: forward_held<T, V, U, 24>(a, grid, stream); break;
        default: forward_held<T, V, U, 36>(a, grid, stream); break;
      }
    }
    return hipGetLastError();
  }
  if (V == 8 && U < 8 && a.plan.chunk > kFold * a.cols[0].rows) group_norm_chunk_kernel<T, V, U, V == 8 && U < 8><<<grid, a.plan.threads, lds_bytes(a, false), stream>>>(a);
  else group_norm_chunk_kernel<T, V, U, false><<<grid, a.plan.threads, lds_bytes(a, false), stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto launch = [&](auto act) { group_norm_apply_kernel<T, V, decltype(act)::value><<<grid, a.plan.threads, (size_t)a.s.groups * (1 + a.spread) * 8, stream>>>(a); };
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
        case 16: backward_held<T, V, 16>(a, grid, stream); break;
        default: backward_held<T, V, 24>(a, grid, stream); break;
      }
    }
    return hipGetLastError();
  }
  auto sums = [&](auto act) { group_norm_gradient_chunk_kernel<T, V, decltype(act)::value><<<grid, a.plan.threads, lds_bytes(a, true), stream>>>(a); };
  BY_ACTIVATION(sums);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.has_dx) return e;
  auto launch = [&](auto act) { group_norm_gradient_apply_kernel<T, V, decltype(act)::value><<<grid, a.plan.threads, (size_t)a.s.groups * (1 + a.spread) * 8, stream>>>(a); };
  BY_ACTIVATION(launch);
  return hipGetLastError();
}

// A launch holds fewer than 2^32 lanes: the images, as many at a time as that takes.  launch(a): those of a.s from a.x, a.y, a.dy, a.dx, a.stats, a.parts and
// a.sums on, which move on behind them.
template <typename F>
static hipError_t by_images(GroupNormArgs& a, F launch) {
  const int64_t parts = a.plan.whole ? a.plan.slabs : a.plan.chunks, most = (((int64_t)1 << 32) - 1) / (parts * a.plan.threads) / 8 * 8;
  const int64_t size = a.s.bf16 ? 2 : 4, all = a.s.images;
  hipError_t e = hipSuccess;
  for (int64_t left = all; left > 0 && e == hipSuccess;) {
    a.s.images = std::min(left, most);
    e = launch(a);
    left -= a.s.images;
    if (left == 0) break;
    a.x += a.s.images * a.x_image * size;
    a.y += a.s.images * a.y_image * size;
    a.dy += a.s.images * a.y_image * size;
    a.dx += a.s.images * a.y_image * size;
    a.stats += a.s.images * a.s.groups * 8;
    a.parts += a.s.images * a.plan.chunks * a.s.groups * 8;
    a.sums += a.s.images * a.plan.chunks * a.s.channels * 8;
  }
  a.s.images = all;
  return e;
}

hipError_t launch_group_norm(GroupNormArgs& a, hipStream_t stream) {
  const int cpg = a.s.channels / a.s.groups;
  return by_images(a, [&](GroupNormArgs& a) {
    if (a.s.bf16 && a.plan.vec == 8) return cpg % 8 == 0 ? forward<bf16_t, 8, 1>(a, stream) : cpg % 2 == 0 ? forward<bf16_t, 8, 4>(a, stream) : forward<bf16_t, 8, 8>(a, stream);
    if (a.s.bf16) return forward<bf16_t, 1, 1>(a, stream);
    if (a.plan.vec == 4) return cpg % 4 == 0 ? forward<float, 4, 1>(a, stream) : forward<float, 4, 4>(a, stream);
    return forward<float, 1, 1>(a, stream);
  });
}

hipError_t launch_group_norm_gradient(GroupNormArgs& a, hipStream_t stream) {
  int64_t from = a.sums;
  hipError_t e = by_images(a, [&](GroupNormArgs& a) {
    set_columns(a, a.plan.vec);
    if (a.s.bf16) return a.plan.vec == 8 ? backward<bf16_t, 8>(a, stream) : backward<bf16_t, 1>(a, stream);
    return a.plan.vec == 4 ? backward<float, 4>(a, stream) : backward<float, 1>(a, stream);
  });
  if (e != hipSuccess || (!a.has_dscale && !a.has_dshift)) return e;
  const int64_t rows = a.s.images * a.plan.chunks, splits = finish_splits(rows);
  const uint32_t strips = (uint32_t)(a.s.channels + 31) / 32, learners = (uint32_t)a.learners;
  int64_t left = rows;
  if (splits > 0) {
    const int64_t to = from + rows * a.s.channels * 8, per = (rows + splits - 1) / splits;
    group_norm_finish_kernel<false><<<dim3(strips, (uint32_t)splits, learners), 1024, 0, stream>>>(a, from, rows, per, to);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    from = to;
    left = splits;
  }
  group_norm_finish_kernel<true><<<dim3(strips, 1, learners), 1024, 0, stream>>>(a, from, left, left, 0);
  return hipGetLastError();
}

}  // namespace sasgd
