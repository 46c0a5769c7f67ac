// AdamW over many tensors in one launch, and the norm over many tensors.
//
// Both walk blocks of 256 consecutive elements of a tensor, a wavefront a block (4 elements a lane), and find a block's tensor in a
// table that the kernel's arguments carry: nothing is copied to the device beforehand, and work is spread over the chip by
// blocks whatever the sizes of the tensors.  Both are bound by HBM.
#include <math.h>

#include "dev_common.hpp"
#include "operators.hpp"

namespace sasgd {

namespace {

constexpr int kRun = 4;            // blocks a wavefront has on their way at a time

// The tensor of block b (a uniform value): the last k with first[k] <= b.  Empty tensors are not in the table.
__device__ __forceinline__ int tensor_of(const TensorTable& tab, uint32_t b) {
  int lo = 0, hi = tab.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.first[mid] <= b) lo = mid; else hi = mid - 1;
  }
  return lo;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void load4(float (&d)[4], const float* p) {
  const f32x4 v = *reinterpret_cast<const f32x4*>(p);
  d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
}
__device__ __forceinline__ void load4(float (&d)[4], const bf16_t* p) {
  const u32x2 v = *reinterpret_cast<const u32x2*>(p);
  d[0] = __uint_as_float(v.x << 16); d[1] = __uint_as_float(v.x & 0xffff0000u);
  d[2] = __uint_as_float(v.y << 16); d[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, const float (&d)[4]) {
  const f32x4 v = {d[0], d[1], d[2], d[3]};
  *reinterpret_cast<f32x4*>(p) = v;
}
__device__ __forceinline__ void store4(bf16_t* p, const float (&d)[4]) {
  const u32x2 v = {pack2bf(d[0], d[1]), pack2bf(d[2], d[3])};
  *reinterpret_cast<u32x2*>(p) = v;
}

// ------------------------------------------------------------------------------------------------ e4m3
__host__ __device__ inline uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xB7E15163u;
  return x ^ (x >> 16);
}

// Largest of the wavefront's values, in every lane: four shifts within rows of 16 lanes, then rows to rows.
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#define STEP(ctrl)                                                                          \
  {                                                                                         \
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, true); \
    v = o > v ? o : v;                                                                      \
  }
  STEP(0x111) STEP(0x112) STEP(0x114) STEP(0x118) STEP(0x142) STEP(0x143)
#undef STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// y in 0 .. 448 (a little beyond by rounding) to an e4m3 value, up with the probability of what is cut off.  e4m3 has 3 bits of
// fraction and even steps of 2^-9 below 2^-6, which are those of the binade from 2^-6 on: values below are moved there and back.
__device__ __forceinline__ float round8(float y, uint32_t chance) {
#pragma clang fp contract(off)
  const bool small = y < 0x1p-6f;
  const float x = small ? y + 0x1p-6f : y;
  const float r = __uint_as_float((__float_as_uint(x) + (chance << 4)) & 0xfff00000u);
  return fminf(small ? r - 0x1p-6f : r, 448.0f);
}

// ------------------------------------------------------------------------------------------------ one block
// What a wavefront holds of a block: element e of lane `lane` is 4 lane + j (vector moves) or lane + 64 j.
template <bool VEC>
__device__ __forceinline__ int element(int lane, int j) { return VEC ? 4 * lane + j : lane + 64 * j; }

struct AdamwStep {
  float pace, vcorr, factor;
  uint32_t key;
  bool scaled, skip;
};

template <typename G, bool E4M3, bool VEC, int R>
__device__ __forceinline__ void adamw_blocks(const AdamwLaunch& A, const AdamwStep& S, const uint64_t* w, const float* share, int64_t at, int64_t left,
                                             int64_t block, int lane) {
#pragma clang fp contract(off)
  // `at`: first element within the tensor, `left`: elements of the tensor from there on, `block`: moments' block
  const float* tin = (const float*)w[1] + at;
  float* tout = A.has_out ? (float*)w[2] + at : const_cast<float*>(tin);
  float th[R][4], g[R][4], m[R][4], v[R][4];
  uint32_t m8[R], u8[R];
  float ms[R], us[R];
  int64_t s0 = block * kMomentBlock;
#pragma unroll
  for (int r = 0; r < R; r++) {
    if (VEC) {
      load4(g[r], (const G*)w[A.grads_at] + at + r * kMomentBlock + 4 * lane);
      load4(th[r], tin + r * kMomentBlock + 4 * lane);
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int e = r * kMomentBlock + element<false>(lane, j);
        g[r][j] = e < left ? ldf((const G*)w[A.grads_at] + at + e) : 0.f;
        th[r][j] = e < left ? tin[e] : 0.f;
      }
    }
    if (E4M3) {
      ms[r] = A.m_scale[block + r];
      us[r] = A.v_scale[block + r];
      if (VEC) {
        m8[r] = *(const uint32_t*)((const uint8_t*)A.m + s0 + r * kMomentBlock + 4 * lane);
        u8[r] = *(const uint32_t*)((const uint8_t*)A.v + s0 + r * kMomentBlock + 4 * lane);
      } else {
        m8[r] = u8[r] = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const int e = element<false>(lane, j);
          if (r * kMomentBlock + e >= left) continue;
          m8[r] |= (uint32_t)((const uint8_t*)A.m)[s0 + r * kMomentBlock + e] << (8 * j);
          u8[r] |= (uint32_t)((const uint8_t*)A.v)[s0 + r * kMomentBlock + e] << (8 * j);
        }
      }
    } else if (VEC) {
      load4(m[r], (const float*)A.m + s0 + r * kMomentBlock + 4 * lane);
      load4(v[r], (const float*)A.v + s0 + r * kMomentBlock + 4 * lane);
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int e = r * kMomentBlock + element<false>(lane, j);
        m[r][j] = e < left ? ((const float*)A.m)[s0 + e] : 0.f;
        v[r][j] = e < left ? ((const float*)A.v)[s0 + e] : 0.f;
      }
    }
  }
  if (A.c > 1) {
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
      for (int j = 0; j < 4; j++) g[r][j] = g[r][j] * share[0];
#pragma unroll 2
    for (int l = 1; l < A.c; l++) {
      const G* gl = (const G*)w[A.grads_at + l] + at;
      const float part = share[l];
      float t[R][4];
#pragma unroll
      for (int r = 0; r < R; r++) {
        if (VEC) {
          load4(t[r], gl + r * kMomentBlock + 4 * lane);
        } else {
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const int e = r * kMomentBlock + element<false>(lane, j);
            t[r][j] = e < left ? ldf(gl + e) : 0.f;
          }
        }
      }
#pragma unroll
      for (int r = 0; r < R; r++)
#pragma unroll
        for (int j = 0; j < 4; j++) g[r][j] = g[r][j] + t[r][j] * part;
    }
  }
#pragma unroll
  for (int r = 0; r < R; r++) {
    if (E4M3) {
      m[r][0] = __builtin_amdgcn_cvt_f32_fp8((int)m8[r], 0) * ms[r];
      m[r][1] = __builtin_amdgcn_cvt_f32_fp8((int)m8[r], 1) * ms[r];
      m[r][2] = __builtin_amdgcn_cvt_f32_fp8((int)m8[r], 2) * ms[r];
      m[r][3] = __builtin_amdgcn_cvt_f32_fp8((int)m8[r], 3) * ms[r];
      v[r][0] = __builtin_amdgcn_cvt_f32_fp8((int)u8[r], 0) * us[r];
      v[r][1] = __builtin_amdgcn_cvt_f32_fp8((int)u8[r], 1) * us[r];
      v[r][2] = __builtin_amdgcn_cvt_f32_fp8((int)u8[r], 2) * us[r];
      v[r][3] = __builtin_amdgcn_cvt_f32_fp8((int)u8[r], 3) * us[r];
#pragma unroll
      for (int j = 0; j < 4; j++) v[r][j] = v[r][j] * v[r][j];
    }
    uint32_t mbits = 0, ubits = 0;
    float u[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      float gg = g[r][j];
      if (S.scaled) gg = gg * S.factor;
      m[r][j] = m[r][j] * A.beta1 + gg * A.rest1;
      v[r][j] = v[r][j] * A.beta2 + (gg * gg) * A.rest2;
      const float move = (m[r][j] * S.pace) / (sqrtf(v[r][j] * S.vcorr) + A.epsilon);
      if (!S.skip) th[r][j] = th[r][j] * A.keep - move;
      if (E4M3) {
        u[j] = sqrtf(v[r][j]);
        mbits = max(mbits, __float_as_uint(fabsf(m[r][j])));       // (bits of NaN are the largest)
        ubits = max(ubits, __float_as_uint(u[j]) & 0x7fffffffu);
      }
    }
    // ---- store
    if (VEC) {
      if (!S.skip || A.has_out) store4(tout + r * kMomentBlock + 4 * lane, th[r]);
      if (A.has_shadow) {
        bf16_t* sh = (bf16_t*)w[2 + A.has_out];
        if (sh) store4(sh + at + r * kMomentBlock + 4 * lane, th[r]);
      }
    } else {
      bf16_t* sh = A.has_shadow ? (bf16_t*)w[2 + A.has_out] : nullptr;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int e = r * kMomentBlock + element<false>(lane, j);
        if (e >= left) continue;
        tout[e] = th[r][j];
        if (sh) sh[at + e] = f2bf(th[r][j]);
      }
    }
    if (S.skip) continue;
    if (E4M3) {
      mbits = wave_umax(mbits);
      ubits = wave_umax(ubits);
      const bool mbad = mbits >= 0x7f800000u, ubad = ubits >= 0x7f800000u;
      float mmost = __uint_as_float(mbits), umost = __uint_as_float(ubits);
      if (mmost < 1e-30f) mmost = 0.f;
      if (umost < 1e-30f) umost = 0.f;
      const float mup = mmost > 0.f ? (1.0f / mmost) * 448.0f : 0.f, uup = umost > 0.f ? (1.0f / umost) * 448.0f : 0.f;
      if (lane == 0) {
        A.m_scale[block + r] = mbad ? NAN : mmost * (1.0f / 448.0f);
        A.v_scale[block + r] = ubad ? NAN : umost * (1.0f / 448.0f);
      }
      float mq[4], uq[4];
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int64_t e = s0 + r * kMomentBlock + element<VEC>(lane, j);
        const uint32_t chance = mix32((uint32_t)e * 0x9E3779B1u ^ (uint32_t)(e >> 32) * 0x243F6A89u ^ S.key);
        const float ym = fabsf(m[r][j]) * mup, yu = u[j] * uup;
        mq[j] = ym > 0.f ? copysignf(round8(ym, chance >> 16), m[r][j]) : 0.f;
        uq[j] = yu > 0.f ? fmaxf(round8(yu, chance & 0xffffu), 0x1p-9f) : 0.f;
      }
      int pm = __builtin_amdgcn_cvt_pk_fp8_f32(mq[0], mq[1], 0, false);
      pm = __builtin_amdgcn_cvt_pk_fp8_f32(mq[2], mq[3], pm, true);
      int pu = __builtin_amdgcn_cvt_pk_fp8_f32(uq[0], uq[1], 0, false);
      pu = __builtin_amdgcn_cvt_pk_fp8_f32(uq[2], uq[3], pu, true);
      if (VEC) {
        *(uint32_t*)((uint8_t*)A.m + s0 + r * kMomentBlock + 4 * lane) = (uint32_t)pm;
        *(uint32_t*)((uint8_t*)A.v + s0 + r * kMomentBlock + 4 * lane) = (uint32_t)pu;
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++) {     // whole blocks: zeros behind a tensor's end
          ((uint8_t*)A.m)[s0 + r * kMomentBlock + element<false>(lane, j)] = (uint8_t)(pm >> (8 * j));
          ((uint8_t*)A.v)[s0 + r * kMomentBlock + element<false>(lane, j)] = (uint8_t)(pu >> (8 * j));
        }
      }
    } else if (VEC) {
      store4((float*)A.m + s0 + r * kMomentBlock + 4 * lane, m[r]);
      store4((float*)A.v + s0 + r * kMomentBlock + 4 * lane, v[r]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int e = r * kMomentBlock + element<false>(lane, j);
        if (e >= left) continue;
        ((float*)A.m)[s0 + e] = m[r][j];
        ((float*)A.v)[s0 + e] = v[r][j];
      }
    }
  }
}

// A wavefront takes kRun consecutive blocks.  fp32 moments: 28 bytes an element (c = 1), e4m3: 16 and 16 a block.
template <typename G, bool E4M3>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwLaunch A) {
  const int lane = threadIdx.x & 63;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const uint32_t total = A.tab.first[A.tab.n];
  uint32_t b = wave * kRun;
  if (b >= total) return;
  const uint32_t b1 = min(b + kRun, total);
  AdamwStep S;
  S.pace = A.pace;
  S.vcorr = A.vcorr;
  int64_t step = A.step;
  if (A.step_dev) {
    step = *A.step_dev;
    S.pace = (float)(A.rate / -expm1((double)step * A.log_beta1));
    S.vcorr = (float)(1.0 / -expm1((double)step * A.log_beta2));
  }
  S.key = mix32(A.seed + (uint32_t)step * 0x9E3779B1u);
  S.scaled = A.factor != nullptr;
  S.factor = S.scaled ? *A.factor : 1.f;
  S.skip = S.scaled && S.factor != S.factor;
  const float* share = (const float*)A.tab.word;
  while (b < b1) {
    const int k = tensor_of(A.tab, b);
    const uint64_t* w = A.tab.word + A.words_at + k * A.tab.stride;
    const int64_t numel = (int64_t)(w[0] & ~kAligned), at = (int64_t)(b - A.tab.first[k]) * kMomentBlock;
    const int64_t left = numel - at, block = A.block0 + b;
    if ((w[0] & kAligned) && left >= kRun * kMomentBlock && b1 - b == kRun) {
      adamw_blocks<G, E4M3, true, kRun>(A, S, w, share, at, left, block, lane);
      b += kRun;
    } else if ((w[0] & kAligned) && left >= kMomentBlock) {
      adamw_blocks<G, E4M3, true, 1>(A, S, w, share, at, left, block, lane);
      b += 1;
    } else {
      adamw_blocks<G, E4M3, false, 1>(A, S, w, share, at, left, block, lane);
      b += 1;
    }
  }
}

// ------------------------------------------------------------------------------------------------ norm
// Squares and their sums in 64 bits: no overflow or underflow whatever the gradients' size, and no error in the last place of
// the norm.  Every workgroup writes one partial sum, one workgroup adds them: the order is fixed.
template <typename G>
__device__ __forceinline__ double block_squares(const uint64_t* w, int64_t at, int64_t left, bool vec, int lane) {
  const G* g = (const G*)w[1] + at;
  double s = 0;
  if (vec && left >= kMomentBlock) {
    float x[4];
    load4(x, g + 4 * lane);
#pragma unroll
    for (int j = 0; j < 4; j++) s = fma((double)x[j], (double)x[j], s);
  } else {
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const int e = lane + 64 * j;
      const double x = e < left ? (double)ldf(g + e) : 0.0;
      s = fma(x, x, s);
    }
  }
  return s;
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <typename G>
__global__ __launch_bounds__(256) void norm_partials_kernel(const NormLaunch A) {
  __shared__ double sums[4];
  const int lane = threadIdx.x & 63;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const uint32_t total = A.tab.first[A.tab.n], waves = gridDim.x * 4;
  double s = 0;
  for (uint32_t b = wave; b < total; b += waves) {
    const int k = tensor_of(A.tab, b);
    const uint64_t* w = A.tab.word + k * A.tab.stride;
    const int64_t at = (int64_t)(b - A.tab.first[k]) * kMomentBlock;
    s += block_squares<G>(w, at, (int64_t)(w[0] & ~kAligned) - at, (w[0] & kAligned) != 0, lane);
  }
  s = wave_sum_f64(s);
  if (lane == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    A.partial[blockIdx.x] = A.add ? A.partial[blockIdx.x] + s : s;
  }
}

__global__ __launch_bounds__(256) void norm_finish_kernel(const double* partial, int n, float max_norm, float* out) {
  __shared__ double sums[4];
  double s = 0;
  for (int k = threadIdx.x; k < n; k += 256) s += partial[k];
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    const double norm = sqrt((sums[0] + sums[1]) + (sums[2] + sums[3]));
    out[0] = (float)norm;
    out[1] = !(norm < INFINITY) ? NAN : max_norm > 0.f && norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
  }
}

}  // namespace

hipError_t launch_adamw(const AdamwLaunch& a, bool grad_bf16, bool e4m3, hipStream_t stream) {
  const uint32_t blocks = a.tab.first[a.tab.n], waves = (blocks + kRun - 1) / kRun;
  const dim3 grid((waves + 3) / 4);
  if (grad_bf16) {
    if (e4m3) adamw_kernel<bf16_t, true><<<grid, 256, 0, stream>>>(a);
    else adamw_kernel<bf16_t, false><<<grid, 256, 0, stream>>>(a);
  } else {
    if (e4m3) adamw_kernel<float, true><<<grid, 256, 0, stream>>>(a);
    else adamw_kernel<float, false><<<grid, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

int norm_grid(int64_t blocks) { return (int)(blocks / 16 < 1 ? 1 : blocks / 16 > kNormPartials ? kNormPartials : blocks / 16); }

hipError_t launch_norm_partials(const NormLaunch& a, bool bf16, hipStream_t stream) {
  if (bf16) norm_partials_kernel<bf16_t><<<a.grid, 256, 0, stream>>>(a);
  else norm_partials_kernel<float><<<a.grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}
hipError_t launch_norm_finish(const NormLaunch& a, hipStream_t stream) {
  norm_finish_kernel<<<1, 256, 0, stream>>>(a.partial, a.grid, a.max_norm, a.out);
  return hipGetLastError();
}

}  // namespace sasgd
