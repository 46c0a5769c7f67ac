// AdamW over many tensors in one launch, and the norm over many tensors.
//
// Both walk blocks of 256 consecutive elements of a tensor, a wavefront a block (4 elements a lane), and find a block's tensor in a
// table that the kernel's arguments carry: nothing is copied to the device beforehand, and work is spread over the chip by
// blocks whatever the sizes of the tensors.  Both are bound by HBM.
#include <math.h>

#include <algorithm>

#include "dev_common.hpp"
#include "operators.hpp"

namespace sasgd {

namespace {

// Blocks that a wavefront has on their way at a time, a wavefront a workgroup: the AlexNet-shaped net's 62 M weights behind a bounded gradient 361 us
// with 2, 358 with 1, 369 with 4; with 8-bit moments and four gradients 314, 323, 321; 397 tensors of 100 M 293, 295, 316 (their launches' ends
// weigh more, the longer a wavefront).  Workgroups of four wavefronts: 368, 321, 295.
// Where the blocks would not fill the chip twice a wavefront takes one, and as many gradients of a long window at a time as registers allow (with two blocks
// and with one: 89 578 weights, 30 gradients 13.8 and 9.3 us; 500 000, one 5.8 and 4.8; from 2.3 M, four gradients, on within 2 %).
constexpr int kRun = 2;
constexpr uint32_t kFewBlocks = 8192;

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
// All streams go past the caches: none is read twice in a step, and a step of a training loop comes long after the one before.  (405 -> 361 us,
// 344 -> 314, 321 -> 293 in the cases above; where three sets of weights and moments fit the memory-side cache together, 3 to 6 M weights, up to 8 % slower.)
template <typename T, typename P>
__device__ __forceinline__ T load_once(const P* p) { return __builtin_nontemporal_load(reinterpret_cast<const T*>(p)); }
template <typename T, typename P>
__device__ __forceinline__ void store_once(P* p, T v) { __builtin_nontemporal_store(v, reinterpret_cast<T*>(p)); }
__device__ __forceinline__ void load4(float (&d)[4], const float* p) {
  const f32x4 v = load_once<f32x4>(p);
  d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
}
__device__ __forceinline__ void load4(float (&d)[4], const bf16_t* p) {
  const u32x2 v = load_once<u32x2>(p);
  d[0] = __uint_as_float(v.x << 16); d[1] = __uint_as_float(v.x & 0xffff0000u);
  d[2] = __uint_as_float(v.y << 16); d[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, const float (&d)[4]) {
  const f32x4 v = {d[0], d[1], d[2], d[3]};
  store_once<f32x4>(p, v);
}
__device__ __forceinline__ void store4(bf16_t* p, const float (&d)[4]) {
  const u32x2 v = {pack2bf(d[0], d[1]), pack2bf(d[2], d[3])};
  store_once<u32x2>(p, v);
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
// fraction and even steps of 2^-9 below 2^-6, which are those of the binade from 2^-6 on: values below are moved there and
// back (0 stays 0).
__device__ __forceinline__ float round8(float y, uint32_t chance) {
#pragma clang fp contract(off)
  const float off = y < 0x1p-6f ? 0x1p-6f : 0.f;
  const float r = __uint_as_float((__float_as_uint(y + off) + (chance << 4)) & 0xfff00000u);
  return fminf(r - off, 448.0f);
}

// The hardware's root, 1 ulp.  It takes denormal numbers for 0, which would leave an epsilon below their roots (1e-19) alone under the fraction: they are
// moved up by 2^64 and back.
__device__ __forceinline__ float root(float v) {
  const bool small = v < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v);
  return small ? r * 0x1p-32f : r;
}

// ------------------------------------------------------------------------------------------------ one block
// What a wavefront holds of a block: element e of lane `lane` is 4 lane + j (vector moves) or lane + 64 j.
template <bool VEC>
__device__ __forceinline__ int element(int lane, int j) { return VEC ? 4 * lane + j : lane + 64 * j; }

struct AdamwStep {
  float pace, root, factor;          // root = sqrt(1 / (1 - beta2^t))
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
        m8[r] = load_once<uint32_t>((const uint8_t*)A.m + s0 + r * kMomentBlock + 4 * lane);
        u8[r] = load_once<uint32_t>((const uint8_t*)A.v + s0 + r * kMomentBlock + 4 * lane);
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
    constexpr int kAhead = R == 1 ? 8 : 2;
#pragma unroll kAhead
    for (int l = 1; l < A.c; l++) {
      const G* gl = (const G*)(A.apart_at ? w[A.grads_at] + A.tab.word[A.apart_at + l] : w[A.grads_at + l]) + at;
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
      // What is kept is rounded operation by operation; the weight's move takes the hardware's root and reciprocal (1 ulp each): a
      // division and two roots by the book were 40 of the 130 instructions of an element with 8-bit moments.
      u[j] = E4M3 ? sqrtf(v[r][j]) : root(v[r][j]);
      const float move = (m[r][j] * S.pace) * __builtin_amdgcn_rcpf(u[j] * S.root + A.epsilon);
      if (!S.skip) th[r][j] = th[r][j] * A.keep - move;
      if (E4M3) {
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
      const int64_t e0 = s0 + r * kMomentBlock;        // (a block does not cross a multiple of 2^32)
      const uint32_t lo = (uint32_t)e0 * 0x9E3779B1u, hi = (uint32_t)(e0 >> 32) * 0x243F6A89u ^ S.key;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const uint32_t chance = mix32((lo + (uint32_t)element<VEC>(lane, j) * 0x9E3779B1u) ^ hi);
        const float yu = u[j] * uup;
        mq[j] = copysignf(round8(fabsf(m[r][j]) * mup, chance >> 16), m[r][j]);
        uq[j] = yu > 0.f ? fmaxf(round8(yu, chance & 0xffffu), 0x1p-9f) : 0.f;
      }
      int pm = __builtin_amdgcn_cvt_pk_fp8_f32(mq[0], mq[1], 0, false);
      pm = __builtin_amdgcn_cvt_pk_fp8_f32(mq[2], mq[3], pm, true);
      int pu = __builtin_amdgcn_cvt_pk_fp8_f32(uq[0], uq[1], 0, false);
      pu = __builtin_amdgcn_cvt_pk_fp8_f32(uq[2], uq[3], pu, true);
      if (VEC) {
        store_once<uint32_t>((uint8_t*)A.m + s0 + r * kMomentBlock + 4 * lane, (uint32_t)pm);
        store_once<uint32_t>((uint8_t*)A.v + s0 + r * kMomentBlock + 4 * lane, (uint32_t)pu);
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

// A wavefront takes R consecutive blocks.  fp32 moments: 28 bytes an element (c = 1), e4m3: 16 and 16 a block.
template <typename G, bool E4M3, int R>
__global__ __launch_bounds__(64) void adamw_kernel(const AdamwLaunch A) {
  const int lane = threadIdx.x;
  const uint32_t wave = blockIdx.x;
  const uint32_t total = A.tab.first[A.tab.n];
  uint32_t b = wave * R;
  if (b >= total) return;
  const uint32_t b1 = min(b + R, total);
  AdamwStep S;
  S.pace = A.pace;
  S.root = A.root;
  int64_t step = A.step;
  if (A.step_dev) {
    step = *A.step_dev;
    S.pace = (float)(A.rate / -expm1((double)step * A.log_beta1));
    S.root = (float)sqrt(1.0 / -expm1((double)step * A.log_beta2));
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
    if (R > 1 && (w[0] & kAligned) && left >= R * kMomentBlock && b1 - b == R) {
      adamw_blocks<G, E4M3, true, R>(A, S, w, share, at, left, block, lane);
      b += R;
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
// 100 M fp32 values 64 us (6.2 TB/s), 40 M 29 us; runs of 1, 2 and 8 blocks: within 3 %.  Up to kLoneBlocks one workgroup of sixteen wavefronts takes
// all and there is no second launch: 30 000 values 5.3 us against 6.7, 90 000 6.6 against 6.7 (and one launch less to make), 130 000 8.2 against 6.6.
constexpr int kNormRun = 4;
constexpr int64_t kLoneBlocks = 384;

// Squares of R blocks of a tensor, `left` elements of it from the first one on.
template <typename G, bool VEC, int R>
__device__ __forceinline__ double block_squares(const G* g, int64_t left, int lane) {
  float x[R][4];
#pragma unroll
  for (int r = 0; r < R; r++) {
    if (VEC) {
      load4(x[r], g + r * kMomentBlock + 4 * lane);
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int e = lane + 64 * j;
        x[r][j] = e < left ? ldf(g + e) : 0.f;
      }
    }
  }
  double s = 0;
#pragma unroll
  for (int r = 0; r < R; r++)
#pragma unroll
    for (int j = 0; j < 4; j++) s = fma((double)x[r][j], (double)x[r][j], s);
  return s;
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The sum over a workgroup of whole wavefronts, in lane 0.
__device__ __forceinline__ double workgroup_sum(double s) {
  __shared__ double sums[16];
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int k = 1; k < (int)blockDim.x >> 6; k++) s += sums[k];
  return s;
}

__device__ __forceinline__ void write_norm(double squares, float max_norm, float* out) {
  const double norm = sqrt(squares);
  out[0] = (float)norm;
  out[1] = !(norm < INFINITY) ? NAN : max_norm > 0.f && norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}

template <typename G>
__global__ __launch_bounds__(1024) void norm_kernel(const NormLaunch A) {
  const int lane = threadIdx.x & 63;
  const uint32_t per = blockDim.x >> 6, waves = gridDim.x * per;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * per + (threadIdx.x >> 6)));
  const uint32_t total = A.tab.first[A.tab.n];
  double s = 0;
  for (uint32_t b0 = wave * kNormRun; b0 < total; b0 += waves * kNormRun) {
    const uint32_t b1 = min(b0 + kNormRun, total);
    for (uint32_t b = b0; b < b1;) {
      const int k = tensor_of(A.tab, b);
      const uint64_t* w = A.tab.word + k * A.tab.stride;
      const int64_t at = (int64_t)(b - A.tab.first[k]) * kMomentBlock, left = (int64_t)(w[0] & ~kAligned) - at;
      const G* g = (const G*)w[1] + at;
      if ((w[0] & kAligned) && left >= kNormRun * kMomentBlock && b1 - b == kNormRun) {
        s += block_squares<G, true, kNormRun>(g, left, lane);
        b += kNormRun;
      } else {
        s += (w[0] & kAligned) && left >= kMomentBlock ? block_squares<G, true, 1>(g, left, lane) : block_squares<G, false, 1>(g, left, lane);
        b += 1;
      }
    }
  }
  s = workgroup_sum(s);
  if (threadIdx.x != 0) return;
  if (A.add) s += A.partial[blockIdx.x];
  if (gridDim.x == 1 && A.last) write_norm(s, A.max_norm, A.out);
  else A.partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void norm_finish_kernel(const double* partial, int n, float max_norm, float* out) {
  double s = 0;
  for (int k = threadIdx.x; k < n; k += 256) s += partial[k];
  s = workgroup_sum(s);
  if (threadIdx.x == 0) write_norm(s, max_norm, out);
}

}  // namespace

template <typename G, bool E4M3>
static void start_adamw(const AdamwLaunch& a, hipStream_t stream) {
  const uint32_t blocks = a.tab.first[a.tab.n];
  const int run = blocks < kFewBlocks ? 1 : kRun;
  const uint32_t waves = (blocks + run - 1) / run;
  if (run == 1) adamw_kernel<G, E4M3, 1><<<waves, 64, 0, stream>>>(a);
  else adamw_kernel<G, E4M3, kRun><<<waves, 64, 0, stream>>>(a);
}

hipError_t launch_adamw(const AdamwLaunch& a, bool grad_bf16, bool e4m3, hipStream_t stream) {
  if (grad_bf16) e4m3 ? start_adamw<bf16_t, true>(a, stream) : start_adamw<bf16_t, false>(a, stream);
  else e4m3 ? start_adamw<float, true>(a, stream) : start_adamw<float, false>(a, stream);
  return hipGetLastError();
}

// Few blocks: one workgroup of sixteen wavefronts, and no second launch.
int norm_grid(int64_t blocks) {
  if (blocks <= kLoneBlocks) return 1;
  return (int)std::min<int64_t>((blocks + 4 * kNormRun - 1) / (4 * kNormRun), kNormPartials);
}

hipError_t launch_norm(const NormLaunch& a, bool bf16, hipStream_t stream) {
  const int threads = a.grid == 1 ? 1024 : 256;
  if (bf16) norm_kernel<bf16_t><<<a.grid, threads, 0, stream>>>(a);
  else norm_kernel<float><<<a.grid, threads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.last || a.grid == 1) return e;
  norm_finish_kernel<<<1, 256, 0, stream>>>(a.partial, a.grid, a.max_norm, a.out);
  return hipGetLastError();
}

}  // namespace sasgd
