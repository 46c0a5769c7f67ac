// C entry points of the context-free operators: argument checks and the tables their kernels read.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>

#include "../../include/sasgd.h"
#include "operators.hpp"

using namespace sasgd;

namespace {

int refuse(char* err, size_t err_len, int code, const char* fmt, ...) {
  if (err && err_len > 0) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(err, err_len, fmt, ap);
    va_end(ap);
  }
  return code;
}
#define REFUSE(...) return refuse(err, err_len, SASGD_EINVAL, __VA_ARGS__)
#define TRY_HIP(x, name)                                                                                     \
  do {                                                                                                       \
    const hipError_t e__ = (x);                                                                              \
    if (e__ != hipSuccess) return refuse(err, err_len, SASGD_EHIP, name ": %s", hipGetErrorString(e__));     \
  } while (0)

inline int64_t blocks_of(int64_t numel) { return (numel + kMomentBlock - 1) / kMomentBlock; }
constexpr int64_t kMostElements = (int64_t)1 << 34;     // of a tensor and of a call: its launch stays below 2^32 lanes

// ---------------------------------------------------------------- group normalisation
const char* shape_error(const sasgd_norm_shape* s) {
  if (!s) return "null shape";
  if (s->images < 0 || s->positions < 1 || s->positions > kNormPositions) return "images or positions out of range";
  if (s->images > ((int64_t)1 << 31)) return "too many images";
  if (s->channels < 1 || s->channels > kWideNormChannels || s->groups < 1 || s->channels % s->groups != 0) return "channels must be 1..4096 and a multiple of groups";
  if ((s->type != SASGD_FP32 && s->type != SASGD_BF16) || (s->param_type != SASGD_FP32 && s->param_type != SASGD_BF16)) return "unknown type";
  if (s->activation < SASGD_ACT_NONE || s->activation > SASGD_ACT_SILU) return "unknown activation";
  if (!(s->eps > 0.f && s->eps < INFINITY)) return "eps must be positive and finite";
  if (s->x_image < 0 || s->x_pixel < 0 || s->y_image < 0 || s->y_pixel < 0) return "negative stride";
  if ((s->x_pixel && s->x_pixel < s->channels) || (s->y_pixel && s->y_pixel < s->channels)) return "pixels overlap";
  return nullptr;
}

GroupNormShape inner_shape(const sasgd_norm_shape& s) { return GroupNormShape{s.images, (int)s.positions, s.channels, s.groups, s.type == SASGD_BF16}; }

// Checks what both directions have in common and fills the launch's arguments; nullptr if all is well.
const char* group_norm_args(const sasgd_norm_shape* shape, const void* x, const void* y, const void* dx, const void* scale, const void* shift,
                            void* work, size_t work_bytes, bool gradient, GroupNormArgs& a) {
  const char* e = shape_error(shape);
  if (e) return e;
  memset(&a, 0, sizeof(a));
  a.s = inner_shape(*shape);
  a.learners = 1;
  a.activation = shape->activation;
  a.eps = shape->eps;
  const int size = a.s.bf16 ? 2 : 4;
  a.x_pixel = shape->x_pixel ? shape->x_pixel : shape->channels;
  a.y_pixel = shape->y_pixel ? shape->y_pixel : shape->channels;
  a.x_image = shape->x_image ? shape->x_image : a.x_pixel * shape->positions;
  a.y_image = shape->y_image ? shape->y_image : a.y_pixel * shape->positions;
  if (a.x_pixel > ((int64_t)1 << 32) || a.y_pixel > ((int64_t)1 << 32) || a.x_image > ((int64_t)1 << 40) || a.y_image > ((int64_t)1 << 40)) return "stride out of range";
  const int64_t reach = (int64_t)1 << 48;      // (of elements: more than there are addresses)
  if (shape->images > 1 && (a.x_image > reach / (shape->images - 1) || a.y_image > reach / (shape->images - 1))) return "stride out of range";
  // images one behind the other, or (positions first) side by side in every position
  if (shape->images > 1 && a.y_image < (shape->positions - 1) * a.y_pixel + shape->channels &&
      (a.y_image < shape->channels || (shape->positions > 1 && a.y_pixel < (shape->images - 1) * a.y_image + shape->channels)))
    return "images that are written overlap";
  if (shape->images > 0 && (!x || !y)) return "null tensor";
  if (!gradient && shape->images > 0 && x == y && (a.x_pixel != a.y_pixel || a.x_image != a.y_image)) return "in place x and y need the same strides";
  const uintptr_t low = (uintptr_t)x | (uintptr_t)y | (uintptr_t)dx;
  if (low & (size - 1)) return "tensors must be aligned to their elements";
  const int psize = shape->param_type == SASGD_BF16 ? 2 : 4;
  if (((uintptr_t)scale | (uintptr_t)shift) & (psize - 1)) return "scale and shift must be aligned to their elements";
  const int vec = 16 / size;
  const bool wide = (low & 15) == 0 && (a.s.channels | a.x_pixel | a.y_pixel | a.x_image | a.y_image) % vec == 0;
  if (!wide && a.s.channels > kNarrowNormChannels) return "more than 1024 channels must be whole 16 bytes, in strides and pointers too";
  a.plan = group_norm_plan(a.s, wide, gradient, a.activation == SASGD_ACT_SILU, 1);
  const size_t need = group_norm_scratch_bytes(a.s, a.plan, gradient);
  if (need > 0 && (!work || ((uintptr_t)work & 15) || work_bytes < need)) return "workspace missing, too small or not 16-byte aligned";
  a.x = (int64_t)(uintptr_t)x;
  (gradient ? a.dy : a.y) = (int64_t)(uintptr_t)y;
  a.dx = (int64_t)(uintptr_t)dx;
  a.parts = (int64_t)(uintptr_t)work;
  a.sums = a.parts + (int64_t)group_norm_sums_at(a.s, a.plan);
  a.scale = (int64_t)(uintptr_t)scale;
  a.shift = (int64_t)(uintptr_t)shift;
  a.has_scale = scale != nullptr;
  a.has_shift = shift != nullptr;
  a.param_bf16 = shape->param_type == SASGD_BF16;
  return nullptr;
}

}  // namespace

extern "C" {

int sasgd_groupNormWorkspace(const sasgd_norm_shape* shape, int32_t gradient, size_t* out_bytes) {
  if (!out_bytes || shape_error(shape)) return SASGD_EINVAL;
  const GroupNormShape s = inner_shape(*shape);
  size_t most = 0;
  for (int wide = 0; wide < 2; wide++) {
    if (wide && s.channels % (s.bf16 ? 8 : 4) != 0) continue;
    if (!wide && s.channels > kNarrowNormChannels) continue;
    for (int silu = 0; silu < 2; silu++)
      most = std::max(most, group_norm_scratch_bytes(s, group_norm_plan(s, wide != 0, gradient != 0, silu != 0, 1), gradient != 0));
  }
  *out_bytes = most;
  return SASGD_OK;
}

int sasgd_groupNorm(const sasgd_norm_shape* shape, const void* x_dev, const void* scale_dev, const void* shift_dev, void* y_dev, float* stats_dev,
                    void* workspace_dev, size_t workspace_bytes, void* stream, char* err, size_t err_len) {
  GroupNormArgs a;
  const char* e = group_norm_args(shape, x_dev, y_dev, nullptr, scale_dev, shift_dev, workspace_dev, workspace_bytes, false, a);
  if (e) REFUSE("groupNorm: %s", e);
  if ((uintptr_t)stats_dev & 7) REFUSE("groupNorm: stats_dev must be 8-byte aligned");
  a.stats = (int64_t)(uintptr_t)stats_dev;
  a.has_stats = stats_dev != nullptr;
  TRY_HIP(launch_group_norm(a, (hipStream_t)stream), "groupNorm");
  return SASGD_OK;
}

int sasgd_groupNormGradient(const sasgd_norm_shape* shape, const void* x_dev, const void* scale_dev, const void* shift_dev, const float* stats_dev,
                            const void* dy_dev, void* dx_dev, float* dscale_dev, float* dshift_dev, void* workspace_dev, size_t workspace_bytes,
                            void* stream, char* err, size_t err_len) {
  GroupNormArgs a;
  const char* e = group_norm_args(shape, x_dev, dy_dev, dx_dev, scale_dev, shift_dev, workspace_dev, workspace_bytes, true, a);
  if (e) REFUSE("groupNormGradient: %s", e);
  if ((shape->images > 0 && !stats_dev) || ((uintptr_t)stats_dev & 7)) REFUSE("groupNormGradient: stats_dev must be an 8-byte aligned device pointer");
  if (((uintptr_t)dscale_dev | (uintptr_t)dshift_dev) & 3) REFUSE("groupNormGradient: dscale_dev and dshift_dev must be 4-byte aligned");
  a.stats = (int64_t)(uintptr_t)stats_dev;
  a.has_dx = dx_dev != nullptr;
  a.dscale = (int64_t)(uintptr_t)dscale_dev;
  a.dshift = (int64_t)(uintptr_t)dshift_dev;
  a.has_dscale = dscale_dev != nullptr;
  a.has_dshift = dshift_dev != nullptr;
  TRY_HIP(launch_group_norm_gradient(a, (hipStream_t)stream), "groupNormGradient");
  return SASGD_OK;
}

int sasgd_momentElements(const int64_t* numel, int32_t count, int64_t* out_elements) {
  if (!out_elements || count < 0 || (count > 0 && !numel)) return SASGD_EINVAL;
  int64_t blocks = 0;
  for (int32_t k = 0; k < count; k++) {
    if (numel[k] < 0 || numel[k] > kMostElements) return SASGD_EINVAL;
    blocks += blocks_of(numel[k]);
  }
  *out_elements = blocks * kMomentBlock;
  return SASGD_OK;
}

int sasgd_gradientNorm(const void* const* grads_dev, const int64_t* numel, int32_t count, int32_t type, float max_norm,
                       float* out_dev, void* workspace_dev, void* stream, char* err, size_t err_len) {
  if (count < 0 || (count > 0 && (!grads_dev || !numel))) REFUSE("gradientNorm: null array or negative count");
  if (type != SASGD_FP32 && type != SASGD_BF16) REFUSE("gradientNorm: unknown type");
  if (!(max_norm >= 0.f)) REFUSE("gradientNorm: max_norm must not be negative");
  if (!out_dev || ((uintptr_t)out_dev & 3)) REFUSE("gradientNorm: out_dev must be a 4-byte aligned device pointer");
  if (!workspace_dev || ((uintptr_t)workspace_dev & 7)) REFUSE("gradientNorm: workspace_dev must be an 8-byte aligned device pointer");
  const bool bf = type == SASGD_BF16;
  int64_t blocks = 0;
  for (int32_t k = 0; k < count; k++) {
    if (numel[k] < 0 || numel[k] > kMostElements) REFUSE("gradientNorm: length of tensor %d out of range", (int)k);
    if (numel[k] > 0 && (!grads_dev[k] || ((uintptr_t)grads_dev[k] & (bf ? 1 : 3)))) REFUSE("gradientNorm: tensor %d is null or not aligned to its elements", (int)k);
    blocks += blocks_of(numel[k]);
  }
  if (blocks * kMomentBlock > kMostElements) REFUSE("gradientNorm: more than 2^34 elements");
  static_assert(kNormPartials * sizeof(double) <= SASGD_NORM_WORKSPACE, "partial sums do not fit the workspace");
  NormLaunch a;
  memset(&a, 0, sizeof(a));
  a.partial = (double*)workspace_dev;
  a.out = out_dev;
  a.max_norm = max_norm;
  a.grid = norm_grid(blocks);
  TensorTable& tab = a.tab;
  tab.stride = 2;
  int32_t k = 0;
  do {
    tab.n = 0;
    for (; k < count && tab.n < kTableTensors; k++) {
      if (numel[k] == 0) continue;
      uint64_t* w = tab.word + tab.n * 2;
      const bool aligned = ((uintptr_t)grads_dev[k] & (bf ? 7 : 15)) == 0;
      w[0] = (uint64_t)numel[k] | (aligned ? kAligned : 0);
      w[1] = (uint64_t)(uintptr_t)grads_dev[k];
      tab.first[tab.n + 1] = tab.first[tab.n] + (uint32_t)blocks_of(numel[k]);
      tab.n++;
    }
    a.last = k == count;
    TRY_HIP(launch_norm(a, bf, (hipStream_t)stream), "gradientNorm");
    a.add = 1;
  } while (k < count);
  return SASGD_OK;
}

int sasgd_applyAdamW(const sasgd_adamw* rule, const sasgd_tensor* tensors, int32_t count, const void* const* grads_dev, int32_t c,
                     const int32_t* staleness, const sasgd_moments* moments, int64_t step, const int64_t* step_dev,
                     const float* factor_dev, void* stream, char* err, size_t err_len) {
  if (!rule || !moments || !staleness || count < 0 || (count > 0 && (!tensors || !grads_dev))) REFUSE("applyAdamW: null argument or negative count");
  if (rule->lr_mode < SASGD_LR_PER_GRADIENT || rule->lr_mode > SASGD_LR_CONSTANT) REFUSE("applyAdamW: unknown lr_mode");
  if (rule->moments != SASGD_MOMENTS_FP32 && rule->moments != SASGD_MOMENTS_E4M3) REFUSE("applyAdamW: unknown type of moments");
  if (rule->grad_type != SASGD_FP32 && rule->grad_type != SASGD_BF16) REFUSE("applyAdamW: unknown type of gradients");
  if (!(rule->alpha0 >= 0 && rule->alpha0 < INFINITY && rule->weight_decay >= 0 && rule->weight_decay < INFINITY))
    REFUSE("applyAdamW: alpha0 and weight_decay must be finite and not negative");
  if (!(rule->beta1 >= 0 && rule->beta1 < 1 && rule->beta2 >= 0 && rule->beta2 < 1)) REFUSE("applyAdamW: beta1 and beta2 must lie in [0, 1)");
  if (!(rule->epsilon >= 1e-30 && rule->epsilon < 1e30)) REFUSE("applyAdamW: epsilon must lie in [1e-30, 1e30)");
  if (c < 1 || c > SASGD_NOALLOC_MAX_GRADIENTS) REFUSE("applyAdamW: c must lie in 1..64");
  if (step < 1 && !step_dev) REFUSE("applyAdamW: steps count from 1");
  if (((uintptr_t)step_dev & 7) || ((uintptr_t)factor_dev & 3)) REFUSE("applyAdamW: step_dev and factor_dev must be aligned to their elements");
  const bool bf = rule->grad_type == SASGD_BF16, e4m3 = rule->moments == SASGD_MOMENTS_E4M3;
  double sum_tau = 0, sum_a = 0, a_of[SASGD_NOALLOC_MAX_GRADIENTS];
  for (int l = 0; l < c; l++) {
    if (staleness[l] < 0) REFUSE("applyAdamW: negative staleness");
    sum_tau += staleness[l];
  }
  for (int l = 0; l < c; l++) {
    a_of[l] = rule->lr_mode == SASGD_LR_PER_GRADIENT ? 1.0 / std::max(staleness[l], 1)
              : rule->lr_mode == SASGD_LR_MEAN_STALENESS ? 1.0 / std::max(sum_tau / c, 1.0) : 1.0;
    sum_a += a_of[l];
  }
  bool has_out = false, has_shadow = false;
  int64_t blocks = 0;
  for (int32_t k = 0; k < count; k++) {
    const sasgd_tensor& t = tensors[k];
    if (t.numel < 0 || t.numel > kMostElements) REFUSE("applyAdamW: length of tensor %d out of range", (int)k);
    if (t.numel == 0) continue;
    if (!t.theta_in || !t.theta_out || (((uintptr_t)t.theta_in | (uintptr_t)t.theta_out) & 3) || ((uintptr_t)t.shadow_out & 1))
      REFUSE("applyAdamW: weights of tensor %d are null or not aligned to their elements", (int)k);
    for (int l = 0; l < c; l++) {
      const void* g = grads_dev[(size_t)k * c + l];
      if (!g || ((uintptr_t)g & (bf ? 1 : 3))) REFUSE("applyAdamW: gradient %d of tensor %d is null or not aligned to its elements", l, (int)k);
    }
    has_out = has_out || t.theta_out != t.theta_in;
    has_shadow = has_shadow || t.shadow_out;
    blocks += blocks_of(t.numel);
  }
  if (blocks * kMomentBlock > kMostElements) REFUSE("applyAdamW: more than 2^34 elements");
  if (blocks == 0) return SASGD_OK;
  if (!moments->m || !moments->v || (((uintptr_t)moments->m | (uintptr_t)moments->v) & 15)) REFUSE("applyAdamW: moments must be 16-byte aligned device pointers");
  if (e4m3 && (!moments->m_scale || !moments->v_scale || (((uintptr_t)moments->m_scale | (uintptr_t)moments->v_scale) & 3)))
    REFUSE("applyAdamW: e4m3 moments need 4-byte aligned scales");
  AdamwLaunch a;
  memset(&a, 0, sizeof(a));
  a.c = c;
  a.has_out = has_out;
  a.has_shadow = has_shadow;
  a.grads_at = 2 + a.has_out + a.has_shadow;
  a.words_at = (c + 1) / 2;
  // Gradients that are flat vectors cut the same way (a learner's, in flat parameter order): their distances do for all tensors, and a launch
  // takes as many as with one gradient (350 tensors, 18 gradients: 4 launches instead of 19)
  int32_t lead = -1;
  bool flat = c > 1;
  for (int32_t k = 0; flat && k < count; k++) {
    if (tensors[k].numel == 0) continue;
    if (lead < 0) lead = k;
    for (int l = 1; flat && l < c; l++)
      flat = (uintptr_t)grads_dev[(size_t)k * c + l] - (uintptr_t)grads_dev[(size_t)k * c] == (uintptr_t)grads_dev[(size_t)lead * c + l] - (uintptr_t)grads_dev[(size_t)lead * c];
  }
  a.seed = rule->seed;
  a.m = moments->m;
  a.v = moments->v;
  a.m_scale = moments->m_scale;
  a.v_scale = moments->v_scale;
  a.factor = factor_dev;
  a.step_dev = step_dev;
  a.step = step;
  a.rate = rule->alpha0 * (sum_a / c);
  a.log_beta1 = log(rule->beta1);          // -inf for 0: 1 - beta^t is 1
  a.log_beta2 = log(rule->beta2);
  if (!step_dev) {
    a.pace = (float)(a.rate / -expm1((double)step * a.log_beta1));
    a.root = (float)sqrt(1.0 / -expm1((double)step * a.log_beta2));
  }
  a.beta1 = (float)rule->beta1;
  a.rest1 = (float)(1.0 - rule->beta1);
  a.beta2 = (float)rule->beta2;
  a.rest2 = (float)(1.0 - rule->beta2);
  a.epsilon = (float)rule->epsilon;
  a.keep = (float)(1.0 - a.rate * rule->weight_decay);
  TensorTable& tab = a.tab;
  for (int l = 0; l < c; l++) {
    const float share = (float)(a_of[l] / sum_a);
    memcpy((char*)tab.word + 4 * l, &share, 4);
  }
  if (flat) {
    a.apart_at = a.words_at;
    a.words_at += c;
    for (int l = 0; l < c; l++) tab.word[a.apart_at + l] = (uint64_t)((uintptr_t)grads_dev[(size_t)lead * c + l] - (uintptr_t)grads_dev[(size_t)lead * c]);
  }
  const int listed = flat ? 1 : c;
  tab.stride = a.grads_at + listed;
  const int most = std::min(kTableTensors, (kTableWords - a.words_at) / tab.stride);
  for (int32_t k = 0; k < count;) {
    tab.n = 0;
    for (; k < count && tab.n < most; k++) {
      const sasgd_tensor& t = tensors[k];
      if (t.numel == 0) continue;
      uint64_t* w = tab.word + a.words_at + tab.n * tab.stride;
      uintptr_t low = (uintptr_t)t.theta_in | (uintptr_t)t.theta_out | ((uintptr_t)t.shadow_out << 1);
      w[1] = (uint64_t)(uintptr_t)t.theta_in;
      if (has_out) w[2] = (uint64_t)(uintptr_t)t.theta_out;
      if (has_shadow) w[2 + a.has_out] = (uint64_t)(uintptr_t)t.shadow_out;
      for (int l = 0; l < c; l++) {
        const uintptr_t g = (uintptr_t)grads_dev[(size_t)k * c + l];
        low |= bf ? g << 1 : g;
        if (l < listed) w[a.grads_at + l] = (uint64_t)g;
      }
      w[0] = (uint64_t)t.numel | ((low & 15) == 0 ? kAligned : 0);
      tab.first[tab.n + 1] = tab.first[tab.n] + (uint32_t)blocks_of(t.numel);
      tab.n++;
    }
    if (tab.n == 0) break;
    TRY_HIP(launch_adamw(a, bf, e4m3, (hipStream_t)stream), "applyAdamW");
    a.block0 += tab.first[tab.n];
  }
  return SASGD_OK;
}

}  // extern "C"
