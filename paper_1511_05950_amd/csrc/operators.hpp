// Launches of the context-free operators (operators.cpp checks their arguments).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastdiv.hpp"

namespace sasgd {

// ---------------------------------------------------------------- many tensors (adamw.hip)
constexpr int kMomentBlock = 256;        // consecutive elements of a tensor that share a scale
constexpr int kTableTensors = 100;       // of one launch
constexpr int kTableWords = 416;
// The tensors of one launch, passed by value (kernel arguments hold 4 KiB).  first[k]: block at which tensor k begins,
// first[n] the number of blocks; empty tensors are left out.  word: per tensor `stride` words, see TensorWords.
struct TensorTable {
  uint64_t word[kTableWords];
  uint32_t first[kTableTensors + 1];
  int32_t n, stride;
};
// A tensor's words: its length, its first pointer, then what the launch has (theta_out, shadow, further gradients).
// The length's top bit: every pointer of the tensor is aligned for vector moves.
constexpr uint64_t kAligned = (uint64_t)1 << 63;

struct AdamwLaunch {
  TensorTable tab;           // words of a tensor: numel, theta_in, [theta_out], [shadow], g_0 .. g_{c-1}; the c shares (float) come first, then distances
  int32_t c, has_out, has_shadow, grads_at;   // grads_at: a tensor's word with g_0;  tensors' words begin at words_at, behind the shares
  int32_t words_at;
  int32_t apart_at;          // not 0: every gradient lies as far from g_0 in all tensors (flat vectors), by c words from here on; tensors have g_0 alone
  uint32_t seed;
  int64_t block0;            // moments' block of the launch's first block
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  const float* factor;
  const int64_t* step_dev;
  int64_t step;
  double rate, log_beta1, log_beta2;
  float pace, root;          // rate / (1 - beta1^step), sqrt(1 / (1 - beta2^step)); computed from step_dev where there is one
  float beta1, rest1, beta2, rest2, epsilon, keep;   // rest = 1 - beta, keep = 1 - rate weight_decay
};
hipError_t launch_adamw(const AdamwLaunch& a, bool grad_bf16, bool e4m3, hipStream_t stream);

constexpr int kNormPartials = 2048;
struct NormLaunch {
  TensorTable tab;           // words of a tensor: numel, gradient
  double* partial;           // [grid]
  float* out;                // norm, factor
  float max_norm;
  int32_t add;               // partial[] holds the sums of the launches before
  int32_t last;              // no more tensors behind these: norm and factor follow
  int32_t grid;              // workgroups, the same in all launches of a call (norm_grid)
};
int norm_grid(int64_t blocks);
hipError_t launch_norm(const NormLaunch& a, bool bf16, hipStream_t stream);

// ---------------------------------------------------------------- group normalisation (group_norm.hip)
// How a call is cut into workgroups (group_norm_plan).
struct GroupNormPlan {
  int vec;         // channels a lane moves at a time: 16 bytes, or 1
  int threads;
  int held;        // vectors of x (and of dy) that a lane keeps in registers
  bool whole;      // a workgroup holds all positions of `slab` channels; otherwise it walks `chunk` positions of all channels, in two launches
  int slab, slabs;
  int chunk, chunks;
  bool once;       // the tensors go past the caches
};
struct GroupNormShape {
  int64_t images;            // of a learner
  int positions, channels, groups;
  bool bf16;
};
GroupNormPlan group_norm_plan(const GroupNormShape& s, bool wide, bool gradient, bool silu, int learners);

// How a workgroup's lanes lie over a pixel's channels: `cols` vectors side by side, `rows` pixels at a time; n = cols x vec channels.
struct GroupNormCols {
  int cols, rows, segs;      // segs: lanes over n
  int fold;                  // n is a power of two below 64
  FastDiv by_cols, by_n;     // of numbers up to 1024: exact
};

// Addresses are base[learner] + a byte offset (workspace), wts[learner] + offset (scale, shift), grads[learner] + offset (their gradients);
// context-free calls have one learner whose bases are 0.
struct GroupNormArgs {
  uintptr_t base[64], wts[64], grads[64];
  int64_t x, y, dy, dx, stats, parts, sums;                 // parts: [image][chunk][group][2], sums: [image][chunk][channel][2], both fp32
  int64_t scale, shift, dscale, dshift;
  int64_t x_image, x_pixel, y_image, y_pixel;               // elements
  GroupNormShape s;
  GroupNormPlan plan;
  int32_t learners, activation;
  int32_t has_scale, has_shift, param_bf16, has_stats, has_dx, has_dscale, has_dshift, mask;   // mask: dx is 0 where x is not positive
  float eps;
  // set by the launch
  GroupNormCols cols[2];
  int32_t cpg;               // channels of a group
  FastDiv by_cpg;            // of channel numbers, up to 4096: exact
  int32_t spread;            // lanes that add one group's chunks in the second launch, a power of two
};
// Scratch of a learner: chunks' statistics, then (from group_norm_sums_at on) the gradient's channel sums.
size_t group_norm_sums_at(const GroupNormShape& s, const GroupNormPlan& p);
size_t group_norm_scratch_bytes(const GroupNormShape& s, const GroupNormPlan& p, bool gradient);
constexpr int kWideNormChannels = 4096, kNarrowNormChannels = 1024;   // sums by channel of a workgroup lie in LDS; narrow: not moved 16 bytes at a time
constexpr int64_t kNormPositions = (int64_t)1 << 26;
hipError_t launch_group_norm(GroupNormArgs& a, hipStream_t stream);
hipError_t launch_group_norm_gradient(GroupNormArgs& a, hipStream_t stream);

}  // namespace sasgd
