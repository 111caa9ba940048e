// Launcher interface of the output layer's losses (linear_loss.cu) and of the top logits (top_logits.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "scalify.h"

namespace scalify {

constexpr int64_t kLossMaxRows = int64_t(1) << 24;
constexpr int64_t kLossMaxVocab = int64_t(1) << 24;
constexpr int64_t kLossMaxDim = int64_t(1) << 16;
constexpr int kLossMaxEntries = 256;  // of a teacher's row

// One call, checked.  Arrays as they came; strides in elements.
struct LinearLossArgs {
  const void* H; const void* W;
  int h_dt, w_dt;
  long long h_ld, w_ld;
  const float* h_scale; const float* w_scale;
  long long n, vocab;
  int d;
  // targets: one id per row (cross entropy, k == 0) or k entries per row (distillation)
  const long long* ids;
  long long padding_id;
  int k;
  const void* T; int t_dt; long long t_ld; const float* t_scale; const float* t_lse;
  float inv_temp, inv_temp_p2, inv_temp_rest;  // 1/temperature, and its power of two times a rest in [1, 2)
  float z_loss;
  // forward
  float* loss; float* lse; float* mean;
  // backward (lse is an input)
  const float* grad; const float* grad_scale;
  void* dH; void* dW;
  int dh_dt, dw_dt;
  long long dh_ld, dw_ld;
  float* dh_scale; float* dw_scale;
};
// What a call on n rows needs, and the most that a call on at most n rows does.
size_t linear_loss_ws_need(long long n, long long vocab, long long d, int operand_bytes, int k, bool backward);
size_t linear_loss_ws_bytes(long long n, long long vocab, long long d, int operand_bytes, int k, bool backward);
int launch_linear_loss(const LinearLossArgs& a, void* ws, cudaStream_t st);
int launch_linear_loss_bwd(const LinearLossArgs& a, void* ws, cudaStream_t st);

struct TopLogitsArgs {
  const void* X; int dt; long long ld;
  const float* x_scale;
  long long n, vocab;
  int k;
  void* V; long long v_ld;
  float* v_scale;
  long long* ids;
  float* lse;
  float inv_temp;
};
int launch_top_logits(const TopLogitsArgs& a, cudaStream_t st);

}  // namespace scalify
