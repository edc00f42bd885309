// Launchers of window_attention*.hip: the arguments as daf_attention.h has them, checked.
#pragma once
#include <hip/hip_runtime.h>

#include "daf_attention.h"

constexpr int kAttentionMaxDim = 128, kAttentionMaxSequences = 1 << 16, kAttentionMaxSteps = 1 << 20;
constexpr int64_t kAttentionMostRows = 1 << 30;       // a window of as many is none, and a position minus it stays an int

struct AttentionTensors {
  daf_heads_t q, k, v, out;
  float* lse;
};

hipError_t daf_launch_window_attention(const daf_window_attention_t& p, const AttentionTensors& t, hipStream_t stream);

struct AttentionGradients {
  daf_heads_t grad_out, grad_q, grad_k, grad_v;
};
// Of a workspace: what a call of these sizes uses, and what is enough for all calls of these sequences and rows or fewer.
int64_t daf_window_attention_backward_workspace_size(int64_t rows, int q_heads, int kv_heads, int head_dim, int64_t sequences, int64_t window, int64_t sinks);
int64_t daf_window_attention_backward_workspace_bound(int64_t rows, int q_heads, int kv_heads, int head_dim, int64_t sequences, int64_t window, int64_t sinks);
hipError_t daf_launch_window_attention_backward(const daf_window_attention_t& p, const AttentionTensors& t, const AttentionGradients& g, char* workspace,
                                                hipStream_t stream);

int64_t daf_window_attention_step_workspace_size(int64_t sequences, int q_heads, int kv_heads, int head_dim, int64_t k_rows, int64_t window, int64_t sinks);
int64_t daf_window_attention_step_workspace_bound(int64_t sequences, int q_heads, int kv_heads, int head_dim, int64_t k_rows, int64_t window, int64_t sinks);
hipError_t daf_launch_window_attention_step(const daf_window_attention_t& p, const AttentionTensors& t, char* workspace, hipStream_t stream);
