// What the checks (amp_ops.cpp) and the kernels of the operators on whole arrays (amp_norm.hip, amp_scan.hip,
// amp_distill.hip, amp_delta.hip, amp_policy.hip, amp_clip.hip) agree on: arguments and launchers.  Sizes have been checked when a launcher is called.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

struct NormArgs {
  size_t rows, cols;
  const void *x, *dy;
  size_t x_stride, dy_stride;
  const float *weight, *bias;
  float eps;
  void *y, *dx;
  size_t y_stride, dx_stride;
  float *mean, *rstd, *dweight, *dbias;
  float* workspace;
};

struct ScanArgs {
  size_t rows, hidden;
  const void *gate, *cand, *dh;
  size_t gate_stride, cand_stride, dh_stride;
  size_t n_seq;
  const void *begin, *end;
  int index_bytes, zero_others;
  const float *h0, *dlast, *carry_in;
  void *h, *dgate, *dcand;
  size_t h_stride, dgate_stride, dcand_stride;
  float *last, *carry, *dh0;
  void* workspace;
};

struct ScanStepArgs {
  size_t rows, hidden;
  const void *gate, *cand;
  size_t gate_stride, cand_stride;
  float* state;
  size_t state_stride;
  void* h;
  size_t h_stride;
};

struct DistillArgs {
  size_t rows, classes, row0;   // row0: a launch's first row
  const void* logits;
  size_t logits_stride;
  int top, teacher_dtype, index_bytes;
  const void *teacher, *index;
  size_t teacher_stride, index_stride;
  float temperature;
  const float* weight;
  float* loss;
  void* dlogits;
  size_t dlogits_stride;
  void* workspace;
};

#define OPS_MAX_TOP 1024

#define DELTA_CHUNK 32   // rows whose errors are solved for together
#define DELTA_BLOCK 64   // rows between two states that the backward pass starts from
#define DELTA_SEGMENT 8  // blocks of the shortest segments that a long sequence is cut into
#define DELTA_ORDER 256  // sequences that are put in order, the longest first
#define DELTA_MAX_KEY 128

struct DeltaZero {   // an output whose rows of no sequence become zeros: bytes between rows, 16-bit halves of a row
  void* p;
  size_t stride, halves;
};

struct DeltaArgs {
  size_t rows, n_seq;
  int heads, key_heads, dk, dv;
  const void *q, *k, *v, *dout;
  size_t q_stride, k_stride, v_stride, dout_stride;
  const float *decay, *beta;
  size_t decay_stride, beta_stride;
  float scale;
  int index_bytes, zero_others;
  const void *begin, *end;
  const float *h0, *dlast, *carry_in;
  void *o, *dq, *dkey, *dvalue;
  size_t o_stride, dq_stride, dk_stride, dv_stride;
  float *ddecay, *dbeta;
  size_t ddecay_stride, dbeta_stride;
  float *last, *dh0, *carry;
  void* workspace;
  DeltaZero zero[5];
  // set by the launchers: how rows are read four elements at a time (whether dk and dv are multiples of 4, at least 4, or less), the workspace's
  // parts, and where the carry's states begin
  int fours;
  size_t blocks, carry_states, segments;   // segments: at most, 0 = sequences stay whole
  size_t slots;                            // places for the segments of sequences that are cut
  long segment;                            // blocks of one, where there is no plan
  int *first, *first_segment, *first_slot, *order, *table;
  float *matrices, *scalars, *x, *behind, *kept, *fronts, *maps;
  double* sums;
};

struct DeltaStepArgs {
  size_t rows;
  int heads, key_heads, dk, dv;
  const void *q, *k, *v;
  size_t q_stride, k_stride, v_stride;
  const float *decay, *beta;
  size_t decay_stride, beta_stride;
  float scale;
  float* state;
  size_t state_stride;
  void* o;
  size_t o_stride;
};

struct PolicyArgs {
  size_t rows, classes, row0;   // row0: a launch's first row
  const void* logits;
  size_t logits_stride;
  const void* index;
  int index_bytes;
  double inverse, scale;                     // 1 and log2(e) over the temperature
  double kl, low, high, log_low, log_high;   // the ratio's limits
  const float *advantage, *old, *reference, *weight;
  float *loss, *logprob;
  void* dlogits;
  size_t dlogits_stride;
};

struct ClipTensor {
  const void* p;
  void* out;
  size_t n;
  int dtype;
};

#define CLIP_LIST 140   // tensors of a launch, whose arguments are at most 4 KB
struct ClipList {
  const void* p[CLIP_LIST];
  void* out[CLIP_LIST];
  size_t count[CLIP_LIST];   // elements << 2 | dtype
  unsigned first[CLIP_LIST + 1];
  int n;
  size_t piece;
};

extern "C" {
size_t amp_norm_workspace_bytes(int dtype, size_t rows, size_t cols);
hipError_t amp_norm_forward_launch(int dtype, const NormArgs* a, hipStream_t stream);
hipError_t amp_norm_backward_launch(int dtype, const NormArgs* a, hipStream_t stream);
size_t amp_scan_carry_rows(int dtype, size_t rows, size_t hidden);
size_t amp_scan_workspace_bytes(int dtype, size_t rows, size_t hidden);
hipError_t amp_scan_forward_launch(int dtype, int tanh, const ScanArgs* a, hipStream_t stream);
hipError_t amp_scan_backward_launch(int dtype, int tanh, const ScanArgs* a, hipStream_t stream);
hipError_t amp_scan_step_launch(int dtype, int tanh, const ScanStepArgs* a, hipStream_t stream);
size_t amp_delta_blocks(size_t rows, size_t n);
size_t amp_delta_workspace_bytes(size_t rows, size_t n, size_t heads, size_t key_heads, size_t dk, size_t dv, int backward);
hipError_t amp_delta_forward_launch(int dtype, const DeltaArgs* a, hipStream_t stream);
hipError_t amp_delta_backward_launch(int dtype, const DeltaArgs* a, hipStream_t stream);
hipError_t amp_delta_step_launch(int dtype, const DeltaStepArgs* a, hipStream_t stream);
hipError_t amp_policy_launch(int dtype, const PolicyArgs* a, hipStream_t stream);
size_t amp_clip_workspace_bytes(size_t n, const ClipTensor* t);
hipError_t amp_clip_launch(size_t n, const ClipTensor* t, double max_norm, float* norm, void* workspace, hipStream_t stream);
size_t amp_distill_workspace_bytes(int dtype, size_t rows, size_t classes);
hipError_t amp_distill_launch(int dtype, const DistillArgs* a, hipStream_t stream);
}
