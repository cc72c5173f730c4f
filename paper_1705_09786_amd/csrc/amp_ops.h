// What the checks (amp_ops.cpp) and the kernels of the operators on whole arrays (amp_norm.hip, amp_scan.hip,
// amp_distill.hip) agree on: arguments and launchers.  Sizes have been checked when a launcher is called.
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

extern "C" {
size_t amp_norm_workspace_bytes(int dtype, size_t rows, size_t cols);
hipError_t amp_norm_forward_launch(int dtype, const NormArgs* a, hipStream_t stream);
hipError_t amp_norm_backward_launch(int dtype, const NormArgs* a, hipStream_t stream);
size_t amp_scan_carry_rows(int dtype, size_t rows, size_t hidden);
size_t amp_scan_workspace_bytes(int dtype, size_t rows, size_t hidden);
hipError_t amp_scan_forward_launch(int dtype, int tanh, const ScanArgs* a, hipStream_t stream);
hipError_t amp_scan_backward_launch(int dtype, int tanh, const ScanArgs* a, hipStream_t stream);
hipError_t amp_scan_step_launch(int dtype, int tanh, const ScanStepArgs* a, hipStream_t stream);
size_t amp_distill_workspace_bytes(int dtype, size_t rows, size_t classes);
hipError_t amp_distill_launch(int dtype, const DistillArgs* a, hipStream_t stream);
}
