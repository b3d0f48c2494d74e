// Int4 projections of whole row batches (moe_linear.hip).
#pragma once

#include "moe_device.h"

namespace moe {

struct LinearArgs {
  const void *q, *sz, *lora_a, *lora_b;  // lora_*: null without an adapter (r = 0)
  int out_dim, in_dim, r, T, y_type;
  float lora_scale;
  const void* x;                         // fp16 [T][x_stride]
  int64_t x_stride, y_stride;
  void* y;
  // workspace, for many rows: [T][linear_extra] and [T]
  __half *e_hi, *e_lo;
  float* e_scale;
  float* sums;                           // of tiles split along the inputs
};

constexpr int kMostIn = 32768, kMostRank = 64;
constexpr int kRowsMost = 192;           // rows that the kernel without tiles takes at most
constexpr size_t kLinearSums = 32u << 20;

// Inputs that the group sums and the adapter add to a row's products.
constexpr int linear_extra(int in_dim, int r) { return (in_dim / 64 + 31) / 32 * 32 + (r + 31) / 32 * 32; }

// Whether the call goes without tiles (it does at fewer rows too, then).
bool linear_by_rows(int out_dim, int in_dim, int T);
hipError_t launch_linear(const LinearArgs& a, hipStream_t st);

}  // namespace moe
