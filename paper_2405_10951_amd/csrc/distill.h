// Distillation from a teacher's top logits (k_distill.hip): raw device pointers and a stream, no allocation, no wait.
#pragma once
#include "bsr_internal.h"

namespace bsr {

constexpr int DISTILL_MAX_TOP = 1024;
struct DistillArgs {
  const void* z = nullptr; bool f32 = false; int64_t rows = 0; int classes = 0; int64_t ldz = 0;     // student logits
  const int32_t* index = nullptr; int64_t ldi = 0;      // [rows, top]: the teacher's classes; outside 0 .. classes - 1: absent
  const void* top = nullptr; bool top_f32 = true; int64_t ldt = 0; int k = 0;                        // its logits
  const int32_t* labels = nullptr;                      // [rows], outside 0 .. classes - 1: none; null: no row has one
  float temperature = 1.f, hard = 0.f;
  float* loss = nullptr;                                // [rows]; null: not wanted
  float* stats = nullptr;                               // [rows, 3]: m = max z, log sum exp((z - m) / temperature), log sum exp(z - m): written by the forward, read by the backward
  const float* row_grad = nullptr;                      // [rows], null: 1 for each
  float grad_scale = 1.f;
  void* dz = nullptr; int64_t ldd = 0;                  // type of z; may be z itself
  float* parts = nullptr;                               // forward: scratch of distill_parts_floats() floats, null: a row is not split
  int segments = 1, writers = 1;                        // (set inside) workgroups that sum up a row, and that write it
};
size_t distill_parts_floats(bool f32, int64_t rows, int classes);      // 0: nothing to split
void distill_forward(const DistillArgs& a, hipStream_t s);      // loss, stats and, where dz is given, the gradient
void distill_backward(const DistillArgs& a, hipStream_t s);     // dz from stats

}  // namespace bsr
