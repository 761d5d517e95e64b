// The norm of many tensors taken together, and the tensors brought down to a largest norm (k_clip.hip): raw device pointers and a stream, no allocation, no wait.
#pragma once
#include "bsr_internal.h"

namespace bsr {

// Tensors of a launch; the table travels as a kernel argument (< 4 KB).
constexpr int CLIP_TENSORS = 144;
struct ClipTable {
  const void* g[CLIP_TENSORS];
  void* out[CLIP_TENSORS];
  int64_t n[CLIP_TENSORS];                          // values; negative: -n values of bf16, else fp32
  int start[CLIP_TENSORS];                          // first piece of each
  int count = 0, pieces = 0;
};
constexpr int CLIP_PIECE = 16384;                   // values of a piece
inline int clip_launches(int count) { return (count + CLIP_TENSORS - 1) / CLIP_TENSORS; }
// workgroups of a launch of the first pass, which leave a part each
inline int clip_share(int count) { const int n = 4096 / clip_launches(count); return n < 64 ? 64 : n > 2048 ? 2048 : n; }
inline size_t clip_workspace_bytes(int count) { return count < 1 ? 0 : sizeof(double) * (size_t)clip_share(count) * clip_launches(count); }

struct ClipArgs {
  const void* const* g = nullptr; const int32_t* f32 = nullptr; const int64_t* n = nullptr; int count = 0;      // host arrays; f32: not 0 where a tensor is fp32
  void* const* out = nullptr;                       // null: the norm alone
  float max_norm = 0.f;
  float* norm = nullptr;
  double* parts = nullptr;                          // clip_workspace_bytes(count)
};
void clip(const ClipArgs& a, hipStream_t s);

}  // namespace bsr
