// Softmax cross-entropy of a linear layer whose logits nobody keeps, and its gradients (k_linear_ce.hip): raw device pointers and a stream, no allocation, no wait.
#pragma once
#include "bsr_internal.h"

namespace bsr {

struct LinearCe {
  const void* x = nullptr; int64_t ldx = 0; int N = 0;          // [N, D]
  const void* w = nullptr; int64_t ldw = 0; int V = 0, D = 0;   // [V, D]
  bool f32 = false;                                             // type of x, w and dx
  const float* bias = nullptr;                                  // [V]; null: none
  const int32_t* labels = nullptr;                              // [N], outside 0 .. V - 1: the row counts for nothing
  float *loss = nullptr, *stats = nullptr;                      // forward: [N], [N, 2]; either may be null.  Backward: stats is read
  const float* row_grad = nullptr; float grad_scale = 1.f;      // [N], null: 1 for each
  void* dx = nullptr; int64_t lddx = 0;                         // null: not wanted
  void* dw = nullptr; int64_t lddw = 0; bool dw_f32 = false;    // null: not wanted
  float* db = nullptr;                                          // [V]; null: not wanted
  void* workspace = nullptr;                                    // 256-byte aligned
};
size_t linear_ce_workspace_bytes(bool f32, int N, int D, int V, bool backward);
void linear_ce_forward(const LinearCe& a, hipStream_t s);
void linear_ce_backward(const LinearCe& a, hipStream_t s);
// one after the other, the second with what the first leaves; stats (not null) is written
size_t linear_ce_both_bytes(bool f32, int N, int D, int V);
void linear_ce_both(const LinearCe& a, hipStream_t s);
// what the forward and the backward of their own take, as bsr.h says; host only
struct LinearCeTiles { int32_t forward = 0, forward_pieces = 0, forward_last = 0, gradient = 0, pieces = 0, gradient_last = 0, products = 0, splits_x = 0, splits_w = 0; };
void linear_ce_tiles(const LinearCe& a, LinearCeTiles& t);

// k_linear_ce_small.hip: scratch of small_ce_bytes() for the logits, or for G, with grad_scale and the rows' weights, [N, small_ce_stride()]
inline int64_t small_ce_stride(int N, int V) { return N <= 64 ? ((int64_t)V + 15) / 16 * 16 : ((int64_t)V + 3) / 4 * 4; }
inline size_t small_ce_bytes(int N, int V) { return sizeof(float) * (size_t)N * small_ce_stride(N, V); }
void small_ce_logits(const LinearCe& a, float* z, hipStream_t s);
void small_ce_forward(const LinearCe& a, float* z, bool grad, hipStream_t s);      // grad (of few rows, below): G in the logits' place
// N up to FEW_ROWS: G (or the logits) at the workspace's beginning, few_ce_bytes() more at few_parts_at()
constexpr int FEW_ROWS = 64;
size_t few_parts_at(int N, int V);
size_t few_ce_bytes(bool f32, int N, int V, int D);
// what G holds: nothing, logits, or G; fused: nothing, and the forward is wanted as well (of few_fused() classes)
enum Few { FEW_NOTHING, FEW_LOGITS, FEW_GRADIENT, FEW_FUSED };
bool few_fused(bool f32, int V);
void few_ce_backward(const LinearCe& a, Few there, hipStream_t s);

}  // namespace bsr
