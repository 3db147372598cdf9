// The losses of include/zb_stage.h for callers inside the library: the gradient may be scaled apart from the loss (a stage's loss is a mean
// over one microbatch, its gradient belongs to the mean over all of them).
#pragma once
#include "../../include/zb_stage.h"
#include "zb_common.h"

namespace zb {

constexpr int kLossMaxRows = (1 << 22) - 1;  // rows and pairs: a launch has less than 2^32 lanes, a row's or pair's workgroup up to 1024
size_t loss_workspace_bytes(int rows, int pairs);
zb_status policy_loss(const zb_logits* x, const zb_policy* p, double grad_scale, float* loss, float* logp, void* dlogits, int64_t dlogits_stride,
                      void* workspace, size_t workspace_size, hipStream_t s);
zb_status preference_loss(const zb_logits* x, const zb_preference* p, double grad_scale, float* loss, float* logp, float* rewards, void* dlogits,
                          int64_t dlogits_stride, void* workspace, size_t workspace_size, hipStream_t s);
bool valid_policy(const zb_policy* p);          // the numbers alone
bool valid_preference(const zb_preference* p);

}  // namespace zb
