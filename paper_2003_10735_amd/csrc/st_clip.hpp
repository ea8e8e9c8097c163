// The norm and the clipping of many gradients: what the kernels and the entry points share.
#pragma once
#include "st_dense.hpp"

namespace st {
struct ClipRule { double scale, max_norm; float* norm; int write; };      // norm: written by the first block, or null; write 0: the norm alone
int64_t clip_parts(const st_grad_tensor* t, int n);
void grad_clip(Ctx& c, const st_grad_tensor* t, int n, const ClipRule& r, double* parts);
}  // namespace st
