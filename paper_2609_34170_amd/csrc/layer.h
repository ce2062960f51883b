// A layer's operators with their gradients (internal; the C ABI is in ravel.h): gated residual and norm,
// cross attention, gated MLP.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <string>

#include "common.h"
#include "ravel.h"

namespace ravel {

ravel_status set_error(ravel_status s, const std::string& msg);  // the calling thread's last error

hipError_t launch_norm_residual(const ravel_norm& n, hipStream_t s);
size_t norm_grad_workspace(const ravel_norm& n, const ravel_norm_grad& g);
hipError_t launch_norm_residual_grad(const ravel_norm& n, const ravel_norm_grad& g, hipStream_t s);

int64_t cross_blocks(const ravel_cross& c);  // of the largest launch
size_t cross_workspace(const ravel_cross& c);
hipError_t launch_cross_attention(const ravel_cross& c, hipStream_t s);
int64_t cross_grad_blocks(const ravel_cross& c, const ravel_cross_grad& g);
size_t cross_grad_workspace(const ravel_cross& c, const ravel_cross_grad& g);
hipError_t launch_cross_attention_grad(const ravel_cross& c, const ravel_cross_grad& g, hipStream_t s);

size_t mlp_workspace(const ravel_mlp& m);
hipError_t launch_gated_mlp(ravel_mlp m, hipStream_t s);
size_t mlp_grad_workspace(const ravel_mlp& m, const ravel_mlp_grad& g);
hipError_t launch_gated_mlp_grad(ravel_mlp m, const ravel_mlp_grad& g, hipStream_t s);

}  // namespace ravel
