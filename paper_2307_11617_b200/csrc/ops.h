// Internal launchers of the training-step operators (gradient norm, AdamW step, group norm).
// The C entry points of rfast.h check their arguments and call these; the engine calls them
// with its own rows.  Nothing here is part of the public ABI.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "rfast.h"
#include "rfast_internal.h"

namespace rfast {

constexpr int kAdamBlock = RFAST_ADAMW_BLOCK;    // values that share a scale of the 8-bit moments

// Scalars of one AdamW step, formed on the host in 64 bits and rounded once.
struct AdamCoef {
    float beta1, omb1, beta2;          // omb = 1 - beta
    float root_beta2, root_omb2;       // square roots of beta2 and 1 - beta2
    float eps, keep;                   // keep = 1 - lr * weight_decay
    float step;                        // lr / (1 - beta1^t)
    float root;                        // 1 / sqrt(1 - beta2^t)
};
AdamCoef adamw_coef(double lr, double beta1, double beta2, double eps, double weight_decay, int64_t t);

// The engine's step: x_i of every active node of a round, its tracker z_i in the role of the
// gradient.  factor[s - 1] = {1 / (1 - beta1^s), 1 / sqrt(1 - beta2^s)} of the event's stamp s.
struct AdamRows {
    const EvDesc* ev;
    float* x;
    const float* z;                    // [n][stride]
    void *m, *v;                       // [n][stride] fp32 or 8-bit codes
    float *m_scale, *v_scale;          // [n][scale_stride], 8-bit moments only
    int64_t p, stride, scale_stride;
    const float2* factor;
    float lr;
};
cudaError_t adamw_rows_launch(const AdamRows& r, const AdamCoef& c, int state_bits, int n_events, cudaStream_t st);

// The engine's hidden layers: rows [n_events][batch][hidden] fp32, event e with the scale and shift of its node.
struct NormRows {
    const EvDesc* ev;
    int n_events, batch, hidden, groups, act;
    float eps;
    const float *gamma, *beta;         // of node 0; a node's are node * stride further on
    int64_t stride;
    const float* x;                    // before the norm
    float* out;                        // forward: the layer's output; backward: the gradient of x
    const float* dy;                   // backward (may be `out`)
    float *mean, *rstd;                // [n_events * batch][groups]
    float *dgamma, *dbeta;             // backward: [n_events][hidden]
    void* workspace;                   // norm_rows_workspace() bytes
};
size_t norm_rows_workspace(int max_events, int batch, int hidden);
cudaError_t norm_rows_launch(const NormRows& r, bool backward, cudaStream_t st, int64_t* launches);

// Sets err and returns RFAST_EINVAL / RFAST_ECUDA unless `p` is memory of the current device.
int check_device_pointer(const void* p, const char* what, char* err, size_t err_len);
int op_fail(char* err, size_t err_len, int code, const char* fmt, ...);

}  // namespace rfast
