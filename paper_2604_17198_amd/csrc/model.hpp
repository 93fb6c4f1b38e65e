// Launchers of the operators that train models: distillation, routing, experts' products and their sums.
#pragma once
#include "dense.hpp"

namespace nacho {

// ---- distillation -----------------------------------------------------------
struct DistillArgs {
    const int32_t *pos, *crd;      // the teacher: CSR, rows x cols
    const float *val;
    const void *logits;            // rows of `ldl` elements
    int64_t ldl;
    const float *weight;           // may be NULL: ones
    float temperature;
    float *loss, *lse;             // may be NULL (both, in a gradient call)
    const float *lse_in;           // a gradient call: what the forward call left
    void *grad;                    // may be NULL
    int64_t ldg;
    int64_t rows;
    int32_t cols;
};
hipError_t launch_distill(int dtype, const DistillArgs &a, hipStream_t s);
hipError_t launch_distill_grad(int dtype, const DistillArgs &a, hipStream_t s);

}  // namespace nacho
