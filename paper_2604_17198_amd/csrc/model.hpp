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
    float *partial;                // distill_partials floats
    bool stream;                   // the gradient is stored past the caches (set by the launch)
};
// Floats that a call keeps of rows that are cut into parts.
int64_t distill_partials(int dtype, int64_t rows, int64_t cols, bool grad);
hipError_t launch_distill(int dtype, const DistillArgs &a, hipStream_t s);
hipError_t launch_distill_grad(int dtype, const DistillArgs &a, hipStream_t s);

// ---- routing ------------------------------------------------------------------
constexpr int kMostExperts = 1024, kMostChoices = 32;
struct RouteArgs {
    const void *logits;            // [tokens] rows of `ldl` elements
    int64_t ldl;
    const uint8_t *keep;           // may be NULL: every token
    int64_t tokens;
    int32_t experts, top_k, normalise;
    nacho_routing out;
};
// Scratch of a routing call: `groups` workgroups work on `per_group` consecutive tokens each.
struct RouteScratch {
    int64_t groups, per_group;
    int32_t *hist;                 // [groups][experts]: entries; after the scan those of the groups before
    float *share;                  // [groups][experts]: sums of probabilities; after the scan row 0 holds the total
    int32_t *entries, *routed;     // [groups] entries and tokens that store one
    uint16_t *choice;              // [tokens * top_k]
    float *gate;                   // [tokens * top_k]
    uint8_t *held;                 // [tokens] entries of a token
};
void route_plan(int64_t tokens, int32_t experts, int64_t *groups, int64_t *per_group);
hipError_t launch_route(int dtype, const RouteArgs &a, const RouteScratch &w, hipStream_t s);
struct RouteGradArgs {
    const void *logits;
    int64_t ldl;
    int64_t tokens;
    int32_t experts, normalise;
    nacho_routing routing;         // (a token that is not kept stores nothing)
    const float *grad_gate;
    float balance;
    void *grad;
    int64_t ldg;
};
hipError_t launch_route_grad(int dtype, const RouteGradArgs &a, hipStream_t s);

// ---- sums of the experts' rows for every token ---------------------------------
struct CombineArgs {
    const int32_t *pos, *slot;     // CSR, tokens x slots
    const float *gate;             // may be NULL: ones
    int64_t tokens;
    const void *y;                 // [slots] rows of `ldy` elements
    int64_t ldy;
    int32_t cols;
    const void *residual;          // forward: may be NULL
    int64_t ldr;
    void *out;
    int64_t ldo;
    const void *grad_out;          // backward
    int64_t ldg;
    void *grad_y;                  // may be NULL
    int64_t ldgy;
    float *grad_gate;              // may be NULL
};
hipError_t launch_combine(int dtype, const CombineArgs &a, hipStream_t s);
hipError_t launch_combine_grad(int dtype, const CombineArgs &a, hipStream_t s);

// ---- the experts' products -----------------------------------------------------
// out[m][n] = sum_k Q(m, k) P(n, k) for every expert, in one of three forms:
//   forward   m: slots, n: outer, k: inner   Q = x[token], P = w[e]            + bias, activation
//   rows      m: slots, n: inner, k: outer   Q = grad_z,   P = w[e] transposed
//   weights   m: outer, n: inner, k: slots   Q = grad_z transposed, P = x[token] transposed
struct ProductArgs {
    const int32_t *bounds, *token; // token: may be NULL (forward, weights)
    int32_t experts, m, n, k;      // sizes, but for the one that is the slots
    int64_t slots;                 // at most
    const void *q, *p;
    int64_t ldq, ldp, p_stride;    // p_stride: from expert to expert
    void *out;
    int64_t ldo, out_stride;
    const void *bias;              // may be NULL
    int64_t bias_stride;
    void *pre;                     // may be NULL
    int64_t ldpre;
    int32_t act;
};
hipError_t launch_experts_forward(int dtype, const ProductArgs &a, hipStream_t s);
hipError_t launch_experts_rows(int dtype, const ProductArgs &a, hipStream_t s);
hipError_t launch_experts_weights(int dtype, const ProductArgs &a, hipStream_t s);
// grad_z = grad_y act'(pre), and the sums of its rows by expert (grad_bias, may be NULL).  grad_z may be NULL: not wanted.
struct SlopeArgs {
    const int32_t *bounds;
    int32_t experts, cols, act;
    int64_t slots;
    const void *grad_y, *pre;
    int64_t ldgy, ldpre;
    void *grad_z;
    int64_t ldgz;
    void *grad_bias;
    int64_t bias_stride;
    float *sums;                   // [experts_slope_tiles][cols], with grad_bias
};
int64_t experts_slope_tiles(int64_t slots, int64_t experts);
hipError_t launch_experts_slope(int dtype, const SlopeArgs &a, hipStream_t s);

}  // namespace nacho
