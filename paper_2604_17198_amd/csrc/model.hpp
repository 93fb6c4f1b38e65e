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
hipError_t launch_experts_forward_kept(int dtype, const ProductArgs &a, const nacho_kept &pre, hipStream_t s);
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
    nacho_kept kept;               // code: pre in 8 bits, or NULL
};
int64_t experts_slope_tiles(int64_t slots, int64_t experts);
hipError_t launch_experts_slope(int dtype, const SlopeArgs &a, hipStream_t s);

// ---- rows kept in 8 bits ----------------------------------------------------------
struct KeepArgs {
    const void *x;                 // rows to keep
    void *out;                     // restored rows
    int64_t ldx;                   // of either
    int64_t rows;
    int32_t cols;
    nacho_kept kept;
};
hipError_t launch_keep(int dtype, const KeepArgs &a, hipStream_t s);
hipError_t launch_restore(int dtype, const KeepArgs &a, hipStream_t s);

// ---- a whole layer of experts for a few tokens -----------------------------------
constexpr int kMostStepTokens = 64;
struct StepArgs {
    const void *logits;            // [tokens] rows of `ldl` elements
    int64_t ldl;
    const uint8_t *keep;           // may be NULL: every token
    int32_t tokens, experts, top_k, normalise, inner, hidden, outer, act;
    const void *x;
    int64_t ldx;
    nacho_dense up, gate, down;    // gate.w: may be NULL
    const void *residual;          // may be NULL
    int64_t ldr;
    void *out;
    int64_t ldo;
    // workspace: the rows between the products by slot (token x top_k + choice), the choice, its gates, the experts that a token
    // chose behind their number
    void *h;
    int64_t ldh;
    uint16_t *choice;
    float *share;
    int32_t *active;
    uint16_t *order;               // the slots by these experts, from `first` of each on
    int32_t *first;
    int32_t tiles, parts;          // of the second product: tiles of rows, workgroups that share one
    float *partial;                // [tiles][parts][tokens][16], several parts
    int32_t *arrived;              // [tiles]
};
void step_plan(int dtype, int64_t tokens, int64_t experts, int64_t top_k, int64_t hidden, int64_t outer, int32_t *tiles, int32_t *parts);
hipError_t launch_step(int dtype, const StepArgs &a, hipStream_t s);

// ---- cross entropy against a vocabulary ---------------------------------------------
struct XentArgs {
    const void *x;                 // [rows], `ldx` apart
    int64_t ldx;
    const void *head;              // [vocabulary], `ldh` apart
    int64_t ldh;
    int64_t rows, vocabulary;
    int32_t inner, elem, label_bytes, half;      // elem: bytes of a value; half: f16
    const void *label;
    const float *weight;           // may be NULL: ones
    float *loss, *lse;             // loss: NULL in a gradient call, which reads lse
    void *grad_x, *grad_head;      // may be NULL
    int64_t ldgx, ldgh;
    // workspace: the rows that count (slots) and their number
    int32_t *bounds, *token, *slot_label;
    // of many rows, by workgroups that list them: how many count, and the largest weight (NULL: they need neither)
    int32_t *counts;
    float *most;
    // of the loss: [tiles of the vocabulary][rows], and the label's logit by slot
    float2 *partial;
    float *at_label;
    // of the gradient: by slot, the slot of a row (or -1), {a power of two that g is multiplied by, its inverse}, g of a piece, sums
    float *slot_lse, *factor;
    int32_t *slot_of;
    float *scale;
    void *g;
    float *sums;
    // of either, where rows start anywhere: the rows that count and a piece of head as rows of whole words (NULL: not wanted)
    void *padded_x, *padded_head;
};
// How a call goes through the vocabulary: `pieces` of `words`, each in `stretches` of `k_part` for the rows' sums.
struct XentPlan {
    int64_t pieces, words, ldg, stretches, shortest, k_part, lds;      // (no stretch shorter than `shortest`)
    bool sums;                     // (of the rows' gradients, in 32 bits: `lds` apart, one set a stretch)
};
int64_t xent_counts(int64_t rows);     // workgroups that `counts` and `most` are by
int64_t xent_partials(int elem, int64_t rows, int64_t vocabulary);
XentPlan xent_plan(int elem, int64_t rows, int64_t vocabulary, int64_t inner, bool pads, bool gradient);
constexpr int64_t kPaddedFrom = 384;   // rows
bool xent_pads(const XentArgs &a);
hipError_t launch_xent(int dtype, const XentArgs &a, const XentPlan &plan, hipStream_t s);
// The logits of up to kFewRows rows (words `first` .. of the vocabulary), which are rows of words of 16 bytes, in_words, or rows of four floats or
// more that start anywhere: statistics by workgroup in a.partial, or, where there is a.g, g.
constexpr int kFewRows = 16;
int64_t xent_few_groups(int64_t vocabulary);
hipError_t launch_xent_few(int dtype, const XentArgs &a, int64_t first, int64_t words, int64_t ldg, bool in_words, hipStream_t s);
// grad_head of a piece from g and the rows of x.
hipError_t launch_xent_few_head(int dtype, const XentArgs &a, int64_t first, int64_t words, int64_t ldg, hipStream_t s);
hipError_t launch_xent_grad(int dtype, const XentArgs &a, const XentPlan &plan, hipStream_t s);

}  // namespace nacho
