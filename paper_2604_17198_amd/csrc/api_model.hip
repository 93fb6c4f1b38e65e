// C-ABI entry points of the operators that train models: argument checks, workspace carving, kernel sequencing.
#include "kernels.hpp"
#include "model.hpp"

using namespace nacho;
using namespace nacho_host;

namespace {

bool value_type(int32_t dtype) { return dtype == NACHO_F32 || dtype == NACHO_BF16 || dtype == NACHO_F16; }
int64_t value_bytes(int32_t dtype) { return dtype == NACHO_F32 ? 4 : 2; }
bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
constexpr int64_t kMostRows = 0x7fffffffLL, kMostStride = (int64_t)1 << 40;

// A dense matrix of `rows` rows of `cols` elements, `ld` apart.
bool matrix(const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t elem)
{
    if (ld < cols || ld > kMostStride) return false;
    return rows == 0 || cols == 0 || (p && aligned(p, (uintptr_t)elem));
}

// Whether two such matrices share a byte of the stretches they span.
bool overlap(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && a_bytes > 0 && b_bytes > 0 && x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}
// Bytes from a matrix's first element to its last one.  (Up to 2^31 rows, 2^40 elements apart: longer stretches than any
// memory count as 2^62 bytes.)
int64_t stretch(__int128 elements, int64_t elem)
{
    const __int128 bytes = elements * elem, most = (__int128)1 << 62;
    return (int64_t)(bytes < most ? bytes : most);
}
int64_t span(int64_t rows, int64_t cols, int64_t ld, int64_t elem)
{
    return rows > 0 ? stretch((__int128)(rows - 1) * ld + cols, elem) : 0;
}

// An array of a call.
struct Array {
    const void *at;
    int64_t bytes;
};
// Whether the outputs share no byte with each other or with an input.
bool apart(std::initializer_list<Array> outputs, std::initializer_list<Array> inputs)
{
    for (const Array *o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Array *p = outputs.begin(); p != o; ++p)
            if (overlap(o->at, o->bytes, p->at, p->bytes)) return false;
        for (const Array &p : inputs)
            if (overlap(o->at, o->bytes, p.at, p.bytes)) return false;
    }
    return true;
}

// Slices of a workspace, 256-byte aligned.
struct Slices {
    char *base;
    size_t off = 0;
    explicit Slices(void *p) : base(static_cast<char *>(p)) {}
    template <typename T> T *take(int64_t n)
    {
        off = align_up(off, 256);
        T *r = base ? reinterpret_cast<T *>(base + off) : nullptr;
        off += (size_t)n * sizeof(T);
        return r;
    }
};

RouteScratch carve_route(void *ws, int64_t tokens, int32_t experts, int32_t top_k, size_t *bytes)
{
    Slices c(ws);
    RouteScratch w;
    route_plan(tokens, experts, &w.groups, &w.per_group);
    w.hist = c.take<int32_t>(w.groups * experts);
    w.share = c.take<float>(w.groups * experts);
    w.entries = c.take<int32_t>(w.groups);
    w.routed = c.take<int32_t>(w.groups);
    w.choice = c.take<uint16_t>(tokens * top_k);
    w.gate = c.take<float>(tokens * top_k);
    w.held = c.take<uint8_t>(tokens);
    *bytes = align_up(c.off, 256);
    return w;
}

// Sizes of a routing call.
int32_t check_route(int64_t tokens, int64_t experts, int32_t top_k)
{
    if (tokens < 0 || experts < 1 || top_k < 1 || top_k > experts) return NACHO_ERR_INVALID_ARG;
    if (experts > kMostExperts || top_k > kMostChoices) return NACHO_ERR_UNSUPPORTED;
    return tokens > kMostRows || tokens * top_k > kMostRows ? NACHO_ERR_INVALID_ARG : NACHO_OK;
}
bool check_routing(const nacho_routing *r)
{
    if (!r || !r->pos || !r->expert || !r->gate || !r->slot || !r->expert_pos || !r->token || !r->counts || !r->lse ||
        !r->balance || !r->routed)
        return false;
    const void *all[] = {r->pos, r->expert, r->gate, r->slot, r->expert_pos, r->token, r->counts, r->lse, r->balance, r->routed};
    for (const void *p : all)
        if (!aligned(p, 4)) return false;
    return true;
}

// The teacher: one CSR operand of floats.
int32_t check_distill(const nacho_tensor *teacher, const void *logits, int64_t ldl, int32_t dtype, const float *weight,
                      float temperature, void *grad, int64_t ldg, DistillArgs *a)
{
    if (!teacher || !value_type(dtype)) return NACHO_ERR_INVALID_ARG;
    if (teacher->nlevels != 2 || teacher->lvl[0].kind != NACHO_DENSE || teacher->lvl[1].kind != NACHO_COMPRESSED)
        return NACHO_ERR_UNSUPPORTED;
    const int64_t rows = teacher->lvl[0].extent, cols = teacher->lvl[1].extent, stored = teacher->lvl[1].count;
    if (rows < 0 || rows > kMostRows || cols < 0 || cols > kMostRows || stored < 0 || stored > kMostRows)
        return NACHO_ERR_INVALID_ARG;
    if (!teacher->lvl[1].pos || (stored > 0 && (!teacher->lvl[1].crd || !teacher->val))) return NACHO_ERR_INVALID_ARG;
    if (!aligned(teacher->lvl[1].pos, 4) || !aligned(teacher->lvl[1].crd, 16) || !aligned(teacher->val, 16) || !aligned(weight, 4))
        return NACHO_ERR_INVALID_ARG;
    const int64_t elem = value_bytes(dtype);
    if (!matrix(logits, rows, cols, ldl, elem) || !(temperature >= 1e-30f && temperature <= 1e18f)) return NACHO_ERR_INVALID_ARG;
    if (grad && !matrix(grad, rows, cols, ldg, elem)) return NACHO_ERR_INVALID_ARG;
    *a = DistillArgs{teacher->lvl[1].pos, teacher->lvl[1].crd, static_cast<const float *>(teacher->val), logits, ldl, weight,
                     temperature, nullptr, nullptr, nullptr, grad, ldg, rows, (int32_t)cols, nullptr, false};
    return NACHO_OK;
}

// The arrays that a distillation call reads, and with them the outputs (`lse` is one or the other).
bool check_distill_arrays(const nacho_tensor *teacher, const DistillArgs &a, int64_t elem, const float *lse_in, float *loss, float *lse,
                          const void *ws, int64_t ws_bytes)
{
    const int64_t by_row = a.rows * 4, stored = teacher->lvl[1].count * 4;
    return apart({{loss, by_row}, {lse, by_row}, {a.grad, a.grad ? span(a.rows, a.cols, a.ldg, elem) : 0}, {ws, ws_bytes}},
                 {{a.pos, by_row + 4}, {a.crd, stored}, {a.val, stored}, {a.logits, span(a.rows, a.cols, a.ldl, elem)}, {a.weight, by_row},
                  {lse_in, by_row}});
}

// The routing matrix of a combine call: CSR, tokens x slots.
int32_t check_combine(const nacho_tensor *m, int64_t n, int32_t dtype, CombineArgs *a)
{
    if (!m || !value_type(dtype) || n < 0 || n > kMostRows) return NACHO_ERR_INVALID_ARG;
    if (m->nlevels != 2 || m->lvl[0].kind != NACHO_DENSE || m->lvl[1].kind != NACHO_COMPRESSED) return NACHO_ERR_UNSUPPORTED;
    const int64_t tokens = m->lvl[0].extent, slots = m->lvl[1].extent, stored = m->lvl[1].count;
    if (tokens < 0 || tokens > kMostRows || slots < 0 || slots > kMostRows || stored < 0 || stored > kMostRows)
        return NACHO_ERR_INVALID_ARG;
    if (!m->lvl[1].pos || !aligned(m->lvl[1].pos, 4) || (stored > 0 && !m->lvl[1].crd) || !aligned(m->lvl[1].crd, 4) ||
        !aligned(m->val, 4))
        return NACHO_ERR_INVALID_ARG;
    *a = CombineArgs{};
    a->pos = m->lvl[1].pos;
    a->slot = m->lvl[1].crd;
    a->gate = static_cast<const float *>(m->val);
    a->tokens = tokens;
    a->cols = (int32_t)n;
    return NACHO_OK;
}

// `count` matrices of rows x cols elements, `ld` and `stride` apart.
bool matrices(const void *p, int64_t count, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int64_t elem)
{
    if (!matrix(p, count > 0 ? rows : 0, cols, ld, elem) || stride > kMostStride) return false;
    return count <= 1 || rows == 0 || stride >= (__int128)(rows - 1) * ld + cols;
}
int64_t span(int64_t count, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int64_t elem)
{
    return count > 0 && rows > 0 ? stretch((__int128)(count - 1) * stride + (__int128)(rows - 1) * ld + cols, elem) : 0;
}

int32_t check_layer(const nacho_experts_layer *l)
{
    if (!l || !value_type(l->dtype) || l->act < NACHO_ACT_NONE || l->act > NACHO_ACT_SILU) return NACHO_ERR_INVALID_ARG;
    if (l->n_experts < 1 || l->n_slots < 0 || l->n_slots > kMostRows || l->n_tokens < 0 || l->n_tokens > kMostRows ||
        l->inner < 1 || l->outer < 1)
        return NACHO_ERR_INVALID_ARG;
    if (l->n_experts > 65536 || l->inner >= 1 << 24 || l->outer >= 1 << 24) return NACHO_ERR_UNSUPPORTED;
    if (!l->expert_pos || !aligned(l->expert_pos, 4) || !aligned(l->token, 4)) return NACHO_ERR_INVALID_ARG;
    // (without a list of tokens a slot reads the row of its own number)
    return !l->token && l->n_tokens < l->n_slots ? NACHO_ERR_INVALID_ARG : NACHO_OK;
}
bool check_x(const nacho_experts_layer *l, int64_t elem) { return matrix(l->x, l->n_tokens, l->inner, l->ldx, elem); }
bool check_w(const nacho_experts_layer *l, int64_t elem)
{
    return matrices(l->w, l->n_experts, l->outer, l->inner, l->ldw, l->w_stride, elem);
}
// The arrays of a layer that a call reads.
Array x_of(const nacho_experts_layer *l, int64_t elem) { return {l->x, l->x ? span(l->n_tokens, l->inner, l->ldx, elem) : 0}; }
Array w_of(const nacho_experts_layer *l, int64_t elem)
{
    return {l->w, l->w ? span(l->n_experts, l->outer, l->inner, l->ldw, l->w_stride, elem) : 0};
}
Array bounds_of(const nacho_experts_layer *l) { return {l->expert_pos, l->n_experts * 4 + 4}; }
Array token_of(const nacho_experts_layer *l) { return {l->token, l->n_slots * 4}; }

// What a gradient call keeps: the gradient before the activation, and sums of its rows.
struct GradWs {
    void *grad_z;
    float *sums;
    size_t bytes;
};
GradWs carve_grad(void *ws, const nacho_experts_layer *l, bool grad_z, bool sums)
{
    Slices c(ws);
    GradWs w{};
    if (grad_z) w.grad_z = c.take<char>(l->n_slots * ((l->outer + 7) / 8 * 8) * value_bytes(l->dtype));
    if (sums) w.sums = c.take<float>(experts_slope_tiles(l->n_slots, l->n_experts) * l->outer);
    w.bytes = align_up(c.off, 256);
    return w;
}

}  // namespace

extern "C" {

int32_t nacho_distill(const nacho_tensor *teacher, const void *logits, int64_t ldl, int32_t dtype, const float *weight,
                      float temperature, float *loss, float *lse, void *grad, int64_t ldg, void *ws, size_t ws_bytes,
                      void *hip_stream)
{
    DistillArgs a;
    const int32_t rc = check_distill(teacher, logits, ldl, dtype, weight, temperature, grad, ldg, &a);
    if (rc != NACHO_OK) return rc;
    if ((a.rows > 0 && (!loss || !lse)) || !aligned(loss, 4) || !aligned(lse, 4)) return NACHO_ERR_INVALID_ARG;
    const size_t need = align_up((size_t)distill_partials(dtype, a.rows, a.cols, grad != nullptr) * sizeof(float), 256);
    if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16))) return NACHO_ERR_WORKSPACE;
    if (!check_distill_arrays(teacher, a, value_bytes(dtype), nullptr, loss, lse, ws, (int64_t)need)) return NACHO_ERR_INVALID_ARG;
    a.partial = static_cast<float *>(ws);
    a.loss = loss;
    a.lse = lse;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    profile_begin(s);
    if (launch_distill(dtype, a, s) != hipSuccess) return NACHO_ERR_HIP;
    profile_mark("distill");
    return NACHO_OK;
}

int32_t nacho_distill_workspace_bytes(int64_t n_rows, int64_t n_cols, int32_t dtype, size_t *bytes)
{
    if (!bytes || !value_type(dtype) || n_rows < 0 || n_rows > kMostRows || n_cols < 0 || n_cols > kMostRows)
        return NACHO_ERR_INVALID_ARG;
    const int64_t with = distill_partials(dtype, n_rows, n_cols, true), without = distill_partials(dtype, n_rows, n_cols, false);
    *bytes = align_up((size_t)(with > without ? with : without) * sizeof(float), 256);
    return NACHO_OK;
}

int32_t nacho_distill_grad(const nacho_tensor *teacher, const void *logits, int64_t ldl, int32_t dtype, const float *weight,
                           float temperature, const float *lse, void *grad, int64_t ldg, void *hip_stream)
{
    DistillArgs a;
    const int32_t rc = check_distill(teacher, logits, ldl, dtype, weight, temperature, grad, ldg, &a);
    if (rc != NACHO_OK) return rc;
    if ((a.rows > 0 && a.cols > 0 && (!lse || !grad)) || !aligned(lse, 4)) return NACHO_ERR_INVALID_ARG;
    if (!check_distill_arrays(teacher, a, value_bytes(dtype), lse, nullptr, nullptr, nullptr, 0)) return NACHO_ERR_INVALID_ARG;
    a.lse_in = lse;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    profile_begin(s);
    if (launch_distill_grad(dtype, a, s) != hipSuccess) return NACHO_ERR_HIP;
    profile_mark("distill_grad");
    return NACHO_OK;
}

int32_t nacho_route_workspace_bytes(int64_t n_tokens, int64_t n_experts, int32_t top_k, size_t *bytes)
{
    if (!bytes) return NACHO_ERR_INVALID_ARG;
    const int32_t rc = check_route(n_tokens, n_experts, top_k);
    if (rc == NACHO_OK) carve_route(nullptr, n_tokens, (int32_t)n_experts, top_k, bytes);
    return rc;
}

int32_t nacho_route(const void *logits, int64_t ldl, int64_t n_tokens, int64_t n_experts, int32_t dtype, int32_t top_k,
                    int32_t normalise, const uint8_t *keep, const nacho_routing *out, void *ws, size_t ws_bytes,
                    void *hip_stream)
{
    int32_t rc = check_route(n_tokens, n_experts, top_k);
    if (rc != NACHO_OK) return rc;
    if (!value_type(dtype) || !matrix(logits, n_tokens, n_experts, ldl, value_bytes(dtype)) || !check_routing(out))
        return NACHO_ERR_INVALID_ARG;
    size_t need = 0;
    const RouteScratch w = carve_route(ws, n_tokens, (int32_t)n_experts, top_k, &need);
    if (!ws || ws_bytes < need || !aligned(ws, 16)) return NACHO_ERR_WORKSPACE;
    const int64_t room = n_tokens * top_k * 4;
    if (!apart({{out->pos, n_tokens * 4 + 4}, {out->expert, room}, {out->gate, room}, {out->slot, room}, {out->expert_pos, n_experts * 4 + 4},
                {out->token, room}, {out->counts, n_experts * 4}, {out->lse, n_tokens * 4}, {out->balance, 4}, {out->routed, 4}, {ws, (int64_t)need}},
               {{logits, span(n_tokens, n_experts, ldl, value_bytes(dtype))}, {keep, n_tokens}}))
        return NACHO_ERR_INVALID_ARG;
    const RouteArgs a{logits, ldl, keep, n_tokens, (int32_t)n_experts, top_k, normalise != 0, *out};
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    profile_begin(s);
    return launch_route(dtype, a, w, s) == hipSuccess ? NACHO_OK : NACHO_ERR_HIP;
}

int32_t nacho_route_grad(const void *logits, int64_t ldl, int64_t n_tokens, int64_t n_experts, int32_t dtype, int32_t top_k,
                         int32_t normalise, const nacho_routing *routing, const float *grad_gate, float balance,
                         void *grad, int64_t ldg, void *hip_stream)
{
    const int32_t rc = check_route(n_tokens, n_experts, top_k);
    if (rc != NACHO_OK) return rc;
    if (!value_type(dtype) || !check_routing(routing) || !aligned(grad_gate, 4)) return NACHO_ERR_INVALID_ARG;
    const int64_t elem = value_bytes(dtype);
    if (!matrix(logits, n_tokens, n_experts, ldl, elem) || !matrix(grad, n_tokens, n_experts, ldg, elem)) return NACHO_ERR_INVALID_ARG;
    const int64_t room = n_tokens * top_k * 4;
    if (!apart({{grad, span(n_tokens, n_experts, ldg, elem)}},
               {{logits, span(n_tokens, n_experts, ldl, elem)}, {grad_gate, room}, {routing->pos, n_tokens * 4 + 4}, {routing->expert, room},
                {routing->gate, room}, {routing->slot, room}, {routing->expert_pos, n_experts * 4 + 4}, {routing->token, room},
                {routing->counts, n_experts * 4}, {routing->lse, n_tokens * 4}, {routing->balance, 4}, {routing->routed, 4}}))
        return NACHO_ERR_INVALID_ARG;
    const RouteGradArgs a{logits, ldl, n_tokens, (int32_t)n_experts, normalise != 0, *routing, grad_gate, balance, grad, ldg};
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    profile_begin(s);
    if (launch_route_grad(dtype, a, s) != hipSuccess) return NACHO_ERR_HIP;
    profile_mark("route_grad");
    return NACHO_OK;
}

int32_t nacho_combine(const nacho_tensor *routing, const void *y, int64_t ldy, int64_t n, int32_t dtype,
                      const void *residual, int64_t ldr, void *out, int64_t ldo, void *hip_stream)
{
    CombineArgs a;
    const int32_t rc = check_combine(routing, n, dtype, &a);
    if (rc != NACHO_OK) return rc;
    const int64_t elem = value_bytes(dtype), slots = routing->lvl[1].extent, bytes = span(a.tokens, n, ldo, elem);
    if (!matrix(y, slots, n, ldy, elem) || !matrix(out, a.tokens, n, ldo, elem) || (residual && !matrix(residual, a.tokens, n, ldr, elem)))
        return NACHO_ERR_INVALID_ARG;
    const bool in_place = residual == out && ldr == ldo;
    const int64_t stored = routing->lvl[1].count * 4;
    if (!apart({{out, bytes}}, {{y, span(slots, n, ldy, elem)}, {in_place ? nullptr : residual, residual ? span(a.tokens, n, ldr, elem) : 0},
                                {a.pos, a.tokens * 4 + 4}, {a.slot, stored}, {a.gate, stored}}))
        return NACHO_ERR_INVALID_ARG;
    a.y = y;
    a.ldy = ldy;
    a.residual = residual;
    a.ldr = ldr;
    a.out = out;
    a.ldo = ldo;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    profile_begin(s);
    if (launch_combine(dtype, a, s) != hipSuccess) return NACHO_ERR_HIP;
    profile_mark("combine");
    return NACHO_OK;
}

int32_t nacho_combine_grad(const nacho_tensor *routing, const void *y, int64_t ldy, int64_t n, int32_t dtype,
                           const void *grad_out, int64_t ldg, void *grad_y, int64_t ldgy, float *grad_val, void *hip_stream)
{
    CombineArgs a;
    const int32_t rc = check_combine(routing, n, dtype, &a);
    if (rc != NACHO_OK) return rc;
    const int64_t elem = value_bytes(dtype), slots = routing->lvl[1].extent, bytes = span(slots, n, ldgy, elem);
    if (!aligned(grad_val, 4) || !matrix(grad_out, a.tokens, n, ldg, elem) || (grad_val && !matrix(y, slots, n, ldy, elem)))
        return NACHO_ERR_INVALID_ARG;
    if (grad_y && !matrix(grad_y, slots, n, ldgy, elem)) return NACHO_ERR_INVALID_ARG;
    const int64_t stored = routing->lvl[1].count * 4;
    // (y is read for grad_val alone)
    if (!apart({{grad_y, grad_y ? bytes : 0}, {grad_val, stored}},
               {{grad_out, span(a.tokens, n, ldg, elem)}, {grad_val ? y : nullptr, grad_val ? span(slots, n, ldy, elem) : 0},
                {a.pos, a.tokens * 4 + 4}, {a.slot, stored}, {a.gate, stored}}))
        return NACHO_ERR_INVALID_ARG;
    a.y = y;
    a.ldy = ldy;
    a.grad_out = grad_out;
    a.ldg = ldg;
    a.grad_y = grad_y;
    a.ldgy = ldgy;
    a.grad_gate = grad_val;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    profile_begin(s);
    if (launch_combine_grad(dtype, a, s) != hipSuccess) return NACHO_ERR_HIP;
    profile_mark("combine_grad");
    return NACHO_OK;
}

int32_t nacho_experts_workspace_bytes(const nacho_experts_layer *layer, size_t *bytes)
{
    if (!bytes) return NACHO_ERR_INVALID_ARG;
    const int32_t rc = check_layer(layer);
    if (rc == NACHO_OK) *bytes = carve_grad(nullptr, layer, layer->act != NACHO_ACT_NONE, true).bytes;
    return rc;
}

int32_t nacho_experts(const nacho_experts_layer *layer, void *y, int64_t ldy, void *pre, int64_t ldpre, void *hip_stream)
{
    const int32_t rc = check_layer(layer);
    if (rc != NACHO_OK) return rc;
    const nacho_experts_layer &l = *layer;
    const int64_t elem = value_bytes(l.dtype), bytes = span(l.n_slots, l.outer, ldy, elem);
    if (!check_x(layer, elem) || !check_w(layer, elem) || !matrix(y, l.n_slots, l.outer, ldy, elem)) return NACHO_ERR_INVALID_ARG;
    if (l.bias && !matrices(l.bias, l.n_experts, 1, l.outer, l.outer, l.bias_stride, elem)) return NACHO_ERR_INVALID_ARG;
    if (pre && !matrix(pre, l.n_slots, l.outer, ldpre, elem)) return NACHO_ERR_INVALID_ARG;
    if (!apart({{y, bytes}, {pre, pre ? span(l.n_slots, l.outer, ldpre, elem) : 0}},
               {x_of(layer, elem), w_of(layer, elem), bounds_of(layer), token_of(layer),
                {l.bias, l.bias ? span(l.n_experts, 1, l.outer, l.outer, l.bias_stride, elem) : 0}}))
        return NACHO_ERR_INVALID_ARG;
    const ProductArgs a{l.expert_pos, l.token, (int32_t)l.n_experts, 0, (int32_t)l.outer, (int32_t)l.inner, l.n_slots, l.x, l.w,
                        l.ldx, l.ldw, l.w_stride, y, ldy, 0, l.bias, l.bias_stride, pre, ldpre, l.act};
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    profile_begin(s);
    if (const hipError_t e = launch_experts_forward(l.dtype, a, s)) return e == hipErrorNotSupported ? NACHO_ERR_UNSUPPORTED : NACHO_ERR_HIP;
    profile_mark("experts");
    return NACHO_OK;
}

int32_t nacho_experts_grad(const nacho_experts_layer *layer, const void *grad_y, int64_t ldgy, const void *pre, int64_t ldpre,
                           void *grad_x, int64_t ldgx, void *grad_w, int64_t ldgw, int64_t gw_stride, void *grad_bias,
                           int64_t gb_stride, void *ws, size_t ws_bytes, void *hip_stream)
{
    const int32_t rc = check_layer(layer);
    if (rc != NACHO_OK) return rc;
    const nacho_experts_layer &l = *layer;
    const int64_t elem = value_bytes(l.dtype), gy_bytes = span(l.n_slots, l.outer, ldgy, elem);
    const bool slope = l.act != NACHO_ACT_NONE;
    if (!matrix(grad_y, l.n_slots, l.outer, ldgy, elem) || (slope && !matrix(pre, l.n_slots, l.outer, ldpre, elem)) ||
        (grad_x && !check_w(layer, elem)) || (grad_w && !check_x(layer, elem)))
        return NACHO_ERR_INVALID_ARG;
    const int64_t pre_bytes = slope ? span(l.n_slots, l.outer, ldpre, elem) : 0;
    const int64_t gx_bytes = grad_x ? span(l.n_slots, l.inner, ldgx, elem) : 0;
    const int64_t gw_bytes = grad_w ? span(l.n_experts, l.outer, l.inner, ldgw, gw_stride, elem) : 0;
    const int64_t gb_bytes = grad_bias ? span(l.n_experts, 1, l.outer, l.outer, gb_stride, elem) : 0;
    if ((grad_x && !matrix(grad_x, l.n_slots, l.inner, ldgx, elem)) ||
        (grad_w && !matrices(grad_w, l.n_experts, l.outer, l.inner, ldgw, gw_stride, elem)) ||
        (grad_bias && !matrices(grad_bias, l.n_experts, 1, l.outer, l.outer, gb_stride, elem)))
        return NACHO_ERR_INVALID_ARG;
    const bool products = grad_x || grad_w;
    const GradWs w = carve_grad(ws, layer, slope && products, grad_bias != nullptr);
    if (w.bytes > 0 && (!ws || ws_bytes < w.bytes || !aligned(ws, 16))) return NACHO_ERR_WORKSPACE;
    if (!apart({{grad_x, gx_bytes}, {grad_w, gw_bytes}, {grad_bias, gb_bytes}, {ws, (int64_t)w.bytes}},
               {x_of(layer, elem), w_of(layer, elem), bounds_of(layer), token_of(layer), {grad_y, gy_bytes}, {pre, pre_bytes}}))
        return NACHO_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    profile_begin(s);
    const void *gz = grad_y;
    int64_t ldgz = ldgy;
    if ((slope && products) || grad_bias) {
        SlopeArgs a{l.expert_pos, (int32_t)l.n_experts, (int32_t)l.outer, l.act, l.n_slots, grad_y, pre, ldgy, ldpre, nullptr, 0,
                    grad_bias, gb_stride, w.sums};
        if (slope && products) {
            gz = a.grad_z = w.grad_z;
            ldgz = a.ldgz = (l.outer + 7) / 8 * 8;
        }
        if (const hipError_t e = launch_experts_slope(l.dtype, a, s)) return e == hipErrorNotSupported ? NACHO_ERR_UNSUPPORTED : NACHO_ERR_HIP;
        profile_mark("experts_slope");
    }
    if (grad_x) {
        const ProductArgs a{l.expert_pos, nullptr, (int32_t)l.n_experts, 0, (int32_t)l.inner, (int32_t)l.outer, l.n_slots, gz, l.w,
                            ldgz, l.ldw, l.w_stride, grad_x, ldgx, 0, nullptr, 0, nullptr, 0, NACHO_ACT_NONE};
        if (const hipError_t e = launch_experts_rows(l.dtype, a, s)) return e == hipErrorNotSupported ? NACHO_ERR_UNSUPPORTED : NACHO_ERR_HIP;
        profile_mark("experts_rows");
    }
    if (grad_w) {
        const ProductArgs a{l.expert_pos, l.token, (int32_t)l.n_experts, (int32_t)l.outer, (int32_t)l.inner, 0, l.n_slots, gz, l.x,
                            ldgz, l.ldx, 0, grad_w, ldgw, gw_stride, nullptr, 0, nullptr, 0, NACHO_ACT_NONE};
        if (const hipError_t e = launch_experts_weights(l.dtype, a, s)) return e == hipErrorNotSupported ? NACHO_ERR_UNSUPPORTED : NACHO_ERR_HIP;
        profile_mark("experts_weights");
    }
    return NACHO_OK;
}

}  // extern "C"
