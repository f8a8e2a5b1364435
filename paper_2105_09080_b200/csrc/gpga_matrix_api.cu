// C entries of the matrix operators (gated feed-forward block, orthogonalisation): argument checks and launch parameters.
// See include/gpga.h.
#include <cmath>
#include <cstdio>
#include <initializer_list>

#include "../../include/gpga.h"
#include "gpga_ff.cuh"
#include "gpga_orth.cuh"
#include "gpga_token.cuh"

using namespace gpga;

namespace {

int32_t bad(const char* text) { return token_error(GPGA_ERR_INVALID_ARG, text); }

int32_t launched(cudaError_t e, const char* where)
{
    if (e == cudaSuccess) return GPGA_OK;
    (void)cudaGetLastError();   // reported here, not by the next call
    char text[256];
    std::snprintf(text, sizeof text, "%s: %s", where, cudaGetErrorString(e));
    return token_error(GPGA_ERR_CUDA, text);
}

int size_of(int64_t dtype) { return dtype == GPGA_DTYPE_F32 ? 4 : dtype == GPGA_DTYPE_BF16 || dtype == GPGA_DTYPE_F16 ? 2 : 0; }
bool element_aligned(const void* p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) == 0; }
bool on_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int64_t kMost = int64_t(1) << 20, kFar = int64_t(1) << 40;

struct Array {
    const void* p;
    int64_t ld, node, rows, cols;
    int size;
};
// nullptr, or what is wrong with a matrix per node: its rows must not overlap, nor its nodes where it is written.
const char* check(const Array& a, int64_t nodes, bool written)
{
    if (a.ld < a.cols || a.ld > kFar) return "strides: rows must not overlap";
    if (nodes > 1 && (a.node < 0 || a.node > kFar)) return "strides: node strides must not be negative";
    if (nodes > 1 && written && a.node < (a.rows - 1) * a.ld + a.cols) return "strides: the nodes of an output must not overlap";
    return nullptr;
}

const char* kSizes = "sizes: need 1 <= nodes <= 65535, rows >= 0, nodes * rows < 2^31, 1 <= d, f <= 2^20, nodes * d * f <= 2^40 and nodes * rows * max(d, f) <= 2^40";
const char* kAlign = "pointers must be aligned to their element";

const char* sizes(int64_t nodes, int64_t rows, int64_t d, int64_t f)
{
    if (nodes < 1 || nodes > 65535 || rows < 0 || rows >= (int64_t(1) << 31) || d < 1 || d > kMost || f < 1 || f > kMost) return kSizes;
    if (nodes * rows >= (int64_t(1) << 31)) return kSizes;
    const int64_t wide = d > f ? d : f;
    if (d * f > kFar / nodes || nodes * rows > kFar / wide) return kSizes;
    return nullptr;
}

const char* types(int64_t dtype, int64_t weight_dtype, int64_t activation)
{
    if (!size_of(dtype)) return "unknown dtype";
    if (weight_dtype != GPGA_DTYPE_F32 && weight_dtype != dtype) return "weights must be fp32 or of the activations' type";
    if (activation < GPGA_ACTIVATION_SILU || activation > GPGA_ACTIVATION_RELU) return "unknown activation";
    return nullptr;
}

Matrix matrix(const void* p, int64_t ld, int64_t node)
{
    Matrix m;
    m.p = const_cast<void*>(p);
    m.ld = ld;
    m.node = node;
    return m;
}

// The launch's parameters; nullptr, or what is wrong.
const char* forward_params(const gpga_feed_forward_forward_args_t* a, FeedForwardParams& q)
{
    if (const char* t = sizes(a->nodes, a->rows, a->d, a->f)) return t;
    if (const char* t = types(a->dtype, a->weight_dtype, a->activation)) return t;
    const int size = size_of(a->dtype), wsize = size_of(a->weight_dtype);
    if ((a->g != nullptr) != (a->u != nullptr)) return "g and u are kept together";
    const Array w[] = {{a->gate, a->ldgate, a->node_gate, a->f, a->d, wsize}, {a->up, a->ldup, a->node_up, a->f, a->d, wsize}, {a->down, a->lddown, a->node_down, a->d, a->f, wsize}};
    for (const Array& x : w) {
        if (const char* t = check(x, a->nodes, false)) return t;
        if (!element_aligned(x.p, x.size)) return kAlign;
    }
    const Array v[] = {{a->x, a->ldx, 0, a->rows, a->d, size}, {a->y, a->ldy, 0, a->rows, a->d, size},
                       {a->g, a->g ? a->ldg : a->f, 0, a->rows, a->f, size}, {a->u, a->u ? a->ldu : a->f, 0, a->rows, a->f, size}};
    for (const Array& x : v) {
        if (const char* t = check(x, 1, true)) return t;
        if (!element_aligned(x.p, x.size)) return kAlign;
    }
    q.x = matrix(a->x, a->ldx, a->rows * a->ldx);
    q.y = matrix(a->y, a->ldy, a->rows * a->ldy);
    q.g = matrix(a->g, a->ldg, a->rows * a->ldg);
    q.u = matrix(a->u, a->ldu, a->rows * a->ldu);
    q.gate = matrix(a->gate, a->ldgate, a->node_gate);
    q.up = matrix(a->up, a->ldup, a->node_up);
    q.down = matrix(a->down, a->lddown, a->node_down);
    q.nodes = a->nodes;
    q.rows = a->rows;
    q.d = a->d;
    q.f = a->f;
    q.dtype = (int)a->dtype;
    q.weight_dtype = (int)a->weight_dtype;
    q.activation = (int)a->activation;
    q.scratch = static_cast<char*>(a->scratch);
    return nullptr;
}

const char* backward_params(const gpga_feed_forward_backward_args_t* a, FeedForwardParams& q)
{
    if (const char* t = sizes(a->nodes, a->rows, a->d, a->f)) return t;
    if (const char* t = types(a->dtype, a->weight_dtype, a->activation)) return t;
    if (a->grad_dtype != GPGA_DTYPE_F32 && a->grad_dtype != a->dtype) return "weight gradients must be fp32 or of the activations' type";
    const int size = size_of(a->dtype), wsize = size_of(a->weight_dtype), gsize = size_of(a->grad_dtype);
    const Array w[] = {{a->gate, a->ldgate, a->node_gate, a->f, a->d, wsize}, {a->up, a->ldup, a->node_up, a->f, a->d, wsize}, {a->down, a->lddown, a->node_down, a->d, a->f, wsize}};
    for (const Array& x : w) {
        if (const char* t = check(x, a->nodes, false)) return t;
        if (!element_aligned(x.p, x.size)) return kAlign;
    }
    const Array g[] = {{a->dgate, a->lddgate, a->node_dgate, a->f, a->d, gsize}, {a->dup, a->lddup, a->node_dup, a->f, a->d, gsize},
                       {a->ddown, a->ldddown, a->node_ddown, a->d, a->f, gsize}};
    for (const Array& x : g) {
        if (const char* t = check(x, a->nodes, true)) return t;
        if (!element_aligned(x.p, x.size)) return kAlign;
        if (!x.p) return "NULL pointer";
    }
    const Array v[] = {{a->dy, a->lddy, 0, a->rows, a->d, size}, {a->x, a->ldx, 0, a->rows, a->d, size}, {a->g, a->ldg, 0, a->rows, a->f, size},
                       {a->u, a->ldu, 0, a->rows, a->f, size}, {a->dx, a->lddx, 0, a->rows, a->d, size}};
    for (const Array& x : v) {
        if (const char* t = check(x, 1, true)) return t;
        if (!element_aligned(x.p, x.size)) return kAlign;
        if (!x.p && a->rows) return "NULL pointer";
    }
    q.dy = matrix(a->dy, a->lddy, a->rows * a->lddy);
    q.x = matrix(a->x, a->ldx, a->rows * a->ldx);
    q.g = matrix(a->g, a->ldg, a->rows * a->ldg);
    q.u = matrix(a->u, a->ldu, a->rows * a->ldu);
    q.dx = matrix(a->dx, a->lddx, a->rows * a->lddx);
    q.gate = matrix(a->gate, a->ldgate, a->node_gate);
    q.up = matrix(a->up, a->ldup, a->node_up);
    q.down = matrix(a->down, a->lddown, a->node_down);
    q.dgate = matrix(a->dgate, a->lddgate, a->node_dgate);
    q.dup = matrix(a->dup, a->lddup, a->node_dup);
    q.ddown = matrix(a->ddown, a->ldddown, a->node_ddown);
    q.nodes = a->nodes;
    q.rows = a->rows;
    q.d = a->d;
    q.f = a->f;
    q.dtype = (int)a->dtype;
    q.weight_dtype = (int)a->weight_dtype;
    q.grad_dtype = (int)a->grad_dtype;
    q.activation = (int)a->activation;
    q.accumulate = a->accumulate != 0;
    q.scratch = static_cast<char*>(a->scratch);
    return nullptr;
}

const char* orth_params(const gpga_orthogonalize_args_t* a, OrthParams& q)
{
    const int size = size_of(a->dtype);
    if (!size) return "unknown dtype";
    if (a->nodes < 1 || a->nodes > 65535 || a->r < 1 || a->c < 1 || a->r > kMost || a->c > kMost || a->r * a->c > kFar / a->nodes)
        return "sizes: need 1 <= nodes <= 65535, 1 <= r, c <= 2^20, nodes * r * c <= 2^40";
    if (a->steps < 1 || a->steps > 1000) return "steps must lie in [1, 1000]";
    if (!(a->eps >= 0.0) || std::isinf(a->eps)) return "eps must be finite and not negative";
    for (double v : {a->c1, a->c3, a->c5, a->scale})
        if (!std::isfinite(v)) return "the coefficients and the scale must be finite";
    const Array in = {a->update, a->ldm, a->node_ldm, a->r, a->c, size}, out = {a->out, a->ldo, a->node_ldo, a->r, a->c, size};
    if (const char* t = check(in, a->nodes, false)) return t;
    if (const char* t = check(out, a->nodes, true)) return t;
    if (!element_aligned(a->update, size) || !element_aligned(a->out, size)) return kAlign;
    q.m = a->update;
    q.out = a->out;
    q.ldm = a->ldm;
    q.node_ldm = a->node_ldm;
    q.ldo = a->ldo;
    q.node_ldo = a->node_ldo;
    q.nodes = a->nodes;
    q.r = a->r;
    q.c = a->c;
    q.steps = a->steps;
    q.dtype = (int)a->dtype;
    q.accumulate = a->accumulate != 0;
    q.c1 = a->c1;
    q.c3 = a->c3;
    q.c5 = a->c5;
    q.scale = a->scale;
    q.eps = a->eps;
    q.scratch = static_cast<char*>(a->scratch);
    return nullptr;
}

const char* scratch_ok(const void* scratch, int64_t have, int64_t need)
{
    if (need && (!scratch || !on_16(scratch))) return "scratch must be 16-byte aligned";
    return have < need ? "scratch is too small: see the _scratch_bytes function" : nullptr;
}

}  // namespace

extern "C" {

int64_t gpga_feed_forward_forward_scratch_bytes(const gpga_feed_forward_forward_args_t* a)
{
    FeedForwardParams q;
    return a && !forward_params(a, q) ? ff_forward_scratch_bytes(q) : 0;
}

int32_t gpga_feed_forward_forward(const gpga_feed_forward_forward_args_t* a, void* stream)
{
    if (!a) return bad("NULL args");
    FeedForwardParams q;
    if (const char* t = forward_params(a, q)) return bad(t);
    if (a->rows == 0) return GPGA_OK;
    if (!a->x || !a->gate || !a->up || !a->down || !a->y) return bad("NULL pointer");
    if (const char* t = scratch_ok(a->scratch, a->scratch_bytes, ff_forward_scratch_bytes(q))) return bad(t);
    return launched(launch_ff_forward(q, static_cast<cudaStream_t>(stream)), "gpga_feed_forward_forward");
}

int64_t gpga_feed_forward_backward_scratch_bytes(const gpga_feed_forward_backward_args_t* a)
{
    FeedForwardParams q;
    return a && !backward_params(a, q) ? ff_backward_scratch_bytes(q) : 0;
}

int32_t gpga_feed_forward_backward(const gpga_feed_forward_backward_args_t* a, void* stream)
{
    if (!a) return bad("NULL args");
    FeedForwardParams q;
    if (const char* t = backward_params(a, q)) return bad(t);
    if (a->rows && (!a->gate || !a->up || !a->down)) return bad("NULL pointer");
    if (const char* t = scratch_ok(a->scratch, a->scratch_bytes, ff_backward_scratch_bytes(q))) return bad(t);
    return launched(launch_ff_backward(q, static_cast<cudaStream_t>(stream)), "gpga_feed_forward_backward");
}

int64_t gpga_orthogonalize_scratch_bytes(const gpga_orthogonalize_args_t* a)
{
    OrthParams q;
    return a && !orth_params(a, q) ? orth_scratch_bytes(q) : 0;
}

int32_t gpga_orthogonalize(const gpga_orthogonalize_args_t* a, void* stream)
{
    if (!a) return bad("NULL args");
    OrthParams q;
    if (const char* t = orth_params(a, q)) return bad(t);
    if (!a->update || !a->out) return bad("NULL pointer");
    if (const char* t = scratch_ok(a->scratch, a->scratch_bytes, orth_scratch_bytes(q))) return bad(t);
    return launched(launch_orth(q, static_cast<cudaStream_t>(stream)), "gpga_orthogonalize");
}

int32_t gpga_selftest_token_wait(void* stream)
{
    return launched(launch_wait_selftest(static_cast<cudaStream_t>(stream)), "gpga_selftest_token_wait");
}

int32_t gpga_token_status(void* stream)
{
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    unsigned int* const flags[] = {ff_forward_gave_up(), ff_backward_gave_up(), orth_gave_up()};
    unsigned int any = 0;
    for (unsigned int* f : flags) {
        if (!f) return launched(cudaErrorUnknown, "gpga_token_status");
        unsigned int v = 0;
        cudaError_t e = cudaMemcpyAsync(&v, f, sizeof v, cudaMemcpyDeviceToHost, s);
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
        if (e == cudaSuccess && v) e = cudaMemsetAsync(f, 0, sizeof v, s);
        if (e != cudaSuccess) return launched(e, "gpga_token_status");
        any |= v;
    }
    return any ? token_error(GPGA_ERR_TIMEOUT, "a bounded wait inside a matrix product gave up; its results are not valid") : GPGA_OK;
}

}  // extern "C"
