// C entries of the token-block operators: argument checks and launch parameters.  See include/gpga.h.
#include <cmath>
#include <cstdio>

#include "../../include/gpga.h"
#include "gpga_embed.cuh"
#include "gpga_norm.cuh"

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

bool sizes_ok(int64_t nodes, int64_t rows, int64_t d)
{
    if (nodes < 1 || nodes > 65535 || rows < 0 || rows >= (int64_t(1) << 31) || d < 1 || d > (int64_t(1) << 20)) return false;
    const int64_t chunks = (d + kChunk - 1) / kChunk;
    return nodes * rows < (int64_t(1) << 31) && rows * chunks < (int64_t(1) << 32) && nodes * rows * chunks <= (int64_t(1) << 38);
}

int size_of(int64_t dtype) { return dtype == GPGA_DTYPE_F32 ? 4 : dtype == GPGA_DTYPE_BF16 || dtype == GPGA_DTYPE_F16 ? 2 : 0; }

bool element_aligned(const void* p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) == 0; }

// Whether every row of an array that is there starts on 16 bytes.
bool vectors(const void* p, int64_t ld, int size) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * size) % 16 == 0); }

bool vocab_ok(int64_t vocab) { return vocab >= 1 && vocab < (int64_t(1) << 31); }

const char* kAlign = "pointers must be aligned to their element";
const char* kStrides = "strides must be at least d";
// Rows of several arrays that are all off the 16-byte alignment alike.
struct Alike {
    bool yes = true, any = false;
    uintptr_t base = 0, step = 0;
    void add(const void* p, int64_t ld, int size)
    {
        if (!p) return;
        const uintptr_t b = reinterpret_cast<uintptr_t>(p) & 15u, s = (uintptr_t)(ld * size) & 15u;
        if (any && (b != base || s != step)) yes = false;
        base = b, step = s, any = true;
    }
};

const char* kSizes = "sizes: need 1 <= nodes <= 65535, rows >= 0, 1 <= d <= 2^20 and the products stated in gpga.h";

// The dropout of a call; nullptr, or what is wrong with its arguments.
const char* drop_mask(DropMask& m, double p, uint64_t seed, int64_t k, int64_t site, int64_t node0, int64_t nodes)
{
    m = DropMask{};
    if (!(p >= 0.0 && p <= 1.0)) return "p must lie in [0, 1]";
    const uint32_t q = (uint32_t)std::floor(65536.0 * p + 0.5);
    m.on = q > 0;
    m.above = (uint32_t)((uint64_t)q * 65536u - 1u);
    m.scale = q < 65536u ? (float)(65536.0 / (65536.0 - q)) : 0.f;
    if (p == 0.0) return nullptr;
    if (k < 0 || k >= (int64_t(1) << 32)) return "k must lie in [0, 2^32)";
    if (site < 0 || site >= (int64_t(1) << 30)) return "site must lie in [0, 2^30)";
    if (node0 < 0 || node0 > (int64_t(1) << 32) - nodes) return "node0 + nodes must not pass 2^32";
    m.keys = make_philox_keys((uint32_t)(seed & 0xFFFFFFFFu), (uint32_t)(seed >> 32));
    m.node0 = (uint32_t)node0;
    m.k = (uint32_t)k;
    m.stream = (uint32_t)GPGA_STREAM_DROPOUT + (uint32_t)site;
    return nullptr;
}

}  // namespace

extern "C" {

int32_t gpga_embedding_forward(const gpga_embedding_forward_args_t* a, void* stream)
{
    if (!a) return bad("NULL args");
    const int size = size_of(a->dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(a->nodes, a->rows, a->d)) return bad(kSizes);
    if (!vocab_ok(a->vocab)) return bad("vocab must lie in [1, 2^31)");
    if (a->token_bytes != 4 && a->token_bytes != 8) return bad("tokens must have 4 or 8 bytes");
    if (a->ldt < a->d || a->ldo < a->d || (a->nodes > 1 && a->node_ldt < 0)) return bad("strides: ldt and ldo must be at least d");
    if (a->rows == 0) return GPGA_OK;
    if (!a->table || !a->tokens || !a->out) return bad("NULL pointer");
    if (!element_aligned(a->table, 4) || !element_aligned(a->tokens, (int)a->token_bytes) || !element_aligned(a->out, size))
        return bad(kAlign);
    LookupParams p;
    p.table = a->table;
    p.tokens = a->tokens;
    p.out = a->out;
    p.ldt = a->ldt;
    p.node_ldt = a->node_ldt;
    p.ldo = a->ldo;
    p.nodes = (uint32_t)a->nodes;
    p.rows = (uint32_t)a->rows;
    p.vocab = (uint32_t)a->vocab;
    p.d = (int32_t)a->d;
    p.tokens64 = a->token_bytes == 8;
    p.scale = (float)a->scale;
    return launched(launch_lookup(p, (int)a->dtype, static_cast<cudaStream_t>(stream)), "gpga_embedding_forward");
}

int64_t gpga_embedding_scratch_bytes(int64_t nodes, int64_t rows, int64_t d, int64_t vocab)
{
    return sizes_ok(nodes, rows, d) && vocab_ok(vocab) ? lookup_grad_scratch_bytes(nodes, rows, d, vocab) : 0;
}

int32_t gpga_embedding_backward(const gpga_embedding_backward_args_t* a, void* stream)
{
    if (!a) return bad("NULL args");
    const int size = size_of(a->dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(a->nodes, a->rows, a->d)) return bad(kSizes);
    if (!vocab_ok(a->vocab)) return bad("vocab must lie in [1, 2^31)");
    if (a->token_bytes != 4 && a->token_bytes != 8) return bad("tokens must have 4 or 8 bytes");
    // rows of grad must not overlap: each has one writer
    if (a->ldo < a->d || a->ldg < a->d || (a->nodes > 1 && a->node_ldg < (a->vocab - 1) * a->ldg + a->d))
        return bad("strides: ldo and ldg must be at least d, node_ldg at least a node's table");
    if (!a->grad || (a->rows && (!a->dout || !a->tokens))) return bad("NULL pointer");
    if (!element_aligned(a->grad, 4) || !element_aligned(a->dout, size) || !element_aligned(a->tokens, (int)a->token_bytes))
        return bad(kAlign);
    const int64_t need = lookup_grad_scratch_bytes(a->nodes, a->rows, a->d, a->vocab);
    if (need && (!a->scratch || (reinterpret_cast<uintptr_t>(a->scratch) & 15u))) return bad("scratch must be 16-byte aligned");
    if (a->scratch_bytes < need)
        return bad("scratch is too small: see gpga_embedding_scratch_bytes");
    if (a->rows == 0 && a->accumulate) return GPGA_OK;
    LookupGradParams p;
    p.dout = a->dout;
    p.tokens = a->tokens;
    p.grad = a->grad;
    p.ldo = a->ldo;
    p.ldg = a->ldg;
    p.node_ldg = a->node_ldg;
    p.nodes = (uint32_t)a->nodes;
    p.rows = (uint32_t)a->rows;
    p.vocab = (uint32_t)a->vocab;
    p.d = (int32_t)a->d;
    p.tokens64 = a->token_bytes == 8;
    p.accumulate = a->accumulate != 0;
    p.scale = (float)a->scale;
    p.scratch = static_cast<char*>(a->scratch);
    return launched(launch_lookup_grad(p, (int)a->dtype, static_cast<cudaStream_t>(stream)), "gpga_embedding_backward");
}

int32_t gpga_dropout(const gpga_dropout_args_t* a, void* stream)
{
    if (!a) return bad("NULL args");
    const int size = size_of(a->dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(a->nodes, a->rows, a->d)) return bad(kSizes);
    if (a->ldx < a->d || a->ldy < a->d) return bad(kStrides);
    DropoutParams q;
    if (const char* text = drop_mask(q.mask, a->p, a->seed, a->k, a->site, a->node0, a->nodes)) return bad(text);
    if (a->rows == 0) return GPGA_OK;
    if (!a->x || !a->y) return bad("NULL pointer");
    if (!element_aligned(a->x, size) || !element_aligned(a->y, size)) return bad(kAlign);
    q.x = a->x;
    q.y = a->y;
    q.ldx = a->ldx;
    q.ldy = a->ldy;
    q.nodes = (uint32_t)a->nodes;
    q.rows = (uint32_t)a->rows;
    q.d = (int32_t)a->d;
    const bool vec = a->d % kChunk == 0 && vectors(a->x, a->ldx, size) && vectors(a->y, a->ldy, size);
    Alike alike;
    alike.add(a->x, a->ldx, size);
    alike.add(a->y, a->ldy, size);
    q.shifted = alike.yes;
    return launched(launch_dropout(q, (int)a->dtype, vec, static_cast<cudaStream_t>(stream)), "gpga_dropout");
}

int32_t gpga_layer_norm_forward(const gpga_layer_norm_forward_args_t* a, void* stream)
{
    if (!a) return bad("NULL args");
    const int size = size_of(a->dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(a->nodes, a->rows, a->d)) return bad(kSizes);
    if (a->ldx < a->d || a->ldy < a->d || (a->residual && a->ldr < a->d) || (a->z && a->ldz < a->d)) return bad(kStrides);
    if (a->nodes > 1 && (a->weight || a->bias) && a->ldw < 0) return bad("ldw must not be negative");
    const float eps = (float)a->eps;
    if (!(eps >= 0.f) || std::isinf(eps)) return bad("eps must be finite and not negative");
    NormForwardParams q;
    if (const char* text = drop_mask(q.mask, a->p, a->seed, a->k, a->site, a->node0, a->nodes)) return bad(text);
    if (a->rows == 0) return GPGA_OK;
    if (!a->x || !a->y || !a->mean || !a->rstd) return bad("NULL pointer");
    if (!element_aligned(a->x, size) || !element_aligned(a->residual, size) || !element_aligned(a->y, size) ||
        !element_aligned(a->z, size) || !element_aligned(a->weight, 4) || !element_aligned(a->bias, 4) ||
        !element_aligned(a->mean, 4) || !element_aligned(a->rstd, 4))
        return bad(kAlign);
    q.x = a->x;
    q.residual = a->residual;
    q.weight = a->weight;
    q.bias = a->bias;
    q.y = a->y;
    q.z = a->z;
    q.mean = a->mean;
    q.rstd = a->rstd;
    q.ldx = a->ldx;
    q.ldr = a->ldr;
    q.ldy = a->ldy;
    q.ldz = a->ldz;
    q.ldw = a->ldw;
    q.nodes = (uint32_t)a->nodes;
    q.rows = (uint32_t)a->rows;
    q.d = (int32_t)a->d;
    q.eps = eps;
    const bool full = a->d % kChunk == 0;
    q.wvec = full && vectors(a->weight, a->ldw, 4) && vectors(a->bias, a->ldw, 4);
    const bool vec = full && vectors(a->x, a->ldx, size) && vectors(a->residual, a->ldr, size) && vectors(a->y, a->ldy, size) &&
                     vectors(a->z, a->ldz, size);
    Alike alike;
    alike.add(a->x, a->ldx, size);
    alike.add(a->residual, a->ldr, size);
    alike.add(a->y, a->ldy, size);
    alike.add(a->z, a->ldz, size);
    q.shifted = alike.yes;
    return launched(launch_norm_forward(q, (int)a->dtype, vec, static_cast<cudaStream_t>(stream)), "gpga_layer_norm_forward");
}

int64_t gpga_layer_norm_scratch_bytes(int64_t nodes, int64_t rows, int64_t d)
{
    if (!sizes_ok(nodes, rows, d)) return 0;
    const int splits = norm_backward_splits(nodes, rows, d);
    return splits > 1 ? nodes * splits * 2 * d * 4 : 0;
}

int32_t gpga_layer_norm_backward(const gpga_layer_norm_backward_args_t* a, void* stream)
{
    if (!a) return bad("NULL args");
    const int size = size_of(a->dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(a->nodes, a->rows, a->d)) return bad(kSizes);
    if (a->lddy < a->d || a->ldz < a->d || (a->dz && a->lddz < a->d) || a->lddr < a->d || (a->dx && a->lddx < a->d))
        return bad(kStrides);
    if (a->nodes > 1 && a->weight && a->ldw < 0) return bad("ldw must not be negative");
    if (a->nodes > 1 && (a->dweight || a->dbias) && a->lddw < a->d) return bad("lddw must be at least d");
    NormBackwardParams q;
    if (const char* text = drop_mask(q.mask, a->p, a->seed, a->k, a->site, a->node0, a->nodes)) return bad(text);
    if ((a->p > 0.0) != (a->dx != nullptr) && (a->rows || a->p == 0.0)) return bad("dx is wanted exactly when p > 0");
    if (a->rows && (!a->dy || !a->z || !a->mean || !a->rstd || !a->dresidual)) return bad("NULL pointer");
    if (!element_aligned(a->dy, size) || !element_aligned(a->z, size) || !element_aligned(a->dz, size) ||
        !element_aligned(a->dresidual, size) || !element_aligned(a->dx, size) || !element_aligned(a->mean, 4) ||
        !element_aligned(a->rstd, 4) || !element_aligned(a->weight, 4) || !element_aligned(a->dweight, 4) ||
        !element_aligned(a->dbias, 4))
        return bad(kAlign);
    const int64_t need = gpga_layer_norm_scratch_bytes(a->nodes, a->rows, a->d);
    if (need && (!a->scratch || (reinterpret_cast<uintptr_t>(a->scratch) & 15u))) return bad("scratch must be 16-byte aligned");
    if (a->scratch_bytes < need) return bad("scratch is too small: see gpga_layer_norm_scratch_bytes");
    q.dy = a->dy;
    q.z = a->z;
    q.dz = a->dz;
    q.mean = a->mean;
    q.rstd = a->rstd;
    q.weight = a->weight;
    q.dres = a->dresidual;
    q.dx = a->dx;
    q.dweight = a->dweight;
    q.dbias = a->dbias;
    q.partial = static_cast<float*>(a->scratch);
    q.lddy = a->lddy;
    q.ldz = a->ldz;
    q.lddz = a->lddz;
    q.lddres = a->lddr;
    q.lddx = a->lddx;
    q.ldw = a->ldw;
    q.lddw = a->lddw;
    q.nodes = (uint32_t)a->nodes;
    q.rows = (uint32_t)a->rows;
    q.d = (int32_t)a->d;
    q.splits = norm_backward_splits(a->nodes, a->rows, a->d);
    q.accumulate = a->accumulate != 0;
    const bool full = a->d % kChunk == 0;
    q.wvec = full && vectors(a->weight, a->ldw, 4);
    const bool vec = full && vectors(a->dy, a->lddy, size) && vectors(a->z, a->ldz, size) && vectors(a->dz, a->lddz, size) &&
                     vectors(a->dresidual, a->lddr, size) && vectors(a->dx, a->lddx, size);
    Alike alike;
    alike.add(a->dy, a->lddy, size);
    alike.add(a->z, a->ldz, size);
    alike.add(a->dz, a->lddz, size);
    alike.add(a->dresidual, a->lddr, size);
    alike.add(a->dx, a->lddx, size);
    q.shifted = alike.yes;
    return launched(launch_norm_backward(q, (int)a->dtype, vec, static_cast<cudaStream_t>(stream)), "gpga_layer_norm_backward");
}

}  // extern "C"
