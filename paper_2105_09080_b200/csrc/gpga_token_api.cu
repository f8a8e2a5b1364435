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

int size_of(int32_t dtype) { return dtype == GPGA_DTYPE_F32 ? 4 : dtype == GPGA_DTYPE_BF16 || dtype == GPGA_DTYPE_F16 ? 2 : 0; }

bool element_aligned(const void* p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) == 0; }

// Whether every row of an array that is there starts on 16 bytes.
bool vectors(const void* p, int64_t ld, int size) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * size) % 16 == 0); }

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

int32_t gpga_embedding_forward(const float* table_dev, int64_t ldt, int64_t node_ldt, const void* tokens_dev,
                               int32_t token_bytes, void* out_dev, int64_t ldo, int32_t dtype, int64_t nodes,
                               int64_t rows, int64_t d, int64_t vocab, float scale, void* stream)
{
    const int size = size_of(dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(nodes, rows, d)) return bad(kSizes);
    if (vocab < 1 || vocab >= (int64_t(1) << 31)) return bad("vocab must lie in [1, 2^31)");
    if (token_bytes != 4 && token_bytes != 8) return bad("tokens must have 4 or 8 bytes");
    if (ldt < d || ldo < d || (nodes > 1 && node_ldt < 0)) return bad("strides: ldt and ldo must be at least d");
    if (rows == 0) return GPGA_OK;
    if (!table_dev || !tokens_dev || !out_dev) return bad("NULL pointer");
    if (!element_aligned(table_dev, 4) || !element_aligned(tokens_dev, token_bytes) || !element_aligned(out_dev, size))
        return bad("pointers must be aligned to their element");
    LookupParams p;
    p.table = table_dev;
    p.tokens = tokens_dev;
    p.out = out_dev;
    p.ldt = ldt;
    p.node_ldt = node_ldt;
    p.ldo = ldo;
    p.nodes = (uint32_t)nodes;
    p.rows = (uint32_t)rows;
    p.vocab = (uint32_t)vocab;
    p.d = (int32_t)d;
    p.tokens64 = token_bytes == 8;
    p.scale = scale;
    return launched(launch_lookup(p, dtype, static_cast<cudaStream_t>(stream)), "gpga_embedding_forward");
}

int64_t gpga_embedding_scratch_bytes(int64_t nodes, int64_t rows, int64_t d, int64_t vocab)
{
    if (!sizes_ok(nodes, rows, d) || vocab < 1 || vocab >= (int64_t(1) << 31)) return 0;
    return lookup_grad_scratch_bytes(nodes, rows, d, vocab);
}

int32_t gpga_embedding_backward(const void* dout_dev, int64_t ldo, int32_t dtype, const void* tokens_dev,
                                int32_t token_bytes, float* grad_dev, int64_t ldg, int64_t node_ldg, int64_t nodes,
                                int64_t rows, int64_t d, int64_t vocab, float scale, int32_t accumulate,
                                void* scratch_dev, int64_t scratch_bytes, void* stream)
{
    const int size = size_of(dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(nodes, rows, d)) return bad(kSizes);
    if (vocab < 1 || vocab >= (int64_t(1) << 31)) return bad("vocab must lie in [1, 2^31)");
    if (token_bytes != 4 && token_bytes != 8) return bad("tokens must have 4 or 8 bytes");
    // rows of grad must not overlap: each has one writer
    if (ldo < d || ldg < d || (nodes > 1 && node_ldg < (vocab - 1) * ldg + d))
        return bad("strides: ldo and ldg must be at least d, node_ldg at least a node's table");
    if (!grad_dev || (rows && (!dout_dev || !tokens_dev))) return bad("NULL pointer");
    if (!element_aligned(grad_dev, 4) || !element_aligned(dout_dev, size) || !element_aligned(tokens_dev, token_bytes))
        return bad("pointers must be aligned to their element");
    if (!scratch_dev || (reinterpret_cast<uintptr_t>(scratch_dev) & 15u)) return bad("scratch must be 16-byte aligned");
    if (scratch_bytes < lookup_grad_scratch_bytes(nodes, rows, d, vocab)) return bad("scratch is too small: see gpga_embedding_scratch_bytes");
    if (rows == 0 && accumulate) return GPGA_OK;
    LookupGradParams p;
    p.dout = dout_dev;
    p.tokens = tokens_dev;
    p.grad = grad_dev;
    p.ldo = ldo;
    p.ldg = ldg;
    p.node_ldg = node_ldg;
    p.nodes = (uint32_t)nodes;
    p.rows = (uint32_t)rows;
    p.vocab = (uint32_t)vocab;
    p.d = (int32_t)d;
    p.tokens64 = token_bytes == 8;
    p.accumulate = accumulate != 0;
    p.scale = scale;
    p.scratch = static_cast<char*>(scratch_dev);
    return launched(launch_lookup_grad(p, dtype, static_cast<cudaStream_t>(stream)), "gpga_embedding_backward");
}

int32_t gpga_dropout(const void* x_dev, int64_t ldx, void* y_dev, int64_t ldy, int32_t dtype, int64_t nodes,
                     int64_t rows, int64_t d, double p, uint64_t seed, int64_t k, int64_t site, int64_t node0,
                     void* stream)
{
    const int size = size_of(dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(nodes, rows, d)) return bad(kSizes);
    if (ldx < d || ldy < d) return bad("strides must be at least d");
    DropoutParams q;
    if (const char* text = drop_mask(q.mask, p, seed, k, site, node0, nodes)) return bad(text);
    if (rows == 0) return GPGA_OK;
    if (!x_dev || !y_dev) return bad("NULL pointer");
    if (!element_aligned(x_dev, size) || !element_aligned(y_dev, size)) return bad("pointers must be aligned to their element");
    q.x = x_dev;
    q.y = y_dev;
    q.ldx = ldx;
    q.ldy = ldy;
    q.nodes = (uint32_t)nodes;
    q.rows = (uint32_t)rows;
    q.d = (int32_t)d;
    const bool vec = d % kChunk == 0 && vectors(x_dev, ldx, size) && vectors(y_dev, ldy, size);
    return launched(launch_dropout(q, dtype, vec, static_cast<cudaStream_t>(stream)), "gpga_dropout");
}

int32_t gpga_layer_norm_forward(const void* x_dev, int64_t ldx, const void* residual_dev, int64_t ldr,
                                const float* weight_dev, const float* bias_dev, int64_t ldw, void* y_dev, int64_t ldy,
                                void* z_dev, int64_t ldz, float* mean_dev, float* rstd_dev, int32_t dtype,
                                int64_t nodes, int64_t rows, int64_t d, float eps, double p, uint64_t seed, int64_t k,
                                int64_t site, int64_t node0, void* stream)
{
    const int size = size_of(dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(nodes, rows, d)) return bad(kSizes);
    if (ldx < d || ldy < d || (residual_dev && ldr < d) || (z_dev && ldz < d)) return bad("strides must be at least d");
    if (nodes > 1 && (weight_dev || bias_dev) && ldw < 0) return bad("ldw must not be negative");
    if (!(eps >= 0.f) || std::isinf(eps)) return bad("eps must be finite and not negative");
    NormForwardParams q;
    if (const char* text = drop_mask(q.mask, p, seed, k, site, node0, nodes)) return bad(text);
    if (rows == 0) return GPGA_OK;
    if (!x_dev || !y_dev || !mean_dev || !rstd_dev) return bad("NULL pointer");
    if (!element_aligned(x_dev, size) || !element_aligned(residual_dev, size) || !element_aligned(y_dev, size) ||
        !element_aligned(z_dev, size) || !element_aligned(weight_dev, 4) || !element_aligned(bias_dev, 4) ||
        !element_aligned(mean_dev, 4) || !element_aligned(rstd_dev, 4))
        return bad("pointers must be aligned to their element");
    q.x = x_dev;
    q.residual = residual_dev;
    q.weight = weight_dev;
    q.bias = bias_dev;
    q.y = y_dev;
    q.z = z_dev;
    q.mean = mean_dev;
    q.rstd = rstd_dev;
    q.ldx = ldx;
    q.ldr = ldr;
    q.ldy = ldy;
    q.ldz = ldz;
    q.ldw = ldw;
    q.nodes = (uint32_t)nodes;
    q.rows = (uint32_t)rows;
    q.d = (int32_t)d;
    q.eps = eps;
    const bool full = d % kChunk == 0;
    q.wvec = full && vectors(weight_dev, ldw, 4) && vectors(bias_dev, ldw, 4);
    const bool vec = full && vectors(x_dev, ldx, size) && vectors(residual_dev, ldr, size) && vectors(y_dev, ldy, size) &&
                     vectors(z_dev, ldz, size);
    return launched(launch_norm_forward(q, dtype, vec, static_cast<cudaStream_t>(stream)), "gpga_layer_norm_forward");
}

int64_t gpga_layer_norm_scratch_bytes(int64_t nodes, int64_t rows, int64_t d)
{
    if (!sizes_ok(nodes, rows, d)) return 0;
    const int splits = norm_backward_splits(nodes, rows, d);
    return splits > 1 ? nodes * splits * 2 * d * 4 : 0;
}

int32_t gpga_layer_norm_backward(const void* dy_dev, int64_t lddy, const void* z_dev, int64_t ldz, const void* dz_dev,
                                 int64_t lddz, const float* mean_dev, const float* rstd_dev, const float* weight_dev,
                                 int64_t ldw, void* dresidual_dev, int64_t lddr, void* dx_dev, int64_t lddx,
                                 float* dweight_dev, float* dbias_dev, int64_t lddw, int32_t accumulate, int32_t dtype,
                                 int64_t nodes, int64_t rows, int64_t d, double p, uint64_t seed, int64_t k,
                                 int64_t site, int64_t node0, void* scratch_dev, int64_t scratch_bytes, void* stream)
{
    const int size = size_of(dtype);
    if (!size) return bad("unknown dtype");
    if (!sizes_ok(nodes, rows, d)) return bad(kSizes);
    if (lddy < d || ldz < d || (dz_dev && lddz < d) || lddr < d || (dx_dev && lddx < d)) return bad("strides must be at least d");
    if (nodes > 1 && weight_dev && ldw < 0) return bad("ldw must not be negative");
    if (nodes > 1 && (dweight_dev || dbias_dev) && lddw < d) return bad("lddw must be at least d");
    NormBackwardParams q;
    if (const char* text = drop_mask(q.mask, p, seed, k, site, node0, nodes)) return bad(text);
    if ((p > 0.0) != (dx_dev != nullptr) && (rows || p == 0.0)) return bad("dx is wanted exactly when p > 0");
    if (rows && (!dy_dev || !z_dev || !mean_dev || !rstd_dev || !dresidual_dev)) return bad("NULL pointer");
    if (!element_aligned(dy_dev, size) || !element_aligned(z_dev, size) || !element_aligned(dz_dev, size) ||
        !element_aligned(dresidual_dev, size) || !element_aligned(dx_dev, size) || !element_aligned(mean_dev, 4) ||
        !element_aligned(rstd_dev, 4) || !element_aligned(weight_dev, 4) || !element_aligned(dweight_dev, 4) ||
        !element_aligned(dbias_dev, 4))
        return bad("pointers must be aligned to their element");
    const int64_t need = gpga_layer_norm_scratch_bytes(nodes, rows, d);
    if (need && (!scratch_dev || (reinterpret_cast<uintptr_t>(scratch_dev) & 15u))) return bad("scratch must be 16-byte aligned");
    if (scratch_bytes < need) return bad("scratch is too small: see gpga_layer_norm_scratch_bytes");
    q.dy = dy_dev;
    q.z = z_dev;
    q.dz = dz_dev;
    q.mean = mean_dev;
    q.rstd = rstd_dev;
    q.weight = weight_dev;
    q.dres = dresidual_dev;
    q.dx = dx_dev;
    q.dweight = dweight_dev;
    q.dbias = dbias_dev;
    q.partial = static_cast<float*>(scratch_dev);
    q.lddy = lddy;
    q.ldz = ldz;
    q.lddz = lddz;
    q.lddres = lddr;
    q.lddx = lddx;
    q.ldw = ldw;
    q.lddw = lddw;
    q.nodes = (uint32_t)nodes;
    q.rows = (uint32_t)rows;
    q.d = (int32_t)d;
    q.splits = norm_backward_splits(nodes, rows, d);
    q.accumulate = accumulate != 0;
    const bool full = d % kChunk == 0;
    q.wvec = full && vectors(weight_dev, ldw, 4);
    const bool vec = full && vectors(dy_dev, lddy, size) && vectors(z_dev, ldz, size) && vectors(dz_dev, lddz, size) &&
                     vectors(dresidual_dev, lddr, size) && vectors(dx_dev, lddx, size);
    return launched(launch_norm_backward(q, dtype, vec, static_cast<cudaStream_t>(stream)), "gpga_layer_norm_backward");
}

}  // extern "C"
