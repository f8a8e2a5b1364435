// Gated feed-forward block, forward: g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T per node.  See include/gpga.h.
#include "gpga_ff_device.cuh"

namespace gpga {

namespace {

struct ForwardPlan {
    PackPlan pack;
    Operand x, gate, up, down, h;
    float* sums;
    int64_t bytes;
};

ForwardPlan plan_forward(const FeedForwardParams& p)
{
    ForwardPlan q;
    const bool f32 = p.dtype == 0, wf32 = p.weight_dtype == 0;
    q.pack.base = p.scratch;
    q.pack.pieces = f32 ? 3 : 1;
    q.x = q.pack.operand(p.x.p, p.x.ld, p.rows * p.x.ld, p.rows, p.d, p.nodes, f32, false, q.pack.pieces);
    q.gate = q.pack.weights(p.gate.p, p.gate.ld, p.gate.node, p.f, p.d, p.nodes, wf32, false);
    q.up = q.pack.weights(p.up.p, p.up.ld, p.up.node, p.f, p.d, p.nodes, wf32, false);
    q.down = q.pack.weights(p.down.p, p.down.ld, p.down.node, p.d, p.f, p.nodes, wf32, false);
    q.h = q.pack.written(p.rows, p.f, p.nodes, false);
    const int64_t parts = f32 ? parts_bytes<3>(p.rows, p.d, p.f, p.nodes, 1, 3) : parts_bytes<1>(p.rows, p.d, p.f, p.nodes, 1, q.down.pieces);
    q.sums = reinterpret_cast<float*>(p.scratch + q.pack.scratch.take(parts));
    q.bytes = q.pack.scratch.bytes;
    return q;
}

template <class T>
cudaError_t forward(const FeedForwardParams& p, cudaStream_t stream)
{
    constexpr int P = PiecesOf<T>::count;
    using T16 = typename PiecesOf<T>::type;
    const ForwardPlan q = plan_forward(p);
    cudaError_t e = q.pack.launch<T16>(stream);
    if (e != cudaSuccess) return e;
    GemmPlan g;
    g.half = std::is_same<T16, __half>::value;
    g.batch = g.bmod = p.nodes;
    g.after = q.pack.jobs.count > 0;
    g.a[0] = q.x;
    g.b[0] = q.gate;
    g.b[1] = q.up;
    g.m = p.rows;
    g.n = p.f;
    g.k = p.d;
    GateUp<T> up;
    up.g = static_cast<T*>(p.g.p);
    up.u = static_cast<T*>(p.u.p);
    up.ldg = p.g.ld;
    up.ldu = p.u.ld;
    up.h = pieces_of<T16>(q.h);
    up.m = (int32_t)p.rows;
    up.kind = p.activation;
    up.keeps = p.g.p != nullptr;
    up.vec = !up.keeps || (rows_on_16(p.g.p, p.g.ld, p.nodes * p.rows, 0, 1, sizeof(T)) && rows_on_16(p.u.p, p.u.ld, p.nodes * p.rows, 0, 1, sizeof(T)));
    e = launch_gemm<P, T>(g, up, stream);
    if (e != cudaSuccess) return e;
    g.after = true;
    g.a[0] = q.h;
    g.b[0] = q.down;
    g.n = p.d;
    g.k = p.f;
    return store_product<T, P>(g, p.y, p.nodes * p.rows, nullptr, false, Exponents(), q.sums, stream);
}

// fp32 as pairs of fp16: no row of x, gate, up, h or down is summed over, so each has a power of two of its own.
struct PairsPlan {
    PackPlan in, between;
    Operand x, gate, up, down, h;
    float *hf, *sums;
    int64_t ldh, bytes;
    int8_t *of_x, *of_gate, *of_up, *of_down, *of_h;    // exponents
};

PairsPlan plan_pairs(const FeedForwardParams& p)
{
    PairsPlan q;
    q.in.base = q.between.base = p.scratch;
    q.in.pieces = q.between.pieces = 2;
    q.in.by_rows(std::min(p.d, p.f));
    q.between.by_rows(p.f);
    q.x = q.in.operand(p.x.p, p.x.ld, p.rows * p.x.ld, p.rows, p.d, p.nodes, true, false, 2);
    q.of_x = q.in.powers();
    q.gate = q.in.operand(p.gate.p, p.gate.ld, p.gate.node, p.f, p.d, p.nodes, true, false, 2);
    q.of_gate = q.in.powers();
    q.up = q.in.operand(p.up.p, p.up.ld, p.up.node, p.f, p.d, p.nodes, true, false, 2);
    q.of_up = q.in.powers();
    q.down = q.in.operand(p.down.p, p.down.ld, p.down.node, p.d, p.f, p.nodes, true, false, 2);
    q.of_down = q.in.powers();
    ScratchPlan& s = q.between.scratch;
    s = q.in.scratch;
    q.ldh = padded(p.f);
    q.hf = reinterpret_cast<float*>(p.scratch + s.take(p.nodes * p.rows * q.ldh * 4));
    q.h = q.between.operand(q.hf, q.ldh, p.rows * q.ldh, p.rows, p.f, p.nodes, true, false, 2);
    q.of_h = q.between.powers();
    q.sums = reinterpret_cast<float*>(p.scratch + s.take(parts_bytes<2>(p.rows, p.d, p.f, p.nodes, 1, 2)));
    q.bytes = s.bytes;
    return q;
}

cudaError_t forward_pairs(const FeedForwardParams& p, cudaStream_t stream)
{
    const PairsPlan q = plan_pairs(p);
    const int32_t nodes = (int32_t)p.nodes;
    cudaError_t e = q.in.launch_rows(false, nullptr, 0, stream);
    if (e != cudaSuccess) return e;
    GemmPlan g;
    g.half = true;
    g.batch = g.bmod = p.nodes;
    g.after = true;
    g.a[0] = q.x;
    g.b[0] = q.gate;
    g.b[1] = q.up;
    g.m = p.rows;
    g.n = p.f;
    g.k = p.d;
    GateUp<float, true> up;
    up.g = static_cast<float*>(p.g.p);
    up.u = static_cast<float*>(p.u.p);
    up.ldg = p.g.ld;
    up.ldu = p.u.ld;
    up.h = {q.hf, q.ldh, p.rows * q.ldh};
    up.of_g = {q.of_x, q.of_gate, padded(p.rows), padded(p.f), nodes};
    up.of_u = {q.of_x, q.of_up, padded(p.rows), padded(p.f), nodes};
    up.m = (int32_t)p.rows;
    up.kind = p.activation;
    up.keeps = p.g.p != nullptr;
    up.vec = !up.keeps || (rows_on_16(p.g.p, p.g.ld, p.nodes * p.rows, 0, 1, 4) && rows_on_16(p.u.p, p.u.ld, p.nodes * p.rows, 0, 1, 4));
    e = launch_gemm<2, float>(g, up, stream);
    if (e == cudaSuccess) e = q.between.launch_rows(true, nullptr, 0, stream);
    if (e != cudaSuccess) return e;
    g.a[0] = q.h;
    g.b[0] = q.down;
    g.n = p.d;
    g.k = p.f;
    return store_product<float, 2>(g, p.y, p.nodes * p.rows, nullptr, false, {q.of_h, q.of_down, padded(p.rows), padded(p.d), nodes}, q.sums, stream);
}

}  // namespace

unsigned int* ff_forward_gave_up()
{
    void* at = nullptr;
    return cudaGetSymbolAddress(&at, gave_up) == cudaSuccess ? static_cast<unsigned int*>(at) : nullptr;
}

int64_t ff_forward_scratch_bytes(const FeedForwardParams& p) 
{
    return !p.rows ? 0 : ff_few(p) ? ff_few_scratch_bytes(p) : ff_pairs(p, false) ? plan_pairs(p).bytes : plan_forward(p).bytes;
}

cudaError_t launch_ff_forward(const FeedForwardParams& p, cudaStream_t stream)
{
    if (ff_few(p)) return launch_ff_few(p, stream);
    if (ff_pairs(p, false)) return forward_pairs(p, stream);
    if (p.dtype == 0) return forward<float>(p, stream);
    if (p.dtype == 1) return forward<__nv_bfloat16>(p, stream);
    return forward<__half>(p, stream);
}

}  // namespace gpga
