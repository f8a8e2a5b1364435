// Gated feed-forward block, backward.  Five products per node and three arrays between them; see include/gpga.h.
#include "gpga_ff_device.cuh"

namespace gpga {

namespace {

struct BackwardPlan {
    PackPlan pack;
    Operand x, dy, gate, up, down, h, dgu;
    float* sums;
    int64_t bytes;
};

// Room for the parts of the three products behind dh (store_product).
template <int P>
int64_t all_parts_bytes(const FeedForwardParams& p, int64_t weight_pieces)
{
    return std::max({parts_bytes<P>(p.d, p.f, p.rows, p.nodes, 1, P), parts_bytes<P>(p.f, p.d, p.rows, 2 * p.nodes, 1, P),
                     parts_bytes<P>(p.rows, p.d, p.f, p.nodes, 2, weight_pieces)});
}

BackwardPlan plan_backward(const FeedForwardParams& p)
{
    BackwardPlan q;
    const bool f32 = p.dtype == 0, wf32 = p.weight_dtype == 0;
    q.pack.base = p.scratch;
    q.pack.pieces = f32 ? 3 : 1;
    q.dy = q.pack.operand(p.dy.p, p.dy.ld, p.rows * p.dy.ld, p.rows, p.d, p.nodes, f32, false, q.pack.pieces);
    q.down = q.pack.weights(p.down.p, p.down.ld, p.down.node, p.d, p.f, p.nodes, wf32, true);
    q.x = q.pack.operand(p.x.p, p.x.ld, p.rows * p.x.ld, p.rows, p.d, p.nodes, f32, true, q.pack.pieces);
    q.gate = q.pack.weights(p.gate.p, p.gate.ld, p.gate.node, p.f, p.d, p.nodes, wf32, true);
    q.up = q.pack.weights(p.up.p, p.up.ld, p.up.node, p.f, p.d, p.nodes, wf32, true);
    q.h = q.pack.written(p.rows, p.f, p.nodes, true);
    q.dgu = q.pack.written(p.rows, p.f, 2 * p.nodes, true);   // dg of all nodes, then du
    const int64_t parts = f32 ? all_parts_bytes<3>(p, 3) : all_parts_bytes<1>(p, q.gate.pieces);
    q.sums = reinterpret_cast<float*>(p.scratch + q.pack.scratch.take(parts));
    q.bytes = q.pack.scratch.bytes;
    return q;
}

template <class T>
cudaError_t weight_gradient(const GemmPlan& g, const FeedForwardParams& p, const Matrix& out, int64_t rows, const Matrix* second, float* sums, cudaStream_t stream)
{
    constexpr int P = PiecesOf<T>::count;
    if (p.grad_dtype == 0) return store_product<float, P>(g, out, rows, second, p.accumulate, Exponents(), sums, stream);
    if constexpr (P == 1) return store_product<T, P>(g, out, rows, second, p.accumulate, Exponents(), sums, stream);
    return cudaErrorInvalidValue;
}

template <class T>
cudaError_t backward(const FeedForwardParams& p, cudaStream_t stream)
{
    constexpr int P = PiecesOf<T>::count;
    using T16 = typename PiecesOf<T>::type;
    const BackwardPlan q = plan_backward(p);
    cudaError_t e = q.pack.launch<T16>(stream);
    if (e != cudaSuccess) return e;
    Operand dg = q.dgu, du = q.dgu;    // halves of one array
    dg.batches = du.batches = p.nodes;
    du.base = static_cast<const T16*>(du.base) + p.nodes * du.batch;

    GemmPlan g;                         // dh = dy Wd, and from it h, dg, du
    g.half = std::is_same<T16, __half>::value;
    g.batch = g.bmod = p.nodes;
    g.after = q.pack.jobs.count > 0;
    g.a[0] = q.dy;
    g.b[0] = q.down;
    g.m = p.rows;
    g.n = p.f;
    g.k = p.d;
    GateGrad<T> grad;
    grad.g = static_cast<const T*>(p.g.p);
    grad.u = static_cast<const T*>(p.u.p);
    grad.ldg = p.g.ld;
    grad.ldu = p.u.ld;
    grad.h = pieces_of<T16>(q.h);
    grad.dg = pieces_of<T16>(dg);
    grad.du = pieces_of<T16>(du);
    grad.m = (int32_t)p.rows;
    grad.kind = p.activation;
    grad.vec = rows_on_16(p.g.p, p.g.ld, p.nodes * p.rows, 0, 1, sizeof(T)) && rows_on_16(p.u.p, p.u.ld, p.nodes * p.rows, 0, 1, sizeof(T));
    if ((e = launch_gemm<P>(g, grad, stream)) != cudaSuccess) return e;

    g.after = true;                     // dWd = dy^T h
    g.a[0] = q.dy;
    g.a[0].mn_major = true;
    g.b[0] = q.h;
    g.m = p.d;
    g.n = p.f;
    g.k = p.rows;
    if ((e = weight_gradient<T>(g, p, p.ddown, p.d, nullptr, q.sums, stream)) != cudaSuccess) return e;

    g.a[0] = q.dgu;                     // dWg = dg^T x, dWu = du^T x
    g.b[0] = q.x;
    g.m = p.f;
    g.n = p.d;
    g.batch = 2 * p.nodes;
    if ((e = weight_gradient<T>(g, p, p.dgate, p.f, &p.dup, q.sums, stream)) != cudaSuccess) return e;

    g.pairs = 2;                        // dx = dg Wg + du Wu, last: it may take dy's or x's place
    g.batch = p.nodes;
    g.a[0] = dg;
    g.a[1] = du;
    g.a[0].mn_major = g.a[1].mn_major = false;
    g.b[0] = q.gate;
    g.b[1] = q.up;
    g.m = p.rows;
    g.n = p.d;
    g.k = p.f;
    return store_product<T, P>(g, p.dx, p.nodes * p.rows, nullptr, false, Exponents(), q.sums, stream);
}

// fp32 as pairs of fp16.  What follows dh is not its product's epilogue: a tile's sums take the registers of its few warps, which
// then wait for g and u and for the activation.  Two passes with all warps take less: one for the largest values of h, and of dg
// and du, one that makes their pieces (2048 x 2048 values: product 46 us with h, dg, du as fp32 and 18 us for their pieces).
struct PairsPlan {
    PackPlan in;
    Operand x, dy, gate, up, down, h, dgu;
    float *dh, *sums;
    int64_t ldh, bytes;
    uint32_t *parts, *peaks;     // of dy, down, x, gate, up (kPeakParts each); of h, of dg and du
    int32_t* exponents;          // of dy, down, x, gate and up, up again, h, dg and du
};

PairsPlan plan_pairs(const FeedForwardParams& p)
{
    PairsPlan q;
    q.in.base = p.scratch;
    q.in.pieces = 2;
    ScratchPlan& s = q.in.scratch;
    q.parts = reinterpret_cast<uint32_t*>(p.scratch + s.take(5 * kPeakParts * 4));
    q.peaks = reinterpret_cast<uint32_t*>(p.scratch + s.take(8));
    q.exponents = reinterpret_cast<int32_t*>(p.scratch + s.take(7 * 4));
    q.dy = q.in.operand(p.dy.p, p.dy.ld, p.rows * p.dy.ld, p.rows, p.d, p.nodes, true, false, 2);
    q.in.scaled(q.parts, kPeakParts, q.exponents);
    q.down = q.in.operand(p.down.p, p.down.ld, p.down.node, p.d, p.f, p.nodes, true, true, 2);
    q.in.scaled(q.parts + kPeakParts, kPeakParts, q.exponents + 1);
    q.x = q.in.operand(p.x.p, p.x.ld, p.rows * p.x.ld, p.rows, p.d, p.nodes, true, true, 2);
    q.in.scaled(q.parts + 2 * kPeakParts, kPeakParts, q.exponents + 2);
    q.gate = q.in.operand(p.gate.p, p.gate.ld, p.gate.node, p.f, p.d, p.nodes, true, true, 2);
    q.in.scaled(q.parts + 3 * kPeakParts, 2 * kPeakParts, q.exponents + 3);   // one power for both: their products are one sum
    q.up = q.in.operand(p.up.p, p.up.ld, p.up.node, p.f, p.d, p.nodes, true, true, 2);
    q.in.scaled(q.parts + 3 * kPeakParts, 2 * kPeakParts, q.exponents + 4);
    q.ldh = (p.f + 7) / 8 * 8;
    q.dh = reinterpret_cast<float*>(p.scratch + s.take(p.nodes * p.rows * q.ldh * 4));
    q.h = q.in.written(p.rows, p.f, p.nodes, true);
    q.dgu = q.in.written(p.rows, p.f, 2 * p.nodes, true);   // dg of all nodes, then du
    const int64_t parts = std::max(parts_bytes<2>(p.rows, p.f, p.d, p.nodes, 1, 2), all_parts_bytes<2>(p, 2));
    q.sums = reinterpret_cast<float*>(p.scratch + s.take(parts));
    q.bytes = s.bytes;
    return q;
}

struct SlopeParams {
    const float *g, *u, *dh;
    int64_t ldg, ldu, ldh;
    int64_t chunks;           // of eight columns, all rows
    int32_t f, kind, vec;
    Pieces<__half> h, dg, du;
    uint32_t* peaks;          // of h; of dg and du
    int32_t* exponents;
};

// PACK: the pieces of h, dg and du; otherwise their largest values.  Bound by memory (12 bytes read per value, 12 written).
template <bool PACK>
__global__ void __launch_bounds__(256) slopes_kernel(const __grid_constant__ SlopeParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    float scale[2] = {1.f, 1.f};
    if constexpr (PACK)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = scale_exponent(p.peaks[i]);
            scale[i] = __int_as_float((e + 127) << 23);
            if (blockIdx.x == 0 && threadIdx.x == 0) p.exponents[i] = -e;
        }
    const int per = (int)(p.ldh / 8);
    uint32_t peak[2] = {0, 0};
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.chunks; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per;
        const int col = (int)(i - row * per) * 8, left = min(8, p.f - col);
        Raw<float> rg, ru, rd;
        rg.load(p.g + row * p.ldg + col, left, p.vec);
        ru.load(p.u + row * p.ldu + col, left, p.vec);
        rd.load(p.dh + row * p.ldh + col, left, true);
        float v[8], w[8], dh[8], dg[8];
        rg.values(v);
        ru.values(w);
        rd.values(dh);
        block_slopes<false>(v, w, dh, dg, p.kind);
        if constexpr (PACK) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= scale[0], dg[k] *= scale[1], dh[k] *= scale[1];
            p.h.store_at<2>(i * 8, v);
            p.dg.store_at<2>(i * 8, dg);
            p.du.store_at<2>(i * 8, dh);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) {
                    peak[0] = max(peak[0], finite_bits(v[k]));
                    peak[1] = max(peak[1], max(finite_bits(dg[k]), finite_bits(dh[k])));
                }
        }
    }
    if constexpr (!PACK)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            peak[i] = __reduce_max_sync(~0u, peak[i]);
            if ((threadIdx.x & 31) == 0 && peak[i] > *reinterpret_cast<volatile uint32_t*>(p.peaks + i)) atomicMax(p.peaks + i, peak[i]);
        }
}

cudaError_t backward_pairs(const FeedForwardParams& p, cudaStream_t stream)
{
    const PairsPlan q = plan_pairs(p);
    cudaError_t e = q.in.launch_peaks(q.parts, q.peaks, stream);
    if (e == cudaSuccess) e = q.in.launch<__half>(stream);
    if (e != cudaSuccess) return e;
    GemmPlan g;
    g.half = true;
    g.batch = g.bmod = p.nodes;
    g.after = true;
    g.a[0] = q.dy;
    g.b[0] = q.down;
    g.m = p.rows;
    g.n = p.f;
    g.k = p.d;
    const Matrix dh{q.dh, q.ldh, p.rows * q.ldh};
    e = store_product<float, 2>(g, dh, p.nodes * p.rows, nullptr, false, {q.exponents, q.exponents + 1}, q.sums, stream);
    if (e != cudaSuccess) return e;
    Operand dg = q.dgu, du = q.dgu;     // halves of one array
    dg.batches = du.batches = p.nodes;
    du.base = static_cast<const __half*>(du.base) + p.nodes * du.batch;
    SlopeParams s;
    s.g = static_cast<const float*>(p.g.p);
    s.u = static_cast<const float*>(p.u.p);
    s.dh = q.dh;
    s.ldg = p.g.ld;
    s.ldu = p.u.ld;
    s.ldh = q.ldh;
    s.chunks = p.nodes * p.rows * (q.ldh / 8);
    s.f = (int32_t)p.f;
    s.kind = p.activation;
    s.vec = rows_on_16(p.g.p, p.g.ld, p.nodes * p.rows, 0, 1, 4) && rows_on_16(p.u.p, p.u.ld, p.nodes * p.rows, 0, 1, 4);
    s.h = pieces_of<__half>(q.h);
    s.dg = pieces_of<__half>(dg);
    s.du = pieces_of<__half>(du);
    s.peaks = q.peaks;
    s.exponents = q.exponents + 5;
    const dim3 blocks((unsigned)std::min<int64_t>((s.chunks + 255) / 256, (int64_t)sm_count() * 8));
    e = launch_after_trigger(slopes_kernel<false>, blocks, dim3(256), 0, stream, true, s);
    if (e == cudaSuccess) e = launch_after_trigger(slopes_kernel<true>, blocks, dim3(256), 0, stream, true, s);
    if (e != cudaSuccess) return e;

    g.a[0] = q.dy;                      // dWd
    g.a[0].mn_major = true;
    g.b[0] = q.h;
    g.m = p.d;
    g.n = p.f;
    g.k = p.rows;
    if ((e = store_product<float, 2>(g, p.ddown, p.d, nullptr, p.accumulate, {q.exponents, q.exponents + 5}, q.sums, stream)) != cudaSuccess) return e;
    g.a[0] = q.dgu;                     // dWg, dWu
    g.b[0] = q.x;
    g.m = p.f;
    g.n = p.d;
    g.batch = 2 * p.nodes;
    if ((e = store_product<float, 2>(g, p.dgate, p.f, &p.dup, p.accumulate, {q.exponents + 6, q.exponents + 2}, q.sums, stream)) != cudaSuccess) return e;
    g.pairs = 2;                        // dx
    g.batch = p.nodes;
    g.a[0] = dg;
    g.a[1] = du;
    g.a[0].mn_major = g.a[1].mn_major = false;
    g.b[0] = q.gate;
    g.b[1] = q.up;
    g.m = p.rows;
    g.n = p.d;
    g.k = p.f;
    return store_product<float, 2>(g, p.dx, p.nodes * p.rows, nullptr, false, {q.exponents + 6, q.exponents + 3}, q.sums, stream);
}

template <class T>
__global__ void zero_rows(T* p, int64_t ld, int64_t node, int64_t rows, int64_t cols, int64_t count)
{
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t r = i / cols, b = r / rows;
        p[b * node + (r - b * rows) * ld + (i - r * cols)] = from_f32<T>(0.f);
    }
}

// A sum over no tokens.
cudaError_t no_tokens(const FeedForwardParams& p, cudaStream_t stream)
{
    if (p.accumulate) return cudaSuccess;
    const Matrix* out[3] = {&p.dgate, &p.dup, &p.ddown};
    for (int i = 0; i < 3; ++i) {
        const int64_t rows = i == 2 ? p.d : p.f, cols = i == 2 ? p.f : p.d, count = p.nodes * rows * cols;
        const unsigned blocks = (unsigned)std::min<int64_t>((count + 255) / 256, (int64_t)sm_count() * 8);
        if (p.grad_dtype == 0)
            zero_rows<<<blocks, 256, 0, stream>>>(static_cast<float*>(out[i]->p), out[i]->ld, out[i]->node, rows, cols, count);
        else if (p.grad_dtype == 1)
            zero_rows<<<blocks, 256, 0, stream>>>(static_cast<__nv_bfloat16*>(out[i]->p), out[i]->ld, out[i]->node, rows, cols, count);
        else
            zero_rows<<<blocks, 256, 0, stream>>>(static_cast<__half*>(out[i]->p), out[i]->ld, out[i]->node, rows, cols, count);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

unsigned int* ff_backward_gave_up()
{
    void* at = nullptr;
    return cudaGetSymbolAddress(&at, gave_up) == cudaSuccess ? static_cast<unsigned int*>(at) : nullptr;
}

int64_t ff_backward_scratch_bytes(const FeedForwardParams& p) { return !p.rows ? 0 : ff_pairs(p, true) ? plan_pairs(p).bytes : plan_backward(p).bytes; }

cudaError_t launch_ff_backward(const FeedForwardParams& p, cudaStream_t stream)
{
    if (p.rows == 0) return no_tokens(p, stream);
    if (ff_pairs(p, true)) return backward_pairs(p, stream);
    if (p.dtype == 0) return backward<float>(p, stream);
    if (p.dtype == 1) return backward<__nv_bfloat16>(p, stream);
    return backward<__half>(p, stream);
}

}  // namespace gpga
