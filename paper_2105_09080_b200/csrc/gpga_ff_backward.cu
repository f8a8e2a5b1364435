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
    if ((e = launch_gemm<P, T>(g, grad, stream)) != cudaSuccess) return e;

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
// then wait for g and u and for the activation.  Two passes with all warps take less: one for the largest values of h, dg
// and du, one that makes their pieces.
// A power of two belongs to a row where the product sums over columns (dy in dh, dg and du in dx), to a column where it sums over
// rows or the matrix is one of weights.  So dy, dg and du are packed both ways.
struct PairsPlan {
    PackPlan rows, columns;
    Operand dy, dyc, x, gate, up, down, h, dgu, dgur;   // dyc: dy by columns; dgu: dg of all nodes, then du, by columns; dgur: by rows
    float *dh, *sums;
    int64_t ldh, bytes;
    uint32_t* peaks;             // largest values of columns of dy, x, down, gate or up, h, dg, du and of rows of dg or du
    uint32_t *peaks_h, *peaks_dgu, *peaks_rows;
    int64_t peak_bytes;
    int8_t *of_dy, *of_dyc, *of_x, *of_gate, *of_down, *of_h, *of_dgu, *of_dgur;   // exponents; of_gate: of gate and up
};

PairsPlan plan_pairs(const FeedForwardParams& p)
{
    PairsPlan q;
    q.rows.base = q.columns.base = p.scratch;
    q.rows.pieces = q.columns.pieces = 2;
    q.rows.by_rows(p.d);
    q.columns.by = PackPlan::kColumns;
    ScratchPlan& s = q.columns.scratch;
    const int64_t d8 = padded(p.d), f8 = padded(p.f), n = p.nodes;
    q.peak_bytes = n * (3 * d8 + 4 * f8 + padded(p.rows)) * 4;
    q.peaks = reinterpret_cast<uint32_t*>(p.scratch + s.take(q.peak_bytes));
    uint32_t* const peaks_x = q.peaks + n * d8;
    uint32_t* const peaks_gate = peaks_x + n * d8;
    uint32_t* const peaks_down = peaks_gate + n * d8;
    q.peaks_h = peaks_down + n * f8;
    q.peaks_dgu = q.peaks_h + n * f8;
    q.peaks_rows = q.peaks_dgu + 2 * n * f8;
    q.rows.scratch = s;
    q.dy = q.rows.operand(p.dy.p, p.dy.ld, p.rows * p.dy.ld, p.rows, p.d, n, true, false, 2);
    q.of_dy = q.rows.powers();
    s = q.rows.scratch;
    PackJobs& jobs = q.columns.jobs;
    jobs.slice = slice_rows(std::max({p.rows, p.d, p.f}), (std::max(p.d, p.f) + 7) / 8, n, sm_count());
    const auto operand = [&](const Matrix& m, int64_t node, int64_t rows, int64_t cols, uint32_t* peaks) {
        const Operand o = q.columns.operand(m.p, m.ld, node, rows, cols, n, true, true, 2);
        jobs.job[jobs.count - 1].peaks = peaks;
        return o;
    };
    q.dyc = operand(p.dy, p.rows * p.dy.ld, p.rows, p.d, q.peaks);
    q.of_dyc = q.columns.powers();
    q.x = operand(p.x, p.rows * p.x.ld, p.rows, p.d, peaks_x);
    q.of_x = q.columns.powers();
    q.down = operand(p.down, p.down.node, p.d, p.f, peaks_down);
    q.of_down = q.columns.powers();
    q.gate = operand(p.gate, p.gate.node, p.f, p.d, peaks_gate);
    q.of_gate = q.columns.powers();
    q.up = operand(p.up, p.up.node, p.f, p.d, peaks_gate);      // one power for both: their products are one sum
    jobs.job[jobs.count - 1].exponents = q.of_gate;
    q.ldh = f8;
    q.dh = reinterpret_cast<float*>(p.scratch + s.take(n * p.rows * q.ldh * 4));
    q.h = q.columns.written(p.rows, p.f, n, true);
    q.dgu = q.columns.written(p.rows, p.f, 2 * n, true);
    q.dgur = q.columns.written(p.rows, p.f, 2 * n, false);
    q.of_h = reinterpret_cast<int8_t*>(p.scratch + s.take(n * f8));
    q.of_dgu = reinterpret_cast<int8_t*>(p.scratch + s.take(2 * n * f8));
    q.of_dgur = reinterpret_cast<int8_t*>(p.scratch + s.take(n * padded(p.rows)));
    const int64_t parts = std::max(parts_bytes<2>(p.rows, p.f, p.d, n, 1, 2), all_parts_bytes<2>(p, 2));
    q.sums = reinterpret_cast<float*>(p.scratch + s.take(parts));
    q.bytes = s.bytes;
    return q;
}

struct SlopeParams {
    const float *g, *u, *dh;
    int64_t ldg, ldu, ldh, rows, nodes, units;
    int32_t f, slice, kind, vec;
    Pieces<__half> h, dg, du, dgr, dur;       // dgr, dur: by rows
    uint32_t *peaks_h, *peaks_dgu, *peaks_rows;
    int8_t *of_h, *of_dgu, *of_dgur;
};

// PACK: the pieces of h, dg and du; otherwise their largest values.  Bound by memory (12 bytes read per value, 20 written).
template <bool PACK>
__global__ void __launch_bounds__(256) slopes_kernel(const __grid_constant__ SlopeParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t chunks = p.ldh / 8;
    __shared__ uint32_t peaks[3][256];
    for (int64_t unit = blockIdx.x; unit < p.units; unit += gridDim.x) {
        const StripPlace s = strip_place(unit, p.rows, chunks, p.slice);
        const bool there = s.chunk < chunks;
        const int col = s.chunk * 8, left = p.f - col;
        const int64_t of_node = s.batch * p.ldh + col, second = p.nodes * p.ldh;    // du's columns behind dg's
        uint32_t ph[8] = {}, pg[8] = {}, pu[8] = {};
        float sh[8], sg[8], su[8];
        if constexpr (PACK) {
            if (there) {
                const bool keep = s.first == 0 && s.group == 0;
                column_scales(p.peaks_h + of_node, sh, keep ? p.of_h + of_node : nullptr);
                column_scales(p.peaks_dgu + of_node, sg, keep ? p.of_dgu + of_node : nullptr);
                column_scales(p.peaks_dgu + second + of_node, su, keep ? p.of_dgu + second + of_node : nullptr);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) peaks[i][threadIdx.x] = 0;
            __syncthreads();
        }
        Raw<float> rg, ru, rd;
        const auto load = [&](int64_t r) {      // a row ahead
            if (!there || r >= s.end) return;
            const int64_t row = s.batch * p.rows + r;
            rg.load(p.g + row * p.ldg + col, left, p.vec);
            ru.load(p.u + row * p.ldu + col, left, p.vec);
            rd.load(p.dh + row * p.ldh + col, left, true);
        };
        load(s.first + s.group);
        // the same turns for all threads, as they exchange their rows' largest values
        for (int64_t first = s.first; first < s.end; first += s.step) {
            const int64_t r = first + s.group, row = s.batch * p.rows + r, place = row * p.ldh + col;
            const bool in = there && r < s.end;
            uint32_t most = 0;
            if (in) {
                float v[8], w[8], dh[8], dg[8];
                rg.values(v);
                ru.values(w);
                rd.values(dh);
                load(r + s.step);
                block_slopes<false>(v, w, dh, dg, p.kind);
                if constexpr (PACK) {
                    float a[8], b[8];
                    const int e = scale_exponent(p.peaks_rows[s.batch * padded(p.rows) + r]);
                    const float scale = power_of_two(e);
                    if (s.chunk == 0) p.of_dgur[s.batch * padded(p.rows) + r] = (int8_t)-e;
#pragma unroll
                    for (int k = 0; k < 8; ++k) a[k] = dg[k] * scale, b[k] = dh[k] * scale;
                    p.dgr.store_at<2>(place, a);
                    p.dur.store_at<2>(place, b);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] *= sh[k], dg[k] *= sg[k], dh[k] *= su[k];
                    p.h.store_at<2>(place, v);
                    p.dg.store_at<2>(place, dg);
                    p.du.store_at<2>(place, dh);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (k < left) {
                            const uint32_t a = finite_bits(dg[k]), b = finite_bits(dh[k]);
                            ph[k] = max(ph[k], finite_bits(v[k]));
                            pg[k] = max(pg[k], a);
                            pu[k] = max(pu[k], b);
                            most = max(most, max(a, b));
                        }
                }
            }
            if constexpr (!PACK) {
                if (s.lanes == 32)
                    most = __reduce_max_sync(~0u, most);
                else
                    for (int o = s.lanes / 2; o; o >>= 1) most = max(most, __shfl_xor_sync(~0u, most, o));
                if ((threadIdx.x & (s.lanes - 1)) == 0 && most) atomicMax(p.peaks_rows + s.batch * padded(p.rows) + r, most);
            }
        }
        if constexpr (!PACK) {
            const int at = (threadIdx.x & (s.lanes - 1)) * 8;
            if (there)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    atomicMax(&peaks[0][at + k], ph[k]);
                    atomicMax(&peaks[1][at + k], pg[k]);
                    atomicMax(&peaks[2][at + k], pu[k]);
                }
            __syncthreads();
            const int64_t column = s.strip * 256 + threadIdx.x;
            if (column < p.ldh) {
                const int64_t to = s.batch * p.ldh + column;
                if (peaks[0][threadIdx.x]) atomicMax(p.peaks_h + to, peaks[0][threadIdx.x]);
                if (peaks[1][threadIdx.x]) atomicMax(p.peaks_dgu + to, peaks[1][threadIdx.x]);
                if (peaks[2][threadIdx.x]) atomicMax(p.peaks_dgu + second + to, peaks[2][threadIdx.x]);
            }
            __syncthreads();
        }
    }
}

cudaError_t backward_pairs(const FeedForwardParams& p, cudaStream_t stream)
{
    const PairsPlan q = plan_pairs(p);
    const int32_t nodes = (int32_t)p.nodes;
    const int64_t d8 = padded(p.d), f8 = padded(p.f), r8 = padded(p.rows);
    cudaError_t e = q.rows.launch_rows(false, q.peaks, q.peak_bytes, stream);
    if (e == cudaSuccess) e = q.columns.launch_columns(false, stream);
    if (e == cudaSuccess) e = q.columns.launch_columns(true, stream);
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
    e = store_product<float, 2>(g, dh, p.nodes * p.rows, nullptr, false, {q.of_dy, q.of_down, r8, f8, nodes}, q.sums, stream);
    if (e != cudaSuccess) return e;
    const auto half_of = [&](const Operand& both, int which) {     // dg's or du's
        Operand o = both;
        o.batches = p.nodes;
        o.base = static_cast<const __half*>(o.base) + which * p.nodes * o.batch;
        return o;
    };
    SlopeParams s;
    s.g = static_cast<const float*>(p.g.p);
    s.u = static_cast<const float*>(p.u.p);
    s.dh = q.dh;
    s.ldg = p.g.ld;
    s.ldu = p.u.ld;
    s.ldh = q.ldh;
    s.rows = p.rows;
    s.nodes = p.nodes;
    s.slice = slice_rows(p.rows, q.ldh / 8, p.nodes, sm_count());
    s.units = p.nodes * ((p.rows + s.slice - 1) / s.slice) * ((q.ldh / 8 + 31) / 32);
    s.f = (int32_t)p.f;
    s.kind = p.activation;
    s.vec = rows_on_16(p.g.p, p.g.ld, p.nodes * p.rows, 0, 1, 4) && rows_on_16(p.u.p, p.u.ld, p.nodes * p.rows, 0, 1, 4);
    s.h = pieces_of<__half>(q.h);
    s.dg = pieces_of<__half>(half_of(q.dgu, 0));
    s.du = pieces_of<__half>(half_of(q.dgu, 1));
    s.dgr = pieces_of<__half>(half_of(q.dgur, 0));
    s.dur = pieces_of<__half>(half_of(q.dgur, 1));
    s.peaks_h = q.peaks_h;
    s.peaks_dgu = q.peaks_dgu;
    s.peaks_rows = q.peaks_rows;
    s.of_h = q.of_h;
    s.of_dgu = q.of_dgu;
    s.of_dgur = q.of_dgur;
    const dim3 blocks((unsigned)std::min<int64_t>(s.units, (int64_t)sm_count() * 16));
    e = launch_after_trigger(slopes_kernel<false>, blocks, dim3(256), 0, stream, true, s);
    if (e == cudaSuccess) e = launch_after_trigger(slopes_kernel<true>, blocks, dim3(256), 0, stream, true, s);
    if (e != cudaSuccess) return e;

    g.a[0] = q.dyc;                     // dWd
    g.b[0] = q.h;
    g.m = p.d;
    g.n = p.f;
    g.k = p.rows;
    if ((e = store_product<float, 2>(g, p.ddown, p.d, nullptr, p.accumulate, {q.of_dyc, q.of_h, d8, f8, nodes}, q.sums, stream)) != cudaSuccess) return e;
    g.a[0] = q.dgu;                     // dWg, dWu
    g.b[0] = q.x;
    g.m = p.f;
    g.n = p.d;
    g.batch = 2 * p.nodes;
    if ((e = store_product<float, 2>(g, p.dgate, p.f, &p.dup, p.accumulate, {q.of_dgu, q.of_x, f8, d8, nodes}, q.sums, stream)) != cudaSuccess) return e;
    g.pairs = 2;                        // dx
    g.batch = p.nodes;
    g.a[0] = half_of(q.dgur, 0);
    g.a[1] = half_of(q.dgur, 1);
    g.b[0] = q.gate;
    g.b[1] = q.up;
    g.m = p.rows;
    g.n = p.d;
    g.k = p.f;
    return store_product<float, 2>(g, p.dx, p.nodes * p.rows, nullptr, false, {q.of_dgur, q.of_gate, r8, d8, nodes}, q.sums, stream);
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
