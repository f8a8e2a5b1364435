// Orthogonalisation of an update by Newton-Schulz products.
//
//     X_0 = M / (|M| + eps),   X <- (a I + b A + c A^2) X with A = X X^T     (M with more rows than columns: X^T X, from the right)
//
// Three products a step: the Gram matrix A, the polynomial B = a I + b A + c A A, and B X.  A and B are symmetric, so
// every operand is read as it lies.  The matrices are held as S times their value in fp16: with |X| about 1 their entries
// lie between 1/columns and a few units, for which fp16 has its full 11 bits (S = 2^11 moves its range down to 2^-25 and
// leaves 2^5 above one).  16-bit updates take one fp16 value (rounding 2^-12, bfloat16's is 2^-9); fp32 updates two, 22
// bits, and three products of fp16 for one, summed as fp32 would be.  X_0 is M times a power of two (nothing is lost), the
// rest of the norm, kappa in [1, 2), is a factor in the first step's epilogues.
#include "gpga_orth.cuh"
#include "gpga_pack.cuh"

namespace gpga {

namespace {

constexpr float kScale = 2048.f;
constexpr int kNormParts = 1024;  // blocks of the sum of squares, over all matrices

// Sum of squares of a part of a matrix in fp64: no overflow, and the order is fixed.
template <class T>
__global__ void __launch_bounds__(256) square_sum_kernel(const T* m, int64_t ld, int64_t node, int64_t rows, int64_t cols, int vec, double* parts)
{
    const T* const base = m + blockIdx.y * node;
    const int64_t chunks = (cols + 7) / 8, count = rows * chunks;
    double sum = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks;
        const int col = (int)(i - r * chunks) * 8, n = (int)min((int64_t)8, cols - col);
        float v[8];
        const T* at = base + r * ld + col;
        Raw<T> x8;
        x8.load(at, n, vec);
        x8.values(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += (double)v[k] * v[k];
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    __shared__ double warps[8];
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) sum += warps[i];
        parts[blockIdx.y * gridDim.x + blockIdx.x] = sum;
    }
}

// M times a power of two as fp16 pieces, and kappa.
template <class T, int P>
__global__ void __launch_bounds__(256) start_kernel(const T* m, int64_t ld, int64_t node, int64_t rows, int64_t cols, int vec, const double* parts,
                                                     int count_parts, double eps, Pieces<__half> x, float* kappa)
{
    grid_launch_dependents();
    __shared__ double factor;
    if (threadIdx.x < 32) {
        double sum = 0;
        for (int i = threadIdx.x; i < count_parts; i += 32) sum += parts[blockIdx.y * count_parts + i];
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        if (threadIdx.x == 0) {
            const double norm = sqrt(sum) + eps;
            double power = 1, rest = 1;
            if (norm > 0 && norm <= 1e300) {
                int e;
                const double f = frexp(kScale / norm, &e);   // f in [1/2, 1)
                power = ldexp(0.5, e);
                rest = 2 * f;
            } else if (norm != 0) {
                rest = nan("");                              // an infinity or NaN in M
            }
            factor = power;
            if (blockIdx.x == 0) kappa[blockIdx.y] = (float)rest;
        }
    }
    __syncthreads();
    const T* const base = m + blockIdx.y * node;
    const int64_t chunks = (cols + 7) / 8, count = rows * chunks;
    const double power = factor;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks;
        const int col = (int)(i - r * chunks) * 8, n = (int)min((int64_t)8, cols - col);
        float v[8];
        const T* at = base + r * ld + col;
        Raw<T> x8;
        x8.load(at, n, vec);
        x8.values(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (float)(v[k] * power);
        const Pieces<__half> to{x.base + blockIdx.y * x.batch + r * x.ld + col, x.piece, 0, 0};
        to.template store<P>(0, 0, 0, v);
    }
}

// factor kappa^power acc + beta R (+ diagonal), as pieces.
template <int P>
struct KeepPieces {
    static constexpr bool kDual = false;
    struct Ahead {
        Raw<__half> r[P];
    };
    Pieces<__half> out, r;
    const float* kappa;
    float factor, beta, diagonal;
    int32_t power, with_r;

    __device__ __forceinline__ bool wide() const { return true; }
    __device__ __forceinline__ void one(float, int, int, int) const {}
    __device__ __forceinline__ void load(Ahead& ahead, int batch, int row, int col, int) const
    {
        if (with_r) r.template load<P>(batch, row, col, ahead.r);
    }
    __device__ __forceinline__ void eight(float (&v)[8], const Ahead& now, int batch, int row, int col, int) const
    {
        float a = factor;
        if (power) {
            const float k = kappa[batch];
            a *= power == 2 ? k * k : k;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= a;
        if (with_r) {
#pragma unroll
            for (int q = P - 1; q >= 0; --q) {
                float s[8];
                now.r[q].values(s);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] += beta * s[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (row == col + k) v[k] += diagonal;
        }
        out.template store<P>(batch, row, col, v);
    }
};

// The last step: factor kappa^power acc, added to what is there or not, in the caller's type.
template <class T>
struct LastStep {
    static constexpr bool kDual = false;
    using Ahead = Raw<T>;
    T* out;
    int64_t ld, node;
    const float* kappa;
    float factor;
    int32_t power, accumulate, vec;

    __device__ __forceinline__ bool wide() const { return vec; }
    __device__ __forceinline__ Rows<T> rows(int batch) const
    {
        return {out + batch * node, ld, power ? factor * kappa[batch] : factor, accumulate != 0};
    }
    __device__ __forceinline__ void load(Ahead& old, int batch, int row, int col, int left) const { rows(batch).ahead(old, row, col, left); }
    __device__ __forceinline__ void eight(float (&v)[8], const Ahead& old, int batch, int row, int col, int left) const
    {
        rows(batch).eight(v, old, row, col, left);
    }
    __device__ __forceinline__ void one(float v, int batch, int row, int col) const { rows(batch).one(v, row, col); }
};

bool on_16(const void* p, int64_t ld, int64_t rows, int64_t node, int64_t nodes, int size)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld * size % 16 == 0) && (nodes <= 1 || node * size % 16 == 0);
}

struct OrthPlan {
    ScratchPlan scratch;
    Operand x[2], a, b;
    double* parts;
    float* kappa;
    int count_parts;
};

OrthPlan plan_orth(const OrthParams& p)
{
    OrthPlan q;
    const int64_t s = std::min(p.r, p.c);
    q.count_parts = (int)std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(1, kNormParts / p.nodes), p.r * p.c / 2048));
    const auto array = [&](int64_t rows, int64_t cols) {
        Operand o;
        o.inner = cols;
        o.outer = rows;
        o.batches = p.nodes;
        o.pieces = p.dtype == 0 ? 2 : 1;
        o.ld = (cols + 7) / 8 * 8;
        o.batch = rows * o.ld;
        o.piece = p.nodes * o.batch;
        o.base = p.scratch + q.scratch.take(o.pieces * o.piece * 2);
        return o;
    };
    q.x[0] = array(p.r, p.c);
    q.x[1] = array(p.r, p.c);
    q.a = array(s, s);
    q.b = array(s, s);
    q.parts = reinterpret_cast<double*>(p.scratch + q.scratch.take(p.nodes * q.count_parts * 8));
    q.kappa = reinterpret_cast<float*>(p.scratch + q.scratch.take(p.nodes * 4));
    return q;
}

template <int P, class Epi>
cudaError_t product(const GemmPlan& g, const Epi& e, cudaStream_t stream)
{
    if (g.m <= 128) return launch_gemm_as<Variant<1, 128, P>>(g, e, stream);
    return launch_gemm_as<Variant<2, 256, P>>(g, e, stream);
}

template <class T>
cudaError_t orth(const OrthParams& p, cudaStream_t stream)
{
    constexpr int P = sizeof(T) == 4 ? 2 : 1;
    const OrthPlan q = plan_orth(p);
    const T* m = static_cast<const T*>(p.m);
    const int vec = on_16(p.m, p.ldm, p.r, p.node_ldm, p.nodes, sizeof(T));
    square_sum_kernel<T><<<dim3(q.count_parts, (unsigned)p.nodes), 256, 0, stream>>>(m, p.ldm, p.node_ldm, p.r, p.c, vec, q.parts);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>((p.r * ((p.c + 7) / 8) + 255) / 256, (int64_t)sm_count() * 8 / std::min<int64_t>(p.nodes, 64)));
    start_kernel<T, P><<<dim3((unsigned)blocks, (unsigned)p.nodes), 256, 0, stream>>>(m, p.ldm, p.node_ldm, p.r, p.c, vec, q.parts, q.count_parts, p.eps,
                                                                                 pieces_of<__half>(q.x[0]), q.kappa);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;

    const bool tall = p.r > p.c;
    const int64_t s = std::min(p.r, p.c);
    KeepPieces<P> keep;
    keep.kappa = q.kappa;
    GemmPlan g;
    g.half = true;
    g.batch = g.bmod = p.nodes;
    g.after = true;
    for (int64_t i = 0; i < p.steps; ++i) {
        const Operand &x = q.x[i & 1], &next = q.x[~i & 1];
        const int first = i == 0;
        g.a[0] = g.b[0] = x;                            // A
        g.a[0].mn_major = g.b[0].mn_major = tall;
        g.m = g.n = s;
        g.k[0] = std::max(p.r, p.c);
        keep.out = pieces_of<__half>(q.a);
        keep.factor = 1.f / kScale;
        keep.power = first ? 2 : 0;
        keep.with_r = 0;
        keep.r = keep.out;
        if ((e = product<P>(g, keep, stream)) != cudaSuccess) return e;
        g.a[0] = g.b[0] = q.a;                          // B = a I + b A + c A A
        g.a[0].mn_major = g.b[0].mn_major = false;
        g.k[0] = s;
        keep.out = pieces_of<__half>(q.b);
        keep.r = pieces_of<__half>(q.a);
        keep.factor = (float)(p.c5 / kScale);
        keep.beta = (float)p.c3;
        keep.diagonal = (float)(p.c1 * kScale);
        keep.power = 0;
        keep.with_r = 1;
        if ((e = product<P>(g, keep, stream)) != cudaSuccess) return e;
        g.a[0] = tall ? x : q.b;                        // B X or X B
        g.b[0] = tall ? q.b : x;
        g.a[0].mn_major = false;
        g.b[0].mn_major = !tall;
        g.m = p.r;
        g.n = p.c;
        g.k[0] = s;
        if (i + 1 < p.steps) {
            keep.out = pieces_of<__half>(next);
            keep.factor = 1.f / kScale;
            keep.power = first;
            keep.with_r = 0;
            if ((e = product<P>(g, keep, stream)) != cudaSuccess) return e;
        } else {
            LastStep<T> last;
            last.out = static_cast<T*>(p.out);
            last.ld = p.ldo;
            last.node = p.node_ldo;
            last.kappa = q.kappa;
            last.factor = (float)(p.scale / ((double)kScale * kScale));
            last.power = first;
            last.accumulate = p.accumulate;
            last.vec = on_16(p.out, p.ldo, p.r, p.node_ldo, p.nodes, sizeof(T));
            if ((e = product<P>(g, last, stream)) != cudaSuccess) return e;
        }
    }
    return cudaSuccess;
}

}  // namespace

unsigned int* orth_gave_up()
{
    void* at = nullptr;
    return cudaGetSymbolAddress(&at, gave_up) == cudaSuccess ? static_cast<unsigned int*>(at) : nullptr;
}

int64_t orth_scratch_bytes(const OrthParams& p) { return plan_orth(p).scratch.bytes; }

cudaError_t launch_orth(const OrthParams& p, cudaStream_t stream)
{
    if (p.dtype == 0) return orth<float>(p, stream);
    if (p.dtype == 1) return orth<__nv_bfloat16>(p, stream);
    return orth<__half>(p, stream);
}

}  // namespace gpga
