// Gated feed-forward block: the activation and its slope, and what the products' epilogues do with them.
#pragma once
#include <type_traits>

#include "gpga_ff.cuh"
#include "gpga_pack.cuh"

namespace gpga {

enum { kSilu = 0, kGelu = 1, kRelu = 2 };

// 2^x and 1 / x by the special-function unit (errors of about 2^-22), results below 2^-126 as zero.
__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fast_reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / (1 + e^-v) and e^(-v^2 / 2).  fp32 results take CUDA's expf and its division to two steps (2^-22); the fast forms' errors
// are below the rounding of 16-bit ones.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float v)
{
    return FAST ? fast_reciprocal(1.f + fast_exp2(-1.44269504f * v)) : __fdividef(1.f, 1.f + expf(-v));
}
template <bool FAST>
__device__ __forceinline__ float bell(float v)
{
    return FAST ? fast_exp2(-0.72134752f * v * v) : expf(-0.5f * v * v);
}

// v <- act(v).
template <bool FAST, int N>
__device__ __forceinline__ void act_values(float (&v)[N], int kind)
{
    if (kind == kSilu) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= sigmoid<FAST>(v[i]);
    } else if (kind == kGelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= 0.5f * (1.f + erff(v[i] * 0.70710678118654752f));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] <= 0.f ? 0.f : v[i];    // NaN stays
    }
}
// v <- act(v), s = act'(v).
template <bool FAST, int N>
__device__ __forceinline__ void act_slopes(float (&v)[N], float (&s)[N], int kind)
{
    if (kind == kSilu) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float sig = sigmoid<FAST>(v[i]), a = v[i] * sig;
            s[i] = fmaf(a, 1.f - sig, sig);
            v[i] = a;
        }
    } else if (kind == kGelu) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float c = 0.5f * (1.f + erff(v[i] * 0.70710678118654752f));
            s[i] = fmaf(v[i] * 0.39894228040143268f, bell<FAST>(v[i]), c);
            v[i] *= c;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = v[i] > 0.f ? 1.f : 0.f;
            v[i] = v[i] <= 0.f ? 0.f : v[i];
        }
    }
}

// The type of the pieces of an activation type, and how many there are.
template <class T> struct PiecesOf { using type = T; static constexpr int count = 1; };
template <> struct PiecesOf<float> { using type = __nv_bfloat16; static constexpr int count = 3; };

// fp32 operands as pairs of fp16 (ff_pairs): a product's element is 2^(a + b) times the product of what was packed, with an
// exponent a of its row and one b of its column.  (A value is 2^-23 of itself off in a pair, or 2^-40 of the largest one that
// shares its power; the product of two rests, at most 2^-22 of a term, is left out.)
struct Exponents {
    const int8_t *a = nullptr, *b = nullptr;
    int64_t a_batch = 0, b_batch = 0;
    int32_t b_mod = 1;        // batches of b, which come twice at most
    __device__ __forceinline__ int row(int batch, int r) const { return a[batch * a_batch + r]; }
    __device__ __forceinline__ const int8_t* column(int batch, int c) const { return b + (batch >= b_mod ? batch - b_mod : batch) * b_batch + c; }
    using Columns = uint2;    // of eight columns, as they lie in memory
    __device__ __forceinline__ Columns columns(int batch, int c) const { return *reinterpret_cast<const uint2*>(column(batch, c)); }
    // 2^(a + b) as two factors with half of the exponent each, as it may be beyond fp32's range.  Exponents are -125 at least, so that
    // a half's sum is that of a normal number.  What lies between the two is between the sum and the result: nothing is lost there.
    struct Factors {
        int32_t one[8], two[8];   // of a column: bits of its halves
    };
    __device__ __forceinline__ static Factors factors(const Columns& w)
    {
        Factors q;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int e = (int8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3)));
            q.one[k] = ((e >> 1) + 127) << 23;
            q.two[k] = (e - (e >> 1) + 127) << 23;
        }
        return q;
    }
    // own: the row's exponent
    __device__ __forceinline__ static void eight(float (&v)[8], const Factors& q, int own)
    {
        const int one = (own >> 1) << 23, two = (own - (own >> 1)) << 23;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] * __int_as_float(q.one[k] + one) * __int_as_float(q.two[k] + two);
    }
    __device__ __forceinline__ float one(float v, int batch, int r, int c) const
    {
        const int own = row(batch, r), e = *column(batch, c);
        return v * power_of_two((own >> 1) + (e >> 1)) * power_of_two(own - (own >> 1) + e - (e >> 1));
    }
};
// An array between two products that is packed after the first: fp32 rows.
struct Between {
    float* base = nullptr;
    int64_t ld = 0, batch = 0;
    __device__ __forceinline__ void store(int64_t place, const float (&v)[8]) const
    {
        reinterpret_cast<float4*>(base + place)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(base + place)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
};

// g, u -> h = act(g) u as pieces (PAIRS: as fp32); g and u themselves where they are kept.
template <class T, bool PAIRS = false>
struct GateUp {
    static constexpr bool kDual = true, kMirror = false, kPair = false;
    static constexpr double kTail = 3.0;
    static constexpr int kWarps = 16;
    using T16 = typename PiecesOf<T>::type;
    static constexpr int P = PiecesOf<T>::count;
    using Ahead = Nothing;
    T *g, *u;
    int64_t ldg, ldu;
    std::conditional_t<PAIRS, Between, Pieces<T16>> h;
    Exponents of_g, of_u;     // PAIRS
    int32_t m, kind, keeps, vec;
    // Of one of the two arrays.
    using Columns = std::conditional_t<PAIRS, Exponents::Columns, Nothing>;

    __device__ __forceinline__ bool wide() const { return vec; }
    __device__ __forceinline__ Columns columns(int which, int batch, int col) const
    {
        if constexpr (PAIRS) return (which ? of_u : of_g).columns(batch, col);
        else return {};
    }
    __device__ __forceinline__ int row(int batch, int r) const { return PAIRS ? of_g.row(batch, r) : 0; }
    __device__ __forceinline__ static auto factors(const Columns& q)
    {
        if constexpr (PAIRS) return Exponents::factors(q);
        else return q;
    }
    template <class Factors>
    __device__ __forceinline__ static void scale(float (&v)[8], const Factors& f, int own)
    {
        if constexpr (PAIRS) Exponents::eight(v, f, own);
    }
    __device__ __forceinline__ void keep(int which, float v, int batch, int row, int col) const
    {
        if constexpr (PAIRS) v = (which ? of_u : of_g).one(v, batch, row, col);
        (which ? u : g)[((int64_t)batch * m + row) * (which ? ldu : ldg) + col] = from_f32<T>(v);
    }
    __device__ __forceinline__ void eight(float (&v)[8], float (&w)[8], int batch, int row, int col, int left) const
    {
        if (keeps && vec) {
            const int64_t at = (int64_t)batch * m + row;
            store8(g + at * ldg + col, left, v);
            store8(u + at * ldu + col, left, w);
        }
        act_values<sizeof(T) == 2>(v, kind);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= w[i];
        if constexpr (PAIRS)
            h.store(batch * h.batch + row * h.ld + col, v);
        else
            h.template store<P>(batch, row, col, v);
    }
};

// v = g, w = u, dh -> v = h = act(g) u, dg = dh u act'(g), dh = du = dh act(g).
template <bool FAST>
__device__ __forceinline__ void block_slopes(float (&v)[8], const float (&w)[8], float (&dh)[8], float (&dg)[8], int kind)
{
    act_slopes<FAST>(v, dg, kind);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        dg[i] *= dh[i] * w[i];
        dh[i] *= v[i];
        v[i] *= w[i];
    }
}

// acc = dh; g, u -> h = act(g) u, du = dh act(g), dg = dh u act'(g), all as pieces.  What it reads and stores per tile bounds it: 16-bit
// values in whole lines (8 x 4096 tokens, 1024 x 2816: 236 us, 268 us in half lines).
template <class T>
struct GateGrad {
    static constexpr bool kDual = false, kMirror = false, kPair = sizeof(T) == 2;
    static constexpr double kTail = 6.0;
    static constexpr int kWarps = 16;
    using T16 = typename PiecesOf<T>::type;
    static constexpr int P = PiecesOf<T>::count;
    struct Ahead {
        Raw<T> g, u;
    };
    using Columns = Nothing;
    using Factors = Nothing;
    const T *g, *u;
    int64_t ldg, ldu;
    Pieces<T16> h, dg, du;
    int32_t m, kind, vec;

    __device__ __forceinline__ bool wide() const { return true; }
    __device__ __forceinline__ void one(float, int, int, int) const {}
    __device__ __forceinline__ Columns columns(int, int) const { return {}; }
    __device__ __forceinline__ static Factors factors(const Columns&) { return {}; }
    __device__ __forceinline__ void load(Ahead& ahead, int batch, int row, int col, int left) const
    {
        const int64_t at = (int64_t)batch * m + row;
        ahead.g.load(g + at * ldg + col, left, vec);
        ahead.u.load(u + at * ldu + col, left, vec);
    }
    __device__ __forceinline__ void eight(float (&dh)[8], const Ahead& now, const Factors&, int batch, int row, int col, int left) const
    {
        float a[8], s[8], uv[8];
        now.g.values(a);
        now.u.values(uv);
        block_slopes<sizeof(T) == 2>(a, uv, dh, s, kind);
        const int64_t at = batch * h.batch + row * h.ld + col;    // of all three
        dg.template store_at<P>(at, s);
        h.template store_at<P>(at, a);
        du.template store_at<P>(at, dh);
    }
};

// acc -> an array of the caller's; batches from `split` on go to the second one.  PAIRS: times the powers of two of its operands.
template <class T, bool PAIRS = false>
struct StoreRows {
    static constexpr bool kDual = false, kMirror = false, kPair = false;
    static constexpr double kTail = 1.0;
    static constexpr int kWarps = 8;
    struct Ahead {
        Raw<T> old;
        int row;              // its exponent
    };
    using Columns = std::conditional_t<PAIRS, Exponents::Columns, Nothing>;
    using Factors = std::conditional_t<PAIRS, Exponents::Factors, Nothing>;
    T* out[2];
    int64_t ld[2], node[2];
    Exponents exponents;
    int32_t split, accumulate, vec;

    __device__ __forceinline__ bool wide() const { return vec; }
    __device__ __forceinline__ Rows<T> rows(int batch) const
    {
        const int which = batch >= split;
        return {out[which] + (batch - which * split) * node[which], ld[which], 1.f, accumulate != 0};
    }
    __device__ __forceinline__ void load(Ahead& ahead, int batch, int row, int col, int left) const
    {
        if constexpr (PAIRS) ahead.row = exponents.row(batch, row);
        rows(batch).ahead(ahead.old, row, col, left);
    }
    __device__ __forceinline__ Columns columns(int batch, int col) const
    {
        if constexpr (PAIRS) return exponents.columns(batch, col);
        else return {};
    }
    __device__ __forceinline__ static Factors factors(const Columns& q)
    {
        if constexpr (PAIRS) return Exponents::factors(q);
        else return {};
    }
    __device__ __forceinline__ void eight(float (&v)[8], const Ahead& now, const Factors& f, int batch, int row, int col, int left) const
    {
        if constexpr (PAIRS) Exponents::eight(v, f, now.row);
        rows(batch).eight(v, now.old, row, col, left);
    }
    __device__ __forceinline__ void one(float v, int batch, int row, int col) const
    {
        if constexpr (PAIRS) v = exponents.one(v, batch, row, col);
        rows(batch).one(v, row, col);
    }
};

// The sums of a product left in parts: [batch][part][m][ld], added in the order of k.  A thread takes eight columns.
template <class T, bool PAIRS>
__global__ void __launch_bounds__(256) sum_parts_kernel(const float* sums, int parts, int m, int n, int64_t ld, int64_t chunks, const __grid_constant__ StoreRows<T, PAIRS> out)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int per = (int)(ld / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per;
        const int col = (int)(i - r * per) * 8, batch = (int)(r / m), row = (int)(r - (int64_t)batch * m);
        typename StoreRows<T, PAIRS>::Ahead old;
        if (out.wide()) out.load(old, batch, row, col, n - col);
        const float* from = sums + ((int64_t)batch * parts * m + row) * ld + col;
        float v[8] = {};
#pragma unroll 4
        for (int q = 0; q < parts; ++q, from += m * ld) {
            const float4 x = *reinterpret_cast<const float4*>(from), y = *reinterpret_cast<const float4*>(from + 4);
            const float z[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += z[k];
        }
        if (out.wide()) {
            out.eight(v, old, out.factors(out.columns(batch, col)), batch, row, col, n - col);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (col + k < n) out.one(v[k], batch, row, col + k);
        }
    }
}

// Bytes of the parts of a product of P pieces, if store_product leaves its sums in parts.
template <int P>
int64_t parts_bytes(int64_t m, int64_t n, int64_t k, int64_t batch, int pairs, int64_t b_pieces)
{
    GemmPlan g;
    g.m = m;
    g.n = n;
    g.k = k;
    g.batch = batch;
    g.pairs = pairs;
    g.a[0].pieces = P;
    g.b[0].pieces = b_pieces;
    const int parts = gemm_parts(g, P * (P + 1) / 2, StoreRows<float>::kTail);
    return parts > 1 ? parts * batch * m * ((n + 7) / 8 * 8) * 4 : 0;
}

// A product stored at its place.  sums: room for parts_bytes().
template <class T, int P>
cudaError_t store_product(const GemmPlan& g, const Matrix& out, int64_t rows, const Matrix* second, bool accumulate, const Exponents& exponents, float* sums, cudaStream_t stream)
{
    StoreRows<T, P == 2> e;
    e.exponents = exponents;
    const Matrix& o2 = second ? *second : out;
    e.out[0] = static_cast<T*>(out.p);
    e.out[1] = static_cast<T*>(o2.p);
    e.ld[0] = out.ld;
    e.ld[1] = o2.ld;
    e.node[0] = out.node;
    e.node[1] = o2.node;
    e.split = (int32_t)(second ? g.batch / 2 : g.batch);
    e.accumulate = accumulate;
    e.vec = rows_on_16(out.p, out.ld, rows, out.node, g.batch, sizeof(T)) && rows_on_16(o2.p, o2.ld, rows, o2.node, g.batch, sizeof(T));
    const int parts = gemm_parts(g, P * (P + 1) / 2, StoreRows<float>::kTail);
    if (parts == 1) return launch_gemm<P, T>(g, e, stream);
    StoreRows<float> to;
    const int64_t ld = (g.n + 7) / 8 * 8, chunks = g.batch * g.m * (ld / 8);
    to.out[0] = to.out[1] = sums;
    to.ld[0] = to.ld[1] = ld;
    to.node[0] = to.node[1] = g.m * ld;
    to.split = INT32_MAX;
    to.accumulate = 0;
    to.vec = 1;
    const cudaError_t r = launch_gemm_up_to<Variant<2, 256, P, 8, false, true>>(most_kblocks<T>, (gemm_kblocks(g) + parts - 1) / parts, g, parts, 0, 0, to, stream);
    if (r != cudaSuccess) return r;
    const dim3 blocks((unsigned)std::min<int64_t>((chunks + 255) / 256, (int64_t)sm_count() * 8));
    return launch_after_trigger(sum_parts_kernel<T, P == 2>, blocks, dim3(256), 0, stream, true, sums, parts, (int)g.m, (int)g.n, ld, chunks, e);
}

}  // namespace gpga
