// Gated feed-forward block: the activation and its slope, and what the products' epilogues do with them.
#pragma once
#include "gpga_ff.cuh"
#include "gpga_pack.cuh"

namespace gpga {

enum { kSilu = 0, kGelu = 1, kRelu = 2 };

// act(v).  fp32 results take CUDA's expf; the fast form's error (2^-21 of the value and more beyond |v| = 8) is below the
// rounding of 16-bit ones.
template <bool FAST>
__device__ __forceinline__ float act_value(float v, int kind)
{
    if (kind == kSilu) return FAST ? __fdividef(v, 1.f + __expf(-v)) : v / (1.f + expf(-v));
    if (kind == kGelu) return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    return v <= 0.f ? 0.f : v;    // NaN stays
}
// act(v) and act'(v).
template <bool FAST>
__device__ __forceinline__ void act_slope(float v, int kind, float& a, float& s)
{
    if (kind == kSilu) {
        const float sig = FAST ? __fdividef(1.f, 1.f + __expf(-v)) : 1.f / (1.f + expf(-v));
        a = v * sig;
        s = sig * (1.f + v * (1.f - sig));
    } else if (kind == kGelu) {
        const float c = 0.5f * (1.f + erff(v * 0.70710678118654752f));
        a = v * c;
        s = c + v * 0.39894228040143268f * (FAST ? __expf(-0.5f * v * v) : expf(-0.5f * v * v));
    } else {
        a = v <= 0.f ? 0.f : v;
        s = v > 0.f ? 1.f : 0.f;
    }
}

// The type of the pieces of an activation type, and how many there are.
template <class T> struct PiecesOf { using type = T; static constexpr int count = 1; };
template <> struct PiecesOf<float> { using type = __nv_bfloat16; static constexpr int count = 3; };

// g, u -> h = act(g) u as pieces; g and u themselves where they are kept.
template <class T>
struct GateUp {
    static constexpr bool kDual = true;
    using T16 = typename PiecesOf<T>::type;
    static constexpr int P = PiecesOf<T>::count;
    using Ahead = NothingAhead;
    T *g, *u;
    int64_t ldg, ldu;
    Pieces<T16> h;
    int32_t m, kind, keeps, vec;

    __device__ __forceinline__ bool wide() const { return vec; }
    __device__ __forceinline__ void keep(int which, float v, int batch, int row, int col) const
    {
        (which ? u : g)[((int64_t)batch * m + row) * (which ? ldu : ldg) + col] = from_f32<T>(v);
    }
    __device__ __forceinline__ void eight(float (&v)[8], float (&w)[8], int batch, int row, int col, int left) const
    {
        if (keeps && vec) {
            const int64_t at = (int64_t)batch * m + row;
            store8(g + at * ldg + col, left, v);
            store8(u + at * ldu + col, left, w);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = act_value<sizeof(T) == 2>(v[i], kind) * w[i];
        h.template store<P>(batch, row, col, v);
    }
};

// acc = dh; g, u -> h = act(g) u, du = dh act(g), dg = dh u act'(g), all as pieces.
template <class T>
struct GateGrad {
    static constexpr bool kDual = false;
    using T16 = typename PiecesOf<T>::type;
    static constexpr int P = PiecesOf<T>::count;
    struct Ahead {
        Raw<T> g, u;
    };
    const T *g, *u;
    int64_t ldg, ldu;
    Pieces<T16> h, dg, du;
    int32_t m, kind, vec;

    __device__ __forceinline__ bool wide() const { return true; }
    __device__ __forceinline__ void one(float, int, int, int) const {}
    __device__ __forceinline__ void load(Ahead& ahead, int batch, int row, int col, int left) const
    {
        const int64_t at = (int64_t)batch * m + row;
        ahead.g.load(g + at * ldg + col, left, vec);
        ahead.u.load(u + at * ldu + col, left, vec);
    }
    __device__ __forceinline__ void eight(float (&dh)[8], const Ahead& now, int batch, int row, int col, int) const
    {
        float a[8], s[8], gu[8];
        now.g.values(gu);
#pragma unroll
        for (int i = 0; i < 8; ++i) act_slope<sizeof(T) == 2>(gu[i], kind, a[i], s[i]);
        now.u.values(gu);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] *= dh[i] * gu[i];
        dg.template store<P>(batch, row, col, s);
#pragma unroll
        for (int i = 0; i < 8; ++i) gu[i] *= a[i];
        h.template store<P>(batch, row, col, gu);
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] *= dh[i];
        du.template store<P>(batch, row, col, a);
    }
};

// acc -> an array of the caller's; batches from `split` on go to the second one.
template <class T>
struct StoreRows {
    static constexpr bool kDual = false;
    using Ahead = Raw<T>;
    T* out[2];
    int64_t ld[2], node[2];
    int32_t split, accumulate, vec;

    __device__ __forceinline__ bool wide() const { return vec; }
    __device__ __forceinline__ Rows<T> rows(int batch) const
    {
        const int which = batch >= split;
        return {out[which] + (batch - which * split) * node[which], ld[which], 1.f, accumulate != 0};
    }
    __device__ __forceinline__ void load(Ahead& old, int batch, int row, int col, int left) const { rows(batch).ahead(old, row, col, left); }
    __device__ __forceinline__ void eight(float (&v)[8], const Ahead& old, int batch, int row, int col, int left) const
    {
        rows(batch).eight(v, old, row, col, left);
    }
    __device__ __forceinline__ void one(float v, int batch, int row, int col) const { rows(batch).one(v, row, col); }
};

inline bool rows_on_16(const void* p, int64_t ld, int64_t rows, int64_t node, int64_t nodes, int size)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld * size % 16 == 0) && (nodes <= 1 || node * size % 16 == 0);
}

// One block a tile where rows are few, pairs of blocks otherwise.
template <int P, class Epi>
cudaError_t launch_gemm(const GemmPlan& g, const Epi& epi, cudaStream_t stream)
{
    if (g.m <= 128) return launch_gemm_as<Variant<1, 128, P>>(g, epi, stream);
    return launch_gemm_as<Variant<2, 256, P>>(g, epi, stream);
}

template <class T, int P>
cudaError_t store_product(const GemmPlan& g, const Matrix& out, int64_t rows, const Matrix* second, bool accumulate, cudaStream_t stream)
{
    StoreRows<T> e;
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
    return launch_gemm<P>(g, e, stream);
}

}  // namespace gpga
