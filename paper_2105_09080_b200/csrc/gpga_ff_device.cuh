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
    int32_t m, n, kind, keep, vec;

    __device__ __forceinline__ void load(Ahead&, int, int, int, int) const {}

    template <bool VEC>
    __device__ __forceinline__ void keep_values(const float (&v)[32], T* to, int64_t ld, float* stage, int lane, int batch, int row0, int col0) const
    {
        along_rows<VEC>(v, stage, lane, [&](int, int row, int c, auto& x) {
            if (row0 + row < m && col0 + c < n) store_values(to + ((int64_t)batch * m + row0 + row) * ld + col0 + c, n - col0 - c, x);
        });
    }
    __device__ __forceinline__ void operator()(float (&v)[32], float (&w)[32], const Ahead&, float* stage, int lane, int batch, int row0, int col0) const
    {
        if (keep) {
            if (vec) {
                keep_values<true>(v, g, ldg, stage, lane, batch, row0, col0);
                keep_values<true>(w, u, ldu, stage, lane, batch, row0, col0);
            } else {
                keep_values<false>(v, g, ldg, stage, lane, batch, row0, col0);
                keep_values<false>(w, u, ldu, stage, lane, batch, row0, col0);
            }
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = act_value<sizeof(T) == 2>(v[i], kind) * w[i];
        along_rows<true>(v, stage, lane, [&](int, int row, int c, auto& x) {
            if (row0 + row < m && col0 + c < n) h.template store<P>(batch, row0 + row, col0 + c, n - col0 - c, x);
        });
    }
};

// acc = dh; g, u -> h = act(g) u, du = dh act(g), dg = dh u act'(g), all as pieces.
template <class T>
struct GateGrad {
    static constexpr bool kDual = false;
    using T16 = typename PiecesOf<T>::type;
    static constexpr int P = PiecesOf<T>::count;
    struct Ahead {
        Raw<T> g[4], u[4];
    };
    const T *g, *u;
    int64_t ldg, ldu;
    Pieces<T16> h, dg, du;
    int32_t m, n, kind, vec;

    __device__ __forceinline__ void load(Ahead& ahead, int lane, int batch, int row0, int col0) const
    {
        ahead_of_rows(lane, [&](int i, int row, int c) {
            const int left = row0 + row < m ? n - col0 - c : 0;
            const int64_t at = (int64_t)batch * m + row0 + row;
            ahead.g[i].load(g + at * ldg + col0 + c, left, vec);
            ahead.u[i].load(u + at * ldu + col0 + c, left, vec);
        });
    }
    __device__ __forceinline__ void operator()(float (&v)[32], float (&)[32], const Ahead& ahead, float* stage, int lane, int batch, int row0, int col0) const
    {
        along_rows<true>(v, stage, lane, [&](int j, int row, int c, auto& dh) {
            const int left = n - col0 - c;
            if (row0 + row >= m || left <= 0) return;
            float gv[8], uv[8];
            ahead.g[j].values(gv);
            ahead.u[j].values(uv);
            float hv[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float a, s;
                act_slope<sizeof(T) == 2>(gv[i], kind, a, s);
                hv[i] = a * uv[i];
                gv[i] = dh[i] * uv[i] * s;
                uv[i] = dh[i] * a;
            }
            h.template store<P>(batch, row0 + row, col0 + c, left, hv);
            dg.template store<P>(batch, row0 + row, col0 + c, left, gv);
            du.template store<P>(batch, row0 + row, col0 + c, left, uv);
        });
    }
};

// acc -> an array of the caller's; batches from `split` on go to the second one.
template <class T>
struct StoreRows {
    static constexpr bool kDual = false;
    using Ahead = NothingAhead;
    T* out[2];
    int64_t ld[2], node[2];
    int32_t m, n, split, accumulate, vec;

    __device__ __forceinline__ void load(Ahead&, int, int, int, int) const {}
    template <bool VEC>
    __device__ __forceinline__ void rows(const float (&v)[32], float* stage, int lane, int batch, int row0, int col0) const
    {
        const int which = batch >= split;
        store_rows<VEC>(v, out[which] + (batch - which * split) * node[which], ld[which], 1.f, accumulate, m, n, stage, lane, row0, col0);
    }
    __device__ __forceinline__ void operator()(float (&v)[32], float (&)[32], const Ahead&, float* stage, int lane, int batch, int row0, int col0) const
    {
        if (vec)
            rows<true>(v, stage, lane, batch, row0, col0);
        else
            rows<false>(v, stage, lane, batch, row0, col0);
    }
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
    e.m = (int32_t)g.m;
    e.n = (int32_t)g.n;
    e.split = (int32_t)(second ? g.batch / 2 : g.batch);
    e.accumulate = accumulate;
    e.vec = rows_on_16(out.p, out.ld, rows, out.node, g.batch, sizeof(T)) && rows_on_16(o2.p, o2.ld, rows, o2.node, g.batch, sizeof(T));
    return launch_gemm<P>(g, e, stream);
}

}  // namespace gpga
