// Orthogonalisation of an update by Newton-Schulz products.
//
//     X_0 = M / (|M| + eps),   X <- (a I + b A + c A^2) X with A = X X^T     (M with more rows than columns: X^T X, from the right)
//
// Three products a step: the Gram matrix A, the polynomial B = a I + b A + c A A, and B X.  A and B are symmetric, so every
// operand is read as it lies.  The matrices are held as S times their value in fp16: with |X| about 1 their entries lie
// between 1 / columns and a few units, for which fp16 has its full 11 bits.  S = 2^11 for X and B moves its range down to 2^-25
// and leaves 2^5 above one; A has 2^9, as its entries are up to 64 where singular values are up to 8.  fp32 and fp16 updates take
// two fp16 values for each (22 bits) and three products of fp16 for one, summed as fp32 would be.  bfloat16 updates of more
// than 128 rows and columns take one value and one product, a third of the time: the result is off by 1.2 to 1.4 times its own
// rounding.  Smaller ones, in which the rounding of X on the way weighs more (500 x 33: 2 times), are computed like fp32.
// X_0 is M times a power of two (nothing is lost, unless the norm is far below eps), the rest of the norm, kappa in [1, 2), is a
// factor in the first step's epilogues.
#include "gpga_orth.cuh"

#include <type_traits>

#include "gpga_pack.cuh"

namespace gpga {

namespace {

constexpr int GPGA_BF16 = 1;     // the type's code
constexpr float kScale = 2048.f, kGramScale = 512.f;   // of X and B; of A
constexpr int kSmallSide = 128;
constexpr int kNormParts = 1024;  // blocks of the sum of squares, over all matrices

// Sum of eight squares, in fp32 where that neither overflows nor vanishes.
__device__ __forceinline__ double squares(const float (&v)[8])
{
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) q = fmaf(v[k], v[k], q);
    if (q > 1e-30f && q < 1e38f) return q;
    double d = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) d += (double)v[k] * v[k];
    return d;
}

// Sum of squares of a part of a matrix: no overflow, and the order is fixed.
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
        sum += squares(v);
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

// What M is multiplied by to be S X_0: S / norm, or the power of two below it.  An infinity or NaN in M makes it NaN.
__device__ __forceinline__ double start_factor(double norm, bool whole)
{
    if (norm == 0) return 1;                   // M = 0 and eps = 0
    if (!(norm <= 1e300)) return whole ? nan("") : 1;
    int e;
    frexp(kScale / norm, &e);
    return whole ? kScale / norm : ldexp(0.5, e);
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
            factor = start_factor(norm, false);
            if (blockIdx.x == 0) kappa[blockIdx.y] = (float)(start_factor(norm, true) / factor);
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

// kappa^power factor acc + beta R (+ diagonal), as P pieces (R in as many).
template <int P>
struct KeepPieces {
    static constexpr bool kDual = false, kMirror = true, kPair = false;
    static constexpr double kTail = 1.0;
    static constexpr int kWarps = 8;
    using Columns = Nothing;
    using Factors = Nothing;
    struct Ahead {
        Raw<__half> r[P];
    };
    Pieces<__half> out, r;
    const float* kappa;
    float factor, beta, diagonal;
    int32_t power, with_r;

    __device__ __forceinline__ bool wide() const { return true; }
    __device__ __forceinline__ void one(float, int, int, int) const {}
    __device__ __forceinline__ Columns columns(int, int) const { return {}; }
    __device__ __forceinline__ static Factors factors(const Columns&) { return {}; }
    __device__ __forceinline__ void load(Ahead& ahead, int batch, int row, int col, int) const
    {
        if (with_r) r.template load<P>(batch, row, col, ahead.r);
    }
    __device__ __forceinline__ void eight(float (&v)[8], const Ahead& now, const Factors&, int batch, int row, int col, int) const
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
                for (int k = 0; k < 8; ++k) v[k] = fmaf(beta, s[k], v[k]);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (row == col + k) v[k] += diagonal;
        }
        out.template store<P>(batch, row, col, v);
    }
    __device__ __forceinline__ void put(const float (&v)[8], int batch, int row, int col) const { out.template store<P>(batch, row, col, v); }
};

// The last step: kappa^power factor acc, added to what is there or not, in the caller's type.
template <class T>
struct LastStep {
    static constexpr bool kDual = false, kMirror = false, kPair = false;
    static constexpr double kTail = 1.0;
    static constexpr int kWarps = 8;
    using Ahead = Raw<T>;
    using Columns = Nothing;
    using Factors = Nothing;
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
    __device__ __forceinline__ Columns columns(int, int) const { return {}; }
    __device__ __forceinline__ static Factors factors(const Columns&) { return {}; }
    __device__ __forceinline__ void eight(float (&v)[8], const Ahead& old, const Factors&, int batch, int row, int col, int left) const
    {
        rows(batch).eight(v, old, row, col, left);
    }
    __device__ __forceinline__ void one(float v, int batch, int row, int col) const { rows(batch).one(v, row, col); }
};

// fp16 values that a matrix is held in.
int pieces_for(const OrthParams& p) { return p.dtype == GPGA_BF16 && std::min(p.r, p.c) > kSmallSide ? 1 : 2; }

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
        o.pieces = pieces_for(p);
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

// Small matrices: one thread block does all of it, X and A (then B) in shared memory, the sums in tensor memory.  X lies as
// [smaller side, padded to 128] x [larger side, in chunks of 64]: chunk after chunk of 128 rows of 128 bytes, swizzled,
// which is an operand with rows along k for X X^T and one with rows along n for B X.  What a launch per product costs
// (about 5 us each, fifteen of them and two before) is left out: 64 x 128 fp32, 97 us that way.
constexpr int kSmallChunk = 128 * 128;   // bytes
constexpr int kSmallHead = 1024;
// Shared memory: two pieces of X and of A.
int64_t small_bytes(const OrthParams& p) { return 2 * ((std::max(p.r, p.c) + 63) / 64 + 2) * kSmallChunk + kSmallHead + 1024; }
bool small_enough(const OrthParams& p)
{
    return std::min(p.r, p.c) <= kSmallSide && std::max(p.r, p.c) <= 320 && small_bytes(p) <= kGemmSmem;
}

struct SmallParams {
    const void* m;
    void* out;
    int64_t ldm, node_ldm, ldo, node_ldo;
    double eps;
    float c1, c3, c5, scale;
    int32_t r, c, steps, accumulate, vec;   // vec: M's rows start on 16 bytes
};

// Eight values of a row to a swizzled chunk array and back, as two pieces.
__device__ __forceinline__ void put8(unsigned char* to, uint32_t piece_bytes, int row, int col, const float (&v)[8])
{
    unsigned char* const at = to + (col >> 6) * kSmallChunk + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4);
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        hi[i] = pack16(v[2 * i], v[2 * i + 1], __half());
        unpack16(hi[i], a, b, __half());
        lo[i] = pack16(v[2 * i] - a, v[2 * i + 1] - b, __half());
    }
    *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(at + piece_bytes) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}
__device__ __forceinline__ void get8(const unsigned char* from, uint32_t piece_bytes, int row, int col, float (&v)[8])
{
    const unsigned char* const at = from + (col >> 6) * kSmallChunk + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4);
    const uint4 h = *reinterpret_cast<const uint4*>(at), o = *reinterpret_cast<const uint4*>(at + piece_bytes);
    const uint32_t hi[4] = {h.x, h.y, h.z, h.w}, lo[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b, c, d;
        unpack16(hi[i], a, b, __half());
        unpack16(lo[i], c, d, __half());
        v[2 * i] = a + c;
        v[2 * i + 1] = b + d;
    }
}

template <class T>
__global__ void __launch_bounds__(256, 1) orth_small_kernel(const __grid_constant__ SmallParams p)
{
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* const smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    uint64_t* const bar = reinterpret_cast<uint64_t*>(smem);
    uint32_t* const tmem_at = reinterpret_cast<uint32_t*>(smem + 8);
    volatile uint32_t* const stop = reinterpret_cast<volatile uint32_t*>(smem + 12);
    double* const parts = reinterpret_cast<double*>(smem + 16);   // [8]
    const bool tall = p.r > p.c;
    const int s = min(p.r, p.c), l = max(p.r, p.c), chunks = (l + 63) >> 6;
    unsigned char* const x = smem + kSmallHead;
    const uint32_t x_piece = chunks * kSmallChunk, a_piece = 2 * kSmallChunk;
    unsigned char* const a = x + 2 * x_piece;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const T* const m = static_cast<const T*>(p.m) + blockIdx.x * p.node_ldm;

    if (tid == 0) {
        mbar_init(bar, 1);
        mbar_init_fence();
        *stop = 0;
    }
    if (warp == 0) tmem_alloc<1>(smem_u32(tmem_at), 512);

    // X's chunks of eight values, four of them to a thread at once, lanes along M's rows; f(row, column, values).
    const auto each_chunk = [&](const auto& f) {
        for (int i0 = tid; i0 < 128 * chunks * 8; i0 += 4 * 256) {
            Raw<T> raw[4];
            int row[4], col[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = i0 + 256 * j;
                row[j] = tall ? i & 127 : i / (chunks * 8);
                col[j] = (tall ? i >> 7 : i - row[j] * chunks * 8) * 8;
                const bool in = row[j] < s && col[j] < l;
                if (!tall && p.vec && in && col[j] + 8 <= l) {
                    raw[j].load16(m + row[j] * p.ldm + col[j]);
                } else {
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = in && col[j] + k < l ? to_f32(tall ? m[(col[j] + k) * p.ldm + row[j]] : m[row[j] * p.ldm + col[j] + k]) : 0.f;
                    raw[j].set(v);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v[8];
                raw[j].values(v);
                if (row[j] < 128) f(row[j], col[j], v);
            }
        }
    };
    // |M|, in a fixed order
    double sum = 0;
    each_chunk([&](int, int, const float(&v)[8]) { sum += squares(v); });
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) parts[warp] = sum;
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = *tmem_at;
    sum = 0;
    for (int i = 0; i < 8; ++i) sum += parts[i];
    const double factor = start_factor(sqrt(sum) + p.eps, true);

    // X_0, zeros around it
    each_chunk([&](int row, int col, float(&v)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (float)(v[k] * factor);
        put8(x, x_piece, row, col, v);
    });

    const WaitState w{stop};
    const int quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    uint32_t parity = 0;
    // D = A B over `count` k-steps of 16, the small products of pieces first.  A's rows run along k (32 bytes a step, a chunk
    // after four), B's too or (b_mn) along n.
    const auto multiply = [&](uint32_t d, uint64_t a0, uint32_t pa, uint64_t b0, uint32_t pb, bool b_mn, int n, int count) {
        const uint32_t idesc = mma_descriptor(128, n, true, false, b_mn), b_step = b_mn ? 2048 >> 4 : 32 >> 4, b_chunk = b_mn ? 8192 >> 4 : kSmallChunk >> 4;
        uint32_t add = 0;
#pragma unroll 1
        for (int q = 0; q < 3; ++q) {     // (1, 0), (0, 1), (0, 0)
            uint64_t da = a0 + (q == 0 ? pa >> 4 : 0), db = b0 + (q == 1 ? pb >> 4 : 0);
#pragma unroll 1
            for (int k = 0; k < count; k += 4, da += kSmallChunk >> 4, db += b_chunk)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (k + j < count) {
                        mma_f16<1>(d, da + j * (32 >> 4), db + j * b_step, idesc, add);
                        add = 1;
                    }
        }
    };
    // What the block has written to shared memory is there for the matrix unit, and what it has read of tensor memory is read.
    const auto hand_over = [&] {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tmem_fence_before();
        __syncthreads();
        tmem_fence_after();
    };
    const auto finished = [&] {
        w.wait(smem_u32(bar), parity);
        parity ^= 1;
        tmem_fence_after();
    };
    const uint32_t xs = smem_u32(x), as = smem_u32(a);
    const uint64_t xk = tile_descriptor(xs, false), xn = tile_descriptor(xs, true, kSmallChunk), ak = tile_descriptor(as, false);
    const int side = (s + 15) >> 4, square = side * 16, wide = chunks * 64;   // columns of A and B that are used; of X
    for (int step = 0; step < p.steps; ++step) {
        hand_over();
        if (tid == 0) {                                       // A = X X^T
            multiply(tmem, xk, x_piece, xk, x_piece, false, square, (l + 15) >> 4);
            mma_commit<1>(smem_u32(bar));
        }
        finished();
#pragma unroll 1
        for (int c = 32 * half; c < square; c += 64) {
            float v[32];
            tmem_load32(lanes + c, v);
            tmem_wait_load();
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = v[j + k] * (kGramScale / (kScale * kScale));
                put8(a, a_piece, row, c + j, o);
            }
        }
        hand_over();
        if (tid == 0) {                                       // B = c1 I + c3 A + c5 A A, in A's place
            multiply(tmem, ak, a_piece, ak, a_piece, false, square, side);
            mma_commit<1>(smem_u32(bar));
        }
        finished();
#pragma unroll 1
        for (int c = 32 * half; c < square; c += 64) {
            float v[32];
            tmem_load32(lanes + c, v);
            tmem_wait_load();
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                float o[8];
                get8(a, a_piece, row, c + j, o);
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = p.c5 * (kScale / (kGramScale * kGramScale)) * v[j + k] + p.c3 * (kScale / kGramScale) * o[k] + (row == c + j + k ? p.c1 * kScale : 0.f);
                put8(a, a_piece, row, c + j, o);
            }
        }
        hand_over();
        if (tid == 0) {                                       // B X, 256 columns to an instruction
            for (int n = 0; n < wide; n += 256)
                multiply(tmem + n, ak, a_piece, xn + (n >> 6) * (kSmallChunk >> 4), x_piece, true, min(256, wide - n), side);
            mma_commit<1>(smem_u32(bar));
        }
        finished();
        const bool last = step + 1 == p.steps;
#pragma unroll 1
        for (int c = 32 * half; c < wide; c += 64) {
            float v[32];
            tmem_load32(lanes + c, v);
            tmem_wait_load();
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = v[j + k] * (1.f / kScale);
                if (!last) put8(x, x_piece, row, c + j, o);
            }
            if (last && row < s) {
                T* const out = static_cast<T*>(p.out) + blockIdx.x * p.node_ldo;
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    if (c + j >= l) break;
                    T* const at = out + (tall ? (c + j) * p.ldo + row : row * p.ldo + c + j);
                    const float o = v[j] * (p.scale / (kScale * kScale));
                    *at = from_f32<T>(p.accumulate ? to_f32(*at) + o : o);
                }
            }
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 0) {
        tmem_fence_after();
        tmem_free<1>(tmem, 512);
    }
}

// A wait that runs out: nothing arrives at its barrier.
__global__ void wait_selftest_kernel()
{
    __shared__ __align__(8) uint64_t bar;
    __shared__ uint32_t stop;
    mbar_init(&bar, 1);
    mbar_init_fence();
    stop = 0;
    const WaitState w{&stop, 64};
    w.wait(smem_u32(&bar), 0);
}

template <class T>
cudaError_t orth_small(const OrthParams& p, cudaStream_t stream)
{
    SmallParams q;
    q.m = p.m;
    q.out = p.out;
    q.ldm = p.ldm;
    q.node_ldm = p.node_ldm;
    q.ldo = p.ldo;
    q.node_ldo = p.node_ldo;
    q.eps = p.eps;
    q.c1 = (float)p.c1;
    q.c3 = (float)p.c3;
    q.c5 = (float)p.c5;
    q.scale = (float)p.scale;
    q.r = (int32_t)p.r;
    q.c = (int32_t)p.c;
    q.steps = (int32_t)p.steps;
    q.accumulate = p.accumulate;
    q.vec = rows_on_16(p.m, p.ldm, p.r, p.node_ldm, p.nodes, sizeof(T));
    static std::atomic<unsigned long long> limit_set{0};
    const cudaError_t e = ensure_smem_limit(orth_small_kernel<T>, kGemmSmem, limit_set);
    if (e != cudaSuccess) return e;
    orth_small_kernel<T><<<(unsigned)p.nodes, 256, (size_t)small_bytes(p), stream>>>(q);
    return cudaGetLastError();
}

template <class T, int P>
cudaError_t orth(const OrthParams& p, cudaStream_t stream)
{
    const OrthPlan q = plan_orth(p);
    const T* m = static_cast<const T*>(p.m);
    const int vec = rows_on_16(p.m, p.ldm, p.r, p.node_ldm, p.nodes, sizeof(T));
    square_sum_kernel<T><<<dim3(q.count_parts, (unsigned)p.nodes), 256, 0, stream>>>(m, p.ldm, p.node_ldm, p.r, p.c, vec, q.parts);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>((p.r * ((p.c + 7) / 8) + 255) / 256, (int64_t)sm_count() * 8 / std::min<int64_t>(p.nodes, 64)));
    start_kernel<T, P><<<dim3((unsigned)blocks, (unsigned)p.nodes), 256, 0, stream>>>(m, p.ldm, p.node_ldm, p.r, p.c, vec, q.parts, q.count_parts, p.eps,
                                                                              pieces_of<__half>(q.x[0]), q.kappa);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;

    const bool tall = p.r > p.c;
    const int64_t s = std::min(p.r, p.c);
    GemmPlan g;
    g.half = true;
    g.batch = g.bmod = p.nodes;
    g.after = true;
    for (int64_t i = 0; i < p.steps; ++i) {
        const Operand &x = q.x[i & 1], &next = q.x[~i & 1];
        const int first = i == 0;
        KeepPieces<P> keep;
        keep.kappa = q.kappa;
        g.a[0] = g.b[0] = x;                            // A
        g.a[0].mn_major = g.b[0].mn_major = tall;
        g.m = g.n = s;
        g.k = std::max(p.r, p.c);
        g.symmetric = true;
        keep.out = keep.r = pieces_of<__half>(q.a);
        keep.factor = kGramScale / (kScale * kScale);
        keep.beta = keep.diagonal = 0.f;
        keep.power = first ? 2 : 0;
        keep.with_r = 0;
        if ((e = launch_gemm<P, __half>(g, keep, stream)) != cudaSuccess) return e;
        g.a[0] = g.b[0] = q.a;                          // B = a I + b A + c A A
        g.a[0].mn_major = g.b[0].mn_major = false;
        g.k = s;
        keep.out = pieces_of<__half>(q.b);
        keep.factor = (float)(p.c5 * (kScale / (kGramScale * kGramScale)));
        keep.beta = (float)(p.c3 * (kScale / kGramScale));
        keep.diagonal = (float)(p.c1 * kScale);
        keep.power = 0;
        keep.with_r = 1;
        if ((e = launch_gemm<P, __half>(g, keep, stream)) != cudaSuccess) return e;
        g.a[0] = tall ? x : q.b;                        // B X or X B
        g.b[0] = tall ? q.b : x;
        g.a[0].mn_major = false;
        g.b[0].mn_major = !tall;
        g.m = p.r;
        g.n = p.c;
        g.k = s;
        g.symmetric = false;
        if (i + 1 < p.steps) {
            keep.out = pieces_of<__half>(next);
            keep.factor = 1.f / kScale;
            keep.power = first;
            keep.with_r = 0;
            if ((e = launch_gemm<P, __half>(g, keep, stream)) != cudaSuccess) return e;
        } else {
            LastStep<T> last;
            last.out = static_cast<T*>(p.out);
            last.ld = p.ldo;
            last.node = p.node_ldo;
            last.kappa = q.kappa;
            last.factor = (float)(p.scale / ((double)kScale * kScale));
            last.power = first;
            last.accumulate = p.accumulate;
            last.vec = rows_on_16(p.out, p.ldo, p.r, p.node_ldo, p.nodes, sizeof(T));
            if ((e = launch_gemm<P, T>(g, last, stream)) != cudaSuccess) return e;
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

cudaError_t launch_wait_selftest(cudaStream_t stream)
{
    wait_selftest_kernel<<<1, 1, 0, stream>>>();
    return cudaGetLastError();
}

int64_t orth_scratch_bytes(const OrthParams& p) { return small_enough(p) ? 0 : plan_orth(p).scratch.bytes; }

cudaError_t launch_orth(const OrthParams& p, cudaStream_t stream)
{
    const bool small = small_enough(p);
    if (p.dtype == 0) return small ? orth_small<float>(p, stream) : orth<float, 2>(p, stream);
    if (p.dtype == 2) return small ? orth_small<__half>(p, stream) : orth<__half, 2>(p, stream);
    if (small) return orth_small<__nv_bfloat16>(p, stream);
    return pieces_for(p) == 1 ? orth<__nv_bfloat16, 1>(p, stream) : orth<__nv_bfloat16, 2>(p, stream);
}

}  // namespace gpga
