// Gated feed-forward block of few tokens per node (a trained model answering): every weight is read once, straight from where it lies,
// and that is what bounds it.
//
// Two launches, h = act(x Wg^T) (x Wu^T) and y = h Wd^T.  16-bit activations: the weights are the rows of m16n8k16 matrix
// instructions (eight of the gate and the same eight of the other projection, or sixteen of Wd) and the tokens their
// columns; as a sum over k may run in any order, a lane takes eight neighbouring k and both operands use them in the same
// places of two instructions.  The tensor memory path would need 128 rows at a time; at up to 32 tokens the instructions
// are not what bounds.  A block's warps take a part of k each and add up through shared memory, in a fixed order.
//
// Rows on 16 bytes are streamed: every warp has 12 to 14 KB of its part on the way to its own ring in shared memory all the time,
// across the tiles that a block goes through (24 tokens, 2048 x 5632, fp32 weights, 138 MB: 38.5 us; 9 us more with loads to
// registers; one token 29 us, 4.8 TB/s).  With more tokens the reading of x for every tile (from L2) adds 3 us for
// each eight of them.
// Others are loaded as they lie, on clusters of blocks where there are few tiles.  fp32 activations: fp32 arithmetic.  The
// second launch begins to read its weights while the first runs.
#include <type_traits>

#include "gpga_ff_device.cuh"

namespace gpga {

namespace {

struct FewParams {
    const void *x, *w1, *w2;        // w2: the second projection (nullptr: only one product)
    int64_t ldx, ld1, node1, ld2, node2;
    void *out, *g, *u;              // out: h or y
    int64_t ldo, ldg, ldu;
    int64_t lo;                     // h: elements from its values to the rests of their rounding (0: not kept)
    int32_t tokens, rows, k, kind, vec_x, vec_w, after, blocks;   // rows: of the weights; blocks: of a cluster
};

template <class T>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2])
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// Eight weights as four pairs of the activations' type; fp32 ones as the sum of two (16 bits more than make a difference).
template <class T, class W, int Q>
__device__ __forceinline__ void as_pairs(const Raw<W>& r, uint32_t (&o)[Q][4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(W) == 2) {
            o[0][i] = r.w[i];
        } else {
            const float x = __uint_as_float(r.w[2 * i]), y = __uint_as_float(r.w[2 * i + 1]);
            float a, b;
            o[0][i] = pack16_finite(x, y, T());
            unpack16(o[0][i], a, b, T());
            o[1][i] = pack16(x - a, y - b, T());
        }
    }
}

// What is done with a finished sum of both projections (or of the one): g, u, h, or y.
template <class T, bool GATE>
__device__ __forceinline__ void finish(const FewParams& p, int node, int token, int row, float a, float b)
{
    const int64_t t = (int64_t)node * p.tokens + token;
    if constexpr (GATE) {
        if (p.g) {
            static_cast<T*>(p.g)[t * p.ldg + row] = from_f32<T>(a);
            static_cast<T*>(p.u)[t * p.ldu + row] = from_f32<T>(b);
        }
        float v[1] = {a};
        act_values<sizeof(T) == 2>(v, p.kind);
        const float h = v[0] * b;
        T* const at = static_cast<T*>(p.out) + t * p.ldo + row;
        *at = from_f32<T>(h);
        if (sizeof(T) == 2 && p.lo) {
            const float rounded = to_f32(*at);    // no rest beside an infinity: it could be NaN
            at[p.lo] = from_f32<T>(fabsf(rounded) <= 3.4028234e38f ? h - rounded : 0.f);
        }
    } else {
        static_cast<T*>(p.out)[t * p.ldo + row] = from_f32<T>(a);
    }
}

// Asks for this warp's part of the weights while the kernel before it runs.
template <class W, int ROWS>
__device__ __forceinline__ void ask_ahead(const W* w, int64_t ld, int row0, int rows, int k0, int k1, int lane)
{
    if (k0 >= k1) return;
    const int bytes = (k1 - k0) * (int)sizeof(W), lines = (bytes + 127) / 128 + 1;
    for (int i = lane; i < ROWS * lines; i += 32) {
        const int r = i / lines, l = i - r * lines;
        if (row0 + r >= rows) break;
        const char* const at = reinterpret_cast<const char*>(w + (row0 + r) * ld + k0);
        asm volatile("prefetch.global.L2 [%0];" ::"l"(at + min(l * 128, bytes - 1)));
    }
}

constexpr int kFewWarps = 8;
// Terms that the matrix instructions add to one sum (they cut off what they add, see gpga_gemm.cuh): 256 instructions, whose
// drift is at most a sixteenth of fp16's half step.  LONG: where a warp has more, they are added to its own in fp32 (in a kernel of
// its own: 24 tokens, 2048 x 5632, fp32 weights 38.4 us, 41.1 us with that in the same loop).
constexpr int kFewSum = 4096;
inline bool few_long(int k) { return k > kFewWarps * kFewSum; }

// Sum of value i of every warp of the cluster, in the order of k.  sums: this block's [warp][count].
__device__ __forceinline__ float cluster_sum(const float* sums, int i, int count, uint32_t blocks)
{
    float s = 0.f;
    for (uint32_t b = 0; b < blocks; ++b) {
        const uint32_t at = map_shared(smem_u32(sums + i), b);
#pragma unroll
        for (int v = 0; v < kFewWarps; ++v) {
            float x;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at + 4 * v * count));
            s += x;
        }
    }
    return s;
}

// NT tiles of eight tokens; XP = 2: x is h with the rests of its rounding.
template <class T, class W, int NT, bool GATE, int XP, bool LONG>
__global__ void __launch_bounds__(kFewWarps * 32) few_tokens_kernel(const __grid_constant__ FewParams p)
{
    constexpr int M = GATE ? 2 : 1, R = 16, N = 8 * NT;
    constexpr int S = R + 4;   // a token's rows in `sums`: no two lanes of a store meet in a bank
    __shared__ __align__(16) float sums[kFewWarps * M * N * S];   // [warp][array][token][row]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, node = blockIdx.y, row0 = (int)(blockIdx.x / p.blocks) * R;
    const int group = lane >> 2, place = (lane & 3) * 8;
    const uint32_t rank = cluster_rank();
    const int parts = kFewWarps * p.blocks, steps = (p.k + 31) / 32, each = (steps + parts - 1) / parts;
    const int k0 = min(((int)rank * kFewWarps + warp) * each * 32, p.k), k1 = min(k0 + each * 32, p.k);
    const W* w[M];
    int64_t ld[M];
    w[0] = static_cast<const W*>(p.w1) + node * p.node1;
    ld[0] = p.ld1;
    if constexpr (GATE) {
        w[1] = static_cast<const W*>(p.w2) + node * p.node2;
        ld[1] = p.ld2;
    }
    grid_launch_dependents();
    if (p.after) {
        ask_ahead<W, R>(w[0], ld[0], row0, p.rows, k0, k1, lane);
        grid_dependency_wait();
    }
    const T* const x = static_cast<const T*>(p.x) + (int64_t)node * p.tokens * p.ldx;

    // Rows and tokens past the last are read as the last: their sums are dropped.
    const W* wr[M][2];
    const T* xr[NT];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) wr[m][h] = w[m] + min(row0 + 8 * h + group, p.rows - 1) * ld[m] + place;
#pragma unroll
    for (int n = 0; n < NT; ++n) xr[n] = x + min(8 * n + group, p.tokens - 1) * p.ldx + place;
    float acc[M][NT][4] = {}, whole[LONG ? M : 1][NT][4] = {};
    const auto add_up = [&] {
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) whole[LONG ? m : 0][n][e] += acc[m][n][e], acc[m][n][e] = 0.f;
    };
    const auto multiply = [&](const Raw<W>(&wv)[M][2], const Raw<T>(&xv)[XP][NT]) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            constexpr int Q = sizeof(W) / 2;
            uint32_t lo[Q][4], hi[Q][4];
            as_pairs<T>(wv[m][0], lo);
            as_pairs<T>(wv[m][1], hi);
#pragma unroll
            for (int q = Q - 1; q >= 0; --q)
#pragma unroll
                for (int z = XP - 1; z >= 0; --z) {
                    if (q + z > 1) continue;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const uint32_t a[4] = {lo[q][2 * s], hi[q][2 * s], lo[q][2 * s + 1], hi[q][2 * s + 1]};
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint32_t b[2] = {xv[z][n].w[2 * s], xv[z][n].w[2 * s + 1]};
                            mma16816<T>(acc[m][n], a, b);
                        }
                    }
                }
        }
    };
#pragma unroll 1
    for (int k = k0; k < k1; k += 32) {
        Raw<W> wv[M][2];
        Raw<T> xv[XP][NT];
        const int left = p.k - k - place;
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) wv[m][h].load(wr[m][h] + k, left, p.vec_w);
#pragma unroll
        for (int z = 0; z < XP; ++z)
#pragma unroll
            for (int n = 0; n < NT; ++n) xv[z][n].load(xr[n] + z * p.lo + k, left, p.vec_x);
        multiply(wv, xv);
        if constexpr (LONG)
            if ((k - k0 + 32) % kFewSum == 0) add_up();
    }
    if constexpr (LONG) add_up();
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[((warp * M + m) * N + 8 * n + 2 * (lane & 3) + (e & 1)) * S + 8 * (e >> 1) + group] = LONG ? whole[LONG ? m : 0][n][e] : acc[m][n][e];
    cluster_barrier();
    for (int i = (int)rank * kFewWarps * 32 + threadIdx.x; i < R * N; i += p.blocks * kFewWarps * 32) {
        const int r = i % R, n = i / R;
        if (row0 + r >= p.rows || n >= p.tokens) continue;
        float s[M];
#pragma unroll
        for (int m = 0; m < M; ++m) s[m] = cluster_sum(sums, (m * N + n) * S + r, M * N * S, p.blocks);
        finish<T, GATE>(p, node, n, row0 + r, s[0], s[M - 1]);
    }
    cluster_farewell();   // nobody goes while its sums are read
}

// Streamed: 16 rows of weights and 64 of k to a stage.
constexpr int kStreamK = 64;
template <class W> constexpr int kStreamStages = sizeof(W) == 4 ? 4 : 8;
template <class W> constexpr int kStreamStage = 16 * kStreamK * (int)sizeof(W);   // bytes

template <class T, class W, int NT, bool GATE, int XP, bool LONG>
__global__ void __launch_bounds__(kFewWarps * 32) few_streamed_kernel(const __grid_constant__ FewParams p)
{
    constexpr int N = 8 * NT, S = 16 + 4, stages = kStreamStages<W>, stage_bytes = kStreamStage<W>;
    constexpr int G = kStreamK * (int)sizeof(W) / 16;    // 16-byte groups of a row
    extern __shared__ __align__(16) unsigned char shared[];
    float* const sums = reinterpret_cast<float*>(shared + kFewWarps * stages * stage_bytes);   // [tile & 1][warp][token][row]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, node = blockIdx.y;
    const int group = lane >> 2, quad = lane & 3;
    unsigned char* const ring = shared + warp * stages * stage_bytes;
    const int tiles = GATE ? (p.rows + 7) / 8 : (p.rows + 15) / 16;
    const int steps = (p.k + kStreamK - 1) / kStreamK, each = (steps + kFewWarps - 1) / kFewWarps;
    const int s0 = min(warp * each, steps), mine = min(each, steps - s0);   // steps of k of this warp
    const W* const w1 = static_cast<const W*>(p.w1) + node * p.node1;
    const W* const w2 = GATE ? static_cast<const W*>(p.w2) + node * p.node2 : nullptr;
    grid_launch_dependents();

    // rows 0 to 7 of a stage: of the gate, 8 to 15 of the other (or 16 of the one); neighbouring rows' groups change places
    const auto swizzle = [](int r) { return sizeof(W) == 4 ? r & 7 : 4 * (r & 1); };
    int ask_tile = blockIdx.x, ask_step = 0, ask_slot = 0;
    const auto ask = [&] {
        if (mine > 0 && ask_tile < tiles) {
            const int k0 = (s0 + ask_step) * kStreamK;
#pragma unroll
            for (int i = 0; i < 16 * G / 32; ++i) {
                const int at = i * 32 + lane, r = at / G, g = at % G;
                const int row = GATE ? min(ask_tile * 8 + (r & 7), p.rows - 1) : min(ask_tile * 16 + r, p.rows - 1);
                const int k = k0 + g * (16 / (int)sizeof(W)), bytes = max(0, min(16, (p.k - k) * (int)sizeof(W)));
                const W* const from = GATE && r >= 8 ? w2 + row * p.ld2 : w1 + row * p.ld1;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(ring + ask_slot * stage_bytes + r * (G * 16) + ((g ^ swizzle(r)) << 4))),
                             "l"(from + (bytes ? k : 0)), "r"(bytes)
                             : "memory");
            }
            if (++ask_step == mine) ask_step = 0, ask_tile += gridDim.x;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++ask_slot == stages) ask_slot = 0;
    };
#pragma unroll 1
    for (int i = 0; i < stages - 1; ++i) ask();
    if (p.after) grid_dependency_wait();

    const T* const x = static_cast<const T*>(p.x) + (int64_t)node * p.tokens * p.ldx + quad * 8;
    const T* xr[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) xr[n] = x + min(8 * n + group, p.tokens - 1) * p.ldx;
    int slot = 0, turn = 0;
#pragma unroll 1
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, turn ^= 1) {
        float acc[NT][4] = {}, whole[NT][4] = {};
        const auto add_up = [&] {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) whole[n][e] += acc[n][e], acc[n][e] = 0.f;
        };
#pragma unroll 1
        for (int step = 0; step < mine; ++step) {
            const int k0 = (s0 + step) * kStreamK;
            Raw<T> xv[2][XP][NT];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int z = 0; z < XP; ++z)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const int k = k0 + 32 * h, left = p.k - k - quad * 8;
                        if (left >= 8)
                            xv[h][z][n].load16(xr[n] + z * p.lo + k);
                        else
                            xv[h][z][n].load(xr[n] + z * p.lo + k, left, false);
                    }
            asm volatile("cp.async.wait_group %0;" ::"n"(stages - 2) : "memory");
            __syncwarp();
            ask();      // into the slot that the step before this one was read from
            const unsigned char* const stage = ring + slot * stage_bytes;
            if (++slot == stages) slot = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                constexpr int Q = sizeof(W) / 2;
                uint32_t lo[Q][4], hi[Q][4];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int r = group + 8 * half;
                    Raw<W> wv;
#pragma unroll
                    for (int i = 0; i < Q; ++i) {
                        const int g = (32 * h + 8 * quad) * (int)sizeof(W) / 16 + i;
                        const uint4 v = *reinterpret_cast<const uint4*>(stage + r * (G * 16) + ((g ^ swizzle(r)) << 4));
                        wv.w[4 * i] = v.x, wv.w[4 * i + 1] = v.y, wv.w[4 * i + 2] = v.z, wv.w[4 * i + 3] = v.w;
                    }
                    if (half)
                        as_pairs<T>(wv, hi);
                    else
                        as_pairs<T>(wv, lo);
                }
#pragma unroll
                for (int q = Q - 1; q >= 0; --q)
#pragma unroll
                    for (int z = XP - 1; z >= 0; --z) {
                        if (q + z > 1) continue;
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const uint32_t a[4] = {lo[q][2 * s], hi[q][2 * s], lo[q][2 * s + 1], hi[q][2 * s + 1]};
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                const uint32_t b[2] = {xv[h][z][n].w[2 * s], xv[h][z][n].w[2 * s + 1]};
                                mma16816<T>(acc[n], a, b);
                            }
                        }
                    }
            }
            __syncwarp();
            if constexpr (LONG)
                if ((step + 1) % (kFewSum / kStreamK) == 0) add_up();
        }
        if constexpr (LONG) add_up();
        float* const here = sums + turn * kFewWarps * N * S;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) here[(warp * N + 8 * n + 2 * quad + (e & 1)) * S + 8 * (e >> 1) + group] = LONG ? whole[n][e] : acc[n][e];
        __syncthreads();
        constexpr int R = GATE ? 8 : 16;
        for (int i = threadIdx.x; i < R * N; i += kFewWarps * 32) {
            const int r = i % R, n = i / R, row = tile * R + r;
            if (row >= p.rows || n >= p.tokens) continue;
            float a = 0.f, b = 0.f;
#pragma unroll
            for (int v = 0; v < kFewWarps; ++v) {
                a += here[(v * N + n) * S + r];
                if constexpr (GATE) b += here[(v * N + n) * S + r + 8];
            }
            finish<T, GATE>(p, node, n, row, a, b);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

template <class T, class W, int NT, bool GATE, int XP, bool LONG>
cudaError_t launch_streamed(FewParams p, int64_t nodes, cudaStream_t stream)
{
    constexpr int bytes = kFewWarps * (kStreamStages<W> * kStreamStage<W> + 2 * 8 * NT * 20 * 4);
    const auto kernel = few_streamed_kernel<T, W, NT, GATE, XP, LONG>;
    static std::atomic<unsigned long long> limit_set{0};
    const cudaError_t e = ensure_smem_limit(kernel, bytes, limit_set);
    if (e != cudaSuccess) return e;
    const int64_t tiles = (p.rows + (GATE ? 7 : 15)) / (GATE ? 8 : 16), blocks = std::max<int64_t>(1, std::min<int64_t>(tiles, (sm_count() + nodes - 1) / nodes));
    return launch_after_trigger(kernel, dim3((unsigned)blocks, (unsigned)nodes), dim3(kFewWarps * 32), bytes, stream, p.after != 0, p);
}

// fp32: R rows of the weights and N tokens to a block, its warps a part of k each.
template <int N, bool GATE>
__global__ void __launch_bounds__(kFewWarps * 32) few_tokens_f32_kernel(const __grid_constant__ FewParams p)
{
    constexpr int M = GATE ? 2 : 1, R = 4;
    __shared__ __align__(16) float sums[kFewWarps * M * R * N];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, node = blockIdx.y, row0 = (int)(blockIdx.x / p.blocks) * R;
    const uint32_t rank = cluster_rank();
    const int parts = kFewWarps * p.blocks, steps = (p.k + 127) / 128, each = (steps + parts - 1) / parts;
    const int k0 = min(((int)rank * kFewWarps + warp) * each * 128, p.k), k1 = min(k0 + each * 128, p.k);
    const float* w[M];
    int64_t ld[M];
    w[0] = static_cast<const float*>(p.w1) + node * p.node1;
    ld[0] = p.ld1;
    if constexpr (GATE) {
        w[1] = static_cast<const float*>(p.w2) + node * p.node2;
        ld[1] = p.ld2;
    }
    grid_launch_dependents();
    if (p.after) {
        ask_ahead<float, R>(w[0], ld[0], row0, p.rows, k0, k1, lane);
        grid_dependency_wait();
    }
    const float* const x = static_cast<const float*>(p.x) + (int64_t)node * p.tokens * p.ldx;
    const auto four = [](const float* q, int n) {
        if (n >= 4) return make_float4(q[0], q[1], q[2], q[3]);
        return make_float4(n > 0 ? q[0] : 0.f, n > 1 ? q[1] : 0.f, n > 2 ? q[2] : 0.f, 0.f);
    };
    // Rows and tokens past the last are read as the last: their sums are dropped.
    const float* wr[M][R];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) wr[m][r] = w[m] + min(row0 + r, p.rows - 1) * ld[m] + 4 * lane;
    float acc[M][R][N] = {};
    const auto multiply = [&](const float4(&wv)[M][R], int n, const float4& v) {
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int r = 0; r < R; ++r)
                acc[m][r][n] = fmaf(wv[m][r].w, v.w, fmaf(wv[m][r].z, v.z, fmaf(wv[m][r].y, v.y, fmaf(wv[m][r].x, v.x, acc[m][r][n]))));
    };
    int k = k0;
    if (p.vec_w && p.vec_x)
        for (; k + 128 <= min(k1, p.k); k += 128) {
            float4 wv[M][R];
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int r = 0; r < R; ++r) wv[m][r] = *reinterpret_cast<const float4*>(wr[m][r] + k);
#pragma unroll
            for (int n = 0; n < N; ++n) multiply(wv, n, *reinterpret_cast<const float4*>(x + min(n, p.tokens - 1) * p.ldx + 4 * lane + k));
        }
#pragma unroll 1
    for (; k < k1; k += 128) {
        const int left = p.k - k - 4 * lane;
        float4 wv[M][R];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int r = 0; r < R; ++r) wv[m][r] = four(wr[m][r] + k, left);
#pragma unroll
        for (int n = 0; n < N; ++n) multiply(wv, n, four(x + min(n, p.tokens - 1) * p.ldx + 4 * lane + k, left));
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float s = acc[m][r][n];
#pragma unroll
                for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
                if (lane == 0) sums[(warp * M * R + m * R + r) * N + n] = s;
            }
    cluster_barrier();
    const int i = (int)rank * kFewWarps * 32 + threadIdx.x;
    if (i < R * N) {
        const int r = i % R, n = i / R;
        if (row0 + r < p.rows && n < p.tokens) {
            float s[M];
#pragma unroll
            for (int m = 0; m < M; ++m) s[m] = cluster_sum(sums, (m * R + r) * N + n, M * R * N, p.blocks);
            finish<float, GATE>(p, node, n, row0 + r, s[0], s[M - 1]);
        }
    }
    cluster_barrier();
}

// Blocks of a cluster: more while the launch has less than a block per SM and every warp still has two steps of k.
cudaError_t launch_clusters(void (*kernel)(FewParams), FewParams p, int rows, int step, int64_t nodes, cudaStream_t stream)
{
    const int64_t tiles = (p.rows + rows - 1) / rows;
    p.blocks = 1;
    while (p.blocks < 8 && tiles * nodes * p.blocks < sm_count() && p.k >= p.blocks * 2 * kFewWarps * step * 2) p.blocks *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * p.blocks), (unsigned)nodes);
    cfg.blockDim = dim3(kFewWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.blocks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.after ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <class T, class W, bool GATE, bool LONG>
cudaError_t few16_as(const FewParams& p, int64_t nodes, cudaStream_t stream)
{
    constexpr int XP = GATE ? 1 : 2;   // up to eight tokens h comes with the rests of its rounding
    if (p.vec_w && p.vec_x)
        return p.tokens <= 8    ? launch_streamed<T, W, 1, GATE, XP, LONG>(p, nodes, stream)
               : p.tokens <= 16 ? launch_streamed<T, W, 2, GATE, 1, LONG>(p, nodes, stream)
                                : launch_streamed<T, W, 4, GATE, 1, LONG>(p, nodes, stream);
    const auto kernel = p.tokens <= 8    ? few_tokens_kernel<T, W, 1, GATE, XP, LONG>
                        : p.tokens <= 16 ? few_tokens_kernel<T, W, 2, GATE, 1, LONG>
                                         : few_tokens_kernel<T, W, 4, GATE, 1, LONG>;
    return launch_clusters(kernel, p, 16, 32, nodes, stream);
}
template <class T, class W, bool GATE>
cudaError_t few16(const FewParams& p, int64_t nodes, cudaStream_t stream)
{
    return few_long(p.k) ? few16_as<T, W, GATE, true>(p, nodes, stream) : few16_as<T, W, GATE, false>(p, nodes, stream);
}

template <bool GATE>
cudaError_t few32(const FewParams& p, int64_t nodes, cudaStream_t stream)
{
    const auto kernel = p.tokens == 1 ? few_tokens_f32_kernel<1, GATE> : p.tokens <= 4 ? few_tokens_f32_kernel<4, GATE> : few_tokens_f32_kernel<8, GATE>;
    return launch_clusters(kernel, p, 4, 128, nodes, stream);
}

template <bool GATE>
cudaError_t few(const FeedForwardParams& q, const FewParams& p, cudaStream_t stream)
{
    if (q.dtype == 0) return few32<GATE>(p, q.nodes, stream);
    if (q.dtype == 1) return q.weight_dtype == 0 ? few16<__nv_bfloat16, float, GATE>(p, q.nodes, stream) : few16<__nv_bfloat16, __nv_bfloat16, GATE>(p, q.nodes, stream);
    return q.weight_dtype == 0 ? few16<__half, float, GATE>(p, q.nodes, stream) : few16<__half, __half, GATE>(p, q.nodes, stream);
}

}  // namespace

// h: fp32, or 16 bits, of up to eight tokens with the rests of its rounding (the second launch is bound by its weights, and y is
// rounded once then).
int64_t ff_few_scratch_bytes(const FeedForwardParams& p) { return p.nodes * p.rows * ((p.f + 7) / 8 * 8) * (p.dtype == 0 || p.rows <= 8 ? 4 : 2); }

cudaError_t launch_ff_few(const FeedForwardParams& q, cudaStream_t stream)
{
    const int size = q.dtype == 0 ? 4 : 2, wsize = q.weight_dtype == 0 ? 4 : 2;
    const int64_t ldh = (q.f + 7) / 8 * 8;
    FewParams p;
    p.x = q.x.p;
    p.ldx = q.x.ld;
    p.vec_x = rows_on_16(q.x.p, q.x.ld, q.nodes * q.rows, 0, 1, size);
    p.w1 = q.gate.p;
    p.ld1 = q.gate.ld;
    p.node1 = q.gate.node;
    p.w2 = q.up.p;
    p.ld2 = q.up.ld;
    p.node2 = q.up.node;
    p.vec_w = rows_on_16(q.gate.p, q.gate.ld, q.f, q.gate.node, q.nodes, wsize) && rows_on_16(q.up.p, q.up.ld, q.f, q.up.node, q.nodes, wsize);
    p.out = q.scratch;
    p.ldo = ldh;
    p.lo = q.dtype != 0 && q.rows <= 8 ? q.nodes * q.rows * ldh : 0;
    p.g = q.g.p;
    p.u = q.u.p;
    p.ldg = q.g.ld;
    p.ldu = q.u.ld;
    p.tokens = (int32_t)q.rows;
    p.rows = (int32_t)q.f;
    p.k = (int32_t)q.d;
    p.kind = q.activation;
    p.after = 0;
    const cudaError_t e = few<true>(q, p, stream);
    if (e != cudaSuccess) return e;
    p.x = q.scratch;
    p.ldx = ldh;
    p.vec_x = 1;
    p.w1 = q.down.p;
    p.ld1 = q.down.ld;
    p.node1 = q.down.node;
    p.vec_w = rows_on_16(q.down.p, q.down.ld, q.d, q.down.node, q.nodes, wsize);
    p.out = q.y.p;
    p.ldo = q.y.ld;
    p.g = p.u = nullptr;
    p.rows = (int32_t)q.d;
    p.k = (int32_t)q.f;
    p.after = 1;
    return few<false>(q, p, stream);
}

}  // namespace gpga
