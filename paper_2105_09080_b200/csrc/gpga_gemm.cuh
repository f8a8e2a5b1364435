// Matrix products of the token-block operators: one persistent kernel for all of them, with an epilogue per use.
//
//     acc(i, j) = sum over k of A(i, k) B(j, k), per node ("batch"), then Epi.
//
// Operands are 16-bit arrays that tiled asynchronous copies bring to shared memory: rows along k, or (mn_major) rows along i
// or j, so no operand is ever transposed in memory.  An operand may be the sum of P arrays of 16 bits ("pieces": a float32
// value is exactly three bfloat16 values); then the products of pieces p + q < P are summed, six of them for P = 3.
// A sum may run over two pairs of operands, and over two pieces of B with one of A (segments), and a tile's columns may
// come from two arrays (DUAL: the left half from B[0], the right half from B[1]), so that both projections of a gate end in
// one thread's registers.  A symmetric product is computed on and above the diagonal and stored twice.
//
// A tile is 128 CG rows by bn columns on CG thread blocks.  Warp 0 loads, warp 1 of the leading block issues the matrix
// instructions, warps 4 to 11 take finished tiles out of tensor memory (two accumulators: the next tile's sums run
// meanwhile) and through shared memory, so that their accesses to global memory are along rows.  Operands pass through a
// ring of stages, each one piece of A and one of B, 64 deep in k.
//
// CHUNKED (operands in pieces, P > 1): the matrix unit cuts what it adds to its fp32 accumulator off, it does not round, so
// that a sum drifts towards zero: by about 2^-26 of itself per instruction where terms have both signs (K = 256 in 96 instructions:
// 1.6e-6 of the result), by up to 2^-23 of the result where they have one (2^15 terms of 16 bits in 2048 instructions: 2e-4).  Where
// the result is to be as good as fp32 gives, the sum is cut into chunks of 64 or 128, the small products of
// a chunk come first, and the epilogue's threads, which then have most of the block's registers, add the chunks' sums.
// LONG: so do long sums of 16-bit operands, in chunks of 512 (most_kblocks).
//
// SPLIT: where there are fewer tiles than SMs, a cluster of blocks takes parts of k of one 128 x 128 tile each.  Every block
// has a part of the columns to finish: it gets the others' sums for them by bulk copies between shared memories, and adds
// in the order of k.
//
// Every wait has a limit (kWaitTries); when one runs out the block notes it in `gave_up`, all of its roles wind down, and
// gpga_token_status reports it.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "gpga_launch.cuh"
#include "gpga_token.cuh"
#include "gpga_umma.cuh"

namespace gpga {

constexpr int kTileK = 64;                                  // columns of k in a stage: 128 bytes
constexpr int kStagingWarp = 32 * 32 * 4;                   // bytes: 32 rows x 32 columns for each epilogue warp
constexpr int kGemmHead = 1024;                             // barriers, before the operand stages
constexpr int kGemmSmem = 227 * 1024;
constexpr uint32_t kWaitTries = 1u << 20;                   // polls of up to some microseconds each: seconds

static __device__ unsigned int gave_up;                     // one per file that launches products

// Instruction descriptor: fp32 accumulator, A and B fp16 or bfloat16.
__host__ __device__ constexpr uint32_t mma_descriptor(int m, int n, bool half, bool a_mn, bool b_mn)
{
    return 1u << 4 | (half ? 0u : 1u << 7 | 1u << 10) | (uint32_t)a_mn << 15 | (uint32_t)b_mn << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

struct GemmMaps {
    CUtensorMap a[2], b[2];
};

struct GemmParams {
    int32_t m, n;                 // of one batch
    int32_t kblocks1, kblocks;    // steps of kTileK of a segment; of all
    int32_t pairs;                // operands that the segments go through, again for every piece of B (GemmPlan)
    int32_t bmod;                 // B's batch index is batch % bmod
    int32_t tiles_m, tiles_n, per_batch;
    int32_t tile0, tiles;         // tiles tile0 to tiles - 1 are this launch's
    int32_t symmetric;            // only tiles on and above the diagonal; the others are their mirror images
    int32_t splits;               // SPLIT: blocks of a cluster, which share a tile's sum; PARTS: parts that its sum is left in
    uint32_t idesc;
    int32_t a_mn, b_mn;
};

struct GemmTile {
    int32_t batch, m0, n0;
};
// Tiles of a batch in columns of eight row tiles, so that tiles that run together share operands in L2.
__device__ __forceinline__ GemmTile gemm_tile(const GemmParams& p, int t, int rows, int columns)
{
    GemmTile g;
    g.batch = t / p.per_batch;
    int r = t - g.batch * p.per_batch;
    if (p.symmetric) {   // column j has j + 1 tiles
        int j = (int)((sqrtf(8.f * r + 1.f) - 1.f) * 0.5f);
        while ((int64_t)j * (j + 1) / 2 > r) --j;
        while ((int64_t)(j + 1) * (j + 2) / 2 <= r) ++j;
        g.m0 = (int)(r - (int64_t)j * (j + 1) / 2) * rows;
        g.n0 = j * columns;
        return g;
    }
    const int group = r / (8 * p.tiles_n);
    const int first = group * 8, height = min(8, p.tiles_m - first);
    r -= first * p.tiles_n;
    g.m0 = (first + r % height) * rows;
    g.n0 = (r / height) * columns;
    return g;
}

// A place in a ring of N stages and the parity of its current round.
template <uint32_t N>
struct Ring {
    uint32_t at = 0, parity = 0;
    __device__ __forceinline__ void next()
    {
        if (++at == N) at = 0, parity ^= 1;
    }
};

struct WaitState {
    volatile uint32_t* stop;
    uint32_t tries = kWaitTries;
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) const
    {
        for (uint32_t t = 0; t < tries; ++t) {
            if (try_wait(bar, parity)) return true;
            if (*stop) return false;
        }
        *stop = 1;
        atomicOr(&gave_up, 1u);
        return false;
    }
};

// A warp's 32 x 32 values pass from thread l holding row l to eight columns of a row per lane: groups of four columns lie at
// group ^ (row & 7), so that neither the writes nor the reads meet in a bank.
__device__ __forceinline__ void stage_rows(const float (&v)[32], float* stage, int lane)
{
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)
        *reinterpret_cast<float4*>(stage + lane * 32 + 4 * (j ^ (lane & 7))) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    __syncwarp();
}
__device__ __forceinline__ void staged8(const float* stage, int row, int c, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4*>(stage + row * 32 + (c ^ (4 * (row & 7))));
    const float4 b = *reinterpret_cast<const float4*>(stage + row * 32 + ((c + 4) ^ (4 * (row & 7))));
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void stage8(float* stage, int row, int c, const float (&v)[8])
{
    *reinterpret_cast<float4*>(stage + row * 32 + (c ^ (4 * (row & 7)))) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(stage + row * 32 + ((c + 4) ^ (4 * (row & 7)))) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ float staged1(const float* stage, int row, int c) { return stage[row * 32 + (c ^ (4 * (row & 7)))]; }

// The same for two warps side by side, each with 32 columns of the same rows: rows of 64, so that a store of 16-bit values to
// memory has whole lines.  `half`: which one this warp is; `id`: of the pair's barrier.
__device__ __forceinline__ void pair_sync(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool pair_all(int id, bool ok)
{
    uint32_t all;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %2, 0;\nbar.red.and.pred q, %1, 64, p;\nselp.u32 %0, 1, 0, q;\n}" : "=r"(all) : "r"(id), "r"((uint32_t)ok) : "memory");
    return all;
}
__device__ __forceinline__ int pair_place(int row, int c) { return row * 64 + (c & 32) + ((c & 31) ^ (4 * ((row & 7) ^ (c >> 5)))); }
__device__ __forceinline__ void pair_staged8(const float* stage, int row, int c, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4*>(stage + pair_place(row, c)), b = *reinterpret_cast<const float4*>(stage + pair_place(row, c + 4));
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void stage_pair(const float (&v)[32], float* stage, int lane, int half, int id)
{
    pair_sync(id);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        *reinterpret_cast<float4*>(stage + pair_place(lane, half * 32 + 4 * j)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    pair_sync(id);
}

// Eight values as they lie in memory; zeros from the n-th on.
template <class T>
struct Raw {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ void load16(const T* p)    // all eight, p on 16 bytes
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4 q = reinterpret_cast<const uint4*>(p)[i];
            w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
        }
    }
    __device__ __forceinline__ void load(const T* p, int n, bool vec)
    {
        if (vec && n >= 8) {
            load16(p);
            return;
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < n ? reinterpret_cast<const uint32_t*>(p)[i] : 0;
        } else {
            const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? h[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)h[2 * i + 1] << 16 : 0u);
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 2 * (int)sizeof(T); ++i) w[i] = 0;
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack16(v[2 * i], v[2 * i + 1], T());
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) unpack16(w[i], v[2 * i], v[2 * i + 1], T());
        }
    }
};
// Eight values to memory, the first n of them where the row ends.
template <class T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[8])
{
    uint32_t w[2 * sizeof(T)];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack16(v[2 * i], v[2 * i + 1], T());
    }
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) {
                if constexpr (sizeof(T) == 4)
                    reinterpret_cast<uint32_t*>(p)[i] = w[i];
                else
                    reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
            }
    }
}

// Rounded to 16 bits as pack16 does, but infinities and what is beyond the range become the largest values: the first of two that
// stand for one value.  The second has what is left, an infinity too, and so neither makes NaN of the other.
__device__ __forceinline__ uint32_t pack16_finite(float lo, float hi, __half)
{
    uint32_t w;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}
__device__ __forceinline__ uint32_t pack16_finite(float lo, float hi, __nv_bfloat16)
{
    uint32_t w;
    asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}

// Where the pieces of an array of rows are (piece, batch, row, column; rows start on 16 bytes and are padded to eight).
// bfloat16, P = 3: the upper 16 bits, the upper 16 of the rest, and what is left of it, which has eight significant bits:
// the sum is exact (an infinity's rest is NaN).  P = 2: rounded, then the rounded rest: 22 bits of
// half, 16 of bfloat16.  P = 1: rounded.
template <class T16>
struct Pieces {
    T16* base;
    int64_t piece, batch, ld;
    __device__ __forceinline__ int64_t at(int b, int row, int col) const { return b * batch + row * ld + col; }
    template <int P>
    __device__ __forceinline__ void store(int b, int row, int col, const float (&v)[8]) const
    {
        store_at<P>(at(b, row, col), v);
    }
    template <int P>
    __device__ __forceinline__ void store_at(int64_t place, const float (&v)[8]) const
    {
        T16* const to = base + place;
        uint32_t w[P][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = v[2 * i], y = v[2 * i + 1];
            if constexpr (P == 3) {
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    w[q][i] = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
                    if (q < 2) {
                        x -= __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
                        y -= __uint_as_float(__float_as_uint(y) & 0xFFFF0000u);
                    }
                }
            } else {
                w[0][i] = P == 2 ? pack16_finite(x, y, T16()) : pack16(x, y, T16());
                if constexpr (P == 2) {
                    float hx, hy;
                    unpack16(w[0][i], hx, hy, T16());
                    w[1][i] = pack16(x - hx, y - hy, T16());
                }
            }
        }
#pragma unroll
        for (int q = 0; q < P; ++q) *reinterpret_cast<uint4*>(to + q * piece) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
    }
    template <int P>
    __device__ __forceinline__ void load(int b, int row, int col, Raw<T16> (&r)[P]) const
    {
        const T16* const from = base + at(b, row, col);
#pragma unroll
        for (int q = 0; q < P; ++q) r[q].load(from + q * piece, 8, true);
    }
};

// Rows of the caller's that a product goes to: factor times it, added to what is there or not.
template <class T>
struct Rows {
    T* base;
    int64_t ld;
    float factor;
    bool accumulate;
    __device__ __forceinline__ void ahead(Raw<T>& old, int row, int col, int left) const
    {
        if (accumulate) old.load(base + row * ld + col, left, true);
    }
    __device__ __forceinline__ void eight(float (&v)[8], const Raw<T>& old, int row, int col, int left) const
    {
        float o[8];
        if (accumulate) old.values(o);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = accumulate ? o[k] + factor * v[k] : factor * v[k];
        store8(base + row * ld + col, left, v);
    }
    __device__ __forceinline__ void one(float v, int row, int col) const
    {
        T* const at = base + row * ld + col;
        *at = from_f32<T>(accumulate ? to_f32(*at) + factor * v : factor * v);
    }
};

// Registers of the CHUNKED kernel's threads: warps 0 to 3, and the others.  128 x (64 + 2 x 208) are no more than a launch
// of 384 threads with 168 (and with 160) has; the launch checks it.
constexpr int kFewRegisters = 64, kManyRegisters = 208;

// Epi, for a product's row and column (bounds are the kernel's care; `left` columns are there from col on):
//   Ahead, load(ahead, batch, row, col, left): what is read of eight columns ahead of their sums;
//   Columns, columns(batch, col): what is read once for the rows of eight columns; Factors, factors(columns): what becomes of it;
//   eight(v, ahead, factors, batch, row, col, left): eight columns.  wide() false: one(v, batch, row, col) is called instead;
//   kDual: scale(v, factors(columns(which, batch, col)), row(batch, row)) of each array, then eight(v, w, batch, row, col, left), v of the first array's columns, w of the second's.  wide() false: keep(which, v,
//   batch, row, col) is called first for every single value.
//   kPair: 16-bit values that are read and stored pass in whole lines of 64 columns, two warps together (wide() is true).
//   kTail: microseconds of 128 x 256 columns, for the choice of the variant.
//   kMirror: eight() leaves in v what it has stored; put(v, batch, row, col) stores it again at its mirror place.
// The loops over eight columns are kept rolled: a warp goes through an epilogue once per tile, and unrolled it waits for
// instructions (an epilogue with the activation and its slopes in fp32, 2048 x 2048 values: 147 us unrolled, 60 us rolled).
struct Nothing {};

// The kernel's shared memory from the first 1024-byte boundary on.
__device__ __forceinline__ unsigned char* gemm_shared()
{
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    return smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
}

// A SPLIT tile's sums: eight columns after eight columns (the block that finishes them has them one after the other), 128 rows of
// 32 bytes and 64 bytes between; the halves of a row change places every four rows, for the banks.
constexpr int kSplitChunk = 128 * 32 + 64;
__device__ __forceinline__ uint32_t split_place(int chunk, int row, int half) { return chunk * kSplitChunk + row * 32 + ((half ^ (row >> 2 & 1)) << 4); }

constexpr int kLongChunk = 8;   // k-blocks

// What a variant of the kernel has: tile columns (of a pair of blocks, where CG = 2), pieces, warps of the epilogue, stages.
// PARTS: batch b of the epilogue is part b % splits of the sums of batch b / splits.
template <int CG_, int BN_, int P_, int WARPS_ = 8, bool SPLIT_ = false, bool PARTS_ = false, bool LONG_ = false>
struct Variant {
    static constexpr int CG = CG_, BN = BN_, P = P_, warps = WARPS_, threads = 128 + 32 * warps;
    static constexpr bool chunked = P > 1 || LONG_, split = SPLIT_, parts = PARTS_;
    static constexpr int staging = split ? 16 * kSplitChunk : warps * kStagingWarp;   // split: the other blocks' sums
    static constexpr bool split_registers = chunked && warps == 8;    // sixteen have few enough sums each
    static_assert(!split || (CG == 1 && BN == 128 && warps == 8), "a SPLIT tile is 128 x 128");
    static constexpr uint32_t a_bytes = 128 * kTileK * 2, b_bytes = BN / CG * kTileK * 2, stage_bytes = a_bytes + b_bytes;
    static constexpr uint32_t room = (kGemmSmem - 1024 - kGemmHead - staging) / stage_bytes;
    static constexpr uint32_t stages = room < 8 ? room : 8;
    static constexpr int chunk = LONG_ ? kLongChunk : P == 3 ? 1 : 2;   // k-blocks of a chunk
    using Long = Variant<CG, BN, P, warps, split, parts, P == 1>;
};

template <class V, class Epi>
__global__ void __launch_bounds__(V::threads, 1)
    gemm_kernel(const __grid_constant__ GemmMaps maps, const __grid_constant__ GemmParams p, const __grid_constant__ Epi epi)
{
    unsigned char* const smem = gemm_shared();
    const uint32_t base = smem_u32(smem);
    // head: full[8], empty[8], acc_full[2], acc_empty[2], tensor memory address, stop flag, SPLIT's copies
    const uint32_t full = base, empty = base + 64, acc_full = base + 128, acc_empty = base + 144;
    uint32_t* const tmem_at = reinterpret_cast<uint32_t*>(smem + 160);
    volatile uint32_t* const stop = reinterpret_cast<volatile uint32_t*>(smem + 164);
    uint64_t* const copies = reinterpret_cast<uint64_t*>(smem + 168);
    float* const staging = reinterpret_cast<float*>(smem + kGemmHead);
    const uint32_t operands = base + kGemmHead + V::staging;
    constexpr int CG = V::CG, BN = V::BN, P = V::P;
    constexpr bool CHUNKED = V::chunked, SPLIT = V::split;
    constexpr uint32_t a_bytes = V::a_bytes, stage_bytes = V::stage_bytes, stages = V::stages;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0, part_of_k = SPLIT ? cluster_rank() : 0;
    const int group = SPLIT ? p.splits : CG, first = p.tile0 + blockIdx.x / group, step = gridDim.x / group;
    const auto k_start = [&](int part) { return (int)((int64_t)p.kblocks * part / p.splits); };
    int kb_first = SPLIT ? k_start(part_of_k) : 0, kb_count = SPLIT ? k_start(part_of_k + 1) - kb_first : p.kblocks;
    const auto take_part = [&](int batch) {
        const int part = batch % p.splits;
        kb_first = k_start(part);
        kb_count = k_start(part + 1) - kb_first;
    };
    const WaitState w{stop};
    // SPLIT: this block's sums, in the order of the blocks that finish them; the place there of the tile's c-th eight columns.
    unsigned char* const sums_at = smem + kGemmHead + V::staging;
    constexpr int columns8 = (Epi::kDual ? BN / 2 : BN) / 8;
    const auto split_chunk = [&](int c) {
        if (!Epi::kDual) return c;
        const int per = columns8 / p.splits, i = c % columns8;   // of both arrays side by side
        return (i / per * 2 + c / columns8) * per + i % per;
    };

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < stages; ++s) {
            mbar_init(reinterpret_cast<uint64_t*>(smem + 8 * s), CG);
            mbar_init(reinterpret_cast<uint64_t*>(smem + 64 + 8 * s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(reinterpret_cast<uint64_t*>(smem + 128 + 8 * i), 1);
            mbar_init(reinterpret_cast<uint64_t*>(smem + 144 + 8 * i), V::warps * CG);
        }
        *stop = 0;
        if constexpr (SPLIT) {
            mbar_init(copies, 1);
            if (p.splits > 1) mbar_arrive_expect_tx(copies, (p.splits - 1) * (16 / p.splits) * kSplitChunk);
        }
        mbar_init_fence();
        prefetch_map(&maps.a[0]);
        prefetch_map(&maps.b[0]);
    }
    if (warp == 2) tmem_alloc<CG>(smem_u32(tmem_at), 512);
    tmem_fence_before();
    __syncthreads();
    if constexpr (CG == 2 || SPLIT) cluster_barrier();
    tmem_fence_after();
    const uint32_t tmem = *tmem_at;
    grid_launch_dependents();
    grid_dependency_wait();

    uint32_t loaded = 0;   // stages filled by this block (warp 0)
    if (warp < 4) {
        if constexpr (V::split_registers) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
        if (warp == 0 && lane == 0) {
            constexpr int nb = BN / CG;
            const uint32_t lead = CG == 2 ? map_shared(full, 0) : full;
            const bool a_mn = p.a_mn, b_mn = p.b_mn;
            Ring<stages> ring;
            bool ok = true;
            for (int t = first; t < p.tiles && ok; t += step) {
                GemmTile g = gemm_tile(p, t, 128 * CG, BN);
                if constexpr (V::parts) take_part(g.batch), g.batch /= p.splits;
                const int m0 = g.m0 + (int)rank * 128, bb = g.batch % p.bmod;
                const int n0 = Epi::kDual ? g.n0 / 2 : g.n0 + (int)rank * nb;   // kDual: BN / 2 columns of each array
                const int segment = kb_first / p.kblocks1;
                int pair = segment % p.pairs, piece = segment / p.pairs, in_segment = kb_first - segment * p.kblocks1;
                for (int kb = 0; kb < kb_count && ok; ++kb) {
                    const int k0 = in_segment * kTileK;
                    const CUtensorMap* const ma = &maps.a[pair];
                    const CUtensorMap* const mb = &maps.b[Epi::kDual ? (CG == 2 ? rank : 0) : pair];
#pragma unroll
                    for (int q = P - 1; q >= 0; --q, ring.next(), ++loaded) {
                        if (loaded >= stages && !(ok = w.wait(empty + 8 * ring.at, ring.parity ^ 1))) break;
                        const uint32_t bar = lead + 8 * ring.at;
                        if constexpr (CG == 2)
                            arrive_expect_cluster(bar, stage_bytes);
                        else
                            mbar_arrive_expect_tx(reinterpret_cast<uint64_t*>(smem + 8 * ring.at), stage_bytes);
                        const uint32_t da = operands + ring.at * stage_bytes, db = da + a_bytes;
                        if (a_mn) {
                            load_box<CG>(da, ma, m0, k0, g.batch, q, bar);
                            load_box<CG>(da + 8192, ma, m0 + 64, k0, g.batch, q, bar);
                        } else {
                            load_box<CG>(da, ma, k0, m0, g.batch, q, bar);
                        }
                        if (!Epi::kDual && b_mn) {
#pragma unroll
                            for (int c = 0; c < nb; c += 64) load_box<CG>(db + c * 128, mb, n0 + c, k0, bb, q + piece, bar);
                        } else {
                            load_box<CG>(db, mb, k0, n0, bb, q + piece, bar);
                            if constexpr (Epi::kDual && CG == 1) load_box<CG>(db + V::b_bytes / 2, &maps.b[1], k0, n0, bb, q + piece, bar);
                        }
                    }
                    if (++in_segment == p.kblocks1) {
                        in_segment = 0;
                        if (++pair == p.pairs) pair = 0, ++piece;
                    }
                }
            }
        } else if (warp == 1 && rank == 0 && lane == 0) {
            const uint32_t a_step = p.a_mn ? 2048 >> 4 : 32 >> 4, b_step = p.b_mn ? 2048 >> 4 : 32 >> 4;
            const uint64_t a_first = tile_descriptor(operands, p.a_mn), b_first = tile_descriptor(operands + a_bytes, p.b_mn);
            const uint32_t idesc = p.idesc;
            Ring<stages> ring;
            uint32_t sums = 0;   // accumulators filled
            bool ok = true;
            for (int t = first; t < p.tiles && ok; t += step) {
                if constexpr (V::parts) take_part(t / p.per_batch);
                const int chunk = CHUNKED ? V::chunk : kb_count;
                for (int k0 = 0; k0 < kb_count && ok; k0 += chunk, ++sums) {
                    const uint32_t buf = sums & 1;
                    if (sums >= 2 && !(ok = w.wait(acc_empty + 8 * buf, (sums / 2 - 1) & 1))) break;
                    tmem_fence_after();
                    const uint32_t d = tmem + buf * 256;
                    const int count = min(chunk, kb_count - k0);
                    for (int kb = 0; kb < count && ok; ++kb) {
                        // The last pieces lie in the first stage of a k-block.  Small products first; a stage is free when its piece
                        // has met all that it meets, which is in the stages' order.
                        uint64_t a[P], b[P];
                        uint32_t free[P];
#pragma unroll
                        for (int q = P - 1; q >= 0; --q, ring.next()) {
                            if (!(ok = w.wait(full + 8 * ring.at, ring.parity))) break;
                            a[q] = a_first + ring.at * (stage_bytes >> 4);
                            b[q] = b_first + ring.at * (stage_bytes >> 4);
                            free[q] = empty + 8 * ring.at;
                        }
                        if (!ok) break;
                        tmem_fence_after();
#pragma unroll
                        for (int q = P - 1; q >= 0; --q) {   // products whose higher piece is q
#pragma unroll
                            for (int r = q; r >= 0; --r) {
                                if (q + r >= P) continue;
#pragma unroll
                                for (int flip = 0; flip < (r < q ? 2 : 1); ++flip)
#pragma unroll
                                    for (int k = 0; k < kTileK / 16; ++k)
                                        mma_f16<CG>(d, a[flip ? r : q] + k * a_step, b[flip ? q : r] + k * b_step, idesc,
                                                    kb > 0 || k > 0 || flip > 0 || q < P - 1 || r < (P - 1) - q);
                            }
                            mma_commit<CG>(free[q]);
                        }
                    }
                    if (!ok) break;
                    mma_commit<CG>(acc_full + 8 * buf);
                }
            }
        }
        __syncwarp();
    } else {
        if constexpr (V::split_registers) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
        const int quarter = warp & 3, part = (warp - 4) >> 2;   // lanes of tensor memory, columns
        // Two warps of a quarter stage 64 columns together where that gives whole lines.
        constexpr bool PAIR = Epi::kPair && !CHUNKED && !SPLIT;
        static_assert(!Epi::kPair || (!Epi::kDual && !Epi::kMirror), "whole lines of one array, which takes eight()");
        const int half = part & 1, pair = quarter + 4 * (part >> 1), pair_id = 1 + pair;
        float* const stage = PAIR ? staging + pair * 64 * 32 : staging + (warp - 4) * 32 * 32;
        const uint32_t release = CG == 2 ? map_shared(acc_empty, 0) : acc_empty;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        uint32_t sums = 0;
        bool ok = true;
        constexpr int width = BN / (V::warps / 4) / (Epi::kDual ? 2 : 1);   // columns of this warp (of each array)
        constexpr int kRows = PAIR ? 4 : 8, kColumns = PAIR ? 64 : 32;   // of a pass over what is staged
        const int lane_row = PAIR ? half * 16 + (lane >> 3) : lane >> 2, lane_col = PAIR ? (lane & 7) * 8 : (lane & 3) * 8;
        const int first_column = PAIR ? (part >> 1) * 2 * width : part * width;
        for (int t = first; t < p.tiles && ok; t += step) {
            const GemmTile g = gemm_tile(p, t, 128 * CG, BN);
            if constexpr (V::parts) take_part(g.batch);
            const int row0 = g.m0 + (int)rank * 128 + quarter * 32, from = (Epi::kDual ? g.n0 / 2 : g.n0) + first_column;
            const int rows = p.m - row0;   // that are there
            const bool mirror = p.symmetric && g.m0 != g.n0;
            constexpr int kAhead = CHUNKED ? 1 : 2;   // calls of eight() that are read ahead
            typename Epi::Ahead ahead[kAhead];
            // SPLIT: 32 columns of this block's sum, where the operands were.
            const auto put_partial = [&](const float(&v)[32], int col) {
                const int r = quarter * 32 + lane;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<float4*>(sums_at + split_place(split_chunk(col / 8 + j / 2), r, j & 1)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            };
            // A 32 x 32 block that is staged (PAIR: 16 x 64); `next`: whether the block to the right follows.
            const auto block = [&](int col0, bool next) {
                if constexpr (!Epi::kDual) {
                if (!epi.wide()) {
                    if (col0 + lane < p.n)
#pragma unroll 1
                        for (int r = 0; r < min(rows, 32); ++r) epi.one(staged1(stage, r, lane), g.batch, row0 + r, col0 + lane);
                    return;
                }
                const int c = col0 + lane_col;
                typename Epi::Factors factors{};
                if (c < p.n) factors = epi.factors(epi.columns(g.batch, c));
#pragma unroll 1
                for (int i = 0; i < 4; i += kAhead) {
#pragma unroll
                    for (int j = 0; j < kAhead; ++j) {
                        const int r = (i + j) * kRows + lane_row;
                        const typename Epi::Ahead now = ahead[j];
                        const bool here = i + kAhead < 4;
                        const int nr = here ? r + kRows * kAhead : j * kRows + lane_row, nc = here ? c : c + kColumns;
                        if (nr < rows && nc < p.n && (here || next)) epi.load(ahead[j], g.batch, row0 + nr, nc, p.n - nc);
                        if (r < rows && c < p.n) {
                            float v[8];
                            if constexpr (PAIR)
                                pair_staged8(stage, r, lane_col, v);
                            else
                                staged8(stage, r, lane_col, v);
                            epi.eight(v, now, factors, g.batch, row0 + r, c, p.n - c);
                            if constexpr (Epi::kMirror)
                                if (mirror) stage8(stage, r, lane_col, v);
                        }
                    }
                }
                if constexpr (Epi::kMirror)
                    if (mirror) {
                        __syncwarp();
#pragma unroll 1
                        for (int i = 0; i < 4; ++i) {
                            const int c = i * 8 + lane_row, r = lane_col;
                            float v[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) v[k] = staged1(stage, r + k, c);
                            if (col0 + c < p.n && r < rows) epi.put(v, g.batch, col0 + c, row0 + r);
                        }
                    }
                }
            };
            const auto start = [&] {
                if constexpr (!Epi::kDual)
#pragma unroll
                    for (int j = 0; j < kAhead; ++j)
                        if (epi.wide() && j * kRows + lane_row < rows && from + lane_col < p.n)
                            epi.load(ahead[j], g.batch, row0 + j * kRows + lane_row, from + lane_col, p.n - from - lane_col);
            };
            // The same of two arrays.
            typename Epi::Columns columns2[2] = {};     // of the 32 columns that are next, of each array
            int own[4] = {};
            const auto start2 = [&](int col0) {
                if constexpr (Epi::kDual) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        if (col0 + lane_col < p.n) columns2[q] = epi.columns(q, g.batch, col0 + lane_col);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i * 8 + lane_row < rows) own[i] = epi.row(g.batch, row0 + i * 8 + lane_row);
                }
            };
            const auto block2 = [&](const float(&a)[32], const float(&b)[32], int col0) {
                if constexpr (Epi::kDual) {
                stage_rows(a, stage, lane);
                if (!epi.wide() && col0 + lane < p.n)
#pragma unroll 1
                    for (int r = 0; r < min(rows, 32); ++r) epi.keep(0, staged1(stage, r, lane), g.batch, row0 + r, col0 + lane);
                float v[4][8];
                {
                    const auto factors = epi.factors(columns2[0]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        staged8(stage, i * 8 + lane_row, lane_col, v[i]);
                        epi.scale(v[i], factors, own[i]);
                    }
                }
                stage_rows(b, stage, lane);
                if (!epi.wide() && col0 + lane < p.n)
#pragma unroll 1
                    for (int r = 0; r < min(rows, 32); ++r) epi.keep(1, staged1(stage, r, lane), g.batch, row0 + r, col0 + lane);
                const auto factors = epi.factors(columns2[1]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = i * 8 + lane_row, c = col0 + lane_col;
                    float w[8];
                    staged8(stage, r, lane_col, w);
                    epi.scale(w, factors, own[i]);
                    if (r < rows && c < p.n) epi.eight(v[i], w, g.batch, row0 + r, c, p.n - c);
                }
                }
            };
            if constexpr (CHUNKED) {
                constexpr int slabs = BN / (V::warps / 4) / 32;   // kDual: those of the first array, then those of the second
                float acc[slabs][32];
#pragma unroll
                for (int j = 0; j < slabs; ++j)
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[j][i] = 0.f;
                if constexpr (!SPLIT) start2(from);
                for (int k0 = 0; k0 < kb_count; k0 += V::chunk, ++sums) {
                    const uint32_t buf = sums & 1;
                    ok = __all_sync(~0u, w.wait(acc_full + 8 * buf, (sums / 2) & 1));
                    if (!ok) break;
                    tmem_fence_after();
#pragma unroll
                    for (int j = 0; j < slabs; ++j) {
                        const uint32_t at = lanes + buf * 256 + part * width + (Epi::kDual ? (j % (slabs / 2)) * 32 + j / (slabs / 2) * (BN / 2) : j * 32);
                        float a[32];
                        tmem_load32(at, a);
                        tmem_wait_load();
#pragma unroll
                        for (int i = 0; i < 32; ++i) acc[j][i] += a[i];
                    }
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_cluster(release + 8 * buf);
                }
                if (!ok) break;
                if constexpr (SPLIT) {
#pragma unroll
                    for (int j = 0; j < slabs; ++j)
                        put_partial(acc[j], part * width + (Epi::kDual ? j * (BN / 2) : j * 32));
                    continue;
                }
                if (rows <= 0) continue;
                if constexpr (!Epi::kDual) start();
#pragma unroll 1
                for (int j = 0; j < (Epi::kDual ? slabs / 2 : slabs); ++j) {
                    const int col0 = from + 32 * j;
                    if (col0 >= p.n) break;
                    if constexpr (Epi::kDual) {
                        if (j) start2(col0);
                        float a[32], b[32];
#pragma unroll
                        for (int q = 0; q < slabs / 2; ++q)
                            if (q == j)
#pragma unroll
                                for (int i = 0; i < 32; ++i) a[i] = acc[q][i], b[i] = acc[q + slabs / 2][i];
                        block2(a, b, col0);
                    } else {
#pragma unroll
                        for (int q = 0; q < slabs; ++q)
                            if (q == j) stage_rows(acc[q], stage, lane);
                        block(col0, j + 1 < slabs);
                    }
                }
            } else {
                const uint32_t buf = sums & 1;
                if constexpr (!Epi::kDual && !SPLIT) start();
                ok = __all_sync(~0u, w.wait(acc_full + 8 * buf, (sums / 2) & 1));
                if constexpr (PAIR) ok = pair_all(pair_id, ok);   // both go on, or neither
                if (!ok) break;
                ++sums;
                tmem_fence_after();
#pragma unroll 1
                for (int c = 0; c < width; c += 32) {
                    float a[32], b[32];
                    const uint32_t at = lanes + buf * 256 + first_column + (PAIR ? 2 * c + half * 32 : c);
                    tmem_load32(at, a);
                    if constexpr (Epi::kDual) tmem_load32(at + BN / 2, b);
                    tmem_wait_load();
                    if (c + 32 >= width) {
                        tmem_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive_cluster(release + 8 * buf);
                    }
                    const int col0 = from + (PAIR ? 2 * c : c);
                    if constexpr (SPLIT) {
                        put_partial(a, part * width + c);
                        if constexpr (Epi::kDual) put_partial(b, part * width + c + BN / 2);
                        continue;
                    }
                    if (rows <= 0 || col0 >= p.n) continue;
                    if constexpr (Epi::kDual) {
                        start2(col0);
                        block2(a, b, col0);
                    } else {
                        if constexpr (PAIR)
                            stage_pair(a, stage, lane, half, pair_id);
                        else
                            stage_rows(a, stage, lane);
                        block(col0, c + 32 < width);
                    }
                }
            }
        }
    }

    if constexpr (SPLIT) {
        __syncthreads();
        const bool sound = !*stop;    // the same for all: what is below has barriers
        __syncthreads();
        if (warp >= 4 && sound) {
            const int thread = threadIdx.x - 128, per = columns8 / p.splits, shift = __ffs(per) - 1;   // chunks of this block: a power of two
            const uint32_t slice = (Epi::kDual ? 2 : 1) * per * kSplitChunk;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (thread == 0)
                for (int b = 0; b < p.splits; ++b)
                    if (b != (int)part_of_k)
                        copy_to_block(map_shared(smem_u32(staging) + part_of_k * slice, b), smem_u32(sums_at) + b * slice, slice, map_shared(smem_u32(copies), b));
            const GemmTile g = gemm_tile(p, first, 128, BN);
            const int n0 = Epi::kDual ? g.n0 / 2 : g.n0;
            const bool mirror = p.symmetric && g.m0 != g.n0;
            unsigned char* const own = sums_at + part_of_k * slice;
            if (p.splits > 1) w.wait(smem_u32(copies), 0);
            // Eight columns' sums over the blocks, in the order of k.
            const auto total = [&](int chunk, int row, float(&v)[8]) {
                const uint32_t lo = split_place(chunk, row, 0), hi = split_place(chunk, row, 1);
#pragma unroll 2
                for (int b = 0; b < p.splits; ++b) {
                    const unsigned char* const from = b == (int)part_of_k ? own : reinterpret_cast<const unsigned char*>(staging) + b * slice;
                    const float4 x = *reinterpret_cast<const float4*>(from + lo), y = *reinterpret_cast<const float4*>(from + hi);
                    const float z[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = b ? v[k] + z[k] : z[k];
                }
            };
#pragma unroll 1
            for (int u = thread; u < 128 * per; u += 256) {
                const int row = u >> shift, chunk = u & (per - 1), c = (int)((part_of_k << shift) + chunk) * 8;
                const int r = g.m0 + row, col = n0 + c, left = p.n - col;
                if (r >= p.m || left <= 0) continue;
                float v[8];
                if constexpr (Epi::kDual) {
                    float x[8];
                    total(chunk, row, v);
                    total(chunk + per, row, x);
                    if (!epi.wide())
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (k < left) {
                                epi.keep(0, v[k], g.batch, r, col + k);
                                epi.keep(1, x[k], g.batch, r, col + k);
                            }
                    epi.scale(v, epi.factors(epi.columns(0, g.batch, col)), epi.row(g.batch, r));
                    epi.scale(x, epi.factors(epi.columns(1, g.batch, col)), epi.row(g.batch, r));
                    epi.eight(v, x, g.batch, r, col, left);
                } else {
                    typename Epi::Ahead ahead;
                    if (epi.wide()) epi.load(ahead, g.batch, r, col, left);
                    total(chunk, row, v);
                    if (epi.wide()) {
                        epi.eight(v, ahead, epi.factors(epi.columns(g.batch, col)), g.batch, r, col, left);
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (k < left) epi.one(v[k], g.batch, r, col + k);
                    }
                    if constexpr (Epi::kMirror)
                        if (mirror) {   // this block's own sums of these columns are not needed again
                            *reinterpret_cast<float4*>(own + split_place(chunk, row, 0)) = make_float4(v[0], v[1], v[2], v[3]);
                            *reinterpret_cast<float4*>(own + split_place(chunk, row, 1)) = make_float4(v[4], v[5], v[6], v[7]);
                        }
                }
            }
            if constexpr (Epi::kMirror)
                if (mirror) {
                    asm volatile("bar.sync 1, 256;" ::: "memory");
#pragma unroll 1
                    for (int u = thread; u < 16 * 8 * per; u += 256) {
                        const int mine = u / 16, row = (u & 15) * 8, c = (int)(part_of_k << shift) * 8 + mine;
                        if (n0 + c >= p.n || g.m0 + row >= p.m) continue;
                        float v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = reinterpret_cast<const float*>(own + split_place(mine >> 3, row + k, mine >> 2 & 1))[mine & 3];
                        epi.put(v, g.batch, n0 + c, g.m0 + row);
                    }
                }
        }
    }

    // Everybody is done, or has given up; copies in flight must land before the block goes.
    tmem_fence_before();
    __syncthreads();
    if (*stop && threadIdx.x == 0)
        for (uint32_t i = loaded > stages ? loaded - stages : 0; i < loaded; ++i)
            for (uint32_t tries = 0; tries < 4096 && !try_wait(full + 8 * (i % stages), (i / stages) & 1); ++tries) {
            }
    __syncthreads();
    if constexpr (CG == 2 || SPLIT) cluster_farewell();
    if (warp == 2) {
        tmem_fence_after();
        tmem_free<CG>(tmem, 512);
    }
}

// ---- host side ----

// A 16-bit array: `outer` rows of `inner` values, batches and pieces of them (strides in elements, multiples of eight).
struct Operand {
    const void* base = nullptr;
    int64_t inner = 0, outer = 0, batches = 1, pieces = 1;
    int64_t ld = 0, batch = 0, piece = 0;
    bool mn_major = false;   // rows run along the product's row (column) index
};

bool operand_fits(const void* base, int64_t ld, int64_t batch);   // whether a tiled copy can read it where it lies

// The driver's encoder of tensor maps, looked up once.
cudaError_t encode_map(CUtensorMap& map, const Operand& o, bool half, int box_rows);

struct GemmPlan {
    // The sum runs over the pairs, for every piece of B beyond those that A has too (their number is a[0].pieces).
    Operand a[2], b[2];
    int pairs = 1;
    int64_t m = 0, n = 0, k = 0, batch = 1, bmod = 1;
    bool half = false;        // fp16 operands (otherwise bfloat16)
    bool after = false;       // the kernel before it on the stream is one of the same call
    bool symmetric = false;
};

int sm_count();

template <class Kernel>
int kernel_registers(Kernel kernel)
{
    cudaFuncAttributes a;
    return cudaFuncGetAttributes(&a, kernel) == cudaSuccess ? a.numRegs : 0;
}

// The tiles from tile0 up to, but not, tile1 (0: the end).
template <class V, class Epi>
cudaError_t launch_gemm_as(const GemmPlan& g, int splits, int64_t tile0, int64_t tile1, const Epi& epi, cudaStream_t stream)
{
    constexpr int CG = V::CG, bn = V::BN;
    GemmParams p;
    GemmMaps maps;
    p.m = (int32_t)g.m;
    p.n = (int32_t)g.n;
    p.pairs = g.pairs;
    p.kblocks1 = (int32_t)((g.k + kTileK - 1) / kTileK);
    p.kblocks = p.kblocks1 * g.pairs * (int32_t)(g.b[0].pieces - g.a[0].pieces + 1);
    p.bmod = (int32_t)g.bmod;
    p.tiles_m = (int32_t)((g.m + 128 * CG - 1) / (128 * CG));
    const int columns = Epi::kDual ? bn / 2 : bn;
    p.tiles_n = (int32_t)((g.n + columns - 1) / columns);
    p.symmetric = g.symmetric;
    p.per_batch = g.symmetric ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
    p.splits = splits;
    if (!tile1) tile1 = g.batch * p.per_batch * (V::parts ? splits : 1);
    const int64_t tiles = tile1 - tile0;
    if (tile1 * splits >= (int64_t(1) << 31) - 65536) return cudaErrorInvalidValue;
    p.tile0 = (int32_t)tile0;
    p.tiles = (int32_t)tile1;
    p.a_mn = g.a[0].mn_major;
    p.b_mn = g.b[0].mn_major;
    p.idesc = mma_descriptor(128 * CG, bn, g.half, p.a_mn, p.b_mn);
    const int b_rows = p.b_mn ? 64 : Epi::kDual ? bn / 2 : bn / CG;
    for (int i = 0; i < 2; ++i) {
        cudaError_t e = cudaSuccess;
        if (i < g.pairs)
            e = encode_map(maps.a[i], g.a[i], g.half, p.a_mn ? 64 : 128);
        else
            maps.a[i] = maps.a[0];
        if (e == cudaSuccess && (i < g.pairs || Epi::kDual))
            e = encode_map(maps.b[i], g.b[i], g.half, b_rows);
        else
            maps.b[i] = maps.b[0];
        if (e != cudaSuccess) return e;
    }
    const auto kernel = gemm_kernel<V, Epi>;
    static std::atomic<unsigned long long> limit_set{0};
    const cudaError_t e = ensure_smem_limit(kernel, kGemmSmem, limit_set);
    if (e != cudaSuccess) return e;
    if (V::split_registers) {
        static const int registers = kernel_registers(kernel);
        if (registers * V::threads < 128 * (kFewRegisters + 2 * kManyRegisters)) return cudaErrorLaunchOutOfResources;
    }
    const int cluster = V::split ? splits : CG;
    const int64_t blocks = (V::split ? tiles : std::min<int64_t>(tiles, sm_count() / CG)) * cluster;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(V::threads);
    cfg.dynamicSmemBytes = kGemmSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)cluster;
        attr[n].val.clusterDim.y = 1;
        attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (g.after) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, maps, p, epi);
}

// Tiles of `side` rows and columns.
inline int64_t gemm_tiles(const GemmPlan& g, int64_t n, int side)
{
    const int64_t tm = (g.m + side - 1) / side, tn = (n + side - 1) / side;
    return g.symmetric ? tm * (tm + 1) / 2 : tm * tn;
}

// Weight of 256 x 256 tiles on pairs of SMs (splits = 0), or of 128 x 128 tiles on clusters of `splits` blocks, for the choice between
// them: microseconds of waves of tiles, k-blocks of a tile, and what a tile costs besides.  A k-block of a 256 x 256 tile counts
// 0.27 us per product of pieces, one of a 128 x 128 tile on its one SM 0.25 us (a quarter of the work on half of the
// SMs: each operand byte is used half as often), which is the matrix unit's time at its highest clock.  They take longer, more so with all SMs at
// work, but alike: 0.34 and 0.37 us one tile alone, 0.62 and 0.49 to 0.58 us (16 bits) or 0.36 to 0.39 and 0.40 to 0.44 us (each of three
// products of two pieces) on all SMs.  A 128 x 128 tile is a block's only one, so nothing hides its start and
// end.  tail: the epilogue of a block's 128 x 256 part of the last tile.  Measured, all of a call with either: 512 x 512 fp32,
// two steps, 117 us and (4 blocks) 60 us; 8 x 1024 x 2816 bfloat16 255 us and (1 block) 456 us; gradient of 8000 tokens x
// 128 x 300, bf16, 145 us and (4 blocks) 84 us.
inline double gemm_microseconds(int64_t tiles, int64_t kblocks, int products, double tail, int splits, int sms)
{
    if (!splits) return (double)((tiles + sms / 2 - 1) / (sms / 2)) * (0.27 * products * kblocks + 0.3) + (products > 1 ? 5.0 : 3.0) + tail;
    const int64_t room = splits == 8 ? sms * 3 / 4 : splits == 4 ? sms * 9 / 10 : sms;   // SMs of whole clusters
    const int64_t waves = (tiles * splits + room - 1) / room;
    // a wave after the first waits for the blocks before it to leave
    return waves * (0.25 * products * ((kblocks + splits - 1) / splits) + 2.6 + (1.4 + 0.5 * tail) / splits + (splits > 1 ? 0.5 : 0.0)) + (1.0 + 1.25 * splits) * (waves - 1);
}

// The last place, at most `limit` 256 x 256 tiles from the start, where the order of those tiles and that of 128 x 128 tiles
// can be cut alike: between batches, columns of a symmetric one, and groups of eight rows of tiles (sixteen) of another.
inline void gemm_cut(const GemmPlan& g, int64_t n, int64_t limit, int64_t& large, int64_t& small)
{
    const int64_t per = gemm_tiles(g, n, 256), batch = limit / per, left = limit - batch * per;
    large = batch * per;
    small = batch * gemm_tiles(g, n, 128);
    if (g.symmetric) {
        int64_t j = 0;
        while ((j + 1) * (j + 2) / 2 <= left) ++j;
        large += j * (j + 1) / 2;
        small += j * (2 * j + 1);
    } else {
        const int64_t tn = (n + 255) / 256, i = left / (8 * tn);
        large += 8 * i * tn;
        small += 16 * i * ((n + 127) / 128);
    }
}

// The variant that should take the least time, of large tiles before the cut and clusters of `splits` blocks (0: none) after it.
struct GemmChoice {
    double microseconds;
    int64_t large, small;   // large tiles before the cut, small ones
    int splits;
};
inline GemmChoice choose_gemm(const GemmPlan& g, int64_t n, int64_t kblocks, int products, double tail)
{
    const int sms = sm_count(), pairs = sms / 2;
    const int64_t large = g.batch * gemm_tiles(g, n, 256), small = g.batch * gemm_tiles(g, n, 128);
    GemmChoice c{gemm_microseconds(large, kblocks, products, tail, 0, sms), large, small, 0};
    int64_t large_cut = 0, small_cut = 0;
    if (large > pairs) gemm_cut(g, n, large / pairs * pairs, large_cut, small_cut);
    const double before = large_cut ? gemm_microseconds(large_cut, kblocks, products, tail, 0, sms) + 3.0 : 0;
    for (int splits = 1; splits <= 8 && splits <= kblocks; splits *= 2) {
        double t = gemm_microseconds(small, kblocks, products, tail, splits, sms);
        if (t < c.microseconds) c = {t, 0, 0, splits};
        if (!large_cut || large_cut == large) continue;
        t = before + gemm_microseconds(small - small_cut, kblocks, products, tail, splits, sms);
        if (t < c.microseconds) c = {t, large_cut, small_cut, splits};
    }
    return c;
}
inline int64_t gemm_kblocks(const GemmPlan& g) { return (g.k + kTileK - 1) / kTileK * g.pairs * (g.b[0].pieces - g.a[0].pieces + 1); }

// K-blocks of 16-bit operands that one accumulator may sum, for a result of type T: fp32 a chunk (32 instructions, 2^-18 at worst);
// 16 bits a sixteenth of the type's half step at worst (bfloat16 1024 instructions, fp16 256).
template <class T> constexpr int64_t most_kblocks = kLongChunk;
template <> constexpr int64_t most_kblocks<__nv_bfloat16> = 256;
template <> constexpr int64_t most_kblocks<__half> = 64;

// V, or where its accumulators (`per` k-blocks each) would sum more than `most`, its LONG form.
template <class V, class Epi>
cudaError_t launch_gemm_up_to(int64_t most, int64_t per, const GemmPlan& g, int splits, int64_t tile0, int64_t tile1, const Epi& epi, cudaStream_t stream)
{
    if (V::P == 1 && per > most) return launch_gemm_as<typename V::Long>(g, splits, tile0, tile1, epi, stream);
    return launch_gemm_as<V>(g, splits, tile0, tile1, epi, stream);
}

// Where whole waves of large tiles leave a few over, those may go to clusters of blocks in a second launch (3 us): X X^T of
// 8 x 1024 x 2816, fp32, has 80 tiles for 74 pairs of SMs (all five steps of its orthogonalisation, replays of a graph: 1378 us
// without, 1211 us with).
// T: the type of the result.
template <int P, class T, class Epi>
cudaError_t launch_gemm(const GemmPlan& g, const Epi& epi, cudaStream_t stream)
{
    const int64_t kblocks = gemm_kblocks(g), most = most_kblocks<T>;
    const GemmChoice c = choose_gemm(g, Epi::kDual ? 2 * g.n : g.n, kblocks, P * (P + 1) / 2, Epi::kTail);
    GemmPlan rest = g;
    if (c.large) {
        const cudaError_t e = launch_gemm_up_to<Variant<2, 256, P, P <= 2 ? Epi::kWarps : 8>>(most, kblocks, g, 1, 0, c.large, epi, stream);
        if (e != cudaSuccess || !c.splits) return e;
        rest.after = true;
    }
    return launch_gemm_up_to<Variant<1, 128, P, 8, true>>(most, (kblocks + c.splits - 1) / c.splits, rest, c.splits, c.small, 0, epi, stream);
}

// Parts that the sums of a product with few large tiles are cut into, so that all pairs of SMs have some; a second launch adds
// them.  1: none.  Measured without and with them, all of a gradient: 14583 tokens x 308 x 683, bfloat16, 199 us and 170 us,
// fp32 373 us and 312 us; 1278 x 934 x 1694 105 us and 96 us, 204 us and 180 us.
inline int gemm_parts(const GemmPlan& g, int products, double tail)
{
    const int64_t tiles = g.batch * gemm_tiles(g, g.n, 256), kblocks = gemm_kblocks(g);
    double least = choose_gemm(g, g.n, kblocks, products, tail).microseconds;
    int best = 1;
    for (int parts = 2; parts <= 8 && parts <= kblocks && tiles * parts <= sm_count() / 2; ++parts) {
        // the second launch, fp32 sums that are not hidden by the next tile's, and the parts' way through L2
        const double t = gemm_microseconds(tiles * parts, (kblocks + parts - 1) / parts, products, 1.0, 0, sm_count()) + (products > 1 ? 6.0 : 4.0) + parts * g.batch * g.m * g.n * 4 / 4e6;
        if (t < least) least = t, best = parts;
    }
    return best;
}

}  // namespace gpga
