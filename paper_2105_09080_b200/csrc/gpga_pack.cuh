// Brings operands into a form that tiled copies can read: 16-bit pieces, rows padded to eight columns, on 16 bytes.
#pragma once
#include "gpga_gemm.cuh"

namespace gpga {

struct PackJob {
    const void* src;
    int64_t ld, batch;        // of the source, in elements
    int64_t rows, cols, batches;
    int64_t chunks;           // ceil(cols / 8)
    int64_t first;            // first of the launch's chunks that belongs to this job
    int vec;                  // every source row starts on 16 bytes
    int src_f32;              // otherwise the type of the pieces
    int pieces;
    void* dst;
    int64_t dst_piece;
};
constexpr int kPackJobs = 5;
struct PackJobs {
    PackJob job[kPackJobs];
    int count;
    int64_t chunks;
};

// A thread takes a chunk of eight columns: one pass over the source, bound by memory (fp32 to three pieces: 4 bytes read,
// 6 written per value).
template <class T16>
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackJobs jobs)
{
    grid_launch_dependents();
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < jobs.chunks; at += (int64_t)gridDim.x * 256) {
        int i = 0;
        while (i + 1 < jobs.count && at >= jobs.job[i + 1].first) ++i;
        const PackJob& j = jobs.job[i];
        const int64_t c = at - j.first, row = c / j.chunks;
        const int col = (int)(c - row * j.chunks) * 8;
        const int64_t b = row / j.rows, r = row - b * j.rows;
        const int n = (int)min((int64_t)8, j.cols - col);
        float v[8];
        const int64_t from = b * j.batch + r * j.ld + col;
        if (j.src_f32) {
            Raw<float> x;
            x.load(static_cast<const float*>(j.src) + from, n, j.vec);
            x.values(v);
        } else {
            Raw<T16> x;
            x.load(static_cast<const T16*>(j.src) + from, n, j.vec);
            x.values(v);
        }
        const Pieces<T16> dst{static_cast<T16*>(j.dst) + c * 8, j.dst_piece, 0, 0};
        if (j.pieces == 1)
            dst.template store<1>(0, 0, 0, v);
        else if (j.pieces == 2)
            dst.template store<2>(0, 0, 0, v);
        else
            dst.template store<3>(0, 0, 0, v);
    }
}

// Scratch handed out from the front, on 256 bytes.
struct ScratchPlan {
    int64_t bytes = 0;
    int64_t take(int64_t n)
    {
        const int64_t at = bytes;
        bytes += (n + 255) / 256 * 256;
        return at;
    }
};

// An operand that a tiled copy can read: where it lies, or packed into scratch by the launch that `jobs` collects.
struct PackPlan {
    PackJobs jobs{};
    ScratchPlan scratch;
    char* base = nullptr;     // nullptr: only the sizes are wanted
    int pieces = 1;           // of activations

    // Weights: fp32 beside 16-bit activations are two pieces of their type.
    Operand weights(const void* p, int64_t ld, int64_t batch, int64_t rows, int64_t cols, int64_t batches, bool f32, bool mn_major)
    {
        return operand(p, ld, batch, rows, cols, batches, f32, mn_major, f32 && pieces == 1 ? 2 : pieces);
    }
    Operand operand(const void* p, int64_t ld, int64_t batch, int64_t rows, int64_t cols, int64_t batches, bool f32, bool mn_major, int pieces)
    {
        Operand o;
        o.inner = cols;
        o.outer = rows;
        o.batches = batches;
        o.pieces = pieces;
        o.mn_major = mn_major;
        if (!f32 && pieces == 1 && operand_fits(p, rows > 1 ? ld : 8, batches > 1 ? batch : 0) && (batches == 1 || batch > 0)) {
            o.base = p;
            o.ld = ld;
            o.batch = batch;
            return o;
        }
        const int64_t chunks = (cols + 7) / 8;
        o.ld = chunks * 8;
        o.batch = rows * o.ld;
        o.piece = batches * o.batch;
        const int64_t at = scratch.take(pieces * o.piece * 2);
        o.base = base + at;
        PackJob& j = jobs.job[jobs.count];
        const int size = f32 ? 4 : 2;
        j.src = p;
        j.ld = ld;
        j.batch = batch;
        j.rows = rows;
        j.cols = cols;
        j.batches = batches;
        j.chunks = chunks;
        j.first = jobs.chunks;
        j.vec = (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows == 1 || ld * size % 16 == 0) && (batches == 1 || batch * size % 16 == 0);
        j.src_f32 = f32;
        j.pieces = pieces;
        j.dst = base + at;
        j.dst_piece = o.piece;
        ++jobs.count;
        jobs.chunks += batches * rows * chunks;
        return o;
    }
    // An array of pieces in scratch that a kernel of the call writes.
    Operand written(int64_t rows, int64_t cols, int64_t batches, bool mn_major)
    {
        Operand o;
        o.inner = cols;
        o.outer = rows;
        o.batches = batches;
        o.pieces = pieces;
        o.mn_major = mn_major;
        o.ld = (cols + 7) / 8 * 8;
        o.batch = rows * o.ld;
        o.piece = batches * o.batch;
        o.base = base + scratch.take(pieces * o.piece * 2);
        return o;
    }
    template <class T16>
    cudaError_t launch(cudaStream_t stream) const
    {
        if (!jobs.count) return cudaSuccess;
        const int64_t blocks = std::min<int64_t>((jobs.chunks + 255) / 256, (int64_t)sm_count() * 8);
        pack_kernel<T16><<<(unsigned)blocks, 256, 0, stream>>>(jobs);
        return cudaGetLastError();
    }
};
template <class T16>
Pieces<T16> pieces_of(const Operand& o)
{
    return {static_cast<T16*>(const_cast<void*>(o.base)), o.piece, o.batch, o.ld};
}

}  // namespace gpga
