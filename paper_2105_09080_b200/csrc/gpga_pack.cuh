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
    // Where the pieces are of the source times a power of two: bits of the largest values of its parts, and where the power's
    // exponent goes, negated.
    const uint32_t* peaks;
    int peak_count;
    int32_t* exponent;
};
constexpr int kPackJobs = 5;
struct PackJobs {
    PackJob job[kPackJobs];
    int count;
    int64_t chunks;
};

__device__ __forceinline__ void pack_load(const PackJob& j, int64_t c, float (&v)[8])
{
    const int64_t row = c / j.chunks, b = row / j.rows, r = row - b * j.rows;
    const int col = (int)(c - row * j.chunks) * 8;
    Raw<float> x;
    x.load(static_cast<const float*>(j.src) + b * j.batch + r * j.ld + col, (int)min((int64_t)8, j.cols - col), j.vec);
    x.values(v);
}

// Largest finite value of an array, as bits.
__device__ __forceinline__ uint32_t finite_bits(float v)
{
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0;
}
constexpr int kPeakParts = 128;   // blocks per array

// Block x of job y: its part of the array.  `cleared`: peaks that a product of the call will find.
template <int PARTS>
__global__ void __launch_bounds__(256) peak_kernel(const __grid_constant__ PackJobs jobs, uint32_t* parts, uint32_t* cleared)
{
    const PackJob& j = jobs.job[blockIdx.y];
    const int64_t count = j.batches * j.rows * j.chunks;
    uint32_t peak = 0;
#pragma unroll 4
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < count; c += PARTS * 256) {
        float v[8];
        pack_load(j, c, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) peak = max(peak, finite_bits(v[k]));
    }
    peak = __reduce_max_sync(~0u, peak);
    __shared__ uint32_t warps[8];
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = peak;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) peak = max(peak, warps[i]);
        parts[blockIdx.y * PARTS + blockIdx.x] = peak;
        if (blockIdx.x == 0 && blockIdx.y == 0) cleared[0] = cleared[1] = 0;
    }
}

// Exponent of the power of two that brings the largest value to 2^14 .. 2^15; an array of zeros stays as it is.
__device__ __forceinline__ int scale_exponent(uint32_t peak) { return peak ? min(14 + 127 - (int)(peak >> 23), 120) : 0; }

// A thread takes a chunk of eight columns: one pass over the source, bound by memory (fp32 to three pieces: 4 bytes read,
// 6 written per value).
template <class T16>
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackJobs jobs)
{
    grid_launch_dependents();
    __shared__ float scale[kPackJobs];
    if (jobs.job[0].peaks) {
        const int i = threadIdx.x >> 5;
        if (i < jobs.count) {
            const PackJob& j = jobs.job[i];
            uint32_t peak = 0;
            for (int k = threadIdx.x & 31; k < j.peak_count; k += 32) peak = max(peak, j.peaks[k]);
            peak = __reduce_max_sync(~0u, peak);
            const int e = scale_exponent(peak);
            if ((threadIdx.x & 31) == 0) {
                scale[i] = __int_as_float((e + 127) << 23);
                if (blockIdx.x == 0) *j.exponent = -e;
            }
        }
        __syncthreads();
    }
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < jobs.chunks; at += (int64_t)gridDim.x * 256) {
        int i = 0;
        while (i + 1 < jobs.count && at >= jobs.job[i + 1].first) ++i;
        const PackJob& j = jobs.job[i];
        const int64_t c = at - j.first;
        float v[8];
        if (j.src_f32) {
            pack_load(j, c, v);
            if (j.peaks)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= scale[i];
        } else {
            const int64_t row = c / j.chunks, b = row / j.rows, r = row - b * j.rows;
            const int col = (int)(c - row * j.chunks) * 8;
            Raw<T16> x;
            x.load(static_cast<const T16*>(j.src) + b * j.batch + r * j.ld + col, (int)min((int64_t)8, j.cols - col), j.vec);
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
    // The last operand is packed times a power of two.
    void scaled(const uint32_t* peaks, int count, int32_t* exponent)
    {
        PackJob& j = jobs.job[jobs.count - 1];
        j.peaks = peaks;
        j.peak_count = count;
        j.exponent = exponent;
    }
    cudaError_t launch_peaks(uint32_t* parts, uint32_t* cleared, cudaStream_t stream) const
    {
        peak_kernel<kPeakParts><<<dim3(kPeakParts, jobs.count), 256, 0, stream>>>(jobs, parts, cleared);
        return cudaGetLastError();
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
