// Brings operands into a form that tiled copies can read: 16-bit pieces, rows padded to eight columns, on 16 bytes.
#pragma once
#include "gpga_gemm.cuh"

namespace gpga {

// fp32 as pairs of fp16 values: times powers of two, one for each row or (where rows are summed over) for each column of a matrix,
// so that what is far larger elsewhere takes no bits from it.
struct PackJob {
    const void* src;
    int64_t ld, batch;        // of the source, in elements
    int64_t rows, cols, batches;
    int64_t chunks;           // ceil(cols / 8)
    int64_t first;            // first of the launch's units that belongs to this job
    int vec;                  // every source row starts on 16 bytes
    int src_f32;              // otherwise the type of the pieces
    int pieces;
    void* dst;
    int64_t dst_piece;
    int8_t* exponents;        // of the powers, negated: [batch][rows, padded to eight], or [batch][8 chunks]
    uint32_t* peaks;          // by columns: bits of their largest finite values, [batch][8 chunks]
};
constexpr int kPackJobs = 5;
struct PackJobs {
    PackJob job[kPackJobs];
    int count;
    int slice;                // by columns: rows of a unit
    int64_t units;            // chunks; what a block holds of rows; or pieces of `slice` rows by 32 chunks
    __device__ __forceinline__ const PackJob& of(int64_t unit) const
    {
        int i = 0;
        while (i + 1 < count && unit >= job[i + 1].first) ++i;
        return job[i];
    }
};

__device__ __forceinline__ void pack_load(const PackJob& j, int64_t c, float (&v)[8])
{
    const int64_t row = c / j.chunks, b = row / j.rows, r = row - b * j.rows;
    const int col = (int)(c - row * j.chunks) * 8;
    Raw<float> x;
    x.load(static_cast<const float*>(j.src) + b * j.batch + r * j.ld + col, (int)min((int64_t)8, j.cols - col), j.vec);
    x.values(v);
}

__host__ __device__ constexpr int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }

// Bits of |v|, 0 for infinities and NaN.
__device__ __forceinline__ uint32_t finite_bits(float v)
{
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0;
}
// Exponent of the power of two that brings the largest value to 2^14 .. 2^15 (as near as fp32 has one); zeros stay as they are.
__device__ __forceinline__ int scale_exponent(uint32_t peak) { return peak ? min(14 + 127 - (int)(peak >> 23), 125) : 0; }
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }

// A thread takes a chunk of eight columns: one pass over the source, bound by memory (fp32 to three pieces: 4 bytes read,
// 6 written per value).
template <class T16>
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackJobs jobs)
{
    grid_launch_dependents();
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < jobs.units; at += (int64_t)gridDim.x * 256) {
        const PackJob& j = jobs.of(at);
        const int64_t c = at - j.first;
        float v[8];
        if (j.src_f32) {
            pack_load(j, c, v);
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

namespace {

// Threads that lie along a row of chunks: a power of two, `most` at most.
__host__ __device__ inline int row_threads(int64_t chunks, int most)
{
    int n = 1;
    while (n < most && n < chunks) n *= 2;
    return n;
}
// A unit of pack_rows_kernel: each thread holds kHeldChunks chunks, `slots` of them of one row.
constexpr int kHeldChunks = 4;
__host__ __device__ inline int row_slots(int64_t chunks) { return chunks > 512 ? 4 : chunks > 256 ? 2 : 1; }
__host__ __device__ inline int rows_of_unit(int64_t chunks) { return kHeldChunks / row_slots(chunks) * (256 / row_threads(chunks, 256)); }

// fp32 rows to pairs, a power of two for each row; bound by memory.  A block takes as many rows as it holds (8192 columns), so
// that they are read once and their reads are under way together; of longer rows the rest comes from L2 again.  A row for each warp,
// one after the other, took 114 us for the operands of 64 x 300 x 130 x 900.  cleared: 16-byte words that later launches find zero.
__global__ void __launch_bounds__(256) pack_rows_kernel(const __grid_constant__ PackJobs jobs, uint4* cleared, int64_t clear)
{
    grid_launch_dependents();
    grid_dependency_wait();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < clear; i += (int64_t)gridDim.x * 256) cleared[i] = make_uint4(0, 0, 0, 0);
    __shared__ uint32_t of_warp[2][kHeldChunks][8];    // of units in turn: one's are read while the next one's are written
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int turn = 0;
    for (int64_t unit = blockIdx.x; unit < jobs.units; unit += gridDim.x) {
        const PackJob& j = jobs.of(unit);
        const int chunks = (int)j.chunks, cols = (int)j.cols, threads = row_threads(chunks, 256), slots = row_slots(chunks), side = 256 / threads;
        const int own = threadIdx.x & (threads - 1);
        const int64_t first = (unit - j.first) * rows_of_unit(chunks) + threadIdx.x / threads, rows = j.batches * j.rows;
        const auto largest = [](const Raw<float>& x) {
            float v[8];
            uint32_t p = 0;
            x.values(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) p = max(p, finite_bits(v[k]));
            return p;
        };
        const auto place = [&](int64_t row, int64_t& b) {      // of a row in the source
            b = row >> 31 ? row / j.rows : (int64_t)((uint32_t)row / (uint32_t)j.rows);
            return static_cast<const float*>(j.src) + b * j.batch + (row - b * j.rows) * j.ld;
        };
        Raw<float> held[kHeldChunks];
        uint32_t peak[kHeldChunks];
#pragma unroll
        for (int q = 0; q < kHeldChunks; ++q) {
            const int64_t row = first + q / slots * side;
            const int c = own + threads * (q & (slots - 1));
            int64_t b;
            if (row < rows && c < chunks)
                held[q].load(place(row, b) + 8 * c, cols - 8 * c, j.vec);
            else
                held[q].zero();
        }
#pragma unroll
        for (int q = 0; q < kHeldChunks; ++q) peak[q] = largest(held[q]);
        const bool longer = chunks > 256 * kHeldChunks;      // one row
        if (longer) {
            int64_t b;
            const float* const from = place(first, b);
            for (int c = own + 256 * kHeldChunks; c < chunks; c += 256) {
                Raw<float> x;
                x.load(from + 8 * c, cols - 8 * c, j.vec);
                peak[0] = max(peak[0], largest(x));
            }
        }
        if (slots > 1) peak[0] = peak[1] = max(peak[0], peak[1]), peak[2] = peak[3] = max(peak[2], peak[3]);
        if (slots > 2) peak[0] = peak[1] = peak[2] = peak[3] = max(peak[0], peak[2]);
#pragma unroll
        for (int q = 0; q < kHeldChunks; ++q) {
            if (threads >= 32)
                peak[q] = __reduce_max_sync(~0u, peak[q]);
            else
                for (int o = threads / 2; o; o >>= 1) peak[q] = max(peak[q], __shfl_xor_sync(~0u, peak[q], o));
        }
        if (threads > 32) {
            const int warps = threads / 32, from = warp & ~(warps - 1);
            if (lane == 0)
#pragma unroll
                for (int q = 0; q < kHeldChunks; ++q) of_warp[turn][q][warp] = peak[q];
            __syncthreads();
            for (int i = 0; i < warps; ++i)
#pragma unroll
                for (int q = 0; q < kHeldChunks; ++q) peak[q] = max(peak[q], of_warp[turn][q][from + i]);
            turn ^= 1;      // with the barrier: units without one may lie between
        }
        const Pieces<__half> dst{static_cast<__half*>(j.dst), j.dst_piece, 0, 0};
        const auto put = [&](const Raw<float>& x, int64_t row, int c, float scale) {
            float v[8];
            x.values(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= scale;
            dst.template store_at<2>((row * chunks + c) * 8, v);
        };
#pragma unroll
        for (int q = 0; q < kHeldChunks; ++q) {
            const int64_t row = first + q / slots * side;
            const int c = own + threads * (q & (slots - 1)), e = scale_exponent(peak[q]);
            if (row >= rows) continue;
            if (c == 0) {
                int64_t b;
                place(row, b);
                j.exponents[b * padded(j.rows) + row - b * j.rows] = (int8_t)-e;
            }
            if (c < chunks) put(held[q], row, c, power_of_two(e));
        }
        if (longer) {
            int64_t b;
            const float* const from = place(first, b);
            const float scale = power_of_two(scale_exponent(peak[0]));
            for (int c = own + 256 * kHeldChunks; c < chunks; c += 256) {
                Raw<float> x;
                x.load(from + 8 * c, cols - 8 * c, j.vec);
                put(x, first, c, scale);
            }
        }
    }
}

// The same, a warp to a row: it holds 2048 columns.  For long rows, where the block's barriers cost more than rows that are read one
// after the other (long_rows).
constexpr int kWarpChunks = 8;
__global__ void __launch_bounds__(256) pack_long_rows_kernel(const __grid_constant__ PackJobs jobs, uint4* cleared, int64_t clear)
{
    grid_launch_dependents();
    grid_dependency_wait();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < clear; i += (int64_t)gridDim.x * 256) cleared[i] = make_uint4(0, 0, 0, 0);
    const int lane = threadIdx.x & 31;
    for (int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); at < jobs.units; at += (int64_t)gridDim.x * 8) {
        const PackJob& j = jobs.of(at);
        const int64_t row = at - j.first, b = row / j.rows, r = row - b * j.rows;
        const float* const from = static_cast<const float*>(j.src) + b * j.batch + r * j.ld;
        const int chunks = (int)j.chunks, cols = (int)j.cols;
        Raw<float> held[kWarpChunks];
        uint32_t peak = 0;
        const auto largest = [&](const Raw<float>& x) {
            float v[8];
            x.values(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) peak = max(peak, finite_bits(v[k]));
        };
#pragma unroll
        for (int q = 0; q < kWarpChunks; ++q) {
            const int c = lane + 32 * q;
            if (c < chunks) held[q].load(from + 8 * c, cols - 8 * c, j.vec);
        }
#pragma unroll
        for (int q = 0; q < kWarpChunks; ++q)
            if (lane + 32 * q < chunks) largest(held[q]);
        for (int c = lane + 32 * kWarpChunks; c < chunks; c += 32) {
            Raw<float> x;
            x.load(from + 8 * c, cols - 8 * c, j.vec);
            largest(x);
        }
        const int e = scale_exponent(__reduce_max_sync(~0u, peak));
        const float scale = power_of_two(e);
        if (lane == 0) j.exponents[b * padded(j.rows) + r] = (int8_t)-e;
        const Pieces<__half> dst{static_cast<__half*>(j.dst) + row * chunks * 8, j.dst_piece, 0, 0};
        const auto put = [&](const Raw<float>& x, int c) {
            float v[8];
            x.values(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= scale;
            dst.template store_at<2>(8 * c, v);
        };
#pragma unroll
        for (int q = 0; q < kWarpChunks; ++q)
            if (lane + 32 * q < chunks) put(held[q], lane + 32 * q);
        for (int c = lane + 32 * kWarpChunks; c < chunks; c += 32) {
            Raw<float> x;
            x.load(from + 8 * c, cols - 8 * c, j.vec);
            put(x, c);
        }
    }
}

// Whether rows of so many columns go to warps.  Measured with warps and with blocks, all of a forward call: 4096 x 768 x 2048 168 us and
// 173 us, 64 x 300 x 130 x 900 324 us and 298 us, 20000 x 64 x 1024 152 us and 148 us.
inline bool long_rows(int64_t cols) { return cols >= 512; }

// Where a thread of a block is in a unit of `slice` rows by 32 chunks (fewer where rows are shorter; a power of two of threads
// lies along a row): chunk `chunk`, if the row has it, of the rows first + group, first + group + step, ... below end.
struct StripPlace {
    int64_t batch, first, end;
    int lanes, chunk, strip, group, step;
};
__device__ __forceinline__ StripPlace strip_place(int64_t unit, int64_t rows, int64_t chunks, int slice)
{
    StripPlace s;
    const int64_t strips = (chunks + 31) / 32, slices = (rows + slice - 1) / slice, t = unit / strips;
    s.strip = (int)(unit - t * strips);
    s.batch = t / slices;
    s.lanes = row_threads(chunks, 32);
    s.chunk = s.strip * 32 + (threadIdx.x & (s.lanes - 1));
    s.first = (t - s.batch * slices) * slice;
    s.group = threadIdx.x / s.lanes;
    s.step = 256 / s.lanes;
    s.end = min(s.first + slice, rows);
    return s;
}
// Rows of a unit: few where there would be too few units for the device otherwise (a thread goes through its rows one after the
// other), and no more adding up of their largest values than that takes.  Gradient of 1024 x 512 x 1024: 79 us, 97 us with 64 rows
// throughout.
inline int slice_rows(int64_t rows, int64_t chunks, int64_t batches, int sms)
{
    int slice = 8;
    const auto units = [&] { return batches * ((rows + slice - 1) / slice) * ((chunks + 31) / 32); };
    while ((slice < 64 && units() > (int64_t)sms * 5 / 2) || (slice < 1024 && units() > (int64_t)sms * 16)) slice *= 2;
    return slice;
}

// Largest finite values of columns, added to what `peaks` holds.
__global__ void __launch_bounds__(256) column_peaks_kernel(const __grid_constant__ PackJobs jobs)
{
    grid_launch_dependents();
    __shared__ uint32_t peaks[256];
    for (int64_t at = blockIdx.x; at < jobs.units; at += gridDim.x) {
        const PackJob& j = jobs.of(at);
        const StripPlace s = strip_place(at - j.first, j.rows, j.chunks, jobs.slice);
        peaks[threadIdx.x] = 0;
        __syncthreads();
        uint32_t p[8] = {};
        if (s.chunk < j.chunks) {
            const float* const from = static_cast<const float*>(j.src) + s.batch * j.batch + 8 * s.chunk;
            const int left = (int)j.cols - 8 * s.chunk;
#pragma unroll 4
            for (int64_t r = s.first + s.group; r < s.end; r += s.step) {
                Raw<float> x;
                float v[8];
                x.load(from + r * j.ld, left, j.vec);
                x.values(v);
#pragma unroll
                for (int k = 0; k < 8; ++k) p[k] = max(p[k], finite_bits(v[k]));
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) atomicMax(&peaks[(threadIdx.x & (s.lanes - 1)) * 8 + k], p[k]);
        }
        __syncthreads();
        if (at == blockIdx.x) grid_dependency_wait();    // the launch before this one clears them and reads what this one reads
        const int64_t column = s.strip * 256 + threadIdx.x;
        if (column < j.chunks * 8 && peaks[threadIdx.x]) atomicMax(j.peaks + s.batch * j.chunks * 8 + column, peaks[threadIdx.x]);
        __syncthreads();
    }
}

// Powers of two of eight columns, and their exponents, negated, to `exponents` where there is one to keep them.
__device__ __forceinline__ void column_scales(const uint32_t* peaks, float (&scale)[8], int8_t* exponents)
{
    const uint4 p = reinterpret_cast<const uint4*>(peaks)[0], q = reinterpret_cast<const uint4*>(peaks)[1];
    const uint32_t peak[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int e = scale_exponent(peak[k]);
        scale[k] = power_of_two(e);
        w[k >> 2] |= ((uint32_t)-e & 0xFFu) << (8 * (k & 3));
    }
    if (exponents) *reinterpret_cast<uint2*>(exponents) = make_uint2(w[0], w[1]);
}

// fp32 to pairs, a power of two for each column.
__global__ void __launch_bounds__(256) pack_columns_kernel(const __grid_constant__ PackJobs jobs)
{
    grid_launch_dependents();
    grid_dependency_wait();
    for (int64_t at = blockIdx.x; at < jobs.units; at += gridDim.x) {
        const PackJob& j = jobs.of(at);
        const StripPlace s = strip_place(at - j.first, j.rows, j.chunks, jobs.slice);
        if (s.chunk >= j.chunks) continue;
        float scale[8];
        const int64_t place = (s.batch * j.chunks + s.chunk) * 8;
        column_scales(j.peaks + place, scale, s.first == 0 && s.group == 0 ? j.exponents + place : nullptr);
        const float* const from = static_cast<const float*>(j.src) + s.batch * j.batch + 8 * s.chunk;
        const int left = (int)j.cols - 8 * s.chunk;
        const Pieces<__half> dst{static_cast<__half*>(j.dst) + s.batch * j.rows * j.chunks * 8 + 8 * s.chunk, j.dst_piece, 0, 0};
#pragma unroll 4
        for (int64_t r = s.first + s.group; r < s.end; r += s.step) {
            Raw<float> x;
            float v[8];
            x.load(from + r * j.ld, left, j.vec);
            x.values(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= scale[k];
            dst.template store_at<2>(r * j.chunks * 8, v);
        }
    }
}

}  // namespace

// Whether all rows of a matrix per node start on 16 bytes.
inline bool rows_on_16(const void* p, int64_t ld, int64_t rows, int64_t node, int64_t nodes, int size)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld * size % 16 == 0) && (nodes <= 1 || node * size % 16 == 0);
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
    enum By { kChunks, kRows, kLongRows, kColumns };
    void by_rows(int64_t cols) { by = long_rows(cols) ? kLongRows : kRows; }    // of `cols` columns at least
    PackJobs jobs{};
    By by = kChunks;          // units of the launch; by rows (blocks or warps) and by columns: pairs times powers of two
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
        j.first = jobs.units;
        j.vec = rows_on_16(p, ld, rows, batch, batches, size);
        j.src_f32 = f32;
        j.pieces = pieces;
        j.dst = base + at;
        j.dst_piece = o.piece;
        ++jobs.count;
        jobs.units += by == kChunks ? batches * rows * chunks
                      : by == kLongRows ? batches * rows
                      : by == kRows ? (batches * rows + rows_of_unit(chunks) - 1) / rows_of_unit(chunks)
                                    : batches * ((rows + jobs.slice - 1) / jobs.slice) * ((chunks + 31) / 32);
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
    // Exponents of the last operand's powers of two.
    int8_t* powers()
    {
        PackJob& j = jobs.job[jobs.count - 1];
        j.exponents = reinterpret_cast<int8_t*>(base + scratch.take(j.batches * padded(by == kColumns ? j.cols : j.rows)));
        return j.exponents;
    }
    template <class T16>
    cudaError_t launch(cudaStream_t stream) const
    {
        if (!jobs.count) return cudaSuccess;
        const int64_t blocks = std::min<int64_t>((jobs.units + 255) / 256, (int64_t)sm_count() * 8);
        pack_kernel<T16><<<(unsigned)blocks, 256, 0, stream>>>(jobs);
        return cudaGetLastError();
    }
    // after: the kernel before it on the stream is one of the same call.
    cudaError_t launch_rows(bool after, void* cleared, int64_t clear_bytes, cudaStream_t stream) const
    {
        const bool warps = by == kLongRows;
        const dim3 blocks((unsigned)std::min<int64_t>(warps ? (jobs.units + 7) / 8 : jobs.units, (int64_t)sm_count() * 8));
        return launch_after_trigger(warps ? pack_long_rows_kernel : pack_rows_kernel, blocks, dim3(256), 0, stream, after, jobs, static_cast<uint4*>(cleared), clear_bytes / 16);
    }
    cudaError_t launch_columns(bool pack, cudaStream_t stream) const
    {
        const dim3 blocks((unsigned)std::min<int64_t>(jobs.units, (int64_t)sm_count() * 16));
        return launch_after_trigger(pack ? pack_columns_kernel : column_peaks_kernel, blocks, dim3(256), 0, stream, true, jobs);
    }
};
template <class T16>
Pieces<T16> pieces_of(const Operand& o)
{
    return {static_cast<T16*>(const_cast<void*>(o.base)), o.piece, o.batch, o.ld};
}

}  // namespace gpga
