// Dropout from a counter-based generator: the mask is formed where it is used, forward and backward alike.
#include "gpga_norm_device.cuh"

namespace gpga {

namespace {

// Both tensors dense and aligned: U chunks per thread, 256 apart, their loads in flight together; no index arithmetic per
// chunk but an addition (with a division by the row's length and 64-bit products it took 134 instructions per chunk instead
// of 97, and issue slots bounded it).  Bound: HBM.  8 x 4096 x 4096 bf16: calls one after the other 88 us = 6.1 TB/s (a plain
// copy: 6.5); replayed in a graph, where part of the last pass is still in L2, 80 us, one chunk per thread 118 us.
template <class T, int U>
__global__ void __launch_bounds__(256) dropout_dense_kernel(const DropoutParams p)
{
    const uint32_t node = blockIdx.y, total = p.rows * p.chunks.d;
    const T* x = static_cast<const T*>(p.x) + (int64_t)node * total * kChunk;
    T* y = static_cast<T*>(p.y) + (int64_t)node * total * kChunk;
    const uint32_t f0 = blockIdx.x * (256 * U) + threadIdx.x;   // the host keeps total + 256 U below 2^32
    Raw8<T, true> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (f0 + u * 256 < total) raw[u].load(x + (int64_t)f0 * kChunk, u * 256 * kChunk, p.d, Span());
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (f0 + u * 256 >= total) return;
        f32x2_t v[4];
        raw[u].get(v);
        drop8(p.mask, f0 + u * 256, node, v);
        store8<T>(y + (int64_t)f0 * kChunk + u * 256 * kChunk, v);
    }
}

// Otherwise TPR lanes take a stretch of NC * TPR chunks of one row.
template <class T, bool VEC, int TPR, int NC>
__global__ void __launch_bounds__(256) dropout_rows_kernel(const DropoutParams p)
{
    const uint32_t node = blockIdx.y, chunks = p.chunks.d;
    const uint32_t g = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    const uint32_t t = divide(g, p.stretches);
    if (t >= p.rows) return;
    const uint32_t first = (g - t * p.stretches.d) * (NC * TPR);
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)node * p.rows + t;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    T* y = static_cast<T*>(p.y) + row * p.ldy;
    const Span span = span_of<T>(p.x, p.ldx, (int64_t)p.nodes * p.rows, p.d);
    Raw8<T, VEC> raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (!VEC || first + c * TPR + lane < chunks) raw[c].load(x, (int)(first + c * TPR + lane) * kChunk, p.d, span);
    RowStore<T, VEC, TPR> store;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint32_t base = first + c * TPR, chunk = base + lane;
        if (base >= chunks) break;
        f32x2_t v[4];
        if (!VEC || chunk < chunks) {
            raw[c].get(v);
            drop8(p.mask, t * chunks + chunk, node, v);
        }
        store.store(y, (int)chunk * kChunk, p.d, v, lane, group_mask<TPR>(), c + 1 == NC || base + TPR >= chunks);
    }
}

// Rows of x and y off the alignment alike: shifted chunks.  p.stretches counts those of the widest shift.  8 x 4096 rows
// of 2001 bf16 columns 70 us (cut chunks 93 us, single elements 157 us; an aligned row's rate would be 40 us): the words of
// a neighbour's generator call, shuffled and cut, are what it pays.
template <class T, int TPR, int NC>
__global__ void __launch_bounds__(256) dropout_shifted_kernel(const DropoutParams p)
{
    const uint32_t node = blockIdx.y, chunks = p.chunks.d;
    const uint32_t g = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    const uint32_t t = divide(g, p.stretches);
    if (t >= p.rows) return;
    const int64_t row = (int64_t)node * p.rows + t;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    T* y = static_cast<T*>(p.y) + row * p.ldy;
    const int lane = threadIdx.x % TPR, shift = shift_of(x);
    const uint32_t first = (g - t * p.stretches.d) * (NC * TPR);
    if ((int)first * kChunk - shift >= p.d) return;
    __shared__ __align__(16) T slots[256 / TPR][16];
    const Span span = span_of<T>(p.x, p.ldx, (int64_t)p.nodes * p.rows, p.d);
    auto col = [&](int c) { return (int)(first + c * TPR + lane) * kChunk - shift; };
    Raw8<T, true> raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (col(c) < p.d) load_shifted(x, col(c), (col(c) >= 0 && col(c) + 8 <= p.d) || span.has(x + col(c), 8 * (int)sizeof(T)), p.d, raw[c], slots[threadIdx.x / TPR]);
    const uint32_t groups = t * chunks + first;
    uint4 before = make_uint4(0, 0, 0, 0);
    if (p.mask.on && shift) before = drop_words(p.mask, groups - 1, node);
    f32x2_t v[NC][4];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        raw[c].get(v[c]);
        if (p.mask.on) {
            const uint4 own = drop_words(p.mask, groups + c * TPR + lane, node);
            const uint4 left = shfl4(group_mask<TPR>(), own, (lane + TPR - 1) % TPR, TPR);
            uint32_t word[4];
            shifted_words(lane ? left : before, own, shift, word);
            before = left;   // lane 0 has the last lane's
            drop8_by(p.mask, word, v[c]);
        }
    }
    store_shifted<T, TPR, NC>(y, col(0), p.d, shift, v, slots[threadIdx.x / TPR], lane, group_mask<TPR>());
}

// ---- launches ---------------------------------------------------------------------------------------
template <class T, bool VEC, int TPR, int NC>
cudaError_t dropout_rows(DropoutParams& p, cudaStream_t s)
{
    p.stretches = make_divisor((p.chunks.d + NC * TPR - 1) / (NC * TPR));
    const uint64_t groups = (uint64_t)p.rows * p.stretches.d;
    dropout_rows_kernel<T, VEC, TPR, NC><<<dim3((unsigned)((groups + 256 / TPR - 1) / (256 / TPR)), p.nodes), 256, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, int TPR, int NC>
cudaError_t dropout_shifted(DropoutParams& p, cudaStream_t s)
{
    p.stretches = make_divisor((p.d + kShiftRows<T> - 1 + NC * TPR * kChunk - 1) / (NC * TPR * kChunk));
    const uint64_t groups = (uint64_t)p.rows * p.stretches.d;
    dropout_shifted_kernel<T, TPR, NC><<<dim3((unsigned)((groups + 256 / TPR - 1) / (256 / TPR)), p.nodes), 256, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool VEC>
cudaError_t dropout_of(DropoutParams p, cudaStream_t s)
{
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const uint64_t total = (uint64_t)p.rows * chunks;   // per node, below 2^32
    p.chunks = make_divisor(chunks);
    if constexpr (VEC) {
        if (p.ldx == p.d && p.ldy == p.d && total < (uint64_t(1) << 32) - 1024) {
            // four chunks per thread where that still fills the SMs with blocks
            if (p.nodes * total < 148 * 8 * 1024) dropout_dense_kernel<T, 1><<<dim3((unsigned)((total + 255) / 256), p.nodes), 256, 0, s>>>(p);
            else dropout_dense_kernel<T, 4><<<dim3((unsigned)((total + 1023) / 1024), p.nodes), 256, 0, s>>>(p);
            return cudaGetLastError();
        }
    }
    if (!VEC && p.shifted) {
        const int d = p.d + (int)kShiftRows<T> - 1;
        return d <= 64    ? dropout_shifted<T, 8, 1>(p, s)
               : d <= 256 ? dropout_shifted<T, 32, 1>(p, s)
               : d <= 512 ? dropout_shifted<T, 32, 2>(p, s)
                          : dropout_shifted<T, 32, 4>(p, s);
    }
    return chunks <= 8    ? dropout_rows<T, VEC, 8, 1>(p, s)
           : chunks <= 32 ? dropout_rows<T, VEC, 32, 1>(p, s)
           : chunks <= 64 ? dropout_rows<T, VEC, 32, 2>(p, s)
                          : dropout_rows<T, VEC, 32, 4>(p, s);
}

}  // namespace

cudaError_t launch_dropout(const DropoutParams& p, int dtype, bool vec, cudaStream_t s)
{
    if (!p.rows) return cudaSuccess;
#define GPGA_CALL(T, V) dropout_of<T, V>(p, s)
    return GPGA_BY_TYPE(GPGA_CALL);
#undef GPGA_CALL
}

}  // namespace gpga
