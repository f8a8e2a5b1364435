// What the token-block kernels (embedding lookup, dropout, layer norm) share: activation types, accesses
// to a row in chunks of eight columns, and the dropout mask.  sm_100a only.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gpga_device.cuh"

namespace gpga {

// Sets the text that gpga_last_error(NULL) returns to the calling thread (defined with the C ABI).
int32_t token_error(int32_t code, const char* text) noexcept;

constexpr int kChunk = 8;   // columns per generator call: eight 16-bit halves of its four words

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void unpack16(uint32_t w, float& lo, float& hi, __nv_bfloat16)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack16(uint32_t w, float& lo, float& hi, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    lo = f.x;
    hi = f.y;
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, __half)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Accesses to rows in chunks of eight columns, column 8 chunk .. 8 chunk + 7.
//
// VEC: every row starts on 16 bytes and d is a multiple of eight (the host has checked): 128-bit accesses.
//
// Otherwise a row starts at any element and its last chunk may be partial, but the accesses stay 128 bits wide: a chunk
// is cut out of the two or three aligned 16-byte pieces ("granules") it lies in, and a granule is written by the lane
// that holds its last columns, which takes the others from its neighbour (a shuffle).  Layer norm of 4 x 8000 rows of 1001
// bf16 columns with residual and dropout: element by element 175 us, this way 121 us, with shifted chunks (below) 69 us.
// A granule that reaches past the array's first or last byte is read element by element; bytes of neighbouring rows
// that come along are dropped, never written.
struct Span {   // bytes of a whole array: first byte of its first row, one past the last of its last row
    const char *lo, *hi;
    __device__ __forceinline__ bool has(const void* p, int bytes) const
    {
        return static_cast<const char*>(p) >= lo && static_cast<const char*>(p) + bytes <= hi;
    }
};
template <class T>
__device__ __forceinline__ Span span_of(const void* p, int64_t ld, int64_t rows, int d)
{
    const char* lo = static_cast<const char*>(p);
    return {lo, lo + ((rows - 1) * ld + d) * (int64_t)sizeof(T)};
}

// Words o[0 .. N) = bytes a .. a + 4 N - 1 of the words w[0 .. N + 4), 0 <= a < 16.
template <int N>
__device__ __forceinline__ void cut(const uint32_t* w, uint32_t a, uint32_t* o)
{
    uint32_t u[N + 2], t[N + 1];
#pragma unroll
    for (int i = 0; i < N + 2; ++i) u[i] = a & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < N + 1; ++i) t[i] = a & 4 ? u[i + 1] : u[i];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = __funnelshift_r(t[i], t[i + 1], (a & 3) * 8);
}

// A chunk in registers is four pairs of fp32, so that its arithmetic takes packed instructions.
template <class T>
__device__ __forceinline__ void unpack8(const uint32_t* w, f32x2_t* v)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            v[j] = pack2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
        } else {
            float lo, hi;
            unpack16(w[j], lo, hi, T());
            v[j] = pack2(lo, hi);
        }
    }
}
template <class T>
__device__ __forceinline__ void pack8(const f32x2_t* v, uint32_t* w)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = unpack2(v[j]);
        if constexpr (sizeof(T) == 4) {
            w[2 * j] = __float_as_uint(f.x);
            w[2 * j + 1] = __float_as_uint(f.y);
        } else {
            w[j] = pack16(f.x, f.y, T());
        }
    }
}
__device__ __forceinline__ float element(const f32x2_t* v, int j) { return j & 1 ? unpack2(v[j >> 1]).y : unpack2(v[j >> 1]).x; }
// Zeroes the columns from the n-th on (the end of a row that is not a multiple of eight).
__device__ __forceinline__ void keep_first(f32x2_t* v, int n)
{
    if (n >= 8) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = unpack2(v[j]);
        v[j] = pack2(2 * j < n ? f.x : 0.f, 2 * j + 1 < n ? f.y : 0.f);
    }
}

// A chunk as read from memory.
template <class T, bool VEC> struct Raw8 {
    static constexpr int W = 2 * sizeof(T);   // words of a chunk
    uint32_t w[VEC ? W : W + 4];
    uint32_t a;   // !VEC: byte offset of the chunk in w
    int n;        // !VEC: columns that the row has here
    // read once (VEC: with the streaming hint)
    __device__ __forceinline__ void load(const T* row, int col, int d, const Span& s) { load_as<true>(row, col, d, s); }
    // kept in the caches: other rows of the launch may be read again
    __device__ __forceinline__ void load_cached(const T* row, int col, int d, const Span& s) { load_as<false>(row, col, d, s); }
    template <bool ONCE>
    __device__ __forceinline__ void load_as(const T* row, int col, int d, const Span& s)
    {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const uint4* at = reinterpret_cast<const uint4*>(row + col) + i;
                const uint4 q = ONCE ? __ldcs(at) : *at;
                w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
            }
        } else {
            n = max(0, min(8, d - col));
            a = 0;
            if (n == 0) return;
            const char* at = reinterpret_cast<const char*>(row + col);
            a = (uint32_t)(uintptr_t)at & 15u;
            const char* g = at - a;
            const int bytes = (int)a + n * (int)sizeof(T);
            if (g >= s.lo && g + (bytes + 15) / 16 * 16 <= s.hi) {
#pragma unroll
                for (int i = 0; i < W / 4 + 1; ++i) {
                    uint4 q = make_uint4(0, 0, 0, 0);
                    if (16 * i < bytes) q = reinterpret_cast<const uint4*>(g)[i];
                    w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
                }
            } else {
                float v[8];
                f32x2_t v2[4];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = j < n && col + j >= 0 ? to_f32(row[col + j]) : 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) v2[j] = pack2(v[2 * j], v[2 * j + 1]);
                pack8<T>(v2, w);
                a = 0;
            }
        }
    }
    // Makes the compiler unpack the words again after this point instead of keeping the values it has (in more registers
    // than the words take, or spilled) since an earlier get().
    __device__ __forceinline__ void unpack_again()
    {
#pragma unroll
        for (int i = 0; i < (VEC ? W : W + 4); ++i) asm volatile("" : "+r"(w[i]));
    }
    __device__ __forceinline__ void get(f32x2_t* v) const
    {
        if constexpr (VEC) {
            unpack8<T>(w, v);
        } else {
            uint32_t o[W];
            cut<W>(w, a, o);
            unpack8<T>(o, v);
            keep_first(v, n);
        }
    }
};

// Stores a chunk to 16-byte aligned memory.
template <class T>
__device__ __forceinline__ void store8(T* at, const f32x2_t* v)
{
    uint32_t o[2 * sizeof(T)];
    pack8<T>(v, o);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
        __stcs(reinterpret_cast<uint4*>(at) + i, make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
}

// Stores the chunks of a row that neighbouring lanes hold.  Lane `lane` of the TPR lanes of `mask` that share the
// call holds chunk `first + lane`, `first` growing by TPR from call to call of one row; every lane of them makes the
// call, with n = 0 where the row has no such chunk.  prev keeps the words of the call before, so that a row leaves only
// its two ends to single elements.
template <class T, bool VEC, int TPR> struct RowStore {
    static constexpr int W = 2 * sizeof(T);
    uint32_t prev[VEC ? 1 : W];
    bool any;   // !VEC: there was a call before
    __device__ __forceinline__ RowStore() : any(false) {}
    // last: no further call follows for this row in these lanes.  VEC: lanes without the chunk need not call.
    __device__ __forceinline__ void store(T* row, int col, int d, const f32x2_t* v, int lane, unsigned mask, bool last)
    {
        if constexpr (VEC) {
            if (col < d) store8<T>(row + col, v);
        } else {
            const int n = max(0, min(8, d - col)), next_n = max(0, min(8, d - col - 8));
            const char* at = reinterpret_cast<const char*>(row + col);
            const uint32_t a = (uint32_t)(uintptr_t)at & 15u;
            const int head = (16 - (int)a) / (int)sizeof(T);   // columns up to the next granule
            constexpr int P = 16 / sizeof(T);                  // columns of a granule
            uint32_t c[W + 4];   // the last 16 bytes of the chunk before, then this chunk
            pack8<T>(v, c + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t mine = c[4 + W - 4 + i];
                c[i] = __shfl_sync(mask, lane == TPR - 1 ? prev[W - 4 + i] : mine, (lane + TPR - 1) % TPR, TPR);
            }
            const bool has_prev = a == 0 || lane > 0 || any;
            const bool has_next = lane < TPR - 1 || !last;
#pragma unroll
            for (int i = 0; i < W; ++i) prev[i] = c[4 + i];
            any = true;
            uint32_t o[W];
            cut<W>(c, a ? 16 - a : 0, o);   // the granules that end inside this chunk
            if (a == 0) {
#pragma unroll
                for (int i = 0; i < W; ++i) o[i] = c[4 + i];
            }
            T* g = row + col - (a ? P - head : 0);   // first granule
            const int first_end = a ? head : P;      // columns of this chunk in it
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const int end = first_end + i * P, begin = i ? end - P : 0;   // columns of this chunk in granule i
                if (n >= end && (i || has_prev))
                    __stcs(reinterpret_cast<uint4*>(g) + i, make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
                else if (n > begin) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j >= begin && j < min(n, end)) row[col + j] = from_f32<T>(element(v, j));
                }
            }
            // the columns behind the last granule: the next lane writes them where it can
            const int tail = first_end + (W / 4 - 1) * P;
            if (n > tail && !(has_next && next_n >= head)) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j >= tail && j < n) row[col + j] = from_f32<T>(element(v, j));
            }
        }
    }
};

// Eight fp32 parameters of a row, kept in the caches; vec: 128-bit accesses (the row starts on 16 bytes and has eight
// columns here).
__device__ __forceinline__ void param8(const float* w, int col, int d, bool vec, f32x2_t* v)
{
    if (vec) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(w + col)), b = __ldg(reinterpret_cast<const float4*>(w + col) + 1);
        v[0] = pack2(a.x, a.y); v[1] = pack2(a.z, a.w);
        v[2] = pack2(b.x, b.y); v[3] = pack2(b.z, b.w);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = pack2(col + 2 * j < d ? __ldg(w + col + 2 * j) : 0.f, col + 2 * j + 1 < d ? __ldg(w + col + 2 * j + 1) : 0.f);
    }
}

// Threads that share a row: TPR, in one warp up to 32 of them.
template <int TPR>
__device__ __forceinline__ unsigned group_mask()
{
    return TPR >= 32 ? 0xFFFFFFFFu : ((1u << (TPR & 31)) - 1u) << ((threadIdx.x & 31) / TPR * TPR);
}

__device__ __forceinline__ f32x2_t both(float v) { return pack2(v, v); }
__device__ __forceinline__ float sum2(f32x2_t v)
{
    const float2 f = unpack2(v);
    return f.x + f.y;
}

// Dropout of one activation tensor: what a launch needs to form any element's mask.
struct DropMask {
    PhiloxKeys keys;
    bool on;          // false: nothing is dropped
    uint32_t above;   // 65536 q - 1: an element is kept iff its 16 bits, as the upper half of a word, are above
    float scale;      // 65536 / (65536 - q), 0 when everything is dropped
    uint32_t node0;   // global index of local node 0
    uint32_t k, stream;
};

// Dropout of chunk `chunk` (columns 8 chunk .. 8 chunk + 7) of row t of local node i: counter (t * chunks + chunk,
// node, k, stream); column 8 chunk + j owns half j & 1 (low half first) of word j >> 1.  A dropped element is a
// selected zero, so that NaN and infinities vanish with it.  The lower half of a word cannot change whether the upper
// one is above (65536 q - 1), so that the upper half is compared in place.
__device__ __forceinline__ uint4 drop_words(const DropMask& m, uint32_t group, uint32_t i)
{
    return philox4x32_10(group, m.node0 + i, m.k, m.stream, m.keys);
}
__device__ __forceinline__ void drop8_by(const DropMask& m, const uint32_t* word, f32x2_t* v)
{
    const f32x2_t scale = both(m.scale);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = unpack2(mul2(v[j], scale));
        v[j] = pack2(word[j] << 16 > m.above ? f.x : 0.f, word[j] > m.above ? f.y : 0.f);
    }
}
__device__ __forceinline__ void drop8(const DropMask& m, uint32_t group, uint32_t i, f32x2_t* v)
{
    if (!m.on) return;
    const uint4 w = drop_words(m, group, i);
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
    drop8_by(m, word, v);
}

// ---- shifted chunks ---------------------------------------------------------------------------------
// Rows that start off a 16-byte boundary but all alike: where every activation of a call has the same distance s (in
// columns) of its rows from the boundary before them, chunk m is taken as columns 8 m - s .. 8 m - s + 7, which is aligned
// memory in each of them; only the first and the last chunk of a row are partial.  s repeats after 16 / sizeof(T) rows,
// and a block takes rows of one s.
// kShiftRows: rows after which s repeats.
template <class T> constexpr uint32_t kShiftRows = 16 / sizeof(T);

template <class T>
__device__ __forceinline__ int shift_of(const T* row) { return (int)((uint32_t)(uintptr_t)row & 15u) / (int)sizeof(T); }

// The columns of a chunk from column `col` on that lie in the row, a bit each; and zero in place of the others.
__device__ __forceinline__ uint32_t columns_there(int col, int d)
{
    const int first = max(0, -col), end = max(first, min(8, d - col));
    return (1u << end) - (1u << first);
}
__device__ __forceinline__ void keep_columns(f32x2_t* v, uint32_t there)
{
    if (there == 0xFFu) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = unpack2(v[j]);
        v[j] = pack2(there & 1u << 2 * j ? f.x : 0.f, there & 2u << 2 * j ? f.y : 0.f);
    }
}

// Whether the memory that a row's partial chunks reach into on both sides belongs to the array.
template <class T>
__device__ __forceinline__ bool inside(const T* row, int d, const Span& s) { return s.has(row - 7, (d + 14) * (int)sizeof(T)); }

// Reads the aligned chunk at column `col` (possibly before the row's start or past its end) into the words of a chunk.
// safe: the whole chunk is in the row or in the array; otherwise bytes beside the row are not touched and come out zero.  slots: two chunks of shared memory for the lanes of a row.
template <class T>
__device__ __forceinline__ void load_shifted(const T* row, int col, bool safe, int d, Raw8<T, true>& raw, T* slots)
{
    constexpr int W = 2 * sizeof(T);
    if (safe) {
        raw.load(row, col, d, Span());
    } else {
        T* to = slots + (col < 0 ? 0 : 8);
#pragma unroll 1
        for (int j = 0; j < 8; ++j) to[j] = col + j >= 0 && col + j < d ? row[col + j] : from_f32<T>(0.f);
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const uint4 q = reinterpret_cast<const uint4*>(to)[i];
            raw.w[4 * i] = q.x; raw.w[4 * i + 1] = q.y; raw.w[4 * i + 2] = q.z; raw.w[4 * i + 3] = q.w;
        }
    }
}

// Stores the NC chunks (the c-th at column col0 + 8 c LANES, col0 = 8 m - shift for the lane's m) that each of LANES lanes
// holds of a row.  The partial chunks at the row's ends go through `slots` (two chunks for these lanes, used once), from where
// a lane stores one element each: element by element from the two lanes that hold them, the ends cost more than all the rest.
template <class T, int LANES, int NC>
__device__ __forceinline__ void store_shifted(T* row, int col0, int d, int shift, const f32x2_t (*v)[4], T* slots, int lane, unsigned mask)
{
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = col0 + 8 * c * LANES;
        if (col >= 0 && col + 8 <= d) {
            store8<T>(row + col, v[c]);
        } else if (col < d) {
            T* to = slots + (col < 0 ? 0 : 8);
            uint32_t o[2 * sizeof(T)];
            pack8<T>(v[c], o);
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                reinterpret_cast<uint4*>(to)[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        }
    }
    // the same for all these lanes: whether the row's ends are theirs
    const int first = col0 - 8 * lane, last = (d + shift - 1) / 8 * 8 - shift;   // column of their first chunk, of the row's last
    const bool head = first < 0, tail = last >= 0 && last + 8 > d && last >= first && last < first + 8 * NC * LANES;
    if (!head && !tail) return;
    __syncwarp(mask);
#pragma unroll
    for (int k = 0; k < (LANES < 16 ? 2 : 1); ++k) {
        const int e = lane + k * LANES, at = e < 8 ? first + e : last + e - 8;
        if (e < 16 && (e < 8 ? head : tail) && at >= 0 && at < d) row[at] = slots[e];
    }
}

// The same for row after row: what depends on the columns alone is worked out once (lookup of 4 x 4096 rows of 1663 fp32, one
// row each: 39 us this way, 35 us with the function above; norm gradient of 4 x 8000 rows of 1001: 126 and 137 us
// when this was measured, 115 us with the tests taken out of full sets since).
template <class T, int LANES, int NC> struct ShiftedStore {
    T* slots;        // two pairs of chunks for these lanes, used in turn: a row's are read while the next one's are written
    int at0, at1;    // columns of the ends that this lane stores, -1: none
    uint32_t whole;  // a bit for every chunk that lies in the row; from bit 8 on, for every one that does in part
    bool ends;       // the same for all these lanes: whether any chunk is partial
    __device__ __forceinline__ ShiftedStore(int col0, int d, int shift, T* slots_, int lane) : slots(slots_), at0(-1), at1(-1), whole(0)
    {
        const int first = col0 - 8 * lane, last = (d + shift - 1) / 8 * 8 - shift;   // column of their first chunk, of the row's last
        const bool head = first < 0, tail = last >= 0 && last + 8 > d && last >= first && last < first + 8 * NC * LANES;
        ends = head || tail;
        auto end_at = [&](int e) {   // element e of the two chunks
            const int at = e < 8 ? first + e : last + e - 8;
            return e < 16 && (e < 8 ? head : tail) && at >= 0 && at < d ? at : -1;
        };
        at0 = end_at(lane);
        if (LANES < 16) at1 = end_at(lane + LANES);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = col0 + 8 * c * LANES;
            if (col >= 0 && col + 8 <= d) whole |= 1u << c;
            else if (col < d) whole |= 256u << c;
        }
    }
    __device__ __forceinline__ void store(T* row, int col0, const f32x2_t (*v)[4], int lane, unsigned mask)
    {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (whole >> c & 1) {
                store8<T>(row + col0 + 8 * c * LANES, v[c]);
            } else if (whole >> c & 256) {
                T* to = slots + (col0 + 8 * c * LANES < 0 ? 0 : 8);
                uint32_t o[2 * sizeof(T)];
                pack8<T>(v[c], o);
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                    reinterpret_cast<uint4*>(to)[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
        }
        if (!ends) return;
        __syncwarp(mask);
        if (at0 >= 0) row[at0] = slots[lane];
        if (LANES < 16 && at1 >= 0) row[at1] = slots[lane + LANES];
        slots = reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(slots) ^ 16 * sizeof(T));   // [2][16] on a boundary of its size
    }
};

// The random words of a shifted chunk: those of generator calls m - 1 (the chunk's first s columns) and m.
__device__ __forceinline__ void shifted_words(const uint4& before, const uint4& own, int s, uint32_t* word)
{
    const uint32_t w[8] = {before.x, before.y, before.z, before.w, own.x, own.y, own.z, own.w};
    if (s) {
        cut<4>(w, (uint32_t)(16 - 2 * s), word);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) word[j] = w[4 + j];
    }
}

__device__ __forceinline__ uint4 shfl4(unsigned mask, const uint4& v, int src, int width)
{
    return make_uint4(__shfl_sync(mask, v.x, src, width), __shfl_sync(mask, v.y, src, width), __shfl_sync(mask, v.z, src, width),
                      __shfl_sync(mask, v.w, src, width));
}

// n / d for n < 2^32 by a multiplication (Granlund and Montgomery's division by an invariant, with a 33-bit multiplier
// whose top bit is the added n).
struct Divisor {
    uint32_t d, mul, shift;
};
inline Divisor make_divisor(uint32_t d)
{
    Divisor v{d, 0, 0};
    while (v.shift < 32 && (uint64_t(1) << v.shift) < d) ++v.shift;
    v.mul = (uint32_t)(((uint64_t(1) << 32) * ((uint64_t(1) << v.shift) - d)) / d + 1);
    return v;
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divisor& v)
{
    return (uint32_t)(((uint64_t)__umulhi(n, v.mul) + n) >> v.shift);
}

}  // namespace gpga
