// Embedding lookup with scaling, and its gradient by sorted tokens.
#include "../../include/gpga.h"
#include "gpga_embed.cuh"
#include "gpga_launch.cuh"

namespace gpga {

namespace {

__device__ __forceinline__ int64_t token_at(const void* tokens, bool is64, int64_t at)
{
    return is64 ? __ldg(static_cast<const long long*>(tokens) + at) : (int64_t)__ldg(static_cast<const int*>(tokens) + at);
}

// ---- lookup -----------------------------------------------------------------------------------------
// TPR lanes take a stretch of NC * TPR chunks of one row.  VEC: the rows of the table and of out are aligned.
template <class T, bool VEC, int TPR, int NC>
__global__ void __launch_bounds__(256) lookup_kernel(const LookupParams p)
{
    const uint32_t node = blockIdx.y, chunks = p.chunks.d;
    const uint32_t g = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    const uint32_t t = divide(g, p.stretches);
    if (t >= p.rows) return;
    const uint32_t first = (g - t * p.stretches.d) * (NC * TPR);
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)node * p.rows + t;
    const int64_t token = token_at(p.tokens, p.tokens64, row);
    const bool named = token >= 0 && token < (int64_t)p.vocab;
    const float* table = p.table + node * p.node_ldt;
    const Span span = span_of<float>(table, p.ldt, p.vocab, p.d);
    const float* from = table + (named ? token : 0) * p.ldt;
    Raw8<float, VEC> raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (!VEC || first + c * TPR + lane < chunks) raw[c].load_cached(from, (int)(first + c * TPR + lane) * kChunk, p.d, span);
    RowStore<T, VEC, TPR> store;
    T* out = static_cast<T*>(p.out) + row * p.ldo;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint32_t base = first + c * TPR;
        if (base >= chunks) break;
        f32x2_t v[4];
        if (!VEC || base + lane < chunks) {
            raw[c].get(v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = named ? mul2(v[j], both(p.scale)) : both(0.f);
        }
        store.store(out, (int)(base + lane) * kChunk, p.d, v, lane, group_mask<TPR>(), c + 1 == NC || base + TPR >= chunks);
    }
}

// ---- gradient: sort -----------------------------------------------------------------------------------
// Layout of the scratch area for one call: sorted tokens and their positions, one bit per vocabulary row that
// some token names, and the partial sums of runs that cross tiles.
constexpr uint32_t kSortPerBlock = 8192, kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr uint32_t kSortMax = 8 * kSortPerBlock;   // tokens of a node sorted by one cluster of eight blocks

struct GradLayout {
    int64_t key_off, pos_off, bit_off, part_off, total;
    uint32_t words;         // words of the bit map per node
    uint32_t tile, tiles;   // sorted entries per tile, tiles per node
    int32_t dpad;
};

// Entries per tile: long tiles leave fewer partial sums, short ones give few tokens more blocks to work on.
uint32_t tile_entries(int64_t nodes, int64_t rows) { return nodes * rows >= 64 * 148 * 4 ? 64 : 16; }

GradLayout grad_layout(int64_t nodes, int64_t rows, int64_t d, int64_t vocab)
{
    auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    if (rows > (int64_t)kSortMax) rows = kSortMax;
    GradLayout L;
    L.tile = tile_entries(nodes, rows);
    L.tiles = (uint32_t)((rows + L.tile - 1) / L.tile);
    L.words = (uint32_t)((vocab + 31) / 32);
    L.dpad = (int32_t)((d + 7) / 8 * 8);
    L.key_off = 0;
    L.pos_off = L.key_off + up(nodes * rows * 4);
    L.bit_off = L.pos_off + up(nodes * rows * 4);
    L.part_off = L.bit_off + up(nodes * (int64_t)L.words * 4);
    L.total = L.part_off + up(L.tiles > 1 ? nodes * (int64_t)L.tiles * 2 * L.dpad * 4 : 0);
    return L;
}

struct SortParams {
    const void* tokens;
    uint32_t *keys, *pos, *bits;
    int64_t node_tokens;   // tokens of one node in `tokens` (this call may sort a part of them)
    uint32_t first, count; // the part: tokens first .. first + count - 1 of every node
    uint32_t vocab, words;
    uint32_t per_block;    // entries a block holds
    int passes, digit_bits;
    bool tokens64;
};

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of this block's shared-memory word in block `rank` of the cluster, and a store to it.
__device__ __forceinline__ uint32_t cluster_address(const void* p, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ void cluster_store(uint32_t address, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(address), "r"(v) : "memory");
}

// Stable radix sort of one node's (token, position) pairs, least significant digit first, by a cluster of blocks
// that hold them in shared memory: entry e lives in block e / per_block.  A pass ranks every entry among the
// equal digits before it (lanes by a match, warps by a scan of their counts, blocks by the counts that every
// block sends to all others) and stores it straight into the block where it belongs.
// A token outside the vocabulary sorts behind all others, as the key `vocab`.
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const SortParams p)
{
    extern __shared__ uint32_t smem[];
    uint32_t* hist = smem;                          // kSortWarps x 256
    uint32_t* totals = hist + kSortWarps * 256;     // 8 x 256: every block's digit counts
    uint32_t* base = totals + 8 * 256;              // 256
    uint32_t* scan = base + 256;                    // 32
    uint32_t* key[2] = {scan + 32, scan + 32 + 2 * p.per_block};
    uint32_t* pos[2] = {key[0] + p.per_block, key[1] + p.per_block};
    uint32_t rank, blocks;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
    const uint32_t node = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t e0 = rank * p.per_block;
    const uint32_t mine = e0 >= p.count ? 0 : min(p.per_block, p.count - e0);
    for (uint32_t e = tid; e < mine; e += kSortThreads) {
        const int64_t token = token_at(p.tokens, p.tokens64, (int64_t)node * p.node_tokens + p.first + e0 + e);
        key[0][e] = token >= 0 && token < (int64_t)p.vocab ? (uint32_t)token : p.vocab;
        pos[0][e] = p.first + e0 + e;
    }
    cluster_barrier();   // every block of the cluster runs before any of them is written to
    uint32_t* bits = p.bits + (int64_t)node * p.words;
    for (uint32_t w = rank * kSortThreads + tid; w < p.words; w += blocks * kSortThreads) bits[w] = 0;

    // a warp's stretch of the block's entries
    const uint32_t stretch = ((mine + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;
    constexpr int kMost = kSortPerBlock / kSortThreads;   // entries of a thread
    const uint32_t digits = 1u << p.digit_bits;
    int cur = 0;
    for (int pass = 0; pass < p.passes; ++pass, cur ^= 1) {
        const int shift = pass * p.digit_bits;
        for (uint32_t h = tid; h < kSortWarps * 256; h += kSortThreads) hist[h] = 0;
        __syncthreads();
        uint32_t before[kMost];   // equal digits before the entry in the warp's stretch
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const uint32_t off = i * 32 + lane, e = warp * stretch + off;
            const bool live = off < stretch && e < mine;
            const unsigned active = __ballot_sync(0xFFFFFFFFu, live);
            if (!active) break;
            if (live) {
                const uint32_t digit = (key[cur][e] >> shift) & (digits - 1);
                const unsigned same = __match_any_sync(active, digit);
                const uint32_t had = hist[warp * 256 + digit];
                __syncwarp(active);
                before[i] = had + __popc(same & ((1u << lane) - 1u));
                if ((int)lane == __ffs(same) - 1) hist[warp * 256 + digit] = had + __popc(same);
            }
            __syncwarp();
        }
        __syncthreads();
        if (tid < digits) {
            uint32_t run = 0;
            for (uint32_t w = 0; w < kSortWarps; ++w) {
                const uint32_t n = hist[w * 256 + tid];
                hist[w * 256 + tid] = run;
                run += n;
            }
            for (uint32_t b = 0; b < blocks; ++b) cluster_store(cluster_address(totals + rank * 256 + tid, b), run);
        }
        cluster_barrier();
        uint32_t all = 0, ahead = 0;   // of this digit: in all blocks, in the blocks before this one
        if (tid < digits)
            for (uint32_t b = 0; b < blocks; ++b) {
                const uint32_t n = totals[b * 256 + tid];
                if (b < rank) ahead += n;
                all += n;
            }
        uint32_t upto = all;   // inclusive scan over the digits
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t n = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= (uint32_t)o) upto += n;
        }
        if (lane == 31 && warp < 8) scan[warp] = upto;
        __syncthreads();
        if (tid < digits) {
            for (uint32_t w = 0; w < warp; ++w) upto += scan[w];
            base[tid] = upto - all + ahead;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const uint32_t off = i * 32 + lane, e = warp * stretch + off;
            if (off < stretch && e < mine) {
                const uint32_t k = key[cur][e], digit = (k >> shift) & (digits - 1);
                const uint32_t to = base[digit] + hist[warp * 256 + digit] + before[i];
                const uint32_t block = to / p.per_block, at = to - block * p.per_block;
                cluster_store(cluster_address(key[cur ^ 1] + at, block), k);
                cluster_store(cluster_address(pos[cur ^ 1] + at, block), pos[cur][e]);
            }
        }
        cluster_barrier();
    }
    const int64_t out = (int64_t)node * p.count + e0;
    for (uint32_t e = tid; e < mine; e += kSortThreads) {
        const uint32_t k = key[cur][e];
        p.keys[out + e] = k;
        p.pos[out + e] = pos[cur][e];
        if (k < p.vocab && (e == 0 || key[cur][e - 1] != k)) atomicOr(bits + (k >> 5), 1u << (k & 31));
    }
}

// ---- gradient: sums -----------------------------------------------------------------------------------
struct SumParams {
    const void* dout;
    float* grad;
    const uint32_t *keys, *pos, *bits;
    float* part;
    int64_t ldo, ldg, node_ldg;
    int64_t node_rows;       // rows of dout per node
    uint32_t count, vocab, words, tile, tiles;
    int32_t d, dpad;
    uint32_t tile_blocks;    // blocks 0 .. tile_blocks - 1 (x) sum, the others write zeros
    uint32_t zero_blocks;
    float scale;
    bool accumulate, gvec;   // gvec: 128-bit accesses to grad
};

// The sorted entries are cut into tiles of p.tile; TX threads walk a tile's entries over 8 TX columns and keep the
// running sum of one token.  A token whose entries all lie in the tile is written to its row of grad; one that
// comes from the tile before or goes on into the next leaves a partial sum (slot 0: came from before, slot 1:
// starts here and goes on).
template <class T, bool VEC, int TX>
__device__ __forceinline__ void sum_tile(const SumParams& p, uint32_t node, uint32_t tile, int c0, int tx)
{
    constexpr int U = VEC && sizeof(T) == 2 ? 8 : 4;   // entries whose loads are in flight together
    constexpr int LANES = TX < 32 ? TX : 32;
    const uint32_t* keys = p.keys + (int64_t)node * p.count;
    const uint32_t* pos = p.pos + (int64_t)node * p.count;
    const T* dout = static_cast<const T*>(p.dout) + (int64_t)node * p.node_rows * p.ldo;
    const Span span = span_of<T>(dout, p.ldo, p.node_rows, p.d);
    const uint32_t begin = tile * p.tile, end = min(begin + p.tile, p.count);
    float* part = p.part + ((int64_t)node * p.tiles + tile) * 2 * p.dpad;
    const uint32_t none = 0xFFFFFFFFu;
    const uint32_t prev = begin ? keys[begin - 1] : none, next = end < p.count ? keys[end] : none;
    const unsigned group = group_mask<TX>();
    const int c = c0 + tx * 8;
    f32x2_t acc[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};
    uint32_t cur = keys[begin];
    bool from_before = cur == prev;
    auto flush = [&](bool goes_on) {
        if (cur >= p.vocab) return;
        if (from_before || goes_on) {
            float* to = part + (from_before ? 0 : p.dpad);
            if (c < p.dpad) {
                *reinterpret_cast<float4*>(to + c) = join4(acc[0], acc[1]);
                *reinterpret_cast<float4*>(to + c + 4) = join4(acc[2], acc[3]);
            }
            return;
        }
        float* to = p.grad + node * p.node_ldg + (int64_t)cur * p.ldg;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = mul2(acc[j], both(p.scale));
        if (p.gvec) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (c + 4 * h < p.d) {
                    float4 a = join4(acc[2 * h], acc[2 * h + 1]);
                    float4* at = reinterpret_cast<float4*>(to + c) + h;
                    if (p.accumulate) a = add4(*at, a);
                    __stcs(at, a);
                }
        } else {
            if (p.accumulate) {
                Raw8<float, false> old;
                f32x2_t v[4];
                old.load(to, c, p.d, span_of<float>(to, 0, 1, p.d));
                old.get(v);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = add2(v[j], acc[j]);
            }
            RowStore<float, false, LANES> store;
            store.store(to, c, p.d, acc, tx % LANES, group, true);
        }
    };
    for (uint32_t e0 = begin; e0 < end; e0 += U) {
        const uint32_t own_e = min(e0 + (tx & (U - 1)), end - 1);
        const uint32_t own_key = keys[own_e], own_pos = pos[own_e];
        uint32_t k[U];
        Raw8<T, VEC> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u] = __shfl_sync(group, own_key, u, U);
            const uint32_t at = __shfl_sync(group, own_pos, u, U);
            if (e0 + u < end && k[u] < p.vocab && (!VEC || c < p.d)) raw[u].load(dout + (int64_t)at * p.ldo, c, p.d, span);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (e0 + u < end) {
                if (k[u] != cur) {
                    flush(false);
                    cur = k[u];
                    from_before = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = both(0.f);
                }
                if (cur < p.vocab && c < p.d) {
                    f32x2_t v[4];
                    raw[u].get(v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = add2(acc[j], v[j]);
                }
            }
        }
    }
    flush(cur == next);
}

// Rows of grad that no token names: eight rows (a byte of the bit map) at a time.
__device__ __forceinline__ void zero_rows(const SumParams& p, uint32_t node, uint32_t first)
{
    const uint32_t eighths = (p.vocab + 7) / 8;
    const uint32_t* bits = p.bits + (int64_t)node * p.words;
    for (uint32_t q = first; q < eighths; q += p.zero_blocks) {
        const uint32_t named = (bits[q >> 2] >> ((q & 3) * 8)) & 0xFFu;
        for (uint32_t r = 0; r < 8; ++r) {
            const uint32_t v = q * 8 + r;
            if (v >= p.vocab || (named >> r & 1)) continue;
            float* to = p.grad + node * p.node_ldg + (int64_t)v * p.ldg;
            if (p.gvec) {
                for (int c = threadIdx.x * 4; c < p.d; c += blockDim.x * 4)
                    __stcs(reinterpret_cast<float4*>(to + c), make_float4(0.f, 0.f, 0.f, 0.f));
            } else {
                for (int c = threadIdx.x; c < p.d; c += blockDim.x) to[c] = 0.f;
            }
        }
    }
}

template <class T, bool VEC, int TX>
__global__ void __launch_bounds__(128) lookup_grad_kernel(const SumParams p)
{
    const uint32_t node = blockIdx.z;
    grid_dependency_wait();
    if (blockIdx.x >= p.tile_blocks) {
        if (blockIdx.y == 0) zero_rows(p, node, blockIdx.x - p.tile_blocks);
        return;
    }
    const uint32_t tile = blockIdx.x * (128 / TX) + threadIdx.x / TX;
    if (tile < p.tiles) sum_tile<T, VEC, TX>(p, node, tile, blockIdx.y * TX * 8, threadIdx.x % TX);
}

// Tokens whose entries span tiles: the sum of the tiles' partial sums, in their order.
// Blocks 0 .. tiles - 1 (x): the token that goes on from tile x and starts there, if it spans at most kShortRun
// more tiles; a thread adds four columns.  The other blocks: a longer run, taken by the first tile inside it
// whose number is a multiple of kShortRun; eight warps add every eighth partial sum of 128 columns.
constexpr uint32_t kShortRun = 16;
__global__ void __launch_bounds__(256) lookup_grad_join_kernel(const SumParams p)
{
    __shared__ float4 sums[8][32];
    grid_dependency_wait();
    const uint32_t node = blockIdx.z;
    const uint32_t* keys = p.keys + (int64_t)node * p.count;
    const bool is_long = blockIdx.x >= p.tiles;
    uint32_t tile = is_long ? (blockIdx.x - p.tiles + 1) * kShortRun : blockIdx.x;
    if (tile >= p.tiles) return;
    uint32_t token;
    if (is_long) {
        // the run that comes into this tile, and the tile where it starts
        const uint32_t begin = tile * p.tile;
        token = keys[begin];
        if (token >= p.vocab || keys[begin - 1] != token) return;
        uint32_t lo = 0, hi = begin;   // first entry of the token
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (keys[mid] < token) lo = mid + 1; else hi = mid;
        }
        const uint32_t start = lo / p.tile;
        if (start + kShortRun < tile) return;   // an earlier multiple of kShortRun is inside the run
        tile = start;
    } else {
        const uint32_t begin = tile * p.tile, end = begin + p.tile;
        if (end >= p.count) return;
        token = keys[end];
        if (token >= p.vocab || keys[end - 1] != token) return;
        if (begin && keys[begin - 1] == token) return;   // starts in an earlier tile
    }
    uint32_t lo = (tile + 1) * p.tile, hi = p.count;   // one past the token's last entry
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (keys[mid] <= token) lo = mid + 1; else hi = mid;
    }
    const uint32_t more = (lo - 1) / p.tile - tile;   // tiles after the first
    if ((more > kShortRun) != is_long) return;
    const float* part = p.part + ((int64_t)node * p.tiles + tile) * 2 * p.dpad;
    const int64_t step = 2 * (int64_t)p.dpad;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = is_long ? blockIdx.y * 128 + lane * 4 : (blockIdx.y * 256 + threadIdx.x) * 4;
    if (!is_long && c >= p.d) return;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < p.d) {
        if (!is_long) {
            sum = *reinterpret_cast<const float4*>(part + p.dpad + c);
            for (uint32_t m = 1; m <= more; ++m) sum = add4(sum, *reinterpret_cast<const float4*>(part + m * step + c));
        } else {
            if (warp == 0) sum = *reinterpret_cast<const float4*>(part + p.dpad + c);
#pragma unroll 8
            for (uint32_t m = 1 + warp; m <= more; m += 8) sum = add4(sum, *reinterpret_cast<const float4*>(part + m * step + c));
        }
    }
    if (is_long) {
        sums[warp][lane] = sum;
        __syncthreads();
        if (warp || c >= p.d) return;
#pragma unroll
        for (int w = 1; w < 8; ++w) sum = add4(sum, sums[w][lane]);
    }
    float* to = p.grad + node * p.node_ldg + (int64_t)token * p.ldg + c;
    sum = scale4(sum, p.scale);
    if (p.gvec && c + 4 <= p.d) {
        if (p.accumulate) sum = add4(*reinterpret_cast<const float4*>(to), sum);
        __stcs(reinterpret_cast<float4*>(to), sum);
    } else {
        const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < p.d) to[j] = (p.accumulate ? to[j] : 0.f) + v[j];
    }
}

template <class T, bool VEC, int TX>
cudaError_t sums_as(SumParams p, uint32_t nodes, cudaStream_t s)
{
    const uint32_t per = 128 / TX;
    p.tile_blocks = (p.tiles + per - 1) / per;
    const uint32_t slabs = (uint32_t)(p.d + 8 * TX - 1) / (8 * TX);
    if (p.accumulate) p.zero_blocks = 0;
    else {
        const uint32_t eighths = (p.vocab + 7) / 8, most = (148 * 16 + nodes - 1) / nodes;
        p.zero_blocks = eighths < most ? eighths : most;
    }
    if (!(p.tile_blocks + p.zero_blocks)) return cudaSuccess;
    return launch_after_trigger(lookup_grad_kernel<T, VEC, TX>, dim3(p.tile_blocks + p.zero_blocks, slabs, nodes), dim3(128), 0, s,
                                true, p);
}

template <class T, bool VEC>
cudaError_t sums_of(const SumParams& p, uint32_t nodes, cudaStream_t s)
{
    if (p.d <= 64) return sums_as<T, VEC, 8>(p, nodes, s);
    if (p.d <= 256) return sums_as<T, VEC, 32>(p, nodes, s);
    return sums_as<T, VEC, 128>(p, nodes, s);
}

bool aligned(const void* p, int64_t ld, int size) { return (((uintptr_t)p) & 15u) == 0 && (ld * size) % 16 == 0; }

template <class T, bool VEC, int TPR, int NC>
cudaError_t lookup_as(LookupParams& p, cudaStream_t s)
{
    p.stretches = make_divisor((p.chunks.d + NC * TPR - 1) / (NC * TPR));
    const uint64_t groups = (uint64_t)p.rows * p.stretches.d;
    lookup_kernel<T, VEC, TPR, NC><<<dim3((unsigned)((groups + 256 / TPR - 1) / (256 / TPR)), p.nodes), 256, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool VEC>
cudaError_t lookup_by_width(LookupParams& p, cudaStream_t s)
{
    const uint32_t chunks = p.chunks.d;
    return chunks <= 8    ? lookup_as<T, VEC, 8, 1>(p, s)
           : chunks <= 32 ? lookup_as<T, VEC, 32, 1>(p, s)
           : chunks <= 64 ? lookup_as<T, VEC, 32, 2>(p, s)
                          : lookup_as<T, VEC, 32, 4>(p, s);
}

template <class T>
cudaError_t lookup_of(LookupParams p, cudaStream_t s)
{
    if (!p.rows) return cudaSuccess;
    p.chunks = make_divisor((uint32_t)(p.d + kChunk - 1) / kChunk);
    const bool vec = p.d % kChunk == 0 && aligned(p.table, p.ldt, 4) && p.node_ldt % 4 == 0 && aligned(p.out, p.ldo, sizeof(T));
    return vec ? lookup_by_width<T, true>(p, s) : lookup_by_width<T, false>(p, s);
}

}  // namespace

cudaError_t launch_lookup(const LookupParams& p, int dtype, cudaStream_t s)
{
    return dtype == GPGA_DTYPE_F32 ? lookup_of<float>(p, s) : dtype == GPGA_DTYPE_BF16 ? lookup_of<__nv_bfloat16>(p, s) : lookup_of<__half>(p, s);
}

int64_t lookup_grad_scratch_bytes(int64_t nodes, int64_t rows, int64_t d, int64_t vocab)
{
    return grad_layout(nodes, rows, d, vocab).total;
}

cudaError_t launch_lookup_grad(const LookupGradParams& g, int dtype, cudaStream_t s)
{
    const GradLayout L = grad_layout(g.nodes, g.rows, g.d, g.vocab);
    SortParams q;
    q.tokens = g.tokens;
    q.keys = reinterpret_cast<uint32_t*>(g.scratch + L.key_off);
    q.pos = reinterpret_cast<uint32_t*>(g.scratch + L.pos_off);
    q.bits = reinterpret_cast<uint32_t*>(g.scratch + L.bit_off);
    q.node_tokens = g.rows;
    q.vocab = g.vocab;
    q.words = L.words;
    q.tokens64 = g.tokens64;
    int key_bits = 1;
    while (g.vocab >> key_bits) ++key_bits;   // keys are 0 .. vocab
    q.passes = (key_bits + 7) / 8;
    q.digit_bits = (key_bits + q.passes - 1) / q.passes;

    SumParams p;
    p.dout = g.dout;
    p.grad = g.grad;
    p.keys = q.keys;
    p.pos = q.pos;
    p.bits = q.bits;
    p.part = reinterpret_cast<float*>(g.scratch + L.part_off);
    p.ldo = g.ldo;
    p.ldg = g.ldg;
    p.node_ldg = g.node_ldg;
    p.node_rows = g.rows;
    p.vocab = g.vocab;
    p.words = L.words;
    p.tile = L.tile;
    p.d = g.d;
    p.dpad = L.dpad;
    p.scale = g.scale;
    p.gvec = g.d % 4 == 0 && aligned(g.grad, g.ldg, 4) && g.node_ldg % 4 == 0;
    const int size = dtype == GPGA_DTYPE_F32 ? 4 : 2;
    const bool vec = g.d % 8 == 0 && aligned(g.dout, g.ldo, size);

    // one cluster sorts up to kSortMax tokens of a node; the parts of a longer row list are added up one after
    // the other
    uint32_t first = 0;
    do {
        const uint32_t count = g.rows - first < kSortMax ? g.rows - first : kSortMax;
        q.first = first;
        q.count = count;
        uint32_t blocks = 1;
        while (blocks < 8 && blocks * 1024 < count) blocks *= 2;
        q.per_block = (count + blocks - 1) / blocks;
        if (q.per_block == 0) q.per_block = 1;
        const size_t smem = (kSortWarps * 256 + 8 * 256 + 256 + 32 + 4 * (size_t)q.per_block) * 4;
        static unsigned long long limit_set = 0;
        cudaError_t e = ensure_smem_limit(sort_tokens_kernel, (kSortWarps * 256 + 8 * 256 + 256 + 32 + 4 * (int)kSortPerBlock) * 4, limit_set);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(blocks, g.nodes);
        cfg.blockDim = dim3(kSortThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = blocks;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, sort_tokens_kernel, q);
        if (e != cudaSuccess) return e;

        p.count = count;
        p.tiles = (count + L.tile - 1) / L.tile;
        p.accumulate = g.accumulate || first > 0;
        e = dtype == GPGA_DTYPE_F32    ? (vec ? sums_of<float, true>(p, g.nodes, s) : sums_of<float, false>(p, g.nodes, s))
            : dtype == GPGA_DTYPE_BF16 ? (vec ? sums_of<__nv_bfloat16, true>(p, g.nodes, s) : sums_of<__nv_bfloat16, false>(p, g.nodes, s))
                                       : (vec ? sums_of<__half, true>(p, g.nodes, s) : sums_of<__half, false>(p, g.nodes, s));
        if (e != cudaSuccess) return e;
        if (p.tiles > 1) {
            // y covers the columns at 1024 per block for the short runs and at 128 for the long ones
            const uint32_t longs = (p.tiles - 1) / kShortRun;
            e = launch_after_trigger(lookup_grad_join_kernel, dim3(p.tiles + longs, (g.d + 127) / 128, g.nodes), dim3(256), 0, s, true, p);
            if (e != cudaSuccess) return e;
        }
        first += count;
    } while (first < g.rows);
    return cudaSuccess;
}

}  // namespace gpga
