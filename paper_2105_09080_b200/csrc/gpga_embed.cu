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
// TPR lanes take a stretch of NC * TPR chunks of one row: one token and one division per 32 NC chunks of loads.  VEC: the
// rows of the table and of out are aligned; otherwise chunks are shifted to out's alignment and cut out of the table's rows.
// Bound: HBM, where words repeat L2.  8 x 4096 tokens of 1024 into bf16 22 us (5.8 TB/s of distinct rows and outputs), a
// chunk per thread 27 us.
template <class T, bool VEC, int TPR, int NC>
__global__ void __launch_bounds__(256) lookup_kernel(const LookupParams p)
{
    __shared__ __align__(16) T slots[VEC ? 1 : 256 / TPR][16];
    const uint32_t node = blockIdx.y;
    const uint32_t g = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    const uint32_t t = divide(g, p.stretches);
    if (t >= p.rows) return;
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)node * p.rows + t;
    T* out = static_cast<T*>(p.out) + row * p.ldo;
    const int shift = VEC ? 0 : shift_of(out);
    const int first = (int)(g - t * p.stretches.d) * (NC * TPR * kChunk) - shift, col0 = first + lane * kChunk;
    if (first >= p.d) return;
    const int64_t token = token_at(p.tokens, p.tokens64, row);
    const bool named = token >= 0 && token < (int64_t)p.vocab;
    const float* table = p.table + node * p.node_ldt;
    const Span span = span_of<float>(table, p.ldt, p.vocab, p.d);
    const float* from = table + (named ? token : 0) * p.ldt;
    Raw8<float, VEC> raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (!VEC || col0 + c * TPR * kChunk < p.d) raw[c].load_cached(from, col0 + c * TPR * kChunk, p.d, span);
    f32x2_t v[NC][4];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        raw[c].get(v[c]);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[c][j] = named ? mul2(v[c][j], both(p.scale)) : both(0.f);
    }
    if constexpr (VEC) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (col0 + c * TPR * kChunk < p.d) store8<T>(out + col0 + c * TPR * kChunk, v[c]);
    } else {
        store_shifted<T, TPR, NC>(out, col0, p.d, shift, v, slots[threadIdx.x / TPR], lane, group_mask<TPR>());
    }
}

// ---- gradient: sort -----------------------------------------------------------------------------------
// A sorted entry is token << 32 | position.  Scratch area of one call: the sorted entries, one bit per vocabulary row
// that some token names, and the partial sums of runs that cross tiles.
constexpr uint32_t kSortPerBlock = 4096, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortBlocks = 16;
constexpr uint32_t kSortMax = kSortBlocks * kSortPerBlock;   // tokens of a node sorted by one cluster of blocks
constexpr uint32_t kDirectTokens = 512;   // up to here no sort: see lookup_grad_direct_kernel

struct GradLayout {
    int64_t entry_off, bit_off, part_off, total;
    uint32_t words;         // words of the bit map per node
    uint32_t tile, tiles;   // sorted entries per tile, tiles per node
    int32_t dpad;
};

GradLayout grad_layout(int64_t nodes, int64_t rows, int64_t d, int64_t vocab)
{
    auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    GradLayout L = {};
    L.dpad = (int32_t)((d + 7) / 8 * 8);
    L.words = (uint32_t)((vocab + 31) / 32);
    if (rows <= kDirectTokens) return L;
    if (rows > (int64_t)kSortMax) rows = kSortMax;
    // entries per tile: 32 leave fewer partial sums, 16 or 8 spread few tokens over the SMs (512 threads each)
    L.tile = 32;
    while (L.tile > 8 && (rows + L.tile - 1) / L.tile * nodes * (L.dpad / 8) < 148 * 512) L.tile /= 2;
    L.tiles = (uint32_t)((rows + L.tile - 1) / L.tile);
    L.entry_off = 0;
    L.bit_off = L.entry_off + up(nodes * rows * 8);
    L.part_off = L.bit_off + up(nodes * (int64_t)L.words * 4);
    L.total = L.part_off + up(L.tiles > 1 ? nodes * (int64_t)L.tiles * 2 * L.dpad * 4 : 0);
    return L;
}

struct SortParams {
    const void* tokens;
    uint64_t* entries;
    uint32_t* bits;
    int64_t node_tokens;   // tokens of one node in `tokens` (this call may sort a part of them)
    uint32_t first, count; // the part: tokens first .. first + count - 1 of every node
    uint32_t vocab, words;
    uint32_t per_block;    // entries a block holds
    int passes, digit_bits;
    bool tokens64;
    bool map_on_chip;      // the bit map fits the blocks' shared memory
};

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of this block's shared-memory word in block `rank` of the cluster, and stores to it.
__device__ __forceinline__ uint32_t cluster_address(const void* p, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ uint32_t cluster_load(uint32_t address)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(address) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_store(uint32_t address, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(address), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_store(uint32_t address, uint64_t v)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(address), "l"(v) : "memory");
}

// Shared memory of the sort, in 32-bit words before the entries.
constexpr uint32_t kSortWords = kSortWarps * 256 + kSortBlocks * 256 + 4 * 256 + 3 * 256 + 32;

// Stable radix sort of one node's entries, least significant digit first, by a cluster of blocks that hold them in
// shared memory: entry e lives in block e / per_block.  A pass ranks every entry among the equal digits before it (lanes
// by ballots, warps by a scan of their counts), brings the block's entries into the order of their digits, and sends the
// runs of one digit to their places in the cluster's blocks (the counts of the other blocks come from a table that every
// block sends to all); the last pass writes them to memory.  A token outside the vocabulary sorts behind all others, as
// the key `vocab`.  65536 tokens of 50021 words 19 us, 4096 of 32000 10 us: barriers and shared-memory latency of two
// passes, 3200 cycles of ranking in each.  On the way the blocks mark the vocabulary rows that are named, each in a map of its own, and join the
// maps (where that does not fit, from 0.9 million rows on at 4096 entries per block, 1.3 million at 700: atomics on the map in memory, which cost 6 us for 65536 tokens).
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const SortParams p)
{
    extern __shared__ __align__(16) uint32_t smem[];
    uint32_t rank, blocks;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
    const uint32_t node = blockIdx.y;
    uint32_t* hist = smem;                            // kSortWarps x 256: equal digits in the block before the warp's
    uint32_t* totals = hist + kSortWarps * 256;       // kSortBlocks x 256: every block's digit counts
    uint32_t* quarter = totals + kSortBlocks * 256;   // 4 x 256: counts of eight warps each
    uint32_t* local = quarter + 4 * 256;              // 256: first place of a digit in the block's order
    uint32_t* global = local + 256;                   // 256: the same in the node's order, for this block's entries
    uint32_t* scan = global + 256;                    // 2 x 8, padded
    uint64_t* buffer[2] = {reinterpret_cast<uint64_t*>(smem + kSortWords), reinterpret_cast<uint64_t*>(smem + kSortWords) + p.per_block};
    uint32_t* map = smem + kSortWords + 4 * p.per_block;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t e0 = rank * p.per_block;
    const uint32_t mine = e0 >= p.count ? 0 : min(p.per_block, p.count - e0);
    const uint32_t digits = 1u << p.digit_bits;
    constexpr int kMost = kSortPerBlock / kSortThreads;   // entries of a thread
    // a warp's stretch of the block's entries
    const uint32_t stretch = ((mine + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;

    uint64_t entry[kMost];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const uint32_t off = i * 32 + lane, e = warp * stretch + off;
        if (off < stretch && e < mine) {
            const int64_t token = token_at(p.tokens, p.tokens64, (int64_t)node * p.node_tokens + p.first + e0 + e);
            const uint32_t key = token >= 0 && token < (int64_t)p.vocab ? (uint32_t)token : p.vocab;
            entry[i] = (uint64_t)key << 32 | (p.first + e0 + e);
        }
    }
    uint32_t* bits = p.bits + (int64_t)node * p.words;
    if (p.map_on_chip) {
        for (uint32_t w = tid; w < p.words; w += kSortThreads) map[w] = 0;
        __syncthreads();
    } else {
        for (uint32_t w = rank * kSortThreads + tid; w < p.words; w += blocks * kSortThreads) bits[w] = 0;
        cluster_barrier();
    }
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const uint32_t off = i * 32 + lane, e = warp * stretch + off, key = (uint32_t)(entry[i] >> 32), bit = 1u << (key & 31);
        if (off < stretch && e < mine && key < p.vocab) {
            // the test spares the frequent words' many atomics
            if (p.map_on_chip) {
                if (!(*(volatile uint32_t*)&map[key >> 5] & bit)) atomicOr(&map[key >> 5], bit);
            } else if (!(__ldcg(bits + (key >> 5)) & bit)) {
                atomicOr(bits + (key >> 5), bit);
            }
        }
    }
    cluster_barrier();   // the maps are complete, and every block of the cluster runs before any of them is written to
    if (p.map_on_chip) {
        const uint32_t slice = (p.words + blocks - 1) / blocks, end = min((rank + 1) * slice, p.words);
        for (uint32_t w = rank * slice + tid; w < end; w += kSortThreads) {
            uint32_t all = 0;
            for (uint32_t b = 0; b < blocks; ++b) all |= cluster_load(cluster_address(map + w, b));
            bits[w] = all;
        }
    }
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = 32 + pass * p.digit_bits;
        if (pass)
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const uint32_t off = i * 32 + lane, e = warp * stretch + off;
                if (off < stretch && e < mine) entry[i] = buffer[pass & 1][e];
            }
        for (uint32_t h = tid; h < kSortWarps * 256; h += kSortThreads) hist[h] = 0;
        __syncthreads();
        uint32_t before[kMost];   // equal digits before the entry in the warp's stretch
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const uint32_t off = i * 32 + lane, e = warp * stretch + off;
            const bool live = off < stretch && e < mine;
            unsigned same = __ballot_sync(0xFFFFFFFFu, live);
            if (!same) break;
            const uint32_t digit = (uint32_t)(entry[i] >> shift) & (digits - 1);
#pragma unroll
            for (int b = 0; b < 8; ++b) {   // lanes that agree in every bit
                const unsigned mine_b = (unsigned)((int)(digit << (31 - b)) >> 31);
                same &= ~(__ballot_sync(0xFFFFFFFFu, mine_b) ^ mine_b);
            }
            uint32_t had = 0;
            if (live) had = hist[warp * 256 + digit];
            __syncwarp();
            before[i] = had + __popc(same & ((1u << lane) - 1u));
            if (live && (int)lane == __ffs(same) - 1) hist[warp * 256 + digit] = had + __popc(same);
            __syncwarp();
        }
        __syncthreads();
        // counts of a digit over the warps, eight warps per quarter of the threads
        const uint32_t digit_t = tid & 255, q = tid >> 8;
        uint32_t sum = 0, count[8];
#pragma unroll
        for (int w = 0; w < 8; ++w) count[w] = hist[(q * 8 + w) * 256 + digit_t];
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const uint32_t n = count[w];
            count[w] = sum;
            sum += n;
        }
        quarter[q * 256 + digit_t] = sum;
        __syncthreads();
        uint32_t total = 0, ahead_q = 0;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            const uint32_t n = quarter[k * 256 + digit_t];
            if (k < q) ahead_q += n;
            total += n;
        }
#pragma unroll
        for (int w = 0; w < 8; ++w) hist[(q * 8 + w) * 256 + digit_t] = count[w] + ahead_q;
        if (q == 0)
            for (uint32_t b = 0; b < blocks; ++b) cluster_store(cluster_address(totals + rank * 256 + digit_t, b), total);
        cluster_barrier();
        uint32_t all = 0, ahead = 0;   // of this digit: in all blocks, in the blocks before this one
        if (q == 0)
            for (uint32_t b = 0; b < blocks; ++b) {
                const uint32_t n = totals[b * 256 + digit_t];
                if (b < rank) ahead += n;
                all += n;
            }
        if (q == 0) {   // inclusive scans over the digits, of the block's counts and of all blocks'
            uint32_t in_block = total, in_all = all;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t n = __shfl_up_sync(0xFFFFFFFFu, in_block, o), m = __shfl_up_sync(0xFFFFFFFFu, in_all, o);
                if (lane >= (uint32_t)o) in_block += n, in_all += m;
            }
            if (lane == 31) scan[warp] = in_block, scan[8 + warp] = in_all;
            local[digit_t] = in_block - total;
            global[digit_t] = in_all - all + ahead;
        }
        __syncthreads();
        if (q == 0) {
            uint32_t n = 0, m = 0;
            for (uint32_t w = 0; w < warp; ++w) n += scan[w], m += scan[8 + w];
            local[digit_t] += n;
            global[digit_t] += m;
        }
        __syncthreads();
        uint64_t* order = buffer[pass & 1];   // its entries are in registers
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const uint32_t off = i * 32 + lane, e = warp * stretch + off;
            if (off < stretch && e < mine) {
                const uint32_t digit = (uint32_t)(entry[i] >> shift) & (digits - 1);
                order[local[digit] + hist[warp * 256 + digit] + before[i]] = entry[i];
            }
        }
        __syncthreads();
        const bool last = pass + 1 == p.passes;
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const uint32_t e = i * kSortThreads + tid;
            if (e < mine) {
                const uint64_t v = order[e];
                const uint32_t digit = (uint32_t)(v >> shift) & (digits - 1);
                const uint32_t to = global[digit] + (e - local[digit]);
                if (last) p.entries[(int64_t)node * p.count + to] = v;
                else {
                    const uint32_t block = to / p.per_block;
                    cluster_store(cluster_address(buffer[pass & 1 ^ 1] + (to - block * p.per_block), block), v);
                }
            }
        }
        if (!last) cluster_barrier();
    }
}

// ---- gradient: sums -----------------------------------------------------------------------------------
struct SumParams {
    const void* dout;
    const void* tokens;      // direct kernel only
    float* grad;
    const uint64_t* entries;
    const uint32_t* bits;
    float* part;
    int64_t ldo, ldg, node_ldg;
    int64_t node_rows;       // rows of dout per node
    uint32_t count, vocab, words, tile, tiles;
    int32_t d, dpad;
    uint32_t sum_blocks;     // blocks 0 .. sum_blocks - 1 (x) sum, the others clear rows
    uint32_t clear_blocks;
    float scale;
    bool tokens64, accumulate, gvec;   // gvec: 128-bit accesses to grad
};

// Writes (or adds) a token's sum to its row of grad; the lanes of `group` that share it make the call together.  GVEC:
// every row of grad is aligned and d is a multiple of four.
template <bool GVEC, int LANES>
__device__ __forceinline__ void write_sum(const SumParams& p, uint32_t node, uint32_t token, int c, int lane, unsigned group, f32x2_t* acc)
{
    float* to = p.grad + node * p.node_ldg + (int64_t)token * p.ldg;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = mul2(acc[j], both(p.scale));
    if constexpr (GVEC) {
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
        store.store(to, c, p.d, acc, lane, group, true);
    }
}

// How a tile [begin, end) of the sorted entries (at most 32) meets the runs (of one token) that cross its ends.  A run
// that holds a whole tile is split: every tile it touches leaves a partial sum.  Any other run belongs to the tile it
// starts in, which follows it into the next tile; that tile skips it.
struct TileEnds {
    uint32_t first, last;   // tokens of the first and the last entry
    bool in, split_in;      // the first run comes from the tile before; it is split
    bool out, split_out;    // the last run goes on into the next tile; it is split
};
// Four lanes read the entries before and behind the tile and one tile further on; L lanes share the call.
template <int L>
__device__ __forceinline__ TileEnds tile_ends(const SumParams& p, const uint64_t* entries, uint32_t tile, uint32_t first, uint32_t last,
                                              uint32_t lane, unsigned mask)
{
    const uint32_t begin = tile * p.tile, end = min(begin + p.tile, p.count), none = 0xFFFFFFFFu;
    uint32_t key = none;
    const uint32_t at = lane == 0 ? begin - 1 : lane == 1 ? begin - p.tile : lane == 2 ? end : end + p.tile - 1;
    if (lane < 2 ? begin > 0 : lane < 4 && at < p.count) key = (uint32_t)(entries[at] >> 32);
    const uint32_t before = __shfl_sync(mask, key, 0, L), tile_before = __shfl_sync(mask, key, 1, L);
    const uint32_t after = __shfl_sync(mask, key, 2, L), tile_after = __shfl_sync(mask, key, 3, L);
    const bool whole = first == last && end - begin == p.tile;
    TileEnds t;
    t.first = first;
    t.last = last;
    t.in = first == before;
    t.split_in = t.in && (tile_before == first || whole);
    t.out = last == after;
    t.split_out = t.out && (whole || tile_after == last);
    return t;
}

// TX threads walk a tile's entries over 8 TX columns and keep the running sum of one token.  A token's sum is written to
// its row of grad, a split run's part to the tile's partial sums (slot 0: came from before, slot 1: starts here and goes
// on).
template <class T, bool VEC, bool GVEC, int TX>
__device__ __forceinline__ void sum_tile(const SumParams& p, uint32_t node, uint32_t tile, int c0, int tx)
{
    constexpr int U = VEC && sizeof(T) == 2 ? 8 : 4;   // entries whose loads are in flight together
    constexpr int L = TX < 32 ? TX : 32, H = 32 / L;   // a lane holds H entries of a tile
    const uint64_t* entries = p.entries + (int64_t)node * p.count;
    const T* dout = static_cast<const T*>(p.dout) + (int64_t)node * p.node_rows * p.ldo;
    const Span span = span_of<T>(dout, p.ldo, p.node_rows, p.d);
    const uint32_t begin = tile * p.tile, end = min(begin + p.tile, p.count), none = 0xFFFFFFFFu, lane = tx % L;
    const unsigned group = group_mask<TX>();
    uint64_t own[H];
    auto read = [&](uint32_t from, uint32_t to) {
#pragma unroll
        for (int h = 0; h < H; ++h) own[h] = from + h * L + lane < to ? entries[from + h * L + lane] : ~0ull;
    };
    auto entry = [&](int i) { return __shfl_sync(group, own[i / L], i % L, L); };   // i: the same in all lanes
    read(begin, end);
    uint32_t last = 0;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const uint32_t k = (uint32_t)(__shfl_sync(group, own[h], (end - 1 - begin) % L, L) >> 32);
        if ((end - 1 - begin) / L == h) last = k;
    }
    const TileEnds ends = tile_ends<L>(p, entries, tile, (uint32_t)(entry(0) >> 32), last, lane, group);
    const uint32_t skip = ends.in && !ends.split_in ? ends.first : none;
    const uint32_t follow = ends.out && !ends.split_out ? ends.last : none;
    float* part = p.part + ((int64_t)node * p.tiles + tile) * 2 * p.dpad;
    const int c = c0 + tx * 8;
    f32x2_t acc[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};
    uint32_t cur = skip == none ? ends.first : none;
    bool from_before = ends.split_in;
    auto flush = [&](bool goes_on) {
        if (cur >= p.vocab) return;
        if (from_before || goes_on) {
            float* to = part + (from_before ? 0 : p.dpad);
            if (c < p.dpad) {
                *reinterpret_cast<float4*>(to + c) = join4(acc[0], acc[1]);
                *reinterpret_cast<float4*>(to + c + 4) = join4(acc[2], acc[3]);
            }
        } else {
            write_sum<GVEC, L>(p, node, cur, c, (int)lane, group, acc);
        }
    };
    for (int half = 0; half < 2; ++half) {
        if (half) {
            if (follow == none) break;
            read(end, min(end + p.tile, p.count));
        }
#pragma unroll
        for (int h = 0; h < H; ++h) {   // entries that are not this tile's: the key `none`
            const uint32_t k = (uint32_t)(own[h] >> 32);
            if (half ? k != follow : k == skip) own[h] = ~0ull;
        }
#pragma unroll 1
        for (int i0 = 0; i0 < (int)p.tile; i0 += U) {
            uint32_t k[U];
            Raw8<T, VEC> raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint64_t e = own[0];
#pragma unroll
                for (int h = 1; h < H; ++h)
                    if ((i0 + u) / L == h) e = own[h];
                e = __shfl_sync(group, e, (i0 + u) % L, L);
                k[u] = (uint32_t)(e >> 32);
                if (k[u] < p.vocab && (!VEC || c < p.d)) raw[u].load(dout + (int64_t)(uint32_t)e * p.ldo, c, p.d, span);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k[u] == none) continue;
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
            if (half && k[U - 1] == none) break;   // the followed run has ended
        }
    }
    flush(ends.split_out);
}

// Zeroes `count` floats from `to` on, by THREADS threads: single ones up to the first 16 bytes and behind the last.
template <int THREADS>
__device__ __forceinline__ void clear_range(float* to, int64_t count, uint32_t thread)
{
    const int64_t head = min(count, (int64_t)(-((uint32_t)(uintptr_t)to >> 2) & 3u)), body = (count - head) / 4;
    float4* at = reinterpret_cast<float4*>(to + head);
    if (thread < head) to[thread] = 0.f;
#pragma unroll 4
    for (int64_t i = thread; i < body; i += THREADS) __stcs(at + i, make_float4(0.f, 0.f, 0.f, 0.f));
    const int64_t tail = head + body * 4 + thread;
    if (tail < count) to[tail] = 0.f;
}

// Clears the rows first .. first + n - 1 (n <= 32) of a node's grad whose bit in `named` is not set.  Neighbouring rows are
// one range where nothing lies between them: rows of an odd width would otherwise leave partial sectors at their ends.
template <int THREADS>
__device__ __forceinline__ void clear_rows(const SumParams& p, uint32_t node, uint32_t first, uint32_t n, uint32_t named, uint32_t thread)
{
    uint32_t open = ~named & (n == 32 ? ~0u : (1u << n) - 1u);
    while (open) {
        const uint32_t a = __ffs(open) - 1, run = p.ldg == p.d ? __ffs(~(open >> a)) : 0;   // run: rows plus one; 0: all 32
        const uint32_t rows = p.ldg == p.d ? (run ? run - 1 : 32 - a) : 1;
        clear_range<THREADS>(p.grad + node * p.node_ldg + (int64_t)(first + a) * p.ldg, (int64_t)rows * p.d, thread);
        open &= rows + a >= 32 ? 0u : ~0u << (a + rows);
    }
}

// Blocks 0 .. sum_blocks - 1 (x) sum tiles; the others clear the rows of grad that no token names, four rows to a warp at a time.
// Both in one launch: reads of dout and writes of grad then share the memory's time (65536 tokens of 1024 bf16, 50021 rows:
// 57 us = 6.0 TB/s with the partial sums; the sums alone take 44 us, the writes 25 us).  (The clearing blocks first, at
// eight per SM beside the sums: 64 us instead of 58 for 65536 tokens, 1024 columns, 50021 rows.)
template <class T, bool VEC, bool GVEC, int TX>
__global__ void __launch_bounds__(128) lookup_grad_kernel(const SumParams p)
{
    const uint32_t node = blockIdx.z;
    grid_dependency_wait();
    if (blockIdx.x >= p.sum_blocks) {
        if (blockIdx.y) return;
        const uint32_t* bits = p.bits + (int64_t)node * p.words;
        const uint32_t warp = (blockIdx.x - p.sum_blocks) * 4 + threadIdx.x / 32;
        if (GVEC) {
            for (uint32_t v = warp; v < p.vocab; v += p.clear_blocks * 4)
                clear_rows<32>(p, node, v, 1, bits[v >> 5] >> (v & 31) & 1u, threadIdx.x & 31);
        } else {
            for (uint32_t q = warp; q * 4 < p.vocab; q += p.clear_blocks * 4)   // four rows
                clear_rows<32>(p, node, q * 4, min(4u, p.vocab - q * 4), bits[q >> 3] >> (q & 7) * 4 & 15u, threadIdx.x & 31);
        }
        return;
    }
    const uint32_t tile = blockIdx.x * (128 / TX) + threadIdx.x / TX;
    if (tile < p.tiles) sum_tile<T, VEC, GVEC, TX>(p, node, tile, blockIdx.y * TX * 8, threadIdx.x % TX);
}

// Adds a float4 of a split run's sum to, or stores it in, the token's row of grad.
__device__ __forceinline__ void write_joined(const SumParams& p, uint32_t node, uint32_t token, int c, float4 sum)
{
    float* to = p.grad + node * p.node_ldg + (int64_t)token * p.ldg + c;
    sum = scale4(sum, p.scale);
    if (p.gvec) {
        if (p.accumulate) sum = add4(*reinterpret_cast<const float4*>(to), sum);
        __stcs(reinterpret_cast<float4*>(to), sum);
    } else {
        const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < p.d) to[j] = (p.accumulate ? to[j] : 0.f) + v[j];
    }
}

// 9 us for 65536 tokens (their most frequent word in 184 tiles): a chain of six dependent reads and the launch.
// Split runs: the sum of the tiles' partial sums, in their order.  Lanes look at 32 boundaries between tiles at a time.
// The first blocks: a warp looks at one of eight tiles, and the block takes the runs that start there and span at most
// kShortRun more tiles, a thread four columns of 1024.  The others: a longer run, taken by the first tile inside it whose
// number is a multiple of kShortRun; sixteen groups of lanes add every sixteenth partial sum of 64 columns, then the
// groups' sums in their order.
constexpr uint32_t kShortRun = 16, kLongGroups = 16, kLongColumns = 64;
__global__ void __launch_bounds__(256) lookup_grad_join_kernel(const SumParams p)
{
    __shared__ float4 sums[kLongGroups][kLongColumns / 4];
    __shared__ uint32_t run_token[8], run_more[8];
    grid_dependency_wait();
    const uint32_t node = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t* entries = p.entries + (int64_t)node * p.count;
    auto key = [&](uint32_t e) { return (uint32_t)(entries[e] >> 32); };
    // Tiles that the run of `tile` reaches after it: the boundaries inside a run are neighbours, so 32 evenly spaced ones
    // at a time narrow its end down.
    auto tiles_behind = [&](uint32_t tile, uint32_t token) {
        uint32_t more = 0, stride = 1;
        for (;;) {   // the next 32, then 32 times as far apart as long as all are inside
            const uint32_t b = tile + more + (lane + 1) * stride;
            const unsigned out = ~__ballot_sync(0xFFFFFFFFu, b < p.tiles && key(b * p.tile) == token);
            more += (out ? __ffs(out) - 1 : 32) * stride;
            if (!out) {
                stride *= 32;
                continue;
            }
            if (stride == 1) return more;
            stride /= 32;
        }
    };
    const int64_t step = 2 * (int64_t)p.dpad;
    const uint32_t slabs = (uint32_t)(p.d + 1023) / 1024, long_slabs = (uint32_t)(p.d + kLongColumns - 1) / kLongColumns;
    const uint32_t short_blocks = (p.tiles + 7) / 8 * slabs;
    if (blockIdx.x < short_blocks) {
        const uint32_t first = blockIdx.x / slabs * 8, tile = first + warp;
        uint32_t token = p.vocab, more = 0;
        if (tile < p.tiles) {
            const uint32_t begin = tile * p.tile, end = min(begin + p.tile, p.count);
            const TileEnds ends = tile_ends<32>(p, entries, tile, key(begin), key(end - 1), lane, 0xFFFFFFFFu);
            // starts here (the tile is not the inside of a run that came in) and is split
            if (ends.split_out && !(ends.in && ends.first == ends.last)) {
                token = ends.last;
                if (token < p.vocab) more = tiles_behind(tile, token);
            }
        }
        if (lane == 0) {
            run_token[warp] = token;
            run_more[warp] = more;
        }
        __syncthreads();
        for (uint32_t w = 0; w < 8; ++w) {
            token = run_token[w], more = run_more[w];
            if (token >= p.vocab || more > kShortRun) continue;
            const float* part = p.part + ((int64_t)node * p.tiles + first + w) * step;
            const int c = (int)(blockIdx.x % slabs * 1024 + threadIdx.x * 4);
            if (c < p.d) {
                float4 sum = *reinterpret_cast<const float4*>(part + p.dpad + c);
#pragma unroll 8
                for (uint32_t m = 1; m <= more; ++m) sum = add4(sum, *reinterpret_cast<const float4*>(part + m * step + c));
                write_joined(p, node, token, c, sum);
            }
        }
        return;
    }
    // the run that comes into this tile, and the tile where it starts
    const uint32_t item = blockIdx.x - short_blocks;
    uint32_t tile = (item / long_slabs + 1) * kShortRun;
    const uint32_t group = threadIdx.x / (kLongColumns / 4), member = threadIdx.x % (kLongColumns / 4);
    const int c = (int)(item % long_slabs * kLongColumns + member * 4);
    const uint32_t token = key(tile * p.tile);
    if (token >= p.vocab) return;
    const unsigned in = __ballot_sync(0xFFFFFFFFu, lane < tile && key((tile - min(lane, tile - 1)) * p.tile - 1) == token);
    const uint32_t back = ~in ? __ffs(~in) - 1 : 32;   // boundaries inside the run from this one back
    if (back == 0 || back > kShortRun) return;   // none, or an earlier multiple of kShortRun is inside it too
    tile -= back;
    const uint32_t more = tiles_behind(tile, token);
    if (more <= kShortRun) return;
    const float* part = p.part + ((int64_t)node * p.tiles + tile) * step;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < p.d) {
        if (group == 0) sum = *reinterpret_cast<const float4*>(part + p.dpad + c);
#pragma unroll 8
        for (uint32_t m = 1 + group; m <= more; m += kLongGroups) sum = add4(sum, *reinterpret_cast<const float4*>(part + m * step + c));
    }
    sums[group][member] = sum;
    __syncthreads();
    if (group || c >= p.d) return;
#pragma unroll
    for (uint32_t g = 1; g < kLongGroups; ++g) sum = add4(sum, sums[g][member]);
    write_joined(p, node, token, c, sum);
}

// Few tokens (at most kDirectTokens per node): one launch, no sort, no scratch: 37 tokens of 257 columns 3.8 us, by the sort
// 17 us; 8 nodes x 512 tokens of 1024, 32000 rows 176 us either way, nearly all of it clearing at 6.0 TB/s.  Blocks 0 .. count - 1 (x): the block
// of a token's first place adds the rows of all its places, in their order, over 1024 columns.  The other blocks clear
// the rows of their share of the vocabulary that no token names.
template <class T, bool VEC, bool GVEC>
__global__ void __launch_bounds__(128) lookup_grad_direct_kernel(const SumParams p)
{
    __shared__ uint32_t keys[kDirectTokens], list[kDirectTokens], found[kDirectTokens / 32];
    constexpr uint32_t kSpan = 1024;   // vocabulary rows of a clearing step
    __shared__ uint32_t named[kSpan / 32];
    const uint32_t node = blockIdx.z, tid = threadIdx.x, lane = tid & 31;
    for (uint32_t i = tid; i < p.count; i += 128) {
        const int64_t token = token_at(p.tokens, p.tokens64, (int64_t)node * p.count + i);
        keys[i] = token >= 0 && token < (int64_t)p.vocab ? (uint32_t)token : p.vocab;
    }
    __syncthreads();
    if (blockIdx.x >= p.sum_blocks) {
        if (blockIdx.y) return;
        // every clear_blocks-th group of eight rows, so that the blocks that run together write one stretch of memory; a row
        // to a warp where rows are aligned (8 tables of 32000 x 1024: 176 us, as ranges by the block 182), neighbouring rows as
        // one range by the block where not (4 tables of 28353 x 1663: 117 us, a row to a warp 125)
        const uint32_t block = blockIdx.x - p.sum_blocks, groups = (p.vocab + 7) / 8;
        for (uint32_t s0 = 0; block + s0 * p.clear_blocks < groups; s0 += kSpan / 8) {
            if (s0) __syncthreads();
            if (tid < kSpan / 32) named[tid] = 0;
            __syncthreads();
            for (uint32_t i = tid; i < p.count; i += 128) {
                const uint32_t group = keys[i] / 8, slot = group / p.clear_blocks;
                if (keys[i] < p.vocab && group - slot * p.clear_blocks == block && slot >= s0 && slot - s0 < kSpan / 8)
                    atomicOr(&named[(slot - s0) >> 2], 1u << (((slot - s0) & 3) * 8 + (keys[i] & 7)));
            }
            __syncthreads();
            for (uint32_t slot = s0; slot < s0 + kSpan / 8; ++slot) {
                const uint32_t first = (block + slot * p.clear_blocks) * 8, of_slot = named[(slot - s0) >> 2] >> ((slot - s0) & 3) * 8 & 0xFFu;
                if (first >= p.vocab) break;
                if (!GVEC) clear_rows<128>(p, node, first, min(8u, p.vocab - first), of_slot, tid);
                else
                    for (uint32_t r = tid / 32; r < min(8u, p.vocab - first); r += 4) clear_rows<32>(p, node, first + r, 1, of_slot >> r & 1u, lane);
            }
        }
        return;
    }
    const uint32_t at = blockIdx.x, token = keys[at];
    if (token >= p.vocab) return;
    bool earlier = false;
    for (uint32_t i = tid; i < kDirectTokens; i += 128) {
        const bool hit = i < p.count && keys[i] == token;
        earlier |= hit && i < at;
        const unsigned hits = __ballot_sync(0xFFFFFFFFu, hit);
        if (lane == 0) found[i >> 5] = hits;
    }
    if (__syncthreads_or(earlier)) return;
    uint32_t places = 0;
#pragma unroll
    for (uint32_t w = 0; w < kDirectTokens / 32; ++w) {
        if (tid >> 5 == (w & 3) && found[w] >> lane & 1) list[places + __popc(found[w] & ((1u << lane) - 1u))] = w * 32 + lane;
        places += __popc(found[w]);
    }
    __syncthreads();
    constexpr int U = VEC && sizeof(T) == 2 ? 8 : 4;
    const T* dout = static_cast<const T*>(p.dout) + (int64_t)node * p.node_rows * p.ldo;
    const Span span = span_of<T>(dout, p.ldo, p.node_rows, p.d);
    const int c = (int)(blockIdx.y * 128 + tid) * 8;
    f32x2_t acc[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};
    for (uint32_t e0 = 0; e0 < places; e0 += U) {
        Raw8<T, VEC> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (e0 + u < places && c < p.d) raw[u].load(dout + (int64_t)list[e0 + u] * p.ldo, c, p.d, span);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (e0 + u < places && c < p.d) {
                f32x2_t v[4];
                raw[u].get(v);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = add2(acc[j], v[j]);
            }
    }
    write_sum<GVEC, 32>(p, node, token, c, lane, 0xFFFFFFFFu, acc);
}

// Blocks that clear rows, per node: four rows at least to a block; at most sixteen such blocks per SM.
uint32_t clear_blocks_for(const SumParams& p, uint32_t nodes)
{
    const uint32_t units = (p.vocab + 3) / 4, most = (148 * 16 + nodes - 1) / nodes;
    return p.accumulate ? 0 : units < most ? units : most;
}

template <class T, bool VEC, bool GVEC, int TX>
cudaError_t sums_as(SumParams p, uint32_t nodes, cudaStream_t s)
{
    const uint32_t per = 128 / TX;
    p.sum_blocks = (p.tiles + per - 1) / per;
    p.clear_blocks = clear_blocks_for(p, nodes);
    const uint32_t slabs = (uint32_t)(p.d + 8 * TX - 1) / (8 * TX);
    return launch_after_trigger(lookup_grad_kernel<T, VEC, GVEC, TX>, dim3(p.sum_blocks + p.clear_blocks, slabs, nodes), dim3(128), 0, s,
                                true, p);
}

template <class T, bool VEC, bool GVEC>
cudaError_t sums_of(SumParams p, bool direct, uint32_t nodes, cudaStream_t s)
{
    if (direct) {
        p.sum_blocks = p.count;
        p.clear_blocks = clear_blocks_for(p, nodes);
        if (!(p.sum_blocks + p.clear_blocks)) return cudaSuccess;
        lookup_grad_direct_kernel<T, VEC, GVEC><<<dim3(p.sum_blocks + p.clear_blocks, (unsigned)(p.d + 1023) / 1024, nodes), 128, 0, s>>>(p);
        return cudaGetLastError();
    }
    if (p.d <= 64) return sums_as<T, VEC, GVEC, 8>(p, nodes, s);
    if (p.d <= 256) return sums_as<T, VEC, GVEC, 32>(p, nodes, s);
    return sums_as<T, VEC, GVEC, 128>(p, nodes, s);
}

template <class T>
cudaError_t sums_by_alignment(const SumParams& p, bool direct, uint32_t nodes, bool vec, cudaStream_t s)
{
    if (!vec) return sums_of<T, false, false>(p, direct, nodes, s);
    return p.gvec ? sums_of<T, true, true>(p, direct, nodes, s) : sums_of<T, true, false>(p, direct, nodes, s);
}

// Clusters of sixteen blocks have to be asked for, once per device.
cudaError_t allow_wide_clusters(std::atomic<unsigned long long>& done_mask)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || done_mask >> (dev & 63) & 1) return e;
    e = cudaFuncSetAttribute(sort_tokens_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) done_mask |= 1ull << (dev & 63);
    return e;
}

bool aligned(const void* p, int64_t ld, int size) { return (((uintptr_t)p) & 15u) == 0 && (ld * size) % 16 == 0; }

template <class T, bool VEC, int TPR, int NC>
cudaError_t lookup_as(LookupParams& p, cudaStream_t s)
{
    p.stretches = make_divisor((uint32_t)(p.d + (VEC ? 0 : (int)kShiftRows<T> - 1) + NC * TPR * kChunk - 1) / (NC * TPR * kChunk));
    const uint64_t groups = (uint64_t)p.rows * p.stretches.d;
    lookup_kernel<T, VEC, TPR, NC><<<dim3((unsigned)((groups + 256 / TPR - 1) / (256 / TPR)), p.nodes), 256, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool VEC>
cudaError_t lookup_by_width(LookupParams& p, cudaStream_t s)
{
    const int d = p.d + (VEC ? 0 : (int)kShiftRows<T> - 1);
    return d <= 64    ? lookup_as<T, VEC, 8, 1>(p, s)
           : d <= 256 ? lookup_as<T, VEC, 32, 1>(p, s)
           : d <= 512 ? lookup_as<T, VEC, 32, 2>(p, s)
                      : lookup_as<T, VEC, 32, 4>(p, s);
}

template <class T>
cudaError_t lookup_of(LookupParams p, cudaStream_t s)
{
    if (!p.rows) return cudaSuccess;
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
    const bool direct = g.rows <= kDirectTokens;
    SumParams p = {};
    p.dout = g.dout;
    p.tokens = g.tokens;
    p.tokens64 = g.tokens64;
    p.grad = g.grad;
    p.ldo = g.ldo;
    p.ldg = g.ldg;
    p.node_ldg = g.node_ldg;
    p.node_rows = g.rows;
    p.count = g.rows;
    p.vocab = g.vocab;
    p.tile = L.tile;
    p.d = g.d;
    p.dpad = L.dpad;
    p.scale = g.scale;
    p.accumulate = g.accumulate;
    p.gvec = g.d % 4 == 0 && aligned(g.grad, g.ldg, 4) && g.node_ldg % 4 == 0;
    const bool vec = g.d % 8 == 0 && aligned(g.dout, g.ldo, dtype == GPGA_DTYPE_F32 ? 4 : 2);
    auto sums = [&]() {
        return dtype == GPGA_DTYPE_F32    ? sums_by_alignment<float>(p, direct, g.nodes, vec, s)
               : dtype == GPGA_DTYPE_BF16 ? sums_by_alignment<__nv_bfloat16>(p, direct, g.nodes, vec, s)
                                          : sums_by_alignment<__half>(p, direct, g.nodes, vec, s);
    };
    if (direct) return sums();

    SortParams q = {};
    q.tokens = g.tokens;
    q.entries = reinterpret_cast<uint64_t*>(g.scratch + L.entry_off);
    q.node_tokens = g.rows;
    q.bits = reinterpret_cast<uint32_t*>(g.scratch + L.bit_off);
    q.vocab = g.vocab;
    q.words = p.words = L.words;
    q.tokens64 = g.tokens64;
    p.bits = q.bits;
    int key_bits = 1;
    while (g.vocab >> key_bits) ++key_bits;   // keys are 0 .. vocab
    q.passes = (key_bits + 7) / 8;
    q.digit_bits = (key_bits + q.passes - 1) / q.passes;
    p.entries = q.entries;
    p.part = reinterpret_cast<float*>(g.scratch + L.part_off);

    // one cluster sorts up to kSortMax tokens of a node; the parts of a longer row list are added up one after
    // the other
    for (uint32_t first = 0; first < g.rows;) {
        const uint32_t count = g.rows - first < kSortMax ? g.rows - first : kSortMax;
        q.first = first;
        q.count = count;
        uint32_t blocks = 1;
        while (blocks < kSortBlocks && blocks * 1024 < count) blocks *= 2;
        q.per_block = (count + blocks - 1) / blocks;
        constexpr size_t kMost = 227 * 1024;
        size_t smem = (kSortWords + 4 * (size_t)q.per_block) * 4;
        q.map_on_chip = smem + 4 * (size_t)L.words <= kMost;
        if (q.map_on_chip) smem += 4 * (size_t)L.words;
        static std::atomic<unsigned long long> limit_set{0}, wide_set{0};
        cudaError_t e = ensure_smem_limit(sort_tokens_kernel, kMost, limit_set);
        if (e == cudaSuccess && blocks > 8) e = allow_wide_clusters(wide_set);
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
        e = sums();
        if (e != cudaSuccess) return e;
        if (p.tiles > 1) {
            const uint32_t blocks_x = (p.tiles + 7) / 8 * ((g.d + 1023) / 1024) + (p.tiles - 1) / kShortRun * ((g.d + kLongColumns - 1) / kLongColumns);
            e = launch_after_trigger(lookup_grad_join_kernel, dim3(blocks_x, g.nodes), dim3(256), 0, s, true, p);
            if (e != cudaSuccess) return e;
        }
        first += count;
    }
    return cudaSuccess;
}

}  // namespace gpga
