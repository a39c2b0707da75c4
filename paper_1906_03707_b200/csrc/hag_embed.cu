// Embedding: rows of a table selected by ids and scaled, and the gradient of the table.
//   forward   out_i = scale * T[id_i]
//   backward  gT_v  = scale * sum over i with id_i = v of g_i
// An id outside 0..V-1 stands for no token: its row is zero and it takes no part in the gradient.
//
// The gradient adds in a fixed order: the ids are sorted (stable radix sort, 8 bits at a time at most, integer
// counters only), so that the tokens of a row lie side by side in ascending order, and each row is a sum over one
// stretch of them.  No atomics on floats: the same inputs give the same bits.
//
// Both are bound by memory.  Measured on B200 (copy rate 6.45 TB/s): lookup of 500 000 x 64 fp32 from 119 rows 23 us (the
// 128 MB written at 5.6 TB/s), of 10^6 x 256 fp32 into bf16 from 50 257 rows 140 us (1 GB of rows out of the L1 and L2
// besides 543 MB of DRAM traffic; none of the three is above half of its rate: the warps, 32 per SM at 64 registers, wait
// for their rows half of the time).  Gradient of 500 000 x 64 fp32 into 119 rows 29 us (128 MB read); of 10^6 x 256 bf16
// into 50 257 fp32 rows 151 us: 94 for the sums (512 MB read, 51 MB written), 9 for the joins, 48 for two sorting passes
// and the zeros; of 4096 x 768 bf16 into that table, which is mostly zeros, 39 us.  Widths without 16-byte vectors go by 4
// or 2 bytes: lookup of 300 000 x 333 106 us, fp32 and bf16 alike.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "hag.h"
#include "hag_kernels.cuh"
#include "hag_launch.h"
#include "hag_rows.cuh"

namespace {

template <typename Args>
cudaError_t launch_with(void (*kernel)(Args), dim3 grid, unsigned threads, size_t shared, const Args &args, cudaStream_t s) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args);
}

// Lets the kernel use that much dynamic shared memory on the current device (asked once per device).
template <auto KERNEL>
bool allow_shared(size_t bytes) {
    static std::atomic<uint64_t> ready{0};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return false;
    const uint64_t bit = uint64_t(1) << (device & 63);
    if (ready.load(std::memory_order_relaxed) & bit) return true;
    if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes)) != cudaSuccess) return false;
    ready.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

constexpr int kCopyThreads = 256;
constexpr int kCopyBlocks = 148 * 4;      // all resident; with 3 per SM 10^6 x 256 takes 179 us, with 4 138, with 6 143

struct LookupArgs {
    const void *ids;
    int32_t ids64;
    int32_t n_rows;          // V
    int64_t n;
    const void *table;
    int64_t ld_table;
    void *out;
    int64_t ld_out;
    int32_t n_vec;           // vectors per row
    int32_t lane_bits;       // log2 of the lanes that cover a row
    float scale;
};

__device__ __forceinline__ int64_t load_id(const void *ids, int ids64, int64_t i) {
    return ids64 ? __ldca(static_cast<const long long *>(ids) + i) : int64_t(__ldca(static_cast<const int *>(ids) + i));
}

// A warp takes U steps of rows at a time (32 / lanes rows per step) and has their loads in flight together; rows of
// more than 32 vectors are taken K * 32 vectors at a time.  The ids of the next rows are read while these are copied.
// The table is read through L1: frequent rows are found there, and without it the few lines of a small table are asked
// of the same corner of the L2 by every SM (500 000 x 64 from 119 rows: 46 us, with L1 34).  The output is stored
// evict-first: it would push the table out of the L2 (that case 26.8 us, so 23.0).
template <typename TT, typename TO, int V, int U, int K>
__global__ void __launch_bounds__(kCopyThreads, 4) embedding_fwd_kernel(const LookupArgs p) {
    hagk::pdl_launch_dependents();
    const int lane = threadIdx.x & 31, gl = lane & ((1 << p.lane_bits) - 1), slice = lane >> p.lane_bits, per_step = 32 >> p.lane_bits;
    const int64_t warps = int64_t(gridDim.x) * (kCopyThreads / 32), stride = warps * U * per_step;
    int64_t row = (int64_t(blockIdx.x) * (kCopyThreads / 32) + (threadIdx.x >> 5)) * U * per_step + slice;
    const TT *table = static_cast<const TT *>(p.table);
    TO *out = static_cast<TO *>(p.out) + row * p.ld_out;
    const int64_t out_step = per_step * p.ld_out, out_stride = stride * p.ld_out;
    int32_t id[U];           // of the rows in turn; -1: no row
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = r + u * per_step;
            const int64_t x = i < p.n ? load_id(p.ids, p.ids64, i) : -1;
            id[u] = uint64_t(x) < uint64_t(p.n_rows) ? int32_t(x) : -1;
        }
    };
    hagk::pdl_wait();
    fetch(row);
    for (; row - slice < p.n; row += stride, out += out_stride) {
        int32_t at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) at[u] = id[u];
        fetch(row + stride);
        for (int c = blockIdx.y * (32 * K) + gl; c < p.n_vec; c += gridDim.y * (32 * K)) {
            hagr::Vec<TT, V> in[U][K];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    in[u][k].zero();
                    if (at[u] >= 0 && c + 32 * k < p.n_vec) in[u][k].template load<hagr::kNear>(table + at[u] * p.ld_table, c + 32 * k);
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (row + u * per_step >= p.n || c + 32 * k >= p.n_vec) continue;
                    float v[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] = at[u] >= 0 ? in[u][k].get(j) * p.scale : 0.0f;      // no row: zero even where the scale is no number
                    hagr::Vec<TO, V> o;
                    o.set(v);
                    o.template store<hagr::kOnce>(out + u * out_step, c + 32 * k);
                }
        }
    }
}

template <typename TT, typename TO, int V, int U, int K>
cudaError_t launch_lookup_rows(const LookupArgs &p, cudaStream_t s) {
    const int64_t rows_per_block = int64_t(kCopyThreads / 32) * U * (32 >> p.lane_bits);
    const int64_t row_blocks = (p.n + rows_per_block - 1) / rows_per_block, chunks = (p.n_vec + 32 * K - 1) / (32 * K);
    const unsigned grid = unsigned(std::min<int64_t>(row_blocks, kCopyBlocks));
    const unsigned columns = unsigned(std::min<int64_t>({chunks, std::max<int64_t>(kCopyBlocks / grid, 1), 65535}));      // few rows: their columns over blocks
    return launch_with(embedding_fwd_kernel<TT, TO, V, U, K>, dim3(grid, columns), kCopyThreads, 0, p, s);
}

template <typename TT, typename TO, int V>
cudaError_t launch_lookup(LookupArgs &p, int32_t D, cudaStream_t s) {
    constexpr int kLoads = V * int(sizeof(TT)) >= 8 ? 4 : 8;              // in flight per lane
    p.n_vec = D / V;
    p.lane_bits = 0;
    while (p.lane_bits < 5 && (1 << p.lane_bits) < p.n_vec) ++p.lane_bits;
    if (p.n_vec <= 32) return launch_lookup_rows<TT, TO, V, kLoads, 1>(p, s);
    if (p.n_vec <= 64) return launch_lookup_rows<TT, TO, V, kLoads / 2, 2>(p, s);
    return launch_lookup_rows<TT, TO, V, kLoads / 4, 4>(p, s);
}

template <typename TT, typename TO>
cudaError_t launch_lookup_v(LookupArgs &p, int32_t D, cudaStream_t s) {
    // 16 bytes of the wider type: neighbouring lanes touch neighbouring words on both sides (8 elements of fp32 per lane
    // would be two stores of every second half sector: 10^6 x 128 from bf16 into fp32 147 us)
    constexpr int kMost = sizeof(TT) == 2 && sizeof(TO) == 2 ? 8 : 4;
    const hagr::Operand ops[] = {{p.table, p.ld_table, int(sizeof(TT))}, {p.out, p.ld_out, int(sizeof(TO))}};
    switch (hagr::vector_elems(kMost, D, ops)) {
        case 8: if constexpr (kMost == 8) return launch_lookup<TT, TO, 8>(p, D, s);
        case 4: return launch_lookup<TT, TO, 4>(p, D, s);
        case 2: return launch_lookup<TT, TO, 2>(p, D, s);
        default: return launch_lookup<TT, TO, 1>(p, D, s);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Zeros for the rows of the gradient, written by blocks of their own next to the sort's in the sort's launches: the
// sort waits for latencies and leaves the memory idle.  The rows that some id names are written again afterwards.
struct FillArgs {
    char *out;
    int64_t row_bytes, ld_bytes;
    int32_t rows_begin, rows_end;      // of this launch
    int32_t elem;                      // bytes
    int32_t blocks;
};
constexpr int kFillThreads = 1024;     // those of the sort's launches

// Threads tid, tid + step, ... clear `bytes` bytes at p (a multiple of the element, 2 or 4).
__device__ __forceinline__ void clear_span(char *p, int64_t bytes, int elem, int64_t tid, int64_t step) {
    int64_t head = int64_t((16 - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u);
    if (head > bytes) head = bytes;
    const int64_t body = (bytes - head) / 16, tail = head + body * 16;
    for (int64_t i = tid; i < body; i += step) *reinterpret_cast<uint4 *>(p + head + i * 16) = make_uint4(0, 0, 0, 0);
    // the ragged ends: at most 7 elements each
    for (int64_t i = tid * elem; i < head; i += step * elem) {
        if (elem == 4) *reinterpret_cast<uint32_t *>(p + i) = 0; else *reinterpret_cast<uint16_t *>(p + i) = 0;
    }
    for (int64_t i = tail + tid * elem; i < bytes; i += step * elem) {
        if (elem == 4) *reinterpret_cast<uint32_t *>(p + i) = 0; else *reinterpret_cast<uint16_t *>(p + i) = 0;
    }
}

__device__ __forceinline__ void fill_rows(const FillArgs &f, int block) {
    if (f.ld_bytes == f.row_bytes) {
        clear_span(f.out + f.rows_begin * f.row_bytes, (f.rows_end - f.rows_begin) * f.row_bytes, f.elem,
                   int64_t(block) * kFillThreads + threadIdx.x, int64_t(f.blocks) * kFillThreads);
    } else {
        const int lane = threadIdx.x & 31;
        for (int64_t r = f.rows_begin + int64_t(block) * (kFillThreads / 32) + (threadIdx.x >> 5); r < f.rows_end;
             r += int64_t(f.blocks) * (kFillThreads / 32))
            clear_span(f.out + r * f.ld_bytes, f.row_bytes, f.elem, lane, 32);
    }
}

__global__ void __launch_bounds__(kFillThreads) fill_kernel(const FillArgs f) {
    hagk::pdl_launch_dependents();
    hagk::pdl_wait();
    fill_rows(f, blockIdx.x);
}

// ---------------------------------------------------------------------------------------------------------------
// Stable radix sort of (key, place) pairs by key; key = the id, or V for a place without a token (those come last).
// Each pass is two launches: every block counts the digits of its own stretch of the list (sort_count_kernel); then
// every block adds up the counts of all blocks and moves its stretch to the places found (sort_move_kernel).  Within a
// block a key's place comes from the lanes of its warp that hold the same digit, the warp's count so far and
// the counts of the warps before it: keys keep their order, and nothing depends on the order of atomics.
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 8;                                 // keys per thread and tile
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kSortBins = 256;
constexpr int kSortMaxBlocks = 148;                           // every block reads the counts of all blocks
constexpr int kSortUnit = kSortThreads;                       // stretches are multiples of one key per thread

struct SortArgs {
    const void *ids;         // first pass: the caller's ids
    int32_t ids64;
    int32_t n_rows;          // V
    const uint2 *in;         // later passes: {key, place}
    uint2 *out;
    uint32_t *count;         // [blocks][bins]
    int32_t n;
    int32_t stretch;         // keys per block, a multiple of kSortUnit
    int32_t shift, bits;
    int32_t passes;          // of the single-launch form
    int32_t blocks;          // that sort; the blocks after them clear rows of the gradient
    FillArgs fill;
};

__device__ __forceinline__ uint2 sort_pair(const SortArgs &p, int32_t i) {
    if (p.in) return __ldcg(p.in + i);
    const int64_t id = load_id(p.ids, p.ids64, i);
    return make_uint2(uint64_t(id) < uint64_t(p.n_rows) ? uint32_t(id) : uint32_t(p.n_rows), uint32_t(i));
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int kCopies = 4;                                // of the counters: fewer warps on one address
    __shared__ uint32_t bin[kCopies][kSortBins];
    const int t = threadIdx.x;
    for (int i = t; i < kCopies * kSortBins; i += kSortThreads) (&bin[0][0])[i] = 0;
    __syncthreads();
    const uint32_t mask = (1u << p.bits) - 1u;
    hagk::pdl_wait();
    if (int(blockIdx.x) >= p.blocks) {
        fill_rows(p.fill, blockIdx.x - p.blocks);
        return;
    }
    const int32_t begin = int32_t(blockIdx.x) * p.stretch, end = int32_t(min(int64_t(p.n), int64_t(begin) + p.stretch));
    uint32_t *mine = bin[(t >> 5) % kCopies];
    for (int32_t tile = begin; tile < end; tile += kSortTile) {
        uint32_t key[kSortItems];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) key[k] = tile + k * kSortThreads + t < end ? sort_pair(p, tile + k * kSortThreads + t).x : 0;
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (tile + k * kSortThreads + t < end) atomicAdd(&mine[(key[k] >> p.shift) & mask], 1u);
    }
    __syncthreads();
    if (t < kSortBins) p.count[blockIdx.x * kSortBins + t] = bin[0][t] + bin[1][t] + bin[2][t] + bin[3][t];
}

// Keys per thread for a tile of so many: no thread works on more empty places than it must.
__device__ __forceinline__ int tile_items(int32_t len) { return min((len + kSortThreads - 1) / kSortThreads, kSortItems); }

// What a block needs to order a tile of pairs by one digit.
struct SortShared {
    uint2 pair[kSortTile];
    uint32_t seen[kSortWarps][kSortBins];      // per warp: keys of the digit so far; then the first place of the warp's keys in the tile
    uint32_t base[kSortBins];                  // next place in the list of each digit of this block
    uint32_t shift_by[kSortBins];              // place in the list minus place in the tile
    uint32_t scan[kSortBins / 32];
};

// Exclusive sums over the bins, for the first kSortBins threads; all threads call it.
__device__ __forceinline__ uint32_t bin_scan(uint32_t count, uint32_t *scan) {
    const int t = threadIdx.x, lane = t & 31;
    uint32_t x = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (t < kSortBins && lane == 31) scan[t >> 5] = x;
    __syncthreads();
    uint32_t lower = 0;
#pragma unroll
    for (int w = 0; w < kSortBins / 32; ++w)
        if (w < (t >> 5)) lower += scan[w];
    return lower + x - count;
}

// Orders a tile by the digit at `shift`: the pairs (in registers, `items` per thread, a warp's are consecutive in the
// list) end in sm.pair.  Returns, for threads below kSortBins, how many keys have digit t; sm.shift_by[t] is set from
// `base`.
__device__ __forceinline__ uint32_t sort_tile(SortShared &sm, const uint2 (&pair)[kSortItems], int items, int shift, uint32_t mask,
                                              uint32_t base) {
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    for (int i = t; i < kSortWarps * kSortBins / 4; i += kSortThreads) reinterpret_cast<uint4 *>(&sm.seen[0][0])[i] = make_uint4(0, 0, 0, 0);
    uint32_t same[kSortItems], rank[kSortItems];
    // lanes with the same digit, bit by bit: a vote per bit costs about a fifth of what the match instruction takes on
    // digits that mostly differ (10 000 cycles per tile there)
#pragma unroll
    for (int k = 0; k < kSortItems; ++k) same[k] = 0xffffffffu;
#pragma unroll
    for (int bit = 0; bit < 8; ++bit) {
        if ((mask >> bit) == 0) break;
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            if (k >= items) break;
            const bool set = (pair[k].x >> (shift + bit)) & 1u;
            const uint32_t votes = __ballot_sync(0xffffffffu, set);
            same[k] &= set ? votes : ~votes;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortItems; ++k) {
        if (k >= items) break;
        uint32_t *count = &sm.seen[warp][(pair[k].x >> shift) & mask];
        rank[k] = *count + __popc(same[k] & ((1u << lane) - 1u));
        __syncwarp();
        if ((same[k] >> lane) == 1u) *count = rank[k] + 1;                // the highest lane of the digit
        __syncwarp();
    }
    __syncthreads();
    uint32_t all = 0, c[kSortWarps];
    if (t < kSortBins) {
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            c[w] = all;
            all += sm.seen[w][t];
        }
    }
    const uint32_t first = bin_scan(all, sm.scan);
    if (t < kSortBins) {
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) sm.seen[w][t] = first + c[w];
        sm.shift_by[t] = base - first;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortItems; ++k)
        if (k < items) sm.pair[sm.seen[warp][(pair[k].x >> shift) & mask] + rank[k]] = pair[k];
    __syncthreads();
    return all;
}

__global__ void __launch_bounds__(kSortThreads) sort_move_kernel(const SortArgs p) {
    hagk::pdl_launch_dependents();
    extern __shared__ __align__(16) char raw[];
    SortShared &sm = *reinterpret_cast<SortShared *>(raw);
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const uint32_t mask = (1u << p.bits) - 1u;
    hagk::pdl_wait();
    if (int(blockIdx.x) >= p.blocks) {
        fill_rows(p.fill, blockIdx.x - p.blocks);
        return;
    }
    const int32_t begin = int32_t(blockIdx.x) * p.stretch, end = int32_t(min(int64_t(p.n), int64_t(begin) + p.stretch));
    uint2 pair[kSortItems];
    // a warp's keys are consecutive: stable.  Places beyond the end hold the largest key and come after all others of
    // the tile, which is the list's last.
    int items = 0;
    auto load = [&](int32_t tile) {
        items = tile_items(end - tile);
        const int32_t mine = tile + warp * (32 * items) + lane;
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (k < items) pair[k] = mine + 32 * k < end ? sort_pair(p, mine + 32 * k) : make_uint2(0xffffffffu, 0);
    };
    load(begin);
    uint32_t base = 0;       // for t < kSortBins: keys with a smaller digit + keys of digit t in the blocks before this one
    {
        constexpr int kQuads = kSortBins / 4, kGroups = kSortThreads / kQuads;           // 64 threads read the counts of one block
        const int quad = t % kQuads, group = t / kQuads;
        uint4 before = make_uint4(0, 0, 0, 0), total = before;
#pragma unroll 10
        for (int b = group; b < p.blocks; b += kGroups) {
            const uint4 c = __ldcg(reinterpret_cast<const uint4 *>(p.count + b * kSortBins) + quad);
            const uint32_t in = b < int(blockIdx.x) ? 0xffffffffu : 0u;
            total.x += c.x; total.y += c.y; total.z += c.z; total.w += c.w;
            before.x += c.x & in; before.y += c.y & in; before.z += c.z & in; before.w += c.w & in;
        }
        static_assert(2 * kGroups <= kSortWarps, "the sums of the groups share the counters' space");
        reinterpret_cast<uint4 *>(sm.seen[group])[quad] = total;
        reinterpret_cast<uint4 *>(sm.seen[kGroups + group])[quad] = before;
        __syncthreads();
        uint32_t all = 0;
        if (t < kSortBins) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                all += sm.seen[g][t];
                base += sm.seen[kGroups + g][t];
            }
        }
        base += bin_scan(all, sm.scan);
    }
    for (int32_t tile = begin; tile < end; tile += kSortTile) {
        if (tile != begin) load(tile);
        __syncthreads();
        base += sort_tile(sm, pair, items, p.shift, mask, base);
        const int32_t len = min(end - tile, kSortTile);
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const int i = k * kSortThreads + t;
            if (i >= len) continue;
            const uint2 q = sm.pair[i];
            p.out[sm.shift_by[(q.x >> p.shift) & mask] + i] = q;          // neighbours mostly go to neighbouring places
        }
    }
}

// A list of one tile: all passes in one launch, the pairs stay in shared memory.
__global__ void __launch_bounds__(kSortThreads) sort_small_kernel(const SortArgs p) {
    hagk::pdl_launch_dependents();
    extern __shared__ __align__(16) char raw[];
    SortShared &sm = *reinterpret_cast<SortShared *>(raw);
    const int t = threadIdx.x;
    const uint32_t mask = (1u << p.bits) - 1u;
    hagk::pdl_wait();
    if (blockIdx.x >= 1) {
        fill_rows(p.fill, blockIdx.x - 1);
        return;
    }
    const int items = tile_items(p.n), mine = (t >> 5) * (32 * items) + (t & 31);
    uint2 pair[kSortItems];
#pragma unroll
    for (int k = 0; k < kSortItems; ++k)
        if (k < items) pair[k] = mine + 32 * k < p.n ? sort_pair(p, mine + 32 * k) : make_uint2(0xffffffffu, 0);
    for (int pass = 0; pass < p.passes; ++pass) {
        sort_tile(sm, pair, items, pass * p.bits, mask, 0);
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (k < items) pair[k] = sm.pair[mine + 32 * k];
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kSortItems; ++k)
        if (k < items && mine + 32 * k < p.n) p.out[mine + 32 * k] = pair[k];
}

// ---------------------------------------------------------------------------------------------------------------
// The sums.  The sorted list is cut into equal stretches, one per worker (a group of lanes that covers a row, or 32
// vectors of it, with one load per lane), so the work does not depend on how often an id occurs.  A worker adds up
// run after run of equal ids; a run that lies inside its stretch is a finished row.  A run that crosses into or out of
// the stretch leaves a partial row: the one that was open at the stretch's start in `head`, the one that is open at its
// end in `tail`; embedding_join_kernel adds those up in the order of the stretches.
struct SumArgs {
    const uint2 *list;               // {key, place} sorted; readable in whole groups of kSumBatch
    int32_t n;
    int32_t n_rows;                  // V
    const void *grad;
    int64_t ld_grad;
    void *out;
    int64_t ld_out;
    int32_t D;
    float scale;
    int32_t stretch;                 // places per worker, a multiple of kSumBatch
    int32_t workers;
    int32_t lanes;                   // per worker: 4, 8, 16 or 32
    float *head, *tail;              // [workers][D up to a multiple of 4]
};
constexpr int kSumThreads = 256;
constexpr int kSumBatch = 8;         // rows in flight per worker

__device__ __forceinline__ uint32_t list_key(const SumArgs &p, int64_t i) { return __ldcg(&p.list[i].x); }

template <typename TO, int V>
__device__ __forceinline__ void store_row(const SumArgs &p, uint32_t key, int vec, const float *acc) {
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = acc[j] * p.scale;
    hagr::Vec<TO, V> o;
    o.set(v);
    o.store(static_cast<TO *>(p.out) + int64_t(key) * p.ld_out, vec);
}

// K: vectors per lane, 32 apart (narrow vectors: a row's loads would else be too small to keep the memory busy).
template <typename TG, typename TO, int V, int K>
__global__ void __launch_bounds__(kSumThreads) embedding_sum_kernel(const SumArgs p) {
    hagk::pdl_launch_dependents();
    const int worker = (blockIdx.x * kSumThreads + threadIdx.x) / p.lanes;
    const int vec = blockIdx.y * (32 * K) + (threadIdx.x & (p.lanes - 1)), n_vec = p.D / V;      // lanes beyond the row only keep step
    const int32_t t0 = worker < p.workers ? worker * p.stretch : p.n;
    const int32_t t1 = int32_t(min(int64_t(p.n), int64_t(t0) + p.stretch));
    hagk::pdl_wait();
    if (t0 >= t1) return;
    const uint32_t none = 0xffffffffu, rows = uint32_t(p.n_rows);
    const uint32_t before = t0 > 0 ? list_key(p, t0 - 1) : none, after = t1 < p.n ? list_key(p, t1) : none;
    const int64_t part = int64_t(worker) * ((p.D + 3) & ~3);
    float acc[K][V];
    auto clear = [&]() {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) acc[k][j] = 0.0f;
    };
    auto leave = [&](float *at) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            hagr::Vec<float, V> o;
            o.set(acc[k]);
            if (vec + 32 * k < n_vec) o.store(at + part, vec + 32 * k);
        }
    };
    auto finish = [&](uint32_t row) {
        if (row >= rows) return;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (vec + 32 * k < n_vec) store_row<TO, V>(p, row, vec + 32 * k, acc[k]);
    };
    uint32_t key[kSumBatch], place[kSumBatch];
    auto fetch = [&](int32_t t) {
#pragma unroll
        for (int h = 0; h < kSumBatch; h += 2) {
            const uint4 q = __ldcg(reinterpret_cast<const uint4 *>(p.list + t + h));
            key[h] = q.x; place[h] = q.y; key[h + 1] = q.z; place[h + 1] = q.w;
        }
    };
    fetch(t0);
    uint32_t cur = key[0];
    bool from_left = cur == before;                            // the current run began in an earlier stretch
    clear();
    for (int32_t t = t0; t < t1; t += kSumBatch) {
        hagr::Vec<TG, V> g[kSumBatch][K];
        uint32_t id[kSumBatch];
#pragma unroll
        for (int u = 0; u < kSumBatch; ++u) {
            id[u] = t + u < t1 ? key[u] : none;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                g[u][k].zero();
                if (id[u] < rows && vec + 32 * k < n_vec)
                    g[u][k].template load<hagr::kOnce>(static_cast<const TG *>(p.grad) + int64_t(place[u]) * p.ld_grad, vec + 32 * k);
            }
        }
        if (t + kSumBatch < t1) fetch(t + kSumBatch);          // the next ids while the rows are on their way
        if (id[kSumBatch - 1] == cur) {                        // sorted: the whole batch belongs to the run
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float even = (g[0][k].get(j) + g[4][k].get(j)) + (g[2][k].get(j) + g[6][k].get(j));
                    const float odd = (g[1][k].get(j) + g[5][k].get(j)) + (g[3][k].get(j) + g[7][k].get(j));
                    acc[k][j] += even + odd;
                }
            continue;
        }
#pragma unroll
        for (int u = 0; u < kSumBatch; ++u) {
            if (t + u < t1 && id[u] != cur) {
                if (from_left) leave(p.head);
                else finish(cur);
                from_left = false;
                cur = id[u];
                clear();
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[k][j] += g[u][k].get(j);
        }
    }
    if (from_left) leave(p.head);
    else if (cur == after) leave(p.tail);
    else finish(cur);
}

// Rows whose runs cross stretches: the tail of the stretch where the run begins and the heads of the following
// stretches that begin with it.  A warp takes one stretch; chains of more than kLongChain heads (an id that fills
// many stretches) are taken by all the warps of the block together, every group of lanes a share of the heads.
constexpr int kJoinThreads = 512;
constexpr int kJoinWarps = kJoinThreads / 32;
constexpr int kLongChain = 12;
constexpr int kJoinQuads = 32;          // a block's columns, in fours

__device__ __forceinline__ float4 add4(float4 a, float4 b) {
    const float2 lo = __fadd2_rn(make_float2(a.x, a.y), make_float2(b.x, b.y)), hi = __fadd2_rn(make_float2(a.z, a.w), make_float2(b.z, b.w));
    return make_float4(lo.x, lo.y, hi.x, hi.y);
}

template <typename TO>
__device__ __forceinline__ void join_store(const SumArgs &p, uint32_t key, int quad, float4 v) {
    const float f[4] = {v.x * p.scale, v.y * p.scale, v.z * p.scale, v.w * p.scale};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (quad * 4 + j >= p.D) break;
        hagr::Vec<TO, 1> o;
        o.set(f + j);
        o.store(static_cast<TO *>(p.out) + int64_t(key) * p.ld_out, quad * 4 + j);
    }
}

template <typename TO>
__global__ void __launch_bounds__(kJoinThreads) embedding_join_kernel(const SumArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ int chain[kJoinWarps];
    __shared__ float4 sum[kJoinWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int w0 = blockIdx.x * kJoinWarps, w = w0 + warp;
    const int quads = (p.D + 3) / 4;                           // of a partial row
    const float4 *head = reinterpret_cast<const float4 *>(p.head), *tail = reinterpret_cast<const float4 *>(p.tail);
    hagk::pdl_wait();
    // heads that continue the run open at the end of stretch `w`; 0: none begins there
    int heads = 0;
    uint32_t key = 0;
    const int64_t t1 = (int64_t(w) + 1) * p.stretch;
    if (w < p.workers && t1 < p.n) {
        key = list_key(p, t1 - 1);
        const int64_t t0 = t1 - p.stretch;
        const bool begins = !(list_key(p, t0) == key && t0 > 0 && list_key(p, t0 - 1) == key);
        if (begins && key < uint32_t(p.n_rows)) {
            for (int j = w + 1;; j += 128) {
                int c = 0;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = j + 32 * u + lane;
                    c += __popc(__ballot_sync(0xffffffffu, i < p.workers && list_key(p, int64_t(i) * p.stretch) == key));
                }
                heads += c;
                if (c < 128) break;
            }
        }
    }
    if (lane == 0) chain[warp] = heads;
    __syncthreads();
    if (heads > 0 && heads <= kLongChain)
        if (const int q = blockIdx.y * kJoinQuads + lane; q < quads) {
            float4 v = __ldcg(tail + int64_t(w) * quads + q);
#pragma unroll 4
            for (int j = 1; j <= heads; ++j) v = add4(v, __ldcg(head + int64_t(w + j) * quads + q));
            join_store<TO>(p, key, q, v);
        }
    int lanes = 4;                                             // that cover the columns of this block
    while (lanes < kJoinQuads && lanes < quads) lanes *= 2;
    const int group = threadIdx.x / lanes, groups = kJoinThreads / lanes;
    for (int x = 0; x < kJoinWarps; ++x) {
        const int count = chain[x];                            // the same for all threads
        if (count <= kLongChain) continue;
        const uint32_t k = list_key(p, (int64_t(w0 + x) + 1) * p.stretch - 1);
        const int q = blockIdx.y * kJoinQuads + threadIdx.x % lanes;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (q < quads) {
            if (group == 0) v = __ldcg(tail + int64_t(w0 + x) * quads + q);
#pragma unroll 8
            for (int j = 1 + group; j <= count; j += groups) v = add4(v, __ldcg(head + int64_t(w0 + x + j) * quads + q));
        }
        for (int o = lanes; o < 32; o *= 2)                    // the groups of a warp, then the warps
            v = add4(v, make_float4(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o),
                                    __shfl_xor_sync(0xffffffffu, v.z, o), __shfl_xor_sync(0xffffffffu, v.w, o)));
        __syncthreads();
        if (lane < lanes) sum[warp][lane] = v;
        __syncthreads();
        if (group == 0 && q < quads) {
#pragma unroll
            for (int y = 1; y < kJoinWarps; ++y) v = add4(v, sum[y][lane]);
            join_store<TO>(p, k, q, v);
        }
    }
}

// (A warp per row of the table instead, whatever its length, took 47.7 ms on the million ids above, 21.3 ms on 119 rows.)
// Warps for the sums: 16 per SM with kSumBatch 16-byte loads per lane in flight keep 64 KB per SM on their way.
constexpr int kSumWarps = 148 * 16;
constexpr int kSumFew = 64;          // ids that one worker takes: the join's launch costs more than the 7 turns it saves

template <typename TG, typename TO, int V, int K>
cudaError_t launch_sum_columns(SumArgs &p, cudaStream_t s) {
    const int n_vec = p.D / V;
    p.lanes = hagl::lanes_per_row(n_vec);
    const int column_blocks = (n_vec + 32 * K - 1) / (32 * K);
    const int64_t most = std::max<int64_t>(int64_t(kSumWarps) / column_blocks, 1) * (32 / p.lanes);
    const int64_t batches = (int64_t(p.n) + kSumBatch - 1) / kSumBatch;
    p.stretch = int32_t((batches + most - 1) / most * kSumBatch);
    if (p.n <= kSumFew) p.stretch = kSumFew;                 // one worker: nothing to join
    p.workers = int32_t((int64_t(p.n) + p.stretch - 1) / p.stretch);
    cudaError_t err = launch_with(embedding_sum_kernel<TG, TO, V, K>,
                                  dim3(unsigned((int64_t(p.workers) * p.lanes + kSumThreads - 1) / kSumThreads), unsigned(column_blocks)),
                                  kSumThreads, 0, p, s);
    if (err == cudaSuccess && p.workers > 1)
        err = launch_with(embedding_join_kernel<TO>,
                          dim3(unsigned((p.workers + kJoinWarps - 1) / kJoinWarps), unsigned(((p.D + 3) / 4 + kJoinQuads - 1) / kJoinQuads)),
                          kJoinThreads, 0, p, s);
    return err;
}

template <typename TG, typename TO, int V>
cudaError_t launch_sum(SumArgs &p, cudaStream_t s) {
    // up to 16 bytes per lane and row, as far as the row fills them
    constexpr int kMost = V * int(sizeof(TG)) >= 8 ? 1 : 4;
    const int n_vec = p.D / V;
    if constexpr (kMost == 4) {
        if (n_vec > 64) return launch_sum_columns<TG, TO, V, 4>(p, s);
        if (n_vec > 32) return launch_sum_columns<TG, TO, V, 2>(p, s);
    }
    return launch_sum_columns<TG, TO, V, 1>(p, s);
}

template <typename TG, typename TO>
cudaError_t launch_sum_v(SumArgs &p, cudaStream_t s) {
    constexpr int kMost = sizeof(TG) == 4 && sizeof(TO) == 4 ? 4 : 8;
    const hagr::Operand ops[] = {{p.grad, p.ld_grad, int(sizeof(TG))}, {p.out, p.ld_out, int(sizeof(TO))}};
    switch (hagr::vector_elems(kMost, p.D, ops)) {
        case 8: if constexpr (kMost == 8) return launch_sum<TG, TO, 8>(p, s);
        case 4: return launch_sum<TG, TO, 4>(p, s);
        case 2: return launch_sum<TG, TO, 2>(p, s);
        default: return launch_sum<TG, TO, 1>(p, s);
    }
}

// Floats of `head` (and of `tail`), at most: workers * columns is bounded by the lanes times the vector, for any width.
int64_t partial_floats(int64_t n, int32_t D) {
    const int64_t width = (int64_t(D) + 3) / 4 * 4, batches = (n + kSumBatch - 1) / kSumBatch;
    // at V elements per lane a worker covers up to 32 V columns: workers <= kSumWarps * 32 V / D (and twice that where D
    // does not fill its lanes), at least 8 per column block
    const int64_t workers = std::max<int64_t>(2 * (int64_t(kSumWarps) * 32 * 8 + D - 1) / D, 8);
    return std::min(workers, batches) * width;
}

// ---------------------------------------------------------------------------------------------------------------
// Few rows (tile_count says which): no sort of the whole list (500 000 x 64 into 119 rows takes 29 us this way and 52 by
// the sort, 100 000 x 64 13 and 32).  Every block sorts a tile of the tokens in shared memory, adds up its runs as above
// (its groups of lanes are the workers, heads and tails stay in shared memory), and leaves a table of its own: all rows,
// its columns.  table_join_kernel adds up the blocks' tables in order.  One tile alone writes the result.
struct TileArgs {
    SortArgs sort;               // ids, n, digits; stretch: tokens per tile
    const void *grad;
    int64_t ld_grad;
    void *out;
    int64_t ld_out;
    int32_t D;
    float scale;
    int32_t lanes;               // per worker
    float *partial;              // [tiles][n_rows][pitch], or null: one tile, whose sums are the result
    int32_t pitch;               // D up to a multiple of 4: rows of a table start on 16 bytes
    int32_t parts;
    hagr::Divisor per_row;       // the pitch (table_join_kernel)
};
constexpr int kTileBatch = 4;    // rows in flight per worker: 32 warps of them (at 64 registers, with 32 bytes spilled by the sort)
// Of a tile's gradient rows, what is asked into the L2 while the ids are sorted, when the memory would be idle: 500 000 x 64
// into 119 rows takes 29.2 us with it and 32.8 without (128 KB 29.7, 384 KB 29.9).  In the launches of the full sort the
// same slowed the sort by what it saved.
constexpr int kTileAhead = 224 << 10;

template <typename TO>
__device__ __forceinline__ void store_scalar(const TileArgs &p, int32_t row, int32_t col, float v) {
    hagr::Vec<TO, 1> o;
    v *= p.scale;
    o.set(&v);
    o.store(static_cast<TO *>(p.out) + int64_t(row) * p.ld_out, col);
}

// A row's sum to this tile's table, or to the result.
template <typename TO, int V>
__device__ __forceinline__ void store_sum(const TileArgs &p, int32_t row, int vec, const float *acc) {
    if (p.partial) {
        hagr::Vec<float, V> o;
        o.set(acc);
        o.store(p.partial + (int64_t(blockIdx.x) * p.sort.n_rows + row) * p.pitch, vec);
    } else {
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = acc[j] * p.scale;
        hagr::Vec<TO, V> o;
        o.set(v);
        o.store(static_cast<TO *>(p.out) + int64_t(row) * p.ld_out, vec);
    }
}

template <typename TG, typename TO, int V>
__global__ void __launch_bounds__(kSortThreads) embedding_tile_kernel(const __grid_constant__ TileArgs p) {
    hagk::pdl_launch_dependents();
    extern __shared__ __align__(16) char raw[];
    SortShared &sm = *reinterpret_cast<SortShared *>(raw);
    float *open_rows = reinterpret_cast<float *>(raw + sizeof(SortShared));      // [head, tail][threads * V]
    const int t = threadIdx.x, rows = p.sort.n_rows;
    const int32_t begin = blockIdx.x * p.sort.stretch, len = min(p.sort.stretch, p.sort.n - begin);
    const uint32_t mask = (1u << p.sort.bits) - 1u;
    hagk::pdl_wait();
    {
        const int items = tile_items(len), mine = (t >> 5) * (32 * items) + (t & 31);
        uint2 pair[kSortItems];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (k < items) pair[k] = mine + 32 * k < len ? sort_pair(p.sort, begin + mine + 32 * k) : make_uint2(0xffffffffu, 0);
        // while the ids are on their way: what the sums will read first, asked into the L2 ...
        if (p.partial) {
            constexpr int kLine = 128;
            const int from = blockIdx.y * p.lanes * V, bytes = min(p.D - from, p.lanes * V) * int(sizeof(TG));
            const int per_row = (bytes + kLine - 1) / kLine, lines = min(len, kTileAhead / bytes) * per_row;
            const char *first = static_cast<const char *>(p.grad) + (begin * p.ld_grad + from) * int64_t(sizeof(TG));
            for (int i = t; i < lines; i += kSortThreads) {
                const int row = i / per_row;
                asm volatile("prefetch.global.L2 [%0];" ::"l"(first + row * p.ld_grad * int64_t(sizeof(TG)) + (i - row * per_row) * kLine));
            }
        }
        // ... and zeros for all rows, of which those that tokens name are written again
        const int vec = blockIdx.y * p.lanes + t % p.lanes;
        const float zeros[V] = {};
        if (vec < p.D / V)
            for (int r = t / p.lanes; r < rows; r += kSortThreads / p.lanes) store_sum<TO, V>(p, r, vec, zeros);
        for (int pass = 0; pass < p.sort.passes; ++pass) {
            if (pass) {
#pragma unroll
                for (int k = 0; k < kSortItems; ++k)
                    if (k < items) pair[k] = sm.pair[mine + 32 * k];
                __syncthreads();
            }
            sort_tile(sm, pair, items, pass * p.sort.bits, mask, 0);             // ends with a barrier: the rows are clear too
        }
    }
    const int worker = t / p.lanes, gl = t % p.lanes, workers = kSortThreads / p.lanes, vec = blockIdx.y * p.lanes + gl;
    const bool column = vec < p.D / V;
    const int stretch = ((len + workers - 1) / workers + kTileBatch - 1) / kTileBatch * kTileBatch;
    const int i0 = min(worker * stretch, len), i1 = min(i0 + stretch, len);
    const uint32_t none = 0xffffffffu;
    auto finish = [&](uint32_t key, const float *acc) {
        if (column && key < uint32_t(rows)) store_sum<TO, V>(p, int32_t(key), vec, acc);
    };
    float *head = open_rows, *tail = open_rows + kSortThreads * V;       // element j of thread t at [j][t]
    uint32_t cur = none, after = none;
    bool from_left = false, begins = false;
    float acc[V];
    if (i0 < i1) {
        const uint32_t before = i0 > 0 ? sm.pair[i0 - 1].x : none;
        after = i1 < len ? sm.pair[i1].x : none;
        cur = sm.pair[i0].x;
        from_left = cur == before;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.0f;
        for (int i = i0; i < i1; i += kTileBatch) {
            uint32_t k[kTileBatch];
            hagr::Vec<TG, V> g[kTileBatch];
#pragma unroll
            for (int u = 0; u < kTileBatch; ++u) {
                const uint2 q = sm.pair[i + u];                          // readable: the tile is whole
                k[u] = i + u < i1 ? q.x : none;
                g[u].zero();
                if (k[u] < uint32_t(rows) && column)
                    g[u].template load<hagr::kOnce>(static_cast<const TG *>(p.grad) + int64_t(q.y) * p.ld_grad, vec);
            }
            if (k[kTileBatch - 1] == cur) {
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += (g[0].get(j) + g[1].get(j)) + (g[2].get(j) + g[3].get(j));
                continue;
            }
#pragma unroll
            for (int u = 0; u < kTileBatch; ++u) {
                if (i + u < i1 && k[u] != cur) {
                    if (from_left) {
#pragma unroll
                        for (int j = 0; j < V; ++j) head[j * kSortThreads + t] = acc[j];
                    } else {
                        finish(cur, acc);
                    }
                    from_left = false;
                    cur = k[u];
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += g[u].get(j);
            }
        }
        if (from_left) {
#pragma unroll
            for (int j = 0; j < V; ++j) head[j * kSortThreads + t] = acc[j];
        } else if (cur == after) {
#pragma unroll
            for (int j = 0; j < V; ++j) tail[j * kSortThreads + t] = acc[j];
            begins = true;
        } else {
            finish(cur, acc);
        }
    }
    __syncthreads();
    if (!begins) return;
    // this worker's last run goes on: the heads of the workers after it that begin with the same id
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = tail[j * kSortThreads + t];
    for (int w = worker + 1; w * stretch < len && sm.pair[w * stretch].x == cur; ++w)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += head[j * kSortThreads + w * p.lanes + gl];
    finish(cur, acc);
}

// The blocks' tables added up: 32 values per block, its warps take every so-many-th table each.
template <typename TO>
__global__ void __launch_bounds__(1024) table_join_kernel(const __grid_constant__ TileArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int64_t values = int64_t(p.sort.n_rows) * p.pitch, i = int64_t(blockIdx.x) * 32 + lane;
    hagk::pdl_wait();
    float v = 0.0f;
    if (i < values) {
#pragma unroll 8
        for (int q = warp; q < p.parts; q += warps) v += __ldcg(p.partial + q * values + i);
    }
    sum[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < values) {
        for (int w = 1; w < warps; ++w) v += sum[w][lane];
        const uint32_t row = hagr::quotient(uint32_t(i), p.per_row);
        const int32_t col = int32_t(i - int64_t(row) * p.pitch);
        if (col < p.D) store_scalar<TO>(p, int32_t(row), col, v);
    }
}

constexpr int64_t kTileValues = 1 << 20;         // of the result that one tile writes
constexpr int64_t kTileTable = 1 << 17;          // of a table, where there are several
// Of the values that one block clears by itself, its columns (at most 128 of fp32) of all the rows: alone and for up to
// kTileLeast tokens, when the sort's second and third launch count; else.
constexpr int64_t kTileAlone = 1 << 17, kTileShare = 5 << 14;
// Tokens per tile of a short list.  256: 1000 x 16 into 100 rows takes 8.0 us, 4000 x 64 into 119 rows 8.9 us; with 1024
// they take 8.8 and 11.4 us.
constexpr int kTileLeast = 256, kTileMost = 2048;
constexpr int kTileBlocks = 148;
// Values of the gradient rows that one block takes alone, without the second launch: 1000 x 16 8.8 us on the device, not
// 8.0, but 2.7 us less on the host, which is what such calls wait for.
constexpr int64_t kTileFew = 32768;

// Tiles for a list, or 0: the sort.  A table costs its clearing, by one block per 128 columns, and its part of the join,
// so that large tables lose however few the tokens are; the sort's zeros are written by up to 592 blocks.  In us, by tiles /
// by the sort (up to 4096 ids whole calls with the host, else the device alone):
//   one tile    64 ids into 1040 x 64 12.2 / 14.1, 2048 x 64 15.3 / 14.0, 16 384 x 64 74 / 14.1, 600 x 336 12.2 / 14.2, 1024 x 1024 15.4 / 14.1
//               256 ids into 1040 x 64 12.2 / 16.4, 2048 x 64 16.1 / 16.1, 600 x 336 13.7 / 16.2; 1024 into 2050 x 32 13.7 / 16.1
//   several     700 ids into 2048 x 64 20.7 / 16.3, 4096 into 2048 x 64 23.2 / 16.3
//               8192 ids into 1024 x 64 18.6 / 24.7, 2048 x 64 26.3 / 26.5, 128 x 1024 18.6 / 22.2, 256 x 1024 25.6 / 26.4
//               10^6 ids into 844 x 64 71 / 82, 1689 x 64 96 / 82, 422 x 128 77 / 87, 844 x 128 105 / 87, 1689 x 128 186 / 89
// All tables together take up to 4 MB (they stay in the L2), or a quarter of the gradient rows' values.
int tile_count(int32_t n, int32_t n_rows, int32_t D) {
    const int64_t values = int64_t(n_rows) * D, columns = (int64_t(D) + 127) / 128;
    if (values > kTileValues || values > (n <= kTileLeast ? kTileAlone : kTileShare) * columns) return 0;
    if (n <= kTileLeast || (n <= kSortThreads && int64_t(n) * D <= kTileFew)) return 1;
    if (values > kTileTable) return 0;
    const int64_t most = std::max<int64_t>(1 << 20, int64_t(n) * D / 4);
    const int64_t waves = (int64_t(n) + kTileBlocks * int64_t(kSortTile) - 1) / (kTileBlocks * int64_t(kSortTile));
    int64_t tiles = waves > 1 ? waves * kTileBlocks : std::min<int64_t>(kTileBlocks, (int64_t(n) + kTileLeast - 1) / kTileLeast);
    while (tiles * values > most && tiles > 1 && (int64_t(n) + tiles / 2 - 1) / (tiles / 2) <= kTileMost) tiles /= 2;
    return tiles * values <= most ? int(tiles) : 0;
}

template <typename TG, typename TO, int V>
cudaError_t launch_tiles(TileArgs p, int tiles, cudaStream_t s) {
    if (!allow_shared<embedding_tile_kernel<TG, TO, V>>(sizeof(SortShared) + 2 * kSortThreads * V * 4)) return cudaErrorInvalidConfiguration;
    const int n_vec = p.D / V;
    p.lanes = hagl::lanes_per_row(n_vec);
    // where a row takes several blocks there are fewer tiles, of at most kSortTile tokens
    const int columns = (n_vec + 31) / 32;
    const int64_t use = std::max<int64_t>(std::min(tiles, std::max(kTileBlocks / columns, 1)), (int64_t(p.sort.n) + kSortTile - 1) / kSortTile);
    p.sort.stretch = int32_t((int64_t(p.sort.n) + use - 1) / use);
    p.parts = int32_t((int64_t(p.sort.n) + p.sort.stretch - 1) / p.sort.stretch);
    if (tiles == 1) p.partial = nullptr;
    p.pitch = (p.D + 3) & ~3;
    p.per_row = hagr::make_divisor(uint32_t(p.pitch));
    cudaError_t err = launch_with(embedding_tile_kernel<TG, TO, V>, dim3(unsigned(p.parts), unsigned(columns)), kSortThreads,
                                  sizeof(SortShared) + 2 * kSortThreads * V * 4, p, s);
    if (err == cudaSuccess && p.partial) {
        const int64_t values = int64_t(p.sort.n_rows) * p.pitch;
        int warps = 1;
        while (warps < 32 && warps < p.parts) warps *= 2;
        err = launch_with(table_join_kernel<TO>, dim3(unsigned((values + 31) / 32)), unsigned(32 * warps), 0, p, s);
    }
    return err;
}

template <typename TG, typename TO>
cudaError_t launch_tiles_v(const TileArgs &p, int tiles, cudaStream_t s) {
    const hagr::Operand ops[] = {{p.grad, p.ld_grad, int(sizeof(TG))}, {tiles == 1 ? p.out : nullptr, p.ld_out, int(sizeof(TO))}};
    switch (hagr::vector_elems(16 / int(sizeof(TG)), p.D, ops)) {
        case 8: if constexpr (sizeof(TG) == 2) return launch_tiles<TG, TO, 8>(p, tiles, s);
        case 4: return launch_tiles<TG, TO, 4>(p, tiles, s);
        case 2: return launch_tiles<TG, TO, 2>(p, tiles, s);
        default: return launch_tiles<TG, TO, 1>(p, tiles, s);
    }
}

int key_bits(int32_t n_rows) {          // of the largest key, V
    int b = 1;
    while ((int64_t(1) << b) <= n_rows) ++b;
    return b;
}

struct SortPlan {
    int blocks, passes, bits;
    int32_t stretch;
};
SortPlan sort_plan(int32_t n, int32_t n_rows) {
    SortPlan s;
    const int64_t least = n <= kSortTile ? kSortTile : (int64_t(n) + kSortMaxBlocks - 1) / kSortMaxBlocks;
    s.stretch = int32_t((least + kSortUnit - 1) / kSortUnit * kSortUnit);
    s.blocks = int((int64_t(n) + s.stretch - 1) / s.stretch);
    const int total = key_bits(n_rows);
    s.passes = (total + 7) / 8;
    s.bits = (total + s.passes - 1) / s.passes;
    return s;
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }
size_t list_bytes(int64_t n) { return up256((size_t(n) + kSumBatch) * sizeof(uint2)); }

// Blocks that clear a launch's share of the rows: 32 KB each, four per SM at most.
int fill_blocks(const FillArgs &f) {
    const int64_t bytes = (int64_t(f.rows_end) - f.rows_begin) * f.row_bytes;
    return int(std::min<int64_t>((bytes + 32767) / 32768, 148 * 4));
}

bool dtype_ok(hag_dtype d) { return d == HAG_F32 || d == HAG_BF16; }
int elem_size(hag_dtype d) { return d == HAG_F32 ? 4 : 2; }

hag_status embed_check(const void *ids, hag_id_type id_type, int64_t n, const void *rows, int64_t ld_rows, hag_dtype dtype,
                       int64_t n_rows, const void *table, int64_t ld_table, hag_dtype table_dtype, int32_t D, bool is_bwd) {
    if (!dtype_ok(dtype) || !dtype_ok(table_dtype)) return HAG_ERR_DTYPE;
    if (id_type != HAG_ID32 && id_type != HAG_ID64) return HAG_ERR_DTYPE;
    if (D <= 0 || n < 0 || n_rows < 0) return HAG_ERR_ARG;
    if (D > (1 << 20) || n_rows > 0x7ffffffeLL) return HAG_ERR_TOO_LARGE;
    if (is_bwd && n > 0x7fffffffLL - kSortTile) return HAG_ERR_TOO_LARGE;
    const int64_t ld_out = is_bwd ? ld_table : ld_rows, ld_in = is_bwd ? ld_rows : ld_table, n_out = is_bwd ? n_rows : n;
    if (ld_in < 0 || ld_out < 0 || (n_out > 1 && ld_out < D)) return HAG_ERR_ARG;
    if ((n > 0 && (!ids || !rows)) || (n_rows > 0 && !table && (is_bwd || n > 0))) return HAG_ERR_NULL;
    if (!hagr::element_aligned(ids, id_type == HAG_ID32 ? 4 : 8) || !hagr::element_aligned(rows, elem_size(dtype)) ||
        !hagr::element_aligned(table, elem_size(table_dtype)))
        return HAG_ERR_ALIGN;
    if (rows && rows == table) return HAG_ERR_ARG;
    return HAG_OK;
}

}  // namespace

extern "C" hag_status hag_embedding_fwd(const void *ids, hag_id_type id_type, int64_t n, int64_t n_rows, const void *table,
                                        hag_dtype table_dtype, int64_t ld_table, hag_dtype dtype, int32_t D, float scale, void *out,
                                        int64_t ld_out, void *cuda_stream) {
    const hag_status st = embed_check(ids, id_type, n, out, ld_out, dtype, n_rows, table, ld_table, table_dtype, D, false);
    if (st != HAG_OK) return st;
    if (n == 0) return HAG_OK;
    LookupArgs p{ids, id_type == HAG_ID64, int32_t(n_rows), n, table, ld_table, out, ld_out, 0, 0, scale};
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    if (table_dtype == HAG_F32)
        err = dtype == HAG_F32 ? launch_lookup_v<float, float>(p, D, s) : launch_lookup_v<float, __nv_bfloat16>(p, D, s);
    else
        err = dtype == HAG_F32 ? launch_lookup_v<__nv_bfloat16, float>(p, D, s) : launch_lookup_v<__nv_bfloat16, __nv_bfloat16>(p, D, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}

extern "C" size_t hag_embedding_bwd_workspace_bytes(int64_t n, int64_t n_rows, int32_t D) {
    if (n <= 0 || n > 0x7fffffffLL - kSortTile || n_rows < 0 || D <= 0) return 0;
    return std::max(2 * list_bytes(n) + up256(size_t(kSortMaxBlocks) * kSortBins * 4) + 2 * up256(size_t(partial_floats(n, D)) * 4),
                    size_t(tile_count(int32_t(n), int32_t(n_rows), D)) * size_t(n_rows) * ((size_t(D) + 3) / 4 * 4) * 4);
}

extern "C" hag_status hag_embedding_bwd(const void *ids, hag_id_type id_type, int64_t n, int64_t n_rows, hag_dtype dtype, int32_t D,
                                        const void *grad_out, int64_t ld_grad_out, float scale, void *grad_table,
                                        hag_dtype table_dtype, int64_t ld_grad_table, void *workspace, void *cuda_stream) {
    const hag_status st = embed_check(ids, id_type, n, grad_out, ld_grad_out, dtype, n_rows, grad_table, ld_grad_table, table_dtype, D, true);
    if (st != HAG_OK) return st;
    if (n_rows == 0) return HAG_OK;
    if (n > 0 && !workspace) return HAG_ERR_WORKSPACE;
    if (!hagl::aligned16(workspace)) return HAG_ERR_ALIGN;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    char *w = static_cast<char *>(workspace);
    const int elem = elem_size(table_dtype);
    FillArgs fill{static_cast<char *>(grad_table), int64_t(D) * elem, ld_grad_table * elem, 0, int32_t(n_rows), elem, 0};
    if (n_rows == 1) fill.ld_bytes = fill.row_bytes;
    cudaError_t err = cudaSuccess;
    if (n == 0) {
        fill.blocks = fill_blocks(fill);
        err = hagl::launch_pdl(fill_kernel, unsigned(fill.blocks), unsigned(kFillThreads), fill, s);
        if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
        return HAG_OK;
    }
    const SortPlan plan = sort_plan(int32_t(n), int32_t(n_rows));
    if (const int tiles = tile_count(int32_t(n), int32_t(n_rows), D)) {
        const SortArgs a{ids, id_type == HAG_ID64, int32_t(n_rows), nullptr, nullptr, nullptr, int32_t(n), 0, 0, plan.bits, plan.passes, 0, fill};
        const TileArgs p{a, grad_out, ld_grad_out, grad_table, ld_grad_table, D, scale, 0, static_cast<float *>(workspace), 0, 0, {}};
        if (dtype == HAG_F32)
            err = table_dtype == HAG_F32 ? launch_tiles_v<float, float>(p, tiles, s) : launch_tiles_v<float, __nv_bfloat16>(p, tiles, s);
        else
            err = table_dtype == HAG_F32 ? launch_tiles_v<__nv_bfloat16, float>(p, tiles, s) : launch_tiles_v<__nv_bfloat16, __nv_bfloat16>(p, tiles, s);
        if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
        return HAG_OK;
    }
    const size_t part = list_bytes(n);
    uint2 *list[2] = {reinterpret_cast<uint2 *>(w), reinterpret_cast<uint2 *>(w + part)};
    uint32_t *count = reinterpret_cast<uint32_t *>(w + 2 * part);
    char *partials = w + 2 * part + up256(size_t(kSortMaxBlocks) * kSortBins * 4);
    int side = 0;
    const int launches = plan.blocks == 1 ? 1 : 2 * plan.passes;
    if (!allow_shared<sort_move_kernel>(sizeof(SortShared)) || !allow_shared<sort_small_kernel>(sizeof(SortShared))) {
        cudaGetLastError();
        return HAG_ERR_CUDA;
    }
    for (int k = 0; k < launches && err == cudaSuccess; ++k) {
        const int pass = k / 2;
        fill.rows_begin = int32_t(n_rows * k / launches);
        fill.rows_end = int32_t(n_rows * (k + 1) / launches);
        fill.blocks = fill_blocks(fill);
        const SortArgs a{ids, id_type == HAG_ID64, int32_t(n_rows), pass ? list[side] : nullptr, list[side ^ 1], count, int32_t(n),
                         plan.stretch, pass * plan.bits, plan.bits, plan.passes, plan.blocks, fill};
        if (launches == 1)
            err = launch_with(sort_small_kernel, dim3(unsigned(1 + fill.blocks)), kSortThreads, sizeof(SortShared), a, s);
        else if (k % 2 == 0)
            err = launch_with(sort_count_kernel, dim3(unsigned(plan.blocks + fill.blocks)), kSortThreads, 0, a, s);
        else
            err = launch_with(sort_move_kernel, dim3(unsigned(plan.blocks + fill.blocks)), kSortThreads, sizeof(SortShared), a, s);
        if (launches == 1 || k % 2) side ^= 1;
    }
    SumArgs q{list[side], int32_t(n), int32_t(n_rows), grad_out, ld_grad_out, grad_table, ld_grad_table, D, scale, 0, 0, 0,
              reinterpret_cast<float *>(partials), reinterpret_cast<float *>(partials + up256(size_t(partial_floats(n, D)) * 4))};
    if (err == cudaSuccess) {
        if (dtype == HAG_F32)
            err = table_dtype == HAG_F32 ? launch_sum_v<float, float>(q, s) : launch_sum_v<float, __nv_bfloat16>(q, s);
        else
            err = table_dtype == HAG_F32 ? launch_sum_v<__nv_bfloat16, float>(q, s) : launch_sum_v<__nv_bfloat16, __nv_bfloat16>(q, s);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
