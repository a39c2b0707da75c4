// Embedding: rows of a table selected by ids and scaled, and the gradient of the table.
//   forward   out_i = scale * T[id_i]
//   backward  gT_v  = scale * sum over i with id_i = v of g_i
// An id outside 0..V-1 stands for no token: its row is zero and it takes no part in the gradient.
//
// The gradient adds in a fixed order: the ids are sorted (stable radix sort, 8 bits at a time at most, integer
// counters only), so that the tokens of a row lie side by side in ascending order, and each row is a sum over one
// stretch of them.  No atomics on floats: the same inputs give the same bits.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "hag.h"
#include "hag_kernels.cuh"
#include "hag_launch.h"
#include "hag_rows.cuh"

namespace {

constexpr int kCopyThreads = 256;
constexpr int kCopyUnroll = 4;

struct LookupArgs {
    const void *ids;
    int32_t ids64;
    int32_t n_rows;          // V
    const void *table;
    int64_t ld_table;
    void *out;
    int64_t ld_out;
    int64_t items;           // n * vectors per row
    float scale;
    hagr::Divisor per_row;   // vectors per row
};

__device__ __forceinline__ int64_t load_id(const void *ids, int ids64, int64_t i) {
    return ids64 ? __ldcg(static_cast<const long long *>(ids) + i) : int64_t(__ldcg(static_cast<const int *>(ids) + i));
}

// One vector per thread and step over the flat list of all output vectors, so that any mix of few wide or many
// narrow rows fills the machine; the row of a vector comes from a multiply-high quotient.
template <typename TT, typename TO, int V>
__global__ void __launch_bounds__(kCopyThreads) embedding_fwd_kernel(const LookupArgs p) {
    hagk::pdl_launch_dependents();
    const int64_t first = int64_t(blockIdx.x) * (kCopyThreads * kCopyUnroll);
    const int64_t row0 = first < (int64_t(1) << 31) ? int64_t(hagr::quotient(uint32_t(first), p.per_row)) : first / p.per_row.d;
    const uint32_t col0 = uint32_t(first - row0 * p.per_row.d);
    int64_t row[kCopyUnroll], id[kCopyUnroll];
    uint32_t col[kCopyUnroll];
    hagk::pdl_wait();
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
        const uint32_t k = u * kCopyThreads + threadIdx.x;
        const uint32_t r = hagr::quotient(col0 + k, p.per_row);
        row[u] = row0 + r;
        col[u] = col0 + k - r * p.per_row.d;
        id[u] = first + k < p.items ? load_id(p.ids, p.ids64, row[u]) : -1;
    }
    hagr::Vec<TT, V> in[kCopyUnroll];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
        in[u].zero();
        if (uint64_t(id[u]) < uint64_t(p.n_rows))
            in[u].template load<hagr::kKeep>(static_cast<const TT *>(p.table) + id[u] * p.ld_table, col[u]);
    }
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
        if (first + u * kCopyThreads + threadIdx.x >= p.items) continue;
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = uint64_t(id[u]) < uint64_t(p.n_rows) ? in[u].get(j) * p.scale : 0.0f;
        hagr::Vec<TO, V> o;
        o.set(v);
        o.store(static_cast<TO *>(p.out) + row[u] * p.ld_out, col[u]);
    }
}

template <typename TT, typename TO, int V>
cudaError_t launch_lookup(LookupArgs &p, int64_t n, int32_t D, cudaStream_t s) {
    p.per_row = hagr::make_divisor(uint32_t(D / V));
    p.items = n * (D / V);
    const int64_t blocks = (p.items + kCopyThreads * kCopyUnroll - 1) / (kCopyThreads * kCopyUnroll);
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    return hagl::launch_pdl(embedding_fwd_kernel<TT, TO, V>, unsigned(blocks), unsigned(kCopyThreads), p, s);
}

template <typename TT, typename TO>
cudaError_t launch_lookup_v(LookupArgs &p, int64_t n, int32_t D, cudaStream_t s) {
    constexpr int kMost = sizeof(TT) == 4 && sizeof(TO) == 4 ? 4 : 8;      // 16 bytes of the narrower type
    const hagr::Operand ops[] = {{p.table, p.ld_table, int(sizeof(TT))}, {p.out, p.ld_out, int(sizeof(TO))}};
    switch (hagr::vector_elems(kMost, D, ops)) {
        case 8: if constexpr (kMost == 8) return launch_lookup<TT, TO, 8>(p, n, D, s);
        case 4: return launch_lookup<TT, TO, 4>(p, n, D, s);
        case 2: return launch_lookup<TT, TO, 2>(p, n, D, s);
        default: return launch_lookup<TT, TO, 1>(p, n, D, s);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Stable radix sort of (key, place) by key; key = the id, or V for a place without a token (those come last).
// Each pass: every block counts the digits of its own stretch of the list (sort_count_kernel); then every block
// adds up the counts before it, and moves its stretch to the places found (sort_move_kernel).
constexpr int kSortThreads = 256;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 16;                                // keys per thread and tile
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kSortBins = 256;
constexpr int kSortMaxBlocks = 296;                           // two per SM

struct SortArgs {
    const void *ids;         // first pass: the caller's ids
    int32_t ids64;
    int32_t n_rows;          // V
    const uint32_t *key_in, *place_in;       // later passes
    uint32_t *key_out, *place_out;
    uint32_t *count;         // [blocks][bins]
    int32_t n;
    int32_t stretch;         // keys per block, a multiple of the tile
    int32_t shift, bits;
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs &p, int32_t i) {
    if (p.key_in) return __ldcg(p.key_in + i);
    const int64_t id = load_id(p.ids, p.ids64, i);
    return uint64_t(id) < uint64_t(p.n_rows) ? uint32_t(id) : uint32_t(p.n_rows);
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ uint32_t bin[kSortBins];
    bin[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t mask = (1u << p.bits) - 1u;
    const int32_t begin = blockIdx.x * p.stretch, end = int32_t(min(int64_t(p.n), int64_t(begin) + p.stretch));
    hagk::pdl_wait();
    for (int32_t i = begin + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&bin[(sort_key(p, i) >> p.shift) & mask], 1u);
    __syncthreads();
    p.count[blockIdx.x * kSortBins + threadIdx.x] = bin[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads) sort_move_kernel(const SortArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ uint32_t base[kSortBins];                      // next place of each digit for this block
    __shared__ uint32_t seen[kSortWarps][kSortBins];          // per warp: keys of the digit so far in this tile
    __shared__ uint32_t scan[kSortWarps];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const uint32_t mask = (1u << p.bits) - 1u;
    hagk::pdl_wait();
    {   // base[d] = keys with a smaller digit + keys of digit d in the blocks before this one
        uint32_t before = 0, total = 0;
        for (int b = 0; b < int(gridDim.x); ++b) {
            const uint32_t c = __ldcg(p.count + b * kSortBins + t);
            if (b < int(blockIdx.x)) before += c;
            total += c;
        }
        uint32_t x = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) scan[warp] = x;
        __syncthreads();
        uint32_t lower = 0;
        for (int w = 0; w < warp; ++w) lower += scan[w];
        base[t] = lower + x - total + before;
    }
    const int32_t begin = blockIdx.x * p.stretch, end = int32_t(min(int64_t(p.n), int64_t(begin) + p.stretch));
    for (int32_t tile = begin; tile < end; tile += kSortTile) {
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) seen[w][t] = 0;
        __syncthreads();
        uint32_t key[kSortItems], rank[kSortItems];
        const int32_t mine = tile + warp * (32 * kSortItems) + lane;      // a warp's keys are consecutive: stable
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) key[k] = mine + 32 * k < end ? sort_key(p, mine + 32 * k) : 0xffffffffu;
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const bool live = mine + 32 * k < end;
            const uint32_t digit = (key[k] >> p.shift) & mask;
            const uint32_t same = __match_any_sync(0xffffffffu, live ? digit : 0xffffffffu);
            const uint32_t old = live ? seen[warp][digit] : 0;
            rank[k] = old + __popc(same & ((1u << lane) - 1u));
            __syncwarp();
            if (live && (same >> lane) == 1u) seen[warp][digit] = old + __popc(same);      // the highest lane of the digit
            __syncwarp();
        }
        __syncthreads();
        {   // per digit: the counts of the warps become their first places; base moves on
            uint32_t at = base[t];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = seen[w][t];
                seen[w][t] = at;
                at += c;
            }
            base[t] = at;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const int32_t i = mine + 32 * k;
            if (i >= end) continue;
            const uint32_t to = seen[warp][(key[k] >> p.shift) & mask] + rank[k];
            p.key_out[to] = key[k];
            p.place_out[to] = p.place_in ? __ldcg(p.place_in + i) : uint32_t(i);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------
struct SumArgs {
    const uint32_t *key, *place;     // sorted
    int32_t n;
    int32_t n_rows;                  // V
    const void *grad;
    int64_t ld_grad;
    void *out;
    int64_t ld_out;
    int32_t D;
    float scale;
};

__device__ __forceinline__ int32_t lower_bound(const uint32_t *key, int32_t n, uint32_t v) {
    int32_t lo = 0, hi = n;
    while (lo < hi) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (__ldcg(key + mid) < v) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// One warp per row of the table.
template <typename TG, typename TO, int V>
__global__ void __launch_bounds__(hagk::kThreads) embedding_sum_kernel(const SumArgs p) {
    hagk::pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int64_t row = int64_t(blockIdx.x) * hagk::kWarps + (threadIdx.x >> 5);
    hagk::pdl_wait();
    if (row >= p.n_rows) return;
    const int32_t b = lower_bound(p.key, p.n, uint32_t(row)), e = lower_bound(p.key, p.n, uint32_t(row) + 1u);
    const int n_vec = p.D / V;
    for (int c = lane; c < n_vec; c += 32) {
        float acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.0f;
        for (int32_t i = b; i < e; ++i) {
            hagr::Vec<TG, V> g;
            g.template load<hagr::kOnce>(static_cast<const TG *>(p.grad) + int64_t(__ldcg(p.place + i)) * p.ld_grad, c);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += g.get(j);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] *= p.scale;
        hagr::Vec<TO, V> o;
        o.set(acc);
        o.store(static_cast<TO *>(p.out) + row * p.ld_out, c);
    }
}

template <typename TG, typename TO, int V>
cudaError_t launch_sum(const SumArgs &p, cudaStream_t s) {
    const int64_t blocks = (int64_t(p.n_rows) + hagk::kWarps - 1) / hagk::kWarps;
    return hagl::launch_pdl(embedding_sum_kernel<TG, TO, V>, unsigned(blocks), unsigned(hagk::kThreads), p, s);
}

template <typename TG, typename TO>
cudaError_t launch_sum_v(const SumArgs &p, cudaStream_t s) {
    constexpr int kMost = sizeof(TG) == 4 && sizeof(TO) == 4 ? 4 : 8;
    const hagr::Operand ops[] = {{p.grad, p.ld_grad, int(sizeof(TG))}, {p.out, p.ld_out, int(sizeof(TO))}};
    switch (hagr::vector_elems(kMost, p.D, ops)) {
        case 8: if constexpr (kMost == 8) return launch_sum<TG, TO, 8>(p, s);
        case 4: return launch_sum<TG, TO, 4>(p, s);
        case 2: return launch_sum<TG, TO, 2>(p, s);
        default: return launch_sum<TG, TO, 1>(p, s);
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
    const int64_t tiles = (int64_t(n) + kSortTile - 1) / kSortTile;
    const int64_t per_block = (tiles + kSortMaxBlocks - 1) / kSortMaxBlocks;
    s.blocks = int((tiles + per_block - 1) / std::max<int64_t>(per_block, 1));
    s.stretch = int32_t(std::min<int64_t>(per_block * kSortTile, 0x7fffffff));
    const int total = key_bits(n_rows);
    s.passes = (total + 7) / 8;
    s.bits = (total + s.passes - 1) / s.passes;
    return s;
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

bool dtype_ok(hag_dtype d) { return d == HAG_F32 || d == HAG_BF16; }
int elem_size(hag_dtype d) { return d == HAG_F32 ? 4 : 2; }

hag_status embed_check(const void *ids, hag_id_type id_type, int64_t n, const void *rows, int64_t ld_rows, hag_dtype dtype,
                       int64_t n_rows, const void *table, int64_t ld_table, hag_dtype table_dtype, int32_t D, bool is_bwd) {
    if (!dtype_ok(dtype) || !dtype_ok(table_dtype)) return HAG_ERR_DTYPE;
    if (id_type != HAG_ID32 && id_type != HAG_ID64) return HAG_ERR_DTYPE;
    if (D <= 0 || n < 0 || n_rows < 0) return HAG_ERR_ARG;
    if (D > (1 << 30) || n_rows > 0x7ffffffeLL) return HAG_ERR_TOO_LARGE;
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
    LookupArgs p{ids, id_type == HAG_ID64, int32_t(n_rows), table, ld_table, out, ld_out, 0, scale, {}};
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    if (table_dtype == HAG_F32)
        err = dtype == HAG_F32 ? launch_lookup_v<float, float>(p, n, D, s) : launch_lookup_v<float, __nv_bfloat16>(p, n, D, s);
    else
        err = dtype == HAG_F32 ? launch_lookup_v<__nv_bfloat16, float>(p, n, D, s) : launch_lookup_v<__nv_bfloat16, __nv_bfloat16>(p, n, D, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}

extern "C" size_t hag_embedding_bwd_workspace_bytes(int64_t n, int64_t n_rows, int32_t D) {
    if (n <= 0 || n > 0x7fffffffLL - kSortTile || n_rows < 0 || D <= 0) return 0;
    return 4 * up256(size_t(n) * 4) + up256(size_t(kSortMaxBlocks) * kSortBins * 4);
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
    const size_t part = up256(size_t(n) * 4);
    uint32_t *key[2] = {reinterpret_cast<uint32_t *>(w), reinterpret_cast<uint32_t *>(w + part)};
    uint32_t *place[2] = {reinterpret_cast<uint32_t *>(w + 2 * part), reinterpret_cast<uint32_t *>(w + 3 * part)};
    uint32_t *count = reinterpret_cast<uint32_t *>(w + 4 * part);
    cudaError_t err = cudaSuccess;
    int side = 0;
    if (n > 0) {
        const SortPlan plan = sort_plan(int32_t(n), int32_t(n_rows));
        for (int pass = 0; pass < plan.passes && err == cudaSuccess; ++pass) {
            SortArgs a{ids, id_type == HAG_ID64, int32_t(n_rows), pass ? key[side] : nullptr, pass ? place[side] : nullptr,
                       key[side ^ 1], place[side ^ 1], count, int32_t(n), plan.stretch, pass * plan.bits, plan.bits};
            err = hagl::launch_pdl(sort_count_kernel, unsigned(plan.blocks), unsigned(kSortThreads), a, s);
            if (err == cudaSuccess) err = hagl::launch_pdl(sort_move_kernel, unsigned(plan.blocks), unsigned(kSortThreads), a, s);
            side ^= 1;
        }
    }
    SumArgs q{key[side], place[side], int32_t(n), int32_t(n_rows), grad_out, ld_grad_out, grad_table, ld_grad_table, D, scale};
    if (err == cudaSuccess) {
        if (dtype == HAG_F32)
            err = table_dtype == HAG_F32 ? launch_sum_v<float, float>(q, s) : launch_sum_v<float, __nv_bfloat16>(q, s);
        else
            err = table_dtype == HAG_F32 ? launch_sum_v<__nv_bfloat16, float>(q, s) : launch_sum_v<__nv_bfloat16, __nv_bfloat16>(q, s);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
