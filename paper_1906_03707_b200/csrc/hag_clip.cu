// The global norm of a list of tensors, and the list scaled so that its norm does not exceed a limit.
//   N = sqrt(sum over all tensors and elements of g^2),  c = min(1, max_norm / (N + 1e-6)),  out_t = c * g_t
// Two launches: every block sums the squares of its pieces of the list; then every block adds up those sums (the
// same order everywhere: the same bits everywhere) and scales its pieces.  The list travels as a kernel parameter,
// so no descriptor is copied to the device first and the calls can be captured in a graph.
//
// Bound by memory: the list is read twice and written once, but for what is still in the L2 the second time.  Measured
// on B200: 40 tensors of 664 MB 322 us (6.2 TB/s over the three), 20 tensors of 80 MB 40 us, 12 tensors of 0.2 MB in one
// launch 6.7 us.  Pointers off 16 bytes are read an element at a time: 40 tensors of 400 MB fp32 382 us (aligned 202), bf16
// 636 (203).
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "hag.h"
#include "hag_kernels.cuh"
#include "hag_launch.h"
#include "hag_rows.cuh"

namespace {

constexpr int kClipThreads = 256;
constexpr int kClipList = 128;                 // tensors per launch: the list must fit in 4 KB of parameters
constexpr int kClipBlocks = 148 * 4;
// A piece of a tensor: U 16-byte loads per thread, all in flight together.  Long lists take 32 KB pieces (40 tensors of
// 664 MB: 322 us, with 16 KB pieces 347); short ones 8 KB, which more SMs share.
constexpr int kLoadsLong = 8, kLoadsShort = 2;
constexpr int64_t kShortList = 8 << 20;        // bytes
// A list for one cluster: 0.2 MB takes 6.7 us and one launch of 2.7 us on the host, by two launches 6.2 us and 5.4; 0.4 MB
// 10.4 us by the cluster, 7 by two launches.  Many small tensors share its eight blocks: on the device 24 take 8.0 us (by two
// launches 6.7), 64 15.5 (9.6); but whole calls, which wait for the host, take 27.7 (30.1) and 50.6 us (52.9), of 128
// tensors 89 (91).
constexpr int64_t kClusterList = 256 << 10;
__host__ __device__ constexpr int piece_bytes(int loads) { return kClipThreads * 16 * loads; }

struct ClipArgs {
    int32_t tensors;
    uint32_t pieces;                           // of this launch's tensors
    double *sums;                              // [launches][kClipBlocks]
    int32_t first_sum, n_sums;                 // where this launch's blocks put theirs; how many there are in all
    float max_norm;
    int32_t scales;                            // clip_cluster_kernel: whether there are outputs
    float *norm;
    const void *in[kClipList];
    void *out[kClipList];
    int64_t len[kClipList];
    uint32_t first_piece[kClipList];
    uint8_t bf16[kClipList];
    uint8_t vec[kClipList];                    // both pointers on 16 bytes
};
static_assert(sizeof(ClipArgs) <= 4096, "the list must fit in the parameters of a launch");

__device__ __forceinline__ double block_sum(double v, double *slot) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kClipThreads / 32; ++w) s += slot[w];
    return s;
}

// Calls f(tensor, first element, end element) for the pieces of this block, from the first to the last or the other way.
template <int U, bool DOWN, typename F>
__device__ __forceinline__ void for_pieces(const ClipArgs &p, F f) {
    if (blockIdx.x >= p.pieces) return;
    int t = DOWN ? p.tensors - 1 : 0;
    const uint32_t turns = (p.pieces - 1 - blockIdx.x) / gridDim.x + 1;
    for (uint32_t i = 0; i < turns; ++i) {
        const uint32_t k = blockIdx.x + (DOWN ? turns - 1 - i : i) * gridDim.x;
        if (DOWN) {
            while (p.first_piece[t] > k) --t;
        } else {
            while (t + 1 < p.tensors && p.first_piece[t + 1] <= k) ++t;
        }
        const int64_t per = piece_bytes(U) / (p.bf16[t] ? 2 : 4), b = int64_t(k - p.first_piece[t]) * per;
        f(t, b, min(p.len[t], b + per));
    }
}

// f(vector, its number) for the vectors of a piece that this thread takes, eight or U of them at a time: all are
// read before the first is used.
template <typename T, int V, int U, hagr::CacheOp OP, typename F>
__device__ __forceinline__ void piece_vectors(const char *at, int32_t len, F f) {
    constexpr int N = piece_bytes(U) / (kClipThreads * V * int(sizeof(T))), B = N < 8 ? N : 8;
    const int32_t full = len / V;
#pragma unroll 1
    for (int u0 = 0; u0 < N && u0 * kClipThreads < full; u0 += B) {
        hagr::Vec<T, V> v[B];
        const bool whole = (u0 + B) * kClipThreads <= full;
#pragma unroll
        for (int u = 0; u < B; ++u) {
            const int32_t i = (u0 + u) * kClipThreads + int32_t(threadIdx.x);
            if (!whole) v[u].zero();
            if (whole || i < full) v[u].template load<OP>(at, i);
        }
#pragma unroll
        for (int u = 0; u < B; ++u) {
            const int32_t i = (u0 + u) * kClipThreads + int32_t(threadIdx.x);
            if (whole || i < full) f(v[u], i);
        }
    }
}

template <typename T, int V, int U>
__device__ __forceinline__ float piece_squares(const void *in, int64_t b, int64_t e) {
    const char *at = static_cast<const char *>(in) + b * sizeof(T);
    const int32_t len = int32_t(e - b), done = len / V * V;
    float2 s0 = make_float2(0.0f, 0.0f), s1 = s0;
    piece_vectors<T, V, U, hagr::kKeep>(at, len, [&](const hagr::Vec<T, V> &v, int32_t) {
        if constexpr (V == 1) {
            s0.x += v.get(0) * v.get(0);
        } else {
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const float2 p = make_float2(v.get(j), v.get(j + 1)), q = make_float2(v.get(j + 2), v.get(j + 3));
                s0 = __ffma2_rn(p, p, s0);
                s1 = __ffma2_rn(q, q, s1);
            }
        }
    });
    if (V > 1 && int32_t(threadIdx.x) < len - done) {
        hagr::Vec<T, 1> v;
        v.template load<hagr::kKeep>(at, done + threadIdx.x);
        s0.x += v.get(0) * v.get(0);
    }
    return (s0.x + s0.y) + (s1.x + s1.y);
}

template <typename T, int V, int U>
__device__ __forceinline__ void piece_scale(const void *in, void *out, int64_t b, int64_t e, float c) {
    const char *at = static_cast<const char *>(in) + b * sizeof(T);
    char *to = static_cast<char *>(out) + b * sizeof(T);
    const int32_t len = int32_t(e - b), done = len / V * V;
    piece_vectors<T, V, U, hagr::kOnce>(at, len, [&](const hagr::Vec<T, V> &v, int32_t i) {
        float f[V];
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = v.get(j) * c;
        hagr::Vec<T, V> o;
        o.set(f);
        o.template store<hagr::kOnce>(to, i);
    });
    if (V > 1 && int32_t(threadIdx.x) < len - done) {
        hagr::Vec<T, 1> v;
        v.template load<hagr::kOnce>(at, done + threadIdx.x);
        const float f = v.get(0) * c;
        v.set(&f);
        v.store(to, done + threadIdx.x);
    }
}

// Squares are added in fp32 within a piece, in fp64 from piece to piece.
template <int U>
__device__ __forceinline__ double piece_sums(const ClipArgs &p) {
    double s = 0.0;
    for_pieces<U, false>(p, [&](int t, int64_t b, int64_t e) {
        if (p.bf16[t])
            s += p.vec[t] ? piece_squares<__nv_bfloat16, 8, U>(p.in[t], b, e) : piece_squares<__nv_bfloat16, 1, U>(p.in[t], b, e);
        else
            s += p.vec[t] ? piece_squares<float, 4, U>(p.in[t], b, e) : piece_squares<float, 1, U>(p.in[t], b, e);
    });
    return s;
}

template <int U>
__global__ void __launch_bounds__(kClipThreads, 2) norm_sums_kernel(const __grid_constant__ ClipArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ double slot[kClipThreads / 32];
    hagk::pdl_wait();
    double s = piece_sums<U>(p);
    s = block_sum(s, slot);
    if (threadIdx.x == 0) p.sums[p.first_sum + blockIdx.x] = s;
}

// The norm from the blocks' sums; called by whole blocks.
__device__ __forceinline__ float total_norm(const ClipArgs &p, double *slot) {
    double s = 0.0;
    for (int i = threadIdx.x; i < p.n_sums; i += kClipThreads) s += __ldcg(p.sums + i);
    return float(sqrt(block_sum(s, slot)));
}

__global__ void __launch_bounds__(kClipThreads) norm_join_kernel(const __grid_constant__ ClipArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ double slot[kClipThreads / 32];
    hagk::pdl_wait();
    const float norm = total_norm(p, slot);
    if (threadIdx.x == 0 && p.norm) *p.norm = norm;
}

// The pieces of this block times the factor.
template <int U>
__device__ __forceinline__ void scale_pieces(const ClipArgs &p, float norm) {
    const float ratio = p.max_norm / (norm + 1e-6f);
    const float c = ratio >= 1.0f ? 1.0f : ratio;          // a norm that is no number gives a factor that is none
    // backwards: what the first launch read last is still in the L2
    for_pieces<U, true>(p, [&](int t, int64_t b, int64_t e) {
        if (c == 1.0f && p.in[t] == p.out[t]) return;      // in place and nothing to change
        if (p.bf16[t]) {
            if (p.vec[t]) piece_scale<__nv_bfloat16, 8, U>(p.in[t], p.out[t], b, e, c);
            else piece_scale<__nv_bfloat16, 1, U>(p.in[t], p.out[t], b, e, c);
        } else {
            if (p.vec[t]) piece_scale<float, 4, U>(p.in[t], p.out[t], b, e, c);
            else piece_scale<float, 1, U>(p.in[t], p.out[t], b, e, c);
        }
    });
}

template <int U>
__global__ void __launch_bounds__(kClipThreads, 2) clip_scale_kernel(const __grid_constant__ ClipArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ double slot[kClipThreads / 32];
    hagk::pdl_wait();
    const float norm = total_norm(p, slot);
    if (p.norm && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = norm;
    scale_pieces<U>(p, norm);
}

// Short lists in one launch: a cluster of blocks exchanges its sums through shared memory.  Its barrier is the
// hardware's, so nothing waits in a loop.
constexpr int kCluster = 8;
__global__ void __launch_bounds__(kClipThreads, 2) __cluster_dims__(kCluster, 1, 1) clip_cluster_kernel(const __grid_constant__ ClipArgs p) {
    hagk::pdl_launch_dependents();
    namespace cg = cooperative_groups;
    __shared__ double slot[kClipThreads / 32], mine;
    cg::cluster_group cluster = cg::this_cluster();
    hagk::pdl_wait();
    double s = piece_sums<kLoadsLong>(p);
    s = block_sum(s, slot);
    if (threadIdx.x == 0) mine = s;
    cluster.sync();
    s = 0.0;
#pragma unroll
    for (unsigned b = 0; b < kCluster; ++b) s += *cluster.map_shared_rank(&mine, b);
    cluster.sync();                                        // no block leaves while another reads its sum
    const float norm = float(sqrt(s));
    if (p.norm && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = norm;
    if (p.scales) scale_pieces<kLoadsLong>(p, norm);
}

constexpr int32_t kClipMost = 1 << 28;         // tensors of a call: the number of their blocks' sums fits in 31 bits
int launches_of(int32_t count) { return std::max(1, (count + kClipList - 1) / kClipList); }

// The part of the list that launch `k` handles; false: it has more pieces than a launch can count.
bool fill(ClipArgs &p, int k, int loads, int32_t count, const void *const *in, void *const *out, const int64_t *len, const hag_dtype *dtype) {
    p.tensors = 0;
    int64_t pieces = 0;
    for (int32_t t = k * kClipList; t < std::min(count, (k + 1) * kClipList); ++t) {
        if (len[t] == 0) continue;
        const int64_t per = piece_bytes(loads) / (dtype[t] == HAG_BF16 ? 2 : 4), here = len[t] / per + (len[t] % per != 0);
        if (pieces + here > 0x7fffffffLL) return false;
        const int i = p.tensors++;
        p.in[i] = in[t];
        p.out[i] = out ? out[t] : nullptr;
        p.len[i] = len[t];
        p.first_piece[i] = uint32_t(pieces);
        p.bf16[i] = dtype[t] == HAG_BF16;
        p.vec[i] = hagl::aligned16(in[t]) && (!out || hagl::aligned16(out[t]));
        pieces += here;
    }
    p.pieces = uint32_t(pieces);
    return true;
}

}  // namespace

extern "C" size_t hag_clip_grad_norm_workspace_bytes(int32_t count) {
    return count < 0 || count > kClipMost ? 0 : size_t(launches_of(count)) * kClipBlocks * sizeof(double);
}

extern "C" hag_status hag_clip_grad_norm(int32_t count, const void *const *grads, void *const *out, const int64_t *lengths,
                                         const hag_dtype *dtypes, float max_norm, float *total_norm, void *workspace,
                                         void *cuda_stream) {
    if (count < 0 || !(max_norm >= 0.0f)) return HAG_ERR_ARG;
    if (count > 0 && (!grads || !lengths || !dtypes)) return HAG_ERR_NULL;
    if (!out && !total_norm) return HAG_ERR_NULL;
    if (count > kClipMost) return HAG_ERR_TOO_LARGE;
    int64_t bytes = 0;
    for (int32_t t = 0; t < count; ++t) {
        if (dtypes[t] != HAG_F32 && dtypes[t] != HAG_BF16) return HAG_ERR_DTYPE;
        if (lengths[t] < 0) return HAG_ERR_ARG;
        if (lengths[t] == 0) continue;
        if (lengths[t] < kShortList) bytes += lengths[t] * (dtypes[t] == HAG_F32 ? 4 : 2);
        else bytes = kShortList;
        bytes = std::min(bytes, kShortList);
        if (!grads[t] || (out && !out[t])) return HAG_ERR_NULL;
        const int elem = dtypes[t] == HAG_F32 ? 4 : 2;
        if (!hagr::element_aligned(grads[t], elem) || (out && !hagr::element_aligned(out[t], elem))) return HAG_ERR_ALIGN;
    }
    if (!hagr::element_aligned(total_norm, 4)) return HAG_ERR_ALIGN;
    if (!workspace) return HAG_ERR_WORKSPACE;
    if (!hagl::aligned16(workspace)) return HAG_ERR_ALIGN;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const int launches = launches_of(count);
    const bool cluster = launches == 1 && bytes <= kClusterList;
    const int loads = bytes < kShortList && !cluster ? kLoadsShort : kLoadsLong;
    void (*const sum)(ClipArgs) = loads == kLoadsShort ? norm_sums_kernel<kLoadsShort> : norm_sums_kernel<kLoadsLong>;
    void (*const scale)(ClipArgs) = loads == kLoadsShort ? clip_scale_kernel<kLoadsShort> : clip_scale_kernel<kLoadsLong>;
    ClipArgs p{};
    p.sums = static_cast<double *>(workspace);
    p.max_norm = max_norm;
    for (int k = 0; k < launches; ++k)      // before the first launch: an error leaves everything as it was
        if (!fill(p, k, loads, count, grads, out, lengths, dtypes)) return HAG_ERR_TOO_LARGE;
    cudaError_t err = cudaSuccess;
    if (cluster) {
        p.norm = total_norm;
        p.scales = out != nullptr;
        err = hagl::launch_pdl<ClipArgs>(clip_cluster_kernel, unsigned(kCluster), unsigned(kClipThreads), p, s);
        if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
        return HAG_OK;
    }
    int32_t sums = 0;
    for (int k = 0; k < launches && err == cudaSuccess; ++k) {
        if (launches > 1) fill(p, k, loads, count, grads, out, lengths, dtypes);
        const unsigned grid = unsigned(std::min<int64_t>(std::max<uint32_t>(p.pieces, 1), kClipBlocks));
        p.first_sum = sums;
        sums += int32_t(grid);
        err = hagl::launch_pdl<ClipArgs>(sum, grid, unsigned(kClipThreads), p, s);
    }
    p.n_sums = sums;
    if (err == cudaSuccess && !out) {
        p.norm = total_norm;
        err = hagl::launch_pdl<ClipArgs>(norm_join_kernel, 1u, unsigned(kClipThreads), p, s);
    }
    for (int k = 0; out && k < launches && err == cudaSuccess; ++k) {
        if (launches > 1) fill(p, k, loads, count, grads, out, lengths, dtypes);
        p.norm = k == 0 ? total_norm : nullptr;
        const unsigned grid = unsigned(std::min<int64_t>(std::max<uint32_t>(p.pieces, 1), kClipBlocks));
        err = hagl::launch_pdl<ClipArgs>(scale, grid, unsigned(kClipThreads), p, s);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
