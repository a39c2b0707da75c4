// The gradient of the root-mean-square norm with the residual's addition.  With hh = h * rstd and q = g * w:
//   grad = rstd * (q - hh * mean(q * hh)) + what arrives along the residual stream,  gw = sum over rows of g * hh
// A row is read once and its gradient written once; gw stays with the threads over all their rows, is joined per block
// and then over the blocks, in a fixed order.  Rows of more columns than a block's registers hold are read twice, the
// second time out of the caches, and gw is kept in shared memory.
#include "hag_rms.cuh"

namespace {

using namespace hagn;

struct RmsBwdArgs {
    int64_t n;
    int32_t D;
    int32_t w_bf16, w_vectors;
    const void *g, *total, *w, *along;      // along: gradient that arrives along the residual stream
    const float *rstd;
    int64_t ld_g, ld_total, ld_along, ld_out, ld_x;
    void *out, *x;                          // x: the gradient in bf16 besides
    float *partial;                         // [parts][D]; NULL: gw is not wanted
    void *gw;
    int32_t parts;                          // blocks that leave a sum of their own
    bool joined;                            // the only block leaves gw itself
};

// A block's sum for column c of gw: a part of it, or, from the only block, the result.
__device__ __forceinline__ void leave(const RmsBwdArgs &p, int64_t c, float v) {
    if (p.parts > 1) p.partial[int64_t(blockIdx.x) * p.D + c] = v;
    else store_weight(p.gw, p.w_bf16, c, v);
}

template <typename S, int V>
__device__ __forceinline__ void store_gradient(const RmsBwdArgs &p, int64_t r, int64_t vec, const float (&o)[V]) {
    Wide<S, V> a;
    a.v.set(o);
    a.store(static_cast<S *>(p.out) + r * p.ld_out, vec);
    if constexpr (sizeof(S) == 4) {
        if (p.x) {
            Wide<__nv_bfloat16, V> b;
            b.v.set(o);
            b.store(static_cast<__nv_bfloat16 *>(p.x) + r * p.ld_x, vec);
        }
    }
}

template <int PER_LANE> constexpr int kTurnRows = PER_LANE <= 8 ? 2 : 1;

template <typename S, typename Y, int V, int L, int K>
__global__ void __launch_bounds__(L ? kWarpRowThreads : kRowThreads, L ? 2 : 1) rms_bwd_kernel(const __grid_constant__ RmsBwdArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int R = L ? kTurnRows<V * K> : 1;
    using P = Place<L, K>;
    __shared__ float slots[2][32];
    const P at;
    const int n_vec = p.D / V;
    const float inverse = 1.0f / float(p.D);
    bool mine[K];
    float w[K][V], sum[K][V];
    hagk::pdl_wait();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        mine[k] = at.first + k * P::kStep < n_vec;
#pragma unroll
        for (int j = 0; j < V; ++j) w[k][j] = sum[k][j] = 0.0f;
        if (mine[k]) load_weights<V>(w[k], p.w, p.w_bf16, p.w_vectors, int64_t(at.first + k * P::kStep) * V);
    }
    int turn = 0;
    for (int64_t lead = at.leader() * R, r0 = at.group * R; lead < p.n; lead += at.groups * R, r0 += at.groups * R, turn ^= 1) {
        Wide<Y, V> g[R][K];
        Wide<S, V> t[R][K], a[R][K];
        float rstd[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            rstd[i] = r0 + i < p.n ? __ldcg(p.rstd + r0 + i) : 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                g[i][k].v.zero();
                t[i][k].v.zero();
                a[i][k].v.zero();
                if (mine[k] && r0 + i < p.n) {
                    const int vec = at.first + k * P::kStep;
                    g[i][k].load(static_cast<const Y *>(p.g) + (r0 + i) * p.ld_g, vec);
                    t[i][k].load(static_cast<const S *>(p.total) + (r0 + i) * p.ld_total, vec);
                    if (p.along) a[i][k].load(static_cast<const S *>(p.along) + (r0 + i) * p.ld_along, vec);
                }
            }
        }
        float s[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float d = g[i][k].v.get(j) * (t[i][k].v.get(j) * rstd[i]);
                    sum[k][j] += d;
                    s[i] = fmaf(d, w[k][j], s[i]);
                }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float m = group_sum<L>(s[i], slots[turn]) * inverse;
            if (r0 + i >= p.n) continue;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float hh = t[i][k].v.get(j) * rstd[i];
                    o[j] = fmaf(rstd[i], fmaf(-hh, m, g[i][k].v.get(j) * w[k][j]), a[i][k].v.get(j));
                }
                if (mine[k]) store_gradient<S, V>(p, r0 + i, at.first + k * P::kStep, o);
            }
        }
    }
    if (!p.partial) return;
    if constexpr (L == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (mine[k]) leave(p, int64_t(at.first + k * 32) * V + j, sum[k][j]);
    } else {
        // groups of the warp, then warps of the block, in a fixed order
        constexpr int C = L * K * V, kWarps = kWarpRowThreads / 32;
        __shared__ float joined[kWarps][C];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
#pragma unroll
                for (int o = L; o < 32; o <<= 1) sum[k][j] += __shfl_xor_sync(0xffffffffu, sum[k][j], o);
                if ((threadIdx.x & 31) < L) joined[threadIdx.x >> 5][(at.first + k * L) * V + j] = sum[k][j];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < p.D; c += kWarpRowThreads) {
            float v = 0.0f;
#pragma unroll
            for (int q = 0; q < kWarps; ++q) v += joined[q][c];
            leave(p, c, v);
        }
    }
}

template <typename S, typename Y, int V>
__global__ void __launch_bounds__(kRowThreads, 1) rms_bwd_long_kernel(const __grid_constant__ RmsBwdArgs p) {
    hagk::pdl_launch_dependents();
    constexpr int K = 2;
    extern __shared__ __align__(16) float sums[];            // [D] where gw is wanted from this kernel
    __shared__ float slots[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n_vec = p.D / V, stride = (kRowThreads / 32) * 32 * K;
    if (p.partial)                                            // a thread's own columns: no barrier is needed
        for (int base = warp * 32 * K; base < n_vec; base += stride)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (base + k * 32 + lane < n_vec) sums[(base + k * 32 + lane) * V + j] = 0.0f;
    hagk::pdl_wait();
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x) {
        const Y *gr = static_cast<const Y *>(p.g) + r * p.ld_g;
        const S *tr = static_cast<const S *>(p.total) + r * p.ld_total;
        const S *ar = static_cast<const S *>(p.along) + (p.along ? r * p.ld_along : 0);
        const float rstd = __ldcg(p.rstd + r);
        float s = 0.0f;
        for (int base = warp * 32 * K; base < n_vec; base += stride) {
            Wide<Y, V> g[K];
            Wide<S, V> t[K];
            float w[K][V];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int vec = base + k * 32 + lane;
                if (vec >= n_vec) continue;
                g[k].load(gr, vec);
                t[k].load(tr, vec);
                load_weights<V>(w[k], p.w, p.w_bf16, p.w_vectors, int64_t(vec) * V);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int vec = base + k * 32 + lane;
                if (vec >= n_vec) continue;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float d = g[k].v.get(j) * (t[k].v.get(j) * rstd);
                    if (p.partial) sums[vec * V + j] += d;
                    s = fmaf(d, w[k][j], s);
                }
            }
        }
        const float m = group_sum<0>(s, slots) / float(p.D);
        for (int base = warp * 32 * K; base < n_vec; base += stride) {
            Wide<Y, V> g[K];
            Wide<S, V> t[K], a[K];
            float w[K][V];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int vec = base + k * 32 + lane;
                a[k].v.zero();
                if (vec >= n_vec) continue;
                g[k].load(gr, vec);
                t[k].load(tr, vec);
                if (p.along) a[k].load(ar, vec);
                load_weights<V>(w[k], p.w, p.w_bf16, p.w_vectors, int64_t(vec) * V);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int vec = base + k * 32 + lane;
                if (vec >= n_vec) continue;
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j)
                    o[j] = fmaf(rstd, fmaf(-(t[k].v.get(j) * rstd), m, g[k].v.get(j) * w[k][j]), a[k].v.get(j));
                store_gradient<S, V>(p, r, vec, o);
            }
        }
        __syncthreads();                                      // the slots are written again
    }
    if (!p.partial) return;
    for (int base = warp * 32 * K; base < n_vec; base += stride)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (base + k * 32 + lane < n_vec) leave(p, int64_t(base + k * 32 + lane) * V + j, sums[(base + k * 32 + lane) * V + j]);
}

// gw of one strip of 32 columns and one part of the rows, for rows whose gw does not fit in shared memory.
constexpr int kStripRows = 8;
template <typename S, typename Y>
__global__ void __launch_bounds__(32 * kStripRows) rms_weight_strips_kernel(const __grid_constant__ RmsBwdArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[kStripRows][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane, step = int64_t(gridDim.y) * kStripRows;
    float a = 0.0f;
    hagk::pdl_wait();
    if (c < p.D)
        for (int64_t r = int64_t(blockIdx.y) * kStripRows + part; r < p.n; r += step)
            a += load_one<Y>(p.g, r * p.ld_g + c) * (load_one<S>(p.total, r * p.ld_total + c) * __ldcg(p.rstd + r));
    sum[part][lane] = a;
    __syncthreads();
    if (part == 0 && c < p.D) {
        a = 0.0f;
#pragma unroll
        for (int k = 0; k < kStripRows; ++k) a += sum[k][lane];
        p.partial[int64_t(blockIdx.y) * p.D + c] = a;
    }
}

// gw from the parts: a block takes 32 columns, its 32 warps every 32nd part each.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps) rms_weight_join_kernel(const __grid_constant__ RmsBwdArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[kJoinWarps][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    hagk::pdl_wait();
    float s = 0.0f;
    if (c < p.D) {
#pragma unroll 8
        for (int q = warp; q < p.parts; q += kJoinWarps) s += __ldcg(p.partial + int64_t(q) * p.D + c);
    }
    sum[warp][lane] = s;
    __syncthreads();
    s = hagr::warp_sum(sum[lane][warp]);                      // column `warp` of this block
    const int64_t k = int64_t(blockIdx.x) * 32 + warp;
    if (lane == 0 && k < p.D) store_weight(p.gw, p.w_bf16, k, s);
}

constexpr int kMostInShared = 48 * 1024;                      // columns
constexpr int kParts = 64;                                    // of the strips
// Parts of gw, i.e. blocks of the other kernels, at most: the wider the rows, the fewer blocks fit an SM.
int most_parts(int32_t D) { return kSms * std::max(1, std::min(8, 16384 / D)); }
// Values of a gradient that one block takes alone, without a second launch.
constexpr int64_t kFewValues = 16384;

// Lets a kernel use the shared memory of the current device's SMs (once per kernel and device).
template <auto KERNEL>
cudaError_t allow_shared() {
    static std::atomic<uint64_t> ready{0};
    int device = 0;
    cudaError_t err = cudaGetDevice(&device);
    const uint64_t bit = uint64_t(1) << (device & 63);
    if (err != cudaSuccess || (ready.load(std::memory_order_relaxed) & bit)) return err;
    err = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostInShared * 4);
    if (err == cudaSuccess) ready.fetch_or(bit, std::memory_order_relaxed);
    return err;
}

template <typename S, typename Y, int V, int L, int K>
cudaError_t launch_rows(RmsBwdArgs &p, cudaStream_t s) {
    constexpr auto kernel = rms_bwd_kernel<S, Y, V, L, K>;
    constexpr int R = L ? kTurnRows<V * K> : 1;
    const unsigned threads = L ? kWarpRowThreads : unsigned((p.D / V + 32 * K - 1) / (32 * K)) * 32;
    const int64_t rows = L ? int64_t(kWarpRowThreads / 32) * (32 / (L ? L : 32)) * R : 1;
    const int64_t most = std::min(kSms * blocks_per_sm<kernel>(threads, 0), most_parts(p.D));
    int64_t grid = std::min<int64_t>((p.n + rows - 1) / rows, most);
    if (L && p.partial && p.n * p.D <= kFewValues) grid = 1;
    p.parts = int32_t(grid);
    p.joined = grid == 1;
    return launch(kernel, dim3(unsigned(grid)), threads, 0, p, s);
}

template <typename S, typename Y, int V>
cudaError_t launch_width(RmsBwdArgs &p, cudaStream_t s) {
    const int32_t n_vec = p.D / V;
    if (p.D > kMostInRegisters) {
        constexpr auto kernel = rms_bwd_long_kernel<S, Y, V>;
        const cudaError_t err = allow_shared<kernel>();
        if (err != cudaSuccess) return err;
        const unsigned grid = unsigned(std::min<int64_t>(p.n, kSms));
        if (p.partial && p.D > kMostInShared) {               // first: the gradient may take the place of what they read
            p.parts = int32_t(std::min<int64_t>((p.n + kStripRows - 1) / kStripRows, kParts));
            const cudaError_t e = launch(rms_weight_strips_kernel<S, Y>, dim3(unsigned((p.D + 31) / 32), unsigned(p.parts)), 32 * kStripRows, 0, p, s);
            if (e != cudaSuccess) return e;
            RmsBwdArgs q = p;
            q.partial = nullptr;
            return launch(kernel, dim3(grid), kRowThreads, 0, q, s);
        }
        p.parts = int32_t(grid);
        p.joined = grid == 1;
        return launch(kernel, dim3(grid), kRowThreads, p.partial ? size_t(p.D) * 4 : 0, p, s);
    }
    if (n_vec <= 4) return launch_rows<S, Y, V, 4, 1>(p, s);
    if (n_vec <= 8) return launch_rows<S, Y, V, 8, 1>(p, s);
    if (n_vec <= 16) return launch_rows<S, Y, V, 16, 1>(p, s);
    if (n_vec <= 32) return launch_rows<S, Y, V, 32, 1>(p, s);
    if (n_vec <= 64) return launch_rows<S, Y, V, 32, 2>(p, s);
    if constexpr (V < 8)
        if (n_vec <= 128) return launch_rows<S, Y, V, 32, 4>(p, s);
    if constexpr (V == 1) {
        if (n_vec <= 256) return launch_rows<S, Y, V, 32, 8>(p, s);
        if (n_vec <= 512) return launch_rows<S, Y, V, 32, 16>(p, s);
    }
    return launch_rows<S, Y, V, 0, kPerThread / V>(p, s);
}

template <typename S, typename Y, int N>
cudaError_t launch_typed(RmsBwdArgs &p, const Matrix (&m)[N], cudaStream_t s) {
    constexpr int kMost = sizeof(Y) == 2 ? 8 : 4;             // the narrowest type fills 16 bytes
    const int we = p.w_bf16 ? 2 : 4;
    if (vectors_fit(kMost, p.D, m)) {
        p.w_vectors = on(p.w, std::min(16, kMost * we));
        return launch_width<S, Y, kMost>(p, s);
    }
    if constexpr (kMost == 8)
        if (vectors_fit(4, p.D, m)) {
            p.w_vectors = on(p.w, 4 * we);
            return launch_width<S, Y, 4>(p, s);
        }
    p.w_vectors = 0;
    return launch_width<S, Y, 1>(p, s);
}

}  // namespace

extern "C" size_t hag_rms_norm_bwd_workspace_bytes(int64_t n, int32_t D) {
    if (n < 0 || D <= 0) return 0;
    return size_t(std::max<int64_t>(std::min<int64_t>(most_parts(D), n), 1)) * size_t(D) * 4;
}

extern "C" hag_status hag_rms_norm_bwd(int64_t n, int32_t D, const void *grad_y, hag_dtype y_dtype, int64_t ld_grad_y,
                                       const void *total, hag_dtype stream_dtype, int64_t ld_total, const float *rstd,
                                       const void *weight, hag_dtype weight_dtype, const void *grad_total, int64_t ld_grad_total,
                                       void *grad_residual, int64_t ld_grad_residual, void *grad_x, int64_t ld_grad_x,
                                       void *grad_weight, void *workspace, void *cuda_stream) {
    if (!dtype_ok(y_dtype) || !dtype_ok(stream_dtype) || !dtype_ok(weight_dtype)) return HAG_ERR_DTYPE;
    if (y_dtype != stream_dtype && stream_dtype != HAG_F32) return HAG_ERR_DTYPE;
    if (grad_x && stream_dtype != HAG_F32) return HAG_ERR_DTYPE;
    const int se = size_of(stream_dtype);
    const Matrix m[] = {{grad_y, ld_grad_y, size_of(y_dtype), false, true}, {total, ld_total, se, false, true},
                        {grad_total, ld_grad_total, se, false, false}, {grad_residual, ld_grad_residual, se, true, true},
                        {grad_x, ld_grad_x, 2, true, false}};
    const hag_status st = check(n, D, weight, weight_dtype, rstd, m);
    if (st != HAG_OK) return st;
    if (n > 0 && !rstd) return HAG_ERR_NULL;
    if (!on(grad_weight, size_of(weight_dtype))) return HAG_ERR_ALIGN;
    if (grad_weight && !workspace) return HAG_ERR_WORKSPACE;
    if (!hagl::aligned16(workspace)) return HAG_ERR_ALIGN;
    RmsBwdArgs p{};
    p.n = n; p.D = D; p.w_bf16 = weight_dtype == HAG_BF16; p.w = weight; p.rstd = rstd;
    p.g = grad_y; p.ld_g = ld_grad_y; p.total = total; p.ld_total = ld_total; p.along = grad_total; p.ld_along = ld_grad_total;
    p.out = grad_residual; p.ld_out = ld_grad_residual; p.x = grad_x; p.ld_x = ld_grad_x;
    p.partial = grad_weight ? static_cast<float *>(workspace) : nullptr;
    p.gw = grad_weight;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err = cudaSuccess;
    if (n > 0) {
        if (y_dtype != stream_dtype) err = launch_typed<float, __nv_bfloat16>(p, m, s);
        else if (y_dtype == HAG_BF16) err = launch_typed<__nv_bfloat16, __nv_bfloat16>(p, m, s);
        else err = launch_typed<float, float>(p, m, s);
    }
    if (err == cudaSuccess && grad_weight && !p.joined)            // no rows: the sum of no parts
        err = launch(rms_weight_join_kernel, dim3(unsigned((int64_t(D) + 31) / 32)), 32 * kJoinWarps, 0, p, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
