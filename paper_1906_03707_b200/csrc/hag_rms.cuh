// What the forward and backward kernels of the root-mean-square norm share.
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "hag.h"
#include "hag_kernels.cuh"
#include "hag_launch.h"
#include "hag_rows.cuh"

namespace hagn {

constexpr int kSms = 148;
constexpr int kWarpRowThreads = 256;      // of a block whose warps take rows of their own
constexpr int kRowThreads = 512;          // at most, of a block that takes a row
constexpr int kWideThreads = 1024;        // of one that takes a row of more than 8192 columns
constexpr int kPerThread = 16;            // columns of a row per thread of such blocks
constexpr int kMostInRegisters = kWideThreads * kPerThread;        // columns

// A vector of V elements, by one access of up to 32 bytes.
template <typename T, int V>
struct Wide {
    hagr::Vec<T, V> v;
    __device__ __forceinline__ void load(const void *row, int64_t i) {
        if constexpr (V * sizeof(T) == 32) {
            uint32_t *w = v.raw.w;
            asm volatile("ld.global.cg.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                         : "l"(static_cast<const char *>(row) + i * 32)
                         : "memory");
        } else {
            v.template load<hagr::kKeep>(row, size_t(i));
        }
    }
    __device__ __forceinline__ void store(void *row, int64_t i) const {
        if constexpr (V * sizeof(T) == 32) {
            const uint32_t *w = v.raw.w;
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<char *>(row) + i * 32), "r"(w[0]),
                         "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                         : "memory");
        } else {
            v.store(row, size_t(i));
        }
    }
};

template <typename T>
__device__ __forceinline__ float load_one(const void *p, int64_t i) {
    hagr::Vec<T, 1> v;
    v.template load<hagr::kKeep>(p, size_t(i));
    return v.get(0);
}
__device__ __forceinline__ void store_weight(void *p, int bf16, int64_t i, float f) {
    if (bf16) {
        hagr::Vec<__nv_bfloat16, 1> v;
        v.set(&f);
        v.store(p, size_t(i));
    } else {
        static_cast<float *>(p)[i] = f;
    }
}
// The weights of a thread's K vectors, zeros beyond the row; `vectors`: whether they can be read as such.  Without weights
// they are ones.  One test of the type for all of them: loads behind a test of their own would wait for one another.
template <int V, int K, typename At>
__device__ __forceinline__ void load_all_weights(hagr::Pairs<V> (&w)[K], const void *p, int bf16, bool vectors, const At &at, int n_vec) {
    auto load = [&](auto type, auto width) {
        using T = decltype(type);
        constexpr int N = decltype(width)::value;
        hagr::Vec<T, N> q[K][V / N];
#pragma unroll
        for (int k = 0; k < K; ++k) w[k].fill(0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V / N; ++j)
                if (at.mine(k, n_vec)) q[k][j].template load<hagr::kNear>(p, size_t(at.vec(k)) * (V / N) + j);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (at.mine(k, n_vec)) w[k].v[j] = q[k][j / N].get(j % N);
    };
    if (!p) {
#pragma unroll
        for (int k = 0; k < K; ++k) w[k].fill(at.mine(k, n_vec) ? 1.0f : 0.0f);
    } else if (vectors) {
        if (bf16) load(__nv_bfloat16(), std::integral_constant<int, V>());
        else load(float(), std::integral_constant<int, V>());
    } else {
        if (bf16) load(__nv_bfloat16(), std::integral_constant<int, 1>());
        else load(float(), std::integral_constant<int, 1>());
    }
}

// Vectors k0, k0 + 1, ... of a thread, for kernels that read the weights of a few at a time, row by row.
template <typename At>
struct From {
    const At &at;
    int k0;
    __device__ __forceinline__ int vec(int k) const { return at.vec(k0 + k); }
    __device__ __forceinline__ bool mine(int k, int n_vec) const { return at.mine(k0 + k, n_vec); }
};
template <int L> constexpr bool kKeepWeights = L >= 0;         // blocks of many threads have no registers for them
template <int L> constexpr int kThreadsOf = L > 0 ? kWarpRowThreads : L == 0 ? kRowThreads : kWideThreads;

// Sums over the L lanes that share a row, or (L <= 0) over the block; every thread receives the sum.  `slot`: of the block's
// sums, another one than that of the sum before, so that one barrier is enough.
template <int L>
__device__ __forceinline__ float group_sum(float v, float *slot) {
#pragma unroll
    for (int o = (L > 0 ? L : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (L <= 0) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = hagr::warp_sum((threadIdx.x & 31) < (blockDim.x >> 5) ? slot[threadIdx.x & 31] : 0.0f);
    }
    return v;
}

// The place of a thread in its row, and of its row among the others.
//   L > 0: L lanes of a warp per row, 32 / L rows per warp; L = 0: a block per row; L = -1: a block of up to kWideThreads.
// A thread has K vectors of the row.  Neighbouring lanes have neighbouring vectors, 32 (or L) of them are a chunk, and the
// warps of a block take chunks in turn; GROUPED: four chunks in turn, so that 128 columns of V = 1 lie in one warp.  Of the
// widths that a kernel is launched with, all chunks but the last kPartial of a thread lie within the row.
template <int L, int K, bool GROUPED>
struct Place {
    static constexpr int kLanes = L > 0 ? L : 32;
    static constexpr bool kWarpRows = L > 0;
    static constexpr int kPartial = GROUPED && L <= 0 ? 4 : K >= 4 ? 2 : 1;
    int lane, warp, warps;                     // lane of the group that shares a row; warp of the row's
    int64_t group, groups;                     // of this thread, and of the launch
    __device__ __forceinline__ Place() {
        if constexpr (kWarpRows) {
            constexpr int G = 32 / kLanes;
            lane = threadIdx.x % kLanes;
            warp = 0;
            warps = 1;
            group = (int64_t(blockIdx.x) * (kWarpRowThreads / 32) + (threadIdx.x >> 5)) * G + (threadIdx.x & 31) / kLanes;
            groups = int64_t(gridDim.x) * (kWarpRowThreads / 32) * G;
        } else {
            lane = threadIdx.x & 31;
            warp = threadIdx.x >> 5;
            warps = blockDim.x >> 5;
            group = blockIdx.x;
            groups = gridDim.x;
        }
    }
    __device__ __forceinline__ int chunk(int k) const {        // first vector of chunk k
        if constexpr (kWarpRows) return k * kLanes;
        else if constexpr (GROUPED) return ((k / 4 * warps + warp) * 4 + k % 4) * 32;
        else return (k * warps + warp) * 32;
    }
    __device__ __forceinline__ int vec(int k) const { return chunk(k) + lane; }
    __device__ __forceinline__ bool mine(int k, int n_vec) const { return k < K - kPartial || vec(k) < n_vec; }
    __device__ __forceinline__ bool first() const { return lane == 0 && warp == 0; }
    // the group whose rows decide how many turns the warp takes
    __device__ __forceinline__ int64_t leader() const { return kWarpRows ? group - (threadIdx.x & 31) / kLanes : group; }
};

// Whether the chunks of a row's warps cover it, and all but the last kPartial of each lie within it.
template <typename P, int K>
inline bool columns_fit(int n_vec, int warps) {
    const int64_t step = P::kWarpRows ? P::kLanes : 32 * int64_t(warps);
    return K * step >= n_vec && (K - P::kPartial) * step <= n_vec;
}

// Sums of R values over the lanes (or the block) that share a row; get(i) is the i-th in every lane, after f was applied to
// it.  Where there are more lanes than rows the sums are spread over the lanes, and f is computed once.
template <int L, int R>
struct Sums {
    static constexpr bool kSpread = L >= 2 * R && R > 1;
    float v[kSpread ? 1 : R];
    template <typename F>
    __device__ __forceinline__ Sums(const float (&s)[R], float *slot, F f) {
        if constexpr (kSpread) {
            v[0] = f(hagr::spread_sums<L, R>(s, threadIdx.x % L));
        } else {
            static_assert(L > 0 || R == 1, "");
#pragma unroll
            for (int i = 0; i < R; ++i) v[i] = f(group_sum<L>(s[i], slot));
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (kSpread) return hagr::spread_get<L, R>(v[0], i, threadIdx.x & 31);
        else return v[i];
    }
};

// Rows on their way into shared memory: chunk k of all groups (or warps) of the block side by side, then chunk k + 1.  A
// chunk is copied 16 bytes per lane at a time; where a vector has 32 bytes, a lane reads what its neighbours copied.
template <typename T, int V, typename P, int K>
struct ChunkCopy {
    static constexpr int kVector = V * int(sizeof(T)), kChunk = P::kLanes * kVector;
    static constexpr bool kCrosses = kVector > 16;             // lanes read each other's copies
    // a row that does not exist, and vectors beyond it, are zeros
    static __device__ __forceinline__ int threads() { return P::kLanes < 32 || P::kWarpRows ? kWarpRowThreads : int(blockDim.x); }
    static __device__ __forceinline__ int group() { return int(threadIdx.x) / P::kLanes * kChunk; }
    static __device__ __forceinline__ int bytes() { return K * threads() * kVector; }          // of a row of each group
    static __device__ __forceinline__ void issue(char *to, const char *row, const P &at, int n_vec, bool live) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < kVector / 16; ++j) {
                const int piece = (j * P::kLanes + at.lane) * 16;
                const int64_t from = int64_t(at.chunk(k)) * kVector + piece;
                char *const slot = to + k * threads() * kVector + group() + piece;
                if (live && (k < K - P::kPartial || from < int64_t(n_vec) * kVector)) hagr::copy_async<16>(slot, row + from);
                else *reinterpret_cast<uint4 *>(slot) = make_uint4(0, 0, 0, 0);
            }
    }
    static __device__ __forceinline__ hagr::Pairs<V> get(const char *from, const P &at, int k) {
        hagr::Vec<T, V> v;
        const char *slot = from + k * threads() * kVector + group() + at.lane * kVector;
#pragma unroll
        for (int j = 0; j < kVector / 16; ++j) {
            const uint4 q = reinterpret_cast<const uint4 *>(slot)[j];
            v.raw.w[4 * j] = q.x; v.raw.w[4 * j + 1] = q.y; v.raw.w[4 * j + 2] = q.z; v.raw.w[4 * j + 3] = q.w;
        }
        return hagr::widen(v);
    }
};

template <typename Args>
cudaError_t launch(void (*kernel)(Args), dim3 grid, unsigned threads, size_t shared, const Args &p, cudaStream_t s) {
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
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

constexpr int kSmShared = 227 * 1024;      // shared memory that the blocks of an SM can use
constexpr int kMostShared = kSmShared - 2048;      // and the dynamic part of one block's
// Lets a kernel use the shared memory of the current device's SMs (once per kernel and device).
template <auto KERNEL>
cudaError_t allow_shared() {
    static std::atomic<uint64_t> ready{0};
    int device = 0;
    cudaError_t err = cudaGetDevice(&device);
    const uint64_t bit = uint64_t(1) << (device & 63);
    if (err != cudaSuccess || (ready.load(std::memory_order_relaxed) & bit)) return err;
    err = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    if (err == cudaSuccess) ready.fetch_or(bit, std::memory_order_relaxed);
    return err;
}

// How many blocks of the kernel an SM runs at once (asked once per kernel and number of warps).
template <auto KERNEL>
int blocks_per_sm(unsigned threads, size_t shared) {
    static std::atomic<int> known[33];
    std::atomic<int> &slot = known[threads / 32];
    int n = slot.load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, KERNEL, int(threads), shared) != cudaSuccess || n < 1) {
            cudaGetLastError();
            n = 1;
        }
        slot.store(n, std::memory_order_relaxed);
    }
    return n;
}

inline bool dtype_ok(hag_dtype d) { return d == HAG_F32 || d == HAG_BF16; }
inline int size_of(hag_dtype d) { return d == HAG_F32 ? 4 : 2; }
inline bool on(const void *p, int bytes) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) == 0; }

// One matrix of a call: rows `ld` elements apart, which may be missing where it is optional.
struct Matrix {
    const void *p;
    int64_t ld;
    int elem;
    bool written, needed;
};

// Whether all matrices can be read V elements at a time, each by one access.
template <int N>
bool vectors_fit(int v, int32_t D, const Matrix (&m)[N]) {
    if (D % v != 0) return false;
    for (const Matrix &x : m)
        if (x.p && (x.ld % v != 0 || !on(x.p, v * x.elem))) return false;
    return true;
}

template <int N>
hag_status check(int64_t n, int32_t D, const void *weight, hag_dtype weight_dtype, const float *rstd, const Matrix (&m)[N]) {
    if (n < 0 || D <= 0) return HAG_ERR_ARG;
    if (D > (1 << 30)) return HAG_ERR_TOO_LARGE;
    for (const Matrix &x : m) {
        if (x.p && (x.ld < 0 || (x.written && n > 1 && x.ld < D))) return HAG_ERR_ARG;
        if (!x.p && x.needed && n > 0) return HAG_ERR_NULL;
    }
    for (const Matrix &x : m)
        if (!on(x.p, x.elem)) return HAG_ERR_ALIGN;
    if (!on(weight, size_of(weight_dtype)) || !on(rstd, 4)) return HAG_ERR_ALIGN;
    for (const Matrix &x : m)            // in place row by row is fine; the same start with other rows or elements is not
        for (const Matrix &y : m)
            if (&x != &y && x.p && x.p == y.p && y.written && n > 0 && (x.written || (n > 1 && x.ld != y.ld) || x.elem != y.elem)) return HAG_ERR_ARG;
    return HAG_OK;
}

}  // namespace hagn
