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
constexpr int kPerThread = 16;            // columns of a row per thread of such a block
constexpr int kMostInRegisters = kRowThreads * kPerThread;     // columns

// A vector of V elements, by one access of up to 32 bytes.
template <typename T, int V>
struct Wide {
    hagr::Vec<T, V> v;
    __device__ __forceinline__ void load(const void *row, int64_t i) {
        if constexpr (V * sizeof(T) == 32) {
            uint32_t *w = v.raw.w;
            asm volatile("ld.global.cg.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                         : "l"(static_cast<const char *>(row) + i * 32));
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
__device__ __forceinline__ float load_weight(const void *p, int bf16, int64_t i) {
    return !p ? 1.0f : bf16 ? load_one<__nv_bfloat16>(p, i) : load_one<float>(p, i);
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
// V weights from column c on; `vectors`: whether they can be read as one
template <int V>
__device__ __forceinline__ void load_weights(float (&w)[V], const void *p, int bf16, bool vectors, int64_t c) {
    if (vectors && p) {
        if (bf16) {
            hagr::Vec<__nv_bfloat16, V> q;
            q.template load<hagr::kNear>(p, size_t(c) / V);
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = q.get(j);
        } else {
            hagr::Vec<float, V> q;
            q.template load<hagr::kNear>(p, size_t(c) / V);
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = q.get(j);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = load_weight(p, bf16, c + j);
    }
}

// Sums over the L lanes that share a row, or (L = 0) over the block; every thread receives the sum.  `slot`: of the block's
// sums, another one than that of the sum before, so that one barrier is enough.
template <int L>
__device__ __forceinline__ float group_sum(float v, float *slot) {
#pragma unroll
    for (int o = (L ? L : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (L == 0) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = hagr::warp_sum((threadIdx.x & 31) < (blockDim.x >> 5) ? slot[threadIdx.x & 31] : 0.0f);
    }
    return v;
}

// The place of a thread in its row, and of its row among the others.
//   L > 0: L lanes of a warp per row, 32 / L rows per warp; L = 0: a block per row, 32 K vectors per warp.
// Vector k of the thread is number first + k * kStep of the row.
template <int L, int K>
struct Place {
    static constexpr int kStep = L ? L : 32;
    int first;
    int64_t group, groups;         // of this thread, and of the launch
    __device__ __forceinline__ Place() {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if constexpr (L) {
            constexpr int G = 32 / (L ? L : 32);
            first = lane % (L ? L : 32);
            group = (int64_t(blockIdx.x) * (kWarpRowThreads / 32) + warp) * G + lane / (L ? L : 32);
            groups = int64_t(gridDim.x) * (kWarpRowThreads / 32) * G;
        } else {
            first = warp * 32 * K + lane;
            group = blockIdx.x;
            groups = gridDim.x;
        }
    }
    // the group whose rows decide how many turns the warp takes
    __device__ __forceinline__ int64_t leader() const { return L ? group - (threadIdx.x & 31) / (L ? L : 32) : group; }
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
