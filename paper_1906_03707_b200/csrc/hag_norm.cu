// Layer norm over the columns of a matrix, forward and backward.
//   forward   mu = mean(x_r), rstd = 1 / sqrt(mean((x_r - mu)^2) + eps), y = (x - mu) * rstd * w + b
//   backward  xh = (x - mu) * rstd, q = g * w:  gx = rstd * (q - mean(q) - xh * mean(q * xh))
//             gw = sum over rows of g * xh,  gb = sum over rows of g
// The variance is the mean of squared differences from the mean (two steps over the row, never
// E[x^2] - mu^2, which cancels when the mean is large against the spread).
//
// Both directions are bound by memory: a row is read once (x, and g backward) and written once.  Measured on B200
// against a copy at 6.45 TB/s: forward 233 000 x 128 fp32 40 us (5.96 TB/s), 10^6 x 256 bf16 160 us (6.45), 32 768 x 4096
// bf16 102 us (5.3); backward with both parameter gradients 10^6 x 256 bf16 232 us in isolation (6.65) and 260 us in a long
// run (5.9), 200 000 x 512 fp32 206 us (6.0).  Contiguous rows of odd widths: 200 000 x 501 fp32 forward 138 us (5.8),
// 300 000 x 333 backward fp32 198 us (6.1), bf16 177 (3.4; forward 139 us): there the two warps of a scheduler wait for their
// own instructions, half of its slots are empty, and the memory is at a third of its rate.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cstdint>
#include <type_traits>

#include "hag.h"
#include "hag_kernels.cuh"
#include "hag_launch.h"
#include "hag_rows.cuh"

namespace {

struct NormArgs {
    int64_t n;
    int32_t D;
    int32_t w_bf16;             // type of w, b, gw, gb
    const void *x, *w, *b;
    const void *g;              // backward: gradient of y
    int64_t ld_x, ld_g, ld_y;
    void *y;                    // forward: y; backward: gx
    float *mean, *rstd;
    const float *mean_in, *rstd_in;
    float eps;
    float *partial;             // backward: [parts][2][D]
    void *gw, *gb;
    int32_t parts;
    int32_t stages;             // of the ring
    int32_t w_vectors;          // whether w and b can be read a vector at a time
    int32_t edge_at;            // where the edges' slots begin in shared memory (EDGE kernels)
    int32_t hop;                // rows from one row of an alignment to the next (EDGE kernels)
};

constexpr int kRowThreads = 256;

template <typename T>
__device__ __forceinline__ float load1(const void *p, int64_t i) {
    hagr::Vec<T, 1> v;
    v.template load<hagr::kKeep>(p, i);
    return v.get(0);
}
template <typename T>
__device__ __forceinline__ void store1(void *p, int64_t i, float f) {
    hagr::Vec<T, 1> v;
    v.set(&f);
    v.store(p, i);
}
__device__ __forceinline__ float load_param(const void *p, int bf16, int64_t i) {
    return bf16 ? load1<__nv_bfloat16>(p, i) : load1<float>(p, i);
}
__device__ __forceinline__ void store_param(void *p, int bf16, int64_t i, float v) {
    if (bf16) store1<__nv_bfloat16>(p, i, v); else store1<float>(p, i, v);
}

// Sum over the block, returned to every thread; `slot` alternates so that one barrier per sum is enough.
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float *slot) {
    v = hagr::warp_sum(v);
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) s += slot[w];
    return s;
}

// Rows of more than kMostInBlock columns: one block per row, which it reads three times (the second and third time out
// of the caches).
template <typename T>
__global__ void __launch_bounds__(kRowThreads) norm_fwd_any_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float slot[2][kRowThreads / 32];
    const float cols = float(p.D);
    hagk::pdl_wait();
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + r * p.ld_x;
        T *y = static_cast<T *>(p.y) + r * p.ld_y;
        float s = 0.0f;
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) s += load1<T>(x, c);
        const float mean = block_sum<kRowThreads>(s, slot[0]) / cols;
        s = 0.0f;
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) {
            const float d = load1<T>(x, c) - mean;
            s += d * d;
        }
        const float rstd = rsqrtf(block_sum<kRowThreads>(s, slot[1]) / cols + p.eps);
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) {
            float v = (load1<T>(x, c) - mean) * rstd;
            if (p.w) v *= load_param(p.w, p.w_bf16, c);
            if (p.b) v += load_param(p.b, p.w_bf16, c);
            store1<T>(y, c, v);
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) norm_bwd_any_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float slot[2][2][kRowThreads / 32];
    const float cols = float(p.D);
    hagk::pdl_wait();
    int turn = 0;
    for (int64_t r = blockIdx.x; r < p.n; r += gridDim.x, turn ^= 1) {
        const T *x = static_cast<const T *>(p.x) + r * p.ld_x;
        const T *g = static_cast<const T *>(p.g) + r * p.ld_g;
        T *gx = static_cast<T *>(p.y) + r * p.ld_y;
        const float mean = __ldcg(p.mean_in + r), rstd = __ldcg(p.rstd_in + r);
        float s1 = 0.0f, s2 = 0.0f;
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) {
            const float q = load1<T>(g, c) * (p.w ? load_param(p.w, p.w_bf16, c) : 1.0f);
            s1 += q;
            s2 += q * ((load1<T>(x, c) - mean) * rstd);
        }
        s1 = block_sum<kRowThreads>(s1, slot[turn][0]) / cols;
        s2 = block_sum<kRowThreads>(s2, slot[turn][1]) / cols;
        for (int32_t c = threadIdx.x; c < p.D; c += kRowThreads) {
            const float q = load1<T>(g, c) * (p.w ? load_param(p.w, p.w_bf16, c) : 1.0f);
            const float xh = (load1<T>(x, c) - mean) * rstd;
            store1<T>(gx, c, rstd * (q - s1 - xh * s2));
        }
    }
}

// gw and gb of one strip of 32 columns and one part of the rows.
constexpr int kStripRows = 8;
template <typename T>
__global__ void __launch_bounds__(32 * kStripRows) norm_params_any_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[2][kStripRows][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    const int64_t step = int64_t(p.parts) * kStripRows;
    float aw = 0.0f, ab = 0.0f;
    hagk::pdl_wait();
    if (c < p.D)
        for (int64_t r = int64_t(blockIdx.y) * kStripRows + part; r < p.n; r += step) {
            const float g = load1<T>(p.g, r * p.ld_g + c);
            aw += g * ((load1<T>(p.x, r * p.ld_x + c) - __ldcg(p.mean_in + r)) * __ldcg(p.rstd_in + r));
            ab += g;
        }
    sum[0][part][lane] = aw;
    sum[1][part][lane] = ab;
    __syncthreads();
    if (part < 2 && c < p.D) {
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < kStripRows; ++k) s += sum[part][k][lane];
        p.partial[(int64_t(blockIdx.y) * 2 + part) * p.D + c] = s;
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Rows read once.  A group of threads owns a row, K vectors of V elements per thread, and reads ahead of the rows it
// works on.
//   L = 4, 8, 16, 32: that many lanes of a warp per row, R rows per group at a time
//   L = 0 or -1  : a whole block per row (of up to kMostThreads or kFewThreads threads), sums over the block through
//                  shared memory
// The rows ahead are on their way into a ring in shared memory (asynchronous copies), so what is in flight does not
// depend on registers.  With 16-byte vectors every thread copies its own vectors into its own slots (Slots).  Rows that
// do not start on 16 bytes go one of two ways:
//   EDGE   : all matrices of the call have the same misalignment in every row (contiguous rows of an odd width).  Rows
//            `hop` apart are misaligned alike; a group keeps to those, so a thread's vectors have the same columns in
//            all its rows.  The up to 2 (V - 1) elements around the vectors are one more element for some threads (Edge).
//   Pieces : else.  Rows are copied as the 16-byte pieces they touch, and the group reads narrow vectors out of those
//            at any place.  (300 000 x 333 bf16: forward 177 us, by EDGE 139; backward 286, by EDGE 175.)
// The weights stay with the thread over all its rows: in registers, or from 16 columns per thread on in shared memory.
constexpr int kMostThreads = 1024;        // of a block per row; up to kFewThreads the compiler may use 128 registers (with more
                                          // threads the backward pass with 16 narrow columns each spills 116 bytes)
constexpr int kFewThreads = 512;
// Stages of the ring.  What is in flight per SM matters more than how many warps are there: about 64 KB (one block of
// eight warps, 64 bytes per lane and turn) is best; with three blocks 10^6 x 256 bf16 forward takes 196 us, with one 160.
constexpr int kFwdStages = 3, kBwdStages = 4, kBlockStages = 2;

template <typename T, int V> constexpr bool kRing = V * int(sizeof(T)) == 16;
constexpr int kWarpThreads = 256;
template <int L> constexpr int kThreads = L == 0 ? kMostThreads : L < 0 ? kFewThreads : kWarpThreads;
// narrow vectors keep the parameters in registers, but for the widest rows; warps of other columns do not share them
template <typename T, int L, int V, int K, bool EDGE> constexpr bool kShared = V * K >= 16 && (kRing<T, V> || L == 0) && !(EDGE && L > 0);
template <typename T, int L, int V, int K, bool BWD> constexpr int kLeastBlocks = L < 0 && !BWD && kRing<T, V> ? 2 : 1;    // per SM
// Rows per turn: 64 bytes per lane and turn (both operands of the backward pass together), but at least one row.
constexpr int rows_per_turn(int bytes, int most) { return bytes >= 64 ? 1 : 64 / bytes < most ? 64 / bytes : most; }
template <typename T, int L, int V, int K> constexpr int kFwdRows = L <= 0 ? 1 : kRing<T, V> ? rows_per_turn(K * V * int(sizeof(T)), 4) : V * K >= 16 ? 1 : 16 / (V * K) < 4 ? 16 / (V * K) : 4;
// rows with edges: more to do per row, so two rows and two blocks per SM (10^6 x 129 fp32 forward 184 us, with four rows
// and one block 208), but with 16 columns per thread one block (200 000 x 501 138 us, with two 167)
template <typename T, int L, int V, int K, bool EDGE> constexpr int kFwdTurn = EDGE && L > 0 && V * K < 16 ? 2 : kFwdRows<T, L, V, K>;
template <int L, int V, int K, bool EDGE> constexpr int kFwdBlocks = EDGE && L > 0 && V * K < 16 ? 2 : 1;
template <typename T, int L, int V, int K> constexpr int kBwdRows = L > 0 && V * K <= 8 ? 2 : 1;

// Sums of R values per lane over the L lanes of a group: lanes trade halves of the list while it has more than one
// value (4 sums over 32 lanes take 6 shuffles, not 20), and each lane ends with ONE of the sums: number (gl * R / L).
// What follows a sum (a division, a root) is then done once, not once per value.
template <int L, int R>
__device__ __forceinline__ float spread_sums(const float (&in)[R], int gl) {
    float v[R];
#pragma unroll
    for (int i = 0; i < R; ++i) v[i] = in[i];
    int o = L / 2;
#pragma unroll
    for (int h = R / 2; h >= 1; h /= 2, o /= 2) {
        const bool upper = gl & o;
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float keep = upper ? v[i + h] : v[i], give = upper ? v[i] : v[i + h];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
#pragma unroll
    for (; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    return v[0];
}
// Value number i of a list spread that way, in every lane of the group.
template <int L, int R>
__device__ __forceinline__ float spread_get(float v, int i, int lane) {
    return __shfl_sync(0xffffffffu, v, (lane & ~(L - 1)) + i * (L / R));
}

// Two fp32 operations per instruction; N is even or 1.
template <int N>
struct Pairs {
    float v[N];
    template <typename F2, typename F1>
    static __device__ __forceinline__ void each(F2 f2, F1 f1) {
#pragma unroll
        for (int j = 0; j + 1 < N; j += 2) f2(j);
        if constexpr (N % 2) f1(N - 1);
    }
    __device__ __forceinline__ float2 two(int j) const { return make_float2(v[j], v[j + 1]); }
    __device__ __forceinline__ void put(int j, float2 t) { v[j] = t.x; v[j + 1] = t.y; }
    __device__ __forceinline__ void fill(float f) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = f;
    }
    __device__ __forceinline__ void add(const Pairs &a) {                                     // v += a
        each([&](int j) { put(j, __fadd2_rn(two(j), a.two(j))); }, [&](int j) { v[j] += a.v[j]; });
    }
    __device__ __forceinline__ void fma(const Pairs &a, const Pairs &b) {                     // v += a * b
        each([&](int j) { put(j, __ffma2_rn(a.two(j), b.two(j), two(j))); }, [&](int j) { v[j] = fmaf(a.v[j], b.v[j], v[j]); });
    }
    __device__ __forceinline__ void mul(const Pairs &a) {
        each([&](int j) { put(j, __fmul2_rn(two(j), a.two(j))); }, [&](int j) { v[j] *= a.v[j]; });
    }
    __device__ __forceinline__ void shift_scale(float s, float m) {                           // v = (v + s) * m
        each([&](int j) { put(j, __fmul2_rn(__fadd2_rn(two(j), make_float2(s, s)), make_float2(m, m))); },
             [&](int j) { v[j] = (v[j] + s) * m; });
    }
    __device__ __forceinline__ void mul_all(float m) {
        each([&](int j) { put(j, __fmul2_rn(two(j), make_float2(m, m))); }, [&](int j) { v[j] *= m; });
    }
    __device__ __forceinline__ void shift(float s) {                                          // v += s
        each([&](int j) { put(j, __fadd2_rn(two(j), make_float2(s, s))); }, [&](int j) { v[j] += s; });
    }
    __device__ __forceinline__ void affine(float m, float s) {                                // v = v * m + s
        each([&](int j) { put(j, __ffma2_rn(two(j), make_float2(m, m), make_float2(s, s))); }, [&](int j) { v[j] = fmaf(v[j], m, s); });
    }
    __device__ __forceinline__ float sum() const {
        float2 s = make_float2(v[0], N > 1 ? v[N > 1] : 0.0f);
#pragma unroll
        for (int j = 2; j + 1 < N; j += 2) s = __fadd2_rn(s, two(j));
        return s.x + s.y;
    }
    __device__ __forceinline__ float dot(const Pairs &a) const {
        if constexpr (N == 1) return v[0] * a.v[0];
        float2 s = __fmul2_rn(two(0), a.two(0));
#pragma unroll
        for (int j = 2; j + 1 < N; j += 2) s = __ffma2_rn(two(j), a.two(j), s);
        return s.x + s.y;
    }
};

template <typename T, int V>
__device__ __forceinline__ Pairs<V> widen(const hagr::Vec<T, V> &a) {
    Pairs<V> f;
#pragma unroll
    for (int j = 0; j < V; ++j) f.v[j] = a.get(j);
    return f;
}

// Waits until the oldest of the stages has arrived (a launch has fewer stages where a row fills the shared memory).
__device__ __forceinline__ void wait_oldest(int stages) {
    if (stages == 4) hagr::wait_copies<3>();
    else if (stages == 3) hagr::wait_copies<2>();
    else if (stages == 2) hagr::wait_copies<1>();
    else hagr::wait_copies<0>();
}

// The rows ahead, 16-byte vectors: slots of the thread (stages x OPS matrices x R rows x K vectors; those of the threads
// lie side by side).  THREADS is the block's size where it is fixed, else 0.
template <typename T, int V, int K, int R, int OPS, int L, int THREADS>
struct Slots {
    static constexpr int kSlot = V * int(sizeof(T)), kStage = OPS * R * K * kSlot;         // bytes per thread
    char *mine;
    int write = 0, read = 0, end;                              // offsets of the stages in turn
    int first, step, n_vec;

    static __device__ __forceinline__ int threads() { return THREADS ? THREADS : int(blockDim.x); }
    __device__ __forceinline__ Slots(char *base, const NormArgs &p, int first_, int step_, int n_vec_)
        : mine(base + threadIdx.x * kSlot), end(p.stages * kStage * threads()), first(first_), step(step_), n_vec(n_vec_) {}
    __device__ __forceinline__ char *slot(int stage, int op, int i, int k) const { return mine + stage + ((op * R + i) * K + k) * (threads() * kSlot); }
    // row i of the turn being issued starts at `row`; a row that does not exist is read as zeros
    __device__ __forceinline__ void issue(int op, int i, const char *row, bool live) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            char *to = slot(write, op, i, k);
            if (live && first + k * step < n_vec) hagr::copy_async<kSlot>(to, row + int64_t(first + k * step) * kSlot);
            else *reinterpret_cast<hagr::Words<kSlot> *>(to) = hagr::Words<kSlot>{};
        }
    }
    __device__ __forceinline__ void issued() {                 // the turn is complete
        hagr::commit_copies();
        write = write + kStage * threads() == end ? 0 : write + kStage * threads();
    }
    __device__ __forceinline__ const char *at(int op, int i, const char *) const { return slot(read, op, i, 0); }
    __device__ __forceinline__ hagr::Vec<T, V> get(const char *row, int k) const {
        hagr::Vec<T, V> v;
        v.raw = *reinterpret_cast<const hagr::Words<kSlot> *>(row + k * (threads() * kSlot));
        return v;
    }
    __device__ __forceinline__ void wait(int stages) const { wait_oldest(stages); }
    template <bool BARRIER> __device__ __forceinline__ void done() {       // with the oldest turn's slots
        read = read + kStage * threads() == end ? 0 : read + kStage * threads();
    }
};

// The rows ahead, at any alignment: per stage, matrix and row the 16-byte pieces that the row touches, and zeros up to
// the last place that a thread looks at.  The last piece is read up to the row's end; the first one from its 16-byte
// boundary on, which never leaves the allocation that holds the row (allocations start on 16 bytes).  The group copies
// together, so it meets before it reads and before a stage is written again.
template <typename T, int V, int K, int R, int OPS, int L>
struct Pieces {
    static constexpr int kBytes = V * int(sizeof(T));
    char *area;                                                // of this group
    int write = 0, read = 0, end, pitch, len;
    int first, step;

    static __host__ __device__ constexpr int row_bytes(int step) { return (K * step * kBytes + 15) / 16 * 16 + 16; }
    __device__ __forceinline__ Pieces(char *base, const NormArgs &p, int first_, int step_, int)
        : pitch(row_bytes(step_)), len(p.D * int(sizeof(T))), first(first_), step(step_) {
        end = p.stages * (OPS * R) * pitch;
        area = base + (L > 0 ? int(threadIdx.x) / (L > 0 ? L : 1) * end : 0);
    }
    __device__ __forceinline__ void issue(int op, int i, const char *row, bool live) {
        char *to = area + write + (op * R + i) * pitch;
        if (live) {
            const int off = int(uint32_t(reinterpret_cast<uintptr_t>(row)) & 15u), bytes = off + len;
            const char *from = row - off;
            for (int c = first * 16; c < pitch; c += step * 16) {      // behind the row: copies of no bytes, i.e. zeros
                const int here = min(16, bytes - c);
                hagr::copy_async_part(to + c, from + (here > 0 ? c : 0), max(here, 0));
            }
        } else {
            for (int c = first * 16; c < pitch; c += step * 16) *reinterpret_cast<uint4 *>(to + c) = make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void issued() {
        hagr::commit_copies();
        write = write + OPS * R * pitch == end ? 0 : write + OPS * R * pitch;
    }
    // where this thread's part of row i, which started at `row`, lies, and vector k of it
    __device__ __forceinline__ const char *at(int op, int i, const char *row) const {
        return area + read + (op * R + i) * pitch + (uint32_t(reinterpret_cast<uintptr_t>(row)) & 15u) + first * kBytes;
    }
    __device__ __forceinline__ hagr::Vec<T, V> get(const char *row, int k) const {
        hagr::Vec<T, V> v;
        v.raw = *reinterpret_cast<const hagr::Words<kBytes> *>(row + k * step * kBytes);
        return v;
    }
    __device__ __forceinline__ void wait(int n) const {
        wait_oldest(n);
        if (L > 0) __syncwarp(); else __syncthreads();
    }
    // BARRIER: the threads of a block have not met since they read
    template <bool BARRIER> __device__ __forceinline__ void done() {
        if (L > 0) __syncwarp();
        else if (BARRIER) __syncthreads();
        read = read + OPS * R * pitch == end ? 0 : read + OPS * R * pitch;
    }
};

template <typename T, int V, int K, int R, int OPS, int L>
using Ahead = std::conditional_t<kRing<T, V>, Slots<T, V, K, R, OPS, L, (L > 0 ? kThreads<L> : 0)>, Pieces<T, V, K, R, OPS, L>>;

// The elements of a row around its vectors: `head` before them (those of an alignment class are the same), up to V - 1
// behind.  Threads 0 .. V - 1 of the group take the former, the next V the latter, one each, out of slots of their own.
template <typename T, int V, int R, int OPS, bool EDGE>
struct Edge {
    int head = 0, n_vec, col = -1;                             // elements before the vectors; vectors; this thread's element
    int high = 0, stage = 0, stages;
    char *mine;

    __device__ __forceinline__ Edge(char *base, const NormArgs &p, const char *row, int first)
        : n_vec(p.D / V), stages(p.stages), mine(base + threadIdx.x * 4) {
        if constexpr (EDGE) {
            head = int((16u - (uint32_t(reinterpret_cast<uintptr_t>(row)) & 15u)) & 15u) / int(sizeof(T));
            n_vec = (p.D - head) / V;
            const int c = first < V ? (first < head ? first : p.D) : first < 2 * V ? head + n_vec * V + first - V : p.D;
            col = c < p.D ? c : -1;
            // a bf16 element is the lower or the upper half of its aligned word
            high = sizeof(T) == 2 ? int(uint32_t(reinterpret_cast<uintptr_t>(row) + uint32_t(c) * 2u) & 2u) : 0;
        }
    }
    __device__ __forceinline__ char *slot(int s, int op, int i) const { return mine + ((s * OPS + op) * R + i) * int(blockDim.x) * 4; }
    __device__ __forceinline__ void issue(int s, int op, int i, const char *row, bool live) const {
        if (!EDGE || col < 0) return;
        if (live) hagr::copy_async_word(slot(s, op, i), row + int64_t(col) * sizeof(T) - high, sizeof(T) == 4 ? 4 : 2 + high);
        else *reinterpret_cast<uint32_t *>(slot(s, op, i)) = 0;
    }
    __device__ __forceinline__ float get(int s, int op, int i) const {
        if (!EDGE || col < 0) return 0.0f;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(slot(s, op, i));
        return __uint_as_float(sizeof(T) == 4 ? w : high ? w & 0xffff0000u : w << 16);
    }
    __device__ __forceinline__ int next(int s) const { return s + 1 == stages ? 0 : s + 1; }
};

// The rows of a group of threads: R at a time, `stride` rows from one turn to the next.
template <int L, int R>
struct Turns {
    static constexpr int G = L <= 0 ? 1 : 32 / (L <= 0 ? 32 : L);        // groups per warp
    int first, step, side;               // this thread's place in its group, the group's threads, the group's place in its warp
    int64_t row, stride;
    int32_t all, live[R];                // turns of the warp (or block); turns in which row i exists

    // `hop`: rows that the group takes are so far apart (the number of groups is a multiple of it)
    __device__ __forceinline__ Turns(int64_t n, int32_t hop) {
        const int lane = threadIdx.x & 31;
        first = L <= 0 ? int(threadIdx.x) : lane % (L <= 0 ? 32 : L);
        step = L <= 0 ? int(blockDim.x) : L;
        side = L <= 0 ? 0 : lane / (L <= 0 ? 32 : L);
        const int64_t group = L <= 0 ? int64_t(blockIdx.x) : (int64_t(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5)) * G + side;
        row = hop == 1 ? group * R : group % hop + group / hop * (R * hop);
        stride = L <= 0 ? int64_t(gridDim.x) * R : int64_t(gridDim.x) * (blockDim.x >> 5) * G * R;
        all = G > 1 ? count(n, (group - side) * R) : count(n, row);
#pragma unroll
        for (int i = 0; i < R; ++i) live[i] = count(n, row + i * hop);
    }
    __device__ __forceinline__ int32_t count(int64_t n, int64_t from) const { return from < n ? int32_t((n - from + stride - 1) / stride) : 0; }
};

// Parameters of a thread's columns, N vectors of them (weights, or weights and biases), in registers or in shared
// memory in planes of up to four columns (so that neighbours read neighbouring words).
template <int V, int K, int N, bool SHARED>
struct Params {
    static constexpr bool kShared = SHARED;
    static constexpr int W = V < 4 ? V : 4;
    struct alignas(4 * W) Piece { float v[W]; };
    float own[kShared ? 1 : N * K * V];
    Piece *shared;
    int first, step;

    static __host__ __device__ constexpr size_t bytes(int step) { return kShared ? size_t(N) * K * V * step * 4 : 0; }
    __device__ __forceinline__ Params(char *base, int first_, int step_) : shared(reinterpret_cast<Piece *>(base)), first(first_), step(step_) {}
    __device__ __forceinline__ Piece *piece(int n, int k, int h) const { return shared + ((n * (V / W) + h) * K + k) * step + first; }
    // `writes`: whether this thread fills the shared copy of its columns
    __device__ __forceinline__ void load(int n, const void *p, int bf16, bool vectors, int32_t n_vec, int head, float fill, bool writes) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float v[V];
            const int32_t vec = first + k * step;
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = fill;
            if (p && vec < n_vec) {
                if (vectors && bf16) {
                    hagr::Vec<__nv_bfloat16, V> q;
                    q.template load<hagr::kKeep>(p, vec);
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] = q.get(j);
                } else if (vectors) {
                    hagr::Vec<float, V> q;
                    q.template load<hagr::kKeep>(p, vec);
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] = q.get(j);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] = load_param(p, bf16, int64_t(vec) * V + head + j);
                }
            }
            if constexpr (kShared) {
                if (writes)
#pragma unroll
                    for (int h = 0; h < V / W; ++h) {
                        Piece q;
#pragma unroll
                        for (int j = 0; j < W; ++j) q.v[j] = v[h * W + j];
                        *piece(n, k, h) = q;
                    }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) own[(n * K + k) * V + j] = v[j];
            }
        }
    }
    __device__ __forceinline__ Pairs<V> get(int n, int k) const {
        Pairs<V> f;
        if constexpr (kShared) {
#pragma unroll
            for (int h = 0; h < V / W; ++h) {
                const Piece q = *piece(n, k, h);
#pragma unroll
                for (int j = 0; j < W; ++j) f.v[h * W + j] = q.v[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) f.v[j] = own[(n * K + k) * V + j];
        }
        return f;
    }
};

// Sums over the group, spread over its lanes (L > 0) or in every thread (L = 0: up to two values; `slot` alternates
// between calls, so one barrier is enough).
template <int L, int R>
__device__ __forceinline__ float group_sums(const float (&s)[R], int gl, float2 *slot) {
    if constexpr (L > 0) {
        return spread_sums<L, R>(s, gl);
    } else {
        static_assert(R == 1, "");
        const float a = hagr::warp_sum(s[0]);
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5].x = a;
        __syncthreads();
        return hagr::warp_sum((threadIdx.x & 31) < (blockDim.x >> 5) ? slot[threadIdx.x & 31].x : 0.0f);
    }
}
__device__ __forceinline__ float2 block_sum2(float a, float b, float2 *slot) {
    a = hagr::warp_sum(a);
    b = hagr::warp_sum(b);
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    const float2 q = (threadIdx.x & 31) < (blockDim.x >> 5) ? slot[threadIdx.x & 31] : make_float2(0.0f, 0.0f);
    return make_float2(hagr::warp_sum(q.x), hagr::warp_sum(q.y));
}

template <typename T, int V, int L, int K, bool EDGE>
__global__ void __launch_bounds__(kThreads<L>, (L > 0 ? kFwdBlocks<L, V, K, EDGE> : kLeastBlocks<T, L, V, K, false>)) norm_fwd_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    extern __shared__ __align__(16) char raw[];
    __shared__ float2 slots[2][32];
    constexpr int R = kFwdTurn<T, L, V, K, EDGE>;
    const int32_t hop = EDGE ? p.hop : 1;
    const Turns<L, R> turns(p.n, hop);
    const int lane = threadIdx.x & 31, first = turns.first, step = turns.step;
    const float cols = float(p.D), inverse = 1.0f / cols;
    Params<V, K, 2, kShared<T, L, V, K, EDGE>> wb(raw, first, step);
    const int64_t ld_x = p.ld_x * int64_t(sizeof(T)), ld_y = p.ld_y * int64_t(sizeof(T));
    const char *x_next = static_cast<const char *>(p.x) + turns.row * ld_x, *x_row = x_next;
    char *y = static_cast<char *>(p.y) + turns.row * ld_y;
    const int64_t step_x = turns.stride * ld_x, step_y = turns.stride * ld_y, hop_x = hop * ld_x, hop_y = hop * ld_y;
    char *const ring = raw + Params<V, K, 2, kShared<T, L, V, K, EDGE>>::bytes(step);
    const Edge<T, V, R, 1, EDGE> edge(raw + p.edge_at, p, x_next, first);
    const int n_vec = edge.n_vec, head = edge.head, head_bytes = head * int(sizeof(T));
    Ahead<T, V, K, R, 1, L> ahead(ring, p, first, step, n_vec);
    int edge_write = 0, edge_read = 0;
    auto issue = [&](int32_t turn) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            edge.issue(edge_write, 0, i, x_next + i * hop_x, turn < turns.live[i]);
            ahead.issue(0, i, x_next + i * hop_x + head_bytes, turn < turns.live[i]);
        }
        ahead.issued();
        edge_write = edge.next(edge_write);
        x_next += step_x;
    };
    hagk::pdl_wait();
    for (int32_t s = 0; s < p.stages; ++s) issue(s);
    wb.load(0, p.w, p.w_bf16, p.w_vectors, n_vec, head, 1.0f, L <= 0 || int(threadIdx.x) < L);
    wb.load(1, p.b, p.w_bf16, p.w_vectors, n_vec, head, 0.0f, L <= 0 || int(threadIdx.x) < L);
    const float edge_w = EDGE && edge.col >= 0 && p.w ? load_param(p.w, p.w_bf16, edge.col) : 1.0f;
    const float edge_b = EDGE && edge.col >= 0 && p.b ? load_param(p.b, p.w_bf16, edge.col) : 0.0f;
    if (L > 0 && wb.kShared) __syncthreads();
    int64_t r = turns.row + (L <= 0 ? 0 : first * R / (L <= 0 ? 1 : L)) * hop;        // the row whose statistics this thread holds
    for (int32_t turn = 0; turn < turns.all; ++turn) {
        ahead.wait(p.stages);
        Pairs<V> x[R][K];
        float s[R], xe[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i] = xe[i] = edge.get(edge_read, 0, i);
            const char *row = ahead.at(0, i, x_row + i * hop_x);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x[i][k] = widen(ahead.get(row, k));
                s[i] += x[i][k].sum();                         // places beyond the row hold zeros
            }
        }
        // divided, not times 1 / D: where the row's sum is exact, the mean of equal values is that value and y the bias
        // (else, as of 72 times 1000.1, the mean is off by the sum's rounding, and rstd is up to 1 / sqrt(eps))
        const float my_mean = group_sums<L, R>(s, first, slots[0]) / cols;
        ahead.template done<false>();
        edge_read = edge.next(edge_read);
        issue(turn + p.stages);                                // into the stage just read
        x_row += step_x;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float mean = L <= 0 ? my_mean : spread_get<L <= 0 ? 32 : L, R>(my_mean, i, lane);
            xe[i] -= mean;
            s[i] = EDGE && edge.col >= 0 ? xe[i] * xe[i] : 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x[i][k].shift(-mean);
                const float q = x[i][k].dot(x[i][k]);
                s[i] += first + k * step < n_vec ? q : 0.0f;
            }
        }
        const float my_rstd = rsqrtf(group_sums<L, R>(s, first, slots[1]) * inverse + p.eps);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float rstd = L <= 0 ? my_rstd : spread_get<L <= 0 ? 32 : L, R>(my_rstd, i, lane);
            const bool live = turn < turns.live[i];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                Pairs<V> o = wb.get(1, k);
                x[i][k].mul_all(rstd);
                o.fma(x[i][k], wb.get(0, k));
                hagr::Vec<T, V> to;
                to.set(o.v);
                if (live && first + k * step < n_vec) to.store(y + i * hop_y + head_bytes, first + k * step);
            }
            if (EDGE && live && edge.col >= 0) store1<T>(y + i * hop_y, edge.col, fmaf(xe[i] * rstd, edge_w, edge_b));
        }
        if (L <= 0 ? first == 0 : first % ((L <= 0 ? R : L) / R) == 0 && r < p.n) {
            if (p.mean) p.mean[r] = my_mean;
            if (p.rstd) p.rstd[r] = my_rstd;
        }
        y += step_y;
        r += turns.stride;
    }
    hagr::wait_copies<0>();
}

// A block's sum for column c of gw (0) or gb (1): a part of it, or, from the only block, the result.
__device__ __forceinline__ void leave_param(const NormArgs &p, int which, int32_t c, float v) {
    if (p.parts > 1) p.partial[(int64_t(blockIdx.x) * 2 + which) * p.D + c] = v;
    else if (void *to = which ? p.gb : p.gw) store_param(to, p.w_bf16, c, v);
}

template <typename T, int V, int L, int K, bool EDGE>
__global__ void __launch_bounds__(kThreads<L>, (kLeastBlocks<T, L, V, K, true>)) norm_bwd_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    extern __shared__ __align__(16) char raw[];
    __shared__ float2 slots[2][32];
    constexpr int R = kBwdRows<T, L, V, K>, S = L <= 0 ? 32 : L;
    constexpr bool HOLD = L != 0 && R * K * V <= 16;                     // keep xh and g * w between their two uses
    const int32_t hop = EDGE ? p.hop : 1;
    const Turns<L, R> turns(p.n, hop);
    const int lane = threadIdx.x & 31, first = turns.first, step = turns.step;
    const float inverse = 1.0f / float(p.D);
    Params<V, K, 1, kShared<T, L, V, K, EDGE>> weights(raw, first, step);
    const int64_t ld_x = p.ld_x * int64_t(sizeof(T)), ld_g = p.ld_g * int64_t(sizeof(T)), ld_y = p.ld_y * int64_t(sizeof(T));
    const char *x_next = static_cast<const char *>(p.x) + turns.row * ld_x, *g_next = static_cast<const char *>(p.g) + turns.row * ld_g;
    const char *x_row = x_next, *g_row = g_next;               // of the turn being worked on
    char *y = static_cast<char *>(p.y) + turns.row * ld_y;
    const int64_t step_x = turns.stride * ld_x, step_g = turns.stride * ld_g, step_y = turns.stride * ld_y;
    const int64_t hop_x = hop * ld_x, hop_g = hop * ld_g, hop_y = hop * ld_y;
    char *const ring = raw + Params<V, K, 1, kShared<T, L, V, K, EDGE>>::bytes(step);
    const Edge<T, V, R, 2, EDGE> edge(raw + p.edge_at, p, x_next, first);
    const int n_vec = edge.n_vec, head = edge.head, head_bytes = head * int(sizeof(T));
    Ahead<T, V, K, R, 2, L> ahead(ring, p, first, step, n_vec);
    int edge_write = 0, edge_read = 0;
    float edge_aw = 0.0f, edge_ab = 0.0f;
    auto issue = [&](int32_t turn) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            edge.issue(edge_write, 0, i, x_next + i * hop_x, turn < turns.live[i]);
            edge.issue(edge_write, 1, i, g_next + i * hop_g, turn < turns.live[i]);
            ahead.issue(0, i, x_next + i * hop_x + head_bytes, turn < turns.live[i]);
            ahead.issue(1, i, g_next + i * hop_g + head_bytes, turn < turns.live[i]);
        }
        ahead.issued();
        edge_write = edge.next(edge_write);
        x_next += step_x;
        g_next += step_g;
    };
    // The rows' statistics: each lane of a group (or warp) reads those of another turn, S turns at once and S turns
    // ahead, and hands them round when the turn comes.
    // Beyond the row xh is (0 - mean) * rstd: where that overflows, 0 times it is no number, and `careful` turns take the
    // sum again without those places.
    float mean[R], rstd[R], mean_next[R], rstd_next[R];
    bool careful = false;
    auto statistics = [&](int32_t turn) {
        const int32_t mine = turn + lane % S;
        const int64_t at = turns.row + int64_t(mine) * turns.stride;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            mean_next[i] = mine < turns.live[i] ? __ldcg(p.mean_in + at + i * hop) : 0.0f;
            rstd_next[i] = mine < turns.live[i] ? __ldcg(p.rstd_in + at + i * hop) : 0.0f;
        }
    };
    Pairs<V> aw[K], ab[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        aw[k].fill(0.0f);
        ab[k].fill(0.0f);
    }
    hagk::pdl_wait();
    for (int32_t s = 0; s < p.stages; ++s) issue(s);
    statistics(0);
    weights.load(0, p.w, p.w_bf16, p.w_vectors, n_vec, head, 1.0f, L <= 0 || int(threadIdx.x) < L);
    const float edge_w = EDGE && edge.col >= 0 && p.w ? load_param(p.w, p.w_bf16, edge.col) : 1.0f;
    if (L > 0 && weights.kShared) __syncthreads();
    for (int32_t turn = 0; turn < turns.all; ++turn) {
        if (turn % S == 0) {
            bool overflows = false;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                mean[i] = mean_next[i];
                rstd[i] = rstd_next[i];
                overflows |= !(fabsf(mean[i] * rstd[i]) <= FLT_MAX);
            }
            careful = __any_sync(0xffffffffu, overflows);
            statistics(turn + S);
        }
        ahead.wait(p.stages);
        Pairs<V> xh[R][K], gw[R][K];
        float m[R], q[R], s[2 * R], xe[R], ge[R];              // xe, ge: xh and g * w of the edge's element
        // where the thread is beyond the row g is zero and its terms vanish
#pragma unroll
        for (int i = 0; i < R; ++i) {
            m[i] = __shfl_sync(0xffffffffu, mean[i], (lane & ~(S - 1)) + turn % S);
            q[i] = __shfl_sync(0xffffffffu, rstd[i], (lane & ~(S - 1)) + turn % S);
            s[2 * i] = s[2 * i + 1] = xe[i] = ge[i] = 0.0f;
            if (EDGE && edge.col >= 0) {
                xe[i] = (edge.get(edge_read, 0, i) - m[i]) * q[i];
                ge[i] = edge.get(edge_read, 1, i);
                edge_ab += ge[i];
                edge_aw = fmaf(ge[i], xe[i], edge_aw);
                ge[i] *= edge_w;
                s[2 * i] = ge[i];
                s[2 * i + 1] = ge[i] * xe[i];
            }
            const char *xs = ahead.at(0, i, x_row + i * hop_x), *gs = ahead.at(1, i, g_row + i * hop_g);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                Pairs<V> a = widen(ahead.get(xs, k)), t = widen(ahead.get(gs, k));
                a.shift_scale(-m[i], q[i]);
                ab[k].add(t);
                aw[k].fma(t, a);
                t.mul(weights.get(0, k));
                s[2 * i] += t.sum();
                s[2 * i + 1] += t.dot(a);
                if (HOLD) {
                    xh[i][k] = a;
                    gw[i][k] = t;
                }
            }
            if (careful) {
                constexpr int kTimes = !HOLD && kShared<T, L, V, K, EDGE> ? 1 : K;         // a rare loop: no registers for it
                s[2 * i + 1] = ge[i] * xe[i];
#pragma unroll kTimes
                for (int k = 0; k < K; ++k) {
                    Pairs<V> a, t;
                    if constexpr (HOLD) {
                        a = xh[i][k];
                        t = gw[i][k];
                    } else {
                        a = widen(ahead.get(xs, k));
                        t = widen(ahead.get(gs, k));
                        a.shift_scale(-m[i], q[i]);
                        t.mul(weights.get(0, k));
                    }
                    if (first + k * step < n_vec) s[2 * i + 1] += t.dot(a);
                }
            }
        }
        float s1[R], s2[R];
        if constexpr (L <= 0) {
            const float2 t = block_sum2(s[0], s[1], slots[turn & 1]);
            s1[0] = t.x * inverse;
            s2[0] = t.y * inverse;
        } else {
            const float mine = spread_sums<L, 2 * R>(s, first) * inverse;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                s1[i] = spread_get<L, 2 * R>(mine, 2 * i, lane);
                s2[i] = spread_get<L, 2 * R>(mine, 2 * i + 1, lane);
            }
        }
        edge_read = edge.next(edge_read);
        if (HOLD) {
            ahead.template done<false>();
            issue(turn + p.stages);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const bool live = turn < turns.live[i];
            const char *xs = ahead.at(0, i, x_row + i * hop_x), *gs = ahead.at(1, i, g_row + i * hop_g);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                Pairs<V> a, t;
                if constexpr (HOLD) {
                    a = xh[i][k];
                    t = gw[i][k];
                } else {
                    a = widen(ahead.get(xs, k));
                    t = widen(ahead.get(gs, k));
                    a.shift_scale(-m[i], q[i]);
                    t.mul(weights.get(0, k));
                }
                a.affine(-s2[i], -s1[i]);
                a.add(t);
                a.mul_all(q[i]);
                hagr::Vec<T, V> o;
                o.set(a.v);
                if (live && first + k * step < n_vec) o.store(y + i * hop_y + head_bytes, first + k * step);
            }
            if (EDGE && live && edge.col >= 0) store1<T>(y + i * hop_y, edge.col, q[i] * (ge[i] - fmaf(xe[i], s2[i], s1[i])));
        }
        if (!HOLD) {
            ahead.template done<true>();
            issue(turn + p.stages);
        }
        x_row += step_x;
        g_row += step_g;
        y += step_y;
    }
    hagr::wait_copies<0>();
    if (!p.partial) return;
    if constexpr (L <= 0) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (first + k * step >= n_vec) continue;
                const int32_t c = head + (first + k * step) * V + j;
                leave_param(p, 0, c, aw[k].v[j]);
                leave_param(p, 1, c, ab[k].v[j]);
            }
        if (EDGE && edge.col >= 0) {
            leave_param(p, 0, edge.col, edge_aw);
            leave_param(p, 1, edge.col, edge_ab);
        }
    } else {
        // groups of the warp, then warps of the block, in a fixed order
#pragma unroll
        for (int o = S; o < 32; o <<= 1)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    aw[k].v[j] += __shfl_xor_sync(0xffffffffu, aw[k].v[j], o);
                    ab[k].v[j] += __shfl_xor_sync(0xffffffffu, ab[k].v[j], o);
                }
        constexpr int C = S * K * V + (EDGE ? 2 * V : 0);
        float *joined = reinterpret_cast<float *>(raw);        // [warps][2][C], over the ring
        const int warp = threadIdx.x >> 5;
        __syncthreads();
        if (lane < S)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (first + k * S >= n_vec) continue;
                    joined[(warp * 2 + 0) * C + head + (first + k * S) * V + j] = aw[k].v[j];
                    joined[(warp * 2 + 1) * C + head + (first + k * S) * V + j] = ab[k].v[j];
                }
        if (EDGE && edge.col >= 0) {
            joined[(warp * 2 + 0) * C + edge.col] = edge_aw;
            joined[(warp * 2 + 1) * C + edge.col] = edge_ab;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * C; c += blockDim.x) {
            const int which = c / C, col = c - which * C;
            if (col >= p.D) continue;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kThreads<L> / 32; ++w) v += joined[w * 2 * C + c];
            leave_param(p, which, col, v);
        }
    }
}

// gw and gb from the parts: a block takes 32 columns of [gw | gb], its 32 warps every 32nd part each.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps) norm_params_join_kernel(const NormArgs p) {
    hagk::pdl_launch_dependents();
    __shared__ float sum[kJoinWarps][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    hagk::pdl_wait();
    float s = 0.0f;
    if (c < 2 * int64_t(p.D)) {
#pragma unroll 8
        for (int q = warp; q < p.parts; q += kJoinWarps) s += __ldcg(p.partial + int64_t(q) * 2 * p.D + c);
    }
    sum[warp][lane] = s;
    __syncthreads();
    s = hagr::warp_sum(sum[lane][warp]);                       // column `warp` of this block
    const int64_t k = int64_t(blockIdx.x) * 32 + warp;
    if (lane == 0 && k < 2 * int64_t(p.D)) {
        void *to = k < p.D ? p.gw : p.gb;
        if (to) store_param(to, p.w_bf16, k < p.D ? k : k - p.D, s);
    }
}

constexpr int kParts = 64;                // of the kernels for rows of any width
constexpr int kSms = 148;
constexpr int kLeastParts = 8;            // the number of parts is a multiple of the hop, 8 at most
constexpr int kSmShared = 227 * 1024;     // shared memory of an SM that blocks can use, and of one block
constexpr int kMostShared = kSmShared - 1024;

cudaError_t launch(void (*kernel)(NormArgs), dim3 grid, unsigned threads, size_t shared, const NormArgs &p, cudaStream_t s) {
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

// Parts of gw and gb, i.e. blocks of the other kernels, at most: the wider the rows, the fewer blocks fit an SM.
int most_parts(int32_t D) { return kSms * std::max(1, std::min(8, 16384 / D)); }

// How many blocks of the kernel the device runs at once (asked once per kernel and block size).
int resident_blocks(void (*kernel)(NormArgs), unsigned threads, size_t shared) {
    int per_sm = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, int(threads), shared) != cudaSuccess || per_sm < 1) {
        cudaGetLastError();
        per_sm = 1;
    }
    return per_sm * kSms;
}

// Values of a gradient that one block takes alone: 34 x 64 2.8 us, two launches 5; 64 x 1024 would be 15 us, two
// launches 8.
constexpr int64_t kFewValues = 16384;

// Lets a kernel use all the shared memory of the current device's SMs (once per kernel and device).
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

template <typename T, int V, int L, int K, bool BWD, bool EDGE>
cudaError_t launch_rows(NormArgs &p, cudaStream_t s) {
    constexpr int R = BWD ? kBwdRows<T, L, V, K> : kFwdTurn<T, L, V, K, EDGE>, OPS = BWD ? 2 : 1;
    constexpr auto kernel = BWD ? norm_bwd_kernel<T, V, L, K, EDGE> : norm_fwd_kernel<T, V, L, K, EDGE>;
    cudaError_t err = allow_shared<kernel>();
    if (err != cudaSuccess) return err;
    const int threads = L <= 0 ? ((p.D / V + K - 1) / K + 31) / 32 * 32 : kThreads<L>;
    const size_t params = Params<V, K, BWD ? 1 : 2, kShared<T, L, V, K, EDGE>>::bytes(L <= 0 ? threads : L);
    size_t stage;
    if constexpr (kRing<T, V>) stage = size_t(Ahead<T, V, K, R, OPS, L>::kStage) * threads;
    else stage = size_t(OPS) * R * Ahead<T, V, K, R, OPS, L>::row_bytes(L > 0 ? L : threads) * (L > 0 ? threads / (L > 0 ? L : 1) : 1);
    const size_t edges = EDGE ? size_t(OPS) * R * 4 * threads : 0;        // of a stage
    // as many stages as leave room for the blocks that the registers allow
    const int blocks = L <= 0 ? std::max(1, std::min(8, 768 / threads)) : BWD || !kRing<T, V> ? 2 : kFwdBlocks<L, V, K, EDGE>;
    p.stages = L <= 0 ? kBlockStages : BWD ? kBwdStages : kFwdStages;
    while (p.stages > 1 && (params + p.stages * (stage + edges) + 1024) * blocks > size_t(kSmShared)) --p.stages;
    p.edge_at = int32_t(params + p.stages * stage);
    size_t shared = params + p.stages * (stage + edges);
    if (BWD && L > 0) shared = std::max(shared, size_t(threads / 32) * 2 * ((L > 0 ? L : 0) * K * V + (EDGE ? 2 * V : 0)) * 4);
    if (shared > size_t(kMostShared)) return cudaErrorInvalidConfiguration;
    static std::atomic<int> resident[kMostThreads / 32 + 1];
    int most = resident[threads / 32].load(std::memory_order_relaxed);
    if (most == 0) resident[threads / 32].store(most = resident_blocks(kernel, threads, shared), std::memory_order_relaxed);
    most = std::min(most, kRing<T, V> && L > 0 ? kSms * (BWD ? 2 : kFwdBlocks<L, V, K, EDGE>) : most_parts(p.D));
    const int64_t rows_per_block = L <= 0 ? 1 : int64_t(threads / 32) * (32 / (L <= 0 ? 32 : L)) * R;
    int64_t grid = std::max<int64_t>(1, std::min<int64_t>((p.n + rows_per_block - 1) / rows_per_block, most));
    // one block does without the second launch
    if (BWD && L > 0 && p.partial && p.n * p.D <= kFewValues) grid = 1;
    if (EDGE && L <= 0) grid = std::max<int64_t>(grid / p.hop, 1) * p.hop;        // the groups are a multiple of the hop
    p.parts = int32_t(grid);
    return launch(kernel, dim3(unsigned(grid)), unsigned(threads), shared, p, s);
}

// Rows of up to 1024 elements (narrow vectors: 512) go to a warp or a part of one, rows of up to
// 1024 * kPerThread to a block.  A warp needs no barrier: 65 536 x 1024 bf16 forward takes 54 us with a warp per row and
// 96 with a block of 64 threads.  Narrow vectors are bound by the instructions around a row, so that a warp takes several
// rows and a lane several vectors: 1 175 089 x 13 bf16 runs forward in 38 us with 8 lanes and two vectors each, in 59
// with 16 lanes and one, in 121 with 32 (backward 65, 96, 185); 1 175 089 x 29 fp32 in 61 with 8 lanes, 69 with 16, 115
// with 32; 775 089 x 49 bf16 in 66 with 16 lanes, 71 with 8, 96 with 32.  Wide vectors are near the memory's rate with
// one each, but where they leave most of the lanes without one: 1 047 213 x 8 bf16 in 20 us with 4 lanes, 41 with 8
// (backward 35 and 60), 32 bf16 in 25 and 42.  Narrow rows of 280 bf16 backward, 123 218 of them, take 97 us with 12
// columns per lane, 117 with 16 and 123 with a block per row (forward 60, 75 with 16); 500 fp32 130 with 16, 140 with a
// block; 223 218 x 150 fp32 86 with 6, 132 with 8; 423 218 x 80 fp32 92 with 3, 123 with 4.
// Rows of more columns are read one element at a time: 4000 x 32 768 bf16 614 us forward and 872 backward.
constexpr int kPerThread = 16;
template <typename T, int V, bool BWD, bool EDGE = false>
cudaError_t launch_width(NormArgs &p, cudaStream_t s) {
    const int32_t n_vec = p.D / V;
    if constexpr (!EDGE) {
        if (n_vec <= 4) return launch_rows<T, V, 4, 1, BWD, EDGE>(p, s);
        if constexpr (kRing<T, V>) {
            if (n_vec <= 8) return launch_rows<T, V, 8, 1, BWD, EDGE>(p, s);
            if (n_vec <= 16) return launch_rows<T, V, 16, 1, BWD, EDGE>(p, s);
        } else {
            if (n_vec <= 8) return launch_rows<T, V, 4, 2, BWD, EDGE>(p, s);
            if (n_vec <= 16) return launch_rows<T, V, 8, 2, BWD, EDGE>(p, s);
            if (n_vec <= 32) return launch_rows<T, V, 8, 4, BWD, EDGE>(p, s);
            if (n_vec <= 64) return launch_rows<T, V, 16, 4, BWD, EDGE>(p, s);
        }
    }
    if (n_vec <= 32) return launch_rows<T, V, 32, 1, BWD, EDGE>(p, s);
    if (n_vec <= 64) return launch_rows<T, V, 32, 2, BWD, EDGE>(p, s);
    constexpr int kMost = (kRing<T, V> && !EDGE ? 32 : 16) / V;       // vectors per lane of a warp
    if constexpr (!kRing<T, V>)
        if (n_vec <= 96) return launch_rows<T, V, 32, 3, BWD, EDGE>(p, s);
    if constexpr (kMost >= 4)
        if (n_vec <= 128) return launch_rows<T, V, 32, 4, BWD, EDGE>(p, s);
    if constexpr (kMost >= 8 && !kRing<T, V>)
        if (n_vec <= 192) return launch_rows<T, V, 32, 6, BWD, EDGE>(p, s);
    if constexpr (kMost >= 8)
        if (n_vec <= 256) return launch_rows<T, V, 32, 8, BWD, EDGE>(p, s);
    if constexpr (kMost >= 16 && !kRing<T, V>)
        if (n_vec <= 384) return launch_rows<T, V, 32, 12, BWD, EDGE>(p, s);
    if constexpr (kMost >= 16)
        if (n_vec <= 512) return launch_rows<T, V, 32, 16, BWD, EDGE>(p, s);
    constexpr int kFew = (kRing<T, V> || !BWD ? kPerThread : 8) / V;
    if (n_vec <= kFewThreads * kFew) return launch_rows<T, V, -1, kFew, BWD, EDGE>(p, s);
    // narrow vectors backward, 8 columns per thread as long as they suffice: 2521 x 7944 fp32 68 us, with 16 105
    if constexpr (BWD && !kRing<T, V>)
        if (n_vec <= kMostThreads * kFew) return launch_rows<T, V, 0, kFew, BWD, EDGE>(p, s);
    return launch_rows<T, V, 0, kPerThread / V, BWD, EDGE>(p, s);
}

constexpr int32_t kMostInBlock = kMostThreads * kPerThread;

constexpr int kEdgeBytes = 256;          // of a row, at least, for vectors with edges

// Whether every row of x, y and g has the same distance from a 16-byte boundary in all of them.
bool same_misalignment(const NormArgs &p, int elem) {
    auto as_x = [&](const void *q, int64_t ld) {
        return (reinterpret_cast<uintptr_t>(q) - reinterpret_cast<uintptr_t>(p.x)) % 16 == 0 && (ld - p.ld_x) * elem % 16 == 0;
    };
    return as_x(p.y, p.ld_y) && (!p.g || as_x(p.g, p.ld_g));
}

template <typename T, bool BWD>
cudaError_t launch_typed(NormArgs &p, cudaStream_t s) {
    const int e = int(sizeof(T)), we = p.w_bf16 ? 2 : 4;
    const hagr::Operand ops[] = {{p.x, p.ld_x, e}, {p.y, p.ld_y, e}, {p.g, p.ld_g, e}};
    int v = hagr::vector_elems(16 / e, p.D, ops);
    p.hop = 1;
    if (v < 16 / e && p.D * e >= kEdgeBytes && same_misalignment(p, e)) {
        p.w_vectors = 0;
        while ((p.ld_x * e * p.hop) % 16 != 0) p.hop *= 2;
        return launch_width<T, 16 / e, BWD, true>(p, s);
    }
    if (v < 16 / e) v = sizeof(T) == 2 && v > 1 ? 2 : 1;
    const hagr::Operand params[] = {{p.w, 0, we}, {p.b, 0, we}};
    p.w_vectors = hagr::vector_elems(v, p.D, params) == v;
    if (v == 16 / e) return launch_width<T, 16 / e, BWD>(p, s);
    if constexpr (sizeof(T) == 2)
        if (v == 2) return launch_width<T, 2, BWD>(p, s);
    return launch_width<T, 1, BWD>(p, s);
}

bool dtype_ok(hag_dtype d) { return d == HAG_F32 || d == HAG_BF16; }
int elem_size(hag_dtype d) { return d == HAG_F32 ? 4 : 2; }

struct Need {
    const void *p;
    int64_t ld;
    bool rows;      // an n x D matrix of `dtype` (else a vector of the parameters' type)
    bool out;
};

template <int N>
hag_status norm_check(int64_t n, int32_t D, hag_dtype dtype, hag_dtype w_dtype, const Need (&a)[N]) {
    if (!dtype_ok(dtype) || !dtype_ok(w_dtype)) return HAG_ERR_DTYPE;
    if (n < 0 || D <= 0) return HAG_ERR_ARG;
    if (D > (1 << 30)) return HAG_ERR_TOO_LARGE;
    for (const Need &x : a) {
        if (!x.rows) continue;
        if (x.ld < 0 || (x.out && n > 1 && x.ld < D)) return HAG_ERR_ARG;
        if (!x.p && n > 0) return HAG_ERR_NULL;
    }
    for (const Need &x : a)
        if (!hagr::element_aligned(x.p, x.rows ? elem_size(dtype) : elem_size(w_dtype))) return HAG_ERR_ALIGN;
    for (const Need &x : a)              // in place row by row is fine; the same start with other rows is not
        for (const Need &y : a)
            if (n > 1 && x.rows && y.rows && y.out && x.p == y.p && x.ld != y.ld) return HAG_ERR_ARG;
    return HAG_OK;
}

}  // namespace

extern "C" hag_status hag_layer_norm_fwd(int64_t n, int32_t D, hag_dtype dtype, const void *x, int64_t ld_x, const void *weight,
                                         const void *bias, hag_dtype weight_dtype, float eps, void *y, int64_t ld_y, float *mean,
                                         float *rstd, void *cuda_stream) {
    const Need need[] = {{x, ld_x, true, false}, {y, ld_y, true, true}, {weight, 0, false, false}, {bias, 0, false, false}};
    const hag_status st = norm_check(n, D, dtype, weight_dtype, need);
    if (st != HAG_OK) return st;
    if (!(eps >= 0.0f)) return HAG_ERR_ARG;
    if (!hagr::element_aligned(mean, 4) || !hagr::element_aligned(rstd, 4)) return HAG_ERR_ALIGN;
    if (n == 0) return HAG_OK;
    NormArgs p{};
    p.n = n; p.D = D; p.w_bf16 = weight_dtype == HAG_BF16;
    p.x = x; p.ld_x = ld_x; p.w = weight; p.b = bias; p.y = y; p.ld_y = ld_y; p.mean = mean; p.rstd = rstd; p.eps = eps;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err;
    if (D <= kMostInBlock)
        err = dtype == HAG_F32 ? launch_typed<float, false>(p, s) : launch_typed<__nv_bfloat16, false>(p, s);
    else
        err = launch(dtype == HAG_F32 ? norm_fwd_any_kernel<float> : norm_fwd_any_kernel<__nv_bfloat16>,
                     dim3(unsigned(std::min<int64_t>(n, kSms * 8))), kRowThreads, 0, p, s);
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}

extern "C" size_t hag_layer_norm_bwd_workspace_bytes(int64_t n, int32_t D) {
    if (n < 0 || D <= 0) return 0;
    return size_t(std::max<int64_t>(std::min<int64_t>(D <= kMostInBlock ? most_parts(D) : kParts, n), kLeastParts)) * 2 * size_t(D) * 4;
}

extern "C" hag_status hag_layer_norm_bwd(int64_t n, int32_t D, hag_dtype dtype, const void *grad_y, int64_t ld_grad_y, const void *x,
                                         int64_t ld_x, const float *mean, const float *rstd, const void *weight,
                                         hag_dtype weight_dtype, void *grad_x, int64_t ld_grad_x, void *grad_weight, void *grad_bias,
                                         void *workspace, void *cuda_stream) {
    const Need need[] = {{grad_y, ld_grad_y, true, false}, {x, ld_x, true, false}, {grad_x, ld_grad_x, true, true},
                         {weight, 0, false, false}, {grad_weight, 0, false, true}, {grad_bias, 0, false, true}};
    const hag_status st = norm_check(n, D, dtype, weight_dtype, need);
    if (st != HAG_OK) return st;
    if (n > 0 && (!mean || !rstd)) return HAG_ERR_NULL;
    if (!hagr::element_aligned(mean, 4) || !hagr::element_aligned(rstd, 4)) return HAG_ERR_ALIGN;
    const bool params = grad_weight || grad_bias;
    if (params && !workspace) return HAG_ERR_WORKSPACE;
    if (!hagl::aligned16(workspace)) return HAG_ERR_ALIGN;
    NormArgs p{};
    p.n = n; p.D = D; p.w_bf16 = weight_dtype == HAG_BF16;
    p.x = x; p.ld_x = ld_x; p.g = grad_y; p.ld_g = ld_grad_y; p.w = weight; p.y = grad_x; p.ld_y = ld_grad_x;
    p.mean_in = mean; p.rstd_in = rstd; p.partial = static_cast<float *>(workspace); p.gw = grad_weight; p.gb = grad_bias;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err = cudaSuccess;
    const bool f32 = dtype == HAG_F32;
    const dim3 join_grid(unsigned((2 * int64_t(D) + 31) / 32));
    if (!params) p.partial = nullptr;
    if (D <= kMostInBlock) {
        if (n > 0 || params) err = f32 ? launch_typed<float, true>(p, s) : launch_typed<__nv_bfloat16, true>(p, s);
        if (params && p.parts > 1 && err == cudaSuccess) err = launch(norm_params_join_kernel, join_grid, 32 * kJoinWarps, 0, p, s);
    } else {
        if (params) {      // first: grad_x may take the place of grad_y or x
            p.parts = int(std::min<int64_t>(std::max<int64_t>((n + kStripRows - 1) / kStripRows, 1), kParts));
            err = launch(f32 ? norm_params_any_kernel<float> : norm_params_any_kernel<__nv_bfloat16>,
                         dim3(unsigned((D + 31) / 32), unsigned(p.parts)), 32 * kStripRows, 0, p, s);
            if (err == cudaSuccess) err = launch(norm_params_join_kernel, join_grid, 32 * kJoinWarps, 0, p, s);
        }
        if (err == cudaSuccess && n > 0)
            err = launch(f32 ? norm_bwd_any_kernel<float> : norm_bwd_any_kernel<__nv_bfloat16>,
                         dim3(unsigned(std::min<int64_t>(n, kSms * 8))), kRowThreads, 0, p, s);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return HAG_ERR_CUDA; }
    return HAG_OK;
}
