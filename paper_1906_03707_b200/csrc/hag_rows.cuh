// Row vectors shared by the kernels around the aggregation (embedding, layer norm, clipping, root-mean-square norm, AdamW),
// and sums and arithmetic on pairs of their elements: V elements of type T as one load or store of V * sizeof(T) bytes (two of 16 bytes where that is 32), kept as raw words
// while in flight and widened to fp32 when used.  V is the largest power of two that the width, the row
// strides and the pointers of a call allow (vector_elems), so any width and any element-aligned pointer works.
// Loads are coherent (ld.global, never .nc): under programmatic dependent launch the kernel that wrote the
// data may still be alive when the reader starts.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace hagr {

template <int B> struct Words;      // B bytes
template <> struct Words<2> { uint16_t w[1]; };
template <> struct Words<4> { uint32_t w[1]; };
template <> struct Words<8> { uint32_t w[2]; };
template <> struct Words<16> { uint32_t w[4]; };
template <> struct Words<32> { uint32_t w[8]; };

// Cache operator of a load: kKeep leaves the line in the L2, kOnce marks it evict-first (data that is read once must
// not push out rows that are read again), kNear also keeps it in the SM's own L1 (rows that the same SM reads again).
enum CacheOp { kKeep, kOnce, kNear };

template <CacheOp OP, typename W>
__device__ __forceinline__ W load_word(const W *p) {
    if constexpr (OP == kOnce) return __ldcs(p);
    else if constexpr (OP == kNear) return __ldca(p);
    else return __ldcg(p);
}

template <CacheOp OP, int B>
__device__ __forceinline__ Words<B> load_words(const void *p) {
    Words<B> r;
    if constexpr (B == 2) {
        r.w[0] = load_word<OP>(static_cast<const uint16_t *>(p));
    } else if constexpr (B == 4) {
        r.w[0] = load_word<OP>(static_cast<const uint32_t *>(p));
    } else if constexpr (B == 8) {
        const uint2 q = load_word<OP>(static_cast<const uint2 *>(p));
        r.w[0] = q.x; r.w[1] = q.y;
    } else {
#pragma unroll
        for (int h = 0; h < B / 16; ++h) {
            const uint4 *s = static_cast<const uint4 *>(p) + h;
            const uint4 q = load_word<OP>(s);
            r.w[4 * h] = q.x; r.w[4 * h + 1] = q.y; r.w[4 * h + 2] = q.z; r.w[4 * h + 3] = q.w;
        }
    }
    return r;
}

// kOnce: written once and not read again soon (evict-first); else an ordinary store.
template <CacheOp OP, typename W>
__device__ __forceinline__ void store_word(W *p, W v) {
    if constexpr (OP == kOnce) __stcs(p, v);
    else *p = v;
}

template <CacheOp OP, int B>
__device__ __forceinline__ void store_words(void *p, const Words<B> &r) {
    if constexpr (B == 2) {
        store_word<OP>(static_cast<uint16_t *>(p), r.w[0]);
    } else if constexpr (B == 4) {
        store_word<OP>(static_cast<uint32_t *>(p), r.w[0]);
    } else if constexpr (B == 8) {
        store_word<OP>(static_cast<uint2 *>(p), make_uint2(r.w[0], r.w[1]));
    } else {
#pragma unroll
        for (int h = 0; h < B / 16; ++h)
            store_word<OP>(static_cast<uint4 *>(p) + h, make_uint4(r.w[4 * h], r.w[4 * h + 1], r.w[4 * h + 2], r.w[4 * h + 3]));
    }
}

template <typename T, int V>
struct Vec {
    static constexpr int kBytes = V * int(sizeof(T));
    Words<kBytes> raw;

    template <CacheOp OP>
    __device__ __forceinline__ void load(const void *row, size_t i) {        // elements i * V .. of the row
        raw = load_words<OP, kBytes>(static_cast<const char *>(row) + i * kBytes);
    }
    template <CacheOp OP = kKeep>
    __device__ __forceinline__ void store(void *row, size_t i) const {
        store_words<OP, kBytes>(static_cast<char *>(row) + i * kBytes, raw);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int k = 0; k < int(sizeof(raw.w) / sizeof(raw.w[0])); ++k) raw.w[k] = 0;
    }
    __device__ __forceinline__ float get(int j) const {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(raw.w[j]);
        } else if constexpr (V == 1) {
            return __uint_as_float(uint32_t(raw.w[0]) << 16);
        } else {
            return (j & 1) ? __uint_as_float(raw.w[j / 2] & 0xffff0000u) : __uint_as_float(raw.w[j / 2] << 16);
        }
    }
    __device__ __forceinline__ void set(const float *v) {                    // one round-to-nearest per element
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < V; ++j) raw.w[j] = __float_as_uint(v[j]);
        } else if constexpr (V == 1) {
            raw.w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
        } else {
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                const __nv_bfloat162 q = __floats2bfloat162_rn(v[j], v[j + 1]);
                raw.w[j / 2] = *reinterpret_cast<const uint32_t *>(&q);
            }
        }
    }
};

// Asynchronous copy of 16 bytes from global to shared memory, straight past the registers.  A thread sees its own copies
// after wait_copies.
template <int B>
__device__ __forceinline__ void copy_async(void *shared, const void *global) {
    static_assert(B == 16, "");
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(uint32_t(__cvta_generic_to_shared(shared))), "l"(global) : "memory");
}
// The same, of which only the first `bytes` (1 to 16) are read; the rest is zeros.
__device__ __forceinline__ void copy_async_part(void *shared, const void *global, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(uint32_t(__cvta_generic_to_shared(shared))), "l"(global), "r"(bytes) : "memory");
}
// Four bytes, of which the first `bytes` (2 or 4) are read.
__device__ __forceinline__ void copy_async_word(void *shared, const void *global, int bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(uint32_t(__cvta_generic_to_shared(shared))), "l"(global), "r"(bytes) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

// Quotients by a divisor fixed per launch: multiply-high, add and shift (Granlund and Montgomery 1994), for
// dividends below 2^31.
struct Divisor {
    uint32_t d, mul, shift;
};
inline Divisor make_divisor(uint32_t d) {
    uint32_t s = 0;
    while ((uint64_t(1) << s) < d) ++s;
    const uint64_t m = ((uint64_t(1) << 32) * ((uint64_t(1) << s) - d)) / d + 1;
    return Divisor{d, uint32_t(m), s};
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Divisor &v) { return (__umulhi(n, v.mul) + n) >> v.shift; }

// One matrix of a call, as far as the vector width goes.
struct Operand {
    const void *p;
    int64_t ld;
    int elem;        // bytes per element
};

// The largest power of two V <= limit such that every operand can be read V elements at a time: V divides the width
// and the row strides, and the pointer is aligned to the V elements or to 16 bytes, whichever is less.
template <int N>
inline int vector_elems(int limit, int32_t D, const Operand (&ops)[N]) {
    int v = limit;
    auto fits = [&](int v_) {
        if (D % v_ != 0) return false;
        for (const Operand &o : ops) {
            if (!o.p) continue;
            const int bytes = v_ * o.elem < 16 ? v_ * o.elem : 16;
            if (o.ld % v_ != 0 || reinterpret_cast<uintptr_t>(o.p) % uintptr_t(bytes) != 0) return false;
        }
        return true;
    };
    while (v > 1 && !fits(v)) v /= 2;
    return v;
}

inline bool element_aligned(const void *p, int elem) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(elem) == 0; }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

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
    __device__ __forceinline__ void affine(float m, const Pairs &s) {                         // v = v * m + s
        each([&](int j) { put(j, __ffma2_rn(two(j), make_float2(m, m), s.two(j))); }, [&](int j) { v[j] = fmaf(v[j], m, s.v[j]); });
    }
    __device__ __forceinline__ void add_scaled(const Pairs &a, float m) {                     // v += a * m
        each([&](int j) { put(j, __ffma2_rn(a.two(j), make_float2(m, m), two(j))); }, [&](int j) { v[j] = fmaf(a.v[j], m, v[j]); });
    }
    // v = v / d, `inverse` an approximate reciprocal of d: the product's remainder, which a fused product gives exactly,
    // corrects it to the rounded quotient (Markstein 1990); a zero keeps its sign.
    __device__ __forceinline__ void divide(float d, float inverse) {
        const Pairs a = *this;
        mul_all(inverse);
        each([&](int j) {
                 const float2 rest = __ffma2_rn(two(j), make_float2(d, d), make_float2(-a.v[j], -a.v[j + 1]));
                 put(j, __ffma2_rn(rest, make_float2(-inverse, -inverse), two(j)));
             },
             [&](int j) { v[j] = fmaf(fmaf(v[j], d, -a.v[j]), -inverse, v[j]); });
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
__device__ __forceinline__ Pairs<V> widen(const Vec<T, V> &a) {
    Pairs<V> f;
#pragma unroll
    for (int j = 0; j < V; ++j) f.v[j] = a.get(j);
    return f;
}

// Waits until the oldest of the stages has arrived (a launch has fewer stages where a row fills the shared memory).
__device__ __forceinline__ void wait_oldest(int stages) {
    if (stages == 4) wait_copies<3>();
    else if (stages == 3) wait_copies<2>();
    else if (stages == 2) wait_copies<1>();
    else wait_copies<0>();
}

}  // namespace hagr
