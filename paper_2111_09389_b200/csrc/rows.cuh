// Rows of logits, read once: 16-byte accesses at any alignment of the row, the running maximum and sums of a softmax, and their
// joining across lanes, warps and the CTAs of a cluster.  Not part of the ABI.
//
// A row of V elements is seen as the 16-byte words of memory that lie wholly inside it, and fewer than 16 bytes before and behind them (the
// edges), which are read element by element: nothing outside the row is touched, and a row may start anywhere.
#pragma once
#include <math.h>
#include "dtypes.cuh"

namespace lpdt {

constexpr float kLowest = -3.402823466e38f, kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }     // 2^x, 2 ulp
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ uint32_t rows_cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t rows_cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void rows_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void rows_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void rows_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// To the same place of shared memory in the CTA of that rank.
__device__ __forceinline__ void st_peer_u64(void *local, uint32_t rank, unsigned long long v) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(rank));
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}

template <typename T>
struct Row {
    static constexpr int VE = 16 / (int)sizeof(T), EDGES = 2 * (VE - 1);
    const T *base;           // of word 0, 16-byte aligned
    int head, V, words;      // elements before word 0; words
    __device__ __forceinline__ Row(const T *p, int V_) : V(V_) {
        head = (int)((16 - ((uintptr_t)p & 15)) % 16 / sizeof(T));
        if (head > V) head = V;
        base = p + head;
        words = (V - head) / VE;
    }
    __device__ __forceinline__ uint4 load(int w) const { return reinterpret_cast<const uint4 *>(base)[w]; }
    __device__ __forceinline__ uint4 load_last(int w) const { return __ldcs(reinterpret_cast<const uint4 *>(base) + w); }    // not to be read again
    __device__ __forceinline__ int index(int w) const { return w * VE + head; }          // of the word's first element
    // Index of the i-th element of the edges (i < EDGES), -1 where there is none.
    __device__ __forceinline__ int edge(int i) const {
        if (i < VE - 1) return i < head ? i : -1;
        const int v = head + words * VE + i - (VE - 1);
        return v < V ? v : -1;
    }
    __device__ __forceinline__ T at(int i) const { return (base - head)[i]; }
};
template <typename T> __device__ __forceinline__ void unpack_vec(const uint4 &v, float *f) {
    constexpr int PER = 4 / (int)sizeof(T);
    unpack_word(v.x, f, T());
    unpack_word(v.y, f + PER, T());
    unpack_word(v.z, f + 2 * PER, T());
    unpack_word(v.w, f + 3 * PER, T());
}

template <typename T> __device__ __forceinline__ uint4 pack_vec(const float *f) {
    constexpr int PER = 4 / (int)sizeof(T);
    return make_uint4(pack_word(f, T()), pack_word(f + PER, T()), pack_word(f + 2 * PER, T()), pack_word(f + 3 * PER, T()));
}

// The largest of a word's elements, NaN passed over; a word of nothing but NaN may answer NaN.
__device__ __forceinline__ float vec_max_of(const uint4 &v, float) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
__device__ __forceinline__ float vec_max_of(const uint4 &v, __nv_bfloat16) {
    const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(&v);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float vec_max_of(const uint4 &v, __half) {
    const __half2 *h = reinterpret_cast<const __half2 *>(&v);
    const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
template <typename T> __device__ __forceinline__ float vec_max(const uint4 &v) { return vec_max_of(v, T()); }

// Running sums relative to the maximum so far: s = sum 2^t, w = sum 2^t * t with t = (x - m) * c, c = log2(e) / temperature.
// A value that is -inf, or far below m, counts as t = -10000 where w is taken: 2^t = 0 and no 0 * inf.  NaN passes through max_nan and
// stays.  Without w, 2^-inf = 0 is enough (4 x 1024 x 131072 distilled: 443 -> 429 us, with the second pass two values at a time).
// m starts at the lowest float, so a row of nothing but -inf ends with s = 0, one of lowest floats is uniform.
constexpr float kFar = -10000.f;
struct Stats {
    float m, s, w;
    __device__ __forceinline__ void reset() { m = kLowest; s = 0.f; w = 0.f; }
    __device__ __forceinline__ void raise(float to, float c) {      // to >= m
        const float t = max_nan((m - to) * c, kFar), r = ex2(t);
        w = r * (w + t * s);
        s *= r;
        m = to;
    }
};
// The largest of the lanes' numbers.
__device__ __forceinline__ float warp_max_f(float v) {
    const uint32_t b = __float_as_uint(v), o = __reduce_max_sync(0xffffffffu, b ^ ((uint32_t)((int)b >> 31) | 0x80000000u));
    return __uint_as_float(o ^ ((uint32_t)(~(int)o >> 31) | 0x80000000u));
}
// Joins the lanes' sums: to their maximum first, then they add.
__device__ __forceinline__ void warp_join(Stats &a, float c) {
    a.raise(warp_max_f(a.m), c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.w += __shfl_xor_sync(0xffffffffu, a.w, o);
    }
}
// Adds a word's elements, two at a time; the maximum has been raised to cover them.
template <int N, bool W> __device__ __forceinline__ void accumulate(Stats &a, const float *f, float c) {
    const F2 minus_m = pack2(-a.m, -a.m), c2 = pack2(c, c);
    F2 s = pack2(a.s, 0.f), w = pack2(a.w, 0.f);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        float t0, t1;
        unpack2(mul2(add2(pack2(f[i], f[i + 1]), minus_m), c2), t0, t1);
        if (W) {
            t0 = max_nan(t0, kFar);
            t1 = max_nan(t1, kFar);
        }
        const F2 e = pack2(ex2(t0), ex2(t1));
        s = add2(s, e);
        if (W) w = fma2(e, pack2(t0, t1), w);
    }
    float s0, s1;
    unpack2(s, s0, s1);
    a.s = s0 + s1;
    if (W) {
        unpack2(w, s0, s1);
        a.w = s0 + s1;
    }
}

// Bits that order like the values, -0 like +0 (NaN is not asked).
__device__ __forceinline__ uint32_t order_bits(float f) {
    const uint32_t b = __float_as_uint(f + 0.f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_order_bits(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }
// Larger values first, of equal ones the lower index.
__device__ __forceinline__ unsigned long long top_key(float f, int index) {
    return ((unsigned long long)order_bits(f) << 32) | (0xffffffffu - (uint32_t)index);
}
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)(0xffffffffu - (uint32_t)k); }
__device__ __forceinline__ float key_value(unsigned long long k) { return from_order_bits((uint32_t)(k >> 32)); }

static inline bool temperature_ok(float t) { return t >= 1e-30f && t <= 1e30f; }

// CTAs of a cluster that share a row: as many (a power of two, at most 8) as leave every SM `per_sm` of them, each with at least
// `least` bytes of the row.
static inline int row_share(int64_t rows, int64_t row_bytes, int per_sm, int64_t least) {
    int cs = 1;
    while (cs < 8 && rows * cs * 2 <= (int64_t)kNumSMs * per_sm && row_bytes / (cs * 2) >= least) cs *= 2;
    return cs;
}

}  // namespace lpdt
