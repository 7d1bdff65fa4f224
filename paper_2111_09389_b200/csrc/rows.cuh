// Rows of logits, read once: 16-byte accesses at any alignment of the row, the running maximum and sums of a softmax, and their
// joining across lanes, warps and the CTAs of a cluster.  Not part of the ABI.
//
// A row of V elements at p is seen as the 16-byte words of memory that it touches: position = index + head, head = elements of the
// first word before the row.  A first or last word that holds others' elements is read element by element, so nothing outside the
// row is touched and a row stride of any parity costs two short accesses per row.
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
// The value at the same place of shared memory in the CTA of that rank.
__device__ __forceinline__ unsigned long long ld_peer_u64(const void *local, uint32_t rank) {
    uint32_t a;
    unsigned long long v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(rank));
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}

template <typename T>
struct Row {
    static constexpr int VE = 16 / (int)sizeof(T);
    const T *base;           // 16-byte aligned; position 0
    int head, V, words;      // words of 16 bytes that the row touches
    __device__ __forceinline__ Row(const T *p, int V_) : V(V_) {
        head = (int)(((uintptr_t)p & 15) / sizeof(T));
        base = p - head;
        words = (int)(((long long)head + V + VE - 1) / VE);
    }
    __device__ __forceinline__ bool whole(int w) const { return (w > 0 || head == 0) && (long long)(w + 1) * VE <= (long long)head + V; }
    __device__ __forceinline__ bool holds(long long pos) const { return pos >= head && pos < (long long)head + V; }
    // Elements of word w as bits; those outside the row are `fill`.
    __device__ __forceinline__ uint4 load(int w, T fill) const {
        if (whole(w)) return reinterpret_cast<const uint4 *>(base)[w];
        union { uint4 v; T e[VE]; } u;
#pragma unroll
        for (int i = 0; i < VE; ++i) u.e[i] = holds((long long)w * VE + i) ? base[(long long)w * VE + i] : fill;
        return u.v;
    }
};
template <typename T> __device__ __forceinline__ void unpack_vec(const uint4 &v, float *f) {
    constexpr int PER = 4 / (int)sizeof(T);
    unpack_word(v.x, f, T());
    unpack_word(v.y, f + PER, T());
    unpack_word(v.z, f + 2 * PER, T());
    unpack_word(v.w, f + 3 * PER, T());
}

// Running sums relative to the maximum so far: s = sum 2^t, w = sum 2^t * t with t = (x - m) * c, c = log2(e) / temperature.
// A value that is -inf, or far below m, counts as t = -10000: 2^t = 0 and no 0 * inf.  NaN passes through max_nan and stays.
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
    __device__ __forceinline__ void join(const Stats &o, float c) {
        Stats b = o;
        const float to = fmaxf(m, b.m);
        raise(to, c);
        b.raise(to, c);
        s += b.s;
        w += b.w;
    }
};
__device__ __forceinline__ Stats shfl_xor(const Stats &a, int o) {
    Stats b;
    b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
    b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
    b.w = __shfl_xor_sync(0xffffffffu, a.w, o);
    return b;
}
__device__ __forceinline__ void warp_join(Stats &a, float c) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a.join(shfl_xor(a, o), c);
}
// Adds a word's elements; the maximum has been raised to cover them.
template <int N, bool W> __device__ __forceinline__ void accumulate(Stats &a, const float *f, float c) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = max_nan((f[i] - a.m) * c, kFar), e = ex2(t);
        a.s += e;
        if (W) a.w = fmaf(e, t, a.w);
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
