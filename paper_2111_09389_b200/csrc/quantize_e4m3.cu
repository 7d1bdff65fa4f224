// lpdt_quantize_e4m3: 8-bit floats with a power-of-two scale for each block of 128 values.
//
// A block's scale is 2^e with e the least integer for which amax <= 448 * 2^e (448: the largest e4m3 value), so x * 2^-e is exact and
// the one rounding is the conversion's own (to nearest, halves to even).  amax is taken on the bits of |x|: as unsigned integers they
// order like the values, infinities and NaN above them, which marks a block that holds one.
//
// Memory is the bound: each value is read once and written as one byte per form.
#include "dtypes.cuh"

namespace lpdt {

constexpr int kBlk = 128;
constexpr uint32_t kInfBits = 0x7f800000u;

// The scale byte (e + 127; 255 = NaN) of a block whose largest |x| has these bits, and the factor 2^-e.
__device__ __forceinline__ uint32_t block_scale(uint32_t amax, float &inv) {
    if (amax >= kInfBits) { inv = __uint_as_float(0x7fc00000u); return 255u; }
    if (amax == 0u) { inv = 1.f; return 127u; }
    int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);     // 448 = 1.75 * 2^8
    if (e < -127) e = -127;                                    // subnormals among them
    inv = __uint_as_float((uint32_t)(127 - e) << 23);          // -e in -120 .. 127
    return (uint32_t)(e + 127);
}
// Two values as e4m3 bytes, `lo` in the lower one.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) { return e4m3x2(a, b) | (e4m3x2(c, d) << 16); }
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// NV consecutive elements at p, of which the first `have` exist (the others read 0); VEC: p is aligned to all of them.
template <typename T, int NV, bool VEC>
__device__ __forceinline__ void load_some(const T *__restrict__ p, int have, float *f) {
    constexpr int WORDS = NV * (int)sizeof(T) / 4, PER = 4 / (int)sizeof(T);
    if (VEC && have >= NV) {
        uint32_t w[WORDS];
        if constexpr (WORDS == 4) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            static_assert(WORDS == 2, "8 or 16 bytes");
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
            w[0] = v.x; w[1] = v.y;
        }
#pragma unroll
        for (int i = 0; i < WORDS; ++i) unpack_word(w[i], f + i * PER, T());
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) f[i] = i < have ? to_f32(p[i]) : 0.f;
    }
}

struct E4m3Args {
    const void *x;
    long long x_node, x_row;                      // strides in elements
    int rows, cols, nb, nbt;                      // blocks of a row, of a column
    uint8_t *q, *s, *qt, *st;
    int qp, sp, qtp, stp;                         // pitches in bytes
};

// Rows only.  128 / NV lanes hold a block, 16 bytes of the row each; U blocks in flight per lane.
template <typename T, bool VEC, int U>
__global__ void __launch_bounds__(256) quantize_e4m3_rows_kernel(const E4m3Args a, unsigned total) {
    constexpr int NV = 16 / (int)sizeof(T), L = kBlk / NV, PER_CTA = 256 / L;
    pdl_enter();
    const int k = threadIdx.x % L;
    unsigned blk = blockIdx.x * (PER_CTA * U) + threadIdx.x / L;
    float f[U][NV];
    unsigned row[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned at = blk + u * PER_CTA;
        row[u] = at / (unsigned)a.nb;             // over all nodes
        b[u] = at - row[u] * (unsigned)a.nb;
        const unsigned n = row[u] / (unsigned)a.rows, r = row[u] - n * (unsigned)a.rows;
        const int c = (int)b[u] * kBlk + k * NV;
        const T *p = (const T *)a.x + n * a.x_node + r * a.x_row + c;
        load_some<T, NV, VEC>(p, at < total ? a.cols - c : 0, f[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned at = blk + u * PER_CTA;
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) amax = max(amax, abs_bits(f[u][i]));
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        float inv;
        const uint32_t s = block_scale(amax, inv);
        if (at >= total) continue;
        if (k == 0) a.s[(size_t)row[u] * a.sp + b[u]] = (uint8_t)s;
        const int c = (int)b[u] * kBlk + k * NV;
        if (c >= a.qp) continue;
        uint8_t *q = a.q + (size_t)row[u] * a.qp + c;
        uint32_t w[NV / 4];
#pragma unroll
        for (int i = 0; i < NV / 4; ++i)
            w[i] = e4m3x4(f[u][4 * i] * inv, f[u][4 * i + 1] * inv, f[u][4 * i + 2] * inv, f[u][4 * i + 3] * inv);
        if constexpr (NV == 4) *reinterpret_cast<uint32_t *>(q) = w[0];
        else *reinterpret_cast<uint2 *>(q) = make_uint2(w[0], w[1]);
    }
}

// A tile of 128 x 128 values, both forms (or the transposed one alone).  A warp holds 16 rows, a lane four columns of them: the
// 16 codes that a lane has of a column are 16 neighbouring bytes of the transposed form, turned through shared memory so that they leave
// in rows of 128 bytes.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) quantize_e4m3_tile_kernel(const E4m3Args a) {
    __shared__ uint32_t s_col[8][kBlk];
    __shared__ uint4 s_t[kBlk][8];
    pdl_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r0 = blockIdx.y * kBlk + warp * 16, c0 = blockIdx.x * kBlk + lane * 4;
    const size_t node = blockIdx.z;
    const T *x = (const T *)a.x + node * a.x_node + c0;
    float f[16][4];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        load_some<T, 4, VEC>(x + (long long)(r0 + i) * a.x_row, r0 + i < a.rows ? a.cols - c0 : 0, f[i]);
    uint32_t cm[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) cm[j] = max(cm[j], abs_bits(f[i][j]));
    *reinterpret_cast<uint4 *>(&s_col[warp][lane * 4]) = make_uint4(cm[0], cm[1], cm[2], cm[3]);
    if (a.q) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            uint32_t amax = max(max(abs_bits(f[i][0]), abs_bits(f[i][1])), max(abs_bits(f[i][2]), abs_bits(f[i][3])));
            amax = __reduce_max_sync(0xffffffffu, amax);
            float inv;
            const uint32_t s = block_scale(amax, inv);
            if (r0 + i >= a.rows) continue;
            const size_t row = node * a.rows + r0 + i;
            if (lane == 0) a.s[row * a.sp + blockIdx.x] = (uint8_t)s;
            if (c0 < a.qp)
                *reinterpret_cast<uint32_t *>(a.q + row * a.qp + c0) = e4m3x4(f[i][0] * inv, f[i][1] * inv, f[i][2] * inv, f[i][3] * inv);
        }
    }
    __syncthreads();
    float inv[4];
    uint32_t sc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) cm[j] = 0u;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const uint4 v = *reinterpret_cast<const uint4 *>(&s_col[w][lane * 4]);
        cm[0] = max(cm[0], v.x); cm[1] = max(cm[1], v.y); cm[2] = max(cm[2], v.z); cm[3] = max(cm[3], v.w);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sc[j] = block_scale(cm[j], inv[j]);
    if (warp == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c0 + j < a.cols) a.st[(node * a.cols + c0 + j) * a.stp + blockIdx.y] = (uint8_t)sc[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = e4m3x4(f[4 * i][j] * inv[j], f[4 * i + 1][j] * inv[j], f[4 * i + 2][j] * inv[j], f[4 * i + 3][j] * inv[j]);
        s_t[lane * 4 + j][warp ^ (lane & 7)] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncthreads();
    const int tr = blockIdx.y * kBlk + (threadIdx.x & 7) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = (threadIdx.x >> 3) + 32 * i, col = blockIdx.x * kBlk + c;
        if (col < a.cols && tr < a.qtp)
            *reinterpret_cast<uint4 *>(a.qt + (node * a.cols + col) * a.qtp + tr) = s_t[c][(threadIdx.x & 7) ^ ((c >> 2) & 7)];
    }
}

}  // namespace lpdt

using namespace lpdt;

extern "C" int64_t lpdt_e4m3_pitch(int64_t cols) { return cols < 0 ? -1 : (int64_t)align_up((size_t)cols, 16); }
extern "C" int64_t lpdt_e4m3_scale_pitch(int64_t cols) { return cols < 0 ? -1 : (int64_t)align_up((size_t)ceil_div(cols, kBlk), 4); }

extern "C" lpdt_status lpdt_quantize_e4m3(const void *x, lpdt_dtype dtype, int32_t nodes, int64_t rows, int64_t cols,
                                          int64_t x_node_stride, int64_t x_row_stride, uint8_t *q, uint8_t *scale,
                                          uint8_t *qt, uint8_t *scale_t, void *stream) {
    LPDT_CHECK_ARG(dtype_ok(dtype) && nodes >= 0 && rows >= 0 && cols >= 0);
    LPDT_CHECK_ARG((q != nullptr) == (scale != nullptr) && (qt != nullptr) == (scale_t != nullptr));
    if (nodes == 0 || rows == 0 || cols == 0) return LPDT_OK;
    LPDT_CHECK_ARG(x && (q || qt) && aligned(x, dtype_size(dtype)));
    LPDT_CHECK_ARG((rows == 1 || x_row_stride >= cols) && (nodes == 1 || x_node_stride >= 0));
    LPDT_CHECK_ARG(!q || aligned(q, 16));
    LPDT_CHECK_ARG(!qt || aligned(qt, 16));
    const int64_t limit = (int64_t)1 << 30;
    if (rows > limit || cols > limit) return LPDT_ERR_UNSUPPORTED;
    E4m3Args a = {};
    a.x = x; a.x_node = nodes == 1 ? 0 : x_node_stride; a.x_row = rows == 1 ? 0 : x_row_stride;
    a.rows = (int)rows; a.cols = (int)cols;
    a.nb = (int)ceil_div(cols, kBlk); a.nbt = (int)ceil_div(rows, kBlk);
    a.q = q; a.s = scale; a.qt = qt; a.st = scale_t;
    a.qp = (int)lpdt_e4m3_pitch(cols); a.sp = (int)lpdt_e4m3_scale_pitch(cols);
    a.qtp = (int)lpdt_e4m3_pitch(rows); a.stp = (int)lpdt_e4m3_scale_pitch(rows);
    const cudaStream_t st = as_stream(stream);
    return with_dtype(dtype, [&](auto t) -> lpdt_status {
        using T = decltype(t);
        if (!qt) {
            constexpr int NV = 16 / (int)sizeof(T), PER_CTA = 256 / (kBlk / NV);
            const bool vec = aligned(x, 16) && (a.x_row % NV == 0) && (a.x_node % NV == 0);
            const int64_t total = (int64_t)nodes * rows * a.nb;
            if (total > (int64_t)0x7fffffff) return LPDT_ERR_UNSUPPORTED;
            if (total >= 4 * PER_CTA * kNumSMs)
                launch_k(vec ? quantize_e4m3_rows_kernel<T, true, 4> : quantize_e4m3_rows_kernel<T, false, 4>,
                                   (unsigned)ceil_div(total, PER_CTA * 4), 256, 0, st, a, (unsigned)total);
            else
                launch_k(vec ? quantize_e4m3_rows_kernel<T, true, 1> : quantize_e4m3_rows_kernel<T, false, 1>,
                                   (unsigned)ceil_div(total, PER_CTA), 256, 0, st, a, (unsigned)total);
            LPDT_LAUNCH_CHECK();
            return LPDT_OK;
        }
        const bool vec = aligned(x, 4 * sizeof(T)) && a.x_row % 4 == 0 && a.x_node % 4 == 0;
        if (a.nbt > 65535 || nodes > 65535) return LPDT_ERR_UNSUPPORTED;
        launch_k(vec ? quantize_e4m3_tile_kernel<T, true> : quantize_e4m3_tile_kernel<T, false>,
                           dim3((unsigned)a.nb, (unsigned)a.nbt, (unsigned)nodes), 256, 0, st, a);
        LPDT_LAUNCH_CHECK();
        return LPDT_OK;
    });
}
