// lpdt_quantize_e4m3: 8-bit floats with a power-of-two scale for each block of 128 values.
//
// A block's scale is 2^e with e the least integer for which amax <= 448 * 2^e (448: the largest e4m3 value), so x * 2^-e is exact and
// the one rounding is the conversion's own (to nearest, halves to even).  amax is taken on the bits of |x|: as unsigned integers they
// order like the values, infinities and NaN above them, which marks a block that holds one.
//
// Memory is the bound: each value is read once and written as one byte per form.  8192 x 8192, calls in a graph: bf16 rows 32.6 us (6.2 TB/s),
// both forms 52.7 (5.1 TB/s), fp32 both forms 72.5 (5.6 TB/s).
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

// NW words of consecutive elements at p, as they lie in memory; the first `have` elements exist, the others read 0.  VEC: p is aligned to
// all of them.
template <typename T, bool VEC, int NW>
__device__ __forceinline__ void load_raw(const T *__restrict__ p, int have, uint32_t (&w)[NW]) {
    constexpr int PER = 4 / (int)sizeof(T);
    if (VEC && have >= NW * PER) {
        if constexpr (NW == 4) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            static_assert(NW == 2, "8 or 16 bytes");
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
            w[0] = v.x; w[1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            float f[2];
#pragma unroll
            for (int j = 0; j < PER; ++j) f[j] = i * PER + j < have ? to_f32(p[i * PER + j]) : 0.f;
            w[i] = pack_word(f, T());
        }
    }
}
// The same at any alignment, for lanes whose neighbours' elements lie in the row on both sides: the two aligned vectors that hold the words,
// from which they are selected and shifted.  16-bit elements only: 8192 x 8190 bf16 in both forms 91 us, 112 element by element, in rows 52
// and 64; fp32 the other way (118 and 94), its elements being words already.
template <typename T, int NW> __device__ __forceinline__ void load_shifted(const T *__restrict__ p, uint32_t (&w)[NW]) {
    const uint32_t o = (uint32_t)((uintptr_t)p & (4 * NW - 1));
    const char *a = reinterpret_cast<const char *>(p) - o;
    uint32_t v[2 * NW];
    if constexpr (NW == 4) {
        const uint4 l = __ldg(reinterpret_cast<const uint4 *>(a)), h = __ldg(reinterpret_cast<const uint4 *>(a) + 1);
        v[0] = l.x; v[1] = l.y; v[2] = l.z; v[3] = l.w; v[4] = h.x; v[5] = h.y; v[6] = h.z; v[7] = h.w;
#pragma unroll
        for (int i = 0; i < 6; ++i) v[i] = o & 8 ? v[i + 2] : v[i];
    } else {
        const uint2 l = __ldg(reinterpret_cast<const uint2 *>(a)), h = __ldg(reinterpret_cast<const uint2 *>(a) + 1);
        v[0] = l.x; v[1] = l.y; v[2] = h.x; v[3] = h.y;
    }
#pragma unroll
    for (int i = 0; i < NW + 1; ++i) v[i] = o & 4 ? v[i + 1] : v[i];
#pragma unroll
    for (int i = 0; i < NW; ++i) w[i] = __funnelshift_r(v[i], v[i + 1], 8 * (o & 2));
}
// Maxima of |x| as bits: one value a word (fp32), or two side by side; then of the two, and as the bits of the same value in fp32.
__device__ __forceinline__ uint32_t amax_word(uint32_t m, uint32_t w, float) { return max(m, w & 0x7fffffffu); }
template <typename H> __device__ __forceinline__ uint32_t amax_word(uint32_t m, uint32_t w, H) { return __vmaxu2(m, w & 0x7fff7fffu); }
__device__ __forceinline__ uint32_t amax_one(uint32_t m, float) { return m; }
template <typename H> __device__ __forceinline__ uint32_t amax_one(uint32_t m, H) { return max(m >> 16, m & 0xffffu); }
__device__ __forceinline__ uint32_t bits_f32(uint32_t b, float) { return b; }
__device__ __forceinline__ uint32_t bits_f32(uint32_t b, __nv_bfloat16) { return b << 16; }
__device__ __forceinline__ uint32_t bits_f32(uint32_t b, __half) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)b))); }
// The elements of a word times a power of two each (exact; what falls below the smallest normal number is below any code's half).
__device__ __forceinline__ void scaled(uint32_t w, float s0, float, float *f, float) { f[0] = __uint_as_float(w) * s0; }
__device__ __forceinline__ void scaled(uint32_t w, float s0, float s1, float *f, __half) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    f[0] = v.x * s0;
    f[1] = v.y * s1;
}
__device__ __forceinline__ void scaled(uint32_t w, float s0, float s1, float *f, __nv_bfloat16) {
    const __nv_bfloat162 p = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&w), __floats2bfloat162_rn(s0, s1));
    unpack_word(*reinterpret_cast<const uint32_t *>(&p), f, __nv_bfloat16());
}

struct E4m3Args {
    const void *x;
    long long x_node, x_row;                      // strides in elements
    int rows, cols, nb, nbt;                      // blocks of a row, of a column
    int chunks;                                   // of a row, for the warps of the rows' kernel
    uint8_t *q, *s, *qt, *st;
    int qp, sp, qtp, stp;                         // pitches in bytes
};

// Rows only.  128 / NV lanes hold a block, 16 bytes of the row each; a warp takes U times as many neighbouring blocks of one row.
template <typename T, bool VEC, int U>
__global__ void __launch_bounds__(256) quantize_e4m3_rows_kernel(const E4m3Args a, unsigned items) {
    constexpr int NV = 16 / (int)sizeof(T), L = kBlk / NV, PER_WARP = 32 / L;
    pdl_enter();
    const unsigned item = blockIdx.x * 8u + (threadIdx.x >> 5);
    if (item >= items) return;
    const unsigned row = item / (unsigned)a.chunks, n = row / (unsigned)a.rows, r = row - n * (unsigned)a.rows;      // row: over all nodes
    const int lane = threadIdx.x & 31, k = lane % L;
    const int b0 = (int)(item - row * (unsigned)a.chunks) * (PER_WARP * U) + lane / L;
    const T *x = (const T *)a.x + n * a.x_node + r * a.x_row + k * NV;
    uint8_t *q = a.q + (size_t)row * a.qp + k * NV, *s = a.s + (size_t)row * a.sp;
    uint32_t w[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = (b0 + u * PER_WARP) * kBlk;
        const int left = a.cols - c - k * NV;
        if (!VEC && sizeof(T) == 2 && c + k * NV >= NV && left >= 2 * NV) load_shifted<T>(x + c, w[u]);
        else load_raw<T, VEC>(x + c, left, w[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) amax = amax_word(amax, w[u][i], T());
        amax = amax_one(amax, T());
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        float inv, f[NV];
        const uint32_t scale = block_scale(bits_f32(amax, T()), inv);
        const int b = b0 + u * PER_WARP;
        if (k == 0 && b < a.nb) s[b] = (uint8_t)scale;
        if (b * kBlk + k * NV >= a.qp) continue;
        uint32_t c[NV / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) scaled(w[u][i], inv, inv, f + i * (NV / 4), T());
#pragma unroll
        for (int i = 0; i < NV / 4; ++i) c[i] = e4m3x4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
        if constexpr (NV == 4) *reinterpret_cast<uint32_t *>(q + b * kBlk) = c[0];
        else *reinterpret_cast<uint2 *>(q + b * kBlk) = make_uint2(c[0], c[1]);
    }
}

// A tile of 128 x 128 values, both forms (or the transposed one alone).  A warp holds R rows, a lane four columns of them as they
// came: the R codes that a lane has of a column are R neighbouring bytes of the transposed form, turned through shared memory so that
// they leave in rows of 128 bytes.  R = 16 rows of 16-bit elements or 8 of fp32 are 32 registers of the 64 that four CTAs an SM leave a
// thread; the rest does not quite fit (spilled: bf16 and fp32 24 bytes, fp16 100; unaligned bf16 128, fp16 276, fp32 36), yet three or
// five CTAs are no faster.
template <typename T> struct TileShape {
    static constexpr int R = 32 / (int)sizeof(T), THREADS = kBlk / R * 32, MIN_CTAS = 1024 / THREADS;
};
template <typename T, bool VEC>
__global__ void __launch_bounds__(TileShape<T>::THREADS, TileShape<T>::MIN_CTAS) quantize_e4m3_tile_kernel(const E4m3Args a) {
    constexpr int W = (int)sizeof(T), PER = 4 / W;             // words of four elements, elements of a word
    constexpr int R = TileShape<T>::R, GROUPS = kBlk / R;
    __shared__ uint32_t s_col[4][32];                          // [column % 4][column / 4]
    __shared__ __align__(16) uint8_t s_t[kBlk][kBlk];          // [column][row], groups of R rows exchanged by column
    pdl_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r0 = blockIdx.y * kBlk + warp * R, c0 = blockIdx.x * kBlk + lane * 4;
    const size_t node = blockIdx.z;
    const T *x = (const T *)a.x + node * a.x_node + (long long)r0 * a.x_row + c0;
    uint32_t w[R][W];
    if (!VEC && sizeof(T) == 2 && c0 >= 4 && a.cols - c0 >= 8) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (r0 + i < a.rows) load_shifted<T>(x + i * a.x_row, w[i]);
            else load_raw<T, false>(x, 0, w[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i)
            load_raw<T, VEC>(x + i * a.x_row, r0 + i < a.rows ? a.cols - c0 : 0, w[i]);
    }
    if (threadIdx.x < kBlk) (&s_col[0][0])[threadIdx.x] = 0u;
    __syncthreads();
    uint32_t cm[W];
#pragma unroll
    for (int k = 0; k < W; ++k) cm[k] = 0u;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int k = 0; k < W; ++k) cm[k] = amax_word(cm[k], w[i][k], T());
#pragma unroll
    for (int j = 0; j < 4; ++j) atomicMax(&s_col[j][lane], PER == 1 ? cm[j % W] : (j & 1) ? cm[j >> 1] >> 16 : cm[j >> 1] & 0xffffu);
    if (a.q) {
        // lane i keeps row i's maximum, so the scales of all rows are one computation
        uint32_t mine = 0u;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            uint32_t amax = 0u;
#pragma unroll
            for (int k = 0; k < W; ++k) amax = amax_word(amax, w[i][k], T());
            amax = __reduce_max_sync(0xffffffffu, amax_one(amax, T()));
            if (lane == i) mine = amax;
        }
        float inv;
        const uint32_t scale = block_scale(bits_f32(mine, T()), inv);
        const size_t row = node * a.rows + r0;
        if (lane < R && r0 + lane < a.rows) a.s[(row + lane) * a.sp + blockIdx.x] = (uint8_t)scale;
        uint8_t *q = a.q + row * a.qp + c0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float s = __shfl_sync(0xffffffffu, inv, i);
            float f[4];
#pragma unroll
            for (int k = 0; k < W; ++k) scaled(w[i][k], s, s, f + k * PER, T());
            if (r0 + i < a.rows && c0 < a.qp) *reinterpret_cast<uint32_t *>(q) = e4m3x4(f[0], f[1], f[2], f[3]);
            q += a.qp;
        }
    }
    __syncthreads();
    float inv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t s = block_scale(bits_f32(s_col[j][lane], T()), inv[j]);
        if (warp == j && c0 + j < a.cols) a.st[(node * a.cols + c0 + j) * a.stp + blockIdx.y] = (uint8_t)s;
    }
    uint32_t t[4][R / 4];
#pragma unroll
    for (int h = 0; h < R / 4; ++h) {
        float f[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < W; ++k) scaled(w[4 * h + i][k], inv[k * PER], inv[k * PER + PER - 1], f[i] + k * PER, T());
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j][h] = e4m3x4(f[0][j], f[1][j], f[2][j], f[3][j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint8_t *to = &s_t[lane * 4 + j][(warp ^ (lane & (GROUPS - 1))) * R];
        if constexpr (R == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(t[j][0], t[j][1]);
        else *reinterpret_cast<uint4 *>(to) = make_uint4(t[j][0], t[j][1], t[j][2], t[j][3]);
    }
    __syncthreads();
    const int piece = threadIdx.x & 7, tr = blockIdx.y * kBlk + piece * 16;
#pragma unroll
    for (int c = threadIdx.x >> 3; c < kBlk; c += TileShape<T>::THREADS / 8) {
        const int col = blockIdx.x * kBlk + c, swz = (c >> 2) & (GROUPS - 1);
        if (col < a.cols && tr < a.qtp) {
            uint4 v = *reinterpret_cast<const uint4 *>(&s_t[c][R == 8 ? ((2 * piece) ^ (swz & 14)) * 8 : (piece ^ swz) * 16]);
            if (R == 8 && (swz & 1)) v = make_uint4(v.z, v.w, v.x, v.y);
            *reinterpret_cast<uint4 *>(a.qt + (node * a.cols + col) * a.qtp + tr) = v;
        }
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
            constexpr int NV = 16 / (int)sizeof(T), PER_WARP = 32 / (kBlk / NV);
            const bool vec = aligned(x, 16) && (a.x_row % NV == 0) && (a.x_node % NV == 0);
            const int64_t all = (int64_t)nodes * rows;
            if (all * a.nb > (int64_t)0x7fffffff) return LPDT_ERR_UNSUPPORTED;
            // four groups of blocks a warp once that leaves every SM some 32 warps
            const bool four = all * ceil_div(a.nb, 4 * PER_WARP) >= 32 * kNumSMs;
            a.chunks = (int)ceil_div(a.nb, (four ? 4 : 1) * PER_WARP);
            const unsigned items = (unsigned)(all * a.chunks), grid = (unsigned)ceil_div(items, 8);
            if (four) launch_k(vec ? quantize_e4m3_rows_kernel<T, true, 4> : quantize_e4m3_rows_kernel<T, false, 4>, grid, 256, 0, st, a, items);
            else launch_k(vec ? quantize_e4m3_rows_kernel<T, true, 1> : quantize_e4m3_rows_kernel<T, false, 1>, grid, 256, 0, st, a, items);
            LPDT_LAUNCH_CHECK();
            return LPDT_OK;
        }
        const bool vec = aligned(x, 4 * sizeof(T)) && a.x_row % 4 == 0 && a.x_node % 4 == 0;
        if (a.nbt > 65535 || nodes > 65535) return LPDT_ERR_UNSUPPORTED;
        launch_k(vec ? quantize_e4m3_tile_kernel<T, true> : quantize_e4m3_tile_kernel<T, false>,
                           dim3((unsigned)a.nb, (unsigned)a.nbt, (unsigned)nodes), TileShape<T>::THREADS, 0, st, a);
        LPDT_LAUNCH_CHECK();
        return LPDT_OK;
    });
}
