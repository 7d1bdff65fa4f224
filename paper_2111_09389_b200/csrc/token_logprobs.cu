// lpdt_token_logprobs and its backward pass: log probabilities of given tokens, entropy, log-sum-exp and the top alternatives of rows
// of logits, in one pass over them.
//
// Memory is the bound: a row is read once.  Each thread keeps the running maximum m and, relative to it, s = sum 2^t and
// w = sum 2^t * t; then lse = m/T + ln s and H = ln s - ln2 * w / s, without a second pass for the maximum or the entropy.
// The top k come out of the same pass: the k-th largest of the threads' maxima over the first tile is a floor that the final k-th value
// cannot lie under, so of the rest of the row only what reaches the floor is written to a list in shared memory; when the list has
// grown, it is cut to its k best, which raises the floor.  Keys hold value and position, so equal values go to the lower position and
// a row of nothing but equal values needs no more than its first k.
//
// Few rows: the CTAs of a cluster share a row and join through distributed shared memory.  Rows of up to 1024 values: a warp each.
#include "rows.cuh"

namespace lpdt {

struct LogprobArgs {
    const void *x; long long x_row;
    long long rows; int V;
    double inv_t; float c;                       // 1 / T, log2(e) / T
    const int32_t *tokens;
    float *logprob, *entropy, *lse, *top_logprob; int32_t *top_index;
    int k;
    int32_t *dev_status;
};

// What one row answers, from its sums.  s = 0: nothing above -inf.
struct RowAnswer {
    double log_s, inv_t; float m; bool none;
    __device__ __forceinline__ RowAnswer(const Stats &a, double inv_t_) : inv_t(inv_t_), m(a.m), none(a.s == 0.f) { log_s = log((double)a.s); }
    __device__ __forceinline__ float of(float x) const {
        return none || x == -INFINITY ? (log_s != log_s ? NAN : -INFINITY) : (float)(((double)x - (double)m) * inv_t - log_s);
    }
    __device__ __forceinline__ float lse() const { return none ? -INFINITY : (float)((double)m * inv_t + log_s); }
    __device__ __forceinline__ float entropy(const Stats &a) const { return none ? 0.f : (float)(log_s - kLn2 * (double)a.w / (double)a.s); }
};
template <typename T>
__device__ __forceinline__ void answer_row(const LogprobArgs &a, long long row, const Stats &st) {
    const RowAnswer r(st, a.inv_t);
    if (a.lse) a.lse[row] = r.lse();
    if (a.entropy) a.entropy[row] = r.entropy(st);
    if (a.logprob) {
        const int t = a.tokens[row];
        float v = 0.f;
        if (t >= 0 && t < a.V) v = r.of(to_f32(((const T *)a.x + row * a.x_row)[t]));
        else if (t >= a.V && a.dev_status) atomicCAS(a.dev_status, 0, (int32_t)LPDT_ERR_INVALID_ARG);
        a.logprob[row] = v;
    }
}

constexpr int kLpThreads = 256, kLpWarps = kLpThreads / 32, kLpUnroll = 4, kTopMax = 128, kTopCap = 2048;

struct TopList {
    unsigned long long key[kTopCap];
    int count;
};
// Cuts the list to its k best, in order.  Each thread ranks its share of the n keys by counting the larger ones.
__device__ __forceinline__ void top_cut(TopList &l, int n, int k) {
    constexpr int PER = kTopCap / kLpThreads;
    unsigned long long mine[PER];
    int rank[PER];
    const int turns = (n + kLpThreads - 1) / kLpThreads;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int at = threadIdx.x + i * kLpThreads;
        rank[i] = kTopCap;
        if (i >= turns || at >= n) continue;
        mine[i] = l.key[at];
        int r = 0;
        for (int j = 0; j < n; ++j) r += l.key[j] > mine[i];
        rank[i] = r;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (rank[i] < k) l.key[rank[i]] = mine[i];
    if (threadIdx.x == 0) l.count = n < k ? n : k;
    __syncthreads();
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kLpThreads) logprobs_row_kernel(const LogprobArgs a) {
    constexpr int VE = Row<T>::VE, U = kLpUnroll;
    __shared__ TopList s_top;
    __shared__ Stats s_warp[kLpWarps];
    __shared__ unsigned long long s_floor;
    pdl_enter();
    const uint32_t rank = rows_cluster_rank(), share = rows_cluster_size();
    const long long row = blockIdx.x / share;
    const Row<T> r((const T *)a.x + row * a.x_row, a.V);
    const int begin = (int)((long long)r.words * rank / share), end = (int)((long long)r.words * (rank + 1) / share);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T fill = from_f32<T>(-INFINITY);
    const int cut_at = kLpThreads + 2 * a.k;

    Stats st;
    st.reset();
    unsigned long long floor_key = 0;            // nothing below it can be among the k best
    float floor_v = -INFINITY;
    if (TOP) {
        if (threadIdx.x == 0) s_top.count = 0;
        __syncthreads();
    }
    for (int w0 = begin; w0 < end; w0 += kLpThreads * U) {
        uint4 v[U];
        int at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at[u] = w0 + u * kLpThreads + (int)threadIdx.x;
            if (at[u] < end) v[u] = r.load(at[u], fill);
        }
        float wmax[U], tmax = kLowest;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            wmax[u] = -INFINITY;
            if (at[u] >= end) continue;
            float f[VE];
            unpack_vec<T>(v[u], f);
#pragma unroll
            for (int i = 0; i < VE; ++i) wmax[u] = fmaxf(wmax[u], f[i]);
            tmax = fmaxf(tmax, wmax[u]);
        }
        if (tmax > st.m) st.raise(tmax, a.c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (at[u] >= end) continue;
            float f[VE];
            unpack_vec<T>(v[u], f);
            accumulate<VE, true>(st, f, a.c);
        }
        if (TOP) {
            const int first_words = end - begin < kLpThreads ? end - begin : kLpThreads;
            if (w0 == begin && first_words >= a.k) {
                // the first tile's floor: the k-th largest of the threads' largest
                unsigned long long best = 0;
                if ((int)threadIdx.x < first_words) {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (at[u] >= end) continue;
                        float f[VE];
                        unpack_vec<T>(v[u], f);
#pragma unroll
                        for (int i = 0; i < VE; ++i)
                            if (r.holds((long long)at[u] * VE + i) && f[i] == f[i]) {
                                const unsigned long long key = top_key(f[i], at[u] * VE + i - r.head);
                                if (key > best) best = key;
                            }
                    }
                }
                s_top.key[threadIdx.x] = best;
                __syncthreads();
                int larger = 0;
                for (int j = 0; j < first_words; ++j) larger += s_top.key[j] > best;
                __syncthreads();
                // (a key of 0: a thread that met nothing but NaN)
                const bool kth = larger == a.k - 1 && best != 0;
                if (kth) s_floor = best;
                floor_key = __syncthreads_or(kth) ? s_floor : 0;
                floor_v = floor_key ? key_value(floor_key) : -INFINITY;
            }
            while (true) {
                const int floor_i = floor_key ? key_index(floor_key) : 0x7fffffff;
                bool grown = false;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (at[u] >= end || !(wmax[u] >= floor_v)) continue;
                    if (wmax[u] == floor_v && at[u] * VE - r.head > floor_i) continue;
                    float f[VE];
                    unpack_vec<T>(v[u], f);
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        if (!(f[i] >= floor_v) || !r.holds((long long)at[u] * VE + i)) continue;
                        const unsigned long long key = top_key(f[i], at[u] * VE + i - r.head);
                        if (key < floor_key) continue;
                        const int to = atomicAdd(&s_top.count, 1);
                        if (to < kTopCap) s_top.key[to] = key;
                        grown |= to >= cut_at;
                    }
                }
                if (!__syncthreads_or(grown)) break;
                const int n = s_top.count;
                __syncthreads();                                   // everyone has read the count
                top_cut(s_top, n < kTopCap ? n : kTopCap, a.k);
                floor_key = s_top.key[a.k - 1];
                floor_v = key_value(floor_key);
                if (n <= kTopCap) break;
                // Some of this tile found no room: its entries leave the list and it is walked again under the higher floor, which
                // at least kTopCap - cut_at - k of its values no longer reach.
                unsigned long long keep = 0;
                if ((int)threadIdx.x < a.k) keep = s_top.key[threadIdx.x];
                const long long pos = (long long)key_index(keep) + r.head;
                const bool stays = keep && pos < (long long)w0 * VE;
                __syncthreads();
                if (threadIdx.x == 0) s_top.count = 0;
                __syncthreads();
                if (stays) s_top.key[atomicAdd(&s_top.count, 1)] = keep;
                __syncthreads();
            }
        }
    }
    warp_join(st, a.c);
    if (lane == 0) s_warp[warp] = st;
    __syncthreads();
    if (warp == 0) {
        st.reset();
        if (lane < kLpWarps) st = s_warp[lane];
        warp_join(st, a.c);
        if (lane == 0) s_warp[0] = st;
    }
    if (TOP) {
        __syncthreads();
        const int n = s_top.count;
        __syncthreads();
        top_cut(s_top, n, a.k);
    }
    if (share > 1) {
        __shared__ unsigned long long s_part[2];
        if (threadIdx.x == 0) {
            s_part[0] = ((unsigned long long)__float_as_uint(s_warp[0].s) << 32) | __float_as_uint(s_warp[0].m);
            s_part[1] = ((unsigned long long)(TOP ? s_top.count : 0) << 32) | __float_as_uint(s_warp[0].w);
        }
        __syncthreads();
        rows_cluster_sync();
        if (rank == 0) {
            int n = TOP ? s_top.count : 0;
            __syncthreads();                                       // before the list grows
            Stats all = s_warp[0];
            for (uint32_t o = 1; o < share; ++o) {
                const unsigned long long p0 = ld_peer_u64(&s_part[0], o), p1 = ld_peer_u64(&s_part[1], o);
                Stats b;
                b.m = __uint_as_float((uint32_t)p0);
                b.s = __uint_as_float((uint32_t)(p0 >> 32));
                b.w = __uint_as_float((uint32_t)p1);
                all.join(b, a.c);
                if (TOP) {
                    const int more = (int)(p1 >> 32);
                    if ((int)threadIdx.x < more) s_top.key[n + threadIdx.x] = ld_peer_u64(&s_top.key[threadIdx.x], o);
                    n += more;
                }
            }
            __syncthreads();
            if (threadIdx.x == 0) s_warp[0] = all;
            if (TOP) top_cut(s_top, n, a.k);
        }
        __syncthreads();
        rows_cluster_sync();                                       // no CTA leaves while its shared memory is read
        if (rank != 0) return;
    }
    __syncthreads();
    if (threadIdx.x == 0) answer_row<T>(a, row, s_warp[0]);
    if (TOP && (int)threadIdx.x < a.k) {
        const RowAnswer ans(s_warp[0], a.inv_t);
        const bool have = (int)threadIdx.x < s_top.count;
        const unsigned long long key = have ? s_top.key[threadIdx.x] : 0;
        a.top_logprob[row * a.k + threadIdx.x] = have ? ans.of(key_value(key)) : NAN;
        a.top_index[row * a.k + threadIdx.x] = have ? key_index(key) : -1;
    }
}

// A warp per row of at most 32 * E values; lane l holds those at l, l + 32, ...
template <typename T, int E>
__global__ void __launch_bounds__(128) logprobs_warp_kernel(const LogprobArgs a) {
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= a.rows) return;
    const T *x = (const T *)a.x + row * a.x_row;
    float f[E];
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = lane + 32 * i < a.V ? to_f32(x[lane + 32 * i]) : -INFINITY;
    Stats st;
    st.reset();
    float m = kLowest;
#pragma unroll
    for (int i = 0; i < E; ++i) m = fmaxf(m, f[i]);
    st.raise(m, a.c);
    accumulate<E, true>(st, f, a.c);
    warp_join(st, a.c);
    if (lane == 0) answer_row<T>(a, row, st);
    if (a.k == 0) return;
    const RowAnswer ans(st, a.inv_t);
    uint32_t taken = 0;
    for (int j = 0; j < a.k; ++j) {
        uint32_t best = 0;                       // order bits of a number are never 0 (that is a NaN's)
        int at = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const bool in = !((taken >> i) & 1u) && f[i] == f[i] && lane + 32 * i < a.V;
            const uint32_t o = in ? order_bits(f[i]) : 0u;
            if (o > best) { best = o; at = i; }
        }
        const uint32_t top = __reduce_max_sync(0xffffffffu, best);
        const uint32_t index = __reduce_min_sync(0xffffffffu, best == top && top ? (uint32_t)(lane + 32 * at) : 0x7fffffffu);
        if (top && index == (uint32_t)(lane + 32 * at) && best == top) taken |= 1u << at;
        if (lane == 0) {
            a.top_logprob[row * a.k + j] = top ? ans.of(from_order_bits(top)) : NAN;
            a.top_index[row * a.k + j] = top ? (int32_t)index : -1;
        }
    }
}

struct LogprobBwdArgs {
    const void *x; long long x_row; void *dx; long long dx_row;
    long long rows; int V, chunks;
    float inv_t;
    const int32_t *tokens;
    const float *lse, *entropy, *g_logprob, *g_entropy, *g_lse;
};
// With p = exp(z - lse), z = x / T:  d x = (1[token] * g - p * (g + h * (ln p + H) - l)) / T.  Elementwise: a warp takes 128 words of a row.
template <typename T>
__global__ void __launch_bounds__(256) logprobs_bwd_kernel(const LogprobBwdArgs a) {
    constexpr int VE = Row<T>::VE, U = 4;
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), row = item / a.chunks;
    if (row >= a.rows) return;
    const int w0 = (int)(item - row * a.chunks) * 32 * U + lane;
    const Row<T> r((const T *)a.x + row * a.x_row, a.V);
    T *dx = (T *)a.dx + row * a.dx_row;
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (w0 + u * 32 < r.words) v[u] = r.load(w0 + u * 32, from_f32<T>(0.f));
    const int t = a.tokens ? a.tokens[row] : -1;
    const bool some = t >= 0 && t < a.V;
    const float lse = a.lse[row], g = a.g_logprob && some ? a.g_logprob[row] : 0.f;
    const float h = a.g_entropy ? a.g_entropy[row] : 0.f, l = a.g_lse ? a.g_lse[row] : 0.f;
    const float base = l - g - (a.g_entropy ? h * a.entropy[row] : 0.f);
    const bool none = lse < -1e30f;              // nothing but mask values: no gradient
    const bool same = (((uintptr_t)dx & 15) / sizeof(T)) == (uintptr_t)r.head;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int w = w0 + u * 32;
        if (w >= r.words) continue;
        float f[VE];
        unpack_vec<T>(v[u], f);
        const int first = w * VE - r.head;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const float lp = max_nan(fmaf(f[i], a.inv_t, -lse), kFar), p = ex2(lp * kLog2e);
            float d = p * fmaf(-h, lp, base);
            if (none) d = 0.f;
            if (first + i == t && !none) d += g;
            f[i] = d * a.inv_t;
        }
        if (same && r.whole(w)) {
            constexpr int PER = 4 / (int)sizeof(T);
            *reinterpret_cast<uint4 *>(dx + first) =
                make_uint4(pack_word(f, T()), pack_word(f + PER, T()), pack_word(f + 2 * PER, T()), pack_word(f + 3 * PER, T()));
        } else {
#pragma unroll
            for (int i = 0; i < VE; ++i)
                if (r.holds((long long)w * VE + i)) dx[first + i] = from_f32<T>(f[i]);
        }
    }
}

}  // namespace lpdt

using namespace lpdt;

extern "C" lpdt_status lpdt_token_logprobs(int64_t rows, int32_t V, const void *logits, lpdt_dtype dtype, int64_t row_stride,
                                           float temperature, const int32_t *tokens, float *logprob, float *entropy, float *lse,
                                           int32_t top_k, float *top_logprob, int32_t *top_index, int32_t *dev_status, void *stream) {
    LPDT_CHECK_ARG(rows >= 0 && V >= 1 && dtype_ok(dtype) && temperature_ok(temperature));
    LPDT_CHECK_ARG(top_k >= 0 && top_k <= V);
    if (rows == 0) return LPDT_OK;
    LPDT_CHECK_ARG(logits && aligned(logits, dtype_size(dtype)) && (rows == 1 || row_stride >= V));
    LPDT_CHECK_ARG((logprob || entropy || lse || top_k > 0) && (!logprob || tokens));
    LPDT_CHECK_ARG(top_k == 0 || (top_logprob && top_index));
    if (top_k > kTopMax || V > (1 << 30) || rows > (1 << 27)) return LPDT_ERR_UNSUPPORTED;
    LogprobArgs a = {};
    a.x = logits; a.x_row = rows == 1 ? 0 : row_stride; a.rows = rows; a.V = V;
    a.inv_t = 1.0 / (double)temperature; a.c = (float)(1.4426950408889634 / (double)temperature);
    a.tokens = tokens; a.logprob = logprob; a.entropy = entropy; a.lse = lse;
    a.top_logprob = top_logprob; a.top_index = top_index; a.k = top_k; a.dev_status = dev_status;
    const cudaStream_t st = as_stream(stream);
    return with_dtype(dtype, [&](auto t) -> lpdt_status {
        using T = decltype(t);
        if (V <= 1024) {
            const unsigned grid = (unsigned)ceil_div(rows, 4);
            if (V <= 64) launch_k(logprobs_warp_kernel<T, 2>, grid, 128, 0, st, a);
            else if (V <= 256) launch_k(logprobs_warp_kernel<T, 8>, grid, 128, 0, st, a);
            else launch_k(logprobs_warp_kernel<T, 32>, grid, 128, 0, st, a);
        } else {
            const int cs = row_share(rows, (int64_t)V * sizeof(T), 4, 4096);
            launch_k_cluster(top_k ? logprobs_row_kernel<T, true> : logprobs_row_kernel<T, false>, (unsigned)(rows * cs), kLpThreads, 0, st, cs, a);
        }
        LPDT_LAUNCH_CHECK();
        return LPDT_OK;
    });
}

extern "C" lpdt_status lpdt_token_logprobs_bwd(int64_t rows, int32_t V, const void *logits, lpdt_dtype dtype, int64_t row_stride,
                                               float temperature, const int32_t *tokens, const float *lse, const float *entropy,
                                               const float *d_logprob, const float *d_entropy, const float *d_lse, void *dlogits,
                                               int64_t dlogits_row_stride, void *stream) {
    LPDT_CHECK_ARG(rows >= 0 && V >= 1 && dtype_ok(dtype) && temperature_ok(temperature));
    if (rows == 0) return LPDT_OK;
    LPDT_CHECK_ARG(logits && dlogits && aligned(logits, dtype_size(dtype)) && aligned(dlogits, dtype_size(dtype)));
    LPDT_CHECK_ARG(rows == 1 || (row_stride >= V && dlogits_row_stride >= V));
    LPDT_CHECK_ARG(lse && (!d_logprob || tokens) && (!d_entropy || entropy) && (d_logprob || d_entropy || d_lse));
    // in place: a row's gradient lies where its logits lay, or the two arrays are apart
    LPDT_CHECK_ARG(dlogits != logits || rows == 1 || dlogits_row_stride == row_stride);
    if (V > (1 << 30) || rows > (1 << 27)) return LPDT_ERR_UNSUPPORTED;
    LogprobBwdArgs a = {};
    a.x = logits; a.x_row = rows == 1 ? 0 : row_stride; a.dx = dlogits; a.dx_row = rows == 1 ? 0 : dlogits_row_stride;
    a.rows = rows; a.V = V; a.inv_t = 1.f / temperature;
    a.tokens = tokens; a.lse = lse; a.entropy = entropy; a.g_logprob = d_logprob; a.g_entropy = d_entropy; a.g_lse = d_lse;
    const cudaStream_t st = as_stream(stream);
    return with_dtype(dtype, [&](auto t) -> lpdt_status {
        using T = decltype(t);
        constexpr int VE = Row<T>::VE;
        a.chunks = (int)ceil_div((int64_t)V + VE - 1, 128 * VE);
        const int64_t blocks = ceil_div(rows * a.chunks, 8);
        if (blocks > 0x7fffffff) return LPDT_ERR_UNSUPPORTED;
        launch_k(logprobs_bwd_kernel<T>, (unsigned)blocks, 256, 0, st, a);
        LPDT_LAUNCH_CHECK();
        return LPDT_OK;
    });
}
