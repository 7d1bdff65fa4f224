// lpdt_distill_topk: distillation from a teacher's top log probabilities, loss and gradient.
//
// With z = x / T, S the listed tokens and p the student's softmax, the loss takes the student's probability of everything outside S as
// one more class.  Its logarithm is lse_R - lse with lse_R over the tokens outside S alone, not ln(1 - sum_S p), which would lose all
// digits once the list holds nearly all of the mass; so the pass over the row leaves S out (a bit per token in shared memory says which)
// and S, gathered by itself, joins at the end.  A token outside S has the gradient e^(z - m) times one number of the row, so the second
// pass is one exponential and one product a value, and the listed tokens' gradients are written over it.
//
// Memory is the bound: the row once in, the gradient once out.
#include "rows.cuh"

namespace lpdt {

constexpr int kDtThreads = 256, kDtWarps = kDtThreads / 32, kDtUnroll = 4, kListMax = 128;
constexpr size_t kDtSmem = 160 * 1024;

struct DistillArgs {
    const void *x; long long x_row; void *dx; long long dx_row;
    int B, V, k, tail;
    long long rows;
    double inv_t;                     // 1 / T
    float c;                          // log2(e) / T
    const float *value; const int32_t *index;
    const float *weight;
    float *row_loss;
    int32_t *dev_status;
};

// A row's list, ready for use: in shared memory.
struct List {
    int id[kListMax];                 // -1: no entry
    float x[kListMax];                // the student's logit
    double t[kListMax], logt[kListMax];
    double sum;                       // of t
    double lse;                       // of the listed tokens' z, each token once; -inf without any
    int first[kListMax];              // the entry is the first one of its token
};

// By all threads of a warp.
__device__ __forceinline__ double warp_max_d(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
// Fills the list of a row; one warp, which may not use it before a barrier of its readers.
template <typename T>
__device__ __forceinline__ void make_list(const DistillArgs &a, long long row, List &l, int lane, bool report) {
    const T *x = (const T *)a.x + row * a.x_row;
    double top = -INFINITY, xmax = -INFINITY;
    bool bad = false;
    for (int j = lane; j < a.k; j += 32) {
        const int id = a.index[row * a.k + j];
        const bool have = id >= 0 && id < a.V;
        if (id >= a.V && report && a.dev_status) atomicCAS(a.dev_status, 0, (int32_t)LPDT_ERR_INVALID_ARG);
        l.id[j] = have ? id : -1;
        l.x[j] = have ? to_f32(x[id]) : -INFINITY;
        l.logt[j] = have ? (double)a.value[row * a.k + j] : -INFINITY;
        top = fmax(top, l.logt[j]);
        xmax = fmax(xmax, (double)l.x[j]);
        bad |= l.x[j] != l.x[j];
    }
    __syncwarp();
    double sum = 0.0, sumx = 0.0;
    if (!a.tail) {
        // the list as a distribution: minus the logarithm of its sum
        top = warp_max_d(top);
        for (int j = lane; j < a.k; j += 32)
            if (l.logt[j] > -INFINITY) sum += exp(l.logt[j] - top);
        const double norm = top + log(warp_sum(sum));
        sum = 0.0;
        for (int j = lane; j < a.k; j += 32)
            if (l.id[j] >= 0 && l.logt[j] > -INFINITY) l.logt[j] -= norm;
    }
    xmax = warp_max_d(xmax);
    const bool some = xmax > -INFINITY;
    bad = __any_sync(0xffffffffu, bad);
    for (int j = lane; j < a.k; j += 32) {
        const int id = l.id[j];
        l.t[j] = id >= 0 ? exp(l.logt[j]) : 0.0;
        sum += l.t[j];
        bool first = id >= 0;
        for (int i = 0; i < j && first; ++i) first = l.id[i] != id;
        l.first[j] = first;
        if (first && some) sumx += exp(((double)l.x[j] - xmax) * a.inv_t);
    }
    sum = warp_sum(sum);
    sumx = warp_sum(sumx);
    if (lane == 0) {
        l.sum = sum;
        l.lse = bad ? NAN : some ? xmax * a.inv_t + log(sumx) : -INFINITY;
    }
    __syncwarp();
}

// What the row's gradient and loss come from, once the sums outside the list are known.  One warp; results in all of its lanes.
// left: the teacher's mass outside the list; rest: the factor of 2^((x - m) c) there.  A student's row of nothing but mask values
// (lse below -1e30) has neither loss nor gradient.
struct RowTerms { double loss, lse, left; float rest; bool masked; };
__device__ __forceinline__ double log_add(double a, double b) {
    if (a != a || b != b) return NAN;
    const double m = fmax(a, b);
    if (m == -INFINITY) return m;
    return m + log(exp(a - m) + exp(b - m));
}
__device__ __forceinline__ RowTerms row_terms(const DistillArgs &a, const List &l, const Stats &st, double g, int lane) {
    RowTerms r;
    const bool outside = !(st.s == 0.f);
    const double lse_r = outside ? (double)st.m * a.inv_t + log((double)st.s) : -INFINITY;
    r.lse = log_add(l.lse, lse_r);
    r.left = a.tail && outside ? fmax(1.0 - l.sum, 0.0) : 0.0;
    r.masked = r.lse < -1e30;
    double loss = 0.0;
    for (int j = lane; j < a.k; j += 32)
        if (l.t[j] != 0.0) loss += l.t[j] * (l.logt[j] - ((double)l.x[j] * a.inv_t - r.lse));
    loss = warp_sum(loss);
    const double p_r = outside ? exp(lse_r - r.lse) : 0.0;
    if (r.left != 0.0) loss += r.left * (log(r.left) - (lse_r - r.lse));
    r.loss = r.masked ? 0.0 : loss;
    r.rest = outside && !r.masked ? (float)(g * ((l.sum + r.left) * p_r - r.left) / (double)st.s) : 0.f;
    return r;
}
// The gradient of listed entry j's token (the first of its entries writes it).
__device__ __forceinline__ float listed_grad(const DistillArgs &a, const List &l, const RowTerms &r, double g, int j) {
    if (r.masked) return 0.f;
    double t = 0.0;
    for (int i = j; i < a.k; ++i)
        if (l.id[i] == l.id[j]) t += l.t[i];
    const double p = l.x[j] == -INFINITY ? 0.0 : exp((double)l.x[j] * a.inv_t - r.lse);
    return (float)(g * (p * (l.sum + r.left) - t));
}

template <typename T>
__global__ void __launch_bounds__(kDtThreads) distill_row_kernel(const DistillArgs a) {
    constexpr int VE = Row<T>::VE, U = kDtUnroll;
    extern __shared__ uint32_t s_bits[];              // a bit per position of this CTA's words: listed
    __shared__ List s_list;
    __shared__ Stats s_warp[kDtWarps];
    __shared__ unsigned long long s_part[2];
    __shared__ RowTerms s_terms;
    pdl_enter();
    const uint32_t rank = rows_cluster_rank(), share = rows_cluster_size();
    const long long row = blockIdx.x / share;
    const Row<T> r((const T *)a.x + row * a.x_row, a.V);
    T *dx = a.dx ? (T *)a.dx + row * a.dx_row : nullptr;
    const bool same = ((uintptr_t)(dx + r.head) & 15) == 0;
    const int begin = (int)((long long)r.words * rank / share), end = (int)((long long)r.words * (rank + 1) / share);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float weight = a.weight ? a.weight[row] : 1.f;
    const double g = (double)weight * a.inv_t / (double)a.B;
    const bool skip = weight == 0.f;                  // the same for the whole cluster
    const int edge = rank == 0 && threadIdx.x < Row<T>::EDGES ? r.edge(threadIdx.x) : -1;
    float at_edge = -INFINITY;

    Stats st;
    st.reset();
    if (!skip) {
        const int bit_words = ((end - begin) * VE + 31) / 32;
        for (int i = threadIdx.x; i < bit_words; i += kDtThreads) s_bits[i] = 0;
        if (warp == 0) make_list<T>(a, row, s_list, lane, rank == 0);
        __syncthreads();
        if ((int)threadIdx.x < a.k && s_list.id[threadIdx.x] >= 0) {
            const int at = s_list.id[threadIdx.x] - r.index(begin);
            if (at >= 0 && at < (end - begin) * VE) atomicOr(&s_bits[at >> 5], 1u << (at & 31));
        }
        if (edge >= 0) {
            at_edge = to_f32(r.at(edge));
            bool out = false;
            for (int j = 0; j < a.k; ++j) out |= s_list.id[j] == edge;
            const float x[2] = {out ? -INFINITY : at_edge, -INFINITY};
            if (x[0] > st.m) st.raise(x[0], a.c);
            accumulate<2, false>(st, x, a.c);
        }
        __syncthreads();
        const uint8_t *bytes = reinterpret_cast<const uint8_t *>(s_bits);
        auto word = [&](const uint4 &v, int i0) {
            float f[VE];
            unpack_vec<T>(v, f);
            const uint32_t out = VE == 8 ? bytes[i0] : (bytes[i0 >> 1] >> (4 * (i0 & 1))) & 15u;
            if (out) {
#pragma unroll
                for (int i = 0; i < VE; ++i) if ((out >> i) & 1u) f[i] = -INFINITY;
            }
            float m = f[0];
#pragma unroll
            for (int i = 1; i < VE; ++i) m = fmaxf(m, f[i]);
            if (m > st.m) st.raise(m, a.c);
            accumulate<VE, false>(st, f, a.c);
        };
        int w = begin + (int)threadIdx.x;
        for (; w + (U - 1) * kDtThreads < end; w += kDtThreads * U) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = r.load(w + u * kDtThreads);
#pragma unroll
            for (int u = 0; u < U; ++u) word(v[u], w + u * kDtThreads - begin);
        }
        for (; w < end; w += kDtThreads) word(r.load(w), w - begin);
        warp_join(st, a.c);
        if (lane == 0) s_warp[warp] = st;
        __syncthreads();
        if (warp == 0) {
            st.reset();
            if (lane < kDtWarps) st = s_warp[lane];
            warp_join(st, a.c);
            if (lane == 0) {
                s_warp[0] = st;
                s_part[0] = ((unsigned long long)__float_as_uint(st.s) << 32) | __float_as_uint(st.m);
            }
        }
    }
    // every CTA of the cluster has read what it gathers before any writes a gradient, which may lie where the logits do
    if (share > 1) {
        __syncthreads();
        rows_cluster_sync();
        if (!skip && warp == 0) {
            st.reset();
            for (uint32_t o = 0; o < share; ++o) {                // in the same order everywhere
                const unsigned long long p0 = ld_peer_u64(&s_part[0], o);
                Stats b;
                b.m = __uint_as_float((uint32_t)p0);
                b.s = __uint_as_float((uint32_t)(p0 >> 32));
                b.w = 0.f;
                st.join(b, a.c);
            }
            if (lane == 0) s_warp[0] = st;
        }
        __syncthreads();
        rows_cluster_sync();
    } else
        __syncthreads();
    if (skip) {
        if (threadIdx.x == 0 && rank == 0) a.row_loss[row] = 0.f;
        if (!dx) return;
    } else {
        if (warp == 0) {
            const RowTerms t = row_terms(a, s_list, s_warp[0], g, lane);
            if (lane == 0) {
                s_terms = t;
                if (rank == 0) a.row_loss[row] = (float)t.loss;
            }
        }
        if (!dx) return;
        __syncthreads();
    }
    const float rest = skip ? 0.f : s_terms.rest, m = skip ? 0.f : s_warp[0].m;
    auto grad = [&](float x) { return rest * ex2(max_nan((x - m) * a.c, kFar)); };
    auto put = [&](int w, const float *f) {
        if (same) *reinterpret_cast<uint4 *>(dx + r.index(w)) = pack_vec<T>(f);
        else {
#pragma unroll
            for (int i = 0; i < VE; ++i) dx[r.index(w) + i] = from_f32<T>(f[i]);
        }
    };
    int w = begin + (int)threadIdx.x;
    if (!skip) {
        auto word = [&](const uint4 &v, int at) {
            float f[VE];
            unpack_vec<T>(v, f);
#pragma unroll
            for (int i = 0; i < VE; ++i) f[i] = grad(f[i]);
            put(at, f);
        };
        for (; w + (U - 1) * kDtThreads < end; w += kDtThreads * U) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = r.load(w + u * kDtThreads);
#pragma unroll
            for (int u = 0; u < U; ++u) word(v[u], w + u * kDtThreads);
        }
        for (; w < end; w += kDtThreads) word(r.load(w), w);
    } else {
        const float zeros[VE] = {};
        for (; w < end; w += kDtThreads) put(w, zeros);
    }
    if (edge >= 0) dx[edge] = from_f32<T>(skip ? 0.f : grad(at_edge));
    if (skip) return;
    __syncthreads();
    if ((int)threadIdx.x < a.k && s_list.first[threadIdx.x]) {
        const int id = s_list.id[threadIdx.x], at = id - r.index(begin);
        const bool here = (at >= 0 && at < (end - begin) * VE) || (rank == 0 && (id < r.head || id >= r.index(r.words)));
        if (here)
            dx[id] = from_f32<T>(listed_grad(a, s_list, s_terms, g, threadIdx.x));
    }
}

// A warp per row of at most 32 * E values; lane l holds those at l, l + 32, ..., bit i of `out` says that the i-th is listed.
template <typename T, int E>
__global__ void __launch_bounds__(128) distill_warp_kernel(const DistillArgs a) {
    __shared__ List s_list[4];
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= a.rows) return;
    const T *x = (const T *)a.x + row * a.x_row;
    T *dx = a.dx ? (T *)a.dx + row * a.dx_row : nullptr;
    const float weight = a.weight ? a.weight[row] : 1.f;
    if (weight == 0.f) {
        if (lane == 0) a.row_loss[row] = 0.f;
        for (int i = lane; dx && i < a.V; i += 32) dx[i] = from_f32<T>(0.f);
        return;
    }
    const double g = (double)weight * a.inv_t / (double)a.B;
    List &l = s_list[threadIdx.x >> 5];
    float f[E];
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = lane + 32 * i < a.V ? to_f32(x[lane + 32 * i]) : -INFINITY;
    make_list<T>(a, row, l, lane, true);
    uint32_t out = 0;
    for (int j = 0; j < a.k; ++j) {
        const int id = l.id[j];
        if (id >= 0 && (id & 31) == lane) out |= 1u << (id >> 5);
    }
    Stats st;
    st.reset();
    float m = kLowest;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if ((out >> i) & 1u) f[i] = -INFINITY;
        m = fmaxf(m, f[i]);
    }
    st.raise(m, a.c);
    accumulate<E, false>(st, f, a.c);
    warp_join(st, a.c);
    const RowTerms t = row_terms(a, l, st, g, lane);
    if (lane == 0) a.row_loss[row] = (float)t.loss;
    if (!dx) return;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (lane + 32 * i < a.V && !((out >> i) & 1u)) dx[lane + 32 * i] = from_f32<T>(t.rest * ex2(max_nan((f[i] - st.m) * a.c, kFar)));
    for (int j = lane; j < a.k; j += 32)
        if (l.first[j]) dx[l.id[j]] = from_f32<T>(listed_grad(a, l, t, g, j));
}

// loss[n] = sum_b weight * row_loss / B, rows of weight 0 left out; sums in double, in a fixed order.
__global__ void __launch_bounds__(256) distill_loss_kernel(int B, const float *__restrict__ row_loss, const float *__restrict__ weight,
                                                           float *__restrict__ loss) {
    __shared__ double s_sum[8];
    pdl_enter();
    const long long first = (long long)blockIdx.x * B;
    double s = 0.0;
    for (int b = threadIdx.x; b < B; b += 256) {
        const float w = weight ? weight[first + b] : 1.f;
        if (w != 0.f) s += (double)w * (double)row_loss[first + b];
    }
    s = warp_sum(s);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int i = 0; i < 8; ++i) s += s_sum[i];
        loss[blockIdx.x] = (float)(s / (double)B);
    }
}

}  // namespace lpdt

using namespace lpdt;

extern "C" lpdt_status lpdt_distill_topk(int32_t nodes, int32_t B, int32_t V, const void *logits, lpdt_dtype dtype, int64_t row_stride,
                                         float temperature, int32_t k, const float *teacher_logprob, const int32_t *teacher_index,
                                         int32_t tail, const float *row_weight, float *loss, float *row_loss, void *dlogits,
                                         int64_t dlogits_row_stride, int32_t *dev_status, void *stream) {
    LPDT_CHECK_ARG(nodes >= 0 && B >= 1 && V >= 1 && dtype_ok(dtype) && temperature_ok(temperature) && k >= 1 && (tail == 0 || tail == 1));
    if (nodes == 0) return LPDT_OK;
    const int64_t rows = (int64_t)nodes * B;
    LPDT_CHECK_ARG(logits && teacher_logprob && teacher_index && loss && row_loss);
    LPDT_CHECK_ARG(aligned(logits, dtype_size(dtype)) && (!dlogits || aligned(dlogits, dtype_size(dtype))));
    LPDT_CHECK_ARG(rows == 1 || (row_stride >= V && (!dlogits || dlogits_row_stride >= V)));
    LPDT_CHECK_ARG(dlogits != logits || rows == 1 || dlogits_row_stride == row_stride);
    if (k > kListMax || V > (1 << 20) || rows > (1 << 27)) return LPDT_ERR_UNSUPPORTED;
    DistillArgs a = {};
    a.x = logits; a.x_row = rows == 1 ? 0 : row_stride; a.dx = dlogits; a.dx_row = rows == 1 ? 0 : dlogits_row_stride;
    a.B = B; a.V = V; a.k = k; a.tail = tail; a.rows = rows;
    a.inv_t = 1.0 / (double)temperature; a.c = (float)(1.4426950408889634 / (double)temperature);
    a.value = teacher_logprob; a.index = teacher_index; a.weight = row_weight; a.row_loss = row_loss; a.dev_status = dev_status;
    const cudaStream_t st = as_stream(stream);
    const lpdt_status s = with_dtype(dtype, [&](auto t) -> lpdt_status {
        using T = decltype(t);
        if (V <= 1024) {
            const unsigned grid = (unsigned)ceil_div(rows, 4);
            if (V <= 64) launch_k(distill_warp_kernel<T, 2>, grid, 128, 0, st, a);
            else if (V <= 256) launch_k(distill_warp_kernel<T, 8>, grid, 128, 0, st, a);
            else launch_k(distill_warp_kernel<T, 32>, grid, 128, 0, st, a);
        } else {
            const int cs = row_share(rows, (int64_t)V * sizeof(T), 4, 4096);
            const size_t smem = align_up(ceil_div((int64_t)V + 2 * Row<T>::VE, cs) / 8 + 16, 16);
            static PerDeviceOnce attr;
            int dev;
            if (attr.pending(&dev)) {
                LPDT_CUDA(cudaFuncSetAttribute(distill_row_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDtSmem));
                attr.mark(dev);
            }
            launch_k_cluster(distill_row_kernel<T>, (unsigned)(rows * cs), kDtThreads, smem, st, cs, a);
        }
        LPDT_LAUNCH_CHECK();
        return LPDT_OK;
    });
    if (s != LPDT_OK) return s;
    launch_k(distill_loss_kernel, (unsigned)nodes, 256, 0, st, (int)B, (const float *)row_loss, row_weight, loss);
    LPDT_LAUNCH_CHECK();
    return LPDT_OK;
}
