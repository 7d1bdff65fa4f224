// lpdt_distill_topk: distillation from a teacher's top log probabilities, loss and gradient.
//
// With z = x / T, S the listed tokens and p the student's softmax, the loss takes the student's probability of everything outside S as
// one more class.  Its logarithm is lse_R - lse with lse_R over the tokens outside S alone, not ln(1 - sum_S p), which would lose all
// digits once the list holds nearly all of the mass; so the pass over the row leaves S out (a bit per token in shared memory says which)
// and S, gathered by itself, joins at the end.  A token outside S has the gradient e^(z - m) times one number of the row, so the second
// pass is one exponential and one product a value; the listed tokens' gradients are written by the warp that has the list.
//
// Memory is the bound: the row once in, the gradient once out.  4096 x 131072 bf16, 64 listed, calls in a graph: 429 us (5.0 TB/s), 180 without the
// gradient (6.0 TB/s).
#include <type_traits>
#include "rows.cuh"

namespace lpdt {

constexpr int kDtUnroll = 4, kListMax = 128;
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

// A row's list in shared memory.
template <int K> struct List {
    double t[K], logt[K];
    double sum;                       // of t
    float x[K];                       // the student's logit
    int id[K];                        // -1: no entry
};
__device__ __forceinline__ double warp_max_d(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
// Makes the teacher's probabilities of a list whose logt are what it says (-inf: no entry): one warp, entries lane, lane + 32, ...
template <int K>
__device__ __forceinline__ void finish_list(const DistillArgs &a, List<K> &l, int lane) {
    constexpr int PER = K / 32;
    double logt[PER], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        logt[i] = lane + 32 * i < a.k ? l.logt[lane + 32 * i] : -INFINITY;
        top = fmax(top, logt[i]);
    }
    double shift = 0.0;
    if (!a.tail) {
        // the list as a distribution: minus the logarithm of its sum (a list of nothing but -inf stays as it is)
        top = warp_max_d(top);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (logt[i] > -INFINITY) sum += exp(logt[i] - top);
        sum = warp_sum(sum);
        if (top > -INFINITY) shift = top + log(sum);
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int j = lane + 32 * i;
        if (j >= a.k) continue;
        l.logt[j] = logt[i] - shift;
        l.t[j] = exp(logt[i] - shift);
        sum += l.t[j];
    }
    sum = warp_sum(sum);
    if (lane == 0) l.sum = sum;
    __syncwarp();
}
// Reads the list of a row first.
template <typename T, int K>
__device__ __forceinline__ void make_list(const DistillArgs &a, long long row, List<K> &l, int lane, bool report) {
    const T *x = (const T *)a.x + row * a.x_row;
    for (int j = lane; j < a.k; j += 32) {
        const int id = a.index[row * a.k + j];
        const bool have = id >= 0 && id < a.V;
        if (id >= a.V && report && a.dev_status) atomicCAS(a.dev_status, 0, (int32_t)LPDT_ERR_INVALID_ARG);
        l.id[j] = have ? id : -1;
        l.x[j] = have ? to_f32(x[id]) : -INFINITY;
        l.logt[j] = have ? (double)a.value[row * a.k + j] : -INFINITY;
    }
    __syncwarp();
    finish_list(a, l, lane);
}

// What a row's gradient comes from once the sums are known: st over the tokens outside the list, sl over those on it, each once.  Only
// sums and quotients: m is the larger maximum, all the sum relative to it.  left: the teacher's mass outside the list; rest: the factor of
// 2^((x - st.m) c) there.  A list that leaves nothing but mask values (-inf, or finite and their lse below -1e30) leaves no class of
// others.  A student's row of nothing but mask values has neither loss nor gradient.  Maxima pass NaN over, so one among mask values shows in
// the sums alone: `all` is NaN then, and so are the row's loss and every gradient.
struct RowTerms { double left, total /* sum t + left */, all; float m, rest; bool outside, masked; };
__device__ __forceinline__ RowTerms row_terms(const DistillArgs &a, double sum, const Stats &st, const Stats &sl, double g) {
    RowTerms r;
    r.outside = !(st.s == 0.f || (st.s == st.s && (double)st.m * a.inv_t < -1e30));
    const bool inside = !(sl.s == 0.f);
    r.m = r.outside && inside ? fmaxf(st.m, sl.m) : r.outside ? st.m : sl.m;
    const double from_rest = r.outside ? (double)st.s * (double)ex2(max_nan((st.m - r.m) * a.c, kFar)) : 0.0;
    const double from_list = inside ? (double)sl.s * (double)ex2(max_nan((sl.m - r.m) * a.c, kFar)) : 0.0;
    r.all = from_rest + from_list;
    r.left = a.tail && r.outside ? fmax(1.0 - sum, 0.0) : 0.0;
    r.total = sum + r.left;
    r.masked = r.all == r.all && ((!r.outside && !inside) || (double)r.m * a.inv_t < -1e30);
    r.rest = r.masked ? 0.f : r.outside ? (float)(g * (r.total * (from_rest / r.all) - r.left) / (double)st.s) : (float)(0.0 * r.all);
    return r;
}
// The loss, by one warp; its three logarithms are one computation on three lanes.  ln of the student's mass outside the list is taken
// from that mass's own sum, however small a part of the whole it is.
template <int K>
__device__ __forceinline__ double row_loss(const DistillArgs &a, const List<K> &l, const RowTerms &r, const Stats &st, int lane) {
    const double o = log(lane == 0 ? r.all : lane == 1 ? (double)st.s : r.left);
    const double log_all = __shfl_sync(0xffffffffu, o, 0), log_out = __shfl_sync(0xffffffffu, o, 1), log_left = __shfl_sync(0xffffffffu, o, 2);
    double loss = 0.0;
    for (int j = lane; j < a.k; j += 32)
        if (l.t[j] != 0.0) loss += l.t[j] * (l.logt[j] - (((double)l.x[j] - (double)r.m) * a.inv_t - log_all));
    loss = warp_sum(loss);
    if (r.left != 0.0) loss += r.left * (log_left - (((double)st.m - (double)r.m) * a.inv_t + log_out - log_all));
    return r.masked ? 0.0 : loss + 0.0 * r.all;                 // (a list without any mass: NaN all the same)
}
// The gradient of listed entry j's token, whose teacher's probability is that of all entries of it (`twice`: some token has several).
template <int K>
__device__ __forceinline__ float listed_grad(const DistillArgs &a, const List<K> &l, const RowTerms &r, double g, int j, bool twice) {
    if (r.masked) return 0.f;
    double t = l.t[j];
    if (twice) {
        t = 0.0;
        for (int i = 0; i < a.k; ++i)
            if (l.id[i] == l.id[j]) t += l.t[i];
    }
    return (float)(g * ((double)ex2(max_nan((l.x[j] - r.m) * a.c, kFar)) / r.all * r.total - t));
}

// A CTA's sums as they travel in its cluster.
__device__ __forceinline__ unsigned long long pack_sums(const Stats &st) { return ((unsigned long long)__float_as_uint(st.s) << 32) | __float_as_uint(st.m); }
__device__ __forceinline__ Stats unpack_sums(unsigned long long v) {
    Stats st;
    st.m = __uint_as_float((uint32_t)v);
    st.s = __uint_as_float((uint32_t)(v >> 32));
    st.w = 0.f;
    return st;
}

// The CTAs of a cluster share a row; the second pass reads its words again, and says of them and of the gradient that they will not be
// needed in L2, which leaves it to the words that wait for theirs.  (Tried instead and slower: words held in shared memory between the passes
// by CTAs that walk over rows, 612 us for 4096 x 131072 bf16 against 456, the exponentials of the two passes no longer side by side.)
template <typename T, int TH>
__global__ void __launch_bounds__(TH + 32, TH == 512 ? 2 : TH == 256 ? 4 : 8) distill_row_kernel(const DistillArgs a) {
    constexpr int VE = Row<T>::VE, U = kDtUnroll, WARPS = TH / 32, PER = kListMax / 32;
    extern __shared__ uint32_t s_bits[];              // a bit per element of this CTA's words: listed
    __shared__ List<kListMax> s_list;
    __shared__ unsigned long long s_warp[WARPS], s_listed, s_in[8], s_list_in[8];
    const uint32_t rank = rows_cluster_rank(), share = rows_cluster_size();
    if (share > 1) rows_cluster_arrive();
    pdl_enter();
    const long long row = blockIdx.x / share;
    const Row<T> r((const T *)a.x + row * a.x_row, a.V);
    T *dx = a.dx ? (T *)a.dx + row * a.dx_row : nullptr;
    const bool same = ((uintptr_t)(dx + r.head) & 15) == 0;
    const int begin = (int)((long long)r.words * rank / share), end = (int)((long long)r.words * (rank + 1) / share);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool lister = warp == WARPS;                // the last warp sees to the list, the others to the row
    const float weight = a.weight ? a.weight[row] : 1.f;
    const double g = (double)weight * a.inv_t / (double)a.B;
    const int edge = rank == 0 && tid < Row<T>::EDGES ? r.edge(tid) : -1;
    float at_edge = -INFINITY;
    // the first turn is asked for before anything else (also of a row of weight 0, which needs none of it)
    const int w0 = begin + tid;
    const bool full = !lister && w0 + (U - 1) * TH < end;
    uint4 ahead[U];
#pragma unroll
    for (int u = 0; u < U; ++u) ahead[u] = full ? r.load(w0 + u * TH) : make_uint4(0, 0, 0, 0);
    auto put = [&](int w, const float *f, uint32_t out) {
        T *to = dx + r.index(w);
        if (same && !out) __stcs(reinterpret_cast<uint4 *>(to), pack_vec<T>(f));
        else {
#pragma unroll
            for (int i = 0; i < VE; ++i)
                if (!((out >> i) & 1u)) to[i] = from_f32<T>(f[i]);
        }
    };

    if (weight == 0.f) {                              // the same for the whole cluster
        if (share > 1) { rows_cluster_wait(); rows_cluster_sync(); }
        if (rank == 0 && tid == 0) a.row_loss[row] = 0.f;
        if (!dx) return;
        const float zeros[VE] = {};
        for (int w = w0; w < end && !lister; w += TH) put(w, zeros, 0);
        if (edge >= 0) dx[edge] = from_f32<T>(0.f);
        return;
    }

    Stats st, sl;
    st.reset();
    sl.reset();
    int id[PER];
    uint32_t mine = 0;                                // the lister's: entry lane + 32 i is the one that stands for its token here
    bool again = false;                               // some token has several entries
    if (lister) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = lane + 32 * i;
            id[i] = j < a.k ? a.index[row * a.k + j] : -1;
            if (id[i] >= a.V) {
                if (rank == 0 && a.dev_status) atomicCAS(a.dev_status, 0, (int32_t)LPDT_ERR_INVALID_ARG);
                id[i] = -1;
            }
            if (j < a.k) s_list.id[j] = id[i] < 0 ? -1 : id[i];
        }
    } else {
        const int bit_words = ((end - begin) * VE + 31) / 32;
        for (int i = tid; i < bit_words; i += TH) s_bits[i] = 0;
    }
    __syncthreads();
    if (lister) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (id[i] < 0) continue;
            const int at = id[i] - r.index(begin);
            bool seen = false, here = true;
            if (at >= 0 && at < (end - begin) * VE) {
                const uint32_t bit = 1u << (at & 31);
                seen = atomicOr(&s_bits[at >> 5], bit) & bit;
            } else if (rank == 0 && (id[i] < r.head || id[i] >= r.index(r.words))) {
                for (int j = 0; j < lane + 32 * i; ++j) seen |= s_list.id[j] == id[i];       // on the edges: few, so by looking
            } else
                here = false;
            again |= here && seen;
            if (here && !seen) mine |= 1u << i;
        }
        if (__any_sync(0xffffffffu, again)) {         // which entry stands for its token does not go by who came first
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = id[i] < 0 ? -1 : id[i] - r.index(begin);
                bool stands = id[i] >= 0 && ((at >= 0 && at < (end - begin) * VE) || (rank == 0 && (id[i] < r.head || id[i] >= r.index(r.words))));
                for (int j = 0; j < lane + 32 * i && stands; ++j) stands = s_list.id[j] != id[i];
                mine = (mine & ~(1u << i)) | ((uint32_t)stands << i);
            }
        }
    }
    const bool twice = __syncthreads_or(again);
    const uint8_t *bytes = reinterpret_cast<const uint8_t *>(s_bits);
    auto listed = [&](int w) -> uint32_t {            // the bits of word w
        const int i = w - begin;
        return VE == 8 ? bytes[i] : (bytes[i >> 1] >> (4 * (i & 1))) & 15u;
    };
    if (lister) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = lane + 32 * i;
            if (j >= a.k) continue;
            const float x = id[i] >= 0 ? to_f32(r.at(id[i])) : -INFINITY;
            s_list.x[j] = x;
            s_list.logt[j] = id[i] >= 0 ? (double)a.value[row * a.k + j] : -INFINITY;
            if ((mine >> i) & 1u) {
                const float y[2] = {x, -INFINITY};
                if (x > sl.m) sl.raise(x, a.c);
                accumulate<2, false>(sl, y, a.c);
            }
        }
        __syncwarp();
        finish_list(a, s_list, lane);
        warp_join(sl, a.c);
        if (lane == 0) s_listed = pack_sums(sl);
    } else {
        auto word = [&](const uint4 &v, int w) {
            float f[VE];
            unpack_vec<T>(v, f);
            float m = vec_max<T>(v);
            const uint32_t out = listed(w);
            if (out) {
                m = kLowest;
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    if ((out >> i) & 1u) f[i] = -INFINITY;
                    m = fmaxf(m, f[i]);
                }
            }
            if (m > st.m) st.raise(m, a.c);
            accumulate<VE, false>(st, f, a.c);
        };
        int w = w0;
        if (full) {
#pragma unroll
            for (int u = 0; u < U; ++u) word(ahead[u], w + u * TH);
            w += U * TH;
        }
        for (; w + (U - 1) * TH < end; w += TH * U) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = r.load(w + u * TH);
#pragma unroll
            for (int u = 0; u < U; ++u) word(v[u], w + u * TH);
        }
        for (; w < end; w += TH) word(r.load(w), w);
        if (edge >= 0) {
            at_edge = to_f32(r.at(edge));
            bool out = false;
            for (int j = 0; j < a.k; ++j) out |= s_list.id[j] == edge;
            const float x[2] = {out ? -INFINITY : at_edge, -INFINITY};
            if (x[0] > st.m) st.raise(x[0], a.c);
            accumulate<2, false>(st, x, a.c);
        }
        warp_join(st, a.c);
        if (lane == 0) s_warp[warp] = pack_sums(st);
    }
    __syncthreads();
    // each warp joins the warps' sums for itself, which saves a barrier
    st.reset();
    if (lane < WARPS) st = unpack_sums(s_warp[lane]);
    warp_join(st, a.c);
    sl = unpack_sums(s_listed);
    if (share > 1) {
        // every CTA hands its sums to all
        rows_cluster_wait();                          // they have started
        if (warp == 0 && lane < (int)share) {
            st_peer_u64(&s_in[rank], lane, pack_sums(st));
            st_peer_u64(&s_list_in[rank], lane, pack_sums(sl));
        }
        // every CTA of the cluster has read what it gathers before any writes a gradient, which may lie where the logits do
        rows_cluster_sync();
        st.reset();
        sl.reset();
        if (lane < (int)share) { st = unpack_sums(s_in[lane]); sl = unpack_sums(s_list_in[lane]); }
        warp_join(st, a.c);
        warp_join(sl, a.c);
    }
    const RowTerms terms = row_terms(a, s_list.sum, st, sl, g);
    if (lister) {
        if (dx) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if ((mine >> i) & 1u) dx[id[i]] = from_f32<T>(listed_grad(a, s_list, terms, g, lane + 32 * i, twice));
        }
        if (rank == 0) {
            const double loss = row_loss(a, s_list, terms, st, lane);
            if (lane == 0) a.row_loss[row] = (float)loss;
        }
        return;
    }
    if (!dx) return;
    auto grad = [&](float x) { return terms.rest * ex2((x - st.m) * a.c); };
    const F2 minus_m = pack2(-st.m, -st.m), c2 = pack2(a.c, a.c), rest2 = pack2(terms.rest, terms.rest);
    auto word = [&](const uint4 &v, int w) {
        float f[VE];
        unpack_vec<T>(v, f);
#pragma unroll
        for (int i = 0; i < VE; i += 2) {
            float t0, t1;
            unpack2(mul2(add2(pack2(f[i], f[i + 1]), minus_m), c2), t0, t1);
            unpack2(mul2(pack2(ex2(t0), ex2(t1)), rest2), f[i], f[i + 1]);
        }
        put(w, f, listed(w));
    };
    int w = w0;
    constexpr int U2 = 32 / VE;                       // words of 32 values: of fp32 twice as many bytes on their way (4 x 512 x 131072: 494 -> 467 us)
    for (; w + (U2 - 1) * TH < end; w += TH * U2) {
        uint4 v[U2];
#pragma unroll
        for (int u = 0; u < U2; ++u) v[u] = r.load_last(w + u * TH);
#pragma unroll
        for (int u = 0; u < U2; ++u) word(v[u], w + u * TH);
    }
    for (; w < end; w += TH) word(r.load_last(w), w);
    if (edge >= 0) {
        bool out = false;
        for (int j = 0; j < a.k; ++j) out |= s_list.id[j] == edge;
        if (!out) dx[edge] = from_f32<T>(grad(at_edge));
    }
}

// A warp per row of at most 32 * E values; lane l holds those at l, l + 32, ..., bit i of `out` says that the i-th is listed.  Returns the
// row's loss times its weight, in lane 0.
template <typename T, int E, int K>
__device__ __forceinline__ double distill_row_of_warp(const DistillArgs &a, long long row, List<K> &l, int lane) {
    const T *x = (const T *)a.x + row * a.x_row;
    T *dx = a.dx ? (T *)a.dx + row * a.dx_row : nullptr;
    const float weight = a.weight ? a.weight[row] : 1.f;
    if (weight == 0.f) {
        if (lane == 0) a.row_loss[row] = 0.f;
        for (int i = lane; dx && i < a.V; i += 32) dx[i] = from_f32<T>(0.f);
        return 0.0;
    }
    const double g = (double)weight * a.inv_t / (double)a.B;
    float f[E];
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = lane + 32 * i < a.V ? to_f32(x[lane + 32 * i]) : -INFINITY;
    make_list<T>(a, row, l, lane, true);
    uint32_t out = 0;
    bool again = false;
    for (int j = 0; j < a.k; ++j) {
        const int id = l.id[j];
        if (id >= 0 && (id & 31) == lane) {
            again |= (out >> (id >> 5)) & 1u;
            out |= 1u << (id >> 5);
        }
    }
    const bool twice = __any_sync(0xffffffffu, again);
    Stats st, sl;
    st.reset();
    sl.reset();
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if ((out >> i) & 1u) sl.m = fmaxf(sl.m, f[i]);
        else st.m = fmaxf(st.m, f[i]);
    }
    float in[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        in[i] = (out >> i) & 1u ? f[i] : -INFINITY;
        if ((out >> i) & 1u) f[i] = -INFINITY;
    }
    accumulate<E, false>(st, f, a.c);
    accumulate<E, false>(sl, in, a.c);
    warp_join(st, a.c);
    warp_join(sl, a.c);
    const RowTerms t = row_terms(a, l.sum, st, sl, g);
    const double loss = row_loss(a, l, t, st, lane);
    if (lane == 0) a.row_loss[row] = (float)loss;
    if (dx) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (lane + 32 * i < a.V && !((out >> i) & 1u)) dx[lane + 32 * i] = from_f32<T>(t.rest * ex2(max_nan((f[i] - st.m) * a.c, kFar)));
        // (entries of one token write the same value)
        for (int j = lane; j < a.k; j += 32)
            if (l.id[j] >= 0) dx[l.id[j]] = from_f32<T>(listed_grad(a, l, t, g, j, twice));
    }
    return (double)weight * (double)(float)loss;
}
// Four rows a CTA.
template <typename T, int E, int K>
__global__ void __launch_bounds__(128) distill_warp_kernel(const DistillArgs a) {
    __shared__ List<K> s_list[4];
    pdl_enter();
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row < a.rows) distill_row_of_warp<T, E, K>(a, row, s_list[threadIdx.x >> 5], threadIdx.x & 31);
}
// A node's rows, at most 32, and its loss, with no launch more.
template <typename T, int E, int K>
__global__ void __launch_bounds__(1024) distill_node_kernel(const DistillArgs a, float *__restrict__ loss) {
    extern __shared__ __align__(16) unsigned char s_lists[];
    __shared__ double s_loss[32];
    pdl_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const double l = distill_row_of_warp<T, E, K>(a, (long long)blockIdx.x * a.B + warp, reinterpret_cast<List<K> *>(s_lists)[warp], lane);
    if (lane == 0) s_loss[warp] = l;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int b = 0; b < a.B; ++b) s += s_loss[b];
        loss[blockIdx.x] = (float)(s / (double)a.B);
    }
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
    LPDT_CHECK_ARG(aligned(teacher_logprob, 4) && aligned(teacher_index, 4) && aligned(loss, 4) && aligned(row_loss, 4) && aligned(row_weight, 4) && aligned(dev_status, 4));
    LPDT_CHECK_ARG(rows == 1 || (row_stride >= V && (!dlogits || dlogits_row_stride >= V)));
    LPDT_CHECK_ARG(dlogits != logits || rows == 1 || dlogits_row_stride == row_stride);
    if (k > kListMax || V > (1 << 20) || rows > (1 << 27)) return LPDT_ERR_UNSUPPORTED;
    DistillArgs a = {};
    a.x = logits; a.x_row = rows == 1 ? 0 : row_stride; a.dx = dlogits; a.dx_row = rows == 1 ? 0 : dlogits_row_stride;
    a.B = B; a.V = V; a.k = k; a.tail = tail; a.rows = rows;
    a.inv_t = 1.0 / (double)temperature; a.c = (float)(1.4426950408889634 / (double)temperature);
    a.value = teacher_logprob; a.index = teacher_index; a.weight = row_weight; a.row_loss = row_loss; a.dev_status = dev_status;
    const cudaStream_t st = as_stream(stream);
    bool done = false;
    const lpdt_status s = with_dtype(dtype, [&](auto t) -> lpdt_status {
        using T = decltype(t);
        if (V <= 1024) {
            // one launch for a node's rows and its loss where a CTA has a warp for each and they are short
            if (B <= 32 && V <= 256 && k <= 32) {
                auto fn = V <= 64 ? distill_node_kernel<T, 2, 32> : distill_node_kernel<T, 8, 32>;
                launch_k(fn, (unsigned)nodes, 32 * B, B * sizeof(List<32>), st, a, loss);
                LPDT_LAUNCH_CHECK();
                done = true;
                return LPDT_OK;
            }
            const unsigned grid = (unsigned)ceil_div(rows, 4);
            if (V <= 64) launch_k(distill_warp_kernel<T, 2, kListMax>, grid, 128, 0, st, a);
            else if (V <= 256) launch_k(distill_warp_kernel<T, 8, kListMax>, grid, 128, 0, st, a);
            else launch_k(distill_warp_kernel<T, 32, kListMax>, grid, 128, 0, st, a);
        } else {
            // Two CTAs for rows above 256 KB, so that the second pass of those in flight finds them in L2 (131072 fp32: 467 -> 424 us)
            int cs = row_share(rows, (int64_t)V * sizeof(T), 4, 4096);
            if (cs == 1 && (int64_t)V * (int64_t)sizeof(T) > 262144) cs = 2;
            const size_t smem = align_up(ceil_div((int64_t)V, cs) / 8 + 16, 16);
            // Threads by what a CTA reads, fewer for short rows, whose barriers and joins cost more than the reading; more where few rows leave
            // SMs idle.  (4096 rows of 30000 bf16 109 us on 128 threads, 117 on 256, 156 on 512; of 131072 bf16 526, 489, 444.)
            const int64_t bytes = (int64_t)V * (int64_t)sizeof(T) / cs * (rows * cs > 2 * kNumSMs ? 1 : 4);
            auto go = [&](auto threads) -> lpdt_status {
                constexpr int TH = decltype(threads)::value;
                static PerDeviceOnce attr;
                int dev;
                if (attr.pending(&dev)) {
                    LPDT_CUDA(cudaFuncSetAttribute(distill_row_kernel<T, TH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDtSmem));
                    attr.mark(dev);
                }
                launch_k_cluster(distill_row_kernel<T, TH>, (unsigned)(rows * cs), TH + 32, smem, st, cs, a);
                return LPDT_OK;
            };
            const lpdt_status s = bytes <= 65536 ? go(std::integral_constant<int, 128>()) : bytes <= 131072 ? go(std::integral_constant<int, 256>())
                                                                                          : go(std::integral_constant<int, 512>());
            if (s != LPDT_OK) return s;
        }
        LPDT_LAUNCH_CHECK();
        return LPDT_OK;
    });
    if (done) return LPDT_OK;
    if (s != LPDT_OK) return s;
    launch_k(distill_loss_kernel, (unsigned)nodes, 256, 0, st, (int)B, (const float *)row_loss, row_weight, loss);
    LPDT_LAUNCH_CHECK();
    return LPDT_OK;
}
