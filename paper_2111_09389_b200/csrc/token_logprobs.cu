// lpdt_token_logprobs and its backward pass: log probabilities of given tokens, entropy, log-sum-exp and the top alternatives of rows
// of logits, in one pass over them.
//
// Memory is the bound: a row is read once.  Each thread keeps the running maximum m and, relative to it, s = sum 2^t and
// w = sum 2^t * t; then lse = m/T + ln s and H = ln s - ln2 * w / s, without a second pass for the maximum or the entropy.
// The top k come out of the same pass: a thread remembers the two of its turns (of four words of 16 bytes) with the largest maxima, which
// costs a comparison a turn and no barrier.  At the end the threads' maxima give a floor that the k-th value cannot lie under, and what
// reaches it, a few more than k, is written to a list in shared memory and ranked.  Keys hold value and position, so equal values go to
// the lower position and a row of nothing but equal values needs no more than its first k.
//
// Few rows: the CTAs of a cluster share a row and join through distributed shared memory.  Rows of up to 1024 values: a warp each.
//
// 2048 x 131072 bf16, calls in a graph: 87.9 us without top k (6.1 TB/s), 107 with top 8, 149 with top 64; one row 4.0 us, top 20 8.8.
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
    RowAnswer() = default;
    __device__ __forceinline__ float lse() const { return none ? -INFINITY : (float)((double)m * inv_t + log_s); }
    __device__ __forceinline__ float entropy(const Stats &a) const { return none ? 0.f : (float)(log_s - kLn2 * (double)a.w / (double)a.s); }
};
template <typename T>
__device__ __forceinline__ void answer_row(const LogprobArgs &a, long long row, const Stats &st, const RowAnswer &r) {
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

constexpr int kLpUnroll = 4, kTopMax = 128;

// What could be among the k best of a row, and then the k best in order.
template <int TH> struct TopList {
    static constexpr int CAP = TH < 256 ? 8 * TH : 2048;
    __align__(16) unsigned long long key[CAP + 8];
    unsigned long long best[kTopMax];
    static constexpr int WORDS = 2 * TH;
    uint4 word[WORDS];                           // words that reach the floor, and the indices of their first elements
    int index[WORDS];
    int again[TH];                               // threads whose every word has to be looked at
    int count, words, agains;
};
// (The code behind a row's end runs once a row: a row by itself waits for each of its instructions to be fetched, so it is written to be
// short, in loops that are not unrolled.  Unrolled over a thread's words and keys the top 20 of one row took 10 us more than none, this 5.)

// The number of the n keys of the list that are larger; n is padded with zeros to a multiple of 8.
template <int TH>
__device__ __forceinline__ int larger_keys(const TopList<TH> &l, int n, unsigned long long mine) {
    const ulonglong2 *keys = reinterpret_cast<const ulonglong2 *>(l.key);
    int r = 0;
#pragma unroll 1
    for (int j = 0; j < n / 2; j += 4) {
        ulonglong2 k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = keys[j + i];
#pragma unroll
        for (int i = 0; i < 4; ++i) r += (k[i].x > mine) + (k[i].y > mine);
    }
    return r;
}
// Cuts the list of n keys to its k best, in order, by counting the larger ones of each: n is near k.
template <int TH>
__device__ __noinline__ void top_cut(TopList<TH> &l, int n, int k) {
    const int padded = (n + 7) & ~7;
    if ((int)threadIdx.x < padded - n) l.key[n + threadIdx.x] = 0;
    __syncthreads();
#pragma unroll 1
    for (int at = threadIdx.x; at < n; at += TH) {
        const unsigned long long mine = l.key[at];
        const int r = larger_keys(l, padded, mine);
        if (r < k) l.best[r] = mine;
    }
    __syncthreads();
    n = n < k ? n : k;
    if ((int)threadIdx.x < n) l.key[threadIdx.x] = l.best[threadIdx.x];
    if (threadIdx.x == 0) l.count = n;
    __syncthreads();
}

// The two turns of a thread (kLpUnroll words each, named by the first) with the largest maxima, of equal ones the earlier; NaN: none yet.
struct Best {
    float v1, v2;
    int w1, w2;
    __device__ __forceinline__ void reset() { v1 = v2 = NAN; w1 = w2 = -1; }
    __device__ __forceinline__ void see(float x, int at) {
        if (x != x) return;
        const bool first = !(x <= v1);
        v2 = first ? v1 : x;
        w2 = first ? w1 : at;
        v1 = first ? x : v1;
        w1 = first ? at : w1;
    }
};
// A warp's keys that reach the floor (0: none) onto the list.
template <int TH>
__device__ __forceinline__ void push(TopList<TH> &l, unsigned long long key, unsigned long long floor_key, int lane) {
    const uint32_t who = __ballot_sync(0xffffffffu, key && key >= floor_key);
    if (!who) return;
    int to = 0;
    if (lane == 0) to = atomicAdd(&l.count, __popc(who));
    to = __shfl_sync(0xffffffffu, to, 0) + __popc(who & ((1u << lane) - 1));
    if (((who >> lane) & 1u) && to < TopList<TH>::CAP) l.key[to] = key;
}
// Puts everything that reaches the floor on the list (`edges`: the row's edges too); its new length, which may exceed the room.  What reaches
// the floor lies in the turns that reach it, whose words that do are kept first, so that memory is waited for once; a thread whose second
// best turn does may have more, so a warp looks at all of its words.  Then the words are looked through, an element a lane.
template <typename T, int TH>
__device__ __noinline__ int collect(const Row<T> r, int begin, int end, bool edges, const Best b, unsigned long long floor_key, TopList<TH> &l) {
    constexpr int VE = Row<T>::VE;
    const float floor_v = floor_key ? key_value(floor_key) : -INFINITY;
    const uint32_t floor_i = (uint32_t)key_index(floor_key);          // the last position that counts among equal ones
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid == 0) l.count = l.words = l.agains = 0;
    __syncthreads();
    auto in = [&](float v, int w) { return v > floor_v || (v == floor_v && (uint32_t)r.index(w) <= floor_i); };
    auto keep = [&](const uint4 &v, int w) {
        if (!in(vec_max<T>(v), w)) return;
        const int to = atomicAdd(&l.words, 1);
        if (to < l.WORDS) { l.word[to] = v; l.index[to] = r.index(w); }
    };
    if (in(b.v1, b.w1)) {
        if (in(b.v2, b.w2)) l.again[atomicAdd(&l.agains, 1)] = begin + tid;
        else {
            const int words = b.w1 + (kLpUnroll - 1) * TH < end ? kLpUnroll : 1;
            uint4 v[kLpUnroll];
#pragma unroll
            for (int u = 0; u < kLpUnroll; ++u) v[u] = r.load(b.w1 + (u < words ? u : 0) * TH);
#pragma unroll
            for (int u = 0; u < kLpUnroll; ++u)
                if (u < words) keep(v[u], b.w1 + u * TH);
        }
    }
    __syncthreads();
    if (l.agains) {                              // a warp for each, two words a lane at a time
#pragma unroll 1
        for (int i = tid >> 5; i < l.agains; i += TH / 32)
#pragma unroll 1
            for (int w = l.again[i] + lane * TH; w < end; w += 64 * TH) {
                const uint4 v = r.load(w), v2 = r.load(w + 32 * TH < end ? w + 32 * TH : w);
                keep(v, w);
                if (w + 32 * TH < end) keep(v2, w + 32 * TH);
            }
        __syncthreads();
    }
    const int given = l.words, words = given < l.WORDS ? given : l.WORDS, elements = words * VE;
#pragma unroll 1
    for (int e0 = tid & ~31; e0 < elements; e0 += TH) {
        const int e = e0 + lane;
        int index = -1;
        float x = -INFINITY;
        if (e < elements) {
            index = l.index[e / VE] + e % VE;
            x = to_f32(reinterpret_cast<const T *>(l.word)[e]);
        }
        unsigned long long key = index >= 0 && x >= floor_v ? top_key(x, index) : 0;
        push(l, key, floor_key, lane);
    }
    if (edges && tid < 32) {
        const int index = tid < Row<T>::EDGES ? r.edge(tid) : -1;
        const float x = index >= 0 ? to_f32(r.at(index)) : 0.f;
        push(l, index >= 0 && x >= floor_v ? top_key(x, index) : 0ull, floor_key, lane);
    }
    __syncthreads();
    const int n = l.count, least = given > l.WORDS ? TopList<TH>::CAP + 1 : 0;
    __syncthreads();
    return n > least ? n : least;
}
// A floor that values tied in many places do not reach: the k-th largest of the threads' best values, each with the last position of the
// first word that holds it (0: fewer than k threads met a number).
template <typename T, int TH>
__device__ __noinline__ unsigned long long exact_floor(const Row<T> r, int end, const Best b, int k, TopList<TH> &l) {
    __shared__ unsigned long long s_floor;
    unsigned long long mine = 0;
    if (b.w1 >= 0) {
        int w = b.w1;
#pragma unroll 1
        while (w + TH < end && w < b.w1 + (kLpUnroll - 1) * TH && vec_max<T>(r.load(w)) != b.v1) w += TH;
        mine = top_key(b.v1, r.index(w) + Row<T>::VE - 1);
    }
    l.key[threadIdx.x] = mine;
    if (threadIdx.x == 0) s_floor = 0;
    __syncthreads();
    if (mine && larger_keys(l, TH, mine) == k - 1) s_floor = mine;
    __syncthreads();
    return s_floor;
}
// The k best of words [begin, end) and perhaps the edges, in order, from the threads' best turns.  A floor comes first: with
// M = ceil(k / warps), the least of the warps' M-th largest maxima; each warp has M lanes that reach it, so k values do.  Where many more
// do (ties: masked rows), a better floor takes less time than ranking them.
template <typename T, int TH>
__device__ __noinline__ void top_of_words(const Row<T> r, int begin, int end, bool edges, const Best b, int k, TopList<TH> &l) {
    __shared__ uint32_t s_least[TH / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int warps = (end - begin) / 32 < TH / 32 ? (end - begin) / 32 : TH / 32;      // whose lanes all have a word
    const int m = warps ? (k + warps - 1) / warps : 33;
    unsigned long long floor_key = 0;
    if (m <= 32) {
        uint32_t mine = b.w1 >= 0 ? order_bits(b.v1) : 0u, best = 0;
#pragma unroll 1
        for (int i = 0; i < m; ++i) {
            best = __reduce_max_sync(0xffffffffu, mine);
            const uint32_t who = __ballot_sync(0xffffffffu, mine == best);
            if (lane == __ffs(who) - 1) mine = 0;
        }
        if (lane == 0) s_least[warp] = best;
        __syncthreads();
        best = s_least[0];
        for (int w = 1; w < warps; ++w) best = min(best, s_least[w]);
        floor_key = (unsigned long long)best << 32;
    }
    int n = 2 * TH + 1;
    if (__syncthreads_count(b.w1 >= 0 && order_bits(b.v1) >= (uint32_t)(floor_key >> 32)) <= 2 * k + TH / 8)
        n = collect<T, TH>(r, begin, end, edges, b, floor_key, l);
    if (n > 2 * TH) {
        floor_key = exact_floor<T, TH>(r, end, b, k, l);
        n = collect<T, TH>(r, begin, end, edges, b, floor_key, l);
    }
    while (n > TopList<TH>::CAP) {
        // Still more than there is room for (rows in an order made for it, rows of mostly NaN): again from the k-th best of those
        // that had room, a floor that all but k of them no longer reach.
        // (a list that has no room for all words holds at least as many keys as words, but for one whose tie lies before the floor)
        top_cut(l, l.count < TopList<TH>::CAP ? l.count : TopList<TH>::CAP, k);
        floor_key = l.key[k - 1];
        __syncthreads();
        n = collect<T, TH>(r, begin, end, edges, b, floor_key, l);
    }
    top_cut(l, n, k);
}

// What the CTAs of a cluster hand to the first: (s, m), (length of the list, w), and the list.
template <int K> struct TopIn { unsigned long long part[8][2], key[8][K]; };          // lists end in zeros

template <typename T, bool TOP, int TH>
__global__ void __launch_bounds__(TH, (TOP ? 1280 : 1536) / TH) logprobs_row_kernel(const LogprobArgs a) {
    constexpr int VE = Row<T>::VE, U = kLpUnroll, WARPS = TH / 32;
    __shared__ TopList<TH> s_top;
    __shared__ Stats s_warp[WARPS];
    extern __shared__ __align__(16) unsigned char s_dynamic[];
    TopIn<TOP ? kTopMax : 1> &s_in = *reinterpret_cast<TopIn<TOP ? kTopMax : 1> *>(s_dynamic);      // in clusters
    const uint32_t rank = rows_cluster_rank(), share = rows_cluster_size();
    if (share > 1) rows_cluster_arrive();
    pdl_enter();
    const long long row = blockIdx.x / share;
    const Row<T> r((const T *)a.x + row * a.x_row, a.V);
    const int begin = (int)((long long)r.words * rank / share), end = (int)((long long)r.words * (rank + 1) / share);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

    Stats st;
    st.reset();
    Best best;
    best.reset();
    int w = begin + (int)threadIdx.x;
    for (; w + (U - 1) * TH < end; w += TH * U) {
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = r.load(w + u * TH);
        float top = vec_max<T>(v[0]);
#pragma unroll
        for (int u = 1; u < U; ++u) top = fmaxf(top, vec_max<T>(v[u]));
        if (TOP && !(top <= best.v2)) best.see(top, w);
        if (top > st.m) st.raise(top, a.c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[VE];
            unpack_vec<T>(v[u], f);
            accumulate<VE, true>(st, f, a.c);
        }
    }
    for (; w < end; w += TH) {
        const uint4 v = r.load(w);
        const float top = vec_max<T>(v);
        if (TOP && !(top <= best.v2)) best.see(top, w);
        if (top > st.m) st.raise(top, a.c);
        float f[VE];
        unpack_vec<T>(v, f);
        accumulate<VE, true>(st, f, a.c);
    }
    if (rank == 0 && threadIdx.x < Row<T>::EDGES && r.edge(threadIdx.x) >= 0) {
        const float x[2] = {to_f32(r.at(r.edge(threadIdx.x))), -INFINITY};
        if (x[0] > st.m) st.raise(x[0], a.c);
        accumulate<2, true>(st, x, a.c);
    }
    warp_join(st, a.c);
    if (lane == 0) s_warp[warp] = st;
    if (TOP) top_of_words<T, TH>(r, begin, end, rank == 0, best, a.k, s_top);
    __syncthreads();
    if (warp == 0) {
        st.reset();
        if (lane < WARPS) st = s_warp[lane];
        warp_join(st, a.c);
        __syncwarp();
        if (lane == 0) s_warp[0] = st;
    }
    if (share > 1) {
        // The others' sums and lists, each in order, go to the first CTA, which merges them.
        rows_cluster_wait();                                       // it has started
        __syncthreads();
        if (threadIdx.x == 0) {
            st_peer_u64(&s_in.part[rank][0], 0, ((unsigned long long)__float_as_uint(st.s) << 32) | __float_as_uint(st.m));
            st_peer_u64(&s_in.part[rank][1], 0, ((unsigned long long)(TOP ? s_top.count : 0) << 32) | __float_as_uint(st.w));
        }
        if (TOP && (int)threadIdx.x < a.k)
            st_peer_u64(&s_in.key[rank][threadIdx.x], 0, (int)threadIdx.x < s_top.count ? s_top.key[threadIdx.x] : 0ull);
        rows_cluster_sync();
        if (rank != 0) return;
        if (warp == WARPS - 1) {
            st.reset();
            if (lane < (int)share) {
                st.m = __uint_as_float((uint32_t)s_in.part[lane][0]);
                st.s = __uint_as_float((uint32_t)(s_in.part[lane][0] >> 32));
                st.w = __uint_as_float((uint32_t)s_in.part[lane][1]);
            }
            warp_join(st, a.c);
        }
        if (TOP) {
            // a key's place: its own in its list, and in each other list the number of larger keys, all found side by side
            int taken = 0;
            for (int i = threadIdx.x; i < (int)share * a.k; i += TH) {
                const int list = i / a.k, j = i - list * a.k;
                const unsigned long long mine = s_in.key[list][j];
                int pos[8] = {};
#pragma unroll 1
                for (int step = kTopMax; step > 0; step >>= 1) {
#pragma unroll
                    for (int o = 0; o < 8; ++o) {
                        const int to = pos[o] + step;
                        const unsigned long long other = s_in.key[o][to < kTopMax ? to - 1 : kTopMax - 1];
                        pos[o] = to <= a.k && other > mine ? to : pos[o];
                    }
                }
                int ahead = j;
#pragma unroll
                for (int o = 0; o < 8; ++o) ahead += o < (int)share && o != list ? pos[o] : 0;
                if (mine && ahead < a.k) { s_top.key[ahead] = mine; ++taken; }
            }
            if (threadIdx.x == 0) s_top.count = 0;
            __syncthreads();
            if (taken) atomicAdd(&s_top.count, taken);
        }
    }
    // One warp answers; the last, which has joined the cluster's sums.
    __shared__ RowAnswer s_answer;
    if (share == 1) __syncthreads();
    if (warp == WARPS - 1) {
        if (share == 1) st = s_warp[0];
        const RowAnswer ans(st, a.inv_t);
        if (lane == 0) {
            s_answer = ans;
            answer_row<T>(a, row, st, ans);
        }
    }
    if (TOP) {
        __syncthreads();
        if ((int)threadIdx.x < a.k) {
            const bool have = (int)threadIdx.x < s_top.count;
            const unsigned long long key = have ? s_top.key[threadIdx.x] : 0;
            a.top_logprob[row * a.k + threadIdx.x] = have ? s_answer.of(key_value(key)) : NAN;
            a.top_index[row * a.k + threadIdx.x] = have ? key_index(key) : -1;
        }
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
    const RowAnswer ans(st, a.inv_t);
    if (lane == 0) answer_row<T>(a, row, st, ans);
    if (a.k == 0) return;
    // Each turn takes the warp's largest.  The values' order bits lie in shared memory (0: no number, or taken; a number's are never 0), a lane
    // keeps the best of each group of eight of its own, and only the group that the taken one was in is looked through again.
    constexpr int GROUP = E < 8 ? E : 8, GROUPS = E / GROUP;
    __shared__ uint32_t s_order[4][E * 32];
    uint32_t *mine = s_order[threadIdx.x >> 5] + lane, best[GROUPS];
    int at[GROUPS];
#pragma unroll
    for (int i = 0; i < E; ++i) mine[32 * i] = f[i] == f[i] && lane + 32 * i < a.V ? order_bits(f[i]) : 0u;
    auto look = [&](int g) {
        uint32_t top = 0;
        int where = g * GROUP;
#pragma unroll
        for (int j = 0; j < GROUP; ++j) {
            const uint32_t o = mine[32 * (g * GROUP + j)];
            if (o > top) { top = o; where = g * GROUP + j; }
        }
#pragma unroll
        for (int q = 0; q < GROUPS; ++q)
            if (q == g) { best[q] = top; at[q] = where; }
    };
#pragma unroll 1
    for (int g = 0; g < GROUPS; ++g) look(g);
#pragma unroll 1
    for (int j = 0; j < a.k; ++j) {
        uint32_t own = best[0];
        int where = at[0];
#pragma unroll
        for (int q = 1; q < GROUPS; ++q)
            if (best[q] > own) { own = best[q]; where = at[q]; }
        const uint32_t top = __reduce_max_sync(0xffffffffu, own);
        const uint32_t index = __reduce_min_sync(0xffffffffu, own == top && top ? (uint32_t)(lane + 32 * where) : 0x7fffffffu);
        if (lane == 0) {
            a.top_logprob[row * a.k + j] = top ? ans.of(from_order_bits(top)) : NAN;
            a.top_index[row * a.k + j] = top ? (int32_t)index : -1;
        }
        if (!top) continue;
        const int gone = (int)(index >> 5);
        if (lane == (int)(index & 31)) mine[32 * gone] = 0;
        look(gone / GROUP);
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
        if (w0 + u * 32 < r.words) v[u] = r.load_last(w0 + u * 32);
    const int t = a.tokens ? a.tokens[row] : -1;
    const bool some = t >= 0 && t < a.V;
    const float lse = a.lse[row], g = a.g_logprob && some ? a.g_logprob[row] : 0.f;
    const float h = a.g_entropy ? a.g_entropy[row] : 0.f, l = a.g_lse ? a.g_lse[row] : 0.f;
    // (0 * lse: an lse beyond fp32 says nothing about p, so NaN and not the gradient of p = 0)
    const float base = fmaf(0.f, lse, l - g - (a.g_entropy ? h * a.entropy[row] : 0.f));
    const bool none = lse < -1e30f;              // nothing but mask values: no gradient
    auto grad = [&](float x, int index) {
        const float lp = max_nan(fmaf(x, a.inv_t, -lse), kFar), p = ex2(lp * kLog2e);
        float d = p * fmaf(-h, lp, base);
        if (none) d = 0.f;
        else if (index == t) d += g;
        return d * a.inv_t;
    };
    const bool same = ((uintptr_t)(dx + r.head) & 15) == 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int w = w0 + u * 32;
        if (w >= r.words) continue;
        float f[VE];
        unpack_vec<T>(v[u], f);
        const int first = r.index(w);
#pragma unroll
        for (int i = 0; i < VE; ++i) f[i] = grad(f[i], first + i);
        if (same) __stcs(reinterpret_cast<uint4 *>(dx + first), pack_vec<T>(f));
        else {
#pragma unroll
            for (int i = 0; i < VE; ++i) dx[first + i] = from_f32<T>(f[i]);
        }
    }
    if (item == row * a.chunks && lane < Row<T>::EDGES && r.edge(lane) >= 0)
        dx[r.edge(lane)] = from_f32<T>(grad(to_f32(r.at(r.edge(lane))), r.edge(lane)));
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
    LPDT_CHECK_ARG(aligned(tokens, 4) && aligned(logprob, 4) && aligned(entropy, 4) && aligned(lse, 4) && aligned(top_logprob, 4) && aligned(top_index, 4) && aligned(dev_status, 4));
    if (top_k > kTopMax || V > (1 << 30) || rows > (1 << 27)) return LPDT_ERR_UNSUPPORTED;
    LogprobArgs a = {};
    a.x = logits; a.x_row = rows == 1 ? 0 : row_stride; a.rows = rows; a.V = V;
    a.inv_t = 1.0 / (double)temperature; a.c = (float)(1.4426950408889634 / (double)temperature);
    a.tokens = tokens; a.logprob = logprob; a.entropy = entropy; a.lse = lse;
    a.top_logprob = top_logprob; a.top_index = top_index; a.k = top_k; a.dev_status = dev_status;
    const cudaStream_t st = as_stream(stream);
    return with_dtype(dtype, [&](auto t) -> lpdt_status {
        using T = decltype(t);
        // A warp's top k takes a turn for each.  Few rows wait for that: a CTA's, where its warps have lanes enough for a floor, is sooner from
        // 13 on (one row of 1000 fp32, top 20 6.7 us by a warp, 5.2 by a CTA; top 5 3.7 and 4.9; 8192 rows, top 20 31 and 41).
        const int full_warps = (int)((int64_t)V * (int64_t)sizeof(T) / 16 / 32);
        const bool by_cta = V > 1024 || (top_k > 12 && rows <= 4 * kNumSMs && top_k <= 32 * (full_warps < 4 ? full_warps : 4));
        if (!by_cta) {
            const unsigned grid = (unsigned)ceil_div(rows, 4);
            if (V <= 64) launch_k(logprobs_warp_kernel<T, 2>, grid, 128, 0, st, a);
            else if (V <= 256) launch_k(logprobs_warp_kernel<T, 8>, grid, 128, 0, st, a);
            else launch_k(logprobs_warp_kernel<T, 32>, grid, 128, 0, st, a);
        } else {
            const int cs = row_share(rows, (int64_t)V * sizeof(T), 4, 4096);
            const unsigned grid = (unsigned)(rows * cs);
            const size_t in = cs == 1 ? 0 : top_k ? sizeof(TopIn<kTopMax>) : sizeof(TopIn<1>);
            if ((int64_t)V * (int64_t)sizeof(T) / cs <= 16384)
                launch_k_cluster(top_k ? logprobs_row_kernel<T, true, 128> : logprobs_row_kernel<T, false, 128>, grid, 128, in, st, cs, a);
            else
                launch_k_cluster(top_k ? logprobs_row_kernel<T, true, 256> : logprobs_row_kernel<T, false, 256>, grid, 256, in, st, cs, a);
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
    LPDT_CHECK_ARG(aligned(tokens, 4) && aligned(lse, 4) && aligned(entropy, 4) && aligned(d_logprob, 4) && aligned(d_entropy, 4) && aligned(d_lse, 4));
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
        a.chunks = (int)ceil_div(V, 128 * VE);
        const int64_t blocks = ceil_div(rows * a.chunks, 8);
        if (blocks > 0x7fffffff) return LPDT_ERR_UNSUPPORTED;
        launch_k(logprobs_bwd_kernel<T>, (unsigned)blocks, 256, 0, st, a);
        LPDT_LAUNCH_CHECK();
        return LPDT_OK;
    });
}
