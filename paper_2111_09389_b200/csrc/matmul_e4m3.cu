// lpdt_matmul_e4m3: C = A * B^T of two matrices of 8-bit floats whose blocks of 128 values along K have power-of-two scales.
//
// The tensor cores apply the scales: tcgen05.mma kind::mxf8f6f4 multiplies e4m3 operands by one UE8M0 factor per row and 32 values, so
// a block of 128 is four instructions that read the same factor, and the accumulator stays in tensor memory over all of K.
//
// The lanes of the accumulator are columns j of C (rows of B), its columns are rows m of C (rows of A): a warp of the epilogue then
// holds 32 neighbouring columns of C and stores each row's piece of 128 bytes in one instruction, whatever the alignment of C, the
// bias is one register, and few rows (one token) make a narrow accumulator instead of 128 rows of which one counts.
//
// G = 2: pairs of SMs (cta_group::2) on tiles of 256 columns by up to 224 rows, each CTA holding the codes of its 128 columns of C and
// of half of the rows; shared memory serves 128 bytes a cycle, which one SM's 128 x 224 would exceed (per 32 values of K 4 KB + 7 KB
// are written and read in 112 cycles).  G = 1: one SM, for what is too small to fill pairs; a cluster of SPLIT CTAs may share a tile's K
// and hand each other groups of eight rows of their accumulators through distributed shared memory, added in the order of
// the CTAs.
//
// Two accumulators of up to 224 columns (the epilogue of one tile runs under the products of the next) and four sets of scale factors
// fill the 512 columns of tensor memory; CTAs of one tile have one accumulator, and two of them fit an SM.  WIDE (G = 2): one accumulator of
// up to 416 columns, made by two instructions that share the codes of the columns of C: a quarter fewer bytes of codes for the same
// products (18 % fewer read from L2 with the scales and what does not fill a tile).  Its epilogue is alone, but the next tile's loads go on
// under it.
//
// Bound by the way from L2 to the SMs on two accumulators (48 bytes a cycle and SM, products 70 % of the cycles), by products (88 %) and the
// clock under the power cap on wide tiles.  8192^3 with a bf16 result 404 us after a pause (2722 TFLOP/s; 470 on two accumulators); seconds
// in a row at 1.34 to 1.41 GHz bf16 472 us (512 on two accumulators), fp32 485 (529), fp32 with an addend 532 (563).  4096^3 58; one token x
// 4096 x 4096 7.5, launch and first loads being most of it.
//
// Roles per CTA: warp 0 fetches codes (TMA), warp 1 copies scale factors to tensor memory and issues the products, warp 2 brings the
// scale bytes into the layout they are copied from, warps 4-11 run the epilogue.  Every wait on a barrier is bounded.
#include "dtypes.cuh"
#include "tc_common.cuh"

namespace lpdt {
namespace tc {

constexpr int kMmThreads = 384, kMmMaxStages = 10, kMmLaneBytes = 16384, kMmScaleSlots = 4, kMmMaxRows = 224 /*2 * 224 + 4 * 16 <= 512*/,
              kMmWideRows = 416 /*416 + 4 * 20 <= 512*/, kMmRaster = 8, kMmSoon = 8;
constexpr size_t kMmSmem = 227 * 1024;

struct MmParams {
    int nodes, M, N, kblocks, bn, bn0;         // bn: rows of C per tile, a multiple of 16; bn0: of the first instruction (WIDE), else bn
    int tilesJ, tilesM, stages, tmem_cols, accs;   // accs: accumulators, 1 where a CTA makes one tile
    int groups, per_cta;                       // SPLIT: groups of 8 rows of a tile that exist, most of them that one CTA adds up
    int slot;                                  // bytes of a stage: codes of both sides
    const uint8_t *sA, *sB;
    int spitch;                                // bytes of a row of scales
    const float *bias; long long bias_node;
    const void *addend;
    bool early;                                // ask for the addend before a tile's products end
    void *C; long long c_node, c_row;
    int32_t *dev_status;
};
struct MmCtl {
    unsigned long long full[kMmMaxStages], empty[kMmMaxStages], sf_full[kMmScaleSlots], sf_done[kMmScaleSlots], tmem_full[2], tmem_empty[2], soon[2];
    uint32_t tmem_base;
    volatile int abort_flag;
};

__device__ __forceinline__ uint32_t mm_cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void mm_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t mm_peer(uint32_t local, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local), "r"(rank));
    return a;
}
__device__ __forceinline__ void mm_arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void mm_prefetch(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ void mm_arrive_relaxed(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void mm_st_peer(uint32_t cluster_addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}
__device__ __forceinline__ void mm_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void mm_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Loads into this CTA that signal the barrier at `bar` (G = 2: the leader's).
template <int G> __device__ __forceinline__ void mm_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2) {
    if constexpr (G == 2)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
    else
        tma_load_3d(dst, map, bar, c0, c1, c2);
}
template <int G> __device__ __forceinline__ void mm_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t acc) {
    if constexpr (G == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc) : "memory");
}
// 32 rows of 16 bytes in shared memory to four columns of tensor memory, the same in each quarter of the lanes.
template <int G> __device__ __forceinline__ void mm_copy_scales(uint32_t taddr, uint64_t desc) {
    if constexpr (G == 2)
        asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
    else
        asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// The barrier (of both CTAs of a pair) is arrived at once what was issued so far has completed.
template <int G> __device__ __forceinline__ void mm_commit(uint32_t bar) {
    if constexpr (G == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        mma_commit(bar);
}
// kind::mxf8f6f4, e4m3 operands (both K-major), UE8M0 scale factors in byte `sf` of their words, M lanes x N columns.
__host__ __device__ constexpr uint32_t idesc_mx_e4m3(int M, int N, uint32_t sf = 0) {
    return (sf << 4) | ((uint32_t)(N >> 3) << 17) | (1u << 23) | ((uint32_t)(M >> 7) << 27) | (sf << 29);
}

struct MmTile { int node, jt, mt; };
// Groups of kMmRaster column tiles sweep all row tiles, so that the tiles in flight share operand panels in L2.
__device__ __forceinline__ MmTile mm_tile(const MmParams &p, int tile) {
    const int rows = p.nodes * p.tilesJ, per_group = kMmRaster * p.tilesM;
    const int g = tile / per_group, rem = tile - g * per_group;
    int gsize = rows - g * kMmRaster;
    if (gsize > kMmRaster) gsize = kMmRaster;
    MmTile t;
    t.mt = rem / gsize;
    const int row = g * kMmRaster + (rem - t.mt * gsize);
    t.node = row / p.tilesJ;
    t.jt = row - t.node * p.tilesJ;
    return t;
}

// WIDE: a tile's rows are those of two instructions, of bn0 and of bn - bn0 rows, and each CTA holds a half of both: the first half of the
// tile's rows is one CTA's, the second the other's, and the first bn0 / 2 rows of each half are the first instruction's.  The row of the tile
// that is column n of the accumulators (which lie side by side).
__device__ __forceinline__ int mm_wide_row(const MmParams &p, int n) {
    const bool second = n >= p.bn0;
    const int i = second ? n - p.bn0 : n, half = (second ? p.bn - p.bn0 : p.bn0) / 2;
    return (i >= half ? p.bn / 2 + i - half : i) + (second ? p.bn0 / 2 : 0);
}
// The rows of scales that a lane brings to tensor memory, every 32nd: of 128 columns of C and of up to 256 rows of it for each instruction.
// They come in sets of 128 rows, four words a lane.
template <bool WIDE> struct MmScaleRows {
    static constexpr int SETS = WIDE ? 5 : 3, BYTES = SETS * 512, COLUMNS = SETS == 3 ? 16 : 20;      // of a slot; columns of tensor memory
    const uint8_t *row[4 * SETS];
    int sets;
    __device__ __forceinline__ void set(const MmParams &p, const MmTile &t, int G, int rank, int lane) {
        sets = WIDE || p.bn > 128 ? SETS : 2;
        const int j0 = (t.jt * G + (G == 2 ? rank : 0)) * 128, m0 = t.mt * p.bn;
        const uint8_t *b = p.sB + (size_t)t.node * p.N * p.spitch, *a = p.sA + (size_t)t.node * p.M * p.spitch;
#pragma unroll
        for (int i = 0; i < 4 * SETS; ++i) {
            const int r = (i & 3) * 32 + lane + (i >= 8 && (i & 4) == 0 ? 128 : 0);      // sets 0; 1, 2; 3, 4
            const int n = i >= 12 ? p.bn0 + r : r, limit = WIDE && i < 12 ? p.bn0 : p.bn;
            const int at = i < 4 ? j0 + r : m0 + (WIDE ? mm_wide_row(p, n) : n);
            const bool have = i < 4 ? at < p.N : (n < limit && at < p.M);
            row[i] = have ? (i < 4 ? b : a) + (size_t)at * p.spitch : nullptr;
        }
    }
    __device__ __forceinline__ void fetch(uint32_t (&w)[4 * SETS], int word) const {
#pragma unroll
        for (int i = 0; i < 4 * SETS; ++i)
            w[i] = (i < 8 || sets > 2) && row[i] ? __ldg(reinterpret_cast<const uint32_t *>(row[i]) + word) : 0x7f7f7f7fu;
    }
};

// 16 rows of C from m on, column j of it per lane: what is added to them, and their storing.
template <typename OutT>
__device__ __forceinline__ void mm_addend(const MmParams &p, int node, int m, int j, OutT (&x)[16]) {
    if (!p.addend || j >= p.N) return;
    const OutT *a = (const OutT *)p.addend + (node * p.c_node + m * p.c_row + j);
    const int have = p.M - m;
    if (have >= 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i, a += p.c_row) x[i] = *a;
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i, a += p.c_row)
            if (i < have) x[i] = *a;
    }
}
template <typename OutT>
__device__ __forceinline__ void mm_store(const MmParams &p, int node, int m, int j, float (&f)[16], float bias, const OutT (&x)[16]) {
    if (j >= p.N) return;
    OutT *c = (OutT *)p.C + (node * p.c_node + m * p.c_row + j);
    const int have = p.M - m;
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = __fadd_rn(f[i], bias);
    }
    if (p.addend) {
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = __fadd_rn(f[i], to_f32(x[i]));
    }
    if (have >= 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i, c += p.c_row) *c = from_f32<OutT>(f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i, c += p.c_row)
            if (i < have) *c = from_f32<OutT>(f[i]);
    }
}

// SPLIT: the clusters' CTAs share one tile's K (G = 1), a CTA makes one tile.  WIDE: two instructions side by side (G = 2), one accumulator.
template <int G, bool SPLIT, bool WIDE, typename OutT>
__global__ void __launch_bounds__(kMmThreads, G == 1 ? 2 : 1)
matmul_e4m3_kernel(const __grid_constant__ CUtensorMap mapL /*B: lanes*/, const __grid_constant__ CUtensorMap mapR /*A: rows*/, const MmParams p) {
    static_assert(!(SPLIT && G == 2) && !(WIDE && G == 1), "one or the other");
    using Rows = MmScaleRows<WIDE>;
    extern __shared__ __align__(1024) unsigned char smem[];
    MmCtl *ctl = reinterpret_cast<MmCtl *>(smem);
    unsigned char *data = smem + 1024, *scales = data + (size_t)p.stages * p.slot;
    [[maybe_unused]] float *parts = reinterpret_cast<float *>(scales + kMmScaleSlots * Rows::BYTES);      // SPLIT: [CTA][group][8 rows][128 columns]
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = (G == 2 || SPLIT) ? mm_cluster_rank() : 0u;
    const uint32_t share = SPLIT ? (uint32_t)gridDim.y : 1u;            // gridDim.y = cluster size
    const int total = p.nodes * p.tilesJ * p.tilesM;
    const int first = (int)blockIdx.x / G, step = (int)gridDim.x / G;
    const int k_begin = SPLIT ? (int)((long long)p.kblocks * rank / share) : 0;
    const int k_end = SPLIT ? (int)((long long)p.kblocks * (rank + 1) / share) : p.kblocks;
    const int halfn = p.bn / G;                                         // rows of A per CTA
    const bool soon = !SPLIT && p.early && p.kblocks > kMmSoon;        // the epilogue hears of a tile's end so many blocks of K before

    // Each role waits for the kernels before this one at its first access of global memory, and does what it can before: the fetching warp
    // sets the barriers up and goes on (its loads need nothing else), the scales' warp asks for the first words, meanwhile.
    // The next kernel's CTAs may start once this one has its tensor memory: theirs, which they would hold while they wait, cannot keep it
    // from this one.  A CTA's first trigger, by whichever warp, is the one that counts, so only the warp that allocates gives it.
    if constexpr (SPLIT) mm_cluster_arrive();
    if (warp == 0) {
        if (lane == 0) {
            for (int i = 0; i < p.stages; ++i) { mbar_init(smem_u32(&ctl->full[i]), 1); mbar_init(smem_u32(&ctl->empty[i]), 1); }
            for (int i = 0; i < kMmScaleSlots; ++i) { mbar_init(smem_u32(&ctl->sf_full[i]), G); mbar_init(smem_u32(&ctl->sf_done[i]), 1); }
            for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&ctl->tmem_full[i]), 1); mbar_init(smem_u32(&ctl->tmem_empty[i]), 8 * G); mbar_init(smem_u32(&ctl->soon[i]), 1); }
            ctl->abort_flag = 0;
            mbar_fence_init();
        }
        __syncwarp();
    }
    if (warp == 1) {
        if constexpr (G == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(p.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            tmem_alloc(smem_u32(&ctl->tmem_base), (uint32_t)p.tmem_cols);
            tmem_relinquish();
        }
        pdl_trigger();
    }
    Rows rows;
    uint32_t next[4 * Rows::SETS];
    if (warp == 2) {
        rows.set(p, mm_tile(p, first < total ? first : 0), G, (int)rank, lane);
        pdl_wait();
        rows.fetch(next, k_begin >> 2);
    }
    tc_fence_before();
    if constexpr (G == 2) {
        __syncthreads();
        mm_cluster_sync();        // the other CTA's barriers are initialised
    } else if (warp == 0)
        asm volatile("bar.arrive 1, %0;" ::"n"(kMmThreads) : "memory");
    else
        named_bar_sync(1, kMmThreads);
    tc_fence_after();
    const uint32_t tmem_base = warp == 0 ? 0u : __shfl_sync(0xffffffffu, ctl->tmem_base, 0);

    if (warp == 0) {
        if (elect_one()) { tma_prefetch_desc(&mapL); tma_prefetch_desc(&mapR); }
        pdl_wait();
        int st = 0; uint32_t ph = 0;
        for (int tile = first; tile < total && !ctl->abort_flag; tile += step) {
            const MmTile t = mm_tile(p, tile);
            const int j0 = (t.jt * G + (G == 2 ? (int)rank : 0)) * 128, m0 = t.mt * p.bn + (G == 2 ? (int)rank * halfn : 0);
            for (int kb = k_begin; kb < k_end; ++kb) {
                if (!mbar_wait(smem_u32(&ctl->empty[st]), ph ^ 1, &ctl->abort_flag, p.dev_status)) break;
                const uint32_t full = G == 2 ? mm_peer(smem_u32(&ctl->full[st]), 0) : smem_u32(&ctl->full[st]);
                if (elect_one()) {
                    if (G == 1 || rank == 0) mbar_expect_tx(smem_u32(&ctl->full[st]), (uint32_t)(G * (kMmLaneBytes + halfn * 128)));
                    const uint32_t dst = smem_u32(data + (size_t)st * p.slot);
                    mm_load<G>(dst, &mapL, full, kb * 128, j0, t.node);
                    mm_load<G>(dst + kMmLaneBytes, &mapR, full, kb * 128, m0, t.node);
                }
                __syncwarp();
                if (++st == p.stages) { st = 0; ph ^= 1; }
            }
        }
        // commits reach the empty barriers (from the other CTA, G = 2): all of them before the CTA may end
        for (int i = 0; i < p.stages && !ctl->abort_flag; ++i) {
            mbar_wait(smem_u32(&ctl->empty[st]), ph ^ 1, &ctl->abort_flag, p.dev_status);
            if (++st == p.stages) { st = 0; ph ^= 1; }
        }
    } else if (warp == 1) {
        if (G == 1 || rank == 0) {
            pdl_wait();               // the limits of the waits below are for this kernel's own loads, not for the kernels before it
            const uint32_t idesc = idesc_mx_e4m3(128 * G, WIDE ? p.bn0 : p.bn);
            [[maybe_unused]] const uint32_t idesc1 = idesc_mx_e4m3(128 * G, p.bn - p.bn0);
            const uint64_t tpl = smem_desc(0, 16, 1024, 2), sc_tpl = smem_desc(0, 16, 128, 0);
            const uint32_t sf0 = tmem_base + p.accs * p.bn;
            // Groups of four blocks of K, counted over all tiles: `copied` have their factors in tensor memory or on their way.  A group's are
            // copied one group ahead of its products, which then do not wait for the copy.
            const uint32_t per_tile = (uint32_t)(((k_end - 1) >> 2) - (k_begin >> 2) + 1);
            const uint32_t groups = first < total ? per_tile * (uint32_t)((total - 1 - first) / step + 1) : 0u;
            uint32_t group = 0, copied = 0;
            auto copy = [&]() {
                const uint32_t slot = copied & (kMmScaleSlots - 1), turn = copied / kMmScaleSlots;
                // the columns' and the slot's last group, kMmScaleSlots before this one, has been used
                if (turn && !mbar_wait(smem_u32(&ctl->sf_done[slot]), (turn - 1) & 1, &ctl->abort_flag, p.dev_status)) return false;
                if (!mbar_wait(smem_u32(&ctl->sf_full[slot]), turn & 1, &ctl->abort_flag, p.dev_status)) return false;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t sc = smem_u32(scales + (size_t)slot * Rows::BYTES) >> 4, sf = sf0 + slot * Rows::COLUMNS;
                    mm_copy_scales<G>(sf, sc_tpl | (sc & 0x3FFFu));
                    mm_copy_scales<G>(sf + 4, sc_tpl | ((sc + 32) & 0x3FFFu));
                    if (WIDE || p.bn > 128) mm_copy_scales<G>(sf + 8, sc_tpl | ((sc + 64) & 0x3FFFu));
                    if constexpr (WIDE) {
                        mm_copy_scales<G>(sf + 12, sc_tpl | ((sc + 96) & 0x3FFFu));
                        mm_copy_scales<G>(sf + 16, sc_tpl | ((sc + 128) & 0x3FFFu));
                    }
                }
                __syncwarp();
                ++copied;
                return true;
            };
            int st = 0; uint32_t ph = 0, tcount = 0;
            bool ok = true;
            for (int tile = first; tile < total && ok && !ctl->abort_flag; tile += step, ++tcount) {
                const int acc = WIDE ? 0 : tcount & 1;
                if (!mbar_wait(smem_u32(&ctl->tmem_empty[acc]), ((WIDE ? tcount : tcount >> 1) & 1) ^ 1, &ctl->abort_flag, p.dev_status)) break;
                tc_fence_after();
                for (int kb = k_begin; kb < k_end && ok; ++kb) {
                    const bool fresh = kb == k_begin || (kb & 3) == 0;
                    if (fresh && copied == group) ok = copy();
                    if (!ok || !mbar_wait(smem_u32(&ctl->full[st]), ph, &ctl->abort_flag, p.dev_status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t slot = group & (kMmScaleSlots - 1);
                    const bool last = (kb & 3) == 3 || kb == k_end - 1;
                    if (elect_one()) {
                        const uint32_t byte = ((uint32_t)(kb & 3) << 4) | ((uint32_t)(kb & 3) << 29), sf = sf0 + slot * Rows::COLUMNS;
                        uint32_t l = smem_u32(data + (size_t)st * p.slot) >> 4, r = l + (kMmLaneBytes >> 4);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            mm_mma<G>(tmem_base + acc * p.bn, tpl | (l & 0x3FFFu), tpl | (r & 0x3FFFu), idesc | byte, sf, sf + 4, (uint32_t)((kb - k_begin) | k));
                            if constexpr (WIDE)
                                mm_mma<G>(tmem_base + p.bn0, tpl | (l & 0x3FFFu), tpl | ((r + p.bn0 * 4) & 0x3FFFu), idesc1 | byte, sf, sf + 12, (uint32_t)((kb - k_begin) | k));
                            l += 2; r += 2;
                        }
                        mm_commit<G>(smem_u32(&ctl->empty[st]));
                        if (last) mm_commit<G>(smem_u32(&ctl->sf_done[slot]));
                        if (soon && kb == k_end - 1 - kMmSoon) mm_commit<G>(smem_u32(&ctl->soon[acc]));
                        if (kb == k_end - 1) mm_commit<G>(smem_u32(&ctl->tmem_full[acc]));
                    }
                    __syncwarp();
                    if (++st == p.stages) { st = 0; ph ^= 1; }
                    if (fresh && copied == group + 1 && copied < groups) ok = copy();
                    if (last) ++group;
                }
            }
        }
    } else if (warp == 2) {
        // Row r of 128 goes to bytes (r % 32) * 16 + (r / 32) * 4 on: the word that holds its scales of four blocks of K (the instruction
        // names the byte).  The next words are on their way while this group waits for its slot.
        uint32_t group = 0;
        const int last = (k_end - 1) >> 2;
        for (int tile = first; tile < total && !ctl->abort_flag; tile += step) {
            if (tile != first) {
                rows.set(p, mm_tile(p, tile), G, (int)rank, lane);
                rows.fetch(next, k_begin >> 2);
            }
            bool ok = true;
            for (int g = k_begin >> 2; g <= last; ++g, ++group) {
                const int slot = group & (kMmScaleSlots - 1);
                uint32_t now[4 * Rows::SETS];
#pragma unroll
                for (int i = 0; i < 4 * Rows::SETS; ++i) now[i] = next[i];
                if (g < last) rows.fetch(next, g + 1);
                if (!mbar_wait(smem_u32(&ctl->sf_done[slot]), ((group / kMmScaleSlots) & 1) ^ 1, &ctl->abort_flag, p.dev_status)) { ok = false; break; }
                uint4 *dst = reinterpret_cast<uint4 *>(scales + (size_t)slot * Rows::BYTES) + lane;
#pragma unroll
                for (int i = 0; i < Rows::SETS; ++i)
                    if (i < rows.sets) dst[i * 32] = make_uint4(now[4 * i], now[4 * i + 1], now[4 * i + 2], now[4 * i + 3]);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (G == 2) mm_arrive_at(mm_peer(smem_u32(&ctl->sf_full[slot]), 0));
                    else mbar_arrive(smem_u32(&ctl->sf_full[slot]));
                }
            }
            if (!ok) break;
        }
        // (commits reach these barriers like the empty ones)
        for (int i = 0; i < kMmScaleSlots && !ctl->abort_flag; ++i, ++group)
            mbar_wait(smem_u32(&ctl->sf_done[group & (kMmScaleSlots - 1)]), ((group / kMmScaleSlots) & 1) ^ 1, &ctl->abort_flag, p.dev_status);
    } else if (warp >= 4) {
        const int q = warp & 3, half = (warp - 4) >> 2, chunks = p.bn / 16;
        const uint32_t empty0 = G == 2 ? mm_peer(smem_u32(&ctl->tmem_empty[0]), 0) : smem_u32(&ctl->tmem_empty[0]);
        uint32_t tcount = 0;
        // This warp's part of the accumulator is in registers.  Relaxed is enough between CTAs: what is handed over is tensor memory alone,
        // every lane's reads of it are complete (the wait for the loads), and they are ordered before the products that follow by the
        // tcgen05 fences on both sides of the arrival, not by the arrival.  A release orders memory, of which the receiver reads none, and would
        // wait for the stores to C of the whole tile (pairs: 8192 x 8192 x 512 77 us with it, 50 without).
        auto done = [&](int acc) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (G == 2) mm_arrive_relaxed(empty0 + acc * 8);
                else mbar_arrive(empty0 + acc * 8);
            }
        };
        pdl_wait();
        if constexpr (SPLIT) mm_cluster_wait();       // the others have started
        for (int tile = first; tile < total && !ctl->abort_flag; tile += step, ++tcount) {
            const MmTile t = mm_tile(p, tile);
            const int j = (t.jt * G + (G == 2 ? (int)rank : 0)) * 128 + q * 32 + lane, m0 = t.mt * p.bn;
            auto row_of = [&](int c) { return m0 + (WIDE ? mm_wide_row(p, c * 16) : c * 16); };
            const float bias = p.bias && j < p.N ? p.bias[t.node * p.bias_node + j] : 0.f;
            const int acc = WIDE ? 0 : tcount & 1;
            const uint32_t phase = (WIDE ? tcount : tcount >> 1) & 1;
            if constexpr (!SPLIT) {
                // what will be added comes to L2 under the last products (any earlier, and long K would drive it out again)
                if (p.early) {
                    if (soon && !mbar_wait(smem_u32(&ctl->soon[acc]), phase, &ctl->abort_flag, p.dev_status)) break;
                    const OutT *a = (const OutT *)p.addend + (t.node * p.c_node + (j - lane));
                    const int last = p.N - 1 - (j - lane);
                    for (int r = lane; r < (chunks - half + 1) / 2 * 16; r += 32) {
                        const int m = row_of(half + r / 16 * 2) + r % 16;
                        if (m < p.M && last >= 0) {
                            mm_prefetch(a + m * p.c_row);
                            mm_prefetch(a + m * p.c_row + (last < 31 ? last : 31));
                        }
                    }
                }
            }
            if (!mbar_wait(smem_u32(&ctl->tmem_full[acc]), phase, &ctl->abort_flag, p.dev_status)) break;
            tc_fence_after();
            const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * p.bn;
            uint32_t v[16];
            OutT next_x[16] = {};
            if (half < chunks) tmem_ld_32x16(t_row + half * 16, v);
            if (G == 2 && half < chunks) mm_addend<OutT>(p, t.node, row_of(half), j, next_x);
            for (int c = half; c < chunks; c += 2) {
                OutT x[16] = {};
                if constexpr (G == 2) {
                    // what is added to a piece is on its way while the piece before it is stored
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = next_x[i];
                    if (c + 2 < chunks) mm_addend<OutT>(p, t.node, row_of(c + 2), j, next_x);
                } else if constexpr (!SPLIT)
                    mm_addend<OutT>(p, t.node, row_of(c), j, x);
                tmem_ld_wait();
                float f[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(v[i]);
                if (c + 2 < chunks) tmem_ld_32x16(t_row + (c + 2) * 16, v);
                else done(acc);
                if constexpr (SPLIT) {
                    // groups of 8 rows go to the CTAs in turn, each to where that CTA keeps this one's
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int g = 2 * c + h;
                        if (g >= p.groups) continue;
                        const uint32_t slot = rank * (uint32_t)p.per_cta + (uint32_t)g / share;
                        const uint32_t to = mm_peer(smem_u32(parts + (size_t)slot * 1024 + q * 32 + lane), (uint32_t)g % share);
#pragma unroll
                        for (int i = 0; i < 8; ++i) mm_st_peer(to + i * 512, f[8 * h + i]);
                    }
                } else if (row_of(c) < p.M)
                    mm_store<OutT>(p, t.node, row_of(c), j, f, bias, x);
            }
            if (half >= chunks) done(acc);
        }
    }
    if constexpr (SPLIT) {
        if (warp < 4) mm_cluster_wait();
        __syncwarp();
        mm_cluster_sync();                        // every part has arrived
        if (warp >= 4 && !ctl->abort_flag) {
            const MmTile t = mm_tile(p, first);
            const int q = warp & 3, j = t.jt * 128 + q * 32 + lane, m0 = t.mt * p.bn;
            const float bias = p.bias && j < p.N ? p.bias[t.node * p.bias_node + j] : 0.f;
            for (int slot = (warp - 4) >> 2; slot < p.per_cta; slot += 2) {
                const int m = m0 + (slot * (int)share + (int)rank) * 8;
                if (slot * (int)share + (int)rank >= p.groups || m >= p.M) break;
                float s[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 0.f;
                for (uint32_t r = 0; r < share; ++r) {                  // in the order of the CTAs
                    const float *part = parts + ((size_t)r * p.per_cta + slot) * 1024 + q * 32 + lane;
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] = __fadd_rn(s[i], part[i * 128]);
                }
                MmParams e = p;
                if (e.M > m + 8) e.M = m + 8;
                OutT x[16] = {};
                mm_addend<OutT>(e, t.node, m, j, x);
                mm_store<OutT>(e, t.node, m, j, s, bias, x);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (G == 2) mm_cluster_sync();                // no CTA leaves while the other may still signal it
    if (warp == 1) {
        tc_fence_after();
        if constexpr (G == 2)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(p.tmem_cols) : "memory");
        else
            tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
    }
}

struct MmPlan { int g, bn, split, dense, wide; };
// What lpdt_last_kernel answers.
static const char *mm_name(const MmPlan &plan) {
    static const char *const wide[] = {"lpdt::tc::matmul_e4m3_kernel<pairs, 256 rows>", "lpdt::tc::matmul_e4m3_kernel<pairs, 288 rows>",
                                       "lpdt::tc::matmul_e4m3_kernel<pairs, 320 rows>", "lpdt::tc::matmul_e4m3_kernel<pairs, 352 rows>",
                                       "lpdt::tc::matmul_e4m3_kernel<pairs, 384 rows>", "lpdt::tc::matmul_e4m3_kernel<pairs, 416 rows>"};
    if (plan.wide) return wide[(plan.bn - 256) / 32];
    if (plan.g == 2) return "lpdt::tc::matmul_e4m3_kernel<pairs>";
    if (plan.split > 1) return plan.split == 2 ? "lpdt::tc::matmul_e4m3_kernel<K by 2>" : plan.split == 4 ? "lpdt::tc::matmul_e4m3_kernel<K by 4>" : "lpdt::tc::matmul_e4m3_kernel<K by 8>";
    return plan.dense ? "lpdt::tc::matmul_e4m3_kernel<two an SM>" : "lpdt::tc::matmul_e4m3_kernel<single>";
}

// The least of an estimate in cycles over pairs and single SMs, rows per tile and shares of K.  A block of 128 values of K takes a tile of bn
// rows the products' 2 * bn cycles or, where that is more, what its codes take from L2: 56 bytes a cycle of an SM by itself, 42 of one of
// a pair, 36 where the pair's tiles are wide.  An epilogue of `row` cycles a row (8, 10 of fp32, 16 with an addend) runs under the next
// tile's products, the last one by itself; three times that, being alone, behind a wide tile's products, and the next tile's loads go on
// meanwhile.  Clusters share K where one round of them is enough (a second would wait for whole clusters to end: 2048 x 2048 x 8192 94 us,
// 34 on wide tiles); those of 8 find room on 96 SMs at once.  `dense`: two CTAs of one tile each on an SM instead of one that walks over
// tiles, where one round of them is enough; one's epilogue then runs beside the other's loads, 32 bytes a cycle each.  (Fitted to every plan's
// time for 36 shapes from 1 x 4096 x 4096 to 8192 x 8192 x 16384, each with bf16 and fp32 results and an addend: 1.4 % above the best plan on
// average.  Wide against pairs of two accumulators: 8192^3 404 us, 470; 8192 x 8192 x 16384 900, 1127; 4096^3 58, 64; short K the other
// way, 8192 x 8192 x 512 64, 49.  Dense 2048^3 12.7, 14.7 wide, 15.3 on single SMs;
// 1 x 28672 x 4096 23.0, 25.1.)
static MmPlan mm_plan(int nodes, int64_t M, int64_t N, int64_t kblocks, double row) {
    MmPlan best = {1, 16, 1, 0, 0};
    double least = 1e300;
    const int64_t rows = (int64_t)align_up((size_t)M, 16);
    for (int g = 1; g <= 2; ++g) {
        const int64_t tj = ceil_div(N, 128 * g);
        for (int bn = 16 * g; bn <= kMmMaxRows; bn += 16 * g) {           // the instruction's column counts: by 16, in pairs by 32
            if (bn > rows) break;
            const int64_t tiles = (int64_t)nodes * tj * ceil_div(M, bn);
            const double bytes = kMmLaneBytes + bn * 128.0 / g;
            const double from_l2 = bytes / (g == 1 ? 56 : 42), per = from_l2 > 2.0 * bn ? from_l2 : 2.0 * bn;
            for (int split = 1; split <= (g == 1 && bn <= 128 ? 8 : 1); split *= 2) {
                if (split > kblocks) break;
                const int64_t slots = split == 8 ? 96 : kNumSMs / (g * split) * (g * split), waves = ceil_div(tiles * g * split, slots);
                if (split > 1 && waves > 1) break;
                const double k = ceil_div(kblocks, split) * per;
                const double cost = split > 1 ? k + 12.0 * bn + 900
                                              : (double)waves * (k + 600 > row * bn ? k + 600 : row * bn) + row / 2 * bn + (g == 2 ? 2000 : 0);
                if (cost < least) { least = cost; best = {g, bn, split, 0, 0}; }
            }
            if (g == 1 && bn <= 128 && tiles > kNumSMs && tiles <= 2 * kNumSMs) {
                const double shared = bytes / 32 > 4.0 * bn ? bytes / 32 : 4.0 * bn;
                const double cost = kblocks * shared + row * bn;
                if (cost < least) { least = cost; best = {1, bn, 1, 1, 0}; }
            }
        }
    }
    for (int bn = 256; bn <= kMmWideRows && (bn <= rows || (bn == 256 && M > kMmMaxRows)); bn += 32) {
        const int64_t waves = ceil_div((int64_t)nodes * ceil_div(N, 256) * ceil_div(M, bn), kNumSMs / 2);
        const double loads = kblocks * (kMmLaneBytes + bn * 64.0) / 36 + 500, work = kblocks * 2.0 * bn + 3 * row * bn;
        const double cost = (double)waves * (loads > work ? loads : work) + row / 2 * bn + 2000;
        if (cost < least) { least = cost; best = {2, bn, 1, 0, 1}; }
    }
    return best;
}

template <int G, bool SPLIT, bool WIDE, typename OutT>
static lpdt_status mm_launch(const CUtensorMap &mL, const CUtensorMap &mR, const MmParams &p, int64_t tiles, int split, size_t smem, cudaStream_t st) {
    static PerDeviceOnce attr;
    int dev;
    if (attr.pending(&dev)) {
        LPDT_CUDA(cudaFuncSetAttribute(matmul_e4m3_kernel<G, SPLIT, WIDE, OutT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMmSmem));
        attr.mark(dev);
    }
    if constexpr (SPLIT) {
        // the cluster runs along y: blockIdx.x is the tile
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)tiles, (unsigned)split); cfg.blockDim = kMmThreads; cfg.dynamicSmemBytes = smem; cfg.stream = st;
        cudaLaunchAttribute a[2];
        a[0].id = cudaLaunchAttributeClusterDimension;
        a[0].val.clusterDim.x = 1; a[0].val.clusterDim.y = (unsigned)split; a[0].val.clusterDim.z = 1;
        a[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        a[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = a;
        cfg.numAttrs = pdl_enabled() ? 2 : 1;
        ++g_launch_count;
        cudaLaunchKernelEx(&cfg, matmul_e4m3_kernel<G, SPLIT, WIDE, OutT>, mL, mR, p);
    } else {
        const int64_t ctas = tiles * G < kNumSMs || (p.accs == 1 && !WIDE) ? tiles * G : kNumSMs;
        launch_k_cluster(matmul_e4m3_kernel<G, SPLIT, WIDE, OutT>, (unsigned)ctas, kMmThreads, smem, st, G, mL, mR, p);
    }
    LPDT_LAUNCH_CHECK();
    return LPDT_OK;
}

}  // namespace tc
}  // namespace lpdt

using namespace lpdt;
using namespace lpdt::tc;

extern "C" lpdt_status lpdt_matmul_e4m3(int32_t nodes, int64_t M, int64_t N, int64_t K, const uint8_t *A, const uint8_t *sA,
                                        const uint8_t *B, const uint8_t *sB, const float *bias, int64_t bias_node_stride,
                                        const void *addend, void *C, lpdt_dtype c_dtype, int64_t c_node_stride,
                                        int64_t c_row_stride, int32_t *dev_status, void *stream) {
    LPDT_CHECK_ARG(nodes >= 0 && M >= 0 && N >= 0 && K >= 1 && dtype_ok(c_dtype));
    if (nodes == 0 || M == 0 || N == 0) return LPDT_OK;
    LPDT_CHECK_ARG(A && sA && B && sB && C);
    LPDT_CHECK_ARG(aligned(A, 16) && aligned(B, 16) && aligned(sA, 4) && aligned(sB, 4));
    LPDT_CHECK_ARG(aligned(C, dtype_size(c_dtype)) && (!addend || aligned(addend, dtype_size(c_dtype))) && aligned(dev_status, 4));
    LPDT_CHECK_ARG((M == 1 || c_row_stride >= N) && (nodes == 1 || c_node_stride >= (M - 1) * c_row_stride + N));
    LPDT_CHECK_ARG(!bias || (aligned(bias, 4) && (nodes == 1 || bias_node_stride >= 0)));
    const int64_t limit = (int64_t)1 << 30;
    if (M > limit || N > limit || K > limit) return LPDT_ERR_UNSUPPORTED;

    const int64_t kblocks = ceil_div(K, 128), pitch = lpdt_e4m3_pitch(K);
    const MmPlan plan = mm_plan(nodes, M, N, kblocks, addend ? 16.0 : c_dtype == LPDT_F32 ? 10.0 : 8.0);
    MmParams p = {};
    p.nodes = nodes; p.M = (int)M; p.N = (int)N; p.kblocks = (int)kblocks; p.bn = plan.bn;
    p.bn0 = plan.wide ? (int)align_up((size_t)plan.bn / 2, 32) : plan.bn;
    p.tilesJ = (int)ceil_div(N, 128 * plan.g); p.tilesM = (int)ceil_div(M, plan.bn);
    const int64_t tiles = (int64_t)nodes * p.tilesJ * p.tilesM;
    if (tiles > 0x3fffffff) return LPDT_ERR_UNSUPPORTED;
    p.slot = kMmLaneBytes + (int)align_up((size_t)(plan.bn / plan.g) * 128, 1024);
    p.groups = (int)ceil_div(M < plan.bn ? M : plan.bn, 8);
    p.per_cta = (int)ceil_div(p.groups, plan.split);
    const size_t rest = 1024 + kMmScaleSlots * (plan.wide ? MmScaleRows<true>::BYTES : MmScaleRows<false>::BYTES) + (plan.split > 1 ? (size_t)plan.split * p.per_cta * 4096 : 0);
    p.stages = (int)((kMmSmem - rest) / p.slot);
    if (p.stages > kMmMaxStages) p.stages = kMmMaxStages;
    // Few rows and short K: half of an SM's shared memory holds enough in flight, and the other half lets the next such call's CTAs start
    // (1 x 4096 x 4096 7.7 us, 8.1 with all of it; 1 x 8192 x 8192 the other way, 16.7 and 15.4).
    const int half = (int)((kMmSmem / 2 - 1024 - rest) / p.slot);
    if (plan.bn <= 64 && tiles * plan.split <= kNumSMs && ceil_div(kblocks, plan.split) <= 16 && half >= 4 && p.stages > half) p.stages = half;
    p.accs = plan.dense || plan.wide || plan.split > 1 ? 1 : 2;
    if (plan.dense) p.stages = half;
    for (p.tmem_cols = 128; p.tmem_cols < p.accs * plan.bn + kMmScaleSlots * (plan.wide ? MmScaleRows<true>::COLUMNS : MmScaleRows<false>::COLUMNS); p.tmem_cols *= 2) {}
    p.sA = sA; p.sB = sB; p.spitch = (int)lpdt_e4m3_scale_pitch(K);
    p.bias = bias; p.bias_node = nodes == 1 ? 0 : bias_node_stride;
    p.addend = addend; p.C = C; p.c_node = nodes == 1 ? 0 : c_node_stride; p.c_row = M == 1 ? 0 : c_row_stride;
    p.dev_status = dev_status;
    // Where the epilogue is not hidden: behind wide tiles (8192^3 fp32 553 -> 540 us), short K (8192 x 8192 x 512 fp32 138 -> 112) or a CTA's only
    // tile (512 x 4096 x 4096 fp32 17.8 -> 16.9).  Elsewhere it only disturbs the loads: 16384 x 4096 x 4096 fp32 257 us, 280 with it.
    p.early = addend && (plan.wide || kblocks <= kMmSoon || tiles * plan.g <= kNumSMs || p.accs == 1);

    CUtensorMap mL, mR;
    const uint64_t dL[3] = {(uint64_t)K, (uint64_t)N, (uint64_t)nodes}, sL[2] = {(uint64_t)pitch, (uint64_t)N * pitch};
    const uint64_t dR[3] = {(uint64_t)K, (uint64_t)M, (uint64_t)nodes}, sR[2] = {(uint64_t)pitch, (uint64_t)M * pitch};
    const uint32_t bL[3] = {128, 128, 1}, bR[3] = {128, (uint32_t)(plan.bn / plan.g), 1};
    if (!make_map_u8(&mL, B, 3, dL, sL, bL, CU_TENSOR_MAP_SWIZZLE_128B) || !make_map_u8(&mR, A, 3, dR, sR, bR, CU_TENSOR_MAP_SWIZZLE_128B))
        return LPDT_ERR_CUDA;
    const size_t smem = rest + (size_t)p.stages * p.slot;
    const cudaStream_t st = as_stream(stream);
    const lpdt_status s = with_dtype(c_dtype, [&](auto t) -> lpdt_status {
        using T = decltype(t);
        if (plan.wide) return mm_launch<2, false, true, T>(mL, mR, p, tiles, 1, smem, st);
        if (plan.g == 2) return mm_launch<2, false, false, T>(mL, mR, p, tiles, 1, smem, st);
        if (plan.split > 1) return mm_launch<1, true, false, T>(mL, mR, p, tiles, plan.split, smem, st);
        return mm_launch<1, false, false, T>(mL, mR, p, tiles, 1, smem, st);
    });
    if (s == LPDT_OK) g_last_kernel = mm_name(plan);
    return s;
}
