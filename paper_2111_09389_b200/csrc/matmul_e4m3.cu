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
// fill the 512 columns of tensor memory; CTAs of one tile have one accumulator, and two of them fit an SM.
//
// Bound by the way from L2 to the SMs (46 to 54 bytes a cycle) and by power where that is long: 8192^3 with a bf16 result 422 us after a pause
// (2606 TFLOP/s), 500 in a row at 1.55 GHz; 4096^3 64; one token x 4096 x 4096 7.5, launch and first loads being most of it.
//
// Roles per CTA: warp 0 fetches codes (TMA), warp 1 copies scale factors to tensor memory and issues the products, warp 2 brings the
// scale bytes into the layout they are copied from, warps 4-11 run the epilogue.  Every wait on a barrier is bounded.
#include "dtypes.cuh"
#include "tc_common.cuh"

namespace lpdt {
namespace tc {

constexpr int kMmThreads = 384, kMmMaxStages = 10, kMmLaneBytes = 16384, kMmScaleBytes = 1536, kMmScaleSlots = 4, kMmMaxRows = 224 /*2 * 224 + 4 * 16 <= 512*/, kMmRaster = 8;
constexpr size_t kMmSmem = 227 * 1024;

struct MmParams {
    int nodes, M, N, kblocks, bn;              // bn: rows of C per tile, a multiple of 16
    int tilesJ, tilesM, stages, tmem_cols, accs;   // accs: accumulators, 1 where a CTA makes one tile
    int groups, per_cta;                       // SPLIT: groups of 8 rows of a tile that exist, most of them that one CTA adds up
    int slot;                                  // bytes of a stage: codes of both sides
    const uint8_t *sA, *sB;
    int spitch;                                // bytes of a row of scales
    const float *bias; long long bias_node;
    const void *addend;
    void *C; long long c_node, c_row;
    int32_t *dev_status;
};
struct MmCtl {
    unsigned long long full[kMmMaxStages], empty[kMmMaxStages], sf_full[kMmScaleSlots], sf_done[kMmScaleSlots], tmem_full[2], tmem_empty[2];
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

// The rows of scales that a lane brings to tensor memory: of 128 columns of C and 256 rows of it, every 32nd.
struct MmScaleRows {
    const uint8_t *row[12];
    int sets;
    __device__ __forceinline__ void set(const MmParams &p, const MmTile &t, int G, int rank, int lane) {
        sets = p.bn > 128 ? 3 : 2;
        const int j0 = (t.jt * G + (G == 2 ? rank : 0)) * 128, m0 = t.mt * p.bn;
        const uint8_t *b = p.sB + (size_t)t.node * p.N * p.spitch, *a = p.sA + (size_t)t.node * p.M * p.spitch;
#pragma unroll
        for (int i = 0; i < 12; ++i) {
            const int r = (i & 3) * 32 + lane + (i >= 8 ? 128 : 0), at = (i < 4 ? j0 : m0) + r;
            const bool have = i < 4 ? at < p.N : (r < p.bn && at < p.M);
            row[i] = have ? (i < 4 ? b : a) + (size_t)at * p.spitch : nullptr;
        }
    }
    __device__ __forceinline__ void fetch(uint32_t (&w)[12], int word) const {
#pragma unroll
        for (int i = 0; i < 12; ++i)
            w[i] = (i < 8 || sets == 3) && row[i] ? __ldg(reinterpret_cast<const uint32_t *>(row[i]) + word) : 0x7f7f7f7fu;
    }
};

// 16 rows of C from m on, column j of it per lane.
template <typename OutT>
__device__ __forceinline__ void mm_store(const MmParams &p, int node, int m, int j, const float (&v)[16], float bias) {
    if (j >= p.N) return;
    const long long at = node * p.c_node + m * p.c_row + j;
    const int have = p.M - m;
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = v[i];
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = __fadd_rn(f[i], bias);
    }
    if (p.addend) {
        const OutT *a = (const OutT *)p.addend + at;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = i < have ? to_f32(a[i * p.c_row]) : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = __fadd_rn(f[i], x[i]);
    }
    OutT *c = (OutT *)p.C + at;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < have) c[i * p.c_row] = from_f32<OutT>(f[i]);
}

// SPLIT: the clusters' CTAs share one tile's K (G = 1), a CTA makes one tile.
template <int G, bool SPLIT, typename OutT>
__global__ void __launch_bounds__(kMmThreads, G == 1 ? 2 : 1)
matmul_e4m3_kernel(const __grid_constant__ CUtensorMap mapL /*B: lanes*/, const __grid_constant__ CUtensorMap mapR /*A: rows*/, const MmParams p) {
    static_assert(!(SPLIT && G == 2), "one or the other");
    extern __shared__ __align__(1024) unsigned char smem[];
    MmCtl *ctl = reinterpret_cast<MmCtl *>(smem);
    unsigned char *data = smem + 1024, *scales = data + (size_t)p.stages * p.slot;
    [[maybe_unused]] float *parts = reinterpret_cast<float *>(scales + kMmScaleSlots * kMmScaleBytes);      // SPLIT: [CTA][group][8 rows][128 columns]
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = (G == 2 || SPLIT) ? mm_cluster_rank() : 0u;
    const uint32_t share = SPLIT ? (uint32_t)gridDim.y : 1u;            // gridDim.y = cluster size
    const int total = p.nodes * p.tilesJ * p.tilesM;
    const int first = (int)blockIdx.x / G, step = (int)gridDim.x / G;
    const int k_begin = SPLIT ? (int)((long long)p.kblocks * rank / share) : 0;
    const int k_end = SPLIT ? (int)((long long)p.kblocks * (rank + 1) / share) : p.kblocks;
    const int halfn = p.bn / G;                                         // rows of A per CTA

    // Each role waits for the kernels before this one at its first access of global memory, and does what it can before: the fetching warp
    // sets the barriers up and goes on (its loads need nothing else), the scales' warp asks for the first words, meanwhile.
    // The next kernel's CTAs may start once this one has its tensor memory: theirs, which they would hold while they wait, cannot keep it
    // from this one.  A CTA's first trigger, by whichever warp, is the one that counts, so only the warp that allocates gives it.
    if constexpr (SPLIT) mm_cluster_arrive();
    if (warp == 0) {
        if (lane == 0) {
            for (int i = 0; i < p.stages; ++i) { mbar_init(smem_u32(&ctl->full[i]), 1); mbar_init(smem_u32(&ctl->empty[i]), 1); }
            for (int i = 0; i < kMmScaleSlots; ++i) { mbar_init(smem_u32(&ctl->sf_full[i]), G); mbar_init(smem_u32(&ctl->sf_done[i]), 1); }
            for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&ctl->tmem_full[i]), 1); mbar_init(smem_u32(&ctl->tmem_empty[i]), 8 * G); }
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
    MmScaleRows rows;
    uint32_t next[12];
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
            const uint32_t idesc = idesc_mx_e4m3(128 * G, p.bn);
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
                    const uint32_t sc = smem_u32(scales + (size_t)slot * kMmScaleBytes) >> 4, sf = sf0 + slot * 16;
                    mm_copy_scales<G>(sf, sc_tpl | (sc & 0x3FFFu));
                    mm_copy_scales<G>(sf + 4, sc_tpl | ((sc + 32) & 0x3FFFu));
                    if (p.bn > 128) mm_copy_scales<G>(sf + 8, sc_tpl | ((sc + 64) & 0x3FFFu));
                }
                __syncwarp();
                ++copied;
                return true;
            };
            int st = 0; uint32_t ph = 0, tcount = 0;
            bool ok = true;
            for (int tile = first; tile < total && ok && !ctl->abort_flag; tile += step, ++tcount) {
                const int acc = tcount & 1;
                if (!mbar_wait(smem_u32(&ctl->tmem_empty[acc]), ((tcount >> 1) & 1) ^ 1, &ctl->abort_flag, p.dev_status)) break;
                tc_fence_after();
                for (int kb = k_begin; kb < k_end && ok; ++kb) {
                    const bool fresh = kb == k_begin || (kb & 3) == 0;
                    if (fresh && copied == group) ok = copy();
                    if (!ok || !mbar_wait(smem_u32(&ctl->full[st]), ph, &ctl->abort_flag, p.dev_status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t slot = group & (kMmScaleSlots - 1);
                    const bool last = (kb & 3) == 3 || kb == k_end - 1;
                    if (elect_one()) {
                        const uint32_t id = idesc | ((uint32_t)(kb & 3) << 4) | ((uint32_t)(kb & 3) << 29), sf = sf0 + slot * 16;
                        uint32_t l = smem_u32(data + (size_t)st * p.slot) >> 4, r = l + (kMmLaneBytes >> 4);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            mm_mma<G>(tmem_base + acc * p.bn, tpl | (l & 0x3FFFu), tpl | (r & 0x3FFFu), id, sf, sf + 4, (uint32_t)((kb - k_begin) | k));
                            l += 2; r += 2;
                        }
                        mm_commit<G>(smem_u32(&ctl->empty[st]));
                        if (last) mm_commit<G>(smem_u32(&ctl->sf_done[slot]));
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
                uint32_t now[12];
#pragma unroll
                for (int i = 0; i < 12; ++i) now[i] = next[i];
                if (g < last) rows.fetch(next, g + 1);
                if (!mbar_wait(smem_u32(&ctl->sf_done[slot]), ((group / kMmScaleSlots) & 1) ^ 1, &ctl->abort_flag, p.dev_status)) { ok = false; break; }
                uint4 *dst = reinterpret_cast<uint4 *>(scales + (size_t)slot * kMmScaleBytes) + lane;
#pragma unroll
                for (int i = 0; i < 3; ++i)
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
        pdl_wait();
        if constexpr (SPLIT) mm_cluster_wait();       // the others have started
        for (int tile = first; tile < total && !ctl->abort_flag; tile += step, ++tcount) {
            const MmTile t = mm_tile(p, tile);
            const int j = (t.jt * G + (G == 2 ? (int)rank : 0)) * 128 + q * 32 + lane, m0 = t.mt * p.bn;
            const float bias = p.bias && j < p.N ? p.bias[t.node * p.bias_node + j] : 0.f;
            const int acc = tcount & 1;
            if (!mbar_wait(smem_u32(&ctl->tmem_full[acc]), (tcount >> 1) & 1, &ctl->abort_flag, p.dev_status)) break;
            tc_fence_after();
            const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * p.bn;
            uint32_t v[16];
            if (half < chunks) tmem_ld_32x16(t_row + half * 16, v);
            for (int c = half; c < chunks; c += 2) {
                tmem_ld_wait();
                float f[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(v[i]);
                if (c + 2 < chunks) tmem_ld_32x16(t_row + (c + 2) * 16, v);
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
                } else if (m0 + c * 16 < p.M)
                    mm_store<OutT>(p, t.node, m0 + c * 16, j, f, bias);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (G == 2) mm_arrive_at(empty0 + acc * 8);
                else mbar_arrive(empty0 + acc * 8);
            }
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
                mm_store<OutT>(e, t.node, m, j, s, bias);
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

struct MmPlan { int g, bn, split, dense; };

// The least of an estimate in cycles over pairs and single SMs, rows per tile and shares of K.  A block of 128 values of K takes a tile of bn
// rows the products' 2 * bn cycles or, where that is more, what its codes take from L2: 48 bytes a cycle of an SM by itself, 34 of one of
// a pair.  An epilogue of some 8 cycles a row runs under the next tile's products, the last one by itself.  Clusters of 8 find room on 96
// SMs at once.  `dense`: two CTAs of one tile each on an SM instead of one that walks over tiles, where one round of them is enough; one's
// epilogue then runs beside the other's loads, whose halves of the SM take 24 bytes a cycle each.  (Fitted to every plan's time for 29
// shapes from 1 x 4096 x 4096 to 4096^3: the plan is within 2 % of the best on average.  Pairs pay for themselves when every SM has
// several tiles of long K: 4096^3 65.0 us against 67.7 on single SMs, 2048^3 17.6 against 16.0; dense 2048^3 13.3 us; narrow tiles or
// dense ones would cost many tiles of short K a third: 2 x 4188 x 4744 x 259 42.9 us, 55.4 by a plan without the epilogue's share.)
static MmPlan mm_plan(int nodes, int64_t M, int64_t N, int64_t kblocks) {
    MmPlan best = {1, 16, 1, 0};
    double least = 1e300;
    for (int g = 1; g <= 2; ++g) {
        const int64_t tj = ceil_div(N, 128 * g);
        for (int bn = 16 * g; bn <= kMmMaxRows; bn += 16 * g) {           // the instruction's column counts: by 16, in pairs by 32
            if (bn > (int64_t)align_up((size_t)M, 16)) break;
            const int64_t tiles = (int64_t)nodes * tj * ceil_div(M, bn);
            const double bytes = kMmLaneBytes + bn * 128.0 / g;
            const double from_l2 = bytes / (g == 1 ? 48 : 34), per = from_l2 > 2.0 * bn ? from_l2 : 2.0 * bn;
            for (int split = 1; split <= (g == 1 && bn <= 128 ? 8 : 1); split *= 2) {
                if (split > kblocks) break;
                const int64_t slots = split == 8 ? 96 : kNumSMs / (g * split) * (g * split);
                const double waves = (double)ceil_div(tiles * g * split, slots), k = ceil_div(kblocks, split) * per;
                const double cost = split > 1 ? waves * (k + 12.0 * bn) + 900
                                              : waves * (k + 200 > 8.0 * bn ? k + 200 : 8.0 * bn) + 12.0 * bn + (g == 2 ? 1500 : 0);
                if (cost < least) { least = cost; best = {g, bn, split, 0}; }
            }
            if (g == 1 && bn >= 64 && bn <= 128 && tiles > kNumSMs && tiles <= 2 * kNumSMs) {
                const double shared = bytes / 24 > 4.0 * bn ? bytes / 24 : 4.0 * bn;
                const double cost = kblocks * shared + 8.0 * bn;
                if (cost < least) { least = cost; best = {1, bn, 1, 1}; }
            }
        }
    }
    return best;
}

template <int G, bool SPLIT, typename OutT>
static lpdt_status mm_launch(const CUtensorMap &mL, const CUtensorMap &mR, const MmParams &p, int64_t tiles, int split, size_t smem, cudaStream_t st) {
    static PerDeviceOnce attr;
    int dev;
    if (attr.pending(&dev)) {
        LPDT_CUDA(cudaFuncSetAttribute(matmul_e4m3_kernel<G, SPLIT, OutT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMmSmem));
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
        cudaLaunchKernelEx(&cfg, matmul_e4m3_kernel<G, SPLIT, OutT>, mL, mR, p);
    } else {
        const int64_t ctas = tiles * G < kNumSMs || p.accs == 1 ? tiles * G : kNumSMs;
        launch_k_cluster(matmul_e4m3_kernel<G, SPLIT, OutT>, (unsigned)ctas, kMmThreads, smem, st, G, mL, mR, p);
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
    const MmPlan plan = mm_plan(nodes, M, N, kblocks);
    MmParams p = {};
    p.nodes = nodes; p.M = (int)M; p.N = (int)N; p.kblocks = (int)kblocks; p.bn = plan.bn;
    p.tilesJ = (int)ceil_div(N, 128 * plan.g); p.tilesM = (int)ceil_div(M, plan.bn);
    const int64_t tiles = (int64_t)nodes * p.tilesJ * p.tilesM;
    if (tiles > 0x3fffffff) return LPDT_ERR_UNSUPPORTED;
    p.slot = kMmLaneBytes + (int)align_up((size_t)(plan.bn / plan.g) * 128, 1024);
    p.groups = (int)ceil_div(M < plan.bn ? M : plan.bn, 8);
    p.per_cta = (int)ceil_div(p.groups, plan.split);
    const size_t rest = 1024 + kMmScaleSlots * kMmScaleBytes + (plan.split > 1 ? (size_t)plan.split * p.per_cta * 4096 : 0);
    p.stages = (int)((kMmSmem - rest) / p.slot);
    if (p.stages > kMmMaxStages) p.stages = kMmMaxStages;
    // Few rows: half of an SM's shared memory holds enough of them in flight, and the other half lets the next such call's CTAs start.
    const int half = (int)((kMmSmem / 2 - 1024 - rest) / p.slot);
    if (plan.bn <= 64 && tiles * plan.split <= kNumSMs && half >= 4 && p.stages > half) p.stages = half;
    p.accs = plan.dense || plan.split > 1 ? 1 : 2;
    if (plan.dense) p.stages = half;
    for (p.tmem_cols = 128; p.tmem_cols < p.accs * plan.bn + kMmScaleSlots * 16; p.tmem_cols *= 2) {}
    p.sA = sA; p.sB = sB; p.spitch = (int)lpdt_e4m3_scale_pitch(K);
    p.bias = bias; p.bias_node = nodes == 1 ? 0 : bias_node_stride;
    p.addend = addend; p.C = C; p.c_node = nodes == 1 ? 0 : c_node_stride; p.c_row = M == 1 ? 0 : c_row_stride;
    p.dev_status = dev_status;

    CUtensorMap mL, mR;
    const uint64_t dL[3] = {(uint64_t)K, (uint64_t)N, (uint64_t)nodes}, sL[2] = {(uint64_t)pitch, (uint64_t)N * pitch};
    const uint64_t dR[3] = {(uint64_t)K, (uint64_t)M, (uint64_t)nodes}, sR[2] = {(uint64_t)pitch, (uint64_t)M * pitch};
    const uint32_t bL[3] = {128, 128, 1}, bR[3] = {128, (uint32_t)(plan.bn / plan.g), 1};
    if (!make_map_u8(&mL, B, 3, dL, sL, bL, CU_TENSOR_MAP_SWIZZLE_128B) || !make_map_u8(&mR, A, 3, dR, sR, bR, CU_TENSOR_MAP_SWIZZLE_128B))
        return LPDT_ERR_CUDA;
    const size_t smem = rest + (size_t)p.stages * p.slot;
    const cudaStream_t st = as_stream(stream);
    return with_dtype(c_dtype, [&](auto t) -> lpdt_status {
        using T = decltype(t);
        if (plan.g == 2) return mm_launch<2, false, T>(mL, mR, p, tiles, 1, smem, st);
        if (plan.split > 1) return mm_launch<1, true, T>(mL, mR, p, tiles, plan.split, smem, st);
        return mm_launch<1, false, T>(mL, mR, p, tiles, 1, smem, st);
    });
}
