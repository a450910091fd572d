// Products of microscaled matrices, large ones of e2m1: tiles of 256 x 256 by pairs of CTAs (see mx_matmul.cu for the others).
//
// A CTA alone moves 51 KB into its shared memory for each stage of a 128 x 256 tile and reads 48 KB out again, 1.5 times what shared
// memory gives while the tensor cores take the stage.  Of a pair each CTA brings its own 128 rows of P and half of the tile's 256 rows
// of S, 35 KB, and the first one's thread issues products (cta_group::2) that read both shared memories; each keeps the sums of its own
// rows.  Codes come as boxes of tensor maps, because their arrival has to be counted at the first CTA's barrier.
//
// Scales: copied into tensor memory by the issuing thread (tcgen05.cp), they stop the tensor cores, about 24 ns for each 512 bytes, 6 a
// stage of e2m1.  Here four warps read them from shared memory and store them to their quarter of the lanes, while earlier stages are
// multiplied; all 8 warps of a pair report to the first CTA before it issues the stage.
//
// Pairs and CTAs alone, us, back to back, rows of k numbers (k at the end):
//   8192 x 8192 x  2048 96.2 and 89.8   2560 98.1 and 100.8   2816 99.0 and 106.5   3584 114 and 125   4096 126 and 138
//   4096 x 4096 x  2048 28.3 and 27.0   2816 31.4 and 31.5    3584 35.8 and 37.6    4096 38.6 and 41.1   8192 62.3 and 69.9
//   16384 x 8192 x 2048 184 and 170     2816 195 and 194      3584 225 and 230;     5000 x 5000 x 2048 39.5 and 39.4   2816 44.4 and 48.0
//   2304 x 4096 x 4096 (144 tiles, one round and a little more) 23.7 and 23.3, 3000 x 3100 x 4096 (156) 28.9 and 29.4
// so that pairs begin at 11 stages (2561 numbers) and 148 tiles.  For e4m3, with 3 copies of scales a stage, the two are equal (8192 x 8192 x 8192
// 474 and 477 us).
//
// What orders what: a stage's shared memory and scale columns are filled again once the commit of its products has come (to both
// CTAs); products begin once both CTAs' codes have landed and both CTAs' scales are stored; a tile's accumulator is given back by all
// 16 warps that read it.  Waits are bounded as in mx_matmul.cu; nobody leaves before the other's arrivals have come.  Whoever gives up, neither CTA takes
// a tile for summed whose last commit has not come to it.
#include <cuda.h>          // types of tensor maps alone; the call comes from the runtime

#include "mx_product.cuh"

namespace divk {

constexpr uint32_t MXR_THREADS = 448, MXR_SCALERS = 10;         // warps 10..13 store scales

struct MxPairParams {
    MxProductParams p;
    alignas(64) CUtensorMap codes_p, codes_s;                    // rows of 128 bytes, 128 a box
};
constexpr uint32_t MXR_CODES = 16384u, MXR_ATOMS = MxFormat<MX_E2M1>::ATOMS, MXR_SCALES = 512u * MXR_ATOMS;      // bytes of 128 rows
constexpr uint32_t MXR_STAGES = 6u, MXR_STAGE_BYTES = 2u * MXR_CODES + 3u * MXR_SCALES, MXR_COLUMNS = 12u * MXR_ATOMS;      // columns of a stage's scales
constexpr uint32_t MXR_SMEM = 1024u + MXR_STAGES * MXR_STAGE_BYTES + (uint32_t)sizeof(MxCtl);
static_assert(MXR_STAGE_BYTES % 1024u == 0u && MXR_SMEM <= 227u * 1024u && 256u + MXR_STAGES * MXR_COLUMNS <= 512u && MXR_STAGES <= MXP_MAX_STAGES,
              "shared and tensor memory");

__device__ __forceinline__ void mxr_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
// arrives at both CTAs when all that this thread has issued is done
__device__ __forceinline__ void mxr_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3)
                 : "memory");
}
// an arrival at the first CTA (relaxed: what it tells of, reads and stores of tensor memory that have ended, is ordered by the fence before it)
__device__ __forceinline__ void mxr_arrive_first(uint64_t* bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_at(smem_u32(bar), 0u)) : "memory");
}
// 128 rows of 128 bytes from row y of the map on, counted at the first CTA's barrier
__device__ __forceinline__ void mxr_box(void* to, const CUtensorMap* map, uint32_t y, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(to)),
                 "l"(map), "r"(0), "r"((int)y), "r"(cluster_at(smem_u32(bar), 0u))
                 : "memory");
}
__device__ __forceinline__ void mxr_store4(uint32_t at, const uint4& v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__global__ void __launch_bounds__(MXR_THREADS, 1)
mx_pair_kernel(const __grid_constant__ MxPairParams g) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    MxCtl* ctl = reinterpret_cast<MxCtl*>(ring + MXR_STAGES * MXR_STAGE_BYTES);
    const MxProductParams& p = g.p;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t half = cluster_rank(), first = blockIdx.x / 2u, step = gridDim.x / 2u, all = p.p.s.stages;

    if (warp == MXP_ISSUER) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&ctl->tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < MXR_STAGES; ++i) {
            mbar_init(&ctl->full[i], 1);
            mbar_init(&ctl->scaled[i], 1);
            mbar_init(&ctl->ready[i], 8);
            mbar_init(&ctl->empty[i], 1);
        }
        mbar_init(&ctl->done, 1);
        mbar_init(&ctl->taken, 16);
        mbar_init(&ctl->last, 1);
        ctl->failed = 0;
        ctl->asked = 0xFFFFFFFFu;
        fence_barrier_init();
        fence_proxy_async();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                                     // (the other's barriers are there)
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *(volatile uint32_t*)&ctl->tmem, scales0 = tmem + 256u;
    griddep_wait();
    griddep_launch();

    if (warp == MXP_PRODUCER && lane == 0) {
        // what a box takes from beyond its matrix (a last block that is no 128 rows high, a block that is not there) ends in lanes and
        // columns that nobody keeps
        const uint32_t blocks_p = (p.p.s.rows + 127u) / 128u, blocks_s = (p.s.s.rows + 127u) / 128u;
        uint32_t asked = 0;
        bool ok = true;
        const uint32_t starved = blockIdx.x == p.starved_cta ? p.starved_copy : 0xFFFFFFFFu;
        for (uint32_t tile = first; tile < p.tiles && ok; tile += step) {
            const uint32_t bp = tile % p.tiles_p * 2u + half, bs = tile / p.tiles_p * 2u;
            const uint32_t mine = bp < blocks_p ? bp : 0u, own = bs + half < blocks_s ? bs + half : 0u, other = bs + 1u < blocks_s ? bs + 1u : 0u;
            const uint32_t hp = mx_tile_rows(p.p.s, mine), hs = mx_tile_rows(p.s.s, own);
            const uint32_t yp = mine * all * 128u, ys = own * all * 128u;              // the first stage's tiles, in rows of 128 bytes
            const unsigned char* zp = p.p.scales + (uint64_t)mine * all * MXR_SCALES;
            const unsigned char* z0 = p.s.scales + (uint64_t)bs * all * MXR_SCALES;
            const unsigned char* z1 = p.s.scales + (uint64_t)other * all * MXR_SCALES;
            for (uint32_t k = 0; k < all; ++k, ++asked) {
                const uint32_t slot = asked % MXR_STAGES, turn = asked / MXR_STAGES;
                if (turn > 0u && !mxp_wait(&ctl->empty[slot], (turn - 1u) & 1u, ctl, p.limit_ns)) {
                    ok = false;
                    break;
                }
                unsigned char *at = ring + slot * MXR_STAGE_BYTES, *sc = at + 2u * MXR_CODES;
                mbar_arrive_expect_tx(&ctl->scaled[slot], 3u * MXR_SCALES);
                bulk_load(sc, zp + (uint64_t)k * MXR_SCALES, MXR_SCALES, &ctl->scaled[slot]);
                bulk_load(sc + MXR_SCALES, z0 + (uint64_t)k * MXR_SCALES, MXR_SCALES, &ctl->scaled[slot]);
                bulk_load(sc + 2u * MXR_SCALES, z1 + (uint64_t)k * MXR_SCALES, MXR_SCALES, &ctl->scaled[slot]);
                if (half == 0u) mbar_arrive_expect_tx(&ctl->full[slot], 4u * MXR_CODES);
                if (asked != starved) mxr_box(at, &g.codes_p, yp + k * hp, &ctl->full[slot]);
                mxr_box(at + MXR_CODES, &g.codes_s, ys + k * hs, &ctl->full[slot]);
            }
        }
        // no copy may land after the CTA has gone, whoever gave up.  (Slots of earlier fills were handed back full.  Both CTAs' codes are
        // counted at the first, and both leave together.)
        const uint64_t t0 = now_ns();
        for (uint32_t i = asked > MXR_STAGES ? asked - MXR_STAGES : 0u; i < asked; ++i) {
            mxp_wait_out(&ctl->scaled[i % MXR_STAGES], (i / MXR_STAGES) & 1u, t0, p.limit_ns);
            if (half == 0u) mxp_wait_out(&ctl->full[i % MXR_STAGES], (i / MXR_STAGES) & 1u, t0, p.limit_ns);
        }
        if (half != 0u) {
            asm volatile("st.release.cluster.shared::cluster.u32 [%0], %1;" ::"r"(cluster_at(smem_u32(&ctl->asked), 0u)), "r"(asked) : "memory");
        } else if (!ok) {
            // stages that the second CTA alone has asked for: its codes are on their way, and complete a fill once they are expected
            const uint32_t other = mxp_wait_word(&ctl->asked, 0xFFFFFFFFu, p.limit_ns);
            const uint64_t t1 = now_ns();
            for (uint32_t i = asked; i < other && other != 0xFFFFFFFFu; ++i) {
                mbar_arrive_expect_tx(&ctl->full[i % MXR_STAGES], 2u * MXR_CODES);
                mxp_wait_out(&ctl->full[i % MXR_STAGES], (i / MXR_STAGES) & 1u, t1, p.limit_ns);
            }
        }
    } else if (warp == MXP_ISSUER && lane == 0 && half == 0u) {
        // dense, both operands e2m1, scales with 8 bits of exponent, 256 columns, 128 lanes of each CTA
        const uint32_t idesc0 = 1u << 7 | 1u << 10 | (256u >> 3) << 17 | 1u << 23 | (256u >> 4) << 24;
        uint32_t n = 0, made = 0;
        bool ok = true;
        for (uint32_t tile = first; tile < p.tiles && ok; tile += step, ++made) {
            if (made > 0u && !mxp_wait_cluster(&ctl->taken, (made - 1u) & 1u, ctl, p.limit_ns)) {
                ok = false;
                break;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (uint32_t k = 0; k < all; ++k, ++n) {
                const uint32_t slot = n % MXR_STAGES, turn = (n / MXR_STAGES) & 1u;
                if (!mxp_wait_cluster(&ctl->full[slot], turn, ctl, p.limit_ns) || !mxp_wait_cluster(&ctl->ready[slot], turn, ctl, p.limit_ns)) {
                    ok = false;
                    break;
                }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t at = smem_u32(ring + slot * MXR_STAGE_BYTES);
                const uint32_t cp = scales0 + slot * MXR_COLUMNS, cs = cp + 4u * MXR_ATOMS;
                const uint64_t dp = mxp_desc(at, 1024u, 2), ds = mxp_desc(at + MXR_CODES, 1024u, 2);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t atom = i >> 1, id = (i & 1u) * 2u;
                    mxr_mma(tmem, dp + 2u * i, ds + 2u * i, idesc0 | id << 4 | id << 29, cp + 4u * atom, cs + 8u * atom, k != 0u || i != 0u);
                }
                mxr_commit(&ctl->empty[slot]);
            }
            if (ok) mxr_commit(&ctl->done);
        }
        if (!ok) {                                                              // (what has been issued ends before the tensor memory goes)
            mxr_commit(&ctl->last);
            mxp_wait_out(&ctl->last, 0u, now_ns(), p.limit_ns);
        }
    } else if (warp >= MXR_SCALERS) {
        // ---- scales: lane l of a quarter holds those of rows l, l + 32, l + 64, l + 96, 4 bytes each, in 4 columns ----
        const uint32_t mine = (warp & 3u) << 21;
        uint32_t n = 0;
        bool ok = true;
        for (uint32_t tile = first; tile < p.tiles && ok; tile += step) {
            for (uint32_t k = 0; k < all; ++k, ++n) {
                const uint32_t slot = n % MXR_STAGES;
                ok = __all_sync(0xFFFFFFFFu, mxp_wait(&ctl->scaled[slot], (n / MXR_STAGES) & 1u, ctl, p.limit_ns));
                if (!ok) break;
                const unsigned char* sc = ring + slot * MXR_STAGE_BYTES + 2u * MXR_CODES + lane * 16u;
                const uint32_t cp = mine + scales0 + slot * MXR_COLUMNS, cs = cp + 4u * MXR_ATOMS;
                uint4 v[3][MXR_ATOMS];
#pragma unroll
                for (uint32_t w = 0; w < 3; ++w)
#pragma unroll
                    for (uint32_t a = 0; a < MXR_ATOMS; ++a) v[w][a] = *reinterpret_cast<const uint4*>(sc + w * MXR_SCALES + a * 512u);
                __syncwarp();
#pragma unroll
                for (uint32_t a = 0; a < MXR_ATOMS; ++a) {
                    mxr_store4(cp + 4u * a, v[0][a]);
                    mxr_store4(cs + 8u * a, v[1][a]);
                    mxr_store4(cs + 8u * a + 4u, v[2][a]);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mxr_arrive_first(&ctl->ready[slot]);
            }
        }
    } else if (warp < 8u) {
        // ---- the way out: a warp has a quarter of the lanes and half of the columns ----
        const uint32_t row = (warp & 3u) * 32u + lane, c0 = (warp >> 2) * 128u;
        const uint32_t from = tmem + ((warp & 3u) << 21) + c0;
        uint32_t made = 0;
        bool good = true;                   // (for good: behind a phase that never ended, the next one's parity reads as ended)
        for (uint32_t tile = first; tile < p.tiles; tile += step, ++made) {
            const uint32_t i = (tile % p.tiles_p * 2u + half) * 128u + row, j = tile / p.tiles_p * 256u + c0;
            good = good && __all_sync(0xFFFFFFFFu, mxp_wait(&ctl->done, made & 1u, ctl, p.limit_ns));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            uint32_t raw[4][32];
            __syncwarp();
#pragma unroll
            for (uint32_t c = 0; c < 4; ++c) mxp_load32(from + 32u * c, raw[c]);
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0 && good) mxr_arrive_first(&ctl->taken);          // (the next tile waits for those who have read this one, and for them alone)
            mxp_row_any<128>(p, i, j, 128u, raw, good);
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                                     // (nobody leaves before the other's arrivals have come)
    if (warp == MXP_ISSUER) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// rows of 128 bytes, 128 of them a box
static bool mxr_map(CUtensorMap* map, const void* at, uint64_t bytes) {
    typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                               CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return (Encode)f;
    }();
    const cuuint64_t dims[2] = {128, bytes / 128u}, strides[1] = {128};
    const cuuint32_t boxes[2] = {128, 128}, steps[2] = {1, 1};
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(at), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

div_status mx_pair_launch(const MxProductParams& p, cudaStream_t st) {
    static SmemAllowed allowed;
    if (!allowed((const void*)mx_pair_kernel, MXR_SMEM)) return DIV_ERR_CUDA;
    MxPairParams g;
    g.p = p;
    if (!mxr_map(&g.codes_p, p.p.codes, mx_codes_bytes(p.p.s)) || !mxr_map(&g.codes_s, p.s.codes, mx_codes_bytes(p.s.s))) return DIV_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2u * (p.tiles < MXP_SMS / 2u ? p.tiles : MXP_SMS / 2u));
    cfg.blockDim = dim3(MXR_THREADS);
    cfg.dynamicSmemBytes = MXR_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, mx_pair_kernel, g) != cudaSuccess) {
        cudaGetLastError();
        return DIV_ERR_CUDA;
    }
    return DIV_OK;
}
}  // namespace divk
