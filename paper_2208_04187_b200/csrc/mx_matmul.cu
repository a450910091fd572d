// Products of microscaled matrices: out[i, j] = sum over k of A[i, k] * B[j, k], both operands blobs by rows (mx.cuh), on the
// 5th-generation tensor cores' block-scaled instructions (kind::mxf8f6f4 for e4m3, kind::mxf4 for e2m1), which take
// the scales from tensor memory and sum in 32 bits.
//
// One of the operands, P, fills the 128 lanes of the accumulator, the other, S, its BN columns.  S is the operand with fewer
// rows where those fit one tile (few tokens: the weights then fill the lanes, and the tile is as narrow as the tokens), else B.
//
// A CTA makes tiles of 128 x BN, one after another.  A producer thread brings stages of 128 bytes of each row, codes and scales, into a
// ring with plain bulk copies: tiles lie in the blobs as the instruction wants them.  The issuer thread waits for a stage, has its
// scales copied into tensor memory, issues the stage's 4 products of 32 bytes of each row, and commits; the commit hands the stage
// back.  The columns of scales go round with the ring, so that no copy meets a product that still reads them.  Eight warps bring a tile
// from tensor memory to registers, give the accumulator back, and store while the next tile is on its way.
//
// Where there are fewer tiles than SMs, the sum over k is split among the CTAs of a cluster: each sums a run of stages, leaves its tile
// in its shared memory, and takes a share of the columns, which it adds up over the cluster in the order of the ranks (the result
// does not depend on timing).
//
// Every wait is bounded (MXP_LIMIT_NS): a CTA that gives up waits for its copies and its products (bounded too), gives its tensor memory back, and
// writes NaN for the tiles that it has not summed.  A tile is taken for summed when the commit behind its last product has come and in no
// other way; in a cluster NaN goes into the ring once no copy can land there any more.
#include "mx_product.cuh"

namespace divk {

constexpr uint32_t MXP_THREADS = 320;

template <int FMT, uint32_t BN> struct MxTile {
    typedef MxFormat<FMT> F;
    static constexpr uint32_t S_BLOCKS = (BN + 127u) / 128u;                  // 128-row blocks of S in a tile
    static constexpr uint32_t P_CODES = 16384u, S_CODES = BN * 128u;
    static constexpr uint32_t SCALES = 512u * F::ATOMS;                       // of 128 rows
    static constexpr uint32_t STAGE_BYTES = (P_CODES + S_CODES + SCALES * (1u + S_BLOCKS) + 1023u) / 1024u * 1024u;
    static constexpr uint32_t FIT = (MXP_SMEM - 1024u - (uint32_t)sizeof(MxCtl)) / STAGE_BYTES;
    static constexpr uint32_t SCALE_COLUMNS = 4u * F::ATOMS * (1u + S_BLOCKS);
    static constexpr uint32_t STAGES = FIT < MXP_MAX_STAGES ? FIT : MXP_MAX_STAGES;
    static constexpr uint32_t SMEM = 1024u + STAGES * STAGE_BYTES + (uint32_t)sizeof(MxCtl);
    static constexpr uint32_t HALVES = BN >= 64u ? 2u : 1u;                   // warps 4..7 take the upper columns of wide tiles
    static constexpr uint32_t MINE = BN / HALVES;                             // columns of a warp
    static constexpr uint32_t NEEDED = BN + SCALE_COLUMNS * STAGES;
    static constexpr uint32_t COLUMNS = NEEDED <= 128u ? 128u : NEEDED <= 256u ? 256u : 512u;
    static_assert(NEEDED <= 512u && STAGES >= 2u, "tensor memory");
    static_assert(BN == 256u || STAGES * STAGE_BYTES >= 128u * BN * 4u, "a split tile waits in the ring");
};

template <int FMT>
__device__ __forceinline__ void mxp_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    if (FMT == MX_E2M1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
            : "memory");
}
__device__ __forceinline__ void mxp_scales(uint32_t columns, uint64_t desc) {      // 512 bytes -> 4 columns, the same for all four quarters of the lanes
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(columns), "l"(desc) : "memory");
}
__device__ __forceinline__ void mxp_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
template <int FMT, uint32_t BN>
__global__ void __launch_bounds__(MXP_THREADS, 1)
mx_product_kernel(const __grid_constant__ MxProductParams p) {
    typedef MxTile<FMT, BN> T;
    typedef MxFormat<FMT> F;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    MxCtl* ctl = reinterpret_cast<MxCtl*>(ring + T::STAGES * T::STAGE_BYTES);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    const uint32_t rank = p.split > 1u ? cluster_rank() : 0u, first = blockIdx.x / p.split, step = gridDim.x / p.split;
    const uint32_t all = p.p.s.stages;
    const uint32_t k0 = (uint32_t)((uint64_t)all * rank / p.split), k1 = (uint32_t)((uint64_t)all * (rank + 1u) / p.split);

    if (warp == MXP_ISSUER) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem)), "n"(T::COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < T::STAGES; ++i) {
            mbar_init(&ctl->full[i], 1);
            mbar_init(&ctl->empty[i], 1);
        }
        mbar_init(&ctl->done, 1);
        mbar_init(&ctl->taken, 4u * T::HALVES);
        mbar_init(&ctl->last, 1);
        ctl->failed = ctl->landed = 0;
        fence_barrier_init();
        fence_proxy_async();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *(volatile uint32_t*)&ctl->tmem;
    griddep_wait();
    griddep_launch();

    if (warp == MXP_PRODUCER && lane == 0) {
        uint32_t asked = 0;
        bool ok = true;
        const uint32_t starved = blockIdx.x == p.starved_cta ? p.starved_copy : 0xFFFFFFFFu;
        for (uint32_t tile = first; tile < p.tiles && ok; tile += step) {
            const uint32_t tp = tile % p.tiles_p, s0 = tile / p.tiles_p * BN;
            const uint32_t hp = mx_tile_rows(p.p.s, tp) * 128u;
            // rows of S: of its only block of 128 (BN < 128), or whole blocks.  (A narrow tile inside a larger block would want its scales at
            // another column of tensor memory than a multiple of 4, which the instruction answered with a misaligned address.)
            uint32_t hs[T::S_BLOCKS], step_s[T::S_BLOCKS];
            const unsigned char *from_s[T::S_BLOCKS], *scales_s[T::S_BLOCKS];
            uint32_t bytes = hp + T::SCALES;
#pragma unroll
            for (uint32_t b = 0; b < T::S_BLOCKS; ++b) {
                const uint32_t row = s0 + b * 128u, rb = row / 128u;
                const bool there = row < p.s.s.rows;
                const uint32_t height = there ? mx_tile_rows(p.s.s, rb) : 0u;
                hs[b] = min(height, BN) * 128u;
                from_s[b] = p.s.codes + (there ? mx_tile_offset(p.s.s, rb, 0) : 0u);
                step_s[b] = height * 128u;
                scales_s[b] = p.s.scales + (uint64_t)(there ? rb : 0u) * p.s.s.stages * T::SCALES;
                bytes += hs[b] + T::SCALES;                   // (scales of a block that is not there: those of the first, for columns that nobody keeps)
            }
            const unsigned char* from_p = p.p.codes + mx_tile_offset(p.p.s, tp, 0);
            const unsigned char* scales_p = p.p.scales + (uint64_t)tp * all * T::SCALES;
            for (uint32_t k = k0; k < k1; ++k, ++asked) {
                const uint32_t slot = asked % T::STAGES, turn = asked / T::STAGES;
                if (turn > 0u && !mxp_wait(&ctl->empty[slot], (turn - 1u) & 1u, ctl, p.limit_ns)) {
                    ok = false;
                    break;
                }
                unsigned char* at = ring + slot * T::STAGE_BYTES;
                uint64_t* bar = &ctl->full[slot];
                mbar_arrive_expect_tx(bar, bytes);
                if (asked != starved) bulk_load(at, from_p + (uint64_t)k * hp, hp, bar);
                bulk_load(at + T::P_CODES + T::S_CODES, scales_p + (uint64_t)k * T::SCALES, T::SCALES, bar);
#pragma unroll
                for (uint32_t b = 0; b < T::S_BLOCKS; ++b) {
                    if (hs[b]) bulk_load(at + T::P_CODES + b * 16384u, from_s[b] + (uint64_t)k * step_s[b], hs[b], bar);
                    bulk_load(at + T::P_CODES + T::S_CODES + (1u + b) * T::SCALES, scales_s[b] + (uint64_t)k * T::SCALES, T::SCALES, bar);
                }
            }
        }
        // no copy may land after the CTA has gone, whoever gave up.  (Slots of earlier fills were handed back full.)
        const uint64_t t0 = now_ns();
        for (uint32_t i = asked > T::STAGES ? asked - T::STAGES : 0u; i < asked; ++i)
            mxp_wait_out(&ctl->full[i % T::STAGES], (i / T::STAGES) & 1u, t0, p.limit_ns);
        __threadfence_block();
        *(volatile uint32_t*)&ctl->landed = 1u;
    } else if (warp == MXP_ISSUER && lane == 0) {
        // dense, both operands of one type, scales with 8 bits of exponent, BN columns, 128 lanes
        const uint32_t type = FMT == MX_E2M1 ? 1u : 0u;
        const uint32_t idesc0 = type << 7 | type << 10 | (BN >> 3) << 17 | 1u << 23 | (128u >> 4) << 24;
        const uint32_t scales0 = tmem + BN;
        uint32_t n = 0, made = 0;
        bool ok = true;
        for (uint32_t tile = first; tile < p.tiles && ok; tile += step, ++made) {
            if (made > 0u && !mxp_wait(&ctl->taken, (made - 1u) & 1u, ctl, p.limit_ns)) {
                ok = false;
                break;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (uint32_t k = k0; k < k1; ++k, ++n) {
                const uint32_t slot = n % T::STAGES;
                if (!mxp_wait(&ctl->full[slot], (n / T::STAGES) & 1u, ctl, p.limit_ns)) {
                    ok = false;
                    break;
                }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t at = smem_u32(ring + slot * T::STAGE_BYTES), sc = at + T::P_CODES + T::S_CODES;
                const uint32_t cp = scales0 + slot * T::SCALE_COLUMNS, cs = cp + 4u * F::ATOMS;
#pragma unroll
                for (uint32_t a = 0; a < F::ATOMS; ++a) {
                    mxp_scales(cp + 4u * a, mxp_desc(sc + 512u * a, 128u, 0));
#pragma unroll
                    for (uint32_t b = 0; b < T::S_BLOCKS; ++b)
                        mxp_scales(cs + 4u * (a * T::S_BLOCKS + b), mxp_desc(sc + (1u + b) * T::SCALES + 512u * a, 128u, 0));
                }
                const uint64_t dp = mxp_desc(at, 1024u, 2), ds = mxp_desc(at + T::P_CODES, 1024u, 2);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t atom = FMT == MX_E2M1 ? i >> 1 : 0u, id = FMT == MX_E2M1 ? (i & 1u) * 2u : i;
                    mxp_mma<FMT>(tmem, dp + 2u * i, ds + 2u * i, idesc0 | id << 4 | id << 29, cp + 4u * atom, cs + 4u * T::S_BLOCKS * atom,
                                 k != k0 || i != 0u);
                }
                mxp_commit(&ctl->empty[slot]);
            }
            if (ok) mxp_commit(&ctl->done);
        }
        if (!ok) {                                                              // (what has been issued ends before the tensor memory goes)
            mxp_commit(&ctl->last);
            mxp_wait_out(&ctl->last, 0u, now_ns(), p.limit_ns);
        }
    } else if (warp < 4u * T::HALVES) {
        // ---- the way out: a warp has a quarter of the lanes, and all columns or half of them ----
        const uint32_t row = (warp & 3u) * 32u + lane, c0 = (warp >> 2) * T::MINE;
        const uint32_t from = tmem + ((warp & 3u) << 21) + c0;          // its first lane in the upper half of the address
        uint32_t made = 0;
        bool good = true;                   // (for good: behind a phase that never ended, the next one's parity reads as ended)
        for (uint32_t tile = first; tile < p.tiles; tile += step, ++made) {
            const uint32_t p0 = tile % p.tiles_p * 128u, s0 = tile / p.tiles_p * BN;
            good = good && __all_sync(0xFFFFFFFFu, mxp_wait(&ctl->done, made & 1u, ctl, p.limit_ns));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            uint32_t raw[(T::MINE + 31u) / 32u][32];
            __syncwarp();
#pragma unroll
            for (uint32_t c = 0; c < T::MINE; c += 32u) {
                if (T::MINE < 32u) mxp_load16(from, raw[0]);
                else mxp_load32(from + c, raw[c / 32u]);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0 && good) mbar_arrive(&ctl->taken);          // (the next tile waits for those who have read this one, and for them alone)
            if (!good && p.split > 1u) mxp_wait_word(&ctl->landed, 0u, p.limit_ns);
            if (p.split == 1u && !p.swapped) {
                mxp_row_any<T::MINE>(p, p0 + row, s0 + c0, T::MINE, raw, good);
                continue;
            }
#pragma unroll
            for (uint32_t c = 0; c < T::MINE; c += 32u) {
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = (T::MINE >= 32u || i < 16) ? (good ? __uint_as_float(raw[c / 32u][i]) : __uint_as_float(0x7FC00000u)) : 0.f;
                if (p.split == 1u) {
                    mxp_column_any(p, p0 + row, s0 + c0 + c, min(T::MINE, 32u), v);
                } else {
                    float* part = reinterpret_cast<float*>(ring);       // [column][lane]; all copies and products are through
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (T::MINE >= 32u || i < 16) part[(c0 + c + i) * 128u + row] = v[i];
                }
            }
        }
    }
    __syncwarp();
    if (p.split > 1u) {
        cluster_sync_all();
        if (warp < 8) {                                                    // (a cluster has one tile)
            // this CTA's share of the columns, half of it for each four warps; reads of 8 columns of two CTAs are under way together
            const uint32_t mine = BN / p.split / 2u, c0 = rank * 2u * mine + (warp >> 2) * mine, row = (warp & 3u) * 32u + lane;
            const uint32_t p0 = first % p.tiles_p * 128u, s0 = first / p.tiles_p * BN;
            float v[32];
#pragma unroll
            for (uint32_t c = 0; c < 32u; c += 8u) {
                const uint32_t n = c < mine ? min(mine - c, 8u) : 0u, at = smem_u32(ring) + ((c0 + c) * 128u + row) * 4u;
                float one[8], two[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c + i] = 0.f;
                if (n == 0u) continue;
                for (uint32_t r = 0; r < p.split; r += 2u) {
                    const uint32_t at1 = cluster_at(at, r), at2 = cluster_at(at, r + 1u);
#pragma unroll
                    for (uint32_t i = 0; i < 8u; ++i) {
                        one[i] = i < n ? ld_cluster(at1 + i * 512u) : 0.f;
                        two[i] = i < n ? ld_cluster(at2 + i * 512u) : 0.f;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[c + i] = (v[c + i] + one[i]) + two[i];
                }
            }
            if (p.swapped) {
                mxp_column_any(p, p0 + row, s0 + c0, mine, v);
            } else {
                uint32_t raw[1][32];
#pragma unroll
                for (int i = 0; i < 32; ++i) raw[0][i] = __float_as_uint(v[i]);
                mxp_row_any<32>(p, p0 + row, s0 + c0, mine, raw, true);
            }
        }
        cluster_sync_all();                                                // nobody leaves while another reads here
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == MXP_ISSUER) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(T::COLUMNS));
    }
}

// ---------------------------------------------------------------------------------------------
// one token, 4 bits
// ---------------------------------------------------------------------------------------------
// One row of S against all rows of P is bound by the reading of P, and by launch and latency before that: of the tensor cores' tile one
// column would be used, and its way out through a cluster takes as long as everything else.  Here a CTA takes 8 rows of P; its 4 warps
// share the stages, 8 lanes a row's stage, a block of 32 numbers each.  S lies in shared memory in 16 bits.  A block sums exactly in
// 16 bits (8 products of at most 36, in steps of 1/4, to a half of a register); the block's sum is scaled by both powers of two at once.
// (The same for e4m3, whose products need 32 bits, took 7.6 us at 4096 x 4096, the tensor cores 6.8; for two tokens 6.4 us, the tensor cores 6.1.)
// From L2, us, against the tensor cores' kernel (rows x numbers a row):
//    512 x  8192  4.8 and  5.3     1024 x 2048 2.3 and 4.2    4096 x 2048 3.5 and 4.9     8192 x  512 3.8 and 3.1
//    512 x 12000  6.5 and  6.1     1024 x 4096 3.0 and 4.7    4096 x 4096 5.2 and 5.7     8192 x 2048 5.1 and 5.1
//   1024 x 16384  8.4 and  7.0     1024 x 8192 4.8 and 5.5    4096 x 6000 7.4 and 6.5    10000 x 1024 4.5 and 7.6
//   2048 x  8192  5.5 and 10.2     3000 x 4096 5.0 and 5.4    6000 x 2048 4.5 and 4.9    12288 x  512 5.0 and 3.3
//   3000 x  6000  7.1 and  6.2     3000 x 8192 8.5 and 6.9    6000 x 4096 6.6 and 6.4    16384 x 1024 6.0 and 4.2
// It takes longer with more than 32 stages (each warp goes through a quarter of them, one after another), with rows of more than a CTA's worth
// for all places of the device (each CTA turns the token into numbers again), and past 65536 rows x stages.
constexpr uint32_t MXV_THREADS = 128, MXV_ROWS = 8;
constexpr uint32_t MXV_MOST = 65536u, MXV_MAX_ROWS = 10240u, MXV_MAX_STAGES = 32u;      // rows x stages, and each, up to which this kernel is the shorter

__host__ __device__ constexpr uint32_t mxv_smem(uint32_t stages) { return stages * (512u + 8u); }       // of S: values and scale bytes
static_assert(mxv_smem(MXV_MAX_STAGES) + 4u * MXV_ROWS * 4u <= 48u * 1024u, "no leave to ask for");
// dot * 2^(a - 127) * 2^(b - 127)
__device__ __forceinline__ float mxv_scaled(float dot, uint32_t a, uint32_t b) {
    if (a == 255u || b == 255u) return __uint_as_float(0x7FC00000u);
    const int t = (int)(a + b) - 254, h = t >> 1;                    // halves, both normal powers: no way round beyond the range
    return dot * __uint_as_float((uint32_t)(h + 127) << 23) * __uint_as_float((uint32_t)(t - h + 127) << 23);
}
__device__ __forceinline__ __half2 mxv_pair(const uint32_t (&w)[4], uint32_t i) {
    return __half2(__nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)((w[i >> 2] >> (8u * (i & 3u))) & 0xFFu), __NV_E2M1));
}

__global__ void __launch_bounds__(MXV_THREADS)
mx_vector_kernel(const __grid_constant__ MxProductParams p) {
    constexpr uint32_t SETS = MXV_ROWS / 4u, AHEAD = 4u;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float joined[4][MXV_ROWS];
    const uint32_t stages = p.p.s.stages, lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint4* values = reinterpret_cast<uint4*>(smem);                                // [stage][quarter of the block][block]: 8 lanes read 128 bytes
    unsigned char* scales = smem + stages * 512u;                                  // [stage][block]
    griddep_wait();
    griddep_launch();

    const uint32_t r0 = blockIdx.x * MXV_ROWS;
    const unsigned char *from[SETS], *scale_of[SETS];
    uint32_t step[SETS], block[SETS];
    bool there[SETS];
#pragma unroll
    for (uint32_t s = 0; s < SETS; ++s) {
        const uint32_t row = r0 + s * 4u + (lane >> 3), rb = row >> 7, rt = row & 127u;
        there[s] = row < p.p.s.rows;
        block[s] = (lane & 7u) ^ (rt & 7u);                                        // where this lane's piece belongs
        step[s] = there[s] ? mx_tile_rows(p.p.s, rb) * 128u : 0u;
        from[s] = p.p.codes + (there[s] ? mx_tile_offset(p.p.s, rb, 0) + rt * 128u + (lane & 7u) * 16u : 0u);
        scale_of[s] = p.p.scales + (there[s] ? (uint64_t)rb * stages * 1024u + (block[s] >> 2) * 512u + mx_scale_slot(rt) + (block[s] & 3u) : 0u);
    }
    uint4 q[AHEAD][SETS];
    uint32_t e[AHEAD][SETS];
    const auto bring = [&](uint32_t k) {
#pragma unroll
        for (uint32_t a = 0; a < AHEAD; ++a)
#pragma unroll
            for (uint32_t s = 0; s < SETS; ++s)
                if (k + a * 4u < stages && there[s]) {
                    q[a][s] = *reinterpret_cast<const uint4*>(from[s] + (uint64_t)(k + a * 4u) * step[s]);
                    e[a][s] = scale_of[s][(uint64_t)(k + a * 4u) * 1024u];
                }
    };
    bring(warp);                                             // under way while the token is brought

    for (uint32_t job = threadIdx.x; job < stages * 8u; job += MXV_THREADS) {
        const uint32_t c = job & 7u, stage = job >> 3;
        const uint4 x = *reinterpret_cast<const uint4*>(p.s.codes + (uint64_t)stage * 1024u + c * 16u);        // (row 0: pieces lie in order)
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            __half2 v[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) v[i] = mxv_pair(w, u * 4u + i);
            values[(stage * 4u + u) * 8u + c] = *reinterpret_cast<const uint4*>(v);
        }
        scales[stage * 8u + c] = p.s.scales[(uint64_t)stage * 1024u + (c >> 2) * 512u + (c & 3u)];
    }
    __syncthreads();

    float sum[SETS];
#pragma unroll
    for (uint32_t s = 0; s < SETS; ++s) sum[s] = 0.f;
    for (uint32_t k = warp; k < stages; k += 4u * AHEAD) {
        if (k != warp) bring(k);
#pragma unroll
        for (uint32_t a = 0; a < AHEAD; ++a) {
            const uint32_t stage = k + a * 4u;
            if (stage >= stages) break;
#pragma unroll
            for (uint32_t s = 0; s < SETS; ++s) {
                if (!there[s]) continue;
                const uint32_t w[4] = {q[a][s].x, q[a][s].y, q[a][s].z, q[a][s].w};
                __half2 part[2] = {__float2half2_rn(0.f), __float2half2_rn(0.f)};
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u) {
                    const uint4 x = values[(stage * 4u + u) * 8u + block[s]];
                    const __half2* v = reinterpret_cast<const __half2*>(&x);
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) part[u >> 1] = __hfma2(mxv_pair(w, u * 4u + i), v[i], part[u >> 1]);
                }
                const float2 lo = __half22float2(part[0]), hi = __half22float2(part[1]);
                sum[s] += mxv_scaled((lo.x + lo.y) + (hi.x + hi.y), e[a][s], scales[stage * 8u + block[s]]);
            }
        }
    }
#pragma unroll
    for (uint32_t s = 0; s < SETS; ++s) {
        float v = sum[s];
#pragma unroll
        for (int d = 4; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
        if ((lane & 7u) == 0) joined[warp][s * 4u + (lane >> 3)] = v;
    }
    __syncthreads();
    const uint32_t r = threadIdx.x;
    if (r < MXV_ROWS && r0 + r < p.p.s.rows) {
        const float v = (joined[0][r] + joined[1][r]) + (joined[2][r] + joined[3][r]);
        const uint64_t at = p.swapped ? r0 + r : (r0 + r) * p.ld;
        if (p.out_dtype == DIV_BF16) static_cast<__nv_bfloat16*>(p.out)[at] = from_f32<__nv_bfloat16>(v);
        else if (p.out_dtype == DIV_F16) static_cast<__half*>(p.out)[at] = from_f32<__half>(v);
        else static_cast<float*>(p.out)[at] = v;
    }
}

}  // namespace divk

namespace {
using namespace divk;

div_status vector_launch(const MxProductParams& p, cudaStream_t st) {
    return launch_pdl(mx_vector_kernel, dim3((p.p.s.rows + MXV_ROWS - 1u) / MXV_ROWS), MXV_THREADS, mxv_smem(p.p.s.stages), st, p);
}

template <int FMT, uint32_t BN>
div_status product_launch(const MxProductParams& p, uint32_t grid, cudaStream_t st) {
    typedef MxTile<FMT, BN> T;
    auto kern = mx_product_kernel<FMT, BN>;
    static SmemAllowed allowed;
    if (!allowed((const void*)kern, T::SMEM)) return DIV_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(MXP_THREADS);
    cfg.dynamicSmemBytes = T::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = p.split;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kern, p) != cudaSuccess) {
        cudaGetLastError();
        return DIV_ERR_CUDA;
    }
    return DIV_OK;
}

template <int FMT>
div_status product_by_width(uint32_t bn, const MxProductParams& p, uint32_t grid, cudaStream_t st) {
    switch (bn) {
        case 16: return product_launch<FMT, 16>(p, grid, st);
        case 32: return product_launch<FMT, 32>(p, grid, st);
        case 64: return product_launch<FMT, 64>(p, grid, st);
        case 128: return product_launch<FMT, 128>(p, grid, st);
    }
    return product_launch<FMT, 256>(p, grid, st);
}

// (p: the limits of waits are set)
div_status product(MxProductParams p, bool starved, const void* a_dev, size_t a_bytes, const void* b_dev, size_t b_bytes, int64_t m, int64_t n, int64_t k, int32_t format,
                   void* out_dev, int64_t out_row_stride, int32_t out_dtype, void* cuda_stream) {
    if (!a_dev || !b_dev || !out_dev) return DIV_ERR_NULL;
    if (!lm_size_ok(m) || !lm_size_ok(n) || !lm_size_ok(k) || (m > 1 && out_row_stride < n)) return DIV_ERR_SHAPE;
    if (!lm_dtype_ok(out_dtype) || !mx_format_ok(format)) return DIV_ERR_PARAM;
    const uint32_t size = lm_dtype_bytes(out_dtype);
    if (!aligned_16(a_dev) || !aligned_16(b_dev) || reinterpret_cast<uintptr_t>(out_dev) % size != 0) return DIV_ERR_ALIGN;
    MxSide a, b;
    a.s = mx_shape((uint32_t)m, (uint32_t)k, format);
    b.s = mx_shape((uint32_t)n, (uint32_t)k, format);
    if (a_bytes < mx_codes_bytes(a.s) + mx_scales_bytes(a.s, format) || b_bytes < mx_codes_bytes(b.s) + mx_scales_bytes(b.s, format)) return DIV_ERR_CAPACITY;
    a.codes = (const unsigned char*)a_dev;
    a.scales = a.codes + mx_scales_at(a.s);
    b.codes = (const unsigned char*)b_dev;
    b.scales = b.codes + mx_scales_at(b.s);

    const bool swapped = m < n && m <= 64;
    p.p = swapped ? b : a;
    p.s = swapped ? a : b;
    p.swapped = swapped;
    p.out = out_dev;
    p.ld = (uint64_t)out_row_stride;
    p.out_dtype = (uint32_t)out_dtype;
    if (format == MX_E2M1 && p.s.s.rows == 1u && p.p.s.rows <= MXV_MAX_ROWS && p.p.s.stages <= MXV_MAX_STAGES && p.p.s.rows * p.p.s.stages <= MXV_MOST)
        return starved ? DIV_ERR_PARAM : vector_launch(p, (cudaStream_t)cuda_stream);
    const uint64_t rows_s = p.s.s.rows;
    const uint64_t blocks_p = (p.p.s.rows + 127u) / 128u;
    uint32_t bn = rows_s <= 16 ? 16u : rows_s <= 32 ? 32u : rows_s <= 64 ? 64u : 128u;
    if (bn == 128u && blocks_p * ((rows_s + 255u) / 256u) >= 120u) bn = 256u;
    const auto tiles_of = [&](uint32_t width) { return blocks_p * ((rows_s + width - 1u) / width); };
    if (tiles_of(bn) >= (1ull << 31)) return DIV_ERR_SHAPE;
    // large products of e2m1: by pairs of CTAs, whose start and end take longer than they save with short rows or fewer than two rounds of tiles
    // (mx_pair.cu has both sides' times; it counts rows of 128 bytes in 31 bits)
    const uint64_t paired = (blocks_p + 1u) / 2u * ((rows_s + 255u) / 256u);
    if (format == MX_E2M1 && bn == 256u && p.p.s.stages >= 11u && paired >= MXP_SMS && ((mx_codes_bytes(p.p.s) | mx_codes_bytes(p.s.s)) >> 38) == 0) {
        p.tiles_p = (uint32_t)((blocks_p + 1u) / 2u);
        p.tiles = (uint32_t)paired;
        p.split = 1;
        return mx_pair_launch(p, (cudaStream_t)cuda_stream);
    }
    // few tiles: the sum is split, as long as a CTA keeps two stages
    uint32_t split = 1;
    while (bn < 256u && split < 8u && tiles_of(bn) * split * 2u <= 160u && p.p.s.stages >= 4u * split) split *= 2u;
    p.tiles_p = (uint32_t)blocks_p;
    p.tiles = (uint32_t)tiles_of(bn);
    p.split = split;
    const uint32_t grid = split > 1u ? p.tiles * split : p.tiles < MXP_SMS ? p.tiles : MXP_SMS;
    return format == MX_E4M3 ? product_by_width<MX_E4M3>(bn, p, grid, (cudaStream_t)cuda_stream)
                             : product_by_width<MX_E2M1>(bn, p, grid, (cudaStream_t)cuda_stream);
}

}  // namespace

extern "C" {

div_status div_mx_matmul(const void* a_dev, size_t a_bytes, const void* b_dev, size_t b_bytes, int64_t m, int64_t n, int64_t k, int32_t format,
                         void* out_dev, int64_t out_row_stride, int32_t out_dtype, void* cuda_stream) {
    return product(MxProductParams(), false, a_dev, a_bytes, b_dev, b_bytes, m, n, k, format, out_dev, out_row_stride, out_dtype, cuda_stream);
}

div_status div_debug_mx_matmul_starved(const void* a_dev, size_t a_bytes, const void* b_dev, size_t b_bytes, int64_t m, int64_t n, int64_t k, int32_t format,
                                       void* out_dev, int64_t out_row_stride, int32_t out_dtype, void* cuda_stream, uint32_t cta, uint32_t copy,
                                       uint64_t timeout_ns) {
    if (timeout_ns == 0 || timeout_ns > 100000000ull) return DIV_ERR_PARAM;
    MxProductParams p;
    p.limit_ns = timeout_ns;
    p.starved_cta = cta;
    p.starved_copy = copy;
    return product(p, true, a_dev, a_bytes, b_dev, b_bytes, m, n, k, format, out_dev, out_row_stride, out_dtype, cuda_stream);
}

}  // extern "C"
