// What the kernels of the microscaled product share: their parameters, matrix descriptors, waits, and the way out.
#pragma once

#include "mx.cuh"

namespace divk {

constexpr uint32_t MXP_PRODUCER = 8, MXP_ISSUER = 9;        // warps 0..7: the way out
constexpr uint32_t MXP_MAX_STAGES = 8, MXP_SMS = 148;
constexpr uint64_t MXP_LIMIT_NS = 2000000000ull;
constexpr uint32_t MXP_SMEM = 224u * 1024u;       // of a CTA, ring and control block

struct MxSide {
    const unsigned char *codes, *scales;
    MxShape s;
};
struct MxProductParams {
    MxSide p, s;
    void* out;
    uint64_t ld;                 // numbers between two rows of out
    uint32_t tiles_p, tiles;
    uint32_t swapped;            // the lanes are columns of out
    uint32_t out_dtype;
    uint32_t split;              // CTAs of a cluster
    uint64_t limit_ns = MXP_LIMIT_NS;      // of every wait
    uint32_t starved_cta = 0xFFFFFFFFu, starved_copy = 0u;      // (a test's: this CTA never gets the codes of that stage, counted over all that it asks for)
};
struct MxCtl {
    uint64_t full[MXP_MAX_STAGES], empty[MXP_MAX_STAGES];
    uint64_t scaled[MXP_MAX_STAGES], ready[MXP_MAX_STAGES];      // pairs: scales are in shared memory, and in tensor memory
    uint64_t done, taken;        // done: a tile is summed; taken: it is in registers
    uint64_t last;               // what a giving-up issuer has issued is through
    uint32_t tmem, failed;
    uint32_t landed;             // (split sums) no copy is on its way any more
    uint32_t asked;              // (pairs) stages that the second CTA has asked for in all, told to the first
};

// shared-memory matrix descriptor: start, stride between groups of 8 rows; version 1 of the layout
__device__ __forceinline__ uint64_t mxp_desc(uint32_t at, uint32_t group_bytes, uint64_t swizzle) {
    return (uint64_t)((at & 0x3FFFFu) >> 4) | (uint64_t)1u << 16 | (uint64_t)(group_bytes >> 4) << 32 | 1ull << 46 | swizzle << 61;
}
__device__ __forceinline__ void mxp_load32(uint32_t at, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
        "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
        "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void mxp_load16(uint32_t at, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(at)
        : "memory");
}
// (a phase that arrivals of another CTA complete)
__device__ __forceinline__ bool mxp_try_wait_cluster(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// waits for a phase, at most limit_ns, and not once another thread of the CTA has given up
template <bool CLUSTER>
__device__ __forceinline__ bool mxp_wait_for(uint64_t* bar, uint32_t parity, MxCtl* ctl, uint64_t limit_ns) {
    uint64_t t0 = 0;
    for (uint32_t polls = 1;; ++polls) {
        if (CLUSTER ? mxp_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity)) return true;
        if ((polls & 63u) == 0u) {                         // (reading the timer takes longer than most waits)
            const uint64_t t = now_ns();
            if (t0 == 0u) t0 = t;
            if (*(volatile uint32_t*)&ctl->failed || t - t0 > limit_ns) {
                *(volatile uint32_t*)&ctl->failed = 1u;
                return false;
            }
        }
    }
}
__device__ __forceinline__ bool mxp_wait(uint64_t* bar, uint32_t parity, MxCtl* ctl, uint64_t limit_ns) { return mxp_wait_for<false>(bar, parity, ctl, limit_ns); }
__device__ __forceinline__ bool mxp_wait_cluster(uint64_t* bar, uint32_t parity, MxCtl* ctl, uint64_t limit_ns) { return mxp_wait_for<true>(bar, parity, ctl, limit_ns); }
// On the way out, for what a CTA has started and must not leave behind (copies, products): whoever has given up.
__device__ __forceinline__ void mxp_wait_out(uint64_t* bar, uint32_t parity, uint64_t t0, uint64_t limit_ns) {
    while (!mbar_try_wait(bar, parity) && now_ns() - t0 < limit_ns) {}
}
// Waits until a word is no longer `until`, three limits at most: another thread's last wait, and what it waits for on its way out
__device__ __forceinline__ uint32_t mxp_wait_word(const uint32_t* word, uint32_t until, uint64_t limit_ns) {
    const uint64_t t0 = now_ns();
    uint32_t v;
    while ((v = *(const volatile uint32_t*)word) == until && now_ns() - t0 < 3u * limit_ns) {}
    __threadfence_block();
    return v;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// an address in the shared memory of another CTA of the cluster; a number there (whose writing a cluster barrier has ordered before)
__device__ __forceinline__ uint32_t cluster_at(uint32_t local, uint32_t rank) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(local), "r"(rank));
    return at;
}
__device__ __forceinline__ float ld_cluster(uint32_t at) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at));
    return v;
}

// up to 32 numbers of a lane into a column of out
template <typename OT>
__device__ __forceinline__ void mxp_column(const MxProductParams& p, uint32_t row_p, uint32_t row_s, uint32_t n, const float (&v)[32]) {
    if (row_p >= p.p.s.rows || row_s >= p.s.s.rows) return;
    const uint32_t count = min(n, p.s.s.rows - row_s);
    OT* to = static_cast<OT*>(p.out) + (uint64_t)row_s * p.ld + row_p;
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if ((uint32_t)i < count) to[i * p.ld] = from_f32<OT>(v[i]);
}
__device__ __forceinline__ void mxp_column_any(const MxProductParams& p, uint32_t row_p, uint32_t row_s, uint32_t n, const float (&v)[32]) {
    if (p.out_dtype == DIV_BF16) mxp_column<__nv_bfloat16>(p, row_p, row_s, n, v);
    else if (p.out_dtype == DIV_F16) mxp_column<__half>(p, row_p, row_s, n, v);
    else mxp_column<float>(p, row_p, row_s, n, v);
}

// C numbers of a row of out, of which `left` are there, in 16-byte stores wherever the row begins
template <typename OT, uint32_t C>
__device__ __forceinline__ void mxp_row(OT* to, uint32_t left, const uint32_t (&raw)[(C + 31u) / 32u][32], bool good) {
    typedef Units<OT> U;
    const uint32_t o = U::offset(to), s = o ? U::E - o : 0u;
    const auto unit = [&](uint32_t u) {
        OT v[U::E];
#pragma unroll
        for (uint32_t i = 0; i < U::E; ++i) {
            const uint32_t c = u * U::E + i;
            v[i] = from_f32<OT>(good ? __uint_as_float(raw[c / 32u][c % 32u]) : __uint_as_float(0x7FC00000u));
        }
        return *reinterpret_cast<const uint4*>(v);
    };
    uint4 one = unit(0);
    U::put(to, one, 0u, min(s, left));
#pragma unroll
    for (uint32_t u = 0; u < C / U::E; ++u) {
        const bool more = u + 1u < C / U::E;
        const uint4 next = more ? unit(u + 1u) : make_uint4(0u, 0u, 0u, 0u);
        if (left >= (u + 1u) * U::E + s && (more || s == 0u)) {
            *reinterpret_cast<uint4*>(to + u * U::E + s) = U::cut(one, next, s);
        } else if (left > u * U::E) {
            U::put(to + u * U::E, one, s, left - u * U::E);
            if (more && left > (u + 1u) * U::E) U::put(to + (u + 1u) * U::E, next, 0u, min(s, left - (u + 1u) * U::E));
        }
        one = next;
    }
}

// the same in out's type: numbers n of row i from column j on
template <uint32_t C>
__device__ __forceinline__ void mxp_row_any(const MxProductParams& p, uint32_t i, uint32_t j, uint32_t n, const uint32_t (&raw)[(C + 31u) / 32u][32], bool good) {
    if (i >= p.p.s.rows || j >= p.s.s.rows) return;
    const uint64_t at = (uint64_t)i * p.ld + j;
    const uint32_t left = min(n, p.s.s.rows - j);
    if (p.out_dtype == DIV_BF16) mxp_row<__nv_bfloat16, C>(static_cast<__nv_bfloat16*>(p.out) + at, left, raw, good);
    else if (p.out_dtype == DIV_F16) mxp_row<__half, C>(static_cast<__half*>(p.out) + at, left, raw, good);
    else mxp_row<float, C>(static_cast<float*>(p.out) + at, left, raw, good);
}

// mx_pair.cu: e2m1, tiles of 256 x 256 (tiles_p, tiles: of those)
div_status mx_pair_launch(const MxProductParams& p, cudaStream_t st);

}  // namespace divk
