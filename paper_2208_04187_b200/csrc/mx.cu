// Microscaled quantisation of a matrix, by rows, by columns or both from one reading, and its way back.
//
//   by rows     the blob of x (rows x cols), blocks of 32 neighbours along a row
//   by columns  the blob of the transposed matrix (cols x rows), blocks of 32 neighbours down a column
//
// Both are bound by memory: x is read once, 1 + 1/32 or 1/2 + 1/32 bytes a number are written for each direction.
//
// A CTA takes 128 x 128 numbers, which are whole tiles of e4m3 codes in both directions (half tiles of e2m1).  A thread reads
// 8 neighbours at a time, 8 times, all reads under way together, and leaves them in shared memory as they are.  From there a
// thread takes whole blocks: 32 neighbours of a row, 32 rows of a column (of two columns of 16-bit types, one word).  So a
// scale costs its dozen instructions once a block; what bounds the kernel next to memory is the issue of instructions (with 8 numbers of
// a block to a thread and shuffles, 75 % of the issue slots at 8192 x 4096).  The columns' codes go through shared memory once more, so
// that whole lines leave the SM.  In a row of shared memory the 16-byte pieces of a block are permuted, so that neither way meets
// bank conflicts: piece j of block b of row r is at j ^ mxq_turn(r, b).
#include "mx.cuh"

namespace divk {

constexpr uint32_t MXQ_TILE = 128, MXQ_THREADS = 256;

struct MxQuantParams {
    const void* x;
    uint64_t stride;           // numbers between the beginnings of two rows
    MxShape r, c;              // of the blob by rows, and by columns
    unsigned char *by_rows, *by_cols;
    uint32_t tiles_x;
};

template <typename XT> __host__ __device__ constexpr uint32_t mxq_smem_bytes(bool cols) {
    // scales by rows; numbers; codes by columns as their tile lies in the blob; scales by columns
    // (16-bit types: in the place of the numbers, which all threads have in registers by then; so 6 CTAs fit an SM instead of 4)
    return 512u + MXQ_TILE * MXQ_TILE * (uint32_t)sizeof(XT) + (cols ? (sizeof(XT) == 4 ? 16384u : 0u) + 512u : 0u);
}
// 4 pieces of 8 numbers or 8 of 4: the 8 lanes that a shared-memory access serves together hold 4 blocks of two rows
template <typename XT> __device__ __forceinline__ uint32_t mxq_turn(uint32_t row, uint32_t block) {
    return sizeof(XT) == 4 ? block ^ (row & 1u) << 2 : block >> 1 ^ (row & 1u) << 1;
}

template <typename XT, int FMT, bool ROWS, bool COLS, bool VEC>
__global__ void __launch_bounds__(MXQ_THREADS)
mx_quantize_kernel(const __grid_constant__ MxQuantParams p) {
    typedef MxFormat<FMT> F;
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char* row_scales = smem;
    XT* numbers = reinterpret_cast<XT*>(smem + 512);
    unsigned char* codes = smem + 512 + (sizeof(XT) == 4 ? MXQ_TILE * MXQ_TILE * sizeof(XT) : 0u);
    unsigned char* col_scales = smem + 512 + MXQ_TILE * MXQ_TILE * sizeof(XT) + (sizeof(XT) == 4 ? 16384u : 0u);

    const uint32_t tx = blockIdx.x % p.tiles_x, ty = blockIdx.x / p.tiles_x;
    const uint32_t r0 = ty * MXQ_TILE, c0 = tx * MXQ_TILE;
    const uint32_t lane16 = threadIdx.x & 15u, row_in = threadIdx.x >> 4;      // 16 lanes to a row of the tile, 16 rows at a time
    const uint32_t c = c0 + lane16 * 8u;
    const uint32_t left = c < p.r.cols ? p.r.cols - c : 0u;                    // numbers from here on in a row
    griddep_wait();
    griddep_launch();

    Row8<XT> raw[8];
    const Rows<XT> x(p.x, p.r.rows, p.r.cols, p.stride);
    constexpr int AT_ONCE = VEC ? 8 : 4;                                       // (what lies unaligned takes more registers on its way)
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += AT_ONCE) {
        Asked8<XT, VEC> a[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const uint32_t r = r0 + row_in + 16u * (i0 + i);
            a[i].ask(x, r, c / 8u, r < p.r.rows ? left : 0u);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const uint32_t r = r0 + row_in + 16u * (i0 + i);
            a[i].take(x, r, c / 8u, r < p.r.rows ? left : 0u, raw[i0 + i]);
        }
    }
    constexpr uint32_t PIECES = sizeof(XT) == 4 ? 8u : 4u, PITCH = MXQ_TILE * (uint32_t)sizeof(XT);       // 16-byte pieces of a block; bytes of a row
    unsigned char* tile_of = reinterpret_cast<unsigned char*>(numbers);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t r = row_in + 16u * i, block = lane16 >> 2, turn = mxq_turn<XT>(r, block), first = (lane16 & 3u) * (PIECES / 4u);
        uint4 q[Raw8<XT>::N];
        to_units(raw[i], q);
#pragma unroll
        for (uint32_t u = 0; u < PIECES / 4u; ++u)
            *reinterpret_cast<uint4*>(tile_of + r * PITCH + (block * PIECES + ((first + u) ^ turn)) * 16u) = q[u];
    }
    __syncthreads();
    if (ROWS) {
        const uint32_t stage = c0 / F::STAGE, atom = (c0 % F::STAGE) / 128u;
        unsigned char* tile = p.by_rows + mx_tile_offset(p.r, ty, stage);
#pragma unroll
        for (uint32_t t = threadIdx.x; t < 512u; t += MXQ_THREADS) {
            const uint32_t r = t >> 2, block = t & 3u, turn = mxq_turn<XT>(r, block);
            uint32_t e = 0u;
            if (r0 + r < p.r.rows) {
                uint4 q[PIECES];
#pragma unroll
                for (uint32_t j = 0; j < PIECES; ++j) q[j] = *reinterpret_cast<const uint4*>(tile_of + r * PITCH + (block * PIECES + (j ^ turn)) * 16u);
                uint32_t big = 0u;
                if constexpr (sizeof(XT) == 2) {
                    uint32_t m = larger_of_each<XT>(larger_of_each<XT>(q[0].x, q[0].y), larger_of_each<XT>(q[0].z, q[0].w));
#pragma unroll
                    for (uint32_t j = 1; j < PIECES; ++j)
                        m = larger_of_each<XT>(m, larger_of_each<XT>(larger_of_each<XT>(q[j].x, q[j].y), larger_of_each<XT>(q[j].z, q[j].w)));
                    big = max(magnitude(half_of<XT>(m, 0u)), magnitude(half_of<XT>(m, 1u)));
                } else {
#pragma unroll
                    for (uint32_t j = 0; j < PIECES; ++j)
                        big = max(big, max(max(q[j].x & 0x7FFFFFFFu, q[j].y & 0x7FFFFFFFu), max(q[j].z & 0x7FFFFFFFu, q[j].w & 0x7FFFFFFFu)));
                }
                e = mx_scale_byte<FMT>(big);
                const float inverse = mx_inverse(e);
                uint2 codes8[4];
#pragma unroll
                for (uint32_t h = 0; h < 4; ++h) {
                    uint4 some[Raw8<XT>::N];
#pragma unroll
                    for (uint32_t u = 0; u < PIECES / 4u; ++u) some[u] = q[h * (PIECES / 4u) + u];
                    Row8<XT> eight;
                    from_units(some, eight);
                    float v[8];
                    eight.get(v);
                    codes8[h] = mx_codes8<FMT>(v, inverse);
                }
                if (FMT == MX_E4M3) {
                    *reinterpret_cast<uint4*>(tile + mx_piece(r, 2u * block)) = make_uint4(codes8[0].x, codes8[0].y, codes8[1].x, codes8[1].y);
                    *reinterpret_cast<uint4*>(tile + mx_piece(r, 2u * block + 1u)) = make_uint4(codes8[2].x, codes8[2].y, codes8[3].x, codes8[3].y);
                } else {
                    *reinterpret_cast<uint4*>(tile + mx_piece(r, atom * 4u + block)) = make_uint4(codes8[0].x, codes8[1].x, codes8[2].x, codes8[3].x);
                }
            }
            row_scales[mx_scale_slot(r) + block] = (unsigned char)e;
        }
        __syncthreads();
        if (threadIdx.x < 128u) {
            uint32_t* to = reinterpret_cast<uint32_t*>(p.by_rows + mx_scales_at(p.r) + (((uint64_t)ty * p.r.stages + stage) * F::ATOMS + atom) * 512u);
            if (r0 < p.r.rows) to[threadIdx.x] = reinterpret_cast<const uint32_t*>(row_scales)[threadIdx.x];
        }
    }
    if (COLS) {
        if (c0 >= p.r.cols) return;                                // (the tile is there for the blob by rows alone)
        constexpr uint32_t W = sizeof(XT) == 4 ? 1u : 2u;          // columns of a thread
        constexpr uint32_t TASKS = 128u / W * 4u;
        const uint32_t stage = r0 / F::STAGE, atom = (r0 % F::STAGE) / 128u;
        for (uint32_t t = threadIdx.x; t < TASKS; t += MXQ_THREADS) {
            const uint32_t col = t % (128u / W) * W, block = t / (128u / W);
            uint32_t word[32];
            // (even rows turn their pieces one way, odd ones the other)
            constexpr uint32_t E = 16u / (uint32_t)sizeof(XT);
            const uint32_t across = col >> 5, j = (col & 31u) / E, in = (col % E) * (uint32_t)sizeof(XT);
            const unsigned char* even = tile_of + block * 32u * PITCH + (across * PIECES + (j ^ mxq_turn<XT>(0u, across))) * 16u + in;
            const unsigned char* odd = tile_of + block * 32u * PITCH + (across * PIECES + (j ^ mxq_turn<XT>(1u, across))) * 16u + in;
#pragma unroll
            for (int i = 0; i < 32; ++i) word[i] = *reinterpret_cast<const uint32_t*>(((i & 1) ? odd : even) + i * PITCH);
            if constexpr (W == 2) {                                // (as many tasks as threads)
                static_assert(TASKS == MXQ_THREADS, "one task a thread");
                __syncthreads();
            }
            uint32_t big_of_each = word[0];                        // of the column, or of the two
            if constexpr (W == 2) {
#pragma unroll
                for (int i = 1; i < 32; ++i) big_of_each = larger_of_each<XT>(big_of_each, word[i]);
            }
#pragma unroll
            for (uint32_t w = 0; w < W; ++w) {
                float v[4][8];
                uint32_t big = 0;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    if constexpr (W == 1) {
                        v[i >> 3][i & 7] = __uint_as_float(word[i]);
                        big = max(big, word[i] & 0x7FFFFFFFu);
                    } else {
                        v[i >> 3][i & 7] = half_of<XT>(word[i], w);
                    }
                }
                if constexpr (W == 2) big = magnitude(half_of<XT>(big_of_each, w));
                const uint32_t e = mx_scale_byte<FMT>(big);
                const float inverse = mx_inverse(e);
                const uint32_t row = col + w;
                col_scales[mx_scale_slot(row) + block] = (unsigned char)e;
                const uint2 q0 = mx_codes8<FMT>(v[0], inverse), q1 = mx_codes8<FMT>(v[1], inverse), q2 = mx_codes8<FMT>(v[2], inverse),
                            q3 = mx_codes8<FMT>(v[3], inverse);
                if (FMT == MX_E4M3) {
                    *reinterpret_cast<uint4*>(codes + mx_piece(row, 2u * block)) = make_uint4(q0.x, q0.y, q1.x, q1.y);
                    *reinterpret_cast<uint4*>(codes + mx_piece(row, 2u * block + 1u)) = make_uint4(q2.x, q2.y, q3.x, q3.y);
                } else {
                    *reinterpret_cast<uint4*>(codes + mx_piece(row, atom * 4u + block)) = make_uint4(q0.x, q1.x, q2.x, q3.x);
                }
            }
        }
        __syncthreads();
        unsigned char* tile = p.by_cols + mx_tile_offset(p.c, tx, stage);
        constexpr uint32_t OUT = FMT == MX_E4M3 ? 8u : 4u;             // pieces of codes in a row
        for (uint32_t t = threadIdx.x; t < 128u * OUT; t += MXQ_THREADS) {
            const uint32_t row = t / OUT, at = mx_piece(row, (FMT == MX_E4M3 ? 0u : atom * 4u) + t % OUT);
            if (c0 + row < p.c.rows) *reinterpret_cast<uint4*>(tile + at) = *reinterpret_cast<const uint4*>(codes + at);
        }
        if (threadIdx.x < 128u) {
            uint32_t* to = reinterpret_cast<uint32_t*>(p.by_cols + mx_scales_at(p.c) + (((uint64_t)tx * p.c.stages + stage) * F::ATOMS + atom) * 512u);
            to[threadIdx.x] = reinterpret_cast<const uint32_t*>(col_scales)[threadIdx.x];
        }
    }
}

// Back: a CTA takes 64 (e4m3) or 32 (e2m1) rows of a tile, a thread 8 numbers of each of 4 rows, whose reads are under way together; a
// warp's stores are whole lines.  Bound by memory: 8192 x 4096 e4m3 to bf16 15.4 us, the copy rate.  (16 numbers a thread from whole
// pieces, whose stores are half lines: 18.4 us.)
template <typename OT, int FMT, bool VEC>
__global__ void __launch_bounds__(256)
mx_dequantize_kernel(const unsigned char* blob, MxShape s, OT* out) {
    typedef MxFormat<FMT> F;
    constexpr uint32_t LANES = F::STAGE / 8u, ROWS = 256u / LANES, AT_ONCE = 4u;      // lanes of a row; rows at a time
    griddep_wait();
    griddep_launch();
    constexpr uint32_t PARTS = 128u / (ROWS * AT_ONCE);                                // CTAs of a tile
    const uint32_t of = blockIdx.x / PARTS, rb = of / s.stages, stage = of % s.stages, r0 = blockIdx.x % PARTS * (ROWS * AT_ONCE);
    const uint32_t lane = threadIdx.x % LANES, first = threadIdx.x / LANES, block = lane / 4u, c = stage * F::STAGE + lane * 8u;
    const uint32_t rows = min(128u, s.rows - rb * 128u), left = c < s.cols ? s.cols - c : 0u;
    const unsigned char* tile = blob + mx_tile_offset(s, rb, stage);
    const unsigned char* scales = blob + mx_scales_at(s) + ((uint64_t)of * F::ATOMS + block / 4u) * 512u + (block & 3u);
    OT* to = out + (uint64_t)rb * 128u * s.cols + (left ? c : 0u);
    if (r0 < rows) {
        uint2 q[AT_ONCE];
        uint32_t e[AT_ONCE];
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i) {
            const uint32_t r = r0 + i * ROWS + first;
            q[i] = make_uint2(0u, 0u);
            e[i] = 0u;
            if (r < rows && left) {
                if (FMT == MX_E4M3) q[i] = *reinterpret_cast<const uint2*>(tile + mx_piece(r, lane >> 1) + (lane & 1u) * 8u);
                else q[i].x = *reinterpret_cast<const uint32_t*>(tile + mx_piece(r, lane >> 2) + (lane & 3u) * 4u);
                e[i] = scales[mx_scale_slot(r)];
            }
        }
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i) {
            const uint32_t r = r0 + i * ROWS + first;
            const float scale = mx_scale(e[i]);
            float v[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t pair = FMT == MX_E4M3 ? ((k < 2 ? q[i].x : q[i].y) >> (16 * (k & 1))) & 0xFFFFu : (q[i].x >> (8 * k)) & 0xFFu;
                const __half2_raw two = FMT == MX_E4M3 ? __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3)
                                                       : __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)pair, __NV_E2M1);
                const float2 f = __half22float2(__half2(two)), g = times(f.x, f.y, scale);
                v[2 * k] = g.x;
                v[2 * k + 1] = g.y;
            }
            Row8<OT> eight;
            eight.set(v);
            if (VEC) {
                if (r < rows && left) eight.store(to + (uint64_t)r * s.cols);
            } else {
                uint4 units[Raw8<OT>::N];
                to_units(eight, units);
                Units<OT>::store(to + (uint64_t)min(r, rows - 1u) * s.cols, r < rows ? left : 0u, units, lane == 0u, lane == LANES - 1u);
            }
        }
    }
}

}  // namespace divk

namespace {
using namespace divk;

template <typename XT, int FMT>
div_status quantize_launch(const MxQuantParams& p, bool rows, bool cols, bool vec, uint32_t grid, cudaStream_t st) {
    const uint32_t smem = mxq_smem_bytes<XT>(cols);
    void (*kern)(const MxQuantParams) =
        rows ? (cols ? (vec ? mx_quantize_kernel<XT, FMT, true, true, true> : mx_quantize_kernel<XT, FMT, true, true, false>)
                     : (vec ? mx_quantize_kernel<XT, FMT, true, false, true> : mx_quantize_kernel<XT, FMT, true, false, false>))
             : (vec ? mx_quantize_kernel<XT, FMT, false, true, true> : mx_quantize_kernel<XT, FMT, false, true, false>);
    static SmemAllowed allowed[8];
    if (smem > 48u * 1024u && !allowed[(cols ? 4 : 0) + (rows ? 2 : 0) + (vec ? 1 : 0)]((const void*)kern, smem)) return DIV_ERR_CUDA;
    return launch_pdl(kern, dim3(grid), MXQ_THREADS, smem, st, p);
}

}  // namespace

extern "C" {

div_status div_mx_bytes(int64_t rows, int64_t cols, int32_t format, div_mx_layout* out) {
    if (!out) return DIV_ERR_NULL;
    if (!lm_size_ok(rows) || !lm_size_ok(cols)) return DIV_ERR_SHAPE;
    if (!mx_format_ok(format)) return DIV_ERR_PARAM;
    const MxShape s = mx_shape((uint32_t)rows, (uint32_t)cols, format);
    out->codes_off = 0;
    out->codes_bytes = mx_codes_bytes(s);
    out->scales_off = mx_scales_at(s);
    out->scales_bytes = mx_scales_bytes(s, format);
    out->total_bytes = out->scales_off + out->scales_bytes;
    const uint64_t blocks = (uint64_t)rows * (((uint64_t)cols + 31u) / 32u);
    out->closed_form_bytes = blocks * (1u + (format == MX_E4M3 ? 32u : 16u));
    return DIV_OK;
}

div_status div_mx_quantize(const void* x_dev, int64_t rows, int64_t cols, int64_t row_stride, int32_t x_dtype, int32_t format,
                           void* by_rows_dev, size_t by_rows_capacity, void* by_columns_dev, size_t by_columns_capacity, void* cuda_stream) {
    if (!x_dev || (!by_rows_dev && !by_columns_dev)) return DIV_ERR_NULL;
    if (!lm_size_ok(rows) || !lm_size_ok(cols) || (rows > 1 && row_stride < cols)) return DIV_ERR_SHAPE;
    if (!lm_dtype_ok(x_dtype) || !mx_format_ok(format)) return DIV_ERR_PARAM;
    const uint32_t size = lm_dtype_bytes(x_dtype);
    if ((reinterpret_cast<uintptr_t>(x_dev) % size) != 0 || !aligned_16(by_rows_dev) || !aligned_16(by_columns_dev)) return DIV_ERR_ALIGN;
    MxQuantParams p;
    p.x = x_dev;
    p.stride = (uint64_t)row_stride;
    p.r = mx_shape((uint32_t)rows, (uint32_t)cols, format);
    p.c = mx_shape((uint32_t)cols, (uint32_t)rows, format);
    p.by_rows = (unsigned char*)by_rows_dev;
    p.by_cols = (unsigned char*)by_columns_dev;
    if (by_rows_dev && by_rows_capacity < mx_codes_bytes(p.r) + mx_scales_bytes(p.r, format)) return DIV_ERR_CAPACITY;
    if (by_columns_dev && by_columns_capacity < mx_codes_bytes(p.c) + mx_scales_bytes(p.c, format)) return DIV_ERR_CAPACITY;
    // whole stages of each direction that is asked for
    const uint64_t stage = mx_stage(format);
    const uint64_t across = by_rows_dev ? p.r.stages * (stage / MXQ_TILE) : ((uint64_t)cols + MXQ_TILE - 1) / MXQ_TILE;
    const uint64_t down = by_columns_dev ? p.c.stages * (stage / MXQ_TILE) : ((uint64_t)rows + MXQ_TILE - 1) / MXQ_TILE;
    if (across * down >= (1ull << 31)) return DIV_ERR_SHAPE;
    p.tiles_x = (uint32_t)across;
    // reads of 16 bytes where every row begins at a multiple of them and holds whole ones
    const bool vec = aligned_16(x_dev) && cols % 8 == 0 && (rows == 1 || row_stride % 8 == 0);
    return with_type(x_dtype, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> XT;
        return format == MX_E4M3 ? quantize_launch<XT, MX_E4M3>(p, by_rows_dev, by_columns_dev, vec, (uint32_t)(across * down), (cudaStream_t)cuda_stream)
                                 : quantize_launch<XT, MX_E2M1>(p, by_rows_dev, by_columns_dev, vec, (uint32_t)(across * down), (cudaStream_t)cuda_stream);
    });
}

div_status div_mx_dequantize(const void* blob_dev, size_t blob_bytes, int64_t rows, int64_t cols, int32_t format, void* out_dev,
                             int32_t out_dtype, void* cuda_stream) {
    if (!blob_dev || !out_dev) return DIV_ERR_NULL;
    if (!lm_size_ok(rows) || !lm_size_ok(cols)) return DIV_ERR_SHAPE;
    if (!lm_dtype_ok(out_dtype) || !mx_format_ok(format)) return DIV_ERR_PARAM;
    if (!aligned_16(blob_dev) || (reinterpret_cast<uintptr_t>(out_dev) % lm_dtype_bytes(out_dtype)) != 0) return DIV_ERR_ALIGN;
    const MxShape s = mx_shape((uint32_t)rows, (uint32_t)cols, format);
    if (blob_bytes < mx_codes_bytes(s) + mx_scales_bytes(s, format)) return DIV_ERR_CAPACITY;
    const uint64_t tiles = (uint64_t)((s.rows + 127u) / 128u) * s.stages;
    const uint64_t grid = tiles * (format == MX_E4M3 ? 2u : 4u);
    if (grid >= (1ull << 31)) return DIV_ERR_SHAPE;
    const bool vec = aligned_16(out_dev) && cols % 8 == 0;
    return with_type(out_dtype, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> OT;
        auto kern = format == MX_E4M3 ? (vec ? mx_dequantize_kernel<OT, MX_E4M3, true> : mx_dequantize_kernel<OT, MX_E4M3, false>)
                                      : (vec ? mx_dequantize_kernel<OT, MX_E2M1, true> : mx_dequantize_kernel<OT, MX_E2M1, false>);
        return launch_pdl(kern, dim3((uint32_t)grid), 256, 0, (cudaStream_t)cuda_stream, (const unsigned char*)blob_dev, s, (OT*)out_dev);
    });
}

}  // extern "C"
