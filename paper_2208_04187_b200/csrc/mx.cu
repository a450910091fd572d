// Microscaled quantisation of a matrix, by rows, by columns or both from one reading, and its way back.
//
//   by rows     the blob of x (rows x cols), blocks of 32 neighbours along a row
//   by columns  the blob of the transposed matrix (cols x rows), blocks of 32 neighbours down a column
//
// Both are bound by memory: x is read once, 1 + 1/32 or 1/2 + 1/32 bytes a number are written for each direction.
//
// A CTA takes 128 x 128 numbers, which are whole tiles of e4m3 codes in both directions (half tiles of e2m1).  A thread reads
// 8 neighbours at a time, 8 times, all reads under way together; 4 lanes hold a block, whose largest magnitude takes two
// shuffles.  For the columns the numbers go through shared memory as they are; a thread then owns 32 rows of one column
// (two columns of 16-bit types, one word), and its codes go through shared memory once more, so that whole lines leave the SM.
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
    // numbers; codes by columns as their tile lies in the blob; scales by columns
    return 512u + (cols ? MXQ_TILE * MXQ_TILE * (uint32_t)sizeof(XT) + 16384u + 512u : 0u);
}

template <typename XT, int FMT, bool ROWS, bool COLS, bool VEC>
__global__ void __launch_bounds__(MXQ_THREADS)
mx_quantize_kernel(const __grid_constant__ MxQuantParams p) {
    typedef MxFormat<FMT> F;
    extern __shared__ __align__(128) unsigned char smem[];
    uint32_t* row_scales = reinterpret_cast<uint32_t*>(smem);
    XT* numbers = reinterpret_cast<XT*>(smem + 512);
    unsigned char* codes = smem + 512 + MXQ_TILE * MXQ_TILE * sizeof(XT);
    unsigned char* col_scales = codes + 16384;

    const uint32_t tx = blockIdx.x % p.tiles_x, ty = blockIdx.x / p.tiles_x;
    const uint32_t r0 = ty * MXQ_TILE, c0 = tx * MXQ_TILE;
    const uint32_t lane16 = threadIdx.x & 15u, row_in = threadIdx.x >> 4;      // 16 lanes to a row of the tile, 16 rows at a time
    const uint32_t c = c0 + lane16 * 8u;
    const uint32_t left = c < p.r.cols ? p.r.cols - c : 0u;                    // numbers from here on in a row
    griddep_wait();
    griddep_launch();

    Row8<XT> raw[8];
    const Rows<XT> x(p.x, p.r.rows, p.r.cols, p.stride);
    constexpr int AT_ONCE = VEC || sizeof(XT) == 2 ? 8 : 4;                    // (what lies unaligned takes more registers on its way)
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
    if (COLS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i].store(numbers + (row_in + 16u * i) * MXQ_TILE + lane16 * 8u);
    }
    if (ROWS) {
        const uint32_t stage = c0 / F::STAGE, atom = (c0 % F::STAGE) / 128u;
        unsigned char* tile = p.by_rows + mx_tile_offset(p.r, ty, stage);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t rt = row_in + 16u * i;
            float v[8];
            raw[i].get(v);
            uint32_t big = raw[i].largest();
            big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
            big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
            const uint32_t e = mx_scale_byte<FMT>(big);
            const uint2 q = mx_codes8<FMT>(v, mx_inverse(e));
            if (r0 + rt < p.r.rows) {
                if (FMT == MX_E4M3) *reinterpret_cast<uint2*>(tile + mx_piece(rt, lane16 >> 1) + (lane16 & 1u) * 8u) = q;
                else *reinterpret_cast<uint32_t*>(tile + mx_piece(rt, atom * 4u + (lane16 >> 2)) + (lane16 & 3u) * 4u) = q.x;
            }
            // the 4 scales of a row in one word
            uint32_t word = e << ((lane16 >> 2) * 8u);
            word |= __shfl_xor_sync(0xFFFFFFFFu, word, 4);
            word |= __shfl_xor_sync(0xFFFFFFFFu, word, 8);
            if (lane16 == 0) row_scales[mx_scale_slot(rt) >> 2] = word;
        }
        __syncthreads();
        if (threadIdx.x < 128u) {
            uint32_t* to = reinterpret_cast<uint32_t*>(p.by_rows + mx_scales_at(p.r) + (((uint64_t)ty * p.r.stages + stage) * F::ATOMS + atom) * 512u);
            if (r0 < p.r.rows) to[threadIdx.x] = row_scales[threadIdx.x];
        }
    } else {
        __syncthreads();
    }
    if (COLS) {
        if (c0 >= p.r.cols) return;                                // (the tile is there for the blob by rows alone)
        constexpr uint32_t W = sizeof(XT) == 4 ? 1u : 2u;          // columns of a thread
        constexpr uint32_t TASKS = 128u / W * 4u;
        const uint32_t stage = r0 / F::STAGE, atom = (r0 % F::STAGE) / 128u;
        for (uint32_t t = threadIdx.x; t < TASKS; t += MXQ_THREADS) {
            const uint32_t col = t % (128u / W) * W, block = t / (128u / W);
            uint32_t word[32];
            const XT* from = numbers + block * 32u * MXQ_TILE + col;
#pragma unroll
            for (int i = 0; i < 32; ++i) word[i] = *reinterpret_cast<const uint32_t*>(from + i * MXQ_TILE);
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
        constexpr uint32_t PIECES = FMT == MX_E4M3 ? 8u : 4u;
        for (uint32_t t = threadIdx.x; t < 128u * PIECES; t += MXQ_THREADS) {
            const uint32_t row = t / PIECES, at = mx_piece(row, (FMT == MX_E4M3 ? 0u : atom * 4u) + t % PIECES);
            if (c0 + row < p.c.rows) *reinterpret_cast<uint4*>(tile + at) = *reinterpret_cast<const uint4*>(codes + at);
        }
        if (threadIdx.x < 128u) {
            uint32_t* to = reinterpret_cast<uint32_t*>(p.by_cols + mx_scales_at(p.c) + (((uint64_t)tx * p.c.stages + stage) * F::ATOMS + atom) * 512u);
            to[threadIdx.x] = reinterpret_cast<const uint32_t*>(col_scales)[threadIdx.x];
        }
    }
}

// Back: a thread takes one 16-byte piece of codes (16 numbers of e4m3, a whole block of e2m1), 8 lanes a tile's row.
template <typename OT, int FMT, bool VEC>
__global__ void __launch_bounds__(256)
mx_dequantize_kernel(const unsigned char* blob, MxShape s, OT* out) {
    typedef MxFormat<FMT> F;
    constexpr uint32_t PER = F::STAGE / 8u;                       // numbers of a piece
    griddep_wait();
    griddep_launch();
    const uint64_t job = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    const uint64_t line = job >> 3;                               // row-major over (128 rows, stage, row of the tile)
    const uint32_t piece = (uint32_t)job & 7u;
    const uint64_t tile = line >> 7;
    const uint32_t rt = (uint32_t)line & 127u, rb = (uint32_t)(tile / s.stages), stage = (uint32_t)(tile % s.stages);
    const uint64_t row = (uint64_t)rb * 128u + rt;
    const uint32_t c = stage * F::STAGE + piece * PER;
    const uint32_t left = row < s.rows && c < s.cols ? s.cols - c : 0u;
    if (VEC && left == 0u) return;
    uint4 q = make_uint4(0u, 0u, 0u, 0u);
    uint32_t e = 0;
    if (left) {
        q = *reinterpret_cast<const uint4*>(blob + mx_tile_offset(s, rb, stage) + mx_piece(rt, piece));
        const uint32_t block = piece * PER / 32u;                 // of the stage
        e = blob[mx_scales_at(s) + ((uint64_t)tile * F::ATOMS + block / 4u) * 512u + mx_scale_slot(rt) + (block & 3u)];
    }
    const float scale = mx_scale(e);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    OT* to = out + (left ? row * s.cols + c : 0u);
    constexpr int N = Raw8<OT>::N;                                // 16-byte units of 8 numbers
    uint4 units[PER / 8u * N];
#pragma unroll
    for (uint32_t h = 0; h < PER / 8u; ++h) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = FMT == MX_E4M3 ? (w[2 * h + (i >> 1)] >> (16 * (i & 1))) & 0xFFFFu : (w[h] >> (8 * i)) & 0xFFu;
            const __half2_raw two = FMT == MX_E4M3 ? __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3)
                                                   : __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)pair, __NV_E2M1);
            const float2 f = __half22float2(__half2(two));
            v[2 * i] = __fmul_rn(f.x, scale);
            v[2 * i + 1] = __fmul_rn(f.y, scale);
        }
        Row8<OT> r;
        r.set(v);
        uint4 some[N];
        to_units(r, some);
#pragma unroll
        for (int u = 0; u < N; ++u) units[h * N + u] = some[u];
    }
    if (VEC) {
#pragma unroll
        for (uint32_t u = 0; u < PER / 8u * N; ++u)
            if (u / N * 8u < left) reinterpret_cast<uint4*>(to)[u] = units[u];
    } else {
        Units<OT>::store(to, left, units, piece == 0u, piece == 7u);
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
    static SmemAllowed allowed[4];
    if (cols && !allowed[(rows ? 2 : 0) + (vec ? 1 : 0)]((const void*)kern, smem)) return DIV_ERR_CUDA;
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
    // (the last tile's rows that are not there would be whole CTAs: 32 rows each)
    const uint64_t grid = tiles * 4u;
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
