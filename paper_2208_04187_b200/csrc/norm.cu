// Root-mean-square normalisation with the residual's addition, forward (output in the input's type, or as a microscaled blob, or both)
// and backward.
//
//   h = round(x + residual)          what the next layers add to; h = x where there is no residual
//   y = h * rstd * w,  rstd = 1 / sqrt(mean(h^2) + eps)
//   dx = dresidual = dh + rstd * (w dy - n * mean(w dy n)),  n = h * rstd;   dw = sum over rows of dy n
//
// Bound by memory: forward reads x and the residual and writes h and y (or 1 + 1/32 bytes a number), backward reads dy, dh and h and writes dx.
// A row is held by G threads, 8 neighbours of each 8 * G, in registers from the first reading to the last use (rows of more than
// NORM_MAX_HELD numbers are read twice).  Sums are in 32 bits: a thread's own numbers, then a tree.  Backward's CTAs stay for many rows and
// keep their columns' sums of dy n in registers; the CTAs' sums are joined by a second kernel in a fixed order.
#include "mx.cuh"

namespace divk {

constexpr int NORM_NONE = -1;                   // no blob
constexpr uint32_t NORM_MAX_THREADS = 512, NORM_MAX_HELD = 16384;       // a thread holds at most 4 pieces of 8 in a row of 512 threads
// Backward's CTAs stay for many rows: as many as fit an SM, by the threads of each (what a thread holds takes 64 registers with one
// piece, 128 with two, 102 where that lets two CTAs of 320 threads in).  More CTAs than fit, or fewer, took longer: 16384 x 4096
// bf16 with 256 threads 161, 97, 119, 101 us for 1, 2, 3, 4 CTAs an SM.
constexpr uint32_t NORM_SMS = 148;
__host__ __device__ constexpr uint32_t norm_resident(int held, uint32_t threads) {
    return held == 1 ? 1024u / threads : held == 2 ? (threads <= 256u ? 512u / threads : threads <= 320u ? 2u : 1u) : 1u;
}

struct NormParams {
    const void *x, *residual, *w;
    uint64_t x_stride, r_stride;
    uint32_t rows, cols;
    float eps;
    void *h, *y;
    float* rstd;
    unsigned char* blob;
    MxShape s;
    uint32_t pieces;           // of 8 numbers: the row's, up to whole stages of the blob where there is one
    uint32_t group;            // threads of a row
};

// sum over the `group` threads of a row (whole warps, all of the CTA's or a power of two that divides them; all threads come here together)
__device__ __forceinline__ float norm_sum(float v, uint32_t group, float* shared) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if (group == 32u) return v;
    const uint32_t warp = threadIdx.x >> 5, warps = group >> 5, first = warp / warps * warps;
    __syncthreads();                               // (what the last row left here has been read)
    if ((threadIdx.x & 31u) == 0) shared[warp] = v;
    __syncthreads();
    v = (threadIdx.x & 31u) < warps ? shared[first + (threadIdx.x & 31u)] : 0.f;
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}
// 8 numbers of a row from `at` * 8 on; `left` of them are there
template <typename T, bool VEC>
__device__ __forceinline__ void norm_load(const Rows<T>& m, uint64_t row, uint32_t at, uint32_t left, float (&v)[8]) {
    Asked8<T, VEC> a;
    a.ask(m, row, at, left);
    a.take(m, row, at, left, v);
}
// all lanes of a warp together, with pieces that follow one another; left 0: nothing
template <typename T, bool VEC>
__device__ __forceinline__ void norm_store(T* p, uint32_t left, const float (&v)[8]) {
    if (VEC) {
        if (left) {
            Row8<T> r;
            r.set(v);
            r.store(p);
        }
    } else {
        store8_row(p, left, v);
    }
}
__device__ __forceinline__ uint32_t norm_left(bool there, uint32_t at, uint32_t cols) { return there && at * 8u < cols ? cols - at * 8u : 0u; }

// h of `M` pieces of a row, `group` apart from `at` on: added in 32 bits, rounded, and stored where there is a residual (as norm_store)
template <typename XT, bool VEC, int M>
__device__ __forceinline__ void norm_h(const NormParams& p, uint32_t row, bool there, uint32_t at, float (&h)[M][8]) {
    const Rows<XT> x(p.x, p.rows, p.cols, p.x_stride), r(p.residual, p.rows, p.cols, p.r_stride);
    Asked8<XT, VEC> ax[M], ar[M];
#pragma unroll
    for (int j = 0; j < M; ++j) {
        const uint32_t left = norm_left(there, at + j * p.group, p.cols);
        ax[j].ask(x, row, at + j * p.group, left);
        if (p.residual) ar[j].ask(r, row, at + j * p.group, left);
    }
#pragma unroll
    for (int j = 0; j < M; ++j) {
        const uint32_t here = at + j * p.group, left = norm_left(there, here, p.cols);
        ax[j].take(x, row, here, left, h[j]);
        if (p.residual) {
            float v[8];
            ar[j].take(r, row, here, left, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[j][i] = to_f32(from_f32<XT>(h[j][i] + v[i]));
            norm_store<XT, VEC>(static_cast<XT*>(p.h) + (uint64_t)row * p.cols + here * 8u, left, h[j]);
        }
    }
}
// y of a piece, and its codes (as norm_store)
template <typename XT, typename WT, int FMT, bool VEC>
__device__ __forceinline__ void norm_out(const NormParams& p, uint32_t row, bool row_there, uint32_t at, const float (&h)[8], float rstd) {
    const uint32_t left = norm_left(row_there, at, p.cols);
    float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (left) {
        float w[8];
        norm_load<WT, VEC>(Rows<WT>(p.w, 1u, p.cols, 0u), 0u, at, left, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = h[i] * rstd * w[i];
        if (!VEC) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = (uint32_t)i < left ? y[i] : 0.f;      // (0 times an infinite rstd would be NaN)
        }
    }
    if (p.y) norm_store<XT, VEC>(static_cast<XT*>(p.y) + (uint64_t)row * p.cols + at * 8u, left, y);
    if (FMT != NORM_NONE) {
        constexpr int F = FMT == NORM_NONE ? 0 : FMT;
        float most = fabsf(y[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(fabsf(y[i])));
        uint32_t big = __float_as_uint(most);                                          // (a NaN's bits order above all)
        big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
        big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
        const uint32_t e = mx_scale_byte<F>(big);
        const uint2 q = mx_codes8<F>(y, mx_inverse(e));
        if (row_there && at < p.pieces) {
            constexpr uint32_t PER = MxFormat<F>::STAGE / 8u;
            const uint32_t rb = row >> 7, rt = row & 127u, stage = at / PER, in = at % PER;
            unsigned char* tile = p.blob + mx_tile_offset(p.s, rb, stage);
            if (F == MX_E4M3) *reinterpret_cast<uint2*>(tile + mx_piece(rt, in >> 1) + (in & 1u) * 8u) = q;
            else *reinterpret_cast<uint32_t*>(tile + mx_piece(rt, in >> 2) + (in & 3u) * 4u) = q.x;
            if ((at & 3u) == 0u)
                p.blob[mx_scales_at(p.s) + (((uint64_t)rb * p.s.stages + stage) * MxFormat<F>::ATOMS + in / 16u) * 512u + mx_scale_slot(rt) + (in / 4u & 3u)] =
                    (unsigned char)e;
        }
    }
}

template <typename XT, typename WT, int FMT, bool VEC, int HELD>       // HELD: pieces that a thread holds; 0: rows are read twice
__global__ void __launch_bounds__(NORM_MAX_THREADS)
norm_forward_kernel(const __grid_constant__ NormParams p) {
    __shared__ float shared[32];
    const uint32_t per = blockDim.x / p.group, t = threadIdx.x % p.group;
    const uint64_t wide = (uint64_t)blockIdx.x * per + threadIdx.x / p.group;
    const bool there = wide < p.rows;
    const uint32_t row = there ? (uint32_t)wide : 0u;
    griddep_wait();
    griddep_launch();
    if (HELD) {
        float h[HELD ? HELD : 1][8];
        float sum = 0.f;
        norm_h<XT, VEC>(p, row, there, t, h);
#pragma unroll
        for (int j = 0; j < HELD; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(h[j][i], h[j][i], sum);
        const float rstd = 1.0f / sqrtf(norm_sum(sum, p.group, shared) / (float)p.cols + p.eps);
        if (there && t == 0 && p.rstd) p.rstd[row] = rstd;
#pragma unroll
        for (int j = 0; j < HELD; ++j) norm_out<XT, WT, FMT, VEC>(p, row, there, j * p.group + t, h[j], rstd);
    } else {
        float sum = 0.f;
        const uint32_t rounds = (p.pieces + p.group - 1u) / p.group;
        for (uint32_t j = 0; j < rounds; ++j) {
            const uint32_t at = j * p.group + t;
            float h[1][8];
            norm_h<XT, VEC>(p, row, there, at, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(h[0][i], h[0][i], sum);
        }
        const float rstd = 1.0f / sqrtf(norm_sum(sum, p.group, shared) / (float)p.cols + p.eps);
        if (there && t == 0 && p.rstd) p.rstd[row] = rstd;
        for (uint32_t j = 0; j < rounds; ++j) {
            const uint32_t at = j * p.group + t;
            float h[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (there && at * 8u < p.cols) {
                // (written by this CTA, before the barriers of the sum)
                if (p.residual) norm_load<XT, VEC>(Rows<XT>(static_cast<const XT*>(p.h) + (uint64_t)row * p.cols, 1u, p.cols, 0u), 0u, at, p.cols - at * 8u, h);
                else norm_load<XT, VEC>(Rows<XT>(p.x, p.rows, p.cols, p.x_stride), row, at, p.cols - at * 8u, h);
            }
            norm_out<XT, WT, FMT, VEC>(p, row, there, at, h, rstd);
        }
    }
}

struct NormBackParams {
    const void *dy, *dh, *h, *w;
    uint64_t dy_stride, dh_stride, h_stride;
    const float* rstd;
    uint32_t rows, cols;
    void* dx;
    float* sums;               // of dy n, one row for each CTA's groups
    uint32_t group;
};

template <typename XT, typename WT, bool VEC, int HELD, uint32_t THREADS>       // THREADS: at most
__global__ void __launch_bounds__(THREADS, norm_resident(HELD, THREADS))
norm_backward_kernel(const __grid_constant__ NormBackParams p) {
    __shared__ float shared[32];
    const uint32_t per = blockDim.x / p.group, t = threadIdx.x % p.group, mine = blockIdx.x * per + threadIdx.x / p.group;
    const uint32_t step = gridDim.x * per, rounds = (p.rows + step - 1u) / step;
    const float inv = 1.0f / (float)p.cols;
    griddep_wait();
    griddep_launch();
    float* sums = p.sums + (uint64_t)mine * p.cols;
    if (HELD) {
        constexpr int N = HELD ? HELD : 1;
        float acc[N][8];
#pragma unroll
        for (int j = 0; j < HELD; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[j][i] = 0.f;
        // the next row's dy and h are under way while this one is summed and written
        Asked8<XT, VEC> dy[N], h[N], dh[N];
        float rstd = 0.f, next_rstd = 0.f;
        const Rows<XT> all_dy(p.dy, p.rows, p.cols, p.dy_stride), all_h(p.h, p.rows, p.cols, p.h_stride), all_dh(p.dh, p.rows, p.cols, p.dh_stride);
        const auto bring = [&](uint32_t k) {
            const uint64_t row = (uint64_t)k * step + mine;
            next_rstd = row < p.rows ? p.rstd[row] : 0.f;
#pragma unroll
            for (int j = 0; j < HELD; ++j) {
                const uint32_t at = j * p.group + t, left = norm_left(row < p.rows, at, p.cols);
                dy[j].ask(all_dy, row, at, left);
                h[j].ask(all_h, row, at, left);
            }
        };
        bring(0);
        for (uint32_t k = 0; k < rounds; ++k) {
            const uint64_t row = (uint64_t)k * step + mine;
            const bool there = row < p.rows;
            float g[N][8], n[N][8];
            float dot = 0.f;
            rstd = next_rstd;
            if (p.dh) {
#pragma unroll
                for (int j = 0; j < HELD; ++j) dh[j].ask(all_dh, row, j * p.group + t, norm_left(there, j * p.group + t, p.cols));
            }
#pragma unroll
            for (int j = 0; j < HELD; ++j) {
                const uint32_t at = j * p.group + t, left = norm_left(there, at, p.cols);
                float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (at * 8u < p.cols) norm_load<WT, VEC>(Rows<WT>(p.w, 1u, p.cols, 0u), 0u, at, p.cols - at * 8u, w);
                dy[j].take(all_dy, row, at, left, g[j]);
                h[j].take(all_h, row, at, left, n[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    n[j][i] *= rstd;
                    acc[j][i] = fmaf(g[j][i], n[j][i], acc[j][i]);
                    g[j][i] *= w[i];
                    dot = fmaf(g[j][i], n[j][i], dot);
                }
            }
            bring(k + 1u);
            const float mean = norm_sum(dot, p.group, shared) * inv;
#pragma unroll
            for (int j = 0; j < HELD; ++j) {
                const uint32_t at = j * p.group + t, left = norm_left(there, at, p.cols);
                float d[8], add[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (p.dh) dh[j].take(all_dh, row, at, left, add);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = fmaf(rstd, fmaf(-n[j][i], mean, g[j][i]), add[i]);
                norm_store<XT, VEC>(static_cast<XT*>(p.dx) + row * p.cols + at * 8u, left, d);
            }
        }
        if (p.sums) {
#pragma unroll
            for (int j = 0; j < HELD; ++j) {
                const uint32_t at = j * p.group + t;
                norm_store<float, VEC>(sums + at * 8u, norm_left(true, at, p.cols), acc[j]);
            }
        }
    } else {
        const uint32_t pieces = (p.cols + 7u) / 8u;                // (the group is the CTA, and every CTA has a first row: its sums are all written)
        for (uint32_t k = 0; k < rounds; ++k) {
            const uint64_t wide = (uint64_t)k * step + mine;
            const bool there = wide < p.rows;
            const uint64_t row = there ? wide : 0u;
            const float rstd = there ? p.rstd[row] : 0.f;
            float dot = 0.f, mean = 0.f;
            for (int pass = 0; pass < 2; ++pass) {
                for (uint32_t j = 0; j * p.group < pieces; ++j) {
                    const uint32_t at = j * p.group + t, left = norm_left(there, at, p.cols);
                    float g[8], n[8], w[8], add[8], sum[8], d[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = n[i] = w[i] = add[i] = sum[i] = 0.f;
                    if (left) {
                        norm_load<XT, VEC>(Rows<XT>(p.dy, p.rows, p.cols, p.dy_stride), row, at, left, g);
                        norm_load<XT, VEC>(Rows<XT>(p.h, p.rows, p.cols, p.h_stride), row, at, left, n);
                        norm_load<WT, VEC>(Rows<WT>(p.w, 1u, p.cols, 0u), 0u, at, left, w);
                        if (pass && p.dh) norm_load<XT, VEC>(Rows<XT>(p.dh, p.rows, p.cols, p.dh_stride), row, at, left, add);
                        if (pass && p.sums && k) load8_any(sums + at * 8u, left, sum);          // (this thread's own writes)
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        n[i] *= rstd;
                        sum[i] = fmaf(g[i], n[i], sum[i]);
                        g[i] *= w[i];
                        if (!pass) dot = fmaf(g[i], n[i], dot);
                        d[i] = fmaf(rstd, fmaf(-n[i], mean, g[i]), add[i]);
                    }
                    if (pass) {
                        norm_store<XT, VEC>(static_cast<XT*>(p.dx) + row * p.cols + at * 8u, left, d);
                        if (p.sums && left) store8_any(sums + at * 8u, left, sum);
                    }
                }
                if (!pass) mean = norm_sum(dot, p.group, shared) * inv;
            }
        }
    }
}

// dw: 32 columns to a CTA, 32 rows of sums at a time, then a tree
template <typename WT>
__global__ void __launch_bounds__(1024)
norm_weight_kernel(const float* sums, uint32_t parts, uint32_t cols, WT* dw) {
    __shared__ float shared[32][33];
    griddep_wait();
    griddep_launch();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, c = blockIdx.x * 32u + lane;
    float v = 0.f;
    if (c < cols)
        for (uint32_t r = warp; r < parts; r += 32u) v += sums[(uint64_t)r * cols + c];
    shared[warp][lane] = v;
    __syncthreads();
    v = shared[lane][warp];
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const uint32_t mine = blockIdx.x * 32u + warp;
    if (lane == 0 && mine < cols) dw[mine] = from_f32<WT>(v);
}

}  // namespace divk

namespace {
using namespace divk;

inline uint32_t pow2_up(uint32_t v) {
    uint32_t p = 32;
    while (p < v) p <<= 1;
    return p;
}
// threads of a row, and pieces that each of them holds (0: too long to hold)
struct NormSplit {
    uint32_t group, held, threads;
};
NormSplit norm_split(uint64_t pieces, uint64_t rows) {
    NormSplit s;
    if (pieces > NORM_MAX_HELD / 8u) return {NORM_MAX_THREADS, 0u, NORM_MAX_THREADS};
    // two pieces a thread once rows fill the device, or where one would take more threads than there are
    s.held = pieces > 2u * NORM_MAX_THREADS ? 4u : pieces > NORM_MAX_THREADS || (rows >= 1024u && pieces >= 64u) ? 2u : 1u;
    const uint32_t need = (uint32_t)((pieces + s.held - 1u) / s.held);
    // rows of up to 128 threads share a CTA of 128; longer ones have a CTA of whole warps
    s.group = need <= 128u ? pow2_up(need) : (need + 31u) / 32u * 32u;
    s.threads = s.group < 128u ? 128u : s.group;
    return s;
}

template <typename XT, typename WT, bool VEC, int HELD>
div_status norm_forward_launch(const NormParams& p, int fmt, uint32_t grid, uint32_t threads, cudaStream_t st) {
    auto kern = fmt == MX_E4M3 ? norm_forward_kernel<XT, WT, MX_E4M3, VEC, HELD>
                               : fmt == MX_E2M1 ? norm_forward_kernel<XT, WT, MX_E2M1, VEC, HELD> : norm_forward_kernel<XT, WT, NORM_NONE, VEC, HELD>;
    return launch_pdl(kern, dim3(grid), threads, 0, st, p);
}
template <typename F>
div_status norm_types(int32_t dtype, int32_t w_dtype, F&& f) {
    return with_type(dtype, [&](auto* x) {
        if (w_dtype == dtype) return f(x, x);
        return f(x, (float*)nullptr);
    });
}
inline bool aligned_type(const void* p, int32_t dtype) { return reinterpret_cast<uintptr_t>(p) % lm_dtype_bytes(dtype) == 0; }
inline bool rows_vec(const void* p, int64_t rows, int64_t stride) { return !p || (aligned_16(p) && (rows == 1 || stride % 8 == 0)); }

// parts of the sums of backward: one for each group of threads
struct NormBack {
    NormSplit s;
    uint32_t grid, parts;
};
NormBack norm_back(int64_t rows, int64_t cols) {
    NormBack b;
    b.s = norm_split(((uint64_t)cols + 7u) / 8u, (uint64_t)rows);
    uint32_t per = b.s.threads / b.s.group;
    const uint64_t all = ((uint64_t)rows + per - 1u) / per;
    if (b.s.held == 4u) b.s = {NORM_MAX_THREADS, 0u, NORM_MAX_THREADS};             // (too many registers with gradients)
    const uint64_t most = b.s.held ? NORM_SMS * norm_resident((int)b.s.held, b.s.threads) : NORM_SMS * 2u;
    b.grid = (uint32_t)(all < most ? all : most);
    b.parts = b.grid * per;
    return b;
}

}  // namespace

extern "C" {

div_status div_rms_norm_forward(const void* x_dev, int64_t x_row_stride, const void* residual_dev, int64_t residual_row_stride,
                                const void* weight_dev, int32_t weight_dtype, int64_t rows, int64_t cols, int32_t dtype, float eps, void* h_dev,
                                void* y_dev, void* blob_dev, size_t blob_capacity, int32_t format, float* rstd_dev, void* cuda_stream) {
    if (!x_dev || !weight_dev || (!y_dev && !blob_dev) || (!h_dev != !residual_dev)) return DIV_ERR_NULL;
    if (!lm_size_ok(rows) || !lm_size_ok(cols) || (rows > 1 && (x_row_stride < cols || (residual_dev && residual_row_stride < cols)))) return DIV_ERR_SHAPE;
    if (!lm_dtype_ok(dtype) || !(weight_dtype == dtype || weight_dtype == DIV_F32) || !(eps >= 0.f) || (blob_dev && !mx_format_ok(format))) return DIV_ERR_PARAM;
    if (!aligned_type(x_dev, dtype) || !aligned_type(residual_dev, dtype) || !aligned_type(weight_dev, weight_dtype) || !aligned_type(h_dev, dtype) ||
        !aligned_type(y_dev, dtype) || !aligned_16(blob_dev) || !aligned_type(rstd_dev, DIV_F32))
        return DIV_ERR_ALIGN;
    const int fmt = blob_dev ? format : NORM_NONE;
    NormParams p;
    p.s = mx_shape((uint32_t)rows, (uint32_t)cols, blob_dev ? format : 0);
    if (blob_dev && blob_capacity < mx_codes_bytes(p.s) + mx_scales_bytes(p.s, format)) return DIV_ERR_CAPACITY;
    p.x = x_dev;
    p.residual = residual_dev;
    p.w = weight_dev;
    p.x_stride = (uint64_t)x_row_stride;
    p.r_stride = (uint64_t)residual_row_stride;
    p.rows = (uint32_t)rows;
    p.cols = (uint32_t)cols;
    p.eps = eps;
    p.h = h_dev;
    p.y = y_dev;
    p.rstd = rstd_dev;
    p.blob = (unsigned char*)blob_dev;
    const uint64_t pieces = blob_dev ? (uint64_t)p.s.stages * mx_stage(format) / 8u : ((uint64_t)cols + 7u) / 8u;
    const NormSplit s = norm_split(pieces, (uint64_t)rows);
    p.pieces = (uint32_t)pieces;
    p.group = s.group;
    const uint64_t per = s.threads / s.group, grid = ((uint64_t)rows + per - 1u) / per;
    const bool vec = cols % 8 == 0 && rows_vec(x_dev, rows, x_row_stride) && rows_vec(residual_dev, rows, residual_row_stride) && aligned_16(weight_dev) &&
                     aligned_16(h_dev) && aligned_16(y_dev);
    return norm_types(dtype, weight_dtype, [&](auto* x, auto* w) {
        typedef std::remove_pointer_t<decltype(x)> XT;
        typedef std::remove_pointer_t<decltype(w)> WT;
        const uint32_t g = (uint32_t)grid, t = s.threads;
        cudaStream_t st = (cudaStream_t)cuda_stream;
        if (s.held == 0) return vec ? norm_forward_launch<XT, WT, true, 0>(p, fmt, g, t, st) : norm_forward_launch<XT, WT, false, 0>(p, fmt, g, t, st);
        if (s.held == 1) return vec ? norm_forward_launch<XT, WT, true, 1>(p, fmt, g, t, st) : norm_forward_launch<XT, WT, false, 1>(p, fmt, g, t, st);
        if (s.held == 2) return vec ? norm_forward_launch<XT, WT, true, 2>(p, fmt, g, t, st) : norm_forward_launch<XT, WT, false, 2>(p, fmt, g, t, st);
        return vec ? norm_forward_launch<XT, WT, true, 4>(p, fmt, g, t, st) : norm_forward_launch<XT, WT, false, 4>(p, fmt, g, t, st);
    });
}

div_status div_rms_norm_workspace(int64_t rows, int64_t cols, uint64_t* out_bytes) {
    if (!out_bytes) return DIV_ERR_NULL;
    if (!lm_size_ok(rows) || !lm_size_ok(cols)) return DIV_ERR_SHAPE;
    *out_bytes = (uint64_t)norm_back(rows, cols).parts * (uint64_t)cols * 4u;
    return DIV_OK;
}

div_status div_rms_norm_backward(const void* dy_dev, int64_t dy_row_stride, const void* dh_dev, int64_t dh_row_stride, const void* h_dev,
                                 int64_t h_row_stride, const void* weight_dev, int32_t weight_dtype, const float* rstd_dev, int64_t rows, int64_t cols,
                                 int32_t dtype, void* dx_dev, void* dweight_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
    if (!dy_dev || !h_dev || !weight_dev || !rstd_dev || !dx_dev || (dweight_dev && !workspace_dev)) return DIV_ERR_NULL;
    if (!lm_size_ok(rows) || !lm_size_ok(cols) || (rows > 1 && (dy_row_stride < cols || h_row_stride < cols || (dh_dev && dh_row_stride < cols)))) return DIV_ERR_SHAPE;
    if (!lm_dtype_ok(dtype) || !(weight_dtype == dtype || weight_dtype == DIV_F32)) return DIV_ERR_PARAM;
    if (!aligned_type(dy_dev, dtype) || !aligned_type(dh_dev, dtype) || !aligned_type(h_dev, dtype) || !aligned_type(weight_dev, weight_dtype) ||
        !aligned_type(rstd_dev, DIV_F32) || !aligned_type(dx_dev, dtype) || !aligned_type(dweight_dev, weight_dtype) || !aligned_16(workspace_dev))
        return DIV_ERR_ALIGN;
    const NormBack b = norm_back(rows, cols);
    if (dweight_dev && workspace_bytes < (uint64_t)b.parts * (uint64_t)cols * 4u) return DIV_ERR_CAPACITY;
    NormBackParams p;
    p.dy = dy_dev;
    p.dh = dh_dev;
    p.h = h_dev;
    p.w = weight_dev;
    p.dy_stride = (uint64_t)dy_row_stride;
    p.dh_stride = (uint64_t)dh_row_stride;
    p.h_stride = (uint64_t)h_row_stride;
    p.rstd = rstd_dev;
    p.rows = (uint32_t)rows;
    p.cols = (uint32_t)cols;
    p.dx = dx_dev;
    p.sums = dweight_dev ? (float*)workspace_dev : nullptr;
    p.group = b.s.group;
    const bool vec = cols % 8 == 0 && rows_vec(dy_dev, rows, dy_row_stride) && rows_vec(dh_dev, rows, dh_row_stride) && rows_vec(h_dev, rows, h_row_stride) &&
                     aligned_16(weight_dev) && aligned_16(dx_dev);
    return norm_types(dtype, weight_dtype, [&](auto* x, auto* w) {
        typedef std::remove_pointer_t<decltype(x)> XT;
        typedef std::remove_pointer_t<decltype(w)> WT;
        cudaStream_t st = (cudaStream_t)cuda_stream;
        void (*kern)(const NormBackParams);
        if (b.s.held == 0) kern = vec ? norm_backward_kernel<XT, WT, true, 0, 512> : norm_backward_kernel<XT, WT, false, 0, 512>;
        else if (b.s.held == 1) kern = vec ? norm_backward_kernel<XT, WT, true, 1, 512> : norm_backward_kernel<XT, WT, false, 1, 512>;
        else if (b.s.threads <= 256) kern = vec ? norm_backward_kernel<XT, WT, true, 2, 256> : norm_backward_kernel<XT, WT, false, 2, 256>;
        else if (b.s.threads <= 320) kern = vec ? norm_backward_kernel<XT, WT, true, 2, 320> : norm_backward_kernel<XT, WT, false, 2, 320>;
        else kern = vec ? norm_backward_kernel<XT, WT, true, 2, 512> : norm_backward_kernel<XT, WT, false, 2, 512>;
        const div_status got = launch_pdl(kern, dim3(b.grid), b.s.threads, 0, st, p);
        if (got != DIV_OK || !dweight_dev) return got;
        return launch_pdl(norm_weight_kernel<WT>, dim3((uint32_t)(((uint64_t)cols + 31u) / 32u)), 1024, 0, st, (const float*)workspace_dev, b.parts,
                          (uint32_t)cols, (WT*)dweight_dev);
    });
}

}  // extern "C"
