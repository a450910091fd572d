// Microscaled operands: where codes and scales of a matrix lie in its blob, and how a block of 32 numbers becomes codes.
//
// A blob holds a matrix of `rows` x `cols` whose rows are cut into blocks of 32 neighbours.  Block b of a row has the scale
// 2^(e - 127), e one byte, and 32 codes, e4m3 (one byte) or e2m1 (half a byte, the first of two in the lower half).
//
//   scale   the smallest power of two with which the block's largest magnitude does not pass the largest number of the
//           format (448 or 6), between 2^-127 and 2^127: nothing is clipped.  A block that holds an infinity or a NaN has
//           the scale byte 255, which stands for NaN, and codes 0.
//   code    value / scale, rounded to nearest, ties to even.  The division is a product with a power of two, so that it is
//           exact but for what lies far below the smallest code: quantising rounds once.
//
// The layout is the one that the product's matrix instruction wants in shared memory, so that a product brings its operands
// with plain copies of whole tiles:
//   codes   K-STAGES of 128 bytes of each row (128 numbers of e4m3, 256 of e2m1).  For each 128 rows, for each stage: a tile of
//           up to 128 rows x 128 bytes, its 16-byte pieces permuted within a row (piece c of row r at c ^ (r mod 8)).  The last
//           tile of each stage is as high as its rows, rounded up to 8.
//   scales  for each 128 rows, for each stage: one ATOM of 512 bytes for each 128 numbers (1 with e4m3, 2 with e2m1).  Byte
//           k of row r, k the block's number among its 4: 16 * (r mod 32) + 4 * (r / 32) + k.
// The columns behind `cols` up to a whole stage hold codes 0 and finite scales.  What lies behind the last row is unspecified.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include <atomic>

#include "../../include/division.h"
#include "fused.cuh"

namespace divk {

constexpr int MX_E4M3 = 0, MX_E2M1 = 1;
template <int FMT> struct MxFormat;
template <> struct MxFormat<MX_E4M3> {
    static constexpr uint32_t STAGE = 128, ATOMS = 1, BLOCK_BYTES = 32;   // numbers of a row in a stage; atoms of scales for it
};
template <> struct MxFormat<MX_E2M1> {
    static constexpr uint32_t STAGE = 256, ATOMS = 2, BLOCK_BYTES = 16;
};
__host__ __device__ inline uint32_t mx_stage(int fmt) { return fmt == MX_E4M3 ? 128u : 256u; }

// a blob's geometry; sizes fit 64 bits for any rows, cols < 2^31
struct MxShape {
    uint32_t rows, cols, stages;      // stages: of a row
};
__host__ __device__ inline MxShape mx_shape(uint32_t rows, uint32_t cols, int fmt) {
    return {rows, cols, (cols + mx_stage(fmt) - 1u) / mx_stage(fmt)};
}
__host__ __device__ inline uint64_t mx_codes_bytes(const MxShape& s) { return (uint64_t)((s.rows + 7u) / 8u) * 1024u * s.stages; }
__host__ __device__ inline uint64_t mx_scales_bytes(const MxShape& s, int fmt) {
    return (uint64_t)((s.rows + 127u) / 128u) * s.stages * (fmt == MX_E4M3 ? 512u : 1024u);
}
// height of the tiles of 128 rows number `rb`, and where the tile of a stage begins
__host__ __device__ inline uint32_t mx_tile_rows(const MxShape& s, uint32_t rb) {
    const uint32_t left = (s.rows + 7u) / 8u * 8u - rb * 128u;
    return left < 128u ? left : 128u;
}
__host__ __device__ inline uint64_t mx_tile_offset(const MxShape& s, uint32_t rb, uint32_t stage) {
    return (uint64_t)rb * s.stages * 16384u + (uint64_t)stage * mx_tile_rows(s, rb) * 128u;
}
// 16-byte piece c (0..7) of row r of a tile
__host__ __device__ inline uint32_t mx_piece(uint32_t r, uint32_t c) { return r * 128u + ((c ^ (r & 7u)) << 4); }
__host__ __device__ inline uint32_t mx_scale_slot(uint32_t r) { return (r & 31u) * 16u + ((r >> 5) & 3u) * 4u; }

// scale byte from the bits of the block's largest magnitude (a float's bits without the sign order like the magnitudes,
// infinities and NaNs above all)
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t largest) {
    if (largest >= 0x7F800000u) return 255u;
    // 448 = 1.75 * 2^8, 6 = 1.5 * 2^2: one power more where the fraction passes that of the largest number
    const int e = (int)(largest >> 23), f = (int)(largest & 0x7FFFFFu);
    const int s = FMT == MX_E4M3 ? e - 8 + (f > 0x600000) : e - 2 + (f > 0x400000);
    return s < 0 ? 0u : (uint32_t)s;
}
__device__ __forceinline__ float mx_inverse(uint32_t scale_byte) {       // 1 / scale, a normal number for 0..253; 0 for NaN blocks
    return scale_byte == 255u ? 0.f : __uint_as_float((254u - scale_byte) << 23);
}
__device__ __forceinline__ float mx_scale(uint32_t scale_byte) {
    return scale_byte == 255u ? __uint_as_float(0x7FC00000u) : scale_byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(scale_byte << 23);
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// codes of N (4 or 8) numbers that are already divided by the scale
__device__ __forceinline__ uint32_t mx_codes4_e4m3(float a, float b, float c, float d) {
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3) << 16;
}
__device__ __forceinline__ uint32_t mx_codes2_e2m1(float a, float b) { return __nv_cvt_float2_to_fp4x2(make_float2(a, b), __NV_E2M1, cudaRoundNearest); }
// 8 numbers -> 8 bytes (e4m3) or 4 bytes in .x (e2m1); a NaN block's numbers are all 0 here
template <int FMT>
__device__ __forceinline__ uint2 mx_codes8(const float (&v)[8], float inverse) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = inverse == 0.f ? 0.f : __fmul_rn(v[i], inverse);
    if (FMT == MX_E4M3) return make_uint2(mx_codes4_e4m3(t[0], t[1], t[2], t[3]), mx_codes4_e4m3(t[4], t[5], t[6], t[7]));
    return make_uint2(mx_codes2_e2m1(t[0], t[1]) | mx_codes2_e2m1(t[2], t[3]) << 8 | mx_codes2_e2m1(t[4], t[5]) << 16 | mx_codes2_e2m1(t[6], t[7]) << 24, 0u);
}

// ---------------------------------------------------------------------------------------------
// 8 neighbours of a row in 32 bits
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <typename T> struct Row8;          // raw: 8 numbers as they are in memory
template <> struct Row8<float> {
    uint4 a, b;
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        a = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        b = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    }
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const uint4*>(p);
        b = *(reinterpret_cast<const uint4*>(p) + 1);
    }
    __device__ __forceinline__ void store(float* p) const {
        *reinterpret_cast<uint4*>(p) = a;
        *(reinterpret_cast<uint4*>(p) + 1) = b;
    }
};
template <typename T> struct Row8 {          // the 16-bit types
    uint4 a;
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = to_f32(bits<T>(w[i] & 0xFFFFu));
            v[2 * i + 1] = to_f32(bits<T>(w[i] >> 16));
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = word(from_f32<T>(v[2 * i])) | word(from_f32<T>(v[2 * i + 1])) << 16;
        a = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void load(const T* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = a; }

   private:
    template <typename U> static __device__ __forceinline__ U bits(uint32_t v) {
        const unsigned short h = (unsigned short)v;
        return *reinterpret_cast<const U*>(&h);
    }
    static __device__ __forceinline__ uint32_t word(T v) { return *reinterpret_cast<const unsigned short*>(&v); }
};
// the same where rows need not begin at a multiple of 16 bytes, or end inside the 8: what is behind `left` is 0
template <typename T>
__device__ __forceinline__ void load8_any(const T* p, uint32_t left, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (uint32_t)i < left ? to_f32(p[i]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store8_any(T* p, uint32_t left, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if ((uint32_t)i < left) p[i] = from_f32<T>(v[i]);
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
inline bool aligned_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool lm_dtype_ok(int32_t t) { return t == DIV_F32 || t == DIV_BF16 || t == DIV_F16; }
inline uint32_t lm_dtype_bytes(int32_t t) { return t == DIV_F32 ? 4u : 2u; }
// a kernel's leave to use more than 48 KB of shared memory, asked for once on each device
struct SmemAllowed {
    std::atomic<uint64_t> devices{0};
    bool operator()(const void* kern, uint32_t bytes) {
        int device = 0;
        if (cudaGetDevice(&device) != cudaSuccess) return false;
        const uint64_t bit = device < 64 ? 1ull << device : 0u;
        if (devices.load(std::memory_order_acquire) & bit) return true;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) {
            cudaGetLastError();
            return false;
        }
        devices.fetch_or(bit, std::memory_order_release);
        return true;
    }
};
inline bool mx_format_ok(int32_t f) { return f == MX_E4M3 || f == MX_E2M1; }
inline bool lm_size_ok(int64_t v) { return v >= 1 && v < (1ll << 31) - 512; }
template <typename F>
div_status with_type(int32_t dtype, F&& f) {
    if (dtype == DIV_F32) return f((float*)nullptr);
    if (dtype == DIV_BF16) return f((__nv_bfloat16*)nullptr);
    return f((__half*)nullptr);
}
__host__ __device__ inline uint64_t mx_scales_at(const MxShape& s) { return mx_codes_bytes(s); }       // (a multiple of 1024)

}  // namespace divk
