// Microscaled operands: where codes and scales of a matrix lie in its blob, and how a block of 32 numbers becomes codes.
//
// A blob holds a matrix of `rows` x `cols` whose rows are cut into blocks of 32 neighbours.  Block b of a row has the scale
// 2^(e - 127), e one byte, and 32 codes, e4m3 (one byte) or e2m1 (half a byte, the first of two in the lower half).
//
//   scale   the smallest power of two with which the block's largest magnitude does not pass the largest number of the
//           format (448 or 6), between 2^-127 and 2^127: nothing is clipped.  A block that holds an infinity or a NaN has
//           the scale byte 255, which stands for NaN, and any codes.
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
    static constexpr uint32_t STAGE = 128, ATOMS = 1;   // numbers of a row in a stage; atoms of scales for it
};
template <> struct MxFormat<MX_E2M1> {
    static constexpr uint32_t STAGE = 256, ATOMS = 2;
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
__device__ __forceinline__ float mx_inverse(uint32_t scale_byte) {       // 1 / scale, a normal number for 0..253; anything for NaN blocks
    return __uint_as_float((254u - scale_byte) << 23);
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
// two products at once
__device__ __forceinline__ float2 times(float a, float b, float f) {
    uint64_t v, g;
    float2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    asm("mov.b64 %0, {%1, %1};" : "=l"(g) : "f"(f));
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(v), "l"(g));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
// 8 numbers -> 8 bytes (e4m3) or 4 bytes in .x (e2m1)
template <int FMT>
__device__ __forceinline__ uint2 mx_codes8(const float (&v)[8], float inverse) {
    float2 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = times(v[2 * i], v[2 * i + 1], inverse);
    if (FMT == MX_E4M3) return make_uint2(mx_codes4_e4m3(t[0].x, t[0].y, t[1].x, t[1].y), mx_codes4_e4m3(t[2].x, t[2].y, t[3].x, t[3].y));
    return make_uint2(mx_codes2_e2m1(t[0].x, t[0].y) | mx_codes2_e2m1(t[1].x, t[1].y) << 8 | mx_codes2_e2m1(t[2].x, t[2].y) << 16 |
                          mx_codes2_e2m1(t[3].x, t[3].y) << 24, 0u);
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

// the larger magnitude of each half of two words, a NaN above all
template <typename T> __device__ __forceinline__ uint32_t larger_of_each(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t larger_of_each<__nv_bfloat16>(uint32_t a, uint32_t b) {
    const __nv_bfloat162 m = __hmax2_nan(__habs2(*reinterpret_cast<const __nv_bfloat162*>(&a)), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&m);
}
template <> __device__ __forceinline__ uint32_t larger_of_each<__half>(uint32_t a, uint32_t b) {
    const __half2 m = __hmax2_nan(__habs2(*reinterpret_cast<const __half2*>(&a)), __habs2(*reinterpret_cast<const __half2*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&m);
}
template <typename T> __device__ __forceinline__ float half_of(uint32_t w, uint32_t which) {
    const unsigned short h = (unsigned short)(w >> (16u * which));
    return to_f32(*reinterpret_cast<const T*>(&h));
}
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
// Rows that do not begin at multiples of 16 bytes, by whole 16-byte units all the same: a unit of the row is cut from two aligned ones.
// (Number by number a warp's store touches 16 sectors for 64 bytes: the norm of 2000 x 4097 bf16 took 41 us that way, its backward 71; by units 30 and 51.)
// ---------------------------------------------------------------------------------------------
template <typename T> struct Units {
    static constexpr uint32_t E = 16u / sizeof(T);                 // numbers of a unit
    static __device__ __forceinline__ uint32_t offset(const T* p) { return (uint32_t)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T)); }
    // E numbers of a and b, one behind the other, from number s (< E) on
    static __device__ __forceinline__ uint4 cut(const uint4& a, const uint4& b, uint32_t s) {
        const uint32_t words = sizeof(T) == 4 ? s : s >> 1;
        uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        if (words & 2u) {
#pragma unroll
            for (int i = 0; i < 6; ++i) x[i] = x[i + 2];
        }
        if (words & 1u) {
#pragma unroll
            for (int i = 0; i < 6; ++i) x[i] = x[i + 1];
        }
        if (sizeof(T) == 2 && (s & 1u)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __funnelshift_r(x[i], x[i + 1], 16);
        }
        return make_uint4(x[0], x[1], x[2], x[3]);
    }
    static __device__ __forceinline__ T number(const uint4& q, uint32_t i) {        // (i known when compiled)
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        if (sizeof(T) == 4) return *reinterpret_cast<const T*>(&w[i & 3u]);
        const unsigned short h = (unsigned short)(w[(i >> 1) & 3u] >> (16u * (i & 1u)));
        return *reinterpret_cast<const T*>(&h);
    }
    // numbers [lo, hi) of a unit, one by one
    static __device__ __forceinline__ void put(T* p, const uint4& q, uint32_t lo, uint32_t hi) {
#pragma unroll
        for (uint32_t i = 0; i < E; ++i)
            if (i >= lo && i < hi) p[i] = number(q, i);
    }
    // N units from p on, of which `left` numbers are there (the rest: 0), in two steps, so that many reads can be under way together:
    // ask() reads the aligned units that they lie in, take() cuts them out.  The matrix lies between `begin` and `end`: nothing outside is
    // read (a row's neighbours may be); what lies at its own two ends ask() reads number by number.
    template <int N> static __device__ __forceinline__ bool inside(const T* p, const T* begin, const T* end) {
        const uint32_t o = offset(p);
        return p - o >= begin && p - o + (o ? N + 1 : N) * E <= end;
    }
    template <typename F> static __device__ __forceinline__ uint4 made(F&& number_at) {        // of numbers 0 .. E-1, as words
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (uint32_t i = 0; i < E; ++i) {
            const T v = number_at(i);
            if (sizeof(T) == 4) w[i & 3u] = *reinterpret_cast<const uint32_t*>(&v);
            else w[(i >> 1) & 3u] |= (uint32_t)*reinterpret_cast<const unsigned short*>(&v) << (16u * (i & 1u));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    template <int N> static __device__ __forceinline__ void ask(const T* p, const T* begin, const T* end, uint32_t left, uint4 (&a)[N + 1]) {
        const uint32_t o = offset(p);
        const uint4* at = reinterpret_cast<const uint4*>(p - o);
        const bool in = inside<N>(p, begin, end);
#pragma unroll
        for (int u = 0; u <= N; ++u) {
            a[u] = make_uint4(0u, 0u, 0u, 0u);
            if (left != 0u && in && (u < N || o != 0u)) a[u] = at[u];
        }
        if (left != 0u && !in) {
#pragma unroll
            for (uint32_t u = 0; u < N; ++u) a[u] = made([&](uint32_t i) { return u * E + i < left ? p[u * E + i] : from_f32<T>(0.f); });
        }
    }
    template <int N> static __device__ __forceinline__ void take(const T* p, const T* begin, const T* end, uint32_t left, const uint4 (&a)[N + 1], uint4 (&q)[N]) {
        const uint32_t o = inside<N>(p, begin, end) ? offset(p) : 0u;
#pragma unroll
        for (int u = 0; u < N; ++u) q[u] = cut(a[u], a[u + 1], o);
        if (left < N * E) {
#pragma unroll
            for (uint32_t u = 0; u < N; ++u) {
                const uint4 whole = q[u];
                q[u] = made([&](uint32_t i) { return u * E + i < left ? number(whole, i) : from_f32<T>(0.f); });
            }
        }
    }
    // the first n (< E) numbers of a unit to p, a multiple of 16 bytes; the last n to where p ends, another: in stores of 8, 4 and 2 bytes
    static __device__ __forceinline__ void put_first(T* p, const uint4& q, uint32_t n) {
        uint32_t words = n, at = 0;
        if (sizeof(T) == 2) words = n >> 1;
        uint32_t* w = reinterpret_cast<uint32_t*>(p);
        if (words & 2u) {
            *reinterpret_cast<uint2*>(w) = make_uint2(q.x, q.y);
            at = 2;
        }
        if (words & 1u) w[at] = at ? q.z : q.x;
        if (sizeof(T) == 2 && (n & 1u)) {
            const uint32_t last = words == 0u ? q.x : words == 1u ? q.y : words == 2u ? q.z : q.w;
            reinterpret_cast<unsigned short*>(p)[n - 1u] = (unsigned short)last;
        }
    }
    static __device__ __forceinline__ void put_last(T* end, const uint4& q, uint32_t n) {        // numbers 0 .. n-1 of q
        const uint4 none = make_uint4(0u, 0u, 0u, 0u);
        T* p = end - n;
        if (sizeof(T) == 2 && (n & 1u)) *reinterpret_cast<unsigned short*>(p) = (unsigned short)q.x;
        const uint32_t odd = sizeof(T) == 2 ? n & 1u : 0u, one = sizeof(T) == 2 ? 2u : 1u;         // numbers of a word
        if (n & one) *reinterpret_cast<uint32_t*>(p + odd) = cut(q, none, odd).x;
        if (n & (2u * one)) {
            const uint4 r = cut(q, none, n & (2u * one - 1u));
            *reinterpret_cast<uint2*>(p + (n & (2u * one - 1u))) = make_uint2(r.x, r.y);
        }
    }
    // N units to p on, of which `left` numbers are wanted (0: none).  All lanes of the warp together; a lane's successor holds what
    // follows in the same row, unless it is the `last` of its run (`first`: no lane before it does so).
    template <int N>
    static __device__ __forceinline__ void store(T* p, uint32_t left, const uint4 (&own)[N], bool first, bool last) {
        uint4 next;
        next.x = __shfl_down_sync(0xFFFFFFFFu, own[0].x, 1);
        next.y = __shfl_down_sync(0xFFFFFFFFu, own[0].y, 1);
        next.z = __shfl_down_sync(0xFFFFFFFFu, own[0].z, 1);
        next.w = __shfl_down_sync(0xFFFFFFFFu, own[0].w, 1);
        uint32_t left_next = __shfl_down_sync(0xFFFFFFFFu, left, 1);
        if (last) left_next = 0u;
        const uint32_t o = offset(p), s = o ? E - o : 0u;             // numbers before the first aligned unit
        const bool joins = left >= N * E && left_next >= s;           // the last unit, with the next lane's first s numbers
        bool joined = __shfl_up_sync(0xFFFFFFFFu, joins ? 1 : 0, 1) != 0;
        if (first) joined = false;
        if (left == 0u) return;
        if (!joined) {
            if (left >= s) put_last(p + s, own[0], s);
            else put(p, own[0], 0u, left);
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const bool whole = u < N - 1 ? left >= (u + 1u) * E + s : joins;
            if (whole) {
                *reinterpret_cast<uint4*>(p + s + u * E) = cut(own[u], u < N - 1 ? own[u + 1 < N ? u + 1 : u] : next, s);
            } else if (u == N - 1 && left >= N * E) {
                put_first(p + s + u * E, cut(own[u], make_uint4(0u, 0u, 0u, 0u), s), E - s);
            } else if (left > u * E) {
                put(p + u * E, own[u], s, left - u * E);
                if (u < N - 1 && left > (u + 1u) * E) put(p + (u + 1u) * E, own[u + 1 < N ? u + 1 : u], 0u, min(s, left - (u + 1u) * E));
            }
        }
    }
};
// Row8 <-> units
template <typename T> struct Raw8 { static constexpr int N = sizeof(T) == 4 ? 2 : 1; };
__device__ __forceinline__ void to_units(const Row8<float>& r, uint4 (&q)[2]) { q[0] = r.a, q[1] = r.b; }
template <typename T> __device__ __forceinline__ void to_units(const Row8<T>& r, uint4 (&q)[1]) { q[0] = r.a; }
__device__ __forceinline__ void from_units(const uint4 (&q)[2], Row8<float>& r) { r.a = q[0], r.b = q[1]; }
template <typename T> __device__ __forceinline__ void from_units(const uint4 (&q)[1], Row8<T>& r) { r.a = q[0]; }
// a matrix to read from: where it begins and ends, numbers between two rows
template <typename T> struct Rows {
    const T *begin, *end;
    uint64_t stride;
    __device__ __forceinline__ Rows(const void* x, uint32_t rows, uint32_t cols, uint64_t s)
        : begin(static_cast<const T*>(x)), end(static_cast<const T*>(x) + (rows - 1u) * s + cols), stride(s) {}
};
// 8 numbers of a row on their way; VEC: they begin at a multiple of 16 bytes and are all there (or none is)
template <typename T, bool VEC> struct Asked8 {
    static constexpr int N = Raw8<T>::N;
    uint4 a[VEC ? N : N + 1];
    __device__ __forceinline__ void ask(const Rows<T>& m, uint64_t row, uint32_t at, uint32_t left) {
        const T* p = m.begin + (left ? row * m.stride + at * 8u : 0u);
        if constexpr (VEC) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                a[u] = make_uint4(0u, 0u, 0u, 0u);
                if (left) a[u] = reinterpret_cast<const uint4*>(p)[u];
            }
        } else {
            Units<T>::template ask<N>(p, m.begin, m.end, left, a);
        }
    }
    __device__ __forceinline__ void take(const Rows<T>& m, uint64_t row, uint32_t at, uint32_t left, Row8<T>& r) const {
        if constexpr (VEC) {
            from_units(a, r);
        } else {
            uint4 q[N];
            Units<T>::template take<N>(m.begin + (left ? row * m.stride + at * 8u : 0u), m.begin, m.end, left, a, q);
            from_units(q, r);
        }
    }
    __device__ __forceinline__ void take(const Rows<T>& m, uint64_t row, uint32_t at, uint32_t left, float (&v)[8]) const {
        Row8<T> r;
        take(m, row, at, left, r);
        r.get(v);
    }
};
// all lanes of the warp together, each with the 8 numbers behind its predecessor's
template <typename T>
__device__ __forceinline__ void store8_row(T* p, uint32_t left, const float (&v)[8]) {
    Row8<T> r;
    r.set(v);
    uint4 q[Raw8<T>::N];
    to_units(r, q);
    Units<T>::store(p, left, q, (threadIdx.x & 31u) == 0u, (threadIdx.x & 31u) == 31u);
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
