// Chunks of eight consecutive values of a row, as the operators' kernels read and write them: from fp32, bf16, or 8 bits with
// scales.  Four lanes with four neighbouring chunks hold one group of 32 values of a matrix in 8 bits.
#pragma once
#include "device_helpers.h"
#include "operators_internal.h"

namespace lf {
namespace ops {

constexpr int kGroup = 32;        // values that share a scale
constexpr int kBlock = 128;       // the same, in blocks of 128
constexpr int kChunk = 8;

typedef unsigned int v2u __attribute__((ext_vector_type(2)));

template <int KIND> struct Stored;
template <> struct Stored<F32> { typedef float type; };
template <> struct Stored<BF16> { typedef __bf16 type; };

template <class T> using global_ptr = T __attribute__((address_space(1)))*;
template <class T, class U> __device__ __forceinline__ global_ptr<T> as_global(U* p) { return (global_ptr<T>)(p); }

// Vectors at any address of their elements: global memory takes wide loads and stores that are not aligned to their
// width, so one instruction serves aligned rows and others (which cost the lines they straddle).  The alignment is part of the
// typedef, which a template's argument loses: these pointers are no template's.  (Of a load that it takes for aligned the compiler
// makes a scalar one where the address is the same for a whole wave, and that leaves out the address's last two bits.)
typedef v4f any_v4f __attribute__((aligned(4)));
typedef v8bf any_v8bf __attribute__((aligned(2)));
typedef __attribute__((address_space(1))) any_v4f* any_v4f_ptr;
typedef __attribute__((address_space(1))) any_v8bf* any_v8bf_ptr;
__device__ __forceinline__ v4f load_vector(const float* p) { return *(any_v4f_ptr)(const_cast<float*>(p)); }
__device__ __forceinline__ v8bf load_vector(const __bf16* p) { return *(any_v8bf_ptr)(const_cast<__bf16*>(p)); }
__device__ __forceinline__ void store_vector(float* p, v4f v) { *(any_v4f_ptr)(p) = v; }
__device__ __forceinline__ void store_vector(__bf16* p, v8bf v) { *(any_v8bf_ptr)(p) = v; }

// n (0..8) values from p; the others are zero.
template <class T>
__device__ __forceinline__ void load_values(const T* p, int n, float (&v)[8]) {
    if (n >= kChunk) {
        if constexpr (sizeof(T) == 4) {
            const v4f a = load_vector(p), b = load_vector(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        } else {
            const v8bf a = load_vector(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)*as_global<const T>(p + i) : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void store_values(T* p, int n, const float (&v)[8]) {
    if (n >= kChunk) {
        if constexpr (sizeof(T) == 4) {
            store_vector(p, v4f{v[0], v[1], v[2], v[3]});
            store_vector(p + 4, v4f{v[4], v[5], v[6], v[7]});
        } else {
            v8bf a;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = (__bf16)v[i];
            store_vector(p, a);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) *as_global<T>(p + i) = (T)v[i];
    }
}

// ---- 8 bits ----------------------------------------------------------------------------------------------------------
// The scale of a group whose largest finite magnitude is m, as e + 127: the least e >= -117 with m <= 448 2^e.  448 is 1.75 2^8,
// so e is m's exponent less 8, one more if its significand is above 1.75: the addition carries into the exponent then.
__device__ __forceinline__ int scale_byte(float m) {
    const int e = (int)((__float_as_uint(m) + 0x1FFFFFu) >> 23) - 8;
    return e < 10 ? 10 : e;
}
// 2^(byte - 127) of bytes from 1 to 254, and a number whose exponent says so of the two others.
__device__ __forceinline__ float scale_power(int byte) { return __uint_as_float((unsigned)byte << 23); }
// What any byte stands for.  This library writes 10 to 247; others' matrices may have 0, 2^-127, which is a number below the
// normal ones, and 255, a NaN: of both the leading bit of the significand is set.
__device__ __forceinline__ float scale_value(int byte) {
    return __uint_as_float((unsigned)byte << 23 | ((byte + 1) & 0xFE ? 0u : 0x400000u));
}
__device__ __forceinline__ float finite_magnitude(float v) {
    const float a = fabsf(v);
    return a < __builtin_inff() ? a : 0.0f;
}
// Largest of the four lanes of a quad (all of them active).
__device__ __forceinline__ unsigned quad_max(unsigned m) {
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));
    return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));
}
// Largest of the 16 lanes of a row of lanes (all of them active).
__device__ __forceinline__ unsigned sixteen_max(unsigned m) {
    m = quad_max(m);
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xF, 0xF, true));
    return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xF, 0xF, true));
}
// Largest among the lanes that hold a group's chunks, four of 32 columns or sixteen of 128.
template <int KIND> __device__ __forceinline__ unsigned group_max(unsigned m) { return KIND == E4M3 ? quad_max(m) : sixteen_max(m); }
template <int KIND> constexpr int kGroupOf = KIND == E4M3 ? kGroup : kBlock;
__device__ __forceinline__ v2u convert_eight(const float (&v)[8]) {
    int w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], w[h], true);
    }
    return v2u{(unsigned)w[0], (unsigned)w[1]};
}
constexpr int kLargestScale = 247;          // of the largest finite numbers
// Codes (rounded to nearest even) and scale of a group's chunk.  The largest of the values' bits without their signs tells what
// the group holds: with every value finite and a scale below the largest no product with the scale's reciprocal passes
// 448 and there is nothing to look at value by value, which would take twice the instructions.
template <int KIND = E4M3>
__device__ __forceinline__ v2u eight_codes(const float (&v)[8], int& byte) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    byte = scale_byte(__uint_as_float(group_max<KIND>(top)));
    float s[8];
    if (byte < kLargestScale) {
        const float inverse = scale_power(254 - byte);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = v[i] * inverse;
    } else {
        unsigned finite = 0;                  // NaN and infinities do not set a scale
#pragma unroll
        for (int i = 0; i < 8; ++i) finite = max(finite, __float_as_uint(finite_magnitude(v[i])));
        byte = scale_byte(__uint_as_float(group_max<KIND>(finite)));
        const float inverse = scale_power(254 - byte);
        const float most = byte == kLargestScale ? 240.0f : 448.0f;      // 256 * 2^120 would be no finite number
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = fminf(fmaxf(v[i] * inverse, -most), most);
            s[i] = fabsf(v[i]) < __builtin_inff() ? a : __builtin_nanf("");
        }
    }
    return convert_eight(s);
}
// Chunk `col` (a multiple of 8) of a row in 8 bits.  Neighbouring lanes (four, or sixteen of blocks of 128) hold the chunks of a group and
// all call this; values past the last column are zero.  live: the chunk's group begins inside the row, so its memory is there.
template <int KIND = E4M3>
__device__ __forceinline__ void store_eight(uint8_t* codes, uint8_t* scales, int col, const float (&v)[8], bool live) {
    int byte;
    const v2u w = eight_codes<KIND>(v, byte);
    if (live) {
        *as_global<v2u>(codes + col) = w;
        if (col % kGroupOf<KIND> == 0) *as_global<uint8_t>(scales + col / kGroupOf<KIND>) = (uint8_t)byte;
    }
}
// The values of eight codes.
__device__ __forceinline__ void eight_values(v2u w, float scale, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
        v[4 * h] = a[0] * scale;
        v[4 * h + 1] = a[1] * scale;
        v[4 * h + 2] = b[0] * scale;
        v[4 * h + 3] = b[1] * scale;
    }
}

// ---- chunks on their way --------------------------------------------------------------------------------------------------
// Elements move down by s places (s >= 8: zeros).
__device__ __forceinline__ void shift_down(v4u& a, int s) {                 // eight of 16 bits
    v4u b = (s & 4) ? v4u{a[2], a[3], 0u, 0u} : a;
    b = (s & 2) ? v4u{b[1], b[2], b[3], 0u} : b;
    const v4u h = {b[0] >> 16 | b[1] << 16, b[1] >> 16 | b[2] << 16, b[2] >> 16 | b[3] << 16, b[3] >> 16};
    b = (s & 1) ? h : b;
    a = s < 8 ? b : v4u{0u, 0u, 0u, 0u};
}
__device__ __forceinline__ void shift_down(v4f& a, int s) {                 // four of 32 bits
    v4f b = (s & 2) ? v4f{a[2], a[3], 0.0f, 0.0f} : a;
    b = (s & 1) ? v4f{b[1], b[2], b[3], 0.0f} : b;
    a = s < 4 ? b : v4f{0.0f, 0.0f, 0.0f, 0.0f};
}
__device__ __forceinline__ void shift_down(v4f (&a)[2], int s) {            // eight of 32 bits
    const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
    if (s & 4) { a[0] = a[1]; a[1] = zero; }
    if (s & 2) { a[0] = v4f{a[0][2], a[0][3], a[1][0], a[1][1]}; a[1] = v4f{a[1][2], a[1][3], 0.0f, 0.0f}; }
    if (s & 1) { a[0] = v4f{a[0][1], a[0][2], a[0][3], a[1][0]}; a[1] = v4f{a[1][1], a[1][2], a[1][3], 0.0f}; }
    if (s >= 8) a[0] = a[1] = zero;
}
// The first n of the codes stay, the others become zeros.
template <class V>
__device__ __forceinline__ void keep_codes(V& a, int n) {
#pragma unroll
    for (int w = 0; w < (int)(sizeof(V) / 4); ++w) {
        const int k = n - 4 * w;
        a[w] &= k >= 4 ? ~0u : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
    }
}

// A chunk as it was loaded.  Loads have no branch around them, so that many are under way: a chunk that the row's end cuts is
// loaded from as far ahead as makes it whole, one past the end from the row's last eight, and both are put right when
// the values are taken.  That needs rows of eight values; NARROW is for fewer.
template <int KIND> struct Chunk;
template <> struct Chunk<F32> { v4f a[2]; };
template <> struct Chunk<BF16> { v4u a; };
template <> struct Chunk<E4M3> { v2u a; int byte; };
template <> struct Chunk<E4M3_128> { v2u a; int byte; };

// Chunk of the row (which is there) from column col on; cols: the matrix's columns.
template <int KIND, bool NARROW>
__device__ __forceinline__ void fetch_chunk(Chunk<KIND>& c, const Mat& m, long long row, int col, int cols) {
    if constexpr (KIND == E4M3 || KIND == E4M3_128) {
        constexpr int kOf = kGroupOf<KIND>;
        const int at = min(col, (cols - 1) / kOf * kOf + (kOf - kChunk));
        c.a = *as_global<const v2u>((const uint8_t*)m.p + row * m.ld + at);
        c.byte = *as_global<const uint8_t>(m.scales + row * m.scale_ld + at / kOf);
    } else {
        typedef typename Stored<KIND>::type T;
        const T* p = (const T*)m.p + row * m.ld;
        if constexpr (NARROW) {
            float v[8];
            load_values(p + col, max(0, cols - col), v);
            if constexpr (KIND == F32) {
                c.a[0] = v4f{v[0], v[1], v[2], v[3]};
                c.a[1] = v4f{v[4], v[5], v[6], v[7]};
            } else {
                v8bf b;
#pragma unroll
                for (int i = 0; i < 8; ++i) b[i] = (__bf16)v[i];
                c.a = __builtin_bit_cast(v4u, b);
            }
        } else {
            p += min(col, cols - kChunk);
            if constexpr (KIND == F32) {
                c.a[0] = load_vector(p);
                c.a[1] = load_vector(p + 4);
            } else {
                c.a = __builtin_bit_cast(v4u, load_vector(p));
            }
        }
    }
}
// Its values; n (0..8) of them are in the row, the others are zero.
template <int KIND, bool NARROW>
__device__ __forceinline__ void take_chunk(Chunk<KIND> c, int n, float (&v)[8]) {
    if constexpr (KIND != E4M3 && KIND != E4M3_128) {
        if (n < kChunk && (!NARROW || n <= 0)) shift_down(c.a, kChunk - max(n, 0));
    }
    if constexpr (KIND == E4M3 || KIND == E4M3_128) {
        eight_values(c.a, scale_value(c.byte), v);
        if (n < kChunk) {                                  // (the scale may be no number)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.0f;
        }
    } else if constexpr (KIND == F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = c.a[0][i]; v[4 + i] = c.a[1][i]; }
    } else {
        const v8bf b = __builtin_bit_cast(v8bf, c.a);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)b[i];
    }
}

// Values col .. col + n - 1 of a row (n <= 8; n <= 0: none), the others zero; col is a multiple of 8.
template <int KIND>
__device__ __forceinline__ void load_chunk(const Mat& m, long long row, int col, int n, float (&v)[8]) {
    if constexpr (KIND >= E4M3) {
        if (n > 0) {
            const v2u w = *as_global<const v2u>((const uint8_t*)m.p + row * m.ld + col);
            const long long scale_row = KIND == E4M3_TILES ? row / kBlock : row;
            eight_values(w, scale_value(*as_global<const uint8_t>(m.scales + scale_row * m.scale_ld + col / kGroupOf<KIND>)), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.0f;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        }
    } else {
        typedef typename Stored<KIND>::type T;
        load_values((const T*)m.p + row * m.ld + col, n, v);
    }
}
// All lanes call this (see store_eight); live: the row is there and col < the row's columns rounded up to whole groups.
template <int KIND>
__device__ __forceinline__ void store_chunk(const Mat& m, long long row, int col, int n, const float (&v)[8], bool live) {
    if constexpr (KIND == E4M3 || KIND == E4M3_128) {
        store_eight<KIND>((uint8_t*)m.p + row * m.ld, m.scales + row * m.scale_ld, col, v, live);
    } else {
        typedef typename Stored<KIND>::type T;
        if (live && n > 0) store_values((T*)m.p + row * m.ld + col, n, v);
    }
}

}  // namespace ops
}  // namespace lf
