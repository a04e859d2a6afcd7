// Chunks of 8 consecutive elements, as a lane of the row passes holds them: loaded, widened to
// binary32, their largest magnitude, and their E4M3 codes with a scale.
#pragma once
#include "cham_device.h"

namespace cham {
namespace {

constexpr int kChunk = 8;  // elements of a lane's chunk

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------------------------
// 8 elements in registers as they were loaded, and as binary32
// ------------------------------------------------------------------------------------
template <int T>
struct Raw {
    uint4 a;
};
template <>
struct Raw<CHAM_T_F32> {
    uint4 a, b;
};

template <int T>
CHAM_DEV const uint4* at8(const void* p, int64_t i) {  // i: element index, a multiple of 8
    return (const uint4*)((const char*)p + i * (T == CHAM_T_F32 ? 4 : 2));
}
template <int T>
CHAM_DEV Raw<T> load8(const void* p, int64_t i) {
    const uint4* q = at8<T>(p, i);
    Raw<T> r;
    r.a = q[0];
    if constexpr (T == CHAM_T_F32) r.b = q[1];
    return r;
}

CHAM_DEV float f16_lo(uint32_t w) { return (float)__builtin_bit_cast(half2v, w)[0]; }
CHAM_DEV float f16_hi(uint32_t w) { return (float)__builtin_bit_cast(half2v, w)[1]; }

template <int T>
CHAM_DEV void widen(const Raw<T>& r, float (&v)[kChunk]) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
    if constexpr (T == CHAM_T_F32) {
        const uint32_t q[4] = {r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = __uint_as_float(w[j]);
            v[4 + j] = __uint_as_float(q[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = T == CHAM_T_F16 ? f16_lo(w[j]) : __uint_as_float(w[j] << 16);
            v[2 * j + 1] = T == CHAM_T_F16 ? f16_hi(w[j]) : __uint_as_float(w[j] & 0xffff0000u);
        }
    }
}

template <int T>
CHAM_DEV void put8(void* p, int64_t i, const float (&v)[kChunk]) {
    uint4* q = (uint4*)at8<T>(p, i);
    if constexpr (T == CHAM_T_F32) {
        q[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        q[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    } else {
        *q = make_uint4(narrow<T>(v[0], v[1]), narrow<T>(v[2], v[3]), narrow<T>(v[4], v[5]), narrow<T>(v[6], v[7]));
    }
}

// The weights g of a chunk, of any type (the same for all rows: they stay in the caches).
CHAM_DEV void load_g(const void* g, int type, int64_t i, float (&v)[kChunk]) {
    if (type == CHAM_T_F32) widen<CHAM_T_F32>(load8<CHAM_T_F32>(g, i), v);
    else if (type == CHAM_T_F16) widen<CHAM_T_F16>(load8<CHAM_T_F16>(g, i), v);
    else widen<CHAM_T_BF16>(load8<CHAM_T_BF16>(g, i), v);
}

// ------------------------------------------------------------------------------------
// scales and codes of a chunk
// ------------------------------------------------------------------------------------
// Largest magnitude as bits: unsigned order puts NaN above infinity above the numbers.
CHAM_DEV uint32_t chunk_amax(const float (&y)[kChunk]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < kChunk; ++j) {
        const uint32_t b = __float_as_uint(y[j]) & 0x7fffffffu;
        m = m > b ? m : b;
    }
    return m;
}
template <int CTRL>
CHAM_DEV uint32_t dpp_maxu(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
    return v > o ? v : o;
}

constexpr uint32_t kInfBits = 0x7f800000u;

// a / 448, correctly rounded: the product with the reciprocal and one correction from the exact
// remainder (equal to the IEEE quotient for every mantissa, checked exhaustively; a tenth of the
// division's instructions).
CHAM_DEV float div448(float a) {
    constexpr float c = 1.0f / 448.0f;
    const float q = a * c;
    return __builtin_fmaf(__builtin_fmaf(-448.0f, q, a), c, q);
}

// The scale of a block of maximum m (bits): its reciprocal, and the value that is stored.  A
// finite scale lies in [2^-126, 2^120), where the corrected estimate is the IEEE reciprocal.
CHAM_DEV float block_scale(uint32_t m, bool pow2, uint32_t* stored) {
    float s = floor_scale(div448(__uint_as_float(m)));
    uint32_t u = __float_as_uint(s);
    if (pow2) {  // the exponent goes up where the mantissa is not zero
        u = (u + 0x7fffffu) & 0x7f800000u;
        s = __uint_as_float(u);
        u >>= 23;
    }
    const bool bad = m >= kInfBits;
    *stored = bad ? (pow2 ? 255u : 0x7fc00000u) : u;
    const float r = __builtin_amdgcn_rcpf(s);
    return __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r);
}

// E4M3 codes of y r.  No clamp is needed: r is the rounded reciprocal of amax / 448 rounded, so
// |y r| <= 448 (1 + 2^-22), which rounds to 448 (the next value of the grid would be 480).
CHAM_DEV uint2 codes8_e4m3(const float (&y)[kChunk], float r) {
    return make_uint2(pack_codes<CHAM_A_FP8_E4M3>(y[0] * r, y[1] * r, y[2] * r, y[3] * r, 0.0f),
                      pack_codes<CHAM_A_FP8_E4M3>(y[4] * r, y[5] * r, y[6] * r, y[7] * r, 0.0f));
}

// The values of 8 E4M3 codes (the gfx950 converter; every value is exact, NaN stays NaN).
CHAM_DEV void decode8_e4m3(uint2 w, float (&y)[kChunk]) {
    typedef float float2v __attribute__((ext_vector_type(2)));
    const float2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
    const float2v c = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
    y[0] = a[0], y[1] = a[1], y[2] = b[0], y[3] = b[1], y[4] = c[0], y[5] = c[1], y[6] = d[0], y[7] = d[1];
}

}  // namespace
}  // namespace cham
