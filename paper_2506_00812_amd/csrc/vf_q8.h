// Matrices in 8 bits: codes in OCP e4m3, and for each 128 columns of a row a scale 2^(byte - 127), which the matrix instruction applies by
// itself.  A row's codes are filled up with zeros to whole blocks of 128; its scale bytes lie in whole 32-bit words.
#pragma once

#include "vf_ops.h"

namespace vf {

constexpr int kBlock = 128;          // columns that share a scale
inline int64_t q8_width(int64_t cols) { return ceil_div(cols, kBlock) * kBlock; }

// The byte of the least scale under which a block's largest finite |value|, `most`, is at most 448 = 1.75 * 2^8: e with most <= 448 * 2^e, from the
// float's own exponent, one more where its significand is above 1.75.  Not less than 2^-127; 1 for a block of zeros.
__device__ __forceinline__ int scale_byte(float most)
{
    if (most == 0.f) return 127;
    return max(0, (int)((__float_as_uint(most) + 0x1FFFFFu) >> 23) - 8);
}
__device__ __forceinline__ float inverse_scale(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }   // byte <= 247: a normal number
__device__ __forceinline__ float scale_value(int byte)
{
    return __uint_as_float((uint32_t)byte << 23 | (((byte + 1) & 254) ? 0u : 0x400000u));   // 2^-127 is below the normal range, byte 255 NaN
}

// Eight values divided by their scale (exact: a power of two), to the nearest code, ties to even; what is not finite becomes NaN.
__device__ __forceinline__ uint2 encode8(const float (&v)[8], float inverse)
{
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse, v[1] * inverse, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse, v[3] * inverse, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inverse, v[5] * inverse, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inverse, v[7] * inverse, hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}
__device__ __forceinline__ float finite_size(float v)
{
    const float a = fabsf(v);
    return a <= kFltMax ? a : 0.f;
}
__device__ __forceinline__ float most_of8(const float (&v)[8])
{
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(v[j]));   // (passes over NaN)
    if (most > kFltMax) {   // only what is finite counts
        most = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, finite_size(v[j]));
    }
    return most;
}
// Sixteen neighbouring lanes have a block, eight columns each (zeros beyond the row): their codes, and from the first lane the scale.
__device__ __forceinline__ void keep_block(const float (&v)[8], uint8_t *codes, uint8_t *scale)
{
    const int byte = scale_byte(max16(most_of8(v)));
    const uint2 c = encode8(v, inverse_scale(byte));
    store_vec(codes, c);
    if ((threadIdx.x & 15) == 0) *scale = (uint8_t)byte;
}

// Eight neighbours of a row as float32, n of which exist; the others are `fill`.  A part of them comes as four, two and one, the last of them first.
template <class T> __device__ __forceinline__ void load8(const T *p, int n, float (&v)[8], float fill = 0.f)
{
    if (n >= 8) {
        constexpr int V = kVec<T>;
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            const Vec<T> u = load_vec<Vec<T>>(p + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) v[i * V + j] = (float)u[j];
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = fill;
    if (n <= 0) return;
    auto some = [&](auto count) {
        constexpr int N = count.value;
        using S = T __attribute__((ext_vector_type(N)));
        if (n & N) {
            const S u = load_vec<S>(p + (n & ~(2 * N - 1)));
#pragma unroll
            for (int j = 7; j >= N; --j) v[j] = v[j - N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (float)u[j];
        }
    };
    some(std::integral_constant<int, 1>());
    some(std::integral_constant<int, 2>());
    some(std::integral_constant<int, 4>());
}
template <class T> __device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    T u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = (T)v[j];
    if (n >= 8) {
        constexpr int V = kVec<T>;
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            Vec<T> w;
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = u[i * V + j];
            store_vec(p + i * V, w);
        }
        return;
    }
    if (n <= 0) return;
    auto some = [&](auto count) {
        constexpr int N = count.value;
        using S = T __attribute__((ext_vector_type(N)));
        if (n & N) {
            S w;
#pragma unroll
            for (int j = 0; j < N; ++j) w[j] = u[j];
            store_vec(p, w);
            p += N;
#pragma unroll
            for (int j = 0; j < N; ++j) u[j] = u[j + N];   // (what is left has fewer than N)
        }
    };
    some(std::integral_constant<int, 4>());
    some(std::integral_constant<int, 2>());
    some(std::integral_constant<int, 1>());
}

// The operand of an entry point.
inline int check_q8(const std::string &what, const Q8Arg &a, int64_t rows, int64_t cols)
{
    if (rows == 0 || cols == 0) return VF_OK;
    VF_REQUIRE(a.codes && a.scales, what + ": codes or scales is NULL");
    VF_REQUIRE(a.ld >= q8_width(cols) && a.ld % 16 == 0 && ((uintptr_t)a.codes & 15) == 0,
               what + ": rows of codes must start on 16 bytes and hold whole blocks of 128");
    VF_REQUIRE(a.lds >= ceil_div(q8_width(cols) / kBlock, 4) * 4 && a.lds % 4 == 0 && ((uintptr_t)a.scales & 3) == 0,
               what + ": rows of scales must start on 4 bytes and hold whole 32-bit words");
    return VF_OK;
}
inline Region codes_region(const Q8Arg &a, int64_t rows, int64_t cols) { return region(a.codes, rows, q8_width(cols), a.ld, 1); }
inline Region scales_region(const Q8Arg &a, int64_t rows, int64_t cols) { return region(a.scales, rows, q8_width(cols) / kBlock, a.lds, 1); }

}  // namespace vf
