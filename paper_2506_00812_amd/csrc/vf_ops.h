// What the kernels and the host code of the encoder operators share: element types, vector loads of any alignment,
// wave and workgroup sums, activations.  Nothing here is part of the C ABI (see include/vecflow.h).
#pragma once

#include <cmath>
#include <type_traits>

#include "vf_host.h"

#pragma clang fp contract(off)

namespace vf {

using bf16 = __bf16;
using f16 = _Float16;

template <class T> constexpr int kVec = 16 / (int)sizeof(T);   // elements of a 16-byte vector
template <class T> using Vec = T __attribute__((ext_vector_type(16 / sizeof(T))));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

// Calls fn with a null pointer of the element type that dtype names.
template <class F> void by_type(int32_t dtype, F &&fn)
{
    if (dtype == VF_F32) fn((float *)nullptr);
    else if (dtype == VF_BF16) fn((bf16 *)nullptr);
    else fn((f16 *)nullptr);
}
inline bool is_float_type(int32_t dtype) { return dtype == VF_F32 || dtype == VF_BF16 || dtype == VF_F16; }
inline size_t type_size(int32_t dtype) { return dtype == VF_F32 ? 4 : 2; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kMaxExtent = INT32_MAX;

inline int check_workspace(const char *op, const void *workspace, size_t have, size_t need)
{
    if (need == 0) return VF_OK;
    VF_REQUIRE(workspace != nullptr && have >= need, std::string(op) + ": the workspace must hold " + std::to_string(need) + " bytes");
    VF_REQUIRE(((uintptr_t)workspace & 15) == 0, std::string(op) + ": the workspace must be aligned to 16 bytes");
    return VF_OK;
}

// A matrix argument in memory: rows of `width` bytes, `ld` bytes apart.  A vector is one row.
struct Region {
    uintptr_t at;
    int64_t rows, width, ld;
    bool same(const Region &o) const { return at == o.at && rows == o.rows && width == o.width && ld == o.ld; }
};
inline Region region(const void *p, int64_t rows, int64_t cols, int64_t ld, size_t size)
{
    if (p == nullptr || cols <= 0) return {0, 0, 0, 0};
    const int64_t s = (int64_t)size;
    if (rows == 1 || ld == cols) return {(uintptr_t)p, rows > 0, rows * cols * s, rows * cols * s};
    return {(uintptr_t)p, rows, cols * s, ld * s};
}
inline Region region(const void *p, int64_t n, size_t size) { return region(p, 1, n, n, size); }

// Whether two regions share a byte.  (Of two slices with unlike row distances it is not asked: that takes a walk over their rows.)
inline bool overlap(Region a, Region b)
{
    if (a.rows == 0 || b.rows == 0) return false;
    if (b.at < a.at) std::swap(a, b);
    const int64_t d = (int64_t)(b.at - a.at);
    if (d >= (a.rows - 1) * a.ld + a.width) return false;
    // b begins in row d / ld of a, or between that one and the next; what begins between them reaches the next one in its first row or never
    if (a.rows == 1) return true;
    if (b.rows > 1 && a.ld != b.ld) return false;
    const int64_t i = d / a.ld, r = d % a.ld;
    return r < a.width || (i + 1 < a.rows && r + b.width > a.ld);
}

// A vector at an address that is aligned to an element only: one 16-byte load or store all the same (global memory
// takes any alignment; rows cut out of a wider matrix start anywhere).
template <class V, class T> __device__ __forceinline__ V load_vec(const T *p)
{
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
template <class V, class T> __device__ __forceinline__ void store_vec(T *p, V v) { __builtin_memcpy(p, &v, sizeof(V)); }

// n elements (0 .. a whole vector) at p, the rest `fill`.
template <class T> __device__ __forceinline__ Vec<T> load_part(const T *p, int n, T fill)
{
    if (n >= kVec<T>) return load_vec<Vec<T>>(p);
    Vec<T> v;
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) v[i] = i < n ? p[i] : fill;
    return v;
}
template <class T> __device__ __forceinline__ void store_part(T *p, Vec<T> v, int n)
{
    if (n >= kVec<T>) { store_vec(p, v); return; }
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
        if (i < n) p[i] = v[i];
}

// Sum and maximum over the 64 lanes of a wave, the same in every lane: within rows of sixteen on DPP moves, the four rows' results
// through scalar registers (no trip through LDS, which a shuffle takes).
template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ float sum16(float v)   // of each row of sixteen lanes
{
    v += dpp<0xB1>(v);           // the neighbour
    v += dpp<0x4E>(v);           // the other pair of four
    v += dpp<0x141>(v);          // the other four of eight
    return v + dpp<0x140>(v);    // the other eight of sixteen
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = sum16(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
__device__ __forceinline__ float max16(float v)
{
    v = fmaxf(v, dpp<0xB1>(v));
    v = fmaxf(v, dpp<0x4E>(v));
    v = fmaxf(v, dpp<0x141>(v));
    return fmaxf(v, dpp<0x140>(v));
}
__device__ __forceinline__ float wave_max(float v)
{
    v = max16(v);
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true));
    const uint32_t a = max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16));
    return max(a, max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
}

// exp(x) on the hardware's 2^x: a relative error of about 2^-23 (1 + |x|), which weighs little where exp(x) is large enough to count.
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }

// Phi(-|z|), the tail of the normal distribution, and exp(-z^2 / 2), for results of type T: a polynomial in t = 1 / (1 + c |z|) times the
// density.
//   2 bytes: Hastings' (Abramowitz and Stegun, Handbook of Mathematical Functions, 26.2.17; off by less than 7.5e-8, a 2^13th of what
//   bfloat16 rounds by; the coefficients here hold the density's 1 / sqrt(2 pi)).  With erff, three times the instructions, an epilogue of
//   10,000 x 4,096 outputs took 50 us of a product's 145; with this one 25.
//   float32: Hastings' loses the tail's digits (0.4 % at z = -6).  A fit of our own to Phi(-z) exp(z^2 / 2) / t over all z >= 0, least squares
//   reweighted towards the largest relative error, 3.2e-8 before rounding (c = 0.32: the best of degree 9), 3.3e-7 after.
template <class T> __device__ __forceinline__ float normal_tail(float z, float &density)
{
    density = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    if constexpr (std::is_same_v<T, float>) {
        const float t = rcp_fast(__builtin_fmaf(0.32f, fabsf(z), 1.f));
        float s = __builtin_fmaf(t, -0.02107816f, 0.0954072177f);
    s = __builtin_fmaf(t, s, -0.146707371f);
    s = __builtin_fmaf(t, s, 0.0653279349f);
    s = __builtin_fmaf(t, s, -0.00937751681f);
    s = __builtin_fmaf(t, s, 0.058653947f);
    s = __builtin_fmaf(t, s, 0.0878291056f);
    s = __builtin_fmaf(t, s, 0.114622362f);
    s = __builtin_fmaf(t, s, 0.127660945f);
    s = __builtin_fmaf(t, s, 0.127661526f);
        return s * t * density;
    }
    constexpr float r = 0.39894228040143268f;
    const float t = rcp_fast(__builtin_fmaf(0.2316419f, fabsf(z), 1.f));
    float s = __builtin_fmaf(t, 1.330274429f * r, -1.821255978f * r);
    s = __builtin_fmaf(t, s, 1.781477937f * r);
    s = __builtin_fmaf(t, s, -0.356563782f * r);
    s = __builtin_fmaf(t, s, 0.319381530f * r);
    return s * t * density;
}
// 1 / (1 + exp(-z)), for results of type T.  float32: with the exponent in two parts, so that its rounding does not grow with |z|.
template <class T> __device__ __forceinline__ float sigmoid(float z)
{
    if constexpr (std::is_same_v<T, float>) {
        const float x = z < -128.f ? 128.f : z > 128.f ? -128.f : -z;   // (beyond it is 0 or 1; NaN stays NaN)
        const float hi = x * 1.4426950408889634f;
        const float lo = __builtin_fmaf(x, 1.4426950408889634f, -hi) + x * 1.92596299e-8f;   // log2 e is these two numbers
        return rcp_fast(1.f + __builtin_amdgcn_exp2f(hi) * __builtin_fmaf(lo, 0.69314718f, 1.f));
    }
    return rcp_fast(1.f + exp_fast(-z));
}

// The activations at infinite z are their limits: a factor that vanishes meets the largest finite number, not an infinity.  NaN stays
// NaN (the other factor still has it).
constexpr float kFltMax = 3.4028234663852886e38f;
template <int ACT, class T> __device__ __forceinline__ float act_value(float z)
{
    if constexpr (ACT == VF_ACT_NONE) return z;
    if constexpr (ACT == VF_ACT_RELU) return z < 0.f ? 0.f : z;
    if constexpr (ACT == VF_ACT_GELU) {   // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
        float density;
        const float tail = normal_tail<T>(z, density);
        return __builtin_fmaf(-fminf(fabsf(z), kFltMax), tail, fmaxf(z, 0.f));
    }
    return fmaxf(z, -kFltMax) * sigmoid<T>(z);
}
template <int ACT, class T> __device__ __forceinline__ float act_slope(float z)
{
    if constexpr (ACT == VF_ACT_NONE) return 1.f;
    if constexpr (ACT == VF_ACT_RELU) return z > 0.f ? 1.f : z != z ? z : 0.f;
    const float u = __builtin_amdgcn_fmed3f(z, -kFltMax, kFltMax);
    if constexpr (ACT == VF_ACT_GELU) {
        float density;
        const float tail = normal_tail<T>(z, density);
        return __builtin_fmaf(u * 0.39894228040143268f, density, z > 0.f ? 1.f - tail : tail);
    }
    const float a = sigmoid<T>(z);
    return a * __builtin_fmaf(u, 1.f - a, 1.f);
}
// Calls fn with the activation as a constant.
template <class F> __host__ __device__ __forceinline__ void by_act(int act, F &&fn)
{
    if (act == VF_ACT_NONE) fn(std::integral_constant<int, VF_ACT_NONE>());
    else if (act == VF_ACT_RELU) fn(std::integral_constant<int, VF_ACT_RELU>());
    else if (act == VF_ACT_GELU) fn(std::integral_constant<int, VF_ACT_GELU>());
    else fn(std::integral_constant<int, VF_ACT_SILU>());
}

// Column sums from partial rows part [parts][sums][d]: 16 columns and one of the sums per workgroup, 64 threads to a column (2,048
// columns of 1,024 rows 18 us with 16 threads to a column, 5 with 64); parts = 0: zeros.
template <class T>
__global__ __launch_bounds__(1024) void join_parts_kernel(int parts, int64_t d, const float *__restrict__ part, T *out0, T *out1)
{
    __shared__ float comb[64][17];
    const int t = threadIdx.x & 15, sub = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + t, stride = (int64_t)gridDim.y * d;
    T *out = blockIdx.y == 0 ? out0 : out1;
    if (out == nullptr) return;
    float a[4] = {};
    if (c < d) {
        const float *from = part + (int64_t)blockIdx.y * d + c;
        int p = sub;
        for (; p + 192 < parts; p += 256) {
#pragma unroll
            for (int u = 0; u < 4; ++u) a[u] += from[(int64_t)(p + 64 * u) * stride];
        }
        for (; p < parts; p += 64) a[0] += from[(int64_t)p * stride];
    }
    comb[sub][t] = (a[0] + a[1]) + (a[2] + a[3]);
    __syncthreads();
    if (sub < 16) {   // sixteen lanes to a column
        const int col = threadIdx.x >> 4, part16 = threadIdx.x & 15;
        float s = (comb[part16][col] + comb[part16 + 16][col]) + (comb[part16 + 32][col] + comb[part16 + 48][col]);
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) s += __shfl_xor(s, w, 16);
        const int64_t at = (int64_t)blockIdx.x * 16 + col;
        if (part16 == 0 && at < d) out[at] = (T)s;
    }
}
template <class T> void launch_join_parts(int parts, int64_t d, int sums, const float *part, T *out0, T *out1, hipStream_t s)
{
    join_parts_kernel<T><<<dim3((unsigned)ceil_div(d, 16), (unsigned)sums), dim3(1024), 0, s>>>(parts, d, part, out0, out1);
}

// ---------------------------------------------------------------- entry points' bodies

struct LinearArgs {
    int32_t dtype, act;
    int64_t m, n, k;
    const void *x, *w, *bias, *residual, *dy;
    int64_t ldx, ldw, ldr, lddy;
    void *y, *z, *dx, *dw, *dbias;
    int64_t ldy, ldz, lddx, lddw;
    void *workspace;
    size_t workspace_bytes;
    hipStream_t stream;
};
int linear_impl(const LinearArgs &a);
int linear_backward_impl(const LinearArgs &a);
int debug_linear_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t product, int32_t direct, int32_t *tiling, int32_t *splits);
int linear_workspace_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act, int32_t backward, size_t *bytes);

struct NormArgs {
    int32_t dtype;
    int64_t m, d;
    const void *x, *dy, *weight, *bias;
    int64_t ldx, lddy, ldy;
    double eps;
    void *y, *dweight, *dbias;   // y: the gradient dx in the backward pass
    float *mean, *rstd;
    void *workspace;
    size_t workspace_bytes;
    hipStream_t stream;
};
int layer_norm_impl(const NormArgs &a);
int layer_norm_backward_impl(const NormArgs &a);
int layer_norm_workspace_impl(int32_t dtype, int64_t m, int64_t d, size_t *bytes);

struct LogProbArgs {
    int32_t dtype, top;
    int64_t m, v, ld, ldd;
    const void *logits;
    const int32_t *targets;
    float *logp, *entropy, *lse;
    int32_t *top_ids;
    float *top_logp;
    const float *d_logp, *d_entropy;
    void *dlogits;
    void *workspace;
    size_t workspace_bytes;
    hipStream_t stream;
};
int log_probs_impl(const LogProbArgs &a);
int log_probs_backward_impl(const LogProbArgs &a);
int log_probs_workspace_impl(int32_t dtype, int64_t m, int64_t v, int32_t top, size_t *bytes);

int adamw_step_impl(const vf_adamw_tensor *tensors, int32_t n_tensors, const vf_adamw_params *params, const int32_t *skip,
                    hipStream_t s);
int adamw_moments_impl(const vf_adamw_tensor *tensors, int32_t n_tensors, float *const *m_out, float *const *v_out,
                       hipStream_t s);

}  // namespace vf
