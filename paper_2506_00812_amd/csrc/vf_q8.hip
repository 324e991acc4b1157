// Products of matrices in 8 bits (vf_q8.h): z = x w^T + bias, y = act(z) + residual or, gated, act(z_gate) z_up + residual, in a wide type or in 8 bits again.
// P = w, Q = x, both along the contraction; P takes the matrix instruction's first operand, so that a lane's accumulators are
// neighbours in a row of the output.  The instruction multiplies codes and applies both rows' scales; a lane's 32 codes may be any of a
// step's, so long as both operands' lanes take the same ones.
#include "vf_q8.h"

namespace vf {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- to and from 8 bits

// Sixteen lanes to a block of 128 columns.
template <class T>
__global__ __launch_bounds__(256) void quantize_kernel(int64_t m, int64_t d, const T *__restrict__ x, int64_t ldx, uint8_t *__restrict__ codes, int64_t ldc,
                                                       uint8_t *__restrict__ scales, int64_t lds)
{
    const int64_t blocks = (d + kBlock - 1) / kBlock, all = m * blocks;
    for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < all; i += (int64_t)gridDim.x * 16) {
        const int64_t row = i / blocks, b = i - row * blocks, c = b * kBlock + (threadIdx.x & 15) * 8;
        float v[8];
        load8(x + row * ldx + c, (int)max((int64_t)0, min((int64_t)8, d - c)), v);
        keep_block(v, codes + row * ldc + c, scales + row * lds + b);
    }
}

template <class T>
__global__ __launch_bounds__(256) void dequantize_kernel(int64_t m, int64_t d, const uint8_t *__restrict__ codes, int64_t ldc, const uint8_t *__restrict__ scales,
                                                         int64_t lds, T *__restrict__ y, int64_t ldy)
{
    const int64_t blocks = (d + kBlock - 1) / kBlock, all = m * blocks;
    for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < all; i += (int64_t)gridDim.x * 16) {
        const int64_t row = i / blocks, b = i - row * blocks, c = b * kBlock + (threadIdx.x & 15) * 8;
        if (c >= d) continue;
        const uint2 u = load_vec<uint2>(codes + row * ldc + c);
        const float s = scale_value(scales[row * lds + b]);
        float v[8];
        v[0] = __builtin_amdgcn_cvt_f32_fp8((int)u.x, 0) * s;
        v[1] = __builtin_amdgcn_cvt_f32_fp8((int)u.x, 1) * s;
        v[2] = __builtin_amdgcn_cvt_f32_fp8((int)u.x, 2) * s;
        v[3] = __builtin_amdgcn_cvt_f32_fp8((int)u.x, 3) * s;
        v[4] = __builtin_amdgcn_cvt_f32_fp8((int)u.y, 0) * s;
        v[5] = __builtin_amdgcn_cvt_f32_fp8((int)u.y, 1) * s;
        v[6] = __builtin_amdgcn_cvt_f32_fp8((int)u.y, 2) * s;
        v[7] = __builtin_amdgcn_cvt_f32_fp8((int)u.y, 3) * s;
        store8(y + row * ldy + c, (int)min((int64_t)8, d - c), v);
    }
}

// ---------------------------------------------------------------- products

struct Q8Product {
    Q8Arg P, Q;
    int64_t np, nq;   // outputs of a row (rows of P; of each of its halves where it is gated), rows of Q
    int64_t blocks;   // of 128 of the contraction
    float *part;      // [nq][np], gated [nq][2 np]
};

template <class T> struct Q8Epilogue {
    const T *bias;       // by p
    int act;
    const T *residual;
    int64_t ldr;
    T *y;                // NULL: 8 bits
    int64_t ldy;
    uint8_t *codes, *scales;
    int64_t ldc, lds;
};

// 32 rows of each operand and 64 of the contraction, 32 codes a lane.  EXACT (float32 outputs): the codes are turned into bfloat16, which holds them
// exactly together with their scales.  The matrix cores add products of codes eight neighbours at a time, to 2^-13 of the largest of them
// (measured: 2^16 + 2^3 is right, 2^16 + 2^2 is 2^16; nine places apart nothing is lost): 1.4e-5 of a result of values of like size, whatever their
// number, where products of bfloat16 have 3e-8.  Outputs in bfloat16 and float16 round by far more.
__device__ __forceinline__ void decode(const int8v &c, float scale, Vec<bf16> (&v)[4])
{
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x2 u = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)c[g * 2 + i / 2], scale, true)
                                     : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)c[g * 2 + i / 2], scale, false);
            v[g][i * 2] = u[0];
            v[g][i * 2 + 1] = u[1];
        }
}

template <bool EXACT>
__device__ __forceinline__ float16v mma32(const int8v &p, int sp, const int8v &q, int sq, float16v acc)
{
    if constexpr (EXACT) {
        Vec<bf16> vp[4], vq[4];
        decode(p, scale_value(sp & 255), vp);
        decode(q, scale_value(sq & 255), vq);
#pragma unroll
        for (int g = 0; g < 4; ++g) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vp[g], vq[g], acc, 0, 0, 0);
        return acc;
    } else {
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, acc, 0, 0, 0, sp, 0, sq);
    }
}

// The sums alone, 32 x 32 a wave straight from memory, sixteen rows at a time of both halves where it is gated.
template <bool EXACT, bool GATED>
__global__ __launch_bounds__(256) void q8_simple_kernel(Q8Product a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int OUT = GATED ? 16 : 32;
    const int64_t tiles_p = (a.np + 2 * OUT - 1) / (2 * OUT);
    const int64_t p0 = (blockIdx.x % tiles_p * 2 + (wave & 1)) * OUT, q0 = (blockIdx.x / tiles_p * 2 + (wave >> 1)) * 32;
    int64_t rp = min(p0 + (GATED ? lane & 15 : lane & 31), a.np - 1);
    if (GATED && (lane & 16)) rp += a.np;
    const int64_t rq = min(q0 + (lane & 31), a.nq - 1);
    const uint8_t *P = a.P.codes + rp * a.P.ld + (lane >> 5) * 32, *Q = a.Q.codes + rq * a.Q.ld + (lane >> 5) * 32;
    const uint8_t *SP = a.P.scales + rp * a.P.lds, *SQ = a.Q.scales + rq * a.Q.lds;
    float16v acc = {};
    for (int64_t b = 0; b < a.blocks; ++b) {
        const int sp = SP[b], sq = SQ[b];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            acc = mma32<EXACT>(load_vec<int8v>(P + b * 128 + h * 64), sp, load_vec<int8v>(Q + b * 128 + h * 64), sq, acc);
    }
    const int64_t q = q0 + (lane & 31);
    if (q >= a.nq) return;
    float *to = a.part + q * a.np * (GATED ? 2 : 1);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
        const int64_t p = p0 + (GATED ? r & 15 : r);
        if (p < a.np) to[GATED && r >= 16 ? a.np + p : p] = acc[i];
    }
}

// The epilogue: eight outputs a thread, sixteen neighbouring lanes have a block of 128.
template <class T, bool GATED, bool Q8>
__global__ __launch_bounds__(256) void q8_join_kernel(Q8Product a, Q8Epilogue<T> e)
{
    constexpr int G = GATED ? 2 : 1;
    const int64_t blocks = (a.np + kBlock - 1) / kBlock, all = a.nq * blocks;
    for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < all; i += (int64_t)gridDim.x * 16) {
        const int64_t q = i / blocks, b = i - q * blocks, p = b * kBlock + (threadIdx.x & 15) * 8;
        const int n = (int)max((int64_t)0, min((int64_t)8, a.np - p));
        if (!Q8 && n == 0) continue;
        float v[G][8], u[8];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            load8(a.part + q * a.np * G + g * a.np + p, n, v[g]);
            if (e.bias) {
                load8(e.bias + g * a.np + p, n, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[g][j] += u[j];
            }
        }
        by_act(e.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[0][j] = act_value<act.value, T>(v[0][j]);
                if constexpr (GATED) v[0][j] *= v[1][j];
            }
        });
        if (e.residual) {
            load8(e.residual + q * e.ldr + p, n, u);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[0][j] += u[j];
        }
        if constexpr (Q8) keep_block(v[0], e.codes + q * e.ldc + p, e.scales + q * e.lds + b);
        else store8(e.y + q * e.ldy + p, n, v[0]);
    }
}

// ---------------------------------------------------------------- host side

constexpr int64_t kMaxTiles = 1 << 22;   // and more are not launched: a launch holds fewer than 2^32 threads

static int check_matrix(const char *op, int32_t dtype, int64_t m, int64_t d, const void *x, int64_t ld)
{
    VF_REQUIRE(is_float_type(dtype), std::string(op) + ": dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && d >= 0 && d <= (1 << 25), std::string(op) + ": sizes out of range");
    if (m == 0 || d == 0) return VF_OK;
    VF_REQUIRE(x != nullptr && ld >= d, std::string(op) + ": the matrix is NULL or its ld less than d");
    return VF_OK;
}

int quantize_impl(int32_t dtype, int64_t m, int64_t d, const void *x, int64_t ldx, const Q8Arg &out, hipStream_t s)
{
    if (int rc = check_matrix("quantize", dtype, m, d, x, ldx); rc != VF_OK) return rc;
    if (int rc = check_q8("quantize", out, m, d); rc != VF_OK) return rc;
    if (m == 0 || d == 0) return VF_OK;
    const Region in = region(x, m, d, ldx, type_size(dtype)), codes = codes_region(out, m, d), scales = scales_region(out, m, d);
    VF_REQUIRE(!overlap(codes, in) && !overlap(scales, in) && !overlap(codes, scales), "quantize: codes or scales overlap x or each other");
    const int64_t items = m * ceil_div(d, kBlock);
    by_type(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        quantize_kernel<T><<<dim3(grid_of(ceil_div(items, 16))), dim3(256), 0, s>>>(m, d, (const T *)x, ldx, (uint8_t *)out.codes, out.ld, (uint8_t *)out.scales, out.lds);
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

int dequantize_impl(int32_t dtype, int64_t m, int64_t d, const Q8Arg &in, void *y, int64_t ldy, hipStream_t s)
{
    if (int rc = check_matrix("dequantize", dtype, m, d, y, ldy); rc != VF_OK) return rc;
    if (int rc = check_q8("dequantize", in, m, d); rc != VF_OK) return rc;
    if (m == 0 || d == 0) return VF_OK;
    const Region out = region(y, m, d, ldy, type_size(dtype));
    VF_REQUIRE(!overlap(out, codes_region(in, m, d)) && !overlap(out, scales_region(in, m, d)), "dequantize: y overlaps codes or scales");
    const int64_t items = m * ceil_div(d, kBlock);
    by_type(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        dequantize_kernel<T><<<dim3(grid_of(ceil_div(items, 16))), dim3(256), 0, s>>>(m, d, in.codes, in.ld, in.scales, in.lds, (T *)y, ldy);
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

static int check_q8_sizes(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act)
{
    VF_REQUIRE(is_float_type(dtype), "linear in 8 bits: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && n >= 0 && n <= (1 << 24) && k >= 0 && k <= (1 << 25), "linear in 8 bits: m, n or k out of range");
    VF_REQUIRE(act >= VF_ACT_NONE && act <= VF_ACT_SILU, "linear in 8 bits: unknown activation");
    return VF_OK;
}

int linear_q8_workspace_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t gated, int32_t quantized, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "linear in 8 bits: bytes is NULL");
    if (int rc = check_q8_sizes(dtype, m, n, k, 0); rc != VF_OK) return rc;
    *bytes = (size_t)m * n * (gated ? 2 : 1) * 4;
    return VF_OK;
}

int linear_q8_impl(const LinearQ8Args &a)
{
    if (int rc = check_q8_sizes(a.dtype, a.m, a.n, a.k, a.act); rc != VF_OK) return rc;
    VF_REQUIRE(a.gated == 0 || a.gated == 1, "linear in 8 bits: gated must be 0 or 1");
    if (a.m == 0 || a.n == 0) return VF_OK;
    const int64_t rows = a.gated ? 2 * a.n : a.n;
    if (int rc = check_q8("linear in 8 bits: x", a.x, a.m, a.k); rc != VF_OK) return rc;
    if (int rc = check_q8("linear in 8 bits: w", a.w, rows, a.k); rc != VF_OK) return rc;
    const bool q8 = a.out.codes != nullptr || a.out.scales != nullptr;
    VF_REQUIRE((a.y != nullptr) != q8, "linear in 8 bits: the output must be either y or codes and scales");
    VF_REQUIRE(q8 || a.ldy >= a.n, "linear in 8 bits: ldy is less than n");
    VF_REQUIRE(!a.residual || a.ldr >= a.n, "linear in 8 bits: ldr is less than n");
    if (q8)
        if (int rc = check_q8("linear in 8 bits: the output", a.out, a.m, a.n); rc != VF_OK) return rc;
    size_t need = 0;
    if (int rc = linear_q8_workspace_impl(a.dtype, a.m, a.n, a.k, a.gated, q8, &need); rc != VF_OK) return rc;
    if (int rc = check_workspace("linear in 8 bits", a.workspace, a.workspace_bytes, need); rc != VF_OK) return rc;
    const size_t size = type_size(a.dtype);
    const Region y = region(a.y, a.m, a.n, a.ldy, size), r = region(a.residual, a.m, a.n, a.ldr, size), codes = codes_region(a.out, a.m, a.n),
                 scales = scales_region(a.out, a.m, a.n);
    for (const Region &in : {codes_region(a.x, a.m, a.k), scales_region(a.x, a.m, a.k), codes_region(a.w, rows, a.k), scales_region(a.w, rows, a.k), region(a.bias, rows, size)})
        VF_REQUIRE(!overlap(y, in) && !overlap(codes, in) && !overlap(scales, in), "linear in 8 bits: an output overlaps an input");
    VF_REQUIRE(y.same(r) || !overlap(y, r), "linear in 8 bits: y overlaps the residual and is not it");
    VF_REQUIRE(!overlap(codes, r) && !overlap(scales, r) && !overlap(codes, scales), "linear in 8 bits: codes or scales overlap the residual or each other");
    VF_REQUIRE(ceil_div(rows, 64) * ceil_div(a.m, 64) < kMaxTiles, "linear in 8 bits: too many output tiles in one call");
    const Q8Product p{a.w, a.x, a.n, a.m, ceil_div(a.k, kBlock), (float *)a.workspace};
    by_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        constexpr bool kExact = std::is_same_v<T, float>;
        const Q8Epilogue<T> e{(const T *)a.bias, a.act, (const T *)a.residual, a.ldr, (T *)a.y, a.ldy, (uint8_t *)a.out.codes, (uint8_t *)a.out.scales, a.out.ld, a.out.lds};
        const dim3 grid((unsigned)(ceil_div(rows, 64) * ceil_div(a.m, 64))), join(grid_of(ceil_div(a.m * ceil_div(a.n, kBlock), 16)));
        auto run = [&](auto gated) {
            q8_simple_kernel<kExact, gated.value><<<grid, dim3(256), 0, a.stream>>>(p);
            if (q8) q8_join_kernel<T, gated.value, true><<<join, dim3(256), 0, a.stream>>>(p, e);
            else q8_join_kernel<T, gated.value, false><<<join, dim3(256), 0, a.stream>>>(p, e);
        };
        if (a.gated) run(std::true_type());
        else run(std::false_type());
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

}  // namespace vf
