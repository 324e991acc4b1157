// Root-mean-square norm of a sum, and its gradients.
//   forward   s = x + residual, rounded to the matrices' type (what the gradient reads is what was normalised);
//             rstd = 1 / sqrt(avg(s^2) + eps);  y = s rstd weight, in that type or in 8 bits straight from float32
//   backward  h = s rstd, g = dy weight:  dx = rstd (g - h avg(g h)) + d_s;  dweight = sum of dy h over all rows
// Both are bound by memory: a row is read once, held in registers while its sum is taken, and written once.  A thread has eight columns at a
// time, so that sixteen neighbouring lanes have the 128 that share a scale.
#include "vf_q8.h"

namespace vf {

template <class T> struct RmsOut {
    T *y;            // NULL: 8 bits
    int64_t ldy;
    T *total;        // s; NULL without a residual
    int64_t ldt;
    float *rstd;
    uint8_t *codes, *scales;
    int64_t ldc, lds;
};

// What a row's last block is filled up with, also where rstd is not finite.
__device__ __forceinline__ void zeros_behind(float (&v)[8], int n)
{
    if (n >= 8) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? v[j] : 0.f;
}

// Rows of up to TPR * NV eights: thread t of a row holds eights t, t + TPR, ...  A wave has a row of up to 1,024 by itself, four rows a workgroup and nothing to
// wait for.  10,000 x 1,024 in bfloat16 with a residual, into 8 bits: 72 MB in 15 us (4.8 TB/s); one such row 3.1 us.
template <class T, int TPR, int NV, bool Q8>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_forward_kernel(int64_t m, int d, const T *x, int64_t ldx, const T *residual, int64_t ldr,
                                                                             const T *__restrict__ weight, float eps, RmsOut<T> o)
{
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    __shared__ float lds[16];
    const int t = threadIdx.x % TPR;
    const int width = Q8 ? (d + kBlock - 1) / kBlock * kBlock : d;
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < m; row += (int64_t)gridDim.x * RPB) {
        float v[NV][8];
        float sum[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * 8;
            if (c < d) {
                load8(x + row * ldx + c, d - c, v[i]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
            }
        }
        if (residual) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TPR) * 8;
                if (c < d) {
                    float r[8];
                    load8(residual + row * ldr + c, d - c, r);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] = (float)(T)(v[i][j] + r[j]);
                    store8(o.total + row * o.ldt + c, d - c, v[i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] += v[i][j] * v[i][j];
        row_sums<TPR>(sum, lds);
        const float rstd = 1.f / sqrtf(sum[0] / (float)d + eps);
        if (t == 0 && o.rstd) o.rstd[row] = rstd;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * 8;
            if (c >= width) continue;
            float w[8];
            if (weight && c < d) {
                load8(weight + c, d - c, w);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = 1.f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * rstd * w[j];
            if constexpr (Q8) zeros_behind(v[i], d - c);
            if constexpr (Q8) keep_block(v[i], o.codes + row * o.ldc + c, o.scales + row * o.lds + c / kBlock);
            else store8(o.y + row * o.ldy + c, d - c, v[i]);
        }
    }
}

// Rows of any length, read twice (the second time mostly from the caches; a sum is read from where it was written, by the thread that did).
template <class T, bool Q8>
__global__ __launch_bounds__(1024) void rms_forward_long_kernel(int64_t m, int64_t d, const T *x, int64_t ldx, const T *residual, int64_t ldr,
                                                                const T *weight, float eps, RmsOut<T> o)
{
    __shared__ float lds[16];
    const int64_t width = Q8 ? (d + kBlock - 1) / kBlock * kBlock : d;
    for (int64_t row = blockIdx.x; row < m; row += gridDim.x) {
        const T *from = residual ? o.total + row * o.ldt : x + row * ldx;
        float sum[1] = {0.f};
        for (int64_t c = (int64_t)threadIdx.x * 8; c < d; c += 1024 * 8) {
            const int n = (int)min((int64_t)8, d - c);
            float v[8];
            load8(x + row * ldx + c, n, v);
            if (residual) {
                float r[8];
                load8(residual + row * ldr + c, n, r);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (float)(T)(v[j] + r[j]);
                store8(o.total + row * o.ldt + c, n, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] += v[j] * v[j];
        }
        row_sums<1024>(sum, lds);
        const float rstd = 1.f / sqrtf(sum[0] / (float)d + eps);
        if (threadIdx.x == 0 && o.rstd) o.rstd[row] = rstd;
        for (int64_t c = (int64_t)threadIdx.x * 8; c < width; c += 1024 * 8) {
            const int n = (int)max((int64_t)0, min((int64_t)8, d - c));
            float v[8], w[8];
            load8(from + c, n, v);
            if (weight) load8(weight + c, n, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] * rstd * (weight ? w[j] : 1.f);
            if constexpr (Q8) zeros_behind(v, n);
            if constexpr (Q8) keep_block(v, o.codes + row * o.ldc + c, o.scales + row * o.lds + c / kBlock);
            else store8(o.y + row * o.ldy + c, n, v);
        }
    }
}

// dx of the rows blockIdx.x * RPB + w, + gridDim.x * RPB, ...; PARTS: every thread also sums its columns' dy h over those rows, and
// the workgroup leaves one row of them in part [gridDim.x][d], or (part NULL: it is the only one) the sums themselves in dweight.
// 100,000 x 1,024 in bfloat16 with d_s: 820 MB in 145 us (5.65 TB/s), the partial rows' join 5.
template <class T, int TPR, int NV, bool PARTS>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR, 4) void rms_backward_kernel(int64_t m, int d, const T *dy, int64_t lddy, const T *__restrict__ s,
                                                                              int64_t lds_, const float *__restrict__ rstd, const T *__restrict__ weight,
                                                                              const T *d_total, int64_t ldt, T *dx, int64_t lddx, float *__restrict__ part,
                                                                              T *dweight)
{
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    __shared__ float lds[16];
    __shared__ float comb[RPB > 1 && PARTS ? TPR * 8 : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float w[NV][8], aw[NV][8] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * 8;
        if (weight && c < d) {
            load8(weight + c, d - c, w[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[i][j] = 1.f;
        }
    }
    for (int64_t row = (int64_t)blockIdx.x * RPB + sub; row < m; row += (int64_t)gridDim.x * RPB) {
        const float rs = rstd[row];
        float y[NV][8], h[NV][8];
        float sum[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * 8;
            if (c < d) {
                load8(dy + row * lddy + c, d - c, y[i]);
                load8(s + row * lds_ + c, d - c, h[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * 8;
            if (c < d) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    h[i][j] *= rs;
                    const float p = y[i][j] * h[i][j];
                    if constexpr (PARTS) aw[i][j] += p;
                    sum[0] += p * w[i][j];
                }
            }
        }
        if (dx) {
            row_sums<TPR>(sum, lds);
            const float b = sum[0] / (float)d;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TPR) * 8;
                if (c < d) {
                    float o[8];
                    if (d_total) {
                        load8(d_total + row * ldt + c, d - c, o);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = 0.f;
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] += rs * (y[i][j] * w[i][j] - h[i][j] * b);
                    store8(dx + row * lddx + c, d - c, o);
                }
            }
        }
    }
    if constexpr (PARTS && TPR == 16) {   // a wave's four rows first: then every wave has one set of sums, in each of its rows
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                aw[i][j] += __shfl_xor(aw[i][j], 16, 64);
                aw[i][j] += __shfl_xor(aw[i][j], 32, 64);
            }
    }
    if constexpr (PARTS) {
        const int group = TPR == 16 ? ((threadIdx.x & 63) < 16 ? threadIdx.x >> 6 : -1) : sub;   // which of `kGroups` sets of sums
        constexpr int kGroups = TPR == 16 ? 4 : RPB;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * 8;
            if constexpr (kGroups > 1) {   // the waves' sums, one wave after the other
                for (int r = kGroups - 1; r > 0; --r) {
                    __syncthreads();
                    if (group == r) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) comb[j * TPR + t] = aw[i][j];
                    }
                    __syncthreads();
                    if (group == 0) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) aw[i][j] += comb[j * TPR + t];
                    }
                }
            }
            if (group == 0 && c < d) {
                if (part) store8(part + (int64_t)blockIdx.x * d + c, d - c, aw[i]);
                else store8(dweight + c, d - c, aw[i]);
            }
        }
    }
}

// dx of rows of any length, one workgroup each; read twice.
template <class T>
__global__ __launch_bounds__(1024) void rms_backward_long_kernel(int64_t m, int64_t d, const T *dy, int64_t lddy, const T *s, int64_t lds_,
                                                                 const float *rstd, const T *weight, const T *d_total, int64_t ldt, T *dx, int64_t lddx)
{
    __shared__ float lds[16];
    for (int64_t row = blockIdx.x; row < m; row += gridDim.x) {
        const float rs = rstd[row];
        float sum[1] = {0.f};
        for (int pass = 0; pass < 2; ++pass) {
            const float b = sum[0] / (float)d;
            for (int64_t c = (int64_t)threadIdx.x * 8; c < d; c += 1024 * 8) {
                const int n = (int)min((int64_t)8, d - c);
                float y[8], h[8], w[8], o[8] = {};
                load8(dy + row * lddy + c, n, y);
                load8(s + row * lds_ + c, n, h);
                if (weight) load8(weight + c, n, w);
                if (pass == 1 && d_total) load8(d_total + row * ldt + c, n, o);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float g = y[j] * (weight ? w[j] : 1.f);
                    h[j] *= rs;
                    if (pass == 0) sum[0] += g * h[j];
                    o[j] += rs * (g - h[j] * b);
                }
                if (pass == 1) store8(dx + row * lddx + c, n, o);
            }
            if (pass == 0) row_sums<1024>(sum, lds);
        }
    }
}

// The same partial sums for rows of any length: blockIdx.x takes 64 columns, blockIdx.y every gridDim.y-th group of 4 rows.
template <class T>
__global__ __launch_bounds__(256) void rms_columns_kernel(int64_t m, int64_t d, const T *dy, int64_t lddy, const T *s, int64_t lds_, const float *rstd,
                                                          float *part)
{
    __shared__ float comb[4][64];
    const int t = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + t;
    float aw = 0.f;
    if (c < d) {
        for (int64_t row = (int64_t)blockIdx.y * 4 + sub; row < m; row += (int64_t)gridDim.y * 4)
            aw += (float)dy[row * lddy + c] * ((float)s[row * lds_ + c] * rstd[row]);
    }
    comb[sub][t] = aw;
    __syncthreads();
    if (sub == 0 && c < d) part[(int64_t)blockIdx.y * d + c] = (comb[0][t] + comb[1][t]) + (comb[2][t] + comb[3][t]);
}

constexpr int64_t kMaxRow = 1 << 24;   // elements of a row

static int64_t eights_of(int64_t d) { return ceil_div(d, 8); }

// Calls fn with the threads of a row and the eights of a thread; false: no kernel holds a row of so many.  Two eights a thread at most: four take so many registers
// that two waves share a SIMD (50,000 x 2,048 in bfloat16 backward: 223 us so, 159 this way; 10,000 x 8,192: 192 and 133).
template <class F> static bool by_eights(int64_t nv, F &&fn)
{
    if (nv <= 16) fn(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    else if (nv <= 32) fn(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
    else if (nv <= 64) fn(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    else if (nv <= 128) fn(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    else if (nv <= 256) fn(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
    else if (nv <= 512) fn(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    else if (nv <= 1024) fn(std::integral_constant<int, 512>(), std::integral_constant<int, 2>());
    else if (nv <= 2048) fn(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
    else return false;
    return true;
}

// Workgroups (and so partial rows) of the backward pass: as many as are in work at the same time, or fewer rows than that need.
static int64_t parts_of(int64_t m, int64_t d)
{
    const int64_t nv = eights_of(d);
    if (m <= (nv <= 32 ? 32 : nv <= 128 ? 8 : nv <= 256 ? 2 : 0)) return 1;   // two rows a wave, or two times four: less than one more launch
    const int64_t most = nv > 512 ? 512 : std::max<int64_t>(512, std::min<int64_t>(1024, m / 16));
    if (nv <= 32) return std::min(ceil_div(m, 16), most);
    if (nv <= 128) return std::min(ceil_div(m, 4), most);
    if (nv <= 2048) return std::min(m, most);
    return std::min<int64_t>(ceil_div(m, 4), 64);
}
static bool sums_at_once(int64_t m, int64_t d) { return eights_of(d) <= 256 && parts_of(m, d) == 1; }

static int check_rms(const RmsArgs &a)
{
    VF_REQUIRE(is_float_type(a.dtype), "rms norm: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(a.m >= 0 && a.m <= kMaxExtent, "rms norm: m out of range");
    VF_REQUIRE(a.d >= 1 && a.d <= kMaxRow, "rms norm: d must be 1 .. 2^24");
    VF_REQUIRE(a.m == 0 || a.x != nullptr, "rms norm: x is NULL");
    VF_REQUIRE(a.ldx >= a.d, "rms norm: ldx is less than d");
    return VF_OK;
}

int rms_norm_impl(const RmsArgs &a)
{
    if (int rc = check_rms(a); rc != VF_OK) return rc;
    VF_REQUIRE(a.eps >= 0 && std::isfinite(a.eps), "rms norm: eps must be finite and not negative");
    const bool q8 = a.codes != nullptr || a.scales != nullptr;
    VF_REQUIRE(a.m == 0 || (a.y != nullptr) != q8, "rms norm: the output must be either y or codes and scales");
    VF_REQUIRE(a.y == nullptr || a.ldy >= a.d, "rms norm: ldy is less than d");
    VF_REQUIRE((a.residual == nullptr) == (a.total == nullptr) || a.m == 0, "rms norm: residual and total go together");
    VF_REQUIRE(a.residual == nullptr || (a.ldr >= a.d && a.ldt >= a.d), "rms norm: ldr or ldt is less than d");
    const Q8Arg out{a.codes, a.scales, a.ldc, a.lds};
    if (q8)
        if (int rc = check_q8("rms norm", out, a.m, a.d); rc != VF_OK) return rc;
    if (a.m == 0) return VF_OK;
    const size_t size = type_size(a.dtype);
    const Region x = region(a.x, a.m, a.d, a.ldx, size), r = region(a.residual, a.m, a.d, a.ldr, size), w = region(a.weight, a.d, size);
    const Region y = region(a.y, a.m, a.d, a.ldy, size), total = region(a.total, a.m, a.d, a.ldt, size), rstd = region(a.rstd, a.m, 4);
    const Region codes = codes_region(out, a.m, a.d), scales = scales_region(out, a.m, a.d);
    VF_REQUIRE((y.same(x) && !a.residual) || !overlap(y, x), "rms norm: y overlaps x and is not it, or there is a residual");
    VF_REQUIRE((total.same(x) || !overlap(total, x)) && (total.same(r) || !overlap(total, r)), "rms norm: total overlaps x or the residual and is not it");
    VF_REQUIRE(!overlap(y, r), "rms norm: y overlaps the residual");
    for (const Region &o : {codes, scales, rstd})
        VF_REQUIRE(!overlap(o, x) && !overlap(o, r) && !overlap(o, y) && !overlap(o, total), "rms norm: codes, scales or rstd overlap another argument");
    for (const Region &o : {y, total, rstd, codes, scales}) VF_REQUIRE(!overlap(o, w), "rms norm: an output overlaps weight");
    VF_REQUIRE(!overlap(y, total) && !overlap(codes, scales) && !overlap(codes, rstd) && !overlap(scales, rstd), "rms norm: the outputs overlap each other");
    by_type(a.dtype, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        const RmsOut<T> o{(T *)a.y, a.ldy, (T *)a.total, a.ldt, a.rstd, a.codes, a.scales, a.ldc, a.lds};
        auto run = [&](auto in8) {
            constexpr bool Q8 = in8.value;
            const bool short_row = by_eights(eights_of(Q8 ? q8_width(a.d) : a.d), [&](auto tpr, auto nv) {
                constexpr int TPR = tpr.value, NV = nv.value;
                const int64_t blocks = TPR < 256 ? ceil_div(a.m, 256 / TPR) : a.m;
                rms_forward_kernel<T, TPR, NV, Q8><<<dim3(grid_of(blocks)), dim3(TPR < 256 ? 256 : TPR), 0, a.stream>>>(
                    a.m, (int)a.d, (const T *)a.x, a.ldx, (const T *)a.residual, a.ldr, (const T *)a.weight, (float)a.eps, o);
            });
            if (!short_row)
                rms_forward_long_kernel<T, Q8><<<dim3(grid_of(a.m)), dim3(1024), 0, a.stream>>>(
                    a.m, a.d, (const T *)a.x, a.ldx, (const T *)a.residual, a.ldr, (const T *)a.weight, (float)a.eps, o);
        };
        if (q8) run(std::true_type());
        else run(std::false_type());
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

int rms_norm_workspace_impl(int32_t dtype, int64_t m, int64_t d, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "rms norm: bytes is NULL");
    VF_REQUIRE(is_float_type(dtype), "rms norm: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && d >= 1 && d <= kMaxRow, "rms norm: sizes out of range");
    *bytes = sums_at_once(m, d) ? 0 : (size_t)parts_of(m, d) * (size_t)d * 4;
    return VF_OK;
}

int rms_norm_backward_impl(const RmsArgs &a)
{
    if (int rc = check_rms(a); rc != VF_OK) return rc;
    VF_REQUIRE(a.m == 0 || (a.dy && a.rstd), "rms norm: dy or rstd is NULL");
    VF_REQUIRE(a.lddy >= a.d, "rms norm: lddy is less than d");
    VF_REQUIRE(a.y == nullptr || a.ldy >= a.d, "rms norm: lddx is less than d");
    VF_REQUIRE(a.residual == nullptr || a.ldr >= a.d, "rms norm: ld of d_total is less than d");
    const bool sums = a.dweight != nullptr;
    const int64_t parts = parts_of(a.m, a.d);
    const bool at_once = sums_at_once(a.m, a.d);
    const size_t need = sums && !at_once ? (size_t)parts * (size_t)a.d * 4 : 0;
    if (int rc = check_workspace("rms norm", a.workspace, a.workspace_bytes, need); rc != VF_OK) return rc;
    const size_t size = type_size(a.dtype);
    const Region dy = region(a.dy, a.m, a.d, a.lddy, size), dx = region(a.y, a.m, a.d, a.ldy, size), dt = region(a.residual, a.m, a.d, a.ldr, size);
    const Region dw = region(a.dweight, a.d, size);
    VF_REQUIRE((dx.same(dy) || !overlap(dx, dy)) && (dx.same(dt) || !overlap(dx, dt)), "rms norm: dx overlaps dy or d_total and is not it");
    for (const Region &in : {region(a.x, a.m, a.d, a.ldx, size), region(a.rstd, a.m, 4), region(a.weight, a.d, size)})
        VF_REQUIRE(!overlap(dx, in) && !overlap(dw, in), "rms norm: dx or dweight overlaps an input");
    VF_REQUIRE(!overlap(dw, dy) && !overlap(dw, dt) && !overlap(dw, dx), "rms norm: dweight overlaps dy, d_total or dx");
    float *part = at_once ? nullptr : (float *)a.workspace;
    by_type(a.dtype, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        const T *dy = (const T *)a.dy, *s = (const T *)a.x, *w = (const T *)a.weight, *dt = (const T *)a.residual;
        if (a.m == 0) {
            if (sums) launch_join_parts<T>(0, a.d, 1, part, (T *)a.dweight, nullptr, a.stream);
            return;
        }
        const bool short_row = by_eights(eights_of(a.d), [&](auto tpr, auto nv) {
            constexpr int TPR = tpr.value, NV = nv.value;
            const dim3 block(TPR < 256 ? 256 : TPR), grid((unsigned)parts);
            if (sums)
                rms_backward_kernel<T, TPR, NV, true><<<grid, block, 0, a.stream>>>(a.m, (int)a.d, dy, a.lddy, s, a.ldx, a.rstd, w, dt, a.ldr, (T *)a.y,
                                                                                    a.ldy, part, (T *)a.dweight);
            else if (a.y)
                rms_backward_kernel<T, TPR, NV, false><<<grid, block, 0, a.stream>>>(a.m, (int)a.d, dy, a.lddy, s, a.ldx, a.rstd, w, dt, a.ldr, (T *)a.y,
                                                                                     a.ldy, part, (T *)a.dweight);
        });
        if (!short_row) {
            if (sums)   // before dx, which may be written over dy
                rms_columns_kernel<T><<<dim3((unsigned)ceil_div(a.d, 64), (unsigned)parts), dim3(256), 0, a.stream>>>(a.m, a.d, dy, a.lddy, s, a.ldx, a.rstd, part);
            if (a.y)
                rms_backward_long_kernel<T><<<dim3(grid_of(a.m)), dim3(1024), 0, a.stream>>>(a.m, a.d, dy, a.lddy, s, a.ldx, a.rstd, w, dt, a.ldr, (T *)a.y, a.ldy);
        }
        if (sums && !at_once) launch_join_parts<T>((int)parts, a.d, 1, part, (T *)a.dweight, nullptr, a.stream);
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

}  // namespace vf
