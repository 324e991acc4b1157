// Layer norm and its gradients.
//   forward   y = (x - mean) rstd weight + bias, mean and variance over a row of d elements
//   backward  h = (x - mean) rstd, g = dy weight:  dx = rstd (g - avg(g) - h avg(g h)); dweight = sum of dy h and dbias = sum
//             of dy over all rows
// Both are bound by memory: a row is read once, held in registers while its sums are taken (the variance from the centred
// values, in a second pass over the registers, so that a large mean cancels nothing), and written once.
#include "vf_ops.h"

namespace vf {

// Rows of up to TPR * NV vectors: thread t of a row holds vectors t, t + TPR, ...  10,000 x 1,024 in float32: 17 us, 4.8 TB/s (a large
// copy moves 4.9).
template <class T, int TPR, int NV>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_forward_kernel(int64_t m, int d, const T *x, int64_t ldx,
                                                                              const T *__restrict__ weight, const T *__restrict__ bias,
                                                                              float eps, T *y, int64_t ldy,
                                                                              float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    constexpr int V = kVec<T>, RPB = TPR < 256 ? 256 / TPR : 1;
    __shared__ float lds[16];
    const int t = threadIdx.x % TPR;
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < m; row += (int64_t)gridDim.x * RPB) {
        const T *xr = x + row * ldx;
        float v[NV][V];
        float sum[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            if (c < d) {
                const Vec<T> u = load_part(xr + c, d - c, (T)0.f);
#pragma unroll
                for (int j = 0; j < V; ++j) { v[i][j] = (float)u[j]; sum[0] += v[i][j]; }
            }
        }
        row_sums<TPR>(sum, lds);
        const float mean = sum[0] / (float)d;
        float sq[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j < d) { v[i][j] -= mean; sq[0] += v[i][j] * v[i][j]; }
        }
        row_sums<TPR>(sq, lds);
        const float rstd = 1.f / sqrtf(sq[0] / (float)d + eps);
        if (t == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
        T *yr = y + row * ldy;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            if (c >= d) continue;
            Vec<T> w, b, o;
            if (weight) w = load_part(weight + c, d - c, (T)0.f);
            if (bias) b = load_part(bias + c, d - c, (T)0.f);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float r = v[i][j] * rstd;
                if (weight) r *= (float)w[j];
                if (bias) r += (float)b[j];
                o[j] = (T)r;
            }
            store_part(yr + c, o, d - c);
        }
    }
}

// Rows of any length, read three times (the second and third time mostly from the caches).
template <class T>
__global__ __launch_bounds__(1024) void norm_forward_long_kernel(int64_t m, int64_t d, const T *x, int64_t ldx, const T *weight, const T *bias,
                                                                 float eps, T *y, int64_t ldy, float *mean_out, float *rstd_out)
{
    constexpr int V = kVec<T>;
    __shared__ float lds[16];
    for (int64_t row = blockIdx.x; row < m; row += gridDim.x) {
        const T *xr = x + row * ldx;
        float sum[1] = {0.f}, sq[1] = {0.f};
        for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
            const Vec<T> u = load_part(xr + c, (int)min((int64_t)V, d - c), (T)0.f);
#pragma unroll
            for (int j = 0; j < V; ++j) sum[0] += (float)u[j];
        }
        row_sums<1024>(sum, lds);
        const float mean = sum[0] / (float)d;
        for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
            const Vec<T> u = load_part(xr + c, (int)min((int64_t)V, d - c), (T)0.f);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c + j < d) sq[0] += ((float)u[j] - mean) * ((float)u[j] - mean);
        }
        row_sums<1024>(sq, lds);
        const float rstd = 1.f / sqrtf(sq[0] / (float)d + eps);
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
        for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
            const int n = (int)min((int64_t)V, d - c);
            const Vec<T> u = load_part(xr + c, n, (T)0.f);
            Vec<T> w, b, o;
            if (weight) w = load_part(weight + c, n, (T)0.f);
            if (bias) b = load_part(bias + c, n, (T)0.f);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float r = ((float)u[j] - mean) * rstd;
                if (weight) r *= (float)w[j];
                if (bias) r += (float)b[j];
                o[j] = (T)r;
            }
            store_part(y + row * ldy + c, o, n);
        }
    }
}

// dx of the rows blockIdx.x * RPB + w, + gridDim.x * RPB, ...; PARTS: every thread also sums its columns' dy h and dy over
// those rows, and the workgroup leaves one row of both in part [gridDim.x][2][d], or (part NULL: it is the only one) the sums
// themselves in dweight and dbias.  100,000 x 1,024 in bfloat16: 119 us, 5.2 TB/s, and 5 us
// for joining the partial rows.
template <class T, int TPR, int NV, bool PARTS>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_backward_kernel(int64_t m, int d, const T *dy, int64_t lddy,
                                                                               const T *__restrict__ x, int64_t ldx,
                                                                               const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                               const T *__restrict__ weight, T *dx, int64_t lddx,
                                                                               float *__restrict__ part, T *dweight, T *dbias)
{
    constexpr int V = kVec<T>, RPB = TPR < 256 ? 256 / TPR : 1;
    __shared__ float lds[32];
    __shared__ float comb[RPB > 1 && PARTS ? TPR * V * 2 : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    Vec<T> w[NV];
    float aw[NV][V] = {}, ab[NV][V] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * V;
        if (weight && c < d) {
            w[i] = load_part(weight + c, d - c, (T)0.f);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) w[i][j] = (T)1.f;
        }
    }
    for (int64_t row = (int64_t)blockIdx.x * RPB + sub; row < m; row += (int64_t)gridDim.x * RPB) {
        const float mu = mean[row], rs = rstd[row];
        Vec<T> vy[NV], vx[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            if (c < d) {
                vy[i] = load_part(dy + row * lddy + c, d - c, (T)0.f);
                vx[i] = load_part(x + row * ldx + c, d - c, (T)mu);
            }
        }
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            if (c < d) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float y = (float)vy[i][j], h = ((float)vx[i][j] - mu) * rs, g = y * (float)w[i][j];
                    const bool in = c + j < d;
                    s[0] += in ? g : 0.f;
                    s[1] += in ? g * h : 0.f;
                    if constexpr (PARTS) { aw[i][j] += in ? y * h : 0.f; ab[i][j] += y; }
                }
            }
        }
        if (dx) {
            row_sums<TPR>(s, lds);
            const float a = s[0] / (float)d, b = s[1] / (float)d;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TPR) * V;
                if (c < d) {
                    Vec<T> o;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float h = ((float)vx[i][j] - mu) * rs, g = (float)vy[i][j] * (float)w[i][j];
                        o[j] = (T)(rs * ((g - a) - h * b));
                    }
                    store_part(dx + row * lddx + c, o, d - c);
                }
            }
        }
    }
    if constexpr (PARTS && TPR == 16) {   // a wave's four rows first: then every wave has one set of sums, in each of its rows
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                aw[i][j] += __shfl_xor(aw[i][j], 16, 64);
                ab[i][j] += __shfl_xor(ab[i][j], 16, 64);
                aw[i][j] += __shfl_xor(aw[i][j], 32, 64);
                ab[i][j] += __shfl_xor(ab[i][j], 32, 64);
            }
    }
    if constexpr (PARTS) {
        const int group = TPR == 16 ? ((threadIdx.x & 63) < 16 ? threadIdx.x >> 6 : -1) : sub;   // which of `kGroups` sets of sums
        constexpr int kGroups = TPR == 16 ? 4 : RPB;
        float *pw = part + (int64_t)blockIdx.x * 2 * d, *pb = pw + d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            if constexpr (kGroups > 1) {   // the waves' sums, one wave after the other
                for (int r = kGroups - 1; r > 0; --r) {
                    __syncthreads();
                    if (group == r) {
#pragma unroll
                        for (int j = 0; j < V; ++j) { comb[(j * 2) * TPR + t] = aw[i][j]; comb[(j * 2 + 1) * TPR + t] = ab[i][j]; }
                    }
                    __syncthreads();
                    if (group == 0) {
#pragma unroll
                        for (int j = 0; j < V; ++j) { aw[i][j] += comb[(j * 2) * TPR + t]; ab[i][j] += comb[(j * 2 + 1) * TPR + t]; }
                    }
                }
            }
            if (group == 0) {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (c + j < d) {
                        if (part) {
                            pw[c + j] = aw[i][j];
                            pb[c + j] = ab[i][j];
                        } else {
                            if (dweight) dweight[c + j] = (T)aw[i][j];
                            if (dbias) dbias[c + j] = (T)ab[i][j];
                        }
                    }
            }
        }
    }
}

// dx of rows of any length, one workgroup each; read twice (2,000 x 20,000 in bfloat16: 102 us with the column sums below, twice the time
// of one reading and writing).
template <class T>
__global__ __launch_bounds__(1024) void norm_backward_long_kernel(int64_t m, int64_t d, const T *dy, int64_t lddy, const T *x, int64_t ldx,
                                                                  const float *mean, const float *rstd, const T *weight, T *dx, int64_t lddx)
{
    constexpr int V = kVec<T>;
    __shared__ float lds[32];
    for (int64_t row = blockIdx.x; row < m; row += gridDim.x) {
        const float mu = mean[row], rs = rstd[row];
        float s[2] = {0.f, 0.f};
        for (int pass = 0; pass < 2; ++pass) {
            const float a = s[0] / (float)d, b = s[1] / (float)d;
            for (int64_t c = (int64_t)threadIdx.x * V; c < d; c += 1024 * V) {
                const int n = (int)min((int64_t)V, d - c);
                const Vec<T> vy = load_part(dy + row * lddy + c, n, (T)0.f), vx = load_part(x + row * ldx + c, n, (T)0.f);
                Vec<T> w, o;
                if (weight) w = load_part(weight + c, n, (T)0.f);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float h = ((float)vx[j] - mu) * rs, g = (float)vy[j] * (weight ? (float)w[j] : 1.f);
                    if (pass == 0 && j < n) { s[0] += g; s[1] += g * h; }
                    o[j] = (T)(rs * ((g - a) - h * b));
                }
                if (pass == 1) store_part(dx + row * lddx + c, o, n);
            }
            if (pass == 0) row_sums<1024>(s, lds);
        }
    }
}

// The same partial sums for rows of any length: blockIdx.x takes 64 columns, blockIdx.y every gridDim.y-th group of 4 rows.
template <class T>
__global__ __launch_bounds__(256) void norm_columns_kernel(int64_t m, int64_t d, const T *dy, int64_t lddy, const T *x, int64_t ldx,
                                                           const float *mean, const float *rstd, float *part)
{
    __shared__ float comb[2][4][64];
    const int t = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + t;
    float aw = 0.f, ab = 0.f;
    if (c < d) {
        for (int64_t row = (int64_t)blockIdx.y * 4 + sub; row < m; row += (int64_t)gridDim.y * 4) {
            const float y = (float)dy[row * lddy + c], h = ((float)x[row * ldx + c] - mean[row]) * rstd[row];
            aw += y * h;
            ab += y;
        }
    }
    comb[0][sub][t] = aw;
    comb[1][sub][t] = ab;
    __syncthreads();
    if (sub < 2 && c < d)
        part[((int64_t)blockIdx.y * 2 + sub) * d + c] = (comb[sub][0][t] + comb[sub][1][t]) + (comb[sub][2][t] + comb[sub][3][t]);
}

// Calls fn(threads per row, vectors per thread) as constants for rows of nv vectors; false: no such kernel, the row is too long.
// A wave takes rows of up to four vectors a lane by itself; beyond that the row's sums would keep too many registers.  Rows of up to 32
// vectors, the index's own dimensions among them, take sixteen lanes each: a wave's instructions then serve four rows.
template <class F> static bool by_row(int64_t nv, F &&fn)
{
    if (nv <= 16) fn(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    else if (nv <= 32) fn(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
    else if (nv <= 64) fn(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    else if (nv <= 128) fn(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    else if (nv <= 256) fn(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
    else if (nv <= 512) fn(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    else if (nv <= 1024) fn(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
    else if (nv <= 2048) fn(std::integral_constant<int, 512>(), std::integral_constant<int, 4>());
    else return false;
    return true;
}

constexpr int64_t kMaxRow = 1 << 24;   // elements of a row

static int64_t vectors_of(int32_t dtype, int64_t d) { return ceil_div(d, 16 / (int64_t)type_size(dtype)); }

// Workgroups (and so partial rows) of the backward pass: 1,024 where there are many rows, so that the partial rows' way through memory
// stays small beside the operands' (5,000 rows of 8,192: 110 us with 1,024, 79 with 512; of 1,200 such rows the 512 partial ones are more than half
// of what is moved: 47 us for 12 of operands).
static int64_t parts_of(int32_t dtype, int64_t m, int64_t d)
{
    const int64_t nv = vectors_of(dtype, d);
    if (m <= (nv <= 32 ? 32 : nv <= 256 ? 8 : 0)) return 1;   // two rows a wave, or two times four: less than one more launch
    const int64_t most = std::max<int64_t>(512, std::min<int64_t>(1024, m / 16));
    if (nv <= 32) return std::min(ceil_div(m, 16), most);
    if (nv <= 256) return std::min(ceil_div(m, 4), most);
    if (nv <= 2048) return std::min(m, most);
    return std::min<int64_t>(ceil_div(m, 4), 64);
}

// Whether the only workgroup of the backward pass writes the weights' gradients itself.
static bool sums_at_once(int32_t dtype, int64_t m, int64_t d) { return vectors_of(dtype, d) <= 256 && parts_of(dtype, m, d) == 1; }

static int check_norm(const NormArgs &a)
{
    VF_REQUIRE(is_float_type(a.dtype), "layer norm: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(a.m >= 0 && a.m <= kMaxExtent, "layer norm: m out of range");
    VF_REQUIRE(a.d >= 1 && a.d <= kMaxRow, "layer norm: d must be 1 .. 2^24");
    VF_REQUIRE(a.m == 0 || a.x != nullptr, "layer norm: x is NULL");
    VF_REQUIRE(a.ldx >= a.d, "layer norm: ldx is less than d");
    return VF_OK;
}

int layer_norm_impl(const NormArgs &a)
{
    if (int rc = check_norm(a); rc != VF_OK) return rc;
    VF_REQUIRE(a.eps >= 0 && std::isfinite(a.eps), "layer norm: eps must be finite and not negative");
    VF_REQUIRE(a.m == 0 || a.y != nullptr, "layer norm: y is NULL");
    VF_REQUIRE(a.ldy >= a.d, "layer norm: ldy is less than d");
    if (a.m == 0) return VF_OK;
    const size_t size = type_size(a.dtype);
    const Region x = region(a.x, a.m, a.d, a.ldx, size), y = region(a.y, a.m, a.d, a.ldy, size);
    const Region mean = region(a.mean, a.m, 4), rstd = region(a.rstd, a.m, 4);
    VF_REQUIRE(y.same(x) || !overlap(y, x), "layer norm: y overlaps x and is not it");
    VF_REQUIRE(!overlap(mean, x) && !overlap(rstd, x), "layer norm: mean or rstd overlaps x");
    for (const Region &in : {region(a.weight, a.d, size), region(a.bias, a.d, size)})
        VF_REQUIRE(!overlap(y, in) && !overlap(mean, in) && !overlap(rstd, in), "layer norm: an output overlaps weight or bias");
    VF_REQUIRE(!overlap(mean, y) && !overlap(rstd, y) && !overlap(mean, rstd), "layer norm: y, mean and rstd overlap each other");
    by_type(a.dtype, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        const bool short_row = by_row(vectors_of(a.dtype, a.d), [&](auto tpr, auto nv) {
            constexpr int TPR = tpr.value, NV = nv.value;
            const int64_t blocks = TPR < 256 ? ceil_div(a.m, 256 / TPR) : a.m;
            norm_forward_kernel<T, TPR, NV><<<dim3(grid_of(blocks)), dim3(TPR < 256 ? 256 : TPR), 0, a.stream>>>(
                a.m, (int)a.d, (const T *)a.x, a.ldx, (const T *)a.weight, (const T *)a.bias, (float)a.eps, (T *)a.y, a.ldy, a.mean, a.rstd);
        });
        if (!short_row)
            norm_forward_long_kernel<T><<<dim3(grid_of(a.m)), dim3(1024), 0, a.stream>>>(
                a.m, a.d, (const T *)a.x, a.ldx, (const T *)a.weight, (const T *)a.bias, (float)a.eps, (T *)a.y, a.ldy, a.mean, a.rstd);
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

int layer_norm_workspace_impl(int32_t dtype, int64_t m, int64_t d, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "layer norm: bytes is NULL");
    VF_REQUIRE(is_float_type(dtype), "layer norm: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && d >= 1 && d <= kMaxRow, "layer norm: sizes out of range");
    *bytes = sums_at_once(dtype, m, d) ? 0 : (size_t)parts_of(dtype, m, d) * 2 * (size_t)d * 4;
    return VF_OK;
}

int layer_norm_backward_impl(const NormArgs &a)
{
    if (int rc = check_norm(a); rc != VF_OK) return rc;
    VF_REQUIRE(a.m == 0 || (a.dy && a.mean && a.rstd), "layer norm: dy, mean or rstd is NULL");
    VF_REQUIRE(a.lddy >= a.d, "layer norm: lddy is less than d");
    VF_REQUIRE(a.y == nullptr || a.ldy >= a.d, "layer norm: lddx is less than d");
    const bool sums = a.dweight != nullptr || a.dbias != nullptr;
    const int64_t parts = parts_of(a.dtype, a.m, a.d);
    const bool at_once = sums_at_once(a.dtype, a.m, a.d);
    const size_t need = sums && !at_once ? (size_t)parts * 2 * (size_t)a.d * 4 : 0;
    if (int rc = check_workspace("layer norm", a.workspace, a.workspace_bytes, need); rc != VF_OK) return rc;
    const size_t size = type_size(a.dtype);
    const Region dy = region(a.dy, a.m, a.d, a.lddy, size), dx = region(a.y, a.m, a.d, a.ldy, size);
    const Region dw = region(a.dweight, a.d, size), db = region(a.dbias, a.d, size);
    VF_REQUIRE(dx.same(dy) || !overlap(dx, dy), "layer norm: dx overlaps dy and is not it");
    VF_REQUIRE(!overlap(dw, dy) && !overlap(db, dy), "layer norm: dweight or dbias overlaps dy");
    for (const Region &in : {region(a.x, a.m, a.d, a.ldx, size), region(a.mean, a.m, 4), region(a.rstd, a.m, 4), region(a.weight, a.d, size)})
        VF_REQUIRE(!overlap(dx, in) && !overlap(dw, in) && !overlap(db, in), "layer norm: dx, dweight or dbias overlaps an input");
    VF_REQUIRE(!overlap(dx, dw) && !overlap(dx, db) && !overlap(dw, db), "layer norm: dx, dweight and dbias overlap each other");
    float *part = at_once ? nullptr : (float *)a.workspace;
    by_type(a.dtype, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        const T *dy = (const T *)a.dy, *x = (const T *)a.x, *w = (const T *)a.weight;
        if (a.m == 0) {
            if (sums) launch_join_parts<T>(0, a.d, 2, part, (T *)a.dweight, (T *)a.dbias, a.stream);
            return;
        }
        const bool short_row = by_row(vectors_of(a.dtype, a.d), [&](auto tpr, auto nv) {
            constexpr int TPR = tpr.value, NV = nv.value;
            const dim3 block(TPR < 256 ? 256 : TPR), grid((unsigned)parts);
            if (sums)
                norm_backward_kernel<T, TPR, NV, true><<<grid, block, 0, a.stream>>>(a.m, (int)a.d, dy, a.lddy, x, a.ldx, a.mean,
                                                                                     a.rstd, w, (T *)a.y, a.ldy, part, (T *)a.dweight, (T *)a.dbias);
            else if (a.y)
                norm_backward_kernel<T, TPR, NV, false><<<grid, block, 0, a.stream>>>(a.m, (int)a.d, dy, a.lddy, x, a.ldx, a.mean,
                                                                                      a.rstd, w, (T *)a.y, a.ldy, part, (T *)a.dweight, (T *)a.dbias);
        });
        if (!short_row) {
            if (sums)   // before dx, which may be written over dy
                norm_columns_kernel<T><<<dim3((unsigned)ceil_div(a.d, 64), (unsigned)parts), dim3(256), 0, a.stream>>>(
                    a.m, a.d, dy, a.lddy, x, a.ldx, a.mean, a.rstd, part);
            if (a.y)
                norm_backward_long_kernel<T><<<dim3(grid_of(a.m)), dim3(1024), 0, a.stream>>>(a.m, a.d, dy, a.lddy, x, a.ldx, a.mean,
                                                                                               a.rstd, w, (T *)a.y, a.ldy);
        }
        if (sums && !at_once)
            launch_join_parts<T>((int)parts, a.d, 2, part, (T *)a.dweight, (T *)a.dbias, a.stream);
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

}  // namespace vf
