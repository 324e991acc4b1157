// The linear layer y = act(x w^T + bias) + residual and its gradients: three matrix products on the matrix cores that share
// one kernel (vf_product.h),
//     forward   P = w  (along c),      Q = x  (along c),     c = k
//     dx        P = w  (along rows),   Q = dz (along c),     c = n
//     dw        P = x  (along rows),   Q = dz (along rows),  c = m
#include "vf_product.h"

namespace vf {

// dz = dy act'(z), and column sums of it: blockIdx.x has 64 vectors of columns, blockIdx.y every gridDim.y-th group of four rows;
// one partial row each, or (dbias given: there is one) the sums themselves.  Bound by memory: 10,000 x 4,096 in bfloat16 47 us, 5.2 TB/s.  (Computed
// while the products load their operands, the slope would be taken once per tile that reads it.)
// dz is rounded to T, which the matrix cores take beside w and x; the sums are not.  That rounding is all that dx and dw differ by from ones of
// an unrounded dz: 0.0024 of their size instead of the 0.0017 of their own rounding (bfloat16).  Two terms per dz would hold it and double both
// products; a caller who needs more digits calls with float32.
template <class T, int ACT>
__global__ __launch_bounds__(256) void slope_kernel(int64_t m, int64_t n, const T *__restrict__ dy, int64_t lddy, const T *__restrict__ z,
                                                    int64_t ldz, T *__restrict__ dz, float *__restrict__ part, T *__restrict__ dbias)
{
    constexpr int V = kVec<T>;
    __shared__ float comb[3][V][64];
    const int t = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + t) * V;
    const int cols = (int)max((int64_t)0, min((int64_t)V, n - c));
    float sum[V] = {};
    if (cols > 0) {
        for (int64_t row = (int64_t)blockIdx.y * 4 + sub; row < m; row += (int64_t)gridDim.y * 4) {
            const Vec<T> g = load_part(dy + row * lddy + c, cols, (T)0.f);
            Vec<T> u, o;
            if (ACT != VF_ACT_NONE) u = load_part(z + row * ldz + c, cols, (T)0.f);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = ACT == VF_ACT_NONE ? (float)g[j] : (float)g[j] * act_slope<ACT, T>((float)u[j]);
                sum[j] += d;
                o[j] = (T)d;
            }
            if (dz) store_part(dz + row * n + c, o, cols);
        }
    }
    if (part == nullptr && dbias == nullptr) return;
    if (sub > 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) comb[sub - 1][j][t] = sum[j];
    }
    __syncthreads();
    if (sub == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < cols) {
                const float s = (sum[j] + comb[0][j][t]) + (comb[1][j][t] + comb[2][j][t]);
                if (dbias) dbias[c + j] = (T)s;
                else part[(int64_t)blockIdx.y * n + c + j] = s;
            }
    }
}

// ---------------------------------------------------------------- host side

// What the backward pass takes of its workspace: dz, the partial column sums, the splits of a product (one at a time).
struct BackwardPlan {
    size_t dz, parts, product;
    int64_t row_parts;
    size_t total() const { return rounded(dz) + rounded(parts) + product; }
};
static BackwardPlan plan_backward(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act)
{
    BackwardPlan b;
    const int64_t across = ceil_div(n, 64 * (16 / (int64_t)type_size(dtype)));
    b.row_parts = m <= 32 ? 1 : std::max<int64_t>(1, std::min<int64_t>(ceil_div(m, 4), 1024 / std::max<int64_t>(1, std::min<int64_t>(across, 1024))));
    b.dz = act == VF_ACT_NONE ? 0 : (size_t)m * n * type_size(dtype);
    b.parts = b.row_parts == 1 ? 0 : (size_t)b.row_parts * n * 4;   // (one: the sums are written at once, which saves a launch)
    b.product = std::max(most_bytes(dtype, k, m, n, false, true, false), most_bytes(dtype, k, n, m, false, false, false));
    return b;
}

constexpr int64_t kMaxWidth = 1 << 25;   // of n and k: kernels give up to 64 threads to a column, a launch holds fewer than 2^32

static const char *const kTooManyTiles = "linear: too many output tiles in one call";

static int check_sizes(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act)
{
    VF_REQUIRE(is_float_type(dtype), "linear: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && n >= 0 && n <= kMaxWidth && k >= 0 && k <= kMaxWidth, "linear: m, n or k out of range");
    VF_REQUIRE(act >= VF_ACT_NONE && act <= VF_ACT_SILU, "linear: unknown activation");
    return VF_OK;
}

int linear_workspace_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act, int32_t backward, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "linear: bytes is NULL");
    if (int rc = check_sizes(dtype, m, n, k, act); rc != VF_OK) return rc;
    *bytes = backward ? plan_backward(dtype, m, n, k, act).total() : most_bytes(dtype, n, m, k, true, true, costly(act));
    return VF_OK;
}

int linear_impl(const LinearArgs &a)
{
    if (int rc = check_sizes(a.dtype, a.m, a.n, a.k, a.act); rc != VF_OK) return rc;
    if (a.m == 0 || a.n == 0) return VF_OK;
    VF_REQUIRE((a.x && a.w) || a.k == 0, "linear: x or w is NULL");
    VF_REQUIRE(a.y != nullptr, "linear: y is NULL");
    VF_REQUIRE(a.ldx >= a.k && a.ldw >= a.k, "linear: ldx or ldw is less than k");
    VF_REQUIRE(a.ldy >= a.n && (!a.z || a.ldz >= a.n) && (!a.residual || a.ldr >= a.n), "linear: ldy, ldz or ldr is less than n");
    const ProductPlan plan = plan_product(a.dtype, a.n, a.m, a.k, {true, true, costly(a.act), direct_rows(a.dtype, a.x, a.ldx) && direct_rows(a.dtype, a.w, a.ldw)});
    VF_REQUIRE(plan.fits, kTooManyTiles);
    if (int rc = check_workspace("linear", a.workspace, a.workspace_bytes, plan.bytes); rc != VF_OK) return rc;
    const size_t size = type_size(a.dtype);
    const Region y = region(a.y, a.m, a.n, a.ldy, size), z = region(a.z, a.m, a.n, a.ldz, size), r = region(a.residual, a.m, a.n, a.ldr, size);
    for (const Region &in : {region(a.x, a.m, a.k, a.ldx, size), region(a.w, a.n, a.k, a.ldw, size), region(a.bias, a.n, size)})
        VF_REQUIRE(!overlap(y, in) && !overlap(z, in), "linear: y or z overlaps an input");
    VF_REQUIRE(y.same(r) || !overlap(y, r), "linear: y overlaps the residual and is not it");
    VF_REQUIRE(!overlap(z, r) && !overlap(z, y), "linear: z overlaps y or the residual");
    int rc = VF_OK;
    by_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const Epilogue<T> e{(const T *)a.bias, a.act, (const T *)a.residual, a.ldr, (T *)a.y, a.ldy, (T *)a.z, a.ldz};
        rc = run_product<T, true, true>(a.dtype, (const T *)a.w, a.ldw, a.n, (const T *)a.x, a.ldx, a.m, a.k, e, plan, (float *)a.workspace,
                                        a.stream);
    });
    return rc;
}

// The backward pass's two products; dz_rows: whether dz's rows can go to LDS directly.
static void plan_products(const LinearArgs &a, bool dz_rows, ProductPlan &plan_dx, ProductPlan &plan_dw)
{
    if (a.dx) plan_dx = plan_product(a.dtype, a.k, a.m, a.n, {false, true, false, a.k % 8 == 0 && direct_rows(a.dtype, a.w, a.ldw) && dz_rows});
    if (a.dw)
        plan_dw = plan_product(a.dtype, a.k, a.n, a.m,
                               {false, false, false, a.k % 8 == 0 && a.n % 8 == 0 && direct_rows(a.dtype, a.x, a.ldx) && dz_rows});
}

bool linear_backward_fits(const LinearArgs &a)
{
    ProductPlan plan_dx, plan_dw;
    plan_products(a, direct_rows(a.dtype, a.dy, a.lddy), plan_dx, plan_dw);
    return plan_dx.fits && plan_dw.fits;
}

int linear_backward_impl(const LinearArgs &a)
{
    if (int rc = check_sizes(a.dtype, a.m, a.n, a.k, a.act); rc != VF_OK) return rc;
    const bool rows = a.m > 0 && a.n > 0;
    VF_REQUIRE(!rows || a.dy, "linear: dy is NULL");
    VF_REQUIRE(a.lddy >= a.n, "linear: lddy is less than n");
    VF_REQUIRE(!rows || a.act == VF_ACT_NONE || (a.z && a.ldz >= a.n), "linear: z is NULL or ldz less than n");
    VF_REQUIRE(!a.dx || ((a.w || !rows || a.k == 0) && a.ldw >= a.k && a.lddx >= a.k), "linear: dx needs w, and ldw and lddx of at least k");
    VF_REQUIRE(!a.dw || ((a.x || !rows || a.k == 0) && a.ldx >= a.k && a.lddw >= a.k), "linear: dw needs x, and ldx and lddw of at least k");
    const BackwardPlan b = plan_backward(a.dtype, a.m, a.n, a.k, a.act);
    if (int rc = check_workspace("linear", a.workspace, a.workspace_bytes, b.total()); rc != VF_OK) return rc;
    // both products are planned before anything is launched: a call that is refused has changed nothing
    const bool none = a.act == VF_ACT_NONE;
    const void *dz_at = none ? a.dy : a.workspace;
    const int64_t lddz = none ? a.lddy : a.n;
    const bool dz_rows = direct_rows(a.dtype, dz_at, lddz);
    ProductPlan plan_dx, plan_dw;
    plan_products(a, dz_rows, plan_dx, plan_dw);
    VF_REQUIRE(plan_dx.fits && plan_dw.fits, kTooManyTiles);
    const size_t size = type_size(a.dtype);
    const Region dx = region(a.dx, a.m, a.k, a.lddx, size), dw = region(a.dw, a.n, a.k, a.lddw, size), db = region(a.dbias, a.n, size);
    for (const Region &in : {region(a.dy, a.m, a.n, a.lddy, size), region(a.dx ? a.w : nullptr, a.n, a.k, a.ldw, size),
                             region(a.dw ? a.x : nullptr, a.m, a.k, a.ldx, size), region(a.act != VF_ACT_NONE ? a.z : nullptr, a.m, a.n, a.ldz, size)})
        VF_REQUIRE(!overlap(dx, in) && !overlap(dw, in) && !overlap(db, in), "linear: dx, dw or dbias overlaps an input");
    VF_REQUIRE(!overlap(dx, dw) && !overlap(dx, db) && !overlap(dw, db), "linear: dx, dw and dbias overlap each other");
    int rc = VF_OK;
    by_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        T *made = (T *)a.workspace;
        float *parts = (float *)((char *)a.workspace + rounded(b.dz));
        float *splits = (float *)((char *)parts + rounded(b.parts));
        const T *dz = (const T *)dz_at;
        const bool products = (a.dx || a.dw) && a.k > 0;
        if (rows && (a.dbias || (!none && products))) {
            const int64_t across = ceil_div(a.n, 64 * kVec<T>);
            by_act(a.act, [&](auto act) {
                slope_kernel<T, act.value><<<dim3((unsigned)across, (unsigned)b.row_parts), dim3(256), 0, a.stream>>>(
                    a.m, a.n, (const T *)a.dy, a.lddy, (const T *)a.z, a.ldz, !none && products ? made : nullptr,
                    a.dbias && b.row_parts > 1 ? parts : nullptr, b.row_parts == 1 ? (T *)a.dbias : nullptr);
            });
        }
        if (a.dbias && a.n > 0 && (!rows || b.row_parts > 1))
            launch_join_parts<T>(rows ? (int)b.row_parts : 0, a.n, 1, parts, (T *)a.dbias, nullptr, a.stream);
        if (a.dx) {
            const Epilogue<T> e{nullptr, VF_ACT_NONE, nullptr, 0, (T *)a.dx, a.lddx, nullptr, 0};
            rc = run_product<T, false, true>(a.dtype, (const T *)a.w, a.ldw, a.k, dz, lddz, a.m, a.n, e, plan_dx, splits, a.stream);
        }
        if (a.dw && rc == VF_OK) {
            const Epilogue<T> e{nullptr, VF_ACT_NONE, nullptr, 0, (T *)a.dw, a.lddw, nullptr, 0};
            rc = run_product<T, false, false>(a.dtype, (const T *)a.x, a.ldx, a.k, dz, lddz, a.n, a.m, e, plan_dw, splits, a.stream);
        }
    });
    if (rc == VF_OK) VF_HIP(hipGetLastError());
    return rc;
}

int debug_linear_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t product, int32_t direct, int32_t *tiling, int32_t *splits)
{
    if (int rc = check_sizes(dtype, m, n, k, VF_ACT_NONE); rc != VF_OK) return rc;
    VF_REQUIRE(product >= 0 && product <= 2 && tiling && splits, "linear: product must be 0 .. 2, tiling and splits not NULL");
    const Operands o{product == 0, product <= 1, false, direct != 0 && dtype != VF_F32};
    const ProductPlan p = product == 0 ? plan_product(dtype, n, m, k, o) : product == 1 ? plan_product(dtype, k, m, n, o) : plan_product(dtype, k, n, m, o);
    VF_REQUIRE(p.fits, kTooManyTiles);
    *tiling = p.tiling;
    *splits = p.splits;
    return VF_OK;
}

}  // namespace vf
