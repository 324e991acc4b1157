// The gated layer y = act(x Wg^T + bg) (x Wu^T + bu) and its gradients.  W holds the rows of Wg and then those of Wu, z = x W^T + b both
// pre-activations side by side, so that
//     forward    one product over all 2 n rows of W, whose tiles have both halves of their outputs (vf_product.h, GATED)
//     backward   dz = [dy up act'(gate) | dy act(gate)], elementwise;  dx = dz W, dw = dz^T x, the linear layer's own products
#include "vf_product.h"

namespace vf {

// dz and column sums of it: blockIdx.x has 64 vectors of columns of each half, blockIdx.y every gridDim.y-th group of four rows; one partial row
// [2][n] each, or (dbias given: there is one) the sums themselves.  Bound by memory: dy and z read, dz written.  dz is rounded
// to T, which the matrix cores take beside w and x (the linear layer's choice too; dx and dw are off by 0.0024 of their size in bfloat16, 0.0017 without it, and two
// terms of dz would take both products twice as long); the sums take it before that.  10,000 x 4,096 in bfloat16: 410 MB in 70 us
// (5.9 TB/s), the partial rows' join 5.  Kept apart from the products: dz is an operand of both, and each reads it many times over.
template <class T, int ACT>
__global__ __launch_bounds__(256) void gated_slope_kernel(int64_t m, int64_t n, const T *__restrict__ dy, int64_t lddy, const T *__restrict__ z,
                                                          int64_t ldz, T *__restrict__ dz, float *__restrict__ part, T *__restrict__ dbias)
{
    constexpr int V = kVec<T>;
    __shared__ float comb[3][2][V][64];
    const int t = threadIdx.x & 63, sub = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + t) * V;
    const int cols = (int)max((int64_t)0, min((int64_t)V, n - c));
    float sum[2][V] = {};
    if (cols > 0) {
        for (int64_t row = (int64_t)blockIdx.y * 4 + sub; row < m; row += (int64_t)gridDim.y * 4) {
            const Vec<T> d = load_part(dy + row * lddy + c, cols, (T)0.f);
            const Vec<T> gate = load_part(z + row * ldz + c, cols, (T)0.f), up = load_part(z + row * ldz + n + c, cols, (T)0.f);
            Vec<T> o[2];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float dg = (float)d[j] * (float)up[j] * act_slope<ACT, T>((float)gate[j]);
                const float du = (float)d[j] * act_value<ACT, T>((float)gate[j]);
                sum[0][j] += dg;
                sum[1][j] += du;
                o[0][j] = (T)dg;
                o[1][j] = (T)du;
            }
            if (dz) {
                store_part(dz + row * 2 * n + c, o[0], cols);
                store_part(dz + row * 2 * n + n + c, o[1], cols);
            }
        }
    }
    if (part == nullptr && dbias == nullptr) return;
    if (sub > 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < V; ++j) comb[sub - 1][h][j][t] = sum[h][j];
    }
    __syncthreads();
    if (sub == 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < cols) {
                    const float s = (sum[h][j] + comb[0][h][j][t]) + (comb[1][h][j][t] + comb[2][h][j][t]);
                    if (dbias) dbias[h * n + c + j] = (T)s;
                    else part[((int64_t)blockIdx.y * 2 + h) * n + c + j] = s;
                }
    }
}

constexpr int64_t kMaxGated = 1 << 24;   // of n: the products have rows of 2 n
static const char *const kTooManyGatedTiles = "gated linear: too many output tiles in one call";

static int check_gated(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act)
{
    VF_REQUIRE(is_float_type(dtype), "gated linear: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && n >= 0 && n <= kMaxGated && k >= 0 && k <= 2 * kMaxGated, "gated linear: m, n or k out of range");
    VF_REQUIRE(act >= VF_ACT_NONE && act <= VF_ACT_SILU, "gated linear: unknown activation");
    return VF_OK;
}

// What the backward pass takes of its workspace: dz, the partial column sums, what the linear layer's backward pass takes.
struct GatedBackward {
    size_t dz, parts, products;
    int64_t row_parts;
    size_t total() const { return rounded(dz) + rounded(parts) + products; }
};
static int plan_gated_backward(int32_t dtype, int64_t m, int64_t n, int64_t k, GatedBackward &b)
{
    const int64_t across = ceil_div(n, 64 * (16 / (int64_t)type_size(dtype)));
    b.row_parts = m <= 32 ? 1 : std::max<int64_t>(1, std::min<int64_t>(ceil_div(m, 4), 1024 / std::max<int64_t>(1, std::min<int64_t>(across, 1024))));
    b.dz = (size_t)m * 2 * n * type_size(dtype);
    b.parts = b.row_parts == 1 ? 0 : (size_t)b.row_parts * 2 * n * 4;
    return linear_workspace_impl(dtype, m, 2 * n, k, VF_ACT_NONE, 1, &b.products);
}

int gated_linear_workspace_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act, int32_t backward, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "gated linear: bytes is NULL");
    if (int rc = check_gated(dtype, m, n, k, act); rc != VF_OK) return rc;
    if (!backward) {
        *bytes = most_bytes(dtype, 2 * n, m, k, true, true, costly(act), true);
        return VF_OK;
    }
    GatedBackward b;
    if (int rc = plan_gated_backward(dtype, m, n, k, b); rc != VF_OK) return rc;
    *bytes = b.total();
    return VF_OK;
}

// The forward product's plan; direct: whether both operands' rows can go to LDS directly.
static ProductPlan plan_gated(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act, bool direct)
{
    return plan_product(dtype, 2 * n, m, k, {true, true, costly(act), direct, true});
}

int debug_gated_linear_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act, int32_t direct, int32_t *tiling, int32_t *splits)
{
    if (int rc = check_gated(dtype, m, n, k, act); rc != VF_OK) return rc;
    VF_REQUIRE(tiling && splits, "gated linear: tiling or splits is NULL");
    const ProductPlan p = plan_gated(dtype, m, n, k, act, direct != 0 && dtype != VF_F32);
    VF_REQUIRE(p.fits, kTooManyGatedTiles);
    *tiling = p.tiling;
    *splits = p.splits;
    return VF_OK;
}

int gated_linear_impl(const LinearArgs &a)
{
    if (int rc = check_gated(a.dtype, a.m, a.n, a.k, a.act); rc != VF_OK) return rc;
    if (a.m == 0 || a.n == 0) return VF_OK;
    VF_REQUIRE((a.x && a.w) || a.k == 0, "gated linear: x or w is NULL");
    VF_REQUIRE(a.y != nullptr, "gated linear: y is NULL");
    VF_REQUIRE(a.ldx >= a.k && a.ldw >= a.k, "gated linear: ldx or ldw is less than k");
    VF_REQUIRE(a.ldy >= a.n && (!a.z || a.ldz >= 2 * a.n), "gated linear: ldy is less than n or ldz less than 2 n");
    const ProductPlan plan = plan_gated(a.dtype, a.m, a.n, a.k, a.act, direct_rows(a.dtype, a.x, a.ldx) && direct_rows(a.dtype, a.w, a.ldw));
    VF_REQUIRE(plan.fits, kTooManyGatedTiles);
    if (int rc = check_workspace("gated linear", a.workspace, a.workspace_bytes, plan.bytes); rc != VF_OK) return rc;
    const size_t size = type_size(a.dtype);
    const Region y = region(a.y, a.m, a.n, a.ldy, size), z = region(a.z, a.m, 2 * a.n, a.ldz, size);
    for (const Region &in : {region(a.x, a.m, a.k, a.ldx, size), region(a.w, 2 * a.n, a.k, a.ldw, size), region(a.bias, 2 * a.n, size)})
        VF_REQUIRE(!overlap(y, in) && !overlap(z, in), "gated linear: y or z overlaps an input");
    VF_REQUIRE(!overlap(z, y), "gated linear: z overlaps y");
    int rc = VF_OK;
    by_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const Epilogue<T> e{(const T *)a.bias, a.act, nullptr, 0, (T *)a.y, a.ldy, (T *)a.z, a.ldz};
        rc = run_product<T, true, true, true>(a.dtype, (const T *)a.w, a.ldw, a.n, (const T *)a.x, a.ldx, a.m, a.k, e, plan, (float *)a.workspace, a.stream);
    });
    return rc;
}

int gated_linear_backward_impl(const LinearArgs &a)
{
    if (int rc = check_gated(a.dtype, a.m, a.n, a.k, a.act); rc != VF_OK) return rc;
    const bool rows = a.m > 0 && a.n > 0;
    VF_REQUIRE(!rows || (a.dy && a.z), "gated linear: dy or z is NULL");
    VF_REQUIRE(a.lddy >= a.n && a.ldz >= 2 * a.n, "gated linear: lddy is less than n or ldz less than 2 n");
    VF_REQUIRE(!a.dx || ((a.w || !rows || a.k == 0) && a.ldw >= a.k && a.lddx >= a.k), "gated linear: dx needs w, and ldw and lddx of at least k");
    VF_REQUIRE(!a.dw || ((a.x || !rows || a.k == 0) && a.ldx >= a.k && a.lddw >= a.k), "gated linear: dw needs x, and ldx and lddw of at least k");
    GatedBackward b;
    if (int rc = plan_gated_backward(a.dtype, a.m, a.n, a.k, b); rc != VF_OK) return rc;
    if (int rc = check_workspace("gated linear", a.workspace, a.workspace_bytes, b.total()); rc != VF_OK) return rc;
    const size_t size = type_size(a.dtype);
    const Region dx = region(a.dx, a.m, a.k, a.lddx, size), dw = region(a.dw, 2 * a.n, a.k, a.lddw, size), db = region(a.dbias, 2 * a.n, size);
    for (const Region &in : {region(a.dy, a.m, a.n, a.lddy, size), region(a.z, a.m, 2 * a.n, a.ldz, size),
                             region(a.dx ? a.w : nullptr, 2 * a.n, a.k, a.ldw, size), region(a.dw ? a.x : nullptr, a.m, a.k, a.ldx, size)})
        VF_REQUIRE(!overlap(dx, in) && !overlap(dw, in) && !overlap(db, in), "gated linear: dx, dw or dbias overlaps an input");
    VF_REQUIRE(!overlap(dx, dw) && !overlap(dx, db) && !overlap(dw, db), "gated linear: dx, dw and dbias overlap each other");
    const bool products = a.dx || a.dw;
    LinearArgs p = a;   // the two products of dz
    p.act = VF_ACT_NONE;
    p.n = 2 * a.n;
    p.dy = a.workspace;
    p.lddy = 2 * a.n;
    p.z = nullptr;
    p.dbias = nullptr;
    p.workspace = (char *)a.workspace + rounded(b.dz) + rounded(b.parts);
    p.workspace_bytes = b.products;
    if (products) VF_REQUIRE(linear_backward_fits(p), kTooManyGatedTiles);   // (before anything is enqueued)
    const bool keep = products && a.k > 0;
    by_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        float *parts = (float *)((char *)a.workspace + rounded(b.dz));
        if (rows && (a.dbias || keep)) {
            const int64_t across = ceil_div(a.n, 64 * kVec<T>);
            by_act(a.act, [&](auto act) {
                gated_slope_kernel<T, act.value><<<dim3((unsigned)across, (unsigned)b.row_parts), dim3(256), 0, a.stream>>>(
                    a.m, a.n, (const T *)a.dy, a.lddy, (const T *)a.z, a.ldz, keep ? (T *)a.workspace : nullptr,
                    a.dbias && b.row_parts > 1 ? parts : nullptr, b.row_parts == 1 ? (T *)a.dbias : nullptr);
            });
        }
        if (a.dbias && a.n > 0 && (!rows || b.row_parts > 1))
            launch_join_parts<T>(rows ? (int)b.row_parts : 0, a.n, 2, parts, (T *)a.dbias, (T *)a.dbias + a.n, a.stream);
    });
    VF_HIP(hipGetLastError());
    return products ? linear_backward_impl(p) : VF_OK;
}

}  // namespace vf
