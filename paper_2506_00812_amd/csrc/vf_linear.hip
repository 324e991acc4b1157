// The linear layer y = act(x w^T + bias) + residual and its gradients: three matrix products on the matrix cores that share
// one kernel.  Every product is written as
//     out[q][p] = sum over c of Q[q][c] P[p][c]
// with each operand either contiguous along c or along its own rows:
//     forward   P = w  (along c),      Q = x  (along c),     c = k
//     dx        P = w  (along rows),   Q = dz (along c),     c = n
//     dw        P = x  (along rows),   Q = dz (along rows),  c = m
// P takes the matrix instruction's first operand, so that a lane's four accumulators are neighbours in a row of the output.
#include "vf_ops.h"

namespace vf {

// A fragment is 16 bytes a lane: lane l has row l % 16 and the elements (l / 16) kVec ... of 64 bytes of the contraction.  float32 takes
// its four elements one after the other, each standing for a product over four of the sixteen c (in the same order on both sides).
__device__ __forceinline__ float4v mma(const Vec<bf16> &p, const Vec<bf16> &q, float4v acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, acc, 0, 0, 0);
}
__device__ __forceinline__ float4v mma(const Vec<f16> &p, const Vec<f16> &q, float4v acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(p, q, acc, 0, 0, 0);
}
__device__ __forceinline__ float4v mma(const Vec<float> &p, const Vec<float> &q, float4v acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(p[i], q[i], acc, 0, 0, 0);
    return acc;
}

template <class T> struct Epilogue {
    const T *bias;       // by p
    int act;
    const T *residual;
    int64_t ldr;
    T *y;
    int64_t ldy;
    T *z;
    int64_t ldz;
};

// Writes n (1 .. 4) neighbouring outputs of row q from column p on.
template <class T>
__device__ __forceinline__ void finish4(const Epilogue<T> &e, int64_t q, int64_t p, int n, float4v a)
{
    using V4 = T __attribute__((ext_vector_type(4)));
    V4 out, pre, res;
    if (e.residual && n == 4) res = load_vec<V4>(e.residual + q * e.ldr + p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= n) break;
        float z = a[i];
        if (e.bias) z += (float)e.bias[p + i];
        pre[i] = (T)z;
        float y = act_value(z, e.act);
        if (e.residual) y += n == 4 ? (float)res[i] : (float)e.residual[q * e.ldr + p + i];
        out[i] = (T)y;
    }
    if (n == 4) {
        if (e.z) store_vec(e.z + q * e.ldz + p, pre);
        store_vec(e.y + q * e.ldy + p, out);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= n) break;
            if (e.z) e.z[q * e.ldz + p + i] = pre[i];
            e.y[q * e.ldy + p + i] = out[i];
        }
    }
}

template <class T> struct Product {
    const T *P, *Q;
    int64_t ldp, ldq;
    int64_t np, nq, nc;   // rows of P and of Q, the contraction's length
    int64_t chunk;        // elements of the contraction per split
    int splits;
    float *part;          // [splits][nq][np] where splits > 1
};

constexpr int kTile = 64;          // rows of either operand per workgroup
constexpr int kRowBytes = 128;     // bytes of the contraction per step

// 64 x 64 outputs per workgroup of four waves, 128 bytes of the contraction per step, staged through LDS by way of registers: any
// alignment, any size.  An LDS row holds its eight 16-byte chunks at chunk ^ (row % 8), which spreads a fragment's reads
// over the banks.
template <class T, bool PC, bool QC>
__global__ __launch_bounds__(256) void product_kernel(Product<T> a, Epilogue<T> e)
{
    constexpr int V = kVec<T>, BC = kRowBytes / (int)sizeof(T);
    __shared__ __align__(16) unsigned char lds[2][kTile * kRowBytes];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t tiles_p = (a.np + kTile - 1) / kTile;
    const int64_t tile = blockIdx.x, p0 = tile % tiles_p * kTile, q0 = tile / tiles_p * kTile;
    const int64_t c_first = (int64_t)blockIdx.y * a.chunk, c_end = min(a.nc, c_first + a.chunk);

    Vec<T> stage[2][2];   // [operand][vector]
    auto load_operand = [&](auto along_c, const T *src, int64_t ld, int64_t r0, int64_t rows, int64_t c0, Vec<T> (&to)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int id = tid + i * 256;
            if constexpr (along_c.value) {
                const int64_t r = r0 + id / 8, c = c0 + id % 8 * V;
                to[i] = load_part(src + r * ld + c, r < rows ? (int)min((int64_t)V, max((int64_t)0, c_end - c)) : 0, (T)0.f);
            } else {
                const int64_t c = c0 + id / (kTile / V), r = r0 + id % (kTile / V) * V;
                to[i] = load_part(src + c * ld + r, c < c_end ? (int)min((int64_t)V, max((int64_t)0, rows - r)) : 0, (T)0.f);
            }
        }
    };
    auto keep_operand = [&](auto along_c, unsigned char *to, const Vec<T> (&from)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int id = tid + i * 256;
            if constexpr (along_c.value) {
                const int r = id / 8, ch = id % 8;
                *(Vec<T> *)(to + r * kRowBytes + ((ch ^ (r & 7)) << 4)) = from[i];
            } else {
                const int c = id / (kTile / V), r = id % (kTile / V) * V;
#pragma unroll
                for (int j = 0; j < V; ++j)
                    *(T *)(to + (r + j) * kRowBytes + ((c / V ^ ((r + j) & 7)) << 4) + c % V * sizeof(T)) = from[i][j];
            }
        }
    };
    using PT = std::integral_constant<bool, PC>;
    using QT = std::integral_constant<bool, QC>;
    const int wp = (wave & 1) * 32, wq = (wave >> 1) * 32;
    float4v acc[2][2] = {};
    if (c_first < c_end) {
        load_operand(PT(), a.P, a.ldp, p0, a.np, c_first, stage[0]);
        load_operand(QT(), a.Q, a.ldq, q0, a.nq, c_first, stage[1]);
    }
    for (int64_t c0 = c_first; c0 < c_end; c0 += BC) {
        __syncthreads();
        keep_operand(PT(), lds[0], stage[0]);
        keep_operand(QT(), lds[1], stage[1]);
        __syncthreads();
        if (c0 + BC < c_end) {
            load_operand(PT(), a.P, a.ldp, p0, a.np, c0 + BC, stage[0]);
            load_operand(QT(), a.Q, a.ldq, q0, a.nq, c0 + BC, stage[1]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Vec<T> fp[2], fq[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int rp = wp + i * 16 + (lane & 15), rq = wq + i * 16 + (lane & 15), ch = h * 4 + (lane >> 4);
                fp[i] = *(const Vec<T> *)(lds[0] + rp * kRowBytes + ((ch ^ (rp & 7)) << 4));
                fq[i] = *(const Vec<T> *)(lds[1] + rq * kRowBytes + ((ch ^ (rq & 7)) << 4));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = mma(fp[i], fq[j], acc[i][j]);
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t q = q0 + wq + j * 16 + (lane & 15);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t p = p0 + wp + i * 16 + (lane >> 4) * 4;
            if (q >= a.nq || p >= a.np) continue;
            const int n = (int)min((int64_t)4, a.np - p);
            if (a.splits > 1) {
                float *to = a.part + ((int64_t)blockIdx.y * a.nq + q) * a.np + p;
                if (n == 4) store_vec(to, acc[i][j]);
                else for (int u = 0; u < n; ++u) to[u] = acc[i][j][u];
            } else {
                finish4(e, q, p, n, acc[i][j]);
            }
        }
    }
}

// The splits' sums, in order, and the epilogue.
template <class T>
__global__ __launch_bounds__(256) void product_join_kernel(int64_t np, int64_t nq, int splits, const float *__restrict__ part, Epilogue<T> e)
{
    const int64_t quads = (np + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quads * nq; i += (int64_t)gridDim.x * 256) {
        const int64_t q = i / quads, p = (i - q * quads) * 4;
        const int n = (int)min((int64_t)4, np - p);
        float4v a = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; ++s) {
            const float *from = part + ((int64_t)s * nq + q) * np + p;
            if (n == 4) a += load_vec<float4v>(from);
            else for (int u = 0; u < n; ++u) a[u] += from[u];
        }
        finish4(e, q, p, n, a);
    }
}

// dz = dy act'(z), and column sums of it: blockIdx.x has 64 vectors of columns, blockIdx.y every gridDim.y-th group of four rows;
// one partial row each.
template <class T>
__global__ __launch_bounds__(256) void slope_kernel(int64_t m, int64_t n, const T *__restrict__ dy, int64_t lddy, const T *__restrict__ z,
                                                    int64_t ldz, int act, T *__restrict__ dz, float *__restrict__ part)
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
            if (act != VF_ACT_NONE) u = load_part(z + row * ldz + c, cols, (T)0.f);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = act == VF_ACT_NONE ? (float)g[j] : (float)g[j] * act_slope((float)u[j], act);
                sum[j] += d;
                o[j] = (T)d;
            }
            if (dz) store_part(dz + row * n + c, o, cols);
        }
    }
    if (part == nullptr) return;
    if (sub > 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) comb[sub - 1][j][t] = sum[j];
    }
    __syncthreads();
    if (sub == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < cols) part[(int64_t)blockIdx.y * n + c + j] = (sum[j] + comb[0][j][t]) + (comb[1][j][t] + comb[2][j][t]);
    }
}

// ---------------------------------------------------------------- host side

struct ProductPlan {
    int splits = 1;
    int64_t chunk = 0;
    size_t bytes = 0;
};

// The contraction is split where there are too few tiles for the chip and it is long enough for that.
static ProductPlan plan_product(int32_t dtype, int64_t np, int64_t nq, int64_t nc)
{
    ProductPlan p;
    const int64_t step = kRowBytes / (int64_t)type_size(dtype);
    const int64_t tiles = ceil_div(np, kTile) * ceil_div(nq, kTile);
    const int64_t most = std::max<int64_t>(1, nc / (4 * step));
    const int64_t splits = tiles >= 256 ? 1 : std::min<int64_t>({ceil_div(512, std::max<int64_t>(1, tiles)), most, 64});
    p.chunk = std::max<int64_t>(step, ceil_div(ceil_div(nc, splits), step) * step);
    p.splits = (int)std::max<int64_t>(1, ceil_div(nc, p.chunk));
    p.bytes = p.splits > 1 ? (size_t)p.splits * nq * np * 4 : 0;
    return p;
}

template <class T, bool PC, bool QC>
static int run_product(int32_t dtype, const T *P, int64_t ldp, int64_t np, const T *Q, int64_t ldq, int64_t nq, int64_t nc,
                       const Epilogue<T> &e, float *part, hipStream_t s)
{
    if (np == 0 || nq == 0) return VF_OK;
    const ProductPlan plan = plan_product(dtype, np, nq, nc);
    const int64_t tiles = ceil_div(np, kTile) * ceil_div(nq, kTile);
    VF_REQUIRE(tiles < (1 << 24), "linear: too many output tiles in one call");
    const Product<T> a{P, Q, ldp, ldq, np, nq, nc, plan.chunk, plan.splits, part};
    product_kernel<T, PC, QC><<<dim3((unsigned)tiles, (unsigned)plan.splits), dim3(256), 0, s>>>(a, e);
    if (plan.splits > 1)
        product_join_kernel<T><<<dim3((unsigned)std::min<int64_t>(ceil_div(ceil_div(np, 4) * nq, 256), 4096)), dim3(256), 0, s>>>(
            np, nq, plan.splits, part, e);
    VF_HIP(hipGetLastError());
    return VF_OK;
}

static size_t rounded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

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
    b.row_parts = std::max<int64_t>(1, std::min<int64_t>(ceil_div(m, 4), 1024 / std::max<int64_t>(1, std::min<int64_t>(across, 1024))));
    b.dz = act == VF_ACT_NONE ? 0 : (size_t)m * n * type_size(dtype);
    b.parts = (size_t)b.row_parts * n * 4;
    b.product = std::max(plan_product(dtype, k, m, n).bytes, plan_product(dtype, k, n, m).bytes);
    return b;
}

static int check_sizes(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act)
{
    VF_REQUIRE(is_float_type(dtype), "linear: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && n >= 0 && n <= kMaxExtent && k >= 0 && k <= kMaxExtent, "linear: m, n or k out of range");
    VF_REQUIRE(act >= VF_ACT_NONE && act <= VF_ACT_SILU, "linear: unknown activation");
    return VF_OK;
}

int linear_workspace_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act, int32_t backward, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "linear: bytes is NULL");
    if (int rc = check_sizes(dtype, m, n, k, act); rc != VF_OK) return rc;
    *bytes = backward ? plan_backward(dtype, m, n, k, act).total() : plan_product(dtype, n, m, k).bytes;
    return VF_OK;
}

int linear_impl(const LinearArgs &a)
{
    size_t need = 0;
    if (int rc = linear_workspace_impl(a.dtype, a.m, a.n, a.k, a.act, 0, &need); rc != VF_OK) return rc;
    if (a.m == 0 || a.n == 0) return VF_OK;
    VF_REQUIRE((a.x && a.w) || a.k == 0, "linear: x or w is NULL");
    VF_REQUIRE(a.y != nullptr, "linear: y is NULL");
    VF_REQUIRE(a.ldx >= a.k && a.ldw >= a.k, "linear: ldx or ldw is less than k");
    VF_REQUIRE(a.ldy >= a.n && (!a.z || a.ldz >= a.n) && (!a.residual || a.ldr >= a.n), "linear: ldy, ldz or ldr is less than n");
    VF_REQUIRE(need == 0 || (a.workspace != nullptr && a.workspace_bytes >= need),
               "linear: the workspace must hold " + std::to_string(need) + " bytes");
    int rc = VF_OK;
    by_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const Epilogue<T> e{(const T *)a.bias, a.act, (const T *)a.residual, a.ldr, (T *)a.y, a.ldy, (T *)a.z, a.ldz};
        rc = run_product<T, true, true>(a.dtype, (const T *)a.w, a.ldw, a.n, (const T *)a.x, a.ldx, a.m, a.k, e, (float *)a.workspace,
                                        a.stream);
    });
    return rc;
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
    VF_REQUIRE(b.total() == 0 || (a.workspace != nullptr && a.workspace_bytes >= b.total()),
               "linear: the workspace must hold " + std::to_string(b.total()) + " bytes");
    int rc = VF_OK;
    by_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        T *made = (T *)a.workspace;
        float *parts = (float *)((char *)a.workspace + rounded(b.dz));
        float *splits = (float *)((char *)parts + rounded(b.parts));
        const T *dz = a.act == VF_ACT_NONE ? (const T *)a.dy : made;
        const int64_t lddz = a.act == VF_ACT_NONE ? a.lddy : a.n;
        const bool products = (a.dx || a.dw) && a.k > 0;
        if (rows && (a.dbias || (a.act != VF_ACT_NONE && products))) {
            const int64_t across = ceil_div(a.n, 64 * kVec<T>);
            slope_kernel<T><<<dim3((unsigned)across, (unsigned)b.row_parts), dim3(256), 0, a.stream>>>(
                a.m, a.n, (const T *)a.dy, a.lddy, (const T *)a.z, a.ldz, a.act, a.act != VF_ACT_NONE && products ? made : nullptr,
                a.dbias ? parts : nullptr);
        }
        if (a.dbias && a.n > 0)
            launch_join_parts<T>(rows ? (int)b.row_parts : 0, a.n, 1, parts, (T *)a.dbias, nullptr, a.stream);
        if (a.dx) {
            const Epilogue<T> e{nullptr, VF_ACT_NONE, nullptr, 0, (T *)a.dx, a.lddx, nullptr, 0};
            rc = run_product<T, false, true>(a.dtype, (const T *)a.w, a.ldw, a.k, dz, lddz, a.m, a.n, e, splits, a.stream);
        }
        if (a.dw && rc == VF_OK) {
            const Epilogue<T> e{nullptr, VF_ACT_NONE, nullptr, 0, (T *)a.dw, a.lddw, nullptr, 0};
            rc = run_product<T, false, false>(a.dtype, (const T *)a.x, a.ldx, a.k, dz, lddz, a.n, a.m, e, splits, a.stream);
        }
    });
    if (rc == VF_OK) VF_HIP(hipGetLastError());
    return rc;
}

}  // namespace vf
