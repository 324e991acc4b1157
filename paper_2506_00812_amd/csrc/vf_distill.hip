// The divergence of a student from a teacher that is known by its top entries, and its gradient.  With u = logits / t, v_j = teacher_j / t over the
// entries j that a row has:
//     q = softmax(v), p = softmax(u) over the whole vocabulary, loss = sum over j of q_j (log q_j - log p at id_j)
//     dlogits_i = d_loss / t (p_i - sum of q_j with id_j = i)
// Both are bound by memory: one reading of the logits, and one writing in the gradient.  The entries are few: each wave that works on a row takes
// q anew from the teacher's values.
#include "vf_device.h"
#include "vf_ops.h"

namespace vf {

constexpr float kInf = __builtin_inff();

// Sum exp(u - m) about an origin m, a maximum so far; turned to another one, where a NaN stays and nothing stays of an empty sum.
struct ExpSum {
    float m, s;
};
__device__ __forceinline__ void move_origin(ExpSum &r, float m)
{
    if (r.m == m) return;
    r.s *= exp_fast(r.m - m);
    r.m = m;
}
__device__ __forceinline__ ExpSum wave_join(ExpSum r)
{
    move_origin(r, wave_max(r.m));
    r.s = wave_sum(r.s);
    return r;
}

// A row's entries, entry lane + 64 i in register i of a lane.
template <int R> struct Entries {
    int32_t id[R];
    float u[R];
    float q[R], log_q[R];     // after soften()
    bool any, bad;            // any: there is an entry; bad: an id is outside of the vocabulary
    __device__ __forceinline__ void load(const int32_t *ids, const float *teacher, int64_t row, int64_t v, int top, float inv_t)
    {
        const int lane = threadIdx.x & 63;
        bool wrong = false;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int j = lane + 64 * i;
            id[i] = -1;
            u[i] = -kInf;
            if (j < top) {
                id[i] = ids[row * top + j];
                u[i] = teacher[row * top + j] * inv_t;
                wrong |= id[i] < -1 || id[i] >= v;
            }
            if (u[i] == -kInf || wrong) id[i] = -1;
            if (id[i] < 0) u[i] = -kInf;
        }
        bad = __ballot(wrong) != 0;
    }
    __device__ __forceinline__ void soften()
    {
        float most = -kInf, total = 0.f;
        bool here = false;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            most = fmaxf(most, u[i]);
            here |= id[i] >= 0;
        }
        any = __ballot(here) != 0;
        most = wave_max(most);
        if (most == -kInf) most = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            log_q[i] = u[i] - most;
            q[i] = exp_fast(log_q[i]);
            total += q[i];
        }
        total = wave_sum(total);
        const float log_total = logf(total), inv = 1.f / total;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            log_q[i] -= log_total;
            q[i] = id[i] >= 0 ? q[i] * inv : 0.f;
        }
    }
};

template <class T> struct DistillRow {
    const T *logits;
    int64_t ld, v;
    const int32_t *ids;
    const float *teacher;
    int top;
    float inv_t;
    float *loss, *lse;
};

// What a row's sums say, by the wave that has them.
template <class T, int R> __device__ __forceinline__ void finish_row(const DistillRow<T> &a, const Entries<R> &e, const float (&x)[R], int64_t row, const ExpSum &r)
{
    const bool empty = r.m == -kInf && r.s == 0.f;
    const float log_s = logf(r.s);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const float log_p = empty ? -kInf : (x[i] - r.m) - log_s;
        sum += e.q[i] == 0.f ? 0.f : e.q[i] * (e.log_q[i] - log_p);
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) {
        a.loss[row] = e.bad ? __uint_as_float(0x7FC00000u) : e.any ? sum : 0.f;
        if (a.lse) a.lse[row] = empty ? -kInf : r.m + log_s;
    }
}
template <class T, int R> __device__ __forceinline__ void load_entries(const DistillRow<T> &a, int64_t row, Entries<R> &e, float (&x)[R])
{
    e.load(a.ids, a.teacher, row, a.v, a.top, a.inv_t);
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = e.id[i] >= 0 ? (float)a.logits[row * a.ld + e.id[i]] * a.inv_t : 0.f;
}

// Segment `item % nseg` of a row: TPR threads take its vectors in turn, 16 elements a thread at a time.  nseg > 1: the segment's sums go to
// part [row][nseg].  Sixteen elements have one maximum and at most one change of origin, so that an element costs one exponential.  64 x 200,000 in bfloat16,
// 13 segments a row: 26 MB in 8.0 us and 2.6 for the join; 10,000 x 10,000: 38 us (5.2 TB/s).  (Asking for the next vectors ahead gained nothing.)
template <class T, int TPR, int R>
__global__ __launch_bounds__(256) void distill_kernel(int64_t m, DistillRow<T> a, int nseg, int64_t seg, float2 *__restrict__ part)
{
    constexpr int V = kVec<T>, RPB = 256 / TPR, W = TPR / 64, E = 16, NV = E / V;
    __shared__ float2 sums[4];
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t items = m * nseg;
    for (int64_t item = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; item < items; item += (int64_t)gridDim.x * RPB) {
        const int64_t row = nseg == 1 ? item : item / nseg, sg = nseg == 1 ? 0 : item - row * nseg;
        const T *x = a.logits + row * a.ld;
        const int64_t c0 = sg * seg, c1 = min(a.v, c0 + seg);
        ExpSum r = {-kInf, 0.f};
        Entries<R> entries;
        float asked[R];
        if (nseg == 1 && (W == 1 || wave == 0)) load_entries(a, row, entries, asked);
        for (int64_t base = c0; base < c1; base += TPR * E) {
            float u[E];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = base + (i * TPR + t) * V;
                Vec<T> raw;
                if (base + TPR * E <= c1) raw = load_vec<Vec<T>>(x + c);
                else raw = load_part(x + c, (int)max((int64_t)0, min((int64_t)V, c1 - c)), (T)-kInf);
#pragma unroll
                for (int j = 0; j < V; ++j) u[i * V + j] = (float)raw[j] * a.inv_t;
            }
            float most = u[0];
#pragma unroll
            for (int j = 1; j < E; ++j) most = fmaxf(most, u[j]);
            if (most > r.m) move_origin(r, most);
            const float origin = r.m == -kInf ? 0.f : r.m;
#pragma unroll
            for (int j = 0; j < E; ++j) r.s += exp_fast(u[j] - origin);   // (a NaN, which the maximum passes over, stays in s)
        }
        r = wave_join(r);
        if constexpr (W > 1) {
            __syncthreads();
            if (lane == 0) sums[wave] = make_float2(r.m, r.s);
            __syncthreads();
            if (wave == 0) {
                float most = -kInf;
#pragma unroll
                for (int w = 0; w < W; ++w) most = fmaxf(most, sums[w].x);
                ExpSum all = {most, 0.f};
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    ExpSum p = {sums[w].x, sums[w].y};
                    move_origin(p, most);
                    all.s += p.s;
                }
                r = all;
            }
        }
        if (W == 1 || wave == 0) {
            if (nseg == 1) {
                entries.soften();
                finish_row(a, entries, asked, row, r);
            } else if (lane == 0) {
                part[item] = make_float2(r.m, r.s);
            }
        }
    }
}

// One wave per row joins the segments.
template <class T, int R> __global__ __launch_bounds__(64) void distill_join_kernel(int64_t m, DistillRow<T> a, int nseg, const float2 *__restrict__ part)
{
    for (int64_t row = blockIdx.x; row < m; row += gridDim.x) {
        Entries<R> entries;
        float asked[R];
        load_entries(a, row, entries, asked);
        ExpSum r = {-kInf, 0.f};
        for (int i = threadIdx.x; i < nseg; i += 64) {
            const float2 p = part[row * nseg + i];
            ExpSum q = {p.x, p.y};
            const float most = fmaxf(r.m, q.m);
            move_origin(r, most);
            move_origin(q, most);
            r.s += q.s;
        }
        r = wave_join(r);
        entries.soften();
        finish_row(a, entries, asked, row, r);
    }
}

// A wave has a segment of a row, 512 columns at a time, and all of the row's entries.  Those that fall into its columns leave their q in LDS at their place,
// where the lanes that have these columns find it.  Two entries of the same label would overwrite each other: what is seen by writing
// their numbers there first, and then they are added one after the other.  Bound by memory: 10,000 x 10,000 in bfloat16 with 32 entries a row 82 us (4.9 TB/s),
// 2,000 x 10,000 with 200 19 us, 22 with random labels, some of them twice.
template <class T, int R>
__global__ __launch_bounds__(256) void distill_backward_kernel(int64_t m, int64_t v, const T *logits, int64_t ld, const float *__restrict__ lse,
                                                               const int32_t *__restrict__ ids, const float *__restrict__ teacher, int top,
                                                               const float *__restrict__ d_loss, float inv_t, int nseg, int64_t seg, T *dlogits, int64_t ldd)
{
    constexpr int V = kVec<T>, NV = 8 / V, kTile = 512;
    __shared__ __align__(16) float places[4][kTile];
    const int lane = threadIdx.x & 63;
    float *place = places[threadIdx.x >> 6];
#pragma unroll
    for (int i = 0; i < kTile / 64; ++i) place[i * 64 + lane] = 0.f;
    wave_sync<true>();
    const int64_t items = m * nseg;
    for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * 4) {
        const int64_t row = item / nseg, c0 = (item - row * nseg) * seg, c1 = min(v, c0 + seg);
        Entries<R> e;
        e.load(ids, teacher, row, v, top, inv_t);
        e.soften();
        const float l = lse[row], g = d_loss[row] * inv_t;
        const bool none = l < -0x1p100f || e.bad || !e.any;   // no gradient (so low, l says nothing of how many labels share p)
        for (int64_t base = c0; base < c1; base += kTile) {
            float x[8];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = base + lane * 8 + i * V;
                const Vec<T> raw = load_part(logits + row * ld + c, (int)max((int64_t)0, min((int64_t)V, c1 - c)), (T)-kInf);
#pragma unroll
                for (int j = 0; j < V; ++j) x[i * V + j] = (float)raw[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = exp_fast(x[j] * inv_t - l);
            int at[R];
            bool here = false;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int64_t off = e.id[i] - base;
                at[i] = off >= 0 && off < kTile ? (int)off : -1;
                here |= at[i] >= 0;
            }
            if (__ballot(here)) {
                bool twice = false;
#pragma unroll
                for (int i = 0; i < R; ++i)
                    if (at[i] >= 0) place[at[i]] = __int_as_float(lane + 64 * i);
                wave_sync<true>();
#pragma unroll
                for (int i = 0; i < R; ++i)
                    if (at[i] >= 0) twice |= __float_as_int(place[at[i]]) != lane + 64 * i;
                wave_sync<true>();
                if (__ballot(twice)) {
#pragma unroll
                    for (int i = 0; i < R; ++i)
                        if (at[i] >= 0) place[at[i]] = 0.f;
                    wave_sync<true>();
#pragma unroll
                    for (int i = 0; i < R; ++i)
#pragma unroll 1
                        for (uint64_t left = __ballot(at[i] >= 0); left != 0; left &= left - 1) {
                            if (lane == __ffsll((unsigned long long)left) - 1) place[at[i]] += e.q[i];
                            wave_sync<true>();
                        }
                } else {
#pragma unroll
                    for (int i = 0; i < R; ++i)
                        if (at[i] >= 0) place[at[i]] = e.q[i];
                }
                wave_sync<true>();
                const float4 a = *(const float4 *)(place + lane * 8), b = *(const float4 *)(place + lane * 8 + 4);
                x[0] -= a.x; x[1] -= a.y; x[2] -= a.z; x[3] -= a.w;
                x[4] -= b.x; x[5] -= b.y; x[6] -= b.z; x[7] -= b.w;
                wave_sync<true>();
#pragma unroll
                for (int i = 0; i < R; ++i)
                    if (at[i] >= 0) place[at[i]] = 0.f;
                wave_sync<true>();
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = base + lane * 8 + i * V;
                Vec<T> o;
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = (T)(none ? 0.f : g * x[i * V + j]);
                store_part(dlogits + row * ldd + c, o, (int)max((int64_t)0, min((int64_t)V, c1 - c)));
            }
        }
    }
}

// Threads per row and segments of a row in the forward pass: rows of up to 2,048 elements, of up to 6,144 where there are many, are a wave's (4,096 x 2,100 in
// bfloat16: 7.7 us, a workgroup to a row 11; 20,000 x 5,000: 63 and 69; 10,000 x 8,000: 34 and 31), longer ones a workgroup's, in segments where there are too
// few rows to fill the chip.
struct DistillPlan {
    int tpr, nseg;
    int64_t seg;
};
static DistillPlan plan_of(int64_t m, int64_t v)
{
    DistillPlan p{64, 1, v};
    if (v <= (m >= 1024 ? 6144 : 2048)) return p;
    p.tpr = 256;
    const int64_t unit = 256 * 16;
    const int64_t want = std::min<int64_t>(ceil_div(1024, m), ceil_div(v, unit));
    p.seg = ceil_div(ceil_div(v, want), unit) * unit;
    p.nseg = (int)ceil_div(v, p.seg);
    return p;
}

static int check_distill(const DistillArgs &a)
{
    VF_REQUIRE(is_float_type(a.dtype), "distill: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(a.m >= 0 && a.m <= kMaxExtent, "distill: m out of range");
    VF_REQUIRE(a.v >= 1 && a.v <= kMaxExtent, "distill: v must be at least 1 and below 2^31");
    VF_REQUIRE(a.top >= 1 && a.top <= VF_DISTILL_MAX_TOP, "distill: top must be 1 .. VF_DISTILL_MAX_TOP");
    VF_REQUIRE(std::isfinite(a.temperature) && a.temperature >= 1e-6 && a.temperature <= 1e6, "distill: temperature must be 1e-6 .. 1e6");
    VF_REQUIRE(a.ld >= a.v, "distill: ld is less than v");
    VF_REQUIRE(a.m == 0 || (a.logits && a.ids && a.teacher), "distill: logits, ids or teacher is NULL");
    return VF_OK;
}

int distill_workspace_impl(int32_t dtype, int64_t m, int64_t v, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "distill: bytes is NULL");
    VF_REQUIRE(is_float_type(dtype), "distill: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && v >= 1 && v <= kMaxExtent, "distill: sizes out of range");
    *bytes = 0;
    if (m == 0) return VF_OK;
    const DistillPlan p = plan_of(m, v);
    if (p.nseg > 1) *bytes = (size_t)m * p.nseg * 8;
    return VF_OK;
}

// Calls fn with the entries of a lane as a constant.
template <class F> static void by_top(int32_t top, F &&fn)
{
    if (top <= 64) fn(std::integral_constant<int, 1>());
    else fn(std::integral_constant<int, 4>());
}

int distill_impl(const DistillArgs &a)
{
    if (int rc = check_distill(a); rc != VF_OK) return rc;
    VF_REQUIRE(a.m == 0 || a.loss != nullptr, "distill: loss is NULL");
    size_t need = 0;
    if (int rc = distill_workspace_impl(a.dtype, a.m, a.v, &need); rc != VF_OK) return rc;
    if (int rc = check_workspace("distill", a.workspace, a.workspace_bytes, need); rc != VF_OK) return rc;
    if (a.m == 0) return VF_OK;
    const size_t size = type_size(a.dtype);
    const Region loss = region(a.loss, a.m, 4), lse = region(a.lse, a.m, 4);
    for (const Region &in : {region(a.logits, a.m, a.v, a.ld, size), region(a.ids, a.m * a.top, 4), region(a.teacher, a.m * a.top, 4)})
        VF_REQUIRE(!overlap(loss, in) && !overlap(lse, in), "distill: loss or lse overlaps an input");
    VF_REQUIRE(!overlap(loss, lse), "distill: loss and lse overlap each other");
    const DistillPlan p = plan_of(a.m, a.v);
    by_type(a.dtype, [&](auto *q) {
        using T = std::remove_pointer_t<decltype(q)>;
        const DistillRow<T> row{(const T *)a.logits, a.ld, a.v, a.ids, a.teacher, a.top, (float)(1.0 / a.temperature), a.loss, a.lse};
        float2 *part = (float2 *)a.workspace;
        by_top(a.top, [&](auto r) {
            constexpr int R = r.value;
            if (p.tpr == 64) {
                distill_kernel<T, 64, R><<<dim3(grid_of(ceil_div(a.m, 4))), dim3(256), 0, a.stream>>>(a.m, row, 1, p.seg, part);
            } else {
                distill_kernel<T, 256, R><<<dim3(grid_of(a.m * p.nseg)), dim3(256), 0, a.stream>>>(a.m, row, p.nseg, p.seg, part);
                if (p.nseg > 1) distill_join_kernel<T, R><<<dim3(grid_of(a.m)), dim3(64), 0, a.stream>>>(a.m, row, p.nseg, part);
            }
        });
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

int distill_backward_impl(const DistillArgs &a)
{
    if (int rc = check_distill(a); rc != VF_OK) return rc;
    VF_REQUIRE(a.ldd >= a.v, "distill: ldd is less than v");
    if (a.m == 0) return VF_OK;
    VF_REQUIRE(a.lse && a.d_loss && a.dlogits, "distill: lse, d_loss or dlogits is NULL");
    const size_t size = type_size(a.dtype);
    const Region x = region(a.logits, a.m, a.v, a.ld, size), dx = region(a.dlogits, a.m, a.v, a.ldd, size);
    VF_REQUIRE(dx.same(x) || !overlap(dx, x), "distill: dlogits overlaps the logits and is not them");
    for (const Region &in : {region(a.lse, a.m, 4), region(a.d_loss, a.m, 4), region(a.ids, a.m * a.top, 4), region(a.teacher, a.m * a.top, 4)})
        VF_REQUIRE(!overlap(dx, in), "distill: dlogits overlaps an input");
    by_type(a.dtype, [&](auto *q) {
        using T = std::remove_pointer_t<decltype(q)>;
        // segments of whole tiles: up to 4,096 columns a wave, fewer where there are few rows
        int64_t seg = 4096;
        while (seg > 512 && a.m * ceil_div(a.v, seg) < 4096) seg /= 2;
        const int nseg = (int)ceil_div(a.v, seg);
        by_top(a.top, [&](auto r) {
            distill_backward_kernel<T, r.value><<<dim3(grid_of(ceil_div(a.m * nseg, 4))), dim3(256), 0, a.stream>>>(
                a.m, a.v, (const T *)a.logits, a.ld, a.lse, a.ids, a.teacher, a.top, a.d_loss, (float)(1.0 / a.temperature), nseg, seg, (T *)a.dlogits, a.ldd);
        });
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

}  // namespace vf
