// Log probabilities over a vocabulary: one pass over the logits takes the running maximum m, S = sum exp(x - m), A = sum
// exp(x - m) (x - m) and the largest entries of a row;  lse = m + log S,  logp = (x_t - m) - log S,  entropy = log S - A / S (a sum
// of two terms that are not negative).  A changed maximum turns (S, A) into f S and f (A + (m - m') S) with f = exp(m - m').
// Bound by memory where there are many rows.  A row is one wave's, one workgroup's, or (few rows) split into segments whose
// (m, S, A, largest) a second kernel joins.
#include "vf_device.h"
#include "vf_ops.h"

namespace vf {

constexpr float kInf = __builtin_inff();

// Orders values as whole numbers: NaN > +inf > ... > -inf, -0 = +0.  Its complement with the label below it is a key that orders
// alternatives ascending (larger values first, ties to the lower label).
__device__ __forceinline__ uint32_t value_order(float x)
{
    if (x != x) return ~0u;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t label) { return (uint64_t)~value_order(x) << 32 | label; }
__device__ __forceinline__ float order_value(uint32_t o)
{
    return __uint_as_float(o == ~0u ? 0x7FC00000u : o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

struct RowSums {
    float m, s, a;
};

// The same sums from another origin m >= r.m.  A factor that vanishes (nothing was summed yet, or the origins are far apart: their
// distance may be infinite) leaves nothing of a; s keeps a NaN.
__device__ __forceinline__ void scale_to(RowSums &r, float m)
{
    if (r.m == m) return;
    const float d = r.m - m, f = exp_fast(d);
    r.a = f > 0.f ? f * (r.a + d * r.s) : 0.f;
    r.s = f * r.s;
    r.m = m;
}

// Over the LANES (16 or 64) lanes that share a row.
template <int LANES = 64> __device__ __forceinline__ RowSums wave_join(RowSums r)
{
    scale_to(r, LANES == 16 ? max16(r.m) : wave_max(r.m));
    r.s = LANES == 16 ? sum16(r.s) : wave_sum(r.s);
    r.a = LANES == 16 ? sum16(r.a) : wave_sum(r.a);
    return r;
}

// The largest keys of a wave, kept as their complements in ascending order: lane i holds the i-th of what was offered (all 64 are kept,
// `top` are asked for).  `bound`: no complement from it on can be among the first `top`.
struct WaveTop {
    uint64_t key = KEY_MAX, bound = KEY_MAX;
    static __device__ __forceinline__ uint64_t of_lane(uint64_t k, int lane)
    {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
    }
    // Before the first offers: of 64 candidates with the value orders o (0: none) at least `top` reach the threshold found here, to 16
    // bits, so that the first thousand entries of a row have some `top` that are looked at and not top (1 + log(1000 / top)).
    __device__ __forceinline__ void expect(uint32_t o, int top)
    {
        uint32_t t = 0;
#pragma unroll 1
        for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit >>= 1)
            if (__popcll(__ballot(o >= (t | bit))) >= top) t |= bit;
        if (t) bound = (uint64_t)(~t + 1) << 32;
    }
    // The least value order that may still be among the first `top`; 0: any.
    __device__ __forceinline__ uint32_t least_order() const { return ~(uint32_t)((bound - 1) >> 32); }
    // One key a lane (KEY_MAX: none).  A few are inserted one by one, some 130 cycles each; more are sorted and merged with the list, some
    // 1,000 cycles however many (10,000 rows of 1,000, 32 alternatives: 24 us, 33 with insertions alone).
    __device__ __forceinline__ void offer(uint64_t k, int top)
    {
        const int lane = threadIdx.x & 63;
        uint64_t mask = __ballot(k < bound);
        if (mask == 0) return;
        if (__popcll(mask) > 8) {
            const uint64_t descending = ~wave_sort64(~(k < bound ? k : KEY_MAX), lane);
            key = wave_merge64(key < descending ? key : descending, lane);
        } else {
            do {
                const uint64_t in = of_lane(k, __builtin_ctzll(mask));
                mask &= mask - 1;
                const int at = __popcll(__ballot(key < in));
                const uint64_t up = wave_shr1_64(key);
                key = lane < at ? key : lane == at ? in : up;
            } while (mask);
        }
        const uint64_t last = of_lane(key, top - 1);
        bound = last < bound ? last : bound;
    }
};

struct LogProbOut {
    const int32_t *targets;
    float *logp, *entropy, *lse;
    int32_t *top_ids;
    float *top_logp;
};

// The label that a row is asked about and its logit, loaded before the sums are known (two loads, one after the other).
template <class T> struct Asked {
    int32_t t = -1;
    float x = 0.f;
    __device__ __forceinline__ void load(const LogProbOut &o, const T *row_x, int64_t row, int64_t v)
    {
        if (!o.targets) return;
        t = o.targets[row];
        if (t >= 0 && t < v) x = (float)row_x[t];
    }
};

// What a row's sums and keys say, written by the wave (or by the sixteen lanes) that has them.
template <class T>
__device__ __forceinline__ void finish_row(const LogProbOut &o, const Asked<T> &asked, int64_t row, int64_t v, int top, const RowSums &r, uint64_t key,
                                           int lane)
{
    const bool empty = r.m == -kInf && r.s == 0.f;
    const float log_s = logf(r.s);
    if (lane == 0) {
        if (o.lse) o.lse[row] = empty ? -kInf : r.m + log_s;
        if (o.entropy) o.entropy[row] = empty ? 0.f : log_s - r.a / r.s;
        if (o.targets) {
            float l = 0.f;
            if (asked.t != -1) {
                if (asked.t < 0 || asked.t >= v) l = __uint_as_float(0x7FC00000u);
                else l = empty ? -kInf : (asked.x - r.m) - log_s;
            }
            o.logp[row] = l;
        }
    }
    if (lane < top) {
        o.top_ids[row * top + lane] = key != KEY_MAX ? (int32_t)(uint32_t)key : -1;
        o.top_logp[row * top + lane] = key != KEY_MAX ? (order_value(~(uint32_t)(key >> 32)) - r.m) - log_s : -kInf;
    }
}

// Segment `item % nseg` of a row: TPR threads take its vectors in turn, 16 elements a thread at a time.  nseg > 1: the segment's sums and
// keys go to part_sums [row][nseg] and part_keys [row][nseg][top].  10,000 rows of 1,000 in float32: 11 us without alternatives (3.8 TB/s), 17
// with eight; finding those is some 400 instructions a row, half of them waiting for the one before.
template <class T, int TPR, bool TOP>
__global__ __launch_bounds__(256) void log_probs_kernel(int64_t m, int64_t v, const T *__restrict__ logits, int64_t ld, int nseg,
                                                        int64_t seg, int top, LogProbOut out, float4 *__restrict__ part_sums,
                                                        uint64_t *__restrict__ part_keys)
{
    constexpr int V = kVec<T>, RPB = 256 / TPR, W = TPR / 64, E = 16, NV = E / V;
    __shared__ float lds_sums[4][3];
    __shared__ uint64_t lds_keys[TOP && W > 1 ? 3 * 64 : 1], lds_chosen[TOP ? 4 * 64 * E / 2 : 1];
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t *chosen = lds_chosen + (TOP ? wave * (64 * E / 2) : 0);
    const int64_t items = m * nseg;
    for (int64_t item = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; item < items; item += (int64_t)gridDim.x * RPB) {
        const int64_t row = nseg == 1 ? item : item / nseg, sg = nseg == 1 ? 0 : item - row * nseg;
        const T *x = logits + row * ld;
        const int64_t c0 = sg * seg, c1 = min(v, c0 + seg);
        RowSums r = {-kInf, 0.f, 0.f};
        WaveTop best;
        Asked<T> asked;
        if (nseg == 1) asked.load(out, x, row, v);
        for (int64_t base = c0; base < c1; base += TPR * E) {
            float u[E];
            const int left = (int)min((int64_t)(TPR * E), c1 - base);   // vectors beyond it are skipped by all lanes at once
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i * TPR * V >= left) {
#pragma unroll
                    for (int j = 0; j < V; ++j) u[i * V + j] = -kInf;
                    continue;
                }
                const int64_t c = base + (i * TPR + t) * V;
                Vec<T> raw;
                if (base + TPR * E <= c1) raw = load_vec<Vec<T>>(x + c);
                else raw = load_part(x + c, (int)max((int64_t)0, min((int64_t)V, c1 - c)), (T)-kInf);
#pragma unroll
                for (int j = 0; j < V; ++j) u[i * V + j] = (float)raw[j];
            }
            float most = u[0];
#pragma unroll
            for (int j = 1; j < E; ++j) most = fmaxf(most, u[j]);
            if (most > r.m) scale_to(r, most);
            const float origin = r.m == -kInf ? 0.f : r.m;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (j % V == 0 && j / V * TPR * V >= left) break;
                // (the distance of a masked entry is -inf and its term 0; a NaN, which the maximum passes over, stays in s)
                const float d = u[j] - origin, e = exp_fast(d);
                r.s += e;
                r.a = __builtin_fmaf(e, fmaxf(d, -kFltMax), r.a);
            }
            if constexpr (TOP) {
                if (base == c0) best.expect(most > -kInf ? value_order(most) : 0, top);
                // what may reach the list is told by its value (NaN is not less than anything), gathered in LDS and offered together
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t least_order = best.least_order();
                    const float least = least_order ? fmaxf(order_value(least_order), -kFltMax) : -kFltMax;
                    int found = 0;
#pragma unroll
                    for (int j = half * (E / 2); j < (half + 1) * (E / 2); ++j) {
                        if (j % V == 0 && j / V * TPR * V >= left) break;
                        const bool in = !(u[j] < least);
                        const uint64_t mask = __ballot(in);
                        if (mask == 0) continue;
                        const uint32_t at = (uint32_t)(base + (j / V * TPR + t) * V + j % V);
                        if (in) chosen[found + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = key_of(u[j], at);
                        found += __popcll(mask);
                    }
                    wave_sync<true>();
#pragma unroll 1
                    for (int i = 0; i < found; i += 64) best.offer(i + lane < found ? chosen[i + lane] : KEY_MAX, top);
                    wave_sync<true>();
                }
            }
        }
        r = wave_join<TPR == 16 ? 16 : 64>(r);
        if constexpr (W > 1) {
            __syncthreads();
            if (lane == 0) { lds_sums[wave][0] = r.m; lds_sums[wave][1] = r.s; lds_sums[wave][2] = r.a; }
            if (TOP && wave > 0 && lane < top) lds_keys[(wave - 1) * top + lane] = best.key;
            __syncthreads();
            if (wave == 0) {
                float most = -kInf;
#pragma unroll
                for (int w = 0; w < W; ++w) most = fmaxf(most, lds_sums[w][0]);
                RowSums all = {most, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    RowSums p = {lds_sums[w][0], lds_sums[w][1], lds_sums[w][2]};
                    scale_to(p, most);
                    all.s += p.s;
                    all.a += p.a;
                }
                r = all;
                if constexpr (TOP) {
                    for (int i = lane; i - lane < (W - 1) * top; i += 64) best.offer(i < (W - 1) * top ? lds_keys[i] : KEY_MAX, top);
                }
            }
        }
        if (W <= 1 || wave == 0) {
            if (nseg == 1) {
                finish_row(out, asked, row, v, TOP ? top : 0, r, best.key, TPR == 16 ? t : lane);
            } else {
                if (lane == 0) part_sums[item] = make_float4(r.m, r.s, r.a, 0.f);
                if (TOP && lane < top) part_keys[item * top + lane] = best.key;
            }
        }
    }
}

// One wave per row joins the segments (one row of 200,000 with eight alternatives: 5 us after the 8 of its 49 segments; both are chains of
// dependent loads and list insertions, far from any rate).
template <class T>
__global__ __launch_bounds__(64) void log_probs_join_kernel(int64_t m, int64_t v, const T *__restrict__ logits, int64_t ld, int nseg,
                                                            int top, LogProbOut out, const float4 *__restrict__ part_sums,
                                                            const uint64_t *__restrict__ part_keys)
{
    const int lane = threadIdx.x;
    for (int64_t row = blockIdx.x; row < m; row += gridDim.x) {
        RowSums r = {-kInf, 0.f, 0.f};
        Asked<T> asked;
        asked.load(out, logits + row * ld, row, v);
        const int n = nseg * top;
        const uint64_t *keys = part_keys + row * n;
        constexpr int kAhead = 8;   // keys a lane, on their way together
        uint64_t ahead[kAhead];
        auto load_keys = [&](int first) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int at = first + i * 64 + lane;
                ahead[i] = at < n ? keys[at] : KEY_MAX;
            }
        };
        load_keys(0);
        for (int i = lane; i < nseg; i += 64) {
            const float4 p = part_sums[row * nseg + i];
            RowSums q = {p.x, p.y, p.z};
            const float most = fmaxf(r.m, q.m);
            scale_to(r, most);
            scale_to(q, most);
            r.s += q.s;
            r.a += q.a;
        }
        r = wave_join(r);
        WaveTop best;
        for (int first = 0; first < n; first += kAhead * 64) {
            if (first > 0) load_keys(first);
            if (first == 0) {
                uint64_t least = KEY_MAX;
#pragma unroll
                for (int i = 0; i < kAhead; ++i) least = ahead[i] < least ? ahead[i] : least;
                best.expect(~(uint32_t)(least >> 32), top);
            }
#pragma unroll 1
            for (int i = 0; i < kAhead && first + i * 64 < n; ++i) {
                uint64_t key = ahead[0];
#pragma unroll
                for (int j = 1; j < kAhead; ++j) key = i == j ? ahead[j] : key;
                best.offer(key, top);
            }
        }
        finish_row(out, asked, row, v, top, r, best.key, lane);
    }
}

// dlogits = d_logp (1[target] - p) - d_entropy p (log p + entropy), p = exp(x - lse).  (lse is one float: its rounding moves all p of a row
// by 2^-24 |lse| of themselves.  A second one per row would take that away; logits as models have them, |lse| < 100, lose 6e-6.)  Elementwise; bound by memory and
// the vector ALUs alike (busy for 89 % of the cycles): 10,000 x 10,000 in bfloat16 81 us, 4.9 TB/s.
template <class T>
__global__ void log_probs_backward_kernel(int64_t m, int64_t v, const T *logits, int64_t ld, const float *__restrict__ lse,
                                          const int32_t *__restrict__ targets, const float *__restrict__ d_logp,
                                          const float *__restrict__ entropy, const float *__restrict__ d_entropy, T *dlogits, int64_t ldd)
{
    constexpr int V = kVec<T>;
    const int64_t c = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * V;
    if (c >= v) return;
    const int n = (int)min((int64_t)V, v - c);
    for (int64_t row = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; row < m; row += (int64_t)gridDim.y * blockDim.y) {
        const float l = lse[row];
        int32_t t = targets ? targets[row] : -1;
        if (t < 0 || t >= v) t = -1;
        const float dl = t >= 0 ? d_logp[row] : 0.f;
        const float dh = d_entropy ? d_entropy[row] : 0.f, h = d_entropy ? entropy[row] : 0.f;
        const Vec<T> x = load_part(logits + row * ld + c, n, (T)-kInf);
        Vec<T> o;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float lp = (float)x[j] - l, p = exp_fast(lp);
            float g = (t == c + j ? dl : 0.f) - dl * p;
            g -= p > 0.f || p != p ? dh * (p * (lp + h)) : 0.f;
            o[j] = (T)(l == -kInf ? 0.f : g);
        }
        store_part(dlogits + row * ldd + c, o, n);
    }
}

// Threads per row and segments of a row.  Rows of up to 2,048 elements are a wave's, without alternatives up to 256 sixteen lanes' (100,000
// rows of 100 labels: 43 us a wave each); longer ones a workgroup's, in segments where there are too few rows to fill the chip.
struct LogProbPlan {
    int tpr, nseg;
    int64_t seg;
};
static LogProbPlan plan_of(int64_t m, int64_t v, int32_t top)
{
    LogProbPlan p{64, 1, v};
    if (v <= 256 && top == 0) p.tpr = 16;
    if (v <= 2048) return p;
    p.tpr = 256;
    const int64_t unit = 256 * 16;
    const int64_t want = std::min<int64_t>(ceil_div(1024, m), ceil_div(v, unit));
    p.seg = ceil_div(ceil_div(v, want), unit) * unit;
    p.nseg = (int)ceil_div(v, p.seg);
    return p;
}

static int check_log_probs(int32_t dtype, int64_t m, int64_t v, int64_t top)
{
    VF_REQUIRE(is_float_type(dtype), "log probs: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent, "log probs: m out of range");
    VF_REQUIRE(v >= 1 && v <= kMaxExtent, "log probs: v must be at least 1 and below 2^31");
    VF_REQUIRE(top >= 0 && top <= VF_LOG_PROBS_MAX_TOP, "log probs: top must be 0 .. VF_LOG_PROBS_MAX_TOP");
    return VF_OK;
}

int log_probs_workspace_impl(int32_t dtype, int64_t m, int64_t v, int32_t top, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "log probs: bytes is NULL");
    if (int rc = check_log_probs(dtype, m, v, top); rc != VF_OK) return rc;
    *bytes = 0;
    if (m == 0) return VF_OK;
    const LogProbPlan p = plan_of(m, v, top);
    if (p.nseg > 1) *bytes = (size_t)m * p.nseg * (16 + 8 * (size_t)top);
    return VF_OK;
}

int log_probs_impl(const LogProbArgs &a)
{
    size_t need = 0;
    if (int rc = log_probs_workspace_impl(a.dtype, a.m, a.v, a.top, &need); rc != VF_OK) return rc;
    VF_REQUIRE(a.ld >= a.v, "log probs: ld is less than v");
    VF_REQUIRE(a.m == 0 || a.logits != nullptr, "log probs: logits is NULL");
    VF_REQUIRE(a.targets == nullptr || a.logp != nullptr || a.m == 0, "log probs: targets without logp");
    VF_REQUIRE(a.top == 0 || a.m == 0 || (a.top_ids && a.top_logp), "log probs: top_ids or top_logp is NULL");
    if (int rc = check_workspace("log probs", a.workspace, a.workspace_bytes, need); rc != VF_OK) return rc;
    if (a.m == 0) return VF_OK;
    const LogProbPlan p = plan_of(a.m, a.v, a.top);
    const LogProbOut out{a.targets, a.logp, a.entropy, a.lse, a.top_ids, a.top_logp};
    float4 *sums = (float4 *)a.workspace;
    uint64_t *keys = (uint64_t *)(sums + (p.nseg > 1 ? a.m * p.nseg : 0));
    by_type(a.dtype, [&](auto *q) {
        using T = std::remove_pointer_t<decltype(q)>;
        const T *x = (const T *)a.logits;
        const int64_t blocks = p.tpr < 256 ? ceil_div(a.m, 256 / p.tpr) : a.m * p.nseg;
        const dim3 grid((unsigned)std::min<int64_t>(blocks, 1 << 20)), block(256);
        auto launch = [&](auto tpr, auto with_top) {
            log_probs_kernel<T, tpr.value, with_top.value><<<grid, block, 0, a.stream>>>(a.m, a.v, x, a.ld, p.nseg, p.seg, a.top, out,
                                                                                         sums, keys);
        };
        using W = std::integral_constant<int, 64>;
        using G = std::integral_constant<int, 256>;
        if (p.tpr == 16) launch(std::integral_constant<int, 16>(), std::false_type());
        else if (p.tpr == 64) { if (a.top) launch(W(), std::true_type()); else launch(W(), std::false_type()); }
        else { if (a.top) launch(G(), std::true_type()); else launch(G(), std::false_type()); }
        if (p.nseg > 1)
            log_probs_join_kernel<T><<<dim3((unsigned)std::min<int64_t>(a.m, 1 << 20)), dim3(64), 0, a.stream>>>(
                a.m, a.v, x, a.ld, p.nseg, a.top, out, sums, keys);
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

int log_probs_backward_impl(const LogProbArgs &a)
{
    if (int rc = check_log_probs(a.dtype, a.m, a.v, 0); rc != VF_OK) return rc;
    VF_REQUIRE(a.ld >= a.v && a.ldd >= a.v, "log probs: ld or ldd is less than v");
    VF_REQUIRE((a.targets == nullptr) == (a.d_logp == nullptr), "log probs: targets and d_logp go together");
    VF_REQUIRE((a.entropy == nullptr) == (a.d_entropy == nullptr), "log probs: entropy and d_entropy go together");
    if (a.m == 0) return VF_OK;
    VF_REQUIRE(a.logits && a.lse && a.dlogits, "log probs: logits, lse or dlogits is NULL");
    const Region x = region(a.logits, a.m, a.v, a.ld, type_size(a.dtype)), dx = region(a.dlogits, a.m, a.v, a.ldd, type_size(a.dtype));
    VF_REQUIRE(dx.same(x) || !overlap(dx, x), "log probs: dlogits overlaps the logits and is not them");
    for (const void *in : {(const void *)a.lse, (const void *)a.targets, (const void *)a.d_logp, (const void *)a.entropy, (const void *)a.d_entropy})
        VF_REQUIRE(!overlap(dx, region(in, a.m, 4)), "log probs: dlogits overlaps an input");
    by_type(a.dtype, [&](auto *q) {
        using T = std::remove_pointer_t<decltype(q)>;
        const int64_t nv = ceil_div(a.v, kVec<T>);
        const dim3 block = nv > 128 ? dim3(256, 1) : nv > 32 ? dim3(64, 4) : dim3(16, 16);
        const int64_t across = ceil_div(nv, block.x);   // (a launch holds fewer than 2^32 threads)
        const dim3 grid((unsigned)across, (unsigned)std::min<int64_t>({ceil_div(a.m, block.y), 65535, std::max<int64_t>(1, (1 << 20) / across)}));
        log_probs_backward_kernel<T><<<grid, block, 0, a.stream>>>(a.m, a.v, (const T *)a.logits, a.ld, a.lse, a.targets, a.d_logp,
                                                                   a.entropy, a.d_entropy, (T *)a.dlogits, a.ldd);
    });
    VF_HIP(hipGetLastError());
    return VF_OK;
}

}  // namespace vf
