// One AdamW step over a list of tensors in few launches: the list travels as a kernel argument (48 tensors a launch), a
// wave takes one or four blocks of 256 elements at a time, four neighbours a lane and block, all of whose loads are on their way before
// the first result.  With moments in 8 bits a block shares a scale, so the wave that holds it takes the largest moment without leaving
// its registers.  Bound by memory: every operand is read and written once.
//
// The operations are single float32 ones in the order that the header states (no fused multiply-add), divisions and square
// roots rounded correctly: a plain evaluation gives the same bits, codes included.
#include "vf_ops.h"

namespace vf {

constexpr int kBlock = VF_ADAMW_BLOCK;
// Blocks that a wave takes at a time.  Moments in 8 bits have much to compute per byte and gain from more loads on their way (18.8 M
// elements: 78 us with four, 87 with one); in 32 bits the smaller pieces spread better (9.6 M elements: 54 us with one, 62 with four).
template <int BITS> constexpr int kUnit = BITS == 8 ? 4 : 1;
constexpr int kLaunchTensors = 48;   // 76 bytes each: the argument block of a kernel holds 4096

struct AdamwItem {
    void *param;
    const void *grad;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    float decay;        // 1 - lr weight_decay
    int32_t types;      // parameter | gradient << 8
};
struct AdamwList {
    AdamwItem item[kLaunchTensors];
    uint32_t first[kLaunchTensors + 1];   // tensor i has the units (of kUnit<BITS> blocks) first[i] .. first[i + 1]
    int32_t n;
};
static_assert(sizeof(AdamwList) <= 3900, "the list must fit a kernel's argument block");

struct AdamwScalars {
    float beta1, one_beta1, beta2, one_beta2, c1, c2, eps, lr, grad_scale;
};

// Four neighbouring elements of a tensor as float32; n: how many there are.
__device__ __forceinline__ void load4(const void *p, int type, int64_t at, int n, float (&o)[4])
{
    if (type == VF_F32) {
        const float *q = (const float *)p + at;
        if (n >= 4) { const float4v u = load_vec<float4v>(q); for (int j = 0; j < 4; ++j) o[j] = u[j]; }
        else for (int j = 0; j < 4; ++j) o[j] = j < n ? q[j] : 0.f;
    } else {
        uint16_t u[4] = {0, 0, 0, 0};
        const uint16_t *q = (const uint16_t *)p + at;
        if (n >= 4) __builtin_memcpy(u, q, 8);
        else for (int j = 0; j < 4; ++j) if (j < n) u[j] = q[j];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            o[j] = type == VF_BF16 ? __uint_as_float((uint32_t)u[j] << 16) : (float)__builtin_bit_cast(f16, u[j]);
    }
}
__device__ __forceinline__ void store4(void *p, int type, int64_t at, int n, const float (&o)[4])
{
    if (type == VF_F32) {
        float *q = (float *)p + at;
        if (n >= 4) { float4v u = {o[0], o[1], o[2], o[3]}; store_vec(q, u); }
        else for (int j = 0; j < 4; ++j) if (j < n) q[j] = o[j];
    } else {
        uint16_t u[4], *q = (uint16_t *)p + at;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            u[j] = type == VF_BF16 ? __builtin_bit_cast(uint16_t, (bf16)o[j]) : __builtin_bit_cast(uint16_t, (f16)o[j]);
        if (n >= 4) __builtin_memcpy(q, u, 8);
        else for (int j = 0; j < 4; ++j) if (j < n) q[j] = u[j];
    }
}

// The moments that codes stand for; the codes of what is not finite aside.
__device__ __forceinline__ float m_of(int8_t c, float scale)
{
    const float a = (float)c * (float)(1.0 / 127);
    return scale * (a * fabsf(a));
}
__device__ __forceinline__ float v_of(uint8_t c, float scale)
{
    const float b = (float)c * (float)(1.0 / 254), r = scale * (b * b);
    return r * r;
}
// The moments of four codes.  Codes of NaN are looked for in all lanes at once (a byte of x is zero where x - 1 borrows into its top bit).
__device__ __forceinline__ void decode4(const uint8_t (&cm)[4], const uint8_t (&cv)[4], float ms, float vs, float (&m)[4], float (&v)[4])
{
    uint32_t wm, wv;
    __builtin_memcpy(&wm, cm, 4);
    __builtin_memcpy(&wv, cv, 4);
    const uint32_t xm = wm ^ 0x80808080u, xv = ~wv;
    const uint32_t odd = ((xm - 0x01010101u) & ~xm | (xv - 0x01010101u) & ~xv) & 0x80808080u;
#pragma unroll
    for (int j = 0; j < 4; ++j) { m[j] = m_of((int8_t)cm[j], ms); v[j] = v_of(cv[j], vs); }
    if (__ballot(odd != 0)) {
        const float nan = __uint_as_float(0x7FC00000u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            m[j] = cm[j] == 0x80 ? nan : m[j];
            v[j] = cv[j] == 0xFF ? nan : v[j];
        }
    }
}
__device__ __forceinline__ void load4_codes(const void *p, int64_t at, int n, uint8_t (&c)[4])
{
    const uint8_t *q = (const uint8_t *)p + at;
    if (n >= 4) __builtin_memcpy(c, q, 4);
    else for (int j = 0; j < 4; ++j) c[j] = j < n ? q[j] : 0;
}
__device__ __forceinline__ void store4_codes(void *p, int64_t at, int n, const uint8_t (&c)[4])
{
    uint8_t *q = (uint8_t *)p + at;
    if (n >= 4) __builtin_memcpy(q, c, 4);
    else for (int j = 0; j < 4; ++j) if (j < n) q[j] = c[j];
}

// Code of x >= 0 under the block's scale, inv = 1 / scale: steps sqrt(x inv), to the nearest whole number, ties to even.
__device__ __forceinline__ float code_of(float x, float inv, float steps)
{
    return x > 0.f ? fminf(rintf(sqrtf(x * inv) * steps), steps) : 0.f;
}
// The same for a finite x and an inverse that did not overflow, with the hardware's square root, which is off by at most one unit
// in the last place: `near` tells that the product may be that close to the middle between two codes (two in 10,000), so that the
// code has to be taken again.
__device__ __forceinline__ float code_fast(float x, float inv, float steps, bool &near)
{
    const float c = __builtin_amdgcn_sqrtf(x * inv) * steps, r = rintf(c);
    near |= fabsf(c - r) > 0.5f - 1e-4f;   // 254 x 2^-22 is 0.6e-4
    return r;
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= kFltMax; }

__device__ __forceinline__ int find_tensor(const AdamwList &l, uint32_t unit)
{
    int lo = 0, hi = l.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (l.first[mid] <= unit) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Four elements a lane of one block, before and after the step.
template <int BITS> struct AdamwBlock {
    float p[4], g[4], m[4], v[4], ms, vs;
    uint8_t cm[4], cv[4];

    __device__ __forceinline__ void load(const AdamwItem &t, uint32_t b, int lane)
    {
        const int64_t at = (int64_t)b * kBlock + lane * 4;
        const int n = (int)max((int64_t)0, min((int64_t)4, t.n - at));
        if (t.master) load4(t.master, VF_F32, at, n, p); else load4(t.param, t.types & 0xFF, at, n, p);
        load4(t.grad, t.types >> 8, at, n, g);
        if constexpr (BITS == 32) {
            load4(t.m, VF_F32, at, n, m);
            load4(t.v, VF_F32, at, n, v);
        } else {
            load4_codes(t.m, at, n, cm);
            load4_codes(t.v, at, n, cv);
            ms = t.m_scale[b];
            vs = t.v_scale[b];
        }
    }
    __device__ __forceinline__ bool encode_fast(const float (&root)[4], float mi, float vi)
    {
        bool near = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            cm[j] = (uint8_t)(int)copysignf(code_fast(fabsf(m[j]), mi, 127.f, near), m[j]);
            cv[j] = (uint8_t)(int)fmaxf(code_fast(root[j], vi, 254.f, near), root[j] > 0.f ? 1.f : 0.f);
        }
        return near;
    }
    // Any values: what is not finite gets its own code and has no part in the scale.
    __device__ __forceinline__ void encode(const float (&root)[4])
    {
        ms = vs = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (finite(m[j])) ms = fmaxf(ms, fabsf(m[j]));
            if (finite(root[j])) vs = fmaxf(vs, root[j]);
        }
        ms = wave_max(ms);
        vs = wave_max(vs);
        const float mi = ms > 0.f ? 1.f / ms : 0.f, vi = vs > 0.f ? 1.f / vs : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int a = (int)code_of(fabsf(m[j]), mi, 127.f);
            const int r = (int)fmaxf(code_of(root[j], vi, 254.f), root[j] > 0.f ? 1.f : 0.f);
            cm[j] = finite(m[j]) ? (uint8_t)(m[j] < 0.f ? -a : a) : (uint8_t)0x80;
            cv[j] = finite(root[j]) ? (uint8_t)r : (uint8_t)255;
        }
    }
    __device__ __forceinline__ void step(const AdamwItem &t, uint32_t b, int lane, const AdamwScalars &c)
    {
        const int64_t at = (int64_t)b * kBlock + lane * 4;
        const int n = (int)max((int64_t)0, min((int64_t)4, t.n - at));
        float root[4];
        if constexpr (BITS == 8) decode4(cm, cv, ms, vs, m, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gj = g[j] * c.grad_scale;
            m[j] = m[j] * c.beta1 + gj * c.one_beta1;
            v[j] = v[j] * c.beta2 + (gj * gj) * c.one_beta2;
            root[j] = sqrtf(v[j]);
            p[j] = p[j] * t.decay - (m[j] * c.c1) / (root[j] * c.c2 + c.eps) * c.lr;
        }
        if (t.master) store4(t.master, VF_F32, at, n, p);
        store4(t.param, t.types & 0xFF, at, n, p);
        if constexpr (BITS == 32) {
            store4(t.m, VF_F32, at, n, m);
            store4(t.v, VF_F32, at, n, v);
        } else {
            // as whole numbers, so that a NaN counts as the largest: blocks with one, or with a scale below the normal range (whose inverse
            // may overflow), take the long way
            uint32_t mb = 0, vb = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mb = max(mb, __float_as_uint(m[j]) & 0x7FFFFFFFu);
                vb = max(vb, __float_as_uint(root[j]));
            }
            mb = wave_max(mb);
            vb = wave_max(vb);
            const uint32_t normal = 0x00800000u, infinite = 0x7F800000u;
            if (mb - normal < infinite - normal && vb - normal < infinite - normal) {
                ms = __uint_as_float(mb);
                vs = __uint_as_float(vb);
                if (__ballot(encode_fast(root, 1.f / ms, 1.f / vs))) encode(root);
            } else {
                encode(root);
            }
            store4_codes(t.m, at, n, cm);
            store4_codes(t.v, at, n, cv);
            if (lane == 0) { t.m_scale[b] = ms; t.v_scale[b] = vs; }
        }
    }
};

// 32 bits, 9.6 M float32 parameters: 55 us, 4.9 TB/s.  8 bits, 18.8 M bfloat16 parameters with masters: 72 us, 4.2 TB/s; there the vector
// ALUs are as busy as memory (three square roots and a division a parameter, some 90 instructions).
template <int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwList l, const AdamwScalars c, const int32_t *skip)
{
    if (skip && *skip != 0) return;
    const int lane = threadIdx.x & 63;
    const uint32_t units = l.first[l.n];
    for (uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); unit < units; unit += gridDim.x * 4) {
        const int i = find_tensor(l, unit);
        const AdamwItem &t = l.item[i];
        const uint32_t b = (unit - l.first[i]) * kUnit<BITS>;
        const int64_t left = t.n - (int64_t)b * kBlock;
        AdamwBlock<BITS> k[kUnit<BITS>];
        if (left >= kUnit<BITS> * kBlock) {
#pragma unroll
            for (int u = 0; u < kUnit<BITS>; ++u) k[u].load(t, b + u, lane);
#pragma unroll
            for (int u = 0; u < kUnit<BITS>; ++u) k[u].step(t, b + u, lane, c);
        } else {
#pragma unroll 1
            for (int u = 0; u < kUnit<BITS> && (int64_t)u * kBlock < left; ++u) {
                k[0].load(t, b + u, lane);
                k[0].step(t, b + u, lane, c);
            }
        }
    }
}

// master: where m goes, param: where v goes.  18.8 M parameters from 8 bits: 30 us, 6 TB/s (half of it in the cache still).
template <int BITS> __global__ __launch_bounds__(256) void adamw_moments_kernel(const AdamwList l)
{
    const int lane = threadIdx.x & 63;
    const uint32_t units = l.first[l.n];
    for (uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); unit < units; unit += gridDim.x * 4) {
        const int i = find_tensor(l, unit);
        const AdamwItem &t = l.item[i];
        const uint32_t first = (unit - l.first[i]) * kUnit<BITS>;
#pragma unroll
        for (int u = 0; u < kUnit<BITS>; ++u) {
            const uint32_t b = first + u;
            if ((int64_t)b * kBlock >= t.n) break;
            const int64_t at = (int64_t)b * kBlock + lane * 4;
            const int n = (int)max((int64_t)0, min((int64_t)4, t.n - at));
            float m[4], v[4];
            if constexpr (BITS == 32) {
                if (t.master) load4(t.m, VF_F32, at, n, m);
                if (t.param) load4(t.v, VF_F32, at, n, v);
            } else {
                uint8_t cm[4], cv[4];
                load4_codes(t.m, at, n, cm);
                load4_codes(t.v, at, n, cv);
                decode4(cm, cv, t.m_scale[b], t.v_scale[b], m, v);
            }
            if (t.master) store4(t.master, VF_F32, at, n, m);
            if (t.param) store4(t.param, VF_F32, at, n, v);
        }
    }
}

// Splits the tensors into launches of one width of moments and calls fn(list, bits) for each.
template <class Fill, class Launch>
static int each_launch(const vf_adamw_tensor *tensors, int32_t n_tensors, Fill &&fill, Launch &&launch)
{
    bool launched = false;
    for (int bits : {32, 8}) {
        AdamwList l;
        l.n = 0;
        l.first[0] = 0;
        for (int32_t i = 0; i < n_tensors; ++i) {
            const vf_adamw_tensor &t = tensors[i];
            if (t.state_bits != bits || t.n == 0) continue;
            if (l.n == kLaunchTensors) {
                launch(l, bits);
                l.n = 0;
            }
            fill(i, l.item[l.n]);
            l.first[l.n + 1] = l.first[l.n] + (uint32_t)ceil_div(t.n, kBlock * (bits == 8 ? kUnit<8> : kUnit<32>));
            ++l.n;
            launched = true;
        }
        if (l.n > 0) launch(l, bits);
    }
    if (launched) VF_HIP(hipGetLastError());
    return VF_OK;
}

// What both entry points ask of a tensor's moments, and that a launch's blocks can be counted in 31 bits.
static int check_tensors(const vf_adamw_tensor *tensors, int32_t n_tensors)
{
    VF_REQUIRE(n_tensors >= 0, "adamw: n_tensors is negative");
    VF_REQUIRE(n_tensors == 0 || tensors != nullptr, "adamw: tensors is NULL");
    int64_t blocks = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const vf_adamw_tensor &t = tensors[i];
        const std::string at = "adamw: tensor " + std::to_string(i);
        VF_REQUIRE(t.n >= 0 && t.n <= (int64_t)INT32_MAX * kBlock, at + ": n out of range");
        blocks += ceil_div(t.n, kBlock);
        VF_REQUIRE(blocks <= INT32_MAX, "adamw: too many elements in one call");
        VF_REQUIRE(t.reserved == 0, at + ": reserved must be zero");
        VF_REQUIRE(t.state_bits == 32 || t.state_bits == 8, at + ": state_bits must be 32 or 8");
        if (t.n == 0) continue;
        VF_REQUIRE(t.m && t.v, at + ": m or v is NULL");
        VF_REQUIRE(t.state_bits == 32 || (t.m_scale && t.v_scale), at + ": moments in 8 bits need scales");
    }
    return VF_OK;
}

static dim3 grid_of(const AdamwList &l)
{
    return dim3((unsigned)std::min<int64_t>(ceil_div((int64_t)l.first[l.n], 4), 256 * 8 * 2));
}

int adamw_step_impl(const vf_adamw_tensor *tensors, int32_t n_tensors, const vf_adamw_params *params, const int32_t *skip,
                    hipStream_t s)
{
    if (int rc = check_tensors(tensors, n_tensors); rc != VF_OK) return rc;
    VF_REQUIRE(params != nullptr, "adamw: params is NULL");
    const vf_adamw_params &h = *params;
    VF_REQUIRE(h.step >= 1, "adamw: step must be at least 1");
    VF_REQUIRE(h.beta1 >= 0 && h.beta1 < 1 && h.beta2 >= 0 && h.beta2 < 1, "adamw: betas must lie in [0, 1)");
    VF_REQUIRE(std::isfinite(h.lr) && h.eps >= 0 && std::isfinite(h.eps) && std::isfinite(h.grad_scale),
               "adamw: lr, eps and grad_scale must be finite, eps not negative");
    for (int32_t i = 0; i < n_tensors; ++i) {
        const vf_adamw_tensor &t = tensors[i];
        const std::string at = "adamw: tensor " + std::to_string(i);
        VF_REQUIRE(is_float_type(t.param_type) && is_float_type(t.grad_type), at + ": types must be VF_F32, VF_BF16 or VF_F16");
        VF_REQUIRE(t.n == 0 || (t.param && t.grad), at + ": param or grad is NULL");
        VF_REQUIRE(std::isfinite(t.weight_decay), at + ": weight_decay must be finite");
    }
    AdamwScalars c;
    c.beta1 = (float)h.beta1; c.one_beta1 = (float)(1 - h.beta1);
    c.beta2 = (float)h.beta2; c.one_beta2 = (float)(1 - h.beta2);
    c.c1 = (float)(1 / (1 - std::pow(h.beta1, (double)h.step)));
    c.c2 = (float)std::sqrt(1 / (1 - std::pow(h.beta2, (double)h.step)));
    c.eps = (float)h.eps; c.lr = (float)h.lr; c.grad_scale = (float)h.grad_scale;
    return each_launch(
        tensors, n_tensors,
        [&](int32_t i, AdamwItem &o) {
            const vf_adamw_tensor &t = tensors[i];
            o = AdamwItem{t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale, t.n,
                          (float)(1 - h.lr * t.weight_decay), t.param_type | t.grad_type << 8};
        },
        [&](const AdamwList &l, int bits) {
            if (bits == 32) adamw_kernel<32><<<grid_of(l), dim3(256), 0, s>>>(l, c, skip);
            else adamw_kernel<8><<<grid_of(l), dim3(256), 0, s>>>(l, c, skip);
        });
}

int adamw_moments_impl(const vf_adamw_tensor *tensors, int32_t n_tensors, float *const *m_out, float *const *v_out,
                       hipStream_t s)
{
    if (int rc = check_tensors(tensors, n_tensors); rc != VF_OK) return rc;
    VF_REQUIRE(n_tensors == 0 || m_out || v_out, "adamw: m_out and v_out are NULL");
    return each_launch(
        tensors, n_tensors,
        [&](int32_t i, AdamwItem &o) {
            const vf_adamw_tensor &t = tensors[i];
            o = AdamwItem{v_out ? v_out[i] : nullptr, nullptr, m_out ? m_out[i] : nullptr, t.m, t.v, t.m_scale, t.v_scale, t.n, 0.f, 0};
        },
        [&](const AdamwList &l, int bits) {
            if (bits == 32) adamw_moments_kernel<32><<<grid_of(l), dim3(256), 0, s>>>(l);
            else adamw_moments_kernel<8><<<grid_of(l), dim3(256), 0, s>>>(l);
        });
}

}  // namespace vf
