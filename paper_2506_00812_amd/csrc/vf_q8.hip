// Products of matrices in 8 bits (vf_q8.h): z = x w^T + bias, y = act(z) + residual or, gated, act(z_gate) z_up + residual, in a wide type or in 8 bits again.
// P = w, Q = x, both along the contraction; P takes the matrix instruction's first operand, so that a lane's accumulators are
// neighbours in a row of the output.  The instruction multiplies codes and applies both rows' scales; a lane's 32 codes may be any of a
// step's, so long as both operands' lanes take the same ones.
#include "vf_product.h"
#include "vf_q8.h"

namespace vf {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- to and from 8 bits

// Sixteen lanes to a block of 128 columns.  Bound by memory: 10,000 x 4,096 to bfloat16 123 MB in 24 us (5.1 TB/s), 10,000 x 1,024 7.
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
    int64_t chunk;    // blocks per split
    int splits;       // 0: the kernel has the epilogue; else its sums go to part, and the join has it
    float *part;      // [splits][nq][np], gated [splits][nq][2 np]
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

// 32 rows of each operand and 64 of the contraction, 32 codes a lane.  EXACT (outputs in float32 and in 8 bits): the codes are turned into bfloat16, which holds
// them exactly together with their scales.  The matrix cores add products of codes eight neighbours at a time, to 2^-13 of the largest of them
// (measured: 2^16 + 2^3 is right, 2^16 + 2^2 is 2^16; nine places apart nothing is lost): 1.4e-5 of a result of values of like size, whatever their
// number, where products of bfloat16 have 3e-8.  Outputs in bfloat16 and float16 round by far more (up to 2^-8 and 2^-11 of themselves) and take it.  Codes do not:
// a sum that is off by so little is on the other side of the middle of two codes once in 2,500 outputs, and a code is 2^-3 of its value further: 0.0015 of the result
// in norm, where float32 sums leave 0.0001.
// (The conversion reads the exponent's bits of the scale alone, and takes 0 for 2^-127 and 255 for NaN, as a scale's byte has them.)
__device__ __forceinline__ void decode(const int8v &c, int byte, Vec<bf16> (&v)[4])
{
    const float scale = __uint_as_float((uint32_t)byte << 23);
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

__device__ __forceinline__ float16v mma32(const Vec<bf16> (&p)[4], const Vec<bf16> (&q)[4], float16v acc)
{
#pragma unroll
    for (int g = 0; g < 4; ++g) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[g], q[g], acc, 0, 0, 0);
    return acc;
}
__device__ __forceinline__ float16v mma32(const int8v &p, int sp, const int8v &q, int sq, float16v acc)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, acc, 0, 0, 0, sp, 0, sq);
}

// ---------------------------------------------------------------- few rows

// Few rows, at most 16 FQ, of Q: one read of P, sixteen rows of it (of each half) a workgroup, whose waves share the contraction block by block, loaded from memory straight
// into the matrix instruction's layout, and add up through LDS.  Bound by memory and latency; the codes are multiplied as bfloat16, which costs nothing
// here and keeps every digit.  One row, 4,096 x 1,024 (4.3 MB): 4.0 us.  Each block of 128 costs a wave's loads in full, 1.5 us and more.
template <class T, int FQ, bool GATED>
__global__ __launch_bounds__(GATED ? 512 : 1024) void q8_few_rows_kernel(Q8Product a, Q8Epilogue<T> e)
{
    constexpr int G = GATED ? 2 : 1;
    __shared__ __align__(16) float4v sums[16 / G][G * FQ][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t p0 = (int64_t)blockIdx.x * 16;
    int64_t rp[G], rq[FQ];   // (rows beyond the last repeat it: their results are not kept)
#pragma unroll
    for (int g = 0; g < G; ++g) rp[g] = g * a.np + min(p0 + (lane & 15), a.np - 1);
#pragma unroll
    for (int j = 0; j < FQ; ++j) rq[j] = min((int64_t)(j * 16 + (lane & 15)), a.nq - 1);
    float4v acc[G][FQ] = {};
    const int at = (lane >> 4) * 32;
    for (int64_t b = wave; b < a.blocks; b += waves) {
        int8v cp[G], cq[FQ];
        int sp[G], sq[FQ];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            cp[g] = load_vec<int8v>(a.P.codes + rp[g] * a.P.ld + b * kBlock + at);
            sp[g] = a.P.scales[rp[g] * a.P.lds + b];
        }
#pragma unroll
        for (int j = 0; j < FQ; ++j) {
            cq[j] = load_vec<int8v>(a.Q.codes + rq[j] * a.Q.ld + b * kBlock + at);
            sq[j] = a.Q.scales[rq[j] * a.Q.lds + b];
        }
        Vec<bf16> vp[G][4];
#pragma unroll
        for (int g = 0; g < G; ++g) decode(cp[g], sp[g], vp[g]);
#pragma unroll
        for (int j = 0; j < FQ; ++j) {
            Vec<bf16> vq[4];
            decode(cq[j], sq[j], vq);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int g = 0; g < G; ++g) acc[g][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vp[g][u], vq[u], acc[g][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int j = 0; j < FQ; ++j)
#pragma unroll
        for (int g = 0; g < G; ++g) sums[wave][g * FQ + j][lane] = acc[g][j];
    __syncthreads();
    for (int j = wave; j < FQ; j += waves) {
        float v[G][4] = {};
        for (int w = 0; w < waves; ++w)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float4v u = sums[w][g * FQ + j][lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[g][i] += u[i];
            }
        const int64_t q = j * 16 + (lane & 15), p = p0 + (lane >> 4) * 4;
        if (q >= a.nq || p >= a.np) continue;
        const int n = (int)min((int64_t)4, a.np - p);
        if (a.splits > 0) {   // the join has the epilogue
#pragma unroll
            for (int g = 0; g < G; ++g) store_row(a.part + q * a.np * G + g * a.np + p, n, v[g]);
            continue;
        }
        float bias[G][4], r[4];
#pragma unroll
        for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) bias[g][i] = 0.f;
            if (e.bias) load_row(e.bias + g * a.np + p, n, bias[g]);
        }
        by_act(e.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[0][i] = act_value<act.value, T>(v[0][i] + bias[0][i]);
                if constexpr (GATED) v[0][i] *= v[1][i] + bias[1][i];
            }
        });
        if (e.residual) {
            load_row(e.residual + q * e.ldr + p, n, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[0][i] += r[i];
        }
        store_row(e.y + q * e.ldy + p, n, v[0]);
    }
}

// ---------------------------------------------------------------- tiles

// Row r of a tile of a gated P, counted in rows of one half: thirty-two of the gate, thirty-two of the other, and so on.
__device__ __forceinline__ int half_row32(int r) { return (r >> 6) * 32 + (r & 31); }

// Rows of 64 bytes, four to a line of the banks: their chunks are permuted so that the sixteen lanes that LDS serves together (0-3,
// 12-15, 20-27 and so on), sixteen of a fragment's thirty-two rows, touch sixteen different ones.
__device__ __forceinline__ int q8_chunk(int r, int ch) { return ch ^ (r >> 2 & 3); }

// The fragment whose lanes have rows `row` of the tile.
__device__ __forceinline__ int8v q8_fragment(const unsigned char *tile, int row, int lane)
{
    typedef int int4v __attribute__((ext_vector_type(4)));
    const int ch = (lane >> 5) * 2;
    const int4v lo = *(const int4v *)(tile + row * 64 + (q8_chunk(row, ch) << 4)), hi = *(const int4v *)(tile + row * 64 + (q8_chunk(row, ch + 1) << 4));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Four bytes a lane from its own address to LDS at `to` + 4 lane.
__device__ __forceinline__ void request4(const void *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}

// BP x BQ sums per workgroup of WP x WQ waves, straight to LDS, STEPS steps of 64 of the contraction deep, as direct_kernel in vf_product.h has them: while
// step t's fragments are multiplied, those of step t + 1 are read, and steps up to t + STEPS - 1 are on their way.  The
// scales of four blocks, eight steps, come a 32-bit word a row; a word's next byte is shifted down every other step.
// Bound by the matrix cores' clock under load and by what a tile has beside its loop: 256 x 256 sums take 1.47 us per block of 128 of the contraction (1.26 without
// any loads), and a tile some 2 us for its first loads and 5 - 8 for its outputs, which only a second workgroup on the compute unit hides.  10,000 x 1,024 x 4,096 with a
// residual: 48 - 53 us in 212 tiles of 256 x 192 (1,600 - 1,740 TFLOP/s; the library's bare product 44.5); 10,000 x (2 x 4,096) x 1,024, gated into bfloat16: 109 us in tiles
// of 256 x 128 (1,540); bare 10,000 x 4,096 x 1,024 67 us (the library 63).  EXACT is bound by the rate of bfloat16 and has sixteen conversions for a fragment beside it: the gated
// product into 8 bits 157 - 171 us (980 - 1,070 TFLOP/s), 10,000 x 1,024 x 4,096 into 8 bits 78, into float32 in tiles of 128 x 128 88; 1,777 x 333 x 777 into float32: 8 us.
template <class T, bool EXACT, bool GATED, int BP, int BQ, int WP, int WQ, int STEPS>
__global__ __launch_bounds__(WP *WQ * 64, BP *BQ == 16384 ? 3 : 2) void q8_tile_kernel(Q8Product a, Q8Epilogue<T> e)
{
    constexpr int G = GATED ? 2 : 1, OUT = BP / G, WAVES = WP * WQ, FP = BP / WP / 32, FQ = BQ / WQ / 32;
    constexpr int NP = BP / 16, NQ = BQ / 16;   // loads of a step; where they do not divide among the waves the last one is made twice
    constexpr int LP = (NP + WAVES - 1) / WAVES, LQ = (NQ + WAVES - 1) / WAVES, LOADS = LP + LQ;
    constexpr int NS = (BP + BQ) / 64, LS = (NS + WAVES - 1) / WAVES, kStep = (BP + BQ) * 64;
    extern __shared__ __align__(16) unsigned char tiles[];   // [STEPS][P, Q][rows of 64 bytes], [2][P, Q] words of scales
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t tiles_p = (a.np + OUT - 1) / OUT;
    int64_t p0, q0;
    place_tile<(BP * BQ > 32768 ? 4 : 8)>(blockIdx.x, gridDim.x, tiles_p, (a.nq + BQ - 1) / BQ, p0, q0);
    p0 *= OUT;
    q0 *= BQ;
    const int64_t b_first = (int64_t)blockIdx.y * a.chunk;
    const int blocks = (int)max((int64_t)0, min(a.blocks - b_first, a.chunk)), steps = 2 * blocks;

    const uint8_t *P = a.P.codes + p0 * a.P.ld + b_first * kBlock, *Q = a.Q.codes + q0 * a.Q.ld + b_first * kBlock;
    uint32_t off_p[LP], off_q[LQ];
#pragma unroll
    for (int i = 0; i < LP; ++i) {
        const int r = min(wave * LP + i, NP - 1) * 16 + (lane >> 2);
        off_p[i] = (uint32_t)(min((int64_t)(GATED ? half_row32(r) : r), a.np - 1 - p0) * a.P.ld) + (q8_chunk(r, lane & 3) << 4);
    }
#pragma unroll
    for (int i = 0; i < LQ; ++i) {
        const int r = min(wave * LQ + i, NQ - 1) * 16 + (lane >> 2);
        off_q[i] = (uint32_t)(min((int64_t)r, a.nq - 1 - q0) * a.Q.ld) + (q8_chunk(r, lane & 3) << 4);
    }
    const uint8_t *scales[LS];
#pragma unroll
    for (int i = 0; i < LS; ++i) {
        int r = min(wave * LS + i, NS - 1) * 64 + lane;
        if (r < BP) {
            int64_t row = min(p0 + (GATED ? half_row32(r) : r), a.np - 1);
            if (GATED && (r & 32)) row += a.np;
            scales[i] = a.P.scales + row * a.P.lds + b_first;
        } else {
            scales[i] = a.Q.scales + min(q0 + r - BP, a.nq - 1) * a.Q.lds + b_first;
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)tiles;
    const unsigned char *words = tiles + STEPS * kStep;
    auto buffer_of = [](int t) { return (STEPS & (STEPS - 1)) == 0 ? t & (STEPS - 1) : t % STEPS; };
    auto request_some = [&](int t, int first, int last) {   // loads first .. last - 1 of a step's
        const uint32_t at = buffer_of(t) * kStep;
        const uint8_t *p = P + t * 64, *q = Q + t * 64;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if (i < first || i >= last) continue;
            if (i < LP) {
                const int piece = min(wave * LP + i, NP - 1);
                request(GATED && (piece & 2) ? p + a.np * a.P.ld : p, off_p[i], lds0 + at + piece * 1024);
            } else {
                request(q, off_q[i - LP], lds0 + BP * 64 + at + min(wave * LQ + i - LP, NQ - 1) * 1024);
            }
        }
    };
    auto request_scales = [&](int group) {   // of blocks 4 group .. 4 group + 3
#pragma unroll
        for (int i = 0; i < LS; ++i)
            request4(scales[i] + group * 4, lds0 + STEPS * kStep + (group & 1) * ((BP + BQ) * 4) + min(wave * LS + i, NS - 1) * 256);
    };
    const int wp = wave % WP * (FP * 32), wq = wave / WP * (FQ * 32), row = lane & 31;
    // Two workgroups share a compute unit: the second of each begins later, by some two thirds of a loop alone, so that one's matrix instructions have the time in
    // which the other's outputs are computed and written (10,000 x 4,096 x 1,024, gated into bfloat16: 108 us, side by side 113; exact sums take longer and gain nothing).
    if (!EXACT && BP * BQ == 32768 && (blockIdx.x >> 8) == 1 && gridDim.x > 512)
        for (int i = 0; i < blocks; ++i) __builtin_amdgcn_s_sleep(32);
    float16v acc[FP][FQ] = {};
    int8v fp[FP], fq[EXACT ? 1 : 2][FQ];
    int sp[FP], sq[FQ];
    auto read_scales = [&](int group) {
        const int *w = (const int *)(words + (group & 1) * ((BP + BQ) * 4));
#pragma unroll
        for (int i = 0; i < FP; ++i) sp[i] = w[wp + i * 32 + row];
#pragma unroll
        for (int j = 0; j < FQ; ++j) sq[j] = w[BP + wq + j * 32 + row];
    };
    // A step in parts, one for each fragment of P: its matrix instructions, then the same fragment of the next step into the registers that they have read; Q's
    // fragments have two sets.  Step t + STEPS - 1 goes into the buffer of step t - 1, whose fragments everybody has used before this step's barrier: the last reads
    // of a step's own may still be on their way there.  MORE: step t + STEPS - 1 exists.
    auto one_step = [&](auto more, int t, int set) __attribute__((always_inline)) {   // (as a function of its own it would take addresses in vector registers)
        constexpr int kParts = FP;
        __builtin_amdgcn_sched_barrier(0);
        if (more.value || t + STEPS - 2 < steps) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((STEPS - 3) * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        const bool request_more = more.value || t + STEPS - 1 < steps;
        const unsigned char *at = tiles + buffer_of(t + 1) * kStep;   // (beyond the last step: a buffer's old contents, not used)
        Vec<bf16> vq[EXACT ? FQ : 1][4];   // Q's fragments as they are multiplied: their codes' registers are free for the next step's
        if constexpr (EXACT) {
#pragma unroll
            for (int j = 0; j < FQ; ++j) decode(fq[0][j], sq[j] & 255, vq[j]);
        }
#pragma unroll
        for (int g = 0; g < kParts; ++g) {
            __builtin_amdgcn_sched_barrier(0);
            if (request_more) request_some(t + STEPS - 1, g * LOADS / kParts, (g + 1) * LOADS / kParts);
            // (the next step begins with these: read early, they are there by then)
#pragma unroll
            for (int f = 0; f < FQ; ++f)
                if (min(f, kParts - 1) == g) fq[EXACT ? 0 : set ^ 1][f] = q8_fragment(at + BP * 64, wq + f * 32 + row, lane);
            if constexpr (EXACT) {
                Vec<bf16> vp[4];
                decode(fp[g], sp[g] & 255, vp);
#pragma unroll
                for (int j = 0; j < FQ; ++j) acc[g][j] = mma32(vp, vq[j], acc[g][j]);
            } else {
#pragma unroll
                for (int j = 0; j < FQ; ++j) acc[g][j] = mma32(fp[g], sp[g], fq[set][j], sq[j], acc[g][j]);
            }
            // (here, and the sums in their own registers: the compiler would gather the step's matrix instructions at its end, and keep all of its reads until then)
#pragma unroll
            for (int j = 0; j < FQ; ++j) asm volatile("" : "+a"(acc[g][j])::"memory");
            fp[g] = q8_fragment(at, wp + g * 32 + row, lane);
        }
    };
    if (steps > 0) {
        request_scales(0);
        for (int t = 0; t < min(steps, STEPS - 1); ++t) request_some(t, 0, LOADS);
        if (steps >= STEPS - 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STEPS - 2) * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        asm volatile("s_barrier" ::: "memory");
#pragma unroll
        for (int j = 0; j < FQ; ++j) fq[0][j] = q8_fragment(tiles + BP * 64, wq + j * 32 + row, lane);
#pragma unroll
        for (int i = 0; i < FP; ++i) fp[i] = q8_fragment(tiles, wp + i * 32 + row, lane);
        read_scales(0);
    }
    // The words of the next four blocks are asked for at the first of four, into the half that the last four have left (their words were read before this
    // block's first barrier), and read at the fourth's end: eight steps' waits lie between.
    auto one_block = [&](auto more, int b) __attribute__((always_inline)) {
        const bool next = (b & 3) == 0 && b + 4 < blocks;
        one_step(more, 2 * b, 0);
        if (next) request_scales(b / 4 + 1);
        one_step(more, 2 * b + 1, 1);
        if ((b & 3) == 3) {
            read_scales(b / 4 + 1);   // (after the last block: old words, not used)
        } else {
#pragma unroll
            for (int i = 0; i < FP; ++i) sp[i] = (int)((uint32_t)sp[i] >> 8);
#pragma unroll
            for (int j = 0; j < FQ; ++j) sq[j] = (int)((uint32_t)sq[j] >> 8);
        }
    };
    int b = 0;
    for (; 2 * b + STEPS < steps; ++b) one_block(std::true_type(), b);
    for (; b < blocks; ++b) one_block(std::false_type(), b);

    // The end: thirty-two rows of sums at a time are turned through LDS, all of a row's by the waves that have them, so that a lane has eight neighbours, a row's lanes
    // whole stretches of it and sixteen of them a block of 128 with its scale.  (Written from where the sums lie it was eight times the code, which runs once a
    // tile and comes from memory each time: 10,000 x 4,096 x 1,024 with GELU 93 us, 78 this way.)
    constexpr int kRow = BP * 4 + 16, kLanes = OUT / 8, kRows = 32 / WP;   // 16 bytes more: rows start in other banks; rows of a wave
    static_assert(kLanes <= 64 && kRows % (64 / kLanes) == 0, "");
    unsigned char *turn = tiles + wave / WP * (32 * kRow);
    const bool raw = a.splits > 0, q8 = EXACT && (!std::is_same_v<T, float> || e.y == nullptr);   // (2-byte types: exact sums are for outputs in 8 bits alone)
    const int64_t p = p0 + lane % kLanes * 8;
    const int m = (int)max((int64_t)0, min((int64_t)8, a.np - p));
    const int col = GATED ? (lane % kLanes >> 2) * 64 + (lane & 3) * 8 : lane % kLanes * 8;   // of the sums; the other half's are 32 further
    float bias[G][8];
    if (e.bias && !raw) {
#pragma unroll
        for (int g = 0; g < G; ++g) load8(e.bias + g * a.np + p, m, bias[g]);
    }
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
        __syncthreads();   // the last step's fragments, or the last rows, have been read
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(float4v *)(turn + row * kRow + (wp + i * 32 + g * 8 + (lane >> 5) * 4) * 4) =
                    float4v{acc[i][j][g * 4], acc[i][j][g * 4 + 1], acc[i][j][g * 4 + 2], acc[i][j][g * 4 + 3]};
        __syncthreads();
        constexpr int kPass = 64 / kLanes;   // rows at a time
        const int r_end = (wave % WP + 1) * kRows;
#pragma unroll 1
        for (int r = wave % WP * kRows + lane / kLanes; r < r_end; r += kPass) {
            const int64_t q = q0 + wq + j * 32 + r;
            float v[G][8];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const unsigned char *from = turn + r * kRow + (col + g * 32) * 4;
                *(float4v *)v[g] = *(const float4v *)from;
                *(float4v *)(v[g] + 4) = *(const float4v *)(from + 16);
            }
            if (raw) {
                if (q < a.nq) {
#pragma unroll
                    for (int g = 0; g < G; ++g) store8(a.part + ((int64_t)blockIdx.y * a.nq + q) * (G * a.np) + g * a.np + p, m, v[g]);
                }
                continue;
            }
            if (e.bias) {
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[g][c] += bias[g][c];
            }
            by_act(e.act, [&](auto act) {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    v[0][c] = act_value<act.value, T>(v[0][c]);
                    if constexpr (GATED) v[0][c] *= v[1][c];
                }
            });
            if (e.residual && q < a.nq) {
                float u[8];
                load8(e.residual + q * e.ldr + p, m, u);
#pragma unroll
                for (int c = 0; c < 8; ++c) v[0][c] += u[c];
            }
            if (!q8) {
                if (q < a.nq) store8(e.y + q * e.ldy + p, m, v[0]);
            } else if constexpr (OUT % kBlock == 0) {
                // (a block's columns beyond the last output are filled up with zeros; blocks beyond the last one are not written)
                if (m < 8) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[0][c] = c < m ? v[0][c] : 0.f;
                }
                if (q < a.nq && p < (a.np + kBlock - 1) / kBlock * kBlock) keep_block(v[0], e.codes + q * e.ldc + p, e.scales + q * e.lds + p / kBlock);
            }
        }
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
        float v[G][8] = {}, bias[G][8] = {}, r[8];
        if (e.bias) {
#pragma unroll
            for (int g = 0; g < G; ++g) load8(e.bias + g * a.np + p, n, bias[g]);
        }
        if (e.residual) load8(e.residual + q * e.ldr + p, n, r);
        join_splits<G, 8>(a.part + q * (a.np * G) + p, a.nq * (a.np * G), a.np, a.splits, n, v);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[g][j] += bias[g][j];
        by_act(e.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[0][j] = act_value<act.value, T>(v[0][j]);
                if constexpr (GATED) v[0][j] *= v[1][j];
            }
        });
        if (e.residual) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[0][j] += r[j];
        }
        if constexpr (Q8) keep_block(v[0], e.codes + q * e.ldc + p, e.scales + q * e.lds + b);
        else store8(e.y + q * e.ldy + p, n, v[0]);
    }
}

// ---------------------------------------------------------------- host side

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

// The kernels of a product, by the sums that a workgroup computes.
enum Q8Tiling {
    kQ8Few,      // 16 rows of P, all rows of Q (at most 64)
    kQ8Slim,     // 256 x 64, four waves: gated outputs in 8 bits, of which a tile of 128 rows would have half a block
    kQ8Small,    // 64 x 64, four waves: outputs in a wide type
    kQ8Square,   // 128 x 128, four waves: all but gated outputs in 8 bits
    kQ8Long,     // 256 x 128, four waves
    kQ8Wide,     // 256 x 192, eight waves
    kQ8Large,    // 256 x 256, eight waves
};
struct Q8Plan {
    bool fits = true;     // false: no tiling has few enough tiles
    Q8Tiling tiling = kQ8Few;
    int splits = 0;       // 0: no join
    int64_t chunk = 0;
    size_t bytes = 0;
};

// What a tiling costs, in microseconds: `step` per block of 128 of the contraction with a compute unit full of `together` workgroups, at least `alone` however few
// there are; `fixed` per workgroup for its first loads and its outputs.  Fitted: 23 sizes from 65 x 1,024 x 1,024 to 8,192 x 4,096 x 2,048, outputs in bfloat16 bare, gated and
// with GELU and a residual, and in float32, every tiling and 1 to 8 splits; outputs in 8 bits: 113 sizes, 1 to 16 splits.  What it picks takes 0.9 % longer than the best of all on average,
// 21 % at worst (65 x 1,024 x 1,024 into 8 bits).  `step` and `fixed` are not told apart well by contractions of 8 to 32 blocks: they are fits, not times of a loop.
struct Q8Cost {
    int bp, bq, together;
    double step, alone, fixed;
};
static Q8Cost q8_cost(Q8Tiling t, bool f32, bool gated, bool quantized)
{
    if (quantized && !f32) {   // exact sums
        switch (t) {
        case kQ8Slim: return Q8Cost{256, 64, 2, 1.43, 1.08, 5.35};
        case kQ8Square: return Q8Cost{128, 128, 3, 2.36, 1.31, 6.16};
        case kQ8Long: return gated ? Q8Cost{256, 128, 2, 2.34, 0.865, 9.04} : Q8Cost{256, 128, 2, 3.6, 0.876, 9.48};
        case kQ8Wide: return gated ? Q8Cost{256, 192, 1, 1.28, 0.383, 10.5} : Q8Cost{256, 192, 1, 1.92, 1.87, 8.93};
        default: return gated ? Q8Cost{256, 256, 1, 1.98, 0.999, 12.6} : Q8Cost{256, 256, 1, 2.45, 0.546, 12.1};
        }
    }
    switch (t) {
    case kQ8Slim: return Q8Cost{256, 64, 2, 2.1, 1.2, 8.0};   // (float32: the others' outputs in 8 bits are above)
    case kQ8Small: return f32 ? Q8Cost{64, 64, 4, 1.36, 0.47, 4.1} : Q8Cost{64, 64, 4, 1.07, 0.33, gated ? 2.5 : 3.0};
    case kQ8Square:
        return f32 ? Q8Cost{128, 128, 3, 2.65, 0.98, 7.5} : gated ? Q8Cost{128, 128, 3, 1.6, 0.6, 6.2} : Q8Cost{128, 128, 3, 1.55, 0.55, 7.2};
    case kQ8Long: return gated ? Q8Cost{256, 128, 2, 1.6, 1.2, 9.0} : Q8Cost{256, 128, 2, 1.64, 1.2, 9.1};
    case kQ8Wide: return gated ? Q8Cost{256, 192, 1, 1.08, 0.3, 10.0} : Q8Cost{256, 192, 1, 0.87, 0.12, 10.0};
    default: return gated ? Q8Cost{256, 256, 1, 1.38, 0.26, 12.0} : Q8Cost{256, 256, 1, 1.03, 0.11, 11.4};
    }
}

constexpr double kJoinCost = 6;   // of one more launch and its workspace, for a host that makes small calls as fast as it can: 4 us and more (in a graph 2)

static int few_waves(int64_t blocks, bool gated) { return (int)std::max<int64_t>(1, std::min<int64_t>(gated ? 8 : 16, blocks)); }

// What the few rows' kernel takes, in microseconds: the longer of a wave's way through its blocks, one after the other, and of all workgroups' loads, Q's in each of
// them.  Fitted to timings of 1,200 products of 1 to 64 rows, 64 to 200,000 outputs and 100 to 16,384 of the contraction.  A few blocks and some thousand outputs go to it
// (4,096 x 1,024: 3.6 us for one row, 4.6 for 32, in tiles of 64 x 64 5.8 and 6.1); long contractions and many outputs go to tiles, which read Q once for
// 64 outputs (16 rows, 200,000 x 1,024: 35 us, here 51; 64 rows, 16,384 x 4,096: 18, here 61; 64 x 16,384: 12, here 55).
static double few_cost(int64_t m, int64_t n, int64_t blocks, bool gated)
{
    const int waves = few_waves(blocks, gated);
    const double groups = (double)ceil_div(n, 16), loads = (gated ? 8.8 : 4.4) + 0.1 * m;
    const double chain = (double)ceil_div(blocks, waves) * (1.5 + 0.005 * m * waves);
    return 1.6 + std::max(chain, groups * 1e-4 * (blocks * loads + (m <= 16 ? 2 : m <= 32 ? 13 : 40)));
}

// quantized: the output is in 8 bits.  heavy: its epilogue has a residual, or GELU or SiLU without a gate.
static Q8Plan plan_q8(int32_t dtype, int64_t m, int64_t n, int64_t k, bool gated, bool quantized, bool heavy)
{
    Q8Plan best;
    const bool f32 = dtype == VF_F32;
    const int64_t blocks = ceil_div(k, kBlock), rows = gated ? 2 * n : n;
    const size_t sums = (size_t)m * rows * 4;
    double least = 0;
    if (m <= 64 && ceil_div(n, 16) < kMaxTiles) {
        least = few_cost(m, n, blocks, gated) + (quantized ? kJoinCost + sums * 2 / 7.5e6 : 0);
        best.splits = quantized ? 1 : 0;
        best.chunk = blocks;
        best.bytes = quantized ? sums : 0;
    }
    for (Q8Tiling t : {kQ8Slim, kQ8Small, kQ8Square, kQ8Long, kQ8Wide, kQ8Large}) {
        if (t == kQ8Slim && !(gated && quantized)) continue;
        if ((t == kQ8Small && quantized) || (t == kQ8Square && gated && quantized)) continue;   // (half a block of outputs)
        if (f32 && t > kQ8Square) continue;
        Q8Cost c = q8_cost(t, f32, gated, quantized);
        if (heavy) c.fixed += 6.0 * c.together * c.bp * c.bq / 65536 * (c.together > 1 ? 0.75 : 1);   // (less where another workgroup multiplies meanwhile)
        const int64_t tiles = ceil_div(n, gated ? c.bp / 2 : c.bp) * ceil_div(m, c.bq);
        if (tiles >= kMaxTiles) continue;
        for (int64_t splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
            const int64_t chunk = std::max<int64_t>(4, ceil_div(ceil_div(blocks, splits), 4) * 4);   // whole words of scales
            const int64_t used = std::max<int64_t>(1, ceil_div(blocks, chunk));
            if (splits > 1 && tiles * splits > 2048) break;
            if (used != splits) continue;
            const int64_t per_cu = ceil_div(tiles * used, 256), rounds = ceil_div(per_cu, c.together);
            const double steps = (double)std::min(chunk, blocks);
            const double last = (double)(per_cu - (rounds - 1) * c.together) / c.together;
            double us = (double)(rounds - 1) * (steps * c.step + c.fixed) + steps * std::max(c.alone, c.step * last) + c.fixed;
            us = std::max(us, 4.0);   // (nothing was quicker)
            if (used > 1) us += kJoinCost + (double)used * sums * 2 / 7.5e6;
            if (least == 0 || us < least) {
                least = us;
                best.tiling = t;
                best.splits = used > 1 ? (int)used : 0;
                best.chunk = chunk;
                best.bytes = best.splits ? sums * best.splits : 0;
            }
        }
    }
    best.fits = least > 0;
    return best;
}

template <class T, bool EXACT, bool GATED, int BP, int BQ, int WP, int WQ, int STEPS>
static int launch_q8(const Q8Product &a, const Q8Epilogue<T> &e, hipStream_t s)
{
    constexpr size_t lds = std::max<size_t>((size_t)STEPS * (BP + BQ) * 64 + 2 * (BP + BQ) * 4, (size_t)WQ * 32 * (BP * 4 + 16));
    static std::atomic<uint64_t> done{0};
    if constexpr (lds > 64 * 1024)
        if (int rc = allow_lds((const void *)q8_tile_kernel<T, EXACT, GATED, BP, BQ, WP, WQ, STEPS>, lds, done); rc != VF_OK) return rc;
    const int64_t tiles = ceil_div(a.np, GATED ? BP / 2 : BP) * ceil_div(a.nq, BQ);
    q8_tile_kernel<T, EXACT, GATED, BP, BQ, WP, WQ, STEPS><<<dim3((unsigned)tiles, (unsigned)std::max(a.splits, 1)), dim3(WP * WQ * 64), lds, s>>>(a, e);
    return VF_OK;
}

// EXACT: outputs in float32 or in 8 bits.
template <class T, bool EXACT, bool GATED> static int run_q8(const Q8Product &a, const Q8Epilogue<T> &e, Q8Tiling t, hipStream_t s)
{
    constexpr bool kWide = std::is_same_v<T, float> || !EXACT, kEight = EXACT;   // outputs that the call may have
    int rc = VF_OK;
    if (t == kQ8Few) {
        const dim3 grid((unsigned)ceil_div(a.np, 16)), block(few_waves(a.blocks, GATED) * 64);
        if (a.nq <= 16) q8_few_rows_kernel<T, 1, GATED><<<grid, block, 0, s>>>(a, e);
        else if (a.nq <= 32) q8_few_rows_kernel<T, 2, GATED><<<grid, block, 0, s>>>(a, e);
        else q8_few_rows_kernel<T, 4, GATED><<<grid, block, 0, s>>>(a, e);
    } else if (t == kQ8Slim) {
        if constexpr (GATED && kEight) rc = launch_q8<T, EXACT, true, 256, 64, 4, 1, 3>(a, e, s);
    } else if (t == kQ8Small) {
        if constexpr (kWide) rc = launch_q8<T, EXACT, GATED, 64, 64, 2, 2, 4>(a, e, s);
    } else if (t == kQ8Square) {
        if constexpr (kWide || !GATED) rc = launch_q8<T, EXACT, GATED, 128, 128, 2, 2, 3>(a, e, s);
    } else if constexpr (!std::is_same_v<T, float>) {
        if (t == kQ8Long) rc = launch_q8<T, EXACT, GATED, 256, 128, 2, 2, 3>(a, e, s);
        else if (t == kQ8Wide) rc = launch_q8<T, EXACT, GATED, 256, 192, 4, 2, 4>(a, e, s);
        else rc = launch_q8<T, EXACT, GATED, 256, 256, 2, 4, 4>(a, e, s);
    }
    if (rc != VF_OK) return rc;
    if (a.splits > 0) {
        const dim3 join(grid_of(ceil_div(a.nq * ceil_div(a.np, kBlock), 16)));
        if (e.y == nullptr) q8_join_kernel<T, GATED, true><<<join, dim3(256), 0, s>>>(a, e);
        else q8_join_kernel<T, GATED, false><<<join, dim3(256), 0, s>>>(a, e);
    }
    VF_HIP(hipGetLastError());
    return VF_OK;
}

static int check_q8_sizes(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t act)
{
    VF_REQUIRE(is_float_type(dtype), "linear in 8 bits: dtype must be VF_F32, VF_BF16 or VF_F16");
    VF_REQUIRE(m >= 0 && m <= kMaxExtent && n >= 0 && n <= (1 << 24) && k >= 0 && k < (1 << 24), "linear in 8 bits: m, n or k out of range");
    VF_REQUIRE(act >= VF_ACT_NONE && act <= VF_ACT_SILU, "linear in 8 bits: unknown activation");
    return VF_OK;
}

int linear_q8_workspace_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t gated, int32_t quantized, size_t *bytes)
{
    VF_REQUIRE(bytes != nullptr, "linear in 8 bits: bytes is NULL");
    if (int rc = check_q8_sizes(dtype, m, n, k, 0); rc != VF_OK) return rc;
    VF_REQUIRE((gated == 0 || gated == 1) && (quantized == 0 || quantized == 1), "linear in 8 bits: gated and quantized must be 0 or 1");
    *bytes = std::max(plan_q8(dtype, m, n, k, gated, quantized, false).bytes, plan_q8(dtype, m, n, k, gated, quantized, true).bytes);
    return VF_OK;
}

int debug_linear_q8_impl(int32_t dtype, int64_t m, int64_t n, int64_t k, int32_t gated, int32_t quantized, int32_t heavy, int32_t *tiling, int32_t *splits)
{
    if (int rc = check_q8_sizes(dtype, m, n, k, 0); rc != VF_OK) return rc;
    VF_REQUIRE(tiling && splits, "linear in 8 bits: tiling or splits is NULL");
    const Q8Plan p = plan_q8(dtype, m, n, k, gated != 0, quantized != 0, heavy != 0);
    VF_REQUIRE(p.fits, "linear in 8 bits: too many output tiles in one call");
    *tiling = p.tiling;
    *splits = p.splits;
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
    VF_REQUIRE(a.x.ld < (1 << 24) && a.w.ld < (1 << 24), "linear in 8 bits: rows of codes lie 2^24 bytes apart or more");   // (offsets within a tile have 32 bits)
    const Q8Plan plan = plan_q8(a.dtype, a.m, a.n, a.k, a.gated, q8, a.residual != nullptr || (!a.gated && costly(a.act)));
    VF_REQUIRE(plan.fits, "linear in 8 bits: too many output tiles in one call");
    if (int rc = check_workspace("linear in 8 bits", a.workspace, a.workspace_bytes, plan.bytes); rc != VF_OK) return rc;
    const size_t size = type_size(a.dtype);
    const Region y = region(a.y, a.m, a.n, a.ldy, size), r = region(a.residual, a.m, a.n, a.ldr, size), codes = codes_region(a.out, a.m, a.n),
                 scales = scales_region(a.out, a.m, a.n);
    for (const Region &in : {codes_region(a.x, a.m, a.k), scales_region(a.x, a.m, a.k), codes_region(a.w, rows, a.k), scales_region(a.w, rows, a.k), region(a.bias, rows, size)})
        VF_REQUIRE(!overlap(y, in) && !overlap(codes, in) && !overlap(scales, in), "linear in 8 bits: an output overlaps an input");
    VF_REQUIRE(y.same(r) || !overlap(y, r), "linear in 8 bits: y overlaps the residual and is not it");
    VF_REQUIRE(!overlap(codes, r) && !overlap(scales, r) && !overlap(codes, scales), "linear in 8 bits: codes or scales overlap the residual or each other");
    const Q8Product p{a.w, a.x, a.n, a.m, ceil_div(a.k, kBlock), plan.chunk, plan.splits, (float *)a.workspace};
    int rc = VF_OK;
    by_type(a.dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const Q8Epilogue<T> e{(const T *)a.bias, a.act, (const T *)a.residual, a.ldr, (T *)a.y, a.ldy, (uint8_t *)a.out.codes, (uint8_t *)a.out.scales, a.out.ld, a.out.lds};
        auto run = [&](auto exact) {
            rc = a.gated ? run_q8<T, exact.value, true>(p, e, plan.tiling, a.stream) : run_q8<T, exact.value, false>(p, e, plan.tiling, a.stream);
        };
        if constexpr (std::is_same_v<T, float>) run(std::true_type());
        else if (q8) run(std::true_type());
        else run(std::false_type());
    });
    return rc;
}

}  // namespace vf
