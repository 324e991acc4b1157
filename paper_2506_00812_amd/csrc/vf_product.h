// Matrix products on the matrix cores, what the linear layer (vf_linear.hip) and the gated layer (vf_gated.hip) share.  Every product
// is written as
//     out[q][p] = sum over c of Q[q][c] P[p][c]
// with each operand either contiguous along c or along its own rows.  P takes the matrix instruction's first operand, so that
// a lane's four accumulators are neighbours in a row of the output.
//
// GATED: P holds the rows of two projections, n of a gate and then n of what it gates, and the output is act(gate) up.  A tile takes its rows
// sixteen by sixteen from both in turn, so that a wave has both halves of its outputs in the same lanes and only the product leaves it.
#pragma once

#include <atomic>

#include "vf_device.h"
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

// N neighbours of a row, n (1 .. N) of which exist.
template <class T, int N> __device__ __forceinline__ void load_row(const T *p, int n, float (&o)[N])
{
    using V = T __attribute__((ext_vector_type(N)));
    if (n == N) {
        const V v = load_vec<V>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = i < n ? (float)p[i] : 0.f;
    }
}
template <class T, int N> __device__ __forceinline__ void store_row(T *p, int n, const float (&o)[N])
{
    using V = T __attribute__((ext_vector_type(N)));
    V v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)o[i];
    if (n == N) {
        store_vec(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = v[i];
    }
}
// The epilogue: outputs p .. p + n - 1 of row q.  bias: of these outputs, loaded by the caller (one that writes many rows loads it
// once: loaded per row it took 15 us of 10,000 x 4,096 outputs' 45).
template <class T, int N> __device__ __forceinline__ void load_bias(const Epilogue<T> &e, int64_t p, int n, float (&bias)[N])
{
    if (e.bias) {
        load_row(e.bias + p, n, bias);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) bias[i] = 0.f;
    }
}
template <class T, int N>
__device__ __forceinline__ void finish(const Epilogue<T> &e, int64_t q, int64_t p, int n, float (&v)[N], const float (&bias)[N])
{
    float u[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += bias[i];
    if (e.z) store_row(e.z + q * e.ldz + p, n, v);
    if (e.act != VF_ACT_NONE)
        by_act(e.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = act_value<act.value, T>(v[i]);
        });
    if (e.residual) {
        load_row(e.residual + q * e.ldr + p, n, u);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += u[i];
    }
    store_row(e.y + q * e.ldy + p, n, v);
}

// The same of a gated layer's n outputs, from both halves of z; z is kept before either is rounded.
template <class T, int N>
__device__ __forceinline__ void finish_gated(const Epilogue<T> &e, int64_t q, int64_t p, int64_t np, int n, float (&gate)[N], float (&up)[N],
                                             const float (&gate_bias)[N], const float (&up_bias)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        gate[i] += gate_bias[i];
        up[i] += up_bias[i];
    }
    if (e.z) {
        store_row(e.z + q * e.ldz + p, n, gate);
        store_row(e.z + q * e.ldz + np + p, n, up);
    }
    by_act(e.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < N; ++i) gate[i] = act_value<act.value, T>(gate[i]) * up[i];
    });
    store_row(e.y + q * e.ldy + p, n, gate);
}

template <class T> struct Product {
    const T *P, *Q;
    int64_t ldp, ldq;
    int64_t np, nq, nc;   // outputs of a row (rows of P; of each of its halves where it is gated), rows of Q, the contraction's length
    int64_t chunk;        // elements of the contraction per split
    int splits;
    float *part;          // [splits][nq][np], gated [splits][nq][2 np], where splits > 1
};

constexpr int kRowBytes = 128;     // bytes of the contraction per step of the tiles below

// ---------------------------------------------------------------- few rows

// At most 16 FQ rows of Q (queries that are served one by one or in small batches): the work is one read of P, so no tile is shared and
// nothing waits for another wave until the end.  A workgroup has 16 rows of P; its waves share the contraction in whole fragments, loaded
// from memory straight into the matrix instruction's layout, several in flight, and add up through LDS.
// One row, 4096 x 1024 in bfloat16 (8 MB of weights): 4.4 us; 64 x 64 tiles over a split contraction and their join took 13.
// Gated: sixteen rows of each half, 8 waves at most; one row, 2 x 4,096 x 1,024 (17 MB) 6.0 us.
template <class T, int FQ, bool GATED = false>
__global__ __launch_bounds__(GATED ? 512 : 1024) void few_rows_kernel(Product<T> a, Epilogue<T> e)
{
    constexpr int V = kVec<T>, BC = 4 * V, G = GATED ? 2 : 1, AHEAD = G * FQ > 2 ? 2 : 4;
    __shared__ __align__(16) float4v sums[16 / G][G * FQ][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t p0 = (int64_t)blockIdx.x * 16;
    const T *P[G];
#pragma unroll
    for (int g = 0; g < G; ++g) P[g] = a.P + (g * a.np + min(p0 + (lane & 15), a.np - 1)) * a.ldp;   // (rows beyond the last repeat it: their results are not kept)
    const T *Q[FQ];
#pragma unroll
    for (int j = 0; j < FQ; ++j) Q[j] = a.Q + min((int64_t)(j * 16 + (lane & 15)), a.nq - 1) * a.ldq;
    float4v acc[G][FQ] = {};
    const int64_t whole = a.nc / BC;   // fragments that the contraction fills
    int64_t f = wave;
    for (; f + (AHEAD - 1) * waves < whole; f += AHEAD * waves) {
        Vec<T> fp[AHEAD][G], fq[AHEAD][FQ];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t c = (f + u * waves) * BC + (lane >> 4) * V;
#pragma unroll
            for (int g = 0; g < G; ++g) fp[u][g] = load_vec<Vec<T>>(P[g] + c);
#pragma unroll
            for (int j = 0; j < FQ; ++j) fq[u][j] = load_vec<Vec<T>>(Q[j] + c);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int j = 0; j < FQ; ++j)
#pragma unroll
                for (int g = 0; g < G; ++g) acc[g][j] = mma(fp[u][g], fq[u][j], acc[g][j]);
    }
    for (; f * BC < a.nc; f += waves) {
        const int64_t c = f * BC + (lane >> 4) * V;
        const int n = (int)max((int64_t)0, min((int64_t)V, a.nc - c));
        Vec<T> fp[G];
#pragma unroll
        for (int g = 0; g < G; ++g) fp[g] = load_part(P[g] + c, n, (T)0.f);
#pragma unroll
        for (int j = 0; j < FQ; ++j) {
            const Vec<T> fq = load_part(Q[j] + c, n, (T)0.f);
#pragma unroll
            for (int g = 0; g < G; ++g) acc[g][j] = mma(fp[g], fq, acc[g][j]);
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
        if (q < a.nq && p < a.np) {
            const int n = (int)min((int64_t)4, a.np - p);
            float bias[G][4];
#pragma unroll
            for (int g = 0; g < G; ++g) load_bias(e, g * a.np + p, n, bias[g]);
            if constexpr (GATED) finish_gated(e, q, p, a.np, n, v[0], v[1], bias[0], bias[1]);
            else finish(e, q, p, n, v[0], bias[0]);
        }
    }
}

// ---------------------------------------------------------------- tiles

// Where element chunks live in a tile in LDS.  An operand that is contiguous along c keeps rows of 128 bytes (eight 16-byte chunks
// at chunk ^ (row % 8)); one that is contiguous along its rows keeps the lines of c as they come, in pieces that the matrix
// instruction's lanes gather with transposing reads (2-byte types) or element by element (float32); the pieces of
// a line are permuted by c so that the lines that one read touches lie in different banks.
template <class T, int ROWS> __device__ __forceinline__ int line_place(int c, int byte)
{
    constexpr int kLine = ROWS * (int)sizeof(T);
    if constexpr (sizeof(T) == 2) return c * kLine + (byte ^ ((((c & 3) | (c >> 1 & 4)) & (kLine / 32 - 1)) << 5));
    else return c * kLine + (byte ^ ((c >> 2 & 3) << 6));
}

typedef short short4v __attribute__((ext_vector_type(4)));

// The fragment of rows r0 .. r0 + 15 and 64 bytes (half h) of the contraction.
template <class T, bool ALONG_C, int ROWS> __device__ __forceinline__ Vec<T> fragment(const unsigned char *tile, int r0, int h, int lane)
{
    if constexpr (ALONG_C) {
        const int r = r0 + (lane & 15), ch = h * 4 + (lane >> 4);
        return *(const Vec<T> *)(tile + r * kRowBytes + ((ch ^ (r & 7)) << 4));
    } else if constexpr (sizeof(T) == 2) {
        // a transposing read hands lane i of sixteen the column i of the four lines whose pieces lanes 4 c .. 4 c + 3 address
        const int c = h * 32 + (lane >> 4) * 8 + (lane >> 2 & 3);
        const unsigned char *at = tile + line_place<T, ROWS>(c, (r0 + (lane & 3) * 4) * 2);
        using P = __attribute__((address_space(3))) short4v *;
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)at);
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at + 4 * ROWS * 2));
        Vec<T> f;
        __builtin_memcpy(&f, &lo, 8);
        __builtin_memcpy((char *)&f + 8, &hi, 8);
        return f;
    } else {
        const int c = h * 16 + (lane >> 4) * 4;
        const unsigned char *at = tile + line_place<T, ROWS>(c, (r0 + (lane & 15)) * 4);
        Vec<T> f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = *(const T *)(at + i * ROWS * 4);
        return f;
    }
}

// Row r of a tile of a gated P, counted in rows of one half: sixteen of the gate, sixteen of the other, and so on.
__device__ __forceinline__ int half_row(int r) { return (r >> 5) * 16 + (r & 15); }

// One thread's share of an operand's tile on its way from memory to LDS.  (Gated: rows, r0 are those of one half.)
template <class T, bool ALONG_C, int ROWS, int THREADS, bool GATED = false> struct Stage {
    static_assert(ALONG_C || !GATED, "");
    static constexpr int V = kVec<T>, BC = kRowBytes / (int)sizeof(T), N = ROWS * 8 / THREADS;
    static constexpr int kLine = ROWS / V;   // vectors of a line of c
    Vec<T> v[N];
    const T *at;        // whole tiles: this thread's first vector in the next step
    int64_t ld, r0, rows;
    const T *src;

    __device__ __forceinline__ void begin(const T *src_, int64_t ld_, int64_t r0_, int64_t rows_, int64_t c0)
    {
        src = src_; ld = ld_; r0 = r0_; rows = rows_;
        const int t = threadIdx.x;
        if constexpr (ALONG_C) at = src + r0 * ld + c0 + t % 8 * V;
        else at = src + (c0 + t / kLine) * ld + r0 + t % kLine * V;
    }
    __device__ __forceinline__ void whole()
    {
        const int t = threadIdx.x;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (ALONG_C) {   // rows beyond the last repeat it: their results are not kept
                const int at_row = t / 8 + i * (THREADS / 8);
                int64_t r = min((int64_t)(GATED ? half_row(at_row) : at_row), rows - 1 - r0);
                if (GATED && (at_row & 16)) r += rows;
                v[i] = load_vec<Vec<T>>(at + r * ld);
            } else {
                v[i] = load_vec<Vec<T>>(at + (int64_t)(i * (THREADS / kLine)) * ld);
            }
        }
        at += ALONG_C ? BC : BC * ld;
    }
    // a step that leaves the operand: zeros beyond its rows and beyond c_end
    __device__ __forceinline__ void part(int64_t c0, int64_t c_end)
    {
        const int t = threadIdx.x;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int id = t + i * THREADS;
            if constexpr (ALONG_C) {
                const int64_t r = r0 + (GATED ? half_row(id / 8) : id / 8), c = c0 + id % 8 * V;
                v[i] = load_part(src + (GATED && (id / 8 & 16) ? r + rows : r) * ld + c, r < rows ? (int)min((int64_t)V, max((int64_t)0, c_end - c)) : 0, (T)0.f);
            } else {
                const int64_t c = c0 + id / kLine, r = r0 + id % kLine * V;
                v[i] = load_part(src + c * ld + r, c < c_end ? (int)min((int64_t)V, max((int64_t)0, rows - r)) : 0, (T)0.f);
            }
        }
        at += ALONG_C ? BC : BC * ld;
    }
    __device__ __forceinline__ void keep(unsigned char *tile) const
    {
        const int t = threadIdx.x;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int id = t + i * THREADS;
            if constexpr (ALONG_C) {
                const int r = id / 8, ch = id % 8;
                *(Vec<T> *)(tile + r * kRowBytes + ((ch ^ (r & 7)) << 4)) = v[i];
            } else {
                *(Vec<T> *)(tile + line_place<T, ROWS>(id / kLine, id % kLine * 16)) = v[i];
            }
        }
    }
};

// The end of a workgroup: each wave turns sixteen rows of its accumulators at a time through LDS, so that its stores are whole stretches
// of a row and not the four neighbours that a lane holds.
// Gated: p_first and the outputs are those of one half; fragments of both lie in turn in a row.
template <class T, int FP, int FQ, int WAVE_P, int WAVE_Q, bool GATED = false>
__device__ __forceinline__ void store_tile(const Product<T> &a, const Epilogue<T> &e, const float4v (&acc)[FP][FQ], unsigned char *lds, int wave,
                                           int lane, int64_t p_first, int64_t q_first)
{
    constexpr int G = GATED ? 2 : 1, kRow = WAVE_P * 4 + 16, kLanes = WAVE_P / 8 / G;   // 16 bytes more: rows start in other banks
    unsigned char *turn = lds + wave * (16 * kRow);   // (at most 68 KiB for eight waves, 35 for four: less than the tiles had)
    const int64_t p = p_first + lane % kLanes * 8;
    const int m = (int)max((int64_t)0, min((int64_t)8, a.np - p));
    float bias[G][8];
#pragma unroll
    for (int g = 0; g < G; ++g) load_bias(e, g * a.np + p, m, bias[g]);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
#pragma unroll
        for (int i = 0; i < FP; ++i) *(float4v *)(turn + (lane & 15) * kRow + (i * 16 + (lane >> 4) * 4) * 4) = acc[i][j];
        wave_sync<true>();
#pragma unroll 1
        for (int r = lane / kLanes; r < 16; r += 64 / kLanes) {
            const int64_t q = q_first + j * 16 + r;
            float v[G][8];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const unsigned char *from = turn + r * kRow + (GATED ? (lane % kLanes >> 1) * 128 + g * 64 + (lane & 1) * 32 : lane % kLanes * 32);
                *(float4v *)v[g] = *(const float4v *)from;
                *(float4v *)(v[g] + 4) = *(const float4v *)(from + 16);
            }
            if (q >= a.nq || m == 0) continue;
            if (a.splits > 1) {
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float *to = a.part + ((int64_t)blockIdx.y * a.nq + q) * (G * a.np) + g * a.np + p;
                    if (m == 8) {
                        store_vec(to, *(float4v *)v[g]);
                        store_vec(to + 4, *(float4v *)(v[g] + 4));
                    } else {
#pragma unroll
                        for (int u = 0; u < 8; ++u)
                            if (u < m) to[u] = v[g][u];
                    }
                }
            } else if constexpr (GATED) {
                finish_gated(e, q, p, a.np, m, v[0], v[1], bias[0], bias[1]);
            } else {
                finish(e, q, p, m, v[0], bias[0]);
            }
        }
        wave_sync<true>();
    }
}

// Where workgroup `group` of `groups` works: tile number p of P and q of Q, of tiles_p and tiles_q.  Neighbouring workgroups go to the eight XCDs in turn: each XCD
// takes a run of tiles, and a run goes through bands of H tiles of Q, so that the tiles in work at the same time share what its L2 has to fetch from either operand.
template <int H> __device__ __forceinline__ void place_tile(int64_t group, int64_t groups, int64_t tiles_p, int64_t tiles_q, int64_t &p, int64_t &q)
{
    const int64_t xcd = group & 7, run = groups / 8, left = groups % 8;
    const int64_t tile = xcd * run + min(xcd, left) + (group >> 3);
    const int64_t band = tile / (H * tiles_p), at = tile - band * (H * tiles_p), high = min((int64_t)H, tiles_q - band * H);
    p = at / high;
    q = band * H + (at - p * high);
}

// BP x BQ outputs per workgroup of WP x WQ waves; two tiles of each operand in LDS, one being read while the other is filled through
// registers, which takes any alignment.  128 x 128 outputs by eight waves, 10,000 x 4,096 x 1,024: float32 123 - 132 TFLOP/s (the library's
// product 137 - 154), bfloat16 with rows that start anywhere 530 - 720; four waves reach half of that (one wave per SIMD waits
// for LDS), 64 x 64 outputs are for products with too few tiles of 128.  Two workgroups of eight waves share a compute unit, which takes at most 128 registers a
// lane: dx in 2-byte types is told so (by itself it came to 140: 11,311 x 2,663 x 968 in bfloat16 158 us, 113 this way).
template <class T, bool PC, bool QC, int BP, int BQ, int WP, int WQ, bool GATED = false>
__global__ __launch_bounds__(WP *WQ * 64, WP *WQ == 8 && !PC && QC && sizeof(T) == 2 ? 4 : 1) void tile_kernel(Product<T> a, Epilogue<T> e)
{
    constexpr int OUT = GATED ? BP / 2 : BP;   // outputs of a row that the tile has
    constexpr int THREADS = WP * WQ * 64, BC = kRowBytes / (int)sizeof(T), FP = BP / WP / 16, FQ = BQ / WQ / 16;
    extern __shared__ __align__(16) unsigned char tiles[];   // [2][(BP + BQ) * kRowBytes]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles_p = (a.np + OUT - 1) / OUT;
    int64_t p0, q0;
    place_tile<8>(blockIdx.x, gridDim.x, tiles_p, (a.nq + BQ - 1) / BQ, p0, q0);
    p0 *= OUT;
    q0 *= BQ;
    const int64_t c_first = (int64_t)blockIdx.y * a.chunk, c_end = min(a.nc, c_first + a.chunk);
    const bool p_whole = PC || p0 + BP <= a.np, q_whole = QC || q0 + BQ <= a.nq;

    Stage<T, PC, BP, THREADS, GATED> sp;
    Stage<T, QC, BQ, THREADS> sq;
    sp.begin(a.P, a.ldp, p0, a.np, c_first);
    sq.begin(a.Q, a.ldq, q0, a.nq, c_first);
    auto fetch = [&](int64_t c0) {
        const bool c_whole = c0 + BC <= c_end;
        if (c_whole && p_whole) sp.whole(); else sp.part(c0, c_end);
        if (c_whole && q_whole) sq.whole(); else sq.part(c0, c_end);
    };
    const int wp = wave % WP * (BP / WP), wq = wave / WP * (BQ / WQ);
    float4v acc[FP][FQ] = {};
    unsigned char *now = tiles, *next = tiles + (BP + BQ) * kRowBytes;
    if (c_first < c_end) {
        fetch(c_first);
        sp.keep(now);
        sq.keep(now + BP * kRowBytes);
    }
    for (int64_t c0 = c_first; c0 < c_end; c0 += BC) {
        __syncthreads();
        const bool more = c0 + BC < c_end;
        if (more) fetch(c0 + BC);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Vec<T> fp[FP], fq[FQ];
#pragma unroll
            for (int i = 0; i < FP; ++i) fp[i] = fragment<T, PC, BP>(now, wp + i * 16, h, lane);
#pragma unroll
            for (int j = 0; j < FQ; ++j) fq[j] = fragment<T, QC, BQ>(now + BP * kRowBytes, wq + j * 16, h, lane);
#pragma unroll
            for (int j = 0; j < FQ; ++j)
#pragma unroll
                for (int i = 0; i < FP; ++i) acc[i][j] = mma(fp[i], fq[j], acc[i][j]);
        }
        if (more) {
            sp.keep(next);
            sq.keep(next + BP * kRowBytes);
        }
        unsigned char *t = now;
        now = next;
        next = t;
    }
    store_tile<T, FP, FQ, BP / WP, BQ / WQ, GATED>(a, e, acc, tiles, wave, lane, p0 + (GATED ? wp / 2 : wp), q0 + wq);
}

// The same for whole, aligned operands of 2-byte types: memory goes to LDS directly (no registers on the way), STEPS steps of 64 bytes of
// the contraction deep.  While step t's fragments are multiplied, those of step t + 1 are read and step t + STEPS is requested into
// the buffer that step t has left, so that a step waits only for loads STEPS - 1 steps old.
//
// The compiler does not see these loads (they have no result); what they need is stated by hand: before a barrier each wave waits for its
// own loads of step t + 1 (loads return in order: all but those of the steps after it) and for its own reads of step t, so
// that beyond the barrier every wave's part of t + 1 is there and nobody reads step t's buffer any more.

// Rows of 64 bytes, four to a line of the banks: their chunks are permuted so that the sixteen lanes that LDS serves together (0-3,
// 12-15, 20-27 and so on) touch sixteen different ones.
__device__ __forceinline__ int direct_chunk(int r, int ch) { return ch ^ ((r >> 1 & 2) ^ (r >> 3 & 1) * 3); }

// Offsets from the tile's first element, in bytes, of what a lane requests with the i-th load of an operand's step.  (Gated: from the first
// element of the half that the piece's sixteen rows belong to.)
template <class T, bool ALONG_C, int ROWS, bool GATED = false>
__device__ __forceinline__ uint32_t direct_offset(int piece, int lane, int64_t ld, int64_t rows_left)
{
    // a piece is 1024 bytes of the tile in LDS
    if constexpr (ALONG_C) {
        const int r = piece * 16 + (lane >> 2);
        return (uint32_t)(min((int64_t)(GATED ? half_row(r) : r), rows_left - 1) * ld * (int64_t)sizeof(T)) + (direct_chunk(r, lane & 3) << 4);
    } else {
        constexpr int kLine = ROWS / 8;   // 16-byte chunks of a line
        const int id = piece * 64 + lane, c = id / kLine;
        const int byte = line_place<T, ROWS>(c, id % kLine * 16) - c * ROWS * 2;
        return (uint32_t)(c * ld * (int64_t)sizeof(T)) + (uint32_t)min((int64_t)byte, rows_left * (int64_t)sizeof(T) - 16);
    }
}

// Sixteen bytes a lane from base + offset to LDS at `to` + 16 lane.  (A load to LDS may read m0 one wait state after its write at the earliest.)
__device__ __forceinline__ void request(const void *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory", "m0");
}

template <class T, bool ALONG_C, int ROWS> __device__ __forceinline__ Vec<T> direct_fragment(const unsigned char *tile, int r0, int lane)
{
    if constexpr (ALONG_C) {
        const int r = r0 + (lane & 15);
        return *(const Vec<T> *)(tile + r * 64 + (direct_chunk(r, lane >> 4) << 4));
    } else {
        return fragment<T, false, ROWS>(tile, r0, 0, lane);
    }
}

// BP x BQ outputs per workgroup of WP x WQ waves.  Bound by the matrix cores' clock under load and by how evenly the tiles fill 256
// compute units.  bfloat16, bare products one after the other: 8,192 x 4,096 x 2,048 forward 115 us, dx 103, dw 130 with its join (the library 96, 105
// and 131); 10,000 x 4,096 x 1,024 forward 95 us, dx 76, dw 85 with its join (880 - 1,100 TFLOP/s; the library 87 - 96, 83 and 116).  In such
// a product with GELU and z the matrix cores are busy for a third of the cycles, in its dx and dw for half.  8,192^3 with rows 8,192 apart on both sides: forward
// 831 us, dx 782 (the library 719 and 787); before the order of place_tile 1,225 and 809.  Gated, 10,000 x (2 x 4,096) x 1,024: 164 us, with z kept 174 (the library's
// bare product of all 8,192 rows 161).  A smaller tile reads more of its operands per product from L2: 128 x 128 takes 15 - 30 % longer where the tiles are many.
template <class T, bool PC, bool QC, int BP, int BQ, int WP, int WQ, int STEPS, bool GATED = false>
__global__ __launch_bounds__(WP *WQ * 64, 2) void direct_kernel(Product<T> a, Epilogue<T> e)
{
    static_assert(!GATED || (PC && BP / WP % 32 == 0), "");
    constexpr int OUT = GATED ? BP / 2 : BP;   // outputs of a row that the tile has
    constexpr int BC = 32, WAVES = WP * WQ, FP = BP / WP / 16, FQ = BQ / WQ / 16;
    constexpr int NP = BP / 16, NQ = BQ / 16;   // loads of a step; where they do not divide among the waves the last one is made twice
    constexpr int LP = (NP + WAVES - 1) / WAVES, LQ = (NQ + WAVES - 1) / WAVES, LOADS = LP + LQ;
    constexpr int kStep = (BP + BQ) * 64;
    extern __shared__ __align__(16) unsigned char tiles[];   // [STEPS][P, Q][rows of 64 bytes, or 32 lines]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t tiles_p = (a.np + OUT - 1) / OUT;
    int64_t p0, q0;
    place_tile<(BP * BQ > 32768 ? 4 : 8)>(blockIdx.x, gridDim.x, tiles_p, (a.nq + BQ - 1) / BQ, p0, q0);
    p0 *= OUT;
    q0 *= BQ;
    const int64_t c_first = (int64_t)blockIdx.y * a.chunk, c_end = min(a.nc, c_first + a.chunk);
    const int steps = (int)max((int64_t)0, (c_end - c_first) / BC);

    const T *P = PC ? a.P + p0 * a.ldp + c_first : a.P + c_first * a.ldp + p0;
    const T *Q = QC ? a.Q + q0 * a.ldq + c_first : a.Q + c_first * a.ldq + q0;
    uint32_t off_p[LP], off_q[LQ];
#pragma unroll
    for (int i = 0; i < LP; ++i) off_p[i] = direct_offset<T, PC, BP, GATED>(min(wave * LP + i, NP - 1), lane, a.ldp, a.np - p0);
#pragma unroll
    for (int i = 0; i < LQ; ++i) off_q[i] = direct_offset<T, QC, BQ>(min(wave * LQ + i, NQ - 1), lane, a.ldq, a.nq - q0);
    const int64_t step_p = PC ? BC : BC * a.ldp, step_q = QC ? BC : BC * a.ldq;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)tiles;
    auto buffer_of = [](int t) { return (STEPS & (STEPS - 1)) == 0 ? t & (STEPS - 1) : t % STEPS; };
    auto request_some = [&](int t, int first, int last) {   // loads first .. last - 1 of a step's
        const uint32_t at = buffer_of(t) * kStep;
        const T *p = P + t * step_p, *q = Q + t * step_q;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if (i < first || i >= last) continue;
            if (i < LP) {
                const int piece = min(wave * LP + i, NP - 1);
                request(GATED && (piece & 1) ? p + a.np * a.ldp : p, off_p[i], lds0 + at + piece * 1024);
            }
            else request(q, off_q[i - LP], lds0 + BP * 64 + at + min(wave * LQ + i - LP, NQ - 1) * 1024);
        }
    };
    const int wp = wave % WP * (FP * 16), wq = wave / WP * (FQ * 16);
    float4v acc[FP][FQ] = {};
    Vec<T> fp[2][FP], fq[2][FQ];
    auto read_step = [&](int t, Vec<T> (&p)[FP], Vec<T> (&q)[FQ]) {
        const unsigned char *at = tiles + buffer_of(t) * kStep;
#pragma unroll
        for (int j = 0; j < FQ; ++j) q[j] = direct_fragment<T, QC, BQ>(at + BP * 64, wq + j * 16, lane);
#pragma unroll
        for (int i = 0; i < FP; ++i) p[i] = direct_fragment<T, PC, BP>(at, wp + i * 16, lane);
    };
    auto multiply = [&](const Vec<T> (&p)[FP], const Vec<T> (&q)[FQ]) {
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FQ; ++j) acc[i][j] = mma(p[i], q[j], acc[i][j]);
    };
    if (steps > 0) {
        for (int t = 0; t < min(steps, STEPS); ++t) request_some(t, 0, LOADS);
        if (steps >= STEPS) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STEPS - 1) * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        asm volatile("s_barrier" ::: "memory");
        read_step(0, fp[0], fq[0]);
    }
    // A step in four parts, each with a quarter of its matrix instructions and between them a quarter of the next step's reads and of the
    // requests.  (Requests in one go at its start held the waves up until the last of them had been taken, 16 cycles each.)
    // MORE: step t + STEPS exists.
    auto one_step = [&](auto more, int t, int set) {
        constexpr int kParts = 4, kFragments = FP + FQ, kRows = FP / kParts;
        __builtin_amdgcn_sched_barrier(0);
        if (more.value || t + STEPS - 1 < steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STEPS - 2) * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const bool request_more = more.value || t + STEPS < steps;
        const unsigned char *at = tiles + buffer_of(t + 1) * kStep;   // (beyond the last step: a buffer's old contents, not used)
#pragma unroll
        for (int g = 0; g < kParts; ++g) {
            __builtin_amdgcn_sched_barrier(0);
            if (request_more) request_some(t + STEPS, g * LOADS / kParts, (g + 1) * LOADS / kParts);
            constexpr int kReads = (kFragments * 2 + kParts - 1) / kParts;
#pragma unroll
            for (int f = g * kFragments / kParts; f < (g + 1) * kFragments / kParts; ++f) {
                if (f < FQ) fq[set ^ 1][f] = direct_fragment<T, QC, BQ>(at + BP * 64, wq + f * 16, lane);
                else fp[set ^ 1][f - FQ] = direct_fragment<T, PC, BP>(at, wp + (f - FQ) * 16, lane);
            }
#pragma unroll
            for (int i = g * kRows; i < (g + 1) * kRows; ++i)
#pragma unroll
                for (int j = 0; j < FQ; ++j) acc[i][j] = mma(fp[set][i], fq[set][j], acc[i][j]);
#pragma unroll
            for (int u = 0; u < kReads; ++u) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a matrix instruction,
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);   // an LDS read
            }
        }
    };
    int t = 0;
    for (; t + 1 + STEPS < steps; t += 2) {
        one_step(std::true_type(), t, 0);
        one_step(std::true_type(), t + 1, 1);
    }
    for (; t + 1 < steps; t += 2) {
        one_step(std::false_type(), t, 0);
        one_step(std::false_type(), t + 1, 1);
    }
    if (t < steps) multiply(fp[0], fq[0]);
    if (c_first + (int64_t)steps * BC < c_end) {   // what is left of the contraction, through registers, with zeros beyond it
        const int64_t c0 = c_first + (int64_t)steps * BC;
        __syncthreads();
        auto keep_part = [&](auto along_c, auto rows_of, auto in_halves, const T *src, int64_t ld, int64_t r0, int64_t rows, unsigned char *to) {
            constexpr int ROWS = rows_of.value, kLine = ROWS / 8;
            constexpr bool kHalves = in_halves.value;
            for (int id = threadIdx.x; id < ROWS * 4; id += WAVES * 64) {
                if constexpr (along_c.value) {
                    const int r = id >> 2, ch = id & 3;
                    const int64_t c = c0 + ch * 8, from = r0 + (kHalves ? half_row(r) : r);
                    *(Vec<T> *)(to + r * 64 + (direct_chunk(r, ch) << 4)) =
                        load_part(src + (kHalves && (r & 16) ? from + rows : from) * ld + c, from < rows ? (int)min((int64_t)8, max((int64_t)0, c_end - c)) : 0, (T)0.f);
                } else {
                    const int64_t c = c0 + id / kLine, r = r0 + id % kLine * 8;
                    *(Vec<T> *)(to + line_place<T, ROWS>(id / kLine, id % kLine * 16)) =
                        load_part(src + c * ld + r, c < c_end ? (int)min((int64_t)8, max((int64_t)0, rows - r)) : 0, (T)0.f);
                }
            }
        };
        keep_part(std::integral_constant<bool, PC>(), std::integral_constant<int, BP>(), std::integral_constant<bool, GATED>(), a.P, a.ldp, p0, a.np, tiles);
        keep_part(std::integral_constant<bool, QC>(), std::integral_constant<int, BQ>(), std::false_type(), a.Q, a.ldq, q0, a.nq, tiles + BP * 64);
        __syncthreads();
        read_step(0, fp[0], fq[0]);
        multiply(fp[0], fq[0]);
    }
    store_tile<T, FP, FQ, FP * 16, FQ * 16, GATED>(a, e, acc, tiles, wave, lane, p0 + (GATED ? wp / 2 : wp), q0 + wq);
}

// a += the splits' sums of n (0 .. N) neighbours, in order; split: elements from one's to the next, half: to the other half's.  Four splits are on their way at a
// time: outputs of few rows have many splits and too few threads to wait for each by itself (288 x 2 x 181 in 8 bits, six splits: 7.5 us, 12 one by one).
template <int G, int N>
__device__ __forceinline__ void join_splits(const float *__restrict__ part, int64_t split, int64_t half, int splits, int n, float (&a)[G][N])
{
    using V = float __attribute__((ext_vector_type(N)));
    if (n <= 0) return;
    if (n >= N) {
        for (int s = 0; s < splits; s += 4) {
            V u[4][G];
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int g = 0; g < G; ++g) u[k][g] = load_vec<V>(part + min(s + k, splits - 1) * split + g * half);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int j = 0; j < N; ++j) a[g][j] += s + k < splits ? u[k][g][j] : 0.f;
        }
        return;
    }
    for (int s = 0; s < splits; s += 4) {   // (the same element by element)
        float u[4][G][N];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int j = 0; j < N; ++j) u[k][g][j] = part[min(s + k, splits - 1) * split + g * half + min(j, n - 1)];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int j = 0; j < N; ++j) a[g][j] += s + k < splits && j < n ? u[k][g][j] : 0.f;
    }
}

// The splits' sums, in order, and the epilogue: 4 x 4,096 x 1,024 in 12 us, 6 TB/s.
template <class T, bool GATED = false>
__global__ __launch_bounds__(256) void product_join_kernel(int64_t np, int64_t nq, int splits, const float *__restrict__ part, Epilogue<T> e)
{
    const int64_t quads = (np + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quads * nq; i += (int64_t)gridDim.x * 256) {
        const int64_t q = i / quads, p = (i - q * quads) * 4;
        const int n = (int)min((int64_t)4, np - p);
        constexpr int G = GATED ? 2 : 1;
        float a[G][4] = {};
        join_splits<G, 4>(part + q * (G * np) + p, nq * (G * np), np, splits, n, a);
        float bias[G][4];
#pragma unroll
        for (int g = 0; g < G; ++g) load_bias(e, g * np + p, n, bias[g]);
        if constexpr (GATED) finish_gated(e, q, p, np, n, a[0], a[1], bias[0], bias[1]);
        else finish(e, q, p, n, a[0], bias[0]);
    }
}

// ---------------------------------------------------------------- host side

// The kernels of a product, by the tile that a workgroup computes.
enum Tiling {
    kFewRows,       // 16 rows of P, all rows of Q (at most 64); both operands along c
    kSmall,         // 64 x 64, any operands
    kMedium,        // 128 x 128, any operands
    kDirect128,     // 128 x 128, aligned operands of 2 bytes, straight to LDS
    kDirectWide,    // 128 x 256, two workgroups per compute unit; both operands along c
    kDirect192,     // 256 x 192, the same, any operands
    kDirect256,     // 256 x 256, the same
};

// What a tiling costs, in microseconds: `step` per 128 bytes of the contraction with a compute unit full of `together` workgroups, at
// least `alone` however few there are; `fixed` per workgroup for its first loads and its stores.  Fitted to 2,255 timings: 39 sizes
// from 32 x 1,024 x 1,024 to 8,192 x 4,096 x 2,048, each product, every tiling and 1 to 32 splits.  Timed again with tiles in place_tile's order and splits joined four at a
// time, what it picks takes 2.9 % longer than the best of all on average, more than 10 % for 10 of 117 products, 31 % at worst (dx of 4,000 x 1,024 x 1,024 whose rows start
// anywhere: 64 x 64 for 128 x 128).
struct TilingCost {
    int bp, bq, together;
    double step, alone, fixed;
};
inline TilingCost cost_of(Tiling t, bool f32, bool both_along)
{
    switch (t) {
    case kSmall:
        return f32 ? (both_along ? TilingCost{64, 64, 4, 2.2, 0.77, 3.9} : TilingCost{64, 64, 4, 2.3, 0.90, 3.9})
                   : (both_along ? TilingCost{64, 64, 4, 0.95, 0.40, 3.4} : TilingCost{64, 64, 4, 0.95, 0.67, 3.5});
    case kMedium:
        return f32 ? TilingCost{128, 128, 2, 3.2, 2.1, 4.6}
                   : (both_along ? TilingCost{128, 128, 2, 1.0, 0.85, 3.6} : TilingCost{128, 128, 2, 1.3, 0.95, 4.0});
    case kDirect128: return both_along ? TilingCost{128, 128, 3, 1.43, 0.46, 4.2} : TilingCost{128, 128, 3, 1.35, 0.68, 4.6};
    case kDirectWide: return TilingCost{128, 256, 2, 1.4, 0.74, 5.6};
    case kDirect192: return both_along ? TilingCost{256, 192, 1, 0.97, 0.60, 4.8} : TilingCost{256, 192, 1, 0.95, 0.60, 5.5};
    default: return both_along ? TilingCost{256, 256, 1, 1.13, 0.61, 6.0} : TilingCost{256, 256, 1, 1.2, 0.61, 6.4};
    }
}
// The few rows' kernel reads P's 16 rows and all of Q's per workgroup, two workgroups per compute unit: latency where there are few
// workgroups (7 us for 64 x 4,096 x 1,024), else P through memory and Q's rows once per workgroup through the caches (200,000 x 1,024
// in bfloat16: 76 us for one row, 99 for 8, 115 for 16; 128 x 128 tiles take 94 for any of these).
inline double few_rows_us(int64_t np, int64_t nq, int64_t row_bytes)
{
    const double groups = (double)ceil_div(np, 16);
    const double latency = 3 + 0.4 * (double)row_bytes / 1024 * (nq <= 16 ? 2 : nq <= 32 ? 3 : 5) * std::ceil(groups / 512);
    return std::max(latency, (double)np * row_bytes / 5.3e6 + groups * nq * row_bytes / 10e6);
}

// The same of a gated layer, np rows of both halves: half as many waves, each with twice the loads, and Q's rows once for both.  The last term is what workgroups cost by
// themselves, which counts where the contraction is short (2 x 65,536 x 100 in bfloat16, 33 rows: 38 us, 14 in tiles of 64 x 64).
inline double few_rows_gated_us(int64_t np, int64_t nq, int64_t row_bytes)
{
    const double groups = (double)ceil_div(np, 16), rows = nq <= 16 ? 16 : nq <= 32 ? 32 : 64;
    const double latency = 3 + 0.6 * (double)row_bytes / 1024 * (nq <= 16 ? 2 : nq <= 32 ? 3 : 5);
    return std::max({latency, 3 + (double)np * row_bytes / 5.3e6 + groups * rows * row_bytes / 25e6, 3 + groups * 1e-4 * (nq <= 16 ? 2 : nq <= 32 ? 13 : 40)});
}

struct ProductPlan {
    bool fits = true;     // false: no tiling has few enough tiles
    Tiling tiling = kSmall;
    int splits = 1;
    int64_t chunk = 0;    // elements of the contraction per split
    size_t bytes = 0;     // of workspace
};

// What the choice of a kernel depends on beside the sizes.
struct Operands {
    bool p_along, q_along;   // contiguous along the contraction
    bool costly_act;         // an epilogue with GELU or SiLU
    bool direct;             // 2-byte types; rows start on 16 bytes, and an operand contiguous along its rows has whole vectors of them
    bool gated = false;
};

constexpr int64_t kMaxTiles = 1 << 22;   // and more are not launched: a launch holds fewer than 2^32 threads

// The tiling and the number of splits of the contraction that should take least time.  A split costs its partial sums' way
// through memory and one more launch (5.5 us: small products come one after the other as fast as the host can launch them); it pays where
// there are too few tiles for the chip's 256 compute units.  Nothing is faster than memory.
inline ProductPlan plan_product(int32_t dtype, int64_t np, int64_t nq, int64_t nc, const Operands &o)
{
    ProductPlan best;
    const bool f32 = dtype == VF_F32;
    const int64_t step = kRowBytes / (int64_t)type_size(dtype);
    const bool both = o.p_along && o.q_along;
    const double floor_us = ((double)np * nc + (double)nq * nc + (double)np * nq) * type_size(dtype) / 5e6;
    double least = 0;
    if (both && nq <= 64) {
        best.tiling = kFewRows;
        best.chunk = nc;
        least = few_rows_us(np, nq, nc * (int64_t)type_size(dtype));
        if (o.gated) least = few_rows_gated_us(np, nq, nc * (int64_t)type_size(dtype));
        // (the quickest that any tile could be: one split, or one step of many; a call of few rows should not wait for its plan)
        if (least <= std::min(3.4 + 0.4 * (double)ceil_div(nc, step), 9.3)) return best;
    }
    for (Tiling t : {kSmall, kMedium, kDirect128, kDirectWide, kDirect192, kDirect256}) {
        if (t >= kDirect128 && !o.direct) continue;
        if (t == kDirectWide && !both) continue;
        TilingCost c = cost_of(t, f32, both);
        // 9 us of a compute unit's vector ALUs for 256 x 256 outputs, three quarters of that where other workgroups multiply meanwhile
        // (10,000 x 4,096 x 1,024 with GELU: 114 us in tiles of 128 x 256, 124 in 256 x 256; without 93 and 98)
        if (o.costly_act) c.fixed += 9.0 * c.together * c.bp * c.bq / 65536 * (c.together > 1 ? 0.75 : 1);
        const int64_t tiles = ceil_div(np, c.bp) * ceil_div(nq, c.bq);
        if (tiles >= kMaxTiles) continue;
        for (int64_t splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            const int64_t chunk = std::max<int64_t>(step, ceil_div(ceil_div(nc, splits), step) * step);
            const int64_t used = std::max<int64_t>(1, ceil_div(nc, chunk));
            if (splits > 1 && (chunk < 2 * step || tiles * splits > 2048)) break;
            if (used != splits) continue;
            const int64_t per_cu = ceil_div(tiles * used, 256), rounds = ceil_div(per_cu, c.together);
            const double steps = (double)ceil_div(chunk, step);
            const double last = (double)(per_cu - (rounds - 1) * c.together) / c.together;   // how full the last round is
            double us = (double)(rounds - 1) * (steps * c.step + c.fixed) + steps * std::max(c.alone, c.step * last) + c.fixed;
            us = std::max(us, floor_us) + 0.05 * us;   // (the second part tells apart what memory makes equal)
            if (used > 1) us += 5.5 + (double)used * np * nq * 8 / 4e6;
            if (least == 0 || us < least) {
                least = us;
                best.tiling = t;
                best.splits = (int)used;
                best.chunk = chunk;
                best.bytes = used > 1 ? (size_t)used * nq * np * 4 : 0;
            }
        }
    }
    best.fits = least > 0;
    return best;
}

// More than 64 KiB of LDS has to be allowed once per kernel and device.  (`done`: the devices where it has been; asking again does no harm.)
inline int allow_lds(const void *kernel, size_t bytes, std::atomic<uint64_t> &done)
{
    int dev = 0;
    VF_HIP(hipGetDevice(&dev));
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return VF_OK;
    VF_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    done.fetch_or(bit, std::memory_order_relaxed);
    return VF_OK;
}

template <class T, bool PC, bool QC, int BP, int BQ, int WP, int WQ, int STEPS, bool GATED>
int launch_direct(const Product<T> &a, const Epilogue<T> &e, dim3 grid, hipStream_t s)
{
    constexpr size_t lds = (size_t)STEPS * (BP + BQ) * 64;
    static std::atomic<uint64_t> done{0};
    if constexpr (lds > 64 * 1024)
        if (int rc = allow_lds((const void *)direct_kernel<T, PC, QC, BP, BQ, WP, WQ, STEPS, GATED>, lds, done); rc != VF_OK) return rc;
    direct_kernel<T, PC, QC, BP, BQ, WP, WQ, STEPS, GATED><<<grid, dim3(WP * WQ * 64), lds, s>>>(a, e);
    return VF_OK;
}

// Gated: np is that of one half, the plan that of both halves' rows.
template <class T, bool PC, bool QC, bool GATED = false>
int run_product(int32_t dtype, const T *P, int64_t ldp, int64_t np, const T *Q, int64_t ldq, int64_t nq, int64_t nc,
                       const Epilogue<T> &e, const ProductPlan &plan, float *part, hipStream_t s)
{
    if (np == 0 || nq == 0) return VF_OK;
    const Product<T> a{P, Q, ldp, ldq, np, nq, nc, plan.chunk, plan.splits, part};
    if (plan.tiling == kFewRows) {
        if constexpr (PC && QC) {
            // four fragments of the contraction and more for each wave
            const int waves = (int)std::max<int64_t>(1, std::min<int64_t>(GATED ? 8 : 16, nc / (4 * 4 * kVec<T>)));
            const dim3 grid((unsigned)ceil_div(np, 16)), block(waves * 64);
            if (nq <= 16) few_rows_kernel<T, 1, GATED><<<grid, block, 0, s>>>(a, e);
            else if (nq <= 32) few_rows_kernel<T, 2, GATED><<<grid, block, 0, s>>>(a, e);
            else few_rows_kernel<T, 4, GATED><<<grid, block, 0, s>>>(a, e);
        }
        VF_HIP(hipGetLastError());
        return VF_OK;
    }
    const TilingCost c = cost_of(plan.tiling, dtype == VF_F32, PC && QC);
    const int64_t tiles = ceil_div(np, GATED ? c.bp / 2 : c.bp) * ceil_div(nq, c.bq);
    const dim3 grid((unsigned)tiles, (unsigned)plan.splits);
    int rc = VF_OK;
    if (plan.tiling == kSmall) {
        tile_kernel<T, PC, QC, 64, 64, 2, 2, GATED><<<grid, dim3(256), (size_t)2 * 128 * kRowBytes, s>>>(a, e);
    } else if (plan.tiling == kMedium) {
        constexpr size_t lds = (size_t)2 * 256 * kRowBytes;   // 64 KiB, which need not be asked for
        static_assert(lds <= 64 * 1024, "");
        tile_kernel<T, PC, QC, 128, 128, 2, 4, GATED><<<grid, dim3(512), lds, s>>>(a, e);
    } else if constexpr (sizeof(T) == 2) {
        if (plan.tiling == kDirect192) rc = launch_direct<T, PC, QC, 256, 192, 4, 2, 4, GATED>(a, e, grid, s);
        else if (plan.tiling == kDirect256) rc = launch_direct<T, PC, QC, 256, 256, 2, 4, 4, GATED>(a, e, grid, s);
        else if (plan.tiling == kDirect128) rc = launch_direct<T, PC, QC, 128, 128, 2, 2, 3, GATED>(a, e, grid, s);
        else if constexpr (PC && QC) rc = launch_direct<T, PC, QC, 128, 256, 2, 2, 3, GATED>(a, e, grid, s);
    }
    if (rc != VF_OK) return rc;
    if (plan.splits > 1)
        product_join_kernel<T, GATED><<<dim3((unsigned)std::min<int64_t>(ceil_div(ceil_div(np, 4) * nq, 256), 4096)), dim3(256), 0, s>>>(
            np, nq, plan.splits, part, e);
    VF_HIP(hipGetLastError());
    return VF_OK;
}

inline size_t rounded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

inline bool costly(int32_t act) { return act == VF_ACT_GELU || act == VF_ACT_SILU; }

// Whether rows of an operand that lie `ld` elements apart can go to LDS directly: the kernel's offsets within a tile have 32 bits.
inline bool direct_rows(int32_t dtype, const void *p, int64_t ld)
{
    return dtype != VF_F32 && ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < (1 << 21);
}

// Workspace of a product whose operands' alignment is not known yet.
inline size_t most_bytes(int32_t dtype, int64_t np, int64_t nq, int64_t nc, bool p_along, bool q_along, bool costly, bool gated = false)
{
    return std::max(plan_product(dtype, np, nq, nc, {p_along, q_along, costly, false, gated}).bytes,
                    dtype == VF_F32 ? 0 : plan_product(dtype, np, nq, nc, {p_along, q_along, costly, true, gated}).bytes);
}

}  // namespace vf
