// The linear layer y = act(x w^T + bias) + residual and its gradients: three matrix products on the matrix cores that share
// one kernel.  Every product is written as
//     out[q][p] = sum over c of Q[q][c] P[p][c]
// with each operand either contiguous along c or along its own rows:
//     forward   P = w  (along c),      Q = x  (along c),     c = k
//     dx        P = w  (along rows),   Q = dz (along c),     c = n
//     dw        P = x  (along rows),   Q = dz (along rows),  c = m
// P takes the matrix instruction's first operand, so that a lane's four accumulators are neighbours in a row of the output.
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

template <class T> struct Product {
    const T *P, *Q;
    int64_t ldp, ldq;
    int64_t np, nq, nc;   // rows of P and of Q, the contraction's length
    int64_t chunk;        // elements of the contraction per split
    int splits;
    float *part;          // [splits][nq][np] where splits > 1
};

constexpr int kRowBytes = 128;     // bytes of the contraction per step of the tiles below

// ---------------------------------------------------------------- few rows

// At most 16 FQ rows of Q (queries that are served one by one or in small batches): the work is one read of P, so no tile is shared and
// nothing waits for another wave until the end.  A workgroup has 16 rows of P; its waves share the contraction in whole fragments, loaded
// from memory straight into the matrix instruction's layout, several in flight, and add up through LDS.
// One row, 4096 x 1024 in bfloat16 (8 MB of weights): 4.4 us; 64 x 64 tiles over a split contraction and their join took 13.
template <class T, int FQ>
__global__ __launch_bounds__(1024) void few_rows_kernel(Product<T> a, Epilogue<T> e)
{
    constexpr int V = kVec<T>, BC = 4 * V, AHEAD = FQ > 2 ? 2 : 4;
    __shared__ __align__(16) float4v sums[16][FQ][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t p0 = (int64_t)blockIdx.x * 16;
    const T *P = a.P + min(p0 + (lane & 15), a.np - 1) * a.ldp;   // (rows beyond the last repeat it: their results are not kept)
    const T *Q[FQ];
#pragma unroll
    for (int j = 0; j < FQ; ++j) Q[j] = a.Q + min((int64_t)(j * 16 + (lane & 15)), a.nq - 1) * a.ldq;
    float4v acc[FQ] = {};
    const int64_t whole = a.nc / BC;   // fragments that the contraction fills
    int64_t f = wave;
    for (; f + (AHEAD - 1) * waves < whole; f += AHEAD * waves) {
        Vec<T> fp[AHEAD], fq[AHEAD][FQ];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t c = (f + u * waves) * BC + (lane >> 4) * V;
            fp[u] = load_vec<Vec<T>>(P + c);
#pragma unroll
            for (int j = 0; j < FQ; ++j) fq[u][j] = load_vec<Vec<T>>(Q[j] + c);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int j = 0; j < FQ; ++j) acc[j] = mma(fp[u], fq[u][j], acc[j]);
    }
    for (; f * BC < a.nc; f += waves) {
        const int64_t c = f * BC + (lane >> 4) * V;
        const int n = (int)max((int64_t)0, min((int64_t)V, a.nc - c));
        const Vec<T> fp = load_part(P + c, n, (T)0.f);
#pragma unroll
        for (int j = 0; j < FQ; ++j) acc[j] = mma(fp, load_part(Q[j] + c, n, (T)0.f), acc[j]);
    }
#pragma unroll
    for (int j = 0; j < FQ; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    for (int j = wave; j < FQ; j += waves) {
        float v[4] = {};
        for (int w = 0; w < waves; ++w) {
            const float4v u = sums[w][j][lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += u[i];
        }
        const int64_t q = j * 16 + (lane & 15), p = p0 + (lane >> 4) * 4;
        if (q < a.nq && p < a.np) {
            const int n = (int)min((int64_t)4, a.np - p);
            float bias[4];
            load_bias(e, p, n, bias);
            finish(e, q, p, n, v, bias);
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

// One thread's share of an operand's tile on its way from memory to LDS.
template <class T, bool ALONG_C, int ROWS, int THREADS> struct Stage {
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
                const int64_t r = min((int64_t)(t / 8 + i * (THREADS / 8)), rows - 1 - r0);
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
                const int64_t r = r0 + id / 8, c = c0 + id % 8 * V;
                v[i] = load_part(src + r * ld + c, r < rows ? (int)min((int64_t)V, max((int64_t)0, c_end - c)) : 0, (T)0.f);
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
template <class T, int FP, int FQ, int WAVE_P, int WAVE_Q>
__device__ __forceinline__ void store_tile(const Product<T> &a, const Epilogue<T> &e, const float4v (&acc)[FP][FQ], unsigned char *lds, int wave,
                                           int lane, int64_t p_first, int64_t q_first)
{
    constexpr int kRow = WAVE_P * 4 + 16, kLanes = WAVE_P / 8;   // 16 bytes more: rows start in other banks
    unsigned char *turn = lds + wave * (16 * kRow);   // (at most 68 KiB for eight waves, 35 for four: less than the tiles had)
    const int64_t p = p_first + lane % kLanes * 8;
    const int m = (int)max((int64_t)0, min((int64_t)8, a.np - p));
    float bias[8];
    load_bias(e, p, m, bias);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
#pragma unroll
        for (int i = 0; i < FP; ++i) *(float4v *)(turn + (lane & 15) * kRow + (i * 16 + (lane >> 4) * 4) * 4) = acc[i][j];
        wave_sync<true>();
#pragma unroll 1
        for (int r = lane / kLanes; r < 16; r += 64 / kLanes) {
            const int64_t q = q_first + j * 16 + r;
            float v[8];
            *(float4v *)v = *(const float4v *)(turn + r * kRow + lane % kLanes * 32);
            *(float4v *)(v + 4) = *(const float4v *)(turn + r * kRow + lane % kLanes * 32 + 16);
            if (q >= a.nq || m == 0) continue;
            if (a.splits > 1) {
                float *to = a.part + ((int64_t)blockIdx.y * a.nq + q) * a.np + p;
                if (m == 8) {
                    store_vec(to, *(float4v *)v);
                    store_vec(to + 4, *(float4v *)(v + 4));
                } else {
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (u < m) to[u] = v[u];
                }
            } else {
                finish(e, q, p, m, v, bias);
            }
        }
        wave_sync<true>();
    }
}

// BP x BQ outputs per workgroup of WP x WQ waves; two tiles of each operand in LDS, one being read while the other is filled through
// registers, which takes any alignment.  128 x 128 outputs by eight waves, 10,000 x 4,096 x 1,024: float32 123 - 132 TFLOP/s (the library's
// product 137 - 154), bfloat16 with rows that start anywhere 530 - 720; four waves reach half of that (one wave per SIMD waits
// for LDS), 64 x 64 outputs are for products with too few tiles of 128.
template <class T, bool PC, bool QC, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__(WP *WQ * 64) void tile_kernel(Product<T> a, Epilogue<T> e)
{
    constexpr int THREADS = WP * WQ * 64, BC = kRowBytes / (int)sizeof(T), FP = BP / WP / 16, FQ = BQ / WQ / 16;
    extern __shared__ __align__(16) unsigned char tiles[];   // [2][(BP + BQ) * kRowBytes]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles_p = (a.np + BP - 1) / BP;
    // neighbouring workgroups go to the eight XCDs in turn: each XCD takes a run of neighbouring tiles, whose operands its L2 holds
    const int64_t n = gridDim.x, xcd = blockIdx.x & 7, run = n / 8, left = n % 8;
    const int64_t tile = xcd * run + min(xcd, left) + (blockIdx.x >> 3);
    const int64_t p0 = tile % tiles_p * BP, q0 = tile / tiles_p * BQ;
    const int64_t c_first = (int64_t)blockIdx.y * a.chunk, c_end = min(a.nc, c_first + a.chunk);
    const bool p_whole = PC || p0 + BP <= a.np, q_whole = QC || q0 + BQ <= a.nq;

    Stage<T, PC, BP, THREADS> sp;
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
    store_tile<T, FP, FQ, BP / WP, BQ / WQ>(a, e, acc, tiles, wave, lane, p0 + wp, q0 + wq);
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

// Offsets from the tile's first element, in bytes, of what a lane requests with the i-th load of an operand's step.
template <class T, bool ALONG_C, int ROWS> __device__ __forceinline__ uint32_t direct_offset(int piece, int lane, int64_t ld, int64_t rows_left)
{
    // a piece is 1024 bytes of the tile in LDS
    if constexpr (ALONG_C) {
        const int r = piece * 16 + (lane >> 2);
        return (uint32_t)(min((int64_t)r, rows_left - 1) * ld * (int64_t)sizeof(T)) + (direct_chunk(r, lane & 3) << 4);
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
// compute units.  bfloat16, bare products one after the other: 8,192 x 4,096 x 2,048 forward 114 us, dx 103, dw 134 with its join (the library 96, 104
// and 131); 10,000 x 4,096 x 1,024 forward 95 us, dx 76, dw 84 with its join (880 - 1,100 TFLOP/s; the library 87 - 95, 82 and 114).  In such
// a product with GELU and z the matrix cores are busy for a third of the cycles, in its dx and dw for half.  Rows 8,192 apart, along c on
// both sides, are slow: 8,192^3 forward 1,225 us, dx 809 (the library 673 and 787).  A smaller tile reads more of its operands per product from L2: 128 x 128 takes 15 - 30 % longer where the tiles are many.
template <class T, bool PC, bool QC, int BP, int BQ, int WP, int WQ, int STEPS>
__global__ __launch_bounds__(WP *WQ * 64, 2) void direct_kernel(Product<T> a, Epilogue<T> e)
{
    constexpr int BC = 32, WAVES = WP * WQ, FP = BP / WP / 16, FQ = BQ / WQ / 16;
    constexpr int NP = BP / 16, NQ = BQ / 16;   // loads of a step; where they do not divide among the waves the last one is made twice
    constexpr int LP = (NP + WAVES - 1) / WAVES, LQ = (NQ + WAVES - 1) / WAVES, LOADS = LP + LQ;
    constexpr int kStep = (BP + BQ) * 64;
    extern __shared__ __align__(16) unsigned char tiles[];   // [STEPS][P, Q][rows of 64 bytes, or 32 lines]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t tiles_p = (a.np + BP - 1) / BP;
    const int64_t n = gridDim.x, xcd = blockIdx.x & 7, run = n / 8, left = n % 8;
    const int64_t tile = xcd * run + min(xcd, left) + (blockIdx.x >> 3);
    const int64_t p0 = tile % tiles_p * BP, q0 = tile / tiles_p * BQ;
    const int64_t c_first = (int64_t)blockIdx.y * a.chunk, c_end = min(a.nc, c_first + a.chunk);
    const int steps = (int)max((int64_t)0, (c_end - c_first) / BC);

    const T *P = PC ? a.P + p0 * a.ldp + c_first : a.P + c_first * a.ldp + p0;
    const T *Q = QC ? a.Q + q0 * a.ldq + c_first : a.Q + c_first * a.ldq + q0;
    uint32_t off_p[LP], off_q[LQ];
#pragma unroll
    for (int i = 0; i < LP; ++i) off_p[i] = direct_offset<T, PC, BP>(min(wave * LP + i, NP - 1), lane, a.ldp, a.np - p0);
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
            if (i < LP) request(p, off_p[i], lds0 + at + min(wave * LP + i, NP - 1) * 1024);
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
        auto keep_part = [&](auto along_c, auto rows_of, const T *src, int64_t ld, int64_t r0, int64_t rows, unsigned char *to) {
            constexpr int ROWS = rows_of.value, kLine = ROWS / 8;
            for (int id = threadIdx.x; id < ROWS * 4; id += WAVES * 64) {
                if constexpr (along_c.value) {
                    const int r = id >> 2, ch = id & 3;
                    const int64_t c = c0 + ch * 8;
                    *(Vec<T> *)(to + r * 64 + (direct_chunk(r, ch) << 4)) =
                        load_part(src + (r0 + r) * ld + c, r0 + r < rows ? (int)min((int64_t)8, max((int64_t)0, c_end - c)) : 0, (T)0.f);
                } else {
                    const int64_t c = c0 + id / kLine, r = r0 + id % kLine * 8;
                    *(Vec<T> *)(to + line_place<T, ROWS>(id / kLine, id % kLine * 16)) =
                        load_part(src + c * ld + r, c < c_end ? (int)min((int64_t)8, max((int64_t)0, rows - r)) : 0, (T)0.f);
                }
            }
        };
        keep_part(std::integral_constant<bool, PC>(), std::integral_constant<int, BP>(), a.P, a.ldp, p0, a.np, tiles);
        keep_part(std::integral_constant<bool, QC>(), std::integral_constant<int, BQ>(), a.Q, a.ldq, q0, a.nq, tiles + BP * 64);
        __syncthreads();
        read_step(0, fp[0], fq[0]);
        multiply(fp[0], fq[0]);
    }
    store_tile<T, FP, FQ, FP * 16, FQ * 16>(a, e, acc, tiles, wave, lane, p0 + wp, q0 + wq);
}

// The splits' sums, in order, and the epilogue: 4 x 4,096 x 1,024 in 12 us, 6 TB/s.
template <class T>
__global__ __launch_bounds__(256) void product_join_kernel(int64_t np, int64_t nq, int splits, const float *__restrict__ part, Epilogue<T> e)
{
    const int64_t quads = (np + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quads * nq; i += (int64_t)gridDim.x * 256) {
        const int64_t q = i / quads, p = (i - q * quads) * 4;
        const int n = (int)min((int64_t)4, np - p);
        float a[4] = {}, u[4];
        for (int s = 0; s < splits; ++s) {
            load_row(part + ((int64_t)s * nq + q) * np + p, n, u);
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] += u[j];
        }
        float bias[4];
        load_bias(e, p, n, bias);
        finish(e, q, p, n, a, bias);
    }
}

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
// from 32 x 1,024 x 1,024 to 8,192 x 4,096 x 2,048, each product, every tiling and 1 to 32 splits; what it picks takes 3.4 % longer than the best of
// all on average, more than 10 % for 16 of 117 products, 53 % at worst (64 x 4,096 -> 128: 16.3 us for 10.7).
struct TilingCost {
    int bp, bq, together;
    double step, alone, fixed;
};
static TilingCost cost_of(Tiling t, bool f32, bool both_along)
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
static double few_rows_us(int64_t np, int64_t nq, int64_t row_bytes)
{
    const double groups = (double)ceil_div(np, 16);
    const double latency = 3 + 0.4 * (double)row_bytes / 1024 * (nq <= 16 ? 2 : nq <= 32 ? 3 : 5) * std::ceil(groups / 512);
    return std::max(latency, (double)np * row_bytes / 5.3e6 + groups * nq * row_bytes / 10e6);
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
};

constexpr int64_t kMaxTiles = 1 << 22;   // and more are not launched: a launch holds fewer than 2^32 threads

// The tiling and the number of splits of the contraction that should take least time.  A split costs its partial sums' way
// through memory and one more launch (5.5 us: small products come one after the other as fast as the host can launch them); it pays where
// there are too few tiles for the chip's 256 compute units.  Nothing is faster than memory.
static ProductPlan plan_product(int32_t dtype, int64_t np, int64_t nq, int64_t nc, const Operands &o)
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
static int allow_lds(const void *kernel, size_t bytes, std::atomic<uint64_t> &done)
{
    int dev = 0;
    VF_HIP(hipGetDevice(&dev));
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return VF_OK;
    VF_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    done.fetch_or(bit, std::memory_order_relaxed);
    return VF_OK;
}

template <class T, bool PC, bool QC, int BP, int BQ, int WP, int WQ, int STEPS>
static int launch_direct(const Product<T> &a, const Epilogue<T> &e, dim3 grid, hipStream_t s)
{
    constexpr size_t lds = (size_t)STEPS * (BP + BQ) * 64;
    static std::atomic<uint64_t> done{0};
    if constexpr (lds > 64 * 1024)
        if (int rc = allow_lds((const void *)direct_kernel<T, PC, QC, BP, BQ, WP, WQ, STEPS>, lds, done); rc != VF_OK) return rc;
    direct_kernel<T, PC, QC, BP, BQ, WP, WQ, STEPS><<<grid, dim3(WP * WQ * 64), lds, s>>>(a, e);
    return VF_OK;
}

template <class T, bool PC, bool QC>
static int run_product(int32_t dtype, const T *P, int64_t ldp, int64_t np, const T *Q, int64_t ldq, int64_t nq, int64_t nc,
                       const Epilogue<T> &e, const ProductPlan &plan, float *part, hipStream_t s)
{
    if (np == 0 || nq == 0) return VF_OK;
    const Product<T> a{P, Q, ldp, ldq, np, nq, nc, plan.chunk, plan.splits, part};
    if (plan.tiling == kFewRows) {
        if constexpr (PC && QC) {
            // four fragments of the contraction and more for each wave
            const int waves = (int)std::max<int64_t>(1, std::min<int64_t>(16, nc / (4 * 4 * kVec<T>)));
            const dim3 grid((unsigned)ceil_div(np, 16)), block(waves * 64);
            if (nq <= 16) few_rows_kernel<T, 1><<<grid, block, 0, s>>>(a, e);
            else if (nq <= 32) few_rows_kernel<T, 2><<<grid, block, 0, s>>>(a, e);
            else few_rows_kernel<T, 4><<<grid, block, 0, s>>>(a, e);
        }
        VF_HIP(hipGetLastError());
        return VF_OK;
    }
    const TilingCost c = cost_of(plan.tiling, dtype == VF_F32, PC && QC);
    const int64_t tiles = ceil_div(np, c.bp) * ceil_div(nq, c.bq);
    const dim3 grid((unsigned)tiles, (unsigned)plan.splits);
    int rc = VF_OK;
    if (plan.tiling == kSmall) {
        tile_kernel<T, PC, QC, 64, 64, 2, 2><<<grid, dim3(256), (size_t)2 * 128 * kRowBytes, s>>>(a, e);
    } else if (plan.tiling == kMedium) {
        constexpr size_t lds = (size_t)2 * 256 * kRowBytes;   // 64 KiB, which need not be asked for
        static_assert(lds <= 64 * 1024, "");
        tile_kernel<T, PC, QC, 128, 128, 2, 4><<<grid, dim3(512), lds, s>>>(a, e);
    } else if constexpr (sizeof(T) == 2) {
        if (plan.tiling == kDirect192) rc = launch_direct<T, PC, QC, 256, 192, 4, 2, 4>(a, e, grid, s);
        else if (plan.tiling == kDirect256) rc = launch_direct<T, PC, QC, 256, 256, 2, 4, 4>(a, e, grid, s);
        else if (plan.tiling == kDirect128) rc = launch_direct<T, PC, QC, 128, 128, 2, 2, 3>(a, e, grid, s);
        else if constexpr (PC && QC) rc = launch_direct<T, PC, QC, 128, 256, 2, 2, 3>(a, e, grid, s);
    }
    if (rc != VF_OK) return rc;
    if (plan.splits > 1)
        product_join_kernel<T><<<dim3((unsigned)std::min<int64_t>(ceil_div(ceil_div(np, 4) * nq, 256), 4096)), dim3(256), 0, s>>>(
            np, nq, plan.splits, part, e);
    VF_HIP(hipGetLastError());
    return VF_OK;
}

static size_t rounded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

static bool costly(int32_t act) { return act == VF_ACT_GELU || act == VF_ACT_SILU; }

// Whether rows of an operand that lie `ld` elements apart can go to LDS directly: the kernel's offsets within a tile have 32 bits.
static bool direct_rows(int32_t dtype, const void *p, int64_t ld)
{
    return dtype != VF_F32 && ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < (1 << 21);
}

// Workspace of a product whose operands' alignment is not known yet.
static size_t most_bytes(int32_t dtype, int64_t np, int64_t nq, int64_t nc, bool p_along, bool q_along, bool costly)
{
    return std::max(plan_product(dtype, np, nq, nc, {p_along, q_along, costly, false}).bytes,
                    dtype == VF_F32 ? 0 : plan_product(dtype, np, nq, nc, {p_along, q_along, costly, true}).bytes);
}

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
    if (a.dx) plan_dx = plan_product(a.dtype, a.k, a.m, a.n, {false, true, false, a.k % 8 == 0 && direct_rows(a.dtype, a.w, a.ldw) && dz_rows});
    if (a.dw)
        plan_dw = plan_product(a.dtype, a.k, a.n, a.m,
                               {false, false, false, a.k % 8 == 0 && a.n % 8 == 0 && direct_rows(a.dtype, a.x, a.ldx) && dz_rows});
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
