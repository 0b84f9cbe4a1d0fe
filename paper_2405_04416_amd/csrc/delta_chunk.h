// The gated delta rule in chunks of 32 tokens: what a workgroup's producing wavefront lays out in LDS for the others, of which each has 16 columns of the
// memory in its registers, all along the sequence.  Internal.
//
// With all rows of 16 columns in one wavefront a chunk needs no exchange between wavefronts: results of the matrix unit are the right operands of the next
// product (split_rows).  Left operands depend on q, k, g and beta alone; one more wavefront makes them, a chunk ahead.
#pragma once
#include "delta_common.h"

namespace dg_delta {

constexpr int kChunk = 32;
constexpr int kPitch = kChunk + 8;      // of rows of 32 values: 16 lanes that read 16 bytes each of neighbouring rows meet all banks once
constexpr int kMostWaves = 4;           // with columns, in a workgroup

// Left operands of a chunk; columns in the order of `place`
template <class T, int KS, bool kBackward>
struct Operands {
    static constexpr int n = Pieces<T>::n, DK = 32 * KS;
    uint16_t K[n][kChunk][DK + 8];
    uint16_t KT[n][DK][kPitch];
    uint16_t Q[n][kBackward ? DK : kChunk][kBackward ? kPitch : DK + 8];       // backward: Q^T
    uint16_t inverse[3][kChunk][kPitch], P[3][kChunk][kPitch];                 // T; backward: T^T, P^T
    float beta[kChunk], read[kChunk], query[kChunk], until[kChunk];            // beta, beta e^G, scale e^G, e^(G[last] - G)
    float whole;                                                               // e^G[last]
};

// The producing wavefront's own
template <class T, int KS, bool kBackward>
struct Scratch {
    double G[kChunk];
    float beta[kChunk];
    float A[2][16][20], inverse[2][16][20];         // A^T and T of the diagonal blocks
    uint16_t Q[kBackward ? Pieces<T>::n : 1][kBackward ? kChunk : 1][kBackward ? 32 * KS + 8 : 8];
};

__device__ __forceinline__ bf16x8 left(const uint16_t *row) { return operand(*reinterpret_cast<const u32x4 *>(row)); }

// eight values that lie aligned, halves of them behind D as 0
template <class T>
__device__ __forceinline__ void load8_aligned(const T *row, uint32_t c, uint32_t D, bool in, dg_rows::Pack<T, 8> &out)
{
    constexpr int n = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < 8 / n; ++h) {
        const bool here = in && c + h * n < D;
        const dg_rows::Pack<T, n> p = *reinterpret_cast<const dg_rows::Pack<T, n> *>(row + (here ? c + h * n : 0));
#pragma unroll
        for (int i = 0; i < n; ++i) out.v[h * n + i] = here ? p.v[i] : (T)0.0f;
    }
}

template <class T, int KS, bool kBackward>
struct Producer {
    using Ops = Operands<T, KS, kBackward>;
    using Own = Scratch<T, KS, kBackward>;
    static constexpr int n = Ops::n, kItems = 2 * KS;

    const Delta &d;
    const Span &span;
    const uint32_t head, hk, lane;
    dg_rows::Pack<T, 8> k[kItems], q[kItems];
    float g, beta;

    __device__ __forceinline__ Producer(const Delta &d, const Span &span, uint32_t head, uint32_t lane)
        : d(d), span(span), head(head), hk(head / (d.H / d.Hk)), lane(lane) {}

    // item `it` of a lane: eight columns of a token of the chunk
    __device__ __forceinline__ uint32_t token(int it) const { return it * (16 / KS) + lane / (4 * KS); }
    __device__ __forceinline__ uint32_t column() const { return lane % (4 * KS) * 8; }

    // rows of chunk c, on their way into registers if vectors divide them; otherwise produce() loads them, value by value
    __device__ __forceinline__ void fetch(uint32_t c)
    {
        if (d.vec_q && d.vec_k) {
            const T *at_k = (const T *)d.k + hk * d.Dk, *at_q = (const T *)d.q + hk * d.Dk;
#pragma unroll
            for (int it = 0; it < kItems; ++it) {
                const uint32_t t = c * kChunk + token(it);
                const bool in = t < span.len;
                const uint64_t row = span.row(in ? t : c * kChunk);
                load8_aligned<T>(at_k + row * d.ldk, column(), d.Dk, in, k[it]);
                load8_aligned<T>(at_q + row * d.ldq, column(), d.Dk, in, q[it]);
            }
        }
        const uint32_t t = c * kChunk + lane % 32;
        const uint64_t row = t < span.len ? span.row(t) : 0;
        g = t < span.len ? fmaxf(d.g[row * d.ldg + head], kShut) : 0.0f;
        beta = t < span.len ? d.beta[row * d.ldb + head] : 0.0f;
    }

    // eight values of a token: as they lie in its row, and each into its column's row
    template <int pitch>
    __device__ __forceinline__ static void put(const dg_rows::Pack<T, 8> &x, uint32_t t, uint32_t col, uint16_t (*rows)[kChunk][pitch], uint16_t (*columns)[32 * KS][kPitch])
    {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)x.v[i];
        uint32_t w[n][4];
        split<n, 8>(v, w);
#pragma unroll
        for (int p = 0; p < n; ++p) {
            if (rows) {
                *reinterpret_cast<u32x2 *>(&rows[p][t][place(col)]) = (u32x2){w[p][0], w[p][1]};
                *reinterpret_cast<u32x2 *>(&rows[p][t][place(col + 4)]) = (u32x2){w[p][2], w[p][3]};
            }
            if (columns)
#pragma unroll
                for (int i = 0; i < 8; ++i) columns[p][col + i][place(t)] = (uint16_t)(w[p][i / 2] >> (i % 2 * 16));
        }
    }

    // four values side by side, in pieces
    __device__ __forceinline__ static void put4(const float (&v)[4], uint16_t (*rows)[kChunk][kPitch], uint32_t row, uint32_t col)
    {
        uint32_t w[3][2];
        split<3, 4>(v, w);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x2 *>(&rows[p][row][place(col)]) = (u32x2){w[p][0], w[p][1]};
    }

    // what never changes: the blocks of T and P behind the diagonal
    __device__ __forceinline__ static void clear(Ops &o, uint32_t lane)
    {
        const float none[4] = {};
        const uint32_t r = lane % 16, c = lane / 16 * 4;
        put4(none, o.inverse, kBackward ? 16 + r : r, kBackward ? c : 16 + c);
        put4(none, o.P, kBackward ? 16 + r : r, kBackward ? c : 16 + c);
    }

    // the product of two 16-row blocks of K or Q
    template <int pa, int pb>
    __device__ __forceinline__ f32x4 rows_product(const uint16_t (*a)[kChunk][pa], uint32_t ra, const uint16_t (*b)[kChunk][pb], uint32_t rb) const
    {
        f32x4 acc = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            bf16x8 x[n], y[n];
#pragma unroll
            for (int p = 0; p < n; ++p) {
                x[p] = left(&a[p][ra + lane % 16][s * 32 + lane / 16 * 8]);
                y[p] = left(&b[p][rb + lane % 16][s * 32 + lane / 16 * 8]);
            }
            acc = multiply<n, n>(x, y, acc);
        }
        return acc;
    }

    __device__ __forceinline__ void produce(Ops &o, Own &own, uint32_t c, uint32_t next, uint32_t chunks)
    {
        constexpr int kRowPitch = 32 * KS + 8;
        auto q_rows = [&] {
            if constexpr (kBackward) return own.Q;
            else return o.Q;
        }();
        auto put_both = [&](const dg_rows::Pack<T, 8> &k8, const dg_rows::Pack<T, 8> &q8, uint32_t t) {
            put<kRowPitch>(k8, t, column(), o.K, o.KT);
            if constexpr (kBackward) put<kRowPitch>(q8, t, column(), own.Q, o.Q);
            else put<kRowPitch>(q8, t, column(), o.Q, nullptr);
        };
        if (d.vec_q && d.vec_k) {
#pragma unroll
            for (int it = 0; it < kItems; ++it) put_both(k[it], q[it], token(it));
        } else
#pragma unroll 1
            for (int it = 0; it < kItems; ++it) {
                const uint32_t t = c * kChunk + token(it);
                dg_rows::Pack<T, 8> k8, q8;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool in = t < span.len && column() + i < d.Dk;
                    const uint64_t row = span.row(in ? t : c * kChunk);
                    const uint32_t at = hk * d.Dk + (in ? column() + i : 0);
                    k8.v[i] = in ? ((const T *)d.k)[row * d.ldk + at] : (T)0.0f;
                    q8.v[i] = in ? ((const T *)d.q)[row * d.ldq + at] : (T)0.0f;
                }
                put_both(k8, q8, token(it));
            }
        double G = (double)g;
#pragma unroll
        for (int s = 1; s < kChunk; s *= 2) {
            const double before = __shfl_up(G, s, kChunk);
            if (lane % kChunk >= (uint32_t)s) G += before;
        }
        const double last = __shfl(G, kChunk - 1, kChunk);
        if (lane < kChunk) {
            const float since = expf((float)G);
            own.G[lane] = G;
            own.beta[lane] = o.beta[lane] = beta;
            o.read[lane] = beta * since;
            o.query[lane] = d.scale * since;
            o.until[lane] = expf((float)(last - G));
            if (lane == 0) o.whole = expf((float)last);
        }
        if (next < chunks) fetch(next);
        wave_fence();
        const uint32_t c16 = lane % 16, r4 = lane / 16 * 4;
        // P
#pragma unroll
        for (int b = 0; b < 3; ++b) {           // blocks (row of tokens i, row of tokens j): (0, 0), (1, 0), (1, 1)
            const uint32_t bi = b ? 16 : 0, bj = b == 2 ? 16 : 0;
            f32x4 acc;
            if constexpr (kBackward) acc = rows_product<kRowPitch, kRowPitch>(q_rows, bi, o.K, bj);      // rows i, columns j
            else acc = rows_product<kRowPitch, kRowPitch>(o.K, bj, q_rows, bi);                          // rows j, columns i
            float v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t i = bi + (kBackward ? r4 + x : c16), j = bj + (kBackward ? c16 : r4 + x);
                v[x] = i >= j ? d.scale * acc[x] * expf((float)(own.G[i] - own.G[j])) : 0.0f;
            }
            if (kBackward) put4(v, o.P, bj + c16, bi + r4);
            else put4(v, o.P, bi + c16, bj + r4);
        }
        // A: the diagonal blocks to LDS, the other stays as an operand
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const f32x4 acc = rows_product<kRowPitch, kRowPitch>(o.K, b * 16, o.K, b * 16);
            f32x4 v;
#pragma unroll
            for (int x = 0; x < 4; ++x) {       // A[r4 + x, c16]
                const uint32_t i = b * 16 + r4 + x, j = b * 16 + c16;
                v[x] = i > j ? own.beta[i] * acc[x] * expf((float)(own.G[i] - own.G[j])) : 0.0f;
            }
            *reinterpret_cast<f32x4 *>(&own.A[b][c16][r4]) = v;
        }
        f32x4 a21;
        {
            // forward: rows i, columns j; backward: rows j, columns i
            const f32x4 acc = kBackward ? rows_product<kRowPitch, kRowPitch>(o.K, 0, o.K, 16) : rows_product<kRowPitch, kRowPitch>(o.K, 16, o.K, 0);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t i = 16 + (kBackward ? c16 : r4 + x), j = kBackward ? r4 + x : c16;
                a21[x] = own.beta[i] * acc[x] * expf((float)(own.G[i] - own.G[j]));
            }
        }
        wave_fence();
        // T (1 + A) = 1 by rows: lane (block, row r), t[j] = [j = r] - sum over m > j of t[m] A[m, j]
        const uint32_t block = lane / 16 % 2;
        float t[16];
#pragma unroll
        for (int j = 15; j >= 0; --j) {
            float sum = 0.0f;
#pragma unroll
            for (int m4 = j / 4 * 4; m4 < 16; m4 += 4) {
                const f32x4 a = *reinterpret_cast<const f32x4 *>(&own.A[block][j][m4]);
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (m4 + x > j) sum = fmaf(t[m4 + x], a[x], sum);
            }
            t[j] = (j == (int)c16 ? 1.0f : 0.0f) - sum;
        }
        if (lane < 32)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                *reinterpret_cast<f32x4 *>(&own.inverse[block][c16][j]) = (f32x4){t[j], t[j + 1], t[j + 2], t[j + 3]};
                if (!kBackward) {
                    const float v[4] = {t[j], t[j + 1], t[j + 2], t[j + 3]};
                    put4(v, o.inverse, block * 16 + c16, block * 16 + j);
                }
            }
        wave_fence();
        if (kBackward && lane < 32)             // rows of T^T
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float v[4] = {own.inverse[block][j][c16], own.inverse[block][j + 1][c16], own.inverse[block][j + 2][c16], own.inverse[block][j + 3][c16]};
                put4(v, o.inverse, block * 16 + c16, block * 16 + j);
            }
        // the block below the diagonal, -T22 A21 T11, in fp32: forward as its transpose (A21^T T22^T, then T11^T times that), so that a lane has four
        // values of a row of T in either case
        const f32x4 t22 = *reinterpret_cast<const f32x4 *>(&own.inverse[1][c16][r4]);
        f32x4 w = {}, x = {};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const float t11 = own.inverse[0][r4 + s][c16];
            w = __builtin_amdgcn_mfma_f32_16x16x4f32(a21[s], kBackward ? t11 : t22[s], w, 0, 0, 0);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const float t11 = own.inverse[0][r4 + s][c16];
            x = __builtin_amdgcn_mfma_f32_16x16x4f32(kBackward ? t22[s] : t11, w[s], x, 0, 0, 0);
        }
        const float v[4] = {-x[0], -x[1], -x[2], -x[3]};
        // forward: lane i, rows j; backward: lane j, rows i
        if (kBackward) put4(v, o.inverse, c16, 16 + r4);
        else put4(v, o.inverse, 16 + c16, r4);
    }
};

// Buffers: two if they fit, so that operands are made while others are used
template <class T, int KS, bool kBackward>
struct Room {
    static constexpr int kBuffers = 2 * sizeof(Operands<T, KS, kBackward>) + sizeof(Scratch<T, KS, kBackward>) <= 160 * 1024 ? 2 : 1;
    Operands<T, KS, kBackward> ops[kBuffers];
    Scratch<T, KS, kBackward> own;
};

// The roles of a workgroup along a sequence's chunks.  use(operands, i): the i-th chunk that is taken.
template <class T, int KS, bool kBackward, class Use>
__device__ __forceinline__ void along(const Delta &d, const Span &span, uint32_t head, bool producer, Room<T, KS, kBackward> &room, uint32_t chunks, Use use)
{
    constexpr int kBuffers = Room<T, KS, kBackward>::kBuffers;
    if (chunks == 0) return;
    if (producer) {
        Producer<T, KS, kBackward> p(d, span, head, threadIdx.x % 64);
        auto chunk = [&](uint32_t i) { return kBackward ? chunks - 1 - i : i; };        // past the end: one that there is not
        p.fetch(chunk(0));
        auto produce = [&](uint32_t i) {
            // the next chunk's rows are fetched on the way
            p.produce(room.ops[i % kBuffers], room.own, chunk(i), chunk(i + 1), chunks);
        };
        if (kBuffers == 2) produce(0);
        __syncthreads();
        for (uint32_t i = 0; i < chunks; ++i) {
            if (kBuffers == 2) {
                if (i + 1 < chunks) produce(i + 1);
                __syncthreads();
            } else {
                produce(i);
                __syncthreads();
                __syncthreads();
            }
        }
    } else {
        __syncthreads();
        for (uint32_t i = 0; i < chunks; ++i) {
            if (kBuffers == 1) __syncthreads();
            use(room.ops[i % kBuffers], i);
            __syncthreads();
        }
    }
}

// columns that a workgroup's wavefronts take, and how many workgroups a head has
struct Columns { uint32_t waves, groups; };

inline Columns columns_of(const Delta &d)
{
    const uint32_t all = (d.Dv + 15) / 16;
    const uint64_t units = (uint64_t)d.n_seq * d.H;
    uint32_t waves = all < (uint32_t)kMostWaves ? all : kMostWaves;
    while (waves > 1 && units * ((all + waves - 1) / waves) < 256) waves = (waves + 1) / 2;        // few heads: as many workgroups as there are compute units
    return {waves, (all + waves - 1) / waves};
}

constexpr uint64_t kMostGroups = 1 << 22;      // of a launch: its lanes have to stay below 2^32

}  // namespace dg_delta
