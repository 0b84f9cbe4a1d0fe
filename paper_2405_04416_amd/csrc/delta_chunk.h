// The gated delta rule in chunks of 32 tokens, along the sequences.  Internal.
//
// A wavefront has all rows of 16 columns of the memory in its registers, so that a chunk needs no exchange between wavefronts: results of the matrix unit
// are the right operands of the next product (split_rows).  Left operands are the same for all columns and lie in LDS.  Those that depend on q, k, g and beta
// alone (T and P) are made by a launch of its own (delta_weights.hip), for all chunks at once, in the workspace, as they are to lie in LDS, and come by loads that write there;
// K and Q come through registers, which cut them into pieces and turn them.
#pragma once
#include "delta_common.h"

namespace dg_delta {

constexpr int kChunk = 32;
constexpr int kPitch = kChunk + 8;      // of rows of 32 values: 16 lanes that read 16 bytes each of neighbouring rows meet all banks once
constexpr int kPage = 1024;             // what a wavefront fetches at once

// The matrix unit's result holds rows 4 q to 4 q + 3 of 16 with lane (column, q); two such results are the right operand of a sum over 32 rows, where lane
// (column, q) has places 8 q to 8 q + 7.  So that sums go over tokens, or columns of keys, in their own order, row r of result h (of two) is number 8 (r / 4) + 4 h + r % 4.
// Rows of left operands lie by result: number i at `line(i)`.
__host__ __device__ constexpr uint32_t line(uint32_t i) { return (i & ~31u) | (i >> 2 & 1) << 4 | (i >> 3 & 3) << 2 | (i & 3); }

template <class T, int KS, bool kBackward>
struct alignas(16) Keys {
    static constexpr int n = Pieces<T>::n, DK = 32 * KS;
    uint16_t K[n][kChunk][DK + 8];
    uint16_t KT[n][DK][kPitch];
    uint16_t Q[n][kBackward ? DK : kChunk][kBackward ? kPitch : DK + 8];       // backward: Q^T
};

struct alignas(16) Weights {
    uint16_t inverse[3][kChunk][kPitch], P[3][kChunk][kPitch];                 // T and P; backward: T^T and P^T
    float beta[kChunk], read[kChunk], query[kChunk], until[kChunk];            // beta, e^G (backward: beta e^G), scale e^G, e^(G[last] - G)
    float whole;                                                               // e^G[last]
    float rest[127];                                                           // of a page
};
static_assert(sizeof(Weights) % kPage == 0, "fetched by pages");

// In the workspace: a chunk's slot has those of its heads.  A sequence's first slot is floor(begin / 32) + its number, which leaves room for all.
inline uint64_t chunk_slots(uint64_t N, uint32_t n_seq) { return N / kChunk + n_seq; }

__device__ __forceinline__ uint64_t first_chunk(const Span &s, uint32_t seq) { return s.begin / kChunk + seq; }

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

// eight values of a row of D from column c on, 0 from D on and without a row
template <class T, bool kVec>
__device__ __forceinline__ void eight(const T *row, uint32_t c, uint32_t D, bool in, float (&out)[8])
{
    if constexpr (kVec) {
        dg_rows::Pack<T, 8> p;
        load8_aligned<T>(row, c, D, in, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = (float)p.v[i];
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool here = in && c + i < D;
            const T v = row[here ? c + i : 0];
            out[i] = here ? (float)v : 0.0f;
        }
}

// ------------------------------------------------------------------------------ along a sequence
constexpr int kMostWaves = 4;           // in a workgroup

template <class T, int KS, bool kBackward>
struct Operands {
    Weights weight;
    Keys<T, KS, kBackward> key;
};

// Buffers: two if they fit, so that a chunk's operands come while the one before is worked on
template <class T, int KS, bool kBackward>
struct Room {
    static constexpr int kBuffers = 2 * sizeof(Operands<T, KS, kBackward>) <= 160 * 1024 ? 2 : 1;
    Operands<T, KS, kBackward> ops[kBuffers];
};

// Where some wavefronts have columns and the others bring what these need and take away what they leave: up to 32 columns of a chunk's tokens
constexpr int kTileColumns = 32;
template <class T, bool kBackward>
struct alignas(16) Tiles {
    T in[kChunk][kTileColumns + 8];                             // v, or gradients of o
    T out[kBackward ? 1 : kChunk][kTileColumns + 8];            // o
    float wide[kChunk][kTileColumns + 4];                       // what tokens miss, or gradients of what they write
};

// eight values of a token: as they lie in its row, and each into its column's row
template <int n, int KS>
__device__ __forceinline__ void put(const float (&v)[8], uint32_t t, uint32_t col, uint16_t (*rows)[kChunk][32 * KS + 8], uint16_t (*columns)[32 * KS][kPitch])
{
    uint32_t w[n][4];
    split<n, 8>(v, w);
#pragma unroll
    for (int p = 0; p < n; ++p) {
        if (rows) *reinterpret_cast<u32x4 *>(&rows[p][line(t)][col]) = (u32x4){w[p][0], w[p][1], w[p][2], w[p][3]};
        if (columns)
#pragma unroll
            for (int i = 0; i < 8; ++i) columns[p][line(col + i)][t] = (uint16_t)(w[p][i / 2] >> (i % 2 * 16));
    }
}

// K and Q of a chunk on their way to LDS, kEach vectors of each for a lane: a workgroup has wavefronts enough for that
template <class T, int KS, bool kBackward, int kEach, bool kVec>
struct Rows {
    static constexpr int n = Pieces<T>::n;
    const T *q, *k;
    uint64_t ldq, ldk;
    uint32_t Dk, wave, waves, lane;
    Span span;
    dg_rows::Pack<T, 8> qs[kEach], ks[kEach];

    __device__ __forceinline__ uint32_t token(int i) const { return (i * waves + wave) * (16 / KS) + lane / (4 * KS); }
    __device__ __forceinline__ uint32_t column() const { return lane % (4 * KS) * 8; }

    // a vector where there is one, otherwise another, which store() clears
    __device__ __forceinline__ void fetch(uint32_t c)
    {
        if (!kVec) return;
        constexpr int m = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t t = c * kChunk + token(i);
            const uint64_t row = span.row(token(i) < kChunk && t < span.len ? t : c * kChunk);
#pragma unroll
            for (int h = 0; h < 8 / m; ++h) {
                const uint32_t col = column() + h * m < Dk ? column() + h * m : 0;
                const dg_rows::Pack<T, m> x = *reinterpret_cast<const dg_rows::Pack<T, m> *>(k + row * ldk + col), y = *reinterpret_cast<const dg_rows::Pack<T, m> *>(q + row * ldq + col);
#pragma unroll
                for (int j = 0; j < m; ++j) {
                    ks[i].v[h * m + j] = x.v[j];
                    qs[i].v[h * m + j] = y.v[j];
                }
            }
        }
    }

    __device__ __forceinline__ void store(uint32_t c, Keys<T, KS, kBackward> &to)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t t = token(i);
            if (t >= kChunk) continue;
            float x[8], y[8];
            const bool in = c * kChunk + t < span.len;
            if constexpr (kVec) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool here = in && column() + j < Dk;
                    x[j] = here ? (float)ks[i].v[j] : 0.0f;
                    y[j] = here ? (float)qs[i].v[j] : 0.0f;
                }
            } else {
                const uint64_t row = span.row(in ? c * kChunk + t : c * kChunk);
                eight<T, false>(k + row * ldk, column(), Dk, in, x);
                eight<T, false>(q + row * ldq, column(), Dk, in, y);
            }
            put<n, KS>(x, t, column(), to.K, to.KT);
            if constexpr (kBackward) put<n, KS>(y, t, column(), nullptr, to.Q);
            else put<n, KS>(y, t, column(), to.Q, nullptr);
        }
    }
};

// use(operands, chunk) for a sequence's chunks in turn, backward from the last one on
template <class T, int KS, bool kBackward, bool kVec, class Use>
__device__ __forceinline__ void along(const Delta &d, const Span &span, uint32_t seq, uint32_t head, Room<T, KS, kBackward> &room, uint32_t wave, uint32_t waves, Use use)
{
    constexpr int kBuffers = Room<T, KS, kBackward>::kBuffers;
    const uint32_t chunks = (span.len + kChunk - 1) / kChunk, hk = head / (d.H / d.Hk);
    if (chunks == 0) return;
    const uint64_t slot0 = first_chunk(span, seq);
    auto chunk = [&](uint32_t i) { return kBackward ? chunks - 1 - i : i; };
    Rows<T, KS, kBackward, 2, kVec> rows = {(const T *)d.q + hk * d.Dk, (const T *)d.k + hk * d.Dk, d.ldq, d.ldk, d.Dk, wave, waves, threadIdx.x % 64, span, {}, {}};
    auto weights = [&](uint32_t i) {
        const uint8_t *from = (const uint8_t *)(d.weights + (slot0 + chunk(i)) * d.H + head) + threadIdx.x % 64 * 16;
        uint8_t *to = (uint8_t *)&room.ops[i % kBuffers].weight;
        for (uint32_t at = wave * kPage; at < sizeof(Weights); at += waves * kPage)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(from + at), (__attribute__((address_space(3))) uint32_t *)(to + at), 16, 0, 0);
    };
    rows.fetch(chunk(0));
    weights(0);
    rows.store(chunk(0), room.ops[0].key);
    for (uint32_t i = 0; i < chunks; ++i) {
        __builtin_amdgcn_s_waitcnt(0x0f70);         // all loads, those that write to LDS among them
        __syncthreads();
        const bool more = i + 1 < chunks;
        if (more) {
            rows.fetch(chunk(i + 1));
            if (kBuffers == 2) weights(i + 1);
        }
        use(room.ops[i % kBuffers], chunk(i));
        if (kBuffers == 1) {
            __syncthreads();
            if (more) weights(i + 1);
        }
        if (more) rows.store(chunk(i + 1), room.ops[(i + 1) % kBuffers].key);
    }
}

// The same with wavefronts `with` on bringing and taking away, of rows in whole 16 bytes.  use(operands, chunk, tile) for those that have columns; in, out, wide: columns of the workgroup in
// rows of tokens.  What is brought is fetched two chunks ahead.
template <class T, int KS, bool kBackward>
struct Helped {
    static constexpr int kWeights = 8;          // of 16 bytes to a lane: all of them with two wavefronts
    static_assert(sizeof(Weights) <= kWeights * 128 * 16, "two wavefronts bring the weights");
    Operands<T, KS, kBackward> ops[2];
    Tiles<T, kBackward> tiles[2];
};

template <class T, int KS, bool kBackward>
struct Helper {
    static constexpr int kWeights = Helped<T, KS, kBackward>::kWeights;
    const Delta &d;
    const Span &span;
    uint64_t slot0;
    uint32_t head, lanes, self, columns, column0;       // lanes that help, this one among them
    Rows<T, KS, kBackward, 4, true> rows;
    u32x4 weights[kWeights];
    dg_rows::Pack<T, 8> in;

    __device__ __forceinline__ uint32_t token() const { return self * 8 / columns; }
    __device__ __forceinline__ uint32_t column() const { return self * 8 % columns; }
    // row of a token of chunk c, another where it is none
    __device__ __forceinline__ uint64_t row_of(uint32_t c, uint32_t t) const { return span.row(c * kChunk + t < span.len ? c * kChunk + t : c * kChunk); }

    __device__ __forceinline__ void fetch(uint32_t c)
    {
        rows.fetch(c);
        const u32x4 *from = (const u32x4 *)(d.weights + (slot0 + c) * d.H + head);
#pragma unroll
        for (int i = 0; i < kWeights; ++i) {
            const uint32_t at = i * lanes + self;
            weights[i] = from[at < sizeof(Weights) / 16 ? at : 0];
        }
        if (self * 8 >= kChunk * columns) return;
        const T *p = kBackward ? (const T *)d.dout + row_of(c, token()) * d.lddo : (const T *)d.v + row_of(c, token()) * d.ldv;
        const uint32_t first = column0 + column();
        p += head * d.Dv;
        constexpr int m = 16 / sizeof(T);
#pragma unroll
        for (int h = 0; h < 8 / m; ++h) {
            const dg_rows::Pack<T, m> x = *reinterpret_cast<const dg_rows::Pack<T, m> *>(p + (first + h * m < d.Dv ? first + h * m : 0));
#pragma unroll
            for (int j = 0; j < m; ++j) in.v[h * m + j] = x.v[j];
        }
    }

    __device__ __forceinline__ void put(uint32_t c, Operands<T, KS, kBackward> &ops, Tiles<T, kBackward> &tile)
    {
        u32x4 *to = (u32x4 *)&ops.weight;
#pragma unroll
        for (int i = 0; i < kWeights; ++i) {
            const uint32_t at = i * lanes + self;
            if (at < sizeof(Weights) / 16) to[at] = weights[i];
        }
        rows.store(c, ops.key);
        if (self * 8 >= kChunk * columns) return;
        const bool there = c * kChunk + token() < span.len;
        dg_rows::Pack<T, 8> x;
#pragma unroll
        for (int j = 0; j < 8; ++j) x.v[j] = there && column0 + column() + j < d.Dv ? in.v[j] : (T)0.0f;
        constexpr int m = 16 / sizeof(T);
#pragma unroll
        for (int h = 0; h < 8 / m; ++h) {
            dg_rows::Pack<T, m> part;
#pragma unroll
            for (int j = 0; j < m; ++j) part.v[j] = x.v[h * m + j];
            *reinterpret_cast<dg_rows::Pack<T, m> *>(&tile.in[token()][column() + h * m]) = part;
        }
    }

    template <class E, int pitch>
    __device__ __forceinline__ void take(const E (&tile)[kChunk][pitch], E *p) const
    {
        constexpr int m = 16 / sizeof(E);
        const uint32_t first = column0 + column();
#pragma unroll
        for (int h = 0; h < 8 / m; ++h)
            if (first + h * m < d.Dv) *reinterpret_cast<dg_rows::Pack<E, m> *>(p + first + h * m) = *reinterpret_cast<const dg_rows::Pack<E, m> *>(&tile[token()][column() + h * m]);
    }

    __device__ __forceinline__ void take_away(uint32_t c, const Tiles<T, kBackward> &tile) const
    {
        if (self * 8 >= kChunk * columns || c * kChunk + token() >= span.len) return;
        const uint64_t row = row_of(c, token());
        if constexpr (!kBackward) take(tile.out, (T *)d.o + row * d.ldo + head * d.Dv);
        float *wide = kBackward ? d.dr : d.y;
        if (wide) take(tile.wide, wide + (row * d.H + head) * d.Dv);
    }
};

template <class T, int KS, bool kBackward, class Use>
__device__ __forceinline__ void along_helped(const Delta &d, const Span &span, uint32_t seq, uint32_t head, uint32_t column0, Helped<T, KS, kBackward> &room, uint32_t wave, uint32_t with,
                                             uint32_t waves, Use use)
{
    const uint32_t chunks = (span.len + kChunk - 1) / kChunk, hk = head / (d.H / d.Hk);
    if (chunks == 0) return;
    auto chunk = [&](uint32_t i) { return kBackward ? chunks - 1 - i : i; };
    if (wave < with) {
        for (uint32_t i = 0; i < chunks; ++i) {
            __syncthreads();
            use(room.ops[i % 2], chunk(i), room.tiles[i % 2]);
        }
        __syncthreads();
        return;
    }
    const uint32_t helpers = waves - with;
    Helper<T, KS, kBackward> h = {d, span, first_chunk(span, seq), head, helpers * 64, threadIdx.x - with * 64, with * 16, column0,
                                  {(const T *)d.q + hk * d.Dk, (const T *)d.k + hk * d.Dk, d.ldq, d.ldk, d.Dk, wave - with, helpers, threadIdx.x % 64, span, {}, {}}, {}, {}};
    h.fetch(chunk(0));
    h.put(chunk(0), room.ops[0], room.tiles[0]);
    if (chunks > 1) h.fetch(chunk(1));
    for (uint32_t i = 0; i < chunks; ++i) {
        __syncthreads();
        if (i + 1 < chunks) h.put(chunk(i + 1), room.ops[(i + 1) % 2], room.tiles[(i + 1) % 2]);
        if (i + 2 < chunks) h.fetch(chunk(i + 2));
        if (i) h.take_away(chunk(i - 1), room.tiles[(i - 1) % 2]);
    }
    __syncthreads();
    h.take_away(chunk(chunks - 1), room.tiles[(chunks - 1) % 2]);
}

// How many wavefronts of a workgroup have columns, how many there are (those that help among them), and how many workgroups a head has
struct Columns { uint32_t with, waves, groups; bool helped; };

// With fewer heads than the chip has room for, one or two wavefronts of a workgroup have columns and the others help; otherwise as many as possible have
// columns and all help.  room: whether there is any for two buffers and the tiles.
inline Columns columns_of(const Delta &d, bool room)
{
    const uint32_t all = (d.Dv + 15) / 16, least = d.Dk <= 32 ? 1 : d.Dk <= 64 ? 2 : 4;
    const uint64_t units = (uint64_t)d.n_seq * d.H;
    if (room && units * all <= 512) {
        const uint32_t with = units * all <= 256 || all == 1 ? 1 : 2;
        return {with, 4, (all + with - 1) / with, true};
    }
    uint32_t with = all < (uint32_t)kMostWaves ? all : kMostWaves;
    while (with > 1 && units * ((all + with - 1) / with) < 256) with = (with + 1) / 2;        // few heads: as many workgroups as there are compute units
    return {with, with < least ? least : with, (all + with - 1) / with, false};
}

// Memories in registers: result t of 2 KS has rows 32 (t / 2) + 8 q + 4 (t % 2) on with lane (column, q)
template <int KS>
__device__ __forceinline__ void load_memory(const float *from, uint32_t Dk, uint32_t Dv, bool in, uint32_t r8, f32x4 (&S)[2 * KS])
{
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t r = t / 2 * 32 + r8 + t % 2 * 4 + x;
            S[t][x] = from && in && r < Dk ? from[(uint64_t)r * Dv] : 0.0f;
        }
}

template <int KS>
__device__ __forceinline__ void store_memory(float *to, uint32_t Dk, uint32_t Dv, bool in, uint32_t r8, const f32x4 (&S)[2 * KS])
{
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t r = t / 2 * 32 + r8 + t % 2 * 4 + x;
            if (in && r < Dk) to[(uint64_t)r * Dv] = S[t][x];
        }
}

// A lane's eight tokens of a chunk in one column of rows [N, ld]: one address for the workgroup, 32-bit distances from it for lanes and tokens
// (32 rows of at most 2^24 values).
struct Column {
    uint64_t row;                       // lowest of the chunk
    uint32_t count, from, step;         // tokens of the chunk; distance of the lane's first token, and from one to the next
    __device__ __forceinline__ Column(const Span &s, uint32_t t0, uint32_t r8, uint64_t ld)
    {
        count = s.len - t0 < kChunk ? s.len - t0 : kChunk;
        row = s.turn ? s.begin + (s.len - t0 - count) : s.begin + t0;
        from = (s.turn ? count - 1 - r8 : r8) * (uint32_t)ld;
        step = s.turn ? 0u - (uint32_t)ld : (uint32_t)ld;
    }
};

// another token's value where there is none, which `held` clears: not before it is used, so that nothing waits for the load
template <class T>
__device__ __forceinline__ void load_column(const T *p, uint64_t ld, uint32_t lane_column, const Span &span, uint32_t t0, uint32_t r8, T (&out)[8])
{
    if (t0 >= span.len) return;
    const Column c(span, t0, r8, ld);
    const T *base = p + c.row * ld;
#pragma unroll
    for (int x = 0; x < 8; ++x) out[x] = base[(r8 + x < c.count ? c.from + x * c.step : 0u) + lane_column];
}

template <class T>
__device__ __forceinline__ float held(T value, const Span &span, uint32_t t, bool in) { return in && t < span.len ? (float)value : 0.0f; }

template <class T>
__device__ __forceinline__ void store_column(T *p, uint64_t ld, uint32_t lane_column, const Span &span, uint32_t t0, uint32_t r8, bool in, const float (&v)[8])
{
    const Column c(span, t0, r8, ld);
    T *base = p + c.row * ld;
    if (!in) return;
    if (c.count == kChunk)
#pragma unroll
        for (int x = 0; x < 8; ++x) base[c.from + x * c.step + lane_column] = (T)v[x];
    else
#pragma unroll
        for (int x = 0; x < 8; ++x)
            if (r8 + x < c.count) base[c.from + x * c.step + lane_column] = (T)v[x];
}

// Left operands: tile h or t of a matrix in LDS, all pieces.  They are read ahead of the products, so that these do not wait for one after the other.
template <int n, int rows, int pitch>
__device__ __forceinline__ void lefts(const uint16_t (&m)[n][rows][pitch], uint32_t row, uint32_t col, bf16x8 (&out)[n])
{
#pragma unroll
    for (int p = 0; p < n; ++p) out[p] = left(&m[p][row][col]);
}

}  // namespace dg_delta
