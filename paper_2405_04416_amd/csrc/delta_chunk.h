// The gated delta rule in chunks of 32 tokens, along the sequences.  Internal.
//
// A wavefront has all rows of 16 columns of the memory in its registers (or, where heads are few, 32 rows of them), so that a chunk needs no exchange between wavefronts: results of the matrix unit
// are the right operands of the next product (split_rows).  Left operands are the same for all columns and lie in LDS.  Those that depend on q, k, g and beta
// alone (T and P) are made by a launch of its own (delta_weights.hip), for all chunks at once, in the workspace, as they are to lie in LDS, and come by loads that write there;
// K and Q come through registers, which cut them into pieces; reads that transpose turn them.
#pragma once
#include <type_traits>
#include "delta_common.h"

namespace dg_delta {

constexpr int kChunk = 32;
constexpr int kPitch = kChunk + 8;      // of rows of 32 values: 16 lanes that read 16 bytes each of neighbouring rows meet all banks once
constexpr int kPage = 1024;             // what a wavefront fetches at once

// The matrix unit's result holds rows 4 q to 4 q + 3 of 16 with lane (column, q); two such results are the right operand of a sum over 32 rows, where lane
// (column, q) has places 8 q to 8 q + 7.  So that sums go over tokens, or columns of keys, in their own order, row r of result h (of two) is number 8 (r / 4) + 4 h + r % 4.
// Rows of left operands lie by result: number i at `line(i)`.
__host__ __device__ constexpr uint32_t line(uint32_t i) { return (i & ~31u) | (i >> 2 & 1) << 4 | (i >> 3 & 3) << 2 | (i & 3); }

template <class T, int KS, bool kQ = true>
struct alignas(16) Keys {
    static constexpr int n = Pieces<T>::n, DK = 32 * KS;
    uint16_t K[n][kChunk][DK + 8], Q[kQ ? n : 1][kQ ? kChunk : 1][DK + 8];
};

struct Nothing {};
struct Inverse { uint16_t inverse[3][kChunk][kPitch]; };                      // T; backward: T^T
struct Pull { uint16_t P[3][kChunk][kPitch]; };                               // P; backward: P^T
struct Fades {
    float beta[kChunk], read[kChunk], query[kChunk], until[kChunk];            // beta, e^G (backward: beta e^G), scale e^G, e^(G[last] - G)
    float whole;                                                               // e^G[last]
    float rest[127];                                                           // of a page
};
template <bool kP>
struct alignas(16) WeightsOf : Inverse, std::conditional_t<kP, Pull, Nothing>, Fades {};
struct Weights : WeightsOf<true> {};
static_assert(sizeof(Weights) == sizeof(Inverse) + sizeof(Pull) + sizeof(Fades) && sizeof(WeightsOf<false>) == sizeof(Inverse) + sizeof(Fades), "one behind the other");
static_assert(sizeof(Weights) % kPage == 0, "fetched by pages");

// In the workspace: a chunk's slot has those of its heads.  A sequence's first slot is floor(begin / 32) + its number, which leaves room for all.
inline uint64_t chunk_slots(uint64_t N, uint32_t n_seq) { return N / kChunk + n_seq; }

__device__ __forceinline__ uint64_t first_chunk(const Span &s, uint32_t seq) { return s.begin / kChunk + seq; }

__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 s16x4_in_lds;

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
// Groups of 16 columns up to which wavefronts share them.  Training, shared / each its own, in us: heads of 128 x 128 384 groups of 2048 tokens 583 / 1007, 512 683 / 747, 768 of 1024 tokens
// 520 / 664, 1024 695 / 597;  of 127 x 128, value by value, 400 groups 801 / 998, 720 (fp32) 1651 / 1571;  of 64 columns of keys 300 groups 636 / 641, 600 746 / 694;  of 32 300 groups 480 / 508,
// 600 561 / 529.
constexpr uint64_t kFewColumns = 512, kFewLargeColumns = 768;

template <class T, int KS, bool kQ = true>
struct Operands {
    WeightsOf<kQ> weight;
    Keys<T, KS, kQ> key;
};

// Two buffers, so that a chunk's operands come while the one before is worked on
template <class T, int KS>
struct Room {
    Operands<T, KS> ops[2];
};
static_assert(sizeof(Room<float, 4>) <= 160 * 1024, "the largest has room");

// eight values of a token
template <int n, int KS>
__device__ __forceinline__ void put(const float (&v)[8], uint32_t t, uint32_t col, uint16_t (&rows)[n][kChunk][32 * KS + 8])
{
    uint32_t w[n][4];
    split<n, 8>(v, w);
#pragma unroll
    for (int p = 0; p < n; ++p) *reinterpret_cast<u32x4 *>(&rows[p][line(t)][col]) = (u32x4){w[p][0], w[p][1], w[p][2], w[p][3]};
}

// Eight values on their way, as they lie: in whole 16 bytes (kVec) or one by one
template <class T, bool kVec>
struct Eight {
    static constexpr int m = 16 / sizeof(T);
    u32x4 w[kVec ? 8 / m : 1];
    T v[kVec ? 1 : 8];

    // of the row that lies `row` bytes behind, from column c on; another column's from D on, which is cleared where they are used: not before, so that nothing waits for the load
    __device__ __forceinline__ void load(const uint8_t *base, uint32_t row, uint32_t c, uint32_t D)
    {
        if constexpr (kVec) {
#pragma unroll
            for (int h = 0; h < 8 / m; ++h) w[h] = *reinterpret_cast<const u32x4 *>(base + (row + (c + h * m < D ? c + h * m : 0) * (uint32_t)sizeof(T)));
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const T *>(base + (row + (c + i < D ? c + i : 0) * (uint32_t)sizeof(T)));
    }

    __device__ __forceinline__ dg_rows::Pack<T, 8> values(bool in, uint32_t c, uint32_t D) const
    {
        dg_rows::Pack<T, 8> p;
        if constexpr (kVec) {
            u32x4 clear[8 / m];
#pragma unroll
            for (int h = 0; h < 8 / m; ++h)
#pragma unroll
                for (int x = 0; x < 4; ++x) clear[h][x] = in && c + h * m < D ? w[h][x] : 0u;
            p = __builtin_bit_cast(dg_rows::Pack<T, 8>, clear);
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i) p.v[i] = in && c + i < D ? v[i] : (T)0.0f;
        return p;
    }
};

// eight of a token, in pieces
template <class T, int KS>
__device__ __forceinline__ void put_eight(const dg_rows::Pack<T, 8> &p, uint32_t t, uint32_t col, uint16_t (&rows)[Pieces<T>::n][kChunk][32 * KS + 8])
{
    if constexpr (Pieces<T>::n == 1) *reinterpret_cast<u32x4 *>(&rows[0][line(t)][col]) = __builtin_bit_cast(u32x4, p);
    else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)p.v[i];
        put<Pieces<T>::n, KS>(x, t, col, rows);
    }
}

// Where a chunk's tokens lie: lowest row, and how many rows behind it a token is (the lowest's place for tokens that are not there)
struct Place {
    uint64_t row;
    uint32_t count;
    int32_t turn;
    __device__ __forceinline__ Place(const Span &s, uint32_t t0) : count(s.len - t0 < kChunk ? s.len - t0 : kChunk), turn(s.turn)
    {
        row = s.turn ? s.begin + (s.len - t0 - count) : s.begin + t0;
    }
    __device__ __forceinline__ uint32_t behind(uint32_t t) const { return t >= count ? 0u : turn ? count - 1 - t : t; }
};

// K and Q of a chunk on their way to LDS, kEach vectors of each for a lane: a workgroup has wavefronts enough for that
template <class T, int kEach, bool kVec>
struct Fetched {
    Eight<T, kVec> qs[kEach], ks[kEach];
};

template <class T, int KS, int kEach, bool kVec>
struct Rows {
    static constexpr int n = Pieces<T>::n;
    const T *q, *k;
    uint64_t ldq, ldk;
    uint32_t Dk, wave, waves, lane;
    Span span;

    __device__ __forceinline__ uint32_t token(int i) const { return (i * waves + wave) * (16 / KS) + lane / (4 * KS); }
    __device__ __forceinline__ uint32_t column() const { return lane % (4 * KS) * 8; }

    // a vector where there is one, otherwise another, which store() clears; one address for the workgroup, 32-bit distances from it (32 rows of at most 2^24 values)
    __device__ __forceinline__ void fetch(uint32_t c, Fetched<T, kEach, kVec> &to) const
    {
        const Place at(span, c * kChunk);
        const uint8_t *const k0 = (const uint8_t *)(k + at.row * ldk), *const q0 = (const uint8_t *)(q + at.row * ldq);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t row = at.behind(token(i));
            to.ks[i].load(k0, row * (uint32_t)ldk * sizeof(T), column(), Dk);
            to.qs[i].load(q0, row * (uint32_t)ldq * sizeof(T), column(), Dk);
        }
    }

    template <bool kQ>
    __device__ __forceinline__ void store(uint32_t c, const Fetched<T, kEach, kVec> &from, Keys<T, KS, kQ> &to) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t t = token(i);
            if (t >= kChunk) continue;
            const bool in = c * kChunk + t < span.len;
            put_eight<T, KS>(from.ks[i].values(in, column(), Dk), t, column(), to.K);
            if constexpr (kQ) put_eight<T, KS>(from.qs[i].values(in, column(), Dk), t, column(), to.Q);
        }
    }
};

// use(operands, chunk) for a sequence's chunks in turn, backward from the last one on
template <class T, int KS, bool kBackward, bool kVec, class Use>
__device__ __forceinline__ void along(const Delta &d, const Span &span, uint32_t seq, uint32_t head, Room<T, KS> &room, uint32_t wave, uint32_t waves, Use use)
{
    const uint32_t chunks = (span.len + kChunk - 1) / kChunk, hk = head / (d.H / d.Hk);
    if (chunks == 0) return;
    const uint64_t slot0 = first_chunk(span, seq);
    auto chunk = [&](uint32_t i) { return kBackward ? chunks - 1 - i : i; };
    Rows<T, KS, 2, kVec> rows = {(const T *)d.q + hk * d.Dk, (const T *)d.k + hk * d.Dk, d.ldq, d.ldk, d.Dk, wave, waves, threadIdx.x % 64, span};
    Fetched<T, 2, kVec> fetched;
    auto weights = [&](uint32_t i) {
        const uint8_t *from = (const uint8_t *)(d.weights + (slot0 + chunk(i)) * d.H + head) + threadIdx.x % 64 * 16;
        uint8_t *to = (uint8_t *)&room.ops[i % 2].weight;
        for (uint32_t at = wave * kPage; at < sizeof(Weights); at += waves * kPage)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(from + at), (__attribute__((address_space(3))) uint32_t *)(to + at), 16, 0, 0);
    };
    rows.fetch(chunk(0), fetched);
    weights(0);
    rows.store(chunk(0), fetched, room.ops[0].key);
    for (uint32_t i = 0; i < chunks; ++i) {
        __builtin_amdgcn_s_waitcnt(0x0f70);         // all loads, those that write to LDS among them
        __syncthreads();
        const bool more = i + 1 < chunks;
        if (more) {
            rows.fetch(chunk(i + 1), fetched);
            weights(i + 1);
        }
        use(room.ops[i % 2], chunk(i));
        if (more) rows.store(chunk(i + 1), fetched, room.ops[(i + 1) % 2].key);
    }
}

// ------------------------------------------------------------------------------ along a sequence, few heads
// With fewer columns than the chip has room for, what bounds is how long a chunk takes a wavefront: so two of them share 16 columns, with up to 64 rows of the memory each.  K S is then a sum
// over the wavefronts, which goes through LDS (Shares): a chunk has two halves, between barriers, what goes before the sum and what comes after.  All that the next chunk does not wait for
// is done by others: two for what is made of a chunk's tokens (o, the gradients' part that does not depend on S), some that bring what all need.
constexpr int kShared = 16;             // columns
constexpr int kAside = 2;

template <int KS>
constexpr int kSharers = KS == 1 ? 1 : 2;
template <int KS>
constexpr int kHelpers = KS == 4 ? 4 : 2;
template <int KS>
constexpr int kSharedWaves = kSharers<KS> + kAside + kHelpers<KS>;

template <class T>
struct alignas(16) Tile {
    T in[kChunk][kShared + 16 / sizeof(T)];     // v, or gradients of o
    // a lane's eight tokens of a column
    __device__ __forceinline__ void read(uint32_t lane, float (&out)[8]) const
    {
        const uint32_t c16 = lane % 16, r8 = lane / 16 * 8;
        if constexpr (sizeof(T) == 2) {
            wave_fence();               // what others have stored is read, of which the compiler sees nothing
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_in_lds *)&in[r8 + h * 4 + c16 / 4][c16 % 4 * 4]);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const short bits = v[x];
                    out[h * 4 + x] = (float)__builtin_bit_cast(T, bits);
                }
            }
            wave_fence();
        } else
#pragma unroll
            for (int x = 0; x < 8; ++x) out[x] = (float)in[r8 + x][c16];
    }
};

// What wavefronts hand each other; for those aside two buffers, since they are a chunk behind
template <int KS>
struct Forward {
    f32x4 left[2][2][64];               // what tokens miss
    u32x4 memory[KS][3][64];            // S in pieces
};
template <bool kEnds>
struct Backward {
    f32x4 left[kEnds ? 1 : 2][2][64];   // gradients of what tokens write
    f32x4 ahead[2][64];                 // P^T dO
    u32x4 queried[3][64];               // scale e^G dO, in pieces
};

template <int KS, bool kBackward, bool kEnds = false>
struct alignas(16) Shares : std::conditional_t<kBackward, Backward<kEnds>, std::conditional_t<kEnds, Nothing, Forward<KS>>> {
    f32x4 keys[kSharers<KS>][2][64];    // K S

    // all wavefronts' sum
    __device__ __forceinline__ static f32x4 sum(const f32x4 (&of)[kSharers<KS>][2][64], int h, uint32_t lane)
    {
        if constexpr (kSharers<KS> == 2) return of[0][h][lane] + of[1][h][lane];
        else return of[0][h][lane];
    }
};

// kEnds: for the memory at the end alone
template <class T, int KS, bool kBackward, bool kEnds = false>
struct Helped {
    static constexpr bool kQ = kBackward || !kEnds;
    using Ops = Operands<T, KS, kQ>;
    Ops ops[2];
    Tile<T> tiles[2];
    Shares<KS, kBackward, kEnds> shares;
};
static_assert(sizeof(Helped<float, 4, false>) <= 160 * 1024 && sizeof(Helped<float, 4, true>) <= 160 * 1024, "the largest has room");

template <class T, int KS, bool kBackward, bool kQ, bool kVec>
struct Helper {
    static constexpr uint32_t kUnits16 = sizeof(WeightsOf<kQ>) / 16, kBehind = sizeof(Inverse) / 16, kSkipped = (sizeof(Weights) - sizeof(WeightsOf<kQ>)) / 16;      // 16 bytes each; P, where nothing needs it
    static constexpr int kLanes = kHelpers<KS> * 64, kEach = (2 * KS + kHelpers<KS> - 1) / kHelpers<KS>, kWeights = (int)(kUnits16 + kLanes - 1) / kLanes;
    static_assert(kLanes * 8 >= kChunk * kShared, "a lane has eight values of the tile at most");
    const Delta &d;
    const Span &span;
    uint64_t slot0;
    uint32_t head, self, column0;
    Rows<T, KS, kEach, kVec> rows;
    struct Chunk {
        Fetched<T, kEach, kVec> rows;
        Eight<T, kVec> in;
        u32x4 weights[kWeights];
    };

    __device__ __forceinline__ uint32_t token() const { return self * 8 / kShared % kChunk; }
    __device__ __forceinline__ uint32_t column() const { return self * 8 % kShared; }

    __device__ __forceinline__ void fetch(uint32_t c, Chunk &to) const
    {
        rows.fetch(c, to.rows);
        const u32x4 *from = (const u32x4 *)(d.weights + (slot0 + c) * d.H + head);
#pragma unroll
        for (int i = 0; i < kWeights; ++i) {
            const uint32_t at = i * kLanes + self;
            to.weights[i] = from[at < kBehind ? at : at < kUnits16 ? at + kSkipped : 0];
        }
        const Place at(span, c * kChunk);
        const uint64_t ld = kBackward ? d.lddo : d.ldv;
        const uint8_t *p = (const uint8_t *)((const T *)(kBackward ? d.dout : d.v) + at.row * ld + head * d.Dv);
        to.in.load(p, at.behind(token()) * (uint32_t)ld * sizeof(T), column0 + column(), d.Dv);
    }

    __device__ __forceinline__ void put_tile(uint32_t c, const Chunk &from, Tile<T> &tile) const
    {
        if (self * 8 >= kChunk * kShared) return;
        const dg_rows::Pack<T, 8> p = from.in.values(c * kChunk + token() < span.len, column0 + column(), d.Dv);
        struct Halves { u32x4 w[sizeof(T) / 2]; };
        const Halves h = __builtin_bit_cast(Halves, p);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) *reinterpret_cast<u32x4 *>(&tile.in[token()][column() + i * (16 / (int)sizeof(T))]) = h.w[i];
    }

    __device__ __forceinline__ void put_operands(uint32_t c, const Chunk &from, Operands<T, KS, kQ> &ops) const
    {
        u32x4 *to = (u32x4 *)&ops.weight;
#pragma unroll
        for (int i = 0; i < kWeights; ++i)
            if (kUnits16 % kLanes == 0 || i * kLanes + self < kUnits16) to[i * kLanes + self] = from.weights[i];
        rows.store(c, from.rows, ops.key);
    }
};

// before(i), after(i) in the wavefronts that have columns, early(i), late(i) in those aside, i counting chunks (backward from the last one): all but early go with the two buffers i % 2; early(i)
// may read what after(i - 1) left, and both early(i) and late(i) run up to i = number of chunks.  The others have a chunk's time for what they bring for the next one.
template <class T, int KS, bool kBackward, bool kEnds, bool kVec, class Before, class After, class Early, class Late>
__device__ __forceinline__ void along_helped(const Delta &d, const Span &span, uint64_t slot0, uint32_t head, uint32_t column0, Helped<T, KS, kBackward, kEnds> &room, uint32_t wave,
                                             Before before, After after, Early early, Late late)
{
    const uint32_t chunks = (span.len + kChunk - 1) / kChunk, hk = head / (d.H / d.Hk);
    if (chunks == 0) return;
    constexpr uint32_t kSharing = kSharers<KS>, kFirst = kSharing + kAside;
    if (wave < kSharing) {
        __builtin_amdgcn_s_setprio(3);          // the others are to wait for these
        for (uint32_t i = 0; i < chunks; ++i) {
            __syncthreads();
            before(i);
            __syncthreads();
            after(i);
        }
        __syncthreads();
        return;
    }
    if (wave < kFirst) {
        for (uint32_t i = 0; i < chunks; ++i) {
            __syncthreads();
            early(i);
            __syncthreads();
            late(i);
        }
        __syncthreads();
        early(chunks);
        late(chunks);
        return;
    }
    using Help = Helper<T, KS, kBackward, Helped<T, KS, kBackward, kEnds>::kQ, kVec>;
    const Help h = {d, span, slot0, head, threadIdx.x - kFirst * 64, column0,
                    {(const T *)d.q + hk * d.Dk, (const T *)d.k + hk * d.Dk, d.ldq, d.ldk, d.Dk, wave - kFirst, kHelpers<KS>, threadIdx.x % 64, span}};
    // A chunk is fetched two before it is put; `coming` holds the next one.  Without a branch about a load (behind the last chunk it comes again), so that a wait is for the oldest loads only.
    typename Help::Chunk held[2];
    auto chunk = [&](uint32_t i) {
        const uint32_t c = i < chunks ? i : chunks - 1;
        return kBackward ? chunks - 1 - c : c;
    };
    auto turn = [&](uint32_t i, typename Help::Chunk &coming) {
        __syncthreads();
        h.put_tile(chunk(i + 1), coming, room.tiles[(i + 1) % 2]);
        __syncthreads();
        h.put_operands(chunk(i + 1), coming, room.ops[(i + 1) % 2]);
        __builtin_amdgcn_sched_barrier(0);          // loads ahead of the stores would go to other registers, which would be copied, and waited for, at once
        h.fetch(chunk(i + 3), coming);
        __builtin_amdgcn_sched_barrier(0);
    };
    h.fetch(chunk(0), held[0]);
    h.fetch(chunk(1), held[1]);
    h.put_tile(chunk(0), held[0], room.tiles[0]);
    h.put_operands(chunk(0), held[0], room.ops[0]);
    h.fetch(chunk(2), held[0]);
    for (uint32_t i = 0; i + 1 < chunks; i += 2) {
        turn(i, held[1]);
        turn(i + 1, held[0]);
    }
    if (chunks % 2) turn(chunks - 1, held[1]);
    __syncthreads();
}

// Which head (of all sequences), part and group of columns a workgroup has.  Those of a head and part read the same operands: they get numbers that differ by 8, and so the same of the eight
// L2 caches.
struct Unit {
    uint32_t seq, head, part, group;
    __device__ __forceinline__ Unit(const Delta &d, uint32_t parts, uint32_t groups, uint64_t from)
    {
        const uint64_t unit = from + blockIdx.x, all = (uint64_t)d.n_seq * d.H * parts, eights = all / 8 * 8 * groups;
        uint64_t of;
        if (unit < eights) {
            of = unit / (8 * groups) * 8 + unit % 8;
            group = (uint32_t)(unit / 8 % groups);
        } else {
            of = unit / groups;
            group = (uint32_t)(unit % groups);
        }
        part = (uint32_t)(of % parts);
        of /= parts;
        seq = (uint32_t)(of / d.H), head = (uint32_t)(of % d.H);
    }
};

// ------------------------------------------------------------------------------ parts
// A sequence of few heads is cut in parts where that fills the chip.  A part turns the memory before it into the one behind it by S' = M S + E: a first launch makes E (from no memory; the first part
// from s0) and M (from the unit matrix, its columns as further columns whose values are 0) of all parts but the last, delta_join.hip goes from part to part, a second launch does the whole work with
// known beginnings.  Backward the same from the other end.  `part` counts in the order of the run.
struct PartPlace {
    Span span;
    uint64_t slot;
    uint32_t mark;
    template <bool kBackward>
    __device__ __forceinline__ static PartPlace of(const Delta &d, const Unit &unit)
    {
        const Span whole = span_of(d, unit.seq);
        const uint64_t slot = first_chunk(whole, unit.seq);
        const uint32_t mark = first_slot(whole, unit.seq);
        if (d.parts == 1) return {whole, slot, mark};
        const uint32_t part = kBackward ? d.parts - 1 - unit.part : unit.part;
        return {part_of(whole, part, d.stretch), slot + part * (d.stretch / kChunk), mark + part * (d.stretch / kMark)};
    }
};

// a lane's part of the unit matrix: column `one`
template <int KS>
__device__ __forceinline__ void unit_memory(uint32_t one, uint32_t row0, uint32_t r8, f32x4 (&S)[2 * KS])
{
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) S[t][x] = row0 + t / 2 * 32 + r8 + t % 2 * 4 + x == one ? 1.0f : 0.0f;
}

constexpr uint32_t kUnits = 256;        // compute units
constexpr uint32_t kMostParts = 16, kLeastStretch = 512;
// Workgroups that a unit runs at once, by the bytes of LDS each has.  Of 160 KB two of 52 KB do, two of 56 KB one after the other (measured; 264 workgroups of 320 lanes take as long as 256, or twice).
constexpr uint32_t side_by_side(size_t bytes) { return bytes <= 52 * 1024 ? (uint32_t)(104 * 1024 / bytes) : 1; }

// Number of parts for the least time by rounds of workgroups: per_first, per_second of the two launches' run on a compute unit at once (the first, which has less to do, counts 0.8).
inline void cut(Delta &d, uint32_t per_first, uint32_t per_second)
{
    d.parts = 1;
    if (d.first || !d.ends || d.N / d.n_seq > 0xffffffffu) return;
    const uint32_t len = (uint32_t)(d.N / d.n_seq), all = (d.Dv + 15) / 16, keys = (d.Dk + 15) / 16;
    const uint64_t heads = (uint64_t)d.n_seq * d.H;
    auto rounds = [](uint64_t groups, uint32_t per) { return (double)((groups + kUnits - 1) / kUnits <= per ? 1 + 0.25 * ((groups - 1) / kUnits) : (double)((groups + kUnits * per - 1) / (kUnits * per)) * (0.75 + 0.25 * per)); };
    double best = 0.8 * rounds(heads * all, per_second);
    for (uint32_t p = 3; p <= kMostParts && heads * p <= kUnits && len / p >= kLeastStretch; ++p) {
        const uint32_t stretch = (len / p + kMark - 1) / kMark * kMark;
        if ((uint64_t)stretch * (p - 1) >= len || (uint64_t)stretch * p < len) continue;
        const double cost = (0.8 * rounds(heads * ((p - 1) * all + (p - 2) * keys), per_first) + rounds(heads * all * p, per_second)) / p;
        if (cost < best) best = cost, d.parts = p, d.stretch = stretch;
    }
}

// How many wavefronts of a workgroup have columns, how many there are (those that help among them), and how many workgroups a head has
struct Columns { uint32_t with, waves, groups; bool helped; };

// With fewer heads than the chip has room for, wavefronts share columns; otherwise each has 16 of its own, as many as possible to a workgroup, and all bring operands.
inline Columns columns_of(const Delta &d)
{
    const uint32_t all = (d.Dv + 15) / 16, least = d.Dk <= 32 ? 1 : d.Dk <= 64 ? 2 : 4;
    const uint64_t units = (uint64_t)d.n_seq * d.H;
    if (units * all <= (d.Dk > 64 && d.vec_all ? kFewLargeColumns : kFewColumns)) return {1, 0, all, true};
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

// four tokens from `first` of the lane's eight on
template <class T>
__device__ __forceinline__ void store_four(T *p, uint64_t ld, uint32_t lane_column, const Span &span, uint32_t t0, uint32_t r8, uint32_t first, bool in, const f32x4 &v)
{
    const Column c(span, t0, r8 + first, ld);
    T *base = p + c.row * ld;
#pragma unroll
    for (int x = 0; x < 4; ++x)
        if (in && r8 + first + x < c.count) base[c.from + x * c.step + lane_column] = (T)v[x];
}

// Left operands: tile h or t of a matrix in LDS, all pieces.  They are read ahead of the products, so that these do not wait for one after the other.
template <int n, int rows, int pitch>
__device__ __forceinline__ void lefts(const uint16_t (&m)[n][rows][pitch], uint32_t row, uint32_t col, bf16x8 (&out)[n])
{
#pragma unroll
    for (int p = 0; p < n; ++p) out[p] = left(&m[p][row][col]);
}

// Columns of K or Q as left operands of a sum over tokens: tile 2 s + h of the memory's rows.  16 lanes read 16 columns of 4 rows and get a column each: of rows of four tokens,
// 4 lanes each, what lane l reads is columns 8 (l % 4) + 4 h on, so that column r is that of the memory's row with number r of result h.
template <int n, int pitch>
__device__ __forceinline__ void lefts_turned(const uint16_t (&m)[n][kChunk][pitch], uint32_t s, uint32_t h, uint32_t lane, bf16x8 (&out)[n])
{
    wave_fence();                       // what others have stored is read, of which the compiler sees nothing
#pragma unroll
    for (int p = 0; p < n; ++p) {
        const uint16_t *at = &m[p][lane / 4][s * 32 + h * 4 + lane % 4 * 8];            // tokens 8 (lane / 16) on lie in rows 4 (lane / 16) on, and 16 rows on
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_in_lds *)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_in_lds *)(at + 16 * pitch));
        out[p] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    wave_fence();
}

// A lane's column of 16 as an operand: column col + lane % 16, eight rows from row + 8 (lane / 16) on.  16 lanes read 16 columns of four rows, 4 values each, and get a column each.
template <int n, int rows, int pitch>
__device__ __forceinline__ void columns(const uint16_t (&m)[n][rows][pitch], uint32_t row, uint32_t col, uint32_t lane, bf16x8 (&out)[n])
{
    wave_fence();                       // what others have stored is read, of which the compiler sees nothing
#pragma unroll
    for (int p = 0; p < n; ++p) {
        const uint16_t *at = &m[p][row + lane / 16 * 8 + lane % 16 / 4][col + lane % 4 * 4];
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_in_lds *)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_in_lds *)(at + 4 * pitch));
        out[p] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    wave_fence();
}

}  // namespace dg_delta
