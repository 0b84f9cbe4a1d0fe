// The gated delta rule, forward, in chunks of 32 tokens: Y = T (V - e^G K S), U = beta Y, O = scale e^G Q S + P U, S' = e^G[last] S + K^T (e^(G[last] - G) U).
//
// Bound by how long a chunk takes after the one before, not by memory or the matrix instructions: cutting S, what tokens miss and what they write into pieces takes 5.5 operations a value, and a
// wavefront issues one in some 6 cycles.  A wavefront with all 128 rows of its columns: 4400 cycles a chunk; two that share them, with o made by others: 2500 (1.05 us).  65536 tokens x 8 heads of
// 128 x 128, bf16: 2.24 ms whole, in four parts 0.67 (ends) + 0.02 (joined) + 0.60; 2 x 8192 tokens x 16 heads 0.39, vector units 31 % of the time busy, matrix units 13.
#include "delta_chunk.h"

namespace {

using namespace dg_delta;

// A chunk for a wavefront with 16 columns of the memory, S.  value: v of the lane's eight tokens; out, missed: o and what they miss.
template <class T, int KS>
__device__ __forceinline__ void take_chunk(const Operands<T, KS> &o, uint32_t c16, uint32_t r8, const float (&value)[8], f32x4 (&S)[2 * KS], float (&out)[8], float (&missed)[8])
{
    constexpr int n = Pieces<T>::n, kTiles = 2 * KS;
    bf16x8 keys[KS][2][n], queries[KS][2][n], inverse[2][3], pull[2][3];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            lefts(o.key.K, h * 16 + c16, s * 32 + r8, keys[s][h]);
            lefts(o.key.Q, h * 16 + c16, s * 32 + r8, queries[s][h]);
        }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        lefts(o.weight.inverse, h * 16 + c16, r8, inverse[h]);
        lefts(o.weight.P, h * 16 + c16, r8, pull[h]);
    }
    __builtin_amdgcn_sched_barrier(0);
    f32x4 ks[2] = {}, qs[2] = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        bf16x8 sp[3];
        split_rows<3, (n > 1)>(S[2 * s], S[2 * s + 1], sp);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            ks[h] = multiply<n, 3>(keys[s][h], sp, ks[h]);
            qs[h] = multiply<n, 3>(queries[s][h], sp, qs[h]);
        }
    }
    bf16x8 turned[kTiles][n];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) lefts_turned(o.key.K, t / 2, t % 2, c16 + r8 * 2, turned[t]);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 r[2], u[2], beta[2], until[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4 read = *reinterpret_cast<const f32x4 *>(&o.weight.read[r8 + h * 4]);
        beta[h] = *reinterpret_cast<const f32x4 *>(&o.weight.beta[r8 + h * 4]);
        until[h] = *reinterpret_cast<const f32x4 *>(&o.weight.until[r8 + h * 4]);
#pragma unroll
        for (int x = 0; x < 4; ++x) r[h][x] = value[h * 4 + x] - read[x] * ks[h][x];
    }
    bf16x8 right[3];
    split_rows<3>(r[0], r[1], right);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4 y = multiply<3, 3>(inverse[h], right, (f32x4){});
#pragma unroll
        for (int x = 0; x < 4; ++x) missed[h * 4 + x] = y[x];
        u[h] = y * beta[h];
    }
    bf16x8 written[3];
    split_rows<3, (n > 1)>(u[0] * until[0], u[1] * until[1], written);
    const float whole = o.weight.whole;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) S[t] = multiply<n, 3>(turned[t], written, S[t] * whole);
    split_rows<3>(u[0], u[1], right);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4 query = *reinterpret_cast<const f32x4 *>(&o.weight.query[r8 + h * 4]);
        const f32x4 sum = multiply<3, 3>(pull[h], right, query * qs[h]);
#pragma unroll
        for (int x = 0; x < 4; ++x) out[h * 4 + x] = sum[x];
    }
}

// The same shared by wavefronts, rows 32 kOwn wave on each.
template <class T, int KS, bool kEnds>
struct Share {
    static constexpr int n = Pieces<T>::n, kOwn = KS / kSharers<KS>;
    f32x4 S[2 * kOwn];
    bf16x8 inverse[2][3], turned[2 * kOwn][n];
    f32x4 read[2], written[2];          // of what tokens miss, what the memory gets: beta e^(G[last] - G)
    float value[8], whole;

    // up to the sum K S; then all that comes after it is read
    __device__ __forceinline__ void before(const Operands<T, KS, !kEnds> &o, const Tile<T> &tile, Shares<KS, false, kEnds> &to, uint32_t wave, uint32_t lane)
    {
        const uint32_t c16 = lane % 16, r8 = lane / 16 * 8;
        bf16x8 keys[kOwn][2][n], sp[kOwn][3];
#pragma unroll
        for (int s = 0; s < kOwn; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) lefts(o.key.K, h * 16 + c16, (wave * kOwn + s) * 32 + r8, keys[s][h]);
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sum[kOwn][2];
#pragma unroll
        for (int s = 0; s < kOwn; ++s) {
            split_rows<3, (n > 1)>(S[2 * s], S[2 * s + 1], sp[s]);
#pragma unroll
            for (int h = 0; h < 2; ++h) sum[s][h] = multiply<n, 3>(keys[s][h], sp[s], (f32x4){});
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (kOwn == 2) sum[0][h] += sum[1][h];
            to.keys[wave][h][lane] = sum[0][h];
        }
        if constexpr (!kEnds)
#pragma unroll
        for (int s = 0; s < kOwn; ++s)
#pragma unroll
            for (int p = 0; p < 3; ++p) to.memory[wave * kOwn + s][p][lane] = __builtin_bit_cast(u32x4, sp[s][p]);
        __builtin_amdgcn_sched_barrier(0);
        tile.read(lane, value);
#pragma unroll
        for (int h = 0; h < 2; ++h) read[h] = *reinterpret_cast<const f32x4 *>(&o.weight.read[r8 + h * 4]);
#pragma unroll
        for (int h = 0; h < 2; ++h) lefts(o.weight.inverse, h * 16 + c16, r8, inverse[h]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            written[h] = *reinterpret_cast<const f32x4 *>(&o.weight.beta[r8 + h * 4]) * *reinterpret_cast<const f32x4 *>(&o.weight.until[r8 + h * 4]);
        }
#pragma unroll
        for (int t = 0; t < 2 * kOwn; ++t) lefts_turned(o.key.K, wave * kOwn + t / 2, t % 2, lane, turned[t]);
        whole = o.weight.whole;
    }

    __device__ __forceinline__ void after(Shares<KS, false, kEnds> &shares, uint32_t parity, uint32_t wave, uint32_t lane)
    {
        f32x4 r[2], y[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 ks = shares.sum(shares.keys, h, lane);
#pragma unroll
            for (int x = 0; x < 4; ++x) r[h][x] = value[h * 4 + x] - read[h][x] * ks[x];
        }
        bf16x8 right[3];
        split_rows<3>(r[0], r[1], right);
#pragma unroll
        for (int h = 0; h < 2; ++h) y[h] = multiply_soon<3, 3>(inverse[h], right, (f32x4){});
        split_rows<3, (n > 1)>(y[0] * written[0], y[1] * written[1], right);
#pragma unroll
        for (int t = 0; t < 2 * kOwn; ++t) S[t] = multiply<n, 3>(turned[t], right, S[t] * whole);
        // for those aside
        if constexpr (!kEnds)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (wave == h % kSharers<KS>) shares.left[parity][h][lane] = y[h];
    }
};

// o of 16 of a chunk's tokens, and what they miss: Q S while the chunk is under way, the rest when it is done
template <class T, int KS>
struct Outputs {
    static constexpr int n = Pieces<T>::n;
    bf16x8 pull[3];
    f32x4 u[2], y, qs;

    __device__ __forceinline__ void query(const Operands<T, KS> &o, const Shares<KS, false> &shares, uint32_t h, uint32_t lane)
    {
        const uint32_t c16 = lane % 16, r8 = lane / 16 * 8;
        f32x4 sum[2] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            bf16x8 queries[n], sp[3];
            lefts(o.key.Q, h * 16 + c16, s * 32 + r8, queries);
#pragma unroll
            for (int p = 0; p < 3; ++p) sp[p] = operand(shares.memory[s][p][lane]);
            sum[s % 2] = multiply<n, 3>(queries, sp, sum[s % 2]);
        }
        qs = (sum[0] + sum[1]) * *reinterpret_cast<const f32x4 *>(&o.weight.query[r8 + h * 4]);
    }
    __device__ __forceinline__ void read(const Operands<T, KS> &o, const Shares<KS, false> &shares, uint32_t parity, uint32_t h, uint32_t lane)
    {
        const uint32_t r8 = lane / 16 * 8;
        lefts(o.weight.P, h * 16 + lane % 16, r8, pull);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 v = shares.left[parity][i][lane];
            u[i] = v * *reinterpret_cast<const f32x4 *>(&o.weight.beta[r8 + i * 4]);
            if (i == (int)h) y = v;
        }
    }
    __device__ __forceinline__ f32x4 make() const
    {
        bf16x8 right[3];
        split_rows<3>(u[0], u[1], right);
        return multiply_soon<3, 3>(pull, right, qs);
    }
};

template <class T, int KS, bool kEnds, bool kVec>
__global__ void __launch_bounds__(kSharedWaves<KS> * 64)
delta_fwd_shared_kernel(Delta d, uint32_t groups, uint64_t from)
{
    using Mine = Share<T, KS, kEnds>;
    __shared__ Helped<T, KS, false, kEnds> room;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c16 = lane % 16, r8 = lane / 16 * 8;
    const Unit unit(d, kEnds ? d.parts - 1 : d.parts, groups, from);
    const uint32_t head = unit.head, seq = unit.seq, column0 = unit.group * kShared, col = column0 + c16, one = (d.Dv + 15) / 16 * 16;
    if (kEnds && unit.part == 0 && column0 >= one) return;
    const PartPlace place = PartPlace::of<false>(d, unit);
    const Span &span = place.span;
    const uint32_t row0 = wave * (Mine::kOwn * 32), rows = d.Dk > row0 ? d.Dk - row0 : 0, chunks = (span.len + kChunk - 1) / kChunk;
    const bool column = col < d.Dv, in = wave < kSharers<KS> && column, mine = wave < kSharers<KS>;
    const uint64_t first = ((uint64_t)seq * d.H + head) * d.Dk + row0, later = (((uint64_t)seq * d.parts + unit.part) * d.H + head) * d.Dk + row0;
    Mine share;
    if (kEnds && column0 >= one) unit_memory<Mine::kOwn>(col - one, row0, r8, share.S);
    else if (unit.part == 0 && (kEnds || d.parts == 1)) load_memory<Mine::kOwn>(d.s0 ? d.s0 + first * d.Dv + col : nullptr, rows, d.Dv, in, r8, share.S);
    else load_memory<Mine::kOwn>(kEnds ? nullptr : d.starts + later * d.Dv + col, rows, d.Dv, in, r8, share.S);
    Outputs<T, KS> outputs;
    along_helped<T, KS, false, kEnds, kVec>(d, span, place.slot, head, column0, room, wave,
        [&](uint32_t c) {
            share.before(room.ops[c % 2], room.tiles[c % 2], room.shares, wave, lane);
            if (!kEnds && d.marks && c % (kMark / kChunk) == 0)
                store_memory<Mine::kOwn>(d.marks + (((uint64_t)(place.mark + c / (kMark / kChunk)) * d.H + head) * d.Dk + row0) * d.Dv + col, rows, d.Dv, in, r8, share.S);
        },
        [&](uint32_t c) { share.after(room.shares, c % 2, wave, lane); },
        [&](uint32_t c) {
            if constexpr (!kEnds) outputs.read(room.ops[(c + 1) % 2], room.shares, (c + 1) % 2, wave - kSharers<KS>, lane);
        },
        [&](uint32_t c) {
            if constexpr (!kEnds) {
                const uint32_t t0 = (c - 1) * kChunk, h = wave - kSharers<KS>;
                if (c) {
                    store_four<T>((T *)d.o + head * d.Dv, d.ldo, col, span, t0, r8, h * 4, column, outputs.make());
                    if (d.y) store_four<float>(d.y + head * d.Dv, (uint64_t)d.H * d.Dv, col, span, t0, r8, h * 4, column, outputs.y);
                }
                if (c < chunks) outputs.query(room.ops[c % 2], room.shares, h, lane);
            }
        });
    if (kEnds) store_memory<Mine::kOwn>(d.ends + later * d.ends_width() + col, rows, d.ends_width(), mine, r8, share.S);
    else if (d.s_last && unit.part == d.parts - 1) store_memory<Mine::kOwn>(d.s_last + first * d.Dv + col, rows, d.Dv, in, r8, share.S);
}

template <class T, int KS, bool kVec>
__global__ void __launch_bounds__(kMostWaves * 64)
delta_fwd_kernel(Delta d, uint32_t with, uint32_t groups, uint64_t from)
{
    __shared__ Room<T, KS> room;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64, c16 = lane % 16, r8 = lane / 16 * 8;
    const Unit unit(d, 1, groups, from);
    const uint32_t head = unit.head, seq = unit.seq, col = unit.group * with * 16 + wave * 16 + c16;
    const Span span = span_of(d, seq);
    const bool in = wave < with && col < d.Dv;
    const uint64_t memory = ((uint64_t)seq * d.H + head) * d.Dk * d.Dv + col;
    f32x4 S[2 * KS];
    load_memory<KS>(d.s0 ? d.s0 + memory : nullptr, d.Dk, d.Dv, in, r8, S);
    float value[8], out[8], missed[8];
    const T *values = (const T *)d.v + head * d.Dv;
    const uint32_t at = in ? col : 0;
    T next[8];
    // of the chunk before: stored when the next one's loads are on their way, so that none waits for a store
    auto store = [&](uint32_t t0) {
        store_column<T>((T *)d.o + head * d.Dv, d.ldo, at, span, t0, r8, in, out);
        if (d.y) store_column<float>(d.y + head * d.Dv, (uint64_t)d.H * d.Dv, at, span, t0, r8, in, missed);
    };
    load_column<T>(values, d.ldv, at, span, 0, r8, next);
    along<T, KS, false, kVec>(d, span, seq, head, room, wave, waves, [&](const Operands<T, KS> &o, uint32_t c) {
        if (wave >= with) return;
        const uint32_t t0 = c * kChunk;
        if (d.marks && c % (kMark / kChunk) == 0)
            store_memory<KS>(d.marks + ((uint64_t)(first_slot(span, seq) + c / (kMark / kChunk)) * d.H + head) * d.Dk * d.Dv + col, d.Dk, d.Dv, in, r8, S);
        if (c) store(t0 - kChunk);
#pragma unroll
        for (int x = 0; x < 8; ++x) value[x] = held(next[x], span, t0 + r8 + x, in);
        load_column<T>(values, d.ldv, at, span, t0 + kChunk, r8, next);
        take_chunk<T, KS>(o, c16, r8, value, S, out, missed);
    });
    if (span.len && wave < with) store((span.len - 1) / kChunk * kChunk);
    if (d.s_last) store_memory<KS>(d.s_last + memory, d.Dk, d.Dv, in, r8, S);
}

template <class T, int KS>
void launch_size(Delta d, hipStream_t st)
{
    const Columns c = columns_of(d);
    if (c.helped) {
        cut(d, side_by_side(sizeof(Helped<T, KS, false, true>)), side_by_side(sizeof(Helped<T, KS, false>)));
        const uint32_t groups = d.ends_width() / kShared, first = d.n_seq * d.H * (d.parts - 1) * groups, all = d.n_seq * d.H * d.parts * c.groups, threads = kSharedWaves<KS> * 64;
        if (d.parts > 1) {
            if (d.vec_all) delta_fwd_shared_kernel<T, KS, true, true><<<first, threads, 0, st>>>(d, groups, 0);
            else delta_fwd_shared_kernel<T, KS, true, false><<<first, threads, 0, st>>>(d, groups, 0);
            launch_join(d, d.s0, st);
        }
        if (d.vec_all) delta_fwd_shared_kernel<T, KS, false, true><<<all, threads, 0, st>>>(d, c.groups, 0);
        else delta_fwd_shared_kernel<T, KS, false, false><<<all, threads, 0, st>>>(d, c.groups, 0);
        return;
    }
    const uint64_t units = (uint64_t)d.n_seq * d.H * c.groups;
    for (uint64_t from = 0; from < units; from += kMostLaunched) {
        const uint32_t grid = (uint32_t)(units - from < kMostLaunched ? units - from : kMostLaunched);
        if (d.vec_keys) delta_fwd_kernel<T, KS, true><<<grid, c.waves * 64, 0, st>>>(d, c.with, c.groups, from);
        else delta_fwd_kernel<T, KS, false><<<grid, c.waves * 64, 0, st>>>(d, c.with, c.groups, from);
    }
}

template <class T>
void launch_type(const Delta &d, hipStream_t st)
{
    if (d.Dk <= 32) launch_size<T, 1>(d, st);
    else if (d.Dk <= 64) launch_size<T, 2>(d, st);
    else launch_size<T, 4>(d, st);
}

}  // namespace

void dg_delta::launch_forward(const Delta &d, uint32_t dtype, hipStream_t st)
{
    if (dtype == DG_F32) launch_type<float>(d, st);
    else if (dtype == DG_F16) launch_type<f16>(d, st);
    else launch_type<bf16>(d, st);
}
