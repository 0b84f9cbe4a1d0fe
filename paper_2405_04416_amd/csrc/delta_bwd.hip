// The gated delta rule, backward along a sequence: the gradient dS of the memory, and that of what the tokens write, dR = T^T dU.
//   dU = P^T dO + e^(G[last] - G) K dS',   dS = e^G[last] dS' + Q^T (scale e^G dO) - K^T (beta e^G dR),   chunk after chunk from the last one on.
// What is left behind (dR of every token, dS' behind every 64) lets delta_grad.hip take all pieces of 64 tokens at once.
// Bound as the forward pass is, by a chunk's time after the one behind it: 2 x 8192 tokens x 16 heads of 128 x 128, bf16, 0.37 ms (256 chunks, 1.4 us each with all units at work).
#include "delta_chunk.h"

namespace {

using namespace dg_delta;

// A chunk for a wavefront with 16 columns of the gradient, S.  dout: that of o of the lane's eight tokens; gradient: that of what they write.
template <class T, int KS>
__device__ __forceinline__ void take_chunk(const Operands<T, KS> &o, uint32_t c16, uint32_t r8, const float (&dout)[8], f32x4 (&S)[2 * KS], float (&gradient)[8])
{
    constexpr int n = Pieces<T>::n, kTiles = 2 * KS;
    bf16x8 keys[KS][2][n], inverse[2][3], pull[2][3];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) lefts(o.key.K, h * 16 + c16, s * 32 + r8, keys[s][h]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        lefts(o.weight.P, h * 16 + c16, r8, pull[h]);
        lefts(o.weight.inverse, h * 16 + c16, r8, inverse[h]);
    }
    __builtin_amdgcn_sched_barrier(0);
    f32x4 ks[2] = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        bf16x8 sp[3];
        split_rows<3, (n > 1)>(S[2 * s], S[2 * s + 1], sp);
#pragma unroll
        for (int h = 0; h < 2; ++h) ks[h] = multiply<n, 3>(keys[s][h], sp, ks[h]);
    }
    bf16x8 turned[kTiles][n], queries[kTiles][n];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        lefts_turned(o.key.K, t / 2, t % 2, c16 + r8 * 2, turned[t]);
        lefts_turned(o.key.Q, t / 2, t % 2, c16 + r8 * 2, queries[t]);
    }
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 exact[n], right[3], right_q[3];
    split8<n>(dout, exact);
    f32x4 du[2], dr[2], back[2];
    float queried[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x4 until = *reinterpret_cast<const f32x4 *>(&o.weight.until[r8 + h * 4]), query = *reinterpret_cast<const f32x4 *>(&o.weight.query[r8 + h * 4]);
        du[h] = multiply<3, n>(pull[h], exact, until * ks[h]);
#pragma unroll
        for (int x = 0; x < 4; ++x) queried[h * 4 + x] = dout[h * 4 + x] * query[x];
    }
    split_rows<3>(du[0], du[1], right);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        dr[h] = multiply<3, 3>(inverse[h], right, (f32x4){});
        back[h] = -dr[h] * *reinterpret_cast<const f32x4 *>(&o.weight.read[r8 + h * 4]);
#pragma unroll
        for (int x = 0; x < 4; ++x) gradient[h * 4 + x] = dr[h][x];
    }
    split8<3, (n > 1)>(queried, right_q);
    split_rows<3, (n > 1)>(back[0], back[1], right);
    const float whole = o.weight.whole;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        S[t] = multiply<n, 3>(queries[t], right_q, S[t] * whole);
        S[t] = multiply<n, 3>(turned[t], right, S[t]);
    }
}

// The same shared by wavefronts, rows 32 kOwn wave on each.
template <class T, int KS, bool kEnds>
struct Share {
    static constexpr int n = Pieces<T>::n, kOwn = KS / kSharers<KS>;
    f32x4 S[2 * kOwn];
    bf16x8 inverse[2][3], turned[2 * kOwn][n], queries[2 * kOwn][n];
    f32x4 read[2], until[2];
    float whole;

    // up to the sum K S; then all that comes after it is read
    __device__ __forceinline__ void before(const Operands<T, KS> &o, Shares<KS, true, kEnds> &to, uint32_t wave, uint32_t lane)
    {
        const uint32_t c16 = lane % 16, r8 = lane / 16 * 8;
        bf16x8 keys[kOwn][2][n], sp[3];
#pragma unroll
        for (int s = 0; s < kOwn; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) lefts(o.key.K, h * 16 + c16, (wave * kOwn + s) * 32 + r8, keys[s][h]);
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sum[kOwn][2];
#pragma unroll
        for (int s = 0; s < kOwn; ++s) {
            split_rows<3, (n > 1)>(S[2 * s], S[2 * s + 1], sp);
#pragma unroll
            for (int h = 0; h < 2; ++h) sum[s][h] = multiply<n, 3>(keys[s][h], sp, (f32x4){});
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (kOwn == 2) sum[0][h] += sum[1][h];
            to.keys[wave][h][lane] = sum[0][h];
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            until[h] = *reinterpret_cast<const f32x4 *>(&o.weight.until[r8 + h * 4]);
            lefts(o.weight.inverse, h * 16 + c16, r8, inverse[h]);
        }
#pragma unroll
        for (int t = 0; t < 2 * kOwn; ++t) lefts_turned(o.key.Q, wave * kOwn + t / 2, t % 2, lane, queries[t]);
#pragma unroll
        for (int h = 0; h < 2; ++h) read[h] = *reinterpret_cast<const f32x4 *>(&o.weight.read[r8 + h * 4]);
#pragma unroll
        for (int t = 0; t < 2 * kOwn; ++t) lefts_turned(o.key.K, wave * kOwn + t / 2, t % 2, lane, turned[t]);
        whole = o.weight.whole;
    }

    __device__ __forceinline__ void after(Shares<KS, true, kEnds> &shares, uint32_t parity, uint32_t wave, uint32_t lane)
    {
        f32x4 du[2], dr[2], back[2];
        bf16x8 right[3], queried[3];
#pragma unroll
        for (int h = 0; h < 2; ++h) du[h] = shares.ahead[h][lane] + until[h] * shares.sum(shares.keys, h, lane);
#pragma unroll
        for (int p = 0; p < 3; ++p) queried[p] = operand(shares.queried[p][lane]);
        split_rows<3>(du[0], du[1], right);
#pragma unroll
        for (int h = 0; h < 2; ++h) dr[h] = multiply_soon<3, 3>(inverse[h], right, (f32x4){});
        // while that is on its way
#pragma unroll
        for (int t = 0; t < 2 * kOwn; ++t) S[t] = multiply<n, 3>(queries[t], queried, S[t] * whole);
#pragma unroll
        for (int h = 0; h < 2; ++h) back[h] = -dr[h] * read[h];
        split_rows<3, (n > 1)>(back[0], back[1], right);
#pragma unroll
        for (int t = 0; t < 2 * kOwn; ++t) S[t] = multiply<n, 3>(turned[t], right, S[t]);
        if constexpr (!kEnds)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (wave == h % kSharers<KS>) shares.left[parity][h][lane] = dr[h];
    }
};

// what does not wait for S: one wavefront makes P^T dO, the other scale e^G dO in pieces
template <class T, int KS, bool kEnds>
__device__ __forceinline__ void make_ahead(const Operands<T, KS> &o, const Tile<T> &tile, Shares<KS, true, kEnds> &to, uint32_t which, uint32_t lane)
{
    constexpr int n = Pieces<T>::n;
    const uint32_t c16 = lane % 16, r8 = lane / 16 * 8;
    float dout[8];
    tile.read(lane, dout);
    if (which == 0) {
        bf16x8 pull[2][3], exact[n];
#pragma unroll
        for (int h = 0; h < 2; ++h) lefts(o.weight.P, h * 16 + c16, r8, pull[h]);
        split8<n>(dout, exact);
#pragma unroll
        for (int h = 0; h < 2; ++h) to.ahead[h][lane] = multiply<3, n>(pull[h], exact, (f32x4){});
    } else {
        bf16x8 pieces[3];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 query = *reinterpret_cast<const f32x4 *>(&o.weight.query[r8 + h * 4]);
#pragma unroll
            for (int x = 0; x < 4; ++x) dout[h * 4 + x] *= query[x];
        }
        split8<3, (n > 1)>(dout, pieces);
#pragma unroll
        for (int p = 0; p < 3; ++p) to.queried[p][lane] = __builtin_bit_cast(u32x4, pieces[p]);
    }
}

template <class T, int KS, bool kEnds, bool kVec>
__global__ void __launch_bounds__(kSharedWaves<KS> * 64)
delta_bwd_shared_kernel(Delta d, uint32_t groups, uint64_t from)
{
    using Mine = Share<T, KS, kEnds>;
    __shared__ Helped<T, KS, true, kEnds> room;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c16 = lane % 16, r8 = lane / 16 * 8;
    const Unit unit(d, kEnds ? d.parts - 1 : d.parts, groups, from);
    const uint32_t head = unit.head, seq = unit.seq, column0 = unit.group * kShared, col = column0 + c16, one = (d.Dv + 15) / 16 * 16;
    if (kEnds && unit.part == 0 && column0 >= one) return;
    const PartPlace place = PartPlace::of<true>(d, unit);
    const Span &span = place.span;
    const uint32_t row0 = wave * (Mine::kOwn * 32), rows = d.Dk > row0 ? d.Dk - row0 : 0, chunks = (span.len + kChunk - 1) / kChunk;
    const bool column = col < d.Dv, in = wave < kSharers<KS> && column, mine = wave < kSharers<KS>;
    const uint64_t first = ((uint64_t)seq * d.H + head) * d.Dk + row0, later = (((uint64_t)seq * d.parts + unit.part) * d.H + head) * d.Dk + row0;
    Mine share;
    if (kEnds && column0 >= one) unit_memory<Mine::kOwn>(col - one, row0, r8, share.S);
    else if (unit.part == 0 && (kEnds || d.parts == 1)) load_memory<Mine::kOwn>(d.ds_last ? d.ds_last + first * d.Dv + col : nullptr, rows, d.Dv, in, r8, share.S);
    else load_memory<Mine::kOwn>(kEnds ? nullptr : d.starts + later * d.Dv + col, rows, d.Dv, in, r8, share.S);
    f32x4 gradient;
    along_helped<T, KS, true, kEnds, kVec>(d, span, place.slot, head, column0, room, wave,
        [&](uint32_t i) {
            const uint32_t c = chunks - 1 - i;
            share.before(room.ops[i % 2], room.shares, wave, lane);
            if (!kEnds && (i == 0 || c % (kMark / kChunk) == kMark / kChunk - 1))
                store_memory<Mine::kOwn>(d.dmarks + (((uint64_t)(place.mark + c / (kMark / kChunk)) * d.H + head) * d.Dk + row0) * d.Dv + col, rows, d.Dv, in, r8, share.S);
        },
        [&](uint32_t i) { share.after(room.shares, i % 2, wave, lane); },
        [&](uint32_t i) {
            if (i < chunks) make_ahead<T, KS, kEnds>(room.ops[i % 2], room.tiles[i % 2], room.shares, wave - kSharers<KS>, lane);
            if constexpr (!kEnds) gradient = room.shares.left[(i + 1) % 2][wave - kSharers<KS>][lane];
        },
        [&](uint32_t i) {
            if (!kEnds && i) store_four<float>(d.dr + head * d.Dv, (uint64_t)d.H * d.Dv, col, span, (chunks - i) * kChunk, r8, (wave - kSharers<KS>) * 4, column, gradient);
        });
    if (kEnds) store_memory<Mine::kOwn>(d.ends + later * d.ends_width() + col, rows, d.ends_width(), mine, r8, share.S);
    else if (d.ds0 && unit.part == d.parts - 1) store_memory<Mine::kOwn>(d.ds0 + first * d.Dv + col, rows, d.Dv, in, r8, share.S);
}

template <class T, int KS, bool kVec>
__global__ void __launch_bounds__(kMostWaves * 64)
delta_bwd_kernel(Delta d, uint32_t with, uint32_t groups, uint64_t from)
{
    __shared__ Room<T, KS> room;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64, c16 = lane % 16, r8 = lane / 16 * 8;
    const Unit unit(d, 1, groups, from);
    const uint32_t head = unit.head, seq = unit.seq, col = unit.group * with * 16 + wave * 16 + c16;
    const Span span = span_of(d, seq);
    const bool in = wave < with && col < d.Dv;
    const uint64_t memory = ((uint64_t)seq * d.H + head) * d.Dk * d.Dv + col;
    const uint32_t last = span.len ? (span.len - 1) / kChunk : 0;
    f32x4 S[2 * KS];
    load_memory<KS>(d.ds_last ? d.ds_last + memory : nullptr, d.Dk, d.Dv, in, r8, S);
    float dout[8], gradient[8];
    const T *gradients = (const T *)d.dout + head * d.Dv;
    const uint32_t at = in ? col : 0;
    T next[8];
    // of the chunk before: stored when the next one's loads are on their way
    auto store = [&](uint32_t t0) { store_column<float>(d.dr + head * d.Dv, (uint64_t)d.H * d.Dv, at, span, t0, r8, in, gradient); };
    load_column<T>(gradients, d.lddo, at, span, last * kChunk, r8, next);
    along<T, KS, true, kVec>(d, span, seq, head, room, wave, waves, [&](const Operands<T, KS> &o, uint32_t c) {
        if (wave >= with) return;
        const uint32_t t0 = c * kChunk;
        if (c == last || c % (kMark / kChunk) == kMark / kChunk - 1)
            store_memory<KS>(d.dmarks + ((uint64_t)(first_slot(span, seq) + c / (kMark / kChunk)) * d.H + head) * d.Dk * d.Dv + col, d.Dk, d.Dv, in, r8, S);
        if (c != last) store(t0 + kChunk);
#pragma unroll
        for (int x = 0; x < 8; ++x) dout[x] = held(next[x], span, t0 + r8 + x, in);
        load_column<T>(gradients, d.lddo, at, span, c ? t0 - kChunk : 0, r8, next);
        take_chunk<T, KS>(o, c16, r8, dout, S, gradient);
    });
    if (span.len && wave < with) store(0);
    if (d.ds0) store_memory<KS>(d.ds0 + memory, d.Dk, d.Dv, in, r8, S);
}

template <class T, int KS>
void launch_size(Delta d, hipStream_t st)
{
    const Columns c = columns_of(d);
    if (c.helped) {
        cut(d, side_by_side(sizeof(Helped<T, KS, true, true>)), side_by_side(sizeof(Helped<T, KS, true>)));
        const uint32_t groups = d.ends_width() / kShared, first = d.n_seq * d.H * (d.parts - 1) * groups, all = d.n_seq * d.H * d.parts * c.groups, threads = kSharedWaves<KS> * 64;
        if (d.parts > 1) {
            if (d.vec_all) delta_bwd_shared_kernel<T, KS, true, true><<<first, threads, 0, st>>>(d, groups, 0);
            else delta_bwd_shared_kernel<T, KS, true, false><<<first, threads, 0, st>>>(d, groups, 0);
            launch_join(d, d.ds_last, st);
        }
        if (d.vec_all) delta_bwd_shared_kernel<T, KS, false, true><<<all, threads, 0, st>>>(d, c.groups, 0);
        else delta_bwd_shared_kernel<T, KS, false, false><<<all, threads, 0, st>>>(d, c.groups, 0);
        return;
    }
    const uint64_t units = (uint64_t)d.n_seq * d.H * c.groups;
    for (uint64_t from = 0; from < units; from += kMostLaunched) {
        const uint32_t grid = (uint32_t)(units - from < kMostLaunched ? units - from : kMostLaunched);
        if (d.vec_keys) delta_bwd_kernel<T, KS, true><<<grid, c.waves * 64, 0, st>>>(d, c.with, c.groups, from);
        else delta_bwd_kernel<T, KS, false><<<grid, c.waves * 64, 0, st>>>(d, c.with, c.groups, from);
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

void dg_delta::launch_backward(const Delta &d, uint32_t dtype, hipStream_t st)
{
    if (dtype == DG_F32) launch_type<float>(d, st);
    else if (dtype == DG_F16) launch_type<f16>(d, st);
    else launch_type<bf16>(d, st);
}
