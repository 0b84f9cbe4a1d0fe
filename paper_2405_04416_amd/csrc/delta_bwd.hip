// The gated delta rule, backward along a sequence: the gradient dS of the memory, and that of what the tokens write, dR = T^T dU.
//   dU = P^T dO + e^(G[last] - G) K dS',   dS = e^G[last] dS' + Q^T (scale e^G dO) - K^T (beta e^G dR),   chunk after chunk from the last one on.
// What is left behind (dR of every token, dS' behind every 64) lets delta_grad.hip take all pieces of 64 tokens at once.
#include "delta_chunk.h"

namespace {

using namespace dg_delta;

template <class T, int KS>
__global__ void __launch_bounds__(kMostWaves * 64)
delta_bwd_kernel(Delta d, uint32_t with, uint32_t groups, uint64_t from)
{
    __shared__ alignas(16) Room<T, KS, true> room;
    constexpr int n = Pieces<T>::n, kTiles = 2 * KS;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64, c16 = lane % 16, r8 = lane / 16 * 8;
    const uint64_t unit = from + blockIdx.x;
    const uint32_t head = (uint32_t)(unit / groups % d.H), seq = (uint32_t)(unit / groups / d.H), col = ((uint32_t)(unit % groups) * with + wave) * 16 + c16;
    const Span span = span_of(d, seq);
    const bool in = wave < with && col < d.Dv;
    const uint64_t memory = ((uint64_t)seq * d.H + head) * d.Dk * d.Dv + col;
    f32x4 S[kTiles];
    load_memory<KS>(d.ds_last ? d.ds_last + memory : nullptr, d.Dk, d.Dv, in, r8, S);
    const T *gradients = (const T *)d.dout + head * d.Dv + (in ? col : 0);
    const uint32_t last = span.len ? (span.len - 1) / kChunk : 0;
    T next[8];
    if (span.len) load_column<T>(gradients, d.lddo, span, last * kChunk + r8, in, next);
    along<T, KS, true>(d, span, seq, head, room, wave, waves, [&](const Operands<T, KS, true> &o, uint32_t c) {
        if (wave >= with) return;
        if (c == last || c % (kMark / kChunk) == kMark / kChunk - 1)
            store_memory<KS>(d.dmarks + ((uint64_t)(first_slot(span, seq) + c / (kMark / kChunk)) * d.H + head) * d.Dk * d.Dv + col, d.Dk, d.Dv, in, r8, S);
        float dout[8], queried[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            dout[x] = (float)next[x];
            queried[x] = dout[x] * o.weight.query[r8 + x];
        }
        load_column<T>(gradients, d.lddo, span, (c ? c - 1 : 0) * kChunk + r8, in, next);
        f32x4 ks[2] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            bf16x8 sp[3];
            split_rows<3>(S[2 * s], S[2 * s + 1], sp);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 a[n];
#pragma unroll
                for (int p = 0; p < n; ++p) a[p] = left(&o.key.K[p][h * 16 + c16][s * 32 + r8]);
                ks[h] = multiply<n, 3>(a, sp, ks[h]);
            }
        }
        bf16x8 exact[n], right[3];
        split8<n>(dout, exact);
        f32x4 du[2], dr[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 until = *reinterpret_cast<const f32x4 *>(&o.weight.until[r8 + h * 4]);
            bf16x8 a[3];
#pragma unroll
            for (int p = 0; p < 3; ++p) a[p] = left(&o.weight.P[p][h * 16 + c16][r8]);
            du[h] = multiply<3, n>(a, exact, until * ks[h]);
        }
        split_rows<3>(du[0], du[1], right);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8 a[3];
#pragma unroll
            for (int p = 0; p < 3; ++p) a[p] = left(&o.weight.inverse[p][h * 16 + c16][r8]);
            dr[h] = multiply<3, 3>(a, right, (f32x4){});
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t t = c * kChunk + r8 + h * 4 + x;
                if (in && t < span.len) d.dr[(span.row(t) * d.H + head) * d.Dv + col] = dr[h][x];
            }
            dr[h] *= -*reinterpret_cast<const f32x4 *>(&o.weight.read[r8 + h * 4]);
        }
        bf16x8 right_q[3];
        split8<3>(queried, right_q);
        split_rows<3>(dr[0], dr[1], right);
        const float whole = o.weight.whole;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            bf16x8 a[n];
#pragma unroll
            for (int p = 0; p < n; ++p) a[p] = left(&o.key.Q[p][t * 16 + c16][r8]);
            S[t] = multiply<n, 3>(a, right_q, S[t] * whole);
#pragma unroll
            for (int p = 0; p < n; ++p) a[p] = left(&o.key.KT[p][t * 16 + c16][r8]);
            S[t] = multiply<n, 3>(a, right, S[t]);
        }
    });
    if (d.ds0) store_memory<KS>(d.ds0 + memory, d.Dk, d.Dv, in, r8, S);
}

template <class T>
void launch_type(const Delta &d, hipStream_t st)
{
    const Columns c = columns_of(d);
    const uint64_t units = (uint64_t)d.n_seq * d.H * c.groups;
    for (uint64_t from = 0; from < units; from += kMostGroups) {
        const uint32_t grid = (uint32_t)(units - from < kMostGroups ? units - from : kMostGroups), threads = c.waves * 64;
        if (d.Dk <= 32) delta_bwd_kernel<T, 1><<<grid, threads, 0, st>>>(d, c.with, c.groups, from);
        else if (d.Dk <= 64) delta_bwd_kernel<T, 2><<<grid, threads, 0, st>>>(d, c.with, c.groups, from);
        else delta_bwd_kernel<T, 4><<<grid, threads, 0, st>>>(d, c.with, c.groups, from);
    }
}

}  // namespace

void dg_delta::launch_backward(const Delta &d, uint32_t dtype, hipStream_t st)
{
    if (dtype == DG_F32) launch_type<float>(d, st);
    else if (dtype == DG_F16) launch_type<f16>(d, st);
    else launch_type<bf16>(d, st);
}
