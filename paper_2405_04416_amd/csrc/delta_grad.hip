// The gated delta rule, backward, what follows from the memories S before and the gradients dS' behind each 64 tokens, and from what the tokens write (U) and its
// gradient (dR): with X = scale D (dO U^T) up to the diagonal, Y = -beta D (dR U^T) below it, and D, G of the 64 tokens,
//   dq = scale e^G dO S^T + X K,
//   dk = -beta e^G dR S^T + e^(G[last] - G) U dS'^T + X^T Q + Y K + Y^T K,    dv = beta dR,
//   dbeta = dR (v - e^G S^T k) - sum over j of D k k[j] (dR U[j]^T),
//   dG[i] = q (first part of dq) + k (first part of dk) - k (second part) + sum over j of Z[i, j] - sum over j of Z[j, i],  Z = X (q k) + Y (k k),
//   dG[last] also + the sum of all k (second part of dk) + e^G[last] <S, dS'>;   dg[t] = sum of dG from t on.
//
// A workgroup takes 64 tokens of a key head, one value head after the other, a wavefront 16 of them: a lane has a token, of which everything above is a column
// of a product, so that what X and Y become are right operands of the next product where they are.  X and Y are made twice, by rows and by columns.
#include "delta_chunk.h"

namespace {

using namespace dg_delta;

constexpr int kTokens = kMark, kTokenPitch = kTokens + 8;

template <class T, int KS>
struct Shared {
    static constexpr int n = Pieces<T>::n;
    uint16_t KT[n][32 * KS][kTokenPitch], QT[n][32 * KS][kTokenPitch];
    double G[kTokens];
    float beta[kTokens], dG[kTokens], end[4];
};

// A lane has rows 4 q to 4 q + 3 of two results of 16, which become places 8 q to 8 q + 7 of the next sum over tokens: where token t stands among the columns
// of its left operands.
__device__ __forceinline__ uint32_t place(uint32_t t) { return (t & ~31u) | (t >> 2 & 3) << 3 | (t >> 4 & 1) << 2 | (t & 3); }

// sum over the four lanes that have a token
__device__ __forceinline__ float of_token(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

template <class T, int KS>
__global__ void __launch_bounds__(256, 1)
delta_grad_kernel(Delta d, uint64_t from)
{
    __shared__ alignas(16) Shared<T, KS> lds;
    constexpr int n = Pieces<T>::n, kTiles = 2 * KS;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c16 = lane % 16, r4 = lane / 16 * 4, r8 = lane / 16 * 8;
    const uint64_t unit = from + blockIdx.x;
    const uint32_t hk = (uint32_t)(unit % d.Hk), group = d.H / d.Hk;
    uint32_t slot = (uint32_t)(unit / d.Hk), seq, block;
    if (d.first) {
        seq = d.slot_seq[slot];
        if (seq >= d.n_seq) return;
    } else {
        const uint32_t each = (uint32_t)((d.N / d.n_seq + kTokens - 1) / kTokens);
        seq = slot / each;
        block = slot % each;
    }
    const Span span = span_of(d, seq);
    if (d.first) block = slot - first_slot(span, seq);
    else slot = first_slot(span, seq) + block;
    if ((uint64_t)block * kTokens >= span.len) return;
    const uint32_t t0 = block * kTokens, count = span.len - t0 < kTokens ? span.len - t0 : kTokens;
    const T *K = (const T *)d.k + hk * d.Dk, *Q = (const T *)d.q + hk * d.Dk;

    // columns of K and Q as rows
    for (uint32_t item = threadIdx.x; item < kTokens * 4 * KS; item += 256) {
        const uint32_t t = item / (4 * KS), col = item % (4 * KS) * 8;
        const bool in = t < count;
        const uint64_t row = span.row(t0 + (in ? t : 0));
        float v[8];
        uint32_t w[n][4];
        eight<T>(K + row * d.ldk, col, d.Dk, in, d.vec_k, v);
        split<n, 8>(v, w);
#pragma unroll
        for (int p = 0; p < n; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) lds.KT[p][col + i][place(t)] = (uint16_t)(w[p][i / 2] >> (i % 2 * 16));
        eight<T>(Q + row * d.ldq, col, d.Dk, in, d.vec_q, v);
        split<n, 8>(v, w);
#pragma unroll
        for (int p = 0; p < n; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) lds.QT[p][col + i][place(t)] = (uint16_t)(w[p][i / 2] >> (i % 2 * 16));
    }

    const uint32_t mine = wave * 16 + c16;              // a lane's token
    const bool in = mine < count;
    const uint64_t row = span.row(t0 + (in ? mine : 0));
    auto row_of = [&](uint32_t t) { return span.row(t0 + (t < count ? t : 0)); };
    f32x4 dq[kTiles] = {}, dk[kTiles] = {};
    const bool vec_f = d.Dv % 4 == 0;

    for (uint32_t h = 0; h < group; ++h) {
        const uint32_t head = hk * group + h;
        __syncthreads();                                // what the last head left in LDS has been read
        if (wave == 0) {
            const bool held = lane < count;
            const uint64_t r = row_of(lane);
            const float value = d.g[r * d.ldg + head], b = d.beta[r * d.ldb + head];
            double G = held ? (double)fmaxf(value, kShut) : 0.0;
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const double before = __shfl_up(G, s);
                if (lane >= (uint32_t)s) G += before;
            }
            lds.G[lane] = G;
            lds.beta[lane] = held ? b : 0.0f;
        }
        __syncthreads();
        const float *S = d.marks + ((uint64_t)slot * d.H + head) * d.Dk * d.Dv, *dS = d.dmarks + ((uint64_t)slot * d.H + head) * d.Dk * d.Dv;
        const float *U = d.u + head * d.Dv, *R = d.dr + head * d.Dv;
        const uint64_t ldu = (uint64_t)d.H * d.Dv;
        const T *O = (const T *)d.dout + head * d.Dv;
        f32x4 from_q[kTiles] = {}, from_k[kTiles] = {}, to_k[kTiles] = {};          // dO S^T, dR S^T, U dS'^T
        f32x4 m1[4] = {}, e1[4] = {}, m2[4] = {}, e2[4] = {};                       // dO U^T, dR U^T of the lane's row and of its column
        float dbeta = 0.0f, dot = 0.0f;
        const float beta = lds.beta[mine];
#pragma unroll 1
        for (uint32_t c0 = 0; c0 < d.Dv; c0 += 32) {
            const uint32_t c = c0 + r8;
            float x[8], y[8];
            bf16x8 o[n], r[3], u[3];
            eight<T>(O + row * d.lddo, c, d.Dv, in, d.vec_o, x);
            split8<n>(x, o);
            eight<float>(U + row * ldu, c, d.Dv, in, vec_f, x);
            split8<3>(x, u);
            eight<float>(R + row * ldu, c, d.Dv, in, vec_f, x);
            split8<3>(x, r);
            eight<T>((const T *)d.v + head * d.Dv + row * d.ldv, c, d.Dv, in, d.vec_v, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) dbeta = fmaf(x[i], y[i], dbeta);
            if (in) {
                T *to = (T *)d.dv + row * d.lddv + head * d.Dv + c;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < d.Dv) to[i] = (T)(beta * x[i]);
            }
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const uint32_t rk = t * 16 + c16;
                float s[8], ds[8];
                bf16x8 a[3];
                eight<float>(S + (uint64_t)(rk < d.Dk ? rk : 0) * d.Dv, c, d.Dv, rk < d.Dk, vec_f, s);
                eight<float>(dS + (uint64_t)(rk < d.Dk ? rk : 0) * d.Dv, c, d.Dv, rk < d.Dk, vec_f, ds);
                if (t % 4 == (int)wave)
#pragma unroll
                    for (int i = 0; i < 8; ++i) dot = fmaf(s[i], ds[i], dot);
                split8<3>(s, a);
                from_q[t] = multiply<3, n>(a, o, from_q[t]);
                from_k[t] = multiply<3, 3>(a, r, from_k[t]);
                split8<3>(ds, a);
                to_k[t] = multiply<3, 3>(a, u, to_k[t]);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t other = t * 16 + c16;
                const bool there = other < count;
                const uint64_t at = row_of(other);
                if (t <= (int)wave) {                   // tokens j: up to the lane's
                    bf16x8 a[3];
                    eight<float>(U + at * ldu, c, d.Dv, there, vec_f, x);
                    split8<3>(x, a);
                    m1[t] = multiply<3, n>(a, o, m1[t]);
                    e1[t] = multiply<3, 3>(a, r, e1[t]);
                }
                if (t >= (int)wave) {                   // tokens i: from the lane's on
                    bf16x8 a[3], b[n];
                    eight<T>(O + at * d.lddo, c, d.Dv, there, d.vec_o, x);
                    split8<n>(x, b);
                    m2[t] = multiply<n, 3>(b, u, m2[t]);
                    eight<float>(R + at * ldu, c, d.Dv, there, vec_f, x);
                    split8<3>(x, a);
                    e2[t] = multiply<3, 3>(a, u, e2[t]);
                }
            }
        }
        // k k and q k, of the lane's row and of its column; X and Y take the places of dO U^T and dR U^T
        f32x4 kk1[4] = {}, qk1[4] = {}, kk2[4] = {}, qk2[4] = {};
#pragma unroll 1
        for (uint32_t c0 = 0; c0 < d.Dk; c0 += 32) {
            const uint32_t c = c0 + r8;
            float x[8];
            bf16x8 k[n], q[n], a[n];
            eight<T>(K + row * d.ldk, c, d.Dk, in, d.vec_k, x);
            split8<n>(x, k);
            eight<T>(Q + row * d.ldq, c, d.Dk, in, d.vec_q, x);
            split8<n>(x, q);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t other = t * 16 + c16;
                const bool there = other < count;
                const uint64_t at = row_of(other);
                eight<T>(K + at * d.ldk, c, d.Dk, there, d.vec_k, x);
                split8<n>(x, a);
                if (t <= (int)wave) {
                    kk1[t] = multiply<n, n>(a, k, kk1[t]);
                    qk1[t] = multiply<n, n>(a, q, qk1[t]);
                }
                if (t >= (int)wave) {
                    kk2[t] = multiply<n, n>(a, k, kk2[t]);
                    eight<T>(Q + at * d.ldq, c, d.Dk, there, d.vec_q, x);
                    split8<n>(x, a);
                    qk2[t] = multiply<n, n>(a, k, qk2[t]);
                }
            }
        }
        const double G = lds.G[mine], last = lds.G[kTokens - 1];
        const float since = expf((float)G), until = expf((float)(last - G));
        float dG = 0.0f;
        dbeta = of_token(dbeta);
        float pulled = 0.0f;                            // sum over j of D k k[j] (dR U[j]^T)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t j = t * 16 + r4 + x;
                const float fade = j <= mine ? expf((float)(G - lds.G[j])) : 0.0f;
                const float e = j < mine ? fade * e1[t][x] : 0.0f;
                m1[t][x] = j <= mine ? d.scale * fade * m1[t][x] : 0.0f;
                pulled = fmaf(e, kk1[t][x], pulled);
                e1[t][x] = -beta * e;
                dG += m1[t][x] * qk1[t][x] + e1[t][x] * kk1[t][x];
                const float grown = j >= mine ? expf((float)(lds.G[j] - G)) : 0.0f;     // j is the later token here
                m2[t][x] = j >= mine ? d.scale * grown * m2[t][x] : 0.0f;
                e2[t][x] = j > mine ? -lds.beta[j] * grown * e2[t][x] : 0.0f;
                dG -= m2[t][x] * qk2[t][x] + e2[t][x] * kk2[t][x];
            }
        dbeta -= of_token(pulled);
        float at_end = 0.0f, read = 0.0f;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const f32x4 rq = from_q[t] * (d.scale * since), rk = from_k[t], wk = to_k[t] * until;
            dq[t] += rq;
            dk[t] += wk - rk * (beta * since);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t c = t * 16 + r4 + x;
                const bool here = in && c < d.Dk;
                const float q = here ? (float)Q[row * d.ldq + c] : 0.0f, k = here ? (float)K[row * d.ldk + c] : 0.0f;
                dG = fmaf(q, rq[x], dG);
                read = fmaf(k, rk[x], read);
                at_end = fmaf(k, wk[x], at_end);
            }
        }
        read = of_token(read) * since;
        dbeta -= read;
        dG = of_token(dG - at_end) - beta * read;
        at_end = of_token(at_end);
        if (lane < 16) lds.dG[mine] = dG;
        // the whole workgroup's share of dG[last]
        float end = fmaf(expf((float)last), dot, lane < 16 ? at_end : 0.0f);
#pragma unroll
        for (int s = 1; s < 64; s *= 2) end += __shfl_xor(end, s);
        if (lane == 0) lds.end[wave] = end;
        if (lane < 16 && in) d.dbeta[row * d.lddb + head] = dbeta;
        __syncthreads();
        if (wave == 0) {
            float sum = lds.dG[lane] + (lane == 63 ? lds.end[0] + lds.end[1] + lds.end[2] + lds.end[3] : 0.0f);
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const float after = __shfl_down(sum, s);
                if (lane + s < 64) sum += after;
            }
            if (lane < count) d.dg[row_of(lane) * d.lddg + head] = sum;
        }
        // what the tokens of the block tell each other
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 x1[3], y1[3], x2[3], y2[3];
            const bool before = 2 * s <= (int)wave, after = 2 * s + 1 >= (int)wave;
            split_rows<3>(m1[2 * s], m1[2 * s + 1], x1);
            split_rows<3>(e1[2 * s], e1[2 * s + 1], y1);
            split_rows<3>(m2[2 * s], m2[2 * s + 1], x2);
            split_rows<3>(e2[2 * s], e2[2 * s + 1], y2);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                bf16x8 a[n], b[n];
#pragma unroll
                for (int p = 0; p < n; ++p) {
                    a[p] = left(&lds.KT[p][t * 16 + c16][s * 32 + r8]);
                    b[p] = left(&lds.QT[p][t * 16 + c16][s * 32 + r8]);
                }
                if (before) {
                    dq[t] = multiply<n, 3>(a, x1, dq[t]);
                    dk[t] = multiply<n, 3>(a, y1, dk[t]);
                }
                if (after) {
                    dk[t] = multiply<n, 3>(b, x2, dk[t]);
                    dk[t] = multiply<n, 3>(a, y2, dk[t]);
                }
            }
        }
    }
    if (!in) return;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t c = t * 16 + r4 + x;
            if (c >= d.Dk) continue;
            ((T *)d.dq)[row * d.lddq + hk * d.Dk + c] = (T)dq[t][x];
            ((T *)d.dk)[row * d.lddk + hk * d.Dk + c] = (T)dk[t][x];
        }
}

// The sequence of each slot, ~0 where it is empty: the last sequence whose slots begin at or before it, if it has so many.
__global__ void __launch_bounds__(256)
delta_slots_kernel(Delta d, uint32_t *slot_seq)
{
    const uint32_t slot = blockIdx.x * 256 + threadIdx.x;
    if (slot >= d.slots) return;
    uint32_t low = 0, high = d.n_seq;               // slots of sequence `low` begin at or before this one, those of `high` behind it
    while (high - low > 1) {
        const uint32_t mid = low + (high - low) / 2;
        if (first_slot(span_of(d, mid), mid) <= slot) low = mid;
        else high = mid;
    }
    const Span span = span_of(d, low);
    const uint32_t begin = first_slot(span, low);
    slot_seq[slot] = begin <= slot && (uint64_t)(slot - begin) * kTokens < span.len ? low : ~0u;
}

template <class T>
void launch_type(const Delta &d, hipStream_t st)
{
    const uint64_t slots = d.first ? d.slots : d.n_seq * ((d.N / d.n_seq + kTokens - 1) / kTokens), units = slots * d.Hk;
    for (uint64_t from = 0; from < units; from += kMostGroups) {
        const uint32_t grid = (uint32_t)(units - from < kMostGroups ? units - from : kMostGroups);
        if (d.Dk <= 32) delta_grad_kernel<T, 1><<<grid, 256, 0, st>>>(d, from);
        else if (d.Dk <= 64) delta_grad_kernel<T, 2><<<grid, 256, 0, st>>>(d, from);
        else delta_grad_kernel<T, 4><<<grid, 256, 0, st>>>(d, from);
    }
}

}  // namespace

void dg_delta::launch_gradients(const Delta &d, uint32_t dtype, hipStream_t st)
{
    if (d.first) delta_slots_kernel<<<(d.slots + 255) / 256, 256, 0, st>>>(d, const_cast<uint32_t *>(d.slot_seq));
    if (dtype == DG_F32) launch_type<float>(d, st);
    else if (dtype == DG_F16) launch_type<f16>(d, st);
    else launch_type<bf16>(d, st);
}
