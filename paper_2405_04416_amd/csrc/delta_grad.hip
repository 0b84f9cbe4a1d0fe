// The gated delta rule, backward, what follows from the memories S before and the gradients dS' behind each 64 tokens, and from what the tokens miss (Y = v - S^T k)
// and the gradient dR of what they write (U = beta Y): with X = scale D (dO U^T) up to the diagonal, Z = -beta D (dR U^T) below it, D and G of the 64 tokens,
//   dq = scale e^G dO S^T + X K,    dk = -beta e^G dR S^T + e^(G[last] - G) U dS'^T + X^T Q + Z K + Z^T K,    dv = beta dR,   dbeta = dR Y.
// With e^-G S for a memory the rule has no decay, values e^-G v and results e^G o: so dG = o do - v dv = q dq - v dv, and dG[last] also the product of the memory
// behind, e^G[last] S + K^T e^(G[last] - G) U, with dS';  dg[t] = sum of dG from t on.
//
// A workgroup takes 64 tokens of a key head, one value head after the other, 32 columns of values at a time through LDS (in pieces, cut once for all), a wavefront
// 16 tokens: a lane has a token, of which everything above is a column of a product, so that what X and Z become are right operands of the next product where
// they are.  X and Z are made twice, by rows and by columns.
#include "delta_chunk.h"

namespace {

using namespace dg_delta;

constexpr int kTokens = kMark, kTokenPitch = kTokens + 8, kColumns = 32, kColumnPitch = kColumns + 8;

template <class T, int KS>
struct Shared {
    static constexpr int n = Pieces<T>::n;
    union {
        struct {                        // 32 columns of values at a time
            uint16_t S[3][32 * KS][kColumnPitch], dS[3][32 * KS][kColumnPitch], U[3][kTokens][kColumnPitch], R[3][kTokens][kColumnPitch], O[n][kTokens][kColumnPitch];
        };
        struct { uint16_t KT[n][32 * KS][kTokenPitch], QT[n][32 * KS][kTokenPitch]; };
    };
    double G[kTokens];
    float beta[kTokens], dG[kTokens], values[kTokens], end[4];
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

// Eight values of a row from column c on, or others where there are none: `cleared` tells them apart when they are used, so that nothing waits for the load
template <class T, bool kVec>
__device__ __forceinline__ void ahead(const T *row, uint32_t c, uint32_t D, dg_rows::Pack<T, 8> &out)
{
    constexpr int m = 16 / sizeof(T);
    if constexpr (kVec) {
#pragma unroll
        for (int h = 0; h < 8 / m; ++h) {
            const dg_rows::Pack<T, m> p = *reinterpret_cast<const dg_rows::Pack<T, m> *>(row + (c + h * m < D ? c + h * m : 0));
#pragma unroll
            for (int i = 0; i < m; ++i) out.v[h * m + i] = p.v[i];
        }
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) out.v[i] = row[c + i < D ? c + i : 0];
}

template <class T>
__device__ __forceinline__ void cleared(const dg_rows::Pack<T, 8> &p, uint32_t c, uint32_t D, bool in, float (&out)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = in && c + i < D ? (float)p.v[i] : 0.0f;
}

template <int n, int rows, int pitch>
__device__ __forceinline__ void put8(const float (&v)[8], uint16_t (&to)[n][rows][pitch], uint32_t row, uint32_t col)
{
    uint32_t w[n][4];
    split<n, 8>(v, w);
#pragma unroll
    for (int p = 0; p < n; ++p) *reinterpret_cast<u32x4 *>(&to[p][row][col]) = (u32x4){w[p][0], w[p][1], w[p][2], w[p][3]};
}

template <class T, int KS, bool kVec>
__global__ void __launch_bounds__(256, 1)
delta_grad_kernel(Delta d, uint64_t from)
{
    __shared__ alignas(16) Shared<T, KS> lds;
    constexpr int n = Pieces<T>::n, kTiles = 2 * KS, kMemoryRows = KS == 4 ? 2 : 1;     // rows of the memory that a thread brings
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
    auto row_of = [&](uint32_t t) { return span.row(t0 + (t < count ? t : 0)); };

    const uint32_t mine = wave * 16 + c16;              // the token that a lane has as a column
    const bool in = mine < count;
    const uint64_t row = row_of(mine);
    const uint32_t brought = threadIdx.x / 4, c8 = threadIdx.x % 4 * 8;         // the token, or row of the memory, of which a thread brings eight columns
    const bool there = brought < count;
    const uint64_t brought_row = row_of(brought);
    f32x4 dq[kTiles] = {}, dk[kTiles] = {};

    for (uint32_t h = 0; h < group; ++h) {
        const uint32_t head = hk * group + h;
        const float *S = d.marks + ((uint64_t)slot * d.H + head) * d.Dk * d.Dv, *dS = d.dmarks + ((uint64_t)slot * d.H + head) * d.Dk * d.Dv;
        const uint64_t at = (brought_row * d.H + head) * d.Dv;
        dg_rows::Pack<float, 8> next_s[kMemoryRows], next_ds[kMemoryRows], next_y, next_r;
        dg_rows::Pack<T, 8> next_o, next_v;
        auto fetch = [&](uint32_t c) {
#pragma unroll
            for (int i = 0; i < kMemoryRows; ++i) {
                const uint64_t r = brought + i * 64 < d.Dk ? brought + i * 64 : 0;
                ahead<float, kVec>(S + r * d.Dv, c, d.Dv, next_s[i]);
                ahead<float, kVec>(dS + r * d.Dv, c, d.Dv, next_ds[i]);
            }
            ahead<float, kVec>(d.y + at, c, d.Dv, next_y);
            ahead<float, kVec>(d.dr + at, c, d.Dv, next_r);
            ahead<T, kVec>((const T *)d.dout + brought_row * d.lddo + head * d.Dv, c, d.Dv, next_o);
            ahead<T, kVec>((const T *)d.v + brought_row * d.ldv + head * d.Dv, c, d.Dv, next_v);
        };
        fetch(c8);
        const float beta_brought = there ? d.beta[brought_row * d.ldb + head] : 0.0f;
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
        f32x4 from_q[kTiles] = {}, from_k[kTiles] = {}, to_k[kTiles] = {};          // dO S^T, dR S^T, U dS'^T
        f32x4 m1[4] = {}, e1[4] = {}, m2[4] = {}, e2[4] = {};                       // dO U^T, dR U^T of the lane's row and of its column
        float dbeta = 0.0f, dot = 0.0f, values = 0.0f;
#pragma unroll 1
        for (uint32_t c0 = 0; c0 < d.Dv; c0 += kColumns) {
            {
                const uint32_t c = c0 + c8;
                float x[8], y[8], r[8];
#pragma unroll
                for (int i = 0; i < kMemoryRows; ++i) {
                    const uint32_t to = brought + i * 64;
                    if (to >= 32 * KS) continue;
                    cleared<float>(next_s[i], c, d.Dv, to < d.Dk, x);
                    put8(x, lds.S, to, c8);
                    cleared<float>(next_ds[i], c, d.Dv, to < d.Dk, y);
                    put8(y, lds.dS, to, c8);
#pragma unroll
                    for (int j = 0; j < 8; ++j) dot = fmaf(x[j], y[j], dot);
                }
                cleared<float>(next_r, c, d.Dv, there, r);
                put8(r, lds.R, brought, c8);
                cleared<float>(next_y, c, d.Dv, there, y);
                cleared<T>(next_v, c, d.Dv, there, x);
                T *dv = (T *)d.dv + brought_row * d.lddv + head * d.Dv + c;
                float out[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    dbeta = fmaf(r[j], y[j], dbeta);
                    y[j] *= beta_brought;
                    out[j] = beta_brought * r[j];
                    values = fmaf(out[j], x[j], values);
                    if (!kVec && there && c + j < d.Dv) dv[j] = (T)out[j];
                }
                if (kVec && there) {
                    constexpr int m = 16 / sizeof(T);
#pragma unroll
                    for (int j = 0; j < 8; j += m) {
                        float part[m];
#pragma unroll
                        for (int i = 0; i < m; ++i) part[i] = out[j + i];
                        if (c + j < d.Dv) dg_rows::store<T, m>(dv + j, part);
                    }
                }
                put8(y, lds.U, brought, c8);
                cleared<T>(next_o, c, d.Dv, there, x);
                put8(x, lds.O, brought, c8);
            }
            __syncthreads();
            if (c0 + kColumns < d.Dv) fetch(c0 + kColumns + c8);
            bf16x8 o[n], r[3], u[3], a[3], b[n];
            lefts(lds.O, mine, r8, o);
            lefts(lds.R, mine, r8, r);
            lefts(lds.U, mine, r8, u);
            // one tile's operands on their way while another's are multiplied, and no more, for which there would not be registers
            bf16x8 s2[2][3], ds2[2][3];
            lefts(lds.S, c16, r8, s2[0]);
            lefts(lds.dS, c16, r8, ds2[0]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if (t + 1 < kTiles) {
                    lefts(lds.S, (t + 1) * 16 + c16, r8, s2[(t + 1) % 2]);
                    lefts(lds.dS, (t + 1) * 16 + c16, r8, ds2[(t + 1) % 2]);
                }
                __builtin_amdgcn_sched_barrier(0);
                from_q[t] = multiply<3, n>(s2[t % 2], o, from_q[t]);
                from_k[t] = multiply<3, 3>(s2[t % 2], r, from_k[t]);
                to_k[t] = multiply<3, 3>(ds2[t % 2], u, to_k[t]);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                __builtin_amdgcn_sched_barrier(0);
                if (t <= (int)wave) {                   // tokens j: up to the lane's
                    lefts(lds.U, t * 16 + c16, r8, a);
                    m1[t] = multiply<3, n>(a, o, m1[t]);
                    e1[t] = multiply<3, 3>(a, r, e1[t]);
                }
                if (t >= (int)wave) {                   // tokens i: from the lane's on
                    lefts(lds.O, t * 16 + c16, r8, b);
                    m2[t] = multiply<n, 3>(b, u, m2[t]);
                    lefts(lds.R, t * 16 + c16, r8, a);
                    e2[t] = multiply<3, 3>(a, u, e2[t]);
                }
            }
            __syncthreads();
        }
        dbeta += __shfl_xor(dbeta, 1);
        dbeta += __shfl_xor(dbeta, 2);
        values += __shfl_xor(values, 1);
        values += __shfl_xor(values, 2);
        if (threadIdx.x % 4 == 0) {
            lds.values[brought] = values;
            if (there) d.dbeta[brought_row * d.lddb + head] = dbeta;
        }
        const double G = lds.G[mine], last = lds.G[kTokens - 1];
        const float since = expf((float)G), until = expf((float)(last - G)), beta = lds.beta[mine];
        // columns of K and Q as rows, where the columns of values have been
        for (uint32_t item = threadIdx.x; item < kTokens * 4 * KS; item += 256) {
            const uint32_t t = item / (4 * KS), col = item % (4 * KS) * 8;
            dg_rows::Pack<T, 8> k8, q8;
            ahead<T, kVec>(K + row_of(t) * d.ldk, col, d.Dk, k8);
            ahead<T, kVec>(Q + row_of(t) * d.ldq, col, d.Dk, q8);
            float v[8];
            uint32_t w[n][4];
            cleared<T>(k8, col, d.Dk, t < count, v);
            split<n, 8>(v, w);
    #pragma unroll
            for (int p = 0; p < n; ++p)
    #pragma unroll
                for (int i = 0; i < 8; ++i) lds.KT[p][col + i][place(t)] = (uint16_t)(w[p][i / 2] >> (i % 2 * 16));
            cleared<T>(q8, col, d.Dk, t < count, v);
            split<n, 8>(v, w);
    #pragma unroll
            for (int p = 0; p < n; ++p)
    #pragma unroll
                for (int i = 0; i < 8; ++i) lds.QT[p][col + i][place(t)] = (uint16_t)(w[p][i / 2] >> (i % 2 * 16));
        }
        // X and Z, of the lane's row and of its column
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t j = t * 16 + r4 + x;
                if (t <= (int)wave) {
                    const float fade = j <= mine ? expf((float)(G - lds.G[j])) : 0.0f;
                    m1[t][x] *= d.scale * fade;
                    e1[t][x] = j < mine ? -beta * fade * e1[t][x] : 0.0f;
                }
                if (t >= (int)wave) {                   // j is the later token here
                    const float fade = j >= mine ? expf((float)(lds.G[j] - G)) : 0.0f;
                    m2[t][x] *= d.scale * fade;
                    e2[t][x] = j > mine ? -lds.beta[j] * fade * e2[t][x] : 0.0f;
                }
            }
        // what the memory before gives and the one behind takes, and what the tokens of the block tell each other
        float at_end = 0.0f, dG = 0.0f;
        f32x4 here[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            here[t] = from_q[t] * (d.scale * since);
            to_k[t] *= until;
            dk[t] += to_k[t] - from_k[t] * (beta * since);
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 x1[3], y1[3], x2[3], y2[3];
            const bool before = 2 * s <= (int)wave, after = 2 * s + 1 >= (int)wave;
            split_rows<3>(m1[2 * s], m1[2 * s + 1], x1);
            split_rows<3>(e1[2 * s], e1[2 * s + 1], y1);
            split_rows<3>(m2[2 * s], m2[2 * s + 1], x2);
            split_rows<3>(e2[2 * s], e2[2 * s + 1], y2);
            bf16x8 a[2][n], b[2][n];
            lefts(lds.KT, c16, s * 32 + r8, a[0]);
            lefts(lds.QT, c16, s * 32 + r8, b[0]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if (t + 1 < kTiles) {
                    lefts(lds.KT, (t + 1) * 16 + c16, s * 32 + r8, a[(t + 1) % 2]);
                    lefts(lds.QT, (t + 1) * 16 + c16, s * 32 + r8, b[(t + 1) % 2]);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (before) {
                    here[t] = multiply<n, 3>(a[t % 2], x1, here[t]);
                    dk[t] = multiply<n, 3>(a[t % 2], y1, dk[t]);
                }
                if (after) {
                    dk[t] = multiply<n, 3>(b[t % 2], x2, dk[t]);
                    dk[t] = multiply<n, 3>(a[t % 2], y2, dk[t]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            dq[t] += here[t];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t c = t * 16 + r4 + x;
                float q = 0.0f, k = 0.0f;       // from their pieces, 0 where there is no token or column
#pragma unroll
                for (int p = 0; p < n; ++p) {
                    q += __uint_as_float((uint32_t)lds.QT[p][c][place(mine)] << 16);
                    k += __uint_as_float((uint32_t)lds.KT[p][c][place(mine)] << 16);
                }
                dG = fmaf(q, here[t][x], dG);
                at_end = fmaf(k, to_k[t][x], at_end);
            }
        }
        dG = of_token(dG);
        if (lane < 16) lds.dG[mine] = dG;
        float end = fmaf(expf((float)last), dot, at_end);
#pragma unroll
        for (int s = 1; s < 64; s *= 2) end += __shfl_xor(end, s);
        if (lane == 0) lds.end[wave] = end;
        __syncthreads();
        if (wave == 0) {
            float sum = lds.dG[lane] - lds.values[lane] + (lane == 63 ? lds.end[0] + lds.end[1] + lds.end[2] + lds.end[3] : 0.0f);
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const float after = __shfl_down(sum, s);
                if (lane + s < 64) sum += after;
            }
            if (lane < count) d.dg[row_of(lane) * d.lddg + head] = sum;
        }
    }
    if (!in) return;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const uint32_t c = t * 16 + r4;
        T *to_q = (T *)d.dq + row * d.lddq + hk * d.Dk + c, *to_k = (T *)d.dk + row * d.lddk + hk * d.Dk + c;
        if constexpr (kVec) {
            if (c >= d.Dk) continue;
            const float a[4] = {dq[t][0], dq[t][1], dq[t][2], dq[t][3]}, b[4] = {dk[t][0], dk[t][1], dk[t][2], dk[t][3]};
            dg_rows::store<T, 4>(to_q, a);
            dg_rows::store<T, 4>(to_k, b);
        } else
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (c + x < d.Dk) {
                    to_q[x] = (T)dq[t][x];
                    to_k[x] = (T)dk[t][x];
                }
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

template <class T, int KS>
void launch_size(const Delta &d, hipStream_t st)
{
    const uint64_t slots = d.first ? d.slots : d.n_seq * ((d.N / d.n_seq + kTokens - 1) / kTokens), units = slots * d.Hk;
    for (uint64_t from = 0; from < units; from += kMostLaunched) {
        const uint32_t grid = (uint32_t)(units - from < kMostLaunched ? units - from : kMostLaunched);
        if (d.vec_all && d.vec_out) delta_grad_kernel<T, KS, true><<<grid, 256, 0, st>>>(d, from);
        else delta_grad_kernel<T, KS, false><<<grid, 256, 0, st>>>(d, from);
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

void dg_delta::launch_slots(const Delta &d, hipStream_t st)
{
    if (d.first) delta_slots_kernel<<<(d.slots + 255) / 256, 256, 0, st>>>(d, const_cast<uint32_t *>(d.slot_seq));
}

void dg_delta::launch_gradients(const Delta &d, uint32_t dtype, hipStream_t st)
{
    if (dtype == DG_F32) launch_type<float>(d, st);
    else if (dtype == DG_F16) launch_type<f16>(d, st);
    else launch_type<bf16>(d, st);
}
