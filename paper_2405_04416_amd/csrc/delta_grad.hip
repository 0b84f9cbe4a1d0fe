// The gated delta rule, backward, what follows from the memories S before and the gradients dS' behind each 64 tokens, and from what the tokens miss (Y = v - S^T k)
// and the gradient dR of what they write (U = beta Y): with X = scale D (dO U^T) up to the diagonal, Z = -beta D (dR U^T) below it, D and G of the 64 tokens,
//   dq = scale e^G dO S^T + X K,    dk = -beta e^G dR S^T + e^(G[last] - G) U dS'^T + X^T Q + Z K + Z^T K,    dv = beta dR,   dbeta = dR Y.
// With e^-G S for a memory the rule has no decay, values e^-G v and results e^G o: so dG = o do - v dv = q dq - v dv, and dG[last] also the product of the memory
// behind, e^G[last] S + K^T e^(G[last] - G) U, with dS';  dg[t] = sum of dG from t on, up to the next gate that keeps nothing.
//
// A workgroup takes 64 tokens of a key head, one value head after the other, 32 columns of values at a time through LDS (in pieces, cut once for all), a wavefront
// 16 tokens and half of the columns of keys: a lane has a token, of which everything above is a column of a product.  X and Z are made once, block by block,
// and go through LDS, from which reads that transpose take them, K and Q by columns too.
// Bound by memory first (memories, gradients and what tokens miss and write are fp32: 2 x 8192 tokens x 16 heads of 128 x 128, bf16, 0.38 ms for some 1.3 GB, 3.4 TB/s), then by cutting into pieces and LDS, which
// do not all hide behind it: vector units 31 % of the time busy, matrix units 20.  2003 ragged sequences x 3 heads of 24 x 40, fp32, 0.34 ms.
#include "delta_chunk.h"
#include "rows_vectors.h"

namespace {

using namespace dg_delta;

constexpr int kTokens = kMark, kTokenPitch = kTokens + 8, kColumns = 32, kColumnPitch = kColumns + 8, kWaves = 8, kThreads = kWaves * 64;

// 32 columns of values at a time
template <class T, int KS>
struct Values {
    uint16_t S[3][32 * KS][kColumnPitch], dS[3][32 * KS][kColumnPitch], U[3][kTokens][kColumnPitch], R[3][kTokens][kColumnPitch], O[Pieces<T>::n][kTokens][kColumnPitch];
};

// X and Z: row i, columns j
struct Pulls { uint16_t X[3][kTokens][kTokenPitch], Z[3][kTokens][kTokenPitch]; };

// K or Q
template <class T, int KS>
struct Turned { uint16_t rows[Pieces<T>::n][kTokens][32 * KS + 8]; };

struct Tokens {
    double G[kTokens];
    float beta[kTokens], dG[2][kTokens], values[kTokens], end[kWaves];
};

// K and Q both stay if there is room; otherwise they come one after the other for every head
template <class T, int KS>
constexpr bool kTogether = (sizeof(Values<T, KS>) > sizeof(Pulls) ? sizeof(Values<T, KS>) : sizeof(Pulls)) + 2 * sizeof(Turned<T, KS>) + sizeof(Tokens) <= 160 * 1024;

template <class T, int KS, bool kBoth>
struct Shared : Tokens {
    union {
        Values<T, KS> value;
        struct { Pulls pull; Turned<T, KS> turned[1]; };
    };
};
template <class T, int KS>
struct Shared<T, KS, true> : Tokens {
    union { Values<T, KS> value; Pulls pull; };
    Turned<T, KS> turned[2];
};

// sum over the four lanes that have a token
__device__ __forceinline__ float of_token(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// W values from an address on that the workgroup shares and a lane's distance in bytes; `left` of them are a row's, the others are whatever comes instead: `cleared`
// tells them apart when they are used, so that nothing waits for the load.
template <class T, int W, bool kVec>
__device__ __forceinline__ void ahead(const T *base, uint32_t bytes, int left, dg_rows::Pack<T, W> &out)
{
    constexpr int m = 16 / sizeof(T) < W ? 16 / sizeof(T) : W;
    if constexpr (kVec) {
#pragma unroll
        for (int h = 0; h < W / m; ++h) {
            const dg_rows::Pack<T, m> p = *reinterpret_cast<const dg_rows::Pack<T, m> *>((const char *)base + (h * m < left ? bytes + h * m * (uint32_t)sizeof(T) : 0u));
#pragma unroll
            for (int i = 0; i < m; ++i) out.v[h * m + i] = p.v[i];
        }
    } else
#pragma unroll
        for (int i = 0; i < W; ++i) out.v[i] = *reinterpret_cast<const T *>((const char *)base + (i < left ? bytes + i * (uint32_t)sizeof(T) : 0u));
}

template <class T, int W>
__device__ __forceinline__ void cleared(const dg_rows::Pack<T, W> &p, uint32_t c, uint32_t D, bool in, float (&out)[W])
{
#pragma unroll
    for (int i = 0; i < W; ++i) out[i] = in && c + i < D ? (float)p.v[i] : 0.0f;
}

template <bool kNear = true, int n, int rows, int pitch>
__device__ __forceinline__ void put4(const float (&v)[4], uint16_t (&to)[n][rows][pitch], uint32_t row, uint32_t col)
{
    uint32_t w[n][2];
    split<n, 4, kNear>(v, w);
#pragma unroll
    for (int p = 0; p < n; ++p) *reinterpret_cast<u32x2 *>(&to[p][row][col]) = (u32x2){w[p][0], w[p][1]};
}

// K or Q from the block's lowest row on; at(t): how many rows behind it token t is
template <class T, int KS, bool kVec, class At>
__device__ __forceinline__ void turn(const T *K, uint32_t ld, uint32_t Dk, uint32_t count, At at, Turned<T, KS> &to)
{
    constexpr int n = Pieces<T>::n, kEach = KS > 2 ? KS / 2 : 1;        // of a thread, if it has any
    // rows are loaded as they lie
    auto token = [](int i) { return (i * kThreads + threadIdx.x) / (4 * KS); };
    const uint32_t col = threadIdx.x % (4 * KS) * 8;
    if (token(0) >= kTokens) return;
    dg_rows::Pack<T, 8> x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) ahead<T, 8, kVec>(K, (at(token(i)) * ld + col) * (uint32_t)sizeof(T), (int)Dk - (int)col, x[i]);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t t = token(i);
        float v[8];
        uint32_t w[n][4];
        cleared<T, 8>(x[i], col, Dk, t < count, v);
        split<n, 8>(v, w);
#pragma unroll
        for (int p = 0; p < n; ++p) *reinterpret_cast<u32x4 *>(&to.rows[p][t][col]) = (u32x4){w[p][0], w[p][1], w[p][2], w[p][3]};
    }
}

template <class T, int KS, bool kVec>
__global__ void __launch_bounds__(kThreads)
delta_grad_kernel(Delta d, uint64_t from)
{
    __shared__ alignas(16) Shared<T, KS, kTogether<T, KS>> lds;
    constexpr int n = Pieces<T>::n, kTiles = KS, kMemoryRows = KS > 2 ? KS / 2 : 1;     // results of 16 columns of keys of a wavefront; rows of the memory of a thread, if it has any
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64 % 4), half = __builtin_amdgcn_readfirstlane(threadIdx.x / 256), key0 = half * 16 * KS;
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
    // rows as distances from the lowest of the block: up to 63 rows of less than 2^24 values
    const uint64_t lowest = span.turn ? span.begin + (span.len - t0 - count) : span.begin + t0;
    auto behind = [&](uint32_t t) { return t >= count ? 0u : span.turn ? count - 1 - t : t; };
    auto row_of = [&](uint32_t t) { return lowest + behind(t); };
    const T *K = (const T *)d.k + lowest * d.ldk + hk * d.Dk, *Q = (const T *)d.q + lowest * d.ldq + hk * d.Dk;

    constexpr bool kBoth = kTogether<T, KS>;
    if constexpr (kBoth) {
        turn<T, KS, kVec>(K, (uint32_t)d.ldk, d.Dk, count, behind, lds.turned[0]);
        turn<T, KS, kVec>(Q, (uint32_t)d.ldq, d.Dk, count, behind, lds.turned[1]);
    }
    // X and Z are made of ten blocks of 16 x 16 on and below the diagonal: one for each wavefront, another for the first two
    const uint32_t blocks = threadIdx.x < 128 ? 2 : 1;
    const uint32_t all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    auto block_row = [&](uint32_t i) -> uint32_t { return all_waves + 8 * i < 1 ? 0 : all_waves + 8 * i < 3 ? 1 : all_waves + 8 * i < 6 ? 2 : 3; };
    auto block_column = [&](uint32_t i) -> uint32_t { return all_waves + 8 * i - block_row(i) * (block_row(i) + 1) / 2; };
    const uint32_t bi[2] = {block_row(0), block_row(1)}, bj[2] = {block_column(0), block_column(1)};
    f32x4 dq[kTiles] = {}, dk[kTiles] = {};

    for (uint32_t h = 0; h < group; ++h) {
        const uint32_t head = hk * group + h;
        const uint32_t thread = again(threadIdx.x), lane = thread % 64, c16 = lane % 16, r4 = lane / 16 * 4, r8 = lane / 16 * 8;
        const uint32_t mine = wave * 16 + c16;              // the token that a lane has as a column
        // A thread brings four columns of rows b, b + 64 of the memory and its gradient, and of token b: eight threads a line
        const uint32_t b = thread / 8, c4 = thread % 8 * 4;
        const uint64_t brought_row = row_of(b);
        const bool there = b < count;
        const uint32_t ldf = d.H * d.Dv;
        uint32_t at_s[kMemoryRows];
#pragma unroll
        for (int i = 0; i < kMemoryRows; ++i) at_s[i] = ((b + i * 64 < d.Dk ? b + i * 64 : 0) * d.Dv + c4) * 4;
        const uint32_t at_f = (behind(b) * ldf + c4) * 4, at_o = (behind(b) * (uint32_t)d.lddo + c4) * (uint32_t)sizeof(T), at_v = (behind(b) * (uint32_t)d.ldv + c4) * (uint32_t)sizeof(T);
        const float *S = d.marks + ((uint64_t)slot * d.H + head) * d.Dk * d.Dv, *dS = d.dmarks + ((uint64_t)slot * d.H + head) * d.Dk * d.Dv;
        dg_rows::Pack<float, 4> next_s[kMemoryRows], next_ds[kMemoryRows], next_y, next_r;
        dg_rows::Pack<T, 4> next_o, next_v;
        const float *Y = d.y + lowest * ldf + head * d.Dv, *R = d.dr + lowest * ldf + head * d.Dv;
        const T *O = (const T *)d.dout + lowest * d.lddo + head * d.Dv, *V = (const T *)d.v + lowest * d.ldv + head * d.Dv;
        auto fetch = [&](uint32_t c0) {
            const int left = (int)d.Dv - (int)(c0 + c4);
#pragma unroll
            for (int i = 0; i < kMemoryRows; ++i) {
                ahead<float, 4, kVec>(S + c0, at_s[i], left, next_s[i]);
                ahead<float, 4, kVec>(dS + c0, at_s[i], left, next_ds[i]);
            }
            ahead<float, 4, kVec>(Y + c0, at_f, left, next_y);
            ahead<float, 4, kVec>(R + c0, at_f, left, next_r);
            ahead<T, 4, kVec>(O + c0, at_o, left, next_o);
            ahead<T, 4, kVec>(V + c0, at_v, left, next_v);
        };
        fetch(0);
        const float rate = there ? d.beta[brought_row * d.ldb + head] : 0.0f;
        uint64_t shut = 0;                              // tokens whose gates keep nothing
        __syncthreads();                                // what the last head left in LDS has been read
        if (thread < 64) {
            const bool held = lane < count;
            const uint64_t r = row_of(lane);
            const float value = d.g[r * d.ldg + head], b = d.beta[r * d.ldb + head];
            double G = held ? (double)cut_off(value) : 0.0;
            shut = __ballot(held && keeps_nothing(value));
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const double before = __shfl_up(G, s);
                if (lane >= (uint32_t)s) G += before;
            }
            lds.G[lane] = G;
            lds.beta[lane] = held ? b : 0.0f;
        }
        f32x4 from_q[kTiles] = {}, from_k[kTiles] = {}, to_k[kTiles] = {};          // dO S^T, dR S^T, U dS'^T
        f32x4 m[2] = {}, e[2] = {};                                                 // dO U^T, dR U^T of the wavefront's blocks: lane i, rows j
        float dbeta = 0.0f, values = 0.0f, dot = 0.0f;
#pragma unroll 1
        for (uint32_t c0 = 0; c0 < d.Dv; c0 += kColumns) {
            {
                const uint32_t c = c0 + c4;
                float x[4], y[4], r[4], out[4];
#pragma unroll
                for (int i = 0; i < kMemoryRows; ++i) {
                    const uint32_t to = b + i * 64;
                    if (to >= 32 * KS) continue;
                    cleared<float, 4>(next_s[i], c, d.Dv, to < d.Dk, x);
                    put4(x, lds.value.S, to, c4);
                    cleared<float, 4>(next_ds[i], c, d.Dv, to < d.Dk, y);
                    put4(y, lds.value.dS, to, c4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) dot = fmaf(x[j], y[j], dot);
                }
                cleared<float, 4>(next_r, c, d.Dv, there, r);
                put4(r, lds.value.R, b, c4);
                cleared<float, 4>(next_y, c, d.Dv, there, y);
                cleared<T, 4>(next_v, c, d.Dv, there, x);
                T *dv = (T *)d.dv + brought_row * d.lddv + head * d.Dv + c;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dbeta = fmaf(r[j], y[j], dbeta);
                    y[j] *= rate;
                    out[j] = rate * r[j];
                    values = fmaf(out[j], x[j], values);
                    if (!kVec && there && c + j < d.Dv) dv[j] = (T)out[j];
                }
                if (kVec && there && c < d.Dv) dg_rows::store<T, 4>(dv, out);
                put4(y, lds.value.U, b, c4);
                cleared<T, 4>(next_o, c, d.Dv, there, x);
                put4(x, lds.value.O, b, c4);
            }
            __syncthreads();
            if (c0 + kColumns < d.Dv) fetch(c0 + kColumns);
            bf16x8 o[n], r[3], u[3], a[3];
            lefts(lds.value.O, mine, r8, o);
            lefts(lds.value.R, mine, r8, r);
            lefts(lds.value.U, mine, r8, u);
            // one tile's operands on their way while another's are multiplied, and no more, for which there would not be registers
            bf16x8 s2[2][3], ds2[2][3];
            lefts(lds.value.S, key0 + c16, r8, s2[0]);
            lefts(lds.value.dS, key0 + c16, r8, ds2[0]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if (t + 1 < kTiles) {
                    lefts(lds.value.S, key0 + (t + 1) * 16 + c16, r8, s2[(t + 1) % 2]);
                    lefts(lds.value.dS, key0 + (t + 1) * 16 + c16, r8, ds2[(t + 1) % 2]);
                }
                __builtin_amdgcn_sched_barrier(0);
                from_q[t] = multiply<3, n>(s2[t % 2], o, from_q[t]);
                from_k[t] = multiply<3, 3>(s2[t % 2], r, from_k[t]);
                to_k[t] = multiply<3, 3>(ds2[t % 2], u, to_k[t]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                if (i >= (int)blocks) continue;
                lefts(lds.value.U, bj[i] * 16 + c16, r8, a);
                lefts(lds.value.O, bi[i] * 16 + c16, r8, o);
                lefts(lds.value.R, bi[i] * 16 + c16, r8, r);
                m[i] = multiply<3, n>(a, o, m[i]);
                e[i] = multiply<3, 3>(a, r, e[i]);
            }
            __syncthreads();
        }
        dbeta = dg_rows::group_sum<8>(dbeta);
        values = dg_rows::group_sum<8>(values);
        if (thread % 8 == 0) {
            lds.values[b] = values;
            if (there) d.dbeta[brought_row * d.lddb + head] = dbeta;
        }
        const double G = lds.G[mine], last = lds.G[kTokens - 1];
        const float since = expf((float)G), until = expf((float)(last - G)), beta = lds.beta[mine];
        if constexpr (!kBoth) turn<T, KS, kVec>(K, (uint32_t)d.ldk, d.Dk, count, behind, lds.turned[0]);
        // X and Z
        float x[2][4];
        const float none[4] = {};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k >= (int)blocks) continue;
            const uint32_t i = bi[k] * 16 + c16, j0 = bj[k] * 16 + r4;
            const double Gi = lds.G[i];
            const float rate_i = lds.beta[i];
            float z[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const float fade = j0 + y <= i ? expf((float)(Gi - lds.G[j0 + y])) : 0.0f;
                x[k][y] = d.scale * fade * m[k][y];
                z[y] = j0 + y < i ? -rate_i * fade * e[k][y] : 0.0f;
            }
            put4<(n > 1)>(x[k], lds.pull.X, i, j0);
            put4<(n > 1)>(z, lds.pull.Z, i, j0);
        }
        // the blocks behind the diagonal that are multiplied with
        if (half == 1 && wave < 2) {
            put4<(n > 1)>(none, lds.pull.X, wave * 32 + c16, wave * 32 + 16 + r4);
            put4<(n > 1)>(none, lds.pull.Z, wave * 32 + c16, wave * 32 + 16 + r4);
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
            bf16x8 x1[3], z1[3], z2[3], a[2][n];
            const bool before = 2 * s <= (int)wave, after = 2 * s + 1 >= (int)wave;
            lefts(lds.pull.X, mine, s * 32 + r8, x1);
            lefts(lds.pull.Z, mine, s * 32 + r8, z1);
            columns(lds.pull.Z, s * 32, wave * 16, lane, z2);
            columns(lds.turned[0].rows, s * 32, key0, lane, a[0]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if (t + 1 < kTiles) columns(lds.turned[0].rows, s * 32, key0 + (t + 1) * 16, lane, a[(t + 1) % 2]);
                __builtin_amdgcn_sched_barrier(0);
                if (before) {
                    here[t] = multiply<n, 3>(a[t % 2], x1, here[t]);
                    dk[t] = multiply<n, 3>(a[t % 2], z1, dk[t]);
                }
                if (after) dk[t] = multiply<n, 3>(a[t % 2], z2, dk[t]);
            }
        }
        auto dot_tokens = [&](const uint16_t (&rows)[n][kTokens][32 * KS + 8], const f32x4 (&with)[kTiles]) {
            float sum = 0.0f;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                float value[4] = {};                // from its pieces, 0 where there is no token or column
#pragma unroll
                for (int p = 0; p < n; ++p) {
                    const u32x2 w = *reinterpret_cast<const u32x2 *>(&rows[p][mine][key0 + t * 16 + r4]);
#pragma unroll
                    for (int y = 0; y < 4; ++y) value[y] += __uint_as_float(y % 2 ? w[y / 2] & 0xffff0000u : w[y / 2] << 16);
                }
#pragma unroll
                for (int y = 0; y < 4; ++y) sum = fmaf(value[y], with[t][y], sum);
            }
            return sum;
        };
        at_end = dot_tokens(lds.turned[0].rows, to_k);
        if constexpr (!kBoth) {
            __syncthreads();
            turn<T, KS, kVec>(Q, (uint32_t)d.ldq, d.Dk, count, behind, lds.turned[0]);
            __syncthreads();
        }
        auto &queries = lds.turned[kBoth ? 1 : 0].rows;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 x2[3], a[2][n];
            const bool after = 2 * s + 1 >= (int)wave;
            columns(lds.pull.X, s * 32, wave * 16, lane, x2);
            columns(queries, s * 32, key0, lane, a[0]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if (t + 1 < kTiles) columns(queries, s * 32, key0 + (t + 1) * 16, lane, a[(t + 1) % 2]);
                __builtin_amdgcn_sched_barrier(0);
                if (after) dk[t] = multiply<n, 3>(a[t % 2], x2, dk[t]);
            }
        }
        dG = dot_tokens(queries, here);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) dq[t] += here[t];
        dG = of_token(dG);
        if (lane < 16) lds.dG[half][mine] = dG;
        float end = fmaf(expf((float)last), dot, at_end);
#pragma unroll
        for (int s = 1; s < 64; s *= 2) end += __shfl_xor(end, s);
        if (lane == 0) lds.end[thread / 64] = end;
        __syncthreads();
        if (thread < 64) {
            float sum = lds.dG[0][lane] + lds.dG[1][lane] - lds.values[lane];
            if (lane == 63)
#pragma unroll
                for (int w = 0; w < kWaves; ++w) sum += lds.end[w];
            // up to the next gate that keeps nothing
            const uint64_t later = lane < 63 ? shut >> (lane + 1) : 0;
            const uint32_t end = later ? lane + 1 + __builtin_ctzll(later) : 64;
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const float after = __shfl_down(sum, s);
                if (lane + s < end) sum += after;
            }
            if (lane < count) d.dg[row_of(lane) * d.lddg + head] = shut >> lane & 1 ? 0.0f : sum;
        }
    }
    const uint32_t mine = wave * 16 + threadIdx.x % 16, r4 = threadIdx.x % 64 / 16 * 4;
    const uint64_t row = row_of(mine);
    if (mine >= count) return;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const uint32_t c = key0 + t * 16 + r4;
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
        if (d.vec_all && d.vec_out) delta_grad_kernel<T, KS, true><<<grid, kThreads, 0, st>>>(d, from);
        else delta_grad_kernel<T, KS, false><<<grid, kThreads, 0, st>>>(d, from);
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
