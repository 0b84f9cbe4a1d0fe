// The gated delta rule: T and P of all chunks of 32 tokens (delta_chunk.h), a workgroup of two wavefronts for each chunk and head, one for T, one for P.
//   T = (1 + A)^-1 of 32 rows: the two diagonal blocks of 16 by substitution, row by row in the lanes' registers, the block below as -T22 A21 T11.
// Forward A has beta of its columns (T gives what tokens miss, Y), backward of its rows (T^T gives dR): so neither divides by a rate, which may be 0.
// Operands come straight from memory and results go straight to the workspace; only the small blocks pass through LDS.  Bound by the substitution, 16 rows that wait for each other, and by
// memory, 16 KB that every chunk and head leaves and as much that it reads: 65536 tokens x 8 heads of 128 150 us (3.8 TB/s).
#include "delta_chunk.h"

namespace {

using namespace dg_delta;

// four values side by side, in pieces, to the workspace
__device__ __forceinline__ void put4(const float (&v)[4], uint16_t (*rows)[kChunk][kPitch], uint32_t row, uint32_t col)
{
    uint32_t w[3][2];
    split<3, 4>(v, w);
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x2 *>(&rows[p][line(row)][col]) = (u32x2){w[p][0], w[p][1]};
}

struct Shared {
    double G[2][kChunk];
    float beta[kChunk];
    float A[2][16][20], inverse[2][16][20];     // A^T and T of the diagonal blocks
};

// 16 rows of K or Q as an operand, in pieces
template <class T, int KS, bool kVec>
struct Block {
    static constexpr int n = Pieces<T>::n;
    bf16x8 v[KS][n];
    __device__ __forceinline__ Block(const T *p, uint64_t ld, const Span &span, uint32_t t0, uint32_t t, uint32_t c8, uint32_t D)
    {
        const bool in = t0 + t < span.len;
        const T *row = p + span.row(in ? t0 + t : t0) * ld;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            float x[8];
            eight<T, kVec>(row, s * 32 + c8, D, in, x);
            split8<n>(x, v[s]);
        }
    }
};

template <class T, int KS, bool kVec>
__device__ __forceinline__ f32x4 product(const Block<T, KS, kVec> &a, const Block<T, KS, kVec> &b)
{
    f32x4 acc = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) acc = multiply(a.v[s], b.v[s], acc);
    return acc;
}

template <class T, int KS, bool kBackward, bool kVec>
__global__ void __launch_bounds__(128)
delta_weights_kernel(Delta d, uint64_t from)
{
    __shared__ Shared lds;
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), c16 = lane % 16, r4 = lane / 16 * 4;
    const uint64_t unit = from + blockIdx.x;
    const uint32_t head = (uint32_t)(unit % d.H), group = d.H / d.Hk, hk = head / group;
    uint64_t slot = unit / d.H;
    uint32_t seq, c;
    if (d.first) {
        seq = d.chunk_seq[slot];
        if (seq >= d.n_seq) return;
    } else {
        const uint64_t each = (d.N / d.n_seq + kChunk - 1) / kChunk;
        seq = (uint32_t)(slot / each);
        c = (uint32_t)(slot % each);
    }
    const Span span = span_of(d, seq);
    if (d.first) c = (uint32_t)(slot - first_chunk(span, seq));
    else slot = first_chunk(span, seq) + c;
    const uint32_t t0 = c * kChunk;
    if (t0 >= span.len) return;

    Weights &out = d.weights[slot * d.H + head];
    const uint32_t mine = lane % kChunk;
    const bool held = t0 + mine < span.len;
    const uint64_t row = span.row(held ? t0 + mine : t0);
    const float gate = d.g[row * d.ldg + head], rate = d.beta[row * d.ldb + head];
    const T *keys = (const T *)d.k + hk * d.Dk, *queries = (const T *)d.q + hk * d.Dk;
    const Block<T, KS, kVec> k0(keys, d.ldk, span, t0, c16, r4 * 2, d.Dk), k1(keys, d.ldk, span, t0, 16 + c16, r4 * 2, d.Dk);
    const float beta = held ? rate : 0.0f;
    double sum = held ? (double)cut_off(gate) : 0.0;
#pragma unroll
    for (int s = 1; s < kChunk; s *= 2) {
        const double before = __shfl_up(sum, s, kChunk);
        if (mine >= (uint32_t)s) sum += before;
    }
    const double last = __shfl(sum, kChunk - 1, kChunk);
    double *G = lds.G[wave];                    // each wavefront has its own, so that none waits for the other
    if (lane < kChunk) {
        G[lane] = sum;
        if (wave == 0) {
            const float since = expf((float)sum);
            lds.beta[lane] = beta;
            out.beta[lane] = beta;
            out.read[lane] = kBackward ? beta * since : since;
            out.query[lane] = d.scale * since;
            out.until[lane] = expf((float)(last - sum));
            if (lane == 0) out.whole = expf((float)last);
        }
    }
    wave_fence();
    const float none[4] = {};
    if (wave == 1) {
        // P; forward rows i, backward rows j
        const Block<T, KS, kVec> q0(queries, d.ldq, span, t0, c16, r4 * 2, d.Dk), q1(queries, d.ldq, span, t0, 16 + c16, r4 * 2, d.Dk);
#pragma unroll
        for (int b = 0; b < 3; ++b) {           // blocks (tokens i, tokens j): (0, 0), (1, 0), (1, 1)
            const uint32_t bi = b ? 16 : 0, bj = b == 2 ? 16 : 0;
            const Block<T, KS, kVec> &q = b ? q1 : q0, &k = b == 2 ? k1 : k0;
            const f32x4 acc = kBackward ? product(q, k) : product(k, q);
            float v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t i = bi + (kBackward ? r4 + x : c16), j = bj + (kBackward ? c16 : r4 + x);
                v[x] = i >= j ? d.scale * acc[x] * expf((float)(G[i] - G[j])) : 0.0f;
            }
            if (kBackward) put4(v, out.P, bj + c16, bi + r4);
            else put4(v, out.P, bi + c16, bj + r4);
        }
        put4(none, out.P, kBackward ? 16 + c16 : c16, kBackward ? r4 : 16 + r4);
    } else {
        put4(none, out.inverse, kBackward ? 16 + c16 : c16, kBackward ? r4 : 16 + r4);
        // A: the diagonal blocks to LDS, the other stays as an operand
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const f32x4 acc = b ? product(k1, k1) : product(k0, k0);
            f32x4 v;
#pragma unroll
            for (int x = 0; x < 4; ++x) {       // A[r4 + x, c16]
                const uint32_t i = b * 16 + r4 + x, j = b * 16 + c16;
                v[x] = i > j ? lds.beta[kBackward ? i : j] * acc[x] * expf((float)(G[i] - G[j])) : 0.0f;
            }
            *reinterpret_cast<f32x4 *>(&lds.A[b][c16][r4]) = v;
        }
        f32x4 a21;
        {
            // forward: rows i, columns j; backward: rows j, columns i
            const f32x4 acc = kBackward ? product(k0, k1) : product(k1, k0);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t i = 16 + (kBackward ? c16 : r4 + x), j = kBackward ? r4 + x : c16;
                a21[x] = lds.beta[kBackward ? i : j] * acc[x] * expf((float)(G[i] - G[j]));
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
                const f32x4 a = *reinterpret_cast<const f32x4 *>(&lds.A[block][j][m4]);
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (m4 + x > j) sum = fmaf(t[m4 + x], a[x], sum);
            }
            t[j] = (j == (int)c16 ? 1.0f : 0.0f) - sum;
        }
        if (lane < 32)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float v[4] = {t[j], t[j + 1], t[j + 2], t[j + 3]};
                *reinterpret_cast<f32x4 *>(&lds.inverse[block][c16][j]) = (f32x4){v[0], v[1], v[2], v[3]};
                if (!kBackward) put4(v, out.inverse, block * 16 + c16, block * 16 + j);
            }
        wave_fence();
        if (kBackward && lane < 32)             // rows of T^T
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float v[4] = {lds.inverse[block][j][c16], lds.inverse[block][j + 1][c16], lds.inverse[block][j + 2][c16], lds.inverse[block][j + 3][c16]};
                put4(v, out.inverse, block * 16 + c16, block * 16 + j);
            }
        // the block below the diagonal in fp32: forward as its transpose (A21^T T22^T, then T11^T times that), so that a lane has four values of a row
        // of what is stored in either case
        const f32x4 t22 = *reinterpret_cast<const f32x4 *>(&lds.inverse[1][c16][r4]);
        f32x4 w = {}, x = {};
        float t11[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) t11[s] = lds.inverse[0][r4 + s][c16];
#pragma unroll
        for (int s = 0; s < 4; ++s) w = __builtin_amdgcn_mfma_f32_16x16x4f32(a21[s], kBackward ? t11[s] : t22[s], w, 0, 0, 0);
#pragma unroll
        for (int s = 0; s < 4; ++s) x = __builtin_amdgcn_mfma_f32_16x16x4f32(kBackward ? t22[s] : t11[s], w[s], x, 0, 0, 0);
        const float v[4] = {-x[0], -x[1], -x[2], -x[3]};
        // forward: lane i, values j; backward: lane j, values i
        if (kBackward) put4(v, out.inverse, c16, 16 + r4);
        else put4(v, out.inverse, 16 + c16, r4);
    }
}

template <class T, int KS, bool kBackward>
void launch_size(const Delta &d, hipStream_t st)
{
    const uint64_t slots = d.first ? chunk_slots(d.N, d.n_seq) : d.n_seq * ((d.N / d.n_seq + kChunk - 1) / kChunk), units = slots * d.H;
    for (uint64_t from = 0; from < units; from += kMostLaunched) {
        const uint32_t grid = (uint32_t)(units - from < kMostLaunched ? units - from : kMostLaunched);
        if (d.vec_keys) delta_weights_kernel<T, KS, kBackward, true><<<grid, 128, 0, st>>>(d, from);
        else delta_weights_kernel<T, KS, kBackward, false><<<grid, 128, 0, st>>>(d, from);
    }
}

template <class T>
void launch_type(const Delta &d, bool backward, hipStream_t st)
{
    if (d.Dk <= 32) backward ? launch_size<T, 1, true>(d, st) : launch_size<T, 1, false>(d, st);
    else if (d.Dk <= 64) backward ? launch_size<T, 2, true>(d, st) : launch_size<T, 2, false>(d, st);
    else backward ? launch_size<T, 4, true>(d, st) : launch_size<T, 4, false>(d, st);
}

// The sequence of each chunk's slot, ~0 where it is empty: the last sequence whose slots begin at or before it, if it has so many.
__global__ void __launch_bounds__(256)
delta_chunks_kernel(Delta d, uint32_t slots, uint32_t *chunk_seq)
{
    const uint32_t slot = blockIdx.x * 256 + threadIdx.x;
    if (slot >= slots) return;
    uint32_t low = 0, high = d.n_seq;               // slots of sequence `low` begin at or before this one, those of `high` behind it
    while (high - low > 1) {
        const uint32_t mid = low + (high - low) / 2;
        if (first_chunk(span_of(d, mid), mid) <= slot) low = mid;
        else high = mid;
    }
    const Span span = span_of(d, low);
    const uint64_t begin = first_chunk(span, low);
    chunk_seq[slot] = begin <= slot && (slot - begin) * kChunk < span.len ? low : ~0u;
}

}  // namespace

size_t dg_delta::weight_bytes(uint64_t N, uint32_t n_seq, uint32_t H) { return chunk_slots(N, n_seq) * H * sizeof(Weights); }
size_t dg_delta::chunk_bytes(uint64_t N, uint32_t n_seq) { return (chunk_slots(N, n_seq) * 4 + 15) / 16 * 16; }

void dg_delta::launch_weights(const Delta &d, uint32_t dtype, bool backward, hipStream_t st)
{
    if (d.first) {
        const uint32_t slots = (uint32_t)chunk_slots(d.N, d.n_seq);
        delta_chunks_kernel<<<(slots + 255) / 256, 256, 0, st>>>(d, slots, const_cast<uint32_t *>(d.chunk_seq));
    }
    if (dtype == DG_F32) launch_type<float>(d, backward, st);
    else if (dtype == DG_F16) launch_type<f16>(d, backward, st);
    else launch_type<bf16>(d, backward, st);
}
