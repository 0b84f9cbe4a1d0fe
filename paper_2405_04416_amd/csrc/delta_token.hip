// The gated delta rule token by token: what a program calls that gets its tokens one after the other.
//
// Bound by memory: the memories go in and out once, 8 Dk Dv bytes per head and sequence (256 sequences of 16 heads of 128 x 128: 121 us, 4.5 TB/s).  A wavefront has 32 columns of a memory in registers, lane
// (r, c) rows 16 r to 16 r + 15 of columns 4 c to 4 c + 3; S^T k and S^T q are summed over r at once, as S'^T q = e^g S^T q + (k q) u.
#include "delta_chunk.h"

namespace {

using namespace dg_delta;

constexpr int kRows = kMaxD / 8;        // per lane

__device__ __forceinline__ float over_rows(float v)
{
    v += __shfl_xor(v, 8);
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

template <class T, bool kVec>
__device__ __forceinline__ void load_rows(const T *p, uint32_t from, uint32_t D, float (&out)[kRows])
{
    float half[8];
#pragma unroll
    for (int h = 0; h < kRows / 8; ++h) {
        eight<T, kVec>(p, from + h * 8, D, true, half);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[h * 8 + i] = half[i];
    }
}

template <class T, bool kVec>
__global__ void __launch_bounds__(256)
delta_token_kernel(Delta d, uint32_t groups, uint64_t units)
{
    const uint32_t lane = threadIdx.x % 64, r = lane / 8 * kRows;
    for (uint64_t unit = (uint64_t)blockIdx.x * 4 + threadIdx.x / 64; unit < units; unit += (uint64_t)gridDim.x * 4) {
        const uint32_t c = (uint32_t)(unit % groups) * 32 + lane % 8 * 4, head = (uint32_t)(unit / groups % d.H), seq = (uint32_t)(unit / groups / d.H);
        const uint32_t hk = head / (d.H / d.Hk);
        const Span span = span_of(d, seq);
        const uint64_t memory = ((uint64_t)seq * d.H + head) * d.Dk * d.Dv;
        float S[kRows][4];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const float *row = d.s0 + memory + (uint64_t)(r + i) * d.Dv + c;
            const bool in = d.s0 && r + i < d.Dk;
            if constexpr (kVec) {
                f32x4 v = {};
                if (in && c < d.Dv) v = *reinterpret_cast<const f32x4 *>(row);
#pragma unroll
                for (int x = 0; x < 4; ++x) S[i][x] = v[x];
            } else
#pragma unroll
                for (int x = 0; x < 4; ++x) S[i][x] = in && c + x < d.Dv ? row[x] : 0.0f;
        }
        for (uint32_t t = 0; t < span.len; ++t) {
            const uint64_t row = span.row(t);
            float k[kRows], q[kRows];
            load_rows<T, kVec>((const T *)d.k + row * d.ldk + hk * d.Dk, r, d.Dk, k);
            load_rows<T, kVec>((const T *)d.q + row * d.ldq + hk * d.Dk, r, d.Dk, q);
            const float a = expf(d.g[row * d.ldg + head]), beta = d.beta[row * d.ldb + head];
            float sk[4] = {}, sq[4] = {}, kq = 0.0f;
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                kq += k[i] * q[i];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    S[i][x] *= a;
                    sk[x] += S[i][x] * k[i];
                    sq[x] += S[i][x] * q[i];
                }
            }
            kq = over_rows(kq);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                sk[x] = over_rows(sk[x]);
                sq[x] = over_rows(sq[x]);
                const float v = c + x < d.Dv ? (float)((const T *)d.v)[row * d.ldv + head * d.Dv + c + x] : 0.0f, u = beta * (v - sk[x]);
#pragma unroll
                for (int i = 0; i < kRows; ++i) S[i][x] = fmaf(k[i], u, S[i][x]);
                if (r == 0 && c + x < d.Dv) ((T *)d.o)[row * d.ldo + head * d.Dv + c + x] = (T)(d.scale * fmaf(kq, u, sq[x]));
            }
        }
        if (!d.s_last) continue;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            float *row = d.s_last + memory + (uint64_t)(r + i) * d.Dv + c;
            if (r + i >= d.Dk) continue;
            if constexpr (kVec) {
                if (c < d.Dv) *reinterpret_cast<f32x4 *>(row) = (f32x4){S[i][0], S[i][1], S[i][2], S[i][3]};
            } else
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (c + x < d.Dv) row[x] = S[i][x];
        }
    }
}

template <class T>
void launch_type(const Delta &d, hipStream_t st)
{
    const uint32_t groups = (d.Dv + 31) / 32;
    const uint64_t units = (uint64_t)d.n_seq * d.H * groups, all = (units + 3) / 4;
    const uint32_t grid = (uint32_t)(all < 1u << 20 ? all : 1u << 20);
    if (d.vec_all && dg::aligned(d.s0, 16) && dg::aligned(d.s_last, 16)) delta_token_kernel<T, true><<<grid, 256, 0, st>>>(d, groups, units);
    else delta_token_kernel<T, false><<<grid, 256, 0, st>>>(d, groups, units);
}

}  // namespace

void dg_delta::launch_tokens(const Delta &d, uint32_t dtype, hipStream_t st)
{
    if (dtype == DG_F32) launch_type<float>(d, st);
    else if (dtype == DG_F16) launch_type<f16>(d, st);
    else launch_type<bf16>(d, st);
}
