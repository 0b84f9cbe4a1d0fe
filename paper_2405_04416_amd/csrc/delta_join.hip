// The gated delta rule, sequences in parts: from part to part.  S before the first part but one is what the first one leaves, E; then S' = M S + E.
// A workgroup has 16 columns of a head's memory, in LDS; M and E come from memory once.  Some 7 us a part (8 heads of 128 x 128), next to the 600 that a part of 16384 tokens takes.
#include "delta_chunk.h"

namespace {

using namespace dg_delta;

constexpr int kThreads = 512, kColumns = 16;         // a lane has a row of M and four columns

__global__ void __launch_bounds__(kThreads)
delta_join_kernel(Delta d, uint32_t groups, const float *before)
{
    __shared__ f32x4 lds[2][kMaxD][kColumns / 4];
    const uint32_t group = blockIdx.x % groups, head = blockIdx.x / groups % d.H, seq = blockIdx.x / groups / d.H, row = threadIdx.x / 4, four = threadIdx.x % 4;
    const uint32_t width = d.ends_width(), one = (d.Dv + 15) / 16 * 16, col = group * kColumns + four * 4;
    // The first part's beginning with the others': what the last one leaves may lie in its place
    for (uint32_t r = row; r < d.Dk; r += kThreads / 4)
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (col + x < d.Dv) {
                const uint64_t at = (((uint64_t)seq * d.H + head) * d.Dk + r) * d.Dv + col + x;
                d.starts[((((uint64_t)seq * d.parts) * d.H + head) * d.Dk + r) * d.Dv + col + x] = before ? before[at] : 0.0f;
            }
    for (uint32_t p = 0; p + 1 < d.parts; ++p) {
        const uint64_t at = (((uint64_t)seq * d.parts + p) * d.H + head) * d.Dk;
        const float *ends = d.ends + at * width;
        float *next = d.starts + (at + (uint64_t)d.H * d.Dk) * d.Dv;
        for (uint32_t r = row; r < d.Dk; r += kThreads / 4) {
            f32x4 sum = *reinterpret_cast<const f32x4 *>(ends + (uint64_t)r * width + col);
            if (p) {
                const float *m = ends + (uint64_t)r * width + one;
                f32x4 part[4] = {};
                for (uint32_t k0 = 0; k0 < d.Dk; k0 += 32) {
                    f32x4 v[8];                 // behind Dk the unit matrix has no columns: rows of 0 and results of 0; behind its sixteens nothing
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const f32x4 *>(m + (one + k0 + i * 4 < width ? k0 + i * 4 : 0));
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (k0 + i * 4 + x < d.Dk) part[x] += v[i][x] * lds[(p + 1) % 2][k0 + i * 4 + x][four];
                }
                sum += (part[0] + part[1]) + (part[2] + part[3]);
            }
            lds[p % 2][r][four] = sum;
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (col + x < d.Dv) next[(uint64_t)r * d.Dv + col + x] = sum[x];
        }
        __syncthreads();
    }
}

}  // namespace

size_t dg_delta::parts_bytes(uint64_t N, uint32_t n_seq, uint32_t H)
{
    const uint64_t heads = (uint64_t)n_seq * H;
    if (n_seq == 0 || heads * 3 > kUnits || N / n_seq < 3 * kLeastStretch) return 0;
    const uint64_t most = heads * kMostParts < kUnits ? heads * kMostParts : kUnits;
    return (size_t)most * kMaxD * 3 * kMaxD * sizeof(float);
}

void dg_delta::launch_join(const Delta &d, const float *before, hipStream_t st)
{
    const uint32_t groups = (d.Dv + kColumns - 1) / kColumns;
    delta_join_kernel<<<d.n_seq * d.H * groups, kThreads, 0, st>>>(d, groups, before);
}
