// Dropout whose mask is never stored: element i is dropped where 16 bits of the counter-based generator of the samplers,
// word offset + i / 4, field i % 4, are below round(65536 p).  The backward pass draws the same bits again.
#include <cmath>
#include "rows_common.h"
#include "sample_common.h"

namespace {

using namespace dg_rows;

constexpr int kBlock = 256;

// four elements, one word of the generator, per lane
template <class T, bool kResidual>
__global__ void __launch_bounds__(kBlock)
dropout_kernel(const T *__restrict__ x, const T *__restrict__ r, uint64_t n, uint32_t below, float scale, uint64_t seed, uint64_t offset, T *y)
{
    const uint64_t q = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const uint64_t bits = dg_sample::mix64(seed, offset + q);
    for (int k = 0; k < 4; ++k) {
        const uint64_t i = 4 * q + k;
        if (i >= n) return;
        // chosen, not multiplied by 0: a dropped infinity or NaN is dropped
        float v = ((bits >> (16 * k)) & 0xffffu) < below ? 0.0f : (float)x[i] * scale;
        if (kResidual) v += (float)r[i];
        y[i] = (T)v;
    }
}

template <class T>
void launch(const void *x, const void *r, uint64_t n, uint32_t below, float scale, uint64_t seed, uint64_t offset, void *y, hipStream_t st)
{
    const uint32_t grid = (uint32_t)(((n + 3) / 4 + kBlock - 1) / kBlock);
    if (r) dropout_kernel<T, true><<<grid, kBlock, 0, st>>>((const T *)x, (const T *)r, n, below, scale, seed, offset, (T *)y);
    else dropout_kernel<T, false><<<grid, kBlock, 0, st>>>((const T *)x, nullptr, n, below, scale, seed, offset, (T *)y);
}

int dropout(const char *who, const void *x, const void *r, uint64_t n, double p, uint64_t seed, uint64_t offset, uint32_t dtype, void *y, hipStream_t st)
{
    DG_REQUIRE(known_type(dtype), DG_ERR_ARG, "%s: unknown element type %u", who, dtype);
    DG_REQUIRE(p >= 0.0 && p <= 1.0, DG_ERR_ARG, "%s: p must lie in [0, 1]", who);
    if (n == 0) return DG_OK;
    const size_t item = item_bytes(dtype);
    DG_REQUIRE(x && y && dg::aligned(x, item) && dg::aligned(y, item) && dg::aligned(r, item), DG_ERR_ARG, "%s: null or misaligned pointer", who);
    DG_REQUIRE(n <= 1ull << 40, DG_ERR_UNSUPPORTED, "%s: n too large for one launch", who);
    const uint32_t below = (uint32_t)std::floor(p * 65536.0 + 0.5);
    const float scale = below == 65536u ? 0.0f : (float)(65536.0 / (65536u - below));
    (dtype == DG_F32 ? launch<float> : dtype == DG_F16 ? launch<f16> : launch<bf16>)(x, r, n, below, scale, seed, offset, y, st);
    return dg::launch_status(who);
}

}  // namespace

extern "C" int dg_dropout_fwd(const void *x, const void *residual, uint64_t n, double p, uint64_t seed, uint64_t offset, uint32_t dtype, void *y,
                              void *stream)
{
    return dropout("dg_dropout_fwd", x, residual, n, p, seed, offset, dtype, y, (hipStream_t)stream);
}

extern "C" int dg_dropout_bwd(const void *dy, uint64_t n, double p, uint64_t seed, uint64_t offset, uint32_t dtype, void *dx, void *stream)
{
    return dropout("dg_dropout_bwd", dy, nullptr, n, p, seed, offset, dtype, dx, (hipStream_t)stream);
}
