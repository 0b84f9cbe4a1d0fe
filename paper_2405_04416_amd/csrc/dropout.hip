// Dropout whose mask is never stored: element i is dropped where 16 bits of the counter-based generator of the samplers,
// word offset + i / 4, field i % 4, are below round(65536 p).  The backward pass draws the same bits again.
#include <cmath>
#include "rows_common.h"
#include "sample_common.h"

namespace {

using namespace dg_rows;

constexpr int kBlock = 256;

struct Drop {
    const void *x, *r;
    void *y;
    uint64_t n, seed, offset;
    uint32_t below;
    float scale;
};

// value k of the four that share a word
__device__ __forceinline__ float dropped(uint64_t bits, int k, uint32_t below, float scale, float x)
{
    const uint32_t field = (uint32_t)(bits >> (k < 2 ? 0 : 32)) >> (16 * (k % 2)) & 0xffffu;
    return field < below ? 0.0f : x * scale;        // chosen, not multiplied by 0: a dropped infinity or NaN is dropped
}

// 16 bytes per lane and array; the values behind the last whole vector are done by the first lanes of the last workgroup, one word each.
// Bound by memory: the generator costs some 14 operations per element, which hide behind the loads.  2^28 fp16 values: with a residual 246 us
// (6.5 TB/s), without 167 (6.4); through the caches 268 with one.
template <class T, bool kResidual, bool kStreamed>
__global__ void __launch_bounds__(kBlock)
dropout_kernel(Drop a)
{
    constexpr int V = 16 / sizeof(T);
    const T *x = (const T *)a.x, *r = (const T *)a.r;
    T *y = (T *)a.y;
    const uint64_t n_vectors = a.n / V, i = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i < n_vectors) {
        Pack<T, V> v = kStreamed ? load_streamed<T, V>(x + i * V) : *reinterpret_cast<const Pack<T, V> *>(x + i * V), b;
        if (kResidual) b = kStreamed ? load_streamed<T, V>(r + i * V) : *reinterpret_cast<const Pack<T, V> *>(r + i * V);
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const uint64_t bits = dg_sample::mix64(a.seed, a.offset + i * (V / 4) + q);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float t = dropped(bits, k, a.below, a.scale, (float)v.v[4 * q + k]);
                if (kResidual) t += (float)b.v[4 * q + k];
                v.v[4 * q + k] = (T)t;
            }
        }
        if (kStreamed) store_streamed<T, V>(y + i * V, v);
        else *reinterpret_cast<Pack<T, V> *>(y + i * V) = v;
    }
    const uint64_t j = n_vectors * V + threadIdx.x;
    if (blockIdx.x == gridDim.x - 1 && j < a.n) {
        const float t = dropped(dg_sample::mix64(a.seed, a.offset + j / 4), j % 4, a.below, a.scale, (float)x[j]);
        y[j] = (T)(kResidual ? t + (float)r[j] : t);
    }
}

// arrays that are not aligned: four values, one word, per lane
template <class T, bool kResidual>
__global__ void __launch_bounds__(kBlock)
dropout_unaligned_kernel(Drop a)
{
    const uint64_t q = (uint64_t)blockIdx.x * kBlock + threadIdx.x, bits = dg_sample::mix64(a.seed, a.offset + q);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t i = 4 * q + k;
        if (i >= a.n) return;
        const float t = dropped(bits, k, a.below, a.scale, (float)((const T *)a.x)[i]);
        ((T *)a.y)[i] = (T)(kResidual ? t + (float)((const T *)a.r)[i] : t);
    }
}

// Values of one launch: 2^31 lanes at most.  A grid of 2^32 lanes and more is cut short without an error.
constexpr uint64_t kMost = 1ull << 33;

template <class T>
void launch_one(const Drop &a, bool streamed, hipStream_t st)
{
    const bool vectors = dg::aligned(a.x, 16) && dg::aligned(a.r, 16) && dg::aligned(a.y, 16);
    const uint64_t per = (vectors ? 16 / sizeof(T) : 4) * kBlock;
    auto go = [&](auto kernel) { kernel<<<(uint32_t)((a.n + per - 1) / per), kBlock, 0, st>>>(a); };
    if (!vectors) return a.r ? go(dropout_unaligned_kernel<T, true>) : go(dropout_unaligned_kernel<T, false>);
    if (streamed) a.r ? go(dropout_kernel<T, true, true>) : go(dropout_kernel<T, false, true>);
    else a.r ? go(dropout_kernel<T, true, false>) : go(dropout_kernel<T, false, false>);
}

template <class T>
void launch(const Drop &a, hipStream_t st)
{
    for (uint64_t at = 0; at < a.n; at += kMost) {
        Drop part = a;
        part.x = (const T *)a.x + at;
        part.r = a.r ? (const T *)a.r + at : nullptr;
        part.y = (T *)a.y + at;
        part.n = a.n - at < kMost ? a.n - at : kMost;
        part.offset += at / 4;
        launch_one<T>(part, a.n * sizeof(T) >= kStreamedBytes, st);
    }
}

int dropout(const char *who, const void *x, const void *r, uint64_t n, double p, uint64_t seed, uint64_t offset, uint32_t dtype, void *y, hipStream_t st)
{
    DG_REQUIRE(known_type(dtype), DG_ERR_ARG, "%s: unknown element type %u", who, dtype);
    DG_REQUIRE(p >= 0.0 && p <= 1.0, DG_ERR_ARG, "%s: p must lie in [0, 1]", who);
    if (n == 0) return DG_OK;
    const size_t item = item_bytes(dtype);
    DG_REQUIRE(x && y && dg::aligned(x, item) && dg::aligned(y, item) && dg::aligned(r, item), DG_ERR_ARG, "%s: null or misaligned pointer", who);
    DG_REQUIRE(n <= 1ull << 40, DG_ERR_UNSUPPORTED, "%s: more than 2^40 values", who);
    const uint32_t below = (uint32_t)std::floor(p * 65536.0 + 0.5);
    const float scale = below == 65536u ? 0.0f : (float)(65536.0 / (65536u - below));
    (dtype == DG_F32 ? launch<float> : dtype == DG_F16 ? launch<f16> : launch<bf16>)({x, r, y, n, seed, offset, below, scale}, st);
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
