// Layer norm of rows of W values, m their mean, s = 1 / sqrt(mean((x - m)^2) + eps):
//   xh = (x - m) s,  y = xh gamma + beta;
//   g = dy gamma,  dx = s (g - mean(g) - xh mean(g xh)),  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy.
// The backward pass computes m and s again; nothing is saved.
#include <cmath>
#include "rows_common.h"

namespace {

using namespace dg_rows;

constexpr int kBlock = 256, kRowsPerPart = 256;

__device__ __forceinline__ float wave_sum(float v)
{
    for (int d = 1; d < dg::kWave; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// mean and 1 / standard deviation of a row, by one wavefront
template <class T>
__device__ __forceinline__ void moments(const T *x, uint32_t W, float eps, float &m, float &s)
{
    const uint32_t lane = threadIdx.x % dg::kWave;
    float sum = 0.0f;
    for (uint32_t c = lane; c < W; c += dg::kWave) sum += (float)x[c];
    m = wave_sum(sum) / W;
    sum = 0.0f;
    for (uint32_t c = lane; c < W; c += dg::kWave) { const float d = (float)x[c] - m; sum += d * d; }
    s = 1.0f / sqrtf(wave_sum(sum) / W + eps);
}

template <class T>
__global__ void __launch_bounds__(kBlock)
norm_fwd_kernel(const T *x, uint64_t ldx, const float *gamma, const float *beta, uint64_t N, uint32_t W, float eps, T *y, uint64_t ldy)
{
    const uint64_t row = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) / dg::kWave;
    if (row >= N) return;
    float m, s;
    x += row * ldx;
    moments(x, W, eps, m, s);
    for (uint32_t c = threadIdx.x % dg::kWave; c < W; c += dg::kWave)
        y[row * ldy + c] = (T)(((float)x[c] - m) * s * (gamma ? gamma[c] : 1.0f) + (beta ? beta[c] : 0.0f));
}

template <class T>
__global__ void __launch_bounds__(kBlock)
norm_bwd_kernel(const T *x, uint64_t ldx, const float *gamma, const T *dy, uint64_t lddy, uint64_t N, uint32_t W, float eps, T *dx, uint64_t lddx)
{
    const uint64_t row = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) / dg::kWave;
    if (row >= N) return;
    float m, s, sg = 0.0f, sgx = 0.0f;
    x += row * ldx;
    dy += row * lddy;
    moments(x, W, eps, m, s);
    for (uint32_t c = threadIdx.x % dg::kWave; c < W; c += dg::kWave) {
        const float g = (float)dy[c] * (gamma ? gamma[c] : 1.0f);
        sg += g;
        sgx += g * ((float)x[c] - m) * s;
    }
    sg = wave_sum(sg) / W;
    sgx = wave_sum(sgx) / W;
    for (uint32_t c = threadIdx.x % dg::kWave; c < W; c += dg::kWave) {
        const float g = (float)dy[c] * (gamma ? gamma[c] : 1.0f);
        dx[row * lddx + c] = (T)(s * (g - sg - ((float)x[c] - m) * s * sgx));
    }
}

// one wavefront per part of the rows; part p of the sums at part[p][0 / 1][W].  Before dx is written, which may be dy.
template <class T>
__global__ void __launch_bounds__(dg::kWave)
norm_parts_kernel(const T *x, uint64_t ldx, const T *dy, uint64_t lddy, uint64_t N, uint32_t W, float eps, uint64_t per_part, float *part)
{
    const uint64_t row0 = blockIdx.x * per_part, row1 = row0 + per_part < N ? row0 + per_part : N;
    part += (uint64_t)blockIdx.x * 2 * W;
    for (uint32_t c = threadIdx.x; c < 2 * W; c += dg::kWave) part[c] = 0.0f;
    for (uint64_t row = row0; row < row1; ++row) {
        float m, s;
        moments(x + row * ldx, W, eps, m, s);
        for (uint32_t c = threadIdx.x; c < W; c += dg::kWave) {
            const float d = (float)dy[row * lddy + c];
            part[c] += d * ((float)x[row * ldx + c] - m) * s;
            part[W + c] += d;
        }
    }
}

__global__ void __launch_bounds__(kBlock)
norm_fold_kernel(const float *part, uint32_t n_parts, uint32_t W, float *dgamma, float *dbeta)
{
    const uint32_t c = blockIdx.x * kBlock + threadIdx.x;
    if (c >= W) return;
    float a = 0.0f, b = 0.0f;
    for (uint32_t p = 0; p < n_parts; ++p) { a += part[(uint64_t)p * 2 * W + c]; b += part[(uint64_t)p * 2 * W + W + c]; }
    if (dgamma) dgamma[c] = a;
    if (dbeta) dbeta[c] = b;
}

uint32_t parts_of(uint64_t N)
{
    const uint64_t p = (N + kRowsPerPart - 1) / kRowsPerPart;
    return (uint32_t)(p < 4096 ? p : 4096);
}

int check(const char *who, uint64_t N, uint32_t W, float eps, uint32_t dtype)
{
    DG_REQUIRE(known_type(dtype), DG_ERR_ARG, "%s: unknown element type %u", who, dtype);
    DG_REQUIRE(W >= 1 && eps >= 0.0f && std::isfinite(eps), DG_ERR_ARG, "%s: W must be positive, eps finite and not negative", who);
    DG_REQUIRE(N <= 1ull << 32 && W <= 1u << 20, DG_ERR_UNSUPPORTED, "%s: more than 2^32 rows or 2^20 values a row", who);
    return DG_OK;
}

int check_rows(const char *who, const void *p, uint64_t ld, uint32_t W, uint32_t dtype)
{
    DG_REQUIRE(p && dg::aligned(p, item_bytes(dtype)), DG_ERR_ARG, "%s: null or misaligned pointer", who);
    DG_REQUIRE(ld >= W && ld <= 1ull << 40, DG_ERR_ARG, "%s: rows of %u values lie %llu apart", who, W, (unsigned long long)ld);
    return DG_OK;
}

template <class T>
void launch_fwd(const void *x, uint64_t ldx, const float *gamma, const float *beta, uint64_t N, uint32_t W, float eps, void *y, uint64_t ldy, hipStream_t st)
{
    norm_fwd_kernel<T><<<(uint32_t)((N + 3) / 4), kBlock, 0, st>>>((const T *)x, ldx, gamma, beta, N, W, eps, (T *)y, ldy);
}

template <class T>
void launch_bwd(const void *x, uint64_t ldx, const float *gamma, const void *dy, uint64_t lddy, uint64_t N, uint32_t W, float eps, void *dx, uint64_t lddx,
                float *dgamma, float *dbeta, float *part, hipStream_t st)
{
    const uint32_t n_parts = parts_of(N);
    if (dgamma || dbeta) {
        if (n_parts)
            norm_parts_kernel<T><<<n_parts, dg::kWave, 0, st>>>((const T *)x, ldx, (const T *)dy, lddy, N, W, eps, (N + n_parts - 1) / n_parts, part);
        norm_fold_kernel<<<(W + kBlock - 1) / kBlock, kBlock, 0, st>>>(part, n_parts, W, dgamma, dbeta);
    }
    if (dx && N) norm_bwd_kernel<T><<<(uint32_t)((N + 3) / 4), kBlock, 0, st>>>((const T *)x, ldx, gamma, (const T *)dy, lddy, N, W, eps, (T *)dx, lddx);
}

}  // namespace

extern "C" int dg_layer_norm_fwd(const void *x, uint64_t ldx, const float *gamma, const float *beta, uint64_t N, uint32_t W, float eps, uint32_t dtype,
                                 void *y, uint64_t ldy, void *stream)
{
    const char *who = "dg_layer_norm_fwd";
    if (int rc = check(who, N, W, eps, dtype)) return rc;
    if (N == 0) return DG_OK;
    if (int rc = check_rows(who, x, ldx, W, dtype)) return rc;
    if (int rc = check_rows(who, y, ldy, W, dtype)) return rc;
    DG_REQUIRE(dg::aligned(gamma, 4) && dg::aligned(beta, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    (dtype == DG_F32 ? launch_fwd<float> : dtype == DG_F16 ? launch_fwd<f16> : launch_fwd<bf16>)(x, ldx, gamma, beta, N, W, eps, y, ldy, (hipStream_t)stream);
    return dg::launch_status(who);
}

extern "C" size_t dg_layer_norm_bwd_workspace_bytes(uint64_t N, uint32_t W) { return (size_t)parts_of(N) * 2 * W * sizeof(float); }

extern "C" int dg_layer_norm_bwd(const void *x, uint64_t ldx, const float *gamma, const void *dy, uint64_t lddy, uint64_t N, uint32_t W, float eps,
                                 uint32_t dtype, void *dx, uint64_t lddx, float *dgamma, float *dbeta, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "dg_layer_norm_bwd";
    if (int rc = check(who, N, W, eps, dtype)) return rc;
    if (N) {
        if (int rc = check_rows(who, x, ldx, W, dtype)) return rc;
        if (int rc = check_rows(who, dy, lddy, W, dtype)) return rc;
        if (dx)
            if (int rc = check_rows(who, dx, lddx, W, dtype)) return rc;
    }
    DG_REQUIRE(dg::aligned(gamma, 4) && dg::aligned(dgamma, 4) && dg::aligned(dbeta, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (!dgamma && !dbeta && (!dx || !N)) return DG_OK;
    const size_t need = dgamma || dbeta ? dg_layer_norm_bwd_workspace_bytes(N, W) : 0;
    DG_REQUIRE(need == 0 || (ws && dg::aligned(ws, 16) && ws_bytes >= need), DG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need,
               ws ? ws_bytes : 0);
    (dtype == DG_F32 ? launch_bwd<float> : dtype == DG_F16 ? launch_bwd<f16> : launch_bwd<bf16>)(x, ldx, gamma, dy, lddy, N, W, eps, dx, lddx, dgamma, dbeta,
                                                                                                 (float *)ws, (hipStream_t)stream);
    return dg::launch_status(who);
}
