// Root-mean-square norm of rows of W values with the residual's addition, and its backward pass:
//   t = x + r,  s = 1 / sqrt(mean(t^2) + eps),  th = t s,  y = th gamma;
//   g = dy gamma,  dx = dr = dt + s (g - th mean(g th)),  dgamma = sum over rows of dy th.
// The backward pass computes s again from t; nothing else is saved.
//
// Both passes are bound by memory: a row is read once into registers and everything is summed there.  The backward pass adds up dgamma of the
// rows that a lane sees in its registers; a workgroup's sums go to the workspace and a second launch folds them.  No atomics: the same bits each time.
// Backward, 8192 rows of 4096 bf16 values with the gradient past the norm: 45 us, 6.0 TB/s of what goes in and out, and the fold 4.8 us.
#include "rms_norm_common.h"

namespace {

using namespace dg_rms;

template <class T, int V, int G, int K, int kThreads, bool kStreamed, bool kLoose, bool kResidual>
__global__ void __launch_bounds__(kThreads)
rms_bwd_kernel(Rms a)
{
    constexpr int kWaves = kThreads / dg::kWave, R = kThreads / G;
    constexpr bool kAhead = K > 1;
    __shared__ float red[kWaves][2];
    const uint32_t lane = threadIdx.x % G;
    float gamma[K][V], sum_g[K][V] = {};
    weights<V, G, K, kLoose>(a.gamma, 1.0f, a, lane, gamma);
    uint32_t c;
    uint64_t row = (uint64_t)blockIdx.x * R + threadIdx.x / G;
    Pack<T, V> next_x[K], next_dy[K], next_dt[K];
    auto fetch = [&] {
        read<T, V, G, K, kStreamed, kLoose, kAhead>(a.x, a.ldx, row, a, lane, next_x);
        read<T, V, G, K, kStreamed, kLoose, kAhead>(a.dy, a.lddy, row, a, lane, next_dy);
        if (kResidual) read<T, V, G, K, kStreamed, kLoose, kAhead>(a.dt, a.lddt, row, a, lane, next_dt);
    };
    if (kAhead) fetch();
    for (uint64_t row0 = (uint64_t)blockIdx.x * R; row0 < a.N; row0 += (uint64_t)gridDim.x * R) {
        const bool held = row < a.N;                // lanes without a row go along: sums are over whole groups of lanes
        T *out = (T *)a.out + row * a.ldo;
        float x[K][V], dy[K][V], dt[K][V];
        if (!kAhead) fetch();
        widen<T, V, G, K, kAhead>(next_x, a, lane, x);
        widen<T, V, G, K, kAhead>(next_dy, a, lane, dy);
        if (kResidual) widen<T, V, G, K, kAhead>(next_dt, a, lane, dt);
        row += (uint64_t)gridDim.x * R;
        if (kAhead) fetch();
        float sum[2] = {0.0f, 0.0f};                // of squares, of g times the value
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int from = skipped<V, kLoose>(a.W, (k * G + lane) * V);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (kLoose && v < from) continue;
                sum[0] += x[k][v] * x[k][v];
                sum[1] += dy[k][v] * gamma[k][v] * x[k][v];
            }
        }
        row_sums<G, kThreads, 2>(sum, red);
        const float s = 1.0f / sqrtf(sum[0] / (float)a.W + a.eps), mean_gx = sum[1] / (float)a.W * s;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float o[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float xh = x[k][v] * s;
                o[v] = s * fmaf(-xh, mean_gx, dy[k][v] * gamma[k][v]);
                if (kResidual) o[v] += dt[k][v];
                if (held) sum_g[k][v] += dy[k][v] * xh;
            }
            if (inside<V>(a.W, lane, k, G, c) && held && a.out) write<T, V, kStreamed, kLoose>(out + begin_of<V, kLoose>(a.W, c), o);
        }
    }
    if (!a.part) return;
    // the rows of a wavefront, then those of the workgroup's wavefronts
    float *part = a.part + (uint64_t)blockIdx.x * a.W;
    __shared__ float sums[G < kThreads ? kWaves : 1][G < kThreads ? G * V : 1];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool in = inside<V>(a.W, lane, k, G, c);
        if (G >= kThreads) {
            if (in) {
                float *to = part + begin_of<V, kLoose>(a.W, c);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (!kLoose || v >= skipped<V, kLoose>(a.W, c)) to[v] = sum_g[k][v];
            }
            continue;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int d = G; d < dg::kWave; d *= 2) sum_g[k][v] += __shfl_xor(sum_g[k][v], d);
        __syncthreads();
        if (threadIdx.x % dg::kWave < G)
#pragma unroll
            for (int v = 0; v < V; ++v) sums[threadIdx.x / dg::kWave][lane * V + v] = sum_g[k][v];
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < G * V; j += kThreads) {
            const uint32_t begin = k * G * V + j / V * V, col = begin_of<V, kLoose>(a.W, begin) + j % V;
            float t = 0.0f;
            for (int w = 0; w < kWaves; ++w) t += sums[w][j];
            if (begin < a.W && (!kLoose || (int)(j % V) >= skipped<V, kLoose>(a.W, begin))) part[col] = t;
        }
    }
}

// dgamma of the workgroups' sums: 16 columns per workgroup, 64 lanes of each share the parts
constexpr int kFoldColumns = 16, kFoldRuns = 64;

__global__ void __launch_bounds__(kFoldColumns *kFoldRuns)
rms_fold_kernel(const float *part, uint32_t n_parts, uint32_t W, float *dgamma)
{
    __shared__ float red[kFoldRuns][kFoldColumns];
    const uint32_t lane = threadIdx.x % kFoldColumns, run = threadIdx.x / kFoldColumns, c = blockIdx.x * kFoldColumns + lane;
    float sum = 0.0f;
    if (c < W)
#pragma unroll 16
        for (uint32_t p = run; p < n_parts; p += kFoldRuns) sum += part[(uint64_t)p * W + c];
    red[run][lane] = sum;
#pragma unroll
    for (int d = kFoldRuns / 2; d > 0; d /= 2) {
        __syncthreads();
        if ((int)run < d) red[run][lane] += red[run + d][lane];
    }
    if (run == 0 && c < W) dgamma[c] = red[0][lane];
}

template <class T>
__global__ void __launch_bounds__(kWide)
rms_bwd_wide_kernel(Rms a)
{
    __shared__ float red[kWide / dg::kWave][1], red2[kWide / dg::kWave][1];
    float *part = a.part ? a.part + (uint64_t)blockIdx.x * a.W : nullptr;
    for (uint32_t c = threadIdx.x; part && c < a.W; c += kWide) part[c] = 0.0f;     // by the lane that adds to them
    for (uint64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.ldx, *dy = (const T *)a.dy + row * a.lddy, *dt = a.dt ? (const T *)a.dt + row * a.lddt : nullptr;
        T *out = (T *)a.out + row * a.ldo;
        const float s = wide_scale<T>(x, nullptr, a, red);
        float sum[1] = {0.0f};
        for (uint32_t c = threadIdx.x; c < a.W; c += kWide) sum[0] += (float)dy[c] * (a.gamma ? a.gamma[c] : 1.0f) * (float)x[c];
        row_sums<kWide, kWide, 1>(sum, red2);
        const float mean_gx = sum[0] / (float)a.W * s;
        for (uint32_t c = threadIdx.x; c < a.W; c += kWide) {
            const float d = (float)dy[c], xh = (float)x[c] * s;
            if (part) part[c] += d * xh;
            if (a.out) out[c] = (T)(s * fmaf(-xh, mean_gx, d * (a.gamma ? a.gamma[c] : 1.0f)) + (dt ? (float)dt[c] : 0.0f));
        }
    }
}

template <bool kResidual>
struct Forward {
    template <class T, int V, int G, int K, bool kStreamed, bool kLoose>
    static void launch(const Call &c, uint32_t grid)
    {
        rms_fwd_kernel<T, V, G, K, kBlock, kStreamed, kLoose, kResidual, kNormed><<<grid, kBlock, 0, c.st>>>(c.a);
    }
    template <class T>
    static void launch_wide(const Call &c)
    {
        rms_fwd_wide_kernel<T, kNormed><<<(uint32_t)(c.a.N < kMostWide ? c.a.N : kMostWide), kWide, 0, c.st>>>(c.a);
    }
};

template <bool kResidual>
struct Backward {
    template <class T, int V, int G, int K, bool kStreamed, bool kLoose>
    static void launch(const Call &c, uint32_t)
    {
        rms_bwd_kernel<T, V, G, K, kBlock, kStreamed, kLoose, kResidual><<<c.parts, kBlock, 0, c.st>>>(c.a);
    }
    template <class T>
    static void launch_wide(const Call &c) { rms_bwd_wide_kernel<T><<<c.parts, kWide, 0, c.st>>>(c.a); }
};

// Workgroups of the backward pass, by layer norm's rule: each leaves W sums, so that wide rows have fewer, and has some 6000 values to itself, but
// there are two for each compute unit, and as many for all.
uint32_t parts_of(uint64_t N, uint32_t W)
{
    const uint64_t most = W <= 512 ? 2048 : W <= 2048 ? 1024 : 512, rows = W <= 512 ? 6144 / W : W <= 2048 ? 16 : 8;
    const uint64_t p = (N + rows - 1) / rows, least = (N + 3) / 4 < 512 ? (N + 3) / 4 : 512;
    return (uint32_t)(p > most ? most : p < least ? least : p >= 512 ? p / 512 * 512 : p);
}

}  // namespace

extern "C" int dg_rms_norm_fwd(const void *x, uint64_t ldx, const void *residual, uint64_t ldr, const float *gamma, uint64_t N, uint32_t W, float eps,
                               uint32_t dtype, void *total, uint64_t ldt, void *y, uint64_t ldy, void *stream)
{
    const char *who = "dg_rms_norm_fwd";
    if (int rc = check_norm(who, N, W, eps, dtype)) return rc;
    if (N == 0) return DG_OK;
    Rms a = {};
    a.x = x, a.r = residual, a.t = total, a.out = y, a.gamma = gamma, a.ldx = ldx, a.ldr = ldr, a.ldt = ldt, a.ldo = ldy, a.N = N, a.W = W, a.eps = eps;
    if (int rc = check_forward(who, a, dtype)) return rc;
    if (int rc = check_rows(who, y, ldy, W, dtype)) return rc;
    DG_REQUIRE(y != total, DG_ERR_ARG, "%s: the sum and the norm in one place", who);
    const bool aligned = may_align(x, ldx, dtype) && may_align(residual, ldr, dtype) && may_align(total, ldt, dtype) && may_align(y, ldy, dtype);
    const Call c = {a, dtype, 0, (hipStream_t)stream};
    residual ? launch<Forward<true>>(c, aligned) : launch<Forward<false>>(c, aligned);
    return dg::launch_status(who);
}

extern "C" size_t dg_rms_norm_bwd_workspace_bytes(uint64_t N, uint32_t W) { return (size_t)parts_of(N, W) * W * sizeof(float); }

extern "C" int dg_rms_norm_bwd(const void *total, uint64_t ldt, const float *gamma, const void *dy, uint64_t lddy, const void *dtotal, uint64_t lddt,
                               uint64_t N, uint32_t W, float eps, uint32_t dtype, void *dx, uint64_t lddx, float *dgamma, void *ws, size_t ws_bytes,
                               void *stream)
{
    const char *who = "dg_rms_norm_bwd";
    if (int rc = check_norm(who, N, W, eps, dtype)) return rc;
    if (N) {
        if (int rc = check_rows(who, total, ldt, W, dtype)) return rc;
        if (int rc = check_rows(who, dy, lddy, W, dtype)) return rc;
        if (dtotal)
            if (int rc = check_rows(who, dtotal, lddt, W, dtype)) return rc;
        if (dx)
            if (int rc = check_rows(who, dx, lddx, W, dtype)) return rc;
    }
    DG_REQUIRE(dg::aligned(gamma, 4) && dg::aligned(dgamma, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (!dgamma && (!dx || !N)) return DG_OK;
    const size_t need = dgamma ? dg_rms_norm_bwd_workspace_bytes(N, W) : 0;
    DG_REQUIRE(need == 0 || (ws && dg::aligned(ws, 16) && ws_bytes >= need), DG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need,
               ws ? ws_bytes : 0);
    const uint32_t parts = parts_of(N, W);
    if (N) {
        Rms a = {};
        a.x = total, a.dy = dy, a.dt = dx ? dtotal : nullptr, a.out = dx, a.gamma = gamma, a.part = dgamma ? (float *)ws : nullptr;
        a.ldx = ldt, a.lddy = lddy, a.lddt = lddt, a.ldo = lddx, a.N = N, a.W = W, a.eps = eps;
        const bool aligned = may_align(total, ldt, dtype) && may_align(dy, lddy, dtype) && may_align(a.dt, lddt, dtype) && may_align(dx, lddx, dtype);
        const Call c = {a, dtype, parts, (hipStream_t)stream};
        a.dt ? launch<Backward<true>>(c, aligned) : launch<Backward<false>>(c, aligned);
    }
    if (dgamma)
        rms_fold_kernel<<<(W + kFoldColumns - 1) / kFoldColumns, kFoldColumns * kFoldRuns, 0, (hipStream_t)stream>>>((const float *)ws, parts, W, dgamma);
    return dg::launch_status(who);
}
