// Layer norm of rows of W values, m their mean, s = 1 / sqrt(mean((x - m)^2) + eps):
//   xh = (x - m) s,  y = xh gamma + beta;
//   g = dy gamma,  dx = s (g - mean(g) - xh mean(g xh)),  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy.
// The backward pass computes m and s again; nothing is saved.
//
// Both passes are bound by memory: a row is read once into registers (K vectors of V values per lane, G lanes per row) and everything
// is summed there, deviations from the mean after the mean itself.  The backward pass adds up dgamma and dbeta of the rows that a
// lane sees in its registers; a workgroup's sums go to the workspace and a second launch folds them.  No atomics: the same bits each time.
// 2^23 rows of 32 fp16 values: forward 194 us (5.5 TB/s), backward 304 (5.3); 2^16 of 4096 bf16 values: 203 (5.3) and 284 (5.7); 2^20 of 37 fp32
// values, unaligned: 58 (5.3) and 106 (4.4).
#include <cmath>
#include "rows_common.h"

namespace {

using namespace dg_rows;

constexpr int kBlock = 256;
// Sum over G neighbouring lanes, in all of them: exchanges inside groups of 4, 8 and 16 lanes on the way to the vector unit, wider ones
// through the LDS crossbar.
template <int kControl>
__device__ __forceinline__ float exchanged(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kControl, 0xf, 0xf, false));
}

template <int G>
__device__ __forceinline__ float group_sum(float v)
{
    if (G >= 2) v += exchanged<0xb1>(v);            // lanes 1 0 3 2
    if (G >= 4) v += exchanged<0x4e>(v);            // lanes 2 3 0 1
    if (G >= 8) v += exchanged<0x141>(v);           // mirrored in 8 lanes: the other four
    if (G >= 16) v += exchanged<0x140>(v);          // mirrored in 16 lanes: the other eight
    if (G >= 32) v += __shfl_xor(v, 16);
    if (G >= 64) v += __shfl_xor(v, 32);
    return v;
}

// The lanes that share a row: G of a wavefront, or all kThreads of the workgroup (G = kThreads).  red: room for one value per
// wavefront and sum.
template <int G, int kThreads, int n>
__device__ __forceinline__ void row_sums(float (&v)[n], float (*red)[n])
{
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = group_sum<(G < dg::kWave ? G : dg::kWave)>(v[i]);
    if (G <= dg::kWave) return;
    constexpr int kWaves = kThreads / dg::kWave;
    __syncthreads();                                // the last use of red is over
    if (threadIdx.x % dg::kWave == 0)
#pragma unroll
        for (int i = 0; i < n; ++i) red[threadIdx.x / dg::kWave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < n; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v[i] += red[w][i];
    }
}

struct Norm {
    const void *x, *dy;
    void *out;                      // y, or dx (NULL: not wanted)
    const float *gamma, *beta;
    float *part;                    // backward: [workgroups][2][W], or NULL
    uint64_t ldx, lddy, ldo, N;
    uint32_t W;
    float eps, per_W;               // 1 / W
};

// Vector k of a lane's share of a row, from value c on; false where the row has ended
template <int V>
__device__ __forceinline__ bool inside(uint32_t W, uint32_t lane, int k, int G, uint32_t &c)
{
    c = (k * G + lane) * V;
    return c < W;
}

// kLoose: rows that no vector divides.  The row's last vector begins early enough to end with it; the first `skipped` of its values are
// the last but one's too: both compute them with the same operations, bit by bit, and store them; sums take them once.
template <int V, bool kLoose>
__device__ __forceinline__ uint32_t begin_of(uint32_t W, uint32_t c)
{
    return kLoose && c + V > W ? W - V : c;
}

template <int V, bool kLoose>
__device__ __forceinline__ int skipped(uint32_t W, uint32_t c)
{
    return kLoose && c < W ? (int)(c - begin_of<V, kLoose>(W, c)) : 0;
}

// 16 bytes that lie as their values do
template <class T>
struct loose { typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2))); };
template <>
struct loose<float> { typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(4))); };

// kAhead: without a branch, so that the compiler can count the loads on their way and does not wait for all of them: the call's last
// row again where there is no further one, the last vector again where the row has ended (widen clears it).  8192 rows of 4096 bf16 values, backward: 50.0 us, with
// branches 55.4; 2^16 rows 284 and 313; 2^17 of 2048 fp32 values 664 and 639.
template <class T, int V, int G, int K, bool kStreamed, bool kLoose, bool kAhead>
__device__ __forceinline__ void read(const void *p, uint64_t ld, uint64_t row, const Norm &a, uint32_t lane, Pack<T, V> (&out)[K])
{
    const T *from = (const T *)p + (!kAhead || row < a.N ? row : a.N - 1) * ld;
    uint32_t c;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool here = inside<V>(a.W, lane, k, G, c) && (kAhead || row < a.N);
        const T *at = from + (here ? begin_of<V, kLoose>(a.W, c) : a.W - V);
        if (!kAhead && !here) {
#pragma unroll
            for (int v = 0; v < V; ++v) out[k].v[v] = (T)0.0f;
        } else if constexpr (kStreamed) out[k] = load_streamed<T, V>(at);
        else if constexpr (kLoose) out[k] = __builtin_bit_cast(Pack<T, V>, *reinterpret_cast<const typename loose<T>::u4 *>(at));
        else out[k] = *reinterpret_cast<const Pack<T, V> *>(at);
    }
}

template <class T, int V, bool kStreamed, bool kLoose>
__device__ __forceinline__ void write(T *p, const float (&in)[V])
{
    Pack<T, V> a;
#pragma unroll
    for (int v = 0; v < V; ++v) a.v[v] = (T)in[v];
    if constexpr (kStreamed) store_streamed<T, V>(p, a);
    else if constexpr (kLoose) *reinterpret_cast<typename loose<T>::u4 *>(p) = __builtin_bit_cast(typename loose<T>::u4, a);
    else *reinterpret_cast<Pack<T, V> *>(p) = a;
}

template <class T, int V, int G, int K, bool kAhead>
__device__ __forceinline__ void widen(const Pack<T, V> (&in)[K], const Norm &a, uint32_t lane, float (&out)[K][V])
{
    uint32_t c;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool here = !kAhead || inside<V>(a.W, lane, k, G, c);
#pragma unroll
        for (int v = 0; v < V; ++v) out[k][v] = here ? (float)in[k].v[v] : 0.0f;
    }
}

// a lane's share of a vector of W values, `none` without one; four at a time, which only lie as fp32 values do
template <int V, int G, int K, bool kLoose>
__device__ __forceinline__ void weights(const float *p, float none, const Norm &a, uint32_t lane, float (&out)[K][V])
{
    constexpr int n = V % 4 == 0 ? 4 : 1;
    uint32_t c;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool in = inside<V>(a.W, lane, k, G, c) && p;
        const float *at = p + begin_of<V, kLoose>(a.W, c);
#pragma unroll
        for (int v = 0; v < V; v += n) {
            Pack<float, n> w;
#pragma unroll
            for (float &each : w.v) each = none;
            if (in) {
                if constexpr (n == 4) w = __builtin_bit_cast(Pack<float, n>, *reinterpret_cast<const loose<float>::u4 *>(at + v));
                else w.v[0] = at[v];
            }
#pragma unroll
            for (int i = 0; i < n; ++i) out[k][v + i] = w.v[i];
        }
    }
}

// mean of a row in registers
template <int V, int G, int K, int kThreads, bool kLoose>
__device__ __forceinline__ float mean(const float (&x)[K][V], const Norm &a, uint32_t lane, float (*red)[1])
{
    float sum[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int from = skipped<V, kLoose>(a.W, (k * G + lane) * V);
#pragma unroll
        for (int v = 0; v < V; ++v) sum[0] += kLoose && v < from ? 0.0f : x[k][v];
    }
    row_sums<G, kThreads, 1>(sum, red);
    return sum[0] * a.per_W;
}

// Workgroups go through the rows side by side: workgroup b takes rows b R, b R + 1, ... of every gridDim.x R, R = kThreads / G at a
// time, with gamma and beta in registers.  Where a row takes more than one vector per lane the next row is on its way while one is worked
// on (2^16 rows of 4096 bf16 values, backward: 284 us, without 523); narrower rows have wavefronts enough (2^20 of 256: 290 without, 322).
template <class T, int V, int G, int K, int kThreads, bool kStreamed, bool kLoose>
__global__ void __launch_bounds__(kThreads)
norm_fwd_kernel(Norm a)
{
    constexpr int R = kThreads / G;
    constexpr bool kAhead = K > 1;
    __shared__ float red[kThreads / dg::kWave][1], red2[kThreads / dg::kWave][1];
    const uint32_t lane = threadIdx.x % G;
    float gamma[K][V], beta[K][V];
    weights<V, G, K, kLoose>(a.gamma, 1.0f, a, lane, gamma);
    weights<V, G, K, kLoose>(a.beta, 0.0f, a, lane, beta);
    uint64_t row = (uint64_t)blockIdx.x * R + threadIdx.x / G;
    Pack<T, V> next[K];
    if (kAhead) read<T, V, G, K, kStreamed, kLoose, kAhead>(a.x, a.ldx, row, a, lane, next);
    for (uint64_t row0 = (uint64_t)blockIdx.x * R; row0 < a.N; row0 += (uint64_t)gridDim.x * R) {
        float x[K][V];
        if (!kAhead) read<T, V, G, K, kStreamed, kLoose, kAhead>(a.x, a.ldx, row, a, lane, next);
        widen<T, V, G, K, kAhead>(next, a, lane, x);
        const uint64_t now = row;
        row += (uint64_t)gridDim.x * R;
        if (kAhead) read<T, V, G, K, kStreamed, kLoose, kAhead>(a.x, a.ldx, row, a, lane, next);
        const float m = mean<V, G, K, kThreads, kLoose>(x, a, lane, red);
        float sum[1] = {0.0f};
        uint32_t c;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (inside<V>(a.W, lane, k, G, c)) {
                const int from = skipped<V, kLoose>(a.W, c);
#pragma unroll
                for (int v = 0; v < V; ++v) { x[k][v] -= m; sum[0] += kLoose && v < from ? 0.0f : x[k][v] * x[k][v]; }
            }
        row_sums<G, kThreads, 1>(sum, red2);
        const float s = 1.0f / sqrtf(sum[0] * a.per_W + a.eps);
        T *y = (T *)a.out + now * a.ldo;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (inside<V>(a.W, lane, k, G, c) && now < a.N) {
#pragma unroll
                for (int v = 0; v < V; ++v) x[k][v] = fmaf(x[k][v] * s, gamma[k][v], beta[k][v]);
                write<T, V, kStreamed, kLoose>(y + begin_of<V, kLoose>(a.W, c), x[k]);
            }
    }
}

template <class T, int V, int G, int K, int kThreads, bool kStreamed, bool kLoose>
__global__ void __launch_bounds__(kThreads)
norm_bwd_kernel(Norm a)
{
    constexpr int kWaves = kThreads / dg::kWave, R = kThreads / G;
    constexpr bool kAhead = K > 1;
    __shared__ float red1[kWaves][1], red3[kWaves][3];
    const uint32_t lane = threadIdx.x % G;
    float gamma[K][V], sum_g[K][V] = {}, sum_b[K][V] = {};
    weights<V, G, K, kLoose>(a.gamma, 1.0f, a, lane, gamma);
    uint32_t c;
    uint64_t row = (uint64_t)blockIdx.x * R + threadIdx.x / G;
    Pack<T, V> next_x[K], next_dy[K];
    auto fetch = [&] {
        read<T, V, G, K, kStreamed, kLoose, kAhead>(a.x, a.ldx, row, a, lane, next_x);
        read<T, V, G, K, kStreamed, kLoose, kAhead>(a.dy, a.lddy, row, a, lane, next_dy);
    };
    if (kAhead) fetch();
    for (uint64_t row0 = (uint64_t)blockIdx.x * R; row0 < a.N; row0 += (uint64_t)gridDim.x * R) {
        const bool held = row < a.N;                // lanes without a row go along: sums are over whole groups of lanes
        T *out = (T *)a.out + row * a.ldo;
        float x[K][V], dy[K][V];
        if (!kAhead) fetch();
        widen<T, V, G, K, kAhead>(next_x, a, lane, x);
        widen<T, V, G, K, kAhead>(next_dy, a, lane, dy);
        row += (uint64_t)gridDim.x * R;
        if (kAhead) fetch();
        const float m = mean<V, G, K, kThreads, kLoose>(x, a, lane, red1);
        float sum[3] = {0.0f, 0.0f, 0.0f};          // of squared deviations, of g, of g times the deviation
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (inside<V>(a.W, lane, k, G, c)) {
                const int from = skipped<V, kLoose>(a.W, c);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    x[k][v] -= m;
                    if (kLoose && v < from) continue;
                    sum[0] += x[k][v] * x[k][v];
                    const float g = dy[k][v] * gamma[k][v];
                    sum[1] += g;
                    sum[2] += g * x[k][v];
                }
            }
        row_sums<G, kThreads, 3>(sum, red3);
        const float s = 1.0f / sqrtf(sum[0] * a.per_W + a.eps), mean_g = sum[1] * a.per_W, mean_gx = sum[2] * a.per_W * s;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float o[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float xh = x[k][v] * s;
                o[v] = s * fmaf(-xh, mean_gx, fmaf(dy[k][v], gamma[k][v], -mean_g));
                if (held) {
                    sum_g[k][v] += dy[k][v] * xh;
                    sum_b[k][v] += dy[k][v];
                }
            }
            if (inside<V>(a.W, lane, k, G, c) && held && a.out) write<T, V, kStreamed, kLoose>(out + begin_of<V, kLoose>(a.W, c), o);
        }
    }
    if (!a.part) return;
    // the rows of a wavefront, then those of the workgroup's wavefronts
    float *part = a.part + (uint64_t)blockIdx.x * 2 * a.W;
    __shared__ float sums[G < kThreads ? kWaves : 1][2][G < kThreads ? G * V : 1];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool in = inside<V>(a.W, lane, k, G, c);
        if (G >= kThreads) {
            if (in) {
                float *to = part + begin_of<V, kLoose>(a.W, c);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (!kLoose || v >= skipped<V, kLoose>(a.W, c)) { to[v] = sum_g[k][v]; to[a.W + v] = sum_b[k][v]; }
            }
            continue;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int d = G; d < dg::kWave; d *= 2) {
                sum_g[k][v] += __shfl_xor(sum_g[k][v], d);
                sum_b[k][v] += __shfl_xor(sum_b[k][v], d);
            }
        __syncthreads();
        if (threadIdx.x % dg::kWave < G)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                sums[threadIdx.x / dg::kWave][0][lane * V + v] = sum_g[k][v];
                sums[threadIdx.x / dg::kWave][1][lane * V + v] = sum_b[k][v];
            }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 2 * G * V; i += kThreads) {
            const uint32_t which = i / (G * V), j = i % (G * V), begin = k * G * V + j / V * V, col = begin_of<V, kLoose>(a.W, begin) + j % V;
            float t = 0.0f;
            for (int w = 0; w < kWaves; ++w) t += sums[w][which][j];
            if (begin < a.W && (!kLoose || (int)(j % V) >= skipped<V, kLoose>(a.W, begin))) part[which * a.W + col] = t;
        }
    }
}

// dgamma and dbeta of the workgroups' sums: 16 columns per workgroup, 64 lanes of each share the parts
constexpr int kFoldColumns = 16, kFoldRuns = 64;

__global__ void __launch_bounds__(kFoldColumns *kFoldRuns)
norm_fold_kernel(const float *part, uint32_t n_parts, uint32_t W, float *dgamma, float *dbeta)
{
    __shared__ float red[kFoldRuns][kFoldColumns];
    const uint32_t lane = threadIdx.x % kFoldColumns, run = threadIdx.x / kFoldColumns, c = blockIdx.x * kFoldColumns + lane;
    float sum = 0.0f;
    if (c < 2 * W)
#pragma unroll 16
        for (uint32_t p = run; p < n_parts; p += kFoldRuns) sum += part[(uint64_t)p * 2 * W + c];
    red[run][lane] = sum;
#pragma unroll
    for (int d = kFoldRuns / 2; d > 0; d /= 2) {
        __syncthreads();
        if ((int)run < d) red[run][lane] += red[run + d][lane];
    }
    if (run != 0 || c >= 2 * W) return;
    sum = red[0][lane];
    if (c < W) {
        if (dgamma) dgamma[c] = sum;
    } else if (dbeta) dbeta[c - W] = sum;
}

// Rows too wide for the registers of a workgroup: read again from the caches for every sum, a workgroup per row.
constexpr int kWide = 1024;

template <class T>
__device__ __forceinline__ void wide_moments(const T *x, const Norm &a, float &m, float &s, float (*red)[1])
{
    float sum[1] = {0.0f};
    for (uint32_t c = threadIdx.x; c < a.W; c += kWide) sum[0] += (float)x[c];
    row_sums<kWide, kWide, 1>(sum, red);
    m = sum[0] * a.per_W;
    sum[0] = 0.0f;
    for (uint32_t c = threadIdx.x; c < a.W; c += kWide) { const float d = (float)x[c] - m; sum[0] += d * d; }
    row_sums<kWide, kWide, 1>(sum, red);
    s = 1.0f / sqrtf(sum[0] * a.per_W + a.eps);
}

template <class T>
__global__ void __launch_bounds__(kWide)
norm_fwd_wide_kernel(Norm a)
{
    __shared__ float red[kWide / dg::kWave][1];
    for (uint64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.ldx;
        T *y = (T *)a.out + row * a.ldo;
        float m, s;
        wide_moments(x, a, m, s, red);
        for (uint32_t c = threadIdx.x; c < a.W; c += kWide) y[c] = (T)(((float)x[c] - m) * s * (a.gamma ? a.gamma[c] : 1.0f) + (a.beta ? a.beta[c] : 0.0f));
    }
}

template <class T>
__global__ void __launch_bounds__(kWide)
norm_bwd_wide_kernel(Norm a)
{
    __shared__ float red[kWide / dg::kWave][1], red2[kWide / dg::kWave][2];
    float *part = a.part ? a.part + (uint64_t)blockIdx.x * 2 * a.W : nullptr;
    for (uint32_t c = threadIdx.x; part && c < a.W; c += kWide) part[c] = part[a.W + c] = 0.0f;     // by the lane that adds to them
    for (uint64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.ldx, *dy = (const T *)a.dy + row * a.lddy;
        T *out = (T *)a.out + row * a.ldo;
        float m, s, sum[2] = {0.0f, 0.0f};
        wide_moments(x, a, m, s, red);
        for (uint32_t c = threadIdx.x; c < a.W; c += kWide) {
            const float g = (float)dy[c] * (a.gamma ? a.gamma[c] : 1.0f);
            sum[0] += g;
            sum[1] += g * ((float)x[c] - m) * s;
        }
        row_sums<kWide, kWide, 2>(sum, red2);
        for (uint32_t c = threadIdx.x; c < a.W; c += kWide) {
            const float d = (float)dy[c], xh = ((float)x[c] - m) * s;
            if (part) {
                part[c] += d * xh;
                part[a.W + c] += d;
            }
            if (a.out) out[c] = (T)(s * (d * (a.gamma ? a.gamma[c] : 1.0f) - sum[0] * a.per_W - xh * sum[1] * a.per_W));
        }
    }
}

int check(const char *who, uint64_t N, uint32_t W, float eps, uint32_t dtype)
{
    DG_REQUIRE(known_type(dtype), DG_ERR_ARG, "%s: unknown element type %u", who, dtype);
    DG_REQUIRE(W >= 1 && eps >= 0.0f && std::isfinite(eps), DG_ERR_ARG, "%s: W must be positive, eps finite and not negative", who);
    DG_REQUIRE(N <= 1ull << 32 && W <= 1u << 20 && N * W <= 1ull << 39, DG_ERR_UNSUPPORTED, "%s: more than 2^32 rows, 2^20 values a row or 2^39 values", who);
    return DG_OK;
}

int check_rows(const char *who, const void *p, uint64_t ld, uint32_t W, uint32_t dtype)
{
    DG_REQUIRE(p && dg::aligned(p, item_bytes(dtype)), DG_ERR_ARG, "%s: null or misaligned pointer", who);
    DG_REQUIRE(ld >= W && ld <= 1ull << 40, DG_ERR_ARG, "%s: rows of %u values lie %llu apart", who, W, (unsigned long long)ld);
    return DG_OK;
}

// How a row of n vectors is spread: up to 64 over as many lanes, rounded up to a power of two; several per lane would leave fewer lanes
// idle, but a load then takes parts of many lines, which loads past the caches fetch again (48 bf16 values a row, two lanes of three
// vectors: 1.9 TB/s forward, eight lanes 5.5).  Then a wavefront with up to 4 each, then a workgroup with up to 8.
struct Spread { int G, K; };

Spread spread_of(uint32_t n)
{
    int G = 1;
    while (G < 64 && (uint32_t)G < n) G *= 2;
    for (int K = 1; K <= 4; ++K)
        if (n <= (uint32_t)(G * K)) return {G, K};
    for (int K = 2; K <= 8; K *= 2)
        if (n <= 256u * K) return {256, K};
    return {0, 0};
}

// Workgroups of the backward pass.  Each leaves 2 W sums, so that wide rows have fewer, and each has some 6000 values to itself, but there are two
// for each compute unit, and as many for all (they run side by side unless a lane has eight vectors, whose registers leave room for one: 8192 rows of 8192 fp32 values
// 156 us, 5.2 TB/s; of 16 384 bf16 values 223, 3.6).  (8192 rows of 4096 bf16 values: 512 workgroups 50 us, 1024 64; 2^23 of 32 fp16
// values: 2048 304 us, 1024 323; 200 000 of 32: 2048 19.7 us, 1563 20.2, 1024 15.3, 781 19.3.)
uint32_t parts_of(uint64_t N, uint32_t W)
{
    const uint64_t most = W <= 512 ? 2048 : W <= 2048 ? 1024 : 512, rows = W <= 512 ? 6144 / W : W <= 2048 ? 16 : 8;
    const uint64_t p = (N + rows - 1) / rows, least = (N + 3) / 4 < 512 ? (N + 3) / 4 : 512;
    return (uint32_t)(p > most ? most : p < least ? least : p >= 512 ? p / 512 * 512 : p);
}

// of the forward pass: as many as the chip holds at once where a lane has one vector; with more of them it holds two to five eighths
constexpr uint64_t kMostBlocks = 2048;

// Of the forward pass of rows too wide for registers: far from the 2^32 lanes from which a grid is cut short without an error.  (20 000 rows of 8200 fp32
// values: a workgroup for each 491 us, 2048 for all 505.)
constexpr uint64_t kMostWide = 1 << 16;

struct Call {
    Norm a;
    uint32_t dtype, parts;
    bool forward;
    hipStream_t st;
};

template <class T, int V, int G, int K, bool kLoose>
void launch_spread(const Call &c)
{
    const uint64_t all = (c.a.N + kBlock / G - 1) / (kBlock / G);
    const uint32_t grid = c.forward ? (uint32_t)(all < kMostBlocks ? all : kMostBlocks) : c.parts;
    auto go = [&](auto kernel) { kernel<<<grid, kBlock, 0, c.st>>>(c.a); };
    if constexpr (V * sizeof(T) == 16 && !kLoose)
        if (c.a.N * c.a.W * sizeof(T) >= kStreamedBytes)
            return c.forward ? go(norm_fwd_kernel<T, V, G, K, kBlock, true, false>) : go(norm_bwd_kernel<T, V, G, K, kBlock, true, false>);
    c.forward ? go(norm_fwd_kernel<T, V, G, K, kBlock, false, kLoose>) : go(norm_bwd_kernel<T, V, G, K, kBlock, false, kLoose>);
}

template <class T, int V, bool kLoose>
void launch_rows(const Call &c)
{
    const Spread s = spread_of((c.a.W + V - 1) / V);
    switch (s.G) {
    case 1: return launch_spread<T, V, 1, 1, kLoose>(c);
    case 2: return launch_spread<T, V, 2, 1, kLoose>(c);
    case 4: return launch_spread<T, V, 4, 1, kLoose>(c);
    case 8: return launch_spread<T, V, 8, 1, kLoose>(c);
    case 16: return launch_spread<T, V, 16, 1, kLoose>(c);
    case 32: return launch_spread<T, V, 32, 1, kLoose>(c);
    case 64:
        return s.K == 1   ? launch_spread<T, V, 64, 1, kLoose>(c)
               : s.K == 2 ? launch_spread<T, V, 64, 2, kLoose>(c)
               : s.K == 3 ? launch_spread<T, V, 64, 3, kLoose>(c)
                          : launch_spread<T, V, 64, 4, kLoose>(c);
    case 256:
        return s.K == 2 ? launch_spread<T, V, 256, 2, kLoose>(c) : s.K == 4 ? launch_spread<T, V, 256, 4, kLoose>(c) : launch_spread<T, V, 256, 8, kLoose>(c);
    }
    if (c.forward) norm_fwd_wide_kernel<T><<<(uint32_t)(c.a.N < kMostWide ? c.a.N : kMostWide), kWide, 0, c.st>>>(c.a);
    else norm_bwd_wide_kernel<T><<<c.parts, kWide, 0, c.st>>>(c.a);
}

// Rows of less than 16 bytes, value by value: up to 4 in a lane with as few idle places as possible (2^20 rows of 6 fp16 values, two lanes of three:
// 9.6 us forward, eight lanes 16).
template <class T>
void launch_narrow(const Call &c)
{
    const uint32_t W = c.a.W;
    if (W == 1) return launch_spread<T, 1, 1, 1, false>(c);
    if (W == 2) return launch_spread<T, 1, 2, 1, false>(c);
    if (W == 3) return launch_spread<T, 1, 1, 3, false>(c);
    if constexpr (sizeof(T) == 2) {
        if (W == 4) return launch_spread<T, 1, 1, 4, false>(c);
        if (W <= 6) return launch_spread<T, 1, 2, 3, false>(c);
        launch_spread<T, 1, 2, 4, false>(c);
    }
}

// Vectors of 16 bytes, whether they are aligned and divide a row or not; rows of less than 16 bytes value by value.  Unaligned vectors / single
// values in us, forward and backward: 2^20 rows of 37 fp32 values 58 / 76 and 106 / 113; 8192 of 4095 44 / 105 and 89 / 283; 2^18 of 999 bf16
// values 218 / 246 and 324 / 437; 8192 of 4095 33 / 92 and 62 / 243; 2^22 of 33 fp16 values 133 / 187 and 246 / 272; 2^21 of 100, eight bytes at a
// time, 182 / 210 and 312 / 278.
template <class T>
void launch(const Call &c)
{
    constexpr int V = 16 / sizeof(T);
    const Norm &a = c.a;
    const bool aligned = a.W % V == 0 && rows_aligned(a.x, a.ldx, c.dtype, 16) && (c.forward || rows_aligned(a.dy, a.lddy, c.dtype, 16)) &&
                         (!a.out || rows_aligned(a.out, a.ldo, c.dtype, 16));
    if (aligned) launch_rows<T, V, false>(c);
    else if (a.W >= V) launch_rows<T, V, true>(c);
    else launch_narrow<T>(c);
}

void launch(const Call &c)
{
    if (c.dtype == DG_F32) launch<float>(c);
    else if (c.dtype == DG_F16) launch<f16>(c);
    else launch<bf16>(c);
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
    launch({{x, nullptr, y, gamma, beta, nullptr, ldx, 0, ldy, N, W, eps, 1.0f / (float)W}, dtype, 0, true, (hipStream_t)stream});
    return dg::launch_status(who);
}

extern "C" size_t dg_layer_norm_bwd_workspace_bytes(uint64_t N, uint32_t W) { return (size_t)parts_of(N, W) * 2 * W * sizeof(float); }

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
    const bool weights = dgamma || dbeta;
    if (!weights && (!dx || !N)) return DG_OK;
    const size_t need = weights ? dg_layer_norm_bwd_workspace_bytes(N, W) : 0;
    DG_REQUIRE(need == 0 || (ws && dg::aligned(ws, 16) && ws_bytes >= need), DG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need,
               ws ? ws_bytes : 0);
    float *part = weights ? (float *)ws : nullptr;
    const uint32_t parts = parts_of(N, W);
    if (N) launch({{x, dy, dx, gamma, nullptr, part, ldx, lddy, lddx, N, W, eps, 1.0f / (float)W}, dtype, parts, false, (hipStream_t)stream});
    if (weights)
        norm_fold_kernel<<<(2 * W + kFoldColumns - 1) / kFoldColumns, kFoldColumns * kFoldRuns, 0, (hipStream_t)stream>>>(part, parts, W, dgamma, dbeta);
    return dg::launch_status(who);
}
