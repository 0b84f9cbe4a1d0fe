// Rows held in the registers of the lanes that share them: how a row is spread, loads, stores and sums.  Internal; what takes `a` takes any description
// of a call that has N rows of W values.
#pragma once
#include <cmath>
#include "rows_common.h"

namespace dg_rows {

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
template <class T, int V, int G, int K, bool kStreamed, bool kLoose, bool kAhead, class A>
__device__ __forceinline__ void read(const void *p, uint64_t ld, uint64_t row, const A &a, uint32_t lane, Pack<T, V> (&out)[K])
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

template <class T, int V, int G, int K, bool kAhead, class A>
__device__ __forceinline__ void widen(const Pack<T, V> (&in)[K], const A &a, uint32_t lane, float (&out)[K][V])
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
template <int V, int G, int K, bool kLoose, class A>
__device__ __forceinline__ void weights(const float *p, float none, const A &a, uint32_t lane, float (&out)[K][V])
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

// How a row of n vectors is spread: up to 64 over as many lanes, rounded up to a power of two; several per lane would leave fewer lanes
// idle, but a load then takes parts of many lines, which loads past the caches fetch again (48 bf16 values a row, two lanes of three
// vectors: 1.9 TB/s forward, eight lanes 5.5).  Then a wavefront with up to 4 each, then a workgroup with up to 8.
struct Spread { int G, K; };

inline Spread spread_of(uint32_t n)
{
    int G = 1;
    while (G < 64 && (uint32_t)G < n) G *= 2;
    for (int K = 1; K <= 4; ++K)
        if (n <= (uint32_t)(G * K)) return {G, K};
    for (int K = 2; K <= 8; K *= 2)
        if (n <= 256u * K) return {256, K};
    return {0, 0};
}

inline int check_norm(const char *who, uint64_t N, uint32_t W, float eps, uint32_t dtype)
{
    DG_REQUIRE(known_type(dtype), DG_ERR_ARG, "%s: unknown element type %u", who, dtype);
    DG_REQUIRE(W >= 1 && eps >= 0.0f && std::isfinite(eps), DG_ERR_ARG, "%s: W must be positive, eps finite and not negative", who);
    DG_REQUIRE(N <= 1ull << 32 && W <= 1u << 20 && N * W <= 1ull << 39, DG_ERR_UNSUPPORTED, "%s: more than 2^32 rows, 2^20 values a row or 2^39 values", who);
    return DG_OK;
}

inline int check_rows(const char *who, const void *p, uint64_t ld, uint32_t W, uint32_t dtype)
{
    DG_REQUIRE(p && dg::aligned(p, item_bytes(dtype)), DG_ERR_ARG, "%s: null or misaligned pointer", who);
    DG_REQUIRE(ld >= W && ld <= 1ull << 40, DG_ERR_ARG, "%s: rows of %u values lie %llu apart", who, W, (unsigned long long)ld);
    return DG_OK;
}

}  // namespace dg_rows
