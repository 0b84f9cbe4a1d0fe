// Root-mean-square norm of rows, forward, with the residual added before and the result in the rows' type or in 8 bits.  Internal.
//   t = x + r, rounded to the rows' type (what the next block adds to);  y = t s gamma,  s = 1 / sqrt(mean(t^2) + eps).
//
// Bound by memory: a row is read once into registers and summed there, as in layer norm, and everything that depends on it is stored from there.
// 8192 rows of 4096 bf16 values with the residual: 47 us, 5.7 TB/s of what goes in and out; 16384 of 2048 into 8 bits 49 us, 4.8 TB/s.  1024 rows of 32: 2.9 us, a launch.
#pragma once
#include "rows_vectors.h"

namespace dg_rms {

using namespace dg_rows;

constexpr int kBlock = 256, kWide = 1024;

struct Rms {
    const void *x, *r, *dy, *dt;
    void *t, *out;                  // sum; y, q or dx (each NULL: not wanted)
    const float *gamma;
    uint8_t *scales;
    float *part;                    // backward: [workgroups][W], or NULL
    uint64_t ldx, ldr, lddy, lddt, ldt, ldo, lds, N;
    uint32_t W;
    float eps;
};

// What a call makes of its rows: the norm in their type, the norm in 8 bits, or 8 bits of the rows themselves
enum Made { kNormed, kNormed8, kPlain8 };

// ------------------------------------------------------------------------------ 8 bits
// A block of 128 columns has the smallest power of two for a scale that leaves no value beyond 448, the largest of e4m3: the matrix
// instruction applies such scales by itself, and values keep all their bits, where a scale of any size would round twice.
constexpr int kScaled = 128;

__device__ __forceinline__ float finite_size(float v)
{
    const float a = fabsf(v);
    return a <= 3.402823466e38f ? a : 0.0f;
}

// exponent byte of the scale: 448 = 1.75 2^8
__device__ __forceinline__ uint32_t scale_byte(float largest)
{
    const uint32_t bits = __float_as_uint(largest), e = bits >> 23;
    const uint32_t up = (bits & 0x7fffff) > 0x600000 ? 1 : 0;
    return e + up > 8 ? e + up - 8 : 0;
}

// two values in the low half of a word; infinities become NaN, which e4m3 has
__device__ __forceinline__ uint32_t pair8(float a, float b, int exponent)
{
    const float nan = __uint_as_float(0x7fc00000u);
    a = __builtin_isinf(a) ? nan : ldexpf(a, exponent);
    b = __builtin_isinf(b) ? nan : ldexpf(b, exponent);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}

template <int V>
__device__ __forceinline__ void bytes_of(const float (&v)[V], int exponent, uint8_t (&out)[V])
{
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const uint32_t two = pair8(v[i], i + 1 < V ? v[i + 1] : 0.0f, exponent);
        out[i] = (uint8_t)two;
        if (i + 1 < V) out[i + 1] = (uint8_t)(two >> 8);
    }
}

template <int G>
__device__ __forceinline__ float group_max(float v)
{
    if (G >= 2) v = fmaxf(v, exchanged<0xb1>(v));
    if (G >= 4) v = fmaxf(v, exchanged<0x4e>(v));
    if (G >= 8) v = fmaxf(v, exchanged<0x141>(v));
    if (G >= 16) v = fmaxf(v, exchanged<0x140>(v));
    if (G >= 32) v = fmaxf(v, __shfl_xor(v, 16));
    return v;
}

// What is rounded to 8 bits is known to some 2^-40 before: fp32 arithmetic would leave one value in half a million on the other side of a step of e4m3, a sixteenth of it away.  Sums of squares
// are taken in 64 bits, the scale and its products in two parts of 32.  The nearest fp32 number to the sum of the two serves as long as it is no border itself: halfway between two of e4m3, or 448 times
// a power of two, where the scale changes.  Borders end in 19 zeros.  There (and at 0) it is rounded to odd, which leaves it on the border's side that the sum is on.  (All of this of values from
// 2^-100 on, below which fp32 has no room for the second part.)  16384 rows of 2048: 49.1 us; with every value rounded to odd 51.1, with none 48.4, but then one in two million falls on the wrong side.
template <int C>
__device__ __forceinline__ double exchanged2(double v)
{
    struct Halves { float lo, hi; };
    Halves h = __builtin_bit_cast(Halves, v);
    h.lo = exchanged<C>(h.lo), h.hi = exchanged<C>(h.hi);
    return __builtin_bit_cast(double, h);
}

template <int G>
__device__ __forceinline__ double group_sum2(double v)
{
    if (G >= 2) v += exchanged2<0xb1>(v);
    if (G >= 4) v += exchanged2<0x4e>(v);
    if (G >= 8) v += exchanged2<0x141>(v);
    if (G >= 16) v += exchanged2<0x140>(v);
    if (G >= 32) v += __shfl_xor(v, 16);
    if (G >= 64) v += __shfl_xor(v, 32);
    return v;
}

template <int G, int kThreads>
__device__ __forceinline__ double row_sum2(double v, double *red)
{
    v = group_sum2<(G < dg::kWave ? G : dg::kWave)>(v);
    if (G <= dg::kWave) return v;
    __syncthreads();                                // the last use of red is over
    if (threadIdx.x % dg::kWave == 0) red[threadIdx.x / dg::kWave] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / dg::kWave; ++w) v += red[w];
    return v;
}

// a + b, |b| <= |a|, towards 0 and then to the odd one if that is not all of it
__device__ __forceinline__ float odd_sum(float a, float b)
{
#pragma clang fp contract(off)
    const float sum = a + b, left = b - (sum - a);
    const uint32_t bits = __float_as_uint(sum), beyond = (bits ^ __float_as_uint(left)) >> 31;
    return left != 0.0f ? __uint_as_float((bits - beyond) | 1u) : sum;
}

struct Scale {
    float s, rest;
    // 1 / sqrt(squares / W + eps): fp32, then a step of Newton's
    __device__ __forceinline__ Scale(double squares, uint32_t W, float eps)
    {
        const double m = squares / W + eps;
        const float s0 = 1.0f / sqrtf((float)m);
        const double off = fma(-m * s0, (double)s0, 1.0), exact = fma(0.5 * s0, off, (double)s0);
        s = off == off ? (float)exact : s0;         // of infinities and NaN as in fp32
        rest = off == off ? (float)(exact - s) : 0.0f;
    }
    template <bool kOdd>
    __device__ __forceinline__ float times(float x, float gamma) const
    {
#pragma clang fp contract(off)
        const float p = x * s, p_off = fmaf(x, rest, fmaf(x, s, -p)), y = p * gamma, y_off = fmaf(p_off, gamma, fmaf(p, gamma, -y));
        return kOdd ? odd_sum(y, y_off) : y + y_off;
    }
    // x <- what is to be rounded to 8 bits
    template <int V>
    __device__ __forceinline__ void apply(float (&x)[V], const float (&gamma)[V]) const
    {
        float y[V];
        uint32_t least = ~0u;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            y[v] = times<false>(x[v], gamma[v]);
            const uint32_t end = __float_as_uint(y[v]) & 0x7ffff;
            least = end < least ? end : least;
        }
        if (least == 0)
#pragma unroll
            for (int v = 0; v < V; ++v) y[v] = times<true>(x[v], gamma[v]);
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = y[v];
    }
};

// A row in registers to 8 bits.  A vector's lane stores it at its own place; of a row's last vector, where it begins early, only what is its own.
template <int V, int G, int K, bool kLoose>
__device__ __forceinline__ void store8(const float (&y)[K][V], const Rms &a, uint64_t row, bool held, uint32_t lane)
{
    constexpr int kLanes = G * V >= kScaled ? kScaled / V : G;      // that share a scale
    constexpr bool kOne = G * V < kScaled && K > 1;                 // all vectors of a lane, in rows of a few values
    float largest[K];
    uint32_t c;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        largest[k] = 0.0f;
        const int from = skipped<V, kLoose>(a.W, (k * G + lane) * V);
        if (inside<V>(a.W, lane, k, G, c))
#pragma unroll
            for (int v = 0; v < V; ++v) largest[k] = kLoose && v < from ? largest[k] : fmaxf(largest[k], finite_size(y[k][v]));
    }
    if (kOne)
#pragma unroll
        for (int k = 1; k < K; ++k) largest[0] = fmaxf(largest[0], largest[k]);
    uint8_t *q = (uint8_t *)a.out + row * a.ldo, *scales = a.scales + row * a.lds;
    uint32_t byte = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (!kOne || k == 0) byte = scale_byte(group_max<kLanes>(largest[k]));
        if (!inside<V>(a.W, lane, k, G, c) || !held) continue;
        if (lane % kLanes == 0 && (!kOne || k == 0)) scales[c / kScaled] = (uint8_t)byte;
        Pack<uint8_t, V> out;
        bytes_of<V>(y[k], 127 - (int)byte, out.v);
        const int from = skipped<V, kLoose>(a.W, c);
        if (kLoose && from) {
            uint8_t *to = q + begin_of<V, kLoose>(a.W, c);
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v >= from) to[v] = out.v[v];
        } else *reinterpret_cast<Pack<uint8_t, V> *>(q + c) = out;
    }
}

// ------------------------------------------------------------------------------ forward
// The norm of rows that layer norm's kernels would take the same way: workgroups side by side, the next row on its way where a lane has several vectors.
template <class T, int V, int G, int K, int kThreads, bool kStreamed, bool kLoose, bool kResidual, Made kMade>
__global__ void __launch_bounds__(kThreads)
rms_fwd_kernel(Rms a)
{
    constexpr int R = kThreads / G;
    constexpr bool kAhead = K > 1;
    __shared__ float red[kThreads / dg::kWave][1];
    __shared__ double red2[kMade == kNormed8 ? kThreads / dg::kWave : 1];
    const uint32_t lane = threadIdx.x % G;
    float gamma[K][V];
    if (kMade != kPlain8) weights<V, G, K, kLoose>(a.gamma, 1.0f, a, lane, gamma);
    uint64_t row = (uint64_t)blockIdx.x * R + threadIdx.x / G;
    Pack<T, V> next[K], next_r[K];
    auto fetch = [&] {
        read<T, V, G, K, kStreamed, kLoose, kAhead>(a.x, a.ldx, row, a, lane, next);
        if (kResidual) read<T, V, G, K, kStreamed, kLoose, kAhead>(a.r, a.ldr, row, a, lane, next_r);
    };
    if (kAhead) fetch();
    for (uint64_t row0 = (uint64_t)blockIdx.x * R; row0 < a.N; row0 += (uint64_t)gridDim.x * R) {
        if (!kAhead) fetch();
        if (kResidual)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) next[k].v[v] = (T)((float)next[k].v[v] + (float)next_r[k].v[v]);
        float x[K][V];
        widen<T, V, G, K, kAhead>(next, a, lane, x);
        Pack<T, V> total[K];
        if (kResidual)
#pragma unroll
            for (int k = 0; k < K; ++k) total[k] = next[k];
        const uint64_t now = row;
        const bool held = now < a.N;
        row += (uint64_t)gridDim.x * R;
        if (kAhead) fetch();
        uint32_t c;
        if (kMade == kNormed8) {
            double sum = 0.0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int from = skipped<V, kLoose>(a.W, (k * G + lane) * V);
#pragma unroll
                for (int v = 0; v < V; ++v) sum = kLoose && v < from ? sum : fma((double)x[k][v], (double)x[k][v], sum);
            }
            const Scale s(row_sum2<G, kThreads>(sum, red2), a.W, a.eps);
#pragma unroll
            for (int k = 0; k < K; ++k) s.apply(x[k], gamma[k]);
        } else if (kMade != kPlain8) {
            float sum[1] = {0.0f};
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int from = skipped<V, kLoose>(a.W, (k * G + lane) * V);
#pragma unroll
                for (int v = 0; v < V; ++v) sum[0] += kLoose && v < from ? 0.0f : x[k][v] * x[k][v];
            }
            row_sums<G, kThreads, 1>(sum, red);
            const float s = 1.0f / sqrtf(sum[0] / (float)a.W + a.eps);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) x[k][v] = x[k][v] * s * gamma[k][v];
        }
        // stores come after the sums, for which all lanes have read the row: the sum may lie where x or r does
        if (kResidual && a.t) {
            T *t = (T *)a.t + now * a.ldt;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (inside<V>(a.W, lane, k, G, c) && held) {
                    T *to = t + begin_of<V, kLoose>(a.W, c);
                    if constexpr (kStreamed) store_streamed<T, V>(to, total[k]);
                    else if constexpr (kLoose) *reinterpret_cast<typename loose<T>::u4 *>(to) = __builtin_bit_cast(typename loose<T>::u4, total[k]);
                    else *reinterpret_cast<Pack<T, V> *>(to) = total[k];
                }
        }
        if constexpr (kMade != kNormed) store8<V, G, K, kLoose>(x, a, now, held, lane);
        else {
            T *y = (T *)a.out + now * a.ldo;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (inside<V>(a.W, lane, k, G, c) && held) write<T, V, kStreamed, kLoose>(y + begin_of<V, kLoose>(a.W, c), x[k]);
        }
    }
}

// Rows too wide for the registers of a workgroup: read again from the caches, a workgroup per row.
template <class T>
__device__ __forceinline__ float wide_scale(const T *x, const T *r, const Rms &a, float (*red)[1])
{
    float sum[1] = {0.0f};
    for (uint32_t c = threadIdx.x; c < a.W; c += kWide) {
        const float t = r ? (float)(T)((float)x[c] + (float)r[c]) : (float)x[c];
        sum[0] += t * t;
    }
    row_sums<kWide, kWide, 1>(sum, red);
    return 1.0f / sqrtf(sum[0] / (float)a.W + a.eps);
}

template <class T>
__device__ __forceinline__ Scale wide_scale2(const T *x, const T *r, const Rms &a, double *red)
{
    double sum = 0.0;
    for (uint32_t c = threadIdx.x; c < a.W; c += kWide) {
        const double t = r ? (double)(float)(T)((float)x[c] + (float)r[c]) : (double)(float)x[c];
        sum = fma(t, t, sum);
    }
    return Scale(row_sum2<kWide, kWide>(sum, red), a.W, a.eps);
}

template <class T, Made kMade>
__global__ void __launch_bounds__(kWide)
rms_fwd_wide_kernel(Rms a)
{
    __shared__ float red[kWide / dg::kWave][1];
    __shared__ double red2[kMade == kNormed8 ? kWide / dg::kWave : 1];
    const uint32_t wave = threadIdx.x / dg::kWave, lane = threadIdx.x % dg::kWave;
    for (uint64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.ldx, *r = a.r ? (const T *)a.r + row * a.ldr : nullptr;
        T *t = a.t ? (T *)a.t + row * a.ldt : nullptr;
        float s = 1.0f;
        Scale exact(1.0, 1, 0.0f);
        if (kMade == kNormed) s = wide_scale<T>(x, r, a, red);
        if (kMade == kNormed8) exact = wide_scale2<T>(x, r, a, red2);
        // a wavefront takes a block of columns, two to a lane; a lane reads the places that it stores to, and no others
        for (uint32_t c0 = wave * kScaled; c0 < a.W; c0 += kWide / dg::kWave * kScaled) {
            float y[2];
            float largest = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t c = c0 + 2 * lane + i;
                y[i] = 0.0f;
                if (c >= a.W) continue;
                const T sum = r ? (T)((float)x[c] + (float)r[c]) : x[c];
                y[i] = (float)sum;
                if (kMade == kNormed) y[i] = y[i] * s * (a.gamma ? a.gamma[c] : 1.0f);
                if (kMade == kNormed8) y[i] = exact.times<true>(y[i], a.gamma ? a.gamma[c] : 1.0f);
                if (t) t[c] = sum;
                if (kMade == kNormed) ((T *)a.out + row * a.ldo)[c] = (T)y[i];
                largest = fmaxf(largest, finite_size(y[i]));
            }
            if (kMade == kNormed) continue;
            largest = group_max<32>(largest);
            const uint32_t byte = scale_byte(fmaxf(largest, __shfl_xor(largest, 32)));
            if (lane == 0) a.scales[row * a.lds + c0 / kScaled] = (uint8_t)byte;
            uint8_t q[2];
            bytes_of<2>(y, 127 - (int)byte, q);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (c0 + 2 * lane + i < a.W) ((uint8_t *)a.out + row * a.ldo)[c0 + 2 * lane + i] = q[i];
        }
    }
}

// ------------------------------------------------------------------------------ launch
// as many workgroups as the chip holds at once where a lane has one vector
constexpr uint64_t kMostBlocks = 2048;
// of rows too wide for registers: far from the 2^32 lanes from which a grid is cut short
constexpr uint64_t kMostWide = 1 << 16;

struct Call {
    Rms a;
    uint32_t dtype, parts;
    hipStream_t st;
};

// `Way` has launch<T, V, G, K, kStreamed, kLoose>(call, grid of the forward pass) and launch_wide<T>(call)
template <class Way, class T, int V, int G, int K, bool kLoose>
void launch_spread(const Call &c)
{
    const uint64_t all = (c.a.N + kBlock / G - 1) / (kBlock / G);
    const uint32_t grid = (uint32_t)(all < kMostBlocks ? all : kMostBlocks);
    if constexpr (V * sizeof(T) == 16 && !kLoose)
        if (c.a.N * c.a.W * sizeof(T) >= kStreamedBytes) return Way::template launch<T, V, G, K, true, false>(c, grid);
    Way::template launch<T, V, G, K, false, kLoose>(c, grid);
}

template <class Way, class T, int V, bool kLoose>
void launch_rows(const Call &c)
{
    const Spread s = spread_of((c.a.W + V - 1) / V);
    switch (s.G) {
    case 1: return launch_spread<Way, T, V, 1, 1, kLoose>(c);
    case 2: return launch_spread<Way, T, V, 2, 1, kLoose>(c);
    case 4: return launch_spread<Way, T, V, 4, 1, kLoose>(c);
    case 8: return launch_spread<Way, T, V, 8, 1, kLoose>(c);
    case 16: return launch_spread<Way, T, V, 16, 1, kLoose>(c);
    case 32: return launch_spread<Way, T, V, 32, 1, kLoose>(c);
    case 64:
        return s.K == 1   ? launch_spread<Way, T, V, 64, 1, kLoose>(c)
               : s.K == 2 ? launch_spread<Way, T, V, 64, 2, kLoose>(c)
               : s.K == 3 ? launch_spread<Way, T, V, 64, 3, kLoose>(c)
                          : launch_spread<Way, T, V, 64, 4, kLoose>(c);
    case 256:
        return s.K == 2   ? launch_spread<Way, T, V, 256, 2, kLoose>(c)
               : s.K == 4 ? launch_spread<Way, T, V, 256, 4, kLoose>(c)
                          : launch_spread<Way, T, V, 256, 8, kLoose>(c);
    }
    Way::template launch_wide<T>(c);
}

// rows of less than 16 bytes, value by value
template <class Way, class T>
void launch_narrow(const Call &c)
{
    const uint32_t W = c.a.W;
    if (W == 1) return launch_spread<Way, T, 1, 1, 1, false>(c);
    if (W == 2) return launch_spread<Way, T, 1, 2, 1, false>(c);
    if (W == 3) return launch_spread<Way, T, 1, 1, 3, false>(c);
    if constexpr (sizeof(T) == 2) {
        if (W == 4) return launch_spread<Way, T, 1, 1, 4, false>(c);
        if (W <= 6) return launch_spread<Way, T, 1, 2, 3, false>(c);
        launch_spread<Way, T, 1, 2, 4, false>(c);
    }
}

// aligned: every array of the rows' type can be loaded and stored 16 bytes at a time
template <class Way, class T>
void launch_type(const Call &c, bool aligned)
{
    constexpr int V = 16 / sizeof(T);
    if (aligned && c.a.W % V == 0) launch_rows<Way, T, V, false>(c);
    else if (c.a.W >= V) launch_rows<Way, T, V, true>(c);
    else launch_narrow<Way, T>(c);
}

template <class Way>
void launch(const Call &c, bool aligned)
{
    if (c.dtype == DG_F32) launch_type<Way, float>(c, aligned);
    else if (c.dtype == DG_F16) launch_type<Way, f16>(c, aligned);
    else launch_type<Way, bf16>(c, aligned);
}

// an array that may be missing
inline bool may_align(const void *p, uint64_t ld, uint32_t dtype) { return !p || rows_aligned(p, ld, dtype, 16); }

inline int check_forward(const char *who, const Rms &a, uint32_t dtype)
{
    if (int rc = check_rows(who, a.x, a.ldx, a.W, dtype)) return rc;
    DG_REQUIRE(a.r || !a.t, DG_ERR_ARG, "%s: a sum without a residual", who);
    if (a.r)
        if (int rc = check_rows(who, a.r, a.ldr, a.W, dtype)) return rc;
    if (a.t)
        if (int rc = check_rows(who, a.t, a.ldt, a.W, dtype)) return rc;
    DG_REQUIRE(dg::aligned(a.gamma, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    return DG_OK;
}

}  // namespace dg_rms
