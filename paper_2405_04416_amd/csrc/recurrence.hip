// Gated linear recurrence along sequences of rows, channel by channel:
//   a = 1 / (1 + e^-z),  c = 1 - a = 1 / (1 + e^z),  h_t = a_t h_{t-1} + c_t u_t,  y_t = h_t.
// Its backward pass: G_t = dy_t + a_{t+1} G_{t+1} from the last token back, du = c G, dz = a c G (h_{t-1} - u_t), dh0 = a_0 G_0.
// From |z| = 87 on a and c are exactly 0 and 1: what a gate of 0 multiplies is not looked at, be it infinite or NaN.
//
// Tokens have a place in the order in which they are gone through: their row, or N - 1 - row back to front.  The forward pass
// keeps the state before every kKeep-th place in fp32; the backward pass computes the states between them again.
//
// Bound by memory: 3 values moved per element forward, 5 backward, for some 16 and 43 operations, an exp2 and a reciprocal at a quarter of
// the rate for each time that a gate is computed.  Many sequences: a lane runs through a sequence's tokens, 16 of them on their way at a
// time.  2^17 rays of 64 samples, 32 channels in fp16: forward 313 us (5.1 TB/s), backward 507 (5.3).  Few long ones: tiles that tell each
// other what they do to a state; each value is still read once.  One sequence of 2^17 tokens, 256 channels in bf16: forward 69 us (2.9 TB/s);
// four of 16 384, 1024 channels: 115 (3.5) and 167 (4.0).  What keeps tiles from 6 TB/s: two workgroups per compute unit
// load, compute, listen and store in turn, and the gates are computed twice and three times.
//
// 16-bit values go in pairs where width and alignment allow it, else one by one: 2^16 sequences of 64 tokens in bf16, 38 / 37 channels: 215 / 231 us and
// 374 / 398; four of 16 384, 1000 / 999 channels, in tiles: 128 / 147 and 201 / 230.  Rows of less than a line: 2^17 rays of 64 samples in fp16, 16 channels:
// 172 us (4.7 TB/s) and 270 (5.0), 8 channels 123 (3.3) and 185 (3.6).
#include <type_traits>
#include "rows_common.h"

namespace {

using namespace dg_rows;

constexpr int kBlock = 256, kKeep = 16;
constexpr float kLeast = 1.17549435e-38f;       // the smallest normal number
constexpr float kShut = 87.0f;                  // up to here e^z, e^-z, a and c are normal numbers
constexpr float kLog2e = 1.44269504f;

struct Gate { float a, c; };

// Both sides of an open gate.  The argument of exp2 is rounded, so that the smaller one is off by some |z| + 3 half units of its own.
__device__ __forceinline__ Gate gate(float z)
{
    const float e = __builtin_amdgcn_exp2f(z * -kLog2e), a = __builtin_amdgcn_rcpf(1.0f + e);
    return {a, e * a};
}

// V neighbouring values as they lie in memory, in one register until they are used: arrays of 16-bit values would be taken apart.
template <class T, int V>
struct Raw {
    static_assert(sizeof(T) * V <= 4, "one register");
    uint32_t bits;
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (sizeof(T) * V == 4) bits = *reinterpret_cast<const uint32_t *>(p);
        else bits = *reinterpret_cast<const uint16_t *>(p);
    }
    __device__ __forceinline__ float operator[](int v) const;
};
template <>
__device__ __forceinline__ float Raw<float, 1>::operator[](int) const { return __uint_as_float(bits); }
template <>
__device__ __forceinline__ float Raw<f16, 1>::operator[](int) const { return (float)__builtin_bit_cast(f16, (uint16_t)bits); }
template <>
__device__ __forceinline__ float Raw<f16, 2>::operator[](int v) const { return (float)__builtin_bit_cast(f16, (uint16_t)(v ? bits >> 16 : bits)); }
template <>
__device__ __forceinline__ float Raw<bf16, 1>::operator[](int) const { return __uint_as_float(bits << 16); }
template <>
__device__ __forceinline__ float Raw<bf16, 2>::operator[](int v) const { return __uint_as_float(v ? bits & 0xffff0000u : bits << 16); }

// Whether a wavefront has a shut gate among the tokens that it has loaded; they are then gone through looking at each gate.  By their
// bits, which without the sign order numbers by magnitude with infinity and NaN on top.
template <class T>
struct Bits;
template <>
struct Bits<float> { using type = uint32_t; static constexpr type kMagnitude = 0x7fffffffu, kShut = 0x42ae0000u; };
template <>
struct Bits<f16> { using type = uint16_t; static constexpr type kMagnitude = 0x7fffu, kShut = 0x5570u; };
template <>
struct Bits<bf16> { using type = uint16_t; static constexpr type kMagnitude = 0x7fffu, kShut = 0x42aeu; };

template <class T, int V, int M>
__device__ __forceinline__ bool any_shut(const Raw<T, V> (&z)[M])
{
    using B = typename Bits<T>::type;
    constexpr int n = 4 / sizeof(B);
    typedef B Vector __attribute__((ext_vector_type(n)));
    Vector most = 0;
#pragma unroll
    for (int k = 0; k < M; ++k) most = __builtin_elementwise_max(most, __builtin_bit_cast(Vector, z[k].bits) & (Vector)Bits<T>::kMagnitude);
    bool shut = false;
#pragma unroll
    for (int v = 0; v < V; ++v) shut = shut || most[v] >= Bits<T>::kShut;
    return __any(shut);
}

// The gate of a token, its input's share b = c u, and h_t.  kShutting: the gate may be shut.
struct Step { float a, c, b; };

template <bool kShutting>
__device__ __forceinline__ Step step_of(float z, float u)
{
    const Gate g = gate(z);
    if (!kShutting) return {g.a, g.c, g.c * u};
    const bool hold = z >= kShut, reset = z <= -kShut;
    return {reset ? 0.0f : g.a, reset ? 1.0f : hold ? 0.0f : g.c, reset ? u : hold ? 0.0f : g.c * u};
}

template <bool kShutting>
__device__ __forceinline__ float advance(const Step &s, float h)
{
    return kShutting && s.a == 0.0f ? s.b : fmaf(s.a, h, s.b);
}

// the gradient before a token from the one behind it
template <bool kShutting>
__device__ __forceinline__ float retreat(const Step &s, float G)
{
    return kShutting && s.a == 0.0f ? 0.0f : s.a * G;
}

// `a` is rounded: near 1 it and its c do not quite add up to 1, and what a state gains or loses by that adds up over the 1 / c tokens that it
// lives.  Over kKeep tokens that is 16 half units at most; a longer chain is written with the smaller share alone, as the value of
// the larger share plus the smaller share of the difference.  2^17 tokens with constant gates of z = 8 / 10 / 12: off by 2.4e-6 / 1.8e-6 / 2.0e-6 of the
// state, with a h + c u throughout by 5.5e-4 / 2.4e-3 / 5.3e-3.  The difference from a state that is infinite would make it NaN; where the end of
// some tokens shows that this may have happened they are gone through once more, kCareful, looking at each.  Finite states are the same both ways.
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.40282347e38f; }

template <bool kCareful>
__device__ __forceinline__ float advance_far(float z, float u, float h)
{
    const Gate g = gate(z);
    const bool more = z > 0.0f;
    const float next = fmaf(more ? g.c : -g.a, u - h, more ? h : u);
    if (!kCareful) return next;
    return fabsf(z) < kShut && finite(next) ? next : advance<true>(step_of<true>(z, u), h);
}

template <bool kCareful>
__device__ __forceinline__ float retreat_far(float z, float G)
{
    const Gate g = gate(z);
    const bool more = z > 0.0f;
    const float next = fmaf(more ? -g.c : g.a, G, more ? G : 0.0f);
    if (!kCareful) return next;
    return fabsf(z) < kShut && finite(next) ? next : retreat<true>(step_of<true>(z, 0.0f), G);
}

// What a stretch of tokens does to the state h before it: A h + B, A the product of its gates and D = 1 - A.  D is summed as what each token
// takes of h, so that it is precise where it is small.  x = code(A, D) is the smaller one of them, A as it is and D with its sign changed, -0 for a stretch that
// only holds.  x is +0 only if a gate of the stretch is 0, and A kLeast where it would be less, so that a state that is infinite or NaN gets
// through a long stretch as it does token by token; to a finite state that adds less than 2^-126 of itself.
__device__ __forceinline__ float code(float A, float D) { return A <= 0.5f ? A : -D; }

// A of x, rounded
__device__ __forceinline__ float share(float x) { return (int)__float_as_uint(x) < 0 ? 1.0f + x : x; }

// A h, as precise as x is, and B
__device__ __forceinline__ float join_finite(float x, float A, float h, float B) { return fmaf(x, h, B) + (A == x ? 0.0f : h); }

__device__ __forceinline__ bool anew(float x) { return __float_as_uint(x) == 0; }

__device__ __forceinline__ float join(float x, float h, float B)
{
    if (anew(x)) return B;
    const float A = share(x), next = join_finite(x, A, h, B);
    return finite(next) ? next : fmaf(A, h, B);
}

__device__ __forceinline__ float clamped(float A, bool zero) { return zero ? 0.0f : fmaxf(A, kLeast); }

// A and D with one more token.  Not kShutting: A is yet to be clamped.
template <bool kShutting>
__device__ __forceinline__ void extend(const Step &s, float &A, float &D)
{
    D = fmaf(s.c, A, D);
    A = kShutting ? clamped(A * s.a, A == 0.0f || s.a == 0.0f) : A * s.a;
}

struct Shape {
    uint64_t N;
    uint32_t n_seq, W, S;           // S: tokens of each sequence, where first is NULL
    const uint32_t *first;
    bool reverse;
    uint32_t n_tiles;               // 0: sequence by sequence
};

// The sequences in the order of their places: sequence(d, k) is the number of the k-th.
__device__ __forceinline__ uint32_t sequence(const Shape &d, uint32_t k) { return d.reverse ? d.n_seq - 1 - k : k; }

// places [begin, end) of the k-th sequence; never outside [0, N), whatever `first` holds
__device__ __forceinline__ void places(const Shape &d, uint32_t k, uint64_t &begin, uint64_t &end)
{
    if (!d.first) {
        begin = (uint64_t)k * d.S;
        end = begin + d.S;
        return;
    }
    const uint32_t seq = sequence(d, k);
    uint64_t b = d.first[seq], e = d.first[seq + 1];
    e = e < d.N ? e : d.N;
    b = b < e ? b : e;
    begin = d.reverse ? d.N - e : b;
    end = d.reverse ? d.N - b : e;
}

// how many sequences begin before place p
__device__ __forceinline__ uint32_t begun_before(const Shape &d, uint64_t p)
{
    if (!d.first) {
        const uint32_t k = p ? ((uint32_t)p - 1) / d.S + 1 : 0;         // places lie below 2^32
        return k < d.n_seq ? k : d.n_seq;
    }
    uint32_t lo = 0, hi = d.n_seq;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        uint64_t b, e;
        places(d, mid, b, e);
        if (b < p) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// V neighbouring channels of the row of a place, walked from token to token: an address at a time, not one for each token in registers
template <class T, int V>
struct Column {
    T *at;
    int64_t step;
    __device__ __forceinline__ Column(const Shape &d, const void *p, uint64_t ld, uint32_t c, uint64_t place)
    {
        at = (T *)p + (d.reverse ? d.N - 1 - place : place) * ld + c;
        step = d.reverse ? -(int64_t)ld : (int64_t)ld;
    }
};

template <class T, int V, int M, bool kFull>
__device__ __forceinline__ void load_tokens(Column<T, V> col, int n, Raw<T, V> (&out)[M])
{
#pragma unroll
    for (int k = 0; k < M; ++k) {
        out[k].load(col.at);
        if (kFull || k + 1 < n) col.at += col.step;         // past the last token: that one again
    }
}

// The compiler takes these values for unknown from here on: what was computed from them is computed again instead of kept in registers.
template <class T, int V, int M>
__device__ __forceinline__ void forget(Raw<T, V> (&a)[M])
{
#pragma unroll
    for (int k = 0; k < M; ++k) asm volatile("" : "+v"(a[k].bits));
}

template <int V>
__device__ __forceinline__ void get(const float *p, uint64_t at, float (&out)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = p ? p[at + v] : 0.0f;
}

template <int V>
__device__ __forceinline__ void put(float *p, uint64_t at, const float (&in)[V])
{
    if (!p) return;
#pragma unroll
    for (int v = 0; v < V; ++v) p[at + v] = in[v];
}

struct Fwd {
    const void *z, *u;
    void *y;
    uint64_t ldz, ldu, ldy;
    const float *h0;
    float *h_last, *states;
};

struct Bwd {
    const void *z, *u, *dy;
    void *dz, *du;
    uint64_t ldz, ldu, lddy, lddz, lddu;
    const float *h0, *states, *dh_last;
    float *dh0;
};

// Runs f(place, number of tokens) over [p, end) in pieces that end where states are kept.
template <class F>
__device__ __forceinline__ void in_pieces(uint64_t p, uint64_t end, F f)
{
    while (p < end) {
        const uint64_t next = (p / kKeep + 1) * kKeep;
        const int n = (int)((next < end ? next : end) - p);
        f(p, n);
        p += n;
    }
}

// kFar: the tokens are some of a longer chain
template <class T, int V, int M, bool kFull, bool kShutting, bool kFar>
__device__ __forceinline__ void advance_loaded(const Raw<T, V> (&z)[M], const Raw<T, V> (&u)[M], Column<T, V> y, int n, float (&h)[V])
{
#pragma unroll
    for (int k = 0; k < M; ++k)
        if (kFull || k < n) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                h[v] = kFar ? advance_far<kShutting>(z[k][v], u[k][v], h[v]) : advance<kShutting>(step_of<kShutting>(z[k][v], u[k][v]), h[v]);
            store<T, V>(y.at, h);
            y.at += y.step;
        }
}

// f(careful, state) from `state` on: without care first, unless `careful` asks for it at once
template <int V, class F>
__device__ __forceinline__ void with_care(bool careful, float (&state)[V], F f)
{
    if (!careful) {
        float to[V];
#pragma unroll
        for (int v = 0; v < V; ++v) to[v] = state[v];
        f(std::false_type(), to);
        bool good = true;
#pragma unroll
        for (int v = 0; v < V; ++v) good = good && finite(to[v]);
        careful = __any(!good);
        if (!careful)
#pragma unroll
            for (int v = 0; v < V; ++v) state[v] = to[v];
    }
    if (careful) f(std::true_type(), state);
}

template <class T, int V, int M, bool kFull, bool kFar>
__device__ __forceinline__ void advance_tokens(const Shape &d, const Fwd &f, uint32_t c, uint64_t p, int n, float (&h)[V])
{
    Raw<T, V> z[M], u[M];
    load_tokens<T, V, M, kFull>(Column<T, V>(d, f.z, f.ldz, c, p), n, z);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, f.u, f.ldu, c, p), n, u);
    const Column<T, V> y(d, f.y, f.ldy, c, p);
    const bool shutting = any_shut<T, V, M>(z);
    if (kFar)
        with_care<V>(shutting, h, [&](auto careful, float (&to)[V]) {
            if (careful) forget<T, V, M>(z), forget<T, V, M>(u);
            advance_loaded<T, V, M, kFull, careful.value, true>(z, u, y, n, to);
        });
    else if (shutting) advance_loaded<T, V, M, kFull, true, false>(z, u, y, n, h);
    else advance_loaded<T, V, M, kFull, false, false>(z, u, y, n, h);
}

// y of places [p, end) of a sequence from the state before them, and the states that are kept
template <class T, int V>
__device__ __forceinline__ void advance_places(const Shape &d, const Fwd &f, uint32_t c, uint64_t p, uint64_t end, float (&h)[V])
{
    in_pieces(p, end, [&](uint64_t q, int n) {
        if (q % kKeep == 0) put<V>(f.states, q / kKeep * d.W + c, h);
        if (n == kKeep) advance_tokens<T, V, kKeep, true, true>(d, f, c, q, n, h);
        else if (n == 1) advance_tokens<T, V, 1, true, true>(d, f, c, q, n, h);
        else advance_tokens<T, V, kKeep, false, true>(d, f, c, q, n, h);
    });
}

// the states before the tokens less their inputs, h_{t-1} - u_t
template <class T, int V, int M, bool kShutting>
__device__ __forceinline__ void steps_taken(const Raw<T, V> (&z)[M], const Raw<T, V> (&u)[M], float (&h)[V], float (&less)[M][V])
{
#pragma unroll
    for (int k = 0; k < M; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float uu = u[k][v];
            less[k][v] = h[v] - uu;
            h[v] = advance<kShutting>(step_of<kShutting>(z[k][v], uu), h[v]);
        }
}

// The gradients of loaded tokens, last first.  The gates are computed again: keeping a, c and a c (h_{t-1} - u) from the way forwards costs
// 96 registers where this takes 48, and half of the wavefronts.
template <class T, int V, int M, bool kFull, bool kShutting, bool kFar>
__device__ __forceinline__ void retreat_loaded(const Raw<T, V> (&z)[M], const Raw<T, V> (&dy)[M], const float (&less)[M][V], Column<T, V> dz,
                                               Column<T, V> du, int n, float (&G)[V])
{
#pragma unroll
    for (int k = M - 1; k >= 0; --k)
        if (kFull || k < n) {
            float oz[V], ou[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Step s = step_of<kShutting>(z[k][v], 0.0f);
                G[v] += dy[k][v];
                ou[v] = kShutting && s.c == 0.0f ? 0.0f : s.c * G[v];
                G[v] = kFar ? retreat_far<kShutting>(z[k][v], G[v]) : retreat<kShutting>(s, G[v]);
                oz[v] = kShutting && (s.c == 0.0f || s.a == 0.0f) ? 0.0f : s.c * less[k][v] * G[v];
            }
            store<T, V>(dz.at, oz);
            store<T, V>(du.at, ou);
            dz.at -= dz.step;
            du.at -= du.step;
        }
}

template <class T, int V, int M, bool kFull, bool kFar>
__device__ __forceinline__ void retreat_tokens(const Shape &d, const Bwd &b, uint32_t c, uint64_t p, int n, float (&h)[V], float (&G)[V])
{
    Raw<T, V> z[M], u[M], dy[M];
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.z, b.ldz, c, p), n, z);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.u, b.ldu, c, p), n, u);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.dy, b.lddy, c, p), n, dy);
    const Column<T, V> dz(d, b.dz, b.lddz, c, p + n - 1), du(d, b.du, b.lddu, c, p + n - 1);      // the last token first
    float less[M][V];
    const bool shutting = any_shut<T, V, M>(z);
    if (shutting) steps_taken<T, V, M, true>(z, u, h, less);
    else steps_taken<T, V, M, false>(z, u, h, less);
    forget<T, V, M>(z);
    if (kFar)
        with_care<V>(shutting, G, [&](auto careful, float (&to)[V]) {
            if (careful) forget<T, V, M>(z), forget<T, V, M>(dy);
            retreat_loaded<T, V, M, kFull, careful.value, true>(z, dy, less, dz, du, n, to);
        });
    else if (shutting) retreat_loaded<T, V, M, kFull, true, false>(z, dy, less, dz, du, n, G);
    else retreat_loaded<T, V, M, kFull, false, false>(z, dy, less, dz, du, n, G);
}

// dz and du of places [p, end) of the sequence that begins at place `begin`, from the gradient G behind them
template <class T, int V>
__device__ __forceinline__ void retreat_places(const Shape &d, const Bwd &b, uint32_t seq, uint32_t c, uint64_t begin, uint64_t p, uint64_t end, float (&G)[V])
{
    while (end > p) {
        const uint64_t keep = (end - 1) / kKeep, q = keep * kKeep > p ? keep * kKeep : p;
        const int n = (int)(end - q);
        float h[V];
        if (q == begin) get<V>(b.h0, (uint64_t)seq * d.W + c, h);
        else get<V>(b.states, keep * d.W + c, h);
        if (n == kKeep) retreat_tokens<T, V, kKeep, true, true>(d, b, c, q, n, h, G);
        else if (n == 1) retreat_tokens<T, V, 1, true, true>(d, b, c, q, n, h, G);
        else retreat_tokens<T, V, kKeep, false, true>(d, b, c, q, n, h, G);
        end = q;
    }
}

// ------------------------------------------------------------------ a lane per sequence and V channels

// of `count` sequences from place `from` on
__device__ __forceinline__ bool lane_place(const Shape &d, uint32_t V, uint32_t from, uint32_t count, uint32_t &k, uint32_t &c)
{
    const uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const uint32_t lanes = d.W / V;
    k = from + (uint32_t)(i / lanes);
    c = (uint32_t)(i % lanes) * V;
    return i < (uint64_t)count * lanes;
}

template <class T, int V>
__global__ void __launch_bounds__(kBlock)
sequence_fwd_kernel(Shape d, Fwd f, uint32_t from, uint32_t count)
{
    uint32_t k, c;
    if (!lane_place(d, V, from, count, k, c)) return;
    uint64_t begin, end;
    places(d, k, begin, end);
    const uint64_t at = (uint64_t)sequence(d, k) * d.W + c;
    float h[V];
    get<V>(f.h0, at, h);
    advance_places<T, V>(d, f, c, begin, end, h);
    put<V>(f.h_last, at, h);
}

// Two wavefronts per SIMD: the registers of a third one keep more tokens on their way.  2^17 rays of 64 samples, 32 channels in fp16: 505 us, with three 527.
template <class T, int V>
__global__ void __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(2, 2)))
sequence_bwd_kernel(Shape d, Bwd b, uint32_t from, uint32_t count)
{
    uint32_t k, c;
    if (!lane_place(d, V, from, count, k, c)) return;
    uint64_t begin, end;
    places(d, k, begin, end);
    const uint32_t seq = sequence(d, k);
    float G[V];
    get<V>(b.dh_last, (uint64_t)seq * d.W + c, G);
    retreat_places<T, V>(d, b, seq, c, begin, begin, end, G);
    put<V>(b.dh0, (uint64_t)seq * d.W + c, G);
}

// ------------------------------------------------------------------ long sequences
//
// A stretch of tokens takes the state before it to join(x, state, B).  A lane has a window of kKeep places and V channels, whose tokens
// it keeps in registers: what they need from memory is read once.  A workgroup has a tile, as many windows one behind the other as
// fit it, for channels that fill the 128 bytes of a line.  It finds x and B of its tile, tells the tiles behind it in a slot of its own,
// joins what those before it have told, and lets its windows run from there, joined in LDS.  A stretch that knows the state behind itself
// tells it as (+0, state); where a sequence begins x is +0 anyway.
//
// Tiles are numbered as workgroups start.  A tile waits only for ones with a lower number, which run or have run, and tell what they do
// before they wait for a state: every wait ends.  A slot is one 64-bit word written at once, so nothing else has to be ordered.
//
// A sequence that begins or ends in a window is gone through piece by piece.

// f(k, p, e, begin, end) for the pieces [p, e) of the sequences [begin, end) that lie in the window from place p0 on, in order.  A
// sequence without a place belongs to the window where it would begin.
template <class F>
__device__ __forceinline__ void forwards(const Shape &d, uint64_t p0, F f)
{
    const uint64_t p1 = p0 + kKeep < d.N ? p0 + kKeep : d.N;
    uint32_t k = begun_before(d, p0);
    uint64_t begin, end;
    if (k > 0) {
        places(d, k - 1, begin, end);
        if (end > p0) f(k - 1, p0, end < p1 ? end : p1, begin, end);
    }
    for (; k < d.n_seq; ++k) {
        places(d, k, begin, end);
        if (begin >= p1 && p1 < d.N) break;
        f(k, begin, end < p1 ? end : p1, begin, end);
    }
}

template <class F>
__device__ __forceinline__ void backwards(const Shape &d, uint64_t p0, F f)
{
    const uint64_t p1 = p0 + kKeep < d.N ? p0 + kKeep : d.N;
    uint32_t k = p1 < d.N ? begun_before(d, p1) : d.n_seq;
    while (k-- > 0) {
        uint64_t begin, end;
        places(d, k, begin, end);
        const uint64_t p = begin > p0 ? begin : p0, e = end < p1 ? end : p1;
        if (begin >= p0 || e > p0) f(k, p, e, begin, end);
        if (begin < p0) break;
    }
}

template <class T, int V, int M, bool kFull, bool kShutting>
__device__ __forceinline__ void sum_loaded(const Raw<T, V> (&z)[M], const Raw<T, V> (&u)[M], int n, float (&A)[V], float (&D)[V], float (&h)[V])
{
    bool zero[V];
#pragma unroll
    for (int v = 0; v < V; ++v) zero[v] = A[v] == 0.0f;
#pragma unroll
    for (int k = 0; k < M; ++k)
        if (kFull || k < n) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Step s = step_of<kShutting>(z[k][v], u[k][v]);
                h[v] = advance<kShutting>(s, h[v]);
                extend<kShutting>(s, A[v], D[v]);
            }
        }
#pragma unroll
    for (int v = 0; v < V && !kShutting; ++v) A[v] = clamped(A[v], zero[v]);
}

template <class T, int V, int M, bool kFull>
__device__ __forceinline__ void sum_tokens(const Shape &d, const Fwd &f, uint32_t c, uint64_t p, int n, float (&A)[V], float (&D)[V], float (&h)[V])
{
    Raw<T, V> z[M], u[M];
    load_tokens<T, V, M, kFull>(Column<T, V>(d, f.z, f.ldz, c, p), n, z);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, f.u, f.ldu, c, p), n, u);
    if (any_shut<T, V, M>(z)) sum_loaded<T, V, M, kFull, true>(z, u, n, A, D, h);
    else sum_loaded<T, V, M, kFull, false>(z, u, n, A, D, h);
}

template <class T, int V, int M, bool kFull, bool kShutting>
__device__ __forceinline__ void sum_gradients_loaded(const Raw<T, V> (&z)[M], const Raw<T, V> (&dy)[M], int n, float (&A)[V], float (&D)[V], float (&G)[V])
{
    bool zero[V];
#pragma unroll
    for (int v = 0; v < V; ++v) zero[v] = A[v] == 0.0f;
#pragma unroll
    for (int k = M - 1; k >= 0; --k)
        if (kFull || k < n) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Step s = step_of<kShutting>(z[k][v], 0.0f);
                G[v] = retreat<kShutting>(s, G[v] + dy[k][v]);
                extend<kShutting>(s, A[v], D[v]);
            }
        }
#pragma unroll
    for (int v = 0; v < V && !kShutting; ++v) A[v] = clamped(A[v], zero[v]);
}

template <class T, int V, int M, bool kFull>
__device__ __forceinline__ void sum_gradients(const Shape &d, const Bwd &b, uint32_t c, uint64_t p, int n, float (&A)[V], float (&D)[V], float (&G)[V])
{
    Raw<T, V> z[M], dy[M];
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.z, b.ldz, c, p), n, z);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.dy, b.lddy, c, p), n, dy);
    if (any_shut<T, V, M>(z)) sum_gradients_loaded<T, V, M, kFull, true>(z, dy, n, A, D, G);
    else sum_gradients_loaded<T, V, M, kFull, false>(z, dy, n, A, D, G);
}

constexpr int kTile = 512;          // lanes of a workgroup
constexpr uint32_t kBundle = 16;    // tiles
constexpr uint32_t kNear = 4;       // bundles that are looked back at

__host__ __device__ __forceinline__ uint32_t bundles_of(uint32_t n_tiles) { return (n_tiles + kBundle - 1) / kBundle; }

// lanes that have a token's channels side by side: a power of two, at most a line of 128 bytes
template <class T, int V>
__host__ __device__ __forceinline__ constexpr uint32_t most_across() { return 128 / (sizeof(T) * V) < dg::kWave ? 128 / (sizeof(T) * V) : dg::kWave; }

__host__ __device__ __forceinline__ uint32_t lanes_across(uint32_t W, uint32_t V, uint32_t most)
{
    uint32_t n = 1;
    while (n < most && n * V < W) n *= 2;
    return n;
}

__host__ __device__ __forceinline__ uint32_t groups_of(uint32_t W, uint32_t V, uint32_t across) { return (W + across * V - 1) / (across * V); }

// Pieces of a window in which a sequence begins or ends, four tokens at a time: they run while other lanes of the wavefront hold their
// windows, so that what they need in registers comes on top.
constexpr int kFew = 4;

template <class T, int V>
__device__ __forceinline__ void advance_few(const Shape &d, const Fwd &f, uint32_t c, uint64_t p, uint64_t end, float (&h)[V])
{
    if (p < end && p % kKeep == 0) put<V>(f.states, p / kKeep * d.W + c, h);
#pragma unroll 1
    for (; p < end; p += kFew) advance_tokens<T, V, kFew, false, false>(d, f, c, p, end - p < kFew ? (int)(end - p) : kFew, h);
}

template <class T, int V>
__device__ __forceinline__ void sum_few(const Shape &d, const Fwd &f, uint32_t c, uint64_t p, uint64_t end, float (&A)[V], float (&D)[V], float (&h)[V])
{
#pragma unroll 1
    for (; p < end; p += kFew) sum_tokens<T, V, kFew, false>(d, f, c, p, end - p < kFew ? (int)(end - p) : kFew, A, D, h);
}

template <class T, int V>
__device__ __forceinline__ void sum_few_gradients(const Shape &d, const Bwd &b, uint32_t c, uint64_t p, uint64_t end, float (&A)[V], float (&D)[V], float (&G)[V])
{
#pragma unroll 1
    while (end > p) {
        const int n = end - p < kFew ? (int)(end - p) : kFew;
        end -= n;
        sum_gradients<T, V, kFew, false>(d, b, c, end, n, A, D, G);
    }
}

// h through places [p, end)
template <class T, int V>
__device__ __forceinline__ void go_few(const Shape &d, const Bwd &b, uint32_t c, uint64_t p, uint64_t end, float (&h)[V])
{
#pragma unroll 1
    for (; p < end; p += kFew) {
        const int n = end - p < kFew ? (int)(end - p) : kFew;
        Raw<T, V> z[kFew], u[kFew];
        load_tokens<T, V, kFew, false>(Column<T, V>(d, b.z, b.ldz, c, p), n, z);
        load_tokens<T, V, kFew, false>(Column<T, V>(d, b.u, b.ldu, c, p), n, u);
#pragma unroll
        for (int k = 0; k < kFew; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (k < n) h[v] = advance<true>(step_of<true>(z[k][v], u[k][v]), h[v]);
    }
}

// every four tokens from the state that was kept, through the tokens in between
template <class T, int V>
__device__ __forceinline__ void retreat_few(const Shape &d, const Bwd &b, uint32_t seq, uint32_t c, uint64_t begin, uint64_t p, uint64_t end, float (&G)[V])
{
#pragma unroll 1
    while (end > p) {
        const int n = end - p < kFew ? (int)(end - p) : kFew;
        end -= n;
        float h[V];
        if (p == begin) get<V>(b.h0, (uint64_t)seq * d.W + c, h);
        else get<V>(b.states, p / kKeep * d.W + c, h);
        go_few<T, V>(d, b, c, p, end, h);
        retreat_tokens<T, V, kFew, false, false>(d, b, c, end, n, h, G);
    }
}

struct Lane {
    uint32_t across, lane, window, windows, c, tile;        // windows of a tile; c: first channel
    bool active;
    __device__ __forceinline__ Lane(const Shape &d, uint32_t V, uint32_t most, uint32_t number)
    {
        across = lanes_across(d.W, V, most);
        lane = threadIdx.x & (across - 1);
        window = threadIdx.x / across;
        windows = kTile / across;
        const uint32_t groups = groups_of(d.W, V, across);
        tile = number / groups;
        c = (number % groups * across + lane) * V;
        active = c < d.W;
    }
};

// What the tiles share: the number of workgroups that have started, and slots with x in the lower half and B in the upper one, for each
// channel of each tile and of each kBundle tiles that follow each other.
struct Board {
    uint32_t *started;
    uint64_t *slots, *bundles;      // [n_tiles, W], [bundles_of(n_tiles), W]
};

constexpr uint64_t kEmpty = ~0ull;  // x would be a NaN that is not told
// Of a lane, a second or so: then it takes NaN for what it has not heard.  A workspace that something else writes to would otherwise never let it go.
constexpr uint32_t kMostPolls = 1u << 20;

__device__ __forceinline__ uint32_t start(const Board &b)
{
    __shared__ uint32_t number;
    if (threadIdx.x == 0) number = __hip_atomic_fetch_add(b.started, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return number;
}

__device__ __forceinline__ uint32_t told_bits(float x) { return x != x ? 0x7fc00000u : __float_as_uint(x); }

template <int V>
__device__ __forceinline__ void tell(uint64_t *slot, const float (&x)[V], const float (&B)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v)
        __hip_atomic_store(slot + v, (uint64_t)told_bits(B[v]) << 32 | told_bits(x[v]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// waits for the first `count` of n slots, step words apart, to be written
template <int V, int n>
__device__ __forceinline__ void hear(const uint64_t *slot, int64_t step, uint32_t count, uint32_t &polls, float (&x)[n][V], float (&B)[n][V])
{
    uint64_t word[n][V];
    for (;;) {
        bool told = true;
#pragma unroll
        for (int i = 0; i < n; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v)
                word[i][v] = (uint32_t)i < count ? __hip_atomic_load(slot + i * step + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
#pragma unroll
        for (int i = 0; i < n; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) told = told && word[i][v] != kEmpty;
        if (told || polls == 0) break;
        --polls;
        __builtin_amdgcn_s_sleep(1);
    }
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) x[i][v] = __uint_as_float((uint32_t)word[i][v]), B[i][v] = __uint_as_float((uint32_t)(word[i][v] >> 32));
}

// The sequence that a window from place p0 on lies in, and whether it begins or ends with the window.
struct Inside {
    bool whole, first, last;        // whole: the window lies in one sequence
    uint32_t seq;
};

__device__ __forceinline__ Inside inside(const Shape &d, uint64_t p0)
{
    Inside in = {};
    const uint32_t k = d.first ? begun_before(d, p0 + 1) : (uint32_t)p0 / d.S + 1;
    if (k == 0) return in;
    uint64_t begin, end;
    places(d, k - 1, begin, end);
    in.whole = begin <= p0 && end >= p0 + kKeep;
    in.first = begin == p0;
    in.last = end == p0 + kKeep;
    in.seq = sequence(d, k - 1);
    return in;
}

// x, A and B of the windows of a tile, or the tiles of a bundle, of at most kTile lanes
template <int V, int n>
struct Stretches {
    float x[n][V], A[n][V], B[n][V];
    __device__ __forceinline__ void put(uint32_t at, const float (&xs)[V], const float (&Bs)[V])
    {
#pragma unroll
        for (int v = 0; v < V; ++v) x[at][v] = xs[v], A[at][v] = share(xs[v]), B[at][v] = Bs[v];
    }
};

// h through n stretches, one every `step` places from `at` on.  As fast as can be first, then with care where that could matter: a state that is not
// finite stays so on the fast way, even past an A of 0.  kFar: they may be more than kKeep (as few lose no more than the tokens of a window).  kAll: x receives that
// of all of them.  (D of the whole is right where it is needed: where A is more than 1/2, and with it that of every stretch.)
template <int V, bool kFar, bool kAll, int n_all>
__device__ __forceinline__ void pass(uint32_t n, const Stretches<V, n_all> &all, uint32_t at, uint32_t step, float (&h)[V], float (&x)[V])
{
    float from[V], A[V], D[V], least[V];
    bool good = true;
#pragma unroll
    for (int v = 0; v < V; ++v) from[v] = h[v], A[v] = least[v] = 1.0f, D[v] = 0.0f;
#pragma unroll 4
    for (uint32_t w = 0; w < n; ++w) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float ax = all.x[at + w * step][v], a = all.A[at + w * step][v], b = all.B[at + w * step][v];
            h[v] = kFar ? join_finite(ax, a, h[v], b) : fmaf(a, h[v], b);
            if (kAll) {
                D[v] = fmaf(-ax, A[v], D[v]);
                A[v] = kFar ? join_finite(ax, a, A[v], 0.0f) : A[v] * a;
                least[v] = fminf(least[v], a);
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (kAll) x[v] = code(clamped(A[v], least[v] == 0.0f), D[v]);
        good = good && finite(h[v]);
    }
    if (good) return;
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = from[v];
#pragma unroll 1
    for (uint32_t w = 0; w < n; ++w)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float a = all.A[at + w * step][v], b = all.B[at + w * step][v];
            h[v] = a == 0.0f ? b : fmaf(a, h[v], b);
        }
}

// The state before a bundle: from the nearest of the kNear bundles before it that knows the state behind itself, through the ones in
// between.  Of lanes that have channels.
template <int V>
__device__ __forceinline__ void before_bundle(const Shape &d, const Board &board, uint32_t bundle, uint32_t c, uint32_t &polls, float (&h)[V])
{
    const uint32_t n = bundle < kNear ? bundle : kNear;
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = 0.0f;
    while (n) {
        float x[kNear][V], B[kNear][V];
        hear<V, kNear>(board.bundles + (uint64_t)(bundle - 1) * d.W + c, -(int64_t)d.W, n, polls, x, B);
        bool known = true;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            bool met = false;                                   // going forwards to the bundle: start anew at each that knows
#pragma unroll
            for (int i = kNear - 1; i >= 0; --i)
                if ((uint32_t)i < n) {
                    h[v] = join(x[i][v], met ? h[v] : 0.0f, B[i][v]);
                    met = met || anew(x[i][v]);
                }
            known = known && met;
        }
        if (known) return;
        if (polls == 0) break;
        --polls;
    }
    if (n)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = __uint_as_float(0x7fc00000u);
}

// From x and B of a lane's window the state before it (backward: the gradient behind it).  All lanes of the workgroup call it.
// mine: the place of the lane's window among those of the tile in the order in which states pass them; tile: likewise.
//
// A tile listens to those before it in its bundle; the last of a bundle tells what the whole bundle does, and, when it knows it, the
// state behind it.  Whoever computes the state behind a bundle computes join(x, the state before it, B): how far back the nearest bundle
// lies that knows its own depends on timing, the result does not.
template <int V>
__device__ __forceinline__ void come_in(const Shape &d, const Board &board, const Lane &l, uint32_t mine, uint32_t tile, const float (&x)[V],
                                        const float (&B)[V], float (&h)[V])
{
    __shared__ Stretches<V, kTile> windows;
    __shared__ Stretches<V, kBundle * dg::kWave> tiles;
    __shared__ float in[dg::kWave][V];
    uint32_t polls = kMostPolls;
    float unused[V];
    auto through_windows = [&](auto all, uint32_t n, float (&to)[V], float (&of_all)[V]) {
        if (l.windows > kKeep) pass<V, true, all.value>(n, windows, l.lane, l.across, to, of_all);      // narrow rows
        else pass<V, false, all.value>(n, windows, l.lane, l.across, to, of_all);
    };
    windows.put(mine * l.across + l.lane, x, B);
    __syncthreads();
    const uint32_t bundle = tile / kBundle, place = tile % kBundle;
    if (mine == 0) {
        float tx[V], tB[V] = {};
        through_windows(std::true_type(), l.windows, tB, tx);
        if (l.active) tell<V>(board.slots + (uint64_t)tile * d.W + l.c, tx, tB);
        tiles.put(place * dg::kWave + l.lane, tx, tB);
    }
    if (l.active)
        for (uint32_t w = mine; w < place; w += l.windows) {
            float tx[1][V], tB[1][V];
            hear<V, 1>(board.slots + (uint64_t)(tile - place + w) * d.W + l.c, 0, 1, polls, tx, tB);
            tiles.put(w * dg::kWave + l.lane, tx[0], tB[0]);
        }
    __syncthreads();
    if (mine == 0 && l.active) {
        uint64_t *told = board.bundles + (uint64_t)bundle * d.W + l.c;
        float bx[V] = {}, bB[V] = {}, state[V];
        if (place == kBundle - 1) {
            pass<V, false, true>(kBundle, tiles, l.lane, dg::kWave, bB, bx);
#pragma unroll
            for (int v = 0; v < V; ++v) bx[v] = bundle == 0 ? 0.0f : bx[v];      // nothing comes before the first
            tell<V>(told, bx, bB);
        }
        before_bundle<V>(d, board, bundle, l.c, polls, state);
        if (place == kBundle - 1 && bundle) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                bB[v] = join(bx[v], state[v], bB[v]);
                bx[v] = 0.0f;
            }
            tell<V>(told, bx, bB);
        }
        pass<V, false, false>(place, tiles, l.lane, dg::kWave, state, unused);
#pragma unroll
        for (int v = 0; v < V; ++v) in[l.lane][v] = state[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = in[l.lane][v];
    through_windows(std::false_type(), mine, h, unused);
}

// 128 registers per lane at most: two workgroups then share a compute unit, and one loads while the other listens.
#define TWO_PER_UNIT __attribute__((amdgpu_waves_per_eu(4)))

// x and B of a window that starts from a state of its own
template <int V>
__device__ __forceinline__ void begin_with(float (&x)[V], float (&B)[V], const float *states, uint64_t at)
{
    float from[V];
    get<V>(states, at, from);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        B[v] = join(x[v], from[v], B[v]);
        x[v] = 0.0f;
    }
}

template <int V>
__device__ __forceinline__ void code(const float (&A)[V], const float (&D)[V], float (&x)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = code(A[v], D[v]);
}

template <class T, int V>
__global__ void __launch_bounds__(kTile) TWO_PER_UNIT
tile_fwd_kernel(Shape d, Fwd f, Board board)
{
    const Lane l(d, V, most_across<T, V>(), start(board));
    const uint64_t p0 = ((uint64_t)l.tile * l.windows + l.window) * kKeep;
    const bool held = l.active && p0 < d.N;
    const Inside in = held ? inside(d, p0) : Inside{};
    auto at = [&] { return (uint64_t)in.seq * d.W + l.c; };
    Raw<T, V> z[kKeep], u[kKeep];
    float A[V], D[V], h[V], x[V];
    bool shutting = false;
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.0f, D[v] = 0.0f, h[v] = 0.0f;
    if (in.whole) {
        load_tokens<T, V, kKeep, true>(Column<T, V>(d, f.z, f.ldz, l.c, p0), kKeep, z);
        load_tokens<T, V, kKeep, true>(Column<T, V>(d, f.u, f.ldu, l.c, p0), kKeep, u);
        shutting = any_shut<T, V, kKeep>(z);
        if (shutting) sum_loaded<T, V, kKeep, true, true>(z, u, kKeep, A, D, h);
        else sum_loaded<T, V, kKeep, true, false>(z, u, kKeep, A, D, h);
    } else if (held)
        forwards(d, p0, [&](uint32_t k, uint64_t p, uint64_t e, uint64_t begin, uint64_t) {
            if (p == begin) {
#pragma unroll
                for (int v = 0; v < V; ++v) A[v] = 0.0f;
                get<V>(f.h0, (uint64_t)sequence(d, k) * d.W + l.c, h);
            }
            sum_few<T, V>(d, f, l.c, p, e, A, D, h);
        });
    code<V>(A, D, x);
    if (in.whole && in.first) begin_with<V>(x, h, f.h0, at());
    forget<T, V, kKeep>(z), forget<T, V, kKeep>(u);
    float state[V];
    come_in<V>(d, board, l, l.window, l.tile, x, h, state);
    if (in.whole) {
        if (in.first) get<V>(f.h0, at(), state);
        put<V>(f.states, p0 / kKeep * d.W + l.c, state);
        const Column<T, V> y(d, f.y, f.ldy, l.c, p0);
        forget<T, V, kKeep>(z);
        if (shutting) advance_loaded<T, V, kKeep, true, true, false>(z, u, y, kKeep, state);
        else advance_loaded<T, V, kKeep, true, false, false>(z, u, y, kKeep, state);
        if (in.last) put<V>(f.h_last, at(), state);
    } else if (held)
        forwards(d, p0, [&](uint32_t k, uint64_t p, uint64_t e, uint64_t begin, uint64_t end) {
            const uint64_t at = (uint64_t)sequence(d, k) * d.W + l.c;
            if (p == begin) get<V>(f.h0, at, state);
            advance_few<T, V>(d, f, l.c, p, e, state);
            if (e == end) put<V>(f.h_last, at, state);
        });
}

// from the last tile to the first
template <class T, int V>
__global__ void __launch_bounds__(kTile) TWO_PER_UNIT
tile_bwd_kernel(Shape d, Bwd b, Board board)
{
    Lane l(d, V, most_across<T, V>(), start(board));
    const uint32_t tile = l.tile;
    l.tile = d.n_tiles - 1 - tile;
    const uint64_t p0 = ((uint64_t)l.tile * l.windows + l.window) * kKeep;
    const bool held = l.active && p0 < d.N;
    const Inside in = held ? inside(d, p0) : Inside{};
    auto at = [&] { return (uint64_t)in.seq * d.W + l.c; };
    Raw<T, V> z[kKeep], u[kKeep], dy[kKeep];
    float A[V], D[V], G[V], x[V];
    bool shutting = false;
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.0f, D[v] = 0.0f, G[v] = 0.0f;
    if (in.whole) {
        load_tokens<T, V, kKeep, true>(Column<T, V>(d, b.z, b.ldz, l.c, p0), kKeep, z);
        load_tokens<T, V, kKeep, true>(Column<T, V>(d, b.dy, b.lddy, l.c, p0), kKeep, dy);
        load_tokens<T, V, kKeep, true>(Column<T, V>(d, b.u, b.ldu, l.c, p0), kKeep, u);
        shutting = any_shut<T, V, kKeep>(z);
        if (shutting) sum_gradients_loaded<T, V, kKeep, true, true>(z, dy, kKeep, A, D, G);
        else sum_gradients_loaded<T, V, kKeep, true, false>(z, dy, kKeep, A, D, G);
    } else if (held)
        backwards(d, p0, [&](uint32_t k, uint64_t p, uint64_t e, uint64_t, uint64_t end) {
            if (e == end) {
#pragma unroll
                for (int v = 0; v < V; ++v) A[v] = 0.0f;
                get<V>(b.dh_last, (uint64_t)sequence(d, k) * d.W + l.c, G);
            }
            sum_few_gradients<T, V>(d, b, l.c, p, e, A, D, G);
        });
    code<V>(A, D, x);
    if (in.whole && in.last) begin_with<V>(x, G, b.dh_last, at());
    forget<T, V, kKeep>(z), forget<T, V, kKeep>(u), forget<T, V, kKeep>(dy);
    float behind[V];
    come_in<V>(d, board, l, l.windows - 1 - l.window, tile, x, G, behind);
    if (in.whole) {
        if (in.last) get<V>(b.dh_last, at(), behind);
        const Column<T, V> dz(d, b.dz, b.lddz, l.c, p0 + kKeep - 1), du(d, b.du, b.lddu, l.c, p0 + kKeep - 1);
        float state[V], less[kKeep][V];
        if (in.first) get<V>(b.h0, at(), state);
        else get<V>(b.states, p0 / kKeep * d.W + l.c, state);
        forget<T, V, kKeep>(z);
        if (shutting) {
            steps_taken<T, V, kKeep, true>(z, u, state, less);
            forget<T, V, kKeep>(z);
            retreat_loaded<T, V, kKeep, true, true, false>(z, dy, less, dz, du, kKeep, behind);
        } else {
            steps_taken<T, V, kKeep, false>(z, u, state, less);
            forget<T, V, kKeep>(z);
            retreat_loaded<T, V, kKeep, true, false, false>(z, dy, less, dz, du, kKeep, behind);
        }
        if (in.first) put<V>(b.dh0, at(), behind);
    } else if (held)
        backwards(d, p0, [&](uint32_t k, uint64_t p, uint64_t e, uint64_t begin, uint64_t end) {
            const uint32_t seq = sequence(d, k);
            const uint64_t at = (uint64_t)seq * d.W + l.c;
            if (e == end) get<V>(b.dh_last, at, behind);
            retreat_few<T, V>(d, b, seq, l.c, begin, p, e, behind);
            if (p == begin) put<V>(b.dh0, at, behind);
        });
}

// Empties the board, and does the sequences without a token: what comes out is what went in.  copy: NULL, or room for `in`, which the
// tiles then read there because `out` lies on it.
__global__ void __launch_bounds__(kBlock)
board_kernel(Shape d, Board board, uint64_t n_slots, const float *in, float *copy, float *out)
{
    const uint64_t i0 = (uint64_t)blockIdx.x * kBlock + threadIdx.x, step = (uint64_t)gridDim.x * kBlock, n = (uint64_t)d.n_seq * d.W;
    if (i0 == 0) *board.started = 0;
    for (uint64_t i = i0; i < n_slots; i += step) board.slots[i] = kEmpty;
    if (copy)
        for (uint64_t i = i0; i < n; i += step) copy[i] = in[i];
    if (d.first && out && in != out)
        for (uint64_t i = i0; i < n; i += step) {
            const uint64_t end = d.first[i / d.W + 1];
            if (d.first[i / d.W] >= (end < d.N ? end : d.N)) out[i] = in ? in[i] : 0.0f;
        }
}

int check(const char *who, Shape &d, uint32_t dtype)
{
    DG_REQUIRE(known_type(dtype), DG_ERR_ARG, "%s: unknown element type %u", who, dtype);
    DG_REQUIRE(d.W >= 1, DG_ERR_ARG, "%s: rows without a channel", who);
    DG_REQUIRE(d.N < 1ull << 32 && d.W <= 1u << 20 && d.N * d.W <= 1ull << 39, DG_ERR_UNSUPPORTED,
               "%s: 2^32 tokens or more, more than 2^20 channels or than 2^39 values", who);
    DG_REQUIRE(dg::aligned(d.first, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    DG_REQUIRE(d.n_seq > 0 || d.N == 0, DG_ERR_ARG, "%s: tokens without a sequence", who);
    DG_REQUIRE(d.first || d.n_seq == 0 || d.N % d.n_seq == 0, DG_ERR_ARG, "%s: %llu tokens are not %u sequences of one length", who, (unsigned long long)d.N,
               d.n_seq);
    d.S = d.n_seq ? (uint32_t)(d.N / d.n_seq) : 0;
    DG_REQUIRE((uint64_t)d.n_seq * d.W <= 1ull << 38, DG_ERR_UNSUPPORTED, "%s: more than 2^38 states", who);
    return DG_OK;
}

int check_rows(const char *who, const void *p, uint64_t ld, const Shape &d, uint32_t dtype)
{
    if (d.N == 0) return DG_OK;
    DG_REQUIRE(p && dg::aligned(p, item_bytes(dtype)), DG_ERR_ARG, "%s: null or misaligned pointer", who);
    DG_REQUIRE(ld >= d.W && ld <= 1ull << 40, DG_ERR_ARG, "%s: rows of %u channels lie %llu apart", who, d.W, (unsigned long long)ld);
    return DG_OK;
}

// Whether tiles serve a call.  Sequence by sequence 16 tokens take some 1.6 us forward however few sequences there are; tiles take 8 us
// and then 3 TB/s with 16-bit values, and longer where many windows hold a sequence's end.  They pay for sequences of more than 120
// tokens and an 80 000th of all values.  Sequences / tiles in us, forward and backward: 256 sequences of 512 tokens, 64 channels, fp16
// 57 / 26 and 93 / 33; 64 of 1024, 256 channels 110 / 42 and 181 / 52; 16 of 4096, 2048 channels, bf16 505 / 186 and 828 / 293; 512 of 1024, 128
// channels 143 / 133 and 225 / 182; 400 of 256, 128 channels 31 / 36 and 49 / 47; 4000 of 400, 64 channels 126 / 199 and 217 / 274; 100 of 400, 32
// channels, fp32 31 / 12 and 47 / 14; 1000 of 200, 32 channels 28 / 31 and 44 / 40; 1000 of 2000, 64 channels 278 / 245 and 442 / 335;
// 300 of 1500, 512 channels, fp16 336 / 448 and 593 / 610.  The rule sees the mean length alone, which is all that the host knows: one long sequence among many
// short ones goes by itself (20 000 of 10 tokens and one of 131 072, 64 channels: 14 ms and 24).  V, most: of the call.
void cut(Shape &d, uint32_t V, uint32_t most)
{
    d.n_tiles = 0;
    if (d.n_seq == 0 || d.N / d.n_seq <= 120 + d.N * d.W / 80000) return;
    const uint32_t tile = kTile / lanes_across(d.W, V, most) * kKeep;
    d.n_tiles = (uint32_t)((d.N + tile - 1) / tile);
}

// Lanes of one launch: a grid of 2^32 lanes and more is cut short without an error.
constexpr uint64_t kMostLanes = 1ull << 31;

// launch(first sequence, sequences, workgroups)
template <class F>
void in_sequences(const Shape &d, uint32_t V, F launch)
{
    const uint64_t lanes = d.W / V, most = kMostLanes / lanes;
    for (uint64_t from = 0; from < d.n_seq; from += most) {
        const uint64_t count = d.n_seq - from < most ? d.n_seq - from : most;
        launch((uint32_t)from, (uint32_t)count, (uint32_t)((count * lanes + kBlock - 1) / kBlock));
    }
}

// launch(workgroups): tiles take their numbers on the device, one launch goes on where the last one has ended
template <class F>
void in_tiles(uint64_t n, F launch)
{
    for (constexpr uint64_t most = kMostLanes / kTile; n > 0; n -= n < most ? n : most) launch((uint32_t)(n < most ? n : most));
}

// the board's counter and slots, and room for a copy of the states
constexpr size_t kSlotsAt = 16;

size_t slots_of(const Shape &d) { return (size_t)(d.n_tiles + bundles_of(d.n_tiles)) * d.W; }

size_t workspace_bytes(const Shape &d) { return d.n_tiles ? kSlotsAt + slots_of(d) * sizeof(uint64_t) + (size_t)d.n_seq * d.W * sizeof(float) : 0; }

// whatever the type and the alignment of the call: the smallest tile makes the most of them
size_t most_workspace_bytes(Shape d)
{
    cut(d, 1, dg::kWave);
    return workspace_bytes(d);
}

int check_workspace(const char *who, const Shape &d, const void *ws, size_t ws_bytes)
{
    const size_t need = most_workspace_bytes(d);
    DG_REQUIRE(need == 0 || (ws && dg::aligned(ws, 16) && ws_bytes >= need), DG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need,
               ws ? ws_bytes : 0);
    return DG_OK;
}

// *in: states (gradients) that the tiles read, out: where they write theirs
Board board_of(const Shape &d, void *ws, const float **in, float *out, hipStream_t st)
{
    const uint64_t n_slots = slots_of(d);
    Board board = {(uint32_t *)ws, (uint64_t *)((char *)ws + kSlotsAt), nullptr};
    board.bundles = board.slots + (uint64_t)d.n_tiles * d.W;
    float *copy = *in && *in == out ? (float *)(board.slots + n_slots) : nullptr;
    const uint64_t n = (n_slots + 4 * kBlock - 1) / (4 * kBlock);
    board_kernel<<<(uint32_t)(n < 2048 ? n : 2048), kBlock, 0, st>>>(d, board, n_slots, *in, copy, out);
    if (copy) *in = copy;
    return board;
}

template <class T, int V>
uint64_t tile_blocks(const Shape &d) { return (uint64_t)d.n_tiles * groups_of(d.W, V, lanes_across(d.W, V, most_across<T, V>())); }

template <class T, int V>
void launch_fwd(Shape d, Fwd f, void *ws, hipStream_t st)
{
    cut(d, V, most_across<T, V>());
    if (!d.n_tiles) {
        in_sequences(d, V, [&](uint32_t from, uint32_t n, uint32_t blocks) { sequence_fwd_kernel<T, V><<<blocks, kBlock, 0, st>>>(d, f, from, n); });
        return;
    }
    const Board board = board_of(d, ws, &f.h0, f.h_last, st);
    in_tiles(tile_blocks<T, V>(d), [&](uint32_t blocks) { tile_fwd_kernel<T, V><<<blocks, kTile, 0, st>>>(d, f, board); });
}

template <class T, int V>
void launch_bwd(Shape d, Bwd b, void *ws, hipStream_t st)
{
    cut(d, V, most_across<T, V>());
    if (!d.n_tiles) {
        in_sequences(d, V, [&](uint32_t from, uint32_t n, uint32_t blocks) { sequence_bwd_kernel<T, V><<<blocks, kBlock, 0, st>>>(d, b, from, n); });
        return;
    }
    const Board board = board_of(d, ws, &b.dh_last, b.dh0, st);
    in_tiles(tile_blocks<T, V>(d), [&](uint32_t blocks) { tile_bwd_kernel<T, V><<<blocks, kTile, 0, st>>>(d, b, board); });
}

}  // namespace

extern "C" size_t dg_recurrence_state_count(uint64_t N, uint32_t W) { return (size_t)((N + kKeep - 1) / kKeep) * W; }

extern "C" size_t dg_recurrence_workspace_bytes(uint64_t N, uint32_t n_seq, uint32_t W)
{
    Shape d = {N, n_seq, W, 0, nullptr, false, 0};
    return most_workspace_bytes(d);
}

extern "C" int dg_recurrence_fwd(const void *z, uint64_t ldz, const void *u, uint64_t ldu, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t W,
                                 uint32_t reverse, uint32_t dtype, const float *h0, void *y, uint64_t ldy, float *h_last, float *states, void *ws,
                                 size_t ws_bytes, void *stream)
{
    const char *who = "dg_recurrence_fwd";
    Shape d = {N, n_seq, W, 0, first, reverse != 0, 0};
    if (int rc = check(who, d, dtype)) return rc;
    if (int rc = check_rows(who, z, ldz, d, dtype)) return rc;
    if (int rc = check_rows(who, u, ldu, d, dtype)) return rc;
    if (int rc = check_rows(who, y, ldy, d, dtype)) return rc;
    DG_REQUIRE(dg::aligned(h0, 4) && dg::aligned(h_last, 4) && dg::aligned(states, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (n_seq == 0) return DG_OK;
    if (int rc = check_workspace(who, d, ws, ws_bytes)) return rc;
    const Fwd f = {z, u, y, ldz, ldu, ldy, h0, h_last, states};
    const bool pairs = dtype != DG_F32 && W % 2 == 0 && rows_aligned(z, ldz, dtype, 4) && rows_aligned(u, ldu, dtype, 4) && rows_aligned(y, ldy, dtype, 4);
    (dtype == DG_F32   ? launch_fwd<float, 1>
     : dtype == DG_F16 ? (pairs ? launch_fwd<f16, 2> : launch_fwd<f16, 1>)
                       : (pairs ? launch_fwd<bf16, 2> : launch_fwd<bf16, 1>))(d, f, ws, (hipStream_t)stream);
    return dg::launch_status(who);
}

extern "C" int dg_recurrence_bwd(const void *z, uint64_t ldz, const void *u, uint64_t ldu, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t W,
                                 uint32_t reverse, uint32_t dtype, const float *h0, const float *states, const void *dy, uint64_t lddy,
                                 const float *dh_last, void *dz, uint64_t lddz, void *du, uint64_t lddu, float *dh0, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "dg_recurrence_bwd";
    Shape d = {N, n_seq, W, 0, first, reverse != 0, 0};
    if (int rc = check(who, d, dtype)) return rc;
    const struct { const void *p; uint64_t ld; } rows[] = {{z, ldz}, {u, ldu}, {dy, lddy}, {dz, lddz}, {du, lddu}};
    for (const auto &r : rows)
        if (int rc = check_rows(who, r.p, r.ld, d, dtype)) return rc;
    DG_REQUIRE(N == 0 || states, DG_ERR_ARG, "%s: the states that the forward pass kept are missing", who);
    DG_REQUIRE(dg::aligned(h0, 4) && dg::aligned(states, 4) && dg::aligned(dh_last, 4) && dg::aligned(dh0, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (n_seq == 0) return DG_OK;
    if (int rc = check_workspace(who, d, ws, ws_bytes)) return rc;
    const Bwd b = {z, u, dy, dz, du, ldz, ldu, lddy, lddz, lddu, h0, states, dh_last, dh0};
    bool pairs = dtype != DG_F32 && W % 2 == 0;
    for (const auto &r : rows) pairs = pairs && rows_aligned(r.p, r.ld, dtype, 4);
    (dtype == DG_F32   ? launch_bwd<float, 1>
     : dtype == DG_F16 ? (pairs ? launch_bwd<f16, 2> : launch_bwd<f16, 1>)
                       : (pairs ? launch_bwd<bf16, 2> : launch_bwd<bf16, 1>))(d, b, ws, (hipStream_t)stream);
    return dg::launch_status(who);
}
