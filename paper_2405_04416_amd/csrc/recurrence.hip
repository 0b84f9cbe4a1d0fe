// Gated linear recurrence along sequences of rows, channel by channel:
//   a = 1 / (1 + e^-z),  c = 1 - a = 1 / (1 + e^z),  h_t = a_t h_{t-1} + c_t u_t,  y_t = h_t.
// Its backward pass: G_t = dy_t + a_{t+1} G_{t+1} from the last token back, du = c G, dz = a c G (h_{t-1} - u_t), dh0 = a_0 G_0.
// From |z| = 87 on a and c are exactly 0 and 1: what a gate of 0 multiplies is not looked at, be it infinite or NaN.
//
// Tokens have a place in the order in which they are gone through: their row, or N - 1 - row back to front.  The forward pass
// keeps the state before every kKeep-th place in fp32; the backward pass computes the states between them again.
#include "rows_common.h"

namespace {

using namespace dg_rows;

constexpr int kBlock = 256, kKeep = 16;
constexpr float kLeast = 1.17549435e-38f;       // the smallest normal number
constexpr float kShut = 87.0f;                  // up to here e^z, e^-z, a and c are normal numbers
constexpr float kLog2e = 1.44269504f;

struct Gate { float a, c; };

// both sides of an open gate to full relative precision
__device__ __forceinline__ Gate gate(float z)
{
    const float e = __builtin_amdgcn_exp2f(z * -kLog2e), a = __builtin_amdgcn_rcpf(1.0f + e);
    return {a, e * a};
}

// Whether a wavefront has a shut gate among the tokens that it has loaded.  One operation per two values finds out; the tokens are then
// gone through without looking at each gate.
template <class T, int V, int M>
__device__ __forceinline__ bool any_shut(const Pack<T, V> (&z)[M])
{
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < M; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) most = fmaxf(most, fabsf((float)z[k].v[v]));
    return __any(most >= kShut);
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

// a stretch of tokens takes the state h to join(A, h, B), A the product of its gates
__device__ __forceinline__ float join(float A, float h, float B) { return (A == 0.0f ? 0.0f : A * h) + B; }

// A product of gates: 0 only if one of them is, so that a state that is infinite or NaN gets through a long stretch as it does token
// by token.  What this adds to a finite state is below 2^-126 of it.
__device__ __forceinline__ float times(float A, float a) { return a == 0.0f ? 0.0f : fmaxf(A * a, A == 0.0f ? 0.0f : kLeast); }

struct Shape {
    uint64_t N;
    uint32_t n_seq, W, S;           // S: tokens of each sequence, where first is NULL
    const uint32_t *first;
    bool reverse;
    uint32_t n_chunks, per_chunk;   // places of a chunk, a multiple of kKeep; 0 chunks: sequence by sequence
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
        const uint64_t k = (p + d.S - 1) / d.S;
        return k < d.n_seq ? (uint32_t)k : d.n_seq;
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

// V neighbouring channels of the row of a place, and the way from there to the next place's
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
__device__ __forceinline__ void load_tokens(const Column<T, V> &col, int n, Pack<T, V> (&out)[M])
{
#pragma unroll
    for (int k = 0; k < M; ++k) {
        const int i = kFull || k < n ? k : n - 1;           // past the last token: that one again
        out[k] = *reinterpret_cast<const Pack<T, V> *>(col.at + i * col.step);
    }
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

// Runs f(place, number of tokens, full) over [p, end) in pieces that end where states are kept.
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

template <class T, int V, int M, bool kFull, bool kShutting>
__device__ __forceinline__ void advance_loaded(const Pack<T, V> (&z)[M], const Pack<T, V> (&u)[M], const Column<T, V> &y, int n, float (&h)[V])
{
#pragma unroll
    for (int k = 0; k < M; ++k)
        if (kFull || k < n) {
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = advance<kShutting>(step_of<kShutting>((float)z[k].v[v], (float)u[k].v[v]), h[v]);
            store<T, V>(y.at + k * y.step, h);
        }
}

template <class T, int V, int M, bool kFull>
__device__ __forceinline__ void advance_tokens(const Shape &d, const Fwd &f, uint32_t c, uint64_t p, int n, float (&h)[V])
{
    Pack<T, V> z[M], u[M];
    load_tokens<T, V, M, kFull>(Column<T, V>(d, f.z, f.ldz, c, p), n, z);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, f.u, f.ldu, c, p), n, u);
    const Column<T, V> y(d, f.y, f.ldy, c, p);
    if (any_shut<T, V, M>(z)) advance_loaded<T, V, M, kFull, true>(z, u, y, n, h);
    else advance_loaded<T, V, M, kFull, false>(z, u, y, n, h);
}

// y of places [p, end) of a sequence from the state before them, and the states that are kept
template <class T, int V>
__device__ __forceinline__ void advance_places(const Shape &d, const Fwd &f, uint32_t c, uint64_t p, uint64_t end, float (&h)[V])
{
    in_pieces(p, end, [&](uint64_t q, int n) {
        if (q % kKeep == 0) put<V>(f.states, q / kKeep * d.W + c, h);
        if (n == kKeep) advance_tokens<T, V, kKeep, true>(d, f, c, q, n, h);
        else if (n == 1) advance_tokens<T, V, 1, true>(d, f, c, q, n, h);
        else advance_tokens<T, V, kKeep, false>(d, f, c, q, n, h);
    });
}

// Forwards through the tokens for what G is multiplied with, a, c and q = a c (h_{t-1} - u), then backwards with G.
template <class T, int V, int M, bool kFull, bool kShutting>
__device__ __forceinline__ void retreat_loaded(const Pack<T, V> (&z)[M], const Pack<T, V> (&u)[M], const Pack<T, V> (&dy)[M], const Column<T, V> &dz,
                                               const Column<T, V> &du, int n, float (&h)[V], float (&G)[V])
{
    float a[M][V], c[M][V], q[M][V];
#pragma unroll
    for (int k = 0; k < M; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float uu = (float)u[k].v[v];
            const Step s = step_of<kShutting>((float)z[k].v[v], uu);
            a[k][v] = s.a;
            c[k][v] = s.c;
            q[k][v] = kShutting && (s.a == 0.0f || s.c == 0.0f) ? 0.0f : s.a * s.c * (h[v] - uu);
            h[v] = advance<kShutting>(s, h[v]);
        }
#pragma unroll
    for (int k = M - 1; k >= 0; --k)
        if (kFull || k < n) {
            float oz[V], ou[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                G[v] += (float)dy[k].v[v];
                oz[v] = kShutting && q[k][v] == 0.0f ? 0.0f : q[k][v] * G[v];
                ou[v] = kShutting && c[k][v] == 0.0f ? 0.0f : c[k][v] * G[v];
                G[v] = kShutting && a[k][v] == 0.0f ? 0.0f : a[k][v] * G[v];
            }
            store<T, V>(dz.at + k * dz.step, oz);
            store<T, V>(du.at + k * du.step, ou);
        }
}

template <class T, int V, int M, bool kFull>
__device__ __forceinline__ void retreat_tokens(const Shape &d, const Bwd &b, uint32_t c, uint64_t p, int n, float (&h)[V], float (&G)[V])
{
    Pack<T, V> z[M], u[M], dy[M];
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.z, b.ldz, c, p), n, z);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.u, b.ldu, c, p), n, u);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.dy, b.lddy, c, p), n, dy);
    const Column<T, V> dz(d, b.dz, b.lddz, c, p), du(d, b.du, b.lddu, c, p);
    if (any_shut<T, V, M>(z)) retreat_loaded<T, V, M, kFull, true>(z, u, dy, dz, du, n, h, G);
    else retreat_loaded<T, V, M, kFull, false>(z, u, dy, dz, du, n, h, G);
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
        if (n == kKeep) retreat_tokens<T, V, kKeep, true>(d, b, c, q, n, h, G);
        else if (n == 1) retreat_tokens<T, V, 1, true>(d, b, c, q, n, h, G);
        else retreat_tokens<T, V, kKeep, false>(d, b, c, q, n, h, G);
        end = q;
    }
}

// ------------------------------------------------------------------ a lane per sequence and V channels

__device__ __forceinline__ bool lane_place(const Shape &d, uint32_t V, uint32_t count, uint32_t &k, uint32_t &c)
{
    const uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const uint32_t lanes = d.W / V;
    k = (uint32_t)(i / lanes);
    c = (uint32_t)(i % lanes) * V;
    return i < (uint64_t)count * lanes;
}

template <class T, int V>
__global__ void __launch_bounds__(kBlock)
sequence_fwd_kernel(Shape d, Fwd f)
{
    uint32_t k, c;
    if (!lane_place(d, V, d.n_seq, k, c)) return;
    uint64_t begin, end;
    places(d, k, begin, end);
    const uint64_t at = (uint64_t)sequence(d, k) * d.W + c;
    float h[V];
    get<V>(f.h0, at, h);
    advance_places<T, V>(d, f, c, begin, end, h);
    put<V>(f.h_last, at, h);
}

template <class T, int V>
__global__ void __launch_bounds__(kBlock)
sequence_bwd_kernel(Shape d, Bwd b)
{
    uint32_t k, c;
    if (!lane_place(d, V, d.n_seq, k, c)) return;
    uint64_t begin, end;
    places(d, k, begin, end);
    const uint32_t seq = sequence(d, k);
    float G[V];
    get<V>(b.dh_last, (uint64_t)seq * d.W + c, G);
    retreat_places<T, V>(d, b, seq, c, begin, begin, end, G);
    put<V>(b.dh0, (uint64_t)seq * d.W + c, G);
}

// ------------------------------------------------------------------ long sequences: a lane per chunk of places and V channels
//
// A chunk takes the state before it to join(A, state, B).  One launch finds A and B of every chunk, one joins them along the
// chunks into the state before each, one runs the chunks from there.  A sequence that begins inside a chunk makes its A 0.

// f(k, p, e, begin, end) for the pieces [p, e) of the sequences [begin, end) that lie in a chunk, in order.  A sequence without a place
// belongs to the chunk where it would begin.
template <class F>
__device__ __forceinline__ void forwards(const Shape &d, uint32_t chunk, F f)
{
    const uint64_t p0 = (uint64_t)chunk * d.per_chunk, p1 = p0 + d.per_chunk < d.N ? p0 + d.per_chunk : d.N;
    uint32_t k = begun_before(d, p0);
    uint64_t begin, end;
    if (k > 0) {
        places(d, k - 1, begin, end);
        if (end > p0) f(k - 1, p0, end < p1 ? end : p1, begin, end);
    }
    for (; k < d.n_seq; ++k) {
        places(d, k, begin, end);
        if (begin >= p1 && chunk + 1 < d.n_chunks) break;
        f(k, begin, end < p1 ? end : p1, begin, end);
    }
}

template <class F>
__device__ __forceinline__ void backwards(const Shape &d, uint32_t chunk, F f)
{
    const uint64_t p0 = (uint64_t)chunk * d.per_chunk, p1 = p0 + d.per_chunk < d.N ? p0 + d.per_chunk : d.N;
    uint32_t k = chunk + 1 < d.n_chunks ? begun_before(d, p1) : d.n_seq;
    while (k-- > 0) {
        uint64_t begin, end;
        places(d, k, begin, end);
        const uint64_t p = begin > p0 ? begin : p0, e = end < p1 ? end : p1;
        if (begin >= p0 || e > p0) f(k, p, e, begin, end);
        if (begin < p0) break;
    }
}

// In both: the product of the gates of these tokens first, which is 0 or underflows only where one of them is shut or times() mends it.
template <class T, int V, int M, bool kFull, bool kShutting>
__device__ __forceinline__ void sum_loaded(const Pack<T, V> (&z)[M], const Pack<T, V> (&u)[M], int n, float (&A)[V], float (&h)[V])
{
    float product[V];
#pragma unroll
    for (int v = 0; v < V; ++v) product[v] = 1.0f;
#pragma unroll
    for (int k = 0; k < M; ++k)
        if (kFull || k < n) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Step s = step_of<kShutting>((float)z[k].v[v], (float)u[k].v[v]);
                h[v] = advance<kShutting>(s, h[v]);
                product[v] = kShutting ? times(product[v], s.a) : product[v] * s.a;
            }
        }
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = times(A[v], kShutting ? product[v] : fmaxf(product[v], kLeast));
}

template <class T, int V, int M, bool kFull>
__device__ __forceinline__ void sum_tokens(const Shape &d, const Fwd &f, uint32_t c, uint64_t p, int n, float (&A)[V], float (&h)[V])
{
    Pack<T, V> z[M], u[M];
    load_tokens<T, V, M, kFull>(Column<T, V>(d, f.z, f.ldz, c, p), n, z);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, f.u, f.ldu, c, p), n, u);
    if (any_shut<T, V, M>(z)) sum_loaded<T, V, M, kFull, true>(z, u, n, A, h);
    else sum_loaded<T, V, M, kFull, false>(z, u, n, A, h);
}

template <class T, int V, int M, bool kFull, bool kShutting>
__device__ __forceinline__ void sum_gradients_loaded(const Pack<T, V> (&z)[M], const Pack<T, V> (&dy)[M], int n, float (&A)[V], float (&G)[V])
{
    float product[V];
#pragma unroll
    for (int v = 0; v < V; ++v) product[v] = 1.0f;
#pragma unroll
    for (int k = M - 1; k >= 0; --k)
        if (kFull || k < n) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Step s = step_of<kShutting>((float)z[k].v[v], 0.0f);
                G[v] += (float)dy[k].v[v];
                G[v] = kShutting && s.a == 0.0f ? 0.0f : s.a * G[v];
                product[v] = kShutting ? times(product[v], s.a) : product[v] * s.a;
            }
        }
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = times(A[v], kShutting ? product[v] : fmaxf(product[v], kLeast));
}

template <class T, int V, int M, bool kFull>
__device__ __forceinline__ void sum_gradients(const Shape &d, const Bwd &b, uint32_t c, uint64_t p, int n, float (&A)[V], float (&G)[V])
{
    Pack<T, V> z[M], dy[M];
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.z, b.ldz, c, p), n, z);
    load_tokens<T, V, M, kFull>(Column<T, V>(d, b.dy, b.lddy, c, p), n, dy);
    if (any_shut<T, V, M>(z)) sum_gradients_loaded<T, V, M, kFull, true>(z, dy, n, A, G);
    else sum_gradients_loaded<T, V, M, kFull, false>(z, dy, n, A, G);
}

// sums[0]: A, sums[1]: B, each [n_chunks, W].  copy: NULL, or room for h0 (backward: dh_last), which the last launch then reads there
// because its own h_last (dh0) lies on it.
template <class T, int V>
__global__ void __launch_bounds__(kBlock)
chunk_sums_fwd_kernel(Shape d, Fwd f, float *sums, float *copy)
{
    uint32_t chunk, c;
    if (!lane_place(d, V, d.n_chunks, chunk, c)) return;
    float A[V], h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.0f, h[v] = 0.0f;
    forwards(d, chunk, [&](uint32_t k, uint64_t p, uint64_t e, uint64_t begin, uint64_t) {
        if (p == begin) {
#pragma unroll
            for (int v = 0; v < V; ++v) A[v] = 0.0f;
            get<V>(f.h0, (uint64_t)sequence(d, k) * d.W + c, h);
            put<V>(copy, (uint64_t)sequence(d, k) * d.W + c, h);
        }
        in_pieces(p, e, [&](uint64_t q, int n) {
            if (n == kKeep) sum_tokens<T, V, kKeep, true>(d, f, c, q, n, A, h);
            else sum_tokens<T, V, kKeep, false>(d, f, c, q, n, A, h);
        });
    });
    put<V>(sums, (uint64_t)chunk * d.W + c, A);
    put<V>(sums, ((uint64_t)d.n_chunks + chunk) * d.W + c, h);
}

template <class T, int V>
__global__ void __launch_bounds__(kBlock)
chunk_sums_bwd_kernel(Shape d, Bwd b, float *sums, float *copy)
{
    uint32_t chunk, c;
    if (!lane_place(d, V, d.n_chunks, chunk, c)) return;
    float A[V], G[V];
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.0f, G[v] = 0.0f;
    backwards(d, chunk, [&](uint32_t k, uint64_t p, uint64_t e, uint64_t, uint64_t end) {
        if (e == end) {
#pragma unroll
            for (int v = 0; v < V; ++v) A[v] = 0.0f;
            get<V>(b.dh_last, (uint64_t)sequence(d, k) * d.W + c, G);
            put<V>(copy, (uint64_t)sequence(d, k) * d.W + c, G);
        }
        while (e > p) {
            const uint64_t keep = (e - 1) / kKeep * kKeep, q = keep > p ? keep : p;
            const int n = (int)(e - q);
            if (n == kKeep) sum_gradients<T, V, kKeep, true>(d, b, c, q, n, A, G);
            else sum_gradients<T, V, kKeep, false>(d, b, c, q, n, A, G);
            e = q;
        }
    });
    put<V>(sums, (uint64_t)chunk * d.W + c, A);
    put<V>(sums, ((uint64_t)d.n_chunks + chunk) * d.W + c, G);
}

// What comes before each chunk (backward: behind it), written over its A.  A workgroup has 16 channels and cuts the chunks into
// 64 runs of at most P, which its threads hold in registers: each joins its run, then the runs before its own, then the chunks of its run.
constexpr int kJoinChannels = 16, kRuns = 64;

template <int P>
__global__ void __launch_bounds__(kJoinChannels *kRuns)
join_chunks_kernel(uint32_t n_chunks, uint32_t W, uint32_t from_the_end, float *sums)
{
    __shared__ float run_A[kRuns][kJoinChannels], run_B[kRuns][kJoinChannels];
    const uint32_t lane = threadIdx.x % kJoinChannels, run = threadIdx.x / kJoinChannels, c = blockIdx.x * kJoinChannels + lane;
    const uint32_t per = (n_chunks + kRuns - 1) / kRuns, k0 = run * per;
    const uint64_t to_B = (uint64_t)n_chunks * W;
    auto held = [&](int i) { return (uint32_t)i < per && k0 + i < n_chunks && c < W; };
    auto at = [&](int i) { return (uint64_t)(from_the_end ? n_chunks - 1 - (k0 + i) : k0 + i) * W + c; };
    float a[P], b[P], A = 1.0f, B = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        a[i] = held(i) ? sums[at(i)] : 1.0f;
        b[i] = held(i) ? sums[to_B + at(i)] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        B = join(a[i], B, b[i]);
        A = times(A, a[i]);
    }
    run_A[run][lane] = A;
    run_B[run][lane] = B;
    __syncthreads();
    float h = 0.0f;
    for (uint32_t r = 0; r < run; ++r) h = join(run_A[r][lane], h, run_B[r][lane]);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if (held(i)) sums[at(i)] = h;
        h = join(a[i], h, b[i]);
    }
}

void join_chunks(uint32_t n_chunks, uint32_t W, uint32_t from_the_end, float *sums, hipStream_t st)
{
    const uint32_t grid = (W + kJoinChannels - 1) / kJoinChannels;
    auto go = [&](auto kernel) { kernel<<<grid, kJoinChannels * kRuns, 0, st>>>(n_chunks, W, from_the_end, sums); };
    n_chunks <= 8 * kRuns ? go(join_chunks_kernel<8>) : go(join_chunks_kernel<32>);
}

template <class T, int V>
__global__ void __launch_bounds__(kBlock)
chunk_fwd_kernel(Shape d, Fwd f, const float *sums)
{
    uint32_t chunk, c;
    if (!lane_place(d, V, d.n_chunks, chunk, c)) return;
    float h[V];
    get<V>(sums, (uint64_t)chunk * d.W + c, h);
    forwards(d, chunk, [&](uint32_t k, uint64_t p, uint64_t e, uint64_t begin, uint64_t end) {
        const uint64_t at = (uint64_t)sequence(d, k) * d.W + c;
        if (p == begin) get<V>(f.h0, at, h);
        advance_places<T, V>(d, f, c, p, e, h);
        if (e == end) put<V>(f.h_last, at, h);
    });
}

template <class T, int V>
__global__ void __launch_bounds__(kBlock)
chunk_bwd_kernel(Shape d, Bwd b, const float *sums)
{
    uint32_t chunk, c;
    if (!lane_place(d, V, d.n_chunks, chunk, c)) return;
    float G[V];
    get<V>(sums, (uint64_t)chunk * d.W + c, G);
    backwards(d, chunk, [&](uint32_t k, uint64_t p, uint64_t e, uint64_t begin, uint64_t end) {
        const uint32_t seq = sequence(d, k);
        const uint64_t at = (uint64_t)seq * d.W + c;
        if (e == end) get<V>(b.dh_last, at, G);
        retreat_places<T, V>(d, b, seq, c, begin, p, e, G);
        if (p == begin) put<V>(b.dh0, at, G);
    });
}

int check(const char *who, Shape &d, uint32_t dtype)
{
    DG_REQUIRE(known_type(dtype), DG_ERR_ARG, "%s: unknown element type %u", who, dtype);
    DG_REQUIRE(d.W >= 1, DG_ERR_ARG, "%s: rows without a channel", who);
    DG_REQUIRE(d.N < 1ull << 32 && d.W <= 1u << 20, DG_ERR_UNSUPPORTED, "%s: 2^32 tokens or more, or more than 2^20 channels", who);
    DG_REQUIRE(dg::aligned(d.first, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    DG_REQUIRE(d.n_seq > 0 || d.N == 0, DG_ERR_ARG, "%s: tokens without a sequence", who);
    DG_REQUIRE(d.first || d.n_seq == 0 || d.N % d.n_seq == 0, DG_ERR_ARG, "%s: %llu tokens are not %u sequences of one length", who, (unsigned long long)d.N,
               d.n_seq);
    d.S = d.n_seq ? (uint32_t)(d.N / d.n_seq) : 0;
    DG_REQUIRE((uint64_t)d.n_seq * d.W <= 1ull << 38, DG_ERR_UNSUPPORTED, "%s: too many sequences for one launch", who);
    return DG_OK;
}

int check_rows(const char *who, const void *p, uint64_t ld, const Shape &d, uint32_t dtype)
{
    if (d.N == 0) return DG_OK;
    DG_REQUIRE(p && dg::aligned(p, item_bytes(dtype)), DG_ERR_ARG, "%s: null or misaligned pointer", who);
    DG_REQUIRE(ld >= d.W && ld <= 1ull << 40, DG_ERR_ARG, "%s: rows of %u channels lie %llu apart", who, d.W, (unsigned long long)ld);
    return DG_OK;
}

// Few sequences: chunks of places instead, enough of them for kWanted lanes of two channels, each of kKeep places at least.
constexpr uint64_t kWanted = 1 << 18;
constexpr uint32_t kMostChunks = 32 * kRuns;

void cut(Shape &d)
{
    d.n_chunks = d.per_chunk = 0;
    const uint64_t pairs = (d.W + 1) / 2;
    if (d.n_seq == 0 || d.N / d.n_seq < 4 * kKeep || d.n_seq * pairs >= kWanted / 4) return;
    uint64_t n = kWanted / pairs;
    n = n < kMostChunks ? n : kMostChunks;
    uint64_t per = (d.N + n - 1) / n;
    per = (per + kKeep - 1) / kKeep * kKeep;
    d.per_chunk = (uint32_t)per;
    d.n_chunks = (uint32_t)((d.N + per - 1) / per);
}

uint32_t blocks(uint64_t count, uint32_t W, uint32_t V) { return (uint32_t)((count * (W / V) + kBlock - 1) / kBlock); }

template <class T, int V>
void launch_fwd(const Shape &d, Fwd f, float *sums, hipStream_t st)
{
    if (!d.n_chunks) {
        sequence_fwd_kernel<T, V><<<blocks(d.n_seq, d.W, V), kBlock, 0, st>>>(d, f);
        return;
    }
    const uint32_t grid = blocks(d.n_chunks, d.W, V);
    float *copy = f.h0 && f.h0 == f.h_last ? sums + (size_t)d.n_chunks * d.W * 2 : nullptr;
    chunk_sums_fwd_kernel<T, V><<<grid, kBlock, 0, st>>>(d, f, sums, copy);
    if (copy) f.h0 = copy;
    join_chunks(d.n_chunks, d.W, 0, sums, st);
    chunk_fwd_kernel<T, V><<<grid, kBlock, 0, st>>>(d, f, sums);
}

template <class T, int V>
void launch_bwd(const Shape &d, Bwd b, float *sums, hipStream_t st)
{
    if (!d.n_chunks) {
        sequence_bwd_kernel<T, V><<<blocks(d.n_seq, d.W, V), kBlock, 0, st>>>(d, b);
        return;
    }
    const uint32_t grid = blocks(d.n_chunks, d.W, V);
    float *copy = b.dh_last && b.dh_last == b.dh0 ? sums + (size_t)d.n_chunks * d.W * 2 : nullptr;
    chunk_sums_bwd_kernel<T, V><<<grid, kBlock, 0, st>>>(d, b, sums, copy);
    if (copy) b.dh_last = copy;
    join_chunks(d.n_chunks, d.W, 1, sums, st);
    chunk_bwd_kernel<T, V><<<grid, kBlock, 0, st>>>(d, b, sums);
}

// sums of the chunks, and room for a copy of the states
size_t workspace_bytes(const Shape &d) { return d.n_chunks ? ((size_t)d.n_chunks * 2 + d.n_seq) * d.W * sizeof(float) : 0; }

int check_workspace(const char *who, const Shape &d, const void *ws, size_t ws_bytes)
{
    const size_t need = workspace_bytes(d);
    DG_REQUIRE(need == 0 || (ws && dg::aligned(ws, 16) && ws_bytes >= need), DG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need,
               ws ? ws_bytes : 0);
    return DG_OK;
}

}  // namespace

extern "C" size_t dg_recurrence_state_count(uint64_t N, uint32_t W) { return (size_t)((N + kKeep - 1) / kKeep) * W; }

extern "C" size_t dg_recurrence_workspace_bytes(uint64_t N, uint32_t n_seq, uint32_t W)
{
    Shape d = {N, n_seq, W, 0, nullptr, false, 0, 0};
    cut(d);
    return workspace_bytes(d);
}

extern "C" int dg_recurrence_fwd(const void *z, uint64_t ldz, const void *u, uint64_t ldu, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t W,
                                 uint32_t reverse, uint32_t dtype, const float *h0, void *y, uint64_t ldy, float *h_last, float *states, void *ws,
                                 size_t ws_bytes, void *stream)
{
    const char *who = "dg_recurrence_fwd";
    Shape d = {N, n_seq, W, 0, first, reverse != 0, 0, 0};
    if (int rc = check(who, d, dtype)) return rc;
    if (int rc = check_rows(who, z, ldz, d, dtype)) return rc;
    if (int rc = check_rows(who, u, ldu, d, dtype)) return rc;
    if (int rc = check_rows(who, y, ldy, d, dtype)) return rc;
    DG_REQUIRE(dg::aligned(h0, 4) && dg::aligned(h_last, 4) && dg::aligned(states, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (n_seq == 0) return DG_OK;
    cut(d);
    if (int rc = check_workspace(who, d, ws, ws_bytes)) return rc;
    const Fwd f = {z, u, y, ldz, ldu, ldy, h0, h_last, states};
    const bool pairs = W % 2 == 0 && rows_aligned(z, ldz, dtype, 4) && rows_aligned(u, ldu, dtype, 4) && rows_aligned(y, ldy, dtype, 4);
    (dtype == DG_F32   ? launch_fwd<float, 1>
     : dtype == DG_F16 ? (pairs ? launch_fwd<f16, 2> : launch_fwd<f16, 1>)
                       : (pairs ? launch_fwd<bf16, 2> : launch_fwd<bf16, 1>))(d, f, (float *)ws, (hipStream_t)stream);
    return dg::launch_status(who);
}

extern "C" int dg_recurrence_bwd(const void *z, uint64_t ldz, const void *u, uint64_t ldu, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t W,
                                 uint32_t reverse, uint32_t dtype, const float *h0, const float *states, const void *dy, uint64_t lddy,
                                 const float *dh_last, void *dz, uint64_t lddz, void *du, uint64_t lddu, float *dh0, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "dg_recurrence_bwd";
    Shape d = {N, n_seq, W, 0, first, reverse != 0, 0, 0};
    if (int rc = check(who, d, dtype)) return rc;
    const struct { const void *p; uint64_t ld; } rows[] = {{z, ldz}, {u, ldu}, {dy, lddy}, {dz, lddz}, {du, lddu}};
    for (const auto &r : rows)
        if (int rc = check_rows(who, r.p, r.ld, d, dtype)) return rc;
    DG_REQUIRE(N == 0 || states, DG_ERR_ARG, "%s: the states that the forward pass kept are missing", who);
    DG_REQUIRE(dg::aligned(h0, 4) && dg::aligned(states, 4) && dg::aligned(dh_last, 4) && dg::aligned(dh0, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (n_seq == 0) return DG_OK;
    cut(d);
    if (int rc = check_workspace(who, d, ws, ws_bytes)) return rc;
    const Bwd b = {z, u, dy, dz, du, ldz, ldu, lddy, lddz, lddu, h0, states, dh_last, dh0};
    bool pairs = W % 2 == 0;
    for (const auto &r : rows) pairs = pairs && rows_aligned(r.p, r.ld, dtype, 4);
    (dtype == DG_F32   ? launch_bwd<float, 1>
     : dtype == DG_F16 ? (pairs ? launch_bwd<f16, 2> : launch_bwd<f16, 1>)
                       : (pairs ? launch_bwd<bf16, 2> : launch_bwd<bf16, 1>))(d, b, (float *)ws, (hipStream_t)stream);
    return dg::launch_status(who);
}
