// The gated delta rule of small heads (up to 32 x 32), token by token: a lane has a column of the memory in its registers along a sequence, or a row of it where
// the gradients of q and k are wanted, so that every sum over the memory stays in a lane; a wavefront has as many heads or sequences as fit side by side.
//
// Forward, and backward along the sequences (dR of what tokens write, with it dv, dbeta): columns.  Then, with what tokens write and its gradient known,
// 64 tokens at a time: rows, once forward (dq, and what dk owes to the memory that was read), once backward (what dk owes to the memory that is written).
// Bound by the vector units: four operations per value of the memory and token in each of the four sweeps.  Vectors that all lanes of a head need lie over 16 lanes, from which
// moves between lanes hand each value to all (when every lane loaded all of them, the first-level cache was what bounded: 2.8 ms for the gradients' rows, 1.7 now).
// 65536 rays of 64 samples, 2 heads of 16 x 16, fp16: forward 0.50 ms, backward along the rays 0.68 (3.4 TB/s), rows 1.70, some 340 operations of a wavefront for 4 tokens.
#include <utility>
#include "delta_common.h"
#include "rows_vectors.h"

namespace {

using namespace dg_delta;

constexpr int kAhead = 4;               // tokens that are loaded before they are needed

template <class F, int... I>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F f) { (f(std::integral_constant<int, I>{}), ...); }
template <int n, class F>
__device__ __forceinline__ void each(F f) { each(std::make_integer_sequence<int, n>{}, f); }

// P values that all lanes of a head need: lane l of 16 has l, l + 16, ...; 0 from D on
template <class T, int P>
struct Vector {
    T v[P / 16];
    __device__ __forceinline__ void load(const T *row, uint32_t D)
    {
#pragma unroll
        for (int i = 0; i < P / 16; ++i) {
            const uint32_t c = i * 16 + threadIdx.x % 16;
            v[i] = row[c < D ? c : 0];
        }
    }
};

// the same in fp32, cleared from D on
template <int P>
struct Spread {
    float v[P / 16];
    template <class T>
    __device__ __forceinline__ Spread(const Vector<T, P> &from, uint32_t D)
    {
#pragma unroll
        for (int i = 0; i < P / 16; ++i) v[i] = i * 16 + threadIdx.x % 16 < D ? (float)from.v[i] : 0.0f;
    }
    template <int i>
    __device__ __forceinline__ float at() const
    {
        return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v[i / 16]), 0x150 + i % 16, 0xf, 0xf, true));       // value i % 16 of the row's lanes
    }
};

// sum of products, in four parts
template <int P>
__device__ __forceinline__ float dot(const float (&a)[P], const Spread<P> &b)
{
    float part[4] = {};
    each<P>([&](auto i) { part[i % 4] = fmaf(b.template at<i>(), a[i], part[i % 4]); });
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// a <- a f + b s
template <int P>
__device__ __forceinline__ void step(float (&a)[P], float f, const Spread<P> &b, float s)
{
    each<P>([&](auto i) { a[i] = fmaf(b.template at<i>(), s, a[i] * f); });
}

// a <- a + b s
template <int P>
__device__ __forceinline__ void add(float (&a)[P], const Spread<P> &b, float s)
{
    each<P>([&](auto i) { a[i] = fmaf(b.template at<i>(), s, a[i]); });
}

// a place in rows that goes from token to token
template <class T>
struct Walk {
    T *p;
    int64_t step;
    __device__ __forceinline__ Walk(T *base, uint64_t ld, const Span &span, uint32_t t, bool back) : p(base + span.row(t) * ld), step((span.turn < 0) != back ? -(int64_t)ld : (int64_t)ld) {}
    __device__ __forceinline__ void next() { p += step; }
};

// use(token) for count tokens, each fetched kAhead before: fetch() loads what the places point at, go() moves these on.  No branch about a load (behind the last token it comes again), so that
// a wait is for the oldest loads only.
template <class Token, class Fetch, class Go, class Use>
__device__ __forceinline__ void along_tokens(uint32_t count, Fetch fetch, Go go, Use use)
{
    Token ahead[kAhead];
    uint32_t at = 0;                    // of the token that is fetched next
    auto get = [&](Token &to) {
        fetch(to);
        if (++at < count) go();
    };
    each<kAhead>([&](auto i) { get(ahead[i]); });
    uint32_t t = 0;
    for (; t + kAhead <= count; t += kAhead)
        each<kAhead>([&](auto i) {
            const Token now = ahead[i];
            __builtin_amdgcn_sched_barrier(0);
            get(ahead[i]);
            __builtin_amdgcn_sched_barrier(0);
            use(t + i, now);
        });
    each<kAhead - 1>([&](auto i) {
        if (t + i < count) use(t + i, ahead[i]);
    });
}

// A lane's place among the heads of all sequences: sequence, head, column
struct Place {
    uint32_t seq, head, column;
    bool in;
    template <int P>
    __device__ __forceinline__ static Place of(const Delta &d, uint64_t from)
    {
        const uint64_t unit = (from + blockIdx.x) * (64 / P) + threadIdx.x / P, all = (uint64_t)d.n_seq * d.H;
        const uint64_t here = unit < all ? unit : all - 1;
        return {(uint32_t)(here / d.H), (uint32_t)(here % d.H), threadIdx.x % P, unit < all};
    }
};

template <class T, int PK, int PV>
__global__ void __launch_bounds__(64)
delta_small_fwd_kernel(Delta d, uint64_t from)
{
    const Place at = Place::of<PV>(d, from);
    const Span span = span_of(d, at.seq);
    const uint32_t hk = at.head / (d.H / d.Hk), c = at.column < d.Dv ? at.column : 0, ldy = d.H * d.Dv;
    const bool in = at.in && at.column < d.Dv;
    const uint32_t len = at.in ? span.len : 0;
    const uint64_t memory = ((uint64_t)at.seq * d.H + at.head) * d.Dk * d.Dv + c;
    float S[PK];
#pragma unroll
    for (int r = 0; r < PK; ++r) S[r] = d.s0 && in && r < (int)d.Dk ? d.s0[memory + (uint64_t)r * d.Dv] : 0.0f;
    if (len) {
        Walk<const T> K((const T *)d.k + hk * d.Dk, d.ldk, span, 0, false), Q((const T *)d.q + hk * d.Dk, d.ldq, span, 0, false), V((const T *)d.v + at.head * d.Dv + c, d.ldv, span, 0, false);
        Walk<const float> G(d.g + at.head, d.ldg, span, 0, false), B(d.beta + at.head, d.ldb, span, 0, false);
        Walk<T> O((T *)d.o + at.head * d.Dv + c, d.ldo, span, 0, false);
        Walk<float> Y(d.y + at.head * d.Dv + c, ldy, span, 0, false);
        float *mark = d.marks + ((uint64_t)first_slot(span, at.seq) * d.H + at.head) * d.Dk * d.Dv + c;
        struct Token {
            Vector<T, PK> k, q;
            T v;
            float g, beta;
        };
        along_tokens<Token>(len,
            [&](Token &to) {
                to.k.load(K.p, d.Dk);
                to.q.load(Q.p, d.Dk);
                to.v = *V.p, to.g = *G.p, to.beta = *B.p;
            },
            [&] { K.next(), Q.next(), V.next(), G.next(), B.next(); },
            [&](uint32_t t, const Token &now) {
                if (d.marks && t % kMark == 0) {
                    if (in)
#pragma unroll
                        for (int r = 0; r < PK; ++r)
                            if (r < (int)d.Dk) mark[(uint64_t)r * d.Dv] = S[r];
                    mark += (uint64_t)d.H * d.Dk * d.Dv;
                }
                const Spread<PK> k(now.k, d.Dk), q(now.q, d.Dk);
                const float a = expf(now.g), y = (float)now.v - a * dot(S, k);
                step(S, a, k, now.beta * y);
                const float o = d.scale * dot(S, q);
                if (in) {
                    *O.p = (T)o;
                    if (d.y) *Y.p = y;
                }
                O.next(), Y.next();
            });
    }
    if (d.s_last && in)
#pragma unroll
        for (int r = 0; r < PK; ++r)
            if (r < (int)d.Dk) d.s_last[memory + (uint64_t)r * d.Dv] = S[r];
}

// dS of a token: + scale q do^T;  dR = dS^T k;  - k (beta dR)^T;  e^g dS goes to the token before.  dg gets v dv, for what follows.
template <class T, int PK, int PV>
__global__ void __launch_bounds__(64)
delta_small_bwd_kernel(Delta d, uint64_t from)
{
    const Place at = Place::of<PV>(d, from);
    const Span span = span_of(d, at.seq);
    const uint32_t hk = at.head / (d.H / d.Hk), c = at.column < d.Dv ? at.column : 0, ldy = d.H * d.Dv;
    const bool in = at.in && at.column < d.Dv;
    const uint32_t len = at.in ? span.len : 0, last = len ? len - 1 : 0;
    const uint64_t memory = ((uint64_t)at.seq * d.H + at.head) * d.Dk * d.Dv + c;
    float S[PK];
#pragma unroll
    for (int r = 0; r < PK; ++r) S[r] = d.ds_last && in && r < (int)d.Dk ? d.ds_last[memory + (uint64_t)r * d.Dv] : 0.0f;
    if (len) {
        Walk<const T> K((const T *)d.k + hk * d.Dk, d.ldk, span, last, true), Q((const T *)d.q + hk * d.Dk, d.ldq, span, last, true);
        Walk<const T> V((const T *)d.v + at.head * d.Dv + c, d.ldv, span, last, true), O((const T *)d.dout + at.head * d.Dv + c, d.lddo, span, last, true);
        Walk<const float> G(d.g + at.head, d.ldg, span, last, true), B(d.beta + at.head, d.ldb, span, last, true), Y(d.y + at.head * d.Dv + c, ldy, span, last, true);
        Walk<T> dV((T *)d.dv + at.head * d.Dv + c, d.lddv, span, last, true);
        Walk<float> R(d.dr + at.head * d.Dv + c, ldy, span, last, true), dB(d.dbeta + at.head, d.lddb, span, last, true), dG(d.dg + at.head, d.lddg, span, last, true);
        float *mark = d.dmarks + ((uint64_t)(first_slot(span, at.seq) + last / kMark) * d.H + at.head) * d.Dk * d.Dv + c;
        struct Token {
            Vector<T, PK> k, q;
            T v, o;
            float g, beta, y;
        };
        along_tokens<Token>(len,
            [&](Token &to) {
                to.k.load(K.p, d.Dk);
                to.q.load(Q.p, d.Dk);
                to.v = *V.p, to.o = *O.p, to.g = *G.p, to.beta = *B.p, to.y = *Y.p;
            },
            [&] { K.next(), Q.next(), V.next(), O.next(), G.next(), B.next(), Y.next(); },
            [&](uint32_t i, const Token &now) {
                const uint32_t t = last - i;
                if (t % kMark == kMark - 1 || i == 0) {
                    if (in)
#pragma unroll
                        for (int r = 0; r < PK; ++r)
                            if (r < (int)d.Dk) mark[(uint64_t)r * d.Dv] = S[r];
                    mark -= (uint64_t)d.H * d.Dk * d.Dv;
                }
                const Spread<PK> k(now.k, d.Dk), q(now.q, d.Dk);
                add(S, q, d.scale * (in ? (float)now.o : 0.0f));
                const float a = expf(now.g), dr = dot(S, k), dv = now.beta * dr;
                step(S, a, k, -a * dv);
                // the lanes of a head go through the same tokens: all of them are here
                const float dbeta = dg_rows::group_sum<PV>(in ? dr * now.y : 0.0f), values = dg_rows::group_sum<PV>(in ? dv * (float)now.v : 0.0f);
                if (in) {
                    *R.p = dr;
                    *dV.p = (T)dv;
                    if (at.column == 0) {
                        *dB.p = dbeta;
                        *dG.p = values;
                    }
                }
                R.next(), dV.next(), dB.next(), dG.next();
            });
    }
    if (d.ds0 && in)
#pragma unroll
        for (int r = 0; r < PK; ++r)
            if (r < (int)d.Dk) d.ds0[memory + (uint64_t)r * d.Dv] = S[r];
}

// Rows: 64 tokens of a key head, one of its value heads after the other
template <class T, int PK, int PV, bool kShared>
__global__ void __launch_bounds__(64)
delta_small_grad_kernel(Delta d, uint64_t from)
{
    constexpr int kUnits = 64 / PK;
    __shared__ float lds_k[kMark][64], lds_q[kShared ? kMark : 1][64], lds_end[kMark][kUnits];      // dk, dq of shared keys, q dq
    const uint32_t lane = threadIdx.x, group = d.H / d.Hk;
    const uint64_t slots = d.first ? d.slots : (uint64_t)d.n_seq * ((d.N / d.n_seq + kMark - 1) / kMark), unit = (from + blockIdx.x) * kUnits + lane / PK;
    const uint32_t hk = (uint32_t)(unit % d.Hk), r = lane % PK < d.Dk ? lane % PK : 0;
    uint64_t slot = unit / d.Hk;
    bool there = slot < slots;
    uint32_t seq = 0, block = 0;
    if (there && d.first) {
        seq = d.slot_seq[slot];
        there = seq < d.n_seq;
    } else if (there) {
        const uint64_t each = (d.N / d.n_seq + kMark - 1) / kMark;
        seq = (uint32_t)(slot / each);
        block = (uint32_t)(slot % each);
    }
    if (!there) seq = 0;
    const Span span = span_of(d, seq);
    if (there && d.first) block = (uint32_t)(slot - first_slot(span, seq));
    slot = first_slot(span, seq) + block;
    const uint32_t t0 = block * kMark;
    there = there && t0 < span.len;
    const uint32_t count = !there ? 0 : span.len - t0 < kMark ? span.len - t0 : kMark;
    const bool in = there && lane % PK < d.Dk;
    if (!there) return;
    const uint32_t last = t0 + count - 1, ldy = d.H * d.Dv;
    for (uint32_t h = 0; h < group; ++h) {
        const uint32_t head = hk * group + h;
        const uint64_t memory = ((slot * d.H + head) * d.Dk + r) * d.Dv;
        float S[PV], end = 0.0f;
        struct Token {
            Vector<float, PV> y, dr;
            Vector<T, PV> o;
            T k, q;
            float g, beta;
        };
        struct Rows {
            Walk<const float> Y, R, G, B;
            Walk<const T> O, K, Q;
            __device__ __forceinline__ Rows(const Delta &d, const Span &span, uint32_t t, bool back, uint32_t head, uint32_t column, uint32_t ldy)
                : Y(d.y + head * d.Dv, ldy, span, t, back), R(d.dr + head * d.Dv, ldy, span, t, back), G(d.g + head, d.ldg, span, t, back), B(d.beta + head, d.ldb, span, t, back),
                  O((const T *)d.dout + head * d.Dv, d.lddo, span, t, back), K((const T *)d.k + column, d.ldk, span, t, back), Q((const T *)d.q + column, d.ldq, span, t, back) {}
            __device__ __forceinline__ void next() { Y.next(), R.next(), G.next(), B.next(), O.next(), K.next(), Q.next(); }
            __device__ __forceinline__ void fetch(Token &to, uint32_t Dv) const
            {
                to.y.load(Y.p, Dv);
                to.dr.load(R.p, Dv);
                to.o.load(O.p, Dv);
                to.k = *K.p, to.q = *Q.p, to.g = *G.p, to.beta = *B.p;
            }
        };
        {
            Rows at(d, span, t0, false, head, hk * d.Dk + r, ldy);
            Walk<T> dQ((T *)d.dq + hk * d.Dk + r, d.lddq, span, t0, false);
#pragma unroll
            for (int i = 0; i < PV; ++i) S[i] = in && i < (int)d.Dv ? d.marks[memory + i] : 0.0f;
            along_tokens<Token>(count, [&](Token &to) { at.fetch(to, d.Dv); }, [&] { at.next(); }, [&](uint32_t t, const Token &now) {
                const float k = in ? (float)now.k : 0.0f, q = in ? (float)now.q : 0.0f, a = expf(now.g);
                const Spread<PV> y(now.y, d.Dv), dr(now.dr, d.Dv), o(now.o, d.Dv);
                const float read = -now.beta * a * dot(S, dr);
                step(S, a, y, k * now.beta);
                float dq = d.scale * dot(S, o);
                const float all = dg_rows::group_sum<PK>(q * dq);
                if (lane % PK == 0) lds_end[t][lane / PK] = all;
                lds_k[t][lane] = kShared && h ? lds_k[t][lane] + read : read;
                if (kShared) lds_q[t][lane] = dq = h ? lds_q[t][lane] + dq : dq;
                if (h + 1 == group && in) *dQ.p = (T)dq;
                dQ.next();
            });
        }
        Rows at(d, span, last, true, head, hk * d.Dk + r, ldy);
        Walk<T> dK((T *)d.dk + hk * d.Dk + r, d.lddk, span, last, true);
        Walk<float> dG(d.dg + head, d.lddg, span, last, true);
        float dS[PV];
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            dS[i] = in && i < (int)d.Dv ? d.dmarks[memory + i] : 0.0f;
            end = fmaf(S[i], dS[i], end);
        }
        end = dg_rows::group_sum<PK>(end);
        along_tokens<Token>(count, [&](Token &to) { at.fetch(to, d.Dv); }, [&] { at.next(); }, [&](uint32_t i, const Token &now) {
            const uint32_t t = count - 1 - i;
            const float k = in ? (float)now.k : 0.0f, q = in ? (float)now.q : 0.0f, a = expf(now.g);
            const Spread<PV> y(now.y, d.Dv), dr(now.dr, d.Dv), o(now.o, d.Dv);
            add(dS, o, d.scale * q);
            const float dk = fmaf(now.beta, dot(dS, y), lds_k[t][lane]);
            step(dS, a, dr, -a * now.beta * k);
            if (lane % PK == 0) {               // values of v dv lie where dg comes
                end += lds_end[t][lane / PK] - *dG.p;
                if (keeps_nothing(now.g)) end = 0.0f;
                *dG.p = end;
            }
            if (h + 1 < group) lds_k[t][lane] = dk;
            else if (in) *dK.p = (T)dk;
            dK.next(), dG.next();
        });
    }
}

// a launch's workgroups of a wavefront each
template <class Go>
void in_turns(uint64_t all, Go go)
{
    for (uint64_t from = 0; from < all; from += kMostLaunched) go((uint32_t)(all - from < kMostLaunched ? all - from : kMostLaunched), from);
}

template <class T, int PK, int PV>
void launch_size(const Delta &d, bool back, hipStream_t st)
{
    const uint64_t along = ((uint64_t)d.n_seq * d.H + 64 / PV - 1) / (64 / PV);
    if (!back) return in_turns(along, [&](uint32_t grid, uint64_t from) { delta_small_fwd_kernel<T, PK, PV><<<grid, 64, 0, st>>>(d, from); });
    in_turns(along, [&](uint32_t grid, uint64_t from) { delta_small_bwd_kernel<T, PK, PV><<<grid, 64, 0, st>>>(d, from); });
    if (d.N == 0) return;
    const uint64_t slots = d.first ? d.slots : (uint64_t)d.n_seq * ((d.N / d.n_seq + kMark - 1) / kMark);
    in_turns((slots * d.Hk + 64 / PK - 1) / (64 / PK), [&](uint32_t grid, uint64_t from) {
        if (d.H == d.Hk) delta_small_grad_kernel<T, PK, PV, false><<<grid, 64, 0, st>>>(d, from);
        else delta_small_grad_kernel<T, PK, PV, true><<<grid, 64, 0, st>>>(d, from);
    });
}

template <class T>
void launch_type(const Delta &d, bool back, hipStream_t st)
{
    if (d.Dk <= 16) d.Dv <= 16 ? launch_size<T, 16, 16>(d, back, st) : launch_size<T, 16, 32>(d, back, st);
    else d.Dv <= 16 ? launch_size<T, 32, 16>(d, back, st) : launch_size<T, 32, 32>(d, back, st);
}

}  // namespace

void dg_delta::launch_small(const Delta &d, uint32_t dtype, bool back, hipStream_t st)
{
    if (dtype == DG_F32) launch_type<float>(d, back, st);
    else if (dtype == DG_F16) launch_type<f16>(d, back, st);
    else launch_type<bf16>(d, back, st);
}
