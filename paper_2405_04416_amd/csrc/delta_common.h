// The gated delta rule: what its kernels share.  Internal.
//
// Per head, with a memory S [Dk, Dv]:  S <- e^g S;  S <- S + beta k (v - S^T k)^T;  o = scale S^T q.
// Over a chunk of tokens, S the memory before it, G the sums of g from its start on, D[i, j] = e^(G[i] - G[j]):
//   A[i, j] = D[i, j] k[i] k[j] beta[j]  (j < i),   T = (1 + A)^-1,   P[i, j] = scale D[i, j] q[i] k[j]  (j <= i),
//   Y = T (V - e^G K S)  (what the tokens miss),   U = beta Y  (what they write),   O = scale e^G Q S + P U,   S' = e^G[last] S + K^T (e^(G[last] - G) U).
//
// Products are taken on the matrix units in bf16, of values that are cut into pieces of 8 bits: one for a bf16 value, two for fp16, three for
// fp32, which lose nothing.  Of the products of pieces the smallest three of nine are left out: at most 2^-22 of the product of two values, of either sign (second pieces are rounded: cut off they would leave
// up to 2^-21, always of the product's sign).  A single product is off by 0.7 U in root mean square, U = 2^-24, where fp32 has 0.4; a sum by its roundings, as in fp32.  All of it at several times the rate
// of the fp32 matrix instruction (139 TFLOP/s measured; three bf16 products 445).
#pragma once
#include "rows_common.h"

namespace dg_delta {

using dg_rows::bf16;
using dg_rows::f16;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMark = 64;               // tokens between memories that the forward pass leaves for the backward pass
constexpr int kMaxD = 128;
constexpr uint64_t kMostLaunched = 1 << 22;     // workgroups of a launch: its lanes have to stay below 2^32
// e^-104 is 0 in fp32: below that a gate is shut.  Logarithms are cut off here so that their differences stay numbers.
constexpr float kShut = -200.0f;
__device__ __forceinline__ float cut_off(float g) { return g < kShut ? kShut : g; }     // NaN stays NaN
// A gate that keeps nothing at all: what comes after it has no part in gradients before it.  That of the gates, a sum of what comes after them of which all but their own part cancels, ends there.
__device__ __forceinline__ bool keeps_nothing(float g) { return g < -104.0f; }

struct Weights;

struct Delta {
    const void *q, *k, *v;
    const float *g, *beta;
    uint64_t ldq, ldk, ldv, ldg, ldb;
    const float *s0, *ds_last;
    void *o;
    const void *dout;
    uint64_t ldo, lddo;
    float *s_last, *ds0;
    float *marks, *dmarks;              // [slots][H][Dk][Dv]: memories before each 64 tokens, gradients of those after
    float *y, *dr;                      // [N][H][Dv]: what tokens miss, v - S^T k, and the gradient of what they write, beta times that
    void *dq, *dk, *dv;
    uint64_t lddq, lddk, lddv;
    float *dg, *dbeta;
    uint64_t lddg, lddb;
    const uint32_t *first;
    const uint32_t *slot_seq, *chunk_seq;       // whose the slots of 64 and of 32 tokens are
    Weights *weights;                           // [chunk slots][H]
    uint64_t N;
    uint32_t n_seq, Hk, H, Dk, Dv, reverse, slots;
    // Sequences cut in parts of `stretch` tokens (1: whole): what a part makes of no memory and of every column of the unit matrix, [n_seq][parts][H][Dk][ends_width()], and memories before them
    uint32_t parts, stretch;
    float *ends, *starts;
    __host__ __device__ uint32_t ends_width() const { return (Dv + 15) / 16 * 16 + (Dk + 15) / 16 * 16; }
    float scale;
    // Whether heads' rows lie in whole 16 bytes: q and k; q, k, v and, backward, the gradient of o, and with them rows of fp32 values; dv, dq and dk too.  Kernels take it as a template
    // argument: of a branch between loads of 16 bytes and single ones the compiler makes single ones for both.
    bool vec_keys, vec_all, vec_out;
};

template <class T>
struct Pieces { static constexpr int n = sizeof(T) == 4 ? 3 : 2; };
template <>
struct Pieces<bf16> { static constexpr int n = 1; };

// ------------------------------------------------------------------------------ sequences
struct Span {
    uint64_t begin;
    uint32_t len;
    int32_t turn;                       // -1: from the last row to the first, else 0
    // row of token i < len, of which there may be 2^31 and more: all in 32 bits without a sign, then added.  Without a branch, which would keep loads apart
    __host__ __device__ __forceinline__ uint64_t row(uint32_t i) const { return begin + ((i ^ (uint32_t)turn) + ((uint32_t)turn & len)); }
};

// no row from N on, whatever the offsets say
__device__ __forceinline__ Span span_of(const Delta &d, uint32_t seq)
{
    if (!d.first) {
        const uint64_t len = d.N / d.n_seq;
        return {seq * len, (uint32_t)len, d.reverse ? -1 : 0};
    }
    const uint64_t b = d.first[seq], e = d.first[seq + 1], begin = b < d.N ? b : d.N, end = e < d.N ? e : d.N;
    return {begin, end > begin ? (uint32_t)(end - begin) : 0u, d.reverse ? -1 : 0};
}

// a part of a sequence
__device__ __forceinline__ Span part_of(const Span &s, uint32_t part, uint32_t stretch)
{
    const uint32_t t0 = part * stretch, len = s.len - t0 < stretch ? s.len - t0 : stretch;
    return {s.turn ? s.begin + (s.len - t0 - len) : s.begin + t0, len, s.turn};
}

// Where the memories of a sequence are left: every sequence begins one slot after floor(begin / 64) more than the one before, which leaves room for all
// of them, whatever the lengths.
__device__ __forceinline__ uint32_t first_slot(const Span &s, uint32_t seq) { return (uint32_t)(s.begin / kMark) + seq; }

// ------------------------------------------------------------------------------ pieces
__device__ __forceinline__ float top(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// the upper halves of two words, a's below b's
__device__ __forceinline__ uint32_t upper(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302); }

// x = sum of n pieces of 8 bits.  Of three the first is cut off, so that no finite value has an infinite one, and with kNear the second is rounded, so that what it leaves has either sign; otherwise it
// is cut off, too: for a product with a single piece, of which nothing is left out.
template <int n, int count, bool kNear = true>
__device__ __forceinline__ void split(const float (&x)[count], uint32_t (&out)[n][count / 2])
{
#pragma unroll
    for (int i = 0; i < count; i += 2) {
        float a = x[i], b = x[i + 1];
#pragma unroll
        for (int p = 0; p < n; ++p) {
            if (kNear && n == 3 && p == 1) {            // a conversion to bf16 takes longer than the addition: 3 % of 65536 tokens x 8 heads
                const float ra = __uint_as_float(__float_as_uint(a) + 0x8000u), rb = __uint_as_float(__float_as_uint(b) + 0x8000u);
                out[p][i / 2] = upper(ra, rb);
                a -= top(ra);
                b -= top(rb);
                continue;
            }
            out[p][i / 2] = upper(a, b);
            if (p + 1 < n) {
                a -= top(a);
                b -= top(b);
            }
        }
    }
}

__device__ __forceinline__ bf16x8 operand(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

template <int n, bool kNear = true>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&out)[n])
{
    uint32_t w[n][4];
    split<n, 8, kNear>(x, w);
#pragma unroll
    for (int p = 0; p < n; ++p) out[p] = operand((u32x4){w[p][0], w[p][1], w[p][2], w[p][3]});
}

// Two 16-row results of the matrix unit as the right operand of a product that sums over their rows
template <int n, bool kNear = true>
__device__ __forceinline__ void split_rows(const f32x4 &a, const f32x4 &b, bf16x8 (&out)[n])
{
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    split8<n, kNear>(x, out);
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Sum of the products of pieces whose orders add up to less than three, the smallest first, which are rounded least while the sum is small
template <int na, int nb>
__device__ __forceinline__ f32x4 multiply(const bf16x8 (&a)[na], const bf16x8 (&b)[nb], f32x4 c)
{
#pragma unroll
    for (int order = na + nb - 2 < 2 ? na + nb - 2 : 2; order >= 0; --order)
#pragma unroll
        for (int i = 0; i < na; ++i)
            if (order >= i && order - i < nb) c = mfma(a[i], b[order - i], c);
    return c;
}

// The same in two sums side by side, for where what bounds is how long one product waits for the one before
template <int na, int nb>
__device__ __forceinline__ f32x4 multiply_soon(const bf16x8 (&a)[na], const bf16x8 (&b)[nb], f32x4 c)
{
    f32x4 other = {};
    int turn = 0;
#pragma unroll
    for (int order = na + nb - 2 < 2 ? na + nb - 2 : 2; order >= 0; --order)
#pragma unroll
        for (int i = 0; i < na; ++i)
            if (order >= i && order - i < nb) {
                if (turn++ % 2) other = mfma(a[i], b[order - i], other);
                else c = mfma(a[i], b[order - i], c);
            }
    return c + other;
}

// ------------------------------------------------------------------------------ memory
// The same number, of which the compiler does not know that it is: what follows from it is computed where it is needed, in place of being kept in registers (and
// beyond them in memory) all along a loop.
__device__ __forceinline__ uint32_t again(uint32_t x)
{
    asm volatile("" : "+v"(x));
    return x;
}

inline bool wide_rows(const void *p, uint64_t ld, uint32_t D, uint32_t dtype)
{
    return dg_rows::rows_aligned(p, ld, dtype, 16) && D * dg_rows::item_bytes(dtype) % 16 == 0;
}

// kernels of the other files, by the rows' type
// bytes of `weights` and of `chunk_seq`
size_t weight_bytes(uint64_t N, uint32_t n_seq, uint32_t H);
size_t chunk_bytes(uint64_t N, uint32_t n_seq);
void launch_weights(const Delta &d, uint32_t dtype, bool backward, hipStream_t st);
void launch_forward(const Delta &d, uint32_t dtype, hipStream_t st);
void launch_small(const Delta &d, uint32_t dtype, bool back, hipStream_t st);        // heads of up to 32 x 32
void launch_slots(const Delta &d, hipStream_t st);
size_t parts_bytes(uint64_t N, uint32_t n_seq, uint32_t H);
void launch_join(const Delta &d, const float *before, hipStream_t st);        // before: memories before the first parts, or NULL
void launch_tokens(const Delta &d, uint32_t dtype, hipStream_t st);
void launch_backward(const Delta &d, uint32_t dtype, hipStream_t st);
void launch_gradients(const Delta &d, uint32_t dtype, hipStream_t st);

}  // namespace dg_delta
