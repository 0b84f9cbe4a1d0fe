// Gated linear recurrence along sequences of rows, channel by channel:
//   a = 1 / (1 + e^-z),  c = 1 - a = 1 / (1 + e^z),  h_t = a_t h_{t-1} + c_t u_t,  y_t = h_t.
// Its backward pass: G_t = dy_t + a_{t+1} G_{t+1} from the last token back, du = c G, dz = a c G (h_{t-1} - u_t), dh0 = a_0 G_0.
// From |z| = 88 on a and c are exactly 0 and 1: what a gate of 0 multiplies is not looked at, be it infinite or NaN.
//
// Tokens have a place in the order in which they are gone through: their row, or N - 1 - row back to front.  The forward pass
// keeps the state before every kKeep-th place in fp32; the backward pass computes the states between them again.
#include "rows_common.h"

namespace {

using namespace dg_rows;

constexpr int kBlock = 256, kKeep = 16;
constexpr float kShut = 88.0f;      // e^-88 is the smallest power that is a normal fp32 number, about

struct Gate { float a, c; };

// both sides of the gate to full relative precision: the larger one is s = 1 / (1 + e^-|z|), the smaller one e^-|z| s
__device__ __forceinline__ Gate gate(float z)
{
    const float e = __expf(-fabsf(z)), s = __builtin_amdgcn_rcpf(1.0f + e), t = e * s;
    return z >= 0.0f ? Gate{s, t} : Gate{t, s};
}

// h_t of h_{t-1}
__device__ __forceinline__ float advance(float z, float u, float h)
{
    const Gate g = gate(z);
    return (z <= -kShut ? 0.0f : g.a * h) + (z >= kShut ? 0.0f : g.c * u);
}

struct Shape {
    uint64_t N;
    uint32_t n_seq, W, S;           // S: tokens of each sequence, where first is NULL
    const uint32_t *first;
    bool reverse;
};

// places [begin, end) of a sequence; never outside [0, N), whatever `first` holds
__device__ __forceinline__ void places(const Shape &d, uint32_t seq, uint64_t &begin, uint64_t &end)
{
    uint64_t b = (uint64_t)seq * d.S, e = b + d.S;
    if (d.first) {
        b = d.first[seq];
        e = d.first[seq + 1];
        e = e < d.N ? e : d.N;
        b = b < e ? b : e;
    }
    begin = d.reverse ? d.N - e : b;
    end = d.reverse ? d.N - b : e;
}

__device__ __forceinline__ uint64_t row_of(const Shape &d, uint64_t place) { return d.reverse ? d.N - 1 - place : place; }

template <class T>
__global__ void __launch_bounds__(kBlock)
recurrence_fwd_kernel(Shape d, const T *z, uint64_t ldz, const T *u, uint64_t ldu, const float *h0, T *y, uint64_t ldy, float *h_last, float *states)
{
    const uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= (uint64_t)d.n_seq * d.W) return;
    const uint32_t seq = (uint32_t)(i / d.W), c = (uint32_t)(i % d.W);
    uint64_t begin, end;
    places(d, seq, begin, end);
    float h = h0 ? h0[i] : 0.0f;
    for (uint64_t p = begin; p < end; ++p) {
        const uint64_t row = row_of(d, p);
        if (states && p % kKeep == 0) states[p / kKeep * d.W + c] = h;
        h = advance((float)z[row * ldz + c], (float)u[row * ldu + c], h);
        y[row * ldy + c] = (T)h;
    }
    if (h_last) h_last[i] = h;
}

template <class T>
__global__ void __launch_bounds__(kBlock)
recurrence_bwd_kernel(Shape d, const T *z, uint64_t ldz, const T *u, uint64_t ldu, const float *h0, const float *states, const T *dy, uint64_t lddy,
                      const float *dh_last, T *dz, uint64_t lddz, T *du, uint64_t lddu, float *dh0)
{
    const uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= (uint64_t)d.n_seq * d.W) return;
    const uint32_t seq = (uint32_t)(i / d.W), c = (uint32_t)(i % d.W);
    uint64_t begin, end;
    places(d, seq, begin, end);
    float G = dh_last ? dh_last[i] : 0.0f;
    while (end > begin) {
        const uint64_t keep = (end - 1) / kKeep, p0 = keep * kKeep > begin ? keep * kKeep : begin;
        const int n = (int)(end - p0);
        float before[kKeep], h = p0 == begin ? (h0 ? h0[i] : 0.0f) : states[keep * d.W + c];
#pragma unroll
        for (int k = 0; k < kKeep; ++k)
            if (k < n) {
                const uint64_t row = row_of(d, p0 + k);
                before[k] = h;
                h = advance((float)z[row * ldz + c], (float)u[row * ldu + c], h);
            }
#pragma unroll
        for (int k = kKeep - 1; k >= 0; --k)
            if (k < n) {
                const uint64_t row = row_of(d, p0 + k);
                const float zz = (float)z[row * ldz + c], uu = (float)u[row * ldu + c];
                const Gate g = gate(zz);
                const bool shut = fabsf(zz) >= kShut;
                G += (float)dy[row * lddy + c];
                dz[row * lddz + c] = (T)(shut ? 0.0f : g.a * g.c * (before[k] - uu) * G);
                du[row * lddu + c] = (T)(zz >= kShut ? 0.0f : g.c * G);
                G = zz <= -kShut ? 0.0f : g.a * G;
            }
        end = p0;
    }
    if (dh0) dh0[i] = G;
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

template <class T>
void launch_fwd(const Shape &d, const void *z, uint64_t ldz, const void *u, uint64_t ldu, const float *h0, void *y, uint64_t ldy, float *h_last,
                float *states, hipStream_t st)
{
    const uint32_t grid = (uint32_t)(((uint64_t)d.n_seq * d.W + kBlock - 1) / kBlock);
    recurrence_fwd_kernel<T><<<grid, kBlock, 0, st>>>(d, (const T *)z, ldz, (const T *)u, ldu, h0, (T *)y, ldy, h_last, states);
}

template <class T>
void launch_bwd(const Shape &d, const void *z, uint64_t ldz, const void *u, uint64_t ldu, const float *h0, const float *states, const void *dy, uint64_t lddy,
                const float *dh_last, void *dz, uint64_t lddz, void *du, uint64_t lddu, float *dh0, hipStream_t st)
{
    const uint32_t grid = (uint32_t)(((uint64_t)d.n_seq * d.W + kBlock - 1) / kBlock);
    recurrence_bwd_kernel<T><<<grid, kBlock, 0, st>>>(d, (const T *)z, ldz, (const T *)u, ldu, h0, states, (const T *)dy, lddy, dh_last, (T *)dz, lddz,
                                                      (T *)du, lddu, dh0);
}

}  // namespace

extern "C" size_t dg_recurrence_state_count(uint64_t N, uint32_t W) { return (size_t)((N + kKeep - 1) / kKeep) * W; }

extern "C" size_t dg_recurrence_workspace_bytes(uint64_t N, uint32_t n_seq, uint32_t W)
{
    (void)N, (void)n_seq, (void)W;
    return 0;
}

extern "C" int dg_recurrence_fwd(const void *z, uint64_t ldz, const void *u, uint64_t ldu, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t W,
                                 uint32_t reverse, uint32_t dtype, const float *h0, void *y, uint64_t ldy, float *h_last, float *states, void *ws,
                                 size_t ws_bytes, void *stream)
{
    const char *who = "dg_recurrence_fwd";
    Shape d = {N, n_seq, W, 0, first, reverse != 0};
    if (int rc = check(who, d, dtype)) return rc;
    if (int rc = check_rows(who, z, ldz, d, dtype)) return rc;
    if (int rc = check_rows(who, u, ldu, d, dtype)) return rc;
    if (int rc = check_rows(who, y, ldy, d, dtype)) return rc;
    DG_REQUIRE(dg::aligned(h0, 4) && dg::aligned(h_last, 4) && dg::aligned(states, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (n_seq == 0) return DG_OK;
    (void)ws, (void)ws_bytes;
    (dtype == DG_F32 ? launch_fwd<float> : dtype == DG_F16 ? launch_fwd<f16> : launch_fwd<bf16>)(d, z, ldz, u, ldu, h0, y, ldy, h_last, states,
                                                                                                 (hipStream_t)stream);
    return dg::launch_status(who);
}

extern "C" int dg_recurrence_bwd(const void *z, uint64_t ldz, const void *u, uint64_t ldu, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t W,
                                 uint32_t reverse, uint32_t dtype, const float *h0, const float *states, const void *dy, uint64_t lddy,
                                 const float *dh_last, void *dz, uint64_t lddz, void *du, uint64_t lddu, float *dh0, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "dg_recurrence_bwd";
    Shape d = {N, n_seq, W, 0, first, reverse != 0};
    if (int rc = check(who, d, dtype)) return rc;
    const struct { const void *p; uint64_t ld; } rows[] = {{z, ldz}, {u, ldu}, {dy, lddy}, {dz, lddz}, {du, lddu}};
    for (const auto &r : rows)
        if (int rc = check_rows(who, r.p, r.ld, d, dtype)) return rc;
    DG_REQUIRE(N == 0 || states, DG_ERR_ARG, "%s: the states that the forward pass kept are missing", who);
    DG_REQUIRE(dg::aligned(h0, 4) && dg::aligned(states, 4) && dg::aligned(dh_last, 4) && dg::aligned(dh0, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (n_seq == 0) return DG_OK;
    (void)ws, (void)ws_bytes;
    (dtype == DG_F32 ? launch_bwd<float> : dtype == DG_F16 ? launch_bwd<f16> : launch_bwd<bf16>)(d, z, ldz, u, ldu, h0, states, dy, lddy, dh_last, dz, lddz, du,
                                                                                                 lddu, dh0, (hipStream_t)stream);
    return dg::launch_status(who);
}
