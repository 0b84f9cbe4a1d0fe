// The gated delta rule: entry points.  Which kernels a call takes, and what it asks of its arguments.
#include <cmath>
#include "delta_common.h"

namespace {

using namespace dg_delta;

// Up to so many tokens a sequence, on average, they are taken one by one.  Heads of 128 x 128, one by one / in chunks, in us: 64 sequences of 16 heads 53 / 98 with 4 tokens each, 127 / 102
// with 16; 4 sequences of 8 heads 14 / 16 with 4, 38 / 15 with 16.
constexpr uint64_t kFewTokens = 4;

// Small heads are taken token by token where those of all sequences fill the chip, or where tokens are few.  Training,
// token by token / in chunks, in us: 768 heads of 16 x 16 270 / 265, 1536 of them 185 / 258; of 16 x 32 1024 223 / 197, 2048 239 / 355; of 32 x 32 2048 847 / 793, 4096 759 / 795.
bool takes_small(uint64_t N, uint32_t n_seq, uint32_t H, uint32_t Dk, uint32_t Dv)
{
    if (Dk > 32 || Dv > 32) return false;
    const uint64_t padded = (Dk <= 16 ? 16 : 32) * (Dv <= 16 ? 16 : 32);
    return (uint64_t)n_seq * H * 2 >= 5 * padded || N <= kFewTokens * n_seq;
}

uint64_t slots_of(uint64_t N, uint32_t n_seq) { return N / kMark + n_seq; }

size_t marks_bytes(uint64_t N, uint32_t n_seq, uint32_t H, uint32_t Dk, uint32_t Dv) { return (size_t)slots_of(N, n_seq) * H * Dk * Dv * sizeof(float); }
size_t rows_bytes(uint64_t N, uint32_t H, uint32_t Dv) { return (size_t)(N * H * Dv * sizeof(float) + 15) / 16 * 16; }
size_t padded(size_t n) { return (n + 15) / 16 * 16; }
size_t slot_bytes(uint64_t N, uint32_t n_seq) { return padded(slots_of(N, n_seq) * 4); }

// The workspace: T and P of the chunks, whose the chunks are, and what parts of sequences leave, for either pass; then what the backward pass hands on.
size_t forward_bytes(uint64_t N, uint32_t n_seq, uint32_t H) { return weight_bytes(N, n_seq, H) + chunk_bytes(N, n_seq) + parts_bytes(N, n_seq, H); }

// The first of these, of which heads that are taken token by token need nothing: it is most of it, 16 KB for 32 tokens of a head, and for 2^20 rays of 64 samples and 2 heads of 16 x 16 96 GiB.
size_t chunks_bytes(uint64_t N, uint32_t n_seq, uint32_t H, uint32_t Dk, uint32_t Dv) { return takes_small(N, n_seq, H, Dk, Dv) ? 0 : forward_bytes(N, n_seq, H); }

void use_workspace(Delta &d, void *ws)
{
    d.weights = (Weights *)ws;
    d.chunk_seq = (const uint32_t *)((char *)ws + weight_bytes(d.N, d.n_seq, d.H));
    d.parts = 1;
    if (const size_t bytes = parts_bytes(d.N, d.n_seq, d.H)) {
        d.ends = (float *)((char *)d.chunk_seq + chunk_bytes(d.N, d.n_seq));
        d.starts = d.ends + bytes / sizeof(float) / 3 * 2;
    }
}

void use_vectors(Delta &d, uint32_t dtype)
{
    d.vec_keys = wide_rows(d.q, d.ldq, d.Dk, dtype) && wide_rows(d.k, d.ldk, d.Dk, dtype);
    d.vec_all = d.vec_keys && wide_rows(d.v, d.ldv, d.Dv, dtype) && (!d.dout || wide_rows(d.dout, d.lddo, d.Dv, dtype));
}

int check_sizes(const char *who, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t Hk, uint32_t H, uint32_t Dk, uint32_t Dv, uint32_t dtype)
{
    DG_REQUIRE(dg_rows::known_type(dtype), DG_ERR_ARG, "%s: unknown element type %u", who, dtype);
    DG_REQUIRE(Hk >= 1 && H >= 1 && H % Hk == 0 && Dk >= 1 && Dv >= 1, DG_ERR_ARG, "%s: heads and their sizes must be positive, and H a multiple of Hk", who);
    DG_REQUIRE(Dk <= kMaxD && Dv <= kMaxD, DG_ERR_UNSUPPORTED, "%s: heads of more than %d values", who, kMaxD);
    // tokens of a sequence are counted in steps of up to 64, in 32 bits
    DG_REQUIRE(N <= (1ull << 32) - kMark && H <= 1u << 16 && n_seq < 1u << 31 && N * H <= 1ull << 36 && (uint64_t)n_seq * H <= 1ull << 32, DG_ERR_UNSUPPORTED,
               "%s: more than 2^32 - 64 rows, 2^31 sequences, 2^16 heads, 2^36 rows of heads or 2^32 memories", who);
    DG_REQUIRE(n_seq >= 1 || N == 0, DG_ERR_ARG, "%s: rows without a sequence", who);
    DG_REQUIRE(first || n_seq == 0 || N % n_seq == 0, DG_ERR_ARG, "%s: %llu rows in %u sequences of one length", who, (unsigned long long)N, n_seq);
    DG_REQUIRE(dg::aligned(first, 4), DG_ERR_ARG, "%s: misaligned offsets", who);
    return DG_OK;
}

int check_rows(const char *who, const char *name, const void *p, uint64_t ld, uint64_t W, uint64_t N, size_t item)
{
    if (N == 0) return DG_OK;
    DG_REQUIRE(p && dg::aligned(p, item), DG_ERR_ARG, "%s: %s: null or misaligned pointer", who, name);
    DG_REQUIRE(ld < 1ull << 24, DG_ERR_UNSUPPORTED, "%s: %s: rows 2^24 values or more apart", who, name);
    DG_REQUIRE(ld >= W, DG_ERR_ARG, "%s: %s: rows of %llu values lie %llu apart", who, name, (unsigned long long)W, (unsigned long long)ld);
    return DG_OK;
}

}  // namespace

extern "C" size_t dg_delta_rule_saved_bytes(uint64_t N, uint32_t n_seq, uint32_t H, uint32_t Dk, uint32_t Dv)
{
    return padded(marks_bytes(N, n_seq, H, Dk, Dv)) + rows_bytes(N, H, Dv);
}

extern "C" size_t dg_delta_rule_fwd_workspace_bytes(uint64_t N, uint32_t n_seq, uint32_t H) { return forward_bytes(N, n_seq, H); }

extern "C" size_t dg_delta_rule_fwd_least_workspace_bytes(uint64_t N, uint32_t n_seq, uint32_t H, uint32_t Dk, uint32_t Dv, uint32_t saves)
{
    return !saves && N <= kFewTokens * n_seq ? 0 : chunks_bytes(N, n_seq, H, Dk, Dv);
}

extern "C" size_t dg_delta_rule_workspace_bytes(uint64_t N, uint32_t n_seq, uint32_t Hk, uint32_t H, uint32_t Dk, uint32_t Dv)
{
    return chunks_bytes(N, n_seq, H, Dk, Dv) + padded(marks_bytes(N, n_seq, H, Dk, Dv)) + rows_bytes(N, H, Dv) + slot_bytes(N, n_seq);
}

extern "C" int dg_delta_rule_fwd(const void *q, uint64_t ldq, const void *k, uint64_t ldk, const void *v, uint64_t ldv, const float *g, uint64_t ldg,
                                 const float *beta, uint64_t ldbeta, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t Hk, uint32_t H, uint32_t Dk,
                                 uint32_t Dv, uint32_t reverse, float scale, uint32_t dtype, const float *s0, void *o, uint64_t ldo, float *s_last, void *saved,
                                 size_t saved_bytes, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "dg_delta_rule_fwd";
    if (int rc = check_sizes(who, N, n_seq, first, Hk, H, Dk, Dv, dtype)) return rc;
    const size_t item = dg_rows::item_bytes(dtype);
    if (int rc = check_rows(who, "q", q, ldq, (uint64_t)Hk * Dk, N, item)) return rc;
    if (int rc = check_rows(who, "k", k, ldk, (uint64_t)Hk * Dk, N, item)) return rc;
    if (int rc = check_rows(who, "v", v, ldv, (uint64_t)H * Dv, N, item)) return rc;
    if (int rc = check_rows(who, "o", o, ldo, (uint64_t)H * Dv, N, item)) return rc;
    if (int rc = check_rows(who, "g", g, ldg, H, N, 4)) return rc;
    if (int rc = check_rows(who, "beta", beta, ldbeta, H, N, 4)) return rc;
    DG_REQUIRE(std::isfinite(scale), DG_ERR_ARG, "%s: scale is not finite", who);
    DG_REQUIRE(dg::aligned(s0, 4) && dg::aligned(s_last, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (n_seq == 0) return DG_OK;
    const size_t need = saved ? dg_delta_rule_saved_bytes(N, n_seq, H, Dk, Dv) : 0;
    DG_REQUIRE(!saved || (dg::aligned(saved, 16) && saved_bytes >= need), DG_ERR_WORKSPACE, "%s: %zu bytes needed for the backward pass, %zu given", who, need, saved_bytes);
    Delta d = {};
    d.q = q, d.k = k, d.v = v, d.g = g, d.beta = beta, d.ldq = ldq, d.ldk = ldk, d.ldv = ldv, d.ldg = ldg, d.ldb = ldbeta, d.s0 = s0, d.o = o, d.ldo = ldo, d.s_last = s_last;
    d.first = first, d.N = N, d.n_seq = n_seq, d.Hk = Hk, d.H = H, d.Dk = Dk, d.Dv = Dv, d.reverse = reverse, d.scale = scale;
    if (saved) d.marks = (float *)saved, d.y = (float *)((char *)saved + padded(marks_bytes(N, n_seq, H, Dk, Dv)));
    use_vectors(d, dtype);
    if (takes_small(N, n_seq, H, Dk, Dv)) launch_small(d, dtype, false, (hipStream_t)stream);
    else if (!saved && N <= kFewTokens * n_seq) launch_tokens(d, dtype, (hipStream_t)stream);
    else {
        const size_t bytes = forward_bytes(N, n_seq, H);
        DG_REQUIRE(ws && dg::aligned(ws, 16) && ws_bytes >= bytes, DG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, bytes, ws ? ws_bytes : 0);
        use_workspace(d, ws);
        if (N) launch_weights(d, dtype, false, (hipStream_t)stream);
        launch_forward(d, dtype, (hipStream_t)stream);
    }
    return dg::launch_status(who);
}

extern "C" int dg_delta_rule_bwd(const void *q, uint64_t ldq, const void *k, uint64_t ldk, const void *v, uint64_t ldv, const float *g, uint64_t ldg,
                                 const float *beta, uint64_t ldbeta, uint64_t N, uint32_t n_seq, const uint32_t *first, uint32_t Hk, uint32_t H, uint32_t Dk,
                                 uint32_t Dv, uint32_t reverse, float scale, uint32_t dtype, const void *saved, size_t saved_bytes, const void *do_, uint64_t lddo,
                                 const float *ds_last, void *dq, uint64_t lddq, void *dk, uint64_t lddk, void *dv, uint64_t lddv, float *dg, uint64_t lddg,
                                 float *dbeta, uint64_t lddbeta, float *ds0, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "dg_delta_rule_bwd";
    if (int rc = check_sizes(who, N, n_seq, first, Hk, H, Dk, Dv, dtype)) return rc;
    const size_t item = dg_rows::item_bytes(dtype);
    const uint64_t wk = (uint64_t)Hk * Dk, wv = (uint64_t)H * Dv;
    const struct { const char *name; const void *p; uint64_t ld, W; size_t item; } rows[] = {
        {"q", q, ldq, wk, item}, {"k", k, ldk, wk, item}, {"v", v, ldv, wv, item}, {"g", g, ldg, H, 4}, {"beta", beta, ldbeta, H, 4}, {"do_", do_, lddo, wv, item},
        {"dq", dq, lddq, wk, item}, {"dk", dk, lddk, wk, item}, {"dv", dv, lddv, wv, item}, {"dg", dg, lddg, H, 4}, {"dbeta", dbeta, lddbeta, H, 4}};
    for (const auto &r : rows)
        if (int rc = check_rows(who, r.name, r.p, r.ld, r.W, N, r.item)) return rc;
    DG_REQUIRE(std::isfinite(scale), DG_ERR_ARG, "%s: scale is not finite", who);
    DG_REQUIRE(dg::aligned(ds_last, 4) && dg::aligned(ds0, 4), DG_ERR_ARG, "%s: misaligned pointer", who);
    if (n_seq == 0) return DG_OK;
    const size_t held = dg_delta_rule_saved_bytes(N, n_seq, H, Dk, Dv), need = dg_delta_rule_workspace_bytes(N, n_seq, Hk, H, Dk, Dv);
    DG_REQUIRE(saved && dg::aligned(saved, 16) && saved_bytes >= held, DG_ERR_WORKSPACE, "%s: the forward pass leaves %zu bytes, %zu given", who, held, saved ? saved_bytes : 0);
    DG_REQUIRE(ws && dg::aligned(ws, 16) && ws_bytes >= need, DG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws ? ws_bytes : 0);
    const size_t marks = padded(marks_bytes(N, n_seq, H, Dk, Dv));
    Delta d = {};
    d.q = q, d.k = k, d.v = v, d.g = g, d.beta = beta, d.ldq = ldq, d.ldk = ldk, d.ldv = ldv, d.ldg = ldg, d.ldb = ldbeta, d.ds_last = ds_last, d.ds0 = ds0;
    d.dout = do_, d.lddo = lddo, d.dq = dq, d.dk = dk, d.dv = dv, d.lddq = lddq, d.lddk = lddk, d.lddv = lddv, d.dg = dg, d.dbeta = dbeta, d.lddg = lddg, d.lddb = lddbeta;
    d.first = first, d.N = N, d.n_seq = n_seq, d.Hk = Hk, d.H = H, d.Dk = Dk, d.Dv = Dv, d.reverse = reverse, d.scale = scale, d.slots = (uint32_t)slots_of(N, n_seq);
    d.marks = (float *)const_cast<void *>(saved), d.y = (float *)((char *)const_cast<void *>(saved) + marks);
    const bool small = takes_small(N, n_seq, H, Dk, Dv);
    if (!small) use_workspace(d, ws);
    char *const rest = (char *)ws + chunks_bytes(N, n_seq, H, Dk, Dv);
    d.dmarks = (float *)rest, d.dr = (float *)(rest + marks), d.slot_seq = (const uint32_t *)(rest + marks + rows_bytes(N, H, Dv));
    use_vectors(d, dtype);
    d.vec_out = wide_rows(dv, lddv, Dv, dtype) && wide_rows(dq, lddq, Dk, dtype) && wide_rows(dk, lddk, Dk, dtype);
    if (N) launch_slots(d, (hipStream_t)stream);
    if (small) launch_small(d, dtype, true, (hipStream_t)stream);
    else {
        if (N) launch_weights(d, dtype, true, (hipStream_t)stream);
        launch_backward(d, dtype, (hipStream_t)stream);
        if (N) launch_gradients(d, dtype, (hipStream_t)stream);
    }
    return dg::launch_status(who);
}
