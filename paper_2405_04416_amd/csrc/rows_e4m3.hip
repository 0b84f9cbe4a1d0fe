// Rows in 8-bit floating point (e4m3: 4 bits of exponent, 3 of mantissa, largest value 448, NaN but no infinity), each block of 128 columns with a scale that
// is a power of two; of the rows themselves (weights) or of their root-mean-square norm, after the residual's addition (what goes into a product).
// Values are rounded once, to the nearest even one: rows from their own type, the norm from what is known to 2^-40 (rms_norm_common.h).
//
// Bound by memory: one pass, rows in registers; the lanes that hold a block of columns find its largest value among themselves.  5003 rows of 1000 fp32 values 6.5 us
// (3.9 TB/s, from the caches), the norm of 16384 rows of 2048 49 us (4.8 TB/s).
#include "rms_norm_common.h"

namespace {

using namespace dg_rms;

template <bool kResidual, Made kMade>
struct To8 {
    template <class T, int V, int G, int K, bool kStreamed, bool kLoose>
    static void launch(const Call &c, uint32_t grid)
    {
        rms_fwd_kernel<T, V, G, K, kBlock, kStreamed, kLoose, kResidual, kMade><<<grid, kBlock, 0, c.st>>>(c.a);
    }
    template <class T>
    static void launch_wide(const Call &c)
    {
        rms_fwd_wide_kernel<T, kMade><<<(uint32_t)(c.a.N < kMostWide ? c.a.N : kMostWide), kWide, 0, c.st>>>(c.a);
    }
};

int check8(const char *who, const Rms &a)
{
    DG_REQUIRE(a.out && dg::aligned(a.out, 16) && a.ldo % 16 == 0, DG_ERR_ARG, "%s: rows in 8 bits have to begin at multiples of 16 bytes", who);
    DG_REQUIRE(a.ldo >= a.W && a.ldo <= 1ull << 40, DG_ERR_ARG, "%s: rows of %u values lie %llu apart", who, a.W, (unsigned long long)a.ldo);
    const uint32_t blocks = (a.W + kScaled - 1) / kScaled;
    DG_REQUIRE(a.scales && a.lds >= blocks && a.lds <= 1ull << 40, DG_ERR_ARG, "%s: null scales, or rows of %u scales %llu apart", who, blocks, (unsigned long long)a.lds);
    return DG_OK;
}

}  // namespace

extern "C" int dg_rms_norm_e4m3_fwd(const void *x, uint64_t ldx, const void *residual, uint64_t ldr, const float *gamma, uint64_t N, uint32_t W, float eps,
                                    uint32_t dtype, void *total, uint64_t ldt, void *q, uint64_t ldq, uint8_t *scales, uint64_t lds, void *stream)
{
    const char *who = "dg_rms_norm_e4m3_fwd";
    if (int rc = check_norm(who, N, W, eps, dtype)) return rc;
    if (N == 0) return DG_OK;
    Rms a = {};
    a.x = x, a.r = residual, a.t = total, a.out = q, a.scales = scales, a.gamma = gamma;
    a.ldx = ldx, a.ldr = ldr, a.ldt = ldt, a.ldo = ldq, a.lds = lds, a.N = N, a.W = W, a.eps = eps;
    if (int rc = check_forward(who, a, dtype)) return rc;
    if (int rc = check8(who, a)) return rc;
    const bool aligned = may_align(x, ldx, dtype) && may_align(residual, ldr, dtype) && may_align(total, ldt, dtype);
    const Call c = {a, dtype, 0, (hipStream_t)stream};
    residual ? launch<To8<true, kNormed8>>(c, aligned) : launch<To8<false, kNormed8>>(c, aligned);
    return dg::launch_status(who);
}

extern "C" int dg_e4m3_rows(const void *x, uint64_t ldx, uint64_t N, uint32_t W, uint32_t dtype, void *q, uint64_t ldq, uint8_t *scales, uint64_t lds,
                            void *stream)
{
    const char *who = "dg_e4m3_rows";
    if (int rc = check_norm(who, N, W, 0.0f, dtype)) return rc;
    if (N == 0) return DG_OK;
    Rms a = {};
    a.x = x, a.out = q, a.scales = scales, a.ldx = ldx, a.ldo = ldq, a.lds = lds, a.N = N, a.W = W;
    if (int rc = check_forward(who, a, dtype)) return rc;
    if (int rc = check8(who, a)) return rc;
    const Call c = {a, dtype, 0, (hipStream_t)stream};
    launch<To8<false, kPlain8>>(c, may_align(x, ldx, dtype));
    return dg::launch_status(who);
}
