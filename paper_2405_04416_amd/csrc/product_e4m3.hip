// Matrix product of rows in 8-bit floating point with a power-of-two scale for each block of 128 columns:
//   y[m, n] = sum over k of a[m, k] 2^(sa[m, k / 128] - 127) b[n, k] 2^(sb[n, k / 128] - 127),   rounded once to 16 bits.
// The matrix instruction takes the exponents with its operands, so that nothing is scaled by hand and the sums stay in its accumulators (fp32).
//
// Three ways, by what bounds them.  Few rows: the bytes of b, which go from memory to the matrix instruction's registers with no stop in LDS.  Many:
// the matrix instruction; tiles are staged through LDS by loads that write there, the next block of columns while one is multiplied.  In between, with
// too few tiles for the chip, the columns are split over workgroups, whose sums a second launch adds in order.
#include <type_traits>
#include "rows_common.h"

namespace {

using dg_rows::bf16;
using dg_rows::f16;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kBlockK = 128;       // columns to a scale, and to a step

struct Side {
    const uint8_t *q, *scales;
    uint64_t ld, lds;
    uint32_t rows;
};

struct Product {
    Side a, b;
    void *y;
    float *part;                        // [splits][M][N], or NULL
    uint64_t ldy;
    uint32_t K, blocks, splits;
    uint32_t tiles_m, tiles_n;
};

// 16 values of a row from column c on, 0 from K on; where the row ends within them they are fetched one by one, so that nothing behind it is read
__device__ __forceinline__ u32x4 sixteen(const uint8_t *row, uint32_t c, uint32_t K)
{
    if (c + 16 <= K) return *reinterpret_cast<const u32x4 *>(row + c);
    u32x4 v = {0, 0, 0, 0};
    for (uint32_t i = 0; c + i < K && i < 16; ++i) v[i / 4] |= (uint32_t)row[c + i] << (8 * (i % 4));
    return v;
}

__device__ __forceinline__ i32x8 both(u32x4 lo, u32x4 hi)
{
    return (i32x8){(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// ------------------------------------------------------------------------------ few rows
constexpr int kFewWaves = 8;

// A workgroup has 16 rows of b and all of a's (up to 16 MT); its wavefronts share the columns, block by block, and their sums meet in LDS.
template <class T, int MT>
__global__ void __launch_bounds__(kFewWaves * 64)
few_rows_kernel(Product p)
{
    __shared__ float sums[kFewWaves][MT][4][64];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n0 = blockIdx.x * 16, part = lane / 16 * 32;
    const uint32_t n = n0 + lane % 16 < p.b.rows ? n0 + lane % 16 : p.b.rows - 1;
    const uint8_t *b = p.b.q + n * p.b.ld, *sb = p.b.scales + n * p.b.lds;
    const uint8_t *a[MT], *sa[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const uint32_t m = t * 16 + lane % 16 < p.a.rows ? t * 16 + lane % 16 : p.a.rows - 1;
        a[t] = p.a.q + m * p.a.ld;
        sa[t] = p.a.scales + m * p.a.lds;
    }
    f32x4 acc[MT] = {};
    const uint32_t full = p.K / kBlockK;
    // kAtOnce blocks are on their way before the first is multiplied
    auto blocks = [&](uint32_t kb, auto count) {
        constexpr int n = decltype(count)::value;
        i32x8 vb[n], va[n][MT];
        int eb[n], ea[n][MT];
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const uint32_t at = kb + i * kFewWaves, c = at * kBlockK + part;
            const u32x4 *from = reinterpret_cast<const u32x4 *>(b + c);
            vb[i] = both(from[0], from[1]);
            eb[i] = sb[at];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                from = reinterpret_cast<const u32x4 *>(a[t] + c);
                va[i][t] = both(from[0], from[1]);
                ea[i][t] = sa[t][at];
            }
        }
#pragma unroll
        for (int i = 0; i < n; ++i)
#pragma unroll
            for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vb[i], va[i][t], acc[t], 0, 0, 0, eb[i], 0, ea[i][t]);
    };
    constexpr int kAtOnce = 4 / MT > 1 ? 4 / MT : 1;
    uint32_t kb = wave;
    for (; kb + (kAtOnce - 1) * kFewWaves < full; kb += kAtOnce * kFewWaves) blocks(kb, std::integral_constant<int, kAtOnce>());
    if (kAtOnce > 1)
        for (; kb < full; kb += kFewWaves) blocks(kb, std::integral_constant<int, 1>());
    if (full < p.blocks && wave == full % kFewWaves) {
        const uint32_t c = full * kBlockK + part;
        const i32x8 vb = both(sixteen(b, c, p.K), sixteen(b, c + 16, p.K));
#pragma unroll
        for (int t = 0; t < MT; ++t)
            acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vb, both(sixteen(a[t], c, p.K), sixteen(a[t], c + 16, p.K)), acc[t], 0, 0, 0,
                                                                      (int)sb[full], 0, (int)sa[t][full]);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][t][i][lane] = acc[t][i];
    __syncthreads();
    // element (n, m) of tile t lies with lane m + 16 (n / 4), register n % 4
    for (uint32_t e = threadIdx.x; e < MT * 256; e += kFewWaves * 64) {
        const uint32_t t = e / 256, m = e / 16 % 16, j = e % 16;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) sum += sums[w][t][j % 4][m + 16 * (j / 4)];
        if (t * 16 + m < p.a.rows && n0 + j < p.b.rows) ((T *)p.y)[(t * 16 + m) * p.ldy + n0 + j] = (T)sum;
    }
}

// ------------------------------------------------------------------------------ tiles
// A workgroup of four wavefronts has a square tile, a wavefront a quarter of it: WT x WT products of 32 x 32.  In LDS a row of 128 bytes lies in
// eight pieces of 16, piece c of row r at place c ^ key(r): the 16 lanes that read together then meet all banks once.
__device__ __forceinline__ uint32_t key(uint32_t r) { return (r & 7) ^ (r >> 3 & 1); }

template <int WT>
struct Tile {
    static constexpr uint32_t kRows = 64 * WT;
    static constexpr uint32_t kBytes = kRows * kBlockK;
};

// One block of columns of a side's rows into LDS.  Loads that write to LDS put lane i's 16 bytes at place i, so lanes choose what they fetch.
template <int WT>
__device__ __forceinline__ void stage(const Side &s, uint32_t row0, uint32_t kb, uint32_t K, uint8_t *to)
{
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const bool whole = (kb + 1) * kBlockK <= K;
#pragma unroll
    for (int i = 0; i < 2 * WT; ++i) {
        const uint32_t first = (i * 4 + wave) * 8, r = first + lane / 8, c = kb * kBlockK + ((lane % 8) ^ key(r)) * 16;
        const uint8_t *row = s.q + (uint64_t)(row0 + r < s.rows ? row0 + r : s.rows - 1) * s.ld;
        if (whole)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(row + c), (__attribute__((address_space(3))) uint32_t *)(to + first * kBlockK), 16, 0,
                                             0);
        else *reinterpret_cast<u32x4 *>(to + first * kBlockK + lane * 16) = sixteen(row, c, K);
    }
}

// Four blocks' exponents of a row, as many as there are
__device__ __forceinline__ int exponents(const uint8_t *scales, uint32_t kb, uint32_t blocks)
{
    typedef uint32_t loose_u32 __attribute__((aligned(1)));
    if (kb + 4 <= blocks) return (int)*reinterpret_cast<const loose_u32 *>(scales + kb);
    uint32_t e = 0;
    for (uint32_t i = 0; kb + i < blocks && i < 4; ++i) e |= (uint32_t)scales[kb + i] << (8 * i);
    return (int)e;
}

template <int WT, int kByte>
__device__ __forceinline__ void multiply(const uint8_t *la, const uint8_t *lb, uint32_t lane, const int (&ea)[WT], const int (&eb)[WT], f32x16 (&acc)[WT][WT])
{
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        i32x8 a[WT], b[WT];
        const uint32_t c = 4 * s + lane / 32 * 2, k = key(lane % 32);
#pragma unroll
        for (int t = 0; t < WT; ++t) {
            const uint8_t *row = la + (t * 32 + lane % 32) * kBlockK;
            a[t] = both(*reinterpret_cast<const u32x4 *>(row + (c ^ k) * 16), *reinterpret_cast<const u32x4 *>(row + ((c + 1) ^ k) * 16));
            row = lb + (t * 32 + lane % 32) * kBlockK;
            b[t] = both(*reinterpret_cast<const u32x4 *>(row + (c ^ k) * 16), *reinterpret_cast<const u32x4 *>(row + ((c + 1) ^ k) * 16));
        }
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
            for (int j = 0; j < WT; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[j], a[i], acc[i][j], 0, 0, kByte, eb[j], kByte, ea[i]);
    }
}

__device__ __forceinline__ void loads_done()
{
    __builtin_amdgcn_s_waitcnt(0x0f70);         // all loads, those that write to LDS among them
    __syncthreads();
}

__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <class T, int WT>
__global__ void __launch_bounds__(256)
tile_kernel(Product p)
{
    constexpr uint32_t kRows = Tile<WT>::kRows, kBytes = Tile<WT>::kBytes, kHalf = kRows / 2;
    __shared__ alignas(16) uint8_t lds[2][2][kBytes];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, tiles = p.tiles_m * p.tiles_n;
    // Workgroups go to the eight chiplets in turn: each gets a run of neighbouring tiles, in columns of eight, so that its cache serves them
    uint32_t id = blockIdx.x;
    const uint32_t all = tiles * p.splits, per = all / 8, more = all % 8, chiplet = id % 8;
    id = chiplet * per + (chiplet < more ? chiplet : more) + id / 8;
    const uint32_t split = id / tiles;
    id %= tiles;
    const uint32_t column = id / (8 * p.tiles_n), high = p.tiles_m - column * 8 < 8 ? p.tiles_m - column * 8 : 8, within = id % (8 * p.tiles_n);
    const uint32_t m0 = (column * 8 + within % high) * kRows, n0 = within / high * kRows;
    const uint32_t begin = (uint64_t)p.blocks * split / p.splits, end = (uint64_t)p.blocks * (split + 1) / p.splits;
    const uint32_t wm = wave / 2 * kHalf, wn = wave % 2 * kHalf;
    const uint8_t *sa[WT], *sb[WT];
#pragma unroll
    for (int t = 0; t < WT; ++t) {
        const uint32_t m = m0 + wm + t * 32 + lane % 32, n = n0 + wn + t * 32 + lane % 32;
        sa[t] = p.a.scales + (uint64_t)(m < p.a.rows ? m : p.a.rows - 1) * p.a.lds;
        sb[t] = p.b.scales + (uint64_t)(n < p.b.rows ? n : p.b.rows - 1) * p.b.lds;
    }
    f32x16 acc[WT][WT] = {};
    int ea[WT], eb[WT], next_a[WT], next_b[WT];
#pragma unroll
    for (int t = 0; t < WT; ++t) {
        next_a[t] = exponents(sa[t], begin, end);
        next_b[t] = exponents(sb[t], begin, end);
    }
    if (begin < end) {
        stage<WT>(p.a, m0, begin, p.K, lds[0][0]);
        stage<WT>(p.b, n0, begin, p.K, lds[0][1]);
    }
    for (uint32_t kb0 = begin; kb0 < end; kb0 += 4) {
#pragma unroll
        for (int t = 0; t < WT; ++t) {
            ea[t] = next_a[t];
            eb[t] = next_b[t];
        }
        auto step = [&](auto byte) {
            constexpr int i = decltype(byte)::value;
            const uint32_t kb = kb0 + i;
            if (kb >= end) return;
            loads_done();                       // this block has come, and the other half of LDS has been read by all
            if (kb + 1 < end) {
                stage<WT>(p.a, m0, kb + 1, p.K, lds[(i + 1) % 2][0]);
                stage<WT>(p.b, n0, kb + 1, p.K, lds[(i + 1) % 2][1]);
            }
            if (i == 0 && kb + 4 < end)
#pragma unroll
                for (int t = 0; t < WT; ++t) {
                    next_a[t] = exponents(sa[t], kb + 4, end);
                    next_b[t] = exponents(sb[t], kb + 4, end);
                }
            multiply<WT, i>(lds[i % 2][0] + wm * kBlockK, lds[i % 2][1] + wn * kBlockK, lane, ea, eb, acc);
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
    }
    // Lane l has row l % 32 of a, and of b rows 8 g + 4 (l / 32) to 3 on, g = 0 to 3
    if (p.part) {
        float *part = p.part + (uint64_t)split * p.a.rows * p.b.rows;
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
            for (int j = 0; j < WT; ++j)
#pragma unroll
                for (int g = 0; g < 16; ++g) {
                    const uint32_t m = m0 + wm + i * 32 + lane % 32, n = n0 + wn + j * 32 + g / 4 * 8 + lane / 32 * 4 + g % 4;
                    if (m < p.a.rows && n < p.b.rows) part[(uint64_t)m * p.b.rows + n] = acc[i][j][g];
                }
        return;
    }
    // 32 rows at a time through LDS, so that a row's stores lie next to each other
    constexpr uint32_t kStride = WT * 32 + 8;
    __syncthreads();
    T *mine = reinterpret_cast<T *>(&lds[0][0][0]) + wave * 32 * kStride;
    static_assert(4 * 32 * kStride * sizeof(T) <= sizeof(lds), "room for the results");
    const bool vectors = p.b.rows % 8 == 0 && p.ldy % 8 == 0 && reinterpret_cast<uintptr_t>(p.y) % 16 == 0;
#pragma unroll
    for (int i = 0; i < WT; ++i) {
        wave_fence();
#pragma unroll
        for (int j = 0; j < WT; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float v[4] = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                dg_rows::store<T, 4>(mine + lane % 32 * kStride + j * 32 + g * 8 + lane / 32 * 4, v);
            }
        wave_fence();
        constexpr uint32_t kVectors = WT * 4;       // of a row
#pragma unroll
        for (uint32_t e = 0; e < 32 * kVectors; e += 64) {
            const uint32_t r = (e + lane) / kVectors, c = (e + lane) % kVectors * 8, m = m0 + wm + i * 32 + r, n = n0 + wn + c;
            if (m >= p.a.rows || n >= p.b.rows) continue;
            const dg_rows::Pack<T, 8> v = *reinterpret_cast<const dg_rows::Pack<T, 8> *>(mine + r * kStride + c);
            T *to = (T *)p.y + m * p.ldy + n;
            if (vectors) *reinterpret_cast<dg_rows::Pack<T, 8> *>(to) = v;
            else
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (n + x < p.b.rows) to[x] = v.v[x];
        }
    }
}

template <class T>
__global__ void __launch_bounds__(256)
join_kernel(Product p)
{
    const uint64_t all = (uint64_t)p.a.rows * p.b.rows;
    for (uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (uint64_t)gridDim.x * 256) {
        float sum = 0.0f;
        for (uint32_t s = 0; s < p.splits; ++s) sum += p.part[s * all + e];
        ((T *)p.y)[e / p.b.rows * p.ldy + e % p.b.rows] = (T)sum;
    }
}

// ------------------------------------------------------------------------------ launch
constexpr uint32_t kFew = 64;           // rows of a up to which b's bytes are what counts

struct Plan { uint32_t tile, tiles_m, tiles_n, splits; };      // tile 0: few rows

// The largest tiles of which there is one for each compute unit; with too few of the smallest, the columns are split.
Plan plan_of(uint32_t M, uint32_t N, uint32_t K)
{
    const uint32_t blocks = (K + kBlockK - 1) / kBlockK;
    if (M <= kFew) return {0, 0, 0, 1};
    uint32_t tile = 256;
    while (tile > 64 && (uint64_t)((M + tile - 1) / tile) * ((N + tile - 1) / tile) < 256) tile /= 2;
    const uint32_t tm = (M + tile - 1) / tile, tn = (N + tile - 1) / tile;
    uint32_t splits = 1;
    while (tile == 64 && (uint64_t)tm * tn * splits * 2 <= 512 && blocks / (splits * 2) >= 4) splits *= 2;
    return {tile, tm, tn, splits};
}

template <class T>
void launch(const Product &p, const Plan &plan, hipStream_t st)
{
    if (plan.tile == 0) {
        const uint32_t grid = (p.b.rows + 15) / 16, mt = (p.a.rows + 15) / 16;
        if (mt == 1) few_rows_kernel<T, 1><<<grid, kFewWaves * 64, 0, st>>>(p);
        else if (mt == 2) few_rows_kernel<T, 2><<<grid, kFewWaves * 64, 0, st>>>(p);
        else few_rows_kernel<T, 4><<<grid, kFewWaves * 64, 0, st>>>(p);
        return;
    }
    const uint32_t grid = plan.tiles_m * plan.tiles_n * plan.splits;
    if (plan.tile == 256) tile_kernel<T, 4><<<grid, 256, 0, st>>>(p);
    else if (plan.tile == 128) tile_kernel<T, 2><<<grid, 256, 0, st>>>(p);
    else tile_kernel<T, 1><<<grid, 256, 0, st>>>(p);
    if (p.part) {
        const uint64_t blocks = ((uint64_t)p.a.rows * p.b.rows + 255) / 256;
        join_kernel<T><<<(uint32_t)(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(p);
    }
}

int check_side(const char *who, const char *name, const Side &s, uint32_t K, uint32_t blocks)
{
    DG_REQUIRE(s.q && s.scales && dg::aligned(s.q, 16) && s.ld % 16 == 0, DG_ERR_ARG, "%s: null pointer, or rows of %s that do not begin at multiples of 16 bytes", who, name);
    DG_REQUIRE(s.ld >= K && s.lds >= blocks && s.ld <= 1ull << 40 && s.lds <= 1ull << 40, DG_ERR_ARG, "%s: rows of %s overlap", who, name);
    return DG_OK;
}

bool in_range(uint64_t M, uint64_t N, uint32_t K) { return M <= 1ull << 24 && N <= 1ull << 24 && M * N <= 1ull << 40 && K >= 1 && K <= 1u << 24; }

}  // namespace

extern "C" size_t dg_e4m3_product_workspace_bytes(uint64_t M, uint64_t N, uint32_t K)
{
    if (!in_range(M, N, K) || M == 0 || N == 0) return 0;
    const Plan plan = plan_of((uint32_t)M, (uint32_t)N, K);
    return plan.splits > 1 ? (size_t)plan.splits * M * N * sizeof(float) : 0;
}

extern "C" int dg_e4m3_product(const void *a, uint64_t lda, const uint8_t *a_scales, uint64_t ldsa, const void *b, uint64_t ldb, const uint8_t *b_scales,
                               uint64_t ldsb, uint64_t M, uint64_t N, uint32_t K, uint32_t dtype, void *y, uint64_t ldy, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "dg_e4m3_product";
    DG_REQUIRE(dtype == DG_F16 || dtype == DG_BF16, DG_ERR_ARG, "%s: the result is fp16 or bf16", who);
    DG_REQUIRE(K >= 1, DG_ERR_ARG, "%s: K must be positive", who);
    DG_REQUIRE(in_range(M, N, K), DG_ERR_UNSUPPORTED, "%s: more than 2^24 rows or columns, or 2^40 results", who);
    if (M == 0 || N == 0) return DG_OK;
    const uint32_t blocks = (K + kBlockK - 1) / kBlockK;
    Product p = {};
    p.a = {(const uint8_t *)a, a_scales, lda, ldsa, (uint32_t)M};
    p.b = {(const uint8_t *)b, b_scales, ldb, ldsb, (uint32_t)N};
    if (int rc = check_side(who, "a", p.a, K, blocks)) return rc;
    if (int rc = check_side(who, "b", p.b, K, blocks)) return rc;
    DG_REQUIRE(y && dg::aligned(y, 2) && ldy >= N && ldy <= 1ull << 40, DG_ERR_ARG, "%s: null or misaligned result, or rows that overlap", who);
    const Plan plan = plan_of((uint32_t)M, (uint32_t)N, K);
    const size_t need = dg_e4m3_product_workspace_bytes(M, N, K);
    DG_REQUIRE(need == 0 || (ws && dg::aligned(ws, 16) && ws_bytes >= need), DG_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws ? ws_bytes : 0);
    p.y = y, p.part = need ? (float *)ws : nullptr, p.ldy = ldy, p.K = K, p.blocks = blocks, p.splits = plan.splits, p.tiles_m = plan.tiles_m, p.tiles_n = plan.tiles_n;
    if (dtype == DG_F16) launch<f16>(p, plan, (hipStream_t)stream);
    else launch<bf16>(p, plan, (hipStream_t)stream);
    return dg::launch_status(who);
}
