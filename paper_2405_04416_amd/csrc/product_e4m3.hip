// Matrix product of rows in 8-bit floating point with a power-of-two scale for each block of 128 columns:
//   y[m, n] = sum over k of a[m, k] 2^(sa[m, k / 128] - 127) b[n, k] 2^(sb[n, k / 128] - 127),   rounded once to 16 bits.
// The matrix instruction takes the exponents with its operands, so that nothing is scaled by hand and the sums stay in its accumulators (fp32).
//
// Three ways, by what bounds them.  Few rows: the bytes of b, which go from memory to the matrix instruction's registers with no stop in LDS.  Many:
// the matrix instruction; tiles are staged through LDS by loads that write there, the next block of columns while one is multiplied.  In between, with
// too few tiles for the chip, the columns are split over workgroups, whose sums a second launch adds in order.
//
// Of eight neighbouring products the instruction cuts off what is below 2^-13 of the largest (measured: a small product beside a large one and its opposite); everything after that is fp32.
// On random values that is 6e-5 of the results in root mean square, where rounding to fp16 is 2e-4: why they are 16 bits.  16384 x 4096 x 4096: 262 us, 2.1 PFLOP/s (249 us when the card has settled, after
// some fifty calls), of 3.9 that the instruction alone reaches on such values; 1003 x 1213 x 968 9.3 us; 8 x 8192 x 4096 10.8 us,
// 3.1 TB/s of b.
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

// 16 values of a row from column c on, 0 from K on.  Where the row ends within them, what lies behind it is cleared; behind the last row nothing may lie, so that there
// they are fetched one by one.
__device__ __forceinline__ u32x4 sixteen(const uint8_t *row, uint32_t c, uint32_t K, bool last)
{
    u32x4 v = {0, 0, 0, 0};
    if (c >= K) return v;
    if (c + 16 <= K || !last) v = *reinterpret_cast<const u32x4 *>(row + c);
    else
        for (uint32_t i = 0; c + i < K; ++i) v[i / 4] |= (uint32_t)row[c + i] << (8 * (i % 4));
    const uint32_t here = K - c;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t bytes = here > 4 * i ? here - 4 * i : 0;
        v[i] = bytes >= 4 ? v[i] : v[i] & ((1u << 8 * bytes) - 1);
    }
    return v;
}

__device__ __forceinline__ i32x8 both(u32x4 lo, u32x4 hi)
{
    return (i32x8){(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// ------------------------------------------------------------------------------ few rows
constexpr int kFewWaves = 8;

// A workgroup has 16 rows of b and all of a's (up to 16 MT); its wavefronts share the columns, block by block, and their sums meet in LDS.  Rows of b are read once, by as many workgroups as
// there are sixteens of them: bound by how soon 34 MB come (8 x 8192 x 4096), and by the launch.
template <class T, int MT>
__global__ void __launch_bounds__(kFewWaves * 64)
few_rows_kernel(Product p)
{
    __shared__ float sums[kFewWaves][MT][4][64];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n0 = blockIdx.x * 16, part = lane / 16 * 32;
    const uint32_t n = n0 + lane % 16 < p.b.rows ? n0 + lane % 16 : p.b.rows - 1;
    const uint8_t *b = p.b.q + n * p.b.ld, *sb = p.b.scales + n * p.b.lds;
    const uint8_t *a[MT], *sa[MT];
    bool last[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const uint32_t m = t * 16 + lane % 16 < p.a.rows ? t * 16 + lane % 16 : p.a.rows - 1;
        a[t] = p.a.q + m * p.a.ld;
        last[t] = m + 1 == p.a.rows;
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
        const bool last_b = n + 1 == p.b.rows;
        const i32x8 vb = both(sixteen(b, c, p.K, last_b), sixteen(b, c + 16, p.K, last_b));
#pragma unroll
        for (int t = 0; t < MT; ++t)
            acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vb, both(sixteen(a[t], c, p.K, last[t]), sixteen(a[t], c + 16, p.K, last[t])), acc[t], 0, 0, 0,
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
// A workgroup has a tile, PM x PN wavefronts side by side in it, each of WM x WN products of 32 x 32.  In LDS a row of 128 bytes lies in
// eight pieces of 16, piece c of row r at place c ^ key(r): the 16 lanes that read together then meet all banks once.
__device__ __forceinline__ uint32_t key(uint32_t r) { return (r & 7) ^ (r >> 3 & 1); }

// Two blocks of columns are in LDS or on their way.
template <int WM, int WN, int PM, int PN>
struct Tile {
    static constexpr int kWM = WM, kWN = WN;
    static constexpr uint32_t kWaves = PM * PN, kThreads = 64 * kWaves, kRowsA = 32 * WM * PM, kRowsB = 32 * WN * PN, kPM = PM, kPN = PN;
};
using Large = Tile<4, 4, 2, 2>;         // 256 x 256
using Middle = Tile<2, 2, 2, 2>;        // 128 x 128
using Small = Tile<1, 1, 2, 2>;         // 64 x 64

// Whole blocks of columns of a side's rows into LDS.  Loads that write to LDS put lane i's 16 bytes at place i, so lanes choose what they fetch: at one address for
// the workgroup and 32-bit distances from it (255 rows of less than 2^24 bytes).
template <uint32_t kRows, uint32_t kWaves>
struct Stage {
    static constexpr uint32_t kEach = kRows / 8 / kWaves;
    const uint8_t *base;
    uint32_t at[kEach], wave;
    __device__ __forceinline__ Stage(const Side &s, uint32_t row0) : base(s.q + row0 * s.ld), wave(__builtin_amdgcn_readfirstlane(threadIdx.x / 64))
    {
        const uint32_t lane = threadIdx.x % 64, last = s.rows - 1 - row0;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            const uint32_t r = (i * kWaves + wave) * 8 + lane / 8;
            at[i] = (r < last ? r : last) * (uint32_t)s.ld + ((lane % 8) ^ key(r)) * 16;
        }
    }
    __device__ __forceinline__ void fetch(uint32_t kb, uint8_t *to) const
    {
        const uint8_t *from = base + kb * kBlockK;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(from + at[i]),
                                             (__attribute__((address_space(3))) uint32_t *)(to + (i * kWaves + wave) * 8 * kBlockK), 16, 0, 0);
    }
};

// The block in which the rows end
template <uint32_t kRows, uint32_t kWaves>
__device__ __forceinline__ void stage_last(const Side &s, uint32_t row0, uint32_t kb, uint32_t K, uint8_t *to)
{
    constexpr uint32_t kEach = kRows / 8 / kWaves;
    u32x4 v[kEach];
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
        const uint32_t i = e * kWaves * 64 + threadIdx.x, r = i / 8, c = kb * kBlockK + ((i % 8) ^ key(r)) * 16, at = row0 + r < s.rows ? row0 + r : s.rows - 1;
        v[e] = sixteen(s.q + at * s.ld, c, K, at + 1 == s.rows);
    }
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) *reinterpret_cast<u32x4 *>(to + (e * kWaves * 64 + threadIdx.x) * 16) = v[e];
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

// Operands of half a block of columns, and their products
template <int WM, int WN>
struct Half {
    i32x8 a[WM], b[WN];
    __device__ __forceinline__ void read(const uint8_t *la, const uint8_t *lb, uint32_t lane, uint32_t half)
    {
        const uint32_t k = key(lane % 32), c = 4 * half + lane / 32 * 2;
        auto operand = [&](const uint8_t *tile, int t) {
            const uint8_t *row = tile + (t * 32 + lane % 32) * kBlockK;
            return both(*reinterpret_cast<const u32x4 *>(row + (c ^ k) * 16), *reinterpret_cast<const u32x4 *>(row + ((c + 1) ^ k) * 16));
        };
#pragma unroll
        for (int t = 0; t < WN; ++t) b[t] = operand(lb, t);
#pragma unroll
        for (int t = 0; t < WM; ++t) a[t] = operand(la, t);
    }
    __device__ __forceinline__ void multiply(const int (&ea)[WM], const int (&eb)[WN], f32x16 (&acc)[WM][WN]) const
    {
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int j = 0; j < WN; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[j], a[i], acc[i][j], 0, 0, 0, eb[j], 0, ea[i]);
    }
};

// Of all wavefronts: reads of LDS, and loads but for the `later` newest (they come in order).  Not __syncthreads(), which would wait for all loads.
template <uint32_t later>
__device__ __forceinline__ void loads_done()
{
    static_assert(later < 64, "as the instruction takes it");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | later % 16 | later / 16 << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <class T, class Tile>
__global__ void __launch_bounds__(Tile::kThreads)
tile_kernel(Product p)
{
    constexpr int WM = Tile::kWM, WN = Tile::kWN;
    constexpr uint32_t kRowsA = Tile::kRowsA, kRowsB = Tile::kRowsB, kBytes = (kRowsA + kRowsB) * kBlockK;
    __shared__ alignas(16) uint8_t lds[2][kBytes];       // blocks of columns: rows of a, then of b
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), tiles = p.tiles_m * p.tiles_n;
    // Workgroups go to the eight chiplets in turn: each gets a run of neighbouring tiles, in columns of eight, so that its cache serves them
    uint32_t id = blockIdx.x;
    const uint32_t all = tiles * p.splits, per = all / 8, more = all % 8, chiplet = id % 8;
    id = chiplet * per + (chiplet < more ? chiplet : more) + id / 8;
    const uint32_t split = id / tiles;
    id %= tiles;
    const uint32_t column = id / (8 * p.tiles_n), high = p.tiles_m - column * 8 < 8 ? p.tiles_m - column * 8 : 8, within = id % (8 * p.tiles_n);
    const uint32_t m0 = (column * 8 + within % high) * kRowsA, n0 = within / high * kRowsB;
    const uint32_t begin = (uint64_t)p.blocks * split / p.splits, end = (uint64_t)p.blocks * (split + 1) / p.splits;
    const uint32_t wm = wave / Tile::kPN * 32 * WM, wn = wave % Tile::kPN * 32 * WN;
    const uint8_t *sa[WM], *sb[WN];
#pragma unroll
    for (int t = 0; t < WM; ++t) {
        const uint32_t m = m0 + wm + t * 32 + lane % 32;
        sa[t] = p.a.scales + (uint64_t)(m < p.a.rows ? m : p.a.rows - 1) * p.a.lds;
    }
#pragma unroll
    for (int t = 0; t < WN; ++t) {
        const uint32_t n = n0 + wn + t * 32 + lane % 32;
        sb[t] = p.b.scales + (uint64_t)(n < p.b.rows ? n : p.b.rows - 1) * p.b.lds;
    }
    f32x16 acc[WM][WN] = {};
    int ea[WM], eb[WN], next_a[WM], next_b[WN];     // a block's exponents lie in the lowest byte
    auto fetch_exponents = [&](uint32_t kb) {
#pragma unroll
        for (int t = 0; t < WM; ++t) next_a[t] = exponents(sa[t], kb, p.blocks);
#pragma unroll
        for (int t = 0; t < WN; ++t) next_b[t] = exponents(sb[t], kb, p.blocks);
    };
    const Stage<kRowsA, Tile::kWaves> stage_a(p.a, m0);
    const Stage<kRowsB, Tile::kWaves> stage_b(p.b, n0);
    auto fetch = [&](uint32_t kb, uint32_t half) {
        stage_a.fetch(kb, lds[half]);
        stage_b.fetch(kb, lds[half] + kRowsA * kBlockK);
    };
    const uint32_t whole = end * kBlockK <= p.K ? end : end - 1;       // blocks before this one are whole
    const uint32_t at_a = wm * kBlockK, at_b = (kRowsA + wn) * kBlockK;
    Half<WM, WN> first, second;
    // behind the last block: something that is there, and is not used, so that as many loads as ever are on their way
    auto fetch_ahead = [&](uint32_t kb) { fetch(kb < whole ? kb : whole - 1, (kb - begin) % 2); };
    if (begin < whole) {
        fetch_exponents(begin);
        fetch(begin, 0);
        fetch_ahead(begin + 1);
        loads_done<(kRowsA + kRowsB) / 8 / Tile::kWaves>();
        first.read(lds[0] + at_a, lds[0] + at_b, lane, 0);
    }
    // Half a block is multiplied while the next half's operands come from LDS, of the next block too: between the halves a block's operands are all in registers,
    // so that its place can be loaded again.
    for (uint32_t kb = begin; kb < whole; ++kb) {
        const uint32_t i = kb - begin;
        if (i % 4 == 0) {
#pragma unroll
            for (int t = 0; t < WM; ++t) ea[t] = next_a[t];
#pragma unroll
            for (int t = 0; t < WN; ++t) eb[t] = next_b[t];
        }
        second.read(lds[i % 2] + at_a, lds[i % 2] + at_b, lane, 1);
        first.multiply(ea, eb, acc);
        __builtin_amdgcn_sched_barrier(0);
        loads_done<0>();
        if (i % 4 == 0 && kb + 4 < whole) fetch_exponents(kb + 4);
        fetch_ahead(kb + 2);
        first.read(lds[(i + 1) % 2] + at_a, lds[(i + 1) % 2] + at_b, lane, 0);
        second.multiply(ea, eb, acc);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < WM; ++t) ea[t] = (int)((uint32_t)ea[t] >> 8);
#pragma unroll
        for (int t = 0; t < WN; ++t) eb[t] = (int)((uint32_t)eb[t] >> 8);
    }
    if (begin < whole) loads_done<0>();
    if (whole < end) {
        stage_last<kRowsA, Tile::kWaves>(p.a, m0, whole, p.K, lds[0]);
        stage_last<kRowsB, Tile::kWaves>(p.b, n0, whole, p.K, lds[0] + kRowsA * kBlockK);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < WM; ++t) ea[t] = sa[t][whole];
#pragma unroll
        for (int t = 0; t < WN; ++t) eb[t] = sb[t][whole];
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            first.read(lds[0] + at_a, lds[0] + at_b, lane, h);
            first.multiply(ea, eb, acc);
        }
    }
    // Lane l has row l % 32 of a, and of b rows 8 g + 4 (l / 32) to 3 on, g = 0 to 3
    if (p.part) {
        float *part = p.part + (uint64_t)split * p.a.rows * p.b.rows;
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int j = 0; j < WN; ++j)
#pragma unroll
                for (int g = 0; g < 16; ++g) {
                    const uint32_t m = m0 + wm + i * 32 + lane % 32, n = n0 + wn + j * 32 + g / 4 * 8 + lane / 32 * 4 + g % 4;
                    if (m < p.a.rows && n < p.b.rows) part[(uint64_t)m * p.b.rows + n] = acc[i][j][g];
                }
        return;
    }
    // 32 rows at a time through LDS, so that a row's stores lie next to each other
    constexpr uint32_t kStride = WN * 32 + 8;
    __syncthreads();
    T *mine = reinterpret_cast<T *>(&lds[0][0]) + wave * 32 * kStride;
    static_assert(Tile::kWaves * 32 * kStride * sizeof(T) <= sizeof(lds), "room for the results");
    const bool vectors = p.b.rows % 8 == 0 && p.ldy % 8 == 0 && reinterpret_cast<uintptr_t>(p.y) % 16 == 0;
#pragma unroll
    for (int i = 0; i < WM; ++i) {
        wave_fence();
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float v[4] = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                dg_rows::store<T, 4>(mine + lane % 32 * kStride + j * 32 + g * 8 + lane / 32 * 4, v);
            }
        wave_fence();
        if (vectors) {
            constexpr uint32_t kVectors = WN * 4;       // of a row
#pragma unroll
            for (uint32_t e = 0; e < 32 * kVectors; e += 64) {
                const uint32_t r = (e + lane) / kVectors, c = (e + lane) % kVectors * 8, m = m0 + wm + i * 32 + r, n = n0 + wn + c;
                if (m < p.a.rows && n < p.b.rows) *reinterpret_cast<dg_rows::Pack<T, 8> *>((T *)p.y + m * p.ldy + n) = *reinterpret_cast<const dg_rows::Pack<T, 8> *>(mine + r * kStride + c);
            }
        } else
#pragma unroll 8
            for (uint32_t e = 0; e < 32 * 32 * WN; e += 64) {
                const uint32_t r = (e + lane) / (32 * WN), c = (e + lane) % (32 * WN), m = m0 + wm + i * 32 + r, n = n0 + wn + c;
                if (m < p.a.rows && n < p.b.rows) ((T *)p.y)[m * p.ldy + n] = mine[r * kStride + c];
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
// Rows of a up to which b's bytes are what counts, and up to which a launch of their own for sums of split columns costs more than that a's rows come from the caches for
// every 16 of b.  Few rows / tiles in us: 64 x 1024 x 1024 8.6 / 11.7, 24 x 4096 x 1024 8.7 / 11.4, 40 x 4096 x 4096 13.7 / 13.2, 32 x 8192 x 4096 18.3 / 13.7,
// 64 x 8192 x 4096 29.3 / 17.4.
constexpr uint32_t kFew = 16, kFewShort = 64, kShort = 2048;

struct Plan { uint32_t tile, tiles_m, tiles_n, splits; };      // tile 0: few rows

// The largest tiles of which there is one for each compute unit; with too few of the smallest, the columns are split.
Plan plan_of(uint32_t M, uint32_t N, uint32_t K)
{
    const uint32_t blocks = (K + kBlockK - 1) / kBlockK;
    if (M <= kFew || (M <= kFewShort && K <= kShort)) return {0, 0, 0, 1};
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
    if (plan.tile == 256) tile_kernel<T, Large><<<grid, Large::kThreads, 0, st>>>(p);
    else if (plan.tile == 128) tile_kernel<T, Middle><<<grid, Middle::kThreads, 0, st>>>(p);
    else tile_kernel<T, Small><<<grid, Small::kThreads, 0, st>>>(p);
    if (p.part) {
        const uint64_t blocks = ((uint64_t)p.a.rows * p.b.rows + 255) / 256;
        join_kernel<T><<<(uint32_t)(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(p);
    }
}

int check_side(const char *who, const char *name, const Side &s, uint32_t K, uint32_t blocks)
{
    DG_REQUIRE(s.q && s.scales && dg::aligned(s.q, 16) && s.ld % 16 == 0, DG_ERR_ARG, "%s: null pointer, or rows of %s that do not begin at multiples of 16 bytes", who, name);
    DG_REQUIRE(s.ld >= K && s.lds >= blocks && s.lds <= 1ull << 40, DG_ERR_ARG, "%s: rows of %s overlap", who, name);
    DG_REQUIRE(s.ld < 1ull << 24, DG_ERR_UNSUPPORTED, "%s: rows of %s 2^24 values or more apart", who, name);
    return DG_OK;
}

// 2^39 results are 2^23 tiles of 256 lanes: a launch has fewer than 2^32 lanes.
bool in_range(uint64_t M, uint64_t N, uint32_t K) { return M <= 1ull << 24 && N <= 1ull << 24 && M * N <= 1ull << 39 && K >= 1 && K < 1u << 24; }

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
    DG_REQUIRE(in_range(M, N, K), DG_ERR_UNSUPPORTED, "%s: more than 2^24 rows or columns, or 2^39 results", who);
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
