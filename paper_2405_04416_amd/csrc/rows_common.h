// Rows of a sequence block (layer norm, recurrence, dropout): element types and loads of several elements.  Internal.
#pragma once
#include "dg_internal.h"

namespace dg_rows {

// DG_F32, DG_F16, DG_BF16 in memory; everything is computed in fp32.  A store rounds to the nearest even value, once.
using f16 = _Float16;
using bf16 = __bf16;

template <class T, int V>
struct alignas(sizeof(T) * V) Pack { T v[V]; };

template <class T, int V>
__device__ __forceinline__ void store(T *p, const float (&in)[V])
{
    Pack<T, V> a;
#pragma unroll
    for (int i = 0; i < V; ++i) a.v[i] = (T)in[i];
    *reinterpret_cast<Pack<T, V> *>(p) = a;
}

// From this size on the arrays of layer norm and dropout go past the caches.  Each call reading what the last one wrote, four arrays in
// turn, through / past the caches in us: 64 MiB norm 23.5 / 25.8, its gradient 43.3 / 41.8, dropout 27.7 / 32.0; 128 MiB 48.0 / 49.1,
// 94.3 / 76.4, 69.7 / 62.8; 512 MiB 202 / 194, 365 / 289, 268 / 250.
constexpr uint64_t kStreamedBytes = 96 << 20;

template <class T, int V>
__device__ __forceinline__ Pack<T, V> load_streamed(const T *p)
{
    static_assert(sizeof(Pack<T, V>) == 16, "one load");
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(Pack<T, V>, __builtin_nontemporal_load(reinterpret_cast<const u4 *>(p)));
}

template <class T, int V>
__device__ __forceinline__ void store_streamed(T *p, const Pack<T, V> &a)
{
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(u4, a), reinterpret_cast<u4 *>(p));
}

inline size_t item_bytes(uint32_t dtype) { return dtype == DG_F32 ? 4 : 2; }
inline bool known_type(uint32_t dtype) { return dtype == DG_F32 || dtype == DG_F16 || dtype == DG_BF16; }

// whether rows of `ld` elements from p on can be loaded `bytes` at a time
inline bool rows_aligned(const void *p, uint64_t ld, uint32_t dtype, size_t bytes)
{
    return dg::aligned(p, bytes) && ld * item_bytes(dtype) % bytes == 0;
}

}  // namespace dg_rows
