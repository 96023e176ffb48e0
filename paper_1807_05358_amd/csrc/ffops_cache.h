// What the paged cache's kernels share: its place in memory, and how elements are held in fewer bits.
#pragma once
#include "ffops_device.h"

namespace ffops {

struct CacheArgs {
    char *k, *v;
    uint8_t *k_scale, *v_scale;
    const int32_t* table;
    int64_t k_stride, v_stride, k_scale_stride, v_scale_stride, table_stride;
    uint32_t pages, page, page_log2, table_pages;
    uint32_t row;               // bytes of a row: one position of one head
    uint32_t blocks;            // scales of a row
};

// positions that sequence b has in the cache: its length, no more than `most`
static __device__ __forceinline__ int cached(const int32_t* lengths, uint32_t most, uint32_t b)
{
    if (!lengths) return (int)most;
    const int n = lengths[b];
    return n < 0 ? 0 : n > (int)most ? (int)most : n;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// A scale's byte as the operand of the converting instructions, which take a float's exponent alone: 0 stands for 2^-127 there, 255 for NaN.
static __device__ __forceinline__ float scale_operand(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// two codes and a scale to two elements, rounded where float16 ends: of e4m3 the half HI of a word, of e2m1 byte AT of it
template <class T, bool HI>
static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w, float scale)
{
    if constexpr (std::is_same<T, BF16>::value) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HI));
}
template <class T, int AT>
static __device__ __forceinline__ uint32_t from_e2m1(uint32_t w, float scale)
{
    if constexpr (std::is_same<T, BF16>::value) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, AT));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, AT));
}

// eight elements from how they are held
template <class T, int HELD>
struct Eight;
template <class T>
struct Eight<T, FF_HELD_SAME> {
    typedef uint4 raw;
    static __device__ __forceinline__ uint4 get(raw r, float) { return r; }
};
template <class T>
struct Eight<T, FF_HELD_E4M3> {
    typedef uint2 raw;
    static __device__ __forceinline__ uint4 get(raw r, float s) { return {from_e4m3<T, false>(r.x, s), from_e4m3<T, true>(r.x, s), from_e4m3<T, false>(r.y, s), from_e4m3<T, true>(r.y, s)}; }
};
template <class T>
struct Eight<T, FF_HELD_E2M1> {
    typedef uint32_t raw;
    static __device__ __forceinline__ uint4 get(raw r, float s) { return {from_e2m1<T, 0>(r, s), from_e2m1<T, 1>(r, s), from_e2m1<T, 2>(r, s), from_e2m1<T, 3>(r, s)}; }
};

// bytes of eight elements
template <int HELD>
constexpr uint32_t EIGHT = HELD == FF_HELD_SAME ? 16 : HELD == FF_HELD_E4M3 ? 8 : 4;

// sizes that all calls on a cache refuse or limit
static inline int check_cache_sizes(const ff_cache_t& c, uint32_t dtype, uint32_t batch, uint32_t kv_heads, uint32_t head_dim)
{
    if (dtype != FF_F16 && dtype != FF_BF16) return FF_EINVAL;
    if (c.held > FF_HELD_E2M1 || kv_heads == 0 || head_dim == 0 || head_dim % (c.held == FF_HELD_SAME ? 8 : c.held == FF_HELD_E4M3 ? 16 : 32)) return FF_EINVAL;
    if (c.page < 16 || (c.page & (c.page - 1)) || c.pages > 0x7fffffffu) return FF_EINVAL;
    if (head_dim > FF_OP_MAX_HEAD_DIM || c.page > FF_OP_MAX_PAGE || (uint64_t)c.table_pages * c.page > FF_OP_MAX_LEN) return FF_ERANGE;
    if (kv_heads > 65535 || batch > 65535 || (uint64_t)batch * kv_heads > 65535u * 32) return FF_ERANGE;
    return FF_OK;
}

// addresses, of a cache that a call looks at
static inline int check_cache(const ff_cache_t& c)
{
    if (c.pages == 0 || !c.table || !c.k || !c.v || !aligned(c.k, 16) || !aligned(c.v, 16) || ((c.k_stride | c.v_stride) & 15)) return FF_EINVAL;
    if (c.held != FF_HELD_SAME && (!c.k_scale || !c.v_scale || !aligned(c.k_scale, 4) || !aligned(c.v_scale, 4) || ((c.k_scale_stride | c.v_scale_stride) & 3))) return FF_EINVAL;
    return FF_OK;
}

static inline CacheArgs cache_args(const ff_cache_t& c, uint32_t head_dim)
{
    CacheArgs a = {(char*)c.k, (char*)c.v, c.k_scale, c.v_scale, c.table, c.k_stride, c.v_stride, c.k_scale_stride, c.v_scale_stride, c.table_stride, c.pages, c.page, 0, c.table_pages, 0, 0};
    while ((1u << a.page_log2) < c.page) ++a.page_log2;
    a.row = c.held == FF_HELD_SAME ? head_dim * 2 : c.held == FF_HELD_E4M3 ? head_dim : head_dim / 2;
    a.blocks = c.held == FF_HELD_SAME ? 0 : c.held == FF_HELD_E4M3 ? 1 : head_dim / 32;
    return a;
}

}  // namespace ffops
