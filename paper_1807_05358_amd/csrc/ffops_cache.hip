// A paged cache of keys and values: as it is written, and read back.
#include "ffops_cache.h"

namespace ffops {
namespace {

struct Moved {
    const char* p;                  // of k or v: bytes
    int64_t batch, head, pos;
};

struct WriteArgs {
    CacheArgs c;
    Moved k, v;
    const int32_t *start, *lengths;
    uint32_t batch, kv_heads, len, dim;
};

struct ReadArgs {
    CacheArgs c;
    Moved k, v;
    const int32_t* lengths;
    uint32_t batch, kv_heads, len, dim;
};

template <class T>
constexpr float MOST(int held)
{
    return (held == FF_HELD_E4M3 ? 1.875f : 1.5f) * (std::is_same<T, F16>::value ? 0x1p15f : 0x1p127f);
}

// The scale's byte of a block whose largest value is `top`: the least power of two with top <= 448 (6) times it.  448 = 1.75 * 2^8 and 6 = 1.5 * 2^2, so it is the
// float's own exponent less 8 (2), and one more where the fraction is beyond .75 (.5).
template <int HELD>
__device__ __forceinline__ uint32_t scale_byte(float top)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, top), less = HELD == FF_HELD_E4M3 ? 8 : 2, fraction = HELD == FF_HELD_E4M3 ? 0x600000 : 0x400000;
    // a float below 2^-126 has exponent 0 and needs a byte below 0: 0 it is then, as for all others below
    const int e = (int)(bits >> 23) - (int)less + ((bits & 0x7fffff) > fraction);
    return (uint32_t)(e < 0 ? 0 : e);
}

// the larger one of both halves of two words
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
{
    typedef uint16_t half2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(half2, a), __builtin_bit_cast(half2, b)));
}

// the largest over a block of lanes: the other of two, the other two of four, then mirrored in 8 and in 16
template <int CTRL>
__device__ __forceinline__ uint32_t larger_of(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false)); }
template <int LANES>
__device__ __forceinline__ uint32_t over_block(uint32_t x)
{
    x = larger_of<0x4e>(larger_of<0xb1>(x));
    if constexpr (LANES >= 8) x = larger_of<0x141>(x);
    if constexpr (LANES >= 16) x = larger_of<0x140>(x);
    return x;
}

// four elements, divided by a power of two, to e4m3, and eight to e2m1: to the nearest, the even one of two as near
typedef short i16x2 __attribute__((ext_vector_type(2)));
template <class T>
__device__ __forceinline__ uint32_t to_e4m3(uint32_t a, uint32_t b, float by)
{
    i16x2 c = {0, 0};
    if constexpr (std::is_same<T, BF16>::value) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, a), by, false);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, b), by, true);
    } else {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c, __builtin_bit_cast(f16x2, a), by, false);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c, __builtin_bit_cast(f16x2, b), by, true);
    }
    return __builtin_bit_cast(uint32_t, c);
}
template <class T>
__device__ __forceinline__ uint32_t to_e2m1(uint4 v, float by)
{
    uint32_t c = 0;
    if constexpr (std::is_same<T, BF16>::value) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v.x), by, 0), c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v.y), by, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v.z), by, 2), c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v.w), by, 3);
    } else {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, v.x), by, 0), c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, v.y), by, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, v.z), by, 2), c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, v.w), by, 3);
    }
    return c;
}

// Both directions: rows of a position and a head, LANES lanes each, 8 elements a lane; a thread has ROWS of them, all of whose loads it asks for before it uses the first.  Memory bounds both; nothing is
// read twice.

// Writing: a block's largest value is found as the bits of its size and takes exchanges between its lanes; codes come from the instructions that divide by a power of two and round to the nearest.
// 55 MB of prompts into e4m3, 28 MB: 25 us by way of 32 bits, 19 so, 4.4 TB/s.
template <class T, int HELD, int LANES, int ROWS>
__global__ __launch_bounds__(256) void k_cache_write(WriteArgs a)
{
    constexpr int GROUPS = 256 / LANES;
    const uint32_t b = blockIdx.y, lane = threadIdx.x % LANES;
    const uint64_t row0 = (uint64_t)blockIdx.x * (GROUPS * ROWS) + threadIdx.x / LANES, rows = (uint64_t)cached(a.lengths, a.len, b) * a.kv_heads;
    if (row0 >= rows) return;           // whole groups of LANES lanes
    const Moved& m = blockIdx.z ? a.v : a.k;
    const int64_t start = a.start[b], stride = blockIdx.z ? a.c.v_stride : a.c.k_stride, scale_stride = blockIdx.z ? a.c.v_scale_stride : a.c.k_scale_stride;
    char* pages = blockIdx.z ? a.c.v : a.c.k;
    uint8_t* scales = blockIdx.z ? a.c.v_scale : a.c.k_scale;
    const bool in = lane * 8 < a.dim;
    uint4 x[ROWS];
    int32_t page[ROWS];                 // -1: the row is not written
    uint32_t head[ROWS], place[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint64_t row = row0 + r * GROUPS;
        page[r] = -1, x[r] = {0, 0, 0, 0};
        if (row >= rows) continue;
        const uint32_t i = (uint32_t)row / a.kv_heads;
        const int64_t at = start + i;
        head[r] = (uint32_t)row % a.kv_heads, place[r] = (uint32_t)at & (a.c.page - 1);
        if (at >= 0 && at < (int64_t)a.c.table_pages << a.c.page_log2) page[r] = a.c.table[b * a.c.table_stride + (at >> a.c.page_log2)];
        if (in) x[r] = *(const uint4*)(m.p + b * m.batch + head[r] * m.head + i * m.pos + lane * 16);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const bool here = (uint32_t)page[r] < a.c.pages;
        char* to = pages + page[r] * stride + ((uint64_t)head[r] * a.c.page + place[r]) * a.c.row + lane * EIGHT<HELD>;
        if constexpr (HELD == FF_HELD_SAME) {
            if (here && in) *(uint4*)to = x[r];
        } else {
            // the largest of the block, as the bits of its size; infinities and NaN are the largest of all
            constexpr int BLOCK = HELD == FF_HELD_E4M3 ? LANES : 4;
            uint4 v = x[r];
            uint32_t top = larger(larger(v.x & 0x7fff7fff, v.y & 0x7fff7fff), larger(v.z & 0x7fff7fff, v.w & 0x7fff7fff));
            top = over_block<BLOCK>(larger(top, top >> 16) & 0xffff);
            const bool bad = top >= (std::is_same<T, F16>::value ? 0x7c00u : 0x7f80u);
            const float most = (float)__builtin_bit_cast(typename T::elem, (uint16_t)top);
            const uint32_t s = bad ? 255 : scale_byte<HELD>(fminf(most, MOST<T>(HELD)));
            if (bad) v = {0, 0, 0, 0};
            else if (most > MOST<T>(HELD)) {
                typename T::vec8 e = __builtin_bit_cast(typename T::vec8, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) e[k] = (typename T::elem)fminf(fmaxf((float)e[k], -MOST<T>(HELD)), MOST<T>(HELD));
                v = __builtin_bit_cast(uint4, e);
            }
            const float by = scale_operand(bad ? 127 : s);
            if constexpr (HELD == FF_HELD_E4M3) {
                const uint2 c = {to_e4m3<T>(v.x, v.y, by), to_e4m3<T>(v.z, v.w, by)};
                if (here && in) *(uint2*)to = c;
            } else {
                const uint32_t c = to_e2m1<T>(v, by);
                if (here && in) *(uint32_t*)to = c;
            }
            if (here && in && lane % BLOCK == 0) scales[page[r] * scale_stride + ((uint64_t)head[r] * a.c.blocks + lane / BLOCK) * a.c.page + place[r]] = (uint8_t)s;
        }
    }
}

// Reading.  The stores pass by the caches (there is more than they hold; where there is not, attention over what was read takes no longer for it): 117 MB of e4m3 and 537 MB written, 148 us with one row
// a thread, 127 with four, 92 with four and such stores, 7.1 TB/s.
template <class T, int HELD, int LANES>
__global__ __launch_bounds__(256) void k_cache_read(ReadArgs a)
{
    constexpr int ROWS = 4, GROUPS = 256 / LANES;
    const uint32_t b = blockIdx.y / a.kv_heads, h = blockIdx.y % a.kv_heads, lane = threadIdx.x % LANES, i0 = blockIdx.x * (ROWS * GROUPS) + threadIdx.x / LANES;
    if (lane * 8 >= a.dim) return;
    const int n = cached(a.lengths, min(a.len, a.c.table_pages << a.c.page_log2), b);
    const Moved& m = blockIdx.z ? a.v : a.k;
    const char* pages = blockIdx.z ? a.c.v : a.c.k;
    const uint8_t* scales = blockIdx.z ? a.c.v_scale : a.c.k_scale;
    const int64_t stride = blockIdx.z ? a.c.v_stride : a.c.k_stride, scale_stride = blockIdx.z ? a.c.v_scale_stride : a.c.k_scale_stride;
    char* to = const_cast<char*>(m.p) + b * m.batch + h * m.head + lane * 16;
    const int32_t* table = a.c.table + b * a.c.table_stride;
    typename Eight<T, HELD>::raw raw[ROWS];
    uint32_t s[ROWS];
    int32_t page[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t i = i0 + r * GROUPS;
        page[r] = (int)i < n ? table[i >> a.c.page_log2] : -1;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t place = (i0 + r * GROUPS) & (a.c.page - 1);
        s[r] = 0, raw[r] = {};
        if ((uint32_t)page[r] < a.c.pages) {
            raw[r] = *(const typename Eight<T, HELD>::raw*)(pages + page[r] * stride + ((uint64_t)h * a.c.page + place) * a.c.row + lane * EIGHT<HELD>);
            if constexpr (HELD != FF_HELD_SAME) s[r] = scales[page[r] * scale_stride + ((uint64_t)h * a.c.blocks + (HELD == FF_HELD_E4M3 ? 0 : lane / 4)) * a.c.page + place];
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t i = i0 + r * GROUPS;
        if (i >= a.len) return;
        typedef uint32_t words __attribute__((ext_vector_type(4)));
        const uint4 x = Eight<T, HELD>::get(raw[r], scale_operand(s[r]));
        const bool lost = (int)i < n && (uint32_t)page[r] >= a.c.pages;
        __builtin_nontemporal_store(lost ? words{0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu} : words{x.x, x.y, x.z, x.w}, (words*)(to + i * m.pos));
    }
}

Moved moved(const ff_heads_t& h) { return {(const char*)h.p, h.batch * 2, h.head * 2, h.pos * 2}; }
bool heads_fit(const ff_heads_t& h) { return h.p && aligned(h.p, 16) && !((h.batch | h.head | h.pos) & 7); }

// Rows of a thread: one where a sequence's rows make no more than 64 blocks, which takes 0.7 to 1.1 us less (a step, 64 positions of 8 heads: 2.7 us and 3.5, in e4m3 3.0 and 4.1); else four, for batches that are mostly padding, whose
// blocks without a row then are a quarter: 64 sequences of up to 2048 positions, 8 heads of 128, seven of eight of them at most 40 long, 24 us and 34 with one row, in e4m3 23 and 33.  Batches that are half or all full pay for it:
// 16 of up to 2048, 34 and 29 us, in e4m3 29 and 24; 4 of 4096 29 and 27; 64 of 128 12.7 and 13.8.
template <class T, int HELD, int LANES>
void launch_lanes(const WriteArgs& a, hipStream_t st)
{
    const uint64_t rows = (uint64_t)a.len * a.kv_heads;
    constexpr int GROUPS = 256 / LANES;
    if (rows >= 64 * GROUPS) k_cache_write<T, HELD, LANES, 4><<<dim3((uint32_t)ceil_div(rows, 4 * GROUPS), a.batch, 2), 256, 0, st>>>(a);
    else k_cache_write<T, HELD, LANES, 1><<<dim3((uint32_t)ceil_div(rows, GROUPS), a.batch, 2), 256, 0, st>>>(a);
}
template <class T, int HELD, int LANES>
void launch_lanes(const ReadArgs& a, hipStream_t st)
{
    k_cache_read<T, HELD, LANES><<<dim3((uint32_t)ceil_div(a.len, 4 * 256 / LANES), a.batch * a.kv_heads, 2), 256, 0, st>>>(a);
}

template <class T, int HELD, class A>
void launch(const A& a, hipStream_t st)
{
    if (a.dim > 64) launch_lanes<T, HELD, 16>(a, st);
    else launch_lanes<T, HELD, 8>(a, st);
}

template <class T, class A>
void launch_held(const A& a, uint32_t held, hipStream_t st)
{
    if (held == FF_HELD_SAME) launch<T, FF_HELD_SAME>(a, st);
    else if (held == FF_HELD_E4M3) launch<T, FF_HELD_E4M3>(a, st);
    else launch<T, FF_HELD_E2M1>(a, st);
}

}  // namespace
}  // namespace ffops

using namespace ffops;

extern "C" int ff_op_cache_write(const ff_cache_write_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check_cache_sizes(p->cache, p->dtype, p->batch, p->kv_heads, p->head_dim)) return rc;
    if (ceil_div((uint64_t)p->new_len * p->kv_heads, 16) * 256 > MOST_THREADS) return FF_ERANGE;
    if (p->batch == 0 || p->new_len == 0 || p->cache.table_pages == 0) return FF_OK;
    if (!heads_fit(p->k) || !heads_fit(p->v) || !p->start) return FF_EINVAL;
    if (const int rc = check_cache(p->cache)) return rc;
    const WriteArgs a = {cache_args(p->cache, p->head_dim), moved(p->k), moved(p->v), p->start, p->lengths, p->batch, p->kv_heads, p->new_len, p->head_dim};
    if (p->dtype == FF_F16) launch_held<F16>(a, p->cache.held, (hipStream_t)stream);
    else launch_held<BF16>(a, p->cache.held, (hipStream_t)stream);
    return launched();
}

extern "C" int ff_op_cache_read(const ff_cache_read_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check_cache_sizes(p->cache, p->dtype, p->batch, p->kv_heads, p->head_dim)) return rc;
    if (ceil_div(p->kv_len, 16) * 256 > MOST_THREADS || (uint64_t)p->batch * p->kv_heads > MOST_BLOCKS_Y) return FF_ERANGE;
    if (p->batch == 0 || p->kv_len == 0) return FF_OK;
    if (!heads_fit(p->k) || !heads_fit(p->v)) return FF_EINVAL;
    if (p->cache.table_pages)
        if (const int rc = check_cache(p->cache)) return rc;
    const ReadArgs a = {cache_args(p->cache, p->head_dim), moved(p->k), moved(p->v), p->lengths, p->batch, p->kv_heads, p->kv_len, p->head_dim};
    if (p->dtype == FF_F16) launch_held<F16>(a, p->cache.held, (hipStream_t)stream);
    else launch_held<BF16>(a, p->cache.held, (hipStream_t)stream);
    return launched();
}
