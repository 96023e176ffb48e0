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

// Rows of positions and heads, LANES lanes each, 8 elements a lane; a row's largest value takes exchanges between the lanes of a block of elements.
// Memory bounds it: reads and writes of 16 bytes a lane (fewer bits: 8 or 4 written), nothing read twice.
template <class T, int HELD, int LANES>
__global__ __launch_bounds__(256) void k_cache_write(WriteArgs a)
{
    const uint32_t b = blockIdx.y, lane = threadIdx.x % LANES;
    const uint64_t row = (uint64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int n = cached(a.lengths, a.len, b);
    if (row >= (uint64_t)n * a.kv_heads) return;           // whole groups of LANES lanes
    const uint32_t i = (uint32_t)(row / a.kv_heads), h = (uint32_t)(row % a.kv_heads);
    const int64_t at = (int64_t)a.start[b] + i;
    if (at < 0 || at >= (int64_t)a.c.table_pages << a.c.page_log2) return;
    const int32_t page = a.c.table[b * a.c.table_stride + (at >> a.c.page_log2)];
    if ((uint32_t)page >= a.c.pages) return;
    const uint32_t place = (uint32_t)at & (a.c.page - 1);
    const bool in = lane * 8 < a.dim;
    const Moved& m = blockIdx.z ? a.v : a.k;
    uint4 x = *(const uint4*)(in ? m.p + b * m.batch + h * m.head + i * m.pos + lane * 16 : (const char*)&zero16);
    char* to = (blockIdx.z ? a.c.v + page * a.c.v_stride : a.c.k + page * a.c.k_stride) + ((uint64_t)h * a.c.page + place) * a.c.row + lane * EIGHT<HELD>;
    if constexpr (HELD == FF_HELD_SAME) {
        if (in) *(uint4*)to = x;
    } else {
        float f[8], top = 0;
        const typename T::vec8 e = __builtin_bit_cast(typename T::vec8, x);
        bool fine = true;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            f[k] = (float)e[k];
            fine &= __builtin_fabsf(f[k]) < INFINITY;
            f[k] = fminf(fmaxf(f[k], -MOST<T>(HELD)), MOST<T>(HELD));
            top = fmaxf(top, __builtin_fabsf(f[k]));
        }
        uint32_t bad = !fine;
        constexpr int BLOCK = HELD == FF_HELD_E4M3 ? LANES : 4;
#pragma unroll
        for (int d = BLOCK / 2; d; d /= 2) {
            top = fmaxf(top, __shfl_xor(top, d));
            bad |= __shfl_xor(bad, d);
        }
        const uint32_t s = bad ? 255 : scale_byte<HELD>(top);
        // times 2^(127 - s): beyond a float's exponents at both ends, so in two steps, which are exact unless the value is far below the smallest code
        const float up = s < 127 ? __builtin_bit_cast(float, (127u + 63) << 23) : 1.0f;
        const float by = __builtin_bit_cast(float, s < 127 ? (254u - 63 - s) << 23 : s < 254 ? (254u - s) << 23 : 1u << 22);
        if (bad)
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = f[k] * by * up;
        if constexpr (HELD == FF_HELD_E4M3) {
            int lo = 0, hi = 0;
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], lo, false), lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], lo, true);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], hi, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], hi, true);
            if (in) *(uint2*)to = uint2{(uint32_t)lo, (uint32_t)hi};
        } else {
            uint32_t c = 0;
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], 1.0f, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], 1.0f, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], 1.0f, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], 1.0f, 3);
            if (in) *(uint32_t*)to = c;
        }
        uint8_t* st = (blockIdx.z ? a.c.v_scale + page * a.c.v_scale_stride : a.c.k_scale + page * a.c.k_scale_stride) + ((uint64_t)h * a.c.blocks + lane / BLOCK) * a.c.page + place;
        if (in && lane % BLOCK == 0) *st = (uint8_t)s;
    }
}

template <class T, int HELD, int LANES>
__global__ __launch_bounds__(256) void k_cache_read(ReadArgs a)
{
    const uint32_t b = blockIdx.y / a.kv_heads, h = blockIdx.y % a.kv_heads, lane = threadIdx.x % LANES;
    const uint32_t i = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (i >= a.len || lane * 8 >= a.dim) return;
    const int n = cached(a.lengths, min(a.len, a.c.table_pages << a.c.page_log2), b);
    const Moved& m = blockIdx.z ? a.v : a.k;
    uint4 x = {0, 0, 0, 0};
    if ((int)i < n) {
        const int32_t page = a.c.table[b * a.c.table_stride + (i >> a.c.page_log2)];
        const uint32_t place = i & (a.c.page - 1);
        if ((uint32_t)page >= a.c.pages) {
            x = {0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
        } else {
            const char* from = (blockIdx.z ? a.c.v + page * a.c.v_stride : a.c.k + page * a.c.k_stride) + ((uint64_t)h * a.c.page + place) * a.c.row + lane * EIGHT<HELD>;
            float s = 0;
            if constexpr (HELD != FF_HELD_SAME)
                s = scale_operand((blockIdx.z ? a.c.v_scale + page * a.c.v_scale_stride : a.c.k_scale + page * a.c.k_scale_stride)[((uint64_t)h * a.c.blocks + (HELD == FF_HELD_E4M3 ? 0 : lane / 4)) * a.c.page + place]);
            x = Eight<T, HELD>::get(*(const typename Eight<T, HELD>::raw*)from, s);
        }
    }
    *(uint4*)(const_cast<char*>(m.p) + b * m.batch + h * m.head + i * m.pos + lane * 16) = x;
}

Moved moved(const ff_heads_t& h) { return {(const char*)h.p, h.batch * 2, h.head * 2, h.pos * 2}; }
bool heads_fit(const ff_heads_t& h) { return h.p && aligned(h.p, 16) && !((h.batch | h.head | h.pos) & 7); }

template <class T, int HELD>
void launch(const WriteArgs& a, hipStream_t st)
{
    const uint32_t lanes = a.dim > 64 ? 16 : 8;
    const dim3 grid((uint32_t)ceil_div((uint64_t)a.len * a.kv_heads, 256 / lanes), a.batch, 2);
    if (lanes == 16) k_cache_write<T, HELD, 16><<<grid, 256, 0, st>>>(a);
    else k_cache_write<T, HELD, 8><<<grid, 256, 0, st>>>(a);
}

template <class T, int HELD>
void launch(const ReadArgs& a, hipStream_t st)
{
    const uint32_t lanes = a.dim > 64 ? 16 : 8;
    const dim3 grid((uint32_t)ceil_div(a.len, 256 / lanes), a.batch * a.kv_heads, 2);
    if (lanes == 16) k_cache_read<T, HELD, 16><<<grid, 256, 0, st>>>(a);
    else k_cache_read<T, HELD, 8><<<grid, 256, 0, st>>>(a);
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
