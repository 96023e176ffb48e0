// What the kernels of the training operators share: element types, matrix instructions, loads into LDS, reductions.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/ff_ops.h"

namespace ffops {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

struct F32 {
    typedef float elem;
    static constexpr int VEC = 4;      // elements of a 16-byte access
};
struct F16 {
    typedef _Float16 elem;
    typedef f16x8 vec8;
    static constexpr int VEC = 8;
    static __device__ __forceinline__ f32x16 mma(vec8 a, vec8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 mma(vec8 a, vec8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ void mma_acc(vec8 a, vec8 b, f32x4& c) { asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};
struct BF16 {
    typedef __bf16 elem;
    typedef bf16x8 vec8;
    static constexpr int VEC = 8;
    static __device__ __forceinline__ f32x16 mma(vec8 a, vec8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 mma(vec8 a, vec8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ void mma_acc(vec8 a, vec8 b, f32x4& c) { asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};
// The 32x32x16 product: lane l gives A[l % 32][8 * (l / 32) + e] and B[8 * (l / 32) + e][l % 32], e = 0..7, and holds
// C[8 * (r / 4) + 4 * (l / 32) + r % 4][l % 32] in register r = 0..15.  Which k the pair (l / 32, e) stands for does not
// matter as long as A and B agree, so eight registers of a C tile are a B operand as they are, with
// k = 16 * step + 8 * (e / 4) + 4 * (l / 32) + e % 4, if A is read in that order.
// The 16x16x32 product: lane l gives A[l % 16][8 * (l / 16) + e] and B[8 * (l / 16) + e][l % 16] and holds
// C[4 * (l / 16) + r][l % 16] in register r = 0..3.  Both do 1024 products a cycle; on numbers that are not zero the device's power sets the
// clock, and the small one gives more of them: 2083 TFLOP/s against 1859 from registers alone, at the same reads of LDS.

// Waits until what this wave has asked of LDS, and of memory but for the latest NEWER loads, is there, and then for all other waves of the block.
// Unlike __syncthreads it lets loads into LDS pass.
template <int NEWER>
static __device__ __forceinline__ void meet()
{
    static_assert(NEWER < 64, "what the counter of loads holds");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0070 | (NEWER & 15) | (NEWER >> 4 << 14));     // vmcnt, lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

static __device__ __forceinline__ int c_row(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

// 16 bytes that rows and columns beyond a matrix are read from
static __device__ const uint4 zero16 = {0, 0, 0, 0};

// 16 bytes per lane from global memory into LDS at dst + 16 * lane, without registers between; dst is uniform
static __device__ __forceinline__ void load_lds16(const char* src, lds_char* dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// 4 bytes per lane, at dst + 4 * lane
static __device__ __forceinline__ void load_lds4(const float* src, lds_char* dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 4, 0, 0);
}

// the same as load_lds16 from base + off, base uniform: the address takes one register of a lane and no arithmetic
static __device__ __forceinline__ void load_lds16(const char* base, uint32_t off, lds_char* dst)
{
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0xffffffffu, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)dst, 16, off, 0, 0, 0);
}

// eight elements at p as an operand
template <class T>
static __device__ __forceinline__ typename T::vec8 read8(const lds_char* p)
{
    return *(const __attribute__((address_space(3))) typename T::vec8*)p;
}

// eight elements as an operand from two transposed reads: in every 16 lanes, lane i gives the address of 4 elements --
// columns 4 * (i % 4) .. + 3 of row i / 4 of a 4 x 16 block -- and receives column i of that block
template <class T>
static __device__ __forceinline__ typename T::vec8 read8_tr(const lds_char* lo, const lds_char* hi)
{
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)lo);
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)hi);
    return __builtin_bit_cast(typename T::vec8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <class T>
static __device__ __forceinline__ typename T::vec8 round8(const float* f)
{
    typename T::vec8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (typename T::elem)f[e];
    return v;
}

template <class T>
static __device__ __forceinline__ void store4(void* p, float a, float b, float c, float d)
{
    typedef typename T::elem v4 __attribute__((ext_vector_type(4)));
    *(v4*)p = v4{(typename T::elem)a, (typename T::elem)b, (typename T::elem)c, (typename T::elem)d};
}

template <class T>
static __device__ __forceinline__ uint2 pack4(f32x4 c)
{
    typedef typename T::elem v4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint2, v4{(typename T::elem)c[0], (typename T::elem)c[1], (typename T::elem)c[2], (typename T::elem)c[3]});
}

static __device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
static __device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }

// the value of lane l ^ 32
static __device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

static __device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

constexpr uint64_t MOST_THREADS = 0xffffffffull;       // of a launch, along x
constexpr uint32_t MOST_BLOCKS_Y = 65535;              // of a launch, along y

static inline int launched() { return hipGetLastError() == hipSuccess ? FF_OK : FF_EHIP; }
static inline bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
static inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
static inline uint64_t round_up(uint64_t a, uint64_t b) { return ceil_div(a, b) * b; }

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

}  // namespace ffops
