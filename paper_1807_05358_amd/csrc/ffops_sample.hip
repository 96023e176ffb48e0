// The choice of a word from its logits.
#include "ffops_device.h"

namespace ffops {
namespace {

struct SampleArgs {
    uint32_t rows, vocab;
    const char* logits;
    int64_t stride;                 // bytes
    const float *u, *temperatures, *top_ps, *min_ps;
    const int32_t* top_ks;
    float temperature, top_p, min_p;
    int32_t top_k;
    int32_t* words;
    float* logprob;
};

constexpr int THREADS = 1024, WAVES = THREADS / 64;

// Logits as whole numbers in the same order, -0 as 0.
template <class T>
struct Key;
template <>
struct Key<F32> {
    static constexpr int BITS = 32;
    static __device__ __forceinline__ uint32_t of(float z)
    {
        const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.0f);
        return b >> 31 ? ~b : b | 0x80000000u;
    }
    static __device__ __forceinline__ float value(uint32_t k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k); }
};
template <class T>
struct Key16 {
    static constexpr int BITS = 16;
    static __device__ __forceinline__ uint32_t of(typename T::elem z)
    {
        uint32_t b = __builtin_bit_cast(uint16_t, z);
        if (b == 0x8000) b = 0;
        return b >> 15 ? ~b & 0xffff : b | 0x8000;
    }
    static __device__ __forceinline__ float value(uint32_t k) { return (float)__builtin_bit_cast(typename T::elem, (uint16_t)(k >> 15 ? k & 0x7fff : ~k)); }
};
template <>
struct Key<F16> : Key16<F16> {};
template <>
struct Key<BF16> : Key16<BF16> {};

struct Shared {
    uint64_t mass[256];
    uint32_t count[256];
    uint64_t a[WAVES], b[WAVES];
    uint32_t c[WAVES];
    uint32_t found, word;
    uint64_t above_mass;
    uint32_t above_count;
};

template <class V>
__device__ __forceinline__ V block_sum(V x, V* at)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = x;
    __syncthreads();
    V s = 0;
    for (int w = 0; w < WAVES; ++w) s += at[w];
    return s;
}
__device__ __forceinline__ uint64_t block_max(uint64_t x, uint64_t* at)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const uint64_t y = __shfl_xor(x, d);
        x = y > x ? y : x;
    }
    __syncthreads();
    if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = x;
    __syncthreads();
    x = at[0];
    for (int w = 1; w < WAVES; ++w) x = at[w] > x ? at[w] : x;
    return x;
}

// Weights as whole numbers of steps of 2^-shift, so that their sums do not depend on an order.
struct Weigh {
    float most;
    double per;                     // 1 / temperature
    double unit;                    // 2^shift
    __device__ __forceinline__ double of(float z) const { return z == most ? 1.0 : exp(((double)z - (double)most) / per); }
    __device__ __forceinline__ uint64_t steps(float z) const { return (uint64_t)rint(of(z) * unit); }
};

// The shortest beginning of the words' order with more than `target` words (BY_COUNT) or steps of weight: its last word's key, the words before it with larger keys and
// their steps (sh.above_...), bit group after bit group of the keys.
template <class T, bool BY_COUNT>
__device__ uint32_t select(const typename T::elem* z, uint32_t vocab, const Weigh& w, uint64_t target, Shared& sh, uint64_t& above_mass, uint32_t& above_count)
{
    uint32_t prefix = 0;
    above_mass = 0, above_count = 0;
    for (int low = Key<T>::BITS - 8; low >= 0; low -= 8) {
        if (threadIdx.x < 256) sh.mass[threadIdx.x] = 0, sh.count[threadIdx.x] = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < vocab; i += THREADS) {
            const uint32_t k = Key<T>::of(z[i]);
            if (low + 8 < Key<T>::BITS && (k >> (low + 8)) != prefix) continue;
            atomicAdd((unsigned long long*)&sh.mass[k >> low & 255], (unsigned long long)w.steps(Key<T>::value(k)));
            atomicAdd(&sh.count[k >> low & 255], 1u);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint64_t m = above_mass;
            uint32_t c = above_count, best = 256;
            for (int d = 255; d >= 0; --d) {
                if (sh.count[d] && (BY_COUNT ? c + (uint64_t)sh.count[d] > target : m + sh.mass[d] > target)) {
                    best = d;
                    break;
                }
                m += sh.mass[d], c += sh.count[d];
            }
            sh.found = best, sh.above_mass = m, sh.above_count = c;
        }
        __syncthreads();
        above_mass = sh.above_mass, above_count = sh.above_count;
        prefix = prefix << 8 | (sh.found & 255);
        __syncthreads();
    }
    return prefix;
}

// A block takes a row and reads it from the cache again for every step.
template <class T>
__global__ __launch_bounds__(THREADS) void k_sample(SampleArgs a)
{
    __shared__ Shared sh;
    const uint32_t row = blockIdx.x, V = a.vocab;
    const typename T::elem* z = (const typename T::elem*)(a.logits + row * a.stride);
    const float temperature = a.temperatures ? a.temperatures[row] : a.temperature, top_p = a.top_ps ? a.top_ps[row] : a.top_p, min_p = a.min_ps ? a.min_ps[row] : a.min_p, u = a.u[row];
    const int32_t top_k = a.top_ks ? a.top_ks[row] : a.top_k;
    // the first word of the order: the largest key, of these the lowest number
    uint64_t first = 0;
    uint32_t nan = 0;
    for (uint32_t i = threadIdx.x; i < V; i += THREADS) {
        const uint32_t k = Key<T>::of(z[i]);
        const float f = (float)z[i];
        nan |= f != f;
        const uint64_t x = (uint64_t)k << 32 | (0xffffffffu - i);
        first = x > first ? x : first;
    }
    first = block_max(first, sh.a);
    nan = block_sum(nan, sh.c);
    const float most = Key<T>::value((uint32_t)(first >> 32));
    const bool fine = nan == 0 && most > -INFINITY && temperature >= 0 && temperature < INFINITY && top_p == top_p && min_p == min_p && u == u;
    if (!fine || temperature == 0) {
        if (threadIdx.x == 0) a.words[row] = fine ? (int32_t)(0xffffffffu - (uint32_t)first) : -1, a.logprob[row] = fine ? 0.0f : NAN;
        return;
    }
    Weigh w = {most, (double)temperature, 1.0};
    int shift = 62;
    while ((1ull << (62 - shift)) < V) --shift;
    w.unit = (double)(1ull << shift);
    uint64_t mass = 0, mass_m = 0;
    uint32_t count_m = 0;
    for (uint32_t i = threadIdx.x; i < V; i += THREADS) {
        const float f = (float)z[i];
        const uint64_t s = w.steps(f);
        mass += s;
        if (w.of(f) >= (double)min_p) mass_m += s, ++count_m;
    }
    mass = block_sum(mass, sh.a), mass_m = block_sum(mass_m, sh.b), count_m = block_sum(count_m, sh.c);
    uint32_t kept = V;
    uint64_t above;
    uint32_t before;
    if (top_k > 0 && (uint32_t)top_k < V) {
        const uint32_t k = select<T, true>(z, V, w, (uint64_t)top_k - 1, sh, above, before);
        kept = (uint32_t)top_k, mass = above + (kept - before) * w.steps(Key<T>::value(k));
    }
    if (top_p < 1) {
        const double t = ceil((double)top_p * (double)mass);
        const uint64_t target = t < 1 ? 0 : t <= (double)(mass - 1) ? (uint64_t)t - 1 : mass - 1;
        const uint32_t k = select<T, false>(z, V, w, target, sh, above, before);
        const uint64_t s = w.steps(Key<T>::value(k)), more = (target - above) / s + 1;
        if (before + more < kept) kept = before + (uint32_t)more, mass = above + more * s;
    }
    if (count_m < kept) {
        kept = count_m, mass = mass_m;
        if (!kept) kept = 1, mass = w.steps(most);
    }
    const double t = floor((double)(u < 0 ? 0 : u) * (double)mass);
    const uint64_t target = t < (double)(mass - 1) ? (uint64_t)t : mass - 1;
    const uint32_t k = select<T, false>(z, V, w, target, sh, above, before);
    const float chosen = Key<T>::value(k);
    uint64_t rank = (target - above) / w.steps(chosen);         // words of that key before it
    if (before + rank >= kept) rank = kept - 1 - before;
    uint32_t seen = 0;
    for (uint32_t base = 0; base < V; base += THREADS) {
        const uint32_t i = base + threadIdx.x;
        const bool is = i < V && Key<T>::of(z[i]) == k;
        const uint64_t votes = __ballot(is);
        __syncthreads();
        if (threadIdx.x % 64 == 0) sh.c[threadIdx.x / 64] = __popcll(votes);
        __syncthreads();
        uint32_t n = seen;
        for (uint32_t x = 0; x < threadIdx.x / 64; ++x) n += sh.c[x];
        n += __popcll(votes & ((1ull << (threadIdx.x % 64)) - 1));
        if (is && n == rank) sh.word = i;
        for (int x = 0; x < WAVES; ++x) seen += sh.c[x];
        if (seen > rank) break;
    }
    __syncthreads();
    if (threadIdx.x == 0) a.words[row] = (int32_t)sh.word, a.logprob[row] = (float)log(w.of(chosen) / ((double)mass / w.unit));
}

int check(const ff_sample_t* p)
{
    if (p->dtype > FF_BF16 || p->vocab == 0) return FF_EINVAL;
    if (p->vocab > FF_OP_MAX_WORDS || p->rows > FF_OP_MAX_CHOICES) return FF_ERANGE;
    return FF_OK;
}

}  // namespace
}  // namespace ffops

using namespace ffops;

extern "C" size_t ff_op_sample_workspace_bytes(const ff_sample_t*) { return 0; }

extern "C" int ff_op_sample(const ff_sample_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check(p)) return rc;
    if (p->rows == 0) return FF_OK;
    if (!p->logits.p || !p->u || !p->words || !p->logprob) return FF_EINVAL;
    const SampleArgs a = {p->rows, p->vocab, (const char*)p->logits.p, p->logits.stride * (p->dtype == FF_F32 ? 4 : 2), p->u, p->temperatures, p->top_ps, p->min_ps, p->top_ks,
                          p->temperature, p->top_p, p->min_p, p->top_k, p->words, p->logprob};
    const hipStream_t st = (hipStream_t)stream;
    if (p->dtype == FF_F32) k_sample<F32><<<p->rows, THREADS, 0, st>>>(a);
    else if (p->dtype == FF_F16) k_sample<F16><<<p->rows, THREADS, 0, st>>>(a);
    else k_sample<BF16><<<p->rows, THREADS, 0, st>>>(a);
    return launched();
}
