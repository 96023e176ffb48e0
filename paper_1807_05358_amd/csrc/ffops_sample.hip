// The choice of a word from its logits.
#include "ffops_device.h"
#include "ffops_sample_bins.h"

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

// A block takes a row.  It reads it twice: once for what decides which words matter, once for these few words, which are put in order and gone through with exact sums.
//   With top_k up to FIRST_MOST, or min_p from FIRST_LEAST on and no top_p, the first reading looks for maxima alone: at least top_k words are as large as the largest of that many threads' shares, and everything from there on is listed,
// a few words more than are kept.  64 rows of 32768 bfloat16, top_k 50: 11 us for 24 by weighing all words; 8 of 200003 float32 24 for 56, 256 of 131071 41 for 54; with top_k 256 21 for 28, 38 for 61 and 50 for 55, one row of 4096
// 17 for 16.  min_p 0.1, 256 rows of 131071 normal logits, deviation 4: 39 us for 49; 2.5: 44 for 49; 1, where the list does not take all of them and the row is read as follows: 95 for 73.
//   Otherwise the first reading sums weights in bins of logits: 24 instructions an element, a third of them in 64 bits, and an addition in LDS.  256 rows of 131071 float32, top_p and min_p, take 61 us (134 MB, 2.2 TB/s; the first reading
// 34 of them, the second, out of the last-level cache, 15), one row of 32768 17 us: fewer rows than compute units leave the rest idle, and two kernels that share a row between blocks take 21 us at least.
//   Bins are 1 / per_nat wide in units of the temperature, from an anchor on, the largest logit of what the block's threads read first.  A word weighs 2^29 e^r steps, r its place
// in its bin: whole numbers, whose sums do not depend on an order, to 2^-30 of the weight whatever its size, one way or the other.  Sums of bins are in 64-bit floats.  Where the anchor was too low, or words may lie beyond the lowest bin
// that weigh more than e^-42, the row is read again with other bins; words that weigh less than that beside the largest do not count.
//   The bins that decide are those in which the border of top_k, that of top_p, that of min_p and the chosen word can lie; they depend on one another, so each is a range
// until the words are there.  Bins with more than MOST words (equal logits, or nearly so) are left to select(), which reads the row for every eight bits of the key of each border.
constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int MOST = 2 * THREADS;           // words of the bins that decide
constexpr uint32_t FIRST_MOST = 256;        // top_k up to which its words are gathered first
constexpr float FIRST_LEAST = 0x1p-6f;      // min_p from which, without top_p, its words are: they are few in most rows (see above)
constexpr uint32_t NONE = 0xffffffffu;      // no word

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

// Weights in steps of 2^-78, so that their sums do not depend on an order; of single ones the upper half, in steps of 2^-39, and the rest, whose sums over 2^24 words fit 64 bits each.  (In 64 bits together a step is 2^-38 of the
// largest weight for as many words, and equal words that weigh less than half of that would count for nothing, all of them 2^-15.)
typedef unsigned __int128 Steps;
struct Halves {
    uint64_t hi, lo;                // lo with its sign, -2^38 .. 2^38
    __device__ __forceinline__ Steps sum() const { return ((Steps)hi << 39) + (Steps)(__int128)(int64_t)lo; }
};
__device__ __forceinline__ double to_double(Steps x) { return (double)(uint64_t)(x >> 64) * 0x1p64 + (double)(uint64_t)x; }
// t: at least 0, below 2^127
__device__ __forceinline__ Steps to_steps(double t)
{
    const uint64_t hi = (uint64_t)(t * 0x1p-64);
    return (Steps)hi << 64 | (uint64_t)(t - (double)hi * 0x1p64);
}
// how many times s, which is more than 0, is in x; at most 2^24 times, so that the quotient in 64 bits is off by one at most
__device__ __forceinline__ uint32_t times(Steps s, Steps x)
{
    uint32_t n = (uint32_t)(to_double(x) / to_double(s));
    if (n * s > x) --n;
    if ((n + 1) * s <= x) ++n;
    return n;
}

// what select() counts
struct Digits {
    uint64_t hi[256], lo[256];      // the halves of sums
    uint32_t count[256];
    uint32_t found;
    Steps target, above_mass;       // (one thread works with these; the others keep no registers for them)
    uint32_t above_count;
    Steps mass, mass_m;             // of the words that are kept, and of those that min_p leaves
    uint32_t kept, rank;
    __device__ __forceinline__ void add(uint32_t digit, uint32_t n, Halves s)
    {
        atomicAdd((unsigned long long*)&hi[digit], (unsigned long long)s.hi);
        atomicAdd((unsigned long long*)&lo[digit], (unsigned long long)s.lo);
        atomicAdd(&count[digit], n);
    }
    __device__ __forceinline__ Steps sum(uint32_t digit) const { return Halves{hi[digit], lo[digit]}.sum(); }
};

struct Shared {
    union {
        uint64_t steps[BINS + 2];   // a bin's sum, at its number + 1; at the ends whether something beyond the bins weighs anything; then:
        double above[BINS];         // the weight of all bins above it
    };
    uint32_t count[BINS + 2];       // words, likewise, then those of all bins above; top_k alone
    union {
        uint64_t list[MOST];        // key and number of each word of the bins that decide
        Digits digits;
    };
    uint64_t a[WAVES], b[WAVES];
    double d[WAVES];
    uint32_t c[WAVES];
    uint32_t n, word, lo, hi, again;
    double value, weight;
    uint32_t found;
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

struct Weigh {
    float most;
    double per;                     // temperature
    __device__ __forceinline__ double of(float z) const { return z == most ? 1.0 : exp(((double)z - (double)most) / per); }
    __device__ __forceinline__ Halves halves(float z) const
    {
        // whole numbers as the lower bits of floats of 2^52 and more, where a step is 1
        constexpr double ONE = 0x1p52, HALF = 0x1.8p52;
        const double w = of(z) * 0x1p39, hi = w + ONE, lo = (w - (hi - ONE)) * 0x1p39 + HALF;
        return {__builtin_bit_cast(uint64_t, hi) - __builtin_bit_cast(uint64_t, ONE), __builtin_bit_cast(uint64_t, lo) - __builtin_bit_cast(uint64_t, HALF)};
    }
    __device__ __forceinline__ Steps steps(float z) const { return halves(z).sum(); }
};

// The shortest beginning of the words' order with more than sh.target words (BY_COUNT) or steps of weight: its last word's key, the words before it with larger keys and
// their steps (sh.above_...), bit group after bit group of the keys.
template <class T, bool BY_COUNT>
__device__ __forceinline__ uint32_t select(const typename T::elem* z, uint32_t vocab, const Weigh& w, Digits& sh)
{
    uint32_t prefix = 0;
    if (threadIdx.x == 0) sh.above_mass = 0, sh.above_count = 0;
    for (int low = Key<T>::BITS - 8; low >= 0; low -= 8) {
        if (threadIdx.x < 256) sh.hi[threadIdx.x] = 0, sh.lo[threadIdx.x] = 0, sh.count[threadIdx.x] = 0;
        __syncthreads();
        for (uint32_t base = 0; base < vocab; base += THREADS) {
            const uint32_t i = base + threadIdx.x, k = i < vocab ? Key<T>::of(z[i]) : 0;
            bool in = i < vocab && !(low + 8 < Key<T>::BITS && (k >> (low + 8)) != prefix);
            const Halves s = in ? w.halves(Key<T>::value(k)) : Halves{0, 0};
            // it is equal logits that this is for: those of a wave are added at once, up to four different ones
            for (int t = 0; t < 4 && __any(in); ++t) {
                const int leader = __builtin_ctzll(__ballot(in));
                const bool same = in && k == (uint32_t)__builtin_amdgcn_readlane((int)k, leader);
                const uint32_t n = __popcll(__ballot(same));
                if ((int)(threadIdx.x % 64) == leader) sh.add(k >> low & 255, n, {n * s.hi, n * s.lo});
                in = in && !same;
            }
            if (in) sh.add(k >> low & 255, 1, s);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            Steps m = sh.above_mass;
            const Steps target = sh.target;
            uint32_t c = sh.above_count, best = 256;
            for (int d = 255; d >= 0; --d) {
                const Steps more = sh.sum(d);
                if (sh.count[d] && (BY_COUNT ? (Steps)c + sh.count[d] > target : m + more > target)) {
                    best = d;
                    break;
                }
                m += more, c += sh.count[d];
            }
            sh.found = best, sh.above_mass = m, sh.above_count = c;
        }
        __syncthreads();
        prefix = prefix << 8 | (sh.found & 255);
        __syncthreads();
    }
    return prefix;
}

// The word by reading the row again for every border; all of its threads.
template <class T>
__device__ __forceinline__ void choose_by_digits(const typename T::elem* z, uint32_t V, float most, float temperature, int32_t top_k, float top_p, float min_p, float u, Shared& sh, uint32_t& word, float& logprob)
{
    const Weigh w = {most, (double)temperature};
    Halves all = {0, 0}, all_m = {0, 0};
    uint32_t count_m = 0;
    for (uint32_t i = threadIdx.x; i < V; i += THREADS) {
        const float f = (float)z[i];
        const Halves s = w.halves(f);
        all.hi += s.hi, all.lo += s.lo;
        if (w.of(f) >= (double)min_p) all_m.hi += s.hi, all_m.lo += s.lo, ++count_m;
    }
    Digits& at = sh.digits;
    const bool one = threadIdx.x == 0;          // of the threads; the others meet it in select() and behind it
    if (threadIdx.x < 2) at.hi[threadIdx.x] = 0, at.lo[threadIdx.x] = 0, at.count[threadIdx.x] = 0;
    __syncthreads();
    at.add(0, 1, all), at.add(1, count_m, all_m);
    __syncthreads();
    if (one) at.mass = at.sum(0), at.mass_m = at.sum(1), at.kept = V, count_m = at.count[1];
    __syncthreads();
    if (top_k > 0 && (uint32_t)top_k < V) {
        if (one) at.target = (Steps)(top_k - 1);
        const uint32_t k = select<T, true>(z, V, w, at);
        if (one) at.kept = (uint32_t)top_k, at.mass = at.above_mass + (at.kept - at.above_count) * w.steps(Key<T>::value(k));
    }
    if (top_p < 1) {
        if (one) {
            const double t = ceil((double)top_p * to_double(at.mass));
            const Steps target = t < 1 ? 0 : to_steps(t) - 1;
            at.target = target < at.mass ? target : at.mass - 1;
        }
        const uint32_t k = select<T, false>(z, V, w, at);
        if (one) {
            const Steps s = w.steps(Key<T>::value(k));
            const uint32_t more = times(s, at.target - at.above_mass) + 1;
            if (at.above_count + more < at.kept) at.kept = at.above_count + more, at.mass = at.above_mass + more * s;
        }
    }
    if (one) {
        if (count_m < at.kept) {
            at.kept = count_m, at.mass = at.mass_m;
            if (!at.kept) at.kept = 1, at.mass = w.steps(most);
        }
        const Steps target = to_steps(floor((u < 0 ? 0.0 : u < 1 ? (double)u : 1.0) * to_double(at.mass)));
        at.target = target < at.mass ? target : at.mass - 1;
    }
    const uint32_t k = select<T, false>(z, V, w, at);
    const float chosen = Key<T>::value(k);
    if (one) {
        const uint32_t n = times(w.steps(chosen), at.target - at.above_mass), before = at.above_count;       // words of that key before it, and of larger ones
        at.rank = before + n < at.kept ? n : at.kept - 1 - before;
    }
    __syncthreads();
    const uint32_t rank = at.rank;
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
    word = sh.word, logprob = (float)log(w.of(chosen) / (to_double(at.mass) * 0x1p-78));
}

// sixteen bytes of a row at any element's place; -inf behind its end
template <class T>
struct Piece {
    typedef typename T::elem vec __attribute__((ext_vector_type(T::VEC), aligned(sizeof(typename T::elem))));
    vec v;
    __device__ __forceinline__ void load(const typename T::elem* z, uint32_t i, uint32_t V)
    {
        if (i + T::VEC <= V) {
            v = *(const vec*)(z + i);
            return;
        }
#pragma unroll
        for (int e = 0; e < T::VEC; ++e) v[e] = (typename T::elem)(-INFINITY);
        if (i < V) {
#pragma unroll
            for (int e = 0; e < T::VEC; ++e)
                if (i + e < V) v[e] = z[i + e];
        }
    }
};

constexpr int GROUP = 2;        // pieces that a thread works between loads; two more groups are on their way (one piece between loads: 256 rows of 131071 69 us, two: 61)

// a thread's first pieces, and all of a row's elements: each calls f(element, its number), a thread's in the order of their numbers
template <class T>
struct Row {
    static constexpr uint32_t STEP = THREADS * T::VEC;
    const typename T::elem* z;
    uint32_t V;
    Piece<T> first[2 * GROUP];
    __device__ __forceinline__ Row(const typename T::elem* z_, uint32_t V_) : z(z_), V(V_)
    {
#pragma unroll
        for (int k = 0; k < 2 * GROUP; ++k) first[k].load(z, threadIdx.x * T::VEC + k * STEP, V);
    }
    // f(piece, number of its first element)
    template <class F>
    __device__ __forceinline__ void each_piece(F f) const
    {
        Piece<T> now[2 * GROUP];
#pragma unroll
        for (int k = 0; k < 2 * GROUP; ++k) now[k] = first[k];
        uint32_t i = threadIdx.x * T::VEC;
        for (uint32_t base = 0; base < V; base += GROUP * STEP) {
            Piece<T> later[GROUP];
#pragma unroll
            for (int k = 0; k < GROUP; ++k) later[k].load(z, i + (2 * GROUP + k) * STEP, V);
#pragma unroll
            for (int k = 0; k < GROUP; ++k)
                if (i + k * STEP < V) f(now[k], i + k * STEP);
#pragma unroll
            for (int k = 0; k < GROUP; ++k) now[k] = now[GROUP + k], now[GROUP + k] = later[k];
            i += GROUP * STEP;
        }
    }
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        each_piece([&](const Piece<T>& p, uint32_t i) {
#pragma unroll
            for (int e = 0; e < T::VEC; ++e) f((float)p.v[e], i + e);
        });
    }
    // f of all elements for which near() holds, which are `lowest` or more: most pieces have none
    template <class N, class F>
    __device__ __forceinline__ void each_near(float lowest, N near, F f) const
    {
        each_piece([&](const Piece<T>& p, uint32_t i) {
            float top = (float)p.v[0];
#pragma unroll
            for (int e = 1; e < T::VEC; ++e) top = fmaxf(top, (float)p.v[e]);
            if (!(top >= lowest)) return;
            bool any = false;
#pragma unroll
            for (int e = 0; e < T::VEC; ++e) any |= near((float)p.v[e]);
            if (!any) return;
#pragma unroll
            for (int e = 0; e < T::VEC; ++e)
                if (near((float)p.v[e])) f((float)p.v[e], i + e);
        });
    }
    __device__ __forceinline__ float largest_of_first() const
    {
        float most = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2 * GROUP; ++k)
#pragma unroll
            for (int e = 0; e < T::VEC; ++e) most = fmaxf(most, (float)first[k].v[e]);
        return most;
    }
};

__device__ __forceinline__ void add_lds(uint64_t* p, uint64_t x) { __hip_atomic_fetch_add(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void add_lds(uint32_t* p, uint32_t x) { __hip_atomic_fetch_add(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

__device__ __forceinline__ uint64_t read_lane(uint64_t x, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}

// x of the lane that a data-parallel primitive names, 0 where there is none: CTRL as the instruction has it, ROWS the rows of 16 lanes that take part
template <int CTRL, int ROWS, class V>
__device__ __forceinline__ V moved(V x)
{
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
    } else {
        const uint64_t b = __builtin_bit_cast(uint64_t, x);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
        return __builtin_bit_cast(V, (uint64_t)hi << 32 | lo);
    }
}

// the sum of x over this lane and those before it: in rows of 16 lanes, then their last lanes' sums to the next row, and to the next two (a shuffle through LDS takes as long as three such steps)
template <class V>
__device__ __forceinline__ V wave_scan(V x)
{
    x += moved<0x111, 0xf>(x);
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);
    x += moved<0x143, 0xc>(x);
    return x;
}

// the largest of a wave, in its last lane
__device__ __forceinline__ uint32_t wave_most(uint32_t x)
{
    x = max(x, moved<0x111, 0xf>(x));
    x = max(x, moved<0x112, 0xf>(x));
    x = max(x, moved<0x114, 0xf>(x));
    x = max(x, moved<0x118, 0xf>(x));
    x = max(x, moved<0x142, 0xa>(x));
    x = max(x, moved<0x143, 0xc>(x));
    return x;
}

// the largest of what threads have and the least of it, of finite ones and infinity
struct Ends {
    float top, least;
};
__device__ __forceinline__ Ends block_ends(float mine, Shared& sh)
{
    const uint32_t key = Key<F32>::of(mine), top_of = wave_most(key), least_of = wave_most(mine > -INFINITY ? ~key : 0);
    __syncthreads();
    if (threadIdx.x % 64 == 63) sh.c[threadIdx.x / 64] = top_of, sh.a[threadIdx.x / 64] = least_of;
    __syncthreads();
    uint32_t top = 0, least = 0;
    for (int w = 0; w < WAVES; ++w) top = max(top, sh.c[w]), least = max(least, (uint32_t)sh.a[w]);
    return {Key<F32>::value(top), Key<F32>::value(~least)};
}

// sums of x over the threads before this one, and over all of them
template <class V>
__device__ __forceinline__ V block_before(V x, V* at, V& all)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const V s = wave_scan(x), own = moved<0x138, 0xf>(s);       // the lane before
    __syncthreads();
    if (lane == 63) at[wave] = s;
    __syncthreads();
    V before = 0;
    all = 0;
    for (int w = 0; w < WAVES; ++w) {
        if (w == wave) before = all;
        all += at[w];
    }
    return before + own;
}

// The bins whose weights a sum from `lo` to `hi` can end in: above[bin] <= sum < above[bin - 1], the lowest one for more than all.  All threads; sh.above is there.
struct Range {
    int lo, hi;
};
__device__ Range bins_of(double lo, double hi, double all, Shared& sh)
{
    __syncthreads();
#pragma unroll
    for (int k = 0; k < BINS / THREADS; ++k) {
        const int b = threadIdx.x + k * THREADS;
        const double from = sh.above[b], to = b ? sh.above[b - 1] : INFINITY;
        if (from <= lo && lo < to) sh.hi = b;
        if (from <= hi && hi < to) sh.lo = b;
    }
    __syncthreads();
    return {(int)sh.lo, (int)sh.hi};
}

constexpr double SLACK = 1e-8;      // of sums: what roundings, and words that do not count, can move them

enum { UNDECIDED, DECIDED, WITHOUT };        // WITHOUT: a row without a word

struct Choice {
    float temperature, top_p, min_p, u;
    uint32_t top_k;                 // 0: all words
    __device__ __forceinline__ Choice(const SampleArgs& a, uint32_t row)
    {
        temperature = a.temperatures ? a.temperatures[row] : a.temperature, top_p = a.top_ps ? a.top_ps[row] : a.top_p, u = a.u[row];
        min_p = a.min_ps ? a.min_ps[row] : a.min_p;
        const int32_t k = a.top_ks ? a.top_ks[row] : a.top_k;
        top_k = k > 0 && (uint32_t)k < a.vocab ? (uint32_t)k : 0;
    }
    // temperature 0, or a min_p that no word weighs: the first weighs 1, as do others that are as large, which are not kept then
    __device__ __forceinline__ bool first_alone() const { return temperature == 0 || min_p > 1; }
    __device__ __forceinline__ bool fine() const { return temperature >= 0 && temperature < INFINITY && top_p == top_p && min_p == min_p && u == u; }
};

// The words that top_k leaves, and some behind them, in the list, from the first one on: those from a logit on that top_k threads or more have.  Nothing is weighed that is not kept.  UNDECIDED: they are
// more than the list takes, or too large.
template <class T>
__device__ __forceinline__ int gather_top(const Row<T>& src, const Choice& c, Shared& sh, Ends& ends, uint32_t& n)
{
    const uint32_t tid = threadIdx.x;
    for (int b = tid; b < BINS; b += THREADS) sh.count[b] = 0;
    if (tid == 0) sh.again = 0, sh.found = NONE, sh.n = 0;
    float mine = -INFINITY;
    bool nan = false;
    src.each([&](float x, uint32_t) { mine = fmaxf(mine, x), nan |= x != x; });
    const bool any = mine > -INFINITY;
    const uint32_t key = Key<F32>::of(mine);
    ends = block_ends(mine, sh);
    if (__any(nan) && tid % 64 == 0) sh.again = 1;
    const float most = ends.top, lo = ends.least, scale = (BINS - 1) / (most - lo);     // of a single value infinite, and places are not numbers: 0
    const bool by_k = c.top_k && c.top_k <= FIRST_MOST;
    const int place = any ? min(max((int)((mine - lo) * scale), 0), BINS - 1) : -1;
    if (by_k && place >= 0) add_lds(&sh.count[place], 1u);
    __syncthreads();
    if (sh.again || most == -INFINITY) return WITHOUT;
    if (most == INFINITY) return UNDECIDED;
    float from = Key<F32>::value(1 + Key<F32>::of(-INFINITY));
    if (by_k) {
        constexpr int EACH = BINS / THREADS;
        uint32_t each[EACH], sum = 0, all;
#pragma unroll
        for (int k = 0; k < EACH; ++k) each[k] = sh.count[BINS - 1 - (tid * EACH + k)], sum += each[k];
        uint32_t before = block_before(sum, sh.c, all);
        if (before < c.top_k && c.top_k <= before + sum) {
            int k = 0;
            while (before + each[k] < c.top_k) before += each[k++];
            sh.lo = BINS - 1 - (tid * EACH + k);
        }
        __syncthreads();
        // from here on are top_k words or more, or all that weigh anything
        if (all >= c.top_k && place == (int)sh.lo) atomicMin(&sh.found, key);
        __syncthreads();
        if (all >= c.top_k) from = Key<F32>::value(sh.found);
    }
    if (c.top_p >= 1 && c.min_p > 0) {
        // on the safe side of it, by a float's rounding, and by those of weights, which are up to 1e-14 of a temperature away
        const double edge = (double)most + (double)c.temperature * log((double)c.min_p);
        from = fmaxf(from, (float)(edge - (fabs(edge) * 1e-6 + c.temperature * 1e-9 + 1e-30)));
    }
    if (tid == 0) sh.above[0] = 0, sh.count[0] = 0;         // the list is one bin, with nothing above it
    bool full = false;
    src.each_near(from, [&](float x) { return x >= from && !full; }, [&](float x, uint32_t i) {
        const uint32_t at = atomicAdd(&sh.n, 1u);
        if (at < MOST) sh.list[at] = (uint64_t)Key<F32>::of(x) << 32 | (0xffffffffu - i);
        else full = true;
    });
    __syncthreads();
    n = sh.n;
    return n <= MOST ? DECIDED : UNDECIDED;
}

// The list in order, the largest first; all threads, which have agreed on it.  Up to 256 words: a word's place is the number of larger ones, counted by 4, 8 or 16 threads together (128 words 1 us); more: by
// exchanges of pairs (128 words took 4 us so, 512 take 7).
__device__ __forceinline__ void sort_list(Shared& sh, uint32_t n)
{
    const uint32_t tid = threadIdx.x;
    if (n <= 256) {
        const uint32_t log = n <= 64 ? 4 : n <= 128 ? 3 : 2, i = tid >> log, each = 1u << log;
        const uint64_t x = i < n ? sh.list[i] : 0;
        uint32_t place = 0;
        if (i < n)
            for (uint32_t j = tid & (each - 1); j < n; j += each) place += sh.list[j] > x;
        place += __builtin_amdgcn_update_dpp(0, place, 0xb1, 0xf, 0xf, false);
        place += __builtin_amdgcn_update_dpp(0, place, 0x4e, 0xf, 0xf, false);
        if (log >= 3) place += __builtin_amdgcn_update_dpp(0, place, 0x141, 0xf, 0xf, false);
        if (log >= 4) place += __builtin_amdgcn_update_dpp(0, place, 0x140, 0xf, 0xf, false);
        __syncthreads();
        if (i < n && !(tid & (each - 1))) sh.list[place] = x;
        __syncthreads();
        return;
    }
    uint32_t size = 512;
    while (size < n) size *= 2;
    for (uint32_t i = n + tid; i < size; i += THREADS) sh.list[i] = 0;
    __syncthreads();
    for (uint32_t k = 2; k <= size; k *= 2)
        for (int log = 30 - __builtin_clz(k); log >= 0; --log) {
            if (tid < size / 2) {
                const uint32_t j = 1u << log, i = (tid >> log << (log + 1)) | (tid & (j - 1));
                const uint64_t x = sh.list[i], y = sh.list[i + j];
                if ((x < y) == ((i & k) == 0)) sh.list[i] = y, sh.list[i + j] = x;
            }
            __syncthreads();
        }
}

// The word from bins, or of the first top_k.  most: the largest logit.
template <class T>
__device__ __forceinline__ int choose_by_bins(const Row<T>& src, const Choice& c, Shared& sh, float& most, uint32_t& word, float& logprob)
{
    const uint32_t tid = threadIdx.x;
    const int lane = tid % 64, wave = tid / 64;
    word = NONE;
    uint32_t n = 0;
    Ends ends = {-INFINITY, -INFINITY};         // of all of the row, if top_k or min_p had it looked over
    const int top = (c.top_k && c.top_k <= FIRST_MOST) || (c.top_p >= 1 && c.min_p >= FIRST_LEAST) ? gather_top(src, c, sh, ends, n) : UNDECIDED;
    if (top == WITHOUT) return WITHOUT;
    most = ends.top;
    const bool whole = top == DECIDED;          // the list has everything from the first word on
    Bins bins;
    double all = 0, m_lo = 0;
    bool need_k = c.top_k && n >= c.top_k;
    Range p_bins = {c.top_p < 1 ? 0 : BINS, BINS - 1}, m_bins = {c.min_p > 0 ? 0 : BINS, BINS - 1}, u_bins = {0, BINS - 1};
    const double share = c.u < 0 ? 0.0 : c.u < 1 ? (double)c.u : 1.0;
    if (!whole) {
        if (!(most > -INFINITY)) ends = block_ends(src.largest_of_first(), sh), most = ends.top;
        int per_nat = bins_per_nat((ends.top - ends.least) / c.temperature);
        __syncthreads();
        for (;;) {
            if (!(most > -INFINITY && most < INFINITY)) {       // no anchor: the largest of all, which may be infinite, or a row without one
                most = -INFINITY;
                uint32_t nan = 0;
                src.each([&](float x, uint32_t) { most = fmaxf(most, x), nan |= x != x; });
                most = Key<F32>::value((uint32_t)block_max(Key<F32>::of(most), sh.a));
                nan = block_sum(nan, sh.c);
                if (nan || most == -INFINITY) {
                    return WITHOUT;
                }
                if (most == INFINITY) return UNDECIDED;
            }
            bins.set(most, c.temperature, per_nat);
            for (int b = tid; b < BINS + 2; b += THREADS) sh.steps[b] = 0;
            if (c.top_k)
                for (int b = tid; b < BINS + 2; b += THREADS) sh.count[b] = 0;
            if (tid == 0) sh.again = 0;
            __syncthreads();
            most = -INFINITY;
            bool nan = false;
            const double light = BELOW + 1 - 42.0 * per_nat;        // places from there on weigh something
            // (words beyond the lowest bin, many of them -inf at times, are kept off the one place in LDS that they would all add to)
            const auto add = [&](float x) {
                most = fmaxf(most, x);
                nan |= x != x;
                const double at = bins.place(x);
                const int slot = bins.slot(at);
                if (slot > 0) add_lds(&sh.steps[slot], (uint64_t)bins.steps((float)__builtin_amdgcn_fract(at)));
                else if (at > light) sh.steps[0] = 1;
                return slot;
            };
            if (c.top_k) src.each([&](float x, uint32_t) {
                const int slot = add(x);
                if (slot > 0) add_lds(&sh.count[slot], 1u);
            });
            else src.each([&](float x, uint32_t) { add(x); });
            if (__any(nan) && tid % 64 == 0) sh.again = 1;
            most = Key<F32>::value((uint32_t)block_max(Key<F32>::of(most), sh.a));
            const bool above = sh.steps[BINS + 1] != 0, below = sh.steps[0] != 0 && per_nat > 64, again = sh.again != 0;
            __syncthreads();
            if (again) {
                return WITHOUT;
            }
            if (!above && !below) break;
            if (!above) per_nat = 64;           // with that what is beyond the lowest bin weighs less than e^-44, and with the largest logit as the anchor nothing is above the highest
        }
        // weights of all bins above each, beside the largest word's, which is 1: a wave has 256 bins, four times 64 side by side, the first wave the highest
        constexpr int EACH = BINS / THREADS;
        const int highest = BINS - 1 - wave * (64 * EACH) - lane;
        uint32_t words_all = 0;
        {
            uint64_t steps[EACH];
            uint32_t n[EACH] = {}, t[EACH] = {}, words_before = 0, row_words = 0;
            double s[EACH] = {}, before = 0, rows = 0;
#pragma unroll
            for (int k = 0; k < EACH; ++k) steps[k] = sh.steps[highest - 64 * k + 1];
            if (__any((steps[0] | steps[1] | steps[2] | steps[3]) != 0)) {          // most waves have empty bins
                static_assert(EACH == 4, "as many rows");
                // e^-h, h at most 1/32, and that for 64 bins
                const double h = 1.0 / per_nat;
                double less = 1 - h * (1 - h / 2 * (1 - h / 3 * (1 - h / 4 * (1 - h / 5 * (1 - h / 6 * (1 - h / 7))))));
#pragma unroll
                for (int k = 0; k < 6; ++k) less *= less;
                double edge = 0x1p-29 * exp(((double)(highest - BELOW) + (bins.anchor - (double)most) * bins.per_logit) * h);
                // sums of a row of 64, up to and with the lane, then of the rows before it, then of the waves before
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    s[k] = wave_scan((double)steps[k] * edge);
                    if (c.top_k) n[k] = sh.count[highest - 64 * k + 1], t[k] = wave_scan(n[k]);
                    edge *= less;
                }
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    const double of_row = __builtin_bit_cast(double, read_lane(__builtin_bit_cast(uint64_t, s[k]), 63));
                    s[k] = moved<0x138, 0xf>(s[k]) + rows, rows += of_row;
                    if (c.top_k) {
                        const uint32_t words = (uint32_t)__builtin_amdgcn_readlane((int)t[k], 63);
                        t[k] = moved<0x138, 0xf>(t[k]) + row_words, row_words += words;
                    }
                }
            }
            if (lane == 0) sh.d[wave] = rows, sh.c[wave] = row_words;
            __syncthreads();
            for (int x = 0; x < WAVES; ++x) {
                if (x == wave) before = all, words_before = words_all;
                all += sh.d[x], words_all += sh.c[x];
            }
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int b = highest - 64 * k;
                sh.above[b] = s[k] + before;
                const uint32_t words = t[k] + words_before;
                if (c.top_k) sh.count[b] = words;
                if (words < c.top_k && c.top_k <= words + n[k]) sh.found = b;
            }
            __syncthreads();
        }
        const auto below = [&](int b) { return b ? sh.above[b - 1] : all; };        // the weight down to the end of bin b
        // what each border leaves, from..to, and the bins it can lie in
        const bool by_k = c.top_k && words_all >= c.top_k;      // otherwise words without weight make up the rest
        double k_lo = all, k_hi = all;
        const int k_bin = by_k ? (int)sh.found : -1;
        if (by_k) k_lo = sh.above[k_bin], k_hi = below(k_bin);
        p_bins = {1, 0}, m_bins = {1, 0};
        double p_lo = k_lo, p_hi = k_hi;
        if (c.top_p < 1) {
            const double p = c.top_p > 0 ? (double)c.top_p : 0.0;
            p_bins = bins_of(p * k_lo * (1 - SLACK), p * k_hi * (1 + SLACK), all, sh);
            p_lo = sh.above[p_bins.hi], p_hi = below(p_bins.lo);
        }
        m_lo = all;
        double m_hi = all;
        if (c.min_p > 0) {
            const double at = fmax(log((double)c.min_p) * per_nat + bins.place(most), 1.0);
            m_bins = {min((int)fmax(at - 1e-6, 1.0), BINS) - 1, min((int)(at + 1e-6), BINS) - 1};
            m_lo = sh.above[m_bins.hi], m_hi = below(m_bins.lo);
        }
        const double lo = fmin(fmin(k_lo, p_lo), m_lo), hi = fmin(fmin(k_hi, p_hi), m_hi);
        // borders that others come before do not count
        if (m_lo > hi * (1 + SLACK)) m_bins = {1, 0};
        const bool no_p = p_lo > hi * (1 + SLACK);
        if (no_p) p_bins = {1, 0};
        need_k = by_k && !(no_p && k_lo > hi * (1 + SLACK));
        u_bins = bins_of(share * lo * (1 - SLACK), fmin(share, 1 - 1e-14) * hi * (1 + SLACK), all, sh);
        const auto decides = [&](int b) { return (need_k && b == k_bin) || (b >= p_bins.lo && b <= p_bins.hi) || (b >= m_bins.lo && b <= m_bins.hi) || (b >= u_bins.lo && b <= u_bins.hi); };
        // their words
        if (tid == 0) sh.n = 0;
        __syncthreads();
        {
            // between these logits are all words of the bins: a piece seldom has one
            int b_lo = BINS, b_hi = -2;
            if (p_bins.lo <= p_bins.hi) b_lo = p_bins.lo, b_hi = p_bins.hi;
            if (m_bins.lo <= m_bins.hi) b_lo = min(b_lo, m_bins.lo), b_hi = max(b_hi, m_bins.hi);
            const int k_at = need_k ? k_bin : u_bins.lo;
            const float b_from = b_hi < 0 ? INFINITY : bins.logit(b_lo, -1), to = b_hi < 0 ? -INFINITY : bins.logit(b_hi + 1, 1), u_from = bins.logit(u_bins.lo, -1), u_to = bins.logit(u_bins.hi + 1, 1), k_from = bins.logit(k_at, -1), k_to = bins.logit(k_at + 1, 1);
            const float lowest = fminf(fminf(b_from, u_from), k_from);
            const auto near = [&](float x) { return ((x >= b_from) & (x <= to)) | ((x >= u_from) & (x <= u_to)) | ((x >= k_from) & (x <= k_to)); };
            src.each_near(lowest, near, [&](float x, uint32_t i) {
                const int b = bins.bin(bins.place(x));
                if (b >= 0 && b < BINS && decides(b)) {
                    const uint32_t n = atomicAdd(&sh.n, 1u);
                    if (n < MOST) sh.list[n] = (uint64_t)Key<F32>::of(x) << 32 | (0xffffffffu - i);
                }
            });
        }
        __syncthreads();
        n = sh.n;
    }
    const Weigh weigh = {most, (double)c.temperature};
    const auto bin_of = [&](float x) { return whole ? 0 : bins.bin(bins.place(x)); };
    if (n <= MOST) sort_list(sh, n);
    if (n <= 64) {
        // one wave, a word a lane
        if (tid < 64) {
            const bool in = lane < (int)n;
            const uint64_t x = in ? sh.list[lane] : 0;
            const float f = Key<F32>::value((uint32_t)(x >> 32));
            const double w = in ? weigh.of(f) : 0;
            const int bin = in ? bin_of(f) : -1;
            const double sum = wave_scan(w);
            if (whole) all = __builtin_bit_cast(double, read_lane(__builtin_bit_cast(uint64_t, sum), 63));
            // the first word of the lane's bin in the list
            const int prev = __shfl_up(bin, 1);
            const uint64_t heads = __ballot(in && (lane == 0 || prev != bin)) & ~0ull >> (63 - lane);
            const int head = heads ? 63 - __builtin_clzll(heads) : 0;
            const double before = (in ? sh.above[bin] : 0) + (sum - w) - __shfl(sum - w, head), to = before + w;
            double left = all;
            bool found = true;
            if (need_k) {
                const uint64_t at = __ballot(in && sh.count[in ? bin : 0] + lane - head == c.top_k - 1);
                found = at != 0;
                left = __shfl(to, at ? __builtin_ctzll(at) : 0);
            }
            if (p_bins.lo <= p_bins.hi) {
                const double target = c.top_p > 0 ? (double)c.top_p * left : 0.0;
                const uint64_t at = __ballot(in && bin >= p_bins.lo && bin <= p_bins.hi && (before < target || before == 0) && !(to < target));
                found = found && at != 0;
                left = fmin(left, __shfl(to, at ? __builtin_ctzll(at) : 0));
            }
            if (m_bins.lo <= m_bins.hi) {
                double m = in && bin >= m_bins.lo && bin <= m_bins.hi && w >= (double)c.min_p ? to : 0;
#pragma unroll
                for (int d = 32; d; d >>= 1) m = fmax(m, __shfl_xor(m, d));
                left = fmin(left, fmax(m, m_lo));
            }
            const double target = fmin(share, 1 - 1e-14) * left;
            const uint64_t at = __ballot(in && bin >= u_bins.lo && bin <= u_bins.hi && before <= target && target < to);
            if (lane == 0) sh.word = NONE;
            if (found && at && lane == (int)__builtin_ctzll(at)) {
                sh.word = 0xffffffffu - (uint32_t)x;
                sh.weight = log(w / left);
            }
        }
        __syncthreads();
        word = sh.word, logprob = (float)sh.weight;
    } else if (n <= MOST) {
        // a thread has two neighbours: their weights, the weight before them, their rank
        double w[2], before[2];
        int bin[2];
        uint32_t rank[2];
        bool in[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t i = 2 * tid + e;
            in[e] = i < n;
            const float x = in[e] ? Key<F32>::value((uint32_t)(sh.list[i] >> 32)) : 0;
            bin[e] = in[e] ? bin_of(x) : -1;
            w[e] = in[e] ? weigh.of(x) : 0;
        }
        double sum_all;
        const double sum = block_before(w[0] + w[1], sh.d, sum_all);
        if (whole) all = sum_all;
        // where each bin's words begin in the list, and the sum there: steps of other bins are not needed any more, but their sums above are
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t i = 2 * tid + e;
            before[e] = sum + (e ? w[0] : 0.0);
            if (!in[e]) continue;
            const float prev = i ? Key<F32>::value((uint32_t)(sh.list[i - 1] >> 32)) : 0;
            if (i == 0 || bin_of(prev) != bin[e]) {     // one thread for each bin
                sh.above[bin[e]] -= before[e];
                sh.count[bin[e]] -= i;
            }
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (in[e]) before[e] += sh.above[bin[e]], rank[e] = sh.count[bin[e]] + 2 * tid + e;
        // the borders, exactly
        double left = all;
        if (need_k) {
            if (tid == 0) sh.value = -1;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (in[e] && rank[e] == c.top_k - 1) sh.value = before[e] + w[e];
            __syncthreads();
            left = sh.value;
        }
        if (p_bins.lo <= p_bins.hi) {
            const double target = c.top_p > 0 ? (double)c.top_p * left : 0.0;
            __syncthreads();
            if (tid == 0) sh.value = -1;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (in[e] && bin[e] >= p_bins.lo && bin[e] <= p_bins.hi && (before[e] < target || before[e] == 0) && !(before[e] + w[e] < target)) sh.value = before[e] + w[e];
            __syncthreads();
            left = fmin(left, sh.value);        // below 0: between two bins, by roundings; no word is found then
        }
        if (m_bins.lo <= m_bins.hi) {
            // the words before the bins, and those of them that weigh enough
            double m = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (in[e] && bin[e] >= m_bins.lo && bin[e] <= m_bins.hi && w[e] >= (double)c.min_p) m = fmax(m, before[e] + w[e]);
            m = __builtin_bit_cast(double, block_max(__builtin_bit_cast(uint64_t, m), sh.a));
            left = fmin(left, fmax(m, m_lo));
        }
        const double target = fmin(share, 1 - 1e-14) * left;
        __syncthreads();
        if (tid == 0) sh.word = NONE;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (left >= 0 && in[e] && bin[e] >= u_bins.lo && bin[e] <= u_bins.hi && before[e] <= target && target < before[e] + w[e]) sh.word = 0xffffffffu - (uint32_t)sh.list[2 * tid + e], sh.weight = w[e];
        __syncthreads();
        word = sh.word;
        if (word != NONE) logprob = (float)log(sh.weight / left);
    }
    return word == NONE ? UNDECIDED : DECIDED;
}

// the whole row, by one block
template <class T>
__device__ __forceinline__ void choose_from_row(const SampleArgs& a, uint32_t row, const Choice& c, Shared& sh)
{
    const typename T::elem* z = (const typename T::elem*)(a.logits + row * a.stride);
    const Row<T> src(z, a.vocab);
    float most = -INFINITY, logprob = NAN;
    uint32_t word;
    const int state = choose_by_bins(src, c, sh, most, word, logprob);
    if (state == UNDECIDED) {
        __syncthreads();
        choose_by_digits<T>(z, a.vocab, most, c.temperature, (int32_t)c.top_k, c.top_p, c.min_p, c.u, sh, word, logprob);
    }
    if (threadIdx.x == 0) a.words[row] = state == WITHOUT ? -1 : (int32_t)word, a.logprob[row] = state == WITHOUT ? NAN : logprob;
}

// the largest key, of these the lowest number; 0 where there is a NaN
template <class T>
__device__ __forceinline__ uint64_t first_word(const Row<T>& src, Shared& sh)
{
    uint64_t first = 0;
    uint32_t nan = 0;
    src.each([&](float x, uint32_t i) {
        nan |= x != x;
        const uint64_t k = (uint64_t)Key<F32>::of(x) << 32 | (0xffffffffu - i);
        first = k > first ? k : first;
    });
    first = block_max(first, sh.a);
    return block_sum(nan, sh.c) ? 0 : first;
}
__device__ __forceinline__ void put_first(const SampleArgs& a, uint32_t row, uint64_t first)
{
    const bool any = first && Key<F32>::value((uint32_t)(first >> 32)) > -INFINITY;
    if (threadIdx.x == 0) a.words[row] = any ? (int32_t)(0xffffffffu - (uint32_t)first) : -1, a.logprob[row] = any ? 0.0f : NAN;
}

template <class T>
__global__ __launch_bounds__(THREADS) void k_sample(SampleArgs a)
{
    __shared__ Shared sh;
    const uint32_t row = blockIdx.x;
    const Choice c(a, row);
    if (!c.fine()) put_first(a, row, 0);
    else if (c.first_alone()) put_first(a, row, first_word(Row<T>((const typename T::elem*)(a.logits + row * a.stride), a.vocab), sh));
    else choose_from_row<T>(a, row, c, sh);
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
