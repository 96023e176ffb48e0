// Attention of new queries over a paged cache.
#include "ffops_attention.h"
#include "ffops_cache.h"
#include "ffops_paged_runs.h"

namespace ffops {
namespace {

struct PagedArgs {
    CacheArgs c;
    uint32_t batch, heads, kv_heads, group, q_len, dim, causal, runs;
    uint32_t cols;                  // queries times heads of a group: what shares the keys of a key head
    float scale_log2, per_group;    // per_group: 1 / group
    Heads q, o;
    float* lse;
    const int32_t *q_lengths, *kv_lengths;
    float* part;                    // runs > 0: [2 * runs][kv_heads][cols][dim], see below
    float* part_lse;                // [2 * runs][kv_heads][cols]
};

// Memory bounds it: every key and value is read once, for all queries and heads that share it.  A block has four waves, a wave takes tiles of 32 positions straight
// into registers and makes s^T = k q^T and o^T += v^T p^T with 16x16x32 products, whose columns are (query, head of the group) pairs.
//   Which k an operand's place stands for does not matter as long as both operands agree, so nothing goes through LDS:
//   keys: lane l gives row l % 16 of each 16 positions, elements as 16-byte pieces l / 16, l / 16 + 4, ...; q is read in that order;
//   scores: the lane then holds positions 4 * (l / 16) + r of both 16, which is as it stands an operand of the second product;
//   values: lane l reads, for those same 8 positions, elements (D / 16) * (l % 16) .. of a row, 16 lanes a whole row, and pairs of positions are put together
//   by one byte permutation a word.
// The running maximum moves when it grows by more than 2^8 (float16: as in the contiguous forward kernel).  bfloat16 keeps probabilities as a sum of two of its numbers,
// which costs products, of which there are plenty, and leaves the output's own rounding the only one that counts.  float16 rounds them once, times 2^8, to 11 bits, as the output is:
// 4 queries over e2m1 are off by 2.8e-4 of their size so, 2.1e-4 with 24 bits, and 4-bit elements wait for vector instructions already.
//   Work is dealt in equal runs of tiles over all sequences, whatever their lengths (ffops_paged_runs.h); parts of a sequence are joined by a second kernel.
//   Measured, 32 heads on 8 of 128: 8 sequences of up to 16384 positions in bfloat16, 233 MB, 38 us, 6.1 TB/s, and 5.5 us for the join; 16 of up to 32768 in e4m3, 404 MB, 71 us, 5.7 TB/s; in 4-bit elements vector
// instructions and the start count as much: 32 sequences of up to 8191, 4 queries of 32 heads on 4, 75 MB, 28 us.
constexpr int WAVES = 4;

template <class T>
constexpr float P_SHIFT = std::is_same<T, F16>::value ? 8.0f : 0.0f;
template <class T>
constexpr float MAX_BEHIND = std::is_same<T, F16>::value ? 7.0f : 8.0f;

// the positions of sequence b that its queries look at
__device__ __forceinline__ int positions(const PagedArgs& a, uint32_t b)
{
    const int n = cached(a.kv_lengths, a.c.table_pages << a.c.page_log2, b);
    return cached(a.q_lengths, a.q_len, b) ? n : 0;
}

// Where a sequence, or a run, begins in the list of all tiles.  Up to 64 sequences: a lane has the length of each, and a wave finds it by itself; more: the block's threads take a stretch of
// sequences each.
struct Finder {
    int64_t sum[WAVES];
    uint32_t b;
    int64_t first;
};

struct List {
    bool few;
    uint32_t b0, b1;                // the thread's sequences
    int nk;                         // few: the length of the lane's sequence
    int64_t before, mine, all;      // places of the list before them, theirs, and all

    __device__ __forceinline__ void make(const PagedArgs& a, Finder& f)
    {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        few = a.batch <= 64;
        if (few) {
            b0 = lane, b1 = lane + 1;
            nk = lane < (int)a.batch ? positions(a, lane) : 0;
            int s = (int)places_of(nk);
            mine = s;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int t = __shfl_up(s, d);
                if (lane >= d) s += t;
            }
            before = s - (int)mine, all = __builtin_amdgcn_readlane(s, 63);
            return;
        }
        const uint32_t per = (a.batch + 255) / 256;
        b0 = min(a.batch, threadIdx.x * per), b1 = min(a.batch, b0 + per), nk = 0, mine = 0;
        for (uint32_t i = b0; i < b1; ++i) mine += places_of(positions(a, i));
        int64_t s = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int64_t t = __shfl_up(s, d);
            if (lane >= d) s += t;
        }
        if (lane == 63) f.sum[wave] = s;
        __syncthreads();
        before = s - mine, all = 0;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) before += f.sum[w];
            all += f.sum[w];
        }
    }
    // the sequence that holds a place of the list, and where it begins there
    __device__ __forceinline__ void sequence_at(const PagedArgs& a, int64_t place, Finder& f, uint32_t& b, int64_t& first) const
    {
        const bool here = before <= place && place < before + mine;
        if (few) {
            b = (uint32_t)__builtin_ctzll(__ballot(here));
            first = __builtin_amdgcn_readlane((int)before, b);
            return;
        }
        if (here) {
            int64_t at = before;
            for (uint32_t i = b0; i < b1; ++i) {
                const uint32_t n = places_of(positions(a, i));
                if (place < at + n) {
                    f.b = i, f.first = at;
                    break;
                }
                at += n;
            }
        }
        __syncthreads();
        b = f.b, first = f.first;
    }
    __device__ __forceinline__ int64_t begin_of(const PagedArgs& a, uint32_t b, Finder& f) const
    {
        if (few) return __builtin_amdgcn_readlane((int)before, b);
        if (b0 <= b && b < b1) {
            int64_t at = before;
            for (uint32_t i = b0; i < b; ++i) at += places_of(positions(a, i));
            f.first = at;
        }
        __syncthreads();
        return f.first;
    }
    __device__ __forceinline__ int length(const PagedArgs& a, uint32_t b) const { return few ? __builtin_amdgcn_readlane(nk, b) : positions(a, b); }
};

struct Lane {
    int lane, wave, x, g;           // x = lane % 16, g = lane / 16
};

// two 16-bit elements of the same column from two rows: the low or the high halves
__device__ __forceinline__ uint32_t low_pair(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100); }
__device__ __forceinline__ uint32_t high_pair(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302); }

// bytes of a row: FULL: the head has all D elements of the kernel's tiles
template <int HELD, int D, bool FULL>
__device__ __forceinline__ uint32_t row_bytes(const PagedArgs& a) { return FULL ? D / 8 * EIGHT<HELD> : a.c.row; }

// ---- a tile's keys ----

// operands of 32 positions: [half][step]; D elements of a row, a.dim of them real
template <class T, int HELD, int D, bool FULL>
struct Keys {
    static constexpr int LOADS = HELD == FF_HELD_SAME ? D / 32 : HELD == FF_HELD_E4M3 ? D / 64 : 1;
    static constexpr bool SHORT = HELD == FF_HELD_E2M1 && D == 64;       // 8-byte pieces
    uint4 raw[2][LOADS];
    uint32_t s[2];

    // elements of step `st`, first of eight, of lane group g
    static __device__ __forceinline__ int element(int st, int g)
    {
        if (HELD == FF_HELD_SAME) return (g + 4 * st) * 8;
        if (HELD == FF_HELD_E4M3) return (g + 4 * (st / 2)) * 16 + st % 2 * 8;
        return g * (D / 4) + st * 8;
    }
    // rows: of 16 positions from a place on, the same for all lanes, so that a lane's address is an offset
    __device__ __forceinline__ void load(const PagedArgs& a, int half, const char* rows, const uint8_t* scales, const Lane& l)
    {
        const uint32_t at = l.x * row_bytes<HELD, D, FULL>(a);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int first = element(HELD == FF_HELD_E4M3 ? 2 * i : i, l.g), place = HELD == FF_HELD_SAME ? first * 2 : HELD == FF_HELD_E4M3 ? first : first / 2;
            const char* from = rows + (at + (FULL || first < (int)a.dim ? (uint32_t)place : 0u));
            if constexpr (SHORT) {
                const uint2 w = *(const uint2*)from;
                raw[half][i] = {w.x, w.y, 0, 0};
            } else {
                raw[half][i] = *(const uint4*)from;
            }
        }
        if constexpr (HELD == FF_HELD_E4M3) s[half] = scales[(uint32_t)l.x];
        if constexpr (HELD == FF_HELD_E2M1) s[half] = scales[min((uint32_t)(l.g * (D / 4) / 32), a.c.blocks - 1) * a.c.page + l.x];
    }
    __device__ __forceinline__ typename T::vec8 operand(const PagedArgs& a, int half, int st, int g) const
    {
        uint4 v;
        if constexpr (HELD == FF_HELD_SAME) v = raw[half][st];
        else if constexpr (HELD == FF_HELD_E4M3) {
            const uint4 r = raw[half][st / 2];
            v = Eight<T, HELD>::get(st % 2 ? uint2{r.z, r.w} : uint2{r.x, r.y}, scale_operand(s[half]));
        } else {
            const uint4 r = raw[half][0];
            v = Eight<T, HELD>::get(st == 0 ? r.x : st == 1 ? r.y : st == 2 ? r.z : r.w, scale_operand(s[half]));
        }
        if (!FULL && element(st, g) >= (int)a.dim) v = {0, 0, 0, 0};
        return __builtin_bit_cast(typename T::vec8, v);
    }
};

// ---- a tile's values ----

// Elements beyond a head's are others', and make sums that are not kept.
template <class T, int HELD, int D, bool FULL>
struct Values {
    static constexpr int EACH = D / 16, WORDS = EACH / 2;       // elements of a row that a lane holds, and words of them as the type
    static constexpr int BYTES = HELD == FF_HELD_SAME ? EACH * 2 : HELD == FF_HELD_E4M3 ? EACH : EACH / 2;
    static constexpr int RAW = BYTES < 4 ? 1 : BYTES / 4;
    uint32_t raw[8][RAW];
    uint32_t s[2];                  // scales of the four positions of each half

    __device__ __forceinline__ void load(const PagedArgs& a, int half, const char* rows, const uint8_t* scales, const Lane& l)
    {
        const uint32_t row = row_bytes<HELD, D, FULL>(a), at = l.g * 4 * row + (FULL || l.x * EACH < (int)a.dim ? l.x * BYTES : 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const char* p = rows + (at + r * row);
            uint32_t* to = raw[half * 4 + r];
            if constexpr (BYTES == 16) {
                const uint4 w = *(const uint4*)p;
                to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
            } else if constexpr (BYTES == 8) {
                const uint2 w = *(const uint2*)p;
                to[0] = w.x, to[1] = w.y;
            } else if constexpr (BYTES == 4) {
                to[0] = *(const uint32_t*)p;
            } else {
                to[0] = *(const uint16_t*)p;
            }
        }
        if constexpr (HELD != FF_HELD_SAME) s[half] = *(const uint32_t*)(scales + ((HELD == FF_HELD_E4M3 ? 0 : min((uint32_t)(l.x * EACH / 32), a.c.blocks - 1)) * a.c.page + l.g * 4));
    }
    // positions from left[half] on (of those of lane group 0) are behind the last, or have no page: what lies there, or was read in its place, may be anything
    __device__ __forceinline__ void clear(const int* left)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool out = e % 4 >= left[e / 4];
#pragma unroll
            for (int i = 0; i < RAW; ++i) raw[e][i] = out ? 0 : raw[e][i];
            if constexpr (HELD != FF_HELD_SAME) s[e / 4] = out ? s[e / 4] & ~(255u << (e % 4 * 8)) : s[e / 4];
        }
    }
    // word i of the lane's elements of position e (of its eight)
    template <int I>
    __device__ __forceinline__ uint32_t word(int e) const
    {
        const float f = HELD == FF_HELD_SAME ? 0 : scale_operand(s[e / 4] >> (e % 4 * 8) & 255);
        if constexpr (HELD == FF_HELD_SAME) return raw[e][I];
        else if constexpr (HELD == FF_HELD_E4M3) return from_e4m3<T, I % 2 == 1>(raw[e][I / 2], f);
        else return from_e2m1<T, I>(raw[e][0], f);
    }
};

// ---- a stretch of a sequence ----

// the columns of a block: which query and head, and how many keys it sees
template <int NT>
struct Columns {
    uint32_t i[NT], h[NT];
    bool in[NT];
    int seen[NT];
};

// the query of a column: col / group.  Columns are below 2^20, so that the quotient of col + 0.5 is off by less than 2^-23 of 2^20 / group, a quarter of what the nearest whole number is away at least
__device__ __forceinline__ uint32_t query_of(const PagedArgs& a, uint32_t col) { return (uint32_t)(((float)col + 0.5f) * a.per_group); }

template <int NT>
__device__ __forceinline__ Columns<NT> columns_of(const PagedArgs& a, uint32_t b, uint32_t kh, uint32_t first, int nk, int x)
{
    Columns<NT> c;
    const int nq = cached(a.q_lengths, a.q_len, b);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t col = first + t * 16 + x;
        c.in[t] = col < a.cols;
        c.i[t] = c.in[t] ? query_of(a, col) : 0, c.h[t] = kh * a.group + (c.in[t] ? col - c.i[t] * a.group : 0);
        int n = 0;
        if (c.in[t] && (int)c.i[t] < nq) {
            n = a.causal ? (int)c.i[t] + 1 + nk - nq : nk;
            n = n < 0 ? 0 : n > nk ? nk : n;
        }
        c.seen[t] = n;
    }
    return c;
}

// A tile as it is asked for.  `bad`: which of its halves has no page; what is read in its place does not count.
template <class T, int HELD, int D, bool FULL>
struct Tile {
    Keys<T, HELD, D, FULL> k;
    Values<T, HELD, D, FULL> v;
    bool bad[2];
};

// The tiles of a wave of a stretch of a sequence: every WAVES-th one.  A lane keeps the table's entry of one half of 32 of them.
struct Stretch {
    const int32_t* table;
    int nk;
    int at0;                        // position of the wave's first tile
    int entries;
    uint64_t head, scale_head;      // of the key head in a page
    __device__ __forceinline__ int at(int i) const { return at0 + i * (WAVES * TILE); }
};

template <class T, int HELD, int D, bool FULL>
__device__ __forceinline__ void ask(const PagedArgs& a, Tile<T, HELD, D, FULL>& x, Stretch& s, int i, const Lane& l)
{
    if (i % 32 == 0) s.entries = s.table[entry_of(s.at(i + l.lane / 2) + l.lane % 2 * 16, s.nk, a.c.page_log2)];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t n = (uint32_t)__builtin_amdgcn_readlane(s.entries, i % 32 * 2 + h);
        x.bad[h] = n >= a.c.pages;
        n = x.bad[h] ? 0 : n;
        const uint64_t page = n;
        const uint32_t place = place_of(s.at(i) + 16 * h, s.nk, a.c.page);
        const uint32_t rows = place * row_bytes<HELD, D, FULL>(a);
        x.k.load(a, h, a.c.k + page * a.c.k_stride + s.head + rows, HELD == FF_HELD_SAME ? nullptr : a.c.k_scale + page * a.c.k_scale_stride + s.scale_head + place, l);
        x.v.load(a, h, a.c.v + page * a.c.v_stride + s.head + rows, HELD == FF_HELD_SAME ? nullptr : a.c.v_scale + page * a.c.v_scale_stride + s.scale_head + place, l);
    }
}

// sums of a wave's columns
template <class T, int D, int NT>
struct Sums {
    typename T::vec8 q[NT][D / 32];
    f32x4 o[NT][D / 16];
    float m[NT], sum[NT];
    int seen_least;                 // keys that all columns see
};

// the largest over lanes l, l ^ 16, l ^ 32 and l ^ 48, by exchanges of halves between two registers
__device__ __forceinline__ float over_groups(float x)
{
    uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];        // (a bit cast of a vector's element itself takes the first one)
    u = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    return fmaxf(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}

// o += v^T p, from the lane's words I on: two columns of v each
template <int I, class T, int HELD, int D, bool FULL, int NT>
__device__ __forceinline__ void values_times(const Values<T, HELD, D, FULL>& v, const typename T::vec8* p, const typename T::vec8* rest, Sums<T, D, NT>& y)
{
    if constexpr (I < D / 32) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = v.template word<I>(e);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint4 u;
            uint32_t* uw = (uint32_t*)&u;
#pragma unroll
            for (int i = 0; i < 4; ++i) uw[i] = j ? high_pair(w[2 * i], w[2 * i + 1]) : low_pair(w[2 * i], w[2 * i + 1]);
            const auto vv = __builtin_bit_cast(typename T::vec8, u);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                y.o[t][2 * I + j] = T::mma(vv, p[t], y.o[t][2 * I + j]);
                if constexpr (std::is_same<T, BF16>::value) y.o[t][2 * I + j] = T::mma(vv, rest[t], y.o[t][2 * I + j]);
            }
        }
        values_times<I + 1, T, HELD, D, FULL, NT>(v, p, rest, y);
    }
}

template <class T, int HELD, int D, bool FULL, int NT>
__device__ __forceinline__ void work(const PagedArgs& a, Tile<T, HELD, D, FULL>& x, Sums<T, D, NT>& y, const Columns<NT>& c, int at, int nk, const Lane& l)
{
    constexpr int STEPS = D / 32, DT = D / 16;
    typedef typename T::vec8 vec8;
    f32x4 s[NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t][h] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            const vec8 kk = x.k.operand(a, h, st, l.g);
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][h] = T::mma(kk, y.q[t][st], s[t][h]);
        }
    }
    const bool bad = x.bad[0] || x.bad[1];
    if (at + TILE > y.seen_least || bad) {
        // a position is left out if the column does not see it, and if it has no page; a column that sees one of those becomes a NaN
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            int first = c.seen[t] - at - 4 * l.g;
            stay_here(first);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * h + r >= first || x.bad[h]) s[t][h][r] = -INFINITY;
            if ((x.bad[0] && at < c.seen[t]) || (x.bad[1] && at + 16 < c.seen[t])) y.sum[t] = NAN;
        }
        if (at + TILE > nk || bad) {
            int left[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                left[h] = x.bad[h] ? 0 : nk - at - 16 * h - 4 * l.g;
                stay_here(left[h]);
            }
            x.v.clear(left);
        }
    }
    vec8 p[NT], rest[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        float top = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])), fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
        top = over_groups(top) * a.scale_log2;
        if (__any(top > y.m[t] + (MAX_BEHIND<T> + P_SHIFT<T>))) {     // m, the maximum less the shift, starts at -inf; a column that sees nothing keeps it
            const float mn = fmaxf(y.m[t], top - P_SHIFT<T>), f = mn == -INFINITY ? 1.0f : exp2_(y.m[t] - mn);
            y.sum[t] *= f;
#pragma unroll
            for (int j = 0; j < DT; ++j) y.o[t][j] *= f;
            y.m[t] = mn;
        }
        const float base = y.m[t] == -INFINITY ? 0.0f : y.m[t];
        float e[8], left[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[i] = exp2_(fmaf(s[t][i / 4][i % 4], a.scale_log2, -base));
            y.sum[t] += e[i];
        }
        if constexpr (std::is_same<T, BF16>::value) {
            // cut off, and the rest, which is never 0 beside more than 0: an infinite value then stays one
            uint4 cut;
            uint32_t* cw = (uint32_t*)&cut;
#pragma unroll
            for (int i = 0; i < 4; ++i) cw[i] = high_pair(__builtin_bit_cast(uint32_t, e[2 * i]), __builtin_bit_cast(uint32_t, e[2 * i + 1]));
            p[t] = __builtin_bit_cast(vec8, cut);
#pragma unroll
            for (int i = 0; i < 8; ++i) left[i] = fmaxf(e[i] - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, e[i]) & 0xffff0000u), e[i] * 0x1p-30f);
            rest[t] = round8<T>(left);
        } else {
            p[t] = round8<T>(e);
        }
    }
    values_times<0, T, HELD, D, FULL, NT>(x.v, p, rest, y);
}

// A tile is asked for while another is worked where registers hold both; else when that one is done with, and the other wave of the SIMD works meanwhile.  16 sequences of 16384 positions, 32 heads on 8 of
// 128, 8 queries: e4m3 129 us with two tiles, 120 with one; e2m1 94 and 102 (keys asked for before the values are worked); one query, e4m3, 73 and 77.
template <int HELD, int D, int NT>
constexpr bool TWO = HELD == FF_HELD_E2M1 || D == 64 || NT == 1;
constexpr int RESIDENT = 2;         // waves of a SIMD: three need the registers of one tile (above), and 512 runs are no more than two

template <class T, int HELD, int D, bool FULL, int NT>
__global__ __launch_bounds__(256, RESIDENT) void k_attention_paged(PagedArgs a)
{
    constexpr int STEPS = D / 32, DT = D / 16;
    typedef typename T::vec8 vec8;
    __shared__ Finder find;
    __shared__ float stat[NT][WAVES][2][16];
    __shared__ float sums[NT][WAVES][16][D + 4];
    Lane l;
    l.lane = threadIdx.x % 64, l.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l.x = l.lane % 16, l.g = l.lane / 16;
    const uint32_t kh = blockIdx.x, run = blockIdx.y, col0 = blockIdx.z * (16 * NT);
    int64_t t0, t1, first;              // places of the run in the list, and where sequence b begins there
    uint32_t b;
    List list;
    if (a.runs) {
        list.make(a, find);
        const Runs runs = runs_used(a.runs, list.all);
        if (run >= runs.n || list.all == 0) return;
        t0 = runs.begin(run), t1 = runs.begin(run + 1);
        list.sequence_at(a, t0, find, b, first);
    } else {
        b = run, t0 = 0, first = 0, t1 = ENTRY + tiles_of(positions(a, b));
    }
    for (;; ++b) {
        const int nk = a.runs ? list.length(a, b) : positions(a, b);
        if (a.runs && nk == 0) continue;
        // its tiles: all of them, and those of this run, from e0 to e1
        const int64_t begin = first + ENTRY, end = begin + tiles_of(nk), e0 = t0 > begin ? t0 : begin, e1 = t1 < end ? t1 : end;
        first = end;
        if (a.runs && e0 >= e1) break;              // the run ends before the first
        const Columns<NT> c = columns_of<NT>(a, b, kh, col0, nk, l.x);
        uint4 q[NT][STEPS];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int d = Keys<T, HELD, D, FULL>::element(s, l.g);
                q[t][s] = *(const uint4*)(a.q.p + b * a.q.batch + c.h[t] * a.q.head + c.i[t] * a.q.pos + (FULL || d < (int)a.dim ? d * 2 : 0));
            }
        Stretch at = {a.c.table + b * a.c.table_stride, nk, (int)(e0 + l.wave - begin) * TILE, 0, (uint64_t)kh * a.c.page * a.c.row, (uint64_t)kh * a.c.page * a.c.blocks};
        const int n = e1 - e0 > l.wave ? (int)((e1 - e0 - l.wave + WAVES - 1) / WAVES) : 0;
        Tile<T, HELD, D, FULL> x0;
        if (n > 0) ask(a, x0, at, 0, l);
        Sums<T, D, NT> y;
        int least = nk;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            least = min(least, c.in[t] ? c.seen[t] : nk);
            y.m[t] = -INFINITY, y.sum[t] = 0;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int d = Keys<T, HELD, D, FULL>::element(s, l.g);
                y.q[t][s] = __builtin_bit_cast(vec8, c.seen[t] > 0 && (FULL || d < (int)a.dim) ? q[t][s] : uint4{0, 0, 0, 0});
            }
#pragma unroll
            for (int j = 0; j < DT; ++j) y.o[t][j] = f32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int d = 8; d; d >>= 1) least = min(least, __shfl_xor(least, d));
        y.seen_least = __builtin_amdgcn_readfirstlane(least);
        if constexpr (TWO<HELD, D, NT>) {
            Tile<T, HELD, D, FULL> x1;
            for (int i = 0; i < n; i += 2) {
                if (i + 1 < n) ask(a, x1, at, i + 1, l);
                work(a, x0, y, c, at.at(i), nk, l);
                if (i + 1 >= n) break;
                if (i + 2 < n) ask(a, x0, at, i + 2, l);
                work(a, x1, y, c, at.at(i + 1), nk, l);
            }
        } else {
            for (int i = 0; i < n; ++i) {
                work(a, x0, y, c, at.at(i), nk, l);
                if (i + 1 < n) ask(a, x0, at, i + 1, l);
            }
        }
        // the four waves' sums together
        const bool whole = e0 == begin && e1 == end;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float total = y.sum[t];
            total += __shfl_xor(total, 16);
            total += __shfl_xor(total, 32);
            if (l.g == 0) stat[t][l.wave][0][l.x] = y.m[t], stat[t][l.wave][1][l.x] = total;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < DT; j += 4)
                    *(f32x4*)&sums[t][l.wave][l.x][(l.g * 4 + r) * DT + j] = f32x4{y.o[t][j][r], y.o[t][j + 1][r], y.o[t][j + 2][r], y.o[t][j + 3][r]};
        }
        __syncthreads();
        // a thread: D / 16 elements of column threadIdx.x / 16
        const uint32_t cc = threadIdx.x / 16, d0 = threadIdx.x % 16 * DT;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t col = col0 + t * 16 + cc;
            if (col >= a.cols) continue;
            float most = -INFINITY, sum = 0, r[DT] = {};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = fmaxf(most, stat[t][w][0][cc]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                // a wave that has seen nothing has sums of 0, or the NaN of a position without a page
                const float m = stat[t][w][0][cc], f = m == -INFINITY ? 1.0f : exp2_(m - most);
                sum += stat[t][w][1][cc] * f;
#pragma unroll
                for (int j = 0; j < DT; ++j) r[j] += sums[t][w][cc][d0 + j] * f;
            }
            const float inv = sum > 0 ? 1.0f / sum : sum == sum ? 0.0f : sum;
            const uint32_t keep = sum == 0 ? 0 : ~0u;           // a query that sees nothing has zeros, whatever values others see
#pragma unroll
            for (int j = 0; j < DT; ++j) r[j] = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, r[j] * inv) & keep);
            const uint32_t i = query_of(a, col), h = kh * a.group + col - i * a.group;
            if (whole) {
                if (d0 == 0) a.lse[((uint64_t)b * a.heads + h) * a.q_len + i] = (most + log2_(sum)) * LN2;
                char* to = a.o.p + b * a.o.batch + h * a.o.head + i * a.o.pos;
#pragma unroll
                for (int j = 0; j < DT; j += 4)
                    if (d0 + j < a.dim) store4<T>(to + (d0 + j) * 2, r[j], r[j + 1], r[j + 2], r[j + 3]);
            } else {
                const uint64_t row = ((uint64_t)slot_of(run, e0 == begin) * a.kv_heads + kh) * a.cols + col;
                if (d0 == 0) a.part_lse[row] = most + log2_(sum);
#pragma unroll
                for (int j = 0; j < DT; j += 4)
                    if (d0 + j < a.dim) *(f32x4*)(a.part + row * a.dim + d0 + j) = f32x4{r[j], r[j + 1], r[j + 2], r[j + 3]};
            }
        }
        if (t1 <= end) break;
        __syncthreads();
    }
}

// Joins the parts of a sequence that several runs share: o = sum_s 2^(lse_s - lse) o_s; a wave per row, as in the contiguous kernel.  Sequences without positions get their zeros here.
template <class T>
__global__ __launch_bounds__(256) void k_attention_paged_join(PagedArgs a)
{
    __shared__ Finder find;
    const uint32_t b = blockIdx.y;
    List list;
    list.make(a, find);
    const int64_t first = list.begin_of(a, b, find) + ENTRY, n = tiles_of(list.length(a, b));
    const uint32_t row = blockIdx.x * WAVES + threadIdx.x / 64, lane = threadIdx.x % 64, x = lane % 16 * 8;      // row: head * q_len + query
    if (row >= a.heads * a.q_len) return;
    const uint32_t h = row / a.q_len, i = row % a.q_len, kh = h / a.group, col = i * a.group + h % a.group;
    char* to = a.o.p + b * a.o.batch + h * a.o.head + i * a.o.pos + x * 2;
    float* lse = a.lse + ((uint64_t)b * a.heads + h) * a.q_len + i;
    if (n == 0) {
        if (lane == 0) *lse = -INFINITY;
        if (lane < 16 && x < a.dim) *(uint4*)to = uint4{0, 0, 0, 0};
        return;
    }
    const Runs runs = runs_used(a.runs, list.all);
    const uint32_t r0 = runs.of(first), r1 = runs.of(first + n - 1);
    if (r0 == r1) return;
    auto slot_row = [&](uint32_t r) { return ((uint64_t)slot_of(r, r == r0) * a.kv_heads + kh) * a.cols + col; };
    // four of the parts at a time, a quarter of the lanes each, with a maximum of its own
    float m = -INFINITY, sum = 0, o[8] = {};
    bool none = false;
#pragma unroll 4
    for (uint32_t r = r0 + lane / 16; r <= r1; r += 4) {
        const uint64_t at = slot_row(r);
        const float s = a.part_lse[at];
        const float* p = a.part + at * a.dim + (x < a.dim ? x : 0);
        const f32x4 u = *(const f32x4*)p, v = *(const f32x4*)(p + 4);
        none |= s != s;
        const float top = fmaxf(m, s), f = m == -INFINITY ? 0.0f : exp2_(m - top), w = s == -INFINITY ? 0.0f : exp2_(s - top);
        sum = sum * f + w, m = top;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * f + w * u[e], o[4 + e] = o[4 + e] * f + w * v[e];
    }
    float base = fmaxf(m, __shfl_xor(m, 16));
    base = fmaxf(base, __shfl_xor(base, 32));
    const float f = m == -INFINITY ? 0.0f : exp2_(m - base);
    sum *= f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= f;
    if (base == -INFINITY) base = 0;
#pragma unroll
    for (int d = 16; d < 64; d *= 2) {
        sum += __shfl_xor(sum, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += __shfl_xor(o[e], d);
    }
    if (__any(none)) sum = NAN;
    if (lane >= 16) return;
    const float inv = sum > 0 ? 1.0f / sum : sum == sum ? 0.0f : sum;
    if (lane == 0) *lse = (base + log2_(sum)) * LN2;
    if (x >= a.dim) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= inv;
    *(typename T::vec8*)to = round8<T>(o);
}

uint32_t column_tiles(const PagedArgs& a) { return a.cols <= 16 ? 1 : 2; }

template <class T, int HELD, int D, bool FULL>
void launch(const PagedArgs& a, hipStream_t st)
{
    const uint32_t nt = column_tiles(a);
    const dim3 grid(a.kv_heads, a.runs ? a.runs : a.batch, (uint32_t)ceil_div(a.cols, 16 * nt));
    if (nt == 1) k_attention_paged<T, HELD, D, FULL, 1><<<grid, 256, 0, st>>>(a);
    else k_attention_paged<T, HELD, D, FULL, 2><<<grid, 256, 0, st>>>(a);
}

template <class T, int HELD>
void launch(const PagedArgs& a, hipStream_t st)
{
    if (a.dim == 64) launch<T, HELD, 64, true>(a, st);
    else if (a.dim < 64) launch<T, HELD, 64, false>(a, st);
    else if (a.dim == 128) launch<T, HELD, 128, true>(a, st);
    else launch<T, HELD, 128, false>(a, st);
}

template <class T>
int run(const PagedArgs& a, uint32_t held, hipStream_t st)
{
    if (held == FF_HELD_SAME) launch<T, FF_HELD_SAME>(a, st);
    else if (held == FF_HELD_E4M3) launch<T, FF_HELD_E4M3>(a, st);
    else launch<T, FF_HELD_E2M1>(a, st);
    if (a.runs) k_attention_paged_join<T><<<dim3((uint32_t)ceil_div((uint64_t)a.heads * a.q_len, WAVES), a.batch), 256, 0, st>>>(a);
    return launched();
}

int check(const ff_attention_paged_fwd_t* p)
{
    if (p->heads == 0 || p->kv_heads == 0 || p->heads % p->kv_heads) return FF_EINVAL;
    if (!(p->scale > 0) || !std::isfinite(p->scale)) return FF_EINVAL;
    if (const int rc = check_cache_sizes(p->cache, p->dtype, p->batch, p->kv_heads, p->head_dim)) return rc;
    // launch grids: blocks of 16 columns along z, a wave for every row of the join along x
    if (p->heads > 65535 || p->q_len > FF_OP_MAX_LEN || (uint64_t)p->q_len * (p->heads / p->kv_heads) > (uint64_t)MOST_BLOCKS_Y * 16 || ceil_div((uint64_t)p->heads * p->q_len, WAVES) * 256 > MOST_THREADS)
        return FF_ERANGE;
    return FF_OK;
}

PagedArgs args_of(const ff_attention_paged_fwd_t* p)
{
    PagedArgs a = {};
    a.c = cache_args(p->cache, p->head_dim);
    a.batch = p->batch, a.heads = p->heads, a.kv_heads = p->kv_heads, a.group = p->heads / p->kv_heads;
    a.q_len = p->q_len, a.dim = p->head_dim, a.causal = p->causal != 0, a.cols = p->q_len * a.group;
    a.scale_log2 = p->scale * LOG2E, a.per_group = 1.0f / (float)a.group;
    a.q = in_bytes(p->q), a.o = in_bytes(p->o);
    a.q_lengths = p->q_lengths, a.kv_lengths = p->kv_lengths;
    a.runs = p->q_len ? runs_of(a.kv_heads * ceil_div(a.cols, 16 * column_tiles(a)), a.batch, (uint64_t)a.c.table_pages * a.c.page) : 0;
    return a;
}

uint64_t part_rows(const PagedArgs& a) { return 2ull * a.runs * a.kv_heads * a.cols; }

}  // namespace
}  // namespace ffops

using namespace ffops;

extern "C" size_t ff_op_attention_paged_fwd_workspace_bytes(const ff_attention_paged_fwd_t* p)
{
    if (!p || check(p) != FF_OK) return 0;
    const PagedArgs a = args_of(p);
    return part_rows(a) * (a.dim + 1) * sizeof(float);
}

extern "C" int ff_op_attention_paged_fwd(const ff_attention_paged_fwd_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check(p)) return rc;
    if (p->batch == 0 || p->q_len == 0) return FF_OK;
    if (!heads_ok(p->q) || !heads_ok(p->o) || !p->lse) return FF_EINVAL;
    if (p->cache.table_pages)
        if (const int rc = check_cache(p->cache)) return rc;
    PagedArgs a = args_of(p);
    a.lse = p->lse;
    const size_t need = ff_op_attention_paged_fwd_workspace_bytes(p);
    if (need) {
        if (!p->workspace || p->workspace_bytes < need || !aligned(p->workspace, 256)) return FF_EWORKSPACE;
        a.part = (float*)p->workspace;
        a.part_lse = a.part + part_rows(a) * a.dim;
    }
    return p->dtype == FF_F16 ? run<F16>(a, p->cache.held, (hipStream_t)stream) : run<BF16>(a, p->cache.held, (hipStream_t)stream);
}
