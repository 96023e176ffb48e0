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
    float scale_log2;
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
// which costs products, of which there are plenty, and leaves the output's own rounding the only one that counts.
//   Work is dealt in equal runs of tiles over all sequences, whatever their lengths (ffops_paged_runs.h); parts of a sequence are joined by a second kernel.
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

// The sums of tiles up to a place, by all 256 threads: each takes a stretch of sequences.
struct Finder {
    int64_t sum[WAVES];
    uint32_t b;
    int64_t first;
};

__device__ __forceinline__ int64_t tiles_of(const PagedArgs& a, uint32_t b) { return (positions(a, b) + TILE - 1) / TILE; }

// the sum of x over the threads before this one; `all`: over all of them
__device__ __forceinline__ int64_t sum_before(int64_t x, Finder& f, int64_t& all)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int64_t s = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t t = __shfl_up(s, d);
        if (lane >= d) s += t;
    }
    if (lane == 63) f.sum[wave] = s;
    __syncthreads();
    int64_t before = 0;
    all = 0;
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += f.sum[w];
        all += f.sum[w];
    }
    return before + s - x;
}

struct Lane {
    int lane, wave, x, g;           // x = lane % 16, g = lane / 16
};

// two 16-bit elements of the same column from two rows: the low or the high halves
__device__ __forceinline__ uint32_t low_pair(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100); }
__device__ __forceinline__ uint32_t high_pair(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302); }

// ---- a tile's keys ----

// operands of 32 positions: [half][step]; D elements of a row, a.dim of them real
template <class T, int HELD, int D>
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
    __device__ __forceinline__ void load(const PagedArgs& a, int half, const char* page, const uint8_t* scales, uint32_t place, const Lane& l)
    {
        const char* p = page + (place + l.x) * a.c.row;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int first = element(HELD == FF_HELD_E4M3 ? 2 * i : i, l.g);
            const uint32_t at = HELD == FF_HELD_SAME ? first * 2 : HELD == FF_HELD_E4M3 ? first : first / 2;
            const char* from = first < (int)a.dim ? p + at : (const char*)&zero16;
            if constexpr (SHORT) {
                const uint2 w = *(const uint2*)from;
                raw[half][i] = {w.x, w.y, 0, 0};
            } else {
                raw[half][i] = *(const uint4*)from;
            }
        }
        if constexpr (HELD == FF_HELD_E4M3) s[half] = scales[place + l.x];
        if constexpr (HELD == FF_HELD_E2M1) s[half] = scales[min((uint32_t)(l.g * (D / 4) / 32), a.c.blocks - 1) * a.c.page + place + l.x];
    }
    __device__ __forceinline__ typename T::vec8 operand(int half, int st) const
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
        return __builtin_bit_cast(typename T::vec8, v);
    }
};

// ---- a tile's values ----

template <class T, int HELD, int D>
struct Values {
    static constexpr int EACH = D / 16, WORDS = EACH / 2;       // elements of a row that a lane holds, and words of them as the type
    static constexpr int BYTES = HELD == FF_HELD_SAME ? EACH * 2 : HELD == FF_HELD_E4M3 ? EACH : EACH / 2;
    static constexpr int RAW = BYTES < 4 ? 1 : BYTES / 4;
    uint32_t raw[8][RAW];
    uint32_t s[2];                  // scales of the four positions of each half

    __device__ __forceinline__ void load(const PagedArgs& a, int half, const char* page, const uint8_t* scales, uint32_t place, const Lane& l)
    {
        const bool in = l.x * EACH < (int)a.dim;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const char* p = in ? page + (place + l.g * 4 + r) * a.c.row + l.x * BYTES : (const char*)&zero16;
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
        if constexpr (HELD != FF_HELD_SAME) s[half] = *(const uint32_t*)(scales + (HELD == FF_HELD_E4M3 ? 0 : min((uint32_t)(l.x * EACH / 32), a.c.blocks - 1)) * a.c.page + place + l.g * 4);
    }
    // words of the lane's elements of position e (of its eight)
    __device__ __forceinline__ void words(int e, uint32_t* w) const
    {
        const float f = HELD == FF_HELD_SAME ? 0 : scale_operand(s[e / 4] >> (e % 4 * 8) & 255);
        if constexpr (HELD == FF_HELD_SAME) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = raw[e][i];
        } else if constexpr (HELD == FF_HELD_E4M3) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = i % 2 ? from_e4m3<T, true>(raw[e][i / 2], f) : from_e4m3<T, false>(raw[e][i / 2], f);
        } else {
            w[0] = from_e2m1<T, 0>(raw[e][0], f), w[1] = from_e2m1<T, 1>(raw[e][0], f);
            if constexpr (WORDS == 4) w[2] = from_e2m1<T, 2>(raw[e][0], f), w[3] = from_e2m1<T, 3>(raw[e][0], f);
        }
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

template <int NT>
__device__ __forceinline__ Columns<NT> columns_of(const PagedArgs& a, uint32_t b, uint32_t kh, uint32_t first, int nk, int x)
{
    Columns<NT> c;
    const int nq = cached(a.q_lengths, a.q_len, b);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t col = first + t * 16 + x;
        c.in[t] = col < a.cols;
        c.i[t] = c.in[t] ? col / a.group : 0, c.h[t] = kh * a.group + (c.in[t] ? col % a.group : 0);
        int n = 0;
        if (c.in[t] && (int)c.i[t] < nq) {
            n = a.causal ? (int)c.i[t] + 1 + nk - nq : nk;
            n = n < 0 ? 0 : n > nk ? nk : n;
        }
        c.seen[t] = n;
    }
    return c;
}

// the page of 16 positions from `at`: its number, 0 in the place of one that there is not
struct Group {
    uint32_t page, place;
    bool bad;
};
__device__ __forceinline__ Group group_at(const PagedArgs& a, const int32_t* table, int at, int nk)
{
    Group g;
    const uint32_t page = (uint32_t)__builtin_amdgcn_readfirstlane(table[entry_of(at, nk, a.c.page_log2)]);
    g.bad = page >= a.c.pages;
    g.page = g.bad ? 0 : page;
    g.place = place_of(at, nk, a.c.page);
    return g;
}

template <class T, int HELD, int D, int NT>
__global__ __launch_bounds__(256) void k_attention_paged(PagedArgs a)
{
    constexpr int STEPS = D / 32, DT = D / 16;
    typedef typename T::vec8 vec8;
    __shared__ Finder find;
    __shared__ float stat[WAVES][2][16];
    __shared__ float sums[WAVES][16][D + 4];
    Lane l;
    l.lane = threadIdx.x % 64, l.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l.x = l.lane % 16, l.g = l.lane / 16;
    const uint32_t kh = blockIdx.x % a.kv_heads, run = blockIdx.x / a.kv_heads, col0 = blockIdx.y * (16 * NT);
    int64_t t0, t1, first, all = 0;     // tiles in the list of all, and the first one of sequence b
    uint32_t b;
    if (a.runs) {
        const uint32_t per = (a.batch + 255) / 256, b0 = min(a.batch, threadIdx.x * per), b1 = min(a.batch, b0 + per);
        int64_t mine = 0;
        for (uint32_t i = b0; i < b1; ++i) mine += tiles_of(a, i);
        int64_t before = sum_before(mine, find, all);
        const uint32_t runs = runs_used(a.runs, all);
        if (run >= runs || all == 0) return;
        t0 = run_begin(run, runs, all), t1 = run_begin(run + 1, runs, all);
        if (before <= t0 && t0 < before + mine)
            for (uint32_t i = b0; i < b1; ++i) {
                const int64_t n = tiles_of(a, i);
                if (t0 < before + n) {
                    find.b = i, find.first = before;
                    break;
                }
                before += n;
            }
        __syncthreads();
        b = find.b, first = find.first;
    } else {
        b = run, first = 0, t0 = 0, t1 = tiles_of(a, b);
        all = t1;
    }
    for (;; ++b) {
        const int nk = positions(a, b);
        const int64_t tiles = (nk + TILE - 1) / TILE, last = first + tiles;
        if (a.runs && tiles == 0) continue;
        const int64_t e1 = t1 < last ? t1 : last;
        const Columns<NT> c = columns_of<NT>(a, b, kh, col0, nk, l.x);
        vec8 q[NT][STEPS];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int d = Keys<T, HELD, D>::element(s, l.g);
                q[t][s] = *(const vec8*)(c.seen[t] > 0 && d < (int)a.dim ? a.q.p + b * a.q.batch + c.h[t] * a.q.head + c.i[t] * a.q.pos + d * 2 : (const char*)&zero16);
            }
        f32x4 o[NT][DT];
        float m[NT], sum[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t] = -INFINITY, sum[t] = 0;
#pragma unroll
            for (int j = 0; j < DT; ++j) o[t][j] = f32x4{0, 0, 0, 0};
        }
        const int32_t* table = a.c.table + b * a.c.table_stride;
        const uint64_t head = (uint64_t)kh * a.c.page * a.c.row, scale_head = (uint64_t)kh * a.c.page * a.c.blocks;
        for (int64_t tile = t0 + l.wave; tile < e1; tile += WAVES) {
            const int at = (int)(tile - first) * TILE;
            Keys<T, HELD, D> k;
            Values<T, HELD, D> v;
            Group g[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                g[h] = group_at(a, table, at + 16 * h, nk);
                const uint64_t page = g[h].page;
                k.load(a, h, a.c.k + page * a.c.k_stride + head, HELD == FF_HELD_SAME ? nullptr : a.c.k_scale + page * a.c.k_scale_stride + scale_head, g[h].place, l);
                v.load(a, h, a.c.v + page * a.c.v_stride + head, HELD == FF_HELD_SAME ? nullptr : a.c.v_scale + page * a.c.v_scale_stride + scale_head, g[h].place, l);
            }
            // scores
            f32x4 s[NT][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int t = 0; t < NT; ++t) s[t][h] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    const vec8 kk = k.operand(h, st);
#pragma unroll
                    for (int t = 0; t < NT; ++t) s[t][h] = T::mma(kk, q[t][st], s[t][h]);
                }
            }
            const bool bad = g[0].bad || g[1].bad;
            vec8 p[NT], rest[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                // a position is left out if the column does not see it, and if it has no page; a column that sees one of those becomes a NaN
                float top = -INFINITY;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (at + 16 * h + 4 * l.g + r >= c.seen[t] || g[h].bad) s[t][h][r] = -INFINITY;
                        top = fmaxf(top, s[t][h][r]);
                    }
                if (bad && ((g[0].bad && at < c.seen[t]) || (g[1].bad && at + 16 < c.seen[t]))) sum[t] = NAN;
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32)) * a.scale_log2;
                if (__any(top > m[t] + (MAX_BEHIND<T> + P_SHIFT<T>))) {     // m, the maximum less the shift, starts at -inf; a column that sees nothing keeps it
                    const float mn = fmaxf(m[t], top - P_SHIFT<T>), f = mn == -INFINITY ? 1.0f : exp2_(m[t] - mn);
                    sum[t] *= f;
#pragma unroll
                    for (int j = 0; j < DT; ++j) o[t][j] *= f;
                    m[t] = mn;
                }
                const float base = m[t] == -INFINITY ? 0.0f : m[t];
                float e[8], left[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    e[i] = exp2_(fmaf(s[t][i / 4][i % 4], a.scale_log2, -base));
                    sum[t] += e[i];
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
            uint32_t w[8][Values<T, HELD, D>::WORDS];
#pragma unroll
            for (int e = 0; e < 8; ++e) v.words(e, w[e]);
            if (at + TILE > nk) {           // what lies behind the last position may be anything
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (at + 16 * (e / 4) + 4 * l.g + e % 4 >= nk)
#pragma unroll
                        for (int i = 0; i < Values<T, HELD, D>::WORDS; ++i) w[e][i] = 0;
            }
#pragma unroll
            for (int j = 0; j < DT; ++j) {
                uint4 u;
                uint32_t* uw = (uint32_t*)&u;
#pragma unroll
                for (int i = 0; i < 4; ++i) uw[i] = j % 2 ? high_pair(w[2 * i][j / 2], w[2 * i + 1][j / 2]) : low_pair(w[2 * i][j / 2], w[2 * i + 1][j / 2]);
                const vec8 vv = __builtin_bit_cast(vec8, u);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    o[t][j] = T::mma(vv, p[t], o[t][j]);
                    if constexpr (std::is_same<T, BF16>::value) o[t][j] = T::mma(vv, rest[t], o[t][j]);
                }
            }
        }
        // the four waves' sums together, 16 columns at a time
        const bool whole = t0 == first && e1 == last;
        const uint32_t slot = slot_of(run, t0 == first);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float total = sum[t];
            total += __shfl_xor(total, 16);
            total += __shfl_xor(total, 32);
            if (l.g == 0) stat[l.wave][0][l.x] = m[t], stat[l.wave][1][l.x] = total;
            __syncthreads();
            float most = -INFINITY;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = fmaxf(most, stat[w][0][l.x]);
            const float f = m[t] == -INFINITY ? 0.0f : exp2_(m[t] - most);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < DT; j += 4)
                    *(f32x4*)&sums[l.wave][l.x][(l.g * 4 + r) * DT + j] = f32x4{o[t][j][r] * f, o[t][j + 1][r] * f, o[t][j + 2][r] * f, o[t][j + 3][r] * f};
            __syncthreads();
            // a thread: column threadIdx.x / 16, D / 16 elements of it
            const uint32_t cc = threadIdx.x / 16, x0 = threadIdx.x % 16 * DT, col = col0 + t * 16 + cc;
            float mm = -INFINITY, ll = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) mm = fmaxf(mm, stat[w][0][cc]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float mw = stat[w][0][cc], lw = stat[w][1][cc];
                ll += mw == -INFINITY ? lw : lw * exp2_(mw - mm);      // a sum beside no maximum is 0, or the NaN of a position without a page
            }
            if (col < a.cols) {
                const float inv = ll > 0 ? 1.0f / ll : ll == ll ? 0.0f : ll;
                float r[DT];
#pragma unroll
                for (int j = 0; j < DT; ++j) {
                    float y = 0;
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) y += sums[w][cc][x0 + j];
                    r[j] = y * inv;
                }
                const uint32_t i = col / a.group, h = kh * a.group + col % a.group;
                if (whole) {
                    if (x0 == 0) a.lse[((uint64_t)b * a.heads + h) * a.q_len + i] = (mm + log2_(ll)) * LN2;
                    char* to = a.o.p + b * a.o.batch + h * a.o.head + i * a.o.pos;
#pragma unroll
                    for (int j = 0; j < DT; j += 4)
                        if (x0 + j < a.dim) store4<T>(to + (x0 + j) * 2, r[j], r[j + 1], r[j + 2], r[j + 3]);
                } else {
                    const uint64_t row = ((uint64_t)slot * a.kv_heads + kh) * a.cols + col;
                    if (x0 == 0) a.part_lse[row] = mm + log2_(ll);
#pragma unroll
                    for (int j = 0; j < DT; j += 4)
                        if (x0 + j < a.dim) *(f32x4*)(a.part + row * a.dim + x0 + j) = f32x4{r[j], r[j + 1], r[j + 2], r[j + 3]};
                }
            }
            __syncthreads();
        }
        t0 = e1, first = last;
        if (t0 >= t1) break;
    }
}

// Joins the parts of a sequence that several runs share: o = sum_s 2^(lse_s - lse) o_s; a wave per row, as in the contiguous kernel.  Sequences without positions get their zeros here.
template <class T>
__global__ __launch_bounds__(256) void k_attention_paged_join(PagedArgs a)
{
    __shared__ Finder find;
    const uint32_t b = blockIdx.y;
    const uint32_t per = (a.batch + 255) / 256, b0 = min(a.batch, threadIdx.x * per), b1 = min(a.batch, b0 + per);
    int64_t mine = 0, all;
    for (uint32_t i = b0; i < b1; ++i) mine += tiles_of(a, i);
    const int64_t before = sum_before(mine, find, all);
    if (b0 <= b && b < b1) {
        int64_t f = before;
        for (uint32_t i = b0; i < b; ++i) f += tiles_of(a, i);
        find.first = f;
    }
    __syncthreads();
    const int64_t first = find.first, n = tiles_of(a, b);
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
    const uint32_t runs = runs_used(a.runs, all);
    const uint32_t r0 = run_of(first, runs, all), r1 = run_of(first + n - 1, runs, all);
    if (r0 == r1) return;
    auto slot_row = [&](uint32_t r) { return ((uint64_t)slot_of(r, r == r0) * a.kv_heads + kh) * a.cols + col; };
    float m = -INFINITY;
    bool none = false;
    for (uint32_t r = r0 + lane; r <= r1; r += 64) {
        const float s = a.part_lse[slot_row(r)];
        none |= s != s;
        m = fmaxf(m, s);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0, o[8] = {};
    for (uint32_t r = r0 + lane / 16; r <= r1; r += 4) {
        const uint64_t at = slot_row(r);
        const float w = exp2_(a.part_lse[at] - base);
        sum += w;
        const float* p = a.part + at * a.dim + (x < a.dim ? x : 0);
        const f32x4 u = *(const f32x4*)p, v = *(const f32x4*)(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += w * u[e], o[4 + e] += w * v[e];
    }
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

template <class T, int HELD, int D>
void launch(const PagedArgs& a, hipStream_t st)
{
    const uint32_t nt = column_tiles(a);
    const dim3 grid((a.runs ? a.runs : a.batch) * a.kv_heads, (uint32_t)ceil_div(a.cols, 16 * nt));
    if (nt == 1) k_attention_paged<T, HELD, D, 1><<<grid, 256, 0, st>>>(a);
    else k_attention_paged<T, HELD, D, 2><<<grid, 256, 0, st>>>(a);
}

template <class T, int HELD>
void launch(const PagedArgs& a, hipStream_t st)
{
    if (a.dim <= 64) launch<T, HELD, 64>(a, st);
    else launch<T, HELD, 128>(a, st);
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
    // launch grids: blocks of 16 columns along y, a wave for every row of the join along x
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
    a.scale_log2 = p->scale * LOG2E;
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
