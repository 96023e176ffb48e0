// Attention, backward: the probabilities are made again from q, k and the forward pass' lse.
#include "ffops_attention.h"

namespace ffops {
namespace {

// Two kernels, one per side of the score matrix, each of which makes the probabilities for itself: seven products instead of
// five, but every sum has one owner -- no atomic additions, the same bits every time -- and nothing of the size of the score matrix moves.
//   k_attention_dq   owns 32 rows a wave: s^T = k q^T, dp^T = v do^T, dq^T += k^T ds^T; and delta_i = <do_i, o_i>, which it leaves to
//   k_attention_dkv  owns 32 keys a wave: s = q k^T, dp = do v^T, dv^T += do^T p, dk^T += q^T ds
// In both, what the wave owns is the column of every product, so that p and ds are second operands as they lie in the registers; they are rounded to the type because the products
// take nothing wider.  2 sequences of 4096, 32 heads on 8 of 128, causal: 950 to 1000 us for both; profiled by themselves dq 383 (matrix units busy 51 % of the time) and dkv 578 (43 %).
// Both are bound by the vector instructions between products; LDS is busy for a quarter of the time.  Around 32 products a body of dkv has, masks aside, 80 for p and ds (16 of them exponentials),
// 32 to 48 copies out of accumulator registers and some 25 for addresses in LDS; dq makes scores, exponentials and sums of 32 keys one after another.
constexpr int STEP = 64;            // rows (keys) of a tile in LDS

// A 16-bit float has too few exponents for probabilities and gradients of small losses: p is kept times 2^10 (it is at most 1), ds relative to a power of two.
// On the keys' side that is 2^-14 of the one below what bounds the key's |dp - delta|: the largest |do| of its heads (as vectors) times |v|, and the largest |do| |o|.  (Relative to |do|
// alone, values of 2000 along do gave infinities.)  On the queries' side it is 2^-14 of the one below the row's sum of p |dp|, and |delta|, where the block sees few keys.  Where they are many that sum is not at hand: there it is the one below the largest
// |do_d| of the row, and if ds has left the type's range with it, which takes values of hundreds that point along do, the block starts again with 2^10 times that for those rows: |dp - delta| is
// below 2 * 128 * 65504 times twice that power, so ds stays below 2^15 then.  bfloat has a float's exponents and needs none of this.
template <class T>
constexpr float P_SHIFT = std::is_same<T, F16>::value ? 10.0f : 0.0f;

// half a step of the type, relative to the value, and near zero
template <class T>
constexpr float HALF_STEP = std::is_same<T, F16>::value ? 0x1p-11f : 0x1p-8f;
template <class T>
constexpr float HALF_LEAST = std::is_same<T, F16>::value ? 0x1p-25f : 0x1p-134f;

// the exponent of the power of two below m, which is above the least float; 0 where there is none
__device__ __forceinline__ int exponent(float m)
{
    return m > 0 && m < INFINITY ? __builtin_amdgcn_frexp_expf(m) - 1 : 0;
}

constexpr int MORE_EXPONENT = 10;

__device__ __forceinline__ void store_part(float* p, const f32x16& c, int x, int dim, int half, float f)
{
#pragma unroll
    for (int r = 0; r < 16; r += 4)
        if (x + c_row(r, half) < dim) *(f32x4*)(p + x + c_row(r, half)) = f32x4{c[r] * f, c[r + 1] * f, c[r + 2] * f, c[r + 3] * f};
}

template <class T>
__device__ __forceinline__ void store_row(char* p, const f32x16& c, int x, int dim, int half, float f)
{
#pragma unroll
    for (int r = 0; r < 16; r += 4)
        if (x + c_row(r, half) < dim) store4<T>(p + (x + c_row(r, half)) * 2, c[r] * f, c[r + 1] * f, c[r + 2] * f, c[r + 3] * f);
}

static __device__ const float infinity = INFINITY, zero = 0;

// Tiles of queries and their gradients, with the rows' statistics: four of them in LDS (three where one wave starts all loads, whose counter ends at 63), all but one on their way, because a tile lasts
// less long than memory takes to answer and nothing else runs on the wave's SIMD meanwhile.
template <class T, int D, int WAVES>
struct Queries {
    static constexpr int STEP = 64, TILE = STEP * D * 2, STAGE = 2 * TILE + 2 * STEP * 4, STAGES = WAVES == 1 || D == 64 ? 3 : 4;
    static constexpr int LOADS = 2 * TILE / 1024 / WAVES;       // of a wave, for a tile, statistics aside
    TileLoads<STEP, D, WAVES> ql, dl;

    // a tile of `rows` queries, none for rows <= 0; as many loads in any case, since they are counted
    __device__ __forceinline__ void load(lds_char* dst, const char* q, const char* d, const float* lse2, const float* delta, int rows) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
        ql.load(dst, q, rows);
        dl.load(dst + TILE, d, rows);
        if (wave == 0) load_lds4(lane < rows ? lse2 + lane : &infinity, dst + 2 * TILE);
        if (wave == WAVES - 1) load_lds4(lane < rows ? delta + lane : &zero, dst + 2 * TILE + STEP * 4);
    }
};

// What a wave of k_attention_dkv holds.  It has its SIMD to itself, so its own products have to hide its exponentials: while it makes p and ds of one block
// of 32 queries, it multiplies for the scores of the next and for the sums of the one before, neither of which waits for them.
template <class T, int D, int WAVES>
struct Keys32 {
    typedef Queries<T, D, WAVES> Q;
    typedef typename T::vec8 vec8;
    static constexpr int DB = D / 32;

    vec8 k[D / 16], v[D / 16];
    f32x16 dk[DB], dv[DB];

    static constexpr int SCORES = D / 8, SUMS = 4 * DB;        // products

    // the first operand of product i of the scores of the queries from row r of a tile, and of the sums over them
    static __device__ __forceinline__ vec8 for_scores(const lds_char* tile, int r, int i) { return along<T, D>(i % 2 ? tile + Q::TILE : tile, r, i / 2); }
    static __device__ __forceinline__ vec8 for_sums(const lds_char* tile, int r, int i) { return across<T, D>(i % 2 ? tile : tile + Q::TILE, r + i / (2 * DB) * 16, i / 2 % DB * 32); }

    __device__ __forceinline__ void scores(const lds_char* tile, int r, f32x16& s, f32x16& dp) const
    {
        s = dp = f32x16{};
#pragma unroll
        for (int i = 0; i < SCORES; ++i) {
            if (i % 2) dp = T::mma(for_scores(tile, r, i), v[i / 2], dp);
            else s = T::mma(for_scores(tile, r, i), k[i / 2], s);
        }
    }

    __device__ __forceinline__ void sums(const lds_char* tile, int r, const vec8 (&p)[2], const vec8 (&ds)[2])
    {
#pragma unroll
        for (int i = 0; i < SUMS; ++i) sum(i, for_sums(tile, r, i), p, ds);
    }
    __device__ __forceinline__ void sum(int i, vec8 f, const vec8 (&p)[2], const vec8 (&ds)[2])
    {
        const int st = i / (2 * DB), d = i / 2 % DB;
        if (i % 2) dk[d] = T::mma(f, ds[st], dk[d]);
        else dv[d] = T::mma(f, p[st], dv[d]);
    }

    // scores of no key, and of queries that do not see it, are -inf
    __device__ __forceinline__ void mask(f32x16& s, int key0, int nk, int i0, int shift, bool causal) const
    {
        if (key0 + 32 <= nk && !(causal && key0 + 31 > i0 + shift)) return;
        const int lane = threadIdx.x % 64, key = key0 + lane % 32;
        // the first of the 32 queries that sees the key, less what c_row adds for this half of the wave
        int first = (key >= nk ? 32 : causal ? key - i0 - shift : 0) - 4 * (lane / 32);
        stay_here(first);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = c_row(r, 0) >= first ? s[r] : -INFINITY;
    }

    // p and ds of the queries from row R of tile `cur` from their scores; meanwhile sn and dpn of the next 32, from row 32 - R of tile `ahead`, and the sums over the
    // 32 before, from row 32 - R of tile `behind`; LOAD: and the loads of a tile into `into`
    template <int R, bool LOAD>
    __device__ __forceinline__ void body(const lds_char* __restrict cur, const lds_char* __restrict ahead, const lds_char* __restrict behind, lds_char* __restrict into, const Q& queries, const char* qn, const char* dn,
                                         const float* ln, const float* en, int rows, const f32x16& s, const f32x16& dp, f32x16& sn, f32x16& dpn, const vec8 (&pl)[2], const vec8 (&dsl)[2], vec8 (&p)[2], vec8 (&ds)[2],
                                         float c, float per)
    {
        typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
        const int half = (threadIdx.x % 64) / 32;
        if (LOAD) queries.load(into, qn, dn, ln, en, rows);
        // One product, the reads of LDS for the one READ later, and a share of the arithmetic; the compiler keeps to that order.
        constexpr int N = SCORES + SUMS, READ = 5;
        const lds_char* stat = cur + (2 * Q::TILE + (R + 4 * half) * 4);
        const auto first_operand = [&](int i) { return i < SCORES ? for_scores(ahead, 32 - R, i) : for_sums(behind, 32 - R, i - SCORES); };
        vec8 f[N];
        f32x4 ls[5], de[5];
        float fp[16];
#pragma unroll
        for (int i = 0; i < READ; ++i) f[i] = first_operand(i);
        ls[0] = *(lds_f32x4*)stat, de[0] = *(lds_f32x4*)(stat + Q::STEP * 4);
        sn = dpn = f32x16{};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i + READ < N) f[i + READ] = first_operand(i + READ);
            const int e0 = i * 32 / N, e1 = (i + 1) * 32 / N;      // halves of the work on an element
#pragma unroll
            for (int h = e0; h < e1; ++h) {
                const int e = h / 2, g = e / 4;
                if (h % 8 == 0 && g < 3) ls[g + 1] = *(lds_f32x4*)(stat + 32 * (g + 1)), de[g + 1] = *(lds_f32x4*)(stat + 32 * (g + 1) + Q::STEP * 4);
            }
            if (i >= SCORES) sum(i - SCORES, f[i], pl, dsl);
            else if (i % 2) dpn = T::mma(f[i], v[i / 2], dpn);
            else sn = T::mma(f[i], k[i / 2], sn);
#pragma unroll
            for (int h = e0; h < e1; ++h) {
                const int e = h / 2, g = e / 4;
                if (h % 2 == 0) fp[e] = exp2_(fmaf(s[e], c, -ls[g][e % 4]));
                else {
                    p[e / 8][e % 8] = (typename T::elem)fp[e];
                    ds[e / 8][e % 8] = (typename T::elem)(fp[e] * ((dp[e] - de[g][e % 4]) * per));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // here, and not in the branches that follow
        asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(ds[0]), "+v"(ds[1]));
    }
};

template <class T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 1) void k_attention_dkv(AttnArgs a)
{
    typedef Queries<T, D, WAVES> Q;
    constexpr int DB = D / 32, STEP = Q::STEP;
    __shared__ __attribute__((aligned(256))) char lds_[Q::STAGES * Q::STAGE];
    lds_char* lds = (lds_char*)lds_;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const uint32_t bk = heads_of_block(a), b = bk / a.kv_heads, kh = bk % a.kv_heads;
    const int nq = seq_len(a.q_lengths, a.q_len, b), nk = seq_len(a.kv_lengths, a.kv_len, b), shift = nk - nq;
    const int block0 = blockIdx.y * (WAVES * 32), key0 = block0 + wave * 32, key = key0 + lane % 32;       // causal: the keys that most queries see first
    const bool own = key < nk;
    const int chunks = a.dim / 8;
    const bool causal = a.causal;
    Keys32<T, D, WAVES> x;
    row_operand<T, D>(x.k, own ? a.k.p + b * a.k.batch + kh * a.k.head + key * a.k.pos : nullptr, a.dim, half);
    row_operand<T, D>(x.v, own ? a.v.p + b * a.v.batch + kh * a.v.head + key * a.v.pos : nullptr, a.dim, half);
    int unit = 0;                   // exponent, of the lane's key
#pragma unroll
    for (int d = 0; d < DB; ++d) x.dk[d] = x.dv[d] = f32x16{};
    // tiles of queries that see a key of the block, for each head of the group; a split takes a run of them
    const int first = causal && block0 - shift > 0 ? (block0 - shift) / STEP : 0;
    const int per_head = block0 < nk ? max(0, (nq + STEP - 1) / STEP - first) : 0;
    int u0 = 0, u1 = per_head * (int)a.group;
    if (a.splits > 1) {
        const int run = (u1 + (int)a.splits - 1) / (int)a.splits;
        u0 = min(u1, run * (int)blockIdx.z);
        u1 = min(u1, u0 + run);
    }
    if (u0 < u1) {
        Q queries;
        queries.ql.init(a.q.pos, chunks);
        queries.dl.init(a.dout.pos, chunks);
        // the tile that is loaded next
        int g = u0 / per_head, t = first + u0 % per_head, ahead = u0;
        const char *qp, *dp;
        const float *lp, *ep;
        int rows;
        const auto aim = [&] {
            const uint32_t h = kh * a.group + min(g, (int)a.group - 1);
            const int64_t i = (int64_t)t * STEP;
            const uint64_t at = ((uint64_t)b * a.heads + h) * a.q_len + i;
            qp = a.q.p + b * a.q.batch + h * a.q.head + i * a.q.pos;
            dp = a.dout.p + b * a.dout.batch + h * a.dout.head + i * a.dout.pos;
            lp = a.lse2 + at, ep = a.delta + at;
            rows = ahead < u1 ? nq - t * STEP : 0;
        };
        const auto advance = [&] {
            ++ahead;
            if (++t == first + per_head) ++g, t = first;
        };
        for (int n = 0; n < Q::STAGES - 1; ++n) {
            aim();
            queries.load(lds + n * Q::STAGE, qp, dp, lp, ep, rows);
            advance();
        }
        queries.load(lds + (Q::STAGES - 1) * Q::STAGE, qp, dp, lp, ep, 0);      // zeros, for the queries before the first
        if constexpr (std::is_same<T, F16>::value) {
            float2 top = make_float2(0, 0);
            for (uint32_t i = lane; i < a.tops; i += 64) {
                const float2 more = a.top[(uint64_t)bk * a.tops + i];
                top = make_float2(fmaxf(top.x, more.x), fmaxf(top.y, more.y));
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) top = make_float2(fmaxf(top.x, __shfl_xor(top.x, d)), fmaxf(top.y, __shfl_xor(top.y, d)));
            float vv = 0;
#pragma unroll
            for (int st = 0; st < D / 16; ++st)
#pragma unroll
                for (int e = 0; e < 8; ++e) vv += (float)x.v[st][e] * (float)x.v[st][e];
            vv += other_half(vv);
            unit = exponent(fmaf(top.x, __builtin_amdgcn_sqrtf(vv), top.y)) - 14;
        }
        // p is 2^P_SHIFT too large in ds, too
        const float per = ldexpf(1.0f, -(int)P_SHIFT<T> - unit);
        meet<0>();
        typedef typename T::vec8 vec8;
        const float c = a.scale_log2;
        f32x16 s0, s1, d0, d1;
        vec8 p0[2], p1[2] = {}, e0[2], e1[2] = {};
        int i0 = (first + u0 % per_head) * STEP, now = 0;
        x.scores(lds, 0, s0, d0);
        x.mask(s0, key0, nk, i0, shift, causal);
        for (int u = u0; u < u1; ++u) {
            const int before = now == 0 ? (Q::STAGES - 1) * Q::STAGE : now - Q::STAGE, next = now == (Q::STAGES - 1) * Q::STAGE ? 0 : now + Q::STAGE;
            x.template body<0, false>(lds + now, lds + now, lds + before, lds, queries, qp, dp, lp, ep, 0, s0, d0, s1, d1, p1, e1, p0, e0, c, per);
            x.mask(s1, key0, nk, i0 + 32, shift, causal);
            i0 = i0 + STEP == (first + per_head) * STEP ? first * STEP : i0 + STEP;
            meet<(Q::STAGES - 3) * Q::LOADS>();        // the next tile has arrived, and the one before has been read by all
            aim();
            x.template body<32, true>(lds + now, lds + next, lds + now, lds + before, queries, qp, dp, lp, ep, rows, s1, d1, s0, d0, p0, e0, p1, e1, c, per);
            advance();
            x.mask(s0, key0, nk, i0, shift, causal);
            now = next;
        }
        x.sums(lds + (now == 0 ? (Q::STAGES - 1) * Q::STAGE : now - Q::STAGE), 32, p1, e1);
    }
    if (key >= (int)a.kv_len) return;
    const float fk = ldexpf(a.scale, unit), fv = exp2_(-P_SHIFT<T>);
    if (a.splits > 1) {
        const uint64_t n = (uint64_t)a.batch * a.kv_heads * a.kv_len, at = ((uint64_t)bk * a.kv_len + key);
        float *pk = a.part + (2 * (uint64_t)blockIdx.z * n + at) * a.dim, *pv = pk + n * a.dim;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            store_part(pk, x.dk[d], d * 32, a.dim, half, fk);
            store_part(pv, x.dv[d], d * 32, a.dim, half, fv);
        }
        return;
    }
    char *pk = a.dk.p + b * a.dk.batch + kh * a.dk.head + key * a.dk.pos, *pv = a.dv.p + b * a.dv.batch + kh * a.dv.head + key * a.dv.pos;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        store_row<T>(pk, x.dk[d], d * 32, a.dim, half, fk);
        store_row<T>(pv, x.dv[d], d * 32, a.dim, half, fv);
    }
}

// whether `x` is true for any lane of the block; uses 4 bytes at lds, which nobody needs
template <int WAVES>
__device__ __forceinline__ bool any_of_block(bool x, lds_char* lds)
{
    if (WAVES == 1) return __any(x);
    volatile __attribute__((address_space(3))) int* flag = (volatile __attribute__((address_space(3))) int*)lds;
    if (threadIdx.x == 0) *flag = 0;
    __syncthreads();
    if (x) *flag = 1;
    __syncthreads();
    const bool any = *flag;
    __syncthreads();
    return any;
}

struct Next {           // what is loaded while a tile is worked on
    const char *a, *b;
    int rows;
    bool more;
};

// s^T and dp^T of 32 keys from row r of the tile at kt, whose values lie behind it
template <class T, int D>
__device__ __forceinline__ void dq_scores(const lds_char* kt, int r, const typename T::vec8* qf, const typename T::vec8* df, f32x16& s, f32x16& dp)
{
    s = dp = f32x16{};
#pragma unroll
    for (int st = 0; st < D / 16; ++st) {
        s = T::mma(along<T, D>(kt, r, st), qf[st], s);
        dp = T::mma(along<T, D>(kt + STEP * D * 2, r, st), df[st], dp);
    }
    interleave<D / 8, 1, 4, 0>();
}

// What a row's probabilities sum to over the tiles (of which 0 is at lds, 1 behind it), and their products with dp and with its size.
template <class T, int D>
__device__ __forceinline__ void dq_row_sums(const lds_char* lds, const typename T::vec8* qf, const typename T::vec8* df, float c, float ls, int seen, int seen_most, float& sum_p, float& sum_pdp, float& sum_abs)
{
    const int half = (threadIdx.x % 64) / 32;
    sum_p = sum_pdp = sum_abs = 0;
#pragma unroll 1
    for (int kb = 0; kb < seen_most; kb += 32) {
        f32x16 s, dp;
        dq_scores<T, D>(lds + kb / STEP * (2 * STEP * D * 2), kb % STEP, qf, df, s, dp);
        int first = seen - kb - 4 * half;       // key that the row does not see
        stay_here(first);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const bool sees = c_row(r, 0) < first;
            const float p = exp2_(fmaf(s[r], c, -ls));
            sum_p += sees ? p : 0.0f;
            sum_pdp += sees ? p * dp[r] : 0.0f;
            sum_abs += sees ? p * fabsf(dp[r]) : 0.0f;
        }
    }
    sum_p += other_half(sum_p);
    sum_pdp += other_half(sum_pdp);
    sum_abs += other_half(sum_abs);
}

template <class T, int D, int WAVES>
__device__ __forceinline__ void dq_step(const lds_char* __restrict cur, lds_char* __restrict next, const Next& n, const TileLoads<STEP, D, WAVES>& la, const TileLoads<STEP, D, WAVES>& lb, const typename T::vec8* qf,
                                        const typename T::vec8* df, f32x16* dq, float c, float ls, float de, float per, int key0, int seen, int seen_least, int seen_most)
{
    constexpr int DB = D / 32;
    const int half = (threadIdx.x % 64) / 32;
    if (n.more) {
        la.load(next, n.a, n.rows);
        lb.load(next + STEP * D * 2, n.b, n.rows);
    }
    const lds_char* kt = cur;
#pragma unroll 1
    for (int b = 0; b < STEP / 32; ++b) {
        const int kb = key0 + b * 32;
        if (kb >= seen_most) break;
        f32x16 s, dp;
        dq_scores<T, D>(kt, b * 32, qf, df, s, dp);
        float ds[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = exp2_(fmaf(s[r], c, -ls)) * fmaf(dp[r], per, -de);
        if (kb + 32 > seen_least) {
            int first = seen - kb - 4 * half;       // key that the row does not see
            stay_here(first);
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] = c_row(r, 0) >= first ? 0.0f : ds[r];
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const typename T::vec8 dsf = round8<T>(ds + st * 8);
#pragma unroll
            for (int d = 0; d < DB; ++d) dq[d] = T::mma(across<T, D>(kt, b * 32 + st * 16, d * 32), dsf, dq[d]);
        }
        interleave<2 * DB, 2, 3, 2>();
    }
}

template <class T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void k_attention_dq(AttnArgs a)
{
    constexpr int DB = D / 32, TILE = STEP * D * 2;
    __shared__ __attribute__((aligned(256))) char lds_[4 * TILE];
    lds_char* lds = (lds_char*)lds_;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const uint32_t bk = heads_of_block(a), b = bk / a.kv_heads, kh = bk % a.kv_heads;
    const Rows w = rows_of_wave<WAVES>(a, b, kh, wave, lane);
    const int nk = w.nk, chunks = a.dim / 8;
    int t0 = 0, t1 = (w.keys + STEP - 1) / STEP;
    const bool few = t1 <= 2;           // all tiles of keys that the block sees fit LDS together: one split takes them
    if (a.splits > 1) {
        const int run = few ? t1 : (t1 + (int)a.splits - 1) / (int)a.splits;
        t0 = min(t1, run * (int)blockIdx.z);
        t1 = min(t1, t0 + run);
    }
    const char* kp = a.k.p + b * a.k.batch + kh * a.k.head;
    const char* vp = a.v.p + b * a.v.batch + kh * a.v.head;
    const bool query = w.in && (int)w.i < w.nq;
    typename T::vec8 qf[D / 16], df[D / 16], of[D / 16];
    row_operand<T, D>(qf, query ? a.q.p + b * a.q.batch + w.h * a.q.head + w.i * a.q.pos : nullptr, a.dim, half);
    row_operand<T, D>(df, query ? a.dout.p + b * a.dout.batch + w.h * a.dout.head + w.i * a.dout.pos : nullptr, a.dim, half);
    const uint64_t at = ((uint64_t)b * a.heads + w.h) * a.q_len + w.i;
    row_operand<T, D>(of, query ? a.o.p + b * a.o.batch + w.h * a.o.head + w.i * a.o.pos : nullptr, a.dim, half);
    float ls = query ? a.lse[at] : -INFINITY;
    TileLoads<STEP, D, WAVES> kl, vl;
    kl.init(a.k.pos, chunks);
    vl.init(a.v.pos, chunks);
    if (t0 < t1) {
        kl.load(lds, kp + (int64_t)t0 * STEP * a.k.pos, nk - t0 * STEP);
        vl.load(lds + TILE, vp + (int64_t)t0 * STEP * a.v.pos, nk - t0 * STEP);
    }
    if (few && t1 == 2) {
        kl.load(lds + 2 * TILE, kp + (int64_t)STEP * a.k.pos, nk - STEP);
        vl.load(lds + 3 * TILE, vp + (int64_t)STEP * a.v.pos, nk - STEP);
    }
    ls = ls != -INFINITY ? ls * LOG2E : INFINITY;
    float de = 0, top = 0, oo = 0;
    float slack = 0;                // how far the rounding of o can take <do, o>
    int unit = 0;                   // exponent
#pragma unroll
    for (int st = 0; st < D / 16; ++st)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            de += (float)df[st][e] * (float)of[st][e];
            slack += fabsf((float)df[st][e]) * fabsf((float)of[st][e]);
            top = fmaxf(top, fabsf((float)df[st][e]));
            oo += (float)of[st][e] * (float)of[st][e];
        }
    de += other_half(de);
    slack += other_half(slack);
    top = fmaxf(top, other_half(top));
    slack = fmaf(slack, HALF_STEP<T>, top * (D * HALF_LEAST<T>));
    if constexpr (std::is_same<T, F16>::value) {
        unit = exponent(top);
        // what bounds the keys' side: the largest of the wave's rows; do as a vector is no longer than sqrt(D) times its largest element
        oo += other_half(oo);
        float2 most = make_float2(top * (D == 64 ? 8.0f : 11.32f), 0);
        most.y = most.x * __builtin_amdgcn_sqrtf(oo);
#pragma unroll
        for (int d = 16; d; d >>= 1) most = make_float2(fmaxf(most.x, __shfl_xor(most.x, d)), fmaxf(most.y, __shfl_xor(most.y, d)));
        if (lane == 0 && blockIdx.z == 0) a.top[(uint64_t)bk * a.tops + (gridDim.y - 1 - blockIdx.y) * WAVES + wave] = most;
    }
    __syncthreads();
    // The rounding of o to the type is in <do, o> for all keys of the row alike, and where few keys share the probability it is the largest error of
    // dq and dk (2^-8 and 8 causal keys: 3.5e-3 of dq, without it 2.3e-3; 128 keys: 2.7e-3).  The sum of p dp has no such part.  It takes the scores twice,
    // so it is taken where that costs no load; and only if these keys hold all of the probability, which they do not where o and lse are
    // of more keys than the call's.  That the probabilities sum to 1, as far as the rounding of lse lets them, does not say so by itself: values of the other keys may be large
    // enough for the rest to count.  But then <do, o> differs from the sum by more than the roundings of o, and of the probabilities that made it, explain.
    if (few && t0 < t1) {
        float sum_p, sum_pdp, sum_abs;
        dq_row_sums<T, D>(lds, qf, df, a.scale_log2, ls, w.seen, w.seen_most, sum_p, sum_pdp, sum_abs);
        if (fabsf(sum_p - 1.0f) < 0x1p-14f * (1.0f + fabsf(ls) * 0x1p-5f) && fabsf(sum_pdp - de) <= fmaf(sum_abs, HALF_STEP<T>, slack)) de = sum_pdp;
        if (std::is_same<T, F16>::value) unit = exponent(sum_abs + fabsf(de)) - 14;
    }
    if (w.in && half == 0 && blockIdx.z == 0) a.delta[at] = de, a.lse2[at] = ls - P_SHIFT<T>;
    f32x16 dq[DB];
#pragma unroll 1
    for (bool again = false;; again = true) {
#pragma unroll
        for (int d = 0; d < DB; ++d) dq[d] = f32x16{};
        const float du = ldexpf(de, -unit), per = ldexpf(1.0f, -unit);
        for (int t = t0; t < t1; ++t) {
            const int now = ((t - t0) & 1) * 2 * TILE, k1 = (t + 1) * STEP;
            const Next n = {kp + (int64_t)k1 * a.k.pos, vp + (int64_t)k1 * a.v.pos, nk - k1, !few && t + 1 < t1};
            dq_step<T, D, WAVES>(lds + now, lds + (2 * TILE - now), n, kl, vl, qf, df, dq, a.scale_log2, ls, du, per, t * STEP, w.seen, w.seen_least, w.seen_most);
            __syncthreads();
        }
        if (!std::is_same<T, F16>::value || few || again) break;
        float z = 0;                // a NaN where a sum is infinite, or one
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) z = fmaf(dq[d][r], 0.0f, z);
        z += other_half(z);
        // all waves of a block start again, since they load together
        const bool left = !(z == 0);
        if (!any_of_block<WAVES>(left, lds)) break;
        if (left) unit += MORE_EXPONENT;
        if (t0 < t1) {
            kl.load(lds, kp + (int64_t)t0 * STEP * a.k.pos, nk - t0 * STEP);
            vl.load(lds + TILE, vp + (int64_t)t0 * STEP * a.v.pos, nk - t0 * STEP);
        }
        __syncthreads();
    }
    if (!w.in) return;
    const float f = ldexpf(a.scale, unit);
    if (a.splits > 1) {
        float* p = a.part + ((uint64_t)blockIdx.z * a.batch * a.heads * a.q_len + at) * a.dim;
#pragma unroll
        for (int d = 0; d < DB; ++d) store_part(p, dq[d], d * 32, a.dim, half, f);
        return;
    }
    char* p = a.dq.p + b * a.dq.batch + w.h * a.dq.head + w.i * a.dq.pos;
#pragma unroll
    for (int d = 0; d < DB; ++d) store_row<T>(p, dq[d], d * 32, a.dim, half, f);
}

// sums of partial sums of rows of heads: part [splits][count][batch * heads * len][dim], of which `which` is meant
template <class T>
__global__ __launch_bounds__(256) void k_attention_add(const float* part, uint32_t splits, uint32_t count, Heads o0, Heads o1, uint32_t batch, uint32_t heads, uint32_t len, uint32_t dim)
{
    const uint64_t n = (uint64_t)batch * heads * len, at = (uint64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const uint32_t x = (threadIdx.x % 16) * 8;
    if (at >= n || x >= dim) return;
    float s[8] = {};
    for (uint32_t k = 0; k < splits; ++k) {
        const float* p = part + (((uint64_t)k * count + blockIdx.y) * n + at) * dim + x;
        const f32x4 u = *(const f32x4*)p, v = *(const f32x4*)(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += u[e], s[4 + e] += v[e];
    }
    const Heads o = blockIdx.y ? o1 : o0;
    const uint64_t i = at % len, bh = at / len;
    *(typename T::vec8*)(o.p + bh / heads * o.batch + bh % heads * o.head + i * o.pos + x * 2) = round8<T>(s);
}

int check_backward(const ff_attention_bwd_t* p)
{
    if (const int rc = check_attention(p)) return rc;
    return p->kv_len > FF_OP_MAX_SIDE ? FF_ERANGE : FF_OK;         // blocks of 128 keys
}

uint32_t waves_of(uint64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

// Work is split over the other axis where the owners alone leave some of the device's 256 compute units without a block: more than half of them by no more than leaves a split four
// tiles; fewer, where the longest block is long enough (32 tiles a split) to pay for the partial sums' way through memory.  Keys' side, 128 blocks of up to 128 tiles
// (32 heads on 8, 2048 x 2048, causal): 308 us for all without, 213 with four splits; 224 blocks of 28 tiles: 89 us without, 101 with two.
uint32_t splits_of(uint64_t blocks, uint64_t tiles)
{
    if (blocks == 0 || blocks >= 256) return 1;
    return (uint32_t)std::max<uint64_t>(1, blocks < 128 ? std::min<uint64_t>(256 / blocks, tiles / 4) : std::min<uint64_t>(512 / blocks, tiles / 32));
}

struct Plan {
    uint32_t kv_waves, kv_splits, q_waves, q_splits, tops;
    uint64_t lse2, top, part, bytes;        // offsets in the workspace, delta first
};

Plan plan_of(const AttnArgs& a)
{
    Plan p = {};
    const uint64_t rows = (uint64_t)a.q_len * a.group, bk = (uint64_t)a.batch * a.kv_heads;
    p.kv_waves = waves_of(a.kv_len), p.q_waves = waves_of(rows);
    p.kv_splits = splits_of(bk * ceil_div(a.kv_len, p.kv_waves * 32), a.group * ceil_div(a.q_len, STEP));
    p.q_splits = splits_of(bk * ceil_div(rows, p.q_waves * 32), ceil_div(a.kv_len, STEP));
    p.lse2 = round_up((uint64_t)a.batch * a.heads * a.q_len * sizeof(float), 256);
    p.top = 2 * p.lse2;
    p.tops = (uint32_t)ceil_div(rows, p.q_waves * 32) * p.q_waves;
    p.part = p.top + round_up(bk * p.tops * sizeof(float2), 256);
    // one area for the partial sums of both: the kernels run one after another
    const uint64_t kv = p.kv_splits > 1 ? 2ull * p.kv_splits * bk * a.kv_len * a.dim : 0, q = p.q_splits > 1 ? (uint64_t)p.q_splits * bk * rows * a.dim : 0;
    p.bytes = p.part + std::max(kv, q) * sizeof(float);
    return p;
}

template <class T, int D>
void launch_dkv(const AttnArgs& a, uint32_t w, hipStream_t st)
{
    const dim3 grid(a.batch * a.kv_heads, (uint32_t)ceil_div(a.kv_len, w * 32), a.splits);
    if (w == 1) k_attention_dkv<T, D, 1><<<grid, 64, 0, st>>>(a);
    else if (w == 2) k_attention_dkv<T, D, 2><<<grid, 128, 0, st>>>(a);
    else k_attention_dkv<T, D, 4><<<grid, 256, 0, st>>>(a);
}

template <class T, int D>
void launch_dq(const AttnArgs& a, uint32_t w, hipStream_t st)
{
    const dim3 grid(a.batch * a.kv_heads, (uint32_t)ceil_div((uint64_t)a.q_len * a.group, w * 32), a.splits);
    if (w == 1) k_attention_dq<T, D, 1><<<grid, 64, 0, st>>>(a);
    else if (w == 2) k_attention_dq<T, D, 2><<<grid, 128, 0, st>>>(a);
    else k_attention_dq<T, D, 4><<<grid, 256, 0, st>>>(a);
}

template <class T>
int run(AttnArgs a, const Plan& p, hipStream_t st)
{
    if (a.q_len) {          // first: delta and the largest |do| are what the keys' side needs of it
        a.splits = p.q_splits;
        if (a.dim <= 64) launch_dq<T, 64>(a, p.q_waves, st);
        else launch_dq<T, 128>(a, p.q_waves, st);
        if (a.splits > 1)
            k_attention_add<T><<<dim3((uint32_t)ceil_div((uint64_t)a.batch * a.heads * a.q_len, 16), 1), 256, 0, st>>>(a.part, a.splits, 1, a.dq, a.dq, a.batch, a.heads, a.q_len, a.dim);
    }
    if (a.kv_len) {
        a.splits = p.kv_splits;
        if (a.dim <= 64) launch_dkv<T, 64>(a, p.kv_waves, st);
        else launch_dkv<T, 128>(a, p.kv_waves, st);
        if (a.splits > 1)
            k_attention_add<T><<<dim3((uint32_t)ceil_div((uint64_t)a.batch * a.kv_heads * a.kv_len, 16), 2), 256, 0, st>>>(a.part, a.splits, 2, a.dk, a.dv, a.batch, a.kv_heads, a.kv_len, a.dim);
    }
    return launched();
}

}  // namespace
}  // namespace ffops

using namespace ffops;

extern "C" size_t ff_op_attention_bwd_workspace_bytes(const ff_attention_bwd_t* p)
{
    if (!p || check_backward(p) != FF_OK) return 0;
    return plan_of(args_of(p)).bytes;
}

extern "C" int ff_op_attention_bwd(const ff_attention_bwd_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check_backward(p)) return rc;
    if (p->batch == 0 || (p->q_len == 0 && p->kv_len == 0)) return FF_OK;
    if (p->q_len && (!heads_ok(p->q) || !heads_ok(p->o) || !heads_ok(p->dout) || !heads_ok(p->dq) || !p->lse)) return FF_EINVAL;
    if (p->kv_len && (!heads_ok(p->k) || !heads_ok(p->v) || !heads_ok(p->dk) || !heads_ok(p->dv))) return FF_EINVAL;
    AttnArgs a = args_of(p);
    const Plan plan = plan_of(a);
    if (plan.bytes && (!p->workspace || p->workspace_bytes < plan.bytes || !aligned(p->workspace, 256))) return FF_EWORKSPACE;
    a.dout = in_bytes(p->dout), a.dq = in_bytes(p->dq), a.dk = in_bytes(p->dk), a.dv = in_bytes(p->dv);
    a.lse = const_cast<float*>(p->lse);
    char* ws = (char*)p->workspace;
    a.delta = (float*)ws;
    a.lse2 = (float*)(ws + plan.lse2);
    a.top = (float2*)(ws + plan.top), a.tops = plan.tops;
    a.part = (float*)(ws + plan.part);
    return p->dtype == FF_F16 ? run<F16>(a, plan, (hipStream_t)stream) : run<BF16>(a, plan, (hipStream_t)stream);
}
