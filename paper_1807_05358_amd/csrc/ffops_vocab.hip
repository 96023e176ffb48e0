// Softmax cross entropy over a vocabulary, forward and backward, from the vectors and the vocabulary's matrix.
#include "ffops_tiles.h"
#include "ffops_vocab_tiling.h"

namespace ffops {
namespace {

struct Mat {
    const char* p;
    int64_t stride;         // bytes from row to row
};

// One side of a product over k, as a block sees it.  Along: p is the tile's first row, rows of k elements; across: p is the
// tile's first column, rows of the tile's elements, one per k.  `count`: rows (columns) of the tile that exist; `ks`: values of k
// that exist, along in multiples of 8 (with zeros where the other side has none).
struct Side {
    Mat m;
    int count;
    int64_t ks;
};

template <int SIZE, int KT, bool ACROSS, int WAVES>
__device__ __forceinline__ void stage_side(lds_char* dst, const Side& s, int64_t k)
{
    const int left = (int)min(s.ks - k, (int64_t)KT);
    if constexpr (ACROSS) stage<KT, SIZE, WAVES>(dst, s.m.p + k * s.m.stride, s.m.stride, left, (s.count + 7) / 8);
    else stage<SIZE, KT, WAVES>(dst, s.m.p + k * 2, s.m.stride, s.count, left / 8);
}

template <class T, int SIZE, int KT, bool ACROSS>
__device__ __forceinline__ typename T::vec8 operand(const lds_char* tile, int at, int step)
{
    if constexpr (ACROSS) return across16<T, SIZE>(tile, step, at);
    else return along16<T, KT>(tile, at, step);
}

// The product of a block: c[m][n] += sum_k a[m][k] b[n][k] over k0 .. k1, M x N of it in WM x WN waves of 16 x 16 tiles, the
// tiles of both sides loaded straight into LDS, STAGES - 1 tiles of k ahead.  Along sides have k in multiples of 8.  A tile of k of 64 x 64 is 8 products of a wave, far less than
// memory takes to answer, so a block alone on its unit needs more than one on the way: 64 x 2472 x 3280 backward (39 blocks) 62 us with two stages, 49 with three, 49 with four.
// 128 x 128 with three leaves room for one block on a unit instead of two: 982 x 4635 x 1892 forward 59 us, 75 then.
template <class T, int M, int N, int WAVES_M, int WAVES_N, bool A_ACROSS, bool B_ACROSS>
struct Product {
    static constexpr int KT = 64;       // k of a tile in LDS
    static constexpr int WM = WAVES_M, WN = WAVES_N, WAVES = WM * WN, TM = M / WM / 16, TN = N / WN / 16, A_BYTES = M * KT * 2, BYTES = (M + N) * KT * 2;
    static constexpr int STAGES = M == 64 ? 3 : 2, LDS = STAGES * BYTES, LOADS = BYTES / 1024 / WAVES;

    static __device__ __forceinline__ void load(lds_char* __restrict dst, const Side& a, const Side& b, int64_t k)
    {
        stage_side<M, KT, A_ACROSS, WAVES>(dst, a, k);
        stage_side<N, KT, B_ACROSS, WAVES>(dst + A_BYTES, b, k);
    }

    template <bool LOAD>
    static __device__ __forceinline__ void step(const lds_char* __restrict cur, lds_char* __restrict into, const Side& a, const Side& b, int64_t k, f32x4 (&c)[TM][TN], int wm, int wn)
    {
        if (LOAD) load(into, a, b, k);
#pragma unroll
        for (int st = 0; st < KT / 32; ++st) {
            typename T::vec8 fa[TM], fb[TN];
#pragma unroll
            for (int n = 0; n < TN; ++n) fb[n] = operand<T, N, KT, B_ACROSS>(cur + A_BYTES, wn + n * 16, st);
#pragma unroll
            for (int m = 0; m < TM; ++m) fa[m] = operand<T, M, KT, A_ACROSS>(cur, wm + m * 16, st);
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int n = 0; n < TN; ++n) c[m][n] = T::mma(fa[m], fb[n], c[m][n]);
        }
    }

    static __device__ __forceinline__ void run(lds_char* lds, const Side& a, const Side& b, int64_t k0, int64_t k1, f32x4 (&c)[TM][TN], int wm, int wn)
    {
        for (int j = 0; j < STAGES - 1 && k0 + j * KT < k1; ++j) load(lds + j * BYTES, a, b, k0 + j * KT);
        int now = 0;
        int64_t k = k0;
        for (; k + (STAGES - 1) * KT < k1; k += KT) {
            meet<(STAGES - 2) * LOADS>();           // the tile is there, and the one before has been read by all
            step<true>(lds + now, lds + (now == 0 ? (STAGES - 1) * BYTES : now - BYTES), a, b, k + (STAGES - 1) * KT, c, wm, wn);
            now = now == (STAGES - 1) * BYTES ? 0 : now + BYTES;
        }
        meet<0>();
        for (; k < k1; k += KT) {
            step<false>(lds + now, lds, a, b, k, c, wm, wn);
            now = now == (STAGES - 1) * BYTES ? 0 : now + BYTES;
        }
        meet<0>();
    }
};

// The same product of 256 x 256 tiles by four waves, one on each SIMD, 128 x 128 each: 16 products of 32 in k need four operands
// of 16 rows and four of 16 columns, a third less from LDS than waves of 128 x 64 would read, and LDS is what two waves a SIMD wait for (its
// reads and the loads' writes share it).  Half a tile of k is 64 products of a wave, 1024 cycles of its SIMD's matrix unit, in eight rows of eight.
// Between the products the wave reads, two rows ahead, the row's operand of a, one of the next half's of b, and starts one load.
// LDS holds three tiles of a and two of b, all of its 160 KB.  Half 0 of tile s starts the loads of a's tile s + 2, half 1 those of b's, whose buffer has been
// read by then; half 1 reads the first operands of tile s + 1, which have had a half at least to arrive.
template <class T, bool A_ACROSS, bool B_ACROSS>
struct Wide {
    static constexpr int KT = 64;               // rows of 128 bytes: caches are asked for whole lines
    static constexpr int M = 256, N = 256, WM = 2, WN = 2, WAVES = 4, TM = 8, TN = 8, TILE = 256 * KT * 2, LDS = 5 * TILE;
    typedef Stager<A_ACROSS ? KT : M, A_ACROSS ? M : KT, WAVES> StageA;
    typedef Stager<B_ACROSS ? KT : N, B_ACROSS ? N : KT, WAVES> StageB;
    typedef typename T::vec8 vec8;
    static constexpr int LOADS = StageA::PER;   // of a wave, for a tile of either side
    static_assert(StageA::PER == 8 && StageB::PER == 8, "one load for every row of products");

    static __device__ __forceinline__ const char* at(const Side& s, bool across, int64_t k) { return across ? s.m.p + k * s.m.stride : s.m.p + k * 2; }
    static __device__ __forceinline__ vec8 of_a(const lds_char* tile, int half, int m, int wm) { return operand<T, M, KT, A_ACROSS>(tile, wm + m * 16, half); }
    static __device__ __forceinline__ vec8 of_b(const lds_char* tile, int half, int n, int wn) { return operand<T, N, KT, B_ACROSS>(tile, wn + n * 16, half); }

    // the products of half HALF of a tile whose a is at `a`; the next half's operands are in `an` and `bn`.  fa: the row's operand and the next two.
    template <int HALF, int LOAD, class S>
    static __device__ __forceinline__ void half(const lds_char* __restrict a, const lds_char* __restrict an, const lds_char* __restrict bn, lds_char* __restrict into, const char* from, const S& stage,
                                                vec8 (&fa)[4], const vec8 (&fb)[TN], vec8 (&gb)[TN], f32x4 (&c)[TM][TN], int wm, int wn)
    {
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            gb[m] = of_b(bn, 1 - HALF, m, wn);
#pragma unroll
            for (int n = 0; n < 3; ++n) T::mma_acc(fa[m % 4], fb[n], c[m][n]);
            fa[(m + 2) % 4] = m + 2 < TM ? of_a(a, HALF, m + 2, wm) : of_a(an, 1 - HALF, m + 2 - TM, wm);
#pragma unroll
            for (int n = 3; n < 6; ++n) T::mma_acc(fa[m % 4], fb[n], c[m][n]);
            if (LOAD) stage.load_one(into, from, m);
#pragma unroll
            for (int n = 6; n < TN; ++n) T::mma_acc(fa[m % 4], fb[n], c[m][n]);
        }
    }

    static __device__ __forceinline__ void run(lds_char* lds, const Side& a, const Side& b, int64_t k0, int64_t k1, f32x4 (&c)[TM][TN], int wm, int wn)
    {
        if (k0 >= k1) return;
        StageA sa;
        StageB sb;
        sa.init(a.m.stride, A_ACROSS ? KT : a.count, A_ACROSS ? (a.count + 7) / 8 : KT / 8);
        sb.init(b.m.stride, B_ACROSS ? KT : b.count, B_ACROSS ? (b.count + 7) / 8 : KT / 8);
        // the order of k is free: what is no whole tile comes first, so that the loop has whole ones
        const int64_t wholes = (min(k1, min(a.ks, b.ks)) - k0) / KT, rest = k0 + wholes * KT;
        const int odd = rest < k1;
        int left = (int)wholes + odd;
        lds_char* lb = lds + 3 * TILE;
        for (int j = 0; j < 2 && j < left; ++j) {
            if (j < odd) {
                stage_side<M, KT, A_ACROSS, WAVES>(lds, a, rest);
                stage_side<N, KT, B_ACROSS, WAVES>(lb, b, rest);
            } else {
                sa.load(lds + j * TILE, at(a, A_ACROSS, k0 + (j - odd) * KT));
                sb.load(lb + j * TILE, at(b, B_ACROSS, k0 + (j - odd) * KT));
            }
        }
        const int64_t as = A_ACROSS ? KT * a.m.stride : KT * 2, bs = B_ACROSS ? KT * b.m.stride : KT * 2;
        const char *pa = at(a, A_ACROSS, k0 + (2 - odd) * KT), *pb = at(b, B_ACROSS, k0 + (2 - odd) * KT);
        vec8 fa[4], fb[TN], gb[TN];
        meet<0>();
        fa[0] = of_a(lds, 0, 0, wm), fa[1] = of_a(lds, 0, 1, wm);
#pragma unroll
        for (int n = 0; n < TN; ++n) fb[n] = of_b(lb, 0, n, wn);
        int ia = 0, ib = 0;
        for (; left > 2; --left) {
            const int next = ia == 2 * TILE ? 0 : ia + TILE, free = next == 2 * TILE ? 0 : next + TILE;
            half<0, 1>(lds + ia, lds + ia, lb + ib, lds + free, pa, sa, fa, fb, gb, c, wm, wn);
            meet<LOADS>();
            half<1, 1>(lds + ia, lds + next, lb + (TILE - ib), lb + ib, pb, sb, fa, gb, fb, c, wm, wn);
            meet<2 * LOADS>();                   // for the reads alone
            pa += as, pb += bs;
            ia = next, ib = TILE - ib;
        }
        for (; left > 0; --left) {              // the last operands read are of what is there, and not used
            const int next = ia == 2 * TILE ? 0 : ia + TILE;
            half<0, 0>(lds + ia, lds + ia, lb + ib, lds, pa, sa, fa, fb, gb, c, wm, wn);
            meet<0>();
            half<1, 0>(lds + ia, lds + next, lb + (TILE - ib), lb, pb, sb, fa, gb, fb, c, wm, wn);
            meet<0>();
            ia = next, ib = TILE - ib;
        }
        // the last products write their registers some cycles after they were issued, of which the compiler knows nothing
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
        for (int m = 0; m < TM; ++m) asm volatile("" : "+a"(c[m][0]), "+a"(c[m][1]), "+a"(c[m][2]), "+a"(c[m][3]), "+a"(c[m][4]), "+a"(c[m][5]), "+a"(c[m][6]), "+a"(c[m][7]));
    }
};

// Blocks go to the 8 dies in turn, each with a cache of its own: a die takes a run of tiles, in groups of 8 along m, so that what
// runs at one time on a die shares its rows of both sides.
__device__ __forceinline__ void tile_of_block(uint32_t id, uint32_t ms, uint32_t ns, uint32_t& m, uint32_t& n)
{
    const uint32_t total = ms * ns, die = id % 8, each = total / 8, rest = total % 8;
    const uint32_t at = die * each + min(die, rest) + id / 8;
    const uint32_t group = at / (8 * ns), first = group * 8, size = min(8u, ms - first), in = at - group * 8 * ns;
    m = first + in % size;
    n = in / size;
}

struct VocabArgs {
    uint32_t rows, dim, words, word0;       // words of this piece, the first of them in the matrix
    uint32_t m_tiles, n_tiles;
    int32_t ignore, first_word;
    Mat x, w;
    const int32_t* targets;
    const float *dloss, *lse_in;
    // Backward: the number of rows that take part, and the bits of their largest |dloss|; row_of has them, in their order, and the others behind.
    // Where there are others, or x does not suit the products, `gathered` has theirs of x: what is in the others reaches no product, and they take no time.
    const uint32_t *live, *row_of;
    Mat gathered;
    float2* part;                           // [rows][m_tiles]: maximum and sum of a tile's words
    float* target_logit;
    char* g;                                // [rows][g_stride]: gradient of the logits of a piece
    uint32_t g_stride;
    float* sum;                             // [splits][rows or words][dim]: dx, over pieces and splits; dw, over splits
    uint32_t splits, first, whole;          // dx: the first piece; one piece and no splits, so that dx is written at once
    char* out;
    int64_t out_stride;                     // bytes
    uint32_t out_vec;                       // rows of the output take 8-byte stores
};

// four neighbouring elements of a row of an output, those below `n`
template <class T>
__device__ __forceinline__ void store_out(char* row, uint32_t x, uint32_t n, bool vec, float a, float b, float c, float d)
{
    if (vec && x + 4 <= n) store4<T>(row + x * 2, a, b, c, d);
    else {
        typename T::elem* p = (typename T::elem*)row;
        if (x < n) p[x] = (typename T::elem)a;
        if (x + 1 < n) p[x + 1] = (typename T::elem)b;
        if (x + 2 < n) p[x + 2] = (typename T::elem)c;
        if (x + 3 < n) p[x + 3] = (typename T::elem)d;
    }
}

// A tile of an output, whose rows are the columns of the products in c, times f: rounded into LDS, which all have read, and from there row by row, so that a wave writes whole lines.  `cols`, `rows`:
// what of it exists; of(r): the output's row of the tile's row r.  From the registers a wave's store is 32 bytes of each of 16 rows, or, where rows start anywhere, 2 bytes of each:
// dw of 16 x 15216 x 3754, of which storing is nearly all, 107 us then, 49 us this way.  All of
// 8192 x 50257 x 2048 4017 us then, 3750 to 3830 this way.
template <class T, class P, int M, class RowOf>
__device__ __forceinline__ void store_tile(lds_char* lds, const f32x4 (&c)[P::TM][P::TN], float f, char* out, int64_t stride, int rows, int cols, int wm, int wn, RowOf of)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
    constexpr int PITCH = M * 2 + 16, THREADS = P::WM * P::WN * 64;
    static_assert(M * PITCH <= P::LDS, "a tile of the result fits in the place of the factors'");
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int n = 0; n < P::TN; ++n)
#pragma unroll
        for (int m = 0; m < P::TM; ++m) *(lds_u32x2*)(lds + (wn + n * 16 + lane % 16) * PITCH + (wm + m * 16 + lane / 16 * 4) * 2) = __builtin_bit_cast(u32x2, pack4<T>(c[m][n] * f));
    __syncthreads();
    typedef u32x4 out16 __attribute__((aligned(2)));        // the device takes them anywhere
#pragma unroll 4
    for (int i = threadIdx.x; i < M * M / 8; i += THREADS) {
        const int r = i / (M / 8), x = i % (M / 8) * 8;
        if (r >= rows || x >= cols) continue;
        const lds_char* from = lds + r * PITCH + x * 2;
        char* to = out + of(r) * stride + x * 2;
        if (x + 8 <= cols) *(out16*)to = *(__attribute__((address_space(3))) const u32x4*)from;
        else
            for (int e = 0; e < cols - x; ++e) ((uint16_t*)to)[e] = ((__attribute__((address_space(3))) const uint16_t*)from)[e];
    }
}

// z^T = w x^T: words down, tokens across, so that a lane holds words of one token.  2560 x 32768 x 1024 forward: 141 to 149 us with its join, 1150 to 1220 TFLOP/s, matrix units busy 51 %, the rest
// the tiles' beginnings and ends around 16 steps of k; 64 x 32768 x 1024: 14 us, w's bytes at 4.8 TB/s.  The gradient of 7782 x 16384 x 2048: 449 us, 1163 TFLOP/s,
// with 255 MB of g written.  GRAD false: maximum and sum of exp per
// token and tile of words, and the target's logit; GRAD true: the gradient of the logits, rounded, into g.
// g is kept relative to the largest |dloss| and times a power of two.  Where all rows weigh the same, a row's entry for its target is then
// p - 1, which for a small p rounds to nearly itself; and a 16-bit float's exponents do not hold a probability of 1 / vocabulary times a loss' weight.
// 2^15 keeps them, and 1 stays below its largest number: a step of g is 2^-39 of the largest |dloss| at least (rows of smaller weight have no smaller one).  With bfloat 2^40 keeps probabilities that a float's exponents do not hold.
template <class T>
constexpr float G_SHIFT = std::is_same<T, F16>::value ? 15.0f : 40.0f;

__device__ __forceinline__ uint32_t live_rows(const VocabArgs& a) { return a.live[0]; }
__device__ __forceinline__ Mat live_x(const VocabArgs& a, uint32_t rows) { return rows == a.rows && a.x.p ? a.x : a.gathered; }

__device__ __forceinline__ float unit_of(const VocabArgs& a)
{
    const float m = __uint_as_float(a.live[1]);
    return m > 0 && m < INFINITY ? m : 1.0f;
}

// maximum (a power of two's exponent) and sum of two sets; an empty one has -inf and 0
__device__ __forceinline__ float2 join(float2 s, float2 o)
{
    const float top = fmaxf(s.x, o.x), base = top == -INFINITY ? 0.0f : top;
    return make_float2(top, s.y * exp2_(s.x - base) + o.y * exp2_(o.x - base));
}

// the product of a tile size
template <class T, int M, bool A_ACROSS, bool B_ACROSS>
struct ProductOf {
    typedef Product<T, M, M, 2, 2, A_ACROSS, B_ACROSS> type;
};
template <class T, bool A_ACROSS, bool B_ACROSS>
struct ProductOf<T, 256, A_ACROSS, B_ACROSS> {
    typedef Wide<T, A_ACROSS, B_ACROSS> type;
};

template <class T, int M, bool GRAD>
__global__ __launch_bounds__(256) void k_vocab_logits(VocabArgs a)
{
    typedef typename ProductOf<T, M, false, false>::type P;
    constexpr int N = M, WM = P::WM, WN = P::WN;
    __shared__ __attribute__((aligned(256))) char lds_[P::LDS];
    lds_char* lds = (lds_char*)lds_;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), quarter = lane / 16;
    const int wm = wave / WN * (M / WM), wn = wave % WN * (N / WN);
    const uint32_t rows = GRAD ? live_rows(a) : a.rows, n_tiles = GRAD ? (rows + N - 1) / N : a.n_tiles;
    if (GRAD && blockIdx.x >= a.m_tiles * n_tiles) return;
    uint32_t tm, tn;
    tile_of_block(blockIdx.x, a.m_tiles, n_tiles, tm, tn);
    const uint32_t m0 = tm * M, n0 = tn * N;
    const Mat x = GRAD ? live_x(a, rows) : a.x;
    const Side sw = {{a.w.p + (int64_t)(a.word0 + m0) * a.w.stride, a.w.stride}, (int)min(a.words - m0, (uint32_t)M), a.dim};
    const Side sx = {{x.p + (int64_t)n0 * x.stride, x.stride}, (int)min(rows - n0, (uint32_t)N), a.dim};
    f32x4 c[P::TM][P::TN];
#pragma unroll
    for (int m = 0; m < P::TM; ++m)
#pragma unroll
        for (int n = 0; n < P::TN; ++n) c[m][n] = f32x4{};
    P::run(lds, sw, sx, 0, a.dim, c, wm, wn);
    float2* stat = (float2*)lds_;           // [WM][N], the tiles have been read
#pragma unroll
    for (int n = 0; n < P::TN; ++n) {
        const uint32_t token = n0 + wn + n * 16 + lane % 16;
        const bool in = token < rows;
        const uint32_t of = GRAD && in ? a.row_of[token] : token;
        const int32_t target = in ? a.targets[of] : a.ignore;
        const bool live = target != a.ignore;
        // the target's place among the words that the lane holds: register r of tile m has word 16 * m + r after its first
        const uint32_t v0 = m0 + wm + 4 * quarter;
        const int64_t at = (int64_t)target - a.first_word - a.word0 - v0;
        const int want = live && at >= 0 && at < M ? (int)at : -1;
        const bool edge = m0 + M > a.words;
        // almost no tile has a lane's target or the last word
        if constexpr (GRAD) {
            // a row that takes no part has exp(-inf)
            const float lse = live ? a.lse_in[of] : INFINITY, ls = fmaf(lse, LOG2E, -G_SHIFT<T>), f = live ? a.dloss[of] / unit_of(a) : 0;
            // The target's entry is p - 1, to which the rounding of ls (2^-19 with bfloat) would be what is left of it where p is near 1: it is made from the difference itself.
            float gt = 0;
            const bool targets = __any(want >= 0);
            if (targets) {
#pragma unroll
                for (int m = 0; m < P::TM; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) gt = m * 16 + e == want ? c[m][n][e] : gt;
                gt = (exp2_((gt - lse) * LOG2E) - 1.0f) * (exp2f(G_SHIFT<T>) * f);
            }
            char* row = a.g + ((uint64_t)token * a.g_stride + v0 + (quarter & 1) * 12) * 2;
#pragma unroll
            for (int m = 0; m < P::TM; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) c[m][n][e] = exp2_(fmaf(c[m][n][e], LOG2E, -ls)) * f;
            if (edge || targets)
#pragma unroll
                for (int m = 0; m < P::TM; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int v = m * 16 + e;
                        if (v == want) c[m][n][e] = gt;
                        if (!live || v0 + v >= a.words) c[m][n][e] = 0;
                    }
            // of two tiles, even quarters take their own and their odd neighbour's words of the first, odd ones of the second: 16 bytes a lane
#pragma unroll
            for (int m = 0; m < P::TM; m += 2) {
                const uint2 x = pack4<T>(c[m][n]), y = pack4<T>(c[m + 1][n]);
                const auto s = __builtin_amdgcn_permlane16_swap(x.x, y.x, false, false), t = __builtin_amdgcn_permlane16_swap(x.y, y.y, false, false);
                if (in) *(uint4*)(row + m * 32) = make_uint4(s[0], t[0], s[1], t[1]);
            }
        } else {
            if (__any(want >= 0)) {
                float z = 0;
#pragma unroll
                for (int m = 0; m < P::TM; ++m)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z = m * 16 + r == want ? c[m][n][r] : z;
                // one lane of the grid has the target among its words
                if (in && want >= 0 && want < P::TM * 16 && (want & 15) < 4 && v0 + want < a.words) a.target_logit[token] = z;
            }
            float top = -INFINITY, sum = 0, base;
            const auto sums = [&](auto last) {
                const auto z = [&](int m, int r) { return last && v0 + m * 16 + r >= a.words ? -INFINITY : c[m][n][r]; };
#pragma unroll
                for (int m = 0; m < P::TM; ++m)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = fmaxf(top, z(m, r));
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, other_half(top));
                base = top == -INFINITY ? 0.0f : top * LOG2E;
#pragma unroll
                for (int m = 0; m < P::TM; ++m)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum += exp2_(fmaf(z(m, r), LOG2E, -base));
            };
            if (edge) sums(std::true_type());
            else sums(std::false_type());
            sum += __shfl_xor(sum, 16);
            sum += other_half(sum);
            if (quarter == 0) stat[wave / WN * N + wn + n * 16 + lane] = make_float2(top * LOG2E, sum);
        }
    }
    if constexpr (!GRAD) {
        __syncthreads();
        for (int n = threadIdx.x; n < N; n += WM * WN * 64) {
            if (n0 + n >= a.rows) break;
            float2 s = stat[n];
#pragma unroll
            for (int k = 1; k < WM; ++k) s = join(s, stat[k * N + n]);
            a.part[(uint64_t)(n0 + n) * a.m_tiles + tm] = s;
        }
    }
}

// joins the statistics of the tiles of words: a wave per token
__global__ __launch_bounds__(256) void k_vocab_join(VocabArgs a, float* loss, float* lse, float* target_logit)
{
    const uint32_t lane = threadIdx.x % 64;
    const uint64_t token = (uint64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (token >= a.rows) return;
    float2 s = make_float2(-INFINITY, 0);
#pragma unroll 4
    for (uint32_t t = lane; t < a.m_tiles; t += 64) s = join(s, a.part[token * a.m_tiles + t]);
#pragma unroll
    for (int d = 32; d; d >>= 1) s = join(s, make_float2(__shfl_xor(s.x, d), __shfl_xor(s.y, d)));
    if (lane) return;
    const float l = (s.x + log2_(s.y)) * LN2;
    const int32_t target = a.targets[token];
    const int64_t at = (int64_t)target - a.first_word;
    const bool here = target != a.ignore && at >= 0 && at < a.words;
    const float z = here ? a.target_logit[token] : 0.0f;
    lse[token] = l;
    if (target_logit) target_logit[token] = z;
    if (loss) loss[token] = target == a.ignore ? 0.0f : here ? l - z : NAN;
}

// dx^T = w^T g^T over the words of a piece: elements down, tokens across.  7782 x 16384 x 2048: 362 us, 1443 TFLOP/s, matrix units busy 67 %.
template <class T, int M>
__global__ __launch_bounds__(256) void k_vocab_dx(VocabArgs a)
{
    typedef typename ProductOf<T, M, true, false>::type P;
    constexpr int N = M, WM = P::WM, WN = P::WN;
    __shared__ __attribute__((aligned(256))) char lds_[P::LDS];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), quarter = lane / 16;
    const int wm = wave / WN * (M / WM), wn = wave % WN * (N / WN);
    const uint32_t rows = live_rows(a), n_tiles = (rows + N - 1) / N;
    if (blockIdx.x >= a.m_tiles * n_tiles) return;
    uint32_t tm, tn;
    tile_of_block(blockIdx.x, a.m_tiles, n_tiles, tm, tn);
    const uint32_t m0 = tm * M, n0 = tn * N;
    const Side sw = {{a.w.p + (int64_t)a.word0 * a.w.stride + m0 * 2, a.w.stride}, (int)min(a.dim - m0, (uint32_t)M), a.words};
    // g has zeros beyond the last word, up to a multiple of 8
    const int64_t ks = ((int64_t)a.words + 7) / 8 * 8;
    const Side sg = {{a.g + (uint64_t)n0 * a.g_stride * 2, (int64_t)a.g_stride * 2}, (int)min(rows - n0, (uint32_t)N), ks};
    const int64_t run = ((ks + a.splits - 1) / a.splits + 63) / 64 * 64;
    const int64_t k0 = min(ks, run * blockIdx.y), k1 = min(ks, k0 + run);
    f32x4 c[P::TM][P::TN];
    const float f = unit_of(a) * exp2f(-G_SHIFT<T>);
    float* sum = a.sum + (uint64_t)blockIdx.y * a.rows * a.dim;
#pragma unroll
    for (int m = 0; m < P::TM; ++m)
#pragma unroll
        for (int n = 0; n < P::TN; ++n) c[m][n] = f32x4{};
    P::run((lds_char*)lds_, sw, sg, k0, k1, c, wm, wn);
    if (a.whole) {
        store_tile<T, P, M>((lds_char*)lds_, c, f, a.out + m0 * 2, a.out_stride, (int)min(rows - n0, (uint32_t)N), (int)min(a.dim - m0, (uint32_t)M), wm, wn, [&](int r) { return a.row_of[n0 + r]; });
        return;
    }
    const auto sums = [&](auto first) {
#pragma unroll
        for (int n = 0; n < P::TN; ++n) {
            const uint32_t token = n0 + wn + n * 16 + lane % 16, x = m0 + wm + 4 * quarter;
            f32x4* p = (f32x4*)(sum + (uint64_t)token * a.dim + x);
            f32x4 old[P::TM];
#pragma unroll
            for (int m = 0; m < P::TM; ++m) old[m] = !first && token < rows && x + m * 16 < a.dim ? p[m * 4] : f32x4{};
#pragma unroll
            for (int m = 0; m < P::TM; ++m)             // dim is a multiple of 8
                if (token < rows && x + m * 16 < a.dim) p[m * 4] = c[m][n] + old[m];
            asm volatile("" ::: "memory");              // no more of them in registers than this
        }
    };
    if (a.first) sums(std::true_type());
    else sums(std::false_type());
}

// rows of an output from the sums of their splits: of dw, and of dx where it has row_of
template <class T, bool DX>
__global__ __launch_bounds__(256) void k_vocab_add(VocabArgs a, uint32_t rows, uint32_t dim)
{
    const uint64_t at = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 4, n = (uint64_t)rows * a.dim;
    const uint32_t row = (uint32_t)(at / a.dim);
    if (row >= (DX ? live_rows(a) : rows)) return;
    f32x4 s = {};
    for (uint32_t k = 0; k < a.splits; ++k) s += *(const f32x4*)(a.sum + k * n + at);
    const float f = unit_of(a) * exp2f(-G_SHIFT<T>);
    store_out<T>(a.out + (int64_t)(DX ? a.row_of[row] : row) * a.out_stride, (uint32_t)(at % a.dim), dim, a.out_vec, s[0] * f, s[1] * f, s[2] * f, s[3] * f);
}

// dw of a piece = g^T x, made transposed over the tokens: elements down, words across.  16384 x 2048 over 7782 rows: 359 us, as dx.
template <class T, int M>
__global__ __launch_bounds__(256) void k_vocab_dw(VocabArgs a, uint32_t dim)
{
    typedef typename ProductOf<T, M, true, true>::type P;
    constexpr int N = M, WM = P::WM, WN = P::WN;
    __shared__ __attribute__((aligned(256))) char lds_[P::LDS];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), quarter = lane / 16;
    const int wm = wave / WN * (M / WM), wn = wave % WN * (N / WN);
    uint32_t tm, tn;
    tile_of_block(blockIdx.x, a.m_tiles, a.n_tiles, tm, tn);
    const uint32_t m0 = tm * M, n0 = tn * N;
    const uint32_t rows = live_rows(a);
    const Mat x = live_x(a, rows);
    const Side sx = {{x.p + m0 * 2, x.stride}, (int)min(a.dim - m0, (uint32_t)M), rows};
    const Side sg = {{a.g + n0 * 2, (int64_t)a.g_stride * 2}, (int)min(a.words - n0, (uint32_t)N), rows};
    f32x4 c[P::TM][P::TN];
#pragma unroll
    for (int m = 0; m < P::TM; ++m)
#pragma unroll
        for (int n = 0; n < P::TN; ++n) c[m][n] = f32x4{};
    const int64_t run = (((int64_t)rows + a.splits - 1) / a.splits + 63) / 64 * 64;
    const int64_t k0 = min((int64_t)rows, run * blockIdx.y), k1 = min((int64_t)rows, k0 + run);
    P::run((lds_char*)lds_, sx, sg, k0, k1, c, wm, wn);
    const float f = unit_of(a) * exp2f(-G_SHIFT<T>);
    float* sum = a.sum + (uint64_t)blockIdx.y * a.words * a.dim;
    if (a.splits == 1) {
        store_tile<T, P, M>((lds_char*)lds_, c, f, a.out + m0 * 2, a.out_stride, (int)min(a.words - n0, (uint32_t)N), (int)dim - (int)m0, wm, wn,
                            [&](int r) { return (int64_t)a.word0 + n0 + r; });
        return;
    }
#pragma unroll
    for (int n = 0; n < P::TN; ++n) {
        const uint32_t word = n0 + wn + n * 16 + lane % 16;
        if (word >= a.words) continue;
#pragma unroll
        for (int m = 0; m < P::TM; ++m) {
            const uint32_t x = m0 + wm + m * 16 + 4 * quarter;
            if (x < a.dim) *(f32x4*)(sum + (uint64_t)word * a.dim + x) = c[m][n];
        }
    }
}

// A row whose length or place does not suit the products' loads, laid out anew by a wave: `dim` elements, zeros up to `to`, a multiple of 8.
template <class E>
__device__ __forceinline__ void lay_out_row(const E* s, uint32_t dim, uint32_t to, E* out)
{
    typedef E chunk __attribute__((ext_vector_type(8)));
    typedef E piece __attribute__((ext_vector_type(8), aligned(sizeof(E))));        // the device takes them anywhere
    const uint32_t lane = threadIdx.x % 64;
#pragma unroll 2
    for (uint32_t x = lane * 8; x < to; x += 512) {
        chunk v;
        if (x + 8 <= dim) v = *(const piece*)(s + x);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = x + e < dim ? s[x + e] : (E)0;
        *(chunk*)(out + x) = v;
    }
}

template <class E>
__global__ __launch_bounds__(256) void k_vocab_lay_out(const E* p, int64_t stride, uint64_t rows, uint32_t dim, uint32_t to, E* out)
{
    const uint64_t row = (uint64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (row < rows) lay_out_row(p + (int64_t)row * stride, dim, to, out + row * to);
}

// The live rows' number and largest |dloss|, and the rows in order: one block, RUN runs of as many rows as it has threads at a time.  More blocks would have to meet in between;
// 8192 rows take this one 5 us.
__global__ __launch_bounds__(1024) void k_vocab_live(const int32_t* targets, int32_t ignore, const float* dloss, uint32_t rows, uint32_t* live, uint32_t* row_of)
{
    constexpr uint32_t RUN = 8;
    __shared__ uint32_t sums[RUN * 16], total;
    __shared__ float tops[16];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    uint32_t before = 0;            // live rows of the rounds before
    float top = 0;
    for (uint64_t r0 = 0; r0 < rows; r0 += blockDim.x * RUN) {
        const uint64_t first = r0 + threadIdx.x;
        int32_t target[RUN];
        float weight[RUN];
        uint64_t lives[RUN];
#pragma unroll
        for (uint32_t i = 0; i < RUN; ++i) {            // all at once
            const uint64_t r = min(first + i * blockDim.x, (uint64_t)rows - 1);
            target[i] = targets[r], weight[i] = dloss[r];
        }
#pragma unroll
        for (uint32_t i = 0; i < RUN; ++i) {
            const bool is = first + i * blockDim.x < rows && target[i] != ignore;
            lives[i] = __ballot(is);
            top = is ? fmaxf(top, fabsf(weight[i])) : top;
            if (lane == 0) sums[i * waves + wave] = __popcll(lives[i]);
        }
        __syncthreads();
        if (wave == 0) {            // sums of what stands before each of them
            const uint32_t n = RUN * waves, u = 2 * lane < n ? sums[2 * lane] : 0, v = 2 * lane < n ? sums[2 * lane + 1] : 0;
            uint32_t upto = u + v;
#pragma unroll
            for (uint32_t d = 1; d < 64; d *= 2) {
                const uint32_t o = __shfl_up(upto, d);
                if (lane >= d) upto += o;
            }
            if (2 * lane < n) sums[2 * lane] = upto - u - v, sums[2 * lane + 1] = upto - v;
            if (lane == 63) total = upto;
        }
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < RUN; ++i) {
            const uint64_t r = first + i * blockDim.x;
            if (r >= rows) break;
            const uint32_t at = before + sums[i * waves + wave] + __popcll(lives[i] & ((1ull << lane) - 1));
            // r - at of the others came before one of them
            row_of[lives[i] >> lane & 1 ? at : rows - 1 - (r - at)] = (uint32_t)r;
        }
        before += total;
        __syncthreads();
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    if (threadIdx.x) return;
    for (uint32_t w = 1; w < waves; ++w) top = fmaxf(top, tops[w]);
    live[0] = before, live[1] = __float_as_uint(top);
}

// a wave per place of row_of: the live rows of x side by side, where some are not live or x does not suit the products (`suits`), and zeros in the others' dx
template <class E>
__global__ __launch_bounds__(256) void k_vocab_gather(VocabArgs a, const E* x, int64_t stride, uint32_t dim, bool suits, char* dx, int64_t dx_stride)
{
    const uint32_t i = blockIdx.x * 4 + threadIdx.x / 64, rows = a.live[0];
    if (i >= a.rows) return;
    if (i < rows) {
        if (rows < a.rows || !suits) lay_out_row(x + (int64_t)a.row_of[i] * stride, dim, a.dim, (E*)(a.gathered.p + (int64_t)i * a.gathered.stride));
    } else if (dx) {
        E* row = (E*)(dx + (int64_t)a.row_of[i] * dx_stride);
        for (uint32_t e = threadIdx.x % 64; e < dim; e += 64) row[e] = (E)0;
    }
}

// ---- host ------------------------------------------------------------------------------

struct Plan {
    uint32_t dim;               // a multiple of 8
    bool copy_x, copy_w;
    uint32_t piece;
    Tiling z, dx;               // of the logits, forward or of a piece; of dx
    uint64_t x, w, part, logit, live, row_of, g, sum, dw, bytes;
};

// 16-byte accesses, and 256 rows within 32 bits
bool suits(const ff_rows_t& m, uint32_t dim) { return aligned(m.p, 16) && m.stride % 8 == 0 && dim % 8 == 0 && m.stride >= 0 && m.stride < (1 << 22); }

bool eight_bytes(const ff_rows_t& m) { return aligned(m.p, 8) && m.stride % 4 == 0; }

template <class A>
Plan plan_of(const A* p, bool back)
{
    Plan q = {};
    q.dim = (uint32_t)round_up(p->dim, 8);
    q.copy_x = !suits(p->x, p->dim), q.copy_w = !suits(p->w, p->dim);
    uint64_t at = 0;
    const auto take = [&](uint64_t bytes) {
        const uint64_t o = at;
        at += round_up(bytes, 256);
        return o;
    };
    q.x = take(q.copy_x || back ? (uint64_t)p->rows * q.dim * 2 : 0);
    q.w = take(q.copy_w ? (uint64_t)p->vocab * q.dim * 2 : 0);
    if (!back) {
        q.z = tiling_of(p->vocab, p->rows, q.dim, false);
        q.part = take((uint64_t)q.z.ms * p->rows * sizeof(float2));
        q.logit = take((uint64_t)p->rows * sizeof(float));
    } else {
        q.live = take(2 * sizeof(uint32_t));
        q.row_of = take((uint64_t)p->rows * sizeof(uint32_t));
        q.piece = piece_of(p->rows, p->vocab);
        q.g = take((uint64_t)p->rows * q.piece * 2);
        q.dx = tiling_of(q.dim, p->rows, std::min(p->vocab, q.piece), true);
        q.sum = take(q.dx.splits > 1 || q.piece < p->vocab ? (uint64_t)q.dx.splits * p->rows * q.dim * sizeof(float) : 0);
        // the last piece may be smaller than the others, and the only one whose dw is split
        uint64_t dw = 0;
        for (const uint64_t words : {(uint64_t)std::min(p->vocab, q.piece), (uint64_t)(p->vocab - 1) % q.piece + 1}) {
            const uint32_t n = tiling_of(q.dim, words, p->rows, true).splits;
            if (n > 1) dw = std::max<uint64_t>(dw, n * words * q.dim * sizeof(float));
        }
        q.dw = take(dw);
    }
    q.bytes = at;
    return q;
}

// whether the blocks of a product are as many as a launch takes
bool fits(const Tiling& t) { return (uint64_t)t.ms * t.ns <= MOST_THREADS / 256; }

// the sizes, and the plan for them
template <class A>
int check_vocab(const A* p, bool back, Plan& q)
{
    if (p->dtype != FF_F16 && p->dtype != FF_BF16) return FF_EINVAL;
    if (p->vocab == 0 || p->dim == 0) return FF_EINVAL;
    static_assert(FF_OP_MAX_TOKENS == MOST_THREADS / 256 * 4, "a wave per row, four in a block");
    if (p->rows > FF_OP_MAX_TOKENS || p->vocab > FF_OP_MAX_TOKENS || p->dim > FF_OP_MAX_DIM) return FF_ERANGE;
    q = plan_of(p, back);
    if (!back) return fits(q.z) ? FF_OK : FF_ERANGE;
    // the last piece is no larger than the others, but may be cut into smaller tiles
    for (const uint32_t words : {std::min(p->vocab, q.piece), (p->vocab - 1) % q.piece + 1})
        if (!fits(tiling_of(words, p->rows, q.dim, false)) || !fits(tiling_of(q.dim, words, p->rows, true))) return FF_ERANGE;
    if (!fits(q.dx) || ((q.dx.splits > 1 || q.piece < p->vocab) && (uint64_t)p->rows * q.dim / 4 > MOST_THREADS / 256 * 256)) return FF_ERANGE;
    return FF_OK;
}

template <class T>
int lay_out(const ff_rows_t& m, uint64_t rows, uint32_t dim, uint32_t to, bool copy, char* ws, Mat& out, hipStream_t st)
{
    if (!copy || rows == 0) {
        out = {(const char*)m.p, m.stride * 2};
        return FF_OK;
    }
    out = {ws, (int64_t)to * 2};
    typedef typename T::elem E;
    k_vocab_lay_out<<<(uint32_t)ceil_div(rows, 4), 256, 0, st>>>((const E*)m.p, m.stride, rows, dim, to, (E*)ws);
    return launched();
}

template <class A>
VocabArgs args_of(const A* p, const Plan& q)
{
    VocabArgs a = {};
    a.rows = p->rows, a.dim = q.dim, a.words = p->vocab, a.ignore = p->ignore_index, a.first_word = p->first_word;
    a.targets = p->targets, a.splits = 1;
    return a;
}

template <class T>
int fwd(const ff_vocab_loss_fwd_t* p, const Plan& q, hipStream_t st)
{
    char* ws = (char*)p->workspace;
    VocabArgs a = args_of(p, q);
    if (const int rc = lay_out<T>(p->x, p->rows, p->dim, q.dim, q.copy_x, ws + q.x, a.x, st)) return rc;
    if (const int rc = lay_out<T>(p->w, p->vocab, p->dim, q.dim, q.copy_w, ws + q.w, a.w, st)) return rc;
    a.part = (float2*)(ws + q.part);
    a.target_logit = (float*)(ws + q.logit);
    a.m_tiles = q.z.ms, a.n_tiles = q.z.ns;
    if (q.z.tile == 256) k_vocab_logits<T, 256, false><<<q.z.blocks(), 256, 0, st>>>(a);
    else if (q.z.tile == 128) k_vocab_logits<T, 128, false><<<q.z.blocks(), 256, 0, st>>>(a);
    else k_vocab_logits<T, 64, false><<<q.z.blocks(), 256, 0, st>>>(a);
    k_vocab_join<<<(uint32_t)ceil_div(p->rows, 4), 256, 0, st>>>(a, p->loss, p->lse, p->target_logit);
    return launched();
}

template <class T>
int bwd(const ff_vocab_loss_bwd_t* p, const Plan& q, hipStream_t st)
{
    char* ws = (char*)p->workspace;
    VocabArgs a = args_of(p, q);
    if (const int rc = lay_out<T>(p->w, p->vocab, p->dim, q.dim, q.copy_w, ws + q.w, a.w, st)) return rc;
    a.dloss = p->dloss, a.lse_in = p->lse, a.live = (uint32_t*)(ws + q.live);
    a.g = ws + q.g, a.g_stride = q.piece, a.sum = (float*)(ws + q.sum);
    a.row_of = (uint32_t*)(ws + q.row_of);
    a.x = {q.copy_x ? nullptr : (const char*)p->x.p, p->x.stride * 2}, a.gathered = {ws + q.x, (int64_t)q.dim * 2};
    k_vocab_live<<<1, p->rows > 512 ? 1024 : 64, 0, st>>>(p->targets, p->ignore_index, p->dloss, p->rows, (uint32_t*)(ws + q.live), (uint32_t*)(ws + q.row_of));
    if (p->rows) {
        typedef typename T::elem E;
        k_vocab_gather<<<(uint32_t)ceil_div(p->rows, 4), 256, 0, st>>>(a, (const E*)p->x.p, p->x.stride, p->dim, !q.copy_x, (char*)p->dx.p, p->dx.stride * 2);
    }
    const bool whole = q.dx.splits == 1 && q.piece >= p->vocab;
    for (uint64_t word0 = 0; word0 < p->vocab; word0 += q.piece) {
        a.word0 = (uint32_t)word0;
        a.words = (uint32_t)std::min<uint64_t>(q.piece, p->vocab - word0);
        if (p->rows) {
            const Tiling z = tiling_of(a.words, p->rows, q.dim, false);
            a.m_tiles = z.ms, a.n_tiles = z.ns;
            if (z.tile == 256) k_vocab_logits<T, 256, true><<<z.blocks(), 256, 0, st>>>(a);
            else if (z.tile == 128) k_vocab_logits<T, 128, true><<<z.blocks(), 256, 0, st>>>(a);
            else k_vocab_logits<T, 64, true><<<z.blocks(), 256, 0, st>>>(a);
        }
        if (p->dx.p && p->rows) {
            a.m_tiles = q.dx.ms, a.n_tiles = q.dx.ns, a.splits = q.dx.splits, a.first = word0 == 0, a.whole = whole;
            a.out = (char*)p->dx.p, a.out_stride = p->dx.stride * 2;
            a.out_vec = eight_bytes(p->dx);
            a.dim = whole ? p->dim : q.dim;         // as many as are stored; the tiles of w have zeros beyond
            const dim3 grid(q.dx.blocks(), q.dx.splits);
            if (q.dx.tile == 256) k_vocab_dx<T, 256><<<grid, 256, 0, st>>>(a);
            else if (q.dx.tile == 128) k_vocab_dx<T, 128><<<grid, 256, 0, st>>>(a);
            else k_vocab_dx<T, 64><<<grid, 256, 0, st>>>(a);
            a.dim = q.dim;
        }
        if (p->dw.p) {
            const Tiling t = tiling_of(q.dim, a.words, p->rows, true);
            a.m_tiles = t.ms, a.n_tiles = t.ns;
            a.out = (char*)p->dw.p, a.out_stride = p->dw.stride * 2;
            a.out_vec = eight_bytes(p->dw);
            a.splits = t.splits, a.sum = (float*)(ws + q.dw);
            const dim3 grid(t.blocks(), t.splits);
            if (t.tile == 256) k_vocab_dw<T, 256><<<grid, 256, 0, st>>>(a, p->dim);
            else if (t.tile == 128) k_vocab_dw<T, 128><<<grid, 256, 0, st>>>(a, p->dim);
            else k_vocab_dw<T, 64><<<grid, 256, 0, st>>>(a, p->dim);
            if (a.splits > 1) {
                VocabArgs o = a;
                o.out += (int64_t)word0 * a.out_stride;
                k_vocab_add<T, false><<<(uint32_t)ceil_div((uint64_t)a.words * q.dim / 4, 256), 256, 0, st>>>(o, a.words, p->dim);
            }
            a.sum = (float*)(ws + q.sum);
        }
    }
    if (p->dx.p && p->rows && !whole) {
        a.splits = q.dx.splits, a.out = (char*)p->dx.p, a.out_stride = p->dx.stride * 2;
        a.out_vec = eight_bytes(p->dx);
        k_vocab_add<T, true><<<(uint32_t)ceil_div((uint64_t)p->rows * q.dim / 4, 256), 256, 0, st>>>(a, p->rows, p->dim);
    }
    return launched();
}

}  // namespace
}  // namespace ffops

using namespace ffops;

extern "C" size_t ff_op_vocab_loss_fwd_workspace_bytes(const ff_vocab_loss_fwd_t* p)
{
    Plan q;
    return p && check_vocab(p, false, q) == FF_OK && p->rows ? q.bytes : 0;
}

extern "C" int ff_op_vocab_loss_fwd(const ff_vocab_loss_fwd_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    Plan q;
    if (const int rc = check_vocab(p, false, q)) return rc;
    if (p->rows == 0) return FF_OK;
    if (!p->x.p || !p->w.p || !p->targets || !p->lse) return FF_EINVAL;
    if (!p->workspace || p->workspace_bytes < q.bytes || !aligned(p->workspace, 256)) return FF_EWORKSPACE;
    return p->dtype == FF_F16 ? fwd<F16>(p, q, (hipStream_t)stream) : fwd<BF16>(p, q, (hipStream_t)stream);
}

extern "C" size_t ff_op_vocab_loss_bwd_workspace_bytes(const ff_vocab_loss_bwd_t* p)
{
    Plan q;
    return p && check_vocab(p, true, q) == FF_OK ? q.bytes : 0;
}

extern "C" int ff_op_vocab_loss_bwd(const ff_vocab_loss_bwd_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    Plan q;
    if (const int rc = check_vocab(p, true, q)) return rc;
    if (!p->w.p || (p->rows && (!p->x.p || !p->targets || !p->dloss || !p->lse))) return FF_EINVAL;
    if (!p->dx.p && !p->dw.p) return FF_OK;
    if (!p->workspace || p->workspace_bytes < q.bytes || !aligned(p->workspace, 256)) return FF_EWORKSPACE;
    return p->dtype == FF_F16 ? bwd<F16>(p, q, (hipStream_t)stream) : bwd<BF16>(p, q, (hipStream_t)stream);
}
