// Attention, backward: the probabilities are made again from q, k and the forward pass' lse.
#include "ffops_attention.h"

namespace ffops {
namespace {

// Two kernels, one per side of the score matrix, each of which makes the probabilities for itself: seven products instead of
// five, but every sum has one owner -- no atomic additions, the same bits every time -- and nothing of the size of the score matrix moves.
//   k_attention_dkv  owns 32 keys a wave: s = q k^T, dp = do v^T, dv^T += do^T p, dk^T += q^T ds
//   k_attention_dq   owns 32 rows a wave: s^T = k q^T, dp^T = v do^T, dq^T += k^T ds^T
// In both, what the wave owns is the column of every product, so that p and ds are second operands as they lie in the registers.
constexpr int STEP = 64;            // rows (keys) of a tile in LDS

// A 16-bit float has too few exponents for probabilities and gradients of small losses: p is kept times 2^10 (it is at most 1),
// ds relative to the power of two below the largest |do| of its heads.  bfloat has a float's exponents and needs neither.
template <class T>
constexpr float P_SHIFT = std::is_same<T, F16>::value ? 10.0f : 0.0f;

__device__ __forceinline__ float unit_below(uint32_t bits)
{
    const float m = __uint_as_float(bits);
    return m > 0 && m < INFINITY ? ldexpf(1.0f, ilogbf(m)) : 1.0f;
}

__global__ void k_attention_clear(uint32_t* top, uint32_t n)
{
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) top[i] = 0;
}

// delta_i = <do_i, o_i>, and the largest |do| per head where the type needs it.  16 lanes per row, 8 elements each.
template <class T>
__global__ __launch_bounds__(256) void k_attention_delta(AttnArgs a)
{
    const uint64_t n = (uint64_t)a.batch * a.heads * a.q_len, at = (uint64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const uint32_t i = at % a.q_len, bh = (uint32_t)(at / a.q_len), b = bh / a.heads, h = bh % a.heads;
    const int x = (threadIdx.x % 16) * 8;
    float s = 0, top = 0;
    if (at < n && (int)i < seq_len(a.q_lengths, a.q_len, b) && x < (int)a.dim) {
        const typename T::vec8 u = *(const typename T::vec8*)(a.dout.p + b * a.dout.batch + h * a.dout.head + i * a.dout.pos + x * 2);
        const typename T::vec8 v = *(const typename T::vec8*)(a.o.p + b * a.o.batch + h * a.o.head + i * a.o.pos + x * 2);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s += (float)u[e] * (float)v[e];
            top = fmaxf(top, fabsf((float)u[e]));
        }
    }
#pragma unroll
    for (int d = 8; d; d >>= 1) s += __shfl_xor(s, d);
    if (at < n && threadIdx.x % 16 == 0) a.delta[at] = s;
    if constexpr (std::is_same<T, F16>::value) {
#pragma unroll
        for (int d = 8; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        // the largest of a set does not depend on the order; most rows find it there already
        if (at < n && threadIdx.x % 16 == 0 && __float_as_uint(top) > __hip_atomic_load(a.top + bh, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))
            atomicMax(a.top + bh, __float_as_uint(top));
    }
}

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

struct Next {           // what is loaded while a tile is worked on
    const char *a, *b;
    int rows;
    bool more;
};

template <class T, int D, int WAVES>
__device__ __forceinline__ void dkv_step(const lds_char* __restrict cur, lds_char* __restrict next, const float* stat, const Next& n, const TileLoads<STEP, D, WAVES>& la, const TileLoads<STEP, D, WAVES>& lb,
                                         const typename T::vec8* kf, const typename T::vec8* vf, f32x16* dk, f32x16* dv, float c, float per, int key0, int nk,
                                         int i0, int shift, bool causal)
{
    constexpr int DB = D / 32;
    const int lane = threadIdx.x % 64, half = lane / 32, key = key0 + lane % 32;
    if (n.more) {
        la.load(next, n.a, n.rows);
        lb.load(next + STEP * D * 2, n.b, n.rows);
    }
    if (key0 >= nk) return;
    const lds_char *qt = cur, *dt = cur + STEP * D * 2;
#pragma unroll 1
    for (int b = 0; b < STEP / 32; ++b) {
        const int ib = i0 + b * 32;
        if (causal && key0 > ib + 31 + shift) continue;
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int st = 0; st < D / 16; ++st) {
            s = T::mma(along<T, D>(qt, b * 32, st), kf[st], s);
            dp = T::mma(along<T, D>(dt, b * 32, st), vf[st], dp);
        }
        interleave<D / 8, 1, 4, 0>();
        const bool edge = key0 + 32 > nk || (causal && key0 + 31 > ib + shift);
        float p[16], ds[16];
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 ls = *(const f32x4*)(stat + b * 32 + c_row(r, half)), de = *(const f32x4*)(stat + STEP + b * 32 + c_row(r, half));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[r + e] = exp2_(fmaf(s[r + e], c, -ls[e]));
                ds[r + e] = p[r + e] * fmaf(dp[r + e], per, -de[e]);
            }
        }
        if (edge) {
            stay_here();
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (key >= nk || (causal && key > ib + c_row(r, half) + shift)) p[r] = ds[r] = 0;
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const typename T::vec8 pf = round8<T>(p + st * 8), df = round8<T>(ds + st * 8);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                dv[d] = T::mma(across<T, D>(dt, b * 32 + st * 16, d * 32), pf, dv[d]);
                dk[d] = T::mma(across<T, D>(qt, b * 32 + st * 16, d * 32), df, dk[d]);
            }
        }
        interleave<4 * DB, 2, 3, 2>();
    }
}

template <class T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 1) void k_attention_dkv(AttnArgs a)
{
    constexpr int DB = D / 32, TILE = STEP * D * 2;
    __shared__ __attribute__((aligned(256))) char lds_[4 * TILE];
    __shared__ __attribute__((aligned(16))) float stat[2][2 * STEP];
    lds_char* lds = (lds_char*)lds_;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const uint32_t bk = blockIdx.x, b = bk / a.kv_heads, kh = bk % a.kv_heads;
    const int nq = seq_len(a.q_lengths, a.q_len, b), nk = seq_len(a.kv_lengths, a.kv_len, b), shift = nk - nq;
    const int block0 = blockIdx.y * (WAVES * 32), key0 = block0 + wave * 32, key = key0 + lane % 32;
    const bool own = key < nk;
    const int chunks = a.dim / 8;
    const bool causal = a.causal;
    float unit = 1.0f;
    if constexpr (std::is_same<T, F16>::value) {
        uint32_t top = 0;
        for (uint32_t g = 0; g < a.group; ++g) top = max(top, a.top[b * a.heads + kh * a.group + g]);
        unit = unit_below(top);
    }
    // p is 2^P_SHIFT too large in ds, too
    const float per = exp2_(-P_SHIFT<T>) / unit;
    typename T::vec8 kf[D / 16], vf[D / 16];
    row_operand<T, D>(kf, own ? a.k.p + b * a.k.batch + kh * a.k.head + key * a.k.pos : nullptr, a.dim, half);
    row_operand<T, D>(vf, own ? a.v.p + b * a.v.batch + kh * a.v.head + key * a.v.pos : nullptr, a.dim, half);
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = f32x16{};
    // tiles of queries that see a key of the block, for each head of the group; a split takes a run of them
    const int first = causal && block0 - shift > 0 ? (block0 - shift) / STEP : 0;
    const int per_head = block0 < nk ? max(0, (nq + STEP - 1) / STEP - first) : 0;
    int u0 = 0, u1 = per_head * (int)a.group;
    if (a.splits > 1) {
        const int run = (u1 + (int)a.splits - 1) / (int)a.splits;
        u0 = min(u1, run * (int)blockIdx.z);
        u1 = min(u1, u0 + run);
    }
    int g = per_head ? u0 / per_head : 0, t = per_head ? first + u0 % per_head : 0;
    const auto tile_of = [&](int g, int t, bool more) {
        const uint32_t h = kh * a.group + g;
        const int64_t i = (int64_t)t * STEP;
        return Next{a.q.p + b * a.q.batch + h * a.q.head + i * a.q.pos, a.dout.p + b * a.dout.batch + h * a.dout.head + i * a.dout.pos, nq - t * STEP, more};
    };
    // the statistics of a tile's rows, for lane r of the first wave those of row r: a row that sees nothing has no probabilities
    const auto stat_of = [&](int g, int t, float& ls, float& de) {
        const int i = t * STEP + lane;
        ls = INFINITY, de = 0;
        if (i >= nq) return;
        const uint64_t at = ((uint64_t)b * a.heads + kh * a.group + g) * a.q_len + i;
        const float x = a.lse[at];
        de = a.delta[at] * per;
        if (x != -INFINITY) ls = x * LOG2E - P_SHIFT<T>;
    };
    TileLoads<STEP, D, WAVES> ql, dl;
    ql.init(a.q.pos, chunks);
    dl.init(a.dout.pos, chunks);
    if (u0 < u1) {
        const Next n = tile_of(g, t, true);
        ql.load(lds, n.a, n.rows);
        dl.load(lds + TILE, n.b, n.rows);
        if (wave == 0) stat_of(g, t, stat[0][lane], stat[0][STEP + lane]);
    }
    __syncthreads();
    for (int u = u0; u < u1; ++u) {
        const int now = (u - u0) & 1;
        int gn = g, tn = t + 1;
        if (tn == first + per_head) ++gn, tn = first;
        const bool more = u + 1 < u1;
        float ls = 0, de = 0;
        if (more && wave == 0) stat_of(gn, tn, ls, de);
        dkv_step<T, D, WAVES>(lds + now * 2 * TILE, lds + (1 - now) * 2 * TILE, stat[now], tile_of(more ? gn : g, more ? tn : t, more), ql, dl, kf, vf, dk, dv,
                              a.scale_log2, per, key0, nk, t * STEP, shift, causal);
        if (more && wave == 0) stat[1 - now][lane] = ls, stat[1 - now][STEP + lane] = de;
        __syncthreads();
        g = gn, t = tn;
    }
    if (key >= (int)a.kv_len) return;
    const float fk = a.scale * unit, fv = exp2_(-P_SHIFT<T>);
    if (a.splits > 1) {
        const uint64_t n = (uint64_t)a.batch * a.kv_heads * a.kv_len, at = ((uint64_t)bk * a.kv_len + key);
        float *pk = a.part + (2 * (uint64_t)blockIdx.z * n + at) * a.dim, *pv = pk + n * a.dim;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            store_part(pk, dk[d], d * 32, a.dim, half, fk);
            store_part(pv, dv[d], d * 32, a.dim, half, fv);
        }
        return;
    }
    char *pk = a.dk.p + b * a.dk.batch + kh * a.dk.head + key * a.dk.pos, *pv = a.dv.p + b * a.dv.batch + kh * a.dv.head + key * a.dv.pos;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        store_row<T>(pk, dk[d], d * 32, a.dim, half, fk);
        store_row<T>(pv, dv[d], d * 32, a.dim, half, fv);
    }
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
    const lds_char *kt = cur, *vt = cur + STEP * D * 2;
#pragma unroll 1
    for (int b = 0; b < STEP / 32; ++b) {
        const int kb = key0 + b * 32;
        if (kb >= seen_most) break;
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int st = 0; st < D / 16; ++st) {
            s = T::mma(along<T, D>(kt, b * 32, st), qf[st], s);
            dp = T::mma(along<T, D>(vt, b * 32, st), df[st], dp);
        }
        interleave<D / 8, 1, 4, 0>();
        float ds[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = exp2_(fmaf(s[r], c, -ls)) * fmaf(dp[r], per, -de);
        if (kb + 32 > seen_least) {
            stay_here();
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (kb + c_row(r, half) >= seen) ds[r] = 0;
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
    const uint32_t bk = blockIdx.x, b = bk / a.kv_heads, kh = bk % a.kv_heads;
    const Rows w = rows_of_wave<WAVES>(a, b, kh, wave, lane);
    const int nk = w.nk, chunks = a.dim / 8;
    int t0 = 0, t1 = (w.keys + STEP - 1) / STEP;
    if (a.splits > 1) {
        const int run = (t1 + (int)a.splits - 1) / (int)a.splits;
        t0 = min(t1, run * (int)blockIdx.z);
        t1 = min(t1, t0 + run);
    }
    const char* kp = a.k.p + b * a.k.batch + kh * a.k.head;
    const char* vp = a.v.p + b * a.v.batch + kh * a.v.head;
    const bool query = w.in && (int)w.i < w.nq;
    typename T::vec8 qf[D / 16], df[D / 16];
    row_operand<T, D>(qf, query ? a.q.p + b * a.q.batch + w.h * a.q.head + w.i * a.q.pos : nullptr, a.dim, half);
    row_operand<T, D>(df, query ? a.dout.p + b * a.dout.batch + w.h * a.dout.head + w.i * a.dout.pos : nullptr, a.dim, half);
    const uint64_t at = ((uint64_t)b * a.heads + w.h) * a.q_len + w.i;
    float ls = INFINITY, de = 0, unit = 1.0f;
    if (query) {
        const float x = a.lse[at];
        if constexpr (std::is_same<T, F16>::value) unit = unit_below(a.top[b * a.heads + w.h]);
        if (x != -INFINITY) ls = x * LOG2E;
        de = a.delta[at] / unit;
    }
    f32x16 dq[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dq[d] = f32x16{};
    TileLoads<STEP, D, WAVES> kl, vl;
    kl.init(a.k.pos, chunks);
    vl.init(a.v.pos, chunks);
    if (t0 < t1) {
        kl.load(lds, kp + (int64_t)t0 * STEP * a.k.pos, nk - t0 * STEP);
        vl.load(lds + TILE, vp + (int64_t)t0 * STEP * a.v.pos, nk - t0 * STEP);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int now = ((t - t0) & 1) * 2 * TILE, k1 = (t + 1) * STEP;
        const Next n = {kp + (int64_t)k1 * a.k.pos, vp + (int64_t)k1 * a.v.pos, nk - k1, t + 1 < t1};
        dq_step<T, D, WAVES>(lds + now, lds + (2 * TILE - now), n, kl, vl, qf, df, dq, a.scale_log2, ls, de, 1.0f / unit, t * STEP, w.seen, w.seen_least, w.seen_most);
        __syncthreads();
    }
    if (!w.in) return;
    const float f = a.scale * unit;
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

uint32_t waves_of(uint64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

// Work is split over the other axis where the owners alone leave more than half of the device's 256 compute units without a block, by no more than leaves
// a split four tiles.
uint32_t splits_of(uint64_t blocks, uint64_t tiles)
{
    if (blocks == 0 || blocks >= 128) return 1;
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(256 / blocks, tiles / 4));
}

struct Plan {
    uint32_t kv_waves, kv_splits, q_waves, q_splits;
    uint64_t delta, top, part, bytes;       // offsets in the workspace
};

Plan plan_of(const AttnArgs& a)
{
    Plan p = {};
    const uint64_t rows = (uint64_t)a.q_len * a.group, bk = (uint64_t)a.batch * a.kv_heads;
    p.kv_waves = waves_of(a.kv_len), p.q_waves = waves_of(rows);
    p.kv_splits = splits_of(bk * ceil_div(a.kv_len, p.kv_waves * 32), a.group * ceil_div(a.q_len, STEP));
    p.q_splits = splits_of(bk * ceil_div(rows, p.q_waves * 32), ceil_div(a.kv_len, STEP));
    p.top = round_up((uint64_t)a.batch * a.heads * a.q_len * sizeof(float), 256);
    p.part = p.top + round_up((uint64_t)a.batch * a.heads * sizeof(uint32_t), 256);
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
    if (a.q_len) {
        if (std::is_same<T, F16>::value) k_attention_clear<<<(uint32_t)ceil_div((uint64_t)a.batch * a.heads, 256), 256, 0, st>>>(a.top, a.batch * a.heads);
        k_attention_delta<T><<<(uint32_t)ceil_div((uint64_t)a.batch * a.heads * a.q_len, 16), 256, 0, st>>>(a);
    }
    if (a.kv_len) {
        a.splits = p.kv_splits;
        if (a.dim <= 64) launch_dkv<T, 64>(a, p.kv_waves, st);
        else launch_dkv<T, 128>(a, p.kv_waves, st);
        if (a.splits > 1)
            k_attention_add<T><<<dim3((uint32_t)ceil_div((uint64_t)a.batch * a.kv_heads * a.kv_len, 16), 2), 256, 0, st>>>(a.part, a.splits, 2, a.dk, a.dv, a.batch, a.kv_heads, a.kv_len, a.dim);
    }
    if (a.q_len) {
        a.splits = p.q_splits;
        if (a.dim <= 64) launch_dq<T, 64>(a, p.q_waves, st);
        else launch_dq<T, 128>(a, p.q_waves, st);
        if (a.splits > 1)
            k_attention_add<T><<<dim3((uint32_t)ceil_div((uint64_t)a.batch * a.heads * a.q_len, 16), 1), 256, 0, st>>>(a.part, a.splits, 1, a.dq, a.dq, a.batch, a.heads, a.q_len, a.dim);
    }
    return launched();
}

}  // namespace
}  // namespace ffops

using namespace ffops;

extern "C" size_t ff_op_attention_bwd_workspace_bytes(const ff_attention_bwd_t* p)
{
    if (!p || check_attention(p) != FF_OK) return 0;
    return plan_of(args_of(p)).bytes;
}

extern "C" int ff_op_attention_bwd(const ff_attention_bwd_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check_attention(p)) return rc;
    if (p->batch == 0 || (p->q_len == 0 && p->kv_len == 0)) return FF_OK;
    if (p->q_len && (!heads_ok(p->q) || !heads_ok(p->o) || !heads_ok(p->dout) || !heads_ok(p->dq) || !p->lse)) return FF_EINVAL;
    if (p->kv_len && (!heads_ok(p->k) || !heads_ok(p->v) || !heads_ok(p->dk) || !heads_ok(p->dv))) return FF_EINVAL;
    AttnArgs a = args_of(p);
    const Plan plan = plan_of(a);
    if (!p->workspace || p->workspace_bytes < plan.bytes || !aligned(p->workspace, 256)) return FF_EWORKSPACE;
    a.dout = in_bytes(p->dout), a.dq = in_bytes(p->dq), a.dk = in_bytes(p->dk), a.dv = in_bytes(p->dv);
    a.lse = const_cast<float*>(p->lse);
    char* ws = (char*)p->workspace;
    a.delta = (float*)ws;
    a.top = (uint32_t*)(ws + plan.top);
    a.part = (float*)(ws + plan.part);
    return p->dtype == FF_F16 ? run<F16>(a, plan, (hipStream_t)stream) : run<BF16>(a, plan, (hipStream_t)stream);
}
