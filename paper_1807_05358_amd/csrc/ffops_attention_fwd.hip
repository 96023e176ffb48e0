// Attention, forward.
#include "ffops_attention.h"

namespace ffops {
namespace {

// A wave owns 32 rows and keeps its q in registers; the block's waves share tiles of KEYS keys
// and values in LDS, loaded one tile ahead.  Scores are made transposed, s^T = k q^T: a lane then holds 16 of 32 keys
// of one row, the softmax of a row needs one exchange with lane ^ 32, its statistics are one register each, and the
// probabilities are the second operand of o^T += v^T p^T as they lie.  The running maximum moves only when it grows by more than
// 2^8: sums then stay within 2^8 of their scale, which costs 32-bit sums nothing and saves most rescalings.  The probabilities are rounded to the type because the products take nothing wider.
// Two waves on a SIMD, so that one's products run beside the other's exponentials, maxima and conversions, which are what bounds it: 2 sequences of 4096, 32 heads on 8 of
// 128, causal, 278 to 292 us, 940 to 990 TFLOP/s, matrix units busy 45 % of the time, LDS 24 %.  One wave with 64 rows, which reads half as much from LDS, takes 352 us.
// A single token (8 sequences of up to 16384 keys, 51622 together, 32 heads on 8): 58 us for 211 MB of keys and values, 3.65 TB/s; the heads of a group share a wave's rows, so that keys are
// read once.  Every sequence has as many splits, so that the longest one's blocks run on when the others' have ended.
constexpr int KEYS = 64;

// A 16-bit float ends at 2^-24: probabilities of 3e-8 of the largest would be none, and of 1e-5 have few bits, which counts where thousands of such keys make up the output beside one whose
// value is small (4096 keys 17.5 below a key without a value: o off by 35 %).  They are kept times 2^8, and the maximum moves when it grows by more than 2^7: they then stay below 2^15.
// Keys of 1e-10 of the largest still count.
template <class T>
constexpr float P_SHIFT = std::is_same<T, F16>::value ? 8.0f : 0.0f;
template <class T>
constexpr float MAX_BEHIND = std::is_same<T, F16>::value ? 7.0f : 8.0f;

template <class T, int D, int WAVES>
__device__ __forceinline__ void tile_step(const lds_char* __restrict cur, lds_char* __restrict next, bool more, const char* kn, const char* vn, int rows_next,
                                          const TileLoads<KEYS, D, WAVES>& kl, const TileLoads<KEYS, D, WAVES>& vl, const typename T::vec8* qf, f32x16* o, float& m, float& l,
                                          float c, int key0, int seen, int seen_least, int seen_most)
{
    constexpr int DB = D / 32;
    const int half = (threadIdx.x % 64) / 32;
    if (more) {
        kl.load(next, kn, rows_next);
        vl.load(next + KEYS * D * 2, vn, rows_next);
    }
    if (key0 >= seen_most) return;
    const lds_char *kt = cur, *vt = cur + KEYS * D * 2;
    f32x16 s[KEYS / 32];
#pragma unroll
    for (int b = 0; b < KEYS / 32; ++b) s[b] = f32x16{};
#pragma unroll
    for (int st = 0; st < D / 16; ++st)
#pragma unroll
        for (int b = 0; b < KEYS / 32; ++b) s[b] = T::mma(along<T, D>(kt, b * 32, st), qf[st], s[b]);
    interleave<D / 16 * (KEYS / 32), 1, 4, 0>();
    if (key0 + KEYS > seen_least) {
        int first = seen - key0 - 4 * half;         // key of the tile that the row does not see
        stay_here(first);
#pragma unroll
        for (int b = 0; b < KEYS / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = b * 32 + c_row(r, 0) >= first ? -INFINITY : s[b][r];
    }
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < KEYS / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
    top = fmaxf(top, other_half(top)) * c;
    if (__any(top > m + (MAX_BEHIND<T> + P_SHIFT<T>))) {        // m, the maximum less the shift, starts at -inf; a row that sees nothing keeps it
        const float mn = fmaxf(m, top - P_SHIFT<T>), f = mn == -INFINITY ? 1.0f : exp2_(m - mn);
        l *= f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] *= f;
        m = mn;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0;
#pragma unroll
    for (int b = 0; b < KEYS / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[b][r] = exp2_(fmaf(s[b][r], c, -base));
            sum += s[b][r];
        }
    l += sum;
#pragma unroll
    for (int b = 0; b < KEYS / 32; ++b)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = s[b][st * 8 + e];
            const typename T::vec8 p = round8<T>(f);
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] = T::mma(across<T, D>(vt, b * 32 + st * 16, d * 32), p, o[d]);
        }
    interleave<KEYS / 16 * DB, 2, 3, 32 / DB>();
}

template <class T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void k_attention_fwd(AttnArgs a)
{
    constexpr int DB = D / 32, TILE = KEYS * D * 2;
    __shared__ __attribute__((aligned(256))) char lds_[4 * TILE];
    lds_char* lds = (lds_char*)lds_;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const uint32_t bk = heads_of_block(a), b = bk / a.kv_heads, kh = bk % a.kv_heads;
    const Rows w = rows_of_wave<WAVES>(a, b, kh, wave, lane);
    const uint32_t i = w.i, h = w.h;
    const int nk = w.nk;
    int t0 = 0, t1 = (w.keys + KEYS - 1) / KEYS;
    if (a.splits > 1) {
        const int per = (t1 + (int)a.splits - 1) / (int)a.splits;
        t0 = min(t1, per * (int)blockIdx.z);
        t1 = min(t1, t0 + per);
    }
    const int chunks = a.dim / 8;
    const char* kp = a.k.p + b * a.k.batch + kh * a.k.head;
    const char* vp = a.v.p + b * a.v.batch + kh * a.v.head;
    typename T::vec8 qf[D / 16];
    row_operand<T, D>(qf, w.in && (int)i < w.nq ? a.q.p + b * a.q.batch + h * a.q.head + i * a.q.pos : nullptr, a.dim, half);
    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x16{};
    float m = -INFINITY, l = 0;
    TileLoads<KEYS, D, WAVES> kl, vl;
    kl.init(a.k.pos, chunks);
    vl.init(a.v.pos, chunks);
    if (t0 < t1) {
        kl.load(lds, kp + (int64_t)t0 * KEYS * a.k.pos, nk - t0 * KEYS);
        vl.load(lds + TILE, vp + (int64_t)t0 * KEYS * a.v.pos, nk - t0 * KEYS);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int now = ((t - t0) & 1) * 2 * TILE, k1 = (t + 1) * KEYS;
        tile_step<T, D, WAVES>(lds + now, lds + (2 * TILE - now), t + 1 < t1, kp + (int64_t)k1 * a.k.pos, vp + (int64_t)k1 * a.v.pos, nk - k1, kl, vl, qf, o, m, l, a.scale_log2, t * KEYS, w.seen, w.seen_least, w.seen_most);
        __syncthreads();
    }
    l += other_half(l);
    if (!w.in) return;
    const float inv = l > 0 ? 1.0f / l : l == l ? 0.0f : l;         // a NaN stays one
    const uint64_t at = ((uint64_t)b * a.heads + h) * a.q_len + i;
    if (a.splits > 1) {
        float* p = a.part + ((uint64_t)blockIdx.z * a.batch * a.heads * a.q_len + at) * a.dim;
        if (half == 0) a.part_lse[(uint64_t)blockIdx.z * a.batch * a.heads * a.q_len + at] = m + log2_(l);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int x = d * 32 + c_row(r, half);
                if (x < (int)a.dim) *(f32x4*)(p + x) = f32x4{o[d][r] * inv, o[d][r + 1] * inv, o[d][r + 2] * inv, o[d][r + 3] * inv};
            }
        return;
    }
    if (half == 0) a.lse[at] = (m + log2_(l)) * LN2;
    char* p = a.o.p + b * a.o.batch + h * a.o.head + i * a.o.pos;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int x = d * 32 + c_row(r, half);
            if (x < (int)a.dim) store4<T>(p + x * 2, o[d][r] * inv, o[d][r + 1] * inv, o[d][r + 2] * inv, o[d][r + 3] * inv);
        }
}

// joins the parts of a row (5 us for 256 rows of 8 splits, most of it the launch): o = sum_s 2^(lse_s - lse) o_s.  A wave per row: 16 lanes cover its elements, 8 each, and four of them the splits in turn.
template <class T>
__global__ __launch_bounds__(256) void k_attention_join(AttnArgs a)
{
    const uint64_t n = (uint64_t)a.batch * a.heads * a.q_len, at = (uint64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (at >= n) return;
    const uint32_t lane = threadIdx.x % 64, x = lane % 16 * 8;
    float m = -INFINITY;
    for (uint32_t s = lane; s < a.splits; s += 64) m = fmaxf(m, a.part_lse[s * n + at]);
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0, o[8] = {};
#pragma unroll 4
    for (uint32_t s = lane / 16; s < a.splits; s += 4) {
        const float w = exp2_(a.part_lse[s * n + at] - base);
        sum += w;
        const float* p = a.part + (s * n + at) * a.dim + (x < a.dim ? x : 0);
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
    if (lane >= 16) return;
    const float inv = sum > 0 ? 1.0f / sum : sum == sum ? 0.0f : sum;
    if (lane == 0) a.lse[at] = (base + log2_(sum)) * LN2;
    if (x >= a.dim) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= inv;
    const uint64_t i = at % a.q_len, bh = at / a.q_len;
    *(typename T::vec8*)(a.o.p + bh / a.heads * a.o.batch + bh % a.heads * a.o.head + i * a.o.pos + x * 2) = round8<T>(o);
}

uint32_t waves_of(const AttnArgs& a)
{
    const uint64_t rows = (uint64_t)a.q_len * a.group;
    return rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
}

// Keys are split over blocks where the rows alone do not fill the device's 512 places (two blocks on each of 256 compute units), by
// no more than leaves a split four tiles.
uint32_t splits_of(const AttnArgs& a)
{
    const uint64_t blocks = (uint64_t)a.batch * a.kv_heads * ceil_div((uint64_t)a.q_len * a.group, waves_of(a) * 32), tiles = ceil_div(a.kv_len, KEYS);
    if (blocks == 0 || blocks >= 256) return 1;
    const uint64_t s = std::min<uint64_t>(512 / blocks, tiles / 4);
    return (uint32_t)std::max<uint64_t>(1, s);
}

template <class T, int D>
void launch(const AttnArgs& a, hipStream_t st)
{
    const uint32_t w = waves_of(a);
    const dim3 grid(a.batch * a.kv_heads, (uint32_t)ceil_div((uint64_t)a.q_len * a.group, w * 32), a.splits);
    if (w == 1) k_attention_fwd<T, D, 1><<<grid, 64, 0, st>>>(a);
    else if (w == 2) k_attention_fwd<T, D, 2><<<grid, 128, 0, st>>>(a);
    else k_attention_fwd<T, D, 4><<<grid, 256, 0, st>>>(a);
}

template <class T>
int run(const AttnArgs& a, hipStream_t st)
{
    if (a.dim <= 64) launch<T, 64>(a, st);
    else launch<T, 128>(a, st);
    if (a.splits > 1) k_attention_join<T><<<(uint32_t)ceil_div((uint64_t)a.batch * a.heads * a.q_len, 4), 256, 0, st>>>(a);
    return launched();
}

uint64_t part_floats(const AttnArgs& a) { return (uint64_t)a.splits * a.batch * a.heads * a.q_len; }

}  // namespace
}  // namespace ffops

using namespace ffops;

extern "C" size_t ff_op_attention_fwd_workspace_bytes(const ff_attention_fwd_t* p)
{
    if (!p || check_attention(p) != FF_OK) return 0;
    AttnArgs a = args_of(p);
    a.splits = splits_of(a);
    return a.splits > 1 ? part_floats(a) * (a.dim + 1) * sizeof(float) : 0;
}

extern "C" int ff_op_attention_fwd(const ff_attention_fwd_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check_attention(p)) return rc;
    if (p->batch == 0 || p->q_len == 0) return FF_OK;
    if (!heads_ok(p->q) || !heads_ok(p->o) || !p->lse || (p->kv_len && (!heads_ok(p->k) || !heads_ok(p->v)))) return FF_EINVAL;
    AttnArgs a = args_of(p);
    a.lse = p->lse;
    a.splits = splits_of(a);
    const size_t need = ff_op_attention_fwd_workspace_bytes(p);
    if (need) {
        if (!p->workspace || p->workspace_bytes < need || !aligned(p->workspace, 256)) return FF_EWORKSPACE;
        a.part = (float*)p->workspace;
        a.part_lse = a.part + part_floats(a) * a.dim;
    }
    return p->dtype == FF_F16 ? run<F16>(a, (hipStream_t)stream) : run<BF16>(a, (hipStream_t)stream);
}
