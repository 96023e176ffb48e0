// What both directions of attention ask of a sequence.
#pragma once
#include "ffops_tiles.h"

namespace ffops {

struct Heads {
    char* p;
    int64_t batch, head, pos;       // bytes
};

struct AttnArgs {
    uint32_t batch, heads, kv_heads, group, q_len, kv_len, dim, causal, splits;
    float scale, scale_log2;        // scale * log2(e): statistics and exponents are powers of two inside
    Heads q, k, v, o, dout, dq, dk, dv;
    float* lse;                     // [batch][heads][q_len]
    float* delta;                   // the same shape: <do_i, o_i>
    float* lse2;                    // the same shape: lse in powers of two, infinite where a query sees nothing
    float2* top;                    // [batch][kv_heads][tops]: the largest |do| and |do| |o| (as vectors) of 32 rows, 16-bit floats only
    uint32_t tops;
    uint32_t deal;                  // 1: a sequence's blocks go to all dies, see heads_of_block
    const int32_t *q_lengths, *kv_lengths;
    float* part;                    // splits > 1: partial sums
    float* part_lse;                // splits > 1, forward: their statistics
};

static __device__ __forceinline__ int seq_len(const int32_t* lengths, uint32_t most, uint32_t b)
{
    if (!lengths) return (int)most;
    const int n = lengths[b];
    return n < 0 ? 0 : n > (int)most ? (int)most : n;
}

// keys that query i of nq sees, of nk
static __device__ __forceinline__ int seen_by(const AttnArgs& a, int i, int nq, int nk)
{
    if (i >= nq) return 0;
    if (!a.causal) return nk;
    const int n = i + 1 + nk - nq;
    return n < 0 ? 0 : n > nk ? nk : n;
}

// Loads of tiles of ROWS positions: whole ones from places worked out once (those of a tile have to fit 32 bits), others with zeros for what is missing.  Elements
// beyond a head's are zeros in the operands in registers, so what a whole tile holds in their place does not matter.
template <int ROWS, int D, int WAVES>
struct TileLoads {
    Stager<ROWS, D, WAVES> whole;
    int64_t stride;
    int chunks;
    bool near;

    __device__ __forceinline__ void init(int64_t pos, int n)
    {
        stride = pos, chunks = n;
        near = pos >= 0 && pos < (1 << 25);
        whole.init(pos, ROWS, n);
    }
    __device__ __forceinline__ void load(lds_char* dst, const char* p, int rows) const
    {
        if (near && rows >= ROWS) whole.load(dst, p);
        else stage<ROWS, D, WAVES>(dst, p, stride, rows, chunks);
    }
};

// keeps what is made of x in its branch: without it the compiler takes comparisons for every tile that only the last ones need
static __device__ __forceinline__ void stay_here(int& x) { asm volatile("" : "+v"(x)); }

// operands in registers: a row of D elements at p (null: zeros), element 16 * step + 8 * half + e
template <class T, int D>
static __device__ __forceinline__ void row_operand(typename T::vec8* f, const char* p, int dim, int half)
{
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        const bool in = p && 16 * s + 8 * half < dim;
        f[s] = *(const typename T::vec8*)(in ? p + (16 * s + 8 * half) * 2 : (const char*)&zero16);
    }
}

// The rows of a head of keys are all (query, head of the group) pairs, row = query * group + head, so that the heads that share
// keys share their loads; a wave owns 32 of them, a lane the row of its place in the half wave.
struct Rows {
    bool in;
    uint32_t i, h;                  // query and head of the lane's row
    int nq, nk;                     // lengths of the sequence
    int seen, seen_least, seen_most;    // keys that the row sees; the fewest and the most of the wave's rows
    int keys;                       // the most of the block's
};

// The sequence and key head of a block.  Blocks go to the 8 dies in turn, so where there are 8 key heads or a multiple, all blocks of one go to one die, whose cache then
// serves them; but where sequences differ in length, dies then differ in work.  Causal, a sequence's blocks are dealt to all dies: 8 of up to 1560 x 1873, 12 heads on 4 of
// 128, backward 328 us, 238 dealt; 16 of up to 2048, 8 heads, forward 107, 92 dealt (9 of up to 1064, 64 heads on 16 of 32, backward 245, 248 dealt).  Where every block reads
// all of its sequence the cache counts for more: 14 of up to 1503 x 3168, 16 heads on 2 of 64, not causal, backward 504 us, 618 dealt.
static __device__ __forceinline__ uint32_t heads_of_block(const AttnArgs& a)
{
    return (blockIdx.x + a.deal * blockIdx.y) % gridDim.x;
}

template <int WAVES>
static __device__ __forceinline__ Rows rows_of_wave(const AttnArgs& a, uint32_t b, uint32_t kh, int wave, int lane)
{
    Rows w;
    const uint32_t rows = a.q_len * a.group;
    const uint32_t tile = gridDim.y - 1 - blockIdx.y;          // causal: the rows with the most keys first
    const uint32_t row0 = tile * (WAVES * 32), row = row0 + wave * 32 + lane % 32;
    w.nq = seq_len(a.q_lengths, a.q_len, b), w.nk = seq_len(a.kv_lengths, a.kv_len, b);
    w.in = row < rows;
    w.i = w.in ? row / a.group : 0, w.h = kh * a.group + (w.in ? row % a.group : 0);
    w.seen = w.in ? seen_by(a, (int)w.i, w.nq, w.nk) : 0;
    int most = w.seen, least = w.in ? w.seen : w.nk;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        most = max(most, __shfl_xor(most, d));
        least = min(least, __shfl_xor(least, d));
    }
    w.seen_most = __builtin_amdgcn_readfirstlane(most);
    w.seen_least = __builtin_amdgcn_readfirstlane(least);
    // the last of the block's rows that is a query sees the most
    const int last = min((int)((min(row0 + WAVES * 32, rows) - 1) / a.group), w.nq - 1);
    w.keys = last * (int64_t)a.group + a.group > (int64_t)row0 ? seen_by(a, last, w.nq, w.nk) : 0;
    return w;
}

static inline Heads in_bytes(const ff_heads_t& h) { return {(char*)h.p, h.batch * 2, h.head * 2, h.pos * 2}; }
static inline bool heads_ok(const ff_heads_t& h) { return h.p && aligned(h.p, 16) && !((h.batch | h.head | h.pos) & 7); }

// sizes that both directions refuse or limit
template <class P>
static int check_attention(const P* p)
{
    if (p->dtype != FF_F16 && p->dtype != FF_BF16) return FF_EINVAL;
    if (p->kv_heads == 0 || p->heads == 0 || p->heads % p->kv_heads || p->head_dim == 0 || p->head_dim % 8) return FF_EINVAL;
    if (!(p->scale > 0) || !std::isfinite(p->scale)) return FF_EINVAL;
    if (p->head_dim > FF_OP_MAX_HEAD_DIM || p->q_len > FF_OP_MAX_LEN || p->kv_len > FF_OP_MAX_LEN) return FF_ERANGE;
    // launch grids: heads of keys of all sequences, and blocks of 128 rows
    if (p->heads > 65535 || p->batch > 65535 || (uint64_t)p->batch * p->kv_heads > 65535u * 32 || (uint64_t)p->q_len * (p->heads / p->kv_heads) > FF_OP_MAX_SIDE)
        return FF_ERANGE;
    static_assert(FF_OP_MAX_SIDE == MOST_BLOCKS_Y * 128, "as many blocks as a launch takes along y");
    return FF_OK;
}

template <class P>
static AttnArgs args_of(const P* p)
{
    AttnArgs a = {};
    a.batch = p->batch, a.heads = p->heads, a.kv_heads = p->kv_heads, a.group = p->heads / p->kv_heads;
    a.q_len = p->q_len, a.kv_len = p->kv_len, a.dim = p->head_dim, a.causal = p->causal != 0, a.splits = 1;
    a.scale = p->scale, a.scale_log2 = p->scale * LOG2E;
    a.q = in_bytes(p->q), a.k = in_bytes(p->k), a.v = in_bytes(p->v), a.o = in_bytes(p->o);
    a.q_lengths = p->q_lengths, a.kv_lengths = p->kv_lengths;
    a.deal = a.causal && (a.q_lengths || a.kv_lengths);
    return a;
}

}  // namespace ffops
