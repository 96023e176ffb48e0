// Layer norm, forward and backward.
#include "ffops_device.h"

namespace ffops {
namespace {

struct FwdArgs {
    uint64_t rows;
    uint32_t cols;
    float eps;
    const void *x, *res;
    void *h, *y;
    int64_t xs, rs, hs, ys;
    const void *w, *b;
    float *mean, *rstd;
};

struct BwdArgs {
    uint64_t rows;
    uint32_t cols, groups;          // groups: partial sums of the weight's gradient
    const void *dy, *h, *dh;
    void* dx;
    int64_t dys, hs, dhs, dxs;
    const void* w;
    const float *mean, *rstd;
    float* part;                    // [2][groups][cols]
};

// The elements of a row that a lane takes at a time: 16 bytes of the type, from element `at`, of which it owns first .. last - 1.  LOOSE: rows start at any element and have any length; the
// device takes accesses of 16 bytes anywhere, and the last ones of a row are moved back to end with it, where their first elements are the lane's before.  That way no load
// stands in a branch, where it would be waited for.  One element at a time 16384 x 4095 bfloats take 101 us forward
// and 250 backward, this way 55 and 98; where rows suit it (4096) 42 and 80.
template <class T, bool LOOSE>
struct Chunk {
    typedef typename T::elem elem;
    static constexpr int V = T::VEC;
    typedef elem vec __attribute__((ext_vector_type(V), aligned(LOOSE ? sizeof(elem) : 16)));
    int64_t at;
    int first, last;
    bool any;

    __device__ __forceinline__ Chunk(uint32_t c, uint32_t cols)
    {
        any = c < cols;
        at = LOOSE ? max(min((int)c, (int)cols - V), 0) : c;
        first = LOOSE ? (int)c - (int)at : 0;
        last = LOOSE ? min(V, (int)cols) : V;
    }
    __device__ __forceinline__ bool owns(int e) const { return !LOOSE || (e >= first && e < last); }
    __device__ __forceinline__ vec fetch(const void* p, int64_t row) const
    {
        const elem* q = (const elem*)p + row + at;
        if (!LOOSE || last == V) return *(const vec*)q;
        vec v;              // a row shorter than that
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = e < last ? q[e] : (elem)0;
        return v;
    }
    __device__ __forceinline__ void load(const void* p, int64_t row, float* f) const
    {
        const vec v = fetch(p, row);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = (float)v[e];
    }
    __device__ __forceinline__ void store(void* p, int64_t row, const float* f) const
    {
        elem* q = (elem*)p + row + at;
        if (!LOOSE || last - first == V) {
            vec v;
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = (elem)f[e];
            *(vec*)q = v;
        } else
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (owns(e)) q[e] = (elem)f[e];
    }
};

// sums of N values over the THREADS lanes that share a row; every lane gets them.  `red` holds N floats per wave.
template <int THREADS, int N>
__device__ __forceinline__ void row_sum(float* s, float* red)
{
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if constexpr (THREADS >= 64) s[n] = wave_sum(s[n]);
        else
#pragma unroll
            for (int d = THREADS / 2; d; d /= 2) s[n] += __shfl_xor(s[n], d);
    }
    if constexpr (THREADS > 64) {
        const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
        __syncthreads();        // the previous sums have been read
        if (lane == 0)
            for (int n = 0; n < N; ++n) red[wave * N + n] = s[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            s[n] = 0;
            for (int w = 0; w < THREADS / 64; ++w) s[n] += red[w * N + n];
        }
    }
}

constexpr int block_of(int threads) { return threads <= 64 ? 256 : threads; }
constexpr int rows_of(int threads) { return block_of(threads) / threads; }

// A row is held in registers by THREADS lanes, E elements each; rows of a wave, or of less of it, go side by side in a
// block.  One read of x (and res), one write of h and y: the kernel is bound by memory (16384 x 4096 bfloats with a residual 97 us, 5.6 TB/s).
template <class T, bool LOOSE, int THREADS, int E>
__global__ __launch_bounds__(block_of(THREADS)) void k_layernorm_fwd(FwdArgs a)
{
    constexpr int V = T::VEC, N = E / V;
    __shared__ float red[THREADS > 64 ? THREADS / 64 : 1];
    const int t = threadIdx.x % THREADS;
    const uint64_t row = (uint64_t)blockIdx.x * rows_of(THREADS) + threadIdx.x / THREADS;
    if (row >= a.rows) return;      // all lanes of a row, and no barrier where a block has several
    const int64_t r = (int64_t)row;
    float f[E];
    float s = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Chunk<T, LOOSE> c((n * THREADS + t) * V, a.cols);
        float* v = f + n * V;
        if (c.any) {
            c.load(a.x, r * a.xs, v);
            if (a.res) {
                float u[V];
                c.load(a.res, r * a.rs, u);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = (float)(typename T::elem)(v[e] + u[e]);     // the sum is an output, and what is normed
                c.store(a.h, r * a.hs, v);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) s += c.owns(e) ? v[e] : 0.0f;
        }
    }
    row_sum<THREADS, 1>(&s, red);
    const float mean = s / (float)a.cols;
    float q = 0;                    // of the differences, from registers: no cancellation
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Chunk<T, LOOSE> c((n * THREADS + t) * V, a.cols);
        if (c.any)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = c.owns(e) ? f[n * V + e] - mean : 0.0f;
                q += d * d;
            }
    }
    row_sum<THREADS, 1>(&q, red);
    const float rstd = 1.0f / sqrtf(q / (float)a.cols + a.eps);
    if (t == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Chunk<T, LOOSE> c((n * THREADS + t) * V, a.cols);
        if (c.any) {
            float w[V], b[V], y[V];
            c.load(a.w, 0, w);
            if (a.b) c.load(a.b, 0, b);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = (f[n * V + e] - mean) * rstd * w[e] + (a.b ? b[e] : 0.0f);
            c.store(a.y, r * a.ys, y);
        }
    }
}

// Rows are dealt to the groups in turn (block b takes rows b, b + groups, ...; a wave, or less, of its own the rows of its place in
// the block too), so that a lane keeps its columns and sums the weight's and the bias's gradient in registers.  One read
// of dy, h (and dh), one write of dx; the partial sums are groups * cols * 8 bytes more, each way.  Bound by memory: 16384 x 4096 bfloats with a residual 102 us, 5.3 TB/s.  Kept as they are in memory, dy and h take
// half the registers of what is made of them: 16384 x 4096 without a residual 80 us, 90 the other way; 3000 x 14233 95 and 130.
template <class T, bool LOOSE, int THREADS, int E>
__global__ __launch_bounds__(block_of(THREADS)) void k_layernorm_bwd(BwdArgs a)
{
    constexpr int RPB = rows_of(THREADS), V = T::VEC, N = E / V, SHARED = THREADS < 64 ? THREADS : 64;
    __shared__ float red[THREADS > 64 ? 2 * THREADS / 64 : 1];
    __shared__ float both[RPB > 1 ? 2 * SHARED * E : 1];
    const int t = threadIdx.x % THREADS, sub = threadIdx.x / THREADS;
    typedef typename Chunk<T, LOOSE>::vec vec;
    constexpr bool KEEP = E < 32;       // the weights, where there is room for them
    vec w[KEEP ? N : 1];
    float dw[E], db[E];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Chunk<T, LOOSE> c((n * THREADS + t) * V, a.cols);
#pragma unroll
        for (int e = 0; e < V; ++e) dw[n * V + e] = db[n * V + e] = 0;
        if (KEEP && c.any) w[n] = c.fetch(a.w, 0);
    }
    for (uint64_t row = (uint64_t)blockIdx.x * RPB + sub; row < a.rows; row += (uint64_t)a.groups * RPB) {
        const int64_t r = (int64_t)row;
        const float mean = a.mean[r], rstd = a.rstd[r];
        vec y[N], h[N];             // as they are in memory: what is made of them takes twice the registers, and is made twice
        float s[2] = {0, 0};
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Chunk<T, LOOSE> c((n * THREADS + t) * V, a.cols);
            if (c.any) {
                y[n] = c.fetch(a.dy, r * a.dys);
                h[n] = c.fetch(a.h, r * a.hs);
                const vec wn = KEEP ? w[KEEP ? n : 0] : c.fetch(a.w, 0);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float dy = c.owns(e) ? (float)y[n][e] : 0.0f, xh = c.owns(e) ? ((float)h[n][e] - mean) * rstd : 0.0f, g = dy * (float)wn[e];
                    dw[n * V + e] += dy * xh;
                    db[n * V + e] += dy;
                    s[0] += g;
                    s[1] += g * xh;
                }
            }
        }
        row_sum<THREADS, 2>(s, red);
        const float mg = s[0] / (float)a.cols, mx = s[1] / (float)a.cols;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Chunk<T, LOOSE> c((n * THREADS + t) * V, a.cols);
            if (c.any) {
                float d[V], u[V];
                if (a.dh) c.load(a.dh, r * a.dhs, u);
                const vec wn = KEEP ? w[KEEP ? n : 0] : c.fetch(a.w, 0);
#pragma unroll
                for (int e = 0; e < V; ++e) d[e] = rstd * ((float)y[n][e] * (float)wn[e] - mg - ((float)h[n][e] - mean) * rstd * mx) + (a.dh ? u[e] : 0.0f);
                c.store(a.dx, r * a.dxs, d);
            }
        }
    }
    if (!a.part) return;
    if constexpr (RPB > 1) {                // the rows of a wave into one, and then the four waves of a block, in turn
#pragma unroll
        for (int d = THREADS; d < 64; d *= 2)
#pragma unroll
            for (int e = 0; e < E; ++e) dw[e] += __shfl_xor(dw[e], d), db[e] += __shfl_xor(db[e], d);
        const int wave = threadIdx.x / 64;
        for (int k = 0; k < 4; ++k) {
            if (wave == k && threadIdx.x % 64 < SHARED)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (k) dw[e] += both[e * SHARED + t], db[e] += both[(E + e) * SHARED + t];
                    both[e * SHARED + t] = dw[e], both[(E + e) * SHARED + t] = db[e];
                }
            __syncthreads();
        }
        if (wave != 3 || threadIdx.x % 64 >= SHARED) return;
    }
    float *pw = a.part + (uint64_t)blockIdx.x * a.cols, *pb = pw + (uint64_t)a.groups * a.cols;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Chunk<T, LOOSE> c((n * THREADS + t) * V, a.cols);
        typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
        if (c.any)
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const float *u = dw + n * V + e, *v = db + n * V + e;
                if (c.owns(e) && c.owns(e + 3)) {
                    *(f32x4*)(pw + c.at + e) = f32x4{u[0], u[1], u[2], u[3]};
                    *(f32x4*)(pb + c.at + e) = f32x4{v[0], v[1], v[2], v[3]};
                } else
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (c.owns(e + i)) pw[c.at + e + i] = u[i], pb[c.at + e + i] = v[i];
            }
    }
}

// sums of the partial sums: 64 columns per block, 16 waves each a sixteenth of the groups
template <class T>
__global__ __launch_bounds__(1024) void k_layernorm_join(const float* part, uint32_t groups, uint32_t cols, void* dw, void* db)
{
    __shared__ float red[16][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.x * 64 + lane;
    void* out = blockIdx.y ? db : dw;
    if (!out) return;
    const float* p = part + (uint64_t)blockIdx.y * groups * cols;
    float s = 0;
    if (c < cols) {
#pragma unroll 8
        for (uint32_t g = wave; g < groups; g += 16) s += p[(uint64_t)g * cols + c];
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
        for (int k = 1; k < 16; ++k) s += red[k][lane];
        ((typename T::elem*)out)[c] = (typename T::elem)s;
    }
}

template <int THREADS, int E>
struct Row {        // lanes that share a row, and elements of a lane
    static constexpr int threads = THREADS, elems = E;
};

// Forward: a wave for rows of up to 2048 elements; its lanes hold little, so wide rows take few lanes and many elements (256 x 16 reads 16384 x 4096 elements
// in 41 us, 512 x 8 in 51).
template <class F>
int by_size_fwd(uint32_t cols, F f)
{
    if (cols <= 128) return f(Row<16, 8>());
    if (cols <= 512) return f(Row<64, 8>());
    if (cols <= 1024) return f(Row<64, 16>());
    if (cols <= 2048) return f(Row<64, 32>());
    if (cols <= 4096) return f(Row<256, 16>());
    if (cols <= 8192) return f(Row<512, 16>());
    if (cols <= 16384) return f(Row<1024, 16>());
    if (cols <= 32768) return f(Row<1024, 32>());
    return f(Row<1024, 64>());
}

// Backward: five values an element, three of them of the type, so few elements a lane (8192 x 8192 elements: 1024 x 8 takes 101 us, 512 x 16 117; 16384 x 2048: 256 x 8 41 us,
// 64 x 32 49), but for rows of a wave's own, whose sums need no barrier.  Beyond 16384 elements the weights are read again for every row (1000 x 30000 bfloats 101 us, kept 211), and a lane's
// values fit its registers barely (bfloat) or not.
template <class F>
int by_size_bwd(uint32_t cols, F f)
{
    if (cols <= 128) return f(Row<16, 8>());
    if (cols <= 512) return f(Row<64, 8>());
    if (cols <= 1024) return f(Row<64, 16>());
    if (cols <= 2048) return f(Row<256, 8>());
    if (cols <= 4096) return f(Row<512, 8>());
    if (cols <= 8192) return f(Row<1024, 8>());
    if (cols <= 16384) return f(Row<1024, 16>());
    if (cols <= 32768) return f(Row<1024, 32>());
    return f(Row<1024, 64>());
}

template <class T>
int fwd(FwdArgs a, bool vec, hipStream_t st)
{
    return by_size_fwd(a.cols, [&](auto row) {
        constexpr int TH = decltype(row)::threads, E = decltype(row)::elems;
        // a launch has fewer than 2^32 threads
        constexpr uint64_t MOST = MOST_THREADS / block_of(TH) * rows_of(TH);
        const dim3 block(block_of(TH));
        for (uint64_t left = a.rows; left; left -= a.rows) {
            a.rows = std::min(left, MOST);
            const dim3 grid((uint32_t)ceil_div(a.rows, rows_of(TH)));
            if (vec) k_layernorm_fwd<T, false, TH, E><<<grid, block, 0, st>>>(a);
            else k_layernorm_fwd<T, true, TH, E><<<grid, block, 0, st>>>(a);
            if (const int rc = launched()) return rc;
            const auto on = [&](auto* p, int64_t stride) { return p ? (decltype(p))((char*)p + (int64_t)a.rows * stride * (int64_t)sizeof(typename T::elem)) : p; };
            a.x = on(a.x, a.xs), a.res = on(a.res, a.rs), a.h = on(a.h, a.hs), a.y = on(a.y, a.ys);
            if (a.mean) a.mean += a.rows;
            if (a.rstd) a.rstd += a.rows;
        }
        return (int)FF_OK;
    });
}

template <class T>
int bwd(const BwdArgs& a, bool vec, void* dw, void* db, hipStream_t st)
{
    if (a.groups) {
        const int rc = by_size_bwd(a.cols, [&](auto row) {
            constexpr int TH = decltype(row)::threads, E = decltype(row)::elems;
            const dim3 grid(a.groups), block(block_of(TH));
            if (vec) k_layernorm_bwd<T, false, TH, E><<<grid, block, 0, st>>>(a);
            else k_layernorm_bwd<T, true, TH, E><<<grid, block, 0, st>>>(a);
            return launched();
        });
        if (rc != FF_OK) return rc;
    }
    if (!dw && !db) return FF_OK;
    k_layernorm_join<T><<<dim3((uint32_t)ceil_div(a.cols, 64), 2), 1024, 0, st>>>(a.part, a.groups, a.cols, dw, db);
    return launched();
}

size_t elem_bytes(uint32_t dtype) { return dtype == FF_F32 ? 4 : 2; }
bool vec_rows(const ff_rows_t& m, size_t e) { return aligned(m.p, 16) && (uint64_t)m.stride * e % 16 == 0; }

int check_size(uint32_t dtype, uint64_t rows, uint32_t cols)
{
    if (dtype > FF_BF16 || cols == 0) return FF_EINVAL;
    if (cols > FF_OP_MAX_COLS || rows > FF_OP_MAX_ROWS) return FF_ERANGE;
    return FF_OK;
}

// partial sums of the weight's gradient: as many blocks as fill the device (twice as many take 10 % longer on 16384 x 4096 elements, half as many 30 %)
uint32_t groups_of(uint64_t rows, uint32_t cols)
{
    return (uint32_t)by_size_bwd(cols, [&](auto row) {
        constexpr uint64_t TH = decltype(row)::threads, most = TH >= 512 ? 512 : 1024;
        return (int)std::min<uint64_t>(ceil_div(rows, rows_of(TH)), most);
    });
}

}  // namespace
}  // namespace ffops

using namespace ffops;

extern "C" int ff_op_layernorm_fwd(const ff_layernorm_fwd_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check_size(p->dtype, p->rows, p->cols)) return rc;
    if (!(p->eps >= 0) || !std::isfinite(p->eps)) return FF_EINVAL;
    if (p->rows == 0) return FF_OK;
    if (!p->x.p || !p->y.p || !p->weight || (p->res.p && !p->h.p)) return FF_EINVAL;
    const size_t e = elem_bytes(p->dtype);
    const bool vec = p->cols * e % 16 == 0 && vec_rows(p->x, e) && vec_rows(p->y, e) && (!p->res.p || (vec_rows(p->res, e) && vec_rows(p->h, e))) &&
                     aligned(p->weight, 16) && aligned(p->bias, 16);
    const FwdArgs a = {p->rows, p->cols, p->eps, p->x.p, p->res.p, p->h.p, p->y.p, p->x.stride, p->res.stride, p->h.stride, p->y.stride,
                       p->weight, p->bias, p->mean, p->rstd};
    const hipStream_t st = (hipStream_t)stream;
    return p->dtype == FF_F32 ? fwd<F32>(a, vec, st) : p->dtype == FF_F16 ? fwd<F16>(a, vec, st) : fwd<BF16>(a, vec, st);
}

extern "C" size_t ff_op_layernorm_bwd_workspace_bytes(const ff_layernorm_bwd_t* p)
{
    if (!p || check_size(p->dtype, p->rows, p->cols) != FF_OK || (!p->dweight && !p->dbias)) return 0;
    return (size_t)2 * groups_of(p->rows, p->cols) * p->cols * sizeof(float);
}

extern "C" int ff_op_layernorm_bwd(const ff_layernorm_bwd_t* p, void* stream)
{
    if (!p) return FF_EINVAL;
    if (const int rc = check_size(p->dtype, p->rows, p->cols)) return rc;
    if (p->rows && (!p->dy.p || !p->h.p || !p->dx.p || !p->weight || !p->mean || !p->rstd)) return FF_EINVAL;
    const size_t need = ff_op_layernorm_bwd_workspace_bytes(p);
    if (need && (!p->workspace || p->workspace_bytes < need || !aligned(p->workspace, 256))) return FF_EWORKSPACE;
    const size_t e = elem_bytes(p->dtype);
    const bool vec = p->cols * e % 16 == 0 && vec_rows(p->dy, e) && vec_rows(p->h, e) && vec_rows(p->dx, e) && (!p->dh.p || vec_rows(p->dh, e)) && aligned(p->weight, 16);
    const BwdArgs a = {p->rows, p->cols, groups_of(p->rows, p->cols), p->dy.p, p->h.p, p->dh.p, p->dx.p, p->dy.stride, p->h.stride, p->dh.stride, p->dx.stride,
                       p->weight, p->mean, p->rstd, need ? (float*)p->workspace : nullptr};
    const hipStream_t st = (hipStream_t)stream;
    return p->dtype == FF_F32 ? bwd<F32>(a, vec, p->dweight, p->dbias, st) : p->dtype == FF_F16 ? bwd<F16>(a, vec, p->dweight, p->dbias, st)
                                                                                               : bwd<BF16>(a, vec, p->dweight, p->dbias, st);
}
