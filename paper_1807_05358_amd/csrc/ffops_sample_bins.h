// The bins of logits that the choice of a word sums weights in: plain arithmetic, for the kernel and for the host.
#pragma once
#include <cstdint>

#ifdef __HIP__
#define FFOPS_BOTH __host__ __device__ __forceinline__
#else
#define FFOPS_BOTH inline
#endif

namespace ffops {

constexpr int BINS = 4096, BELOW = 2816;    // bins; those below the anchor

// The bins of a row; the anchor, a finite logit, is at the lower edge of bin BELOW.
struct Bins {
    double anchor, per_logit, width;        // bins in a unit of the logits, and its inverse
    float c[4];                             // 2^29 (e^(r / per_nat) - 1) as a sum of powers of r, and 0.5

    FFOPS_BOTH void set(float anchor_, float temperature, int per_nat)
    {
        anchor = anchor_, per_logit = per_nat / (double)temperature, width = (double)temperature / per_nat;
        const float h = 1.0f / per_nat;
        c[0] = 0x1p29f * h, c[1] = 0x1p28f * h * h, c[2] = 0x1p29f / 6 * h * h * h, c[3] = 0x1p29f / 24 * h * h * h * h;
    }
    // the place of a logit in bins, the lowest of which begins at 1: what is below is then cut off to 0
    FFOPS_BOTH double place(float z) const { return __builtin_fma((double)z - anchor, per_logit, (double)(BELOW + 1)); }
    // A logit on the safe side (-1: below, 1: above) of a bin's lower edge.  place() is off by 2^-39 of a bin at most (two roundings of what it adds, up to 2^12 bins, and one of a sum up to 2^13), an edge by 2^-41 of one and a
    // float's rounding, so a thousandth of a bin is plenty, also where the edge is at or near 0.  Words between that and the edge are found out when their bins are looked at.
    FFOPS_BOTH float logit(int bin, int side) const
    {
        const double edge = __builtin_fma((double)(bin - BELOW), width, anchor);
        return (float)(edge + side * (__builtin_fabs(edge) * 1e-6 + width * 1e-3 + 1e-30));
    }
    // a bin's number, -1 and BINS beyond them, and that + 1
    FFOPS_BOTH int slot(double at) const { const int n = (int)at; return n < 0 ? 0 : n > BINS + 1 ? BINS + 1 : n; }
    FFOPS_BOTH int bin(double at) const { return slot(at) - 1; }
    // e^(r / per_nat), 0 <= r < 1, in steps of 2^-29, to the nearest: what is beyond 1 is below 2^-4.9, so a float has it to half of such a step
    FFOPS_BOTH uint32_t steps(float r) const { return (1u << 29) + (uint32_t)__builtin_fmaf(r, __builtin_fmaf(r, __builtin_fmaf(r, __builtin_fmaf(r, c[3], c[2]), c[1]), c[0]), 0.5f); }
};

// Bins in a unit of the temperature, where the largest logits of the threads' shares lie so many units apart: in most rows the others are no more than three times that, and a little, below the largest, so bins are as narrow as
// reaches that far and the words of a few of them are few.  Where it does not, the row is read again.  256 rows of 131071 normal logits, top_p 0.9, with 64 bins a unit and so: deviation 1 unit 1100 us and 80, 2.5 units
// 71 and 66, 4 units 51 and 50.
FFOPS_BOTH int bins_per_nat(float apart)
{
    const int n = (int)(BELOW / (3 * apart + (apart < 2.0f ? apart : 2.0f)));
    return n < 32 ? 32 : n > 1 << 16 ? 1 << 16 : n;
}

}  // namespace ffops
