// What the kernels over normalised rows share: a row's elements, its columns' factors, sums of squares, the scale of an output in 8 bits.
#pragma once

#include "head_util.h"

namespace tron {
namespace {

constexpr int kWaveRows = 4;            // wavefronts, each with rows of its own, of a workgroup over narrow rows

// What an output in 8 bits is scaled to
template <typename O>
constexpr float kLargest = __is_same(O, whole8) ? 127.f : 448.f;
constexpr float kLeastSquares = 0x1p-60f, kMostSquares = 0x1p100f;   // where a sum of squares has its digits in 32 bits, whatever parts are lost

template <typename T>
struct Elements {
    const T *p;
    int64_t d;
    __device__ __forceinline__ Raw8<T> at(int64_t j) const { return load_row8(p, j, d, static_cast<T>(0.f)); }
};

// eight factors of columns, 1 without any (or terms: `none`)
__device__ __forceinline__ void gain8(float *g, const float *gain, int64_t j, int64_t d, float none = 1.f)
{
    if (!gain) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) g[i] = none;
        return;
    }
    const Raw8<float> r = Elements<float>{gain, d}.at(j);
#pragma unroll
    for (int i = 0; i < kVec; ++i) g[i] = r.v[i];
}

// A thread's sum of squares: in 64 bits anew where 32 have lost its range.  (All sums in 64 bits: 16384 x 8192 bf16 to e4m3 167 us instead of 162.)
template <int CH>
__device__ __forceinline__ double squares(const float (&s)[CH][kVec])
{
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum = fmaf(s[c][i], s[c][i], sum);
    if (sum >= kLeastSquares && sum <= kMostSquares) return sum;
    double wide = 0.0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < kVec; ++i) wide = fma((double)s[c][i], (double)s[c][i], wide);
    return wide;
}

// Scale of a row whose largest |y| is `largest`.  A row of zeros has scale 1; the smallest normal number as the least scale has a finite
// reciprocal.  e4m3 holds NaN itself (and a row with one has the scale of the others, or 1); a row of whole numbers where some y is not finite has the scale NaN.
template <typename O>
__device__ __forceinline__ float scale_for(float largest)
{
    if (__is_same(O, whole8) && !(largest < INFINITY)) return NAN;
    return largest > 0.f ? fmaxf(largest / kLargest<O>, 0x1p-126f) : 1.f;
}

// threads of a workgroup that holds a row in CH chunks a thread
inline unsigned row_threads(int64_t d, int ch) { return (unsigned)(ceil_div(ceil_div(d, kVec), (int64_t)ch * kWave) * kWave); }

}  // namespace
}  // namespace tron
