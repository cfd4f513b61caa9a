// Root-mean-square norm of the sum of a row and its residual, with an output in the input's type or in 8 bits, and its gradient.
//
//   s = x + r,  rstd = (mean s^2 + eps)^-1/2,  y = s rstd gain          (e4m3: y / scale with scale = max |y| / 448)
//   dx = rstd (a - s rstd^2 mean(a s)) + dtotal,  a = dy gain;          dgain_j = sum_i dy_ij s_ij rstd_i
//
// Both are bound by memory: every matrix is read or written once, and a row stays in registers between the sums over it and the
// outputs that need them.  A row belongs to one wavefront (narrow rows: no barriers) or to one workgroup.  The sums are taken in
// 32 bits over the unrounded s (those of squares in 64 where 32 lose their range); `total` is s rounded to its type, and the gradient
// reads that.  The scale's maximum is taken with the sum of squares, over s gain, so 8 bits cost no further pass.
//
// Measured: 16384 x 8192 bf16 with a residual to e4m3 158 us (939 MB, 5.95 TB/s: outputs larger than 32 MB go past the caches, which keep what
// is read); one row of 4096 3.7 us of the device's time, 9 us a call; gradient of 20011 x 2047 f16 with all its inputs 100 us, of which 5 us
// the columns' sums (328 MB, 3.3 TB/s, rows at odd places; 16384 x 1024: 4.4 TB/s).
#include "head_util.h"

namespace tron {
namespace {

constexpr int kWaveRows = 4;            // wavefronts, each with rows of its own, of a workgroup over narrow rows
// Columns up to which a wavefront holds a row, and above which rows are read twice.  Both sides: 16384 x 2048 bf16 to e4m3 45 us by workgroups
// and 50 us by wavefronts, x 1024 19.4 us by either; 2048 x 32768 99 us held and 118 us read twice.
constexpr int64_t kNarrow = 1024;
constexpr int64_t kWide = 32768;

struct NormArgs {
    const void *x, *residual;
    const float *gain;
    void *total, *y;
    float *scale, *rstd;
    int64_t m, d, ldx, ldr, ldt, ldy;
    float eps, inv_d;
};

constexpr float kE4m3Max = 448.f;
constexpr float kLeastSquares = 0x1p-60f, kMostSquares = 0x1p100f;   // where a sum of squares has its digits in 32 bits, whatever parts are lost

template <typename T>
struct Elements {
    const T *p;
    int64_t d;
    __device__ __forceinline__ Raw8<T> at(int64_t j) const { return load_row8(p, j, d, static_cast<T>(0.f)); }
};

__device__ __forceinline__ void gain8(float *g, const float *gain, int64_t j, int64_t d)
{
    if (!gain) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) g[i] = 1.f;
        return;
    }
    const Raw8<float> r = Elements<float>{gain, d}.at(j);
#pragma unroll
    for (int i = 0; i < kVec; ++i) g[i] = r.v[i];
}

// What a row's sums give: its factors
struct RowFactors {
    float rstd, scale, per_scale;
};
// From a thread's sum of squares and its max |s gain|, by a wavefront or a workgroup.  The sum is joined in 32 bits, and in 64 once more where
// these have lost its range, so that rows of any size have their rstd.
template <bool WAVE, bool EIGHT>
__device__ __forceinline__ RowFactors row_factors(double own, float top, float eps, float inv_d)
{
    __shared__ float room[2 * kMostWaves];
    __shared__ double wide_room[kMostWaves];
    float sum2 = (float)own;
    if (WAVE) {
        sum2 = wave_sumf(sum2);
        if (EIGHT) top = wave_maxf(top);
    } else if (EIGHT) {
        block_sum_max(sum2, top, room);
    } else {
        sum2 = block_sum_all(sum2, room);
    }
    RowFactors f;
    if (sum2 >= kLeastSquares && sum2 <= kMostSquares) f.rstd = 1.f / sqrtf(sum2 * inv_d + eps);
    else f.rstd = (float)(1.0 / sqrt((WAVE ? wave_sum(own) : block_sum_all(own, wide_room)) * (double)inv_d + (double)eps));
    // max |y| = rstd max |s gain|; a row of zeros (and one with a NaN, which every y then is) has scale 1.  The smallest normal
    // number as the least scale has a finite reciprocal.
    const float largest = top * f.rstd;
    f.scale = largest > 0.f ? fmaxf(largest / kE4m3Max, 0x1p-126f) : 1.f;
    f.per_scale = 1.f / f.scale;
    return f;
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

// CH chunks of eight elements a thread; WAVE: a wavefront a row, otherwise a workgroup
template <typename T, typename O, int CH, bool WAVE, bool PAST>
__global__ __launch_bounds__(WAVE ? kWaveRows * kWave : 1024) void k_rms_norm(NormArgs A)
{
    constexpr bool kEight = sizeof(O) == 1;
    const int team = WAVE ? kWave : (int)blockDim.x, me = WAVE ? (int)threadIdx.x % kWave : (int)threadIdx.x;
    const int64_t row = WAVE ? block_number() * kWaveRows + threadIdx.x / kWave : block_number();
    if (row >= A.m) return;
    const int64_t d = A.d;
    const Elements<T> x{static_cast<const T *>(A.x) + row * A.ldx, d};
    float s[CH][kVec];
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t j = (int64_t)(me + c * team) * kVec;
        if (j < d) {
            const Raw8<T> v = x.at(j);
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[c][i] = static_cast<float>(v.v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[c][i] = 0.f;
        }
    }
    if (A.residual) {
        const Elements<T> r{static_cast<const T *>(A.residual) + row * A.ldr, d};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t j = (int64_t)(me + c * team) * kVec;
            if (j < d) {
                const Raw8<T> v = r.at(j);
#pragma unroll
                for (int i = 0; i < kVec; ++i) s[c][i] += static_cast<float>(v.v[i]);
            }
        }
    }
    const double sum2 = squares(s);
    if (A.total) {
        T *t = static_cast<T *>(A.total) + row * A.ldt;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t j = (int64_t)(me + c * team) * kVec;
            if (j < d) store8_of<T, PAST>(t + j, s[c], d - j);
        }
    }
    // s gain from here on
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t j = (int64_t)(me + c * team) * kVec;
        if (j < d) {
            float g[kVec];
            gain8(g, A.gain, j, d);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                s[c][i] *= g[i];
                if (kEight) top = fmaxf(top, fabsf(s[c][i]));
            }
        }
    }
    const RowFactors f = row_factors<WAVE, kEight>(sum2, top, A.eps, A.inv_d);
    if (me == 0) {
        if (A.rstd) A.rstd[row] = f.rstd;
        if (kEight) A.scale[row] = f.scale;
    }
    O *y = static_cast<O *>(A.y) + row * A.ldy;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t j = (int64_t)(me + c * team) * kVec;
        if (j < d) {
            float v[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = kEight ? s[c][i] * f.rstd * f.per_scale : s[c][i] * f.rstd;
            store8_of<O, PAST>(y + j, v, d - j);
        }
    }
}

// Rows that registers do not hold: read twice.  What is written lies behind the thread's last read of it, so `total` may be x or r.
template <typename T, typename O, bool PAST>
__global__ __launch_bounds__(1024) void k_rms_norm_wide(NormArgs A)
{
    constexpr bool kEight = sizeof(O) == 1;
    const int64_t row = block_number(), d = A.d, step = (int64_t)blockDim.x * kVec;
    if (row >= A.m) return;
    const Elements<T> x{static_cast<const T *>(A.x) + row * A.ldx, d}, r{static_cast<const T *>(A.residual) + (A.residual ? row * A.ldr : 0), d};
    auto sum8 = [&](float *s, int64_t j) {
        const Raw8<T> v = x.at(j);
#pragma unroll
        for (int i = 0; i < kVec; ++i) s[i] = static_cast<float>(v.v[i]);
        if (A.residual) {
            const Raw8<T> u = r.at(j);
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[i] += static_cast<float>(u.v[i]);
        }
    };
    double sum2 = 0.0;
    float top = 0.f;
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        float s[kVec], g[kVec];
        sum8(s, j);
        if (kEight) gain8(g, A.gain, j, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            sum2 = fma((double)s[i], (double)s[i], sum2);
            if (kEight) top = fmaxf(top, fabsf(s[i] * g[i]));
        }
    }
    const RowFactors f = row_factors<false, kEight>(sum2, top, A.eps, A.inv_d);
    if (threadIdx.x == 0) {
        if (A.rstd) A.rstd[row] = f.rstd;
        if (kEight) A.scale[row] = f.scale;
    }
    O *y = static_cast<O *>(A.y) + row * A.ldy;
    T *t = static_cast<T *>(A.total) + (A.total ? row * A.ldt : 0);
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        float s[kVec], g[kVec];
        sum8(s, j);
        if (A.total) store8_of<T, PAST>(t + j, s, d - j);
        gain8(g, A.gain, j, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i) s[i] = kEight ? s[i] * g[i] * f.rstd * f.per_scale : s[i] * g[i] * f.rstd;
        store8_of<O, PAST>(y + j, s, d - j);
    }
}

// ------------------------------------------------------------------ gradient
struct NormGradArgs {
    const void *total, *dy, *dtotal;
    const float *gain, *rstd;
    void *dx;
    float *partial;   // [workgroups][d]: their shares of dgain, or NULL
    int64_t m, d, lds, lddy, lddt, lddx;
    float inv_d;
};

// Teams (wavefronts or workgroups) keep their columns' shares of dgain in registers.  Where a thread holds one chunk of a row, they take two rows
// at a time: one barrier and one wait for memory serve both (20011 x 4096 f16: 175 us one at a time, 141 us; with two chunks of two rows
// the registers are short, and it is slower).
template <typename T, int CH, bool WAVE, bool PAST>
__global__ __launch_bounds__(WAVE ? kWaveRows * kWave : 1024) void k_rms_norm_grad(NormGradArgs A)
{
    constexpr int kRows = CH == 1 ? 2 : 1;
    __shared__ float room[2][kRows][kMostWaves];
    const int team = WAVE ? kWave : (int)blockDim.x, me = WAVE ? (int)threadIdx.x % kWave : (int)threadIdx.x;
    const int64_t teams = WAVE ? (int64_t)gridDim.x * kWaveRows : gridDim.x;
    const int64_t first = WAVE ? (int64_t)blockIdx.x * kWaveRows + threadIdx.x / kWave : blockIdx.x;
    const int64_t d = A.d;
    float g[CH][kVec], dg[CH][kVec];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t j = (int64_t)(me + c * team) * kVec;
#pragma unroll
        for (int i = 0; i < kVec; ++i) g[c][i] = dg[c][i] = 0.f;
        if (j < d) gain8(g[c], A.gain, j, d);
    }
    int turn = 0;
    for (int64_t row0 = first; row0 < A.m; row0 += kRows * teams, turn ^= 1) {
        Raw8<T> s[kRows][CH], dy[kRows][CH], dt[kRows][CH];
        float rstd[kRows], dot[kRows];
#pragma unroll
        for (int q = 0; q < kRows; ++q) {
            const int64_t row = row0 + q * teams;
            const bool there = row < A.m;
            const Elements<T> sv{static_cast<const T *>(A.total) + row * A.lds, d}, dyv{static_cast<const T *>(A.dy) + row * A.lddy, d};
            const Elements<T> dtv{static_cast<const T *>(A.dtotal) + (A.dtotal ? row * A.lddt : 0), d};
            rstd[q] = there ? A.rstd[row] : 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t j = (int64_t)(me + c * team) * kVec;
                if (there && j < d) {
                    s[q][c] = sv.at(j);
                    dy[q][c] = dyv.at(j);
                    if (A.dtotal) dt[q][c] = dtv.at(j);
                } else {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) s[q][c].v[i] = dy[q][c].v[i] = static_cast<T>(0.f);
                }
            }
        }
#pragma unroll
        for (int q = 0; q < kRows; ++q) {
            dot[q] = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float a = static_cast<float>(dy[q][c].v[i]), v = static_cast<float>(s[q][c].v[i]);
                    dot[q] = fmaf(a * g[c][i], v, dot[q]);
                    dg[c][i] = fmaf(a, v * rstd[q], dg[c][i]);
                }
            dot[q] = wave_sumf(dot[q]);
        }
        if (!WAVE) {
            // two rooms in turn: who writes the next rows' sums has passed the barrier behind which the last ones of this room were read
            const int waves = blockDim.x / kWave;
            if (threadIdx.x % kWave == 0) {
#pragma unroll
                for (int q = 0; q < kRows; ++q) room[turn][q][threadIdx.x / kWave] = dot[q];
            }
            __syncthreads();
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                dot[q] = 0.f;
                for (int w = 0; w < waves; ++w) dot[q] += room[turn][q][w];
            }
        }
#pragma unroll
        for (int q = 0; q < kRows; ++q) {
            const int64_t row = row0 + q * teams;
            if (row >= A.m) break;
            const float back = rstd[q] * (rstd[q] * (dot[q] * A.inv_d));   // not rstd^2, which may be no number of 32 bits
            T *dx = static_cast<T *>(A.dx) + row * A.lddx;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t j = (int64_t)(me + c * team) * kVec;
                if (j < d) {
                    float v[kVec];
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        v[i] = rstd[q] * (static_cast<float>(dy[q][c].v[i]) * g[c][i] - static_cast<float>(s[q][c].v[i]) * back);
                        if (A.dtotal) v[i] += static_cast<float>(dt[q][c].v[i]);
                    }
                    store8_of<T, PAST>(dx + j, v, d - j);
                }
            }
        }
    }
    if (!A.partial) return;
    if (WAVE) {   // the wavefronts of a workgroup join their shares, a chunk of columns at a time
        __shared__ float join[kWaveRows][kWave * kVec];
        const int wave = threadIdx.x / kWave;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (c) __syncthreads();
#pragma unroll
            for (int i = 0; i < kVec; ++i) join[wave][me * kVec + i] = dg[c][i];
            __syncthreads();
            for (int k = threadIdx.x; k < kWave * kVec; k += kWaveRows * kWave) {
                const int64_t j = (int64_t)c * kWave * kVec + k;
                if (j >= d) break;
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < kWaveRows; ++w) sum += join[w][k];
                A.partial[(int64_t)blockIdx.x * d + j] = sum;
            }
        }
    } else {
        float *p = A.partial + first * d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t j = (int64_t)(me + c * team) * kVec;
            if (j < d) store8_of<float>(p + j, dg[c], d - j);
        }
    }
}

template <typename T, bool PAST>
__global__ __launch_bounds__(1024) void k_rms_norm_grad_wide(NormGradArgs A)
{
    __shared__ float room[kMostWaves];
    const int64_t row = block_number(), d = A.d, step = (int64_t)blockDim.x * kVec;
    if (row >= A.m) return;
    const Elements<T> sv{static_cast<const T *>(A.total) + row * A.lds, d}, dyv{static_cast<const T *>(A.dy) + row * A.lddy, d};
    const Elements<T> dtv{static_cast<const T *>(A.dtotal) + (A.dtotal ? row * A.lddt : 0), d};
    float dot = 0.f;
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        const Raw8<T> s = sv.at(j), dy = dyv.at(j);
        float g[kVec];
        gain8(g, A.gain, j, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i) dot = fmaf(static_cast<float>(dy.v[i]) * g[i], static_cast<float>(s.v[i]), dot);
    }
    dot = block_sum_all(dot, room);
    const float rstd = A.rstd[row], back = rstd * (rstd * (dot * A.inv_d));
    T *dx = static_cast<T *>(A.dx) + row * A.lddx;
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        const Raw8<T> s = sv.at(j), dy = dyv.at(j);
        float g[kVec], v[kVec];
        gain8(g, A.gain, j, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = rstd * (static_cast<float>(dy.v[i]) * g[i] - static_cast<float>(s.v[i]) * back);
        if (A.dtotal) {
            const Raw8<T> dt = dtv.at(j);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += static_cast<float>(dt.v[i]);
        }
        store8_of<T, PAST>(dx + j, v, d - j);
    }
}

// shares of dgain of rows that registers do not hold: a thread a column, gridDim.y shares
template <typename T>
__global__ __launch_bounds__(kBlock) void k_gain_shares(NormGradArgs A)
{
    const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (j >= A.d) return;
    float sum = 0.f;
    for (int64_t row = blockIdx.y; row < A.m; row += gridDim.y)
        sum = fmaf(static_cast<float>(static_cast<const T *>(A.dy)[row * A.lddy + j]),
                   static_cast<float>(static_cast<const T *>(A.total)[row * A.lds + j]) * A.rstd[row], sum);
    A.partial[blockIdx.y * A.d + j] = sum;
}

}  // namespace

// out_j = sum over the rows of shares, in a fixed order: 16 columns a workgroup, which 64 groups of 16 lanes walk down, four loads ahead
__global__ __launch_bounds__(1024) void k_column_sums(const float *shares, int64_t count, int64_t d, float *out)
{
    constexpr int kColumns = 16, kGroups = 1024 / kColumns;
    __shared__ float room[kGroups][kColumns + 1];
    const int c = threadIdx.x % kColumns, group = threadIdx.x / kColumns;
    const int64_t j = (int64_t)blockIdx.x * kColumns + c;
    float sum = 0.f;
    if (j < d) {
        int64_t i = group;
        for (; i + 3 * kGroups < count; i += 4 * kGroups) {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = shares[(i + k * kGroups) * d + j];
            sum += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; i < count; i += kGroups) sum += shares[i * d + j];
    }
    room[group][c] = sum;
    __syncthreads();
    for (int half = kGroups / 2; half; half /= 2) {
        if (group < half) room[group][c] += room[group + half][c];
        __syncthreads();
    }
    if (group == 0 && j < d) out[j] = room[0][c];
}

int column_sums(const float *shares, int64_t count, int64_t d, float *out, hipStream_t st)
{
    k_column_sums<<<(unsigned)ceil_div(d, 16), 1024, 0, st>>>(shares, count, d, out);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

namespace {

// threads of a workgroup that holds a row in CH chunks a thread
inline unsigned row_threads(int64_t d, int ch) { return (unsigned)(ceil_div(ceil_div(d, kVec), (int64_t)ch * kWave) * kWave); }

template <typename T, typename O, bool PAST>
int norm_launch(const NormArgs &A, hipStream_t st)
{
    const int64_t d = A.d;
    if (d <= kNarrow) {
        const dim3 grid = block_grid(ceil_div(A.m, kWaveRows));
        if (d <= 512) k_rms_norm<T, O, 1, true, PAST><<<grid, kWaveRows * kWave, 0, st>>>(A);
        else k_rms_norm<T, O, 2, true, PAST><<<grid, kWaveRows * kWave, 0, st>>>(A);
    } else if (d <= 8192) {
        k_rms_norm<T, O, 2, false, PAST><<<block_grid(A.m), row_threads(d, 2), 0, st>>>(A);
    } else if (d <= kWide) {
        k_rms_norm<T, O, 4, false, PAST><<<block_grid(A.m), row_threads(d, 4), 0, st>>>(A);
    } else {
        k_rms_norm_wide<T, O, PAST><<<block_grid(A.m), 1024, 0, st>>>(A);
    }
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

template <typename T>
int norm_typed(const NormArgs &A, bool eight, hipStream_t st)
{
    const bool past = goes_past(A.m, A.d, (A.total ? sizeof(T) : 0) + (eight ? 1 : sizeof(T)));
    if (eight) return past ? norm_launch<T, e4m3, true>(A, st) : norm_launch<T, e4m3, false>(A, st);
    return past ? norm_launch<T, T, true>(A, st) : norm_launch<T, T, false>(A, st);
}

// Columns up to which a wavefront of the gradient holds its rows (gain, share and two rows of three matrices), and above which rows are
// read twice.  Both sides: 16384 x 1024 f16 30.5 us by wavefronts and 41.6 us by workgroups, 4096 x 16384 125 us held and 191 us read twice.
constexpr int64_t kGradNarrow = 1024;
constexpr int64_t kGradWide = 16384;

// workgroups of the gradient, each with a share of dgain
int64_t grad_shares(int64_t m, int64_t d)
{
    if (d <= kGradNarrow) return std::min<int64_t>(ceil_div(m, kWaveRows), 1024);
    return std::min<int64_t>(m, d <= 2048 ? 1024 : d <= kGradWide ? 512 : 64);
}

template <typename T, bool PAST>
int norm_grad_typed(const NormGradArgs &A, float *dgain, hipStream_t st)
{
    const int64_t d = A.d;
    const unsigned shares = (unsigned)grad_shares(A.m, d);
    if (d <= kGradNarrow) {
        if (d <= 512) k_rms_norm_grad<T, 1, true, PAST><<<shares, kWaveRows * kWave, 0, st>>>(A);
        else k_rms_norm_grad<T, 2, true, PAST><<<shares, kWaveRows * kWave, 0, st>>>(A);
    } else if (d <= 8192) {
        k_rms_norm_grad<T, 1, false, PAST><<<shares, row_threads(d, 1), 0, st>>>(A);
    } else if (d <= kGradWide) {
        k_rms_norm_grad<T, 2, false, PAST><<<shares, row_threads(d, 2), 0, st>>>(A);
    } else {
        // before dx is written, which may be dy
        if (A.partial) k_gain_shares<T><<<dim3((unsigned)ceil_div(d, kBlock), shares), kBlock, 0, st>>>(A);
        k_rms_norm_grad_wide<T, PAST><<<block_grid(A.m), 1024, 0, st>>>(A);
    }
    TRON_HIP(hipGetLastError());
    return dgain ? column_sums(A.partial, shares, d, dgain, st) : TRON_OK;
}

template <typename T>
int norm_grad_typed(const NormGradArgs &A, float *dgain, hipStream_t st)
{
    return goes_past(A.m, A.d, sizeof(T)) ? norm_grad_typed<T, true>(A, dgain, st) : norm_grad_typed<T, false>(A, dgain, st);
}

}  // namespace
}  // namespace tron

using namespace tron;

extern "C" {

int tron_rms_norm(int64_t m, int64_t d, int type, const void *x, int64_t ldx, const void *residual, int64_t ldr, const float *gain, double eps,
                  void *total, int64_t ldt, int out_type, void *y, int64_t ldy, float *scale, float *rstd, void *hip_stream)
{
    const bool eight = out_type == TRON_TYPE_E4M3;
    if (m < 0 || d < 1 || m > INT32_MAX || !type_is_float(type) || (out_type != type && !eight) || !(eps >= 0.0) || !(eps < HUGE_VAL)) {
        set_error("tron_rms_norm: bad argument (need 0 <= m < 2^31, d >= 1, type f32, bf16 or f16, out_type that type or e4m3, finite eps >= 0)");
        return TRON_EINVAL;
    }
    if (m > 0 && (!x || !y || (eight && !scale) || !rows_ok(m, d, ldx, false) || (residual && !rows_ok(m, d, ldr, false)) ||
                  (total && !rows_ok(m, d, ldt, true)) || !rows_ok(m, d, ldy, true) || !extent_ok(m, ldx, d) || !extent_ok(m, residual ? ldr : 0, d) ||
                  !extent_ok(m, total ? ldt : 0, d) || !extent_ok(m, ldy, d))) {
        set_error("tron_rms_norm: bad argument (x, y and, for e4m3, scale are needed; rows that are written may not overlap)");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    if (m == 0) return TRON_OK;
    const NormArgs A{x, residual, gain, total, y, scale, rstd, m, d, ldx, ldr, ldt, ldy, (float)eps, (float)(1.0 / (double)d)};
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    return type == TRON_TYPE_F32 ? norm_typed<float>(A, eight, st) : type == TRON_TYPE_BF16 ? norm_typed<__bf16>(A, eight, st) : norm_typed<_Float16>(A, eight, st);
}

int64_t tron_rms_norm_grad_work(int64_t m, int64_t d)
{
    if (m < 1 || d < 1 || m > INT32_MAX || !extent_ok(grad_shares(m, d), d, d)) return 0;
    return grad_shares(m, d) * d * (int64_t)sizeof(float);
}

int tron_rms_norm_grad(int64_t m, int64_t d, int type, const void *total, int64_t lds, const float *rstd, const float *gain, const void *dy, int64_t lddy,
                       const void *dtotal, int64_t lddt, void *dx, int64_t lddx, float *dgain, void *work, int64_t work_bytes, void *hip_stream)
{
    if (m < 0 || d < 1 || m > INT32_MAX || !type_is_float(type)) {
        set_error("tron_rms_norm_grad: bad argument (need 0 <= m < 2^31, d >= 1, type f32, bf16 or f16)");
        return TRON_EINVAL;
    }
    if (m > 0 && (!total || !rstd || !dy || !dx || !rows_ok(m, d, lds, false) || !rows_ok(m, d, lddy, false) || (dtotal && !rows_ok(m, d, lddt, false)) ||
                  !rows_ok(m, d, lddx, true) || !extent_ok(m, lds, d) || !extent_ok(m, lddy, d) || !extent_ok(m, dtotal ? lddt : 0, d) || !extent_ok(m, lddx, d))) {
        set_error("tron_rms_norm_grad: bad argument (total, rstd, dy and dx are needed; the rows of dx may not overlap)");
        return TRON_EINVAL;
    }
    if (dgain && !work_ok(work, work_bytes, tron_rms_norm_grad_work(m, d))) {
        set_error("tron_rms_norm_grad: dgain needs a work space of tron_rms_norm_grad_work(m, d) bytes at a multiple of 16");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    if (m == 0) return dgain ? column_sums(nullptr, 0, d, dgain, st) : TRON_OK;
    const NormGradArgs A{total, dy, dtotal, gain, rstd, dx, dgain ? static_cast<float *>(work) : nullptr, m, d, lds, lddy, lddt, lddx, (float)(1.0 / (double)d)};
    return type == TRON_TYPE_F32 ? norm_grad_typed<float>(A, dgain, st)
           : type == TRON_TYPE_BF16 ? norm_grad_typed<__bf16>(A, dgain, st) : norm_grad_typed<_Float16>(A, dgain, st);
}

}  // extern "C"
