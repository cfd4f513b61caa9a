// Layer norm of the sum of a row and its residual, with an output in the input's type or in 8 bits, and its gradient.
//
//   s = x + r,  rstd = (mean (s - mean s)^2 + eps)^-1/2,  h = (s - mean s) rstd,  y = h gain + shift     (8 bits: y / scale, scale = max |y| / 448 or 127)
//   dx = rstd (a - mean a - h mean(a h)) + dtotal,  a = dy gain;     dgain_j = sum_i dy_ij h_ij,  dshift_j = sum_i dy_ij
//
// Both are bound by memory: every matrix is read or written once, and a row stays in the registers of a wavefront (narrow rows: no barriers) or
// of a workgroup.  The mean is taken first and the squares are those of differences to it, so that rows that lie far from 0 keep the
// digits of their variance: with m the mean rounded to 32 bits and c = s - m,  mean s = m + mean c  and  variance = mean c^2 - (mean c)^2.  mean c is what
// the rounding of m and the order of its sum left; it is subtracted from c once more.
#include "head_rows.h"

namespace tron {
namespace {

// Columns up to which a wavefront holds a row, and above which rows are read twice
constexpr int64_t kNarrow = 1024;
constexpr int64_t kWide = 32768;

struct LayerArgs {
    const void *x, *residual;
    const float *gain, *shift;
    void *total, *y;
    float *scale, *mean, *rstd;
    int64_t m, d, ldx, ldr, ldt, ldy;
    double eps, inv_d;
};

struct Moments {
    float mean, rest, rstd;   // c = (s - mean) - rest
};

// CH chunks of eight elements a thread; WAVE: a wavefront a row, otherwise a workgroup
template <typename T, typename O, int CH, bool WAVE, bool PAST>
__global__ __launch_bounds__(WAVE ? kWaveRows * kWave : 1024) void k_layer_norm(LayerArgs A)
{
    constexpr bool kEight = sizeof(O) == 1, kWhole = __is_same(O, whole8);
    __shared__ float room[5 * kMostWaves];
    __shared__ double wide_room[3 * kMostWaves];
    const int team = WAVE ? kWave : (int)blockDim.x, me = WAVE ? (int)threadIdx.x % kWave : (int)threadIdx.x;
    const int64_t row = WAVE ? block_number() * kWaveRows + threadIdx.x / kWave : block_number();
    if (row >= A.m) return;
    const int64_t d = A.d;
    const Elements<T> x{static_cast<const T *>(A.x) + row * A.ldx, d};
    float s[CH][kVec];
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
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum += s[c][i];
    if (A.total) {
        T *t = static_cast<T *>(A.total) + row * A.ldt;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t j = (int64_t)(me + c * team) * kVec;
            if (j < d) store8_of<T, PAST>(t + j, s[c], d - j);
        }
    }
    Moments M;
    sum = WAVE ? wave_sumf(sum) : block_sum_all(sum, room);
    M.mean = sum * (float)A.inv_d;
    if (!(fabsf(sum) <= kMostSquares)) {   // more than 32 bits hold, or no number
        double wide = 0.0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < kVec; ++i) wide += (double)s[c][i];
        M.mean = (float)((WAVE ? wave_sum(wide) : block_sum_all(wide, wide_room)) * A.inv_d);
    }
    float own = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        // columns behind the row's end stay 0
        const int64_t n = d - (int64_t)(me + c * team) * kVec;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            s[c][i] = i < n ? s[c][i] - M.mean : 0.f;
            own += s[c][i];
        }
    }
    const double own2 = squares(s);
    float left = own, sum2 = (float)own2;
    if (WAVE) {
        left = wave_sumf(left);
        sum2 = wave_sumf(sum2);
    } else {
        block_sum_two(left, sum2, room + kMostWaves);
    }
    if (sum2 >= kLeastSquares && sum2 <= kMostSquares) {
        const float inv_d = (float)A.inv_d;
        M.rest = left * inv_d;
        M.rstd = 1.f / sqrtf(fmaxf((sum2 - left * M.rest) * inv_d, 0.f) + (float)A.eps);
    } else {
        double wide = 0.0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < kVec; ++i) wide += (double)s[c][i];
        const double l = WAVE ? wave_sum(wide) : block_sum_all(wide, wide_room + kMostWaves);
        const double l2 = WAVE ? wave_sum(own2) : block_sum_all(own2, wide_room + 2 * kMostWaves);
        M.rest = (float)(l * A.inv_d);
        const double variance = (l2 - l * (l * A.inv_d)) * A.inv_d;
        M.rstd = (float)(1.0 / sqrt((variance < 0.0 ? 0.0 : variance) + A.eps));   // NaN stays NaN
    }
    // y from here on
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t j = (int64_t)(me + c * team) * kVec;
        if (j < d) {
            float g[kVec], b[kVec];
            gain8(g, A.gain, j, d);
            gain8(b, A.shift, j, d, 0.f);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                s[c][i] = fmaf((s[c][i] - M.rest) * M.rstd, g[i], b[i]);
                if (kEight && i < d - j) top = larger<kWhole>(top, fabsf(s[c][i]));
            }
        }
    }
    float scale = 1.f, per_scale = 1.f;
    if (kEight) {
        if (kWhole) top = WAVE ? wave_top<true>(top) : block_top<true>(top, room + 3 * kMostWaves);
        else top = WAVE ? wave_top<false>(top) : block_top<false>(top, room + 3 * kMostWaves);
        scale = scale_for<O>(top);
        per_scale = 1.f / scale;
    }
    if (me == 0) {
        if (A.mean) A.mean[row] = M.mean + M.rest;
        if (A.rstd) A.rstd[row] = M.rstd;
        if (kEight) A.scale[row] = scale;
    }
    O *y = static_cast<O *>(A.y) + row * A.ldy;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t j = (int64_t)(me + c * team) * kVec;
        if (j < d) {
            if (kEight) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) s[c][i] *= per_scale;
            }
            store8_of<O, PAST>(y + j, s[c], d - j);
        }
    }
}

// Rows that registers do not hold: read twice, or three times for an output in 8 bits.  The squares are those of differences to the row's first
// element, in 64 bits: it is one of the row's own, so that the variance is at least the d-th part of its squared distance to the mean.
// What is written lies behind the thread's last read of it, so `total` may be x or r.
template <typename T, typename O, bool PAST>
__global__ __launch_bounds__(1024) void k_layer_norm_wide(LayerArgs A)
{
    constexpr bool kEight = sizeof(O) == 1, kWhole = __is_same(O, whole8);
    __shared__ double room[2 * kMostWaves];
    __shared__ float top_room[kMostWaves];
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
    const double pivot = (double)(static_cast<float>(x.p[0]) + (A.residual ? static_cast<float>(r.p[0]) : 0.f));
    double sum = 0.0, sum2 = 0.0;
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        float s[kVec];
        sum8(s, j);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const double c = i < d - j ? (double)s[i] - pivot : 0.0;
            sum += c;
            sum2 = fma(c, c, sum2);
        }
    }
    sum = block_sum_all(sum, room);
    sum2 = block_sum_all(sum2, room + kMostWaves);
    const double from_pivot = sum * A.inv_d, variance = (sum2 - sum * from_pivot) * A.inv_d, mean = pivot + from_pivot;
    const float rstd = (float)(1.0 / sqrt((variance < 0.0 ? 0.0 : variance) + A.eps)), high = (float)mean, rest = (float)(mean - (double)high);
    auto out8 = [&](float *s, int64_t j) {
        float g[kVec], b[kVec];
        gain8(g, A.gain, j, d);
        gain8(b, A.shift, j, d, 0.f);
#pragma unroll
        for (int i = 0; i < kVec; ++i) s[i] = fmaf(((s[i] - high) - rest) * rstd, g[i], b[i]);
    };
    float scale = 1.f, per_scale = 1.f;
    if (kEight) {
        float top = 0.f;
        for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
            float s[kVec];
            sum8(s, j);
            out8(s, j);
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i < d - j) top = larger<kWhole>(top, fabsf(s[i]));
        }
        scale = scale_for<O>(block_top<kWhole>(top, top_room));
        per_scale = 1.f / scale;
    }
    if (threadIdx.x == 0) {
        if (A.mean) A.mean[row] = (float)mean;
        if (A.rstd) A.rstd[row] = rstd;
        if (kEight) A.scale[row] = scale;
    }
    O *y = static_cast<O *>(A.y) + row * A.ldy;
    T *t = static_cast<T *>(A.total) + (A.total ? row * A.ldt : 0);
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        float s[kVec];
        sum8(s, j);
        if (A.total) store8_of<T, PAST>(t + j, s, d - j);
        out8(s, j);
        if (kEight) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[i] *= per_scale;
        }
        store8_of<O, PAST>(y + j, s, d - j);
    }
}

// ------------------------------------------------------------------ gradient
struct LayerGradArgs {
    const void *total, *dy, *dtotal;
    const float *gain, *mean, *rstd;
    void *dx;
    float *gain_shares, *shift_shares;   // [workgroups][d] each, or NULL
    int64_t m, d, lds, lddy, lddt, lddx;
    float inv_d;
};

// Teams (wavefronts or workgroups) keep their columns' shares of dgain and dshift in registers, and take two rows at a time where a thread holds one
// chunk of a row: one barrier and one wait for memory serve both.
template <typename T, int CH, bool WAVE, bool PAST>
__global__ __launch_bounds__(WAVE ? kWaveRows * kWave : 1024) void k_layer_norm_grad(LayerGradArgs A)
{
    constexpr int kRows = CH == 1 ? 2 : 1;
    __shared__ float room[2][2 * kRows][kMostWaves];
    const int team = WAVE ? kWave : (int)blockDim.x, me = WAVE ? (int)threadIdx.x % kWave : (int)threadIdx.x;
    const int64_t teams = WAVE ? (int64_t)gridDim.x * kWaveRows : gridDim.x;
    const int64_t first = WAVE ? (int64_t)blockIdx.x * kWaveRows + threadIdx.x / kWave : blockIdx.x;
    const int64_t d = A.d;
    float g[CH][kVec], dg[CH][kVec], db[CH][kVec];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t j = (int64_t)(me + c * team) * kVec;
#pragma unroll
        for (int i = 0; i < kVec; ++i) g[c][i] = dg[c][i] = db[c][i] = 0.f;
        if (j < d) gain8(g[c], A.gain, j, d);
    }
    int turn = 0;
    for (int64_t row0 = first; row0 < A.m; row0 += kRows * teams, turn ^= 1) {
        Raw8<T> s[kRows][CH], dy[kRows][CH], dt[kRows][CH];
        float mean[kRows], rstd[kRows], along[kRows], level[kRows];
#pragma unroll
        for (int q = 0; q < kRows; ++q) {
            const int64_t row = row0 + q * teams;
            const bool there = row < A.m;
            const Elements<T> sv{static_cast<const T *>(A.total) + row * A.lds, d}, dyv{static_cast<const T *>(A.dy) + row * A.lddy, d};
            const Elements<T> dtv{static_cast<const T *>(A.dtotal) + (A.dtotal ? row * A.lddt : 0), d};
            mean[q] = there ? A.mean[row] : 0.f;
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
            along[q] = level[q] = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    // behind the row's end dy is 0
                    const float u = static_cast<float>(dy[q][c].v[i]), a = u * g[c][i], h = (static_cast<float>(s[q][c].v[i]) - mean[q]) * rstd[q];
                    along[q] = fmaf(a, h, along[q]);
                    level[q] += a;
                    dg[c][i] = fmaf(u, h, dg[c][i]);
                    db[c][i] += u;
                }
            along[q] = wave_sumf(along[q]);
            level[q] = wave_sumf(level[q]);
        }
        if (!WAVE) {
            // two rooms in turn: who writes the next rows' sums has passed the barrier behind which the last ones of this room were read
            const int waves = blockDim.x / kWave;
            if (threadIdx.x % kWave == 0) {
#pragma unroll
                for (int q = 0; q < kRows; ++q) {
                    room[turn][q][threadIdx.x / kWave] = along[q];
                    room[turn][kRows + q][threadIdx.x / kWave] = level[q];
                }
            }
            __syncthreads();
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                along[q] = level[q] = 0.f;
                for (int w = 0; w < waves; ++w) {
                    along[q] += room[turn][q][w];
                    level[q] += room[turn][kRows + q][w];
                }
            }
        }
#pragma unroll
        for (int q = 0; q < kRows; ++q) {
            const int64_t row = row0 + q * teams;
            if (row >= A.m) break;
            const float a_mean = level[q] * A.inv_d, back = along[q] * A.inv_d;
            T *dx = static_cast<T *>(A.dx) + row * A.lddx;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t j = (int64_t)(me + c * team) * kVec;
                if (j < d) {
                    float v[kVec];
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        const float h = (static_cast<float>(s[q][c].v[i]) - mean[q]) * rstd[q];
                        v[i] = rstd[q] * (fmaf(static_cast<float>(dy[q][c].v[i]), g[c][i], -a_mean) - h * back);
                        if (A.dtotal) v[i] += static_cast<float>(dt[q][c].v[i]);
                    }
                    store8_of<T, PAST>(dx + j, v, d - j);
                }
            }
        }
    }
    auto shares = [&](float *to, float (&mine)[CH][kVec]) {
        if (!to) return;
        if (WAVE) {   // the wavefronts of a workgroup join their shares, a chunk of columns at a time
            __shared__ float join[kWaveRows][kWave * kVec];
            const int wave = threadIdx.x / kWave;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kVec; ++i) join[wave][me * kVec + i] = mine[c][i];
                __syncthreads();
                for (int k = threadIdx.x; k < kWave * kVec; k += kWaveRows * kWave) {
                    const int64_t j = (int64_t)c * kWave * kVec + k;
                    if (j >= d) break;
                    float sum = 0.f;
#pragma unroll
                    for (int w = 0; w < kWaveRows; ++w) sum += join[w][k];
                    to[(int64_t)blockIdx.x * d + j] = sum;
                }
            }
        } else {
            float *p = to + first * d;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int64_t j = (int64_t)(me + c * team) * kVec;
                if (j < d) store8_of<float>(p + j, mine[c], d - j);
            }
        }
    };
    shares(A.gain_shares, dg);
    shares(A.shift_shares, db);
}

// Rows that registers do not hold: read twice.  dx may be dy or dtotal.
template <typename T, bool PAST>
__global__ __launch_bounds__(1024) void k_layer_norm_grad_wide(LayerGradArgs A)
{
    __shared__ float room[2 * kMostWaves];
    const int64_t row = block_number(), d = A.d, step = (int64_t)blockDim.x * kVec;
    if (row >= A.m) return;
    const Elements<T> sv{static_cast<const T *>(A.total) + row * A.lds, d}, dyv{static_cast<const T *>(A.dy) + row * A.lddy, d};
    const Elements<T> dtv{static_cast<const T *>(A.dtotal) + (A.dtotal ? row * A.lddt : 0), d};
    const float mean = A.mean[row], rstd = A.rstd[row];
    float along = 0.f, level = 0.f;
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        const Raw8<T> s = sv.at(j), dy = dyv.at(j);
        float g[kVec];
        gain8(g, A.gain, j, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float a = static_cast<float>(dy.v[i]) * g[i];
            along = fmaf(a, (static_cast<float>(s.v[i]) - mean) * rstd, along);
            level += a;
        }
    }
    block_sum_two(along, level, room);
    const float a_mean = level * A.inv_d, back = along * A.inv_d;
    T *dx = static_cast<T *>(A.dx) + row * A.lddx;
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        const Raw8<T> s = sv.at(j), dy = dyv.at(j);
        float g[kVec], v[kVec];
        gain8(g, A.gain, j, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = rstd * (fmaf(static_cast<float>(dy.v[i]), g[i], -a_mean) - (static_cast<float>(s.v[i]) - mean) * rstd * back);
        if (A.dtotal) {
            const Raw8<T> dt = dtv.at(j);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += static_cast<float>(dt.v[i]);
        }
        store8_of<T, PAST>(dx + j, v, d - j);
    }
}

// shares of dgain and dshift of rows that registers do not hold: a thread a column, gridDim.y shares
template <typename T>
__global__ __launch_bounds__(kBlock) void k_layer_shares(LayerGradArgs A)
{
    const int64_t j = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (j >= A.d) return;
    float sum = 0.f, level = 0.f;
    for (int64_t row = blockIdx.y; row < A.m; row += gridDim.y) {
        const float u = static_cast<float>(static_cast<const T *>(A.dy)[row * A.lddy + j]);
        sum = fmaf(u, (static_cast<float>(static_cast<const T *>(A.total)[row * A.lds + j]) - A.mean[row]) * A.rstd[row], sum);
        level += u;
    }
    if (A.gain_shares) A.gain_shares[blockIdx.y * A.d + j] = sum;
    if (A.shift_shares) A.shift_shares[blockIdx.y * A.d + j] = level;
}

template <typename T, typename O, bool PAST>
int layer_launch(const LayerArgs &A, hipStream_t st)
{
    const int64_t d = A.d;
    if (d <= kNarrow) {
        const dim3 grid = block_grid(ceil_div(A.m, kWaveRows));
        if (d <= 512) k_layer_norm<T, O, 1, true, PAST><<<grid, kWaveRows * kWave, 0, st>>>(A);
        else k_layer_norm<T, O, 2, true, PAST><<<grid, kWaveRows * kWave, 0, st>>>(A);
    } else if (d <= 8192) {
        k_layer_norm<T, O, 2, false, PAST><<<block_grid(A.m), row_threads(d, 2), 0, st>>>(A);
    } else if (d <= kWide) {
        k_layer_norm<T, O, 4, false, PAST><<<block_grid(A.m), row_threads(d, 4), 0, st>>>(A);
    } else {
        k_layer_norm_wide<T, O, PAST><<<block_grid(A.m), 1024, 0, st>>>(A);
    }
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

template <typename T>
int layer_typed(const LayerArgs &A, int out_type, hipStream_t st)
{
    const bool past = goes_past(A.m, A.d, (A.total ? sizeof(T) : 0) + type_bytes(out_type));
    if (out_type == TRON_TYPE_E4M3) return past ? layer_launch<T, e4m3, true>(A, st) : layer_launch<T, e4m3, false>(A, st);
    if (out_type == TRON_TYPE_I8) return past ? layer_launch<T, whole8, true>(A, st) : layer_launch<T, whole8, false>(A, st);
    return past ? layer_launch<T, T, true>(A, st) : layer_launch<T, T, false>(A, st);
}

// Columns up to which a wavefront of the gradient holds its rows, and above which rows are read twice
constexpr int64_t kGradNarrow = 1024;
constexpr int64_t kGradWide = 16384;

// workgroups of the gradient, each with a share of dgain and of dshift
int64_t layer_shares(int64_t m, int64_t d)
{
    if (d <= kGradNarrow) return std::min<int64_t>(ceil_div(m, kWaveRows), 1024);
    return std::min<int64_t>(m, d <= 2048 ? 1024 : d <= kGradWide ? 512 : 64);
}

template <typename T, bool PAST>
int layer_grad_typed(const LayerGradArgs &A, float *dgain, float *dshift, const float *work, hipStream_t st)
{
    const int64_t d = A.d;
    const unsigned shares = (unsigned)layer_shares(A.m, d);
    if (d <= kGradNarrow) {
        if (d <= 512) k_layer_norm_grad<T, 1, true, PAST><<<shares, kWaveRows * kWave, 0, st>>>(A);
        else k_layer_norm_grad<T, 2, true, PAST><<<shares, kWaveRows * kWave, 0, st>>>(A);
    } else if (d <= 8192) {
        k_layer_norm_grad<T, 1, false, PAST><<<shares, row_threads(d, 1), 0, st>>>(A);
    } else if (d <= kGradWide) {
        k_layer_norm_grad<T, 2, false, PAST><<<shares, row_threads(d, 2), 0, st>>>(A);
    } else {
        // before dx is written, which may be dy
        if (dgain || dshift) k_layer_shares<T><<<dim3((unsigned)ceil_div(d, kBlock), shares), kBlock, 0, st>>>(A);
        k_layer_norm_grad_wide<T, PAST><<<block_grid(A.m), 1024, 0, st>>>(A);
    }
    TRON_HIP(hipGetLastError());
    return dgain || dshift ? column_sums(work, shares, d, dgain, st, dshift) : TRON_OK;
}

template <typename T>
int layer_grad_typed(const LayerGradArgs &A, float *dgain, float *dshift, const float *work, hipStream_t st)
{
    return goes_past(A.m, A.d, sizeof(T)) ? layer_grad_typed<T, true>(A, dgain, dshift, work, st) : layer_grad_typed<T, false>(A, dgain, dshift, work, st);
}

}  // namespace
}  // namespace tron

using namespace tron;

extern "C" {

int tron_layer_norm(int64_t m, int64_t d, int type, const void *x, int64_t ldx, const void *residual, int64_t ldr, const float *gain, const float *shift,
                    double eps, void *total, int64_t ldt, int out_type, void *y, int64_t ldy, float *scale, float *mean, float *rstd, void *hip_stream)
{
    const bool eight = out_type == TRON_TYPE_E4M3 || out_type == TRON_TYPE_I8;
    if (m < 0 || d < 1 || m > INT32_MAX || !type_is_float(type) || (out_type != type && !eight) || !(eps >= 0.0) || !(eps < HUGE_VAL)) {
        set_error("tron_layer_norm: bad argument (need 0 <= m < 2^31, d >= 1, type f32, bf16 or f16, out_type that type, e4m3 or i8, finite eps >= 0)");
        return TRON_EINVAL;
    }
    if (m > 0 && (!x || !y || (eight && !scale) || !rows_ok(m, d, ldx, false) || (residual && !rows_ok(m, d, ldr, false)) ||
                  (total && !rows_ok(m, d, ldt, true)) || !rows_ok(m, d, ldy, true) || !extent_ok(m, ldx, d) || !extent_ok(m, residual ? ldr : 0, d) ||
                  !extent_ok(m, total ? ldt : 0, d) || !extent_ok(m, ldy, d))) {
        set_error("tron_layer_norm: bad argument (x, y and, for 8 bits, scale are needed; rows that are written may not overlap)");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    if (m == 0) return TRON_OK;
    const LayerArgs A{x, residual, gain, shift, total, y, scale, mean, rstd, m, d, ldx, ldr, ldt, ldy, eps, 1.0 / (double)d};
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    return type == TRON_TYPE_F32 ? layer_typed<float>(A, out_type, st)
           : type == TRON_TYPE_BF16 ? layer_typed<__bf16>(A, out_type, st) : layer_typed<_Float16>(A, out_type, st);
}

int64_t tron_layer_norm_grad_work(int64_t m, int64_t d)
{
    if (m < 1 || d < 1 || m > INT32_MAX || !extent_ok(2 * layer_shares(m, d), d, d)) return 0;
    return 2 * layer_shares(m, d) * d * (int64_t)sizeof(float);
}

int tron_layer_norm_grad(int64_t m, int64_t d, int type, const void *total, int64_t lds, const float *mean, const float *rstd, const float *gain, const void *dy,
                         int64_t lddy, const void *dtotal, int64_t lddt, void *dx, int64_t lddx, float *dgain, float *dshift, void *work, int64_t work_bytes,
                         void *hip_stream)
{
    if (m < 0 || d < 1 || m > INT32_MAX || !type_is_float(type)) {
        set_error("tron_layer_norm_grad: bad argument (need 0 <= m < 2^31, d >= 1, type f32, bf16 or f16)");
        return TRON_EINVAL;
    }
    if (m > 0 && (!total || !mean || !rstd || !dy || !dx || !rows_ok(m, d, lds, false) || !rows_ok(m, d, lddy, false) || (dtotal && !rows_ok(m, d, lddt, false)) ||
                  !rows_ok(m, d, lddx, true) || !extent_ok(m, lds, d) || !extent_ok(m, lddy, d) || !extent_ok(m, dtotal ? lddt : 0, d) || !extent_ok(m, lddx, d))) {
        set_error("tron_layer_norm_grad: bad argument (total, mean, rstd, dy and dx are needed; the rows of dx may not overlap)");
        return TRON_EINVAL;
    }
    if ((dgain || dshift) && !work_ok(work, work_bytes, tron_layer_norm_grad_work(m, d))) {
        set_error("tron_layer_norm_grad: dgain and dshift need a work space of tron_layer_norm_grad_work(m, d) bytes at a multiple of 16");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    if (m == 0) return dgain || dshift ? column_sums(nullptr, 0, d, dgain, st, dshift) : TRON_OK;
    float *gain_shares = static_cast<float *>(work), *shift_shares = gain_shares + (dshift ? layer_shares(m, d) * d : 0);
    const LayerGradArgs A{total, dy, dtotal, gain, mean, rstd, dx, dgain ? gain_shares : nullptr, dshift ? shift_shares : nullptr, m, d, lds, lddy, lddt, lddx,
                          (float)(1.0 / (double)d)};
    return type == TRON_TYPE_F32 ? layer_grad_typed<float>(A, dgain, dshift, gain_shares, st)
           : type == TRON_TYPE_BF16 ? layer_grad_typed<__bf16>(A, dgain, dshift, gain_shares, st) : layer_grad_typed<_Float16>(A, dgain, dshift, gain_shares, st);
}

}  // extern "C"
