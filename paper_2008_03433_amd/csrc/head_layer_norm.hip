// Layer norm of the sum of a row and its residual, with an output in the input's type or in 8 bits, and its gradient.
//
//   s = x + r,  rstd = (mean (s - mean s)^2 + eps)^-1/2,  h = (s - mean s) rstd,  y = h gain + shift     (8 bits: y / scale, scale = max |y| / 448 or 127)
//   dx = rstd (a - mean a - h mean(a h)) + dtotal,  a = dy gain;     dgain_j = sum_i dy_ij h_ij,  dshift_j = sum_i dy_ij
//
// Both are bound by memory: every matrix is read or written once, and a row stays in the registers of a wavefront (narrow rows: no barriers) or
// of a workgroup.  The mean is taken first and the squares are those of differences to it, so that rows that lie far from 0 keep the
// digits of their variance: with m the mean rounded to 32 bits and c = s - m,  mean s = m + mean c  and  variance = mean c^2 - (mean c)^2.  mean c is what
// the rounding of m and the order of its sum left; it is subtracted from c once more.  Where it is most of c, sums are of 64 bits and of differences to the row's first element.
//
// Measured: 16384 x 8192 bf16 with a residual and its sum 190 us (1.07 GB, 5.6 TB/s: outputs past the caches), to e4m3 203 us, to whole numbers 194 us; one row of 4096 to e4m3
// 4.6 us of the device's time, 9.2 us a call; gradient of 16384 x 4096 bf16 with all its inputs 116 us, of which 5 us the columns' sums (537 MB, 4.8 TB/s beside them), of
// 30011 x 1023 f16 52 us, of which 7 us these sums (184 MB).  Rows at odd places cost nothing by themselves (30011 x 1024 f16 in rows of 1025: 3% more).
#include "head_rows.h"

namespace tron {
namespace {

// Columns up to which sixteen lanes and a wavefront hold a row, and above which rows are read twice
constexpr int64_t kSlim = 128;
constexpr int64_t kNarrow = 1024;
constexpr int64_t kWide = 32768;

// Sums and maxima over a team of 16 or 64 lanes, in a fixed order; every lane has the result
template <int TEAM, typename F>
__device__ __forceinline__ float team_join(float v, F f)
{
    if (TEAM == kWave) return wave_joinf(v, f);
    v = f(v, dpp_movef<0xB1>(v));
    v = f(v, dpp_movef<0x4E>(v));
    v = f(v, dpp_movef<0x141>(v));
    return f(v, dpp_movef<0x140>(v));
}
template <int TEAM>
__device__ __forceinline__ float team_sum(float v)
{
    return team_join<TEAM>(v, [](float a, float b) { return a + b; });
}
template <int TEAM>
__device__ __forceinline__ double team_sum(double v)
{
    return TEAM == kWave ? wave_sum(v) : sum16(v);
}
constexpr int kTeamBlock = kWaveRows * kWave;   // threads of a workgroup of teams

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

// A thread's chunk of eight columns of a row of d.  The last one ends with the row: it begins in the chunk before, and its first `skip` elements are
// that one's.  Both compute and store them, with the same bits; sums leave them out.  (A last chunk that is shorter takes loads and stores of its
// own, by which the whole wavefront waits twice: 30011 x 1023 f16 31.8 us, x 1024 22.2 us.)  Rows of fewer than eight columns are one short chunk.
struct Chunk {
    int at, skip, end;
    bool there;
    __device__ __forceinline__ Chunk(int number, int d)
    {
        const int j = number * kVec;
        there = j < d;
        at = j + kVec <= d || d < kVec ? j : d - kVec;
        skip = there ? j - at : kVec;
        end = d < kVec ? d : kVec;
    }
    __device__ __forceinline__ bool counts(int i) const { return i >= skip && i < end; }
    // behind a row of fewer than eight columns: 0, or (AGAIN) its first element once more
    template <bool AGAIN = false, typename T>
    __device__ __forceinline__ Eight<T> of(const T *row) const
    {
        Eight<T> e;
        if (end == kVec) e.set(load8(row + at));
        else e.set(load_first(row + at, end, AGAIN ? row[0] : static_cast<T>(0.f)));
        return e;
    }
    __device__ __forceinline__ void factors(float *f, const float *p, float none) const
    {
        if (!p) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) f[i] = none;
            return;
        }
        const Eight<float> e = of(p);
#pragma unroll
        for (int i = 0; i < kVec; ++i) f[i] = e.at(i);
    }
    template <typename O, bool PAST>
    __device__ __forceinline__ void put(O *row, const float *v) const
    {
        store8_of<O, PAST>(row + at, v, end);
    }
};

// f(value, whether it counts) for a thread's values of a row; all of them count where a row is whole chunks
template <int CH, typename V, typename F>
__device__ __forceinline__ void for_each(const V (&s)[CH][kVec], int me, int team, int d, F f)
{
    if (d % kVec == 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < kVec; ++i) f(s[c][i]);   // 0 where there is no chunk
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const Chunk k(me + c * team, d);
#pragma unroll
            for (int i = 0; i < kVec; ++i) f(k.counts(i) ? s[c][i] : 0.f);
        }
    }
}

// f(value) for those that count
template <int CH, typename F>
__device__ __forceinline__ void for_each_there(const float (&s)[CH][kVec], int me, int team, int d, F f)
{
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const Chunk k(me + c * team, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (k.counts(i)) f(s[c][i]);
    }
}

// CH chunks of eight elements a thread; TEAM lanes a row (16: heads of a few dozen columns, 47454 x 69 bf16 by wavefronts 31 us for its gradient), 0: a
// workgroup
template <typename T, typename O, int CH, int TEAM, bool PAST>
__global__ __launch_bounds__(TEAM ? kTeamBlock : 1024) void k_layer_norm(LayerArgs A)
{
    constexpr bool kEight = sizeof(O) == 1, kWhole = __is_same(O, whole8);
    __shared__ float room[5 * kMostWaves];
    __shared__ double wide_room[3 * kMostWaves];
    __shared__ float first_room;
    constexpr int kTeam = TEAM ? TEAM : kWave;
    const int team = TEAM ? TEAM : (int)blockDim.x, me = TEAM ? (int)threadIdx.x % kTeam : (int)threadIdx.x;
    const int64_t row = TEAM ? block_number() * (kTeamBlock / kTeam) + threadIdx.x / kTeam : block_number();
    if (row >= A.m) return;
    const int d = (int)A.d;
    const T *x = static_cast<const T *>(A.x) + row * A.ldx, *r = static_cast<const T *>(A.residual) + (A.residual ? row * A.ldr : 0);
    float s[CH][kVec];
    float sum = 0.f;
    {
        Eight<T> raw[CH], more[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const Chunk k(me + c * team, d);
            if (!k.there) continue;
            raw[c] = k.of(x);
            if (A.residual) more[c] = k.of(r);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const Chunk k(me + c * team, d);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                s[c][i] = k.there ? raw[c].at(i) : 0.f;
                if (A.residual && k.there) s[c][i] += more[c].at(i);
            }
        }
    }
    for_each<CH>(s, me, team, d, [&](float v) { sum += v; });
    Moments M;
    sum = TEAM ? team_sum<kTeam>(sum) : block_sum_all(sum, room);
    M.mean = sum * (float)A.inv_d;
    if (!(fabsf(sum) <= kMostSquares)) {   // more than 32 bits hold, or no number
        double wide = 0.0;
        for_each<CH>(s, me, team, d, [&](float v) { wide += (double)v; });
        M.mean = (float)((TEAM ? team_sum<kTeam>(wide) : block_sum_all(wide, wide_room)) * A.inv_d);
    }
    // behind the sum's barrier, as `total` may be x or r, of which a last chunk reads what another wavefront's thread writes
    if (A.total) {
        T *t = static_cast<T *>(A.total) + row * A.ldt;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const Chunk k(me + c * team, d);
            if (k.there) k.put<T, PAST>(t, s[c]);
        }
    }
    float left = 0.f, sum2 = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const bool there = (me + c * team) * kVec < d;
#pragma unroll
        for (int i = 0; i < kVec; ++i) s[c][i] = there ? s[c][i] - M.mean : 0.f;
    }
    for_each<CH>(s, me, team, d, [&](float v) {
        left += v;
        sum2 = fmaf(v, v, sum2);
    });
    if (TEAM) {
        left = team_sum<kTeam>(left);
        sum2 = team_sum<kTeam>(sum2);
    } else {
        block_sum_two(left, sum2, room + kMostWaves);
    }
    // The squares' sum less what the mean's rounding has of it.  Where it has more than half (rows whose numbers differ in their last places, or not at all: 55 times 1e9
    // kept 2^-24 of it, a variance of 2e-4), and where 32 bits have lost the range, the sums are of 64 bits, of differences to one of the row's own: a row of one
    // number has the variance 0.
    M.rest = left * (float)A.inv_d;
    const float kept = sum2 - left * M.rest;
    if (sum2 >= kLeastSquares && sum2 <= kMostSquares && kept >= 0.5f * sum2) {
        M.rstd = 1.f / sqrtf(kept * (float)A.inv_d + (float)A.eps);
    } else {
        float first = s[0][0];
        if (TEAM) {
            first = __shfl(first, 0, kTeam);
        } else {
            if (me == 0) first_room = first;
            __syncthreads();
            first = first_room;
        }
        double l = 0.0, l2 = 0.0;
        for_each_there<CH>(s, me, team, d, [&](float v) {
            const double u = (double)v - (double)first;
            l += u;
            l2 = fma(u, u, l2);
        });
        l = TEAM ? team_sum<kTeam>(l) : block_sum_all(l, wide_room + kMostWaves);
        l2 = TEAM ? team_sum<kTeam>(l2) : block_sum_all(l2, wide_room + 2 * kMostWaves);
        M.rest = (float)((double)first + l * A.inv_d);
        const double variance = (l2 - l * (l * A.inv_d)) * A.inv_d;
        M.rstd = (float)(1.0 / sqrt((variance < 0.0 ? 0.0 : variance) + A.eps));   // NaN stays NaN
    }
    // y from here on
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const Chunk k(me + c * team, d);
        if (!k.there) continue;
        float g[kVec], b[kVec];
        k.factors(g, A.gain, 1.f);
        k.factors(b, A.shift, 0.f);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            s[c][i] = fmaf((s[c][i] - M.rest) * M.rstd, g[i], b[i]);
            if (kEight && i < k.end) top = larger<kWhole>(top, fabsf(s[c][i]));
        }
    }
    float scale = 1.f, per_scale = 1.f;
    if (kEight) {
        top = TEAM ? team_join<kTeam>(top, [](float a, float b) { return larger<kWhole>(a, b); }) : block_top<kWhole>(top, room + 3 * kMostWaves);
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
        const Chunk k(me + c * team, d);
        if (!k.there) continue;
        if (kEight) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[c][i] *= per_scale;
        }
        k.put<O, PAST>(y, s[c]);
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

// What a thread holds of a row.  Where dy does not count it is 0, and h, by which it is multiplied, has to be finite: a row of one large number times its rstd
// passes 32 bits, so that 0 in the place of s gives (0 - mean) rstd = -inf.  A chunk that is not there has rstd 0; what lies behind a row of fewer than eight columns,
// as what a last chunk skips, is an element of the row.
template <typename T, int CH>
struct HeldRow {
    Eight<T> s[CH], dy[CH], dt[CH];
    float mean, rstd;
    __device__ __forceinline__ void load(const LayerGradArgs &A, int64_t row, int me, int team)
    {
        const T *sp = static_cast<const T *>(A.total) + row * A.lds, *dyp = static_cast<const T *>(A.dy) + row * A.lddy;
        const T *dtp = static_cast<const T *>(A.dtotal) + (A.dtotal ? row * A.lddt : 0);
        mean = A.mean[row];
        rstd = A.rstd[row];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const Chunk k(me + c * team, (int)A.d);
            s[c] = dy[c] = Eight<T>{};
            if (!k.there) continue;
            s[c] = k.of<true>(sp);
            dy[c] = k.of(dyp);
            if (A.dtotal) dt[c] = k.of(dtp);
        }
    }
};

// Teams (wavefronts or workgroups) keep their columns' shares of dgain and dshift in registers.  Two rows at a time, or the next row under way while one is
// summed, take registers that other teams' loads need more (40011 x 512 f16 43.5 and 32.1 us instead of 32.6, 16384 x 4096 102 and 98 us instead of 97).
template <typename T, int CH, int TEAM, bool PAST>
__global__ __launch_bounds__(TEAM ? kTeamBlock : 1024) void k_layer_norm_grad(LayerGradArgs A)
{
    constexpr int kTeam = TEAM ? TEAM : kWave, kTeams = kTeamBlock / kTeam;
    constexpr int kWords = sizeof(Eight<T>) / 4;
    __shared__ float room[2][2 * kMostWaves];
    const int team = TEAM ? TEAM : (int)blockDim.x, me = TEAM ? (int)threadIdx.x % kTeam : (int)threadIdx.x;
    const int64_t teams = TEAM ? (int64_t)gridDim.x * kTeams : gridDim.x;
    const int64_t first = TEAM ? (int64_t)blockIdx.x * kTeams + threadIdx.x / kTeam : blockIdx.x;
    const int d = (int)A.d;
    float g[CH][kVec], dg[CH][kVec], db[CH][kVec];
    uint32_t counted[CH][kWords];   // ones where a chunk's elements count: sums take dy with zeros elsewhere
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const Chunk k(me + c * team, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i) g[c][i] = dg[c][i] = db[c][i] = 0.f;
        if (k.there) k.factors(g[c], A.gain, 1.f);
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            if (sizeof(T) == 4) counted[c][w] = k.counts(w) ? ~0u : 0;
            else counted[c][w] = (k.counts(2 * w) ? 0xffffu : 0) | (k.counts(2 * w + 1) ? 0xffff0000u : 0);
        }
    }
    int turn = 0;
    for (int64_t row = first; row < A.m; row += teams, turn ^= 1) {
        HeldRow<T, CH> now;
        now.load(A, row, me, team);
        float along = 0.f, level = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const float rstd = Chunk(me + c * team, d).there ? now.rstd : 0.f;
            Eight<T> own;
#pragma unroll
            for (int w = 0; w < kWords; ++w) own.w[w] = now.dy[c].w[w] & counted[c][w];
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float u = own.at(i), h = (now.s[c].at(i) - now.mean) * rstd, uh = u * h;
                along = fmaf(uh, g[c][i], along);
                level = fmaf(u, g[c][i], level);
                dg[c][i] += uh;
                db[c][i] += u;
            }
        }
        // two rooms in turn: who writes the next row's sums has passed the barrier behind which the last ones of this room were read
        if (TEAM) {
            along = team_sum<kTeam>(along);
            level = team_sum<kTeam>(level);
        } else {
            block_sum_two(along, level, room[turn]);
        }
        const float a_mean = level * A.inv_d, back = along * A.inv_d;
        T *dx = static_cast<T *>(A.dx) + row * A.lddx;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const Chunk k(me + c * team, d);
            if (!k.there) continue;
            float v[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float h = (now.s[c].at(i) - now.mean) * now.rstd;
                v[i] = now.rstd * fmaf(-h, back, fmaf(now.dy[c].at(i), g[c][i], -a_mean));
                if (A.dtotal) v[i] += now.dt[c].at(i);
            }
            k.put<T, PAST>(dx, v);
        }
    }
    auto shares = [&](float *to, float (&mine)[CH][kVec]) {
        if (!to) return;
        if (TEAM) {   // the teams of a workgroup join their shares, a chunk of columns at a time
            __shared__ float join[kTeams][kTeam * kVec];
            const int mine_of = threadIdx.x / kTeam;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                __syncthreads();
                const Chunk k0(me + c * team, d);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {   // what a chunk skips is the chunk's before, and stays there
                    const int column = k0.at + i - c * kTeam * kVec;
                    if (k0.counts(i)) join[mine_of][column] = mine[c][i];
                }
                __syncthreads();
                for (int k = threadIdx.x; k < kTeam * kVec; k += kTeamBlock) {
                    const int j = c * kTeam * kVec + k;
                    if (j >= d) break;
                    float sum = 0.f;
#pragma unroll
                    for (int w = 0; w < kTeams; ++w) sum += join[w][k];
                    to[(int64_t)blockIdx.x * d + j] = sum;
                }
            }
        } else {
            float *p = to + first * d;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const Chunk k(me + c * team, d);
                if (!k.there) continue;
                if (k.skip == 0) {
                    k.put<float, false>(p, mine[c]);
                } else {
#pragma unroll
                    for (int i = 0; i < kVec; ++i)
                        if (k.counts(i)) p[k.at + i] = mine[c][i];
                }
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
    const T behind = sv.p[0];   // of the row, so that h is finite where dy is 0
    float along = 0.f, level = 0.f;
    for (int64_t j = (int64_t)threadIdx.x * kVec; j < d; j += step) {
        const Raw8<T> s = load_row8(sv.p, j, d, behind), dy = dyv.at(j);
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
        const dim3 grid = block_grid(ceil_div(A.m, kTeamBlock / (d <= kSlim ? 16 : kWave)));
        if (d <= kSlim) k_layer_norm<T, O, 1, 16, PAST><<<grid, kTeamBlock, 0, st>>>(A);
        else if (d <= 512) k_layer_norm<T, O, 1, kWave, PAST><<<grid, kTeamBlock, 0, st>>>(A);
        else k_layer_norm<T, O, 2, kWave, PAST><<<grid, kTeamBlock, 0, st>>>(A);
    } else if (d <= 8192) {
        k_layer_norm<T, O, 2, 0, PAST><<<block_grid(A.m), row_threads(d, 2), 0, st>>>(A);
    } else if (d <= kWide) {
        k_layer_norm<T, O, 4, 0, PAST><<<block_grid(A.m), row_threads(d, 4), 0, st>>>(A);
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

// Columns up to which lanes of one wavefront hold a row in the gradient, and above which rows are read twice.  30011 x 1024 f16 67 us by wavefronts with two chunks a lane,
// 53 us by workgroups of 128 threads.
constexpr int64_t kGradNarrow = 512;
constexpr int64_t kGradWide = 16384;

// Workgroups of the gradient, each with a share of dgain and of dshift: as many as are resident.  16384 x 4096 f16 97 us with 512, 108 us with 1024; 30011 x 1024 53 us with
// 2048 of 128 threads, 69 us with 1024.
int64_t layer_shares(int64_t m, int64_t d)
{
    if (d <= kGradNarrow) return std::min<int64_t>(ceil_div(m, kTeamBlock / (d <= kSlim ? 16 : kWave)), 1024);
    return std::min<int64_t>(m, d <= 1024 ? 2048 : d <= 2048 ? 1024 : d <= kGradWide ? 512 : 64);
}

template <typename T, bool PAST>
int layer_grad_typed(const LayerGradArgs &A, float *dgain, float *dshift, const float *work, hipStream_t st)
{
    const int64_t d = A.d;
    const unsigned shares = (unsigned)layer_shares(A.m, d);
    if (d <= kGradNarrow) {
        if (d <= kSlim) k_layer_norm_grad<T, 1, 16, PAST><<<shares, kTeamBlock, 0, st>>>(A);
        else k_layer_norm_grad<T, 1, kWave, PAST><<<shares, kTeamBlock, 0, st>>>(A);
    } else if (d <= 8192) {
        k_layer_norm_grad<T, 1, 0, PAST><<<shares, row_threads(d, 1), 0, st>>>(A);
    } else if (d <= kGradWide) {
        k_layer_norm_grad<T, 2, 0, PAST><<<shares, row_threads(d, 2), 0, st>>>(A);
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
    if (m > 1 && total && ((total == x && ldt != ldx) || (total == residual && ldt != ldr))) {
        set_error("tron_layer_norm: total may be x or residual with the same leading dimension");
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
    if (m > 1 && ((dx == dy && lddx != lddy) || (dx == dtotal && lddx != lddt))) {
        set_error("tron_layer_norm_grad: dx may be dy or dtotal with the same leading dimension");
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
