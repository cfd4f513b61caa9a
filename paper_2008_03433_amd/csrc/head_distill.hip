// Loss of a softmax head against a teacher that gives its top entries only, its gradient and its Hessian-vector product.
//
// Row i, temperature T, weight w_i:  q = softmax(t / T) over the K listed entries,  p = softmax(z / T) over all V columns,
//   loss = w T^2 sum_j q_j (log q_j - log p_j),   dz = w T (p - q),   H u = w (p u - p (p.u)).
//
// All of it is bound by reading z and writing a matrix of its size.  A pass keeps a running maximum m and the sum of exp((z - m) / T)
// (in 32 bits; exponents are differences, so masks of the type's lowest value neither overflow nor lose the row).
//
// Loss and gradient: a workgroup a row, which it streams twice; the second read comes from the caches, because few long rows are under way.
// 4096 x 128000 bf16, 64 entries: 446 us, 4.70 TB/s of the 2.1 GB that have to move (with workgroups of 512 threads, stores that
// stay in the caches and exponents in 64 bits 704 us).  The gradient alone reads z once: 2011 x 50021 f16 94 us, 4.30 TB/s, rows at
// odd places.  Hessian product: z and u stay in registers between p.u and the product, exponentials are taken twice: 8192 x 32000
// bf16 273 us, 5.76 TB/s.  Where long rows are fewer than compute units they are split, and the second launch joins the parts'
// maxima and sums.
//
// The teacher's part of a row, K entries, is one wavefront's work: its exponents and its terms are held in 64 bits, because they and the
// logarithm of the sum cancel to the loss; its masses q in 32.
#include <type_traits>

#include "head_util.h"

namespace tron {
namespace {

constexpr int kThreads = 512;         // of a workgroup over a part of a row, at most
constexpr int kMostTop = 1024;        // listed entries a row
constexpr double kLog2e = 1.4426950408889634;

struct DistillArgs {
    const void *z, *u;
    int64_t ldz, ldu;
    const void *ids;
    int64_t ldi;
    const float *t;
    int64_t ldt;
    const float *weight;
    float *loss, *lse;
    const float *lse_in;
    void *out;           // dz or H u
    int64_t ldo;
    float *part_max, *part_sum;   // [m][splits]
    double *part_teacher;         // [m][2]: the teacher's terms and their base
    int64_t m, V;
    int64_t per;         // columns of a part
    int splits, top;
    bool lists;          // whether there are lists (of no entry, where top = 0)
    bool ids64;
    bool past;           // outputs go past the caches
    float temperature;
    double inv_t;
    float c;             // log2(e) / T
    float it_hi, it_lo;  // 1 / T in two parts
};

template <typename T>
constexpr bool kFull = sizeof(T) == 4;   // results in 32 bits: 1 / T in two parts

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }
// what exponents are differences to: no -inf minus -inf
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

// ------------------------------------------------------------------ the teacher's part of a row
// In LDS, as long as the launch says: three arrays of the listed entries
struct Teacher {
    float *q, *z;        // mass and logit
    int *id;             // -1: an entry that is missing
};
// A bit for every column's hash: where no bit is met twice, no column is listed twice, and nobody has to compare all pairs (loss
// and gradient of 2000 x 4000, 64 entries a row: 21.8 -> 16.2 us).  64 entries meet by chance in one row of sixteen.
constexpr int kSeenWords = 1024;
__device__ __forceinline__ unsigned column_hash(int id) { return (unsigned)id * 2654435761u >> 17; }
struct TeacherSums {
    double terms;        // sum_j q_j (log q_j - (z_j - base) / T)
    float base;          // the largest z_j that has mass: terms of masks of the type's lowest value keep their other parts
    int any;             // whether an entry has mass
    int twice;           // whether a column may be listed twice
};
extern __shared__ float g_lists[];
__device__ __forceinline__ Teacher teacher_of(const DistillArgs &A) { return {g_lists, g_lists + A.top, reinterpret_cast<int *>(g_lists + 2 * A.top)}; }
unsigned teacher_bytes(const DistillArgs &A) { return 3u * sizeof(float) * A.top; }

__device__ __forceinline__ int64_t listed_id(const DistillArgs &A, int64_t row, int j)
{
    return A.ids64 ? static_cast<const int64_t *>(A.ids)[row * A.ldi + j] : static_cast<const int32_t *>(A.ids)[row * A.ldi + j];
}

// By one wavefront.  Ids outside [0, V) are missing entries, whatever their t.
template <typename T>
__device__ __forceinline__ TeacherSums teacher_part(const DistillArgs &A, int64_t row, const Teacher &S, int lane, unsigned *seen = nullptr)
{
    if (seen) {
        typedef unsigned words __attribute__((ext_vector_type(4)));
        for (int i = lane; i < kSeenWords / 4; i += kWave) reinterpret_cast<words *>(seen)[i] = words{0, 0, 0, 0};
    }
    bool met = false;
    const float *t = A.t + row * A.ldt;
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    float top = -INFINITY, base = -INFINITY;
    bool bad = false;
    for (int j = lane; j < A.top; j += kWave) {
        const int64_t id = listed_id(A, row, j);
        const bool there = id >= 0 && id < A.V;
        const float v = there ? t[j] : -INFINITY, x = there ? static_cast<float>(z[id]) : 0.f;
        S.id[j] = there ? (int)id : -1;
        S.q[j] = v;
        S.z[j] = x;
        top = fmaxf(top, v);
        bad |= v != v;
        if (v > -INFINITY) base = fmaxf(base, x);
        if (seen && there) {
            const unsigned h = column_hash((int)id), bit = 1u << (h & 31);
            met |= (atomicOr(&seen[h >> 5], bit) & bit) != 0;
        }
    }
    top = wave_maxf(top);
    base = base_of(wave_maxf(base));
    TeacherSums R;
    R.any = __any(bad) || top > -INFINITY;
    // a wavefront's own LDS operations complete in order.  Exponents in 64 bits, of which the instruction takes 32 and a factor the rest: a
    // small q keeps its digits, for the difference to a p that is as small.  Masks of the type's lowest value have exponents that no float
    // holds: from -200 on, where the mass is 0, they are that.
    const double per_t = A.inv_t * kLog2e, from_top = base_of(top);
    auto mass = [&](double t_top) {
        const double exact = t_top * per_t, e = exact < -200.0 ? -200.0 : exact;   // NaN stays
        const float hi = (float)e;
        return exp2_(hi) * fmaf((float)(e - (double)hi), 0.69314718f, 1.f);
    };
    float sum = 0.f;
    for (int j = lane; j < A.top; j += kWave) {
        const float v = S.q[j];
        if (S.id[j] >= 0 && v != -INFINITY) sum += mass((double)v - from_top);
    }
    sum = wave_sumf(sum);
    const float per = 1.f / sum;
    const double log_sum = (double)logf(sum);
    double terms = 0.0;
    for (int j = lane; j < A.top; j += kWave) {
        const float v = S.q[j];
        const double t_top = (double)v - from_top;
        const float q = S.id[j] < 0 || v == -INFINITY ? 0.f : mass(t_top) * per;
        S.q[j] = q;
        if (q != 0.f) terms += (double)q * ((t_top - ((double)S.z[j] - (double)base)) * A.inv_t - log_sum);
    }
    R.terms = wave_sum(terms);
    R.base = base;
    R.twice = __any(met);
    return R;
}

// The listed columns in [from, to) of a row whose workgroup has stored w T p everywhere and passed a barrier: w T (p - q), where a
// column that is listed several times has the sum of its q.  scaled(z) = w T p.
template <typename T, typename P>
__device__ __forceinline__ void subtract_teacher(const DistillArgs &A, const Teacher &S, T *out, int64_t from, int64_t to, float wt, bool twice, P scaled)
{
    for (int j = threadIdx.x; j < A.top; j += blockDim.x) {
        const int id = S.id[j];
        if (id < from || id >= to) continue;
        if (!twice) {
            out[id] = static_cast<T>(scaled(S.z[j]) - wt * S.q[j]);
            continue;
        }
        float q = 0.f;
        bool first = true;
        for (int i = 0; i < A.top; ++i)
            if (S.id[i] == id) {
                first &= i >= j;
                q += S.q[i];
            }
        if (first) out[id] = static_cast<T>(scaled(S.z[j]) - wt * q);
    }
}

// ------------------------------------------------------------------ running maximum and sum
struct Running {
    float m = -INFINITY, s = 0.f;   // s = sum exp2((z - m) c); m = -inf: nothing yet, or nothing but -inf
};


template <typename T>
__device__ __forceinline__ void take8(Running &r, const Raw8<T> &raw, float c)
{
    float v[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = static_cast<float>(raw.v[i]);
    const float top = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    if (top > r.m) {
        r.s *= exp2_((r.m - top) * c);   // 0 * exp2(-inf) at first
        r.m = top;
    }
    const float m = base_of(r.m);
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < kVec; i += 2) {
        s0 += exp2_((v[i] - m) * c);
        s1 += exp2_((v[i + 1] - m) * c);
    }
    r.s += s0 + s1;
}

__device__ __forceinline__ Running join(const Running &a, const Running &b, float c)
{
    Running r;
    r.m = fmaxf(a.m, b.m);
    const float m = base_of(r.m);
    r.s = a.s * exp2_((a.m - m) * c) + b.s * exp2_((b.m - m) * c);
    return r;
}

// over the wavefront; every lane has the result
__device__ __forceinline__ Running join_wave(const Running &r, float c)
{
    const float top = wave_maxf(r.m);
    return {top, wave_sumf(r.s * exp2_((r.m - base_of(top)) * c))};
}

// over the workgroup; every thread has the result, behind a barrier.  room: 2 * kMostWaves floats
__device__ __forceinline__ Running join_block(Running r, float c, float *room)
{
    r = join_wave(r, c);
    const int waves = blockDim.x / kWave;
    if (threadIdx.x % kWave == 0) {
        room[threadIdx.x / kWave] = r.m;
        room[kMostWaves + threadIdx.x / kWave] = r.s;
    }
    __syncthreads();
    Running all{room[0], room[kMostWaves]};
    for (int w = 1; w < waves; ++w) all = join(all, Running{room[w], room[kMostWaves + w]}, c);
    return all;
}

// log sum_i exp(z_i / T), in 64 bits
__device__ __forceinline__ double log_sum(const Running &r, double inv_t)
{
    return r.m == -INFINITY && r.s == 0.f ? -INFINITY : (double)r.m * inv_t + log((double)r.s);
}

__device__ __forceinline__ float loss_of(const DistillArgs &A, double terms, double base, const Running &r, float w)
{
    // a row of nothing but -inf gives its teacher's entries no probability
    if (r.m == -INFINITY && r.s == 0.f) return INFINITY;
    return (float)((double)w * A.temperature * A.temperature * (terms + (((double)r.m - base) * A.inv_t + log((double)r.s))));
}

// ------------------------------------------------------------------ whole rows
template <typename T>
__device__ __forceinline__ Raw8<T> at8(const T *row, int64_t j, int64_t to, float fill = -INFINITY)
{
    return load_row8(row, j, to, static_cast<T>(fill));
}

// f p = f exp2((z - m) c) / s where the row's maximum m and sum s are known, with per = f / s
struct ByMax {
    float m, c, per;
    __device__ __forceinline__ float operator()(float z) const { return per * exp2_((z - m) * c); }
};
__device__ __forceinline__ ByMax by_max(const Running &r, float c, float f) { return {base_of(r.m), c, r.s == 0.f ? 0.f : f / r.s}; }

// f p = f exp((z - m) / T - less), the exponent as that difference times log2(e); m = 0 and less = lse where lse is known well enough.
// A row of nothing but -inf has p = 0.
template <typename T>
struct ByLse {
    float hi, lo, m, less, f;
    __device__ __forceinline__ float operator()(float z) const
    {
        const float d = z - m;
        float e = fmaf(d, hi, -less);
        if (kFull<T>) e += d == -INFINITY ? 0.f : d * lo;
        return f * exp2_(e * (float)kLog2e);
    }
};

// Columns that a workgroup takes at once, and how many of these a thread has under way
constexpr int kAhead = 2;
__device__ __forceinline__ int64_t block_step() { return (int64_t)blockDim.x * kVec; }

// f(j, eight elements of z from j on) over [from, to), kAhead loads at a time
template <typename T, typename F>
__device__ __forceinline__ void over_row(const T *z, int64_t from, int64_t to, F f)
{
    const int64_t step = block_step();
    int64_t j = from + (int64_t)threadIdx.x * kVec;
    for (; j + (kAhead - 1) * step + kVec <= to; j += kAhead * step) {
        Raw8<T> raw[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) raw[k] = load8(z + j + k * step);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) f(j + k * step, raw[k]);
    }
    for (; j < to; j += step) f(j, at8(z, j, to));
}

// the same over two rows; beyond `to` the second has zeros
template <typename T, typename F>
__device__ __forceinline__ void over_rows(const T *z, const T *u, int64_t from, int64_t to, F f)
{
    const int64_t step = block_step();
    int64_t j = from + (int64_t)threadIdx.x * kVec;
    for (; j + (kAhead - 1) * step + kVec <= to; j += kAhead * step) {
        Raw8<T> x[kAhead], y[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            x[k] = load8(z + j + k * step);
            y[k] = load8(u + j + k * step);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) f(j + k * step, x[k], y[k]);
    }
    for (; j < to; j += step) f(j, at8(z, j, to), at8(u, j, to, 0.f));
}

// A float holds lse to 2^-24 of its size, and p is off by that in proportion: rows of logits far from 0 (masks of the type's lowest value, whose
// lse is that value or infinite; small temperatures) would have any p.  From here on, where it is 2^-17 of p (16 bits: 2^-13), the row's
// maximum and sum are taken again from z.
template <typename T>
constexpr float kCoarseLse = kFull<T> ? 256.f : 4096.f;
template <typename T>
__device__ __forceinline__ bool coarse(float lse) { return fabsf(lse) >= kCoarseLse<T>; }

// By the whole workgroup.  room: 2 * kMostWaves floats, free again on return
template <typename T>
__device__ __forceinline__ ByLse<T> by_lse(const DistillArgs &A, const T *z, float lse, float f, float *room)
{
    if (!coarse<T>(lse)) return {A.it_hi, A.it_lo, 0.f, lse, f};
    Running r;
    over_row(z, 0, A.V, [&](int64_t, const Raw8<T> &x) { take8(r, x, A.c); });
    r = join_block(r, A.c, room);
    __syncthreads();
    const float m = base_of(r.m), less = r.s == 0.f ? 0.f : logf(r.s);
    return {A.it_hi, A.it_lo, read_lanef(m, 0), read_lanef(less, 0), f};
}

template <typename T, typename P>
__device__ __forceinline__ void write_scaled(const DistillArgs &A, const T *z, T *out, int64_t from, int64_t to, P scaled)
{
    auto all = [&](auto past) {
        over_row(z, from, to, [&](int64_t j, const Raw8<T> &x) {
            float v[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = scaled(static_cast<float>(x.v[i]));
            store8_of<T, past.value>(out + j, v, to - j);
        });
    };
    if (A.past) all(std::true_type{});
    else all(std::false_type{});
}

template <typename T>
__device__ __forceinline__ void write_zeros(const DistillArgs &A, T *out, int64_t from, int64_t to)
{
    const float zero[kVec] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t j = from + (int64_t)threadIdx.x * kVec; j < to; j += block_step()) store8_of<T>(out + j, zero, to - j);
}

// A workgroup a row, which is read again for the gradient: a running maximum needs no second look at what is behind it, so nothing is held.
template <typename T, bool GRAD>
__global__ __launch_bounds__(1024) void k_distill_row(DistillArgs A)
{
    __shared__ TeacherSums sums;
    __shared__ float room[2 * kMostWaves];
    __shared__ __align__(16) unsigned seen[GRAD ? kSeenWords : 4];
    const int64_t row = block_number();
    if (row >= A.m) return;
    const Teacher S = teacher_of(A);
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    if (threadIdx.x < kWave) {
        const TeacherSums R = teacher_part<T>(A, row, S, threadIdx.x, GRAD ? seen : nullptr);
        if (threadIdx.x == 0) sums = R;
    }
    Running r;
    over_row(z, 0, A.V, [&](int64_t, const Raw8<T> &x) { take8(r, x, A.c); });
    r = join_block(r, A.c, room);   // its barrier shows the teacher's part too
    const float w = sums.any ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    if (threadIdx.x == 0) {
        if (A.lse) A.lse[row] = (float)log_sum(r, A.inv_t);
        A.loss[row] = w == 0.f ? 0.f : loss_of(A, sums.terms, sums.base, r, w);
    }
    if (!GRAD) return;
    T *out = static_cast<T *>(A.out) + row * A.ldo;
    if (w == 0.f) {
        write_zeros(A, out, 0, A.V);
        return;
    }
    const float wt = w * A.temperature;
    const ByMax scaled = by_max(r, A.c, wt);
    write_scaled(A, z, out, 0, A.V, scaled);
    __syncthreads();
    subtract_teacher(A, S, out, 0, A.V, wt, sums.twice, scaled);
}

// ------------------------------------------------------------------ parts of rows
// blockIdx.x: the part; blockIdx.y, z: the row
__device__ __forceinline__ int64_t part_row() { return (int64_t)blockIdx.z * gridDim.y + blockIdx.y; }

template <typename T>
__global__ __launch_bounds__(1024) void k_distill_part(DistillArgs A)
{
    __shared__ float room[2 * kMostWaves];
    const int64_t row = part_row();
    if (row >= A.m) return;
    const int64_t from = blockIdx.x * A.per, to = from + A.per < A.V ? from + A.per : A.V;
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    if (blockIdx.x == 0 && threadIdx.x < kWave) {
        const TeacherSums R = teacher_part<T>(A, row, teacher_of(A), threadIdx.x);
        if (threadIdx.x == 0) {
            A.part_teacher[2 * row] = R.terms;
            A.part_teacher[2 * row + 1] = R.base;
        }
    }
    Running r;
    over_row(z, from, to, [&](int64_t, const Raw8<T> &x) { take8(r, x, A.c); });
    r = join_block(r, A.c, room);
    if (threadIdx.x == 0) {
        A.part_max[row * A.splits + blockIdx.x] = r.m;
        A.part_sum[row * A.splits + blockIdx.x] = r.s;
    }
}

__device__ __forceinline__ bool row_listed(const DistillArgs &A, int64_t row);

// Behind k_distill_part where there is no gradient: a wavefront a row joins its parts
template <typename T>
__global__ __launch_bounds__(kWave) void k_distill_join(DistillArgs A)
{
    const int64_t row = block_number();
    if (row >= A.m) return;
    const float w = row_listed(A, row) ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    Running r;
    for (int k = threadIdx.x; k < A.splits; k += kWave) r = join(r, Running{A.part_max[row * A.splits + k], A.part_sum[row * A.splits + k]}, A.c);
    r = join_wave(r, A.c);
    if (threadIdx.x == 0) {
        if (A.lse) A.lse[row] = (float)log_sum(r, A.inv_t);
        A.loss[row] = w == 0.f ? 0.f : loss_of(A, A.part_teacher[2 * row], A.part_teacher[2 * row + 1], r, w);
    }
}

// The gradient of a part of a row.  JOIN: behind k_distill_part, whose maxima and sums every wavefront joins, and the first part writes
// loss and lse; otherwise lse is given.
template <typename T, bool JOIN>
__global__ __launch_bounds__(1024) void k_distill_grad(DistillArgs A)
{
    __shared__ int any, twice;
    __shared__ float room[2 * kMostWaves];
    __shared__ __align__(16) unsigned seen[kSeenWords];
    const int64_t row = part_row();
    if (row >= A.m) return;
    const int64_t V = A.V;
    int64_t from = blockIdx.x * A.per, to = from + A.per < V ? from + A.per : V;
    const float lse = JOIN ? 0.f : A.lse_in[row];
    if (!JOIN && coarse<T>(lse)) {   // the whole row is read before any of `out`, which may be z, is written: by one workgroup
        if (blockIdx.x) return;
        from = 0;
        to = V;
    }
    const Teacher S = teacher_of(A);
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    // z of the listed columns too, before `out`, which may be z, is written
    if (threadIdx.x < kWave) {
        const TeacherSums R = teacher_part<T>(A, row, S, threadIdx.x, seen);
        if (threadIdx.x == 0) {
            any = R.any;
            twice = R.twice;
        }
    }
    Running r;
    if (JOIN) {
        const int lane = threadIdx.x % kWave;
        for (int k = lane; k < A.splits; k += kWave) r = join(r, Running{A.part_max[row * A.splits + k], A.part_sum[row * A.splits + k]}, A.c);
        r = join_wave(r, A.c);
    }
    __syncthreads();
    const float w = any ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    if (JOIN && blockIdx.x == 0 && threadIdx.x == 0) {
        if (A.lse) A.lse[row] = (float)log_sum(r, A.inv_t);
        A.loss[row] = w == 0.f ? 0.f : loss_of(A, A.part_teacher[2 * row], A.part_teacher[2 * row + 1], r, w);
    }
    T *out = static_cast<T *>(A.out) + row * A.ldo;
    if (w == 0.f) {
        write_zeros(A, out, from, to);
        return;
    }
    const float wt = w * A.temperature;
    const auto scaled = [&] {
        if constexpr (JOIN) return by_max(r, A.c, wt);
        else return by_lse<T>(A, z, lse, wt, room);
    }();
    write_scaled(A, z, out, from, to, scaled);
    __syncthreads();
    subtract_teacher(A, S, out, from, to, wt, twice, scaled);
}

// ------------------------------------------------------------------ Hessian-vector product
// whether an id of the row lies in [0, V) and its entry has mass, by the whole workgroup
__device__ __forceinline__ bool row_listed(const DistillArgs &A, int64_t row)
{
    if (!A.lists) return true;
    bool any = false;
    for (int j = threadIdx.x; j < A.top; j += blockDim.x) {
        const int64_t id = listed_id(A, row, j);
        any |= id >= 0 && id < A.V && !(A.t && A.t[row * A.ldt + j] == -INFINITY);
    }
    return __syncthreads_or(any);
}

// The same values, of which the compiler no longer knows what it has computed from them: exponentials are taken again where their
// registers would cost a workgroup.
template <typename T>
__device__ __forceinline__ void forget(Raw8<T> &r)
{
    typedef int words __attribute__((ext_vector_type(4)));
    words w[sizeof(r) / 16];
    __builtin_memcpy(w, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < (int)sizeof(r) / 16; ++i) asm volatile("" : "+v"(w[i]));
    __builtin_memcpy(&r, w, sizeof(r));
}

// CH > 0: z and u of a row stay in registers, CH chunks of eight a thread; 0, rows that 64 registers a thread do not hold: they are read
// again (8192 x 32000 bf16: 273 us held, 313 us read twice).
template <typename T, int CH, bool PAST>
__global__ __launch_bounds__(1024, CH * sizeof(T) <= 8 ? 8 : 4) void k_distill_hv_row(DistillArgs A)
{
    constexpr bool kAnew = CH * sizeof(T) >= 8;   // 32 registers hold z and u (two workgroups of 1024 a compute unit), or 64
    __shared__ float room[2 * kMostWaves];
    const int64_t row = block_number();
    if (row >= A.m) return;
    const int64_t V = A.V;
    const int64_t step = CH > 1 ? 1024 * kVec : block_step();   // CH > 1: launched with 1024 threads
    T *out = static_cast<T *>(A.out) + row * A.ldo;
    const float w = row_listed(A, row) ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    if (w == 0.f) {
        write_zeros(A, out, 0, V);
        return;
    }
    const T *z = static_cast<const T *>(A.z) + row * A.ldz, *u = static_cast<const T *>(A.u) + row * A.ldu;
    const ByLse<T> p = by_lse<T>(A, z, A.lse_in[row], 1.f, room);
    Raw8<T> zr[CH ? CH : 1], ur[CH ? CH : 1];
    float dot = 0.f;
    auto dot8 = [&](const Raw8<T> &x, const Raw8<T> &y) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            dot = fmaf(p(static_cast<float>(x.v[i])), static_cast<float>(y.v[i]), dot);
    };
    auto write8 = [&](const Raw8<T> &x, const Raw8<T> &y, int64_t j) {
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = w * (p(static_cast<float>(x.v[i])) * (static_cast<float>(y.v[i]) - dot));
        store8_of<T, PAST>(out + j, v, V - j);
    };
    if (CH) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t j = threadIdx.x * kVec + k * step;
            if (j < V) {
                zr[k] = at8(z, j, V);
                ur[k] = at8(u, j, V, 0.f);
            }
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t j = threadIdx.x * kVec + k * step;
            if (j < V) dot8(zr[k], ur[k]);
        }
    } else {
        over_rows(z, u, 0, V, [&](int64_t, const Raw8<T> &x, const Raw8<T> &y) { dot8(x, y); });
    }
    dot = block_sum_all(dot, room);
    if (CH) {
        if (kAnew) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                forget(zr[k]);
                forget(ur[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t j = threadIdx.x * kVec + k * step;
            if (j < V) write8(zr[k], ur[k], j);
        }
    } else {
        over_rows(z, u, 0, V, [&](int64_t j, const Raw8<T> &x, const Raw8<T> &y) { write8(x, y, j); });
    }
}

// FIRST: p.u of the parts; otherwise the product, behind that
template <typename T, bool FIRST>
__global__ __launch_bounds__(1024) void k_distill_hv_part(DistillArgs A)
{
    __shared__ float room[2 * kMostWaves];
    const int64_t row = part_row();
    if (row >= A.m) return;
    const int64_t V = A.V, from = blockIdx.x * A.per, to = from + A.per < V ? from + A.per : V;
    T *out = static_cast<T *>(A.out) + row * A.ldo;
    const float w = row_listed(A, row) ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    if (w == 0.f) {
        if (!FIRST) write_zeros(A, out, from, to);
        return;
    }
    const T *z = static_cast<const T *>(A.z) + row * A.ldz, *u = static_cast<const T *>(A.u) + row * A.ldu;
    const ByLse<T> p = by_lse<T>(A, z, A.lse_in[row], 1.f, room);
    float dot = 0.f;
    if (!FIRST)
        for (int k = 0; k < A.splits; ++k) dot += A.part_sum[row * A.splits + k];
    over_rows(z, u, from, to, [&](int64_t j, const Raw8<T> &x, const Raw8<T> &y) {
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float e = p(static_cast<float>(x.v[i])), f = static_cast<float>(y.v[i]);
            if (FIRST) dot = fmaf(e, f, dot);
            else v[i] = w * (e * (f - dot));
        }
        if (!FIRST) store8_of<T>(out + j, v, to - j);
    });
    if (FIRST) {
        dot = block_sum_all(dot, room);
        if (threadIdx.x == 0) A.part_sum[row * A.splits + blockIdx.x] = dot;
    }
}

// ------------------------------------------------------------------ launches
constexpr int64_t kLeastPart = 4096;   // columns of a part: one chunk of eight a thread
constexpr int64_t kWhole = 32768;      // columns of a row that one workgroup takes whatever the number of rows
constexpr int64_t kUnits = 256;        // compute units

// Parts of a row for the loss and the Hessian product, for which parts cost a second launch and a second read: only of rows that are long, and
// fewer than compute units.  One part and many: loss of 13 x 32000 f32 10 and 14 us, with the gradient of 400 x 32000 bf16 21 and
// 26 us, product of 200 x 100000 29 and 37 us; but with the gradient of 13 x 128000 21 and 15 us, of 64 x 64000 20 and 17 us.
int parts_of(int64_t m, int64_t V)
{
    return V <= kWhole ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(V, kLeastPart), kUnits / std::max<int64_t>(m, 1)));
}

// and for the gradient alone, one launch in either case: four workgroups a compute unit (300 x 32000 f16 12.3 us, with two 14.0 us)
int grad_parts(int64_t m, int64_t V)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(V, kLeastPart), 4 * kUnits / std::max<int64_t>(m, 1)));
}

void set_parts(DistillArgs &A, int parts)
{
    A.per = ceil_div(ceil_div(A.V, parts), kVec) * kVec;
    A.splits = (int)ceil_div(A.V, A.per);
}

dim3 part_grid(const DistillArgs &A)
{
    const int64_t y = std::min<int64_t>(A.m, 32768);
    return dim3((unsigned)A.splits, (unsigned)y, (unsigned)ceil_div(A.m, y));
}

int64_t work_of(int64_t m, int64_t V) { return parts_of(m, V) > 1 ? ceil_div(m * (16 + 2 * 4 * (int64_t)parts_of(m, V)), 16) * 16 : 0; }

// Threads of a workgroup over a row, with so many chunks of eight each, up to 1024.  Eight: the barriers of rows of some thousand columns wait
// for fewer, and long rows have few workgroups under way, whose rows are still in the caches when they are read again.
unsigned row_threads(int64_t V, int chunks) { return (unsigned)std::min<int64_t>(1024, ceil_div(ceil_div(V, kVec * chunks), kWave) * kWave); }

template <typename T>
int distill_typed(DistillArgs A, void *work, hipStream_t st)
{
    const int parts = parts_of(A.m, A.V);
    if (parts == 1) {
        const unsigned threads = row_threads(A.V, 8);
        if (A.out) k_distill_row<T, true><<<block_grid(A.m), threads, teacher_bytes(A), st>>>(A);
        else k_distill_row<T, false><<<block_grid(A.m), threads, teacher_bytes(A), st>>>(A);
        TRON_HIP(hipGetLastError());
        return TRON_OK;
    }
    set_parts(A, parts);
    A.part_teacher = static_cast<double *>(work);
    A.part_max = reinterpret_cast<float *>(A.part_teacher + 2 * A.m);
    A.part_sum = A.part_max + A.m * A.splits;
    k_distill_part<T><<<part_grid(A), kThreads, teacher_bytes(A), st>>>(A);
    if (A.out) k_distill_grad<T, true><<<part_grid(A), kThreads, teacher_bytes(A), st>>>(A);
    else k_distill_join<T><<<block_grid(A.m), kWave, 0, st>>>(A);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

template <typename T>
int distill_grad_typed(DistillArgs A, hipStream_t st)
{
    set_parts(A, grad_parts(A.m, A.V));
    k_distill_grad<T, false><<<part_grid(A), std::min<unsigned>(kThreads, row_threads(A.per, 8)), teacher_bytes(A), st>>>(A);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

template <typename T>
int distill_hv_typed(DistillArgs A, void *work, hipStream_t st)
{
    const int parts = parts_of(A.m, A.V);
    if (parts == 1) {
        const dim3 grid = block_grid(A.m);
        const unsigned threads = row_threads(A.V, 1);
        const int64_t chunks = ceil_div(A.V, (int64_t)threads * kVec);
        constexpr int kHeld = sizeof(T) == 2 ? 8 : 4;   // 64 registers
        auto launch = [&](auto past) {
            if (chunks == 1) k_distill_hv_row<T, 1, past.value><<<grid, threads, 0, st>>>(A);
            else if (chunks <= kHeld / 4) k_distill_hv_row<T, kHeld / 4, past.value><<<grid, threads, 0, st>>>(A);
            else if (chunks <= kHeld / 2) k_distill_hv_row<T, kHeld / 2, past.value><<<grid, threads, 0, st>>>(A);
            else if (chunks <= kHeld) k_distill_hv_row<T, kHeld, past.value><<<grid, threads, 0, st>>>(A);
            else k_distill_hv_row<T, 0, past.value><<<grid, threads, 0, st>>>(A);
        };
        if (A.past) launch(std::true_type{});
        else launch(std::false_type{});
    } else {
        set_parts(A, parts);
        A.part_sum = static_cast<float *>(work);
        k_distill_hv_part<T, true><<<part_grid(A), kThreads, 0, st>>>(A);
        k_distill_hv_part<T, false><<<part_grid(A), kThreads, 0, st>>>(A);
    }
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

// what the three calls check alike
int check(const char *name, int64_t m, int64_t V, int type, const void *z, int64_t ldz, int64_t K, const void *ids, int id_bytes, int64_t ldi, const void *t,
          int64_t ldt, bool lists, double temperature, const void *out, int64_t ldo, DistillArgs &A)
{
    if (m < 0 || m > INT32_MAX || V < 1 || V > INT32_MAX - 64 || !type_is_float(type) || K < (lists ? 0 : -1) || K > kMostTop || (id_bytes != 4 && id_bytes != 8)) {
        set_error("%s: bad argument (need 0 <= m < 2^31, 1 <= V < 2^31 - 64, type f32, bf16 or f16, 0 <= K <= %d, ids of 4 or 8 bytes)", name, kMostTop);
        return TRON_EINVAL;
    }
    if (!(temperature >= 0x1p-20) || !(temperature <= 0x1p20)) {
        set_error("%s: the temperature %g is not between 2^-20 and 2^20", name, temperature);
        return TRON_EINVAL;
    }
    if (m > 0 && (!z || !rows_ok(m, V, ldz, false) || !extent_ok(m, ldz, V) || (out && (!rows_ok(m, V, ldo, true) || !extent_ok(m, ldo, V))))) {
        set_error("%s: bad argument (z is needed; rows that are written may not overlap)", name);
        return TRON_EINVAL;
    }
    if (m > 0 && K > 0 && (!ids || !t || ldi < 0 || ldt < 0 || !extent_ok(m, ldi, K) || !extent_ok(m, ldt, K))) {
        set_error("%s: bad argument (the teacher's ids and values are needed)", name);
        return TRON_EINVAL;
    }
    A = DistillArgs{};
    A.z = z;
    A.ldz = ldz;
    A.ids = ids;
    A.ldi = ldi;
    A.t = static_cast<const float *>(t);
    A.ldt = ldt;
    A.out = const_cast<void *>(out);
    A.ldo = ldo;
    A.m = m;
    A.V = V;
    A.lists = K >= 0;
    A.top = K > 0 ? (int)K : 0;
    A.ids64 = id_bytes == 8;
    A.past = goes_past(m, V, type_bytes(type));
    A.temperature = (float)temperature;
    A.inv_t = 1.0 / temperature;
    A.c = (float)(kLog2e / temperature);
    A.it_hi = (float)A.inv_t;
    A.it_lo = (float)(A.inv_t - (double)A.it_hi);
    return TRON_OK;
}

}  // namespace
}  // namespace tron

using namespace tron;

extern "C" {

int64_t tron_distill_work(int64_t m, int64_t V) { return m < 1 || V < 1 || m > INT32_MAX || V > INT32_MAX - 64 ? 0 : work_of(m, V); }

int tron_distill(int64_t m, int64_t V, int type, const void *z, int64_t ldz, int64_t K, const void *ids, int id_bytes, int64_t ldi, const float *t, int64_t ldt,
                 double temperature, const float *weight, float *loss, float *lse, void *dz, int64_t lddz, void *work, int64_t work_bytes, void *hip_stream)
{
    DistillArgs A;
    TRON_TRY(check("tron_distill", m, V, type, z, ldz, K, ids, id_bytes, ldi, t, ldt, true, temperature, dz, lddz, A));
    if (m > 0 && !loss) {
        set_error("tron_distill: loss is needed");
        return TRON_EINVAL;
    }
    if (!work_ok(work, work_bytes, tron_distill_work(m, V))) {
        set_error("tron_distill: needs a work space of tron_distill_work(m, V) bytes at a multiple of 16");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    if (m == 0) return TRON_OK;
    A.weight = weight;
    A.loss = loss;
    A.lse = lse;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    return type == TRON_TYPE_F32 ? distill_typed<float>(A, work, st) : type == TRON_TYPE_BF16 ? distill_typed<__bf16>(A, work, st) : distill_typed<_Float16>(A, work, st);
}

int tron_distill_grad(int64_t m, int64_t V, int type, const void *z, int64_t ldz, const float *lse, int64_t K, const void *ids, int id_bytes, int64_t ldi,
                      const float *t, int64_t ldt, double temperature, const float *weight, void *dz, int64_t lddz, void *hip_stream)
{
    DistillArgs A;
    TRON_TRY(check("tron_distill_grad", m, V, type, z, ldz, K, ids, id_bytes, ldi, t, ldt, true, temperature, dz, lddz, A));
    if (m > 0 && (!lse || !dz)) {
        set_error("tron_distill_grad: lse and dz are needed");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    if (m == 0) return TRON_OK;
    A.weight = weight;
    A.lse_in = lse;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    return type == TRON_TYPE_F32 ? distill_grad_typed<float>(A, st) : type == TRON_TYPE_BF16 ? distill_grad_typed<__bf16>(A, st) : distill_grad_typed<_Float16>(A, st);
}

int tron_distill_hv(int64_t m, int64_t V, int type, const void *z, int64_t ldz, const float *lse, const void *u, int64_t ldu, int64_t K, const void *ids, int id_bytes,
                    int64_t ldi, const float *t, int64_t ldt, double temperature, const float *weight, void *hu, int64_t ldhu, void *work, int64_t work_bytes,
                    void *hip_stream)
{
    DistillArgs A;
    TRON_TRY(check("tron_distill_hv", m, V, type, z, ldz, K, ids, id_bytes, ldi, t, ldt, false, temperature, hu, ldhu, A));
    if (m > 0 && (!lse || !u || !hu || !rows_ok(m, V, ldu, false) || !extent_ok(m, ldu, V))) {
        set_error("tron_distill_hv: lse, u and hu are needed");
        return TRON_EINVAL;
    }
    if (!work_ok(work, work_bytes, tron_distill_work(m, V))) {
        set_error("tron_distill_hv: needs a work space of tron_distill_work(m, V) bytes at a multiple of 16");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    if (m == 0) return TRON_OK;
    A.u = u;
    A.ldu = ldu;
    A.weight = weight;
    A.lse_in = lse;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    return type == TRON_TYPE_F32 ? distill_hv_typed<float>(A, work, st) : type == TRON_TYPE_BF16 ? distill_hv_typed<__bf16>(A, work, st) : distill_hv_typed<_Float16>(A, work, st);
}

}  // extern "C"
