// Loss of a softmax head against a teacher that gives its top entries only, its gradient and its Hessian-vector product.
//
// Row i, temperature T, weight w_i:  q = softmax(t / T) over the K listed entries,  p = softmax(z / T) over all V columns,
//   loss = w T^2 sum_j q_j (log q_j - log p_j),   dz = w T (p - q),   H u = w (p u - p (p.u)).
//
// All of it is bound by reading z and writing a matrix of its size.  A pass keeps a running maximum m and the sum of exp((z - m) / T)
// (in 32 bits; exponents are differences, so masks of the type's lowest value neither overflow nor lose the row).  Rows that fit
// registers are read once; the others are read again for the gradient, while they are still in the caches.  Few rows are split
// over many workgroups, whose maxima and sums the second launch joins.  The teacher's part of a row, K entries, is one wavefront's
// work, in 64 bits: its terms and the logarithm of the sum cancel to the loss.
#include "head_util.h"

namespace tron {
namespace {

constexpr int kThreads = 512;         // of a workgroup over a row or a part of one
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
    float temperature;
    double inv_t;
    float c;             // log2(e) / T
    float it_hi, it_lo;  // 1 / T in two parts
};

template <typename T>
constexpr bool kFull = sizeof(T) == 4;   // results in 32 bits: 1 / T in two parts

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

// ------------------------------------------------------------------ the teacher's part of a row
struct Teacher {
    float q[kMostTop];
    int id[kMostTop];    // -1: an entry that is missing
    double terms;        // sum_j q_j (log q_j - (z_j - base) / T)
    float base;          // the largest z_j that has mass: terms of masks of the type's lowest value keep their other parts
    int any;             // whether an entry has mass
};

__device__ __forceinline__ int64_t listed_id(const DistillArgs &A, int64_t row, int j)
{
    return A.ids64 ? static_cast<const int64_t *>(A.ids)[row * A.ldi + j] : static_cast<const int32_t *>(A.ids)[row * A.ldi + j];
}

// By one wavefront.  Ids outside [0, V) are missing entries, whatever their t.
template <typename T, bool TERMS>
__device__ __forceinline__ void teacher_part(const DistillArgs &A, int64_t row, Teacher &S, int lane)
{
    const float *t = A.t + row * A.ldt;
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    float top = -INFINITY;
    bool bad = false;
    for (int j = lane; j < A.top; j += kWave) {
        const int64_t id = listed_id(A, row, j);
        const bool there = id >= 0 && id < A.V;
        const float v = there ? t[j] : -INFINITY;
        S.id[j] = there ? (int)id : -1;
        S.q[j] = v;
        top = fmaxf(top, v);
        bad |= v != v;
    }
    top = wave_maxf(top);
    bad = __any(bad);
    double sum = 0.0;
    // a wavefront's own LDS operations complete in order
    for (int j = lane; j < A.top; j += kWave)
        if (S.id[j] >= 0) sum += exp(((double)S.q[j] - (double)top) * A.inv_t);
    sum = wave_sum(sum);
    const bool any = bad || top > -INFINITY;
    const double log_sum = log(sum);
    float base = -INFINITY;
    if (TERMS) {
        for (int j = lane; j < A.top; j += kWave)
            if (S.id[j] >= 0 && S.q[j] > -INFINITY) base = fmaxf(base, static_cast<float>(z[S.id[j]]));
        base = wave_maxf(base);
        if (base == -INFINITY) base = 0.f;
    }
    double terms = 0.0;
    for (int j = lane; j < A.top; j += kWave) {
        const int id = S.id[j];
        if (id < 0) {
            S.q[j] = 0.f;
            continue;
        }
        const double log_q = any ? ((double)S.q[j] - (double)top) * A.inv_t - log_sum : 0.0, q = any ? exp(log_q) : 0.0;
        S.q[j] = (float)q;
        if (TERMS && q != 0.0) terms += q * (log_q - ((double)static_cast<float>(z[id]) - (double)base) * A.inv_t);
    }
    if (TERMS) terms = wave_sum(terms);
    if (lane == 0) {
        S.any = any;
        S.terms = terms;
        S.base = base;
    }
}

// The listed columns in [from, to) of a row whose workgroup has stored w T p everywhere and passed a barrier: w T (p - q), where a
// column that is listed several times has the sum of its q.  `keep` holds the listed z, scaled(z) = w T p.
template <typename T, typename P>
__device__ __forceinline__ void subtract_teacher(const DistillArgs &A, const Teacher &S, const float *keep, T *out, int64_t from, int64_t to, float wt, P scaled)
{
    for (int j = threadIdx.x; j < A.top; j += blockDim.x) {
        const int id = S.id[j];
        if (id < from || id >= to) continue;
        float q = 0.f;
        bool first = true;
        for (int i = 0; i < A.top; ++i)
            if (S.id[i] == id) {
                first &= i >= j;
                q += S.q[i];
            }
        if (first) out[id] = static_cast<T>(scaled(keep[j]) - wt * q);
    }
}

// ------------------------------------------------------------------ running maximum and sum
struct Running {
    float m = -INFINITY, s = 0.f;   // s = sum exp2((z - m) c); m = -inf: nothing yet, or nothing but -inf
};

__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

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

// over the workgroup; every thread has the result.  room: 2 * kMostWaves floats
__device__ __forceinline__ Running join_block(Running r, float c, float *room)
{
    const float m = base_of(wave_maxf(r.m));
    const float top = wave_maxf(r.m);
    r.s = wave_sumf(r.s * exp2_((r.m - m) * c));
    r.m = top;
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
__device__ __forceinline__ Raw8<T> at8(const T *row, int64_t j, int64_t to)
{
    return j + kVec <= to ? load8(row + j) : load_first(row + j, (int)(to - j), static_cast<T>(-INFINITY));
}

// f p = f exp2((z - m) c) / s where the row's maximum m and sum s are known, with per = f / s
struct ByMax {
    float m, c, per;
    __device__ __forceinline__ float operator()(float z) const { return per * exp2_((z - m) * c); }
};
__device__ __forceinline__ ByMax by_max(const Running &r, float c, float f) { return {base_of(r.m), c, r.s == 0.f ? 0.f : f / r.s}; }

// f p = f exp(z / T - lse), the exponent as that difference times log2(e): rows of the type's lowest value stay finite.  lse = -inf: a
// row of nothing but -inf, p = 0.
template <typename T>
struct ByLse {
    float hi, lo, less, f;
    __device__ __forceinline__ float operator()(float z) const
    {
        float e = fmaf(z, hi, -less);
        if (kFull<T>) e += z == -INFINITY ? 0.f : z * lo;
        return f * exp2_(e * (float)kLog2e);
    }
};
template <typename T>
__device__ __forceinline__ ByLse<T> by_lse(const DistillArgs &A, int64_t row, float f)
{
    const float lse = A.lse_in[row];
    return {A.it_hi, A.it_lo, lse == -INFINITY ? 0.f : lse, f};
}

template <typename T>
__device__ __forceinline__ void fill8(T *out, int64_t j, int64_t to)
{
    const float zero[kVec] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    store8_of<T>(out + j, zero, to - j);
}

// A workgroup a row.  CH > 0: the row stays in registers, CH chunks of eight a thread; 0: it is read again for the gradient.
template <typename T, int CH, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_distill_row(DistillArgs A)
{
    __shared__ Teacher S;
    __shared__ float keep[GRAD ? kMostTop : 1];
    __shared__ float room[2 * kMostWaves];
    const int64_t row = block_number();
    if (row >= A.m) return;
    const int64_t V = A.V;
    constexpr int64_t kStep = (int64_t)kThreads * kVec;
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    const float c = A.c;
    Raw8<T> raw[CH ? CH : 1];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int64_t j = threadIdx.x * kVec + k * kStep;
        if (j < V) raw[k] = at8(z, j, V);
    }
    if (threadIdx.x < kWave) teacher_part<T, true>(A, row, S, threadIdx.x);
    Running r;
    if (CH) {
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if ((int64_t)threadIdx.x * kVec + k * kStep < V) take8(r, raw[k], c);
    } else {
        int64_t j = (int64_t)threadIdx.x * kVec;
        for (; j + 3 * kStep + kVec <= V; j += 4 * kStep) {
            Raw8<T> four[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) four[k] = load8(z + j + k * kStep);
#pragma unroll
            for (int k = 0; k < 4; ++k) take8(r, four[k], c);
        }
        for (; j < V; j += kStep) take8(r, at8(z, j, V), c);
    }
    r = join_block(r, c, room);   // its barrier shows the teacher's part too
    const float w = S.any ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    if (threadIdx.x == 0) {
        if (A.lse) A.lse[row] = (float)log_sum(r, A.inv_t);
        A.loss[row] = w == 0.f ? 0.f : loss_of(A, S.terms, S.base, r, w);
    }
    if (!GRAD) return;
    T *out = static_cast<T *>(A.out) + row * A.ldo;
    if (w == 0.f) {
        for (int64_t j = (int64_t)threadIdx.x * kVec; j < V; j += kStep) fill8(out, j, V);
        return;
    }
    // z of the listed columns, before `out`, which may be z, is written
    for (int j = threadIdx.x; j < A.top; j += kThreads) keep[j] = S.id[j] >= 0 ? static_cast<float>(z[S.id[j]]) : 0.f;
    __syncthreads();
    const float wt = w * A.temperature;
    const ByMax scaled = by_max(r, c, wt);
    auto write8 = [&](int64_t j, const Raw8<T> &x) {
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = scaled(static_cast<float>(x.v[i]));
        store8_of<T>(out + j, v, V - j);
    };
    if (CH) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t j = threadIdx.x * kVec + k * kStep;
            if (j < V) write8(j, raw[k]);
        }
    } else {
        for (int64_t j = (int64_t)threadIdx.x * kVec; j < V; j += kStep) write8(j, at8(z, j, V));
    }
    __syncthreads();
    subtract_teacher(A, S, keep, out, 0, V, wt, scaled);
}

// ------------------------------------------------------------------ parts of rows
// blockIdx.x: the part; blockIdx.y, z: the row
__device__ __forceinline__ int64_t part_row() { return (int64_t)blockIdx.z * gridDim.y + blockIdx.y; }

template <typename T>
__global__ __launch_bounds__(kThreads) void k_distill_part(DistillArgs A)
{
    __shared__ Teacher S;
    __shared__ float room[2 * kMostWaves];
    const int64_t row = part_row();
    if (row >= A.m) return;
    const int64_t from = blockIdx.x * A.per, to = from + A.per < A.V ? from + A.per : A.V;
    constexpr int64_t kStep = (int64_t)kThreads * kVec;
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    if (blockIdx.x == 0 && threadIdx.x < kWave) {
        teacher_part<T, true>(A, row, S, threadIdx.x);
        if (threadIdx.x == 0) {
            A.part_teacher[2 * row] = S.terms;
            A.part_teacher[2 * row + 1] = S.base;
        }
    }
    Running r;
    for (int64_t j = from + (int64_t)threadIdx.x * kVec; j < to; j += kStep) take8(r, at8(z, j, to), A.c);
    r = join_block(r, A.c, room);
    if (threadIdx.x == 0) {
        A.part_max[row * A.splits + blockIdx.x] = r.m;
        A.part_sum[row * A.splits + blockIdx.x] = r.s;
    }
}

// The gradient of a part of a row.  JOIN: behind k_distill_part, whose maxima and sums it joins, and the first part writes loss and
// lse (without GRAD that is all there is); otherwise lse is given.
template <typename T, bool JOIN, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_distill_grad(DistillArgs A)
{
    __shared__ Teacher S;
    __shared__ float keep[GRAD ? kMostTop : 1];
    const int64_t row = part_row();
    if (row >= A.m) return;
    const int64_t V = A.V, from = blockIdx.x * A.per, to = from + A.per < V ? from + A.per : V;
    constexpr int64_t kStep = (int64_t)kThreads * kVec;
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    if (threadIdx.x < kWave) teacher_part<T, false>(A, row, S, threadIdx.x);
    __syncthreads();
    const float w = S.any ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    Running r;
    if (JOIN) {
        for (int k = 0; k < A.splits; ++k) r = join(r, Running{A.part_max[row * A.splits + k], A.part_sum[row * A.splits + k]}, A.c);
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            if (A.lse) A.lse[row] = (float)log_sum(r, A.inv_t);
            A.loss[row] = w == 0.f ? 0.f : loss_of(A, A.part_teacher[2 * row], A.part_teacher[2 * row + 1], r, w);
        }
    }
    if (!GRAD) return;
    T *out = static_cast<T *>(A.out) + row * A.ldo;
    if (w == 0.f) {
        for (int64_t j = from + (int64_t)threadIdx.x * kVec; j < to; j += kStep) fill8(out, j, to);
        return;
    }
    for (int j = threadIdx.x; j < A.top; j += kThreads) {
        const int id = S.id[j];
        keep[j] = id >= from && id < to ? static_cast<float>(z[id]) : 0.f;
    }
    __syncthreads();
    const float wt = w * A.temperature;
    const auto scaled = [&] {
        if constexpr (JOIN) return by_max(r, A.c, wt);
        else return by_lse<T>(A, row, wt);
    }();
    for (int64_t j = from + (int64_t)threadIdx.x * kVec; j < to; j += kStep) {
        const Raw8<T> x = at8(z, j, to);
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = scaled(static_cast<float>(x.v[i]));
        store8_of<T>(out + j, v, to - j);
    }
    __syncthreads();
    subtract_teacher(A, S, keep, out, from, to, wt, scaled);
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

template <typename T, int CH>
__global__ __launch_bounds__(kThreads) void k_distill_hv_row(DistillArgs A)
{
    __shared__ float room[kMostWaves];
    const int64_t row = block_number();
    if (row >= A.m) return;
    const int64_t V = A.V;
    constexpr int64_t kStep = (int64_t)kThreads * kVec;
    T *out = static_cast<T *>(A.out) + row * A.ldo;
    const float w = row_listed(A, row) ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    if (w == 0.f) {
        for (int64_t j = (int64_t)threadIdx.x * kVec; j < V; j += kStep) fill8(out, j, V);
        return;
    }
    const T *z = static_cast<const T *>(A.z) + row * A.ldz, *u = static_cast<const T *>(A.u) + row * A.ldu;
    const ByLse<T> p = by_lse<T>(A, row, 1.f);
    Raw8<T> zr[CH ? CH : 1], ur[CH ? CH : 1];
    float dot = 0.f;
    auto dot8 = [&](const Raw8<T> &x, const Raw8<T> &y, int64_t j) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (j + i < V) dot = fmaf(p(static_cast<float>(x.v[i])), static_cast<float>(y.v[i]), dot);
    };
    auto write8 = [&](const Raw8<T> &x, const Raw8<T> &y, int64_t j) {
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = w * (p(static_cast<float>(x.v[i])) * (static_cast<float>(y.v[i]) - dot));
        store8_of<T>(out + j, v, V - j);
    };
    if (CH) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t j = threadIdx.x * kVec + k * kStep;
            if (j < V) {
                zr[k] = at8(z, j, V);
                ur[k] = at8(u, j, V);
            }
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t j = threadIdx.x * kVec + k * kStep;
            if (j < V) dot8(zr[k], ur[k], j);
        }
    } else {
        for (int64_t j = (int64_t)threadIdx.x * kVec; j < V; j += kStep) dot8(at8(z, j, V), at8(u, j, V), j);
    }
    dot = block_sumf(dot, room);
    if (CH) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int64_t j = threadIdx.x * kVec + k * kStep;
            if (j < V) write8(zr[k], ur[k], j);
        }
    } else {
        for (int64_t j = (int64_t)threadIdx.x * kVec; j < V; j += kStep) write8(at8(z, j, V), at8(u, j, V), j);
    }
}

// FIRST: p.u of the parts; otherwise the product, behind that
template <typename T, bool FIRST>
__global__ __launch_bounds__(kThreads) void k_distill_hv_part(DistillArgs A)
{
    __shared__ float room[kMostWaves];
    const int64_t row = part_row();
    if (row >= A.m) return;
    const int64_t V = A.V, from = blockIdx.x * A.per, to = from + A.per < V ? from + A.per : V;
    constexpr int64_t kStep = (int64_t)kThreads * kVec;
    T *out = static_cast<T *>(A.out) + row * A.ldo;
    const float w = row_listed(A, row) ? (A.weight ? A.weight[row] : 1.f) : 0.f;
    if (w == 0.f) {
        if (!FIRST)
            for (int64_t j = from + (int64_t)threadIdx.x * kVec; j < to; j += kStep) fill8(out, j, to);
        return;
    }
    const T *z = static_cast<const T *>(A.z) + row * A.ldz, *u = static_cast<const T *>(A.u) + row * A.ldu;
    const ByLse<T> p = by_lse<T>(A, row, 1.f);
    float dot = 0.f;
    if (!FIRST)
        for (int k = 0; k < A.splits; ++k) dot += A.part_sum[row * A.splits + k];
    for (int64_t j = from + (int64_t)threadIdx.x * kVec; j < to; j += kStep) {
        const Raw8<T> x = at8(z, j, to), y = at8(u, j, to);
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float e = p(static_cast<float>(x.v[i])), f = static_cast<float>(y.v[i]);
            if (FIRST) dot = j + i < to ? fmaf(e, f, dot) : dot;
            else v[i] = w * (e * (f - dot));
        }
        if (!FIRST) store8_of<T>(out + j, v, to - j);
    }
    if (FIRST) {
        dot = block_sumf(dot, room);
        if (threadIdx.x == 0) A.part_sum[row * A.splits + blockIdx.x] = dot;
    }
}

// ------------------------------------------------------------------ launches
constexpr int64_t kLeastPart = 4096;   // columns of a part: one chunk of eight a thread
constexpr int64_t kWanted = 1024;      // workgroups that fill the device: four of kThreads a compute unit

int parts_of(int64_t m, int64_t V)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(V, kLeastPart), kWanted / std::max<int64_t>(m, 1)));
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

template <typename T, bool GRAD>
int distill_rows(const DistillArgs &A, hipStream_t st)
{
    const dim3 grid = block_grid(A.m);
    constexpr int64_t kStep = (int64_t)kThreads * kVec;
    if (A.V <= kStep) k_distill_row<T, 1, GRAD><<<grid, kThreads, 0, st>>>(A);
    else if (A.V <= 4 * kStep) k_distill_row<T, 4, GRAD><<<grid, kThreads, 0, st>>>(A);
    else if (A.V <= 8 * kStep && sizeof(T) == 2) k_distill_row<T, sizeof(T) == 2 ? 8 : 4, GRAD><<<grid, kThreads, 0, st>>>(A);
    else k_distill_row<T, 0, GRAD><<<grid, kThreads, 0, st>>>(A);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

template <typename T>
int distill_typed(DistillArgs A, void *work, hipStream_t st)
{
    const int parts = parts_of(A.m, A.V);
    if (parts == 1) return A.out ? distill_rows<T, true>(A, st) : distill_rows<T, false>(A, st);
    set_parts(A, parts);
    A.part_teacher = static_cast<double *>(work);
    A.part_max = reinterpret_cast<float *>(A.part_teacher + 2 * A.m);
    A.part_sum = A.part_max + A.m * A.splits;
    k_distill_part<T><<<part_grid(A), kThreads, 0, st>>>(A);
    if (A.out) {
        k_distill_grad<T, true, true><<<part_grid(A), kThreads, 0, st>>>(A);
    } else {
        dim3 grid = part_grid(A);
        grid.x = 1;
        k_distill_grad<T, true, false><<<grid, kWave, 0, st>>>(A);
    }
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

template <typename T>
int distill_grad_typed(DistillArgs A, hipStream_t st)
{
    set_parts(A, parts_of(A.m, A.V));
    k_distill_grad<T, false, true><<<part_grid(A), kThreads, 0, st>>>(A);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

template <typename T>
int distill_hv_typed(DistillArgs A, void *work, hipStream_t st)
{
    const int parts = parts_of(A.m, A.V);
    if (parts == 1) {
        const dim3 grid = block_grid(A.m);
        constexpr int64_t kStep = (int64_t)kThreads * kVec;
        if (A.V <= kStep) k_distill_hv_row<T, 1><<<grid, kThreads, 0, st>>>(A);
        else if (A.V <= 4 * kStep) k_distill_hv_row<T, 4><<<grid, kThreads, 0, st>>>(A);
        else if (A.V <= 8 * kStep && sizeof(T) == 2) k_distill_hv_row<T, sizeof(T) == 2 ? 8 : 4><<<grid, kThreads, 0, st>>>(A);
        else k_distill_hv_row<T, 0><<<grid, kThreads, 0, st>>>(A);
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
