// Matrix product with bias, activation and residual in its epilogue, and its gradients.
//
//   y = act(x w' (x_scale_i w_scale_j) + b) + r;    dpre = dy act'(pre),  dx = dpre w,  dw = dpre' x,  db = sum_i dpre_i
//
// Both operands of a product lie with the inner index k contiguous.  A step of the inner loop takes 128 bytes of every row: 64
// elements of 16 bits, or 128 of 8.  In LDS the sixteen-byte chunks of a row are exchanged among themselves by the row's number, so that
// sixteen rows of one column of chunks lie in different banks, and a chunk is what a lane of a matrix instruction takes: the
// order of k among chunks is the same for both operands and does not matter to the sum.
//
// Which kernel runs is a rule on the sizes (linear_plan): tiles of 256 x 256 or 128 x 128 of the result for many rows, a kernel that reads w
// once, straight into registers, for up to 32 rows.  The inner index is cut where tiles leave compute units idle, and the parts are
// added in a fixed order.
//
// Many rows are bound by the matrix units and what feeds them: 8192 x 32000 x 4096 bf16 1.70 ms, 1262 TFLOP/s; the units are busy 57% of the cycles of a
// clock that falls to 2.0 GHz under them.  Without the fetches the same loop runs at 1500 to 1600 TFLOP/s.  Few rows are bound by reading w: one
// row of 32000 x 4096 bf16 55 us, 4.8 TB/s.  In between the way to memory and the launch count: 777 x 1001 x 2049 f16 23 us.
// Whole numbers of 8 bits take the same bytes a step and twice the inner index: 8192 x 8192 x 4096 with silu 292 us, 1880 TOP/s; eight rows of
// 32000 x 4096 32.5 us, 4.0 TB/s; 515 x 1003 x 2051 20 us.
#include <type_traits>

#include "head_util.h"

namespace tron {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ operand types
template <typename T>
constexpr int kStepElems = 128 / (int)sizeof(T);   // elements of a row that a step takes
template <typename T>
constexpr int kChunkElems = 16 / (int)sizeof(T);

// What a lane has of a chunk, as operands of matrix instructions.  e4m3 is made bf16 on the way, which holds each of its values: the
// matrix instructions for 8 bits keep 13 bits below the largest product of a step (a product 2^14 times smaller than another adds
// nothing), those for 16 bits sum in 32.  Whole numbers have instructions of their own, which sum in whole numbers of 32 bits: exactly, for inner lengths
// up to kMostWhole.
template <typename T>
struct Fragment {
    static constexpr int kCount = 1;
    i32x4 v[1];
};
template <>
struct Fragment<e4m3> {
    static constexpr int kCount = 2;
    i32x4 v[2];
};

constexpr int64_t kMostWhole = (1 << 17) - 1;   // (-128)^2 times that is below 2^31

// Four sums of a lane.  Whole numbers stay such until the epilogue, and in the parts of a cut inner index, which hold their bits: whatever the tiles
// and parts are, the sum is the same.
template <typename T>
struct SumOf {
    typedef f32x4 four;
    typedef float one;
};
template <>
struct SumOf<whole8> {
    typedef i32x4 four;
    typedef int one;
};
template <typename T>
using Sums = typename SumOf<T>::four;

template <typename T>
__device__ __forceinline__ Fragment<T> fragment(i32x4 chunk)
{
    Fragment<T> f;
    if constexpr (__is_same(T, e4m3)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f.v[i / 2][i % 2 * 2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(chunk[i], 1.f, false));
            f.v[i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(chunk[i], 1.f, true));
        }
    } else {
        f.v[0] = chunk;
    }
    return f;
}

template <typename T>
__device__ __forceinline__ Sums<T> mma(const Fragment<T> &a, const Fragment<T> &b, Sums<T> c)
{
#pragma unroll
    for (int i = 0; i < Fragment<T>::kCount; ++i) {
        if constexpr (__is_same(T, whole8))
            c = __builtin_amdgcn_mfma_i32_16x16x64_i8(a.v[i], b.v[i], c, 0, 0, 0);
        else if constexpr (sizeof(T) == 2 && !__is_same(T, __bf16))
            c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.v[i]), __builtin_bit_cast(f16x8, b.v[i]), c, 0, 0, 0);
        else
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.v[i]), __builtin_bit_cast(bf16x8, b.v[i]), c, 0, 0, 0);
    }
    return c;
}

// ------------------------------------------------------------------ epilogue
struct Epilogue {
    const float *x_scale, *w_scale, *bias;
    const void *residual;
    void *y, *pre;
    int64_t m, n, ldr, ldy, ldpre;
    int act, out;
    float *part;   // [parts][m][n]: sums of a part of the inner index instead (whole numbers: their bits)
    bool past;     // y goes past the caches
    const float *factor;   // one number that every sum is multiplied by, or NULL
};

// exp(-v) from the two parts hi + lo = -v log2(e), |lo| at most a unit of the last place of hi: one part alone is off by 2^-24 of the exponent
__device__ __forceinline__ float exp_of_parts(float hi, float lo)
{
    const float e = __builtin_amdgcn_exp2f(hi);
    return fmaf(e, lo * 0.69314718f, e);
}

// Phi(a) = (1 + erf(a / sqrt 2)) / 2 = bell t P(t) for a <= 0, with t = 1 / (1 + p |a| / sqrt 2), bell = exp(-a^2 / 2), and 1 minus that
// of -a above.  P is a polynomial fitted to exp(a^2 / 2) Phi(a) / t by the least largest relative error, 1.9e-7 over |a| <= 20; in 32 bits Phi of
// either sign is off by 6e-7 of itself, so small values of gelu have their digits too.  Beyond 13 bell is 0.  8192 x 8192 x
// 4096 e4m3 operands with gelu: 438 us, 428 us by a shorter formula that is off by 0.6% of Phi(-7), a tenth more by erff.
__device__ __forceinline__ float normal_cdf(float a, float &bell)
{
    const float b = fminf(fabsf(a), 20.f), t = __builtin_amdgcn_rcpf(fmaf(0.44f * 0.70710678f, b, 1.f));
    const float square = b * b, hi = square * -0.72134752f;
    const float lo = fmaf(square, -0.72134752f, -hi) + fmaf(fmaf(b, b, -square), -0.72134752f, square * -9.629815e-9f);   // b^2 and log2(e) / 2 to 48 bits
    bell = exp_of_parts(hi, lo);
    float p = fmaf(t, 0.0357501879f, -0.139577508f);
    p = fmaf(t, p, 0.149435416f);
    p = fmaf(t, p, -0.0111487368f);
    p = fmaf(t, p, 0.108497597f);
    p = fmaf(t, p, 0.108467117f);
    p = fmaf(t, p, 0.124467745f);
    p = fmaf(t, p, 0.124108262f);
    const float beyond = t * p * bell;   // Phi(-|a|)
    return a < 0.f ? beyond : 1.f - beyond;
}

// h = 1 / (1 + exp(-a)) and 1 - h, both with their digits
__device__ __forceinline__ float logistic(float a, float &rest)
{
    const float b = fminf(fabsf(a), 120.f), hi = b * -1.44269502f;
    const float e = exp_of_parts(hi, fmaf(b, -1.44269502f, -hi) + b * -1.925963e-8f), r = __builtin_amdgcn_rcpf(1.f + e);
    rest = a < 0.f ? r : e * r;
    return a < 0.f ? e * r : r;
}

__device__ __forceinline__ float act_of(float a, int act)
{
    float other;
    switch (act) {
    case TRON_ACT_RELU: return a > 0.f || a != a ? a : 0.f;
    case TRON_ACT_GELU: return a * normal_cdf(a, other);
    case TRON_ACT_SILU: return a * logistic(a, other);
    default: return a;
    }
}

__device__ __forceinline__ float act_slope(float a, int act)
{
    float other;
    switch (act) {
    case TRON_ACT_RELU: return a > 0.f || a != a ? 1.f : 0.f;
    case TRON_ACT_GELU: {
        const float phi = normal_cdf(a, other);
        return phi + a * 0.39894228f * other;
    }
    case TRON_ACT_SILU: {
        const float h = logistic(a, other);
        return h * (1.f + a * other);
    }
    default: return 1.f;
    }
}

template <typename O>
__device__ __forceinline__ void load_as(float *v, const void *base, int64_t at, int64_t n)
{
    const O *p = static_cast<const O *>(base) + at;
    const Raw8<O> r = n >= kVec ? load8(p) : load_first(p, (int)n, static_cast<O>(0.f));
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = static_cast<float>(r.v[i]);
}

__device__ __forceinline__ void load_out(float *v, const void *base, int out, int64_t at, int64_t n)
{
    if (out == TRON_TYPE_F32) load_as<float>(v, base, at, n);
    else if (out == TRON_TYPE_BF16) load_as<__bf16>(v, base, at, n);
    else load_as<_Float16>(v, base, at, n);
}

template <bool PAST = false>
__device__ __forceinline__ void store_out(void *base, int out, int64_t at, const float *v, int64_t n)
{
    if (out == TRON_TYPE_F32) store8_of<float, PAST>(static_cast<float *>(base) + at, v, n);
    else if (out == TRON_TYPE_BF16) store8_of<__bf16, PAST>(static_cast<__bf16 *>(base) + at, v, n);
    else store8_of<_Float16, PAST>(static_cast<_Float16 *>(base) + at, v, n);
}

// A scale as fraction and exponent: the product of a row's and a column's may lie outside the range of 32 bits where the result does not.
struct Scale {
    float fraction;
    int exponent;
};
__device__ __forceinline__ Scale scale_of(float s) { return {__builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s)}; }
__device__ __forceinline__ float scaled(float v, const Scale &a, const Scale &b) { return ldexpf(v * (a.fraction * b.fraction), a.exponent + b.exponent); }

// what eight columns have
struct Columns {
    Scale scale[kVec];
    float bias[kVec], factor;
};
__device__ __forceinline__ Columns columns_of(const Epilogue &E, int64_t j)
{
    Columns c;
#pragma unroll
    for (int e = 0; e < kVec; ++e) c.bias[e] = 0.f;
    c.factor = E.factor ? *E.factor : 1.f;
    if (j < E.n && E.w_scale) {
        float s[kVec];
        load_as<float>(s, E.w_scale, j, E.n - j);
#pragma unroll
        for (int e = 0; e < kVec; ++e) c.scale[e] = scale_of(s[e]);
    }
    if (j < E.n && E.bias) load_as<float>(c.bias, E.bias, j, E.n - j);
    return c;
}

// N times eight neighbouring sums, of rows that lie `step` apart: what is read before what is written
template <bool PAST, int N>
__device__ __forceinline__ void finish8(const Epilogue &E, const Columns &C, float (&v)[N][kVec], int64_t i, int64_t step, int64_t j)
{
    const int64_t n = E.n - j;
    float f[N][kVec];
    Scale xs[N];
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const int64_t row = i + q * step;
        if (row >= E.m) break;
        if (E.residual) load_out(f[q], E.residual, E.out, row * E.ldr + j, n);
        if (E.x_scale) xs[q] = scale_of(E.x_scale[row]);
    }
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const int64_t row = i + q * step;
        if (row >= E.m) break;
        if (E.factor) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[q][e] *= C.factor;
        }
        if (E.x_scale) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[q][e] = scaled(v[q][e], xs[q], C.scale[e]);
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[q][e] += C.bias[e];
        if (E.pre) store_out(E.pre, E.out, row * E.ldpre + j, v[q], n);
        if (E.act != TRON_ACT_NONE) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[q][e] = act_of(v[q][e], E.act);
        }
        if (E.residual) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[q][e] += f[q][e];
        }
        store_out<PAST>(E.y, E.out, row * E.ldy + j, v[q], n);
    }
}

template <bool PAST, int N>
__device__ __forceinline__ void put8(const Epilogue &E, const Columns &C, float (&v)[N][kVec], int64_t i, int64_t step, int64_t j, int part)
{
    if (E.part) {
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (i + q * step < E.m) store8_of<float>(E.part + ((int64_t)part * E.m + i + q * step) * E.n + j, v[q], E.n - j);
    } else {
        finish8<PAST>(E, C, v, i, step, j);
    }
}

// Behind a product whose inner index was cut: eight sums a thread, four parts at a time, the lanes of a wavefront on one row after the other
// (9 parts of 3368 x 18: 18.6 us with a workgroup a row, 4.1 us so).  More parts than kJoinAlone are shared out over W wavefronts, whose sums
// meet in LDS in their order (64 parts of 16 x 4096: 13.8 us by one, 5 us by eight).
constexpr int kJoinAlone = 8, kJoinWaves = 8;

// WHOLE: the parts hold whole numbers.
template <bool WHOLE>
__device__ __forceinline__ float join(float a, float b)
{
    return WHOLE ? __int_as_float(__float_as_int(a) + __float_as_int(b)) : a + b;
}

template <int W, bool WHOLE>
__global__ __launch_bounds__(W == 1 ? kBlock : W * kWave) void k_linear_join(Epilogue E, int parts)
{
    const int wave = W == 1 ? 0 : threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t chunks = (E.n + kVec - 1) / kVec, unit = W == 1 ? block_number() * blockDim.x + threadIdx.x : block_number() * kWave + lane;
    const int64_t i = unit / chunks, j = (unit - i * chunks) * kVec, n = i < E.m ? E.n - j : 0, each = E.m * E.n;
    const float *p = E.part + i * E.n + j;
    float v[1][kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[0][e] = 0.f;
    if (n > 0) {
        int q = wave;
        for (; q + 3 * W < parts; q += 4 * W) {
            float f[4][kVec];
#pragma unroll
            for (int r = 0; r < 4; ++r) load_as<float>(f[r], p + (q + r * W) * each, 0, n);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < kVec; ++e) v[0][e] = join<WHOLE>(v[0][e], f[r][e]);
        }
        for (; q < parts; q += W) {
            float f[kVec];
            load_as<float>(f, p + q * each, 0, n);
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[0][e] = join<WHOLE>(v[0][e], f[e]);
        }
    }
    if constexpr (W > 1) {
        __shared__ float share[W - 1][kVec][kWave];
        if (wave)
#pragma unroll
            for (int e = 0; e < kVec; ++e) share[wave - 1][e][lane] = v[0][e];
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int u = 0; u < W - 1; ++u)
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[0][e] = join<WHOLE>(v[0][e], share[u][e][lane]);
    }
    if (WHOLE) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[0][e] = (float)__float_as_int(v[0][e]);
    }
    if (n > 0) finish8<false>(E, columns_of(E, j), v, i, 0, j);
}

template <bool WHOLE = false>
int join_parts(const Epilogue &E, int parts, hipStream_t st)
{
    const int64_t units = E.m * ceil_div(E.n, kVec);
    const bool alone = parts <= kJoinAlone;
    const unsigned across = alone ? (unsigned)std::min<int64_t>(kBlock, ceil_div(units, kWave) * kWave) : kWave;
    const int64_t blocks = ceil_div(units, across), x = std::min<int64_t>(blocks, 1 << 20);
    const dim3 grid((unsigned)x, (unsigned)ceil_div(blocks, x));
    if (alone) k_linear_join<1, WHOLE><<<grid, across, 0, st>>>(E, parts);
    else k_linear_join<kJoinWaves, WHOLE><<<grid, kJoinWaves * kWave, 0, st>>>(E, parts);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

// ------------------------------------------------------------------ tiles
struct Operand {
    const void *p;
    int64_t rows, ld;   // in elements
};

struct ProductArgs {
    Operand x, w;
    int64_t k;          // inner length
    int64_t k_part;     // of a part; a multiple of a step
    int64_t tiles_m, tiles_n;
    Epilogue E;
};

// a chunk's place in LDS: rows of 128 bytes
__device__ __forceinline__ int chunk_place(int row, int chunk) { return row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4); }

// Sixteen bytes of a row from element k on; elements from `end` on are zeros.
template <typename T>
__device__ __forceinline__ i32x4 load_chunk(const T *row, int64_t k, int64_t end)
{
    i32x4 v = {0, 0, 0, 0};
    if (k + kChunkElems<T> <= end) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < end) {
        T some[kChunkElems<T>];
#pragma unroll
        for (int i = 0; i < kChunkElems<T>; ++i) {
            if (k + i < end) some[i] = row[k + i];
            else __builtin_memset(&some[i], 0, sizeof(T));
        }
        __builtin_memcpy(&v, some, 16);
    }
    return v;
}

// Which tile a workgroup takes.  Workgroups go to the eight XCDs in turn; each XCD gets a contiguous range of tiles, walked in groups
// of eight tiles of m, so that what its L2 holds is used by the tiles that run there together.
__device__ __forceinline__ void tile_of(const ProductArgs &A, int64_t block, int64_t &tm, int64_t &tn)
{
    const int64_t count = A.tiles_m * A.tiles_n, xcd = block % 8, each = count / 8, more = count % 8;
    const int64_t t = xcd * each + (xcd < more ? xcd : more) + block / 8;
    constexpr int64_t kGroup = 8;
    const int64_t group = t / (kGroup * A.tiles_n), first = group * kGroup, high = A.tiles_m - first < kGroup ? A.tiles_m - first : kGroup;
    const int64_t in = t - group * kGroup * A.tiles_n;
    tm = first + in % high;
    tn = in / high;
}

// LDS of a tile: two steps' chunks, or 128 rows of results
template <int BM, int BN>
constexpr int kTileLds = 2 * (BM + BN) * 128 > 128 * (BN + 4) * 4 ? 2 * (BM + BN) * 128 : 128 * (BN + 4) * 4;

// What a lane has of half a step: four of the eight chunks of a row
template <int FM, int FN>
struct Half {
    i32x4 a[FM], b[FN];
};

template <int BM, int FM, int FN>
__device__ __forceinline__ void load_half(Half<FM, FN> &f, const char *lds, int h, int wm, int wn, int lane)
{
#pragma unroll
    for (int j = 0; j < FN; ++j) f.b[j] = *reinterpret_cast<const i32x4 *>(lds + chunk_place(BM + wn * FN * 16 + j * 16 + lane % 16, lane / 16 + 4 * h));
#pragma unroll
    for (int i = 0; i < FM; ++i) f.a[i] = *reinterpret_cast<const i32x4 *>(lds + chunk_place(wm * FM * 16 + i * 16 + lane % 16, lane / 16 + 4 * h));
}

template <typename T, int FM, int FN>
__device__ __forceinline__ void mma_half(const Half<FM, FN> &f, Sums<T> (&acc)[FM][FN])
{
    Fragment<T> b[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) b[j] = fragment<T>(f.b[j]);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const Fragment<T> a = fragment<T>(f.a[i]);
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mma<T>(b[j], a, acc[i][j]);
    }
}

// a step's products of a wavefront's part of the tile
template <typename T, int BM, int FM, int FN>
__device__ __forceinline__ void tile_step(const char *lds, int wm, int wn, int lane, Sums<T> (&acc)[FM][FN])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        Fragment<T> a[FM], b[FN];
#pragma unroll
        for (int i = 0; i < FM; ++i) a[i] = fragment<T>(*reinterpret_cast<const i32x4 *>(lds + chunk_place(wm * FM * 16 + i * 16 + lane % 16, lane / 16 + 4 * h)));
#pragma unroll
        for (int j = 0; j < FN; ++j)
            b[j] = fragment<T>(*reinterpret_cast<const i32x4 *>(lds + chunk_place(BM + wn * FN * 16 + j * 16 + lane % 16, lane / 16 + 4 * h)));
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mma<T>(b[j], a[i], acc[i][j]);
    }
}

// Sums on their way out: whole numbers as the nearest floats, or their bits where a part's sums go to memory.
__device__ __forceinline__ f32x4 as_floats(f32x4 v, const float *) { return v; }
__device__ __forceinline__ f32x4 as_floats(i32x4 v, const float *part) { return part ? __builtin_bit_cast(f32x4, v) : __builtin_convertvector(v, f32x4); }

// Lane l holds row l % 16 and columns l / 16 * 4 .. + 3 of a 16 x 16 piece.  Through LDS, 128 rows at a time, to stores of whole lines: a
// thread keeps its eight columns and takes rows that lie apart, several at once.
template <typename T, int BM, int BN, int WM, int WN, int FM, int FN>
__device__ __forceinline__ void tile_out(const Epilogue &E, char *lds, int wm, int wn, int lane, const Sums<T> (&acc)[FM][FN], int64_t m0, int64_t n0, int part)
{
    constexpr int kThreads = WM * WN * kWave, kRows = BM < 128 ? BM : 128, kPitch = BN + 4, kAcross = BN / kVec, kDown = kThreads / kAcross;
    static_assert(kThreads % kAcross == 0 && kRows % (4 * kDown) == 0, "whole rows at once");
    float *out = reinterpret_cast<float *>(lds);
    const int c = threadIdx.x % kAcross * kVec;
    const int64_t j = n0 + c;
    const Columns C = columns_of(E, j);
#pragma unroll
    for (int half = 0; half < BM / kRows; ++half) {
        if (half) __syncthreads();
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int r = wm * FM * 16 + i * 16 + lane % 16 - half * kRows;
            if (r >= 0 && r < kRows) {
#pragma unroll
                for (int k = 0; k < FN; ++k) *reinterpret_cast<f32x4 *>(out + r * kPitch + wn * FN * 16 + k * 16 + lane / 16 * 4) = as_floats(acc[i][k], E.part);
            }
        }
        __syncthreads();
        if (j >= E.n) continue;
        auto rows = [&](auto past) {
#pragma unroll 1
            for (int r = threadIdx.x / kAcross; r < kRows; r += 4 * kDown) {
                float v[4][kVec];
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int e = 0; e < kVec; e += 4) {
                        const f32x4 four = *reinterpret_cast<const f32x4 *>(out + (r + q * kDown) * kPitch + c + e);
                        v[q][e] = four[0], v[q][e + 1] = four[1], v[q][e + 2] = four[2], v[q][e + 3] = four[3];
                    }
                put8<past.value>(E, C, v, m0 + half * kRows + r, kDown, j, part);
            }
        };
        if (E.past) rows(std::true_type{});
        else rows(std::false_type{});
    }
}

// Every wavefront's loads into LDS have arrived and its reads of LDS are done, for all of the workgroup.
__device__ __forceinline__ void all_arrived()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A tile whose operands' rows lie at multiples of 16 bytes and are whole chunks: chunks go from memory to LDS without registers, a step
// ahead of the products.  A wavefront's load takes eight rows of 128 bytes; which chunk a lane fetches makes the exchange of places.
// Eight wavefronts of 128 x 64 each: four of 128 x 128 read less of LDS, but one a SIMD had nothing to run while it waits (4096^3: 1104 against
// 1174 TFLOP/s).  8192 x 32000 x 4096 bf16 through registers 2119 us, straight to
// LDS 1964 us, with half a step read ahead 1907 us, and with what the epilogue and priorities gave 1.70 ms.
template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN *kWave) void k_linear_direct(ProductArgs A)
{
    constexpr int kWaves = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int kX = BM / 8 / kWaves, kW = BN / 8 / kWaves, kStage = (BM + BN) * 128;
    static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0, "whole loads");
    extern __shared__ __align__(16) char lds[];
    const int64_t count = A.tiles_m * A.tiles_n;
    if (block_number() >= count) return;
    int64_t tm, tn;
    tile_of(A, block_number(), tm, tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    const int part = blockIdx.z;
    const int64_t k_from = part * A.k_part, k_to = k_from + A.k_part < A.k ? k_from + A.k_part : A.k;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, wm = wave / WN, wn = wave % WN;

    // offsets from the tile's first row; rows past the end repeat the last one, and their results are not stored
    constexpr unsigned kNowhere = 0x80000000u;   // past the buffer's end: zeros arrive
    unsigned at[kX + kW];
    static_assert(kWaves % 2 == 0 && BM % 16 == 0, "a wavefront's groups of eight rows are all even or all odd");
    const int chunk16 = ((lane % 8) ^ (wave % 2 * 4 + lane / 16)) << 4;
#pragma unroll
    for (int i = 0; i < kX + kW; ++i) {
        const int r = (i < kX ? wave + kWaves * i : wave + kWaves * (i - kX)) * 8 + lane / 8;
        const int64_t left = i < kX ? A.x.rows - m0 : A.w.rows - n0;
        at[i] = (unsigned)((r < left ? r : left - 1) * (i < kX ? A.x.ld : A.w.ld) * (int64_t)sizeof(T)) + chunk16;
    }
    const __amdgpu_buffer_rsrc_t xs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<T *>(static_cast<const T *>(A.x.p) + m0 * A.x.ld + k_from), 0, 0x7ffffff0, 0x00020000);
    const __amdgpu_buffer_rsrc_t ws = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<T *>(static_cast<const T *>(A.w.p) + n0 * A.w.ld + k_from), 0, 0x7ffffff0, 0x00020000);
    const int bytes = (int)((k_to - k_from) * (int64_t)sizeof(T)), steps = (bytes + 127) / 128;   // of a row
    auto fetch = [&](char *to, int from) {
        const int left = bytes - from;   // below 128: the rest of a row
#pragma unroll
        for (int i = 0; i < kX + kW; ++i) {
            const int group = i < kX ? wave + kWaves * i : BM / 8 + wave + kWaves * (i - kX);
            const unsigned offset = chunk16 < left ? at[i] : kNowhere;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(i < kX ? xs : ws, (__attribute__((address_space(3))) void *)(to + group * 1024), 16, offset, from, 0, 0);
        }
    };
    Sums<T> acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Sums<T>{0, 0, 0, 0};
    // Half a step is read from LDS while the other half's products run.  The wait for the next step lies in the middle: behind it
    // nobody reads this step's chunks any more, and the step after the next is fetched to their place.
    auto all = [&](char *__restrict__ even, char *__restrict__ odd) {
        Half<FM, FN> first, second;
        auto one = [&](char *now, char *next, int i) {
            load_half<BM>(second, now, 1, wm, wn, lane);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);   // who multiplies goes before who loads
            mma_half<T>(first, acc);
            __builtin_amdgcn_s_setprio(0);
            all_arrived();
            if (i + 2 < steps) fetch(now, (i + 2) * 128);
            if (i + 1 < steps) load_half<BM>(first, next, 0, wm, wn, lane);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            mma_half<T>(second, acc);
            __builtin_amdgcn_s_setprio(0);
        };
        fetch(even, 0);
        all_arrived();
        if (steps > 1) fetch(odd, 128);
        load_half<BM>(first, even, 0, wm, wn, lane);
        for (int i = 0;;) {
            one(even, odd, i);
            if (++i == steps) break;
            one(odd, even, i);
            if (++i == steps) break;
        }
    };
    // e4m3: its operands as bf16 leave no registers for a second half
    auto plain = [&](char *__restrict__ even, char *__restrict__ odd) {
        auto one = [&](char *now, char *next, int i) {
            all_arrived();
            if (i + 1 < steps) fetch(next, (i + 1) * 128);
            tile_step<T, BM, FM, FN>(now, wm, wn, lane, acc);
        };
        fetch(even, 0);
        for (int i = 0;;) {
            one(even, odd, i);
            if (++i == steps) break;
            one(odd, even, i);
            if (++i == steps) break;
        }
    };
    if constexpr (__is_same(T, e4m3)) plain(lds, lds + kStage);
    else all(lds, lds + kStage);
    __syncthreads();
    tile_out<T, BM, BN, WM, WN>(A.E, lds, wm, wn, lane, acc, m0, n0, part);
}

// A tile whose operands lie anywhere: chunks go through registers, which know where a row ends (8192 x 32000 x 4096 bf16: 2.1 ms).
template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN *kWave) void k_linear_tile(ProductArgs A)
{
    constexpr int kThreads = WM * WN * kWave, FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int kChunks = (BM + BN) * 8 / kThreads;   // that a thread moves in a step
    constexpr int kRowsAtOnce = kThreads / 8;
    extern __shared__ __align__(16) char lds[];
    const int64_t count = A.tiles_m * A.tiles_n;
    if (block_number() >= count) return;
    int64_t tm, tn;
    tile_of(A, block_number(), tm, tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    const int part = blockIdx.z;
    const int64_t k_from = part * A.k_part, k_to = k_from + A.k_part < A.k ? k_from + A.k_part : A.k;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, wm = wave / WN, wn = wave % WN;

    // rows of x first, rows of w behind them; rows past the end repeat the last one, and their results are not stored
    const T *rows[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int r = c * kRowsAtOnce + threadIdx.x / 8;
        if (r < BM) {
            const int64_t i = m0 + r < A.x.rows ? m0 + r : A.x.rows - 1;
            rows[c] = static_cast<const T *>(A.x.p) + i * A.x.ld;
        } else {
            const int64_t i = n0 + r - BM < A.w.rows ? n0 + r - BM : A.w.rows - 1;
            rows[c] = static_cast<const T *>(A.w.p) + i * A.w.ld;
        }
    }
    Sums<T> acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Sums<T>{0, 0, 0, 0};

    i32x4 next[kChunks];
    auto fetch = [&](int64_t k) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) next[c] = load_chunk(rows[c], k + (threadIdx.x % 8) * kChunkElems<T>, k_to);
    };
    auto put = [&] {
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            *reinterpret_cast<i32x4 *>(lds + chunk_place(c * kRowsAtOnce + threadIdx.x / 8, threadIdx.x % 8)) = next[c];
    };
    fetch(k_from);
    put();
    __syncthreads();
    for (int64_t k = k_from; k < k_to; k += kStepElems<T>) {
        const bool more = k + kStepElems<T> < k_to;
        if (more) fetch(k + kStepElems<T>);
        tile_step<T, BM, FM, FN>(lds, wm, wn, lane, acc);
        __syncthreads();
        if (more) {
            put();
            __syncthreads();
        }
    }
    tile_out<T, BM, BN, WM, WN>(A.E, lds, wm, wn, lane, acc, m0, n0, part);
}

// Tiles of 128 x 128 of operands that lie anywhere, where there are few and the way to memory is what a step waits for: kDeep steps are under
// way in registers, and two workgroups share a compute unit (1024^3 bf16 14 us, against 19 us with one step under way).
constexpr int kDeep = 2;

template <typename T, int WM, int WN>
__device__ __forceinline__ void deep_tile(const ProductArgs &A, int64_t block, int part, char *lds)
{
    constexpr int BM = 128, BN = 128, kThreads = WM * WN * kWave, FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int kChunks = (BM + BN) * 8 / kThreads, kRowsAtOnce = kThreads / 8, kStage = (BM + BN) * 128;
    int64_t tm, tn;
    tile_of(A, block, tm, tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    const int64_t k_from = part * A.k_part, k_to = k_from + A.k_part < A.k ? k_from + A.k_part : A.k;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, wm = wave / WN, wn = wave % WN;

    // rows of x first, rows of w behind them; rows past the end repeat the last one, and their results are not stored
    const T *rows[kChunks];
    int place[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int r = c * kRowsAtOnce + threadIdx.x / 8;
        const bool of_x = r < BM;
        const int64_t i = of_x ? m0 + r : n0 + r - BM, end = of_x ? A.x.rows : A.w.rows;
        rows[c] = static_cast<const T *>(of_x ? A.x.p : A.w.p) + (i < end ? i : end - 1) * (of_x ? A.x.ld : A.w.ld) + threadIdx.x % 8 * kChunkElems<T>;
        place[c] = chunk_place(r, threadIdx.x % 8);
    }
    Sums<T> acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Sums<T>{0, 0, 0, 0};

    i32x4 under_way[kDeep][kChunks];
    auto fetch_whole = [&](i32x4 (&to)[kChunks], int64_t k) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) __builtin_memcpy(&to[c], rows[c] + k, 16);
    };
    auto fetch = [&](i32x4 (&to)[kChunks], int64_t k) {
        if (k + kStepElems<T> <= k_to) {
            fetch_whole(to, k);
        } else if (k < k_to) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) to[c] = load_chunk(rows[c], k, k_to - threadIdx.x % 8 * kChunkElems<T>);
        }
    };
    auto put = [&](char *to, const i32x4 (&from)[kChunks]) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) *reinterpret_cast<i32x4 *>(to + place[c]) = from[c];
    };
    // two places in turn: who writes one again has passed the next step's barrier, behind which all have read it.  Neither the compiler's
    // stores to LDS before nor its reads behind may pass the barrier.
    auto multiply = [&](const char *now) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the loads from memory go on
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        tile_step<T, BM, FM, FN>(now, wm, wn, lane, acc);
    };
    const int whole = (int)((k_to - k_from) / kStepElems<T>), steps = (int)((k_to - k_from + kStepElems<T> - 1) / kStepElems<T>);
    auto place_of = [&](int i) { return k_from + (int64_t)i * kStepElems<T>; };
#pragma unroll
    for (int q = 0; q < kDeep; ++q) fetch(under_way[q], place_of(q));
    int i = 0;
    // without a condition between the loads, so that only the oldest are waited for
    for (; i + 2 * kDeep <= whole; i += kDeep) {
#pragma unroll
        for (int q = 0; q < kDeep; ++q) {
            put(lds + q % 2 * kStage, under_way[q]);
            fetch_whole(under_way[q], place_of(i + q + kDeep));
            multiply(lds + q % 2 * kStage);
        }
    }
    while (i < steps) {
#pragma unroll
        for (int q = 0; q < kDeep; ++q, ++i) {
            if (i >= steps) break;
            put(lds + q % 2 * kStage, under_way[q]);
            fetch(under_way[q], place_of(i + kDeep));
            multiply(lds + q % 2 * kStage);
        }
    }
    __syncthreads();
    tile_out<T, BM, BN, WM, WN>(A.E, lds, wm, wn, lane, acc, m0, n0, part);
}

// e4m3: one workgroup a compute unit, because its operands as bf16 do not fit 128 registers (1024^3 17.3 us, with two and spilt ones 19.8 us)
template <typename T, int WM, int WN>
__global__ __launch_bounds__(WM *WN *kWave, __is_same(T, e4m3) ? 2 : 4) void k_linear_deep(ProductArgs A)
{
    extern __shared__ __align__(16) char lds[];
    if (block_number() < A.tiles_m * A.tiles_n) deep_tile<T, WM, WN>(A, block_number(), blockIdx.z, lds);
}

// Two products in one launch, where the device has room for both: neither fills it.  Tiles of one after tiles of the other, parts in turn
// (all gradients of 1024^3: 50 us with one after the other, 38 us together).
template <typename T, int WM, int WN>
__global__ __launch_bounds__(WM *WN *kWave, 4) void k_linear_deep_two(ProductArgs A, ProductArgs B, int first)
{
    extern __shared__ __align__(16) char lds[];
    const int block = (int)blockIdx.x < first ? blockIdx.x : blockIdx.x - first;
    const ProductArgs P = (int)blockIdx.x < first ? A : B;
    const int tiles = (int)(P.tiles_m * P.tiles_n);
    deep_tile<T, WM, WN>(P, block % tiles, block / tiles, lds);
}

// ------------------------------------------------------------------ few rows
constexpr int kFewWaves = 4;

// Up to 16 MT rows of x, 16 NT rows of w a workgroup.  Its wavefronts take the inner index in turns of two steps of 128 bytes; a lane
// loads the chunks of its row straight into the registers of the matrix instruction, each row of w once.  Bound by that: one row of x,
// 32000 x 4096 bf16, 55 us, 4.8 TB/s.
template <typename T, int MT, int NT>
__global__ __launch_bounds__(kFewWaves *kWave) void k_linear_few(ProductArgs A)
{
    typedef typename SumOf<T>::one Sum;
    __shared__ __align__(16) Sum room[kFewWaves][MT * 16][NT * 16 + 4];
    const int64_t tn = block_number();
    if (tn >= A.tiles_n) return;
    const int part = blockIdx.z;
    const int64_t n0 = tn * NT * 16, k_from = part * A.k_part, k_to = k_from + A.k_part < A.k ? k_from + A.k_part : A.k;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const T *x[MT], *w[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = static_cast<const T *>(A.x.p) + (i * 16 + lane % 16 < A.x.rows ? i * 16 + lane % 16 : 0) * A.x.ld;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t r = n0 + j * 16 + lane % 16;
        w[j] = static_cast<const T *>(A.w.p) + (r < A.w.rows ? r : A.w.rows - 1) * A.w.ld;
    }
    Sums<T> acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = Sums<T>{0, 0, 0, 0};
    constexpr int kSteps = 2;
    constexpr int64_t kTurn = kSteps * kStepElems<T>;
    for (int64_t k = k_from + wave * kTurn; k < k_to; k += kFewWaves * kTurn) {
        i32x4 a[MT][kSteps][2], b[NT][kSteps][2];
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t at = k + s * kStepElems<T> + (lane / 16 + 4 * h) * kChunkElems<T>;
#pragma unroll
                for (int j = 0; j < NT; ++j) b[j][s][h] = load_chunk(w[j], at, k_to);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    a[i][s][h] = i32x4{0, 0, 0, 0};
                    if (i * 16 + lane % 16 < A.x.rows) a[i][s][h] = load_chunk(x[i], at, k_to);
                }
            }
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Fragment<T> f[MT];
#pragma unroll
                for (int i = 0; i < MT; ++i) f[i] = fragment<T>(a[i][s][h]);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const Fragment<T> g = fragment<T>(b[j][s][h]);
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[i][j] = mma<T>(g, f[i], acc[i][j]);
                }
            }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<Sums<T> *>(&room[wave][i * 16 + lane % 16][j * 16 + lane / 16 * 4]) = acc[i][j];
    __syncthreads();
    for (int at = threadIdx.x; at < MT * 16 * NT * 2; at += kFewWaves * kWave) {
        const int r = at / (NT * 2), c = at % (NT * 2) * kVec;
        if (r >= A.E.m || n0 + c >= A.E.n) continue;
        float v[1][kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            Sum sum = room[0][r][c + e];
            for (int u = 1; u < kFewWaves; ++u) sum += room[u][r][c + e];
            v[0][e] = __is_same(T, whole8) && A.E.part ? __builtin_bit_cast(float, sum) : (float)sum;
        }
        put8<false>(A.E, columns_of(A.E, n0 + c), v, r, 0, n0 + c, part);
    }
}

// ------------------------------------------------------------------ dx of few rows
// dx = dpre w for up to M rows: w is read once, as it lies.  A lane has eight columns and sums over the rows that its wavefront takes; dpre's
// factors of 256 rows of w lie in LDS, in 32 bits: no matrix unit takes them here, so they are not rounded.  Bound by reading w: 262 MB of it in 52 us
// (5.0 TB/s) for one row.  Against a turned copy of w and a product with it: all gradients of 3 x 29367 x 4841 f16 242 us (414 us), of
// 8 x 4096 x 4096 51 us (54 us), of 16 x 32000 x 4096 245 us (323 us), but of 16 x 4096 x 4096 61 us (54 us) - hence the rule of few_grad_rows.
inline bool few_grad_rows(int64_t m, int64_t n, int64_t k) { return m <= 8 || (m <= 16 && n * k >= (int64_t)1 << 25); }
constexpr int kFewGradCols = kWave * kVec, kFewGradStage = kBlock;

struct FewGradArgs {
    const void *w, *dy, *pre;
    int64_t m, n, k, ldw, lddy, ldpre, per;   // rows of w a part
    int act;
    Epilogue E;
};

template <typename T, int M>
__global__ __launch_bounds__(kBlock) void k_few_grad(FewGradArgs A)
{
    __shared__ __align__(16) float factor[kFewGradStage][M];
    __shared__ float sum[M][kVec][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t c0 = (int64_t)blockIdx.x * kFewGradCols, j = c0 + lane * kVec;
    const int64_t from = blockIdx.z * A.per, to = from + A.per < A.n ? from + A.per : A.n;
    const T *w = static_cast<const T *>(A.w);
    float acc[M][kVec];
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) acc[i][e] = 0.f;
    for (int64_t r0 = from; r0 < to; r0 += kFewGradStage) {
        const int here = (int)(to - r0 < kFewGradStage ? to - r0 : kFewGradStage);
        __syncthreads();
        {
            const int r = threadIdx.x;
            const T *dy = static_cast<const T *>(A.dy) + r0 + r, *pre = static_cast<const T *>(A.pre) + r0 + r;
            float v[M], at[M];
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const bool there = i < A.m && r < here;
                v[i] = there ? static_cast<float>(dy[i * A.lddy]) : 0.f;
                at[i] = there && A.act != TRON_ACT_NONE ? static_cast<float>(pre[i * A.ldpre]) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < M; ++i) factor[r][i] = A.act == TRON_ACT_NONE ? v[i] : v[i] * act_slope(at[i], A.act);
        }
        __syncthreads();
        if (j >= A.k) continue;
        auto add = [&](const Raw8<T> &raw, int r) {
#pragma unroll
            for (int i = 0; i < M; ++i)
#pragma unroll
                for (int e = 0; e < kVec; ++e) acc[i][e] = fmaf(factor[r][i], static_cast<float>(raw.v[e]), acc[i][e]);
        };
        constexpr int kAhead = M == 16 ? 2 : 4;
        int r = wave;
#pragma unroll 1
        for (; r + (kAhead - 1) * kWavesPerBlock < here; r += kAhead * kWavesPerBlock) {
            Raw8<T> raw[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) raw[q] = load_row8(w + (r0 + r + q * kWavesPerBlock) * A.ldw, j, A.k, static_cast<T>(0.f));
#pragma unroll
            for (int q = 0; q < kAhead; ++q) add(raw[q], r + q * kWavesPerBlock);
        }
#pragma unroll 1
        for (; r < here; r += kWavesPerBlock) add(load_row8(w + (r0 + r) * A.ldw, j, A.k, static_cast<T>(0.f)), r);
    }
    // the wavefronts' sums, one after the other
    for (int u = 0; u < kWavesPerBlock; ++u) {
        __syncthreads();
        if (wave != u) continue;
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[i][e][lane] = u ? sum[i][e][lane] + acc[i][e] : acc[i][e];
    }
    __syncthreads();
    if (j >= A.k) return;
#pragma unroll 1
    for (int i = wave; i < A.m; i += kWavesPerBlock) {
        float v[1][kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[0][e] = sum[i][e][lane];
        put8<false>(A.E, columns_of(A.E, j), v, i, 0, j, blockIdx.z);
    }
}

// ------------------------------------------------------------------ which kernel
enum Shape { SHAPE_FEW = 0, SHAPE_128, SHAPE_256 };
struct Plan {
    Shape shape;
    int64_t tiles_m, tiles_n;
    int parts;
    int64_t k_part;
};

constexpr int64_t kFewRows = 32;   // 33 rows of 32000 x 4096 bf16 took 72 us by that kernel and 67 us in tiles of 128 rows
constexpr int64_t kUnits = 256;    // compute units
constexpr int64_t kMostParts = 64;

// What p parts of the inner index cost beside their products: the second launch, and the way of 32-bit sums to memory and back at some 4 TB/s
double cut_us(int64_t p, double results) { return p > 1 ? 4.0 + (double)p * results * 8.0 / 4e6 : 0.0; }

// Tiles and parts by the time that they take, measured in microseconds on bf16: a step of a tile of 256 x 256 1.5 (one workgroup a compute
// unit) and its beginning and end 12; a step of a tile of 128 x 128 0.65 where a compute unit has one, 1.0 where it has two, and
// 4.  Both sides: 4096^3 111 us in large tiles, 2048 x 2048 x 4096 47 us in small ones (70 us in large ones cut in four),
// 1024^3 14 us in one part and 18 us in two, 777 x 1001 x 2049 26 us in two and 23 us in four.
Plan linear_plan(int64_t m, int64_t n, int64_t k, int type)
{
    const int64_t step = 128 / type_bytes(type), steps = std::max<int64_t>(1, ceil_div(k, step));
    const double results = (double)m * (double)n, slow = type == TRON_TYPE_E4M3 ? 2.0 : 1.0;   // twice the inner index a step
    Plan best{SHAPE_FEW, 1, ceil_div(n, 64), 1, 0};
    double best_us = HUGE_VAL;
    int64_t parts = 1;
    if (m <= kFewRows) {
        // eight steps a turn of its wavefronts, one microsecond
        const int64_t turns = ceil_div(steps, 2 * kFewWaves);
        for (int64_t p = 1; p == 1 || p <= std::min({2 * kUnits / best.tiles_n, turns, kMostParts}); ++p) {
            const double us = (double)ceil_div(turns, p) + cut_us(p, results);
            if (us < best_us) {
                best_us = us;
                parts = p;
            }
        }
    } else {
        for (const Shape shape : {SHAPE_256, SHAPE_128}) {
            if (g_tuning.linear_tile == (shape == SHAPE_256 ? 128 : 256)) continue;
            const int64_t b = shape == SHAPE_256 ? 256 : 128, tiles_m = ceil_div(m, b), tiles_n = ceil_div(n, b), tiles = tiles_m * tiles_n;
            for (int64_t p = 1; p == 1 || p <= std::min({2 * kUnits / tiles, steps, kMostParts}); ++p) {
                const int64_t each = ceil_div(steps, p);
                const double rounds = shape == SHAPE_256 ? (double)ceil_div(tiles * p, kUnits) * 1.5 : tiles * p <= kUnits ? 0.65 : (double)ceil_div(tiles * p, 2 * kUnits);
                const double us = rounds * slow * (double)each + (shape == SHAPE_256 ? 12.0 : 4.0) + cut_us(p, results);
                if (us < best_us) {
                    best_us = us;
                    best = Plan{shape, tiles_m, tiles_n, 1, 0};
                    parts = p;
                }
            }
        }
    }
    best.k_part = ceil_div(steps, parts) * step;
    best.parts = (int)ceil_div(steps * step, best.k_part);
    return best;
}

int64_t plan_bytes(const Plan &P, int64_t m, int64_t n) { return P.parts > 1 ? ceil_div(P.parts * m * n * 4, 16) * 16 : 0; }

template <typename K>
int allow_lds(K kernel, int bytes)
{
    TRON_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return TRON_OK;
}

template <typename T, int MT>
void launch_few(const ProductArgs &A, dim3 grid, hipStream_t st)
{
    k_linear_few<T, MT, 4><<<grid, kFewWaves * kWave, 0, st>>>(A);
}

// whether rows are whole chunks at multiples of 16 bytes, and a tile's offsets and a row's bytes fit 31 bits
template <typename T>
bool direct_ok(const Operand &a, int64_t k)
{
    return ((uintptr_t)a.p & 15) == 0 && a.ld % kChunkElems<T> == 0 && k % kChunkElems<T> == 0 && (a.ld * 256 + k) * (int64_t)sizeof(T) < 0x7fff0000;
}

// Kernels that take more LDS than a launch may without having said so
template <typename T>
int launch_256(const ProductArgs &A, dim3 grid, hipStream_t st)
{
    constexpr int kLds = kTileLds<256, 256>;
    if (direct_ok<T>(A.x, A.k) && direct_ok<T>(A.w, A.k)) {
        TRON_TRY(allow_lds(k_linear_direct<T, 256, 256, 2, 4>, kLds));
        k_linear_direct<T, 256, 256, 2, 4><<<grid, 512, kLds, st>>>(A);
    } else {
        TRON_TRY(allow_lds(k_linear_tile<T, 256, 256, 2, 4>, kLds));
        k_linear_tile<T, 256, 256, 2, 4><<<grid, 512, kLds, st>>>(A);
    }
    return TRON_OK;
}

template <typename T>
int launch_128(const ProductArgs &A, dim3 grid, hipStream_t st)
{
    constexpr int kLds = kTileLds<128, 128>;
    TRON_TRY(allow_lds(k_linear_deep<T, 2, 4>, kLds));
    k_linear_deep<T, 2, 4><<<grid, 512, kLds, st>>>(A);
    return TRON_OK;
}

ProductArgs product_args(Operand x, Operand w, int64_t k, const Plan &P, Epilogue E, float *part)
{
    E.part = P.parts > 1 ? part : nullptr;
    E.past = goes_past(E.m, E.n, type_bytes(E.out));
    return ProductArgs{x, w, k, P.k_part, P.tiles_m, P.tiles_n, E};
}

template <typename T>
int product(const ProductArgs &A, const Plan &P, hipStream_t st)
{
    dim3 grid = block_grid(P.tiles_m * P.tiles_n);
    grid.z = (unsigned)P.parts;
    if (P.shape == SHAPE_FEW) {
        if (A.x.rows <= 16) launch_few<T, 1>(A, grid, st);
        else launch_few<T, 2>(A, grid, st);
    } else if (P.shape == SHAPE_128) {
        TRON_TRY(launch_128<T>(A, grid, st));
    } else {
        TRON_TRY(launch_256<T>(A, grid, st));
    }
    TRON_HIP(hipGetLastError());
    return P.parts > 1 ? join_parts<__is_same(T, whole8)>(A.E, P.parts, st) : TRON_OK;
}

// whether two products go into one launch: both in tiles of 128 x 128, and all of these under way at once, two a compute unit
bool together(const Plan &P, const Plan &Q)
{
    return P.shape == SHAPE_128 && Q.shape == SHAPE_128 && P.tiles_m * P.tiles_n * P.parts + Q.tiles_m * Q.tiles_n * Q.parts <= 2 * kUnits;
}

template <typename T>
int two_products(const ProductArgs &A, const Plan &P, const ProductArgs &B, const Plan &Q, hipStream_t st)
{
    constexpr int kLds = kTileLds<128, 128>;
    const int first = (int)(P.tiles_m * P.tiles_n * P.parts), second = (int)(Q.tiles_m * Q.tiles_n * Q.parts);
    TRON_TRY(allow_lds(k_linear_deep_two<T, 2, 4>, kLds));
    k_linear_deep_two<T, 2, 4><<<first + second, 512, kLds, st>>>(A, B, first);
    TRON_HIP(hipGetLastError());
    if (P.parts > 1) TRON_TRY(join_parts(A.E, P.parts, st));
    return Q.parts > 1 ? join_parts(B.E, Q.parts, st) : TRON_OK;
}

// ------------------------------------------------------------------ gradients
constexpr int kPatch = 64;   // rows and columns of a patch that one wavefront turns

struct TurnArgs {
    const void *a, *pre;       // [rows][cols]; pre: a is multiplied by act'(pre)
    int64_t rows, cols, lda, ldpre;
    int act;
    void *same, *turned;       // [rows][ldsame], [cols][ldturned], zeros from the last element to the end of its chunk; or NULL
    int64_t ldsame, ldturned;
    float *shares;             // [patches of rows][cols]: column sums of the products before rounding, or NULL
    float *factor;             // f16: see k_range_parts; or NULL, and the products are rounded as they are
    int range_parts;
    int64_t again_same, again_turned;   // elements of a row of `same` and of `turned` behind which it is there again, for dpre in two parts; 0: it is not
    int64_t blocks;
};

struct TurnList {
    TurnArgs list[3];
    int count;
};

// Eight rows of eight elements in a lane, turned: pairs of rows change elements, words and pairs of words.
template <typename T>
__device__ __forceinline__ void turn8(Raw8<T> (&r)[kVec])
{
    uint32_t w[kVec][4];
#pragma unroll
    for (int i = 0; i < kVec; ++i) __builtin_memcpy(w[i], &r[i], 16);
    uint32_t t[kVec][4];   // t[c][p]: column c's elements of rows 2p and 2p + 1
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            t[2 * q][p] = __builtin_amdgcn_perm(w[2 * p + 1][q], w[2 * p][q], 0x05040100);
            t[2 * q + 1][p] = __builtin_amdgcn_perm(w[2 * p + 1][q], w[2 * p][q], 0x07060302);
        }
#pragma unroll
    for (int i = 0; i < kVec; ++i) __builtin_memcpy(&r[i], t[i], 16);
}

// f16: dpre is dy times a slope of up to 1.13, which may lie above the largest value or below the smallest where the products' results
// do not.  It is held times a power of two, by which the largest |dy| comes to lie in [2^14, 2^15), and the results are multiplied by its
// reciprocal.  This launch takes the maximum, in parts behind that factor; the next one joins them, and its first wavefront writes the
// factor.  8192 x 4096: 25 us.
constexpr int kRangeBlocks = 512;

__global__ __launch_bounds__(kBlock) void k_range_parts(const _Float16 *dy, int64_t m, int64_t n, int64_t ld, float *parts)
{
    __shared__ float room[2 * kMostWaves];
    const int64_t across = (n + kVec - 1) / kVec, chunks = m * across;
    float top = 0.f, none = 0.f;
    for (int64_t c = (int64_t)blockIdx.x * kBlock + threadIdx.x; c < chunks; c += (int64_t)gridDim.x * kBlock) {
        const int64_t i = c / across;
        const Raw8<_Float16> r = load_row8(dy + i * ld, (c - i * across) * kVec, n, static_cast<_Float16>(0.f));
#pragma unroll
        for (int e = 0; e < kVec; ++e) top = fmaxf(top, fabsf(static_cast<float>(r.v[e])));
    }
    block_sum_max(none, top, room);
    if (threadIdx.x == 0) parts[blockIdx.x] = top;
}

int range_blocks(int64_t m, int64_t n) { return (int)std::min<int64_t>(kRangeBlocks, ceil_div(m * ceil_div(n, kVec), kBlock)); }

// by a wavefront; `writes`: whether it is the one that writes the reciprocal
__device__ __forceinline__ float range_factor(float *factor, int parts, int lane, bool writes)
{
    float top = 0.f;
    for (int i = lane; i < parts; i += kWave) top = fmaxf(top, factor[1 + i]);
    top = wave_maxf(top);
    // infinities stay what they are; all others are safe as beside 65504
    const int e = top == 0.f ? 0 : top < INFINITY ? 14 - ilogbf(top) : -1;
    if (writes && lane == 0) *factor = ldexpf(1.f, -e);
    return ldexpf(1.f, e);
}

// A wavefront a patch: lane 8 a + b holds rows 8 a .. + 7 and columns 8 b .. + 7, reads them as eight pieces of 16 bytes, and writes them so or
// turned in its registers.  The four of a workgroup take patches one below the other: their pieces of a turned row are 512 bytes (side by
// side 42 us, so 35 us for 8192 x 4096 bf16, 3.8 TB/s).
// All copies of a call are one launch, and the activation is chosen once a patch: its code is long, and a small copy waits for it to be fetched.
// TWO: dpre is followed by what its rounding left, none where it is not finite, and the other operands by themselves, with 0 for what is not
// finite (its products are in the first part's sum).
template <typename T, int ACT, bool TWO>
__device__ __forceinline__ void turn_patch(const TurnArgs &A, int64_t block)
{
    static_assert(sizeof(T) == 2, "two elements a word");
    const int64_t across = (A.cols + kPatch - 1) / kPatch, down = (A.rows + kPatch - 1) / kPatch;
    const int64_t patch_row = block / across * kWavesPerBlock + threadIdx.x / kWave, patch_col = block % across;
    if (patch_row >= down) return;
    const int lane = threadIdx.x % kWave;
    const int64_t i0 = patch_row * kPatch + lane / 8 * kVec, j = patch_col * kPatch + lane % 8 * kVec, n = A.cols - j;
    Raw8<T> raw[kVec], p[kVec];
#pragma unroll
    for (int r = 0; r < kVec; ++r) {
        const bool there = i0 + r < A.rows && n > 0;
        if (there) raw[r] = load_row8(static_cast<const T *>(A.a) + (i0 + r) * A.lda, j, A.cols, static_cast<T>(0.f));
        if (there && ACT != TRON_ACT_NONE) p[r] = load_row8(static_cast<const T *>(A.pre) + (i0 + r) * A.ldpre, j, A.cols, static_cast<T>(0.f));
    }
    float sum[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) sum[e] = 0.f;
    const float factor = ACT != TRON_ACT_NONE && !__is_same(T, __bf16) && A.factor ? range_factor(A.factor, A.range_parts, lane, patch_row == 0 && patch_col == 0) : 1.f;
#pragma unroll
    for (int r = 0; r < kVec; ++r) {
        if (i0 + r < A.rows && n > 0) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                float v = static_cast<float>(raw[r].v[e]);
                if (ACT != TRON_ACT_NONE) {
                    v = e < n ? v * act_slope(static_cast<float>(p[r].v[e]), ACT) : 0.f;
                    raw[r].v[e] = static_cast<T>(v * factor);
                    if (TWO) {
                        const float left = v * factor - static_cast<float>(raw[r].v[e]);
                        p[r].v[e] = static_cast<T>(__builtin_isfinite(left) ? left : 0.f);
                    }
                } else if (TWO) {
                    p[r].v[e] = static_cast<T>(__builtin_isfinite(v) ? v : 0.f);
                }
                sum[e] += v;
            }
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) raw[r].v[e] = p[r].v[e] = static_cast<T>(0.f);
        }
        if (A.same && i0 + r < A.rows && j < A.ldsame) {
            T *row = static_cast<T *>(A.same) + (i0 + r) * A.ldsame + j;
            store8(row, raw[r]);
            if (TWO) store8(row + A.again_same, p[r]);
        }
    }
    if (A.shares) {
        // over the eight lanes of a column
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            sum[e] += __shfl_xor(sum[e], 8);
            sum[e] += __shfl_xor(sum[e], 16);
            sum[e] += __shfl_xor(sum[e], 32);
        }
        if (lane < 8 && n > 0) store8_of<float>(A.shares + patch_row * A.cols + j, sum, n);
    }
    if (!A.turned) return;
    auto put = [&](Raw8<T> (&r)[kVec], int64_t at) {
        turn8(r);
        if (at >= A.ldturned) return;
#pragma unroll
        for (int c = 0; c < kVec; ++c)
            if (j + c < A.cols) store8(static_cast<T *>(A.turned) + (j + c) * A.ldturned + at, r[c]);
    };
    put(raw, i0);
    if (TWO) put(p, A.again_turned + i0);
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_turn(TurnList L)
{
    int64_t block = block_number();
    int which = 0;
    while (which < L.count && block >= L.list[which].blocks) block -= L.list[which++].blocks;
    if (which == L.count) return;
    const TurnArgs A = L.list[which];
    const bool two = A.again_turned != 0;
    switch (A.act) {
    case TRON_ACT_RELU: return turn_patch<T, TRON_ACT_RELU, false>(A, block);
    case TRON_ACT_GELU: return two ? turn_patch<T, TRON_ACT_GELU, true>(A, block) : turn_patch<T, TRON_ACT_GELU, false>(A, block);
    case TRON_ACT_SILU: return two ? turn_patch<T, TRON_ACT_SILU, true>(A, block) : turn_patch<T, TRON_ACT_SILU, false>(A, block);
    default: return two ? turn_patch<T, TRON_ACT_NONE, true>(A, block) : turn_patch<T, TRON_ACT_NONE, false>(A, block);
    }
}

template <typename T>
int turn(TurnList &L, hipStream_t st)
{
    int64_t blocks = 0;
    for (int i = 0; i < L.count; ++i) blocks += L.list[i].blocks = ceil_div(L.list[i].rows, kPatch * kWavesPerBlock) * ceil_div(L.list[i].cols, kPatch);
    if (!blocks) return TRON_OK;
    k_turn<T><<<block_grid(blocks), kBlock, 0, st>>>(L);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

// Row length of the copies: whole chunks, and no multiple of 1 KB, whose rows' equal columns lie in one channel of the L2 (8192 x 8192 x 4096:
// 478 us with rows of 8 KB, 441 us with 128 bytes more).
inline int64_t whole(int64_t n) { return ceil_div(n, kVec) * kVec; }
inline int64_t padded(int64_t n) { return whole(n) % 512 == 0 ? whole(n) + 64 : whole(n); }

// Parts of the rows of w for dx of few rows: workgroups for four a compute unit, 64 rows of w each at least
int64_t few_grad_parts(int64_t n, int64_t k)
{
    return std::max<int64_t>(1, std::min<int64_t>(ceil_div(n, 64), 4 * kUnits / ceil_div(k, kFewGradCols)));
}

template <typename T>
int few_grad(FewGradArgs A, float *part, hipStream_t st)
{
    A.per = ceil_div(A.n, few_grad_parts(A.n, A.k));
    const int parts = (int)ceil_div(A.n, A.per);
    A.E.part = parts > 1 ? part : nullptr;
    const dim3 grid((unsigned)ceil_div(A.k, kFewGradCols), 1, (unsigned)parts);
    if (A.m <= 4) k_few_grad<T, 4><<<grid, kBlock, 0, st>>>(A);
    else if (A.m <= 8) k_few_grad<T, 8><<<grid, kBlock, 0, st>>>(A);
    else k_few_grad<T, 16><<<grid, kBlock, 0, st>>>(A);
    TRON_HIP(hipGetLastError());
    return parts > 1 ? join_parts(A.E, parts, st) : TRON_OK;
}

// the work space of the gradients, in the order of its parts
struct GradSpace {
    int64_t dpre, dpre_t, w_t, x_t, shares, factor, part_dx, part_dw, total;
    int64_t again_n, again_m;   // dpre in two parts: elements of each part of a row; 0: in one
    int64_t inner_n, inner_m;   // inner lengths of dx and of dw in the copies
    Plan for_dx, for_dw;
    bool few, both;   // dx of few rows; dx and dw in one launch
};
// slopes other than 0 and 1, so that dpre has more bits than dy
bool smooth(int act) { return act == TRON_ACT_GELU || act == TRON_ACT_SILU; }

// The products take dpre as two operands of 16 bits, rounded and what the rounding left, one behind the other along the inner index, against
// the other operand twice: results have their own rounding alone.  narrow, the caller's choice: rounded alone.  8192 x 4096 x 4096
// bf16 gelu, error against 64 bits as a share of the result: dx and dw in bf16 1.66e-3, dw in f32 2.6e-6, in 1046 us; narrow 2.35e-3, 1.7e-3,
// in 566 us.  Parts of whole patches, whose ends are zeros.
GradSpace grad_space(int64_t m, int64_t n, int64_t k, int act, bool narrow, bool dx, bool dw, bool db)
{
    GradSpace S;
    int64_t at = 0;
    auto take = [&](bool want, int64_t bytes) {
        const int64_t from = at;
        if (want) at += ceil_div(bytes, 256) * 256;
        return from;
    };
    const bool two = smooth(act) && !narrow;
    S.again_n = two ? ceil_div(n, kPatch) * kPatch : 0;
    S.again_m = two ? ceil_div(m, kPatch) * kPatch : 0;
    S.inner_n = two ? 2 * S.again_n : whole(n);
    S.inner_m = two ? 2 * S.again_m : whole(m);
    S.few = few_grad_rows(m, n, k);
    S.for_dx = linear_plan(m, k, S.inner_n, TRON_TYPE_BF16);
    S.for_dw = linear_plan(n, k, S.inner_m, TRON_TYPE_BF16);
    S.both = dx && dw && !S.few && together(S.for_dx, S.for_dw);
    S.dpre = take(dx && act != TRON_ACT_NONE && !S.few, m * padded(S.inner_n) * 2);
    S.dpre_t = take(dw, n * padded(S.inner_m) * 2);
    S.w_t = take(dx && !S.few, k * padded(S.inner_n) * 2);
    S.x_t = take(dw, k * padded(S.inner_m) * 2);
    S.shares = take(db, ceil_div(m, kPatch) * n * 4);
    S.factor = take(smooth(act) && (dw || (dx && !S.few)), (1 + kRangeBlocks) * 4);
    const int64_t of_dx = !dx ? 0 : S.few ? few_grad_parts(n, k) * m * k * 4 : plan_bytes(S.for_dx, m, k), of_dw = dw ? plan_bytes(S.for_dw, n, k) : 0;
    S.part_dx = take(true, S.both ? of_dx : std::max(of_dx, of_dw));
    S.part_dw = S.both ? take(true, of_dw) : S.part_dx;
    S.total = at;
    return S;
}

struct GradArgs {
    int64_t m, n, k;
    const void *x, *w, *dy, *pre;
    int64_t ldx, ldw, lddy, ldpre;
    int act, type;
    bool narrow;
    void *dx, *dw;
    int64_t lddx, lddw;
    int dw_type;
    float *dbias;
    char *work;
};

template <typename T>
int linear_grad_typed(const GradArgs &G, hipStream_t st)
{
    const int64_t m = G.m, n = G.n, k = G.k;
    const bool act = G.act != TRON_ACT_NONE;
    const GradSpace S = grad_space(m, n, k, G.act, G.narrow, G.dx, G.dw, G.dbias);
    const int64_t np = padded(S.inner_n), mp = padded(S.inner_m);
    float *shares = reinterpret_cast<float *>(G.work + S.shares), *part_dx = reinterpret_cast<float *>(G.work + S.part_dx);
    void *dpre = G.work + S.dpre, *dpre_t = G.work + S.dpre_t, *w_t = G.work + S.w_t, *x_t = G.work + S.x_t;
    const bool same = G.dx && act && !S.few, rounds = smooth(G.act) && (same || G.dw);
    float *factor = nullptr;
    if (!__is_same(T, __bf16) && rounds) {
        factor = reinterpret_cast<float *>(G.work + S.factor);
        k_range_parts<<<range_blocks(m, n), kBlock, 0, st>>>(static_cast<const _Float16 *>(G.dy), m, n, G.lddy, factor + 1);
    }
    TurnList L{};
    if (G.dbias || G.dw || same)
        L.list[L.count++] = TurnArgs{G.dy, G.pre, m, n, G.lddy, G.ldpre, G.act, same ? dpre : nullptr, G.dw ? dpre_t : nullptr, np, mp, G.dbias ? shares : nullptr, factor,
                                     range_blocks(m, n), rounds ? S.again_n : 0, rounds ? S.again_m : 0, 0};
    if (G.dx && !S.few) L.list[L.count++] = TurnArgs{G.w, nullptr, n, k, G.ldw, 0, TRON_ACT_NONE, nullptr, w_t, 0, np, nullptr, nullptr, 0, 0, S.again_n, 0};
    if (G.dw) L.list[L.count++] = TurnArgs{G.x, nullptr, m, k, G.ldx, 0, TRON_ACT_NONE, nullptr, x_t, 0, mp, nullptr, nullptr, 0, 0, S.again_m, 0};
    TRON_TRY(turn<T>(L, st));
    if (G.dbias) TRON_TRY(column_sums(shares, ceil_div(m, kPatch), n, G.dbias, st));
    Epilogue E{}, F{};
    E.y = G.dx;
    E.m = m;
    E.n = k;
    E.ldy = G.lddx;
    E.out = G.type;
    F.y = G.dw;
    F.m = n;
    F.n = k;
    F.ldy = G.lddw;
    F.out = G.dw_type;
    Epilogue few = E;   // which multiplies dy itself
    E.factor = F.factor = factor;
    // without an activation dy itself, whose rows end at n
    const ProductArgs A = product_args(act ? Operand{dpre, m, np} : Operand{G.dy, m, G.lddy}, Operand{w_t, k, np}, act ? S.inner_n : n, S.for_dx, E, part_dx);
    const ProductArgs B = product_args(Operand{dpre_t, n, mp}, Operand{x_t, k, mp}, S.inner_m, S.for_dw, F, reinterpret_cast<float *>(G.work + S.part_dw));
    if (S.both) return two_products<T>(A, S.for_dx, B, S.for_dw, st);
    if (G.dx && S.few) TRON_TRY(few_grad<T>(FewGradArgs{G.w, G.dy, G.pre, m, n, k, G.ldw, G.lddy, G.ldpre, 0, G.act, few}, part_dx, st));
    else if (G.dx) TRON_TRY(product<T>(A, S.for_dx, st));
    return G.dw ? product<T>(B, S.for_dw, st) : TRON_OK;
}

bool sizes_ok(int64_t m, int64_t n, int64_t k)
{
    return m >= 0 && n >= 1 && k >= 1 && m <= INT32_MAX && n <= INT32_MAX && k <= INT32_MAX && extent_ok(m, n, n) && extent_ok(m, k, k) && extent_ok(n, k, k);
}
bool operand_ok(int type, int64_t k) { return type >= TRON_TYPE_BF16 && type <= TRON_TYPE_I8 && (type != TRON_TYPE_I8 || k <= kMostWhole); }
bool act_ok(int act) { return act >= TRON_ACT_NONE && act <= TRON_ACT_SILU; }

}  // namespace
}  // namespace tron

using namespace tron;

extern "C" {

int64_t tron_linear_work(int64_t m, int64_t n, int64_t k, int type)
{
    return sizes_ok(m, n, k) && m > 0 && operand_ok(type, k) ? plan_bytes(linear_plan(m, n, k, type), m, n) : 0;
}

int tron_linear(int64_t m, int64_t n, int64_t k, int type, const void *x, int64_t ldx, const float *x_scale, const void *w, int64_t ldw, const float *w_scale,
                const float *bias, int act, const void *residual, int64_t ldr, int out_type, void *y, int64_t ldy, void *pre, int64_t ldpre, void *work,
                int64_t work_bytes, void *hip_stream)
{
    const bool eight = type == TRON_TYPE_E4M3 || type == TRON_TYPE_I8;
    if (!sizes_ok(m, n, k) || !operand_ok(type, k) || !type_is_float(out_type) || !act_ok(act)) {
        set_error("tron_linear: bad argument (need 0 <= m < 2^31, 1 <= n, k < 2^31, operands bf16, f16, e4m3 or, up to k < 2^17, i8, out_type f32, bf16 or f16, a known activation)");
        return TRON_EINVAL;
    }
    if (m > 0 && (!x || !w || !y || (eight && (!x_scale || !w_scale)) || (!eight && (x_scale || w_scale)))) {
        set_error("tron_linear: bad argument (x, w and y are needed; operands of 8 bits, and they alone, have scales)");
        return TRON_EINVAL;
    }
    if (m > 0 && (!rows_ok(m, k, ldx, false) || !rows_ok(n, k, ldw, false) || (residual && !rows_ok(m, n, ldr, false)) || !rows_ok(m, n, ldy, true) ||
                  (pre && !rows_ok(m, n, ldpre, true)) || !extent_ok(m, ldx, k) || !extent_ok(n, ldw, k) || !extent_ok(m, residual ? ldr : 0, n) ||
                  !extent_ok(m, ldy, n) || !extent_ok(m, pre ? ldpre : 0, n))) {
        set_error("tron_linear: bad leading dimension (rows that are written may not overlap)");
        return TRON_EINVAL;
    }
    if (m > 0 && !work_ok(work, work_bytes, tron_linear_work(m, n, k, type))) {
        set_error("tron_linear: needs a work space of tron_linear_work(m, n, k, type) bytes at a multiple of 16");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    if (m == 0) return TRON_OK;
    const Epilogue E{x_scale, w_scale, bias, residual, y, pre, m, n, ldr, ldy, ldpre, act, out_type, nullptr, false, nullptr};
    const Operand a{x, m, ldx}, b{w, n, ldw};
    const Plan P = linear_plan(m, n, k, type);
    const ProductArgs A = product_args(a, b, k, P, E, static_cast<float *>(work));
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    return type == TRON_TYPE_BF16 ? product<__bf16>(A, P, st)
           : type == TRON_TYPE_F16 ? product<_Float16>(A, P, st) : type == TRON_TYPE_E4M3 ? product<e4m3>(A, P, st) : product<whole8>(A, P, st);
}

int64_t tron_linear_grad_work(int64_t m, int64_t n, int64_t k, int act, int want_dx, int want_dw, int want_dbias)
{
    const bool narrow = (act & TRON_ACT_NARROW) != 0;
    act &= ~TRON_ACT_NARROW;
    return sizes_ok(m, n, k) && m > 0 && act_ok(act) ? grad_space(m, n, k, act, narrow, want_dx != 0, want_dw != 0, want_dbias != 0).total : 0;
}

int tron_linear_grad(int64_t m, int64_t n, int64_t k, int type, const void *x, int64_t ldx, const void *w, int64_t ldw, const void *dy, int64_t lddy, int act,
                     const void *pre, int64_t ldpre, void *dx, int64_t lddx, int dw_type, void *dw, int64_t lddw, float *dbias, void *work, int64_t work_bytes,
                     void *hip_stream)
{
    const int act_and_narrow = act;
    act &= ~TRON_ACT_NARROW;
    if (!sizes_ok(m, n, k) || (type != TRON_TYPE_BF16 && type != TRON_TYPE_F16) || !act_ok(act) || (dw && !type_is_float(dw_type))) {
        set_error("tron_linear_grad: bad argument (need 0 <= m < 2^31, 1 <= n, k < 2^31, type bf16 or f16, dw_type f32, bf16 or f16, a known activation)");
        return TRON_EINVAL;
    }
    if (m > 0 && ((dw && !x) || (dx && !w) || !dy || (act != TRON_ACT_NONE && !pre))) {
        set_error("tron_linear_grad: bad argument (dy is needed, x for dw, w for dx, pre where there is an activation)");
        return TRON_EINVAL;
    }
    if (m > 0 && ((dw && !rows_ok(m, k, ldx, false)) || (dx && !rows_ok(n, k, ldw, false)) || !rows_ok(m, n, lddy, false) ||
                  (act != TRON_ACT_NONE && !rows_ok(m, n, ldpre, false)) || !extent_ok(m, dw ? ldx : 0, k) || !extent_ok(n, dx ? ldw : 0, k) ||
                  !extent_ok(m, lddy, n) || !extent_ok(m, act != TRON_ACT_NONE ? ldpre : 0, n) || (dx && (!rows_ok(m, k, lddx, true) || !extent_ok(m, lddx, k))))) {
        set_error("tron_linear_grad: bad leading dimension (rows that are written may not overlap)");
        return TRON_EINVAL;
    }
    if (dw && (!rows_ok(n, k, lddw, true) || !extent_ok(n, lddw, k))) {
        set_error("tron_linear_grad: bad leading dimension of dw");
        return TRON_EINVAL;
    }
    if (m > 0 && !work_ok(work, work_bytes, tron_linear_grad_work(m, n, k, act_and_narrow, dx != nullptr, dw != nullptr, dbias != nullptr))) {
        set_error("tron_linear_grad: needs a work space of tron_linear_grad_work(...) bytes at a multiple of 16");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    if (m == 0) {
        // sums over no rows
        if (dbias) TRON_TRY(column_sums(nullptr, 0, n, dbias, st));
        if (!dw) return TRON_OK;
        Epilogue E{};
        E.y = dw;
        E.m = n;
        E.n = k;
        E.ldy = lddw;
        E.out = dw_type;
        return join_parts(E, 0, st);
    }
    const GradArgs G{m, n, k, x, w, dy, pre, ldx, ldw, lddy, ldpre, act, type, act != act_and_narrow, dx, dw, lddx, lddw, dw_type, dbias, static_cast<char *>(work)};
    return type == TRON_TYPE_BF16 ? linear_grad_typed<__bf16>(G, st) : linear_grad_typed<_Float16>(G, st);
}

}  // extern "C"
