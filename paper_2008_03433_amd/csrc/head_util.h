// What the operators of multi-class heads share: element types, loads and stores of eight elements, sums over wavefronts and
// workgroups in 32 bits, argument checks.
#pragma once

#include <cmath>

#include "common.h"
#include "device_util.h"

namespace tron {

// ---------------------------------------------------------------- element types
// e4m3 has no arithmetic type of its own: a byte that the conversion instructions read and write
struct e4m3 {
    uint8_t bits;
};

// whole numbers of 8 bits, -127 .. 127 as outputs
struct whole8 {
    int8_t v;
};

inline int type_bytes(int type) { return type == TRON_TYPE_F32 ? 4 : type == TRON_TYPE_E4M3 || type == TRON_TYPE_I8 ? 1 : 2; }
inline bool type_is_float(int type) { return type == TRON_TYPE_F32 || type == TRON_TYPE_BF16 || type == TRON_TYPE_F16; }

// ---------------------------------------------------------------- eight elements at a time
// A thread moves eight neighbouring elements with one or two wide instructions.  Rows may start at any multiple of the element's
// size: the copies are declared with that alignment, and the memory pipeline takes wide accesses at any address.
constexpr int kVec = 8;

template <typename T>
struct Raw8 {
    T v[kVec];
};

// The same in whole registers: elements of 16 bits that are copied from one place to another take a register each
template <typename T>
struct Eight {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ void set(const Raw8<T> &r) { __builtin_memcpy(w, &r, sizeof(w)); }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (__is_same(T, __bf16)) return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return static_cast<float>(__builtin_bit_cast(_Float16, (uint16_t)(i % 2 ? w[i / 2] >> 16 : w[i / 2])));
    }
};

template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T *p)
{
    Raw8<T> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}

template <typename T>
__device__ __forceinline__ void store8(T *p, const Raw8<T> &r)
{
    __builtin_memcpy(p, &r, sizeof(r));
}

// the first n of eight; the others are `fill`
template <typename T>
__device__ __forceinline__ Raw8<T> load_first(const T *p, int n, T fill)
{
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) r.v[i] = i < n ? p[i] : fill;
    return r;
}

// Eight elements of a row from j < to on; from `to` on they are `fill`.  A row's end is read with the wide load that ends there, whose
// elements are moved down: single loads of up to seven elements one after the other hold up the whole workgroup.
template <typename T>
__device__ __forceinline__ Raw8<T> load_row8(const T *row, int64_t j, int64_t to, T fill)
{
    if (j + kVec <= to) return load8(row + j);
    const int n = (int)(to - j);
    if (to < kVec) return load_first(row + j, n, fill);
    Raw8<T> r = load8(row + to - kVec);
#pragma unroll
    for (int by = 4; by; by /= 2)
        if ((kVec - n) & by) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) r.v[i] = i + by < kVec ? r.v[i + by] : fill;
        }
    return r;
}

template <typename T>
__device__ __forceinline__ void store_first(T *p, int n, const Raw8<T> &r)
{
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < n) p[i] = r.v[i];
}

// past the caches: for matrices that no cache holds until they are read, so that what others still read stays there
template <typename T>
__device__ __forceinline__ void store8_past(T *p, const Raw8<T> &r)
{
    typedef int words __attribute__((ext_vector_type(4), aligned(2)));
    const words *w = reinterpret_cast<const words *>(&r);
#pragma unroll
    for (int i = 0; i < (int)sizeof(r) / 16; ++i) __builtin_nontemporal_store(w[i], reinterpret_cast<words *>(p) + i);
}

// e4m3 (finite numbers up to 448, NaN), rounded to nearest, ties to even
template <bool PAST>
__device__ __forceinline__ void store8_e4m3(e4m3 *p, const float *v, int64_t n)
{
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
    if (n >= kVec) {
        typedef int words __attribute__((ext_vector_type(2), aligned(1)));
        const words both = {lo, hi};
        if (PAST) __builtin_nontemporal_store(both, reinterpret_cast<words *>(p));
        else *reinterpret_cast<words *>(p) = both;
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < n) p[i].bits = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
}

// whole numbers, rounded to nearest, ties to even; NaN: 0.  What is given lies within +-127.
template <bool PAST>
__device__ __forceinline__ void store8_whole(whole8 *p, const float *v, int64_t n)
{
    int both[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kVec; ++i) both[i / 4] |= ((v[i] == v[i] ? (int)rintf(v[i]) : 0) & 255) << (8 * (i & 3));
    if (n >= kVec) {
        typedef int words __attribute__((ext_vector_type(2), aligned(1)));
        const words w = {both[0], both[1]};
        if (PAST) __builtin_nontemporal_store(w, reinterpret_cast<words *>(p));
        else *reinterpret_cast<words *>(p) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (i < n) p[i].v = (int8_t)(both[i / 4] >> (8 * (i & 3)));
}

// rounded to nearest, ties to even; above the largest finite value of f16: infinity
template <typename T, bool PAST = false>
__device__ __forceinline__ void store8_of(T *p, const float *v, int64_t n)
{
    if constexpr (__is_same(T, whole8)) {
        store8_whole<PAST>(p, v, n);
    } else if constexpr (sizeof(T) == 1) {
        store8_e4m3<PAST>(p, v, n);
    } else {
        Raw8<T> r;
#pragma unroll
        for (int i = 0; i < kVec; ++i) r.v[i] = static_cast<T>(v[i]);
        if (n < kVec) store_first(p, (int)n, r);
        else if (PAST) store8_past(p, r);
        else store8(p, r);
    }
}

// ---------------------------------------------------------------- sums and maxima in 32 bits
template <int CTRL>
__device__ __forceinline__ float dpp_movef(float v)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}

__device__ __forceinline__ float read_lanef(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// over the 64 lanes of a wavefront, in a fixed order; every lane has the result
template <typename F>
__device__ __forceinline__ float wave_joinf(float v, F f)
{
    v = f(v, dpp_movef<0xB1>(v));
    v = f(v, dpp_movef<0x4E>(v));
    v = f(v, dpp_movef<0x141>(v));
    v = f(v, dpp_movef<0x140>(v));
    return f(f(read_lanef(v, 0), read_lanef(v, 16)), f(read_lanef(v, 32), read_lanef(v, 48)));
}
__device__ __forceinline__ float wave_sumf(float v)
{
    return wave_joinf(v, [](float a, float b) { return a + b; });
}
// NaN is left out, as fmaxf leaves it out
__device__ __forceinline__ float wave_maxf(float v)
{
    return wave_joinf(v, [](float a, float b) { return fmaxf(a, b); });
}

// the larger one, or NaN where there is one
__device__ __forceinline__ float max_or_nan(float a, float b) { return b > a || b != b ? b : a; }
// NAN_TOO: NaN is kept, otherwise left out
template <bool NAN_TOO>
__device__ __forceinline__ float larger(float a, float b)
{
    return NAN_TOO ? max_or_nan(a, b) : fmaxf(a, b);
}
template <bool NAN_TOO>
__device__ __forceinline__ float wave_top(float v)
{
    return wave_joinf(v, [](float a, float b) { return larger<NAN_TOO>(a, b); });
}

// in 32 or 64 bits
__device__ __forceinline__ float wave_sum_of(float v) { return wave_sumf(v); }
__device__ __forceinline__ double wave_sum_of(double v) { return wave_sum(v); }

// Largest workgroup of these kernels
constexpr int kMostWaves = 16;

// Sums of a and maxima of b over the workgroup, in a fixed order.  `room`: 2 * kMostWaves floats of LDS that nobody reads or writes at
// that time; after a call it may be used again behind one barrier.
template <bool NAN_TOO = false>
__device__ __forceinline__ void block_sum_max(float &a, float &b, float *room)
{
    const int waves = blockDim.x / kWave, wave = threadIdx.x / kWave;
    a = wave_sumf(a);
    b = wave_top<NAN_TOO>(b);
    if (waves == 1) return;
    if (threadIdx.x % kWave == 0) {
        room[wave] = a;
        room[kMostWaves + wave] = b;
    }
    __syncthreads();
    a = 0.f;
    b = room[kMostWaves];
    for (int w = 0; w < waves; ++w) {
        a += room[w];
        b = larger<NAN_TOO>(b, room[kMostWaves + w]);
    }
}

// Sums of a and b over the workgroup, in the same way.
__device__ __forceinline__ void block_sum_two(float &a, float &b, float *room)
{
    const int waves = blockDim.x / kWave, wave = threadIdx.x / kWave;
    a = wave_sumf(a);
    b = wave_sumf(b);
    if (waves == 1) return;
    if (threadIdx.x % kWave == 0) {
        room[wave] = a;
        room[kMostWaves + wave] = b;
    }
    __syncthreads();
    a = b = 0.f;
    for (int w = 0; w < waves; ++w) {
        a += room[w];
        b += room[kMostWaves + w];
    }
}

// The maximum over the workgroup.  `room`: kMostWaves floats.
template <bool NAN_TOO>
__device__ __forceinline__ float block_top(float a, float *room)
{
    const int waves = blockDim.x / kWave;
    a = wave_top<NAN_TOO>(a);
    if (waves == 1) return a;
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = a;
    __syncthreads();
    a = room[0];
    for (int w = 1; w < waves; ++w) a = larger<NAN_TOO>(a, room[w]);
    return a;
}

template <typename S>
__device__ __forceinline__ S block_sum_all(S a, S *room)
{
    const int waves = blockDim.x / kWave;
    a = wave_sum_of(a);
    if (waves == 1) return a;
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = a;
    __syncthreads();
    a = 0;
    for (int w = 0; w < waves; ++w) a += room[w];
    return a;
}

// ---------------------------------------------------------------- launches of many workgroups
// One dimension of a launch holds fewer than 2^32 threads: blocks are numbered over two.  Numbers from `blocks` on have no work.
inline dim3 block_grid(int64_t blocks)
{
    const int64_t x = blocks < (1 << 20) ? blocks : (1 << 20);
    return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}
__device__ __forceinline__ int64_t block_number() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// out_j = sum over `count` rows of shares [count][d], in a fixed order (head_norm.hip); a second matrix behind the first one goes to out2, where
// that is not NULL, and either may be left out
int column_sums(const float *shares, int64_t count, int64_t d, float *out, hipStream_t st, float *out2 = nullptr);

// ---------------------------------------------------------------- checks of arguments
// Rows that are read may lie anywhere, one on another too (ld 0: one row for all); rows that are written may not overlap.
inline bool rows_ok(int64_t rows, int64_t cols, int64_t ld, bool written) { return written ? rows <= 1 || ld >= cols : ld >= 0; }
// whether the last element's byte offset fits into 62 bits
inline bool extent_ok(int64_t rows, int64_t ld, int64_t cols) { return rows < 1 || (long double)(rows - 1) * (long double)ld + (long double)cols < 4.6e18L / 4; }

// `bytes` of a caller's work space, at 16 bytes
inline bool work_ok(const void *work, int64_t bytes, int64_t needed) { return needed == 0 || (work && bytes >= needed && ((uintptr_t)work & 15) == 0); }

// Whether an output is stored past the caches: above 32 MB, what the eight L2s hold together.  Norm of 16384 x 8192 in bf16 with its sum,
// output in 8 bits: 233 us through them, 195 us past them.
inline bool goes_past(int64_t rows, int64_t cols, int64_t bytes) { return (double)rows * (double)cols * (double)bytes > 32e6; }

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace tron
