// A step of a beam search over a softmax head's logits, and the states of the beams that go on.
//
// Row r = item * beams + beam holds z, score_r the beam's sum of log-probabilities so far:
//   lse_r = log sum_v exp z_rv,   c_rv = score_r + (z_rv - lse_r),
// and the K largest c of an item's beams * V are taken, ties to the lowest beam, then its largest z, then the lowest token.
//
// Bound by reading z, once.  Within a row c grows with z, so a row offers its K largest z whatever its lse will be.  A first launch
// reads the rows (or parts of them): every wavefront keeps a running maximum and sum a lane, and a list in LDS of what may be among the K
// largest.  A value enters the list only above the K-th largest seen so far, so that of n values some K log n are looked at more closely, and
// the others cost a conversion, a maximum and an exponential.  A second launch, a workgroup an item, joins sums and lists.  Keys are unique (the value's
// bits in order, then the column's complement), so lists may be filled in any order and the result is still the same.
//
// The sum is the more exact the more rows are compared by it: exponents are products with log2(e) in two parts, lanes' sums are joined in 64 bits,
// scores are compared in 64 bits.
//
// Measured: 64 items of 8 beams over 128000 bf16, 16 picks: 39.5 us the rows (118 MB that are read, 3.0 TB/s; the vector units are busy two thirds of the cycles), 6.5 us
// the joining; 2 layers of 129 x 128 bf16 states of 512 rows 9.6 us (50 MB, 5.2 TB/s).  One item of 4 beams over 32000 f32: 8 + 4 us.
#include "head_util.h"

namespace tron {
namespace {

constexpr int kMostPicks = 64;       // one a lane
constexpr int kMostBeams = 64;
constexpr int kAhead = 4;            // chunks of eight columns of a lane under way
constexpr int kTurn = kAhead * kWave * kVec;   // columns of a wavefront's turn
constexpr int kSlack = 128;          // entries of a list beyond which it is cut to the K largest
// Lanes whose columns of a turn are looked at more closely at once.  Beside other wavefronts' first turns few pass in any; a wavefront alone has all of the K.
template <int WAVES>
constexpr int kLooked = WAVES == 1 ? 16 : 4;
template <int WAVES>
constexpr int kList = kSlack + kLooked<WAVES> * kAhead * kVec;   // behind kSlack entries, all that is looked at at once has its place
constexpr int kMostParts = 64;       // of a row, one a lane
constexpr int kMostOffers = kMostBeams * kMostPicks;   // of an item's rows' parts together

typedef unsigned long long key_t64;

struct BeamArgs {
    const void *z;
    int64_t ldz;
    const float *score;
    const uint8_t *ended;
    int64_t batch, V, end, per;   // per: columns of a part
    int beams, picks, parts;
    double *part_sum;      // [rows][parts]
    key_t64 *part_key;     // [rows][parts][picks]; 0: none
    float *part_max;       // [rows][parts]
    float *next_score;
    int32_t *parent, *token;
    uint8_t *next_ended;
};

// Bits whose order as whole numbers is that of the values; no number's are 0
__device__ __forceinline__ uint32_t in_order(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);   // -0 is 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ key_t64 in_order(double v)
{
    const key_t64 b = (key_t64)__double_as_longlong(v + 0.0);
    return b >> 63 ? ~b : b | (key_t64)1 << 63;
}
__device__ __forceinline__ double of_order(key_t64 o) { return __longlong_as_double((long long)(o >> 63 ? o & ~((key_t64)1 << 63) : ~o)); }
constexpr uint32_t kOrderOfNothing = 0x007fffffu;   // of -inf

__device__ __forceinline__ key_t64 key_of(float v, int64_t column) { return (key_t64)in_order(v) << 32 | (uint32_t)~(uint32_t)column; }

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }   // what exponents are differences to: no -inf minus -inf
// exp(d) for d <= 0
__device__ __forceinline__ float exp_of(float d) { return exp2_(fmaf(d, 1.44269502f, d * 1.925963e-8f)); }

// The largest of three, one instruction: fmaxf first makes a quiet NaN of an argument that may be another one, as bits shifted to a float may (bf16: 46
// instructions for 32 columns, 12 so; 512 rows of 128000 with 16 picks, both launches on fresh logits, 48.6 us by fmaxf, 47.5 us so).  A NaN may hide the others here: its row has no candidates.
__device__ __forceinline__ float top3(float a, float b, float c)
{
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}

// whether a row is read: a beam that has ended, or has no finite score, offers nothing of its logits
__device__ __forceinline__ bool is_read(const BeamArgs &A, int64_t row) { return !(A.ended && A.ended[row]) && fabsf(A.score[row]) < INFINITY; }

__device__ __forceinline__ int lanes_before(uint64_t mask) { return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0)); }

// The largest number that K of the wavefront's words reach, N a lane, of those that take part (0 for fewer), or one that exactly K reach: bit by bit from
// the highest on to `last`
template <int N, typename F>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&word)[N], int K, int last, bool &exactly, F takes_part)
{
    uint32_t bound = 0;
    exactly = false;
#pragma unroll 1
    for (int b = 31; b >= last; --b) {
        const uint32_t trial = bound | 1u << b;
        int reach = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) reach += __popcll(__ballot(takes_part(i) && word[i] >= trial));
        if (reach >= K) bound = trial;
        if ((exactly = reach == K)) break;
    }
    return bound;
}

// The K largest of the first `count` keys of a wavefront's list, N a lane, go to its front, in no order; fewer are all kept.  Returns, in order, a value that
// they reach: 0 where there are fewer than K.  Keys are unique: the values' words decide, or among the same ones the columns'.  (Keys of 64 bits at once: 4096
// rows of 3000, 32 picks, 43 us.)
template <int N>
__device__ __forceinline__ uint32_t cut_to(key_t64 *list, int &count, int K, int lane)
{
    uint32_t high[N], low[N];
    wave_lds_fence();   // other lanes put keys here
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const key_t64 key = i * kWave + lane < count ? list[i * kWave + lane] : 0;
        high[i] = (uint32_t)(key >> 32);
        low[i] = (uint32_t)key;
    }
    if (count < K) return 0;
    bool exactly;
    const uint32_t bound = reached_by(high, K, 0, exactly, [](int) { return true; });
    uint32_t least = 0;   // of the low words beside the bound itself
    if (!exactly) {
        int above = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) above += __popcll(__ballot(high[i] > bound));
        least = reached_by(low, K - above, 0, exactly, [&](int i) { return high[i] == bound; });
    }
    count = 0;
    wave_lds_fence();   // all have read theirs
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool keep = high[i] && (high[i] > bound || (high[i] == bound && low[i] >= least));
        const uint64_t mask = __ballot(keep);
        if (keep) list[count + lanes_before(mask)] = (key_t64)high[i] << 32 | low[i];
        count += __popcll(mask);
    }
    wave_lds_fence();
    return bound;
}

// `count` is one of the wavefront's; the compiler keeps what it may not know to be such in a register of each lane, and branches by masks
template <int LIST>
__device__ __forceinline__ uint32_t cut(key_t64 *list, int &count, int K, int lane)
{
    const uint32_t bound = count <= kWave ? cut_to<1>(list, count, K, lane) : count <= 2 * kWave ? cut_to<2>(list, count, K, lane) : cut_to<LIST / kWave>(list, count, K, lane);
    count = __builtin_amdgcn_readfirstlane(count);
    return bound;
}

struct Running {
    float m = -INFINITY, s = 0.f;   // s = sum exp(z - m); m = -inf: nothing yet, or nothing but -inf
};

// What a wavefront knows of the K largest values of its workgroup's columns: K of those that its list, or another's, holds are `least` or more.
// `beyond`: K of its own, of earlier columns, are, so that a later value has to lie above.
struct Bound {
    float least = -INFINITY;
    bool beyond = false;
    __device__ __forceinline__ bool passes(float v) const { return beyond ? v > least : v >= least; }
    __device__ __forceinline__ void raise(uint32_t order, bool own)
    {
        const float v = order > kOrderOfNothing ? of_order(order) : -INFINITY;
        if (v > least) least = v, beyond = own;
        else if (v == least && own) beyond = true;
    }
};

// A turn's columns of a wavefront: eight neighbouring ones a lane, kAhead times
template <typename T>
struct Turn {
    Eight<T> e[kAhead];
    __device__ __forceinline__ void load(const T *z, int64_t j0, int64_t to, int lane)
    {
        if (j0 + kTurn <= to) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) e[u].set(load8(z + j0 + (u * kWave + lane) * kVec));
            return;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t j = j0 + (u * kWave + lane) * kVec;
            Raw8<T> r;
#pragma unroll
            for (int i = 0; i < kVec; ++i) r.v[i] = static_cast<T>(-INFINITY);
            if (j < to) r = load_row8(z, j, to, static_cast<T>(-INFINITY));
            e[u].set(r);
        }
    }
};

// A workgroup of WAVES wavefronts a part of a row: blockIdx.x the part, y and z the row
template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES *kWave, 4) void k_beam_offers(BeamArgs A)
{
    constexpr int kMine = kList<WAVES>;
    __shared__ key_t64 lists[WAVES][kMine];
    __shared__ __align__(16) uint32_t looked[WAVES][kLooked<WAVES>][kAhead * 2 * sizeof(T)];
    __shared__ uint32_t firsts[WAVES][kWave];   // the lanes' largest values of the first turns, in order
    __shared__ double sums[WAVES];
    __shared__ float tops[WAVES];
    __shared__ key_t64 join[WAVES > 1 ? WAVES * kWave : 1];
    __shared__ int joined;
    __shared__ uint32_t common;   // in order: what K of some wavefront's values reach
    const int64_t row = (int64_t)blockIdx.z * gridDim.y + blockIdx.y, part = blockIdx.x;
    if (row >= A.batch * A.beams || !is_read(A, row)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, K = A.picks;
    const int64_t from = part * A.per, to = from + A.per < A.V ? from + A.per : A.V;
    const T *z = static_cast<const T *>(A.z) + row * A.ldz;
    key_t64 *list = lists[wave];
    Running run;
    Bound bound;
    int count = 0;
    const int64_t begin = from + (int64_t)wave * kTurn;
    Turn<T> now;
    now.load(z, begin, to, lane);
    for (int64_t j0 = begin;;) {
        const int64_t next = j0 + WAVES * kTurn;
        Turn<T> ahead;
        if (next < to) ahead.load(z, next, to, lane);
        float most = -INFINITY;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float v[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = now.e[u].at(i);
            if (__is_same(T, __bf16)) most = top3(top3(most, v[0], v[1]), top3(v[2], v[3], v[4]), top3(v[5], v[6], v[7]));
            else most = fmaxf(most, fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7]))));
        }
        if (most > run.m) {
            run.s *= exp_of(run.m - most);   // 0 * exp(-inf) at first
            run.m = most;
        }
        const float base = base_of(run.m);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float s0 = exp_of(now.e[u].at(0) - base), s1 = exp_of(now.e[u].at(1) - base);
#pragma unroll
            for (int i = 2; i < kVec; i += 2) {
                s0 += exp_of(now.e[u].at(i) - base);
                s1 += exp_of(now.e[u].at(i + 1) - base);
            }
            run.s += s0 + s1;   // NaN from here on, where there is a NaN or +inf
        }
        uint32_t reached = 0;   // in order: what K values of this turn, or of earlier ones, reach
        if (j0 == begin) {
            // The workgroup's first turns: of the lanes' largest values the K-th largest is a bound that K values reach
            const uint32_t mine = j0 + (int64_t)lane * kVec < to ? in_order(most) : 0;
            uint32_t all[WAVES] = {mine};
            if (WAVES > 1) {
                firsts[wave][lane] = mine;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < WAVES; ++w) all[w] = firsts[w][lane];
            }
            bool exactly;
            reached = reached_by(all, K, 16, exactly, [](int) { return true; });   // sixteen bits of it are enough
            if (WAVES > 1) {
                if (threadIdx.x == 0) {
                    common = reached;
                    joined = 0;
                }
                __syncthreads();   // behind which `common` only rises
            }
            bound.raise(reached, false);
        } else if (WAVES > 1) {
            bound.raise(__builtin_amdgcn_readfirstlane(*(volatile uint32_t *)&common), false);
        }
        // Few lanes have a value that passes.  Four of them at a time put theirs into LDS, and every lane takes two neighbouring ones of those.
        uint64_t some = __ballot(bound.passes(most));
        while (some) {
            if (count > kSlack) {
                const uint32_t order = cut<kMine>(list, count, K, lane);
                bound.raise(order, false);   // lower columns of this turn may still come
                if (WAVES > 1 && lane == 0) atomicMax(&common, order);
                reached = reached > order ? reached : order;
            }
            // words of a lane's columns; lanes that read one lane's, and the columns that each of these takes
            constexpr int kWords = kAhead * 2 * sizeof(T), kAcross = kWave / kLooked<WAVES>, kEach = kAhead * kVec / kAcross, kTaken = kWords / kAcross;
            static_assert(kEach <= kVec && kVec % kEach == 0, "neighbouring columns");
            uint64_t rest = some;
            int from_lane = 0;
            wave_lds_fence();   // the ones before have been read
#pragma unroll
            for (int q = 0; q < kLooked<WAVES>; ++q) {
                const int l = rest ? __builtin_ctzll(rest) : 0;
                if (lane / kAcross == q) from_lane = rest ? l : -1;
                if (rest && lane == l) {
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
#pragma unroll
                        for (int i = 0; i < kWords / kAhead; ++i) looked[wave][q][u * (kWords / kAhead) + i] = now.e[u].w[i];
                }
                rest &= rest - 1;
            }
            some = rest;
            wave_lds_fence();
            const int mine = lane % kAcross * kEach;   // first one of its columns
            Eight<T> w;
#pragma unroll
            for (int i = 0; i < kTaken; ++i) w.w[i] = looked[wave][lane / kAcross][lane % kAcross * kTaken + i];
            const int64_t j = j0 + (mine / kVec * kWave + from_lane) * kVec + mine % kVec;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const float v = w.at(i);
                const bool in = from_lane >= 0 && bound.passes(v) && j + i < to;
                const uint64_t mask = __ballot(in);
                if (in) list[count + lanes_before(mask)] = key_of(v, j + i);
                count = __builtin_amdgcn_readfirstlane(count + __popcll(mask));
            }
        }
        // later turns' columns are higher ones, and higher than those of all first turns, so their values have to lie above
        if (reached) bound.raise(reached, true);
        if (next >= to) break;
        now = ahead;
        j0 = next;
    }
    float all_most = wave_maxf(run.m);
    double total = wave_sum((double)run.s * (double)exp_of(run.m - base_of(all_most)));
    wave_lds_fence();   // the list is read from here on
    if (WAVES > 1) {
        // one list of the wavefronts' keys that may be among the K, 64 of each at most
        if (count > kWave) cut<kMine>(list, count, K, lane);
        if (lane == 0) {
            tops[wave] = all_most;
            sums[wave] = total;
        }
        const key_t64 key = lane < count ? list[lane] : 0;
        const bool in = key && (uint32_t)(key >> 32) >= *(volatile uint32_t *)&common;
        const uint64_t mask = __ballot(in);
        int place = 0;
        if (lane == 0) place = atomicAdd(&joined, __popcll(mask));
        if (in) join[__builtin_amdgcn_readfirstlane(place) + lanes_before(mask)] = key;
        __syncthreads();
        if (wave) return;
        const float m = lane < WAVES ? tops[lane % WAVES] : -INFINITY;
        all_most = wave_maxf(m);
        total = wave_sum(lane < WAVES ? sums[lane % WAVES] * exp((double)m - (double)base_of(all_most)) : 0.0);
        list = join;
        const int keys = __builtin_amdgcn_readfirstlane(joined);
        count = keys < kMine ? keys : kMine;
        for (int read = count; read < keys;) {   // as many as a list holds at a time
            cut<kMine>(list, count, K, lane);
            const int more = keys - read < kMine - count ? keys - read : kMine - count;
            for (int i = lane; i < more; i += kWave) {   // from later places to earlier ones
                const key_t64 key = join[read + i];
                wave_lds_fence();
                list[count + i] = key;
            }
            count += more;
            read += more;
        }
    }
    if (count > K) cut<kMine>(list, count, K, lane);
    const int64_t at = row * A.parts + part;
    if (lane < K) A.part_key[at * K + lane] = lane < count ? list[lane] : 0;
    if (lane == 0) {
        A.part_max[at] = all_most;
        A.part_sum[at] = total;
    }
}

// ------------------------------------------------------------------ joining
constexpr int kPickThreads = 256;
constexpr int kRanked = kPickThreads;   // offers that are ranked, one a thread

// Offers of an item: score in 64 bits, in order (0: none), beam, z, in order (0 where it does not count), and token.  The better one of two has the higher score, then
// the lower beam, the higher z and the lower token: a score of large size takes the differences of its beam's z, and they still decide.
struct Offers {
    key_t64 *order;
    uint32_t *z, *token;
    int of_beam;   // offers a beam
    // digits of eight bits, the first ones of the score, the higher the better
    static constexpr int kDigits = 17;
    __device__ __forceinline__ unsigned digit(int e, int d) const
    {
        return (d < 8 ? (unsigned)(order[e] >> (56 - 8 * d)) : d == 8 ? ~(unsigned)(e / of_beam) : d < 13 ? z[e] >> (96 - 8 * d) : ~token[e] >> (128 - 8 * d)) & 255u;
    }
};
constexpr int kOfferBytes = 16;

typedef uint32_t words4 __attribute__((ext_vector_type(4)));

// count += a > b, the last word, of a number's lowest bits, first: the borrow of b - a.  (Comparisons make two of each word, and of 64 bits take four times as long: 144
// offers were ranked in 9 us of a launch.)
__device__ __forceinline__ void count_larger(int &count, const words4 &a, uint32_t a_last, const words4 &b, uint32_t b_last)
{
    uint32_t difference;
    asm("v_sub_co_u32_e32 %0, vcc, %2, %3\n\t"
        "v_subb_co_u32_e32 %0, vcc, %4, %5, vcc\n\t"
        "v_subb_co_u32_e32 %0, vcc, %6, %7, vcc\n\t"
        "v_subb_co_u32_e32 %0, vcc, %8, %9, vcc\n\t"
        "v_subb_co_u32_e32 %0, vcc, %10, %11, vcc\n\t"
        "v_addc_co_u32_e32 %1, vcc, 0, %1, vcc"
        : "=&v"(difference), "+v"(count)
        : "v"(b_last), "v"(a_last), "v"(b[0]), "v"(a[0]), "v"(b[1]), "v"(a[1]), "v"(b[2]), "v"(a[2]), "v"(b[3]), "v"(a[3])
        : "vcc");
}

// How many of `highs`, of one a thread, are larger and how many the same
__device__ __forceinline__ void compare_high(const uint32_t *highs, uint32_t high, int &larger, int &same)
{
    for (int i = 0; i < kPickThreads; i += 8) {
        const words4 a = *reinterpret_cast<const words4 *>(highs + i), b = *reinterpret_cast<const words4 *>(highs + i + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            larger += (a[k] > high) + (b[k] > high);
            same += (a[k] == high) + (b[k] == high);
        }
    }
}

enum { LIVE = 0, OVER, DEAD };   // a beam whose logits make its offers, one that has ended, one of which nothing is possible

// A workgroup an item
__global__ __launch_bounds__(kPickThreads) void k_beam_pick(BeamArgs A)
{
    extern __shared__ __align__(16) key_t64 room[];
    __shared__ double lse[kMostBeams];
    __shared__ int kind[kMostBeams];
    __shared__ bool had_ended[kMostBeams];   // as next_ended may be ended
    __shared__ unsigned digits[256];
    __shared__ uint32_t bound;
    __shared__ int found[2], survivors, left, chosen[kRanked];
    __shared__ __align__(16) uint32_t highs[kPickThreads];   // of the scores' bits
    __shared__ words4 keys[kRanked + 32];                    // score, beam and z as one number, the higher the better; 0 behind the last one
    __shared__ __align__(16) uint32_t lasts[kRanked + 32];   // and its last word, of the token
    const int64_t item = block_number();
    if (item >= A.batch) return;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, K = A.picks;
    const int of_beam = A.parts * K, count = A.beams * of_beam;
    const Offers O{room, reinterpret_cast<uint32_t *>(room + count), reinterpret_cast<uint32_t *>(room + count) + count, of_beam};
    const int64_t row0 = item * A.beams;
    const key_t64 early = threadIdx.x < count ? A.part_key[row0 * of_beam + threadIdx.x] : 0;   // under way while the sums are joined
    // a beam's parts lie in neighbouring lanes, a power of two of them
    int lanes = 1;
    while (lanes < A.parts) lanes *= 2;
    for (int first = 0; first < A.beams; first += kPickThreads / lanes) {
        const int b = first + (int)threadIdx.x / lanes, part = threadIdx.x % lanes;
        const bool beam = b < A.beams, there = beam && part < A.parts;
        const int64_t row = row0 + (beam ? b : 0);
        const float score = A.score[row];
        const float m = there ? A.part_max[row * A.parts + part] : -INFINITY;
        const double s = there ? A.part_sum[row * A.parts + part] : 0.0;
        float most = m;
        for (int by = 1; by < lanes; by *= 2) most = fmaxf(most, __shfl_xor(most, by));
        double total = there ? s * exp((double)m - (double)base_of(most)) : 0.0;
        for (int by = 1; by < lanes; by *= 2) total += __shfl_xor(total, by);
        if (beam && part == 0) {
            const bool possible = total > 0.0 && total < INFINITY;   // not: nothing but -inf; a NaN or +inf
            kind[b] = !(fabsf(score) < INFINITY) ? DEAD : A.ended && A.ended[row] ? OVER : possible ? LIVE : DEAD;
            lse[b] = (double)most + log(total);
            had_ended[b] = A.ended && A.ended[row];
        }
    }
    if (threadIdx.x == 0) {
        survivors = left = 0;
        bound = 0;
    }
    __syncthreads();
    const int64_t listed = A.V < K ? A.V : K;
    for (int e = threadIdx.x; e < count; e += kPickThreads) {
        const int b = e / of_beam, i = e - b * of_beam;
        const int64_t row = item * A.beams + b;
        const bool live = kind[b] == LIVE, over = kind[b] == OVER;
        // One condition after the other.  Of a choice of three in one the compiler makes a switch, and of its default, which lanes of two branches reach (kinds below and
        // above the ones named), ROCm 7.2 sets the token in one branch alone: the optimized intermediate code has the value for all, the machine code not for
        // kind 2, also where this loop is compiled by itself.  There is no switch in this file's intermediate code.
        key_t64 key = 1;
        if (live) key = e == (int)threadIdx.x ? early : A.part_key[row * of_beam + i];
        const uint32_t other = over ? i == 0 ? (uint32_t)A.end : (uint32_t)(i - (i <= A.end)) : (uint32_t)i;   // columns in order, behind `end` where it is first
        const uint32_t token = live ? ~(uint32_t)key : other;
        const bool there = live ? key != 0 : i < listed;
        const double score = A.score[row], logit = of_order((uint32_t)(key >> 32));
        const double c = live ? score + (logit - lse[b]) : over && i == 0 ? score : -INFINITY;
        O.order[e] = there ? in_order(c) : 0;
        O.z[e] = live ? (uint32_t)(key >> 32) : 0;
        O.token[e] = token;
    }
    __syncthreads();
    static_assert(kMostOffers <= 32 * kPickThreads, "one bit an offer of a thread");
    const int each = (count + kPickThreads - 1) / kPickThreads;
    unsigned taken = 0;
    key_t64 top = 0;
#pragma unroll 1
    for (int i = 0; i < each; ++i) {
        const int e = i * kPickThreads + threadIdx.x;
        const key_t64 order = e < count ? O.order[e] : 0;
        taken |= (order != 0) << i;
        top = order > top ? order : top;
    }
    if (count > kRanked) {
        // Of the threads' best scores the K-th best is a bound that K offers reach; those that do are nearly always few enough
        const uint32_t high = (uint32_t)(top >> 32);
        highs[threadIdx.x] = high;
        __syncthreads();
        int better = 0, alike = 0;
        compare_high(highs, high, better, alike);
        if (high && better < K && better + alike >= K) bound = high;
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < each; ++i)
            if (taken >> i & 1 && (uint32_t)(O.order[i * kPickThreads + threadIdx.x] >> 32) < bound) taken &= ~(1u << i);
        if (taken) atomicAdd(&left, __popc(taken));
        __syncthreads();
    }
    if (left > kRanked) {
        // Digit by digit: who has a higher digit than the K-th best is chosen, who has the same is looked at further, until what is left fits
        unsigned under = taken;
        taken = 0;
        int need = K, have = 0;
#pragma unroll 1
        for (int d = 0; d < Offers::kDigits; ++d) {
            digits[threadIdx.x] = 0;
            __syncthreads();
#pragma unroll 1
            for (int i = 0; i < each; ++i)
                if (under >> i & 1) atomicAdd(&digits[O.digit(i * kPickThreads + threadIdx.x, d)], 1u);
            __syncthreads();
            if (wave == 0) {
                // the digit at which counts from the highest one on reach `need`: lane 0 has the four highest
                int mine[4], own = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) own += mine[q] = (int)digits[255 - 4 * lane - q];
                int before = wave_scan_add(own) - own;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (before < need && before + mine[q] >= need) {
                        found[0] = 255 - 4 * lane - q;
                        found[1] = before;
                    }
                    before += mine[q];
                }
            }
            __syncthreads();
            const unsigned at = (unsigned)found[0];
            const int same = (int)digits[at];
            need -= found[1];
            have += found[1];
#pragma unroll 1
            for (int i = 0; i < each; ++i)
                if (under >> i & 1) {
                    const unsigned mine = O.digit(i * kPickThreads + threadIdx.x, d);
                    if (mine > at) taken |= 1u << i;
                    if (mine != at) under &= ~(1u << i);
                }
            if (have + same <= kRanked) break;
            __syncthreads();
        }
        taken |= under;
    }
    {
        const int mine = __popc(taken), scanned = wave_scan_add(mine);
        int at = 0;
        if (lane == kWave - 1) at = atomicAdd(&survivors, scanned);
        at = __builtin_amdgcn_readlane(at, kWave - 1) + scanned - mine;
        for (unsigned rest = taken; rest; rest &= rest - 1) chosen[at++] = __builtin_ctz(rest) * kPickThreads + threadIdx.x;
    }
    __syncthreads();
    const int n = survivors;
    for (int i = threadIdx.x; i < kRanked + 32; i += kPickThreads) {
        words4 key = {0, 0, 0, 0};
        uint32_t last = 0;
        if (i < n) {
            const int e = chosen[i];
            const key_t64 order = O.order[e];
            key = words4{O.z[e], ~(uint32_t)(e / of_beam), (uint32_t)order, (uint32_t)(order >> 32)};
            last = ~O.token[e];
        }
        keys[i] = key;
        lasts[i] = last;
    }
    __syncthreads();
    // one, two or four threads an offer
    const int share = n <= kRanked / 4 ? 4 : n <= kRanked / 2 ? 2 : 1, mine = threadIdx.x / share;
    const words4 own = keys[mine];
    const uint32_t own_last = lasts[mine];
    int rank = 0;
    if (mine < n) {
        const int some = ((n + share - 1) / share + 7) / 8 * 8, first = threadIdx.x % share * some;   // eights: share * some <= n + 32
        for (int i = first; i < first + some; i += 8) {
            words4 other[8], last[2];
#pragma unroll
            for (int k = 0; k < 8; ++k) other[k] = keys[i + k];
#pragma unroll
            for (int k = 0; k < 2; ++k) last[k] = *reinterpret_cast<const words4 *>(lasts + i + 4 * k);
#pragma unroll
            for (int k = 0; k < 8; ++k) count_larger(rank, other[k], last[k / 4][k % 4], own, own_last);
        }
    }
    if (share > 1) rank += __shfl_xor(rank, 1);
    if (share > 2) rank += __shfl_xor(rank, 2);
    if (mine >= n || threadIdx.x % share || rank >= K) return;
    const int e = chosen[mine];
    const key_t64 order = (key_t64)own[3] << 32 | own[2];
    const int b = e / of_beam;
    const int64_t out = item * K + rank, row = item * A.beams + b;
    const uint32_t token = O.token[e];
    A.next_score[out] = (float)of_order(order);
    A.parent[out] = (int32_t)row;
    A.token[out] = (int32_t)token;
    if (A.next_ended) A.next_ended[out] = had_ended[b] || (int64_t)token == A.end;
}

// ------------------------------------------------------------------ states
struct ReorderArgs {
    const int32_t *rows, *lengths;
    const char *src;
    char *dst;
    int64_t ld, per, count, rows_in, src_layer, src_row, dst_layer, dst_row, positions, step, pieces;   // strides in bytes
};

constexpr int kPiece = 16 * 1024;   // bytes that a workgroup copies, four loads a thread under way

// Bound by memory: a workgroup copies a piece of a row; blockIdx.z the layer
__global__ __launch_bounds__(kBlock) void k_beam_reorder(ReorderArgs A)
{
    const int64_t block = block_number(), i = block / A.pieces, piece = block - i * A.pieces;
    if (i >= A.count) return;
    const int64_t from = A.rows[i / A.per * A.ld + i % A.per];
    if (from < 0 || from >= A.rows_in) return;
    int64_t n = A.positions;
    if (A.lengths) {
        const int64_t l = A.lengths[from];
        n = l < 0 ? 0 : l < n ? l : n;
    }
    const int64_t bytes = n * A.step, at = piece * kPiece;
    if (at >= bytes) return;
    const char *src = A.src + blockIdx.z * A.src_layer + from * A.src_row + at;
    char *dst = A.dst + blockIdx.z * A.dst_layer + i * A.dst_row + at;
    const int left = (int)(bytes - at < kPiece ? bytes - at : kPiece);
    constexpr int kLoads = kPiece / (kBlock * 16);
    typedef int words __attribute__((ext_vector_type(4), aligned(1)));
    words v[kLoads];
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int b = (q * kBlock + threadIdx.x) * 16;
        if (b + 16 <= left) v[q] = *reinterpret_cast<const words *>(src + b);
    }
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int b = (q * kBlock + threadIdx.x) * 16;
        if (b + 16 <= left) *reinterpret_cast<words *>(dst + b) = v[q];
    }
    // the rest of a row
    const int rest = left % 16;
    if ((int)threadIdx.x < rest) dst[left - rest + threadIdx.x] = src[left - rest + threadIdx.x];
}

// ------------------------------------------------------------------ host
struct Split {
    int waves, parts;
    int64_t per;
};

// Wavefronts a workgroup by the row's length, so that each has two turns or more where it can; parts of a row where there are fewer rows than 512, which are
// resident at once.  us of both launches, 8 beams, 16 picks, fresh logits.
//   By eight, four and one wavefronts: 512 rows of 128000 bf16 47, 62, 197; 64 rows 26, 26, 62; 512 of 32000 f32 28.5, 30, 77; 2048 of 32000 bf16 65, 52, 96; 2048 of 6000
//   49, 29, 34.  Long rows of few items want eight; many shorter rows would do better by four.
//   Whole rows, and in parts by the rule (or, from 512 rows on, in two): 128000 bf16 64 rows 32, 26; 256 rows 35, 37; 304 rows 42, 46; 400 rows 44, 54; 512 rows 47, 56; 520 rows 58,
//   61; 768 rows 68, 74; 1024 rows 77, 92; 2048 rows 133, 161.  32000 f32 64 rows 18.6, 20; 256 rows 22, 26; 400 rows 27, 34; 512 rows 28.5, 36; 768 rows 40, 47.  Parts gain where
//   rows are long and few; from 256 to 511 rows, and of 32000 columns, whole rows would be faster by 5 to 25%.
Split split_of(int64_t rows, int64_t beams, int64_t V, int64_t picks)
{
    const int64_t turns = ceil_div(V, kTurn);
    Split S{turns >= 16 ? 8 : turns >= 4 ? 4 : 1, 1, V};
    const int64_t most = std::min<int64_t>({kMostParts, kMostOffers / (beams * picks), ceil_div(turns, S.waves)});
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(most, ceil_div(512, rows)));
    S.per = ceil_div(turns, parts) * kTurn;
    S.parts = (int)ceil_div(V, S.per);
    return S;
}

bool beam_sizes_ok(int64_t batch, int64_t beams, int64_t V, int64_t picks)
{
    return batch >= 0 && beams >= 1 && beams <= kMostBeams && V >= 1 && V < INT32_MAX - 64 && picks >= 1 && picks <= kMostPicks && picks <= beams * V &&
           batch <= INT32_MAX / kMostBeams;
}

template <typename T>
void launch_offers(const BeamArgs &A, int waves, hipStream_t st)
{
    const int64_t rows = A.batch * A.beams, y = std::min<int64_t>(rows, 65535);
    const dim3 grid((unsigned)A.parts, (unsigned)y, (unsigned)ceil_div(rows, y));
    if (waves == 1) k_beam_offers<T, 1><<<grid, kWave, 0, st>>>(A);
    else if (waves == 4) k_beam_offers<T, 4><<<grid, 4 * kWave, 0, st>>>(A);
    else k_beam_offers<T, 8><<<grid, 8 * kWave, 0, st>>>(A);
}

struct Range {
    const void *p;   // or NULL: nothing
    int64_t bytes;
};
bool meet(const Range &a, const Range &b)
{
    return a.p && b.p && static_cast<const char *>(a.p) < static_cast<const char *>(b.p) + b.bytes && static_cast<const char *>(b.p) < static_cast<const char *>(a.p) + a.bytes;
}

// whether `layers` ranges of a_bytes that lie a_layer apart, and the same of b, have no byte in common: one behind the other, or side by side in each layer
bool apart(int64_t layers, const char *a, int64_t a_layer, int64_t a_bytes, const char *b, int64_t b_layer, int64_t b_bytes)
{
    if (a + (layers - 1) * a_layer + a_bytes <= b || b + (layers - 1) * b_layer + b_bytes <= a) return true;
    if (a_layer != b_layer || a_layer == 0) return false;
    const int64_t behind = ((b - a) % a_layer + a_layer) % a_layer;
    return behind >= a_bytes && behind + b_bytes <= a_layer;
}

}  // namespace
}  // namespace tron

using namespace tron;

extern "C" {

int64_t tron_beam_select_work(int64_t batch, int64_t beams, int64_t V, int64_t picks)
{
    if (!beam_sizes_ok(batch, beams, V, picks) || batch == 0) return 0;
    const int64_t parts = batch * beams * split_of(batch * beams, beams, V, picks).parts;
    return ceil_div(parts * (picks * 8 + 8 + 4), 16) * 16;
}

int tron_beam_select(int64_t batch, int64_t beams, int64_t V, int type, const void *z, int64_t ldz, const float *score, const uint8_t *ended, int64_t end,
                     int64_t picks, float *next_score, int32_t *parent, int32_t *token, uint8_t *next_ended, void *work, int64_t work_bytes, void *hip_stream)
{
    if (!beam_sizes_ok(batch, beams, V, picks) || !type_is_float(type) || end < -1 || end >= V) {
        set_error("tron_beam_select: bad argument (need batch >= 0, 1 <= beams <= 64, 1 <= V < 2^31 - 64, 1 <= picks <= 64, picks <= beams V, batch < 2^25, "
                  "type f32, bf16 or f16, -1 <= end < V)");
        return TRON_EINVAL;
    }
    if (batch > 0 && (!z || !score || !next_score || !parent || !token || (ended && end < 0) || !rows_ok(batch * beams, V, ldz, false) || !extent_ok(batch * beams, ldz, V))) {
        set_error("tron_beam_select: bad argument (z, score, next_score, parent and token are needed, and an end where beams may have ended)");
        return TRON_EINVAL;
    }
    if (batch > 0 && !work_ok(work, work_bytes, tron_beam_select_work(batch, beams, V, picks))) {
        set_error("tron_beam_select: needs a work space of tron_beam_select_work(batch, beams, V, picks) bytes at a multiple of 16");
        return TRON_EINVAL;
    }
    // A workgroup writes an item's picks while others read their items' scores and flags: only where it writes over its own, and has read them, may they be the same
    const int64_t of = batch * beams, go_on = batch * picks;
    const Range in[3] = {{score, of * 4}, {ended, of}, {work, tron_beam_select_work(batch, beams, V, picks)}};
    const Range out[4] = {{next_score, go_on * 4}, {next_ended, go_on}, {parent, go_on * 4}, {token, go_on * 4}};
    for (int o = 0; o < 4; ++o) {
        bool over = false;
        for (int i = 0; i < 3; ++i) over = over || (meet(out[o], in[i]) && !(o == i && picks == beams && out[o].p == in[i].p));
        for (int p = 0; p < o; ++p) over = over || meet(out[o], out[p]);
        if (over) {
            set_error("tron_beam_select: next_score, parent, token and next_ended may overlap neither score, ended, the work space nor each other, but next_score may be score and "
                      "next_ended ended where picks = beams");
            return TRON_EINVAL;
        }
    }
    TRON_TRY(check_device());
    if (batch == 0) return TRON_OK;
    const int64_t rows = batch * beams;
    const Split S = split_of(rows, beams, V, picks);
    double *part_sum = static_cast<double *>(work);
    key_t64 *part_key = reinterpret_cast<key_t64 *>(part_sum + rows * S.parts);
    float *part_max = reinterpret_cast<float *>(part_key + rows * S.parts * picks);
    const BeamArgs A{z, ldz, score, ended, batch, V, end, S.per, (int)beams, (int)picks, S.parts, part_sum, part_key, part_max, next_score, parent, token, next_ended};
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    if (type == TRON_TYPE_F32) launch_offers<float>(A, S.waves, st);
    else if (type == TRON_TYPE_BF16) launch_offers<__bf16>(A, S.waves, st);
    else launch_offers<_Float16>(A, S.waves, st);
    TRON_HIP(hipGetLastError());
    const int lds = (int)(beams * S.parts * picks) * kOfferBytes;   // 64 KB at most, beside 12 KB
    if (lds > 48 << 10) TRON_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(k_beam_pick), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    k_beam_pick<<<block_grid(batch), kPickThreads, lds, st>>>(A);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

int tron_beam_reorder(int64_t layers, int64_t batch, int64_t per, const int32_t *rows, int64_t ldrows, int64_t rows_in, const void *src, int64_t src_layer,
                      int64_t src_row, void *dst, int64_t dst_layer, int64_t dst_row, int64_t positions, int64_t step, const int32_t *lengths, void *hip_stream)
{
    if (layers < 0 || batch < 0 || per < 0 || rows_in < 0 || positions < 0 || step < 0 || layers > 65535 || rows_in > INT32_MAX || batch > INT32_MAX || per > INT32_MAX ||
        !extent_ok(positions, step, step)) {
        set_error("tron_beam_reorder: bad argument (sizes are not negative; layers < 65536, batch, per and rows_in < 2^31)");
        return TRON_EINVAL;
    }
    const int64_t count = batch * per, row_bytes = positions * step;
    if (layers == 0 || count == 0 || row_bytes == 0) return check_device();
    if (!rows || (rows_in && !src) || !dst || !rows_ok(batch, per, ldrows, false) || count > INT32_MAX || src_layer < 0 || src_row < 0 || !extent_ok(rows_in, src_row, row_bytes) ||
        !extent_ok(layers, src_layer, row_bytes) || !extent_ok(count, dst_row, row_bytes) || !extent_ok(layers, dst_layer, row_bytes)) {
        set_error("tron_beam_reorder: bad argument (rows, src and dst are needed; strides are not negative)");
        return TRON_EINVAL;
    }
    const int64_t in_layer = rows_in ? (rows_in - 1) * src_row + row_bytes : 0, out_layer = (count - 1) * dst_row + row_bytes;
    // rows in layers, or layers in rows
    const bool whole = (count == 1 || dst_row >= row_bytes) &&
                       (layers == 1 || dst_layer >= out_layer || (dst_layer >= row_bytes && (count == 1 || dst_row >= (layers - 1) * dst_layer + row_bytes)));
    if (!whole || !apart(layers, static_cast<const char *>(src), src_layer, in_layer, static_cast<const char *>(dst), dst_layer, out_layer)) {
        set_error("tron_beam_reorder: rows that are written may overlap neither each other nor src");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    if (rows_in == 0) return TRON_OK;
    const int64_t pieces = ceil_div(row_bytes, kPiece);
    const ReorderArgs A{rows, lengths, static_cast<const char *>(src), static_cast<char *>(dst), ldrows, per, count, rows_in, src_layer, src_row, dst_layer, dst_row,
                        positions, step, pieces};
    dim3 grid = block_grid(count * pieces);
    if (grid.y > 65535 || count > ((int64_t)1 << 36) / pieces) {
        set_error("tron_beam_reorder: more than 2^36 pieces of 16 KB a layer");
        return TRON_EINVAL;
    }
    grid.z = (unsigned)layers;
    k_beam_reorder<<<grid, kBlock, 0, reinterpret_cast<hipStream_t>(hip_stream)>>>(A);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

}  // extern "C"
