// Embeddings of tokens, and the gradient of their table.
//
//   y_i = scale row_scale[id_i] table[id_i];      dtable_v = scale sum_{i: id_i = v} dy_i  (+ dtable_v)
//
// The lookup is bound by reading the rows of the tokens and writing y.  The gradient is bound by reading dy once and writing the table; its
// sums are those of the rows of equal tokens in the order of their places, so that the same call gives the same bits.  Where a token's sum is cut depends on all ids: other
// tokens' number moves its places over the tiles' borders.
// Three launches: tokens are sorted (k_sort_tokens); the sorted places are cut into tiles of equal length, whatever tokens they hold, so that a frequent
// token is many tiles' work, and a wavefront sums a tile's rows over 512 columns and stores those tokens that lie in its tile alone
// (k_embed_sums, whose further workgroups fill the rows of tokens that are not there); the others' shares are joined (k_embed_join).
//
// Measured: 32768 tokens of 4096 bf16, a table of 128000 rows in f32: 15 us the sort, 402 us the sums and rows of zeros (2.35 GB, 5.8 TB/s), 10 us the joining,
// 461 us a call; 9001 of 511 f16, 50021 rows: 8 + 16 + 5 us; lookup of 8 rows of 4096 i8 3 us, of 32768 rows of 4096 bf16 94 us (4.7 TB/s).  Every workgroup of the sort reads all
// ids, so that many take it long: 32768, 262144 and 1000000 tokens of 1024 bf16 15 + 117 + 9, 170 + 238 + 14 and 701 + 557 + 16 us.
#include "head_util.h"

namespace tron {
namespace {

constexpr int kColumns = kWave * kVec;   // of a wavefront

template <typename T>
__device__ __forceinline__ void floats_of(float *v, const Raw8<T> &r)
{
    if constexpr (__is_same(T, e4m3)) {
        int w[2];
        __builtin_memcpy(w, &r, 8);
        v[0] = __builtin_amdgcn_cvt_f32_fp8(w[0], 0), v[1] = __builtin_amdgcn_cvt_f32_fp8(w[0], 1);
        v[2] = __builtin_amdgcn_cvt_f32_fp8(w[0], 2), v[3] = __builtin_amdgcn_cvt_f32_fp8(w[0], 3);
        v[4] = __builtin_amdgcn_cvt_f32_fp8(w[1], 0), v[5] = __builtin_amdgcn_cvt_f32_fp8(w[1], 1);
        v[6] = __builtin_amdgcn_cvt_f32_fp8(w[1], 2), v[7] = __builtin_amdgcn_cvt_f32_fp8(w[1], 3);
    } else if constexpr (__is_same(T, whole8)) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = (float)r.v[i].v;
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = static_cast<float>(r.v[i]);
    }
}

template <typename T>
__device__ __forceinline__ T zero_of()
{
    T z;
    __builtin_memset(&z, 0, sizeof(T));
    return z;
}

struct Ids {
    const void *p;
    bool wide;
    __device__ __forceinline__ int64_t at(int64_t i) const { return wide ? static_cast<const int64_t *>(p)[i] : (int64_t)static_cast<const int32_t *>(p)[i]; }
};

// ------------------------------------------------------------------ lookup
struct EmbedArgs {
    Ids ids;
    const void *table;
    const float *row_scale;
    void *y;
    int64_t m, d, V, ldtable, ldy, across;   // across: wavefronts a row
    float scale;
};

// A wavefront 512 columns of a row
template <typename T, typename O, bool PAST>
__global__ __launch_bounds__(kBlock) void k_embed(EmbedArgs A)
{
    const int64_t unit = block_number() * kWavesPerBlock + threadIdx.x / kWave, i = unit / A.across;
    const int64_t j = (unit - i * A.across) * kColumns + threadIdx.x % kWave * kVec;
    if (i >= A.m || j >= A.d) return;
    const int64_t id = A.ids.at(i);
    float v[kVec];
    if (id >= 0 && id < A.V) {
        floats_of(v, load_row8(static_cast<const T *>(A.table) + id * A.ldtable, j, A.d, zero_of<T>()));
        const float by = A.row_scale ? A.scale * A.row_scale[id] : A.scale;
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] *= by;
    } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = 0.f;
    }
    store8_of<O, PAST>(static_cast<O *>(A.y) + i * A.ldy + j, v, A.d - j);
}

// ------------------------------------------------------------------ sorted tokens
constexpr int kSortWaves = 16;
constexpr int kMostIds = 1024;    // of a workgroup: counts of each for every wavefront lie in LDS
constexpr int kMostFound = 256;   // of a wavefront's own tokens that LDS keeps between the counting and the placing

struct Sorted {
    int32_t *start, *stop; // [V]: first place of a token among the sorted ones, and the first behind it
    int32_t *count;        // places
    int32_t *key, *from;   // [m]: token and row of dy of a place
};

// Of 2^shift workgroups, number g has the tokens g, g + 2^shift, ... of the table, so that neighbouring ones, which vocabularies sort by frequency, are many
// workgroups' (32768 tokens of 128000 by a cubic law 28 us in ranges).  It reads all m ids, counts those of the workgroups before it and its own by
// wavefront; each wavefront has a contiguous range of the ids, and puts its places in their order behind those of the wavefronts before it.
template <typename Id>
__global__ __launch_bounds__(kSortWaves *kWave) void k_sort_tokens(const Id *ids, int64_t m, int64_t V, int shift, Sorted S)
{
    __shared__ int counts[kSortWaves][kMostIds];
    __shared__ int totals[2][kSortWaves];
    __shared__ uint8_t marks[kSortWaves][kMostIds];
    __shared__ uint64_t found[kSortWaves][kMostFound];   // token's number of the workgroup's, row of dy
    const int64_t group = block_number(), below = (int64_t)1 << shift;
    if (group >= below) return;
    const int here = (int)((V - group + below - 1) >> shift);   // tokens; at most kMostIds
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    if ((int)threadIdx.x < here) {
        for (int w = 0; w < kSortWaves; ++w) counts[w][threadIdx.x] = 0;
    }
    __syncthreads();
    // ids in 32 bits, the highest one for what is no token: V is less than 2^31
    constexpr uint32_t kNone = ~0u;
    auto token_at = [&](int64_t i, int64_t end) {   // without a branch, so that several are under way
        const Id id = ids[i < end ? i : end - 1];
        return i >= end || (sizeof(Id) == 8 && (uint64_t)id >> 32) ? kNone : (uint32_t)id;
    };
    const uint32_t tokens = (uint32_t)V, mask = (uint32_t)below - 1, mine_of = (uint32_t)group;
    const int64_t share = (m + kSortWaves * kWave - 1) / (kSortWaves * kWave) * kWave, begin = wave * share, end = begin + share < m ? begin + share : m;
    constexpr int kAhead = 8;
    int before = 0, own_here = 0;
    for (int64_t i0 = begin; i0 < end; i0 += kAhead * kWave) {
        uint32_t id[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) id[u] = token_at(i0 + u * kWave + lane, end);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t of = id[u] & mask;
            const uint64_t there = __ballot(id[u] < tokens), some = there & __ballot(of == mine_of);
            before += __popcll(there & __ballot(of < mine_of));   // of the wavefront
            if (!some) continue;
            // the first one's token at once, as it may be most of them
            const int k = (int)(id[u] >> shift), lead = __builtin_ctzll(some), token = __builtin_amdgcn_readlane(k, lead);
            const uint64_t same = some & __ballot(k == token);
            if (lane == lead) atomicAdd(&counts[wave][token], __popcll(same));
            if ((some & ~same) >> lane & 1) atomicAdd(&counts[wave][k], 1);
            const int at = own_here + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(some >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)some, 0));
            if ((some >> lane & 1) && at < kMostFound) found[wave][at] = (uint64_t)k << 32 | (uint32_t)(i0 + u * kWave + lane);
            own_here += __popcll(some);
        }
    }
    // places of the tokens: a thread a token
    __syncthreads();
    int mine = 0;
    const int k = threadIdx.x;
    if (k < here)
        for (int w = 0; w < kSortWaves; ++w) mine += counts[w][k];
    const int scanned = wave_scan_add(mine);
    if (lane == kWave - 1) {
        totals[0][wave] = before;
        totals[1][wave] = scanned;
    }
    __syncthreads();
    int place = scanned - mine;
    for (int w = 0; w < kSortWaves; ++w) {
        place += totals[0][w];
        if (w < wave) place += totals[1][w];
    }
    if (k < here) {
        const int64_t v = ((int64_t)k << shift) + group;
        S.start[v] = place;
        S.stop[v] = place + mine;
        if (group == below - 1 && k == here - 1) *S.count = place + mine;
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = counts[w][k];
            counts[w][k] = place;
            place += c;
        }
    }
    __syncthreads();
    // A wavefront of tokens, in the order of their rows
    auto place_tokens = [&](bool own, int k, int from) {
        uint64_t left = __ballot(own);
        if (!left) return;
        auto put = [&](int to) {
            S.key[to] = (int32_t)((uint32_t)k << shift | mine_of);
            S.from[to] = from;
        };
        // Every lane writes its number to its token's mark.  Whose number is not there has a token that is there twice: these go one token after the other,
        // in the order of their lanes; the others all at once
        volatile uint8_t *mark = marks[wave];
        if (own) mark[k] = (uint8_t)lane;
        wave_lds_fence();
        uint64_t twice = __ballot(own && mark[k] != lane);
        while (twice) {
            const int token = __builtin_amdgcn_readlane(k, __builtin_ctzll(twice));
            const uint64_t same = left & __ballot(k == token);
            const int at = counts[wave][token];
            if (same >> lane & 1) put(at + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(same >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)same, 0)));
            wave_lds_fence();   // all have read it
            if (lane == 0) counts[wave][token] = at + __popcll(same);
            wave_lds_fence();
            left &= ~same;
            twice &= ~same;
        }
        if (left >> lane & 1) {
            const int at = counts[wave][k];
            put(at);
            counts[wave][k] = at + 1;
        }
        wave_lds_fence();
    };
    if (own_here <= kMostFound) {
#pragma unroll 1
        for (int i = 0; i < own_here; i += kWave) {
            const bool own = i + lane < own_here;
            const uint64_t one = own ? found[wave][i + lane] : 0;
            place_tokens(own, (int)(one >> 32), (int)(uint32_t)one);
        }
        return;
    }
    // more than LDS keeps: they are read once more
#pragma unroll 1
    for (int64_t i0 = begin; i0 < end; i0 += kAhead * kWave) {
        uint32_t id[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) id[u] = token_at(i0 + u * kWave + lane, end);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) place_tokens(id[u] < tokens && (id[u] & mask) == mine_of, (int)(id[u] >> shift), (int)(i0 + u * kWave + lane));
    }
}

// ------------------------------------------------------------------ sums
struct EmbedGradArgs {
    Sorted S;
    const void *dy;
    void *dtable;
    float *shares;     // [tiles][2][d]: sums of a tile's first token, where its places begin before the tile, and of its last one, where they go on behind it
    int64_t m, d, V, lddy, ldtable, across, tiles, tile_units;
    int tile;          // places of a tile
    int rows_each;     // rows of the table that a workgroup looks at, 64 at most
    float scale;
    bool add;
};

template <typename O, bool PAST>
__device__ __forceinline__ void put_row(const EmbedGradArgs &A, int64_t v, int64_t j, const float *sum)
{
    O *row = static_cast<O *>(A.dtable) + v * A.ldtable;
    float out[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) out[e] = sum[e] * A.scale;
    if (A.add) {
        const Raw8<O> was = load_row8(row, j, A.d, static_cast<O>(0.f));
#pragma unroll
        for (int e = 0; e < kVec; ++e) out[e] += static_cast<float>(was.v[e]);
    }
    store8_of<O, PAST>(row + j, out, A.d - j);
}

// The first wavefronts have a tile's 512 columns each, the workgroups behind them rows_each rows of the table, one for each wavefront, pair or four of them by
// its length: some 16 KB, which lie side by side.  (A row a wavefront, which waits for its tokens' places first: rows of 69 f32 67 us for 256000, 36 us so; of
// 4096 f32 399 us for 128000, 363 us so.)
template <typename T, typename O, bool PAST>
__global__ __launch_bounds__(kBlock) void k_embed_sums(EmbedGradArgs A)
{
    const int64_t unit = block_number() * kWavesPerBlock + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lane = threadIdx.x % kWave;
    const int64_t filler = block_number() - (A.tile_units + kWavesPerBlock - 1) / kWavesPerBlock;
    if (filler >= 0) {
        constexpr int kEach = 16 / (int)sizeof(O);
        // wavefronts a row
        const int team = A.d <= kWave * kEach ? 1 : A.d <= 2 * kWave * kEach ? 2 : 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int64_t v0 = filler * A.rows_each, v = v0 + lane, step = team * kWave * kEach;
        const bool mine = lane % (kWavesPerBlock / team) == wave / team;
        uint64_t none = __ballot(mine && lane < A.rows_each && v < A.V && A.S.start[v] == A.S.stop[v]);
        for (; none; none &= none - 1) {
            // sixteen bytes a lane, side by side: whole lines from one instruction
            typedef int words __attribute__((ext_vector_type(4), aligned(2)));
            O *row = static_cast<O *>(A.dtable) + (v0 + __builtin_ctzll(none)) * A.ldtable;
            for (int64_t j = (wave % team * kWave + lane) * kEach; j < A.d; j += step) {
                if (j + kEach <= A.d) {
                    if (PAST) __builtin_nontemporal_store(words{0, 0, 0, 0}, reinterpret_cast<words *>(row + j));
                    else *reinterpret_cast<words *>(row + j) = words{0, 0, 0, 0};
                } else {
                    for (int64_t k = j; k < A.d; ++k) row[k] = static_cast<O>(0.f);
                }
            }
        }
        return;
    }
    if (unit >= A.tile_units) return;
    const int64_t t = unit / A.across, j = (unit - t * A.across) * kColumns + lane * kVec;
    // All that does not wait for the number of places is read beside it: what lies behind the last place is nobody's token, but in the work space.  The
    // places of the first 64, one a lane.
    const int64_t begin = t * A.tile, last = A.m - 1;
    auto clamped = [&](int64_t i) { return i < last ? i : last; };
    int key = A.S.key[clamped(begin + lane)], from = A.S.from[clamped(begin + lane)];
    const int key_before = A.S.key[begin > 0 ? begin - 1 : 0], key_end = A.S.key[clamped(begin + A.tile)], key_last = A.S.key[clamped(begin + A.tile - 1)];
    const int64_t count = *A.S.count, end = begin + A.tile < count ? begin + A.tile : count;
    if (begin >= count) return;
    const bool enters = begin > 0 && key_before == __builtin_amdgcn_readfirstlane(key), leaves = end < count && key_end == key_last;
    const bool there = j < A.d;
    const T *dy = static_cast<const T *>(A.dy);
    float sum[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) sum[e] = 0.f;
    bool first = enters;
    constexpr int kAhead = 8;
    for (int64_t c0 = begin; c0 < end; c0 += kWave) {
        // behind the tile's last place the token is -1, and the row that place's
        const int here = (int)(end - c0 < kWave ? end - c0 : kWave), at = lane < here ? lane : here - 1;
        if (c0 > begin) {
            key = A.S.key[c0 + at];
            from = A.S.from[c0 + at];
        } else {
            from = lane < here ? from : __builtin_amdgcn_readlane(from, here - 1);
        }
        const int after = c0 + kWave < end ? A.S.key[c0 + kWave] : -1;
        if (lane >= here) key = -1;
        for (int i0 = 0; i0 < here; i0 += kAhead) {
            Raw8<T> raw[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (there) raw[u] = load_row8(dy + (int64_t)__builtin_amdgcn_readlane(from, i0 + u) * A.lddy, j, A.d, static_cast<T>(0.f));
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = i0 + u;
                if (i >= here) break;
                float v[kVec];
                floats_of(v, raw[u]);
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum[e] += v[e];
                const int token = __builtin_amdgcn_readlane(key, i), next = i + 1 < kWave ? __builtin_amdgcn_readlane(key, (i + 1) % kWave) : after;
                if (next == token) continue;
                const bool last = next < 0;
                if (there) {
                    if (first) store8_of<float>(A.shares + 2 * t * A.d + j, sum, A.d - j);
                    else if (last && leaves) store8_of<float>(A.shares + (2 * t + 1) * A.d + j, sum, A.d - j);
                    else put_row<O, PAST>(A, token, j, sum);
                }
                first = false;
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum[e] = 0.f;
            }
        }
    }
}

// Tokens of several tiles: the workgroup of the tile in which one begins adds the shares of those that follow.  Its wavefronts have a range of them each, four
// loads ahead, and their sums are added in their order; a token that is everywhere is thousands of tiles' (65536 x 1024 f32, half of them one token: 524 us by
// one wavefront).
constexpr int kJoinWaves = 8;

template <typename O, bool PAST>
__global__ __launch_bounds__(kJoinWaves *kWave) void k_embed_join(EmbedGradArgs A)
{
    __shared__ float room[kJoinWaves - 1][kVec][kWave];
    const int64_t unit = block_number();
    if (unit >= A.tile_units) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int64_t t = unit / A.across, j = (unit - t * A.across) * kColumns + lane * kVec;
    const int64_t begin = t * A.tile, end = begin + A.tile;
    if (end >= A.m) return;
    const int v = A.S.key[end - 1], next = A.S.key[end];   // read beside the number of places, behind which there are no tokens
    if (end >= *A.S.count || next != v) return;
    const int64_t start = A.S.start[v], stop = A.S.stop[v];
    if (start < begin) return;
    const int64_t last = (stop - 1) / A.tile, each = (last - t + kJoinWaves - 1) / kJoinWaves;
    const int64_t from = t + 1 + wave * each, to = from + each < last + 1 ? from + each : last + 1;
    float sum[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) sum[e] = 0.f;
    if (j < A.d) {
        auto take = [&](const float *p, float *into) {
            const Raw8<float> r = load_row8(p, j, A.d, 0.f);
#pragma unroll
            for (int e = 0; e < kVec; ++e) into[e] = r.v[e];
        };
        if (wave == 0) take(A.shares + (2 * t + 1) * A.d, sum);
        int64_t u = from;
        for (; u + 3 < to; u += 4) {
            float four[4][kVec];
#pragma unroll
            for (int q = 0; q < 4; ++q) take(A.shares + 2 * (u + q) * A.d, four[q]);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum[e] += four[q][e];
        }
        for (; u < to; ++u) {
            float one[kVec];
            take(A.shares + 2 * u * A.d, one);
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] += one[e];
        }
    }
    if (wave) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) room[wave - 1][e][lane] = sum[e];
    }
    __syncthreads();
    if (wave || j >= A.d) return;
    for (int w = 0; w < kJoinWaves - 1; ++w)
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum[e] += room[w][e][lane];
    put_row<O, PAST>(A, v, j, sum);
}

// ------------------------------------------------------------------ host
template <typename T, typename O>
void embed_launch(const EmbedArgs &A, hipStream_t st)
{
    const dim3 grid = block_grid(ceil_div(A.m * A.across, kWavesPerBlock));
    if (goes_past(A.m, A.d, sizeof(O))) k_embed<T, O, true><<<grid, kBlock, 0, st>>>(A);
    else k_embed<T, O, false><<<grid, kBlock, 0, st>>>(A);
}

template <typename T>
void embed_typed(const EmbedArgs &A, int out, hipStream_t st)
{
    if (out == TRON_TYPE_F32) embed_launch<T, float>(A, st);
    else if (out == TRON_TYPE_BF16) embed_launch<T, __bf16>(A, st);
    else embed_launch<T, _Float16>(A, st);
}

// Places of a tile (65536 x 2048 bf16 over 200 tokens 101 us with these, 108 and 118 us with a half and a quarter): tiles of 512 columns for some 16 wavefronts a compute unit, of 8 places at least, one turn's loads, and of 512 at most
int tile_of_places(int64_t m, int64_t d)
{
    int tile = 8;
    while (tile < 512 && ceil_div(m, tile) * ceil_div(d, kColumns) > 4096) tile *= 2;
    return tile;
}

struct EmbedSpace {
    int64_t start, stop, count, key, from, shares, total;
};
EmbedSpace embed_space(int64_t m, int64_t d, int64_t V)
{
    EmbedSpace S;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t from = at;
        at += ceil_div(bytes, 256) * 256;
        return from;
    };
    S.start = take(V * 4);
    S.stop = take(V * 4);
    S.count = take(4);
    S.key = take(m * 4);
    S.from = take(m * 4);
    S.shares = take(ceil_div(m, tile_of_places(m, d)) * 2 * d * 4);
    S.total = at;
    return S;
}

template <typename T, typename O, bool PAST>
int embed_grad_launch(const EmbedGradArgs &A, hipStream_t st)
{
    const int64_t blocks = ceil_div(A.tile_units, kWavesPerBlock) + (A.add ? 0 : ceil_div(A.V, A.rows_each));
    if (blocks) k_embed_sums<T, O, PAST><<<block_grid(blocks), kBlock, 0, st>>>(A);
    TRON_HIP(hipGetLastError());
    if (A.tiles > 1) k_embed_join<O, PAST><<<block_grid(A.tile_units), kJoinWaves * kWave, 0, st>>>(A);
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

template <typename T, typename O>
int embed_grad_to(const EmbedGradArgs &A, hipStream_t st)
{
    return !A.add && goes_past(A.V, A.d, sizeof(O)) ? embed_grad_launch<T, O, true>(A, st) : embed_grad_launch<T, O, false>(A, st);
}

template <typename T>
int embed_grad_typed(const EmbedGradArgs &A, int out, hipStream_t st)
{
    return out == TRON_TYPE_F32 ? embed_grad_to<T, float>(A, st) : out == TRON_TYPE_BF16 ? embed_grad_to<T, __bf16>(A, st) : embed_grad_to<T, _Float16>(A, st);
}

bool embed_sizes_ok(int64_t m, int64_t d, int64_t V)
{
    return m >= 0 && m <= INT32_MAX && d >= 1 && V >= 1 && V < INT32_MAX - 64 && extent_ok(m, d, d) && extent_ok(V, d, d);
}

}  // namespace
}  // namespace tron

using namespace tron;

extern "C" {

int tron_embed(int64_t m, int64_t d, int64_t V, const void *ids, int id_bytes, int type, const void *table, int64_t ldtable, const float *row_scale, double scale,
               int out_type, void *y, int64_t ldy, void *hip_stream)
{
    const bool eight = type == TRON_TYPE_E4M3 || type == TRON_TYPE_I8;
    if (!embed_sizes_ok(m, d, V) || (id_bytes != 4 && id_bytes != 8) || (!eight && !type_is_float(type)) || !type_is_float(out_type)) {
        set_error("tron_embed: bad argument (need 0 <= m < 2^31, d >= 1, 1 <= V < 2^31 - 64, ids of 4 or 8 bytes, type f32, bf16, f16, e4m3 or i8, out_type f32, bf16 or f16)");
        return TRON_EINVAL;
    }
    if (m > 0 && (!ids || !table || !y || eight != (row_scale != nullptr) || !rows_ok(V, d, ldtable, false) || !rows_ok(m, d, ldy, true) || !extent_ok(V, ldtable, d) ||
                  !extent_ok(m, ldy, d))) {
        set_error("tron_embed: bad argument (ids, table and y are needed, tables of 8 bits, and they alone, have scales; rows that are written may not overlap)");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    if (m == 0) return TRON_OK;
    const EmbedArgs A{Ids{ids, id_bytes == 8}, table, row_scale, y, m, d, V, ldtable, ldy, ceil_div(d, kColumns), (float)scale};
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    switch (type) {
    case TRON_TYPE_F32: embed_typed<float>(A, out_type, st); break;
    case TRON_TYPE_BF16: embed_typed<__bf16>(A, out_type, st); break;
    case TRON_TYPE_F16: embed_typed<_Float16>(A, out_type, st); break;
    case TRON_TYPE_E4M3: embed_typed<e4m3>(A, out_type, st); break;
    default: embed_typed<whole8>(A, out_type, st);
    }
    TRON_HIP(hipGetLastError());
    return TRON_OK;
}

int64_t tron_embed_grad_work(int64_t m, int64_t d, int64_t V) { return embed_sizes_ok(m, d, V) ? embed_space(m, d, V).total : 0; }

int tron_embed_grad(int64_t m, int64_t d, int64_t V, const void *ids, int id_bytes, int type, const void *dy, int64_t lddy, double scale, int add, int out_type,
                    void *dtable, int64_t ldtable, void *work, int64_t work_bytes, void *hip_stream)
{
    if (!embed_sizes_ok(m, d, V) || (id_bytes != 4 && id_bytes != 8) || !type_is_float(type) || !type_is_float(out_type)) {
        set_error("tron_embed_grad: bad argument (need 0 <= m < 2^31, d >= 1, 1 <= V < 2^31 - 64, ids of 4 or 8 bytes, types f32, bf16 or f16)");
        return TRON_EINVAL;
    }
    if ((m > 0 && (!ids || !dy || !rows_ok(m, d, lddy, false) || !extent_ok(m, lddy, d))) || !dtable || !rows_ok(V, d, ldtable, true) || !extent_ok(V, ldtable, d)) {
        set_error("tron_embed_grad: bad argument (ids, dy and dtable are needed; rows that are written may not overlap)");
        return TRON_EINVAL;
    }
    if (!work_ok(work, work_bytes, tron_embed_grad_work(m, d, V))) {
        set_error("tron_embed_grad: needs a work space of tron_embed_grad_work(m, d, V) bytes at a multiple of 16");
        return TRON_EINVAL;
    }
    TRON_TRY(check_device());
    const EmbedSpace S = embed_space(m, d, V);
    char *w = static_cast<char *>(work);
    auto at = [&](int64_t offset) { return reinterpret_cast<int32_t *>(w + offset); };
    const Sorted sorted{at(S.start), at(S.stop), at(S.count), at(S.key), at(S.from)};
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    // a workgroup a compute unit, of whom each reads all ids, or as many as the tokens' counts need
    int shift = 0;
    while ((shift < 8 && (V >> shift) > 1) || (V >> shift) >= kMostIds) ++shift;
    const dim3 groups = block_grid((int64_t)1 << shift);
    if (id_bytes == 8) k_sort_tokens<<<groups, kSortWaves * kWave, 0, st>>>(static_cast<const int64_t *>(ids), m, V, shift, sorted);
    else k_sort_tokens<<<groups, kSortWaves * kWave, 0, st>>>(static_cast<const int32_t *>(ids), m, V, shift, sorted);
    TRON_HIP(hipGetLastError());
    const int tile = tile_of_places(m, d);
    const int64_t across = ceil_div(d, kColumns), tiles = ceil_div(m, tile);
    const int64_t row_bytes = d * (out_type == TRON_TYPE_F32 ? 4 : 2);
    const int rows_each = (int)std::min<int64_t>(std::max<int64_t>(16384 / row_bytes, 1), kWave);
    const EmbedGradArgs A{sorted, dy, dtable, reinterpret_cast<float *>(w + S.shares), m, d, V, lddy, ldtable, across, tiles, tiles * across, tile, rows_each, (float)scale, add != 0};
    return type == TRON_TYPE_F32 ? embed_grad_typed<float>(A, out_type, st)
           : type == TRON_TYPE_BF16 ? embed_grad_typed<__bf16>(A, out_type, st) : embed_grad_typed<_Float16>(A, out_type, st);
}

}  // extern "C"
