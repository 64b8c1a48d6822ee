// Rows of a table by token, and the table's gradient:
//     Y[i] = scale T[index[i]],   dT[v] (+)= scale sum_{i: index[i] = v} dY[i]
// A token outside [0, V) stands for a padded place: a row of zeros, no gradient.
//
// The gradient sorts the tokens (stable, so each sum's order is that of the batch), cuts the sorted list into
// pieces of equal length whatever the tokens' frequencies, and sums each piece's rows token by token.  A token that
// reaches over pieces leaves fp32 partial sums, joined in order: no floating-point atomics, the same bits every run.
#include "common.hpp"
#include "internal.hpp"

namespace cogdl {
namespace {

// VEC values (4 or 8, or one) of a row of any type.
template <typename T, int VEC>
__device__ __forceinline__ void read_row(const T *__restrict__ row, int at, float (&v)[VEC])
{
    if constexpr (VEC == 1 || (int)sizeof(T) * VEC == 16) {
        load_vec<T, VEC>(row, at, v);
    } else if constexpr (sizeof(T) == 4) {
        float h[2][4];
        load_vec<float, 4>(row, at, h[0]);
        load_vec<float, 4>(row, at + 4, h[1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = h[e / 4][e % 4];
    } else {
        const u32x2_u w = *reinterpret_cast<const u32x2_u *>(row + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t h = (e < 2 ? w.x : w.y) >> (16 * (e & 1)) & 0xffffu;
            v[e] = RowGather<T, 1, false>::widen1(h);
        }
    }
}

constexpr int kBlock = 256;

// ---------------------------------------------------------------- lookup
// Bound by memory: 1.5M rows of 256 bytes out of 2.4M 127 us (751 MB of HBM, 5.9 TB/s).  A thread takes a vector of
// 16 bytes, kLookupDeep at a time and all of them consecutive, so that ragged rows leave no lane idle.
struct LookupArgs {
    int64_t n;
    int32_t V, k;
    float scale;
    const void *table;
    const int32_t *index;
    void *out;
    int32_t vecs;                // 16-byte vectors of a row, the last moved back to the row's end
    int32_t rows;                // of a workgroup's turn
    uint32_t magic;              // ceil(2^32 / vecs)
};

constexpr int kLookupDeep = 4;   // vectors a thread has in flight

template <typename TI, typename TO, int VEC>
__global__ __launch_bounds__(kBlock) void k_lookup(LookupArgs a)
{
    const TI *__restrict__ table = static_cast<const TI *>(a.table);
    TO *__restrict__ out = static_cast<TO *>(a.out);
    for (int64_t r0 = (int64_t)blockIdx.x * a.rows; r0 < a.n; r0 += (int64_t)gridDim.x * a.rows) {
        const int rows = a.n - r0 < a.rows ? (int)(a.n - r0) : a.rows;
        const int items = rows * a.vecs;
        for (int i0 = threadIdx.x; i0 < items; i0 += kBlock * kLookupDeep) {
            int32_t token[kLookupDeep];
            int64_t row[kLookupDeep];
            int col[kLookupDeep];
            float v[kLookupDeep][VEC];
#pragma unroll
            for (int u = 0; u < kLookupDeep; ++u) {
                int i = i0 + u * kBlock;
                if (i >= items) i = i0;
                // (exact: i < 2048 where there is more than one row)
                const int r = rows == 1 ? 0 : a.vecs == 1 ? i : (int)__umulhi((uint32_t)i, a.magic);
                const int c = (i - r * a.vecs) * VEC;
                col[u] = c + VEC <= a.k ? c : a.k - VEC;
                row[u] = r0 + r;
                token[u] = a.index[row[u]];
            }
#pragma unroll
            for (int u = 0; u < kLookupDeep; ++u) {
                const bool in = (uint32_t)token[u] < (uint32_t)a.V;
                load_vec<TI, VEC>(table, (int64_t)(in ? token[u] : 0) * a.k + col[u], v[u]);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[u][e] = in ? v[u][e] * a.scale : 0.f;
            }
#pragma unroll
            for (int u = 0; u < kLookupDeep; ++u)
                if (i0 + u * kBlock < items) store_out<TO, VEC>(out, row[u] * a.k + col[u], v[u]);
        }
    }
}

// -------------------------------------------------------------- gradient
struct ScatterArgs {
    int64_t n;
    int32_t V, k;
    float scale;
    const int32_t *index;
    const void *dY;
    void *out;
    bool add;
    int32_t out_bytes;           // of an element
    uint32_t *keys;              // n: the tokens, V for those outside
    const uint32_t *sorted;      // n
    const uint32_t *order;       // n: their places
    float *slots;                // [2 x pieces][k]: partial sums of a piece's first token, begun before, and of its last
    int32_t *counts;             // [digit][tile] (lists of the middle lengths)
    int32_t tiles;
    int32_t per, pieces;
    int32_t lanes, log_lanes, vecs, chunks;
};

// The gradient of tokens that do not occur: thread `me` of `all`.
__device__ __forceinline__ void write_zeros(const ScatterArgs &a, int64_t me, int64_t all)
{
    const int64_t halves = (int64_t)a.V * a.k * (a.out_bytes / 2);
    uint16_t *__restrict__ out = static_cast<uint16_t *>(a.out);
    for (int64_t i = me * 8; i < halves; i += all * 8) {
        if (i + 8 <= halves) {
            *reinterpret_cast<u32x4_u *>(out + i) = u32x4_u{0u, 0u, 0u, 0u};
        } else {
            for (int64_t j = i; j < halves; ++j) out[j] = 0;
        }
    }
}

__device__ __forceinline__ uint32_t key_of(const ScatterArgs &a, int64_t i)
{
    const uint32_t t = (uint32_t)a.index[i];
    return t < (uint32_t)a.V ? t : (uint32_t)a.V;
}

__global__ __launch_bounds__(kBlock) void k_tokens(ScatterArgs a)
{
    const int64_t me = (int64_t)blockIdx.x * kBlock + threadIdx.x, all = (int64_t)gridDim.x * kBlock;
    for (int64_t i = me; i < a.n; i += all) {
        a.keys[i] = key_of(a, i);
    }
    if (!a.add) write_zeros(a, me, all);
}

// Short lists are sorted by one workgroup in LDS, while the others of its launch write the zeros: a stable radix sort
// of up to 8 bits a pass.  Each wavefront owns a run of the list and counts its digits, one scan over (digit,
// wavefront) gives every run's places, and a key's rank in its run is the count of lower lanes with its digit (a
// ballot a bit) behind the run's keys so far.  4096 tokens of 7 bits 8 us, by the sort for any length, four
// launches, 16.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kSortBits = 8, kSortEach = (kSortWaves << kSortBits) / kSortThreads;
constexpr int kShortList = 8192;

__global__ __launch_bounds__(kSortThreads) void k_sort_short(ScatterArgs a, int bits)
{
    __shared__ uint32_t keys[2][kShortList];
    __shared__ uint16_t vals[2][kShortList];
    __shared__ int counts[kSortWaves << kSortBits];
    __shared__ int sums[kSortWaves];
    if (blockIdx.x > 0) {
        if (!a.add) write_zeros(a, (int64_t)(blockIdx.x - 1) * kSortThreads + threadIdx.x, (int64_t)(gridDim.x - 1) * kSortThreads);
        return;
    }
    const int n = (int)a.n, lane = lane_id(), wave = threadIdx.x / kWave;
    for (int i = threadIdx.x; i < n; i += kSortThreads) {
        keys[0][i] = key_of(a, i);
        vals[0][i] = (uint16_t)i;
    }
    const int run = ((n + kSortWaves - 1) / kSortWaves + kWave - 1) / kWave * kWave;
    const int from = wave * run < n ? wave * run : n, to = from + run < n ? from + run : n;
    const int passes = (bits + kSortBits - 1) / kSortBits;
    int now = 0, shift = 0;
    for (int pass = 0; pass < passes; ++pass, now ^= 1) {
        const int dbits = (bits - shift + passes - pass - 1) / (passes - pass), mask = (1 << dbits) - 1;
        // (digit d of wavefront w: place 16 d + w)
        for (int e = threadIdx.x; e < kSortWaves << dbits; e += kSortThreads) counts[e] = 0;
        __syncthreads();
        for (int i = from + lane; i < to; i += kWave) atomicAdd(&counts[(keys[now][i] >> shift & mask) * kSortWaves + wave], 1);
        __syncthreads();
        int c[kSortEach], mine = 0;
#pragma unroll
        for (int e = 0; e < kSortEach; ++e) {
            const int at = threadIdx.x * kSortEach + e;
            c[e] = at < kSortWaves << dbits ? counts[at] : 0;
            mine += c[e];
        }
        const int scan = wave_inclusive_scan(mine);
        if (lane == kWave - 1) sums[wave] = scan;
        __syncthreads();
        int before = scan - mine;
        for (int w = 0; w < wave; ++w) before += sums[w];
#pragma unroll
        for (int e = 0; e < kSortEach; ++e) {
            const int at = threadIdx.x * kSortEach + e;
            if (at < kSortWaves << dbits) counts[at] = before;
            before += c[e];
        }
        __syncthreads();
        for (int i0 = from; i0 < to; i0 += kWave) {
            const int i = i0 + lane;
            const bool in = i < to;
            const uint32_t key = in ? keys[now][i] : 0u;
            const int digit = (int)(key >> shift) & mask;
            uint64_t same = __ballot(in);
            for (int b = 0; b < dbits; ++b) {
                const uint64_t ones = __ballot(digit >> b & 1);
                same &= digit >> b & 1 ? ones : ~ones;
            }
            if (in) {
                int *const run_place = &counts[digit * kSortWaves + wave];
                const int place = *run_place + __popcll(same & ((1ull << lane) - 1));
                keys[now ^ 1][place] = key;
                vals[now ^ 1][place] = vals[now][i];
                // the last lane of a digit moves the run's place on (the next round reads it behind this write)
                if (same >> lane == 1) *run_place = place + 1;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        shift += dbits;
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n; i += kSortThreads) {
        const_cast<uint32_t *>(a.sorted)[i] = keys[now][i];
        const_cast<uint32_t *>(a.order)[i] = vals[now][i];
    }
}

// Lists up to kMiddleList are sorted so in tiles of kTile keys, by digits of up to 9 bits: a launch counts each tile's
// digits (the first one of the tokens themselves, its further workgroups writing the zeros), one sums a digit's
// counts over the tiles, one moves the keys.  262144 tokens of 18 bits 53 us, by the library's sort of 8 bits a pass
// behind a launch that makes its keys 85; 1M 60 and 88, 4M 102 and 132; 16M 302 and 308, of 13 bits 231 and 220: short
// runs of a digit cost there.
constexpr int kTile = 4096, kTileEach = kTile / kSortThreads, kTileBits = 9;
constexpr int64_t kMiddleList = 1 << 23;

__global__ __launch_bounds__(kSortThreads) void k_token_counts(ScatterArgs a, const uint32_t *__restrict__ keys, int shift, int dbits)
{
    __shared__ int counts[kSortWaves << kTileBits];
    if ((int)blockIdx.x >= a.tiles) {
        write_zeros(a, (int64_t)(blockIdx.x - a.tiles) * kSortThreads + threadIdx.x, (int64_t)(gridDim.x - a.tiles) * kSortThreads);
        return;
    }
    const int64_t from = (int64_t)blockIdx.x * kTile;
    const int wave = threadIdx.x / kWave;
    const uint32_t mask = (1u << dbits) - 1;
    uint32_t key[kTileEach];
#pragma unroll
    for (int u = 0; u < kTileEach; ++u) {
        const int64_t i = from + u * kSortThreads + threadIdx.x, in = i < a.n ? i : a.n - 1;
        key[u] = keys ? keys[in] : key_of(a, in);
    }
    for (int e = threadIdx.x; e < kSortWaves << dbits; e += kSortThreads) counts[e] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kTileEach; ++u)
        if (from + u * kSortThreads + threadIdx.x < a.n) atomicAdd(&counts[(wave << dbits) + (key[u] >> shift & mask)], 1);
    __syncthreads();
    if ((int)threadIdx.x > (int)mask) return;
    int all = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) all += counts[(w << dbits) + threadIdx.x];
    a.counts[(int64_t)threadIdx.x * a.tiles + blockIdx.x] = all;
}

// Inclusive sums over the tiles, a wavefront a digit.
__global__ __launch_bounds__(kBlock) void k_token_scan(ScatterArgs a, int digits)
{
    constexpr int each = 4;
    const int digit = (int)(blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave);
    if (digit >= digits) return;
    int32_t *__restrict__ row = a.counts + (int64_t)digit * a.tiles;
    int carry = 0;
    for (int base = 0; base < a.tiles; base += each * kWave) {
        int v[each], sum = 0;
#pragma unroll
        for (int e = 0; e < each; ++e) {
            const int at = base + lane_id() * each + e;
            sum += v[e] = at < a.tiles ? row[at] : 0;
        }
        const int scan = wave_inclusive_scan(sum);
        int run = carry + scan - sum;
#pragma unroll
        for (int e = 0; e < each; ++e) {
            const int at = base + lane_id() * each + e;
            run += v[e];
            if (at < a.tiles) row[at] = run;
        }
        carry += __builtin_amdgcn_readlane(scan, kWave - 1);
    }
}

__global__ __launch_bounds__(kSortThreads) void k_token_move(ScatterArgs a, const uint32_t *__restrict__ keys,
                                                             const uint32_t *__restrict__ vals, uint32_t *__restrict__ keys_out,
                                                             uint32_t *__restrict__ vals_out, int shift, int dbits)
{
    __shared__ int counts[kSortWaves << kTileBits];
    __shared__ int to[1 << kTileBits];                   // where a digit's keys go, less where they lie in the tile
    __shared__ uint32_t stage[2][kTile];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const uint32_t mask = (1u << dbits) - 1;
    // (an XCD takes neighbouring tiles, whose runs of a digit share cache lines)
    const int xcd = blockIdx.x % 8, per = a.tiles / 8, rest = a.tiles % 8;
    const int tile = xcd * per + (xcd < rest ? xcd : rest) + (int)blockIdx.x / 8;
    const int64_t from = (int64_t)tile * kTile;
    const int count = a.n - from < kTile ? (int)(a.n - from) : kTile;
    const int run = wave * (kTile / kSortWaves);
    uint32_t key[kTileEach], val[kTileEach];
    int place[kTileEach];
#pragma unroll
    for (int u = 0; u < kTileEach; ++u) {
        const int64_t i = from + run + u * kWave + lane, in = i < a.n ? i : a.n - 1;
        key[u] = keys ? keys[in] : key_of(a, in);
        val[u] = vals ? vals[in] : (uint32_t)in;
    }
    const bool mine = (int)threadIdx.x <= (int)mask;
    const int32_t *__restrict__ row = a.counts + (int64_t)(mine ? threadIdx.x : 0) * a.tiles;
    const int whole = mine ? row[a.tiles - 1] : 0, before = mine && tile > 0 ? row[tile - 1] : 0;
    for (int e = threadIdx.x; e < kSortWaves << dbits; e += kSortThreads) counts[e] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kTileEach; ++u) {
        const bool in = run + u * kWave + lane < count;
        const uint32_t digit = key[u] >> shift & mask;
        uint64_t same = __ballot(in);
        for (int b = 0; b < dbits; ++b) {
            const uint64_t ones = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? ones : ~ones;
        }
        if (in) {
            int *const so_far = &counts[(wave << dbits) + digit];
            place[u] = *so_far + __popcll(same & ((1ull << lane) - 1));
            // (the last lane of a digit moves it on; the next round reads it behind this write)
            if (same >> lane == 1) *so_far = place[u] + 1;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    int first[2] = {0, whole}, all[2];
    if (mine) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) first[0] += counts[(w << dbits) + threadIdx.x];
    }
    block_exclusive_scans<2, kSortWaves>(first, all);
    if (mine) {
        int at = first[0];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = counts[(w << dbits) + threadIdx.x];
            counts[(w << dbits) + threadIdx.x] = at;
            at += c;
        }
        to[threadIdx.x] = first[1] + before - first[0];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kTileEach; ++u) {
        if (run + u * kWave + lane >= count) continue;
        const int at = place[u] + counts[(wave << dbits) + (key[u] >> shift & mask)];
        stage[0][at] = key[u];
        stage[1][at] = val[u];
    }
    __syncthreads();
    for (int q = threadIdx.x; q < count; q += kSortThreads) {
        const uint32_t k = stage[0][q];
        const int at = to[k >> shift & mask] + q;
        keys_out[at] = k;
        vals_out[at] = stage[1][q];
    }
}

// Columns [at + gone, at + VEC) of a row of the gradient: scale v, onto `was` where sums are added to it.
template <typename TO, int VEC>
__device__ __forceinline__ void put(const ScatterArgs &a, uint32_t token, int at, int gone, const float (&v)[VEC],
                                    const float (&was)[VEC])
{
    TO *__restrict__ out = static_cast<TO *>(a.out) + (int64_t)token * a.k;
    float w[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = fmaf(v[e], a.scale, was[e]);
    if (gone == 0) {
        store_out<TO, VEC>(out, at, w);
        return;
    }
    // (the columns before are the lane's before)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const float one[1] = {w[e]};
        if (e >= gone) store_out<TO, 1>(out, at + e, one);
    }
}

// VEC elements as they lie in memory: 16 bytes, or one.
template <typename T, int VEC>
struct Packed {
    std::conditional_t<VEC == 1, float, uint4> w;
    __device__ __forceinline__ void load(const T *__restrict__ p, int64_t i)
    {
        if constexpr (VEC == 1) {
            float one[1];
            load_vec<T, 1>(p, i, one);
            w = one[0];
        } else {
            // (read once: past the caches, 1M rows of 512 bytes 139 us, so 136; 262144 of 600, added, 111 and 104)
            const u32x4_u u = __builtin_nontemporal_load(reinterpret_cast<const u32x4_u *>(p + i));
            w = make_uint4(u.x, u.y, u.z, u.w);
        }
    }
    __device__ __forceinline__ void add_to(float (&t)[VEC]) const
    {
        if constexpr (VEC == 1) {
            t[0] += w;
        } else {
            float v[VEC];
            RowGather<T, VEC, false>::unpack16(w.x, w.y, w.z, w.w, v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) t[e] += v[e];
        }
    }
};

// A group of lanes a piece (and a chunk of its columns), a vector a lane.  Bound by the rows' reads, in the tokens'
// order: 1M rows of 512 bytes 132 us (4.5 TB/s of HBM).  ADD: the rows that sums are added to are read with the batch
// that names them first: 262144 rows of 600 bytes onto 1200 100 us (5.1 TB/s), where a read at each sum's end took 194.
constexpr int kDeep = 8;         // rows a lane has in flight

template <typename TI, typename TO, int VEC, bool ADD>
__global__ __launch_bounds__(kBlock) void k_scatter_sums(ScatterArgs a)
{
    constexpr int D = ADD && sizeof(TI) == 2 ? kDeep / 2 : kDeep;
    const int lane = lane_id() & (a.lanes - 1);
    const int64_t groups = (int64_t)gridDim.x * kBlock >> a.log_lanes;
    const int64_t all = (int64_t)a.pieces * a.chunks;
    const TI *__restrict__ dY = static_cast<const TI *>(a.dY);
    for (int64_t u = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> a.log_lanes; u < all; u += groups) {
        const int64_t piece = u / a.chunks;
        const int vec = (int)(u % a.chunks) * a.lanes + lane;
        const int c = vec * VEC;
        if (vec >= a.vecs) continue;
        const int64_t from = piece * a.per, to = from + a.per < a.n ? from + a.per : a.n;
        // (the last vector is moved back to the row's end)
        const int at = c + VEC <= a.k ? c : a.k - VEC;
        const int gone = c - at;
        const uint32_t before = from > 0 ? a.sorted[from - 1] : ~0u;
        const uint32_t after = to < a.n ? a.sorted[to] : ~0u;
        uint32_t token = a.sorted[from];
        bool begun = token == before;
        float t[VEC], was[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) t[e] = was[e] = 0.f;
        if (ADD && token < (uint32_t)a.V) read_row<TO, VEC>(static_cast<const TO *>(a.out) + (int64_t)token * a.k, at, was);
        const auto flush = [&](int slot) {
            // (columns of two lanes: both write the same sum)
            if (slot < 0) put<TO, VEC>(a, token, at, gone, t, was);
            else store_vec<float, VEC>(a.slots, (2 * piece + slot) * (int64_t)a.k + at, t);
        };
        for (int64_t i0 = from; i0 < to && token < (uint32_t)a.V; i0 += D) {
            uint32_t tok[D];
            Packed<TI, VEC> v[D];
            float base[ADD ? D : 1][VEC];
#pragma unroll
            for (int d = 0; d < D; ++d) {
                const int64_t i = i0 + d < to ? i0 + d : to - 1;
                tok[d] = i0 + d < to ? a.sorted[i] : (uint32_t)a.V;
                v[d].load(dY, (int64_t)a.order[i] * a.k + at);
                if constexpr (ADD) {
                    if (tok[d] < (uint32_t)a.V && tok[d] != (d > 0 ? tok[d > 0 ? d - 1 : 0] : token))
                        read_row<TO, VEC>(static_cast<const TO *>(a.out) + (int64_t)tok[d] * a.k, at, base[d]);
                }
            }
#pragma unroll
            for (int d = 0; d < D; ++d) {
                if (tok[d] != token) {
                    if (i0 + d >= to || token >= (uint32_t)a.V) continue;
                    flush(begun ? 0 : -1);
                    begun = false;
                    token = tok[d];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        t[e] = 0.f;
                        if constexpr (ADD) was[e] = base[d][e];
                    }
                    if (token >= (uint32_t)a.V) continue;
                }
                v[d].add_to(t);
            }
        }
        if (token < (uint32_t)a.V) flush(begun ? 0 : token == after ? 1 : -1);
    }
}

// Tokens that reach over pieces: the slot of the piece that begins one, then those of the pieces after.  A
// wavefront looks at a piece; tokens of more pieces than kShort are summed by the whole workgroup, in 16 parts, or
// more where rows are short.  Latency, mostly: 1M tokens, 10417 pieces of 256 columns, 17 us.
constexpr int kShort = 16;

// The sums of slots [q0, q1) of a token that begins in `piece`, columns [c, c + 4) below k.
__device__ __forceinline__ void sum_slots(const ScatterArgs &a, int64_t piece, int64_t q0, int64_t q1, int c, float (&t)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = 0.f;
    const bool whole = c + 4 <= a.k;
    for (int64_t q = q0; q < q1; q += kDeep) {
        float v[kDeep][4];
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            const int64_t at = q + d < q1 ? q + d : q1 - 1;
            const float *__restrict__ row = a.slots + (2 * (piece + at) + (at == 0 ? 1 : 0)) * (int64_t)a.k + c;
            if (whole) {
                load_vec<float, 4>(row, 0, v[d]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[d][e] = c + e < a.k ? row[e] : 0.f;
            }
        }
#pragma unroll
        for (int d = 0; d < kDeep; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] += q + d < q1 ? v[d][e] : 0.f;
    }
}

template <typename TO>
__global__ __launch_bounds__(kBlock) void k_scatter_join(ScatterArgs a)
{
    constexpr int W = kBlock / kWave;
    __shared__ float4 sums[kBlock];
    __shared__ int64_t long_count[W];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const auto finish = [&](uint32_t token, int c, const float (&t)[4]) {
        const TO *__restrict__ out = static_cast<const TO *>(a.out) + (int64_t)token * a.k;
        if (c + 4 <= a.k) {
            float was[4] = {0.f, 0.f, 0.f, 0.f};
            if (a.add) read_row<TO, 4>(out, c, was);
            put<TO, 4>(a, token, c, 0, t, was);
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= a.k) continue;
            const float one[1] = {t[e]};
            float was[1] = {0.f};
            if (a.add) read_row<TO, 1>(out, c + e, was);
            put<TO, 1>(a, token, c + e, 0, one, was);
        }
    };
    for (int64_t p0 = (int64_t)blockIdx.x * W; p0 + 1 < a.pieces; p0 += (int64_t)gridDim.x * W) {
        const int64_t piece = p0 + wave;
        int64_t count = 0;
        uint32_t token = 0;
        if (piece + 1 < a.pieces) {
            const int64_t from = piece * a.per, next = from + a.per;
            token = a.sorted[next - 1];
            const uint32_t after = a.sorted[next], first = a.sorted[from], before = from > 0 ? a.sorted[from - 1] : ~0u;
            if (token < (uint32_t)a.V && after == token && !(first == token && before == token)) {
                // the last piece that has it: the first that ends otherwise (most often the next one)
                int64_t lo = piece + 1, hi = a.pieces - 1;
                for (int64_t step = 1; lo < hi; step *= 2) {
                    const int64_t mid = lo + step - 1 < hi ? lo + step - 1 : hi - 1;
                    if (a.sorted[(mid + 1) * a.per] != token) {
                        hi = mid;
                        break;
                    }
                    lo = mid + 1;
                }
                while (lo < hi) {
                    const int64_t mid = (lo + hi) / 2;
                    if (a.sorted[(mid + 1) * a.per] == token) lo = mid + 1;
                    else hi = mid;
                }
                count = lo - piece + 1;
            }
        }
        if (count > 0 && count <= kShort) {
            for (int c = 4 * lane; c < a.k; c += 4 * kWave) {
                float t[4];
                sum_slots(a, piece, 0, count, c, t);
                finish(token, c, t);
            }
        }
        if (lane == 0) long_count[wave] = count > kShort ? count : 0;
        __syncthreads();
        for (int w = 0; w < W; ++w) {
            const int64_t many = long_count[w];
            if (many == 0) continue;                     // (uniform)
            const int64_t mine = p0 + w;
            const uint32_t its = a.sorted[(mine + 1) * a.per];
            // lanes by 4 columns: 16, fewer of short rows
            int lanes = 16;
            while (lanes > 1 && lanes * 2 >= a.k) lanes /= 2;
            const int parts = kBlock / lanes, part = threadIdx.x / lanes;
            for (int c0 = 0; c0 < a.k; c0 += 4 * lanes) {
                const int c = c0 + 4 * ((int)threadIdx.x % lanes);
                float t[4];
                sum_slots(a, mine, many * part / parts, many * (part + 1) / parts, c, t);
                __syncthreads();
                sums[threadIdx.x] = make_float4(t[0], t[1], t[2], t[3]);
                __syncthreads();
                for (int half = parts / 2; half > 0; half /= 2) {
                    if (part < half) {
                        const float4 o = sums[threadIdx.x + half * lanes];
                        t[0] += o.x; t[1] += o.y; t[2] += o.z; t[3] += o.w;
                        sums[threadIdx.x] = make_float4(t[0], t[1], t[2], t[3]);
                    }
                    __syncthreads();
                }
                if (part == 0) finish(its, c, t);
            }
        }
        __syncthreads();
    }
}

// Short lists over small tables, in one launch: a workgroup a token (and a chunk of its columns) looks through the list
// for its places, and sums their rows in runs of 16 or more, which are joined in order.  Launches and latency: 4096
// rows of 64 fp32 into 90, by sort, sums and join 30 us, so 10; all of 8192 rows of one token 36 and 25; 1000 rows of
// 256 into 90 24 and 8.  With 2000 workgroups (500 tokens of 4 chunks) 4096 rows take 32 and 23, with 8000 33 and 59.
constexpr int kFewTokens = 2048;             // tokens times chunks

template <typename TI, typename TO, int VEC>
__global__ __launch_bounds__(kSortThreads) void k_scatter_few(ScatterArgs a)
{
    constexpr int Rounds = kShortList / kSortThreads;
    __shared__ uint16_t places[kShortList];
    __shared__ int counts[kSortWaves];
    __shared__ float sums[VEC][kSortThreads];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int token = (int)(blockIdx.x / a.chunks), vec = (int)(blockIdx.x % a.chunks) * a.lanes + ((int)threadIdx.x & (a.lanes - 1));
    // the token's places in order: a wavefront's are those of a run of the list
    const int n = (int)a.n, run = ((n + kSortWaves - 1) / kSortWaves + kWave - 1) / kWave * kWave;
    const int from = wave * run, to = from + run < n ? from + run : n;
    uint64_t hits[Rounds];
    int here = 0, before = 0, all = 0;
#pragma unroll
    for (int u = 0; u < Rounds; ++u) {
        const int i = from + u * kWave + lane;
        hits[u] = __ballot(i < to && a.index[i] == token);
        here += __popcll(hits[u]);
    }
    if (lane == 0) counts[wave] = here;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        before += w < wave ? counts[w] : 0;
        all += counts[w];
    }
#pragma unroll
    for (int u = 0; u < Rounds; ++u) {
        if (hits[u] >> lane & 1) places[before + __popcll(hits[u] & ((1ull << lane) - 1))] = (uint16_t)(from + u * kWave + lane);
        before += __popcll(hits[u]);
    }
    __syncthreads();
    const bool on = vec < a.vecs;
    const int c = vec * VEC, at = c + VEC <= a.k ? c : a.k - VEC;
    float t[VEC], was[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = was[e] = 0.f;
    if (all == 0) {
        a.scale = 0.f;
        if (!a.add && (int)threadIdx.x < a.lanes && on) put<TO, VEC>(a, token, at, c - at, t, was);
        return;
    }
    const int group = (int)threadIdx.x >> a.log_lanes, groups = kSortThreads >> a.log_lanes;
    int per = (all + groups - 1) / groups;
    if (per < 16) per = 16;
    const int p0 = group * per, p1 = p0 + per < all ? p0 + per : all;
    const TI *__restrict__ dY = static_cast<const TI *>(a.dY);
    for (int p = p0; on && p < p1; p += kDeep) {
        Packed<TI, VEC> v[kDeep];
#pragma unroll
        for (int d = 0; d < kDeep; ++d) v[d].load(dY, (int64_t)places[p + d < p1 ? p + d : p1 - 1] * a.k + at);
#pragma unroll
        for (int d = 0; d < kDeep; ++d)
            if (p + d < p1) v[d].add_to(t);
    }
    const int parts = (all + per - 1) / per;
    if (parts > 1) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) sums[e][threadIdx.x] = t[e];
        __syncthreads();
        for (int half = 1 << (31 - __builtin_clz(parts - 1)); half > 0; half /= 2) {
            if (group < half && group + half < parts) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) sums[e][threadIdx.x] = t[e] += sums[e][threadIdx.x + (half << a.log_lanes)];
            }
            __syncthreads();
        }
    }
    if (group != 0 || !on) return;
    if (a.add) read_row<TO, VEC>(static_cast<const TO *>(a.out) + (int64_t)token * a.k, at, was);
    put<TO, VEC>(a, token, at, c - at, t, was);
}

// ------------------------------------------------------------- launching
template <typename F>
auto by_type(int dtype, F f)
{
    if (dtype == COGDL_F32) return f(float{});
    if (dtype == COGDL_BF16) return f(bf16_t{});
    return f(f16_t{});
}

cogdl_status check_table(int64_t n, int32_t V, int32_t k)
{
    if (n < 0 || V < 1 || k < 0) return COGDL_ERR_INVALID;
    if (n > COGDL_MAX_NNZ || k > (1 << 22) || V == INT32_MAX) return COGDL_ERR_TOO_LARGE;
    return COGDL_OK;
}

struct Scatter {
    size_t keys, ping_k, ping_v, sorted, order, sort, slots, total;
};

size_t al(size_t b) { return (b + 255) & ~size_t(255); }

// The sorted list's pieces: all of them at once on the chip, 16 tokens or more, and no more than the join takes in a
// few us.  With 4608 wavefronts of pieces 1M rows of 512 bytes take 140 us and their join 17, 262144 rows of 600, added,
// 111; with a third less 161, 12 and 129, with a third more 133, 19 and 142, with 8192 154, 25 and 116.
int32_t piece_of(int64_t n, int32_t vecs)
{
    const int lanes = vecs >= kWave ? kWave : next_pow2(vecs);
    const int64_t wide = (int64_t)((vecs + lanes - 1) / lanes) * lanes;      // of a piece
    int64_t per = (n * wide + kWave * 4608 - 1) / (kWave * 4608);
    if (per < n / 16384) per = n / 16384;
    if (per > 256) per = 256;
    per = (per + kDeep - 1) / kDeep * kDeep;
    return (int32_t)(per < 16 ? 16 : per);
}

// 16-byte vectors of a row, or its elements where it has under one.
int32_t vecs_of(int32_t k, int bytes)
{
    const int vec = 16 / bytes;
    return k >= vec ? (k + vec - 1) / vec : k;
}

Scatter scatter_layout(int64_t n, int32_t k)
{
    Scatter s;
    // (the type is not known here: the more pieces of the two)
    const int32_t p2 = piece_of(n, vecs_of(k, 2)), p4 = piece_of(n, vecs_of(k, 4));
    const int64_t pieces = (n + (p2 < p4 ? p2 : p4) - 1) / (p2 < p4 ? p2 : p4);
    size_t off = 0;
    s.keys = off; off += al(4 * (size_t)n);
    s.ping_k = off; off += al(8 * (size_t)n);
    s.ping_v = off; off += al(8 * (size_t)n);
    s.sorted = off; off += al(4 * (size_t)n);
    s.order = off; off += al(4 * (size_t)n);
    s.sort = off; off += al(n <= kMiddleList ? (4ull << kTileBits) * ((n + kTile - 1) / kTile) : radix_workspace_bytes(n));
    s.slots = off; off += al(8 * (size_t)pieces * k);
    s.total = off;
    return s;
}

template <typename TI, typename TO, int VEC>
cogdl_status run_lookup(LookupArgs a, hipStream_t stream)
{
    a.vecs = (a.k + VEC - 1) / VEC;
    a.rows = 2048 / a.vecs > 1 ? 2048 / a.vecs : 1;
    a.magic = (uint32_t)((((uint64_t)1 << 32) + a.vecs - 1) / a.vecs);
    int64_t blocks = (a.n + a.rows - 1) / a.rows;
    if (blocks > (1 << 20)) blocks = 1 << 20;
    COGDL_LAUNCH("embedding", (k_lookup<TI, TO, VEC>), (unsigned)blocks, kBlock, stream, a);
    return COGDL_OK;
}

template <typename TI, typename TO, int VEC>
cogdl_status run_few(ScatterArgs a, bool &done, hipStream_t stream)
{
    a.vecs = (a.k + VEC - 1) / VEC;
    a.lanes = a.vecs >= 16 ? 16 : next_pow2(a.vecs);
    a.log_lanes = log2i(a.lanes);
    a.chunks = (a.vecs + a.lanes - 1) / a.lanes;
    const int64_t blocks = (int64_t)a.V * a.chunks;
    done = a.n <= kShortList && blocks <= kFewTokens;
    if (done) COGDL_LAUNCH("embedding_few", (k_scatter_few<TI, TO, VEC>), (unsigned)blocks, kSortThreads, stream, a);
    return COGDL_OK;
}

template <typename TI, typename TO, int VEC>
cogdl_status run_scatter(ScatterArgs a, hipStream_t stream)
{
    a.vecs = (a.k + VEC - 1) / VEC;
    a.lanes = a.vecs >= kWave ? kWave : next_pow2(a.vecs);
    a.log_lanes = log2i(a.lanes);
    a.chunks = (a.vecs + a.lanes - 1) / a.lanes;
    const int64_t groups = (int64_t)a.pieces * a.chunks;
    int64_t blocks = ((groups << a.log_lanes) + kBlock - 1) / kBlock;
    if (blocks > (1 << 20)) blocks = 1 << 20;
    if (a.add) COGDL_LAUNCH("embedding_sums", (k_scatter_sums<TI, TO, VEC, true>), (unsigned)blocks, kBlock, stream, a);
    else COGDL_LAUNCH("embedding_sums", (k_scatter_sums<TI, TO, VEC, false>), (unsigned)blocks, kBlock, stream, a);
    if (a.pieces > 1) {
        const int64_t joins = (a.pieces + kBlock / kWave - 2) / (kBlock / kWave);
        COGDL_LAUNCH("embedding_join", k_scatter_join<TO>, (unsigned)(joins < (1 << 16) ? joins : 1 << 16), kBlock, stream, a);
    }
    return COGDL_OK;
}

}  // namespace
}  // namespace cogdl

using namespace cogdl;

extern "C" {

cogdl_status cogdl_embedding(int64_t n, int32_t V, int32_t k, const void *table, cogdl_dtype dtype, const int32_t *index,
                             float scale, void *Y, cogdl_dtype y_dtype, hipStream_t stream)
{
    const cogdl_status st = check_table(n, V, k);
    if (st != COGDL_OK) return st;
    if (!dtype_ok(dtype) || !dtype_ok(y_dtype)) return COGDL_ERR_DTYPE;
    if (n == 0 || k == 0) return COGDL_OK;
    if (!index || !Y || !table) return COGDL_ERR_INVALID;
    LookupArgs a{};
    a.n = n; a.V = V; a.k = k;
    a.scale = scale;
    a.table = table;
    a.index = index;
    a.out = Y;
    return by_type(dtype, [&](auto ti) {
        using TI = decltype(ti);
        return by_type(y_dtype, [&](auto to) {
            using TO = decltype(to);
            constexpr int VEC = 16 / (int)sizeof(TI);
            return a.k >= VEC ? run_lookup<TI, TO, VEC>(a, stream) : run_lookup<TI, TO, 1>(a, stream);
        });
    });
}

cogdl_status cogdl_embedding_backward_workspace(int64_t n, int32_t V, int32_t k, size_t *bytes)
{
    if (!bytes) return COGDL_ERR_INVALID;
    const cogdl_status st = check_table(n, V, k);
    if (st != COGDL_OK) return st;
    *bytes = n > 0 && k > 0 ? scatter_layout(n, k).total : 0;
    return COGDL_OK;
}

cogdl_status cogdl_embedding_backward(int64_t n, int32_t V, int32_t k, const void *dY, cogdl_dtype dtype,
                                      const int32_t *index, float scale, void *dtable, cogdl_dtype d_dtype,
                                      int32_t accumulate, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    const cogdl_status st = check_table(n, V, k);
    if (st != COGDL_OK) return st;
    if (!dtype_ok(dtype) || !dtype_ok(d_dtype)) return COGDL_ERR_DTYPE;
    if (k == 0) return COGDL_OK;
    if (!dtable) return COGDL_ERR_INVALID;
    ScatterArgs a{};
    a.n = n; a.V = V; a.k = k;
    a.scale = scale;
    a.index = index;
    a.dY = dY;
    a.out = dtable;
    a.add = accumulate != 0;
    a.out_bytes = dtype_bytes(d_dtype);
    if (n > 0) {
        if (!dY || !index) return COGDL_ERR_INVALID;
        const Scatter s = scatter_layout(n, k);
        if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < s.total) return COGDL_ERR_INVALID;
        char *ws = static_cast<char *>(workspace);
        a.keys = reinterpret_cast<uint32_t *>(ws + s.keys);
        a.sorted = reinterpret_cast<uint32_t *>(ws + s.sorted);
        a.order = reinterpret_cast<uint32_t *>(ws + s.order);
        a.slots = reinterpret_cast<float *>(ws + s.slots);
        a.per = piece_of(n, vecs_of(k, dtype_bytes(dtype)));
        a.pieces = (int32_t)((n + a.per - 1) / a.per);
        bool done = false;
        const cogdl_status few = by_type(dtype, [&](auto ti) {
            using TI = decltype(ti);
            return by_type(d_dtype, [&](auto to) {
                using TO = decltype(to);
                constexpr int VEC = 16 / (int)sizeof(TI);
                return a.k >= VEC ? run_few<TI, TO, VEC>(a, done, stream) : run_few<TI, TO, 1>(a, done, stream);
            });
        });
        if (done || few != COGDL_OK) return few;
    } else if (a.add) {
        return COGDL_OK;
    }
    const int64_t zeros = a.add ? 0 : ((int64_t)V * k * a.out_bytes + 15) / 16;      // threads for them
    const int bits = bits_for((uint64_t)V);
    if (n > 0 && n <= kShortList) {
        int64_t blocks = (zeros + kSortThreads - 1) / kSortThreads;
        if (blocks > 1024) blocks = 1024;
        COGDL_LAUNCH("embedding_sort", k_sort_short, (unsigned)(blocks + 1), kSortThreads, stream, a, bits);
    } else if (n > 0 && n <= kMiddleList) {
        char *ws = static_cast<char *>(workspace);
        const Scatter s = scatter_layout(n, k);
        a.counts = reinterpret_cast<int32_t *>(ws + s.sort);
        a.tiles = (int32_t)((n + kTile - 1) / kTile);
        int64_t blocks = (zeros + kSortThreads - 1) / kSortThreads;
        if (blocks > 1024) blocks = 1024;
        const int passes = (bits + kTileBits - 1) / kTileBits;
        const uint32_t *keys = nullptr, *vals = nullptr;
        for (int p = 0, shift = 0; p < passes; ++p) {
            const int dbits = (bits - shift) / (passes - p);
            const bool last = p == passes - 1;
            uint32_t *const keys_to = last ? const_cast<uint32_t *>(a.sorted) : reinterpret_cast<uint32_t *>(ws + s.ping_k) + (p & 1) * n;
            uint32_t *const vals_to = last ? const_cast<uint32_t *>(a.order) : reinterpret_cast<uint32_t *>(ws + s.ping_v) + (p & 1) * n;
            COGDL_LAUNCH("embedding_count", k_token_counts, (unsigned)(a.tiles + (p == 0 ? blocks : 0)), kSortThreads, stream, a, keys, shift, dbits);
            COGDL_LAUNCH("embedding_scan", k_token_scan, (1u << dbits) / 4 + 1, kBlock, stream, a, 1 << dbits);
            COGDL_LAUNCH("embedding_move", k_token_move, (unsigned)a.tiles, kSortThreads, stream, a, keys, vals, keys_to, vals_to, shift, dbits);
            keys = keys_to;
            vals = vals_to;
            shift += dbits;
        }
    } else {
        int64_t blocks = ((n > zeros ? n : zeros) + kBlock - 1) / kBlock;
        if (blocks > 4096) blocks = 4096;
        COGDL_LAUNCH("embedding_tokens", k_tokens, (unsigned)blocks, kBlock, stream, a);
        if (n == 0) return COGDL_OK;
        char *ws = static_cast<char *>(workspace);
        const Scatter s = scatter_layout(n, k);
        COGDL_HIP_TRY(radix_sort_pairs(a.keys, nullptr, const_cast<uint32_t *>(a.sorted), const_cast<uint32_t *>(a.order),
                                       n, bits, reinterpret_cast<uint32_t *>(ws + s.ping_k),
                                       reinterpret_cast<uint32_t *>(ws + s.ping_v), ws + s.sort, stream));
    }
    return by_type(dtype, [&](auto ti) {
        using TI = decltype(ti);
        return by_type(d_dtype, [&](auto to) {
            using TO = decltype(to);
            constexpr int VEC = 16 / (int)sizeof(TI);
            return a.k >= VEC ? run_scatter<TI, TO, VEC>(a, stream) : run_scatter<TI, TO, 1>(a, stream);
        });
    });
}

}  // extern "C"
