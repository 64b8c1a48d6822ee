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

constexpr int kBlock = 256;

// ---------------------------------------------------------------- lookup
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
    int32_t per, pieces;
    int32_t lanes, log_lanes, vecs, chunks;
};

__global__ __launch_bounds__(kBlock) void k_tokens(ScatterArgs a)
{
    const int64_t me = (int64_t)blockIdx.x * kBlock + threadIdx.x, all = (int64_t)gridDim.x * kBlock;
    for (int64_t i = me; i < a.n; i += all) {
        const uint32_t t = (uint32_t)a.index[i];
        a.keys[i] = t < (uint32_t)a.V ? t : (uint32_t)a.V;
    }
    if (a.add) return;
    // the gradient of tokens that do not occur
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

// Columns [at + gone, at + VEC) of a row of the gradient: (out +) scale v.
template <typename TO, int VEC>
__device__ __forceinline__ void put(const ScatterArgs &a, uint32_t token, int at, int gone, const float (&v)[VEC])
{
    TO *__restrict__ out = static_cast<TO *>(a.out) + (int64_t)token * a.k;
    if (!a.add && gone == 0) {
        float w[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = v[e] * a.scale;
        store_out<TO, VEC>(out, at, w);
        return;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        if (e < gone) continue;
        float was[1] = {0.f};
        if (a.add) load_vec<TO, 1>(out, at + e, was);
        const float sum[1] = {fmaf(v[e], a.scale, was[0])};
        store_out<TO, 1>(out, at + e, sum);
    }
}

constexpr int kDeep = 8;         // rows a lane has in flight

template <typename TI, typename TO, int VEC>
__global__ __launch_bounds__(kBlock) void k_scatter_sums(ScatterArgs a)
{
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
        float t[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) t[e] = 0.f;
        const auto flush = [&](int slot) {
            if (slot < 0) {
                put<TO, VEC>(a, token, at, gone, t);
                return;
            }
            // (columns of two lanes: both write the same sum)
            store_vec<float, VEC>(a.slots, (2 * piece + slot) * (int64_t)a.k + at, t);
        };
        for (int64_t i0 = from; i0 < to && token < (uint32_t)a.V; i0 += kDeep) {
            uint32_t tok[kDeep];
            float v[kDeep][VEC];
#pragma unroll
            for (int d = 0; d < kDeep; ++d) {
                const int64_t i = i0 + d < to ? i0 + d : to - 1;
                tok[d] = i0 + d < to ? a.sorted[i] : (uint32_t)a.V;
                load_vec<TI, VEC>(dY, (int64_t)a.order[i] * a.k + at, v[d]);
            }
#pragma unroll
            for (int d = 0; d < kDeep; ++d) {
                if (tok[d] != token) {
                    if (i0 + d >= to || token >= (uint32_t)a.V) continue;
                    flush(begun ? 0 : -1);
                    begun = false;
                    token = tok[d];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) t[e] = 0.f;
                    if (token >= (uint32_t)a.V) continue;
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) t[e] += v[d][e];
            }
        }
        if (token < (uint32_t)a.V) flush(begun ? 0 : token == after ? 1 : -1);
    }
}

// Tokens that reach over pieces: the slot of the piece that begins one, then those of the pieces after.
template <typename TO>
__global__ __launch_bounds__(kBlock) void k_scatter_join(ScatterArgs a)
{
    constexpr int kCols = 16, kParts = kBlock / kCols;
    __shared__ float sums[kParts][kCols];
    const int part = threadIdx.x / kCols, col = threadIdx.x % kCols;
    for (int64_t piece = blockIdx.x; piece + 1 < a.pieces; piece += gridDim.x) {
        const int64_t from = piece * a.per, next = from + a.per;
        const uint32_t token = a.sorted[next - 1];
        if (token >= (uint32_t)a.V || a.sorted[next] != token) continue;
        if (a.sorted[from] == token && from > 0 && a.sorted[from - 1] == token) continue;      // begun before
        // the last piece that has it: the first that ends otherwise
        int64_t lo = piece + 1, hi = a.pieces - 1;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            const int64_t end = (mid + 1) * a.per;         // (of a piece before the last)
            if (a.sorted[end] == token) lo = mid + 1;
            else hi = mid;
        }
        const int64_t count = lo - piece + 1;
        const int64_t p0 = count * part / kParts, p1 = count * (part + 1) / kParts;
        for (int c0 = 0; c0 < a.k; c0 += kCols) {
            const int c = c0 + col;
            float t = 0.f;
            if (c < a.k) {
#pragma unroll 4
                for (int64_t q = p0; q < p1; ++q) t += a.slots[(2 * (piece + q) + (q == 0 ? 1 : 0)) * (int64_t)a.k + c];
            }
            __syncthreads();
            sums[part][col] = t;
            __syncthreads();
            if (part == 0 && c < a.k) {
                for (int q = 1; q < kParts; ++q) t += sums[q][col];
                const float one[1] = {t};
                put<TO, 1>(a, token, c, 0, one);
            }
        }
    }
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
    size_t keys, ping_k, ping_v, sorted, order, radix, slots, total;
    int32_t per;
    int64_t pieces;
};

size_t al(size_t b) { return (b + 255) & ~size_t(255); }

Scatter scatter_layout(int64_t n, int32_t k)
{
    Scatter s;
    s.per = n < (1 << 16) ? 16 : n < (1 << 18) ? 32 : 64;
    s.pieces = (n + s.per - 1) / s.per;
    size_t off = 0;
    s.keys = off; off += al(4 * (size_t)n);
    s.ping_k = off; off += al(8 * (size_t)n);
    s.ping_v = off; off += al(8 * (size_t)n);
    s.sorted = off; off += al(4 * (size_t)n);
    s.order = off; off += al(4 * (size_t)n);
    s.radix = off; off += al(radix_workspace_bytes(n));
    s.slots = off; off += al(8 * (size_t)s.pieces * k);
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
cogdl_status run_scatter(ScatterArgs a, hipStream_t stream)
{
    a.vecs = (a.k + VEC - 1) / VEC;
    a.lanes = a.vecs >= kWave ? kWave : next_pow2(a.vecs);
    a.log_lanes = log2i(a.lanes);
    a.chunks = (a.vecs + a.lanes - 1) / a.lanes;
    const int64_t groups = (int64_t)a.pieces * a.chunks;
    int64_t blocks = ((groups << a.log_lanes) + kBlock - 1) / kBlock;
    if (blocks > (1 << 20)) blocks = 1 << 20;
    COGDL_LAUNCH("embedding_sums", (k_scatter_sums<TI, TO, VEC>), (unsigned)blocks, kBlock, stream, a);
    if (a.pieces > 1) {
        const unsigned joins = a.pieces < (1 << 16) ? (unsigned)a.pieces : 1u << 16;
        COGDL_LAUNCH("embedding_join", k_scatter_join<TO>, joins, kBlock, stream, a);
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
        a.per = s.per;
        a.pieces = (int32_t)s.pieces;
    } else if (a.add) {
        return COGDL_OK;
    }
    int64_t blocks = a.add ? (n + kBlock - 1) / kBlock : ((int64_t)V * k * a.out_bytes / 16 + n + kBlock - 1) / kBlock + 1;
    if (blocks > 4096) blocks = 4096;
    COGDL_LAUNCH("embedding_tokens", k_tokens, (unsigned)blocks, kBlock, stream, a);
    if (n == 0) return COGDL_OK;
    char *ws = static_cast<char *>(workspace);
    const Scatter s = scatter_layout(n, k);
    COGDL_HIP_TRY(radix_sort_pairs(a.keys, nullptr, const_cast<uint32_t *>(a.sorted), const_cast<uint32_t *>(a.order), n,
                                   bits_for((uint64_t)V), reinterpret_cast<uint32_t *>(ws + s.ping_k),
                                   reinterpret_cast<uint32_t *>(ws + s.ping_v), ws + s.radix, stream));
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
