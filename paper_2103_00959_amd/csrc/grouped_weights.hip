// The gradients of the grouped products' weights and biases:
//     dW[g, c, j] = sum_{i in g} dZ[i, c] X[i, j],   db[g, c] = sum_{i in g} dZ[i, c]
//
// The sums run over rows, and which group they belong to only the device knows: the rows are cut into
// slices, and a workgroup goes through a slice's groups.  A group inside a slice is written as it
// is, one that reaches over several as fp32 partial sums into the workspace, added up in a
// fixed order by k_reduce_slices (no atomics: the same bits every run).
#include "grouped_tile.hpp"

namespace cogdl {
namespace {

// The matrix of a group without rows is zeroed in pieces of so many elements (of size 0 in one: db's zeros are with
// the first), which all workgroups share evenly: bound by memory.  8 rows in the first 8 of 64 groups, 2048 -> 1024
// bf16: 48 us (5.6 TB/s); one row among 256 groups of 1024 x 1024 111 (4.8 TB/s); 4096 groups of 64 x 64, two of
// them with rows, 14.  (As tiles of the slice at their place 354, 1558 and 6459: a workgroup zeroed a run of them one
// after another.)
constexpr int kZeroPiece = 16384;
__host__ __device__ inline int64_t zero_pieces(int64_t size) { return size > 0 ? (size + kZeroPiece - 1) / kZeroPiece : 1; }

// dW and db: TM x TN outputs (c by j) of a group's matrix at a time, over a slice's rows of it.
// One group of 32768 rows, 2048 x 2048 bf16: 270 us (1.02 PFLOP/s); from 8 bits 365: each of the 8 rows of
// tiles decodes the codes again, and the matrix cores wait meanwhile.  64 groups of 280 to 2244 rows
// 435 and 500: a workgroup stores 17 groups' tiles one after another.  2.4M rows of 8 groups, 256 -> 128,
// from 8 bits 353 us (3.5 TB/s); 600k rows of 12, 256 -> 256, 157 (2.9 TB/s): the decoding.  Under an activation dZ is
// formed anew for each tile: from the input, ReLU 530 us and ELU 570 (386 without) for those 2.4M rows, 262 and 282
// (161) for the 600k; from 8 bits 615 and 670, 311 and 340.
template <typename T, int WAVES, int TM, int TN, int SRC, int SRCB>
__global__ __launch_bounds__(WAVES * kWave) void k_grouped_weights(GroupedArgs a)
{
    constexpr int N = WAVES * kWave;
    constexpr int WAVES_C = TN >= 256 ? 4 : 2, WAVES_R = WAVES / WAVES_C;
    constexpr int WR = TM / WAVES_R / 32, WC = TN / WAVES_C / 32;
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int r0 = wave / WAVES_C * (32 * WR), c0 = wave % WAVES_C * (32 * WC);
    const int tiles_k = a.k > 0 ? (a.k + TN - 1) / TN : 1, nb = (a.k + kCkptBlock - 1) / kCkptBlock;
    const int64_t mk = (int64_t)a.m * a.k;
    // db: staged operands sum their own columns on the way; direct ones are summed from the
    // fragments of the wavefronts that hold the first columns
    constexpr bool STAGED_SUM = SRC != kDirect;
    SliceWalk walk;
    walk.start(a.off, a.E, a.n, a.per, a.tiles_c);
    ColOperand<T, TM, N, SRC, STAGED_SUM> A;
    ColOperand<T, TN, N, SRCB, false> B;
    A.clear_sums();
    const auto sums = [&](const Span &s) { return a.db && s.tile % tiles_k == 0; };
    const auto open = [&](const Span &s) {
        A.open(static_cast<const T *>(a.dY) + s.lo * a.m, SRC == kSloped ? static_cast<const T *>(a.Y) + s.lo * a.m : nullptr,
               nullptr, nullptr, s.tile / tiles_k * TM, a.m, s.have, a.act, sums(s));
        B.open(static_cast<const T *>(a.X) + (SRCB == kCodes ? 0 : s.lo * a.k), nullptr,
               SRCB == kCodes ? a.codes + s.lo * a.k : nullptr, SRCB == kCodes ? a.exps + s.lo * nb : nullptr,
               s.tile % tiles_k * TN, a.k, s.have, 0, false);
        return s.have;
    };
    // (db comes from the wavefronts of the first columns, whatever k)
    const auto busy = [&](const Span &s) {
        return s.tile / tiles_k * TM + r0 < a.m && (c0 == 0 || s.tile % tiles_k * TN + c0 < a.k);
    };
    float fsum[STAGED_SUM ? 1 : WR], colsum[STAGED_SUM ? 8 : 1];
#pragma unroll
    for (int i = 0; i < (STAGED_SUM ? 1 : WR); ++i) fsum[i] = 0.f;
    constexpr uint32_t kOnes = Fmt<T>::code == COGDL_BF16 ? 0x3f803f80u : 0x3c003c00u;
    const auto each = [&](const Span &s, const uint4 (&fa)[WR]) {
        if constexpr (!STAGED_SUM) {
            if (c0 != 0 || !sums(s)) return;
#pragma unroll
            for (int i = 0; i < WR; ++i) {
                fsum[i] = dot2_acc<T>(fa[i].x, kOnes, fsum[i]);
                fsum[i] = dot2_acc<T>(fa[i].y, kOnes, fsum[i]);
                fsum[i] = dot2_acc<T>(fa[i].z, kOnes, fsum[i]);
                fsum[i] = dot2_acc<T>(fa[i].w, kOnes, fsum[i]);
            }
        }
    };
    const auto settle = [&](const Span &) {
        if constexpr (STAGED_SUM) {
#pragma unroll
            for (int e = 0; e < 8; ++e) colsum[e] = A.sum[e];
            A.clear_sums();
        }
    };
    char *const outs = lds + 2 * (TM + TN) * kX * 2;
    run_tiles<T, decltype(A), decltype(B), WR, WC>(lds, walk, A, B, r0, c0, open, busy, each, settle, [&](const Span &s,
                                                                                             const Acc<WR, WC> &acc) {
        const int row0 = s.tile / tiles_k * TM, col0 = s.tile % tiles_k * TN;
        if (a.out) {
            float *__restrict__ part = a.part + s.slot * mk;
            for_outputs<WR, WC>(outs + wave * kOutBytes, acc, [&](int, int r, int c, float (&v)[8]) {
                r += row0 + r0;
                c += col0 + c0;
                if (r >= a.m || c >= a.k) return;
                if (s.slot < 0) store8(a.out, a.out_dtype, s.g * mk + (int64_t)r * a.k, c, a.k, v);
                else store8(part + (int64_t)r * a.k, c, a.k, v);
            });
        }
        if (!sums(s)) return;
        float *__restrict__ db = s.slot < 0 ? a.db + (int64_t)s.g * a.m : a.part_db + (int64_t)s.slot * a.m;
        if constexpr (STAGED_SUM) {
            // the threads that share 8 columns add up in order
            constexpr int P = TM / 8, S = N / P;
            static_assert(S * TM * (int)sizeof(float) <= WAVES * kOutBytes, "the sums fit the outputs' part");
            float *const shared = reinterpret_cast<float *>(outs);
            meet();
#pragma unroll
            for (int e = 0; e < 8; ++e) shared[(threadIdx.x / P) * TM + (threadIdx.x % P) * 8 + e] = colsum[e];
            meet();
            const int c = row0 + (int)threadIdx.x;
            if ((int)threadIdx.x < TM && c < a.m) {
                float t = 0.f;
#pragma unroll
                for (int q = 0; q < S; ++q) t += shared[q * TM + threadIdx.x];
                db[c] = t;
            }
            meet();
        } else if (c0 == 0) {
            const int lane = lane_id();
#pragma unroll
            for (int i = 0; i < WR; ++i) {
                const float t = fsum[i] + bfly_partner<32>(fsum[i]);
                const int c = row0 + r0 + 32 * i + (lane & 31);
                if (lane < 32 && c < a.m) db[c] = t;
                fsum[i] = 0.f;
            }
        }
    });
    const float zeros[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int64_t size = a.out ? mk : 0;
    deal_empty_groups(a.off, a.E, a.n, zero_pieces(size), [&](int g, int64_t piece) {
        const int64_t end = (piece + 1) * kZeroPiece < size ? (piece + 1) * kZeroPiece : size;
        for (int64_t i = piece * kZeroPiece + threadIdx.x * 8; i < end; i += N * 8)
            store8(a.out, a.out_dtype, g * mk + i, 0, end - i < 8 ? (int)(end - i) : 8, zeros);
        if (piece == 0 && a.db)
            for (int c = threadIdx.x; c < a.m; c += N) a.db[(int64_t)g * a.m + c] = 0.f;
    });
}

// Sums over a group's partial sums: slot 2 i + 1 of its first slice i, then slots 2 i of the
// others, in order; of many, 4 or 16 parts are added up by threads of their own and then joined in
// order (one group of 1024 slices, 19 x 19: 50 us with 4 parts, 16 with 16).  kBatch loads are in flight.  Bound by memory where the partial sums are many: 64 groups over 4
// slices, 2048 x 2048, 28 us (100 MB read).
constexpr int kBlock = 256;
constexpr int kBatch = 8;

// Parts of so many slots.
__host__ __device__ inline int parts_of(int64_t slots) { return slots >= 64 ? 16 : slots >= 16 ? 4 : 1; }

// V values from p on in the slots of slices [at, end), the group's first slice being `first`; slots
// are `stride` floats apart.
template <int V>
__device__ __forceinline__ void sum_slots(const float *__restrict__ p, int64_t stride, int first, int at, int end, float (&t)[V])
{
    for (; at < end; at += kBatch) {
        float v[kBatch][V];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (at + u >= end) break;
            const int64_t slot = 2 * (int64_t)(at + u) + (at + u == first ? 1 : 0);
            if constexpr (V == 4) load_vec<float, 4>(p, slot * stride, v[u]);
            else v[u][0] = p[slot * stride];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (at + u >= end) break;
#pragma unroll
            for (int e = 0; e < V; ++e) t[e] += v[u][e];
        }
    }
}

// dW and db of the groups that reach over several slices, V values a thread.  Block row y looks at
// group y or, where there are fewer borders between slices than groups, at the group that reaches
// over border y first.
template <int V>
__global__ __launch_bounds__(kBlock) void k_reduce_slices(GroupedArgs a, bool by_border)
{
    __shared__ float sums[kBlock][V];
    int g = blockIdx.y;
    const int64_t border = (int64_t)(g + 1) * a.per;
    if (by_border) g = a.off[0] < border ? (int)RowCursor::find(a.off, a.E, border - 1) : 0;
    const int64_t lo = offset_at(a.off, g, a.n), hi = offset_at(a.off, g + 1, a.n);
    if (hi <= lo || (by_border && (lo >= border || hi <= border || lo < border - a.per))) return;
    const int first = (int)(lo / a.per), count = (int)((hi - 1) / a.per) - first + 1;
    if (count <= 1) return;
    const int parts = parts_of(count), width = kBlock / parts;
    const int part = threadIdx.x / width, mine = threadIdx.x % width;
    const int at = first + (int)((int64_t)count * part / parts), end = first + (int)((int64_t)count * (part + 1) / parts);
    const int64_t mk = a.out ? (int64_t)a.m * a.k : 0, all = mk + (a.db ? a.m : 0);
    const int64_t step = (int64_t)gridDim.x * width * V;
    for (int64_t i0 = (int64_t)blockIdx.x * width * V; i0 < all; i0 += step) {
        const int64_t i = i0 + mine * V;
        float t[V];
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = 0.f;
        if (i < mk) sum_slots<V>(a.part + i, mk, first, at, end, t);
        else if (i < all) sum_slots<V>(a.part_db + (i - mk), a.m, first, at, end, t);
        if (parts > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) sums[threadIdx.x][e] = t[e];
            __syncthreads();
            if (part == 0) {
                for (int q = 1; q < parts; ++q)
#pragma unroll
                    for (int e = 0; e < V; ++e) t[e] += sums[q * width + mine][e];
            }
        }
        if (part != 0 || i >= all) continue;
        if (i >= mk) {
            store_vec<float, V>(a.db, (int64_t)g * a.m + (i - mk), t);
        } else if (a.out_dtype == COGDL_F32) {
            store_vec<float, V>(static_cast<float *>(a.out), g * mk + i, t);
        } else if (a.out_dtype == COGDL_BF16) {
            store_vec<bf16_t, V>(static_cast<bf16_t *>(a.out), g * mk + i, t);
        } else {
            store_vec<f16_t, V>(static_cast<f16_t *>(a.out), g * mk + i, t);
        }
    }
}

struct Tiles {
    int tm, tn;
};

template <typename T, int WAVES, int TM, int TN>
GroupedKernel pick(bool act, bool codes, bool direct_dy, bool direct_x)
{
    if (act) return codes ? k_grouped_weights<T, WAVES, TM, TN, kSloped, kCodes> : k_grouped_weights<T, WAVES, TM, TN, kSloped, kStaged>;
    if (codes) return direct_dy ? k_grouped_weights<T, WAVES, TM, TN, kDirect, kCodes> : k_grouped_weights<T, WAVES, TM, TN, kStaged, kCodes>;
    return direct_dy && direct_x ? k_grouped_weights<T, WAVES, TM, TN, kDirect, kDirect>
                                 : k_grouped_weights<T, WAVES, TM, TN, kStaged, kStaged>;
}

template <typename T>
GroupedKernel pick_tile(const Tiles &c, bool act, bool codes, bool direct_dy, bool direct_x)
{
    if (c.tm == 256) return codes ? k_grouped_weights<T, 8, 256, 256, kDirect, kCodes>
                                  : k_grouped_weights<T, 8, 256, 256, kDirect, kDirect>;
    if (c.tm == 128) return c.tn == 128 ? pick<T, 4, 128, 128>(act, codes, direct_dy, direct_x)
                                        : pick<T, 4, 128, 64>(act, codes, direct_dy, direct_x);
    return c.tn == 128 ? pick<T, 4, 64, 128>(act, codes, direct_dy, direct_x) : pick<T, 4, 64, 64>(act, codes, direct_dy, direct_x);
}

int64_t tiles_of(int64_t m, int64_t k, int tm, int tn) { return (m + tm - 1) / tm * (k > 0 ? (k + tn - 1) / tn : 1); }

}  // namespace

// Slices of rows: a group that is cut costs its partial sums, so there are no more slices than
// make two tiles of 128 x 128 (one of 256 x 256) for each resident workgroup, and of few rows a
// slice for 128 of them or 4 groups or, where the partial sums are small, as many as they leave
// under 4 MB.  Slices have 16 rows or more, or 4 groups each: few rows can be as many groups (46 rows
// in 253 groups, 104 x 28: 49 us in 2 slices, 9 in 46; 64 groups of one row, 1024 x 1024, 105 and 35).
Slices slices_of(int64_t n, int32_t E, int32_t k, int32_t m)
{
    const int64_t tiles = tiles_of(m, k, m > 64 ? 128 : 64, k > 64 ? 128 : 64);
    int64_t count = tiles > 0 ? (1024 + tiles - 1) / tiles : 1;
    const int64_t small = (4 << 20) / (16 * ((int64_t)m * k + m + 1));
    int64_t most = n / 128 > E / 4 ? n / 128 : E / 4;
    if (most < small) most = small;
    if (count > most) count = most;
    const int64_t rows = n / 16 > E / 4 ? n / 16 : E / 4;
    if (count > rows) count = rows;
    if (count > n) count = n;
    if (count < 1) count = 1;
    Slices c;
    c.per = (n + count - 1) / count;
    if (c.per < 1) c.per = 1;
    c.count = n > 0 ? (n + c.per - 1) / c.per : 1;
    return c;
}

cogdl_status grouped_weights_launch(GroupedArgs a, const Slices &c, cogdl_dtype dtype, hipStream_t stream)
{
    a.per = (int32_t)c.per;
    if (!a.out) {               // db alone: one column of tiles
        a.k = 0;
        a.X = a.codes = nullptr;
    }
    a.part_db = a.part + (size_t)c.slots() * a.m * a.k;
    const bool act = a.act != COGDL_ACT_NONE, codes = a.codes != nullptr;
    const bool direct_dy = on_grid(a.dY, a.m), direct_x = a.out && !codes && on_grid(a.X, a.k);
    Tiles t{a.m > 64 ? 128 : 64, a.k > 64 ? 128 : 64};
    // (from 8 bits, with 256 x 256 and with 128 x 128: 64 groups of 32768 rows, 2048 x 2048, 541 and 756 us; 600k
    // rows, 256 x 256, 170 and 208)
    if (a.m > 128 && a.k > 128 && !act && direct_dy && (codes || direct_x)) t = {256, 256};
    a.tiles_c = (int32_t)tiles_of(a.m, a.k, t.tm, t.tn);
    const GroupedKernel kern = dtype == COGDL_BF16 ? pick_tile<bf16_t>(t, act, codes, direct_dy, direct_x)
                                                   : pick_tile<f16_t>(t, act, codes, direct_dy, direct_x);
    const int waves = t.tm == 256 ? 8 : 4;
    // (with any number of groups without rows: which, only the device knows)
    const int64_t zeros = a.E * zero_pieces(a.out ? (int64_t)a.m * a.k : 0);
    const int64_t all = c.count * a.tiles_c > zeros ? c.count * a.tiles_c : zeros;
    const cogdl_status st = launch_tiles("grouped_linear_dw", kern, a, all, waves, lds_of(waves, t.tm, t.tn), 2, stream);
    if (st != COGDL_OK || c.slots() == 0) return st;
    // whole vectors of 4 where the matrices and rows of db are
    const int64_t values = (a.out ? (int64_t)a.m * a.k : 0) + (a.db ? a.m : 0);
    const int vec = a.m % 4 == 0 ? 4 : 1;
    const bool by_border = c.count - 1 < a.E;
    const int64_t rows = by_border ? c.count - 1 : a.E;
    int64_t bx = (values + kBlock * vec - 1) / (kBlock * vec);
    bx *= parts_of(c.count);
    const int64_t most = 8192 / rows > 1 ? 8192 / rows : 1;
    if (bx > most) bx = most;
    const dim3 grid((unsigned)bx, (unsigned)rows);
    if (vec == 4) COGDL_LAUNCH("grouped_linear_sum", k_reduce_slices<4>, grid, kBlock, stream, a, by_border);
    else COGDL_LAUNCH("grouped_linear_sum", k_reduce_slices<1>, grid, kBlock, stream, a, by_border);
    return COGDL_OK;
}

}  // namespace cogdl
