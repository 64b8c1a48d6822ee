// The gradients of the grouped products' weights and biases:
//     dW[g, c, j] = sum_{i in g} dZ[i, c] X[i, j],   db[g, c] = sum_{i in g} dZ[i, c]
//
// The sums run over rows, whose number only the device knows: groups are cut into chunks of
// rows; a group of one chunk writes its result, the others write fp32 partial sums into the
// workspace, added up in chunk order by k_reduce_chunks (no atomics: the same bits every run).
#include "grouped_tile.hpp"

namespace cogdl {
namespace {

// dW and db of chunks of a group's rows: TM x TN outputs (c by j) of its matrix at a time.
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
    Walk walk;
    walk.start(a.off, a.E, a.n, a.per, a.tiles_c, true);
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
    run_tiles<T, decltype(A), decltype(B), WR, WC>(lds, walk, A, B, r0, c0, open, each, settle, [&](const Span &s,
                                                                                             const Acc<WR, WC> &acc) {
        const int row0 = s.tile / tiles_k * TM, col0 = s.tile % tiles_k * TN;
        if (a.out) {
            float *__restrict__ part = a.part + (s.slot + s.local) * mk;
            for_outputs<WR, WC>(outs + wave * kOutBytes, acc, [&](int r, int c, float (&v)[8]) {
                r += row0 + r0;
                c += col0 + c0;
                if (r >= a.m || c >= a.k) return;
                if (s.count == 1) store8(a.out, a.out_dtype, s.g * mk + (int64_t)r * a.k, c, a.k, v);
                else store8(part + (int64_t)r * a.k, c, a.k, v);
            });
        }
        if (!sums(s)) return;
        float *__restrict__ db = s.count == 1 ? a.db + (int64_t)s.g * a.m : a.part_db + (s.slot + s.local) * a.m;
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
}

// Sums over a group's partial sums.  Four quarters of the slots, each added up in order by a
// thread of its own with kBatch loads in flight, then the quarters in order.
constexpr int kBlock = 256;
constexpr int kQuarters = 4;
constexpr int kBatch = 8;

// V values from p on in each of the slots [0, count), `stride` floats apart.
template <int V>
__device__ __forceinline__ void sum_slots(const float *__restrict__ p, int64_t stride, int count, float (&t)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = 0.f;
    for (int c = 0; c < count; c += kBatch) {
        float v[kBatch][V];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int at = c + u < count ? c + u : count - 1;
            if constexpr (V == 4) load_vec<float, 4>(p, at * stride, v[u]);
            else v[u][0] = p[at * stride];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) t[e] += c + u < count ? v[u][e] : 0.f;
    }
}

// dW and db of the groups of several chunks (sums of their slots) and of none (zeros).
// Group blockIdx.y, V values a thread of each quarter.
template <int V>
__global__ __launch_bounds__(kBlock) void k_reduce_chunks(GroupedArgs a)
{
    __shared__ float sums[kQuarters][kBlock / kQuarters][V];
    const int g = blockIdx.y, lane = lane_id();
    const int64_t lo = offset_at(a.off, g, a.n), hi = offset_at(a.off, g + 1, a.n);
    const int count = hi > lo ? (int)((hi - lo + a.per - 1) / a.per) : 0;
    if (count == 1) return;
    int64_t slot = 0;
    if (count > 1) {
        for (int e = lane; e < g; e += kWave) {
            const int64_t from = offset_at(a.off, e, a.n), to = offset_at(a.off, e + 1, a.n);
            if (to - from > a.per) slot += (to - from + a.per - 1) / a.per;
        }
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) slot += __shfl_xor(slot, d);
    }
    const int quarter = threadIdx.x / (kBlock / kQuarters), mine = threadIdx.x % (kBlock / kQuarters);
    const int first = count * quarter / kQuarters, end = count * (quarter + 1) / kQuarters;
    const int64_t mk = a.out ? (int64_t)a.m * a.k : 0, all = mk + (a.db ? a.m : 0);
    const int64_t step = (int64_t)gridDim.x * (kBlock / kQuarters) * V;
    for (int64_t i0 = (int64_t)blockIdx.x * (kBlock / kQuarters) * V; i0 < all; i0 += step) {
        const int64_t i = i0 + mine * V;
        float t[V];
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = 0.f;
        if (i < mk) sum_slots<V>(a.part + (slot + first) * mk + i, mk, end - first, t);
        else if (i < all) sum_slots<V>(a.part_db + (slot + first) * a.m + (i - mk), a.m, end - first, t);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) sums[quarter][mine][e] = t[e];
        __syncthreads();
        if (quarter != 0 || i >= all) continue;
#pragma unroll
        for (int q = 1; q < kQuarters; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) t[e] += sums[q][mine][e];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float one[1] = {t[e]};
            if (i >= mk) a.db[(int64_t)g * a.m + (i - mk) + e] = t[e];
            else if (a.out_dtype == COGDL_BF16) store_out<bf16_t, 1>(static_cast<bf16_t *>(a.out), g * mk + i + e, one);
            else if (a.out_dtype == COGDL_F16) store_out<f16_t, 1>(static_cast<f16_t *>(a.out), g * mk + i + e, one);
            else static_cast<float *>(a.out)[g * mk + i + e] = t[e];
        }
    }
}

struct Tiles {
    int tm, tn;
};

template <typename T, int WAVES, int TM, int TN>
GroupedKernel pick(bool act, bool codes, bool direct)
{
    if (act) return codes ? k_grouped_weights<T, WAVES, TM, TN, kSloped, kCodes> : k_grouped_weights<T, WAVES, TM, TN, kSloped, kStaged>;
    if (codes) return k_grouped_weights<T, WAVES, TM, TN, kStaged, kCodes>;
    return direct ? k_grouped_weights<T, WAVES, TM, TN, kDirect, kDirect> : k_grouped_weights<T, WAVES, TM, TN, kStaged, kStaged>;
}

template <typename T>
GroupedKernel pick_tile(const Tiles &c, bool act, bool codes, bool direct)
{
    if (c.tm == 256) return codes ? k_grouped_weights<T, 8, 256, 256, kStaged, kCodes>
                                  : k_grouped_weights<T, 8, 256, 256, kDirect, kDirect>;
    if (c.tm == 128) return c.tn == 128 ? pick<T, 4, 128, 128>(act, codes, direct) : pick<T, 4, 128, 64>(act, codes, direct);
    return c.tn == 128 ? pick<T, 4, 64, 128>(act, codes, direct) : pick<T, 4, 64, 64>(act, codes, direct);
}

int64_t tiles_of(int64_t m, int64_t k, int tm, int tn) { return (m + tm - 1) / tm * (k > 0 ? (k + tn - 1) / tn : 1); }

}  // namespace

// Rows of a piece: a partial sum is written and read once for each, so there are no more pieces
// than make two tiles of 128 x 128 (one of 256 x 256) for each resident workgroup, E groups ending
// in a short one each; 512 rows at least.  A group of several pieces has under 2 n_g / per.
Chunks chunks_of(int64_t n, int32_t E, int32_t k, int32_t m)
{
    Chunks c;
    const int64_t tiles = tiles_of(m, k, m > 64 ? 128 : 64, k > 64 ? 128 : 64);
    const int64_t want = 1024 / (tiles < 1 ? 1 : tiles < 1024 ? tiles : 1024);
    int64_t pieces = want - E > want / 2 ? want - E : want / 2;
    if (pieces < 1) pieces = 1;
    int64_t per = (n + pieces - 1) / pieces;
    per = (per + 63) / 64 * 64;
    if (per < 512) per = 512;
    if (per > (1 << 30)) per = 1 << 30;
    c.per = per;
    c.slots = n > per ? 2 * (n / per) : 0;
    return c;
}

cogdl_status grouped_weights_launch(GroupedArgs a, const Chunks &c, cogdl_dtype dtype, hipStream_t stream)
{
    a.per = (int32_t)c.per;
    if (!a.out) {               // db alone: one column of tiles
        a.k = 0;
        a.X = a.codes = nullptr;
    }
    a.part_db = a.part + (size_t)c.slots * a.m * a.k;
    const bool act = a.act != COGDL_ACT_NONE, codes = a.codes != nullptr;
    if (a.n > 0) {
        const bool direct = a.out && !codes && on_grid(a.dY, a.m) && on_grid(a.X, a.k);
        Tiles t{a.m > 64 ? 128 : 64, a.k > 64 ? 128 : 64};
        if (a.m > 128 && a.k > 128 && !act && (codes || direct)) t = {256, 256};
        const int64_t tiles = tiles_of(a.m, a.k, t.tm, t.tn);
        a.tiles_c = (int32_t)tiles;
        const GroupedKernel kern = dtype == COGDL_BF16 ? pick_tile<bf16_t>(t, act, codes, direct)
                                                       : pick_tile<f16_t>(t, act, codes, direct);
        const cogdl_status st = launch_tiles("grouped_linear_dw", kern, a, most_pieces(a.n, a.E, c.per), t.tm == 256 ? 8 : 4, t.tm,
                                             t.tn, stream);
        if (st != COGDL_OK) return st;
    }
    // whole vectors of 4 where the matrices and rows of db are
    const int64_t values = (a.out ? (int64_t)a.m * a.k : 0) + (a.db ? a.m : 0);
    const int vec = a.m % 4 == 0 ? 4 : 1;
    int64_t bx = (values + kBlock / kQuarters * vec - 1) / (kBlock / kQuarters * vec);
    const int64_t most = 8192 / a.E > 1 ? 8192 / a.E : 1;
    if (bx > most) bx = most;
    const dim3 grid_r((unsigned)bx, (unsigned)a.E);
    if (vec == 4) COGDL_LAUNCH("grouped_linear_sum", k_reduce_chunks<4>, grid_r, kBlock, stream, a);
    else COGDL_LAUNCH("grouped_linear_sum", k_reduce_chunks<1>, grid_r, kBlock, stream, a);
    return COGDL_OK;
}

}  // namespace cogdl
