// Softmax losses over a large vocabulary, backward (the formulas: vocab.hpp): the vocabulary in pieces, for
// each of which the logits are computed again, turned into dz in 16 bits, and multiplied with W (into dX's
// sums) and with X (into the piece's rows of dW).
#include "vocab.hpp"

namespace cogdl {
namespace {

constexpr int kBlock = 256;

// Notes a term of db[v] that is not finite.
__device__ __forceinline__ void note_odd(const VocabArgs &a, int32_t v, float term)
{
    if (fabsf(term) < INFINITY) return;
    const uint32_t bit = term == INFINITY ? kOddPlus : term == -INFINITY ? kOddMinus : kOddNan;
    if (!(a.db_odd[v] & bit)) atomicOr(&a.db_odd[v], bit);
}

// The entries' part of dz (distillation), in fp32 from their log-probabilities: dz = g T (p - sum q), where p may
// be near sum q and dz of it was rounded as g T p.  Several entries of a row on the same answer all write their
// common value.  On the first piece also the entries' part of db, in whole numbers (any order gives the same
// sum).  Those hold no infinity and no NaN, and db's other part has g T p where dz is g T (p - sum q): terms of db
// that are not finite are noted apart, those of an entry (a teacher's NaN or +inf makes its row's q NaN) and, of a row
// whose weight or lse is not finite, dz of every answer (4096 rows by 65536 answers, all of them NaN: 880 us).  A
// wavefront a row, an entry a lane.  4096 rows of 64 entries 16 us, every store a cache line of its own.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_vocab_entries(VocabArgs a)
{
    const int64_t live = a.head->live;
    const float scale = a.head->scale;
    T *__restrict__ dz = static_cast<T *>(a.dz);
    const int64_t waves = (int64_t)gridDim.x * (kBlock / kWave);
    for (int64_t p = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave; p < live; p += waves) {
        const int64_t i = a.rows[p];
        const int32_t *__restrict__ index = a.index + i * a.entries;
        const float *__restrict__ teacher = a.teacher + i * a.entries;
        const float g = a.g[p] * scale;
        const float2 tlse = a.tlse[i];
        for (int e = lane_id(); e < a.entries; e += kWave) {
            const int32_t v = index[e];
            if ((uint32_t)v >= (uint32_t)a.V) continue;
            const bool here = v >= a.v0 && v - a.v0 < a.width, db = a.first && a.db_q;
            if (!here && !db) continue;
            const float mine = expf(log_share(teacher[e], a.T, tlse));
            if (here) {
                float q = 0.f;
                for (int o = 0; o < a.entries; ++o)
                    if (index[o] == v) q += o == e ? mine : expf(log_share(teacher[o], a.T, tlse));
                const float one[1] = {(expf(a.logp_in[i * a.entries + e]) - q) * g};
                store_out<T, 1>(dz + p * a.pitch, v - a.v0, one);
                if (a.db_q) note_odd(a, v, one[0]);
            }
            if (db) {
                const float w = ldexpf(mine * g, a.unit_bits);
                // (2^61 at most where it is finite; else the term is noted as odd)
                if (fabsf(w) < 9e18f) atomicAdd(&a.db_q[v], (unsigned long long)(long long)rintf(w));
            }
        }
        if (!a.db_q || (fabsf(g) < INFINITY && fabsf(a.lse2[p]) < INFINITY)) continue;       // (uniform)
        __threadfence_block();                           // (the entries' dz, by other lanes)
        __builtin_amdgcn_wave_barrier();
        for (int c = lane_id(); c < a.width; c += kWave) {
            float term[1];
            load_vec<T, 1>(dz + p * a.pitch, c, term);
            note_odd(a, a.v0 + c, term[0]);
        }
    }
}

// Those of 8 packed outputs from column c on that lie below width.
template <typename T>
__device__ __forceinline__ void store_packed(T *__restrict__ row, int c, int width, uint4 w)
{
    if (c + 8 <= width) {
        *reinterpret_cast<u32x4_u *>(row + c) = u32x4_u{w.x, w.y, w.z, w.w};
        return;
    }
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < width) row[c + e].bits = (uint16_t)(u[e / 2] >> (16 * (e & 1)));
}

// Both products of a piece, each workgroup's tiles of dX's sums (rows by k, a slice of the piece's columns each),
// then its tiles of dW (vocabulary by k, over the live rows): workgroups that have no tile of the first begin with
// the second.  Bound by the matrix cores: 8192 rows, vocabulary 131072, 1024 features 3750 us in four pieces (1.17
// PFLOP/s; library products of these sizes 1.19); 2867 rows, 40943 x 512, 235 to 250 us (0.96 to 1.02): tiles do not come
// out even.
template <typename T, int WAVES, int TM, int TN, int SRCB>
__global__ __launch_bounds__(WAVES * kWave, 2) void k_vocab_products(VocabArgs a)
{
    constexpr int N = WAVES * kWave;
    constexpr int WAVES_C = TN >= 256 ? 4 : 2, WAVES_R = WAVES / WAVES_C;
    constexpr int WR = TM / WAVES_R / 32, WC = TN / WAVES_C / 32;
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int r0 = wave / WAVES_C * (32 * WR), c0 = wave % WAVES_C * (32 * WC);
    const int live = a.head->live;
    char *const mine = lds + 2 * (TM + TN) * kX * 2 + wave * kOutBytes;
    const auto busy = [&](const Span &s) { return r0 < s.have && s.tile * TN + c0 < a.k; };
    const auto nothing = [](const Span &) {};
    uint32_t block = blockIdx.x;
    GridWalk walk;
    if (a.dX) {
        const int slices = a.head->slices;
        const int cols = (a.width + 7) / 8 * 8, per = ((cols + slices - 1) / slices + kX - 1) / kX * kX;
        walk.start(live, TM, a.tiles_c, slices, block, kPanel, false);
        block = (uint32_t)((block + gridDim.x - (((uint32_t)(walk.R * walk.C) * (uint32_t)slices + 7) / 8 * 8) % gridDim.x) % gridDim.x);
        RowOperand<T, TM, N, kDirect> A;
        ColOperand<T, TN, N, SRCB, false> B;
        const auto open = [&](const Span &s) {
            const int x0 = s.slot * per < cols ? s.slot * per : cols;
            const int wide = cols - x0 < per ? cols - x0 : per;
            const int real = a.width - x0 < wide ? a.width - x0 : wide;
            A.open(static_cast<const T *>(a.dz) + s.lo * a.pitch + x0, nullptr, s.have, a.pitch, 0);
            A.width = wide;
            B.open(static_cast<const T *>(a.W) + ((int64_t)a.v0 + x0) * a.k, nullptr, nullptr, nullptr, s.tile * TN, a.k,
                   real > 0 ? real : 0, 0, false);
            return wide;
        };
        run_tiles<T, decltype(A), decltype(B), WR, WC>(
            lds, walk, A, B, r0, c0, open, busy, [](const Span &, const uint4 (&)[WR]) {}, nothing,
            [&](const Span &s, const Acc<WR, WC> &acc) {
                const int col0 = s.tile * TN + c0;
                if (a.direct) {
                    const float unscale = a.head->unscale;
                    for_rows16<T, WR, WC>(
                        mine, acc,
                        [&](int, int, int, float (&v)[4]) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] *= unscale;
                        },
                        [&](int r, int c, uint4 w) {
                            r += r0;
                            c += col0;
                            if (r < s.have && c < a.k) store_packed(static_cast<T *>(a.dX) + a.rows[s.lo + r] * (int64_t)a.k, c, a.k, w);
                        });
                    return;
                }
                float *__restrict__ part = a.dx_part + (s.slot * a.n + s.lo) * a.kp;
                for_outputs<WR, WC>(mine, acc, [&](int, int r, int c, float (&v)[8]) {
                    r += r0;
                    c += col0;
                    if (r >= s.have || c >= a.kp) return;
                    float *__restrict__ to = part + (int64_t)r * a.kp + c;
                    if (!a.first) {
                        float w[2][4];
                        load_vec<float, 4>(to, 0, w[0]);
                        load_vec<float, 4>(to, 4, w[1]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += w[e / 4][e % 4];
                    }
                    store_vec<float, 8>(to, 0, v);
                });
            });
        __syncthreads();                                 // (the LDS is the next product's)
    }
    if (a.dW) {
        const float unscale = a.head->unscale;
        const int parts = a.plan.parts, per = ((live + parts - 1) / parts + kX - 1) / kX * kX;
        walk.start(a.width, TM, a.tiles_c, parts, block, kPanel, false);
        ColOperand<T, TM, N, kDirect, false> A;
        ColOperand<T, TN, N, kDirect, false> B;
        const auto open = [&](const Span &s) {
            const int x0 = s.slot * per < live ? s.slot * per : live, rows = live - x0 < per ? live - x0 : per;
            A.open(static_cast<const T *>(a.dz) + (int64_t)x0 * a.pitch, nullptr, nullptr, nullptr, (int)s.lo, a.pitch, rows, 0, false);
            B.open(static_cast<const T *>(a.Xr) + (int64_t)x0 * a.kp, nullptr, nullptr, nullptr, s.tile * TN, a.kp, rows, 0, false);
            return rows;
        };
        run_tiles<T, decltype(A), decltype(B), WR, WC>(
            lds, walk, A, B, r0, c0, open, busy, [](const Span &, const uint4 (&)[WR]) {}, nothing,
            [&](const Span &s, const Acc<WR, WC> &acc) {
                const int col0 = s.tile * TN + c0;
                if (parts > 1) {
                    float *__restrict__ part = a.dw_part + ((int64_t)s.slot * a.plan.width + s.lo) * a.kp;
                    for_outputs<WR, WC>(mine, acc, [&](int, int r, int c, float (&v)[8]) {
                        r += r0;
                        c += col0;
                        if (r < s.have && c < a.kp) store_vec<float, 8>(part + (int64_t)r * a.kp, c, v);
                    });
                    return;
                }
                T *__restrict__ dW = static_cast<T *>(a.dW) + (a.v0 + s.lo) * a.k;
                for_rows16<T, WR, WC>(
                    mine, acc,
                    [&](int, int, int, float (&v)[4]) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] *= unscale;
                    },
                    [&](int r, int c, uint4 w) {
                        r += r0;
                        c += col0;
                        if (r < s.have && c < a.k) store_packed(dW + (int64_t)r * a.k, c, a.k, w);
                    });
            });
    }
}

// db's sums over kJoin row tiles each, where there are many: 64 columns a workgroup, 4 parts of them.  1821 row tiles
// of 41 columns 7 us, and vocab_out, whose one workgroup had read them all, 139 -> 27.
constexpr int kJoin = 64, kManyTiles = 256;

__global__ __launch_bounds__(kBlock) void k_vocab_db(VocabArgs a, int rows_a_part)
{
    __shared__ float sums[kBlock];
    const int64_t live = a.head->live;
    const int parts = (int)((live + rows_a_part - 1) / rows_a_part);
    const int c = (int)blockIdx.y * kWave + lane_id(), q = threadIdx.x / kWave;
    const int from = (int)blockIdx.x * kJoin + q * (kJoin / 4);
    float t = 0.f;
    if (c < a.width) {
#pragma unroll
        for (int p = 0; p < kJoin / 4; ++p) t += from + p < parts ? a.db_part[(int64_t)(from + p) * a.pitch + c] : 0.f;
    }
    sums[threadIdx.x] = t;
    __syncthreads();
    if (q == 0 && c < a.width)
        a.db_join[(int64_t)blockIdx.x * a.pitch + c] = ((t + sums[threadIdx.x + kWave]) + sums[threadIdx.x + 2 * kWave]) + sums[threadIdx.x + 3 * kWave];
}

// 8 values' sums over slots, `stride` floats apart.
__device__ __forceinline__ void sum_slots(const float *__restrict__ from, int64_t stride, int slots, float unscale, float (&t)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = 0.f;
#pragma unroll 4
    for (int s = 0; s < slots; ++s) {
        float w[2][4];
        load_vec<float, 4>(from, s * stride, w[0]);
        load_vec<float, 4>(from, s * stride + 4, w[1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] += w[e / 4][e % 4];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] *= unscale;
}

// The piece's db from the row tiles' sums and the entries' part (`db_blocks` workgroups from `dx_blocks` on), its dW from
// its parts' sums (those behind), and, with the last piece, dX of the live rows from their slices' sums.  Bound by
// memory: 8192 x 1024 of two slices 20 us (4.3 TB/s).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_vocab_out(VocabArgs a, int dx_blocks, int db_blocks, int rows_a_part)
{
    const int64_t live = a.head->live;
    const float unscale = a.head->unscale;
    if ((int)blockIdx.x >= dx_blocks + db_blocks) {
        const int vecs = a.kp / 8;
        const int64_t all = (int64_t)a.width * vecs, from = (int64_t)(blockIdx.x - dx_blocks - db_blocks) * kBlock + threadIdx.x;
        for (int64_t u = from; u < all; u += (int64_t)(gridDim.x - dx_blocks - db_blocks) * kBlock) {
            const int64_t r = u / vecs;
            const int c = (int)(u % vecs) * 8;
            float t[8];
            sum_slots(a.dw_part + r * a.kp + c, (int64_t)a.plan.width * a.kp, a.plan.parts, unscale, t);
            store8(static_cast<T *>(a.dW) + (a.v0 + r) * a.k, c, a.k, t);
        }
        return;
    }
    if ((int)blockIdx.x >= dx_blocks) {
        const bool joined = a.row_tiles > kManyTiles;
        const int rows = joined ? rows_a_part * kJoin : rows_a_part, parts = (int)((live + rows - 1) / rows);
        const float *__restrict__ part = joined ? a.db_join : a.db_part;
        const int c = (int)(blockIdx.x - dx_blocks) * kBlock + (int)threadIdx.x;
        if (c >= a.width) return;
        float t = 0.f;
#pragma unroll 8
        for (int p = 0; p < parts; ++p) t += part[(int64_t)p * a.pitch + c];
        if (a.db_q) {
            t = (float)((double)t - ldexp((double)(long long)a.db_q[a.v0 + c], -a.unit_bits));
            const uint32_t odd = a.db_odd[a.v0 + c];
            if (odd) t = odd == kOddPlus ? INFINITY : odd == kOddMinus ? -INFINITY : NAN;
        }
        a.db[a.v0 + c] = t * unscale;
        return;
    }
    const int vecs = a.kp / 8, slices = a.head->slices;
    const int64_t all = live * vecs;
    for (int64_t u = (int64_t)blockIdx.x * kBlock + threadIdx.x; u < all; u += (int64_t)dx_blocks * kBlock) {
        const int64_t p = u / vecs;
        const int c = (int)(u % vecs) * 8;
        float t[8];
        sum_slots(a.dx_part + p * a.kp + c, a.n * a.kp, slices, unscale, t);
        store8(static_cast<T *>(a.dX) + a.rows[p] * (int64_t)a.k, c, a.k, t);
    }
}

template <typename T>
VocabKernel pick_products(bool wide, bool direct)
{
    if (wide) return k_vocab_products<T, 8, 256, 256, kDirect>;
    return direct ? k_vocab_products<T, 4, 128, 128, kDirect> : k_vocab_products<T, 4, 128, 128, kStaged>;
}

int64_t tiles_of(int64_t rows, int64_t cols, int tile) { return (rows + tile - 1) / tile * ((cols + tile - 1) / tile); }

// The columns of a piece: its dz takes at most so many bytes (and 256 columns at least).  With 256 MB, 512 and 1024,
// loss and gradients: 8192 rows, vocabulary 131072, 1024 features 8000, 7900 and 7900 us; 4096 rows, 65536 x 768, 1730,
// 1623 and 1625.
constexpr int64_t kPieceBytes = 512ll << 20;

// Parts of the rows that dW of a piece is summed in: many rows and few classes make few tiles, each a sum over all
// rows.  As many as the chip holds tiles, of 1024 rows or more.  232965 rows, 41 classes, 128 features: the products
// 3248 us with one part, 46 so.
int32_t dw_parts(int64_t n, int32_t width, int32_t k, int tile)
{
    const int64_t tiles = tiles_of(width, k, tile), want = tile == 256 ? 256 : 512;
    int64_t parts = tiles > 0 ? want / tiles : 1;
    if (parts > n / 1024) parts = n / 1024;
    return (int32_t)(parts < 1 ? 1 : parts);
}

// The plan of a piece's products with tiles of 256 x 256 or of 128 x 128, whichever ends first.
void plan_products(ProductsPlan &p, int64_t n, const void *W)
{
    p.parts = 1;
    float best[2];
    for (int wide = 0; wide < 2; ++wide) {
        p.tile = wide ? 256 : 128;
        p.resident = wide ? 32 : 64;
        best[wide] = p.cost((int32_t)n, 1);
        for (int s = 2; s <= p.most; ++s) best[wide] = fminf(best[wide], p.cost((int32_t)n, s));
    }
    const bool wide = on_grid(W, p.k) && p.k > 128 && best[1] * kWideChunk < best[0] * kNarrowChunks;
    p.tile = wide ? 256 : 128;
    p.resident = wide ? 32 : 64;
    if (p.dw) p.parts = dw_parts(n, p.width, p.k, p.tile);
}

int32_t piece_width(int64_t n, int32_t V)
{
    int64_t cols = kPieceBytes / (2 * (n > 0 ? n : 1)) / 256 * 256;
    if (cols < 256) cols = 256;
    if (cols > kMaxWidth) cols = kMaxWidth;
    const int64_t count = (V + cols - 1) / cols;
    const int64_t width = ((V + count - 1) / count + 255) / 256 * 256;
    return (int32_t)(width < V ? width : V);
}

// Slices of 256 columns or more, and no more than make 1024 tiles of dX.
int32_t most_slices(int64_t n, int32_t width, int32_t k)
{
    const int64_t tiles = tiles_of(n, k, 128);
    int64_t most = tiles > 0 ? (1024 + tiles - 1) / tiles : 1;
    if (most > width / 256) most = width / 256;
    if (most > kMostSlices) most = kMostSlices;
    return (int32_t)(most < 1 ? 1 : most);
}

size_t lay_backward(VocabArgs &a, char *ws)
{
    a.width = piece_width(a.n, a.V);
    a.pitch = (int32_t)odd_pitch(a.width);
    a.plan.most = most_slices(a.n, a.width, a.k);
    a.row_tiles = (int32_t)((a.n + 127) / 128 * 2);
    const size_t n = (size_t)a.n;
    Layout l;
    a.head = reinterpret_cast<RowsHead *>(ws + l.take(sizeof(RowsHead)));
    a.live = reinterpret_cast<int32_t *>(ws + l.take(a.distill ? 4 * n : 0));
    a.tlse = reinterpret_cast<float2 *>(ws + l.take(a.distill ? 8 * n : 0));
    a.counts = reinterpret_cast<int32_t *>(ws + l.take(a.n > kManyRows ? 4 * kMostRuns : 0));
    a.tops = reinterpret_cast<float *>(ws + l.take(a.n > kManyRows ? 4 * kMostRuns : 0));
    a.rows = reinterpret_cast<int32_t *>(ws + l.take(4 * n));
    a.lse2 = reinterpret_cast<float *>(ws + l.take(4 * n));
    a.g = reinterpret_cast<float *>(ws + l.take(4 * n));
    a.col = reinterpret_cast<int32_t *>(ws + l.take(a.distill ? 0 : 4 * n));
    a.at_col = reinterpret_cast<float *>(ws + l.take(a.distill ? 0 : 4 * n));
    a.Xr = ws + l.take(2 * n * a.kp);
    a.dz = ws + l.take(2 * n * a.pitch);
    a.direct = a.width == a.V && a.plan.most == 1;
    a.dx_part = reinterpret_cast<float *>(ws + l.take(a.direct ? 0 : 4 * n * a.kp * a.plan.most));
    const int32_t small = dw_parts(a.n, a.width, a.k, 128), large = dw_parts(a.n, a.width, a.k, 256);
    const int32_t parts = small > large ? small : large;           // (which tiles, W's alignment decides)
    a.dw_part = reinterpret_cast<float *>(ws + l.take(parts > 1 ? 4 * (size_t)parts * a.width * a.kp : 0));
    a.db_part = reinterpret_cast<float *>(ws + l.take(4 * (size_t)a.row_tiles * a.pitch));
    a.db_join = reinterpret_cast<float *>(ws + l.take(a.row_tiles > kManyTiles ? 4 * (size_t)((a.row_tiles + kJoin - 1) / kJoin) * a.pitch : 0));
    a.db_q = reinterpret_cast<unsigned long long *>(ws + l.take(a.distill ? 8 * (size_t)a.V : 0));
    a.db_odd = reinterpret_cast<uint32_t *>(ws + l.take(a.distill ? 4 * (size_t)a.V : 0));
    return l.total;
}

#define COGDL_TRY(expr)                              \
    do {                                             \
        const cogdl_status _s = (expr);              \
        if (_s != COGDL_OK) return _s;               \
    } while (0)

cogdl_status run_backward(VocabArgs a, cogdl_dtype dtype, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (dtype != COGDL_BF16 && dtype != COGDL_F16) return COGDL_ERR_DTYPE;
    COGDL_TRY(check_sizes(a));
    if (a.n > 0 && (!a.index || !a.dloss || !a.lse_in || (a.k > 0 && (!a.X || !a.W)))) return COGDL_ERR_INVALID;
    if (a.n > 0 && (a.distill ? !a.teacher || !a.logp_in : !a.loss_in)) return COGDL_ERR_INVALID;
    if (a.k == 0) a.dX = a.dW = nullptr;
    if (a.n == 0) a.dX = nullptr;
    if (!a.dX && !a.dW && !a.db) return COGDL_OK;
    a.kp = (a.k + 7) / 8 * 8;
    a.per_z = kLog2e / a.T;
    const size_t need = lay_backward(a, static_cast<char *>(workspace));
    if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < need) return COGDL_ERR_INVALID;
    const int piece = a.width;
    if (!a.db) a.db_part = nullptr;
    if (!a.db || !a.distill) a.db_q = nullptr;
    // n terms below 2^15, in 62 bits
    a.unit_bits = 46 - bits_for((uint64_t)a.n);
    const bool bf16 = dtype == COGDL_BF16;
    const bool wide_logits = vocab_wide(a.n, piece, a.k, a.W);
    a.plan.width = piece;
    a.plan.k = a.k;
    a.plan.dx = a.dX != nullptr;
    a.plan.dw = a.dW != nullptr;
    plan_products(a.plan, a.n, a.W);
    const int tile = a.plan.tile, waves = tile == 256 ? 8 : 4;
    const bool wide = tile == 256;
    COGDL_TRY(vocab_rows_launch(a, dtype, true, stream));
    for (int64_t v0 = 0; v0 < a.V; v0 += piece) {
        a.v0 = (int32_t)v0;
        a.width = (int32_t)(a.V - v0 < piece ? a.V - v0 : piece);
        a.first = v0 == 0;
        if (a.n > 0) {
            COGDL_TRY(vocab_logits_launch(a, dtype, true, wide_logits, stream));
            if (a.distill) {
                const int64_t blocks = (a.n * kWave + kBlock - 1) / kBlock;
                const unsigned grid = (unsigned)(blocks < 2048 ? blocks : 2048);
                if (bf16) COGDL_LAUNCH("vocab_entries", k_vocab_entries<bf16_t>, grid, kBlock, stream, a);
                else COGDL_LAUNCH("vocab_entries", k_vocab_entries<f16_t>, grid, kBlock, stream, a);
            }
        }
        if (a.dX || a.dW) {
            a.tiles_c = (a.k + tile - 1) / tile;
            const int64_t tiles = (a.dX ? tiles_of(a.n, a.k, tile) * a.plan.most : 0) + (a.dW ? tiles_of(a.width, a.k, tile) * a.plan.parts : 0);
            COGDL_TRY(launch_vocab("vocab_products", bf16 ? pick_products<bf16_t>(wide, on_grid(a.W, a.k)) : pick_products<f16_t>(wide, on_grid(a.W, a.k)),
                                   a, tiles, waves, lds_of(waves, tile, tile), stream));
        }
        if (a.db && a.row_tiles > kManyTiles)
            COGDL_LAUNCH("vocab_db", k_vocab_db, dim3((unsigned)((a.row_tiles + kJoin - 1) / kJoin), (unsigned)((a.width + kWave - 1) / kWave)),
                         kBlock, stream, a, wide_logits ? 128 : 64);
        const bool last = a.V - v0 <= piece;
        int64_t dx_blocks = a.dX && last && !a.direct ? (a.n * (a.kp / 8) + kBlock - 1) / kBlock : 0;
        if (dx_blocks > 4096) dx_blocks = 4096;
        const int db_blocks = a.db ? (a.width + kBlock - 1) / kBlock : 0;
        int64_t dw_blocks = a.dW && a.plan.parts > 1 ? ((int64_t)a.width * (a.kp / 8) + kBlock - 1) / kBlock : 0;
        if (dw_blocks > 4096) dw_blocks = 4096;
        const unsigned grid = (unsigned)(dx_blocks + db_blocks + dw_blocks);
        if (grid == 0) continue;
        if (bf16) COGDL_LAUNCH("vocab_out", k_vocab_out<bf16_t>, grid, kBlock, stream, a, (int)dx_blocks, db_blocks, wide_logits ? 128 : 64);
        else COGDL_LAUNCH("vocab_out", k_vocab_out<f16_t>, grid, kBlock, stream, a, (int)dx_blocks, db_blocks, wide_logits ? 128 : 64);
    }
    return COGDL_OK;
}

}  // namespace
}  // namespace cogdl

using namespace cogdl;

extern "C" {

cogdl_status cogdl_linear_loss_backward_workspace(int64_t n, int32_t V, int32_t k, int32_t K, size_t *bytes)
{
    if (!bytes || K < 0) return COGDL_ERR_INVALID;
    VocabArgs a{};
    a.n = n; a.V = V; a.k = k;
    a.entries = K > 0 ? K : 1;
    a.distill = K > 0;
    a.T = 1.f;
    COGDL_TRY(check_sizes(a));
    a.kp = (k + 7) / 8 * 8;
    *bytes = lay_backward(a, nullptr);
    return COGDL_OK;
}

cogdl_status cogdl_linear_cross_entropy_backward(int64_t n, int32_t V, int32_t k, const float *dloss, const void *X,
                                                 const void *W, cogdl_dtype dtype, const float *bias,
                                                 const int32_t *target, const float *loss, const float *lse, void *dX,
                                                 void *dW, float *db, void *workspace, size_t workspace_bytes,
                                                 hipStream_t stream)
{
    VocabArgs a{};
    a.n = n; a.V = V; a.k = k;
    a.entries = 1;
    a.T = 1.f;
    a.X = X; a.W = W;
    a.bias = bias;
    a.index = target;
    a.dloss = dloss;
    a.loss_in = loss; a.lse_in = lse;
    a.dX = dX; a.dW = dW; a.db = db;
    return run_backward(a, dtype, workspace, workspace_bytes, stream);
}

cogdl_status cogdl_linear_distill_backward(int64_t n, int32_t V, int32_t k, int32_t K, const float *dloss, const void *X,
                                           const void *W, cogdl_dtype dtype, const float *bias, const int32_t *index,
                                           const float *teacher, float temperature, const float *lse, const float *logp,
                                           void *dX, void *dW, float *db, void *workspace, size_t workspace_bytes,
                                           hipStream_t stream)
{
    VocabArgs a{};
    a.n = n; a.V = V; a.k = k;
    a.entries = K;
    a.distill = true;
    a.T = temperature;
    a.X = X; a.W = W;
    a.bias = bias;
    a.index = index;
    a.teacher = teacher;
    a.dloss = dloss;
    a.lse_in = lse; a.logp_in = logp;
    a.dX = dX; a.dW = dW; a.db = db;
    return run_backward(a, dtype, workspace, workspace_bytes, stream);
}

}  // extern "C"
