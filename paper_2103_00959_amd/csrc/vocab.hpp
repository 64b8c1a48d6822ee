// The softmax losses over a large vocabulary (vocab.hip, vocab_grad.hip): what their launches share.
//
//     z[i, v] = sum_j X[i, j] W[v, j] + bias[v],   lse[i] = log sum_v exp(z[i, v] / T)
//     cross entropy:  loss[i] = lse[i] - z[i, t_i]                                   (T = 1)
//     distillation:   loss[i] = T^2 sum_e q[i, e] (log q[i, e] - logp[i, e])
//                     logp[i, e] = z[i, v_ie] / T - lse[i],  q[i, :] = softmax(teacher[i, :] / T)
//     dz[i, v] = g[i] T (exp(z[i, v] / T - lse[i]) - sum_{e: v_ie = v} q[i, e]),  dX = dz W,  dW = dz^T X
//
// Logits are never kept.  Rows that count (a target inside the vocabulary, a teacher's entry) are gathered
// first, so that padded rows cost nothing and what they hold reaches no sum: every product below runs over
// `live` rows, a number that only the device knows.
#pragma once

#include "grouped_tile.hpp"

namespace cogdl {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// Most entries of a teacher's row.
constexpr int kMaxEntries = COGDL_MAX_TEACHER;
// Slices of dX's sums over a piece, at most.
constexpr int kMostSlices = 64;
// Rows of one call.
constexpr int64_t kMaxRows = 1 << 24;

// Runs that many rows are counted in before they are gathered.
constexpr int kMostRuns = 4096;
// Terms of a sum that are not finite, together: any two of them make NaN.
constexpr uint32_t kOddPlus = 1, kOddMinus = 2, kOddNan = 4;
constexpr int64_t kManyRows = 16384;

// Header of a workspace, written by k_vocab_rows.
struct RowsHead {
    int32_t live;                // rows that count
    float scale, unscale;        // |g T| scale <= 2^15 for every live row where it is finite, and 1 / scale
    int32_t slices;              // of dX's sums over a piece
};

// The two products of a piece as tiles of tile x tile on `resident` workgroups of each XCD, one after another: dX's
// sums (rows x k, a slice of the piece's `width` columns each), then dW (width x k, summed over the rows, a part of
// `parts` each).  The time of the busiest workgroup where dX's sums are cut into s slices, in chunks of 64: a tile
// costs its chunks and kTileStart more, dX's kTileSums besides (its sums go to memory in fp32).  4096 rows, 30% of
// them padded, 40943 x 512 fp16: the products in launches of their own, slices by the rows given, 319 us, together by
// the rows that count 270 (both before rows of dz lay apart as odd_pitch has them; 235 to 250 since).
constexpr int kTileStart = 4, kTileSums = 2;

struct ProductsPlan {
    int32_t tile, resident, width, k, most, parts;
    bool dx, dw;

    // (in floats: sizes are far apart, and no whole number has to come out)
    __host__ __device__ __forceinline__ float cost(int32_t live, int32_t s) const
    {
        const float tr = (float)((live + tile - 1) / tile), tk = (float)((k + tile - 1) / tile), tw = (float)((width + tile - 1) / tile);
        const float n1 = dx ? ceilf(tr * tk * s * 0.125f) : 0.f, n2 = dw ? ceilf(tw * tk * parts * 0.125f) : 0.f, each = 1.f / resident;
        const float c1 = ceilf((float)width / (64.f * s)) + kTileStart + kTileSums, c2 = ceilf((float)live / (64.f * parts)) + kTileStart;
        // workgroup w of the XCD has the tiles w, w + resident, ... of n1 + n2: the most of it at the first, and at
        // the first that begins with dW
        float most_of = 0.f;
        for (int h = 0; h < 2; ++h) {
            const float w = h == 0 ? 0.f : n1 - floorf(n1 * each) * resident;
            const float all = ceilf((n1 + n2 - w) * each), of_dx = n1 > w ? ceilf((n1 - w) * each) : 0.f;
            most_of = fmaxf(most_of, of_dx * c1 + fmaxf(all - of_dx, 0.f) * c2);
        }
        return most_of + s * tr * tk * each * (1.f / 16);       // (what the sum over slices reads)
    }
};

struct VocabArgs {
    int64_t n;                   // rows given
    int32_t V, k, kp;            // kp: k rounded up to 8
    int32_t entries;             // of a row: 1 (cross entropy), K (distillation)
    bool distill;
    bool plain;                  // the rows as they were given stand for the gathered ones (few of them, forward)
    float T, per_z;              // per_z = log2(e) / T
    const void *X, *W;
    const float *bias;           // V, nullable
    const int32_t *index;        // n x entries
    const float *teacher;        // n x entries (distillation)
    const float *dloss;          // n (backward)
    const float *loss_in, *lse_in, *logp_in;
    float *loss, *lse, *logp;
    void *dX, *dW;
    float *db;
    // workspace
    RowsHead *head;
    int32_t *live;               // n: >= 0 where the row counts (distillation; else the targets are read)
    float2 *tlse;                // n: the largest teacher / T, and the log of the sum of exp over it (distillation)
    int32_t *counts;             // [kMostRuns]: rows that count in each run of rows (many rows)
    float *tops;                 // [kMostRuns]: their largest |g T| (backward)
    int32_t *rows;               // live: the rows that count
    float *lse2, *g;             // live: lse log2(e), g T
    int32_t *col;                // live: the target (cross entropy)
    float *at_col;               // live: g (p - 1) there
    void *Xr;                    // live x kp: their features, zeros from k on
    float2 *part;                // [slot][block]: (max, sum) of a row's logits in a slot of columns, in powers of two
    int32_t slots;
    int32_t block;               // rows whose statistics are kept at once
    int64_t p0;                  // the first of them
    void *dz;                    // live x pitch: scaled by head->scale, zeros from width to the next multiple of 8
    float *dx_part;              // [slice][live][kp]
    ProductsPlan plan;           // (backward)
    float *db_part;              // [row tile][pitch]: a piece's
    float *db_join;              // [kJoin row tiles][pitch] (many row tiles)
    int32_t row_tiles;
    unsigned long long *db_q;    // V: the entries' part of db, in units of 2^-unit_bits (distillation)
    uint32_t *db_odd;            // V: what of db is not finite, kOdd... (distillation)
    int32_t unit_bits;
    // this launch
    int32_t v0, width;           // the vocabulary piece [v0, v0 + width)
    int32_t pitch;               // of dz
    int32_t tiles_c;             // column tiles of the logits, of both products
    float *dw_part;              // [part][piece's width][kp] (more than one part)
    bool first;                  // the first piece
    bool direct;                 // dX leaves the products as it is: one piece, one slice
};

// log q of a teacher's logit: the two parts of its row's log sum apart, which one float would round by more than
// the loss can be told to (4096 rows of 64 entries: 6e-7 of it, so 1e-7).
__device__ __forceinline__ float log_share(float teacher, float T, float2 of_row) { return (teacher / T - of_row.x) - of_row.y; }

// Sizes and temperature of a call.  (Temperatures past 2^20 either way: logits over them leave fp32's range.)
inline cogdl_status check_sizes(const VocabArgs &a)
{
    if (a.n < 0 || a.V < 1 || a.k < 0 || a.entries < 1) return COGDL_ERR_INVALID;
    if (!(a.T >= 1.f / (1 << 20) && a.T <= (float)(1 << 20))) return COGDL_ERR_INVALID;
    if (a.n > kMaxRows || a.k > kMaxWidth || a.entries > kMaxEntries) return COGDL_ERR_TOO_LARGE;
    const int64_t tr = (a.n + 127) / 128, tv = ((int64_t)a.V + 127) / 128, tk = ((int64_t)a.k + 127) / 128;
    return countable(tr, tv) && countable(tr, tk) && countable(tv, tk) ? COGDL_OK : COGDL_ERR_TOO_LARGE;
}

// Parts of a workspace, one after another on 256 bytes.
struct Layout {
    size_t total = 0;
    size_t take(size_t bytes)
    {
        const size_t at = total;
        total += (bytes + 255) & ~size_t(255);
        return at;
    }
};

using VocabKernel = void (*)(VocabArgs);

// The tiles of one output of R x C tiles (R >= 0, known on the device), S slices of the sum each.  Tiles are
// numbered slice by slice, then in panels of so many row tiles, in a panel column by column; the XCDs take equal runs
// of them, their workgroups one after another: those that run together on an XCD take a panel's rows of tiles by a
// few columns, and share both operands in its L2.  TURNED: each XCD begins an eighth of its run further on than the
// one before.  Those that go through the same columns side by side store to the same channels of the memory: dz of
// 8192 x 131072 logits, 1024 features, 2390 us, turned 2110.  The statistics store little (1920 us, turned 1905), and so
// do the products.
constexpr int kPanel = 4;

struct GridWalk {
    int R, C, tm, tallest;
    int64_t rows;
    uint32_t j, step, end;       // the next tile in the XCD's own order, the way to the one after, its tiles
    uint32_t first, turn;        // the XCD's first tile, and where in its run it begins

    // `block`: this workgroup's number among those of the grid.
    __device__ __forceinline__ void start(int64_t n, int rows_a_tile, int col_tiles, int slices, uint32_t block, int panel, bool turned)
    {
        tallest = panel;
        rows = n;
        tm = rows_a_tile;
        R = (int)((n + tm - 1) / tm);
        C = col_tiles;
        const int64_t all = (int64_t)R * C * slices;
        const uint32_t xcd = block & 7;
        first = (uint32_t)(all * xcd / 8);
        end = (uint32_t)(all * (xcd + 1) / 8) - first;
        turn = turned ? (uint32_t)((uint64_t)end * xcd / 8) : 0;
        j = block >> 3;
        step = gridDim.x >> 3;
    }
    __device__ __forceinline__ bool next(Span &s)
    {
        if (j >= end) return false;
        const uint32_t one = (uint32_t)R * (uint32_t)C;
        const uint32_t at = first + (j + turn < end ? j + turn : j + turn - end);
        const uint32_t slice = at / one, u = at % one;
        j = end - j > step ? j + step : end;
        const uint32_t panel = u / (uint32_t)(tallest * C), w = u % (uint32_t)(tallest * C);
        const int left = R - (int)panel * tallest, tall = left < tallest ? left : tallest;
        s.g = (int)panel * tallest + (int)(w % (uint32_t)tall);          // row tile
        s.tile = (int)(w / (uint32_t)tall);
        s.slot = (int)slice;
        s.lo = (int64_t)s.g * tm;
        s.have = rows - s.lo < tm ? (int)(rows - s.lo) : tm;
        return true;
    }
};

// The lane's number as the outputs of a tile use it: what follows from it is computed anew for each tile, and takes
// no registers from the products (hoisted out of the loop over tiles, it made 256 x 256 tiles spill).
__device__ __forceinline__ int lane_of_outputs()
{
    int lane = lane_id();
    asm volatile("" : "+v"(lane));
    return lane;
}

// A wavefront's 16-bit outputs, 64 columns of them: calls map(row block, column block, g, v) for its outputs four at a
// time, of row lane % 32 and columns 8 g + 4 (lane / 32) ... + 3 of the block, rounds them, and calls out(row, column,
// w) for 8 of a row as 16 bytes, through the wavefront's part of the LDS: eight neighbouring lanes then hold a row's 128
// bytes, a whole cache line.  (dz of 8192 x 131072 logits, 1024 features, not turned, 2440 us; straight from the
// accumulators, 32 bytes of a row at a time, 2990.)
template <typename T, int WR, int WC, typename Map, typename Out>
__device__ __forceinline__ void for_rows16(char *mine, const Acc<WR, WC> &acc, Map map, Out out)
{
    static_assert(WC == 2 && 32 * 64 * 2 == kOutBytes, "32 rows of 64 columns");
    const int lane = lane_of_outputs(), r = lane & 31, hi = lane >> 5;
#pragma unroll
    for (int i = 0; i < WR; ++i) {
#pragma unroll
        for (int j = 0; j < WC; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float v[4] = {acc.a[i][j][4 * g], acc.a[i][j][4 * g + 1], acc.a[i][j][4 * g + 2], acc.a[i][j][4 * g + 3]};
                map(i, j, g, v);
                // (the 16-byte pieces of a row permuted by the row)
                *reinterpret_cast<uint2 *>(mine + r * 128 + (((4 * j + g) ^ (r & 7)) << 4) + 8 * hi) =
                    make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int row = 8 * u + (lane >> 3), piece = lane & 7;
            out(32 * i + row, 8 * piece, *reinterpret_cast<const uint4 *>(mine + row * 128 + ((piece ^ (row & 7)) << 4)));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// The pitch of rows of `cols` 16-bit elements: an odd number of 256 bytes, so that the rows of a tile start on
// different channels of the memory.  (4096 rows, 30% of them padded, 40943 x 512 fp16, between events: dz 173 us, so
// 168; the products 258 and 255.)
inline int64_t odd_pitch(int64_t cols)
{
    const int64_t lines = (cols + 127) / 128;
    return (lines | 1) * 128;
}

// Launches a kernel of resident workgroups over at most `all` tiles.
inline cogdl_status launch_vocab(const char *name, VocabKernel kern, const VocabArgs &a, int64_t all, int waves, size_t lds,
                                 hipStream_t stream)
{
    const int64_t resident = resident_blocks(reinterpret_cast<const void *>(kern), waves * kWave, lds, 0) / 8;
    if (resident < 1) return COGDL_ERR_LAUNCH;
    const int64_t need = (all + 7) / 8;
    COGDL_LAUNCH_SHM(name, kern, dim3((unsigned)(8 * (need < resident ? need : resident))), waves * kWave, lds, stream, a);
    return COGDL_OK;
}

// The rows that count, gathered (and, for a backward pass, the gradients of the others zeroed).
cogdl_status vocab_rows_launch(const VocabArgs &a, cogdl_dtype dtype, bool backward, hipStream_t stream);
// The logits: their (max, sum) by slots of columns, or the piece's dz.
cogdl_status vocab_logits_launch(VocabArgs a, cogdl_dtype dtype, bool grad, bool wide, hipStream_t stream);

// Time of a chunk of 64 for a compute unit, us: a tile of 256 x 256, or two of 128 x 128 (one alone).
constexpr float kWideChunk = 1.85f, kNarrowChunks = 1.23f, kNarrowChunk = 0.75f;

// Whether the logits of n rows by `cols` columns take tiles of 256 x 256 (else 128 x 128).
bool vocab_wide(int64_t n, int64_t cols, int32_t k, const void *W);

}  // namespace cogdl
