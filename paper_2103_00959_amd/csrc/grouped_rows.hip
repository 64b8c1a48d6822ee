// Products of rows that lie sorted by group (node types, relations, experts), each group
// with a weight matrix of its own, and the gradient of their input:
//     Y[i, c]  = act(sum_j X[i, j] W[g, c, j] + bias[g, c])        rows i of group g
//     dX[i, j] = sum_c dZ[i, c] W[g, c, j]                          dZ = dY act'(Y)
// The offsets stay on the device: each of the resident workgroups finds its tiles' groups by a scan of
// the group sizes.
#include "grouped_tile.hpp"

namespace cogdl {
namespace {

// WAVES wavefronts, tiles of TM rows by TN columns; DX: the gradient.  The operands from SRC, SRCB.
// Bound by the matrix cores' clock where both widths are large: one group of 32768 rows, 2048 ->
// 2048 bf16, 263 us (1.05 PFLOP/s; a large library product reaches 1.43), 229 without the loads
// from memory and 211 without the reads of LDS too.  64 groups of 280 to 2244 rows there: 375, a quarter of
// the tiles' rows are no group's.  Bound by memory elsewhere: 2.5M rows of 90 groups, 64 -> 64, fp16
// to fp32, 183 us (5.2 TB/s); dX of 2.4M rows, 128 -> 256, 378 us (4.9 TB/s); rows of 602 bf16 start
// off the cache lines: 232965 of them to 128 outputs 120 us (2.8 TB/s).  dX under an activation forms dZ from dY
// and Y anew for each tile, through registers: ReLU 649 us and ELU 690 for those 378, 600k rows of 256 267 and 285
// (150 without).
template <typename T, int WAVES, int TM, int TN, bool DX, int SRC, int SRCB>
__global__ __launch_bounds__(WAVES * kWave) void k_grouped_rows(GroupedArgs a)
{
    constexpr int N = WAVES * kWave;
    constexpr int WAVES_C = TN >= 256 ? 4 : TN >= 128 ? 2 : 1, WAVES_R = WAVES / WAVES_C;
    constexpr int WR = TM / WAVES_R / 32, WC = TN / WAVES_C / 32;
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int r0 = wave / WAVES_C * (32 * WR), c0 = wave % WAVES_C * (32 * WC);
    const int wx = DX ? a.m : a.k;                      // x
    const int wc = DX ? a.k : a.m;                      // outputs of a row
    PieceWalk walk;
    walk.start(a.off, a.E, a.n, TM, a.tiles_c);
    RowOperand<T, TM, N, SRC> A;
    std::conditional_t<DX, ColOperand<T, TN, N, SRCB, false>, RowOperand<T, TN, N, SRCB>> B;
    const auto open = [&](const Span &s) {
        const T *__restrict__ W = static_cast<const T *>(a.W) + (int64_t)s.g * a.m * a.k;
        const int col0 = s.tile * TN;
        A.open(static_cast<const T *>(DX ? a.dY : a.X) + s.lo * wx,
               SRC == kSloped ? static_cast<const T *>(a.Y) + s.lo * wx : nullptr, s.have, wx, a.act);
        if constexpr (DX) B.open(W, nullptr, nullptr, nullptr, col0, a.k, a.m, 0, false);
        else B.open(W + (int64_t)col0 * a.k, nullptr, a.m - col0 < TN ? a.m - col0 : TN, a.k, 0);
        return wx;
    };
    char *const mine = lds + 2 * (TM + TN) * kX * 2 + wave * kOutBytes;
    run_tiles<T, decltype(A), decltype(B), WR, WC>(
        lds, walk, A, B, r0, c0, open, [&](const Span &s) { return r0 < s.have && s.tile * TN + c0 < wc; },
        [](const Span &, const uint4 (&)[WR]) {}, [](const Span &) {},
        [&](const Span &s, const Acc<WR, WC> &acc) {
            const int col0 = s.tile * TN + c0;
            const float *__restrict__ bias = !DX && a.bias ? a.bias + (int64_t)s.g * a.m : nullptr;
            // a lane's columns are the same in every row
            float add[DX ? 1 : WC][8];
            if constexpr (!DX) {
#pragma unroll
                for (int bc = 0; bc < WC; ++bc)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int c = col0 + 32 * bc + 8 * (lane_id() & 3) + e;
                        add[bc][e] = bias && c < wc ? bias[c] : 0.f;
                    }
            }
            for_outputs<WR, WC>(mine, acc, [&](int bc, int r, int c, float (&v)[8]) {
                r += r0;
                c += col0;
                if (r >= s.have || c >= wc) return;
                if constexpr (!DX) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += add[bc][e];
                    if (a.act != COGDL_ACT_NONE) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = output_act(v[e], a.act);
                    }
                }
                store8(a.out, a.out_dtype, (s.lo + r) * wc, c, wc, v);
            });
        });
}

// The forward of few rows a group (single tokens): the reads of the weights are all there is.  A
// workgroup owns 16 rows by 16 columns and its four wavefronts a quarter of x each, kFewSteps
// steps of 32 loaded at once, straight into the operands of the 16 x 16 x 32 matrix
// instructions; the quarters are added up through LDS.  8 rows of 8 among 64 groups, 2048 -> 1024,
// bf16: 64 workgroups of 128 x 128 tiles took 20 us, these 512 take 6.
constexpr int kFewRows = 16, kFewCols = 16, kFewSteps = 8, kFewWaves = 4;

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ f32x4 mfma_16x16x32(uint4 a, uint4 b, f32x4 c)
{
    if constexpr (Fmt<T>::code == COGDL_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <typename T>
__global__ __launch_bounds__(kFewWaves * kWave) void k_grouped_few(GroupedArgs a)
{
    __shared__ f32x4 part[kFewWaves][kWave];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int i = lane & 15, q = lane >> 4;             // row of either operand, its 8 of a step's 32 x
    // this wavefront's x: whole steps
    const int steps = (a.k + 31) / 32;
    const int x_lo = steps * wave / kFewWaves * 32, x_hi = steps * (wave + 1) / kFewWaves * 32;
    PieceWalk walk;
    walk.start(a.off, a.E, a.n, kFewRows, a.tiles_c);
    Span s;
    while (walk.next(s)) {
        const int col0 = s.tile * kFewCols;
        const Buffer X = buffer_of(static_cast<const T *>(a.X) + s.lo * a.k, (int64_t)s.have * a.k * 2);
        const int cols = a.m - col0 < kFewCols ? a.m - col0 : kFewCols;
        const Buffer W = buffer_of(static_cast<const T *>(a.W) + ((int64_t)s.g * a.m + col0) * a.k, (int64_t)cols * a.k * 2);
        const uint32_t row = (uint32_t)i * (uint32_t)a.k * 2u;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int x0 = x_lo; x0 < x_hi; x0 += 32 * kFewSteps) {
            uint4 w[kFewSteps], x[kFewSteps];
#pragma unroll
            for (int u = 0; u < kFewSteps; ++u) {
                // pieces at the row's end are read from its last 8 elements, those past it from nowhere
                const int at = x0 + 32 * u + 8 * q;
                const bool in = x0 + 32 * u < x_hi && at < a.k;
                const uint32_t off = in ? row + (uint32_t)(at + 8 <= a.k ? at : a.k - 8) * 2u : kNowhere;
                w[u] = load16(W, off);
                x[u] = load16(X, off);
            }
#pragma unroll
            for (int u = 0; u < kFewSteps; ++u) {
                if (x0 + 32 * u + 32 > a.k) {            // (uniform)
                    const int gone = x0 + 32 * u + 8 * q + 8 - a.k;
                    w[u] = shift_down(w[u], gone);
                    x[u] = shift_down(x[u], gone);
                }
                acc = mfma_16x16x32<T>(w[u], x[u], acc);
            }
        }
        __syncthreads();                                 // (the tile before is read)
        part[wave][lane] = acc;
        __syncthreads();
        if (wave != 0) continue;
        // lane l: columns 4 (l / 16) ... of row l % 16
        f32x4 t = part[0][lane];
#pragma unroll
        for (int p = 1; p < kFewWaves; ++p) t += part[p][lane];
        const int c = col0 + 4 * q;
        if (i >= s.have || c >= a.m) continue;
        float v[4] = {t.x, t.y, t.z, t.w};
        const float *__restrict__ bias = a.bias ? a.bias + (int64_t)s.g * a.m : nullptr;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = output_act(v[e] + (bias && c + e < a.m ? bias[c + e] : 0.f), a.act);
        store4(a.out, a.out_dtype, (s.lo + i) * a.m, c, a.m, v);
    }
}

struct Variant {
    GroupedKernel kern;
    int waves, tm, tn;
};

template <typename T, int WAVES, int TM, int TN>
Variant pick(bool dx, bool act, bool direct)
{
    GroupedKernel k;
    if (!dx) k = direct ? k_grouped_rows<T, WAVES, TM, TN, false, kDirect, kDirect>
                        : k_grouped_rows<T, WAVES, TM, TN, false, kStaged, kStaged>;
    else if (act) k = k_grouped_rows<T, WAVES, TM, TN, true, kSloped, kStaged>;
    else k = direct ? k_grouped_rows<T, WAVES, TM, TN, true, kDirect, kDirect>
                    : k_grouped_rows<T, WAVES, TM, TN, true, kStaged, kStaged>;
    return {k, WAVES, TM, TN};
}

// Tiles of 256 x 256 read each operand from the L2s half as often as those of 128 x 128, and hold a whole
// compute unit: for groups that fill them, and where there are enough for half of the chip.  2048 -> 2048
// bf16, dX with 256 and with 128: one group of 32768 rows 265 and 340 us, of 300 rows 48 and 32; 64
// groups, 8192 rows 212 and 172, 16384 rows 216 and 231, 32768 rows 377 and 410 (forward 376 and 417);
// 8 groups of 2.4M rows, 128 -> 256: 381 and 434.
bool wide_tiles(int64_t n, int32_t E, int wc)
{
    return wc > 128 && n >= 256 * (int64_t)E && n / 256 * ((wc + 255) / 256) > 128;
}

template <typename T>
Variant pick_tile(int64_t n, int32_t E, int wc, bool dx, bool act, bool direct)
{
    if (direct && !act && wide_tiles(n, E, wc))
        return {dx ? k_grouped_rows<T, 8, 256, 256, true, kDirect, kDirect>
                   : k_grouped_rows<T, 8, 256, 256, false, kDirect, kDirect>, 8, 256, 256};
    if (wc > 64) return pick<T, 4, 128, 128>(dx, act, direct);
    return pick<T, 4, 128, 64>(dx, act, direct);
}

// Whether the kernel for few rows is the faster one.  It reads a group's weights once for every 16 rows, at 5 TB/s;
// tiles read them once, at 5.5, but take 9.5 ns for each of k features besides.  With G groups that have rows and
// P pieces of 16 rows in them (as if they were even) that is in favour of few rows while
//     2 k m P / 5 TB/s < 9.5 ns k + 2 k m G / 5.5 TB/s,  or  m (11 (P - G) + G) < 2^18,
// whatever k.  bf16, us, with tiles in brackets: 64 groups, 2048 -> 1024, 32 / 512 rows: 25 (39) / 61 (77); 2048 -> 2048,
// one group of 16 / 64 / 128 / 256 rows: 9 (23) / 13 (24) / 21 (26) / 35 (26); 64 groups of 1 / 8 rows 96 (125) / 115
// (126), 256 groups 365 (346) / 446 (352); 4096 -> 4096, one group of 64 / 128 / 256: 35 (52) / 63 (55) / 121 (56), 64 of
// one row 356 (344); 8192 -> 8192, one of 16 / 64 / 256: 35 (92) / 119 (95) / 453 (105), with odd k three times that
// (256 rows of 8191: 1556 (169)).  More rows (64 groups, 2048 -> 1024, 1024 / 2048 rows: 74 (78) / 130 (78)) are
// tiles' whatever the widths.
bool few_rows(int64_t n, int32_t E, int32_t m)
{
    if (n > 256 && (n > 8 * (int64_t)E || n > 2048)) return false;
    const int64_t G = n < E ? n : E, P = G * (((n + G - 1) / G + kFewRows - 1) / kFewRows);
    return m * (11 * (P - G) + G) < 1 << 18;
}

}  // namespace

cogdl_status grouped_rows_launch(const char *name, GroupedArgs a, bool dx, cogdl_dtype dtype, hipStream_t stream)
{
    const bool act = dx && a.act != COGDL_ACT_NONE;
    // direct loads: every row of both operands on the 4-byte grid
    const bool direct = on_grid(dx ? a.dY : a.X, dx ? a.m : a.k) && on_grid(a.W, a.k);
    const int wc = dx ? a.k : a.m;
    if (!dx && a.k >= 8 && few_rows(a.n, a.E, a.m)) {
        const GroupedKernel kern = dtype == COGDL_BF16 ? k_grouped_few<bf16_t> : k_grouped_few<f16_t>;
        a.tiles_c = (a.m + kFewCols - 1) / kFewCols;
        return launch_tiles(name, kern, a, most_pieces(a.n, a.E, kFewRows) * a.tiles_c, kFewWaves, 0, 0, stream);
    }
    const Variant v = dtype == COGDL_BF16 ? pick_tile<bf16_t>(a.n, a.E, wc, dx, act, direct)
                                          : pick_tile<f16_t>(a.n, a.E, wc, dx, act, direct);
    a.tiles_c = (int32_t)(((int64_t)wc + v.tn - 1) / v.tn);
    return launch_tiles(name, v.kern, a, most_pieces(a.n, a.E, v.tm) * a.tiles_c, v.waves, lds_of(v.waves, v.tm, v.tn), 0, stream);
}

}  // namespace cogdl

using namespace cogdl;

extern "C" {

static cogdl_status check_grouped(int64_t n, int32_t E, int32_t k, int32_t m, const int32_t *offsets, int dtype)
{
    if (n < 0 || E < 1 || k < 0 || m < 0) return COGDL_ERR_INVALID;
    if (dtype != COGDL_BF16 && dtype != COGDL_F16) return COGDL_ERR_DTYPE;
    if (n > INT32_MAX || E > COGDL_MAX_GROUPS || k > kMaxWidth || m > kMaxWidth) return COGDL_ERR_TOO_LARGE;
    if (!offsets) return COGDL_ERR_INVALID;
    return COGDL_OK;
}

// More of the smallest tiles than the walks number: refused before anything runs.  (The kernel for few rows
// has smaller ones, of 16 x 16: 2176 pieces at most, under 2^30 tiles at any width.)
static bool too_many_tiles(int64_t n, int32_t E, int64_t wc)
{
    return !countable(most_pieces(n, E, 128), (wc + 63) / 64);
}

cogdl_status cogdl_grouped_linear(int64_t n, int32_t E, int32_t k, int32_t m, const int32_t *offsets,
                                  const void *X, const void *W, cogdl_dtype dtype, const float *bias,
                                  cogdl_act act, void *Y, cogdl_dtype y_dtype, int8_t *codes, uint8_t *exps,
                                  hipStream_t stream)
{
    const cogdl_status st = check_grouped(n, E, k, m, offsets, dtype);
    if (st != COGDL_OK) return st;
    if (act < COGDL_ACT_NONE || act > COGDL_ACT_ELU) return COGDL_ERR_INVALID;
    if (!dtype_ok(y_dtype)) return COGDL_ERR_DTYPE;
    if ((codes == nullptr) != (exps == nullptr)) return COGDL_ERR_INVALID;
    if (n > 0 && m > 0 && !Y) return COGDL_ERR_INVALID;
    if (n > 0 && k > 0 && !X) return COGDL_ERR_INVALID;
    if (n > 0 && m > 0 && k > 0 && !W) return COGDL_ERR_INVALID;
    if (n == 0) return COGDL_OK;
    if (m > 0 && too_many_tiles(n, E, m)) return COGDL_ERR_TOO_LARGE;
    if (codes && k > 0) {
        const cogdl_status cs = cogdl_act_checkpoint(n, k, X, dtype, codes, exps, stream);
        if (cs != COGDL_OK) return cs;
    }
    if (m == 0) return COGDL_OK;
    GroupedArgs a{};
    a.n = n; a.E = E; a.k = k; a.m = m;
    a.off = offsets;
    a.X = X; a.W = W;
    a.bias = bias;
    a.act = (int32_t)act;
    a.out = Y;
    a.out_dtype = (int32_t)y_dtype;
    return grouped_rows_launch("grouped_linear", a, false, dtype, stream);
}

cogdl_status cogdl_grouped_linear_backward_workspace(int64_t n, int32_t E, int32_t k, int32_t m, size_t *bytes)
{
    if (n < 0 || E < 1 || k < 0 || m < 0 || !bytes) return COGDL_ERR_INVALID;
    if (n > INT32_MAX || E > COGDL_MAX_GROUPS || k > kMaxWidth || m > kMaxWidth) return COGDL_ERR_TOO_LARGE;
    *bytes = (size_t)slices_of(n, E, k, m).slots() * ((size_t)m * k + m) * sizeof(float);
    return COGDL_OK;
}

cogdl_status cogdl_grouped_linear_backward(int64_t n, int32_t E, int32_t k, int32_t m, const int32_t *offsets,
                                           const void *dY, const void *W, const void *X, const int8_t *codes,
                                           const uint8_t *exps, cogdl_dtype dtype, const void *Y, cogdl_act act,
                                           void *dX, void *dW, cogdl_dtype dw_dtype, float *db, void *workspace,
                                           size_t workspace_bytes, hipStream_t stream)
{
    const cogdl_status st = check_grouped(n, E, k, m, offsets, dtype);
    if (st != COGDL_OK) return st;
    if (act < COGDL_ACT_NONE || act > COGDL_ACT_ELU) return COGDL_ERR_INVALID;
    if (dw_dtype != COGDL_F32 && dw_dtype != dtype) return COGDL_ERR_DTYPE;
    const bool rows = n > 0 && m > 0;
    if (rows && (dX || dW || db) && (!dY || (act != COGDL_ACT_NONE && !Y))) return COGDL_ERR_INVALID;
    if (rows && k > 0 && dX && !W) return COGDL_ERR_INVALID;
    if ((codes == nullptr) != (exps == nullptr)) return COGDL_ERR_INVALID;
    if (rows && k > 0 && dW && (X != nullptr) == (codes != nullptr)) return COGDL_ERR_INVALID;
    const Slices c = slices_of(n, E, k, m);
    const size_t need = (size_t)c.slots() * ((size_t)m * k + m) * sizeof(float);
    const bool weights = (dW && k > 0 && m > 0) || (db && m > 0);
    if (weights && need > 0 && (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < need))
        return COGDL_ERR_INVALID;
    if (n > 0 && dX && k > 0 && too_many_tiles(n, E, k)) return COGDL_ERR_TOO_LARGE;
    if (weights && !countable(c.count, (int64_t)((m + 63) / 64) * (k > 0 ? (k + 63) / 64 : 1))) return COGDL_ERR_TOO_LARGE;
    GroupedArgs a{};
    a.n = n; a.E = E; a.k = k; a.m = m;
    a.off = offsets;
    a.X = X; a.codes = codes; a.exps = exps;
    a.W = W;
    a.act = (int32_t)act;
    a.dY = dY; a.Y = Y;
    if (dX && n > 0 && k > 0) {
        a.out = dX;
        a.out_dtype = (int32_t)dtype;
        const cogdl_status s = grouped_rows_launch("grouped_linear_dx", a, true, dtype, stream);
        if (s != COGDL_OK) return s;
    }
    if (!weights) return COGDL_OK;
    a.out = k > 0 ? dW : nullptr;
    a.out_dtype = (int32_t)dw_dtype;
    a.db = db;
    a.part = static_cast<float *>(workspace);
    return grouped_weights_launch(a, c, dtype, stream);
}

}  // extern "C"
