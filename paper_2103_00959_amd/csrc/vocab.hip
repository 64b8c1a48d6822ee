// Softmax losses over a large vocabulary, forward: cross entropy and distillation from a teacher's top
// logits, of logits X W^T + bias that are never kept (the formulas: vocab.hpp).
//
// A tile of logits stays in the accumulators of the matrix cores; what leaves it is each row's (max, sum of
// exp) over a slot of 64 columns.  A last kernel joins the slots.  The logits of the targets are
// plain dot products, as the rows are gathered.
#include "vocab.hpp"

namespace cogdl {
namespace {

constexpr int kBlock = 256;

__device__ __forceinline__ bool counts(int32_t t, int32_t V) { return (uint32_t)t < (uint32_t)V; }

// |g T| for the call's factor: a weight that is not finite makes its own row NaN or infinite under any, and has no part
// in what the others' is.
__device__ __forceinline__ float finite_weight(float dloss, float T)
{
    const float w = fabsf(dloss * T);
    return w < INFINITY ? w : 0.f;
}

// 8 features from column 8 v on of a row of k, zeros behind its end.
template <typename T>
__device__ __forceinline__ uint4 load_vec8(const T *__restrict__ row, int v, int k)
{
    if (8 * v + 8 > k) return load_short(row + 8 * v, k - 8 * v);
    const u32x4_u u = *reinterpret_cast<const u32x4_u *>(row + 8 * v);
    return make_uint4(u.x, u.y, u.z, u.w);
}

template <typename T>
__device__ __forceinline__ float dot8(uint4 a, uint4 b, float t)
{
    float f[8], g[8];
    unpack8<T>(a, f);
    unpack8<T>(b, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) t = fmaf(f[e], g[e], t);
    return t;
}

// The teacher's rows: whether any entry counts (inside the vocabulary, its logit above -inf), and the log of
// the sum of their exponentials.  FORWARD: also the student's logits of the entries, by 4 entries of 16 lanes a
// wavefront, into logp, and a workgroup a row (its wavefronts each find the row's sum); else a wavefront a row.  Bound
// by the gather of W: 4096 rows of 64 entries of 768 bf16 52 us (5.6 TB/s of HBM).
template <typename T, bool FORWARD>
__global__ __launch_bounds__(kBlock) void k_teacher_rows(VocabArgs a)
{
    constexpr int W = kBlock / kWave;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int64_t step = FORWARD ? gridDim.x : (int64_t)gridDim.x * W;
    for (int64_t i = FORWARD ? blockIdx.x : (int64_t)blockIdx.x * W + wave; i < a.n; i += step) {
        const int32_t *__restrict__ index = a.index + i * a.entries;
        const float *__restrict__ teacher = a.teacher + i * a.entries;
        float m = -INFINITY;
        bool any = false;
        for (int e = lane; e < a.entries; e += kWave) {
            const float t = teacher[e] / a.T;
            if (!counts(index[e], a.V)) continue;
            any = any || !(t == -INFINITY);
            m = fmaxf(m, t);
        }
        m = group_reduce(m, kWave, [](float x, float y) { return fmaxf(x, y); });
        const bool live = __ballot(any) != 0;
        const float from = m == -INFINITY ? 0.f : m;
        float s = 0.f;
        for (int e = lane; e < a.entries; e += kWave)
            if (counts(index[e], a.V)) s += expf(teacher[e] / a.T - from);
        s = group_sum(s, kWave);
        if (lane == 0 && (!FORWARD || wave == 0)) {
            a.live[i] = live ? 0 : -1;
            a.tlse[i] = make_float2(from, logf(s));
        }
        if constexpr (FORWARD) {
            const T *__restrict__ x = static_cast<const T *>(a.X) + i * a.k;
            const int sub = lane & 15, vecs = (a.k + 7) / 8;
            for (int e0 = 4 * wave; e0 < a.entries; e0 += 4 * W) {
                const int e = e0 + (lane >> 4);
                const int32_t v = e < a.entries ? index[e] : -1;
                const bool on = live && counts(v, a.V);
                const T *__restrict__ w = static_cast<const T *>(a.W) + (int64_t)(on ? v : 0) * a.k;
                float z = 0.f;
                if (on) {
#pragma unroll 4
                    for (int c = sub; c < vecs; c += 16) z = dot8<T>(load_vec8(w, c, a.k), load_vec8(x, c, a.k), z);
                }
                z = group_sum(z, 16);
                if (sub == 0 && e < a.entries) a.logp[i * a.entries + e] = on ? (a.bias ? z + a.bias[v] : z) / a.T : 0.f;
            }
        }
    }
}

// How many rows of each run of `per` count, and their largest weight.
template <bool BACKWARD>
__global__ __launch_bounds__(kBlock) void k_count_rows(VocabArgs a, int per)
{
    constexpr int W = kBlock / kWave;
    __shared__ int wsum[W];
    __shared__ float wmax[W];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int32_t *__restrict__ live = a.distill ? a.live : a.index;
    const int32_t limit = a.distill ? INT32_MAX : a.V;
    const int64_t from = (int64_t)blockIdx.x * per, to = from + per < a.n ? from + per : a.n;
    int count = 0;
    float top = 0.f;
    for (int64_t i = from + threadIdx.x; i < to; i += kBlock) {
        if (!counts(live[i], limit)) continue;
        ++count;
        if (BACKWARD) top = fmaxf(top, finite_weight(a.dloss[i], a.T));
    }
    count = wave_inclusive_scan(count);
    top = group_reduce(top, kWave, [](float x, float y) { return fmaxf(x, y); });
    if (lane == kWave - 1) {
        wsum[wave] = count;
        wmax[wave] = top;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int w = 1; w < W; ++w) {
        wsum[0] += wsum[w];
        wmax[0] = fmaxf(wmax[0], wmax[w]);
    }
    a.counts[blockIdx.x] = wsum[0];
    if (BACKWARD) a.tops[blockIdx.x] = wmax[0];
}

// The rows that count, in order, and their features; in the forward of the cross entropy also their targets'
// logits, into loss.  A workgroup takes `per` rows; how many count before them it finds by itself, from the targets
// (up to n a workgroup, from the L2s), which a launch of its own would not do sooner.  8192 rows of 1024 bf16 20 us.
// Of more than kManyRows a launch before counts them run by run (k_count_rows), and finds the largest weight: 232965
// rows 14 us, and the gathering of 128 features, forward and backward, 679 -> 112.
constexpr int kRowsDeep = 4;     // rows a wavefront moves at once

template <typename T, bool BACKWARD>
__global__ __launch_bounds__(kBlock) void k_vocab_rows(VocabArgs a, int per)
{
    constexpr int W = kBlock / kWave;
    __shared__ int wsum[W];
    __shared__ float wmax[W];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int32_t *__restrict__ live = a.distill ? a.live : a.index;
    const int32_t limit = a.distill ? INT32_MAX : a.V;
    const int64_t from = (int64_t)blockIdx.x * per, to = from + per < a.n ? from + per : a.n;
    const bool many = a.n > kManyRows;
    int before = 0;
    if (many) {
        for (int b = threadIdx.x; b < (int)blockIdx.x; b += kBlock) before += a.counts[b];
    }
    for (int64_t i0 = threadIdx.x; !many && i0 < from; i0 += kBlock * 16) {
        int32_t t[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) t[u] = i0 + u * kBlock < from ? live[i0 + u * kBlock] : -1;
#pragma unroll
        for (int u = 0; u < 16; ++u) before += counts(t[u], limit) ? 1 : 0;
    }
    before = wave_inclusive_scan(before);
    if (lane == kWave - 1) wsum[wave] = before;
    __syncthreads();
    int at = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) at += wsum[w];
    if (BACKWARD && blockIdx.x == 0) {
        // The largest finite |g T| that counts, for a factor that brings it to 2^15: fp16 then keeps what it can of the small
        // ones, and of rows that weigh the same, as in a mean, a target's dz, near -g T, lies just under a power of
        // two, where a rounding takes least of it (256 rows of 1433 answers, bf16: the gradients are, with a
        // power of two for the factor, 0.0020 to 0.0031, so 0.0019; rounded once they are 0.0017).
        float top = 0.f;
        if (many) {
            for (int b = threadIdx.x; b < (int)gridDim.x; b += kBlock) top = fmaxf(top, a.tops[b]);
        }
        for (int64_t i0 = threadIdx.x; !many && i0 < a.n; i0 += kBlock * 8) {
            float g[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int64_t i = i0 + u * kBlock;
                g[u] = i < a.n && counts(live[i], limit) ? a.dloss[i] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) top = fmaxf(top, finite_weight(g[u], a.T));
        }
        top = group_reduce(top, kWave, [](float x, float y) { return fmaxf(x, y); });
        if (lane == 0) wmax[wave] = top;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, wmax[w]);
            top = fmaxf(top, 0x1p-100f);
            a.head->scale = 32768.f / top;
            a.head->unscale = top / 32768.f;
        }
    }
    if (BACKWARD && a.db_q) {
        for (int64_t v = (int64_t)blockIdx.x * kBlock + threadIdx.x; v < a.V; v += (int64_t)gridDim.x * kBlock) {
            a.db_q[v] = 0;
            a.db_odd[v] = 0;
        }
    }
    const T *__restrict__ X = static_cast<const T *>(a.X);
    T *__restrict__ Xr = static_cast<T *>(a.Xr);
    T *__restrict__ dX = static_cast<T *>(a.dX);
    const int vecs = a.kp / 8;
    const bool dots = !BACKWARD && !a.distill;
    // 64 rows at a time, every wavefront alike; a wavefront moves every fourth row
    for (int64_t r0 = from; r0 < to; r0 += kWave) {
        const int64_t i = r0 + lane;
        const int32_t t = i < to ? live[i] : -1;
        const uint64_t mask = __ballot(counts(t, limit));
        if (wave == 0 && i < to) {
            if (counts(t, limit)) {
                const int p = at + __popcll(mask & ((1ull << lane) - 1));
                a.rows[p] = (int32_t)i;
                if constexpr (BACKWARD) {
                    const float g = a.dloss[i] * a.T;
                    a.lse2[p] = a.lse_in[i] * kLog2e;
                    a.g[p] = g;
                    if (!a.distill) {
                        a.col[p] = t;
                        a.at_col[p] = g * expm1f(-a.loss_in[i]);      // p - 1, exact where p is near 1 too
                    }
                }
            } else if constexpr (!BACKWARD) {
                a.loss[i] = 0.f;
                a.lse[i] = 0.f;
            }
        }
        const int here = to - r0 < kWave ? (int)(to - r0) : kWave;
        for (int b = wave; b < here; b += W * kRowsDeep) {
            int64_t row[kRowsDeep];
            int p[kRowsDeep];
            int32_t target[kRowsDeep];
            float z[kRowsDeep];
#pragma unroll
            for (int u = 0; u < kRowsDeep; ++u) {
                const int r = b + u * W < kWave ? b + u * W : 0;
                const bool on = b + u * W < here && (mask >> r & 1);
                row[u] = r0 + r;
                p[u] = on ? at + __popcll(mask & ((1ull << r) - 1)) : -1;
                target[u] = __builtin_amdgcn_readlane(t, r);
                z[u] = 0.f;
            }
            for (int v = lane; v < vecs; v += kWave) {
                uint4 f[kRowsDeep], w[kRowsDeep];
#pragma unroll
                for (int u = 0; u < kRowsDeep; ++u) {
                    f[u] = w[u] = make_uint4(0u, 0u, 0u, 0u);
                    if (p[u] < 0) continue;
                    f[u] = load_vec8(X + row[u] * a.k, v, a.k);
                    if (dots) w[u] = load_vec8(static_cast<const T *>(a.W) + (int64_t)target[u] * a.k, v, a.k);
                }
#pragma unroll
                for (int u = 0; u < kRowsDeep; ++u) {
                    if (p[u] < 0) continue;
                    *reinterpret_cast<uint4 *>(Xr + (int64_t)p[u] * a.kp + 8 * v) = f[u];
                    if (dots) z[u] = dot8<T>(f[u], w[u], z[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < kRowsDeep; ++u) {
                if (p[u] >= 0 && dots) {
                    z[u] = group_sum(z[u], kWave);
                    if (lane == 0) a.loss[row[u]] = a.bias ? z[u] + a.bias[target[u]] : z[u];
                }
                if (BACKWARD && p[u] < 0 && b + u * W < here && dX) {
                    const float zeros[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    for (int v = lane; v < vecs; v += kWave) store8(dX + row[u] * a.k, 8 * v, a.k, zeros);
                }
            }
        }
        at += __popcll(mask);
    }
    if (to == a.n && wave == 0) {
        if (lane == 0) a.head->live = at;
        if constexpr (BACKWARD) {
            // the slices of dX's sums that end soonest for so many rows: a candidate a lane
            static_assert(kMostSlices == kWave, "a candidate a lane");
            const float cost = lane < a.plan.most ? a.plan.cost(at, lane + 1) : INFINITY;
            const float best = group_reduce(cost, kWave, [](float x, float y) { return fminf(x, y); });
            const int first = __builtin_ctzll(__ballot(cost == best));
            if (lane == 0) a.head->slices = first + 1;
        }
    }
}

// Tiles of logits.  GRAD: dz of the piece, else each row's (max, sum) over the wavefront's columns.  EXTRA: with a
// bias, or db's sums over the tile's rows.  Bound by the matrix cores and, of narrow features, by what is done with
// their outputs (an exponential each, a quarter of the other instructions' rate; about 3 chunks of 64 features' time
// a tile): 8192 x 131072 of 1024 features the statistics 1912 us (1.15 PFLOP/s; a library product that writes the logits
// 1.16 to 1.21), dz 2103; 2867 x 40943 of 512 125 (0.96 PFLOP/s) and 148; 2048 x 14951 of 200 27 (0.45).
// dz is rounded to T, by half a step at most: the matrix instructions of the products behind take 16 bits, and W and X
// are T.  The gradients are then 0.0018 to 0.0023 of their size off in bf16 and 0.0003 to 0.0004 in fp16, where the
// rounding of the outputs alone makes 0.0017 and 0.0002 to 0.0004.  dz in two parts of 16 bits would take that away and
// double the products: 3750 us more of the 7900 of the first of those sizes.
template <typename T, int WAVES, int TM, int TN, int SRCB, bool GRAD, bool EXTRA>
__global__ __launch_bounds__(WAVES * kWave, 2) void k_vocab_logits(VocabArgs a)
{
    constexpr int N = WAVES * kWave;
    constexpr int WAVES_C = TN >= 256 ? 4 : 2, WAVES_R = WAVES / WAVES_C;
    constexpr int WR = TM / WAVES_R / 32, WC = TN / WAVES_C / 32;
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wr = wave / WAVES_C, wc = wave % WAVES_C;
    const int r0 = wr * (32 * WR), c0 = wc * (32 * WC);
    GridWalk walk;
    int64_t rows = !GRAD && a.plain ? a.n : a.head->live;
    if constexpr (!GRAD) {
        rows -= a.p0;
        rows = rows < 0 ? 0 : rows < a.block ? rows : a.block;
    }
    walk.start(rows, TM, a.tiles_c, 1, blockIdx.x, GRAD ? kPanel : 2 * kPanel, GRAD);
    RowOperand<T, TM, N, kDirect> A;
    RowOperand<T, TN, N, SRCB> B;
    const auto open = [&](const Span &s) {
        const int col = s.tile * TN, cols = a.width - col < TN ? a.width - col : TN;
        A.open(static_cast<const T *>(a.Xr) + ((GRAD ? 0 : a.p0) + s.lo) * a.kp, nullptr, s.have, a.kp, 0);
        B.open(static_cast<const T *>(a.W) + ((int64_t)a.v0 + col) * a.k, nullptr, cols, a.k, 0);
        return a.kp;
    };
    const float scale = GRAD ? a.head->scale : 1.f;
    char *const mine = lds + 2 * (TM + TN) * kX * 2 + wave * kOutBytes;
    run_tiles<T, decltype(A), decltype(B), WR, WC>(
        lds, walk, A, B, r0, c0, open, [&](const Span &s) { return r0 < s.have && s.tile * TN + c0 < a.width; },
        [](const Span &, const uint4 (&)[WR]) {}, [](const Span &) {},
        [&](const Span &s, Acc<WR, WC> &acc) {
            const int col0 = s.tile * TN + c0;
            if (col0 >= a.width || r0 >= s.have) return;
            const int lane = lane_of_outputs();
            // the bias, and -inf behind the last column: no part of a sum, no gradient
            // (col0 + 32 WC may pass 32 bits)
            if (EXTRA || col0 > a.width - 32 * WC) {
#pragma unroll
                for (int j = 0; j < WC; ++j)
#pragma unroll
                    for (int t = 0; t < 16; ++t) {
                        const int c = col0 + 32 * j + 8 * (t / 4) + 4 * (lane >> 5) + t % 4;
                        const float add = c < a.width ? EXTRA && a.bias ? a.bias[a.v0 + c] : 0.f : -INFINITY;
#pragma unroll
                        for (int i = 0; i < WR; ++i) acc.a[i][j][t] += add;
                    }
            }
            if constexpr (!GRAD) {
                const int slot = s.tile * WAVES_C + wc;
#pragma unroll
                for (int i = 0; i < WR; ++i) {
                    float m = -INFINITY;
#pragma unroll
                    for (int j = 0; j < WC; ++j)
#pragma unroll
                        for (int t = 0; t < 16; ++t) m = fmaxf(m, acc.a[i][j][t]);
                    m = fmaxf(m, bfly_partner<32>(m)) * a.per_z;
                    const float from = m == -INFINITY ? 0.f : m;
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < WC; ++j)
#pragma unroll
                        for (int t = 0; t < 16; ++t) sum += __builtin_amdgcn_exp2f(fmaf(acc.a[i][j][t], a.per_z, -from));
                    sum += bfly_partner<32>(sum);
                    const int r = r0 + 32 * i + (lane & 31);
                    if (lane < 32 && r < s.have) a.part[(int64_t)slot * a.block + s.lo + r] = make_float2(m, sum);
                }
            } else {
                T *__restrict__ dz = static_cast<T *>(a.dz) + s.lo * a.pitch;
                float sums[EXTRA ? 16 * WC : 1] = {};
                float less = 0.f, g = 0.f;
                int32_t col = -1;
                int64_t p = 0;
                for_rows16<T, WR, WC>(
                    mine, acc,
                    [&](int i, int j, int q, float (&v)[4]) {
                        const int r = r0 + 32 * i + (lane & 31), c = col0 + 32 * j + 8 * q + 4 * (lane >> 5);
                        if (j == 0 && q == 0) {          // (a row block's first)
                            p = s.lo + (r < s.have ? r : 0);
                            less = a.lse2[p];
                            g = r < s.have ? a.g[p] * scale : 0.f;
                            col = a.distill ? -1 : a.col[p] - a.v0;
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_exp2f(fmaf(v[e], a.per_z, -less)) * g;
                        if ((uint32_t)(col - c) < 4u) {  // (seldom)
                            const float there = r < s.have ? a.at_col[p] * scale : 0.f;
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = col == c + e ? there : v[e];
                        }
                        if constexpr (EXTRA) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) sums[16 * j + 4 * q + e] += r < s.have ? v[e] : 0.f;
                        }
                    },
                    [&](int r, int c, uint4 w) {
                        r += r0;
                        c += col0;
                        // (past the caches: it is read when the whole piece is there; of 8192 x 131072, 1024 features, the
                        // products took 3885 us, so 3790)
                        if (r < s.have && c < a.width)
                            __builtin_nontemporal_store(__builtin_bit_cast(u32x4_u, w), reinterpret_cast<u32x4_u *>(dz + (int64_t)r * a.pitch + c));
                    });
                if constexpr (EXTRA) {
                    if (!a.db_part) return;
                    // over the 32 rows' lanes, in a fixed order: two lanes share what either has left, and keep a half
                    // each, down to one column a lane
#pragma unroll
                    for (int half = 16; half > 0; half /= 2) {
                        const bool upper = lane & half;
#pragma unroll
                        for (int t = 0; t < half; ++t) {
                            const float keep = upper ? sums[t + half] : sums[t], give = upper ? sums[t] : sums[t + half];
                            sums[t] = keep + __shfl_xor(give, half);
                        }
                    }
                    const int t = lane & 31, c = col0 + 32 * (t / 16) + 8 * (t / 4 % 4) + 4 * (lane >> 5) + t % 4;
                    if (c < a.width) a.db_part[((int64_t)s.g * WAVES_R + wr) * a.pitch + c] = sums[0];
                }
            }
        });
}

// The statistics of up to 16 rows (single queries), where one tile a wavefront covers W: the reads of W are all there
// is.  A wavefront owns 16 columns over all features, 8 steps of 32 loaded at once straight into the operands of the
// 16 x 16 x 32 matrix instructions; the rows lie in LDS.  Lane l holds columns 4 (l / 16) ... + 3 of row l % 16; the
// (max, sum) of a workgroup's 64 columns are one slot.  In place of 128 x 128 tiles: 1 row, 14541 classes of 512
// features 7.5 us for 10.6, 8000 of 2048 14 for 27.  Not for more rows or columns: 64 of those rows 12.8 for 10.7, and
// 1 row, 50257 of 2048 (two tiles a wavefront) 40 for 33.
constexpr int kFewRows = 16, kFewSteps = 8, kFewWaves = 4;

inline int few_stride(int k) { return (k + 31) / 32 * 32 + 8; }       // of a row in LDS: 16 of them on all banks

template <typename T>
__global__ __launch_bounds__(kFewWaves * kWave) void k_vocab_few(VocabArgs a, int stride)
{
    extern __shared__ __align__(16) char lds[];
    T *const x = reinterpret_cast<T *>(lds);
    __shared__ float2 part[kFewWaves][kFewRows];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int i = lane & 15, q = lane >> 4;              // column of W (row of X), its 8 of a step's 32 features
    const int n = (int)a.n, vecs = (stride - 8) / 8;
    for (int u = threadIdx.x; u < kFewRows * vecs; u += kFewWaves * kWave) {
        const int r = u / vecs, v = u % vecs;
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (r < n && 8 * v < a.k) w = load_vec8(static_cast<const T *>(a.X) + (int64_t)r * a.k, v, a.k);
        *reinterpret_cast<uint4 *>(x + r * stride + 8 * v) = w;
    }
    __syncthreads();
    const int64_t col0 = ((int64_t)blockIdx.x * kFewWaves + wave) * 16;
    const int cols = (int)(a.V - col0 < 16 ? a.V - col0 > 0 ? a.V - col0 : 0 : 16);
    const Buffer W = buffer_of(static_cast<const T *>(a.W) + (cols ? col0 : 0) * a.k, (int64_t)cols * a.k * 2);
    const uint32_t row = (uint32_t)i * (uint32_t)a.k * 2u;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int x0 = 0; x0 < a.k; x0 += 32 * kFewSteps) {
        uint4 w[kFewSteps];
#pragma unroll
        for (int u = 0; u < kFewSteps; ++u) {
            // pieces at the row's end are read from its last 8 elements, those past it from nowhere
            const int at = x0 + 32 * u + 8 * q;
            w[u] = load16(W, at < a.k ? row + (uint32_t)(at + 8 <= a.k ? at : a.k - 8) * 2u : kNowhere);
        }
#pragma unroll
        for (int u = 0; u < kFewSteps; ++u) {
            if (x0 + 32 * u >= a.k) break;               // (uniform)
            if (x0 + 32 * u + 32 > a.k) w[u] = shift_down(w[u], x0 + 32 * u + 8 * q + 8 - a.k);
            acc = mfma_16x16x32<T>(w[u], *reinterpret_cast<const uint4 *>(x + i * stride + x0 + 32 * u + 8 * q), acc);
        }
    }
    float m = -INFINITY, z = 0.f, v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool in = 4 * q + e < cols;
        v[e] = in ? (acc[e] + (a.bias ? a.bias[col0 + 4 * q + e] : 0.f)) * a.per_z : -INFINITY;
        m = fmaxf(m, v[e]);
    }
    const auto base = [](float top) { return top == -INFINITY ? 0.f : top; };
#pragma unroll
    for (int e = 0; e < 4; ++e) z += __builtin_amdgcn_exp2f(v[e] - base(m));
    const auto merge = [&](float m2, float z2) {
        const float top = fmaxf(m, m2), from = base(top);
        z = z * __builtin_amdgcn_exp2f(m - from) + z2 * __builtin_amdgcn_exp2f(m2 - from);
        m = top;
    };
    for (int half = 16; half < kWave; half *= 2) {
        const float m2 = __shfl_xor(m, half), z2 = __shfl_xor(z, half);
        merge(m2, z2);
    }
    if (q == 0) part[wave][i] = make_float2(m, z);
    __syncthreads();
    if (wave != 0 || lane >= n) return;
    m = part[0][lane].x;
    z = part[0][lane].y;
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) merge(part[w][lane].x, part[w][lane].y);
    a.part[(int64_t)blockIdx.x * a.block + lane] = make_float2(m, z);
}

// The slots of a row joined to its lse, and the loss from its targets' logits.  R rows a workgroup (a power of
// two up to 16), 256 / R threads each.  Of rows as they were given, which count, and their targets' logits, are found
// here.  8192 rows, 2048 slots 27 us (4.9 TB/s).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_vocab_finish(VocabArgs a, int R)
{
    constexpr int W = kBlock / kWave;
    __shared__ float2 part[kBlock];
    __shared__ float lse_of[16], dots[16];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    int64_t live = a.plain ? a.n : a.head->live;
    live = live < a.p0 + a.block ? live : a.p0 + a.block;
    const int r = threadIdx.x & (R - 1), sg = threadIdx.x / R, S = kBlock / R;
    for (int64_t r0 = a.p0 + (int64_t)blockIdx.x * R; r0 < live; r0 += (int64_t)gridDim.x * R) {
        if (a.plain && !a.distill) {
            for (int q = wave; q < R && r0 + q < live; q += W) {
                const int32_t t = a.index[r0 + q];
                float dot = 0.f;
                if (counts(t, a.V))
                    for (int v = lane; v < (a.k + 7) / 8; v += kWave)
                        dot = dot8<T>(load_vec8(static_cast<const T *>(a.X) + (r0 + q) * a.k, v, a.k),
                                      load_vec8(static_cast<const T *>(a.W) + (int64_t)t * a.k, v, a.k), dot);
                dot = group_sum(dot, kWave);
                if (lane == 0) dots[q] = dot;
            }
        }
        float m = -INFINITY, z = 0.f;
        // (the exponents are powers of two here)
        const auto merge = [&](float2 p) {
            const float top = fmaxf(m, p.x);
            const float from = top == -INFINITY ? 0.f : top;
            z = z * __builtin_amdgcn_exp2f(m - from) + p.y * __builtin_amdgcn_exp2f(p.x - from);
            m = top;
        };
        if (r0 + r < live) {
            for (int s0 = sg; s0 < a.slots; s0 += 8 * S) {
                float2 p[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int s = s0 + u * S;
                    p[u] = s < a.slots ? a.part[(int64_t)s * a.block + (r0 - a.p0) + r] : make_float2(-INFINITY, 0.f);
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) merge(p[u]);
            }
        }
        part[threadIdx.x] = make_float2(m, z);
        __syncthreads();
        for (int half = S / 2; half > 0; half /= 2) {
            if (sg < half) {
                merge(part[threadIdx.x + half * R]);
                part[threadIdx.x] = make_float2(m, z);
            }
            __syncthreads();
        }
        if ((int)threadIdx.x < R) {
            const float lse = ((m == -INFINITY ? 0.f : m) + log2f(z)) * kLn2;
            lse_of[r] = lse;
            if (r0 + r < live) {
                const int64_t i = a.plain ? r0 + r : a.rows[r0 + r];
                if (a.plain && !counts(a.distill ? a.live[i] : a.index[i], a.distill ? INT32_MAX : a.V)) {
                    a.lse[i] = 0.f;
                    if (!a.distill) a.loss[i] = 0.f;
                } else {
                    a.lse[i] = lse;
                    if (!a.distill) {
                        const float dot = a.plain ? dots[r] + (a.bias ? a.bias[a.index[i]] : 0.f) : a.loss[i];
                        // (above 0 by definition; the two sums' roundings may differ)
                        const float loss = lse - dot;
                        a.loss[i] = loss < 0.f ? 0.f : loss;
                    }
                }
            }
        }
        __syncthreads();                                 // (lse_of; part and dots are read)
        if (!a.distill) continue;
        for (int q = wave; q < R && r0 + q < live; q += W) {
            const int64_t i = a.plain ? r0 + q : a.rows[r0 + q];
            if (a.plain && a.live[i] < 0) {
                if (lane == 0) a.loss[i] = 0.f;
                continue;
            }
            const float lse = lse_of[q];
            const float2 tlse = a.tlse[i];
            float loss = 0.f;
            for (int e = lane; e < a.entries; e += kWave) {
                if (!counts(a.index[i * a.entries + e], a.V)) continue;       // (logp is 0)
                const float logp = a.logp[i * a.entries + e] - lse, logq = log_share(a.teacher[i * a.entries + e], a.T, tlse);
                a.logp[i * a.entries + e] = logp;
                const float share = expf(logq);
                if (!(share == 0.f)) loss += share * (logq - logp);
            }
            loss = group_sum(loss, kWave);
            if (lane == 0) a.loss[i] = loss * a.T * a.T;
        }
        __syncthreads();
    }
}

template <typename T, bool GRAD, bool EXTRA>
VocabKernel pick(bool wide, bool direct)
{
    if (wide) return k_vocab_logits<T, 8, 256, 256, kDirect, GRAD, EXTRA>;
    return direct ? k_vocab_logits<T, 4, 128, 128, kDirect, GRAD, EXTRA> : k_vocab_logits<T, 4, 128, 128, kStaged, GRAD, EXTRA>;
}

template <typename T>
VocabKernel pick(bool grad, bool extra, bool wide, bool direct)
{
    if (grad) return extra ? pick<T, true, true>(wide, direct) : pick<T, true, false>(wide, direct);
    return extra ? pick<T, false, true>(wide, direct) : pick<T, false, false>(wide, direct);
}

}  // namespace

// The fewer rounds of resident workgroups, at their chunks' times (a tile's start and outputs take about 3 chunks of
// either).  With tiles of 256 x 256 and of 128 x 128: 1000 rows by 10007, 602 features, 160 and 632 tiles, 25 and 30 us;
// 2048 by 14951, 200 features, 472 and 1872, 28 and 37; 256 by 1433, 128 features, 6 and 24, 9 and 5.
bool vocab_wide(int64_t n, int64_t cols, int32_t k, const void *W)
{
    if (!on_grid(W, k)) return false;
    const int64_t w = ((n + 255) / 256) * ((cols + 255) / 256), s = ((n + 127) / 128) * ((cols + 127) / 128);
    return (float)((w + 255) / 256) * kWideChunk < (float)((s + 511) / 512) * (s <= 256 ? kNarrowChunk : kNarrowChunks);
}

// k_vocab_few where its rule holds.
template <typename T>
cogdl_status few_launch(const VocabArgs &a, bool &done, hipStream_t stream)
{
    const size_t lds = (size_t)kFewRows * few_stride(a.k) * 2;
    done = a.plain && on_grid(a.W, a.k) && a.n <= kFewRows && a.k >= 8 && lds <= (156 << 10);
    if (!done) return COGDL_OK;
    const int64_t resident = resident_blocks(reinterpret_cast<const void *>(k_vocab_few<T>), kFewWaves * kWave, lds, 0);
    if (resident < 1) return COGDL_ERR_LAUNCH;
    done = a.slots <= resident;
    if (!done) return COGDL_OK;
    COGDL_LAUNCH_SHM("vocab_few", k_vocab_few<T>, (unsigned)a.slots, kFewWaves * kWave, lds, stream, a, few_stride(a.k));
    return COGDL_OK;
}

cogdl_status vocab_rows_launch(const VocabArgs &a, cogdl_dtype dtype, bool backward, hipStream_t stream)
{
    if (a.distill && a.n > 0) {
        const int64_t blocks = backward ? (a.n + kBlock / kWave - 1) / (kBlock / kWave) : a.n;
        const unsigned grid = (unsigned)(blocks < 8192 ? blocks : 8192);
        if (backward) COGDL_LAUNCH("teacher_rows", (k_teacher_rows<bf16_t, false>), grid, kBlock, stream, a);    // (no features)
        else if (dtype == COGDL_BF16) COGDL_LAUNCH("teacher_rows", (k_teacher_rows<bf16_t, true>), grid, kBlock, stream, a);
        else COGDL_LAUNCH("teacher_rows", (k_teacher_rows<f16_t, true>), grid, kBlock, stream, a);
    }
    if (a.plain) return COGDL_OK;
    const bool many = a.n > kManyRows;
    const int64_t runs = many ? kMostRuns : 512;
    int64_t per = (a.n + runs - 1) / runs;
    per = per < 8 ? 8 : per;
    const unsigned blocks = a.n > 0 ? (unsigned)((a.n + per - 1) / per) : 1;
    if (many && backward) COGDL_LAUNCH("vocab_count", k_count_rows<true>, blocks, kBlock, stream, a, (int)per);
    else if (many) COGDL_LAUNCH("vocab_count", k_count_rows<false>, blocks, kBlock, stream, a, (int)per);
    if (dtype == COGDL_BF16) {
        if (backward) COGDL_LAUNCH("vocab_rows", (k_vocab_rows<bf16_t, true>), blocks, kBlock, stream, a, (int)per);
        else COGDL_LAUNCH("vocab_rows", (k_vocab_rows<bf16_t, false>), blocks, kBlock, stream, a, (int)per);
    } else {
        if (backward) COGDL_LAUNCH("vocab_rows", (k_vocab_rows<f16_t, true>), blocks, kBlock, stream, a, (int)per);
        else COGDL_LAUNCH("vocab_rows", (k_vocab_rows<f16_t, false>), blocks, kBlock, stream, a, (int)per);
    }
    return COGDL_OK;
}

cogdl_status vocab_logits_launch(VocabArgs a, cogdl_dtype dtype, bool grad, bool wide, hipStream_t stream)
{
    const bool direct = on_grid(a.W, a.k);
    const int tile = wide ? 256 : 128, waves = wide ? 8 : 4;
    const bool extra = a.bias || (grad && a.db_part);
    const VocabKernel kern = dtype == COGDL_BF16 ? pick<bf16_t>(grad, extra, wide, direct) : pick<f16_t>(grad, extra, wide, direct);
    a.tiles_c = (int32_t)(((int64_t)a.width + tile - 1) / tile);
    const int64_t rows = grad ? a.n : a.block;
    const int64_t all = (rows + tile - 1) / tile * a.tiles_c;
    return launch_vocab(grad ? "vocab_dz" : "vocab_stats", kern, a, all, waves, lds_of(waves, tile, tile), stream);
}

}  // namespace cogdl

using namespace cogdl;

namespace {

// Bytes of statistics kept at once, about (256 rows' at least).
constexpr int64_t kPartBytes = 256ll << 20;

// The forward's workspace.
size_t lay_forward(VocabArgs &a, char *ws)
{
    Layout l;
    a.slots = (int32_t)(((int64_t)a.V + 63) / 64);
    int64_t block = kPartBytes / ((int64_t)sizeof(float2) * a.slots) / 256 * 256;
    if (block < 256) block = 256;
    a.block = (int32_t)(block < a.n ? block : a.n);
    a.head = reinterpret_cast<RowsHead *>(ws + l.take(sizeof(RowsHead)));
    a.live = reinterpret_cast<int32_t *>(ws + l.take(a.distill ? 4 * (size_t)a.n : 0));
    a.tlse = reinterpret_cast<float2 *>(ws + l.take(a.distill ? 8 * (size_t)a.n : 0));
    a.counts = reinterpret_cast<int32_t *>(ws + l.take(a.n > kManyRows ? 4 * kMostRuns : 0));
    a.rows = reinterpret_cast<int32_t *>(ws + l.take(4 * (size_t)a.n));
    a.Xr = ws + l.take(2 * (size_t)a.n * a.kp);
    a.part = reinterpret_cast<float2 *>(ws + l.take(sizeof(float2) * (size_t)a.block * a.slots));
    return l.total;
}

cogdl_status run_forward(VocabArgs a, cogdl_dtype dtype, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (dtype != COGDL_BF16 && dtype != COGDL_F16) return COGDL_ERR_DTYPE;
    const cogdl_status st = check_sizes(a);
    if (st != COGDL_OK) return st;
    if (a.n == 0) return COGDL_OK;
    if (!a.index || !a.loss || !a.lse || (a.k > 0 && (!a.X || !a.W))) return COGDL_ERR_INVALID;
    if (a.distill && (!a.teacher || !a.logp)) return COGDL_ERR_INVALID;
    a.kp = (a.k + 7) / 8 * 8;
    a.per_z = kLog2e / a.T;
    const size_t need = lay_forward(a, static_cast<char *>(workspace));
    if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < need) return COGDL_ERR_INVALID;
    a.v0 = 0;
    a.width = a.V;
    // Rows do not meet in the forward: they need not be gathered where that costs more than the tiles of rows that
    // do not count (one tile of rows costs the same anyway).  One row, 50000 x 512: 22 us a call gathered, 19 so.
    a.plain = on_grid(a.X, a.k) && (a.n <= 128 || (a.n <= 4096 && (double)a.n * a.V * a.k <= (double)(1ll << 33)));
    if (a.plain) {
        a.Xr = const_cast<void *>(a.X);
        a.kp = a.k;
    }
    cogdl_status s = vocab_rows_launch(a, dtype, false, stream);
    if (s != COGDL_OK) return s;
    const bool wide = vocab_wide(a.block, a.V, a.k, a.W);
    const int R = a.block <= 256 ? 1 : a.block <= 1024 ? 4 : 16;
    int64_t blocks = (a.block + R - 1) / R;
    if (blocks > 4096) blocks = 4096;
    for (a.p0 = 0; a.p0 < a.n; a.p0 += a.block) {
        bool few = false;
        s = dtype == COGDL_BF16 ? few_launch<bf16_t>(a, few, stream) : few_launch<f16_t>(a, few, stream);
        if (s == COGDL_OK && !few) s = vocab_logits_launch(a, dtype, false, wide, stream);
        if (s != COGDL_OK) return s;
        if (dtype == COGDL_BF16) COGDL_LAUNCH("vocab_finish", k_vocab_finish<bf16_t>, (unsigned)blocks, kBlock, stream, a, R);
        else COGDL_LAUNCH("vocab_finish", k_vocab_finish<f16_t>, (unsigned)blocks, kBlock, stream, a, R);
    }
    return COGDL_OK;
}

}  // namespace

extern "C" {

cogdl_status cogdl_linear_loss_workspace(int64_t n, int32_t V, int32_t k, int32_t K, size_t *bytes)
{
    if (!bytes || K < 0) return COGDL_ERR_INVALID;
    VocabArgs a{};
    a.n = n; a.V = V; a.k = k;
    a.entries = K > 0 ? K : 1;
    a.distill = K > 0;
    a.T = 1.f;
    const cogdl_status st = check_sizes(a);
    if (st != COGDL_OK) return st;
    a.kp = (k + 7) / 8 * 8;
    *bytes = n > 0 ? lay_forward(a, nullptr) : 0;
    return COGDL_OK;
}

cogdl_status cogdl_linear_cross_entropy(int64_t n, int32_t V, int32_t k, const void *X, const void *W,
                                        cogdl_dtype dtype, const float *bias, const int32_t *target, float *loss,
                                        float *lse, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    VocabArgs a{};
    a.n = n; a.V = V; a.k = k;
    a.entries = 1;
    a.T = 1.f;
    a.X = X; a.W = W;
    a.bias = bias;
    a.index = target;
    a.loss = loss; a.lse = lse;
    return run_forward(a, dtype, workspace, workspace_bytes, stream);
}

cogdl_status cogdl_linear_distill(int64_t n, int32_t V, int32_t k, int32_t K, const void *X, const void *W,
                                  cogdl_dtype dtype, const float *bias, const int32_t *index, const float *teacher,
                                  float temperature, float *loss, float *lse, float *logp, void *workspace,
                                  size_t workspace_bytes, hipStream_t stream)
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
    a.loss = loss; a.lse = lse; a.logp = logp;
    return run_forward(a, dtype, workspace, workspace_bytes, stream);
}

}  // extern "C"
