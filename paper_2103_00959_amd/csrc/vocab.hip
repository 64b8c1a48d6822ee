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
// the sum of their exponentials.  FORWARD: also the student's logits of the entries, by 4 entries of 16 lanes,
// into logp.  A wavefront a row.
template <typename T, bool FORWARD>
__global__ __launch_bounds__(kBlock) void k_teacher_rows(VocabArgs a)
{
    const int lane = lane_id();
    const int64_t waves = (int64_t)gridDim.x * (kBlock / kWave);
    for (int64_t i = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave; i < a.n; i += waves) {
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
        if (lane == 0) {
            a.live[i] = live ? 0 : -1;
            a.tlse[i] = from + logf(s);
        }
        if constexpr (FORWARD) {
            const T *__restrict__ x = static_cast<const T *>(a.X) + i * a.k;
            const int sub = lane & 15, vecs = a.kp / 8;
            for (int e0 = 0; e0 < a.entries; e0 += kWave / 16) {
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

// The rows that count, in order, and their features; in the forward of the cross entropy also their targets'
// logits, into loss.  A workgroup takes `per` rows; how many count before them
// it finds by itself, from the targets (n targets a workgroup, from the L2s).
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
    int before = 0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < from; i += kBlock) before += counts(live[i], limit) ? 1 : 0;
    before = wave_inclusive_scan(before);
    if (lane == kWave - 1) wsum[wave] = before;
    __syncthreads();
    int at = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) at += wsum[w];
    if (BACKWARD && blockIdx.x == 0) {
        // the largest |g T| that counts, for a power of two that brings every dz below 2^15 (and keeps what
        // fp16 can of the small ones)
        float top = 0.f;
#pragma unroll 4
        for (int64_t i = threadIdx.x; i < a.n; i += kBlock)
            if (counts(live[i], limit)) top = fmaxf(top, fabsf(a.dloss[i] * a.T));
        top = group_reduce(top, kWave, [](float x, float y) { return fmaxf(x, y); });
        if (lane == 0) wmax[wave] = top;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 0; w < W; ++w) top = fmaxf(top, wmax[w]);
            int e = 0;
            if (top > 0.f && top <= 3.4e38f) {
                (void)frexpf(top, &e);                     // top < 2^e
                e = 15 - e;
                e = e > 120 ? 120 : e < -120 ? -120 : e;
            }
            a.head->scale = ldexpf(1.f, e);
            a.head->unscale = ldexpf(1.f, -e);
        }
    }
    if (BACKWARD && a.db_q) {
        for (int64_t v = (int64_t)blockIdx.x * kBlock + threadIdx.x; v < a.V; v += (int64_t)gridDim.x * kBlock) a.db_q[v] = 0;
    }
    const T *__restrict__ X = static_cast<const T *>(a.X);
    T *__restrict__ Xr = static_cast<T *>(a.Xr);
    T *__restrict__ dX = static_cast<T *>(a.dX);
    const int vecs = a.kp / 8;
    // 64 rows at a time, every wavefront alike; a wavefront moves every fourth row
    for (int64_t r0 = from; r0 < to; r0 += kWave) {
        const int64_t i = r0 + lane;
        const bool mine = i < to && counts(live[i], limit);
        const uint64_t mask = __ballot(mine);
        if (wave == 0 && i < to) {
            if (mine) {
                const int p = at + __popcll(mask & ((1ull << lane) - 1));
                a.rows[p] = (int32_t)i;
                if constexpr (BACKWARD) {
                    a.lse2[p] = a.lse_in[i] * kLog2e;
                    a.g[p] = a.dloss[i] * a.T;
                }
            } else if constexpr (!BACKWARD) {
                a.loss[i] = 0.f;
                a.lse[i] = 0.f;
            }
        }
        const int here = to - r0 < kWave ? (int)(to - r0) : kWave;
#pragma unroll 2
        for (int r = wave; r < here; r += W) {
            const bool on = mask >> r & 1;
            const int64_t i1 = r0 + r;
            if (on) {
                const int64_t p = at + __popcll(mask & ((1ull << r) - 1));
                const T *__restrict__ x = X + i1 * a.k;
                const int32_t v1 = !BACKWARD && !a.distill ? a.index[i1] : 0;
                const T *__restrict__ w = static_cast<const T *>(a.W) + (int64_t)v1 * a.k;
                float z = 0.f;
                for (int v = lane; v < vecs; v += kWave) {
                    const uint4 f = load_vec8(x, v, a.k);
                    *reinterpret_cast<uint4 *>(Xr + p * a.kp + 8 * v) = f;
                    if constexpr (!BACKWARD)
                        if (!a.distill) z = dot8<T>(f, load_vec8(w, v, a.k), z);
                }
                if constexpr (!BACKWARD) {
                    if (!a.distill) {
                        z = group_sum(z, kWave);
                        if (lane == 0) a.loss[i1] = a.bias ? z + a.bias[v1] : z;
                    }
                }
            } else if constexpr (BACKWARD) {
                if (dX) {
                    const float zeros[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    for (int v = lane; v < vecs; v += kWave) store8(dX + i1 * a.k, 8 * v, a.k, zeros);
                }
            }
        }
        at += __popcll(mask);
    }
    if (to == a.n && threadIdx.x == 0) {
        a.head->off[0] = 0;
        a.head->off[1] = at;
    }
}

// Tiles of logits.  GRAD: dz of the piece, else each row's (max, sum) over the wavefront's columns.
template <typename T, int WAVES, int TM, int TN, int SRCB, bool GRAD>
__global__ __launch_bounds__(WAVES * kWave) void k_vocab_logits(VocabArgs a)
{
    constexpr int N = WAVES * kWave;
    constexpr int WAVES_C = TN >= 256 ? 4 : 2, WAVES_R = WAVES / WAVES_C;
    constexpr int WR = TM / WAVES_R / 32, WC = TN / WAVES_C / 32;
    extern __shared__ __align__(16) char lds[];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int wr = wave / WAVES_C, wc = wave % WAVES_C;
    const int r0 = wr * (32 * WR), c0 = wc * (32 * WC);
    GridWalk walk;
    walk.start(a.head->off[1], TM, a.tiles_c, 1);
    RowOperand<T, TM, N, kDirect> A;
    RowOperand<T, TN, N, SRCB> B;
    const auto open = [&](const Span &s) {
        const int col = s.tile * TN, cols = a.width - col < TN ? a.width - col : TN;
        A.open(static_cast<const T *>(a.Xr) + s.lo * a.kp, nullptr, s.have, a.kp, 0);
        B.open(static_cast<const T *>(a.W) + ((int64_t)a.v0 + col) * a.k, nullptr, cols, a.k, 0);
        return a.kp;
    };
    char *const mine = lds + 2 * (TM + TN) * kX * 2 + wave * kOutBytes;
    run_tiles<T, decltype(A), decltype(B), WR, WC>(
        lds, walk, A, B, r0, c0, open, [&](const Span &s) { return r0 < s.have && s.tile * TN + c0 < a.width; },
        [](const Span &, const uint4 (&)[WR]) {}, [](const Span &) {},
        [&](const Span &s, const Acc<WR, WC> &acc) {
            const int col0 = s.tile * TN + c0;
            if constexpr (!GRAD) {
                // this lane's columns of a block: 8 (t / 4) + 4 (lane / 32) + t % 4, of row lane % 32
                float add[WC][16];
                const int first = col0 + 4 * (lane >> 5);
#pragma unroll
                for (int j = 0; j < WC; ++j)
#pragma unroll
                    for (int t = 0; t < 16; ++t) {
                        const int c = first + 32 * j + 8 * (t / 4) + t % 4;
                        add[j][t] = c < a.width ? a.bias ? a.bias[a.v0 + c] : 0.f : -INFINITY;
                    }
                const int slot = s.tile * WAVES_C + wc;
                if (slot >= a.slots) return;
#pragma unroll
                for (int i = 0; i < WR; ++i) {
                    float m = -INFINITY;
                    float z[WC][16];
#pragma unroll
                    for (int j = 0; j < WC; ++j)
#pragma unroll
                        for (int t = 0; t < 16; ++t) {
                            z[j][t] = acc.a[i][j][t] + add[j][t];
                            m = fmaxf(m, z[j][t]);
                        }
                    m = fmaxf(m, bfly_partner<32>(m)) * a.per_z;
                    const float from = m == -INFINITY ? 0.f : m;
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < WC; ++j)
#pragma unroll
                        for (int t = 0; t < 16; ++t) sum += __builtin_amdgcn_exp2f(fmaf(z[j][t], a.per_z, -from));
                    sum += bfly_partner<32>(sum);
                    const int r = r0 + 32 * i + (lane & 31);
                    if (lane < 32 && r < s.have) a.part[(int64_t)slot * a.n + s.lo + r] = make_float2(m, sum);
                }
            } else {
                const float scale = a.head->scale;
                T *__restrict__ dz = static_cast<T *>(a.dz) + s.lo * a.pitch;
                float add[WC][8], sums[WC][8];
#pragma unroll
                for (int j = 0; j < WC; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int c = col0 + 32 * j + 8 * (lane & 3) + e;
                        add[j][e] = c < a.width ? a.bias ? a.bias[a.v0 + c] : 0.f : -INFINITY;
                        sums[j][e] = 0.f;
                    }
                for_outputs<WR, WC>(mine, acc, [&](int bc, int r, int c, float (&v)[8]) {
                    r += r0;
                    c += col0;
                    if (r >= s.have || c >= a.pitch) return;
                    const float less = a.lse2[s.lo + r], g = a.g[s.lo + r] * scale;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[e] = __builtin_amdgcn_exp2f(fmaf(v[e] + add[bc][e], a.per_z, -less)) * g;
                        sums[bc][e] += v[e];
                    }
                    store_vec<T, 8>(dz + (int64_t)r * a.pitch, c, v);
                });
                if (a.db_part) {
                    // over the 16 lanes that share 8 columns, in a fixed order
                    float *__restrict__ to = a.db_part + ((int64_t)s.g * WAVES_R + wr) * a.V + a.v0;
#pragma unroll
                    for (int j = 0; j < WC; ++j)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            float t = sums[j][e];
                            t += __shfl_xor(t, 4);
                            t += __shfl_xor(t, 8);
                            t += __shfl_xor(t, 16);
                            t += __shfl_xor(t, 32);
                            const int c = col0 + 32 * j + 8 * (lane & 3) + e;
                            if (lane < 4 && c < a.width) to[c] = t;
                        }
                }
            }
        });
}

// The slots of a row joined to its lse, and the loss from its targets' logits.  kRowsBlock rows a workgroup.
constexpr int kRowsBlock = 16;

__global__ __launch_bounds__(kBlock) void k_vocab_finish(VocabArgs a)
{
    constexpr int W = kBlock / kWave, S = kBlock / kRowsBlock;
    __shared__ float2 part[S][kRowsBlock];
    __shared__ float lse_of[kRowsBlock];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int64_t live = a.head->off[1];
    const int r = threadIdx.x % kRowsBlock, sg = threadIdx.x / kRowsBlock;
    for (int64_t r0 = (int64_t)blockIdx.x * kRowsBlock; r0 < live; r0 += (int64_t)gridDim.x * kRowsBlock) {
        float m = -INFINITY, z = 0.f;
        if (r0 + r < live) {
#pragma unroll 4
            for (int s = sg; s < a.slots; s += S) {
                const float2 p = a.part[(int64_t)s * a.n + r0 + r];
                const float top = fmaxf(m, p.x);
                const float from = top == -INFINITY ? 0.f : top;
                z = z * __builtin_amdgcn_exp2f(m - from) + p.y * __builtin_amdgcn_exp2f(p.x - from);
                m = top;
            }
        }
        part[sg][r] = make_float2(m, z);
        __syncthreads();
        if (threadIdx.x < kRowsBlock) {
            float top = -INFINITY;
            for (int s = 0; s < S; ++s) top = fmaxf(top, part[s][r].x);
            const float from = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            for (int s = 0; s < S; ++s) sum += part[s][r].y * __builtin_amdgcn_exp2f(part[s][r].x - from);
            const float lse = (from + log2f(sum)) * kLn2;
            lse_of[r] = lse;
            if (r0 + r < live) {
                const int64_t i = a.rows[r0 + r];
                a.lse[i] = lse;
                if (!a.distill) {
                    // (above 0 by definition; the two sums' roundings may differ)
                    const float loss = lse - a.loss[i];
                    a.loss[i] = loss < 0.f ? 0.f : loss;
                }
            }
        }
        __syncthreads();
        if (!a.distill) continue;
        for (int q = wave; q < kRowsBlock && r0 + q < live; q += W) {
            const int64_t i = a.rows[r0 + q];
            const float lse = lse_of[q], tlse = a.tlse[i];
            float loss = 0.f;
            for (int e = lane; e < a.entries; e += kWave) {
                if (!counts(a.index[i * a.entries + e], a.V)) continue;       // (logp is 0)
                const float logp = a.logp[i * a.entries + e] - lse, logq = a.teacher[i * a.entries + e] / a.T - tlse;
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

template <typename T, int WAVES, int TM, int TN>
VocabKernel pick(bool direct, bool grad)
{
    if (grad) return direct ? k_vocab_logits<T, WAVES, TM, TN, kDirect, true> : k_vocab_logits<T, WAVES, TM, TN, kStaged, true>;
    return direct ? k_vocab_logits<T, WAVES, TM, TN, kDirect, false> : k_vocab_logits<T, WAVES, TM, TN, kStaged, false>;
}

}  // namespace

bool vocab_wide(int64_t n, int64_t cols, int32_t k, const void *W)
{
    return on_grid(W, k) && ((n + 255) / 256) * ((cols + 255) / 256) >= 256;
}

cogdl_status vocab_rows_launch(const VocabArgs &a, cogdl_dtype dtype, bool backward, hipStream_t stream)
{
    if (a.distill && a.n > 0) {
        const int64_t blocks = (a.n + kBlock / kWave - 1) / (kBlock / kWave);
        const unsigned grid = (unsigned)(blocks < 8192 ? blocks : 8192);
        if (backward) COGDL_LAUNCH("teacher_rows", (k_teacher_rows<bf16_t, false>), grid, kBlock, stream, a);    // (no features)
        else if (dtype == COGDL_BF16) COGDL_LAUNCH("teacher_rows", (k_teacher_rows<bf16_t, true>), grid, kBlock, stream, a);
        else COGDL_LAUNCH("teacher_rows", (k_teacher_rows<f16_t, true>), grid, kBlock, stream, a);
    }
    int64_t per = (a.n + 511) / 512;
    per = per < 8 ? 8 : per;
    const unsigned blocks = a.n > 0 ? (unsigned)((a.n + per - 1) / per) : 1;
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
    VocabKernel kern;
    if (dtype == COGDL_BF16) kern = wide ? pick<bf16_t, 8, 256, 256>(true, grad) : pick<bf16_t, 4, 128, 128>(direct, grad);
    else kern = wide ? pick<f16_t, 8, 256, 256>(true, grad) : pick<f16_t, 4, 128, 128>(direct, grad);
    a.tiles_c = (int32_t)(((int64_t)a.width + tile - 1) / tile);
    const int64_t all = (a.n + tile - 1) / tile * a.tiles_c;
    return launch_vocab(grad ? "vocab_dz" : "vocab_stats", kern, a, all, waves, lds_of(waves, tile, tile), stream);
}

}  // namespace cogdl

using namespace cogdl;

namespace {

struct Layout {
    size_t total = 0;
    size_t take(size_t bytes)
    {
        const size_t at = total;
        total += (bytes + 255) & ~size_t(255);
        return at;
    }
};

// The forward's workspace.
size_t lay_forward(VocabArgs &a, char *ws)
{
    Layout l;
    a.slots = (int32_t)(((int64_t)a.V + 63) / 64);
    a.head = reinterpret_cast<RowsHead *>(ws + l.take(sizeof(RowsHead)));
    a.live = reinterpret_cast<int32_t *>(ws + l.take(a.distill ? 4 * (size_t)a.n : 0));
    a.tlse = reinterpret_cast<float *>(ws + l.take(a.distill ? 4 * (size_t)a.n : 0));
    a.rows = reinterpret_cast<int32_t *>(ws + l.take(4 * (size_t)a.n));
    a.Xr = ws + l.take(2 * (size_t)a.n * a.kp);
    a.part = reinterpret_cast<float2 *>(ws + l.take(sizeof(float2) * (size_t)a.n * a.slots));
    return l.total;
}

cogdl_status check_sizes(int64_t n, int32_t V, int32_t k, int32_t K)
{
    if (n < 0 || V < 1 || k < 0 || K < 1) return COGDL_ERR_INVALID;
    if (n > kMaxRows || k > kMaxWidth || K > kMaxEntries) return COGDL_ERR_TOO_LARGE;
    if (!countable((n + 127) / 128, ((int64_t)V + 127) / 128)) return COGDL_ERR_TOO_LARGE;
    return COGDL_OK;
}

cogdl_status run_forward(VocabArgs a, cogdl_dtype dtype, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (dtype != COGDL_BF16 && dtype != COGDL_F16) return COGDL_ERR_DTYPE;
    const cogdl_status st = check_sizes(a.n, a.V, a.k, a.entries);
    if (st != COGDL_OK) return st;
    if (!(a.T > 0.f) || a.T > 3.4e38f) return COGDL_ERR_INVALID;
    if (a.n == 0) return COGDL_OK;
    if (!a.index || !a.loss || !a.lse || (a.k > 0 && (!a.X || !a.W))) return COGDL_ERR_INVALID;
    if (a.distill && (!a.teacher || !a.logp)) return COGDL_ERR_INVALID;
    a.kp = (a.k + 7) / 8 * 8;
    a.per_z = kLog2e / a.T;
    const size_t need = lay_forward(a, static_cast<char *>(workspace));
    if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < need) return COGDL_ERR_INVALID;
    a.v0 = 0;
    a.width = a.V;
    cogdl_status s = vocab_rows_launch(a, dtype, false, stream);
    if (s != COGDL_OK) return s;
    s = vocab_logits_launch(a, dtype, false, vocab_wide(a.n, a.V, a.k, a.W), stream);
    if (s != COGDL_OK) return s;
    int64_t blocks = (a.n + kRowsBlock - 1) / kRowsBlock;
    if (blocks > 4096) blocks = 4096;
    COGDL_LAUNCH("vocab_finish", k_vocab_finish, (unsigned)blocks, kBlock, stream, a);
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
    const cogdl_status st = check_sizes(n, V, k, a.entries);
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
