// Products of rows that lie sorted by group (node types, relations, experts), each group
// with a weight matrix of its own, and their gradients:
//     Y[i, c]     = act(sum_j X[i, j] W[g, c, j] + bias[g, c])        rows i of group g
//     dX[i, j]    = sum_c dZ[i, c] W[g, c, j]                          dZ = dY act'(Y)
//     dW[g, c, j] = sum_{i in g} dZ[i, c] X[i, j],   db[g, c] = sum_{i in g} dZ[i, c]
//
// All three are C[r, c] = sum_x A(r, x) B(c, x) on one tile engine: a workgroup of four
// wavefronts owns kTileR x TN outputs of one group and walks x in chunks of 64, both
// operands' chunks staged in LDS.  An operand lies in memory with x along its rows (X and W
// of the forward, dZ of dX: "row" operands) or with x down its rows (W of dX, both of dW:
// "col" operands); a row operand's matrix fragments are plain 16-byte LDS reads, a col
// operand's are the LDS reads that transpose 4 x 16 elements.  The offsets stay on the device:
// the grid covers the most tiles that n rows in E groups can have, and each workgroup finds
// its group by a scan of the group sizes.
//
// dW sums over the rows, whose number only the device knows: groups are cut into chunks of
// rows; a group of one chunk writes its result, the others write fp32 partial sums into the
// workspace, added up in chunk order by k_reduce_chunks (no atomics: the same bits every run).
#include "checkpoint.hpp"
#include "internal.hpp"

namespace cogdl {
namespace {

constexpr int kBlock = 256;
constexpr int kTileR = 128;      // rows of a tile (forward, dX); outputs c of a tile (dW)
constexpr int kX = 64;           // x elements of a chunk
constexpr int kPieces = kX / 8;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_b __attribute__((ext_vector_type(2), aligned(1)));

template <typename T>
__device__ __forceinline__ f32x16 mfma_32x32x16(uint4 a, uint4 b, f32x16 c)
{
    if constexpr (Fmt<T>::code == COGDL_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// ---------------------------------------------------------------- groups

// Rows [lo, hi) of group g: piece `local` of the pieces of `per` rows that the groups are
// cut into, `count` pieces in this group, `slot` pieces of groups with several before it.
struct Span {
    int g;
    int64_t lo, hi;
    int local, count;
    int64_t slot;
};

// Offsets as the kernels use them: inside [0, n], so that no contents of the device array
// lead outside the operands.
__device__ __forceinline__ int64_t offset_at(const int32_t *__restrict__ off, int e, int64_t n)
{
    const int64_t o = off[e];
    return o < 0 ? 0 : (o < n ? o : n);
}

// Piece t of all pieces (false past the last one), found by one wavefront (uniform).
__device__ __forceinline__ bool find_span(const int32_t *__restrict__ off, int E, int64_t n, int per, int64_t t,
                                          Span &s)
{
    const int lane = lane_id();
    int64_t slot = 0;
    for (int base = 0; base < E; base += kWave) {
        const int e = base + lane;
        int64_t lo = 0, hi = 0;
        if (e < E) {
            lo = offset_at(off, e, n);
            hi = offset_at(off, e + 1, n);
        }
        const int size = hi > lo ? (int)(hi - lo) : 0;
        const int pieces = (int)(((int64_t)size + per - 1) / per);
        const int before = wave_inclusive_scan(pieces);
        const int total = __builtin_amdgcn_readlane(before, kWave - 1);
        const int many = pieces > 1 ? pieces : 0;
        const int many_before = wave_inclusive_scan(many);
        if (t < total) {
            const int l = __builtin_ctzll(__ballot((int64_t)before > t));
            s.g = base + l;
            s.count = __builtin_amdgcn_readlane(pieces, l);
            s.local = (int)t - (__builtin_amdgcn_readlane(before, l) - s.count);
            const int64_t first = __builtin_amdgcn_readlane((int)lo, l);
            const int64_t end = first + __builtin_amdgcn_readlane(size, l);
            s.lo = first + (int64_t)s.local * per;
            s.hi = s.lo + per < end ? s.lo + per : end;
            s.slot = slot + __builtin_amdgcn_readlane(many_before - many, l);
            return true;
        }
        t -= total;
        slot += __builtin_amdgcn_readlane(many_before, kWave - 1);
    }
    return false;
}

// -------------------------------------------------------- pieces of memory

__device__ __forceinline__ uint4 load16(const void *p)
{
    const u32x4_u v = *reinterpret_cast<const u32x4_u *>(p);
    return make_uint4(v.x, v.y, v.z, v.w);
}

// Elements [at, at + 8) of a row of `width` 16-bit elements, zeros past its end: a ragged end
// is the row's last 16 bytes shifted down.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T *__restrict__ row, int at, int width)
{
    if (at + 8 <= width) return load16(row + at);
    if (at >= width) return make_uint4(0u, 0u, 0u, 0u);
    if (width >= 8) {
        const uint4 v = load16(row + width - 8);
        const int gone = at + 8 - width;              // 1 to 7 elements
        const unsigned __int128 all = ((unsigned __int128)(((uint64_t)v.w << 32) | v.z) << 64) |
                                      (((uint64_t)v.y << 32) | v.x);
        const unsigned __int128 r = all >> (16 * gone);
        return make_uint4((uint32_t)r, (uint32_t)(r >> 32), (uint32_t)(r >> 64), (uint32_t)(r >> 96));
    }
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t lo = at + 2 * j < width ? row[at + 2 * j].bits : 0u;
        const uint32_t hi = at + 2 * j + 1 < width ? row[at + 2 * j + 1].bits : 0u;
        w[j] = lo | (hi << 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Codes [at, at + 8) of a row of a checkpoint, zeros past its end.
__device__ __forceinline__ uint2 load_codes(const int8_t *__restrict__ row, int at, int width)
{
    if (at + 8 <= width) {
        const u32x2_b v = *reinterpret_cast<const u32x2_b *>(row + at);
        return make_uint2(v.x, v.y);
    }
    uint64_t r = 0;
    if (at < width) {
        if (width >= 8) {
            const u32x2_b v = *reinterpret_cast<const u32x2_b *>(row + width - 8);
            r = (((uint64_t)v.y << 32) | v.x) >> (8 * (at + 8 - width));
        } else {
            for (int j = 0; j < 8; ++j)
                if (at + j < width) r |= (uint64_t)(uint8_t)row[at + j] << (8 * j);
        }
    }
    return make_uint2((uint32_t)r, (uint32_t)(r >> 32));
}

template <typename T>
__device__ __forceinline__ void unpack8(uint4 v, float (&o)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (Fmt<T>::code == COGDL_BF16) {
            o[2 * j] = bf16_lo(w[j]);
            o[2 * j + 1] = bf16_hi(w[j]);
        } else {
            o[2 * j] = f16_bits_to_f32(w[j] & 0xffffu);
            o[2 * j + 1] = f16_bits_to_f32(w[j] >> 16);
        }
    }
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (Fmt<T>::code == COGDL_BF16) return f32x2_to_bf16(a, b);
    else return f32_to_f16(a) | (f32_to_f16(b) << 16);
}

template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&v)[8])
{
    return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}

// 8 codes as 8 elements of T: exact in bf16, and in fp16 from fp16 activations.
template <typename T>
__device__ __forceinline__ uint4 decode8(uint2 codes, uint32_t b)
{
    const float s = ckpt_scale(b);
    float lo[4], hi[4];
    ckpt_decode4(codes.x, s, lo);
    ckpt_decode4(codes.y, s, hi);
    return make_uint4(pack2<T>(lo[0], lo[1]), pack2<T>(lo[2], lo[3]), pack2<T>(hi[0], hi[1]),
                      pack2<T>(hi[2], hi[3]));
}

// d act'(y) from the activation's output y: relu 1 where y > 0 and 0 elsewhere, ELU 1 where
// y > 0 and y + 1 = exp(v) elsewhere.
__device__ __forceinline__ float act_grad(float d, float y, int act)
{
    if (act == COGDL_ACT_RELU) return y > 0.f ? d : 0.f;
    return y > 0.f ? d : d * (y + 1.f);
}

// ------------------------------------------------------------- LDS tiles
// A row tile holds R rows of 64 x (128 bytes): 16-byte piece p of row r lies at p ^ (r / 2
// mod 8), so that the 16 rows that a phase of fragment reads takes cover all banks.  A col
// tile holds 64 x of C elements: the 32-byte granules of a row are permuted by the row, so
// that the four rows a transposing read takes lie on different banks.

__device__ __forceinline__ int row_tile_at(int r, int p) { return r * (kX * 2) + ((p ^ ((r >> 1) & 7)) << 4); }

template <int C>
__device__ __forceinline__ int col_tile_at(int x, int byte)
{
    const int f = C >= 128 ? (x & 3) << 1 : ((x >> 1) & 1) << 1;
    return x * (C * 2) + (byte ^ (f << 5));
}

// 8 consecutive x (16 s + 8 (lane / 32) ...) of index idx0 + lane % 32 of a tile.
__device__ __forceinline__ uint4 row_fragment(const char *tile, int idx0, int s)
{
    const int lane = lane_id();
    return *reinterpret_cast<const uint4 *>(tile + row_tile_at(idx0 + (lane & 31), 2 * s + (lane >> 5)));
}

template <int C>
__device__ __forceinline__ uint4 col_fragment(char *tile, int idx0, int s)
{
    const int lane = lane_id(), q = lane >> 4, l = lane & 15;
    const int x = 16 * s + 8 * (q >> 1) + (l >> 2);
    const int byte = 2 * (idx0 + 16 * (q & 1) + 4 * (l & 3));
    typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + col_tile_at<C>(x, byte)));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + col_tile_at<C>(x + 4, byte)));
    const uint2 u = __builtin_bit_cast(uint2, a), v = __builtin_bit_cast(uint2, b);
    return make_uint4(u.x, u.y, v.x, v.y);
}

// ------------------------------------------------------------- operands
// An operand's chunk on its way from memory to LDS: fetch() starts the loads of the pieces
// this thread brings, put() writes them once the tile is free.

// R indices (rows of the matrix) x 64 x along the row; indices from `have` on repeat the last.
template <typename T, int R, bool ACT>
struct RowOperand {
    static constexpr int N = R * kPieces / kBlock;
    const T *row[N];
    const T *yrow[ACT ? N : 1];
    int width, act;
    uint4 v[N], y[ACT ? N : 1];

    __device__ __forceinline__ void open(const T *base, const T *ybase, int64_t stride, int have, int w, int a)
    {
        width = w;
        act = a;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            int r = ((int)threadIdx.x + q * kBlock) / kPieces;
            r = r < have ? r : have - 1;
            row[q] = base + r * stride;
            if constexpr (ACT) yrow[q] = ybase + r * stride;
        }
    }
    __device__ __forceinline__ void fetch(int x0)
    {
        const int at = x0 + (threadIdx.x % kPieces) * 8;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            v[q] = load_piece<T>(row[q], at, width);
            if constexpr (ACT) y[q] = load_piece<T>(yrow[q], at, width);
        }
    }
    __device__ __forceinline__ void put(char *tile)
    {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            uint4 w = v[q];
            if constexpr (ACT) {
                float d[8], o[8];
                unpack8<T>(w, d);
                unpack8<T>(y[q], o);
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = act_grad(d[e], o[e], act);
                w = pack8<T>(d);        // the matrix cores take 16 bits
            }
            const int r = ((int)threadIdx.x + q * kBlock) / kPieces;
            *reinterpret_cast<uint4 *>(tile + row_tile_at(r, threadIdx.x % kPieces)) = w;
        }
    }
};

// 64 x (rows of the matrix, those from x_end on zero) by C indices along the row, from column c0.
// SUM: keeps this thread's share of the sums over x of its 8 columns.
template <typename T, int C, bool ACT, bool CODES, bool SUM>
struct ColOperand {
    static constexpr int P = C / 8;
    static constexpr int N = kX * P / kBlock;
    const T *base, *ybase;
    const int8_t *codes;
    const uint8_t *exps;
    int64_t stride;
    int at, width, act, nb;
    uint4 v[N], y[ACT ? N : 1];
    uint32_t b[CODES ? N : 1];
    float sum[SUM ? 8 : 1];

    __device__ __forceinline__ void open(const T *p, const T *py, const int8_t *pc, const uint8_t *pe, int c0, int w,
                                         int a)
    {
        base = p;
        ybase = py;
        codes = pc;
        exps = pe;
        stride = w;
        width = w;
        act = a;
        nb = (w + kCkptBlock - 1) / kCkptBlock;
        at = c0 + (threadIdx.x % P) * 8;
#pragma unroll
        for (int e = 0; e < (SUM ? 8 : 1); ++e) sum[e] = 0.f;
    }
    __device__ __forceinline__ void fetch(int64_t x0, int64_t x_end)
    {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int64_t x = x0 + ((int)threadIdx.x + q * kBlock) / P;
            if constexpr (CODES) b[q] = 0u;
            v[q] = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (ACT) y[q] = v[q];
            if (x >= x_end || at >= width) continue;
            if constexpr (CODES) {
                const uint2 w = load_codes(codes + x * stride, at, width);
                v[q].x = w.x;
                v[q].y = w.y;
                b[q] = exps[x * nb + at / kCkptBlock];
            } else {
                v[q] = load_piece<T>(base + x * stride, at, width);
                if constexpr (ACT) y[q] = load_piece<T>(ybase + x * stride, at, width);
            }
        }
    }
    __device__ __forceinline__ void put(char *tile)
    {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            uint4 w = v[q];
            if constexpr (CODES) w = decode8<T>(make_uint2(w.x, w.y), b[q]);
            if constexpr (ACT || SUM) {
                float d[8];
                unpack8<T>(w, d);
                if constexpr (ACT) {
                    float o[8];
                    unpack8<T>(y[q], o);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[e] = act_grad(d[e], o[e], act);
                    w = pack8<T>(d);    // the matrix cores take 16 bits; the sums do not round
                }
                if constexpr (SUM) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += d[e];
                }
            }
            const int x = ((int)threadIdx.x + q * kBlock) / P;
            *reinterpret_cast<uint4 *>(tile + col_tile_at<C>(x, (threadIdx.x % P) * 16)) = w;
        }
    }
};

// ------------------------------------------------------------ the engine

// A wavefront's WR x WC blocks of 32 x 32 outputs.  The c operand goes first into the matrix
// instruction: register t of lane l is then c = 8 (t / 4) + 4 (l / 32) + t % 4 of row l % 32.
template <int WR, int WC>
struct Acc {
    f32x16 a[WR][WC];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < WR; ++i)
#pragma unroll
            for (int j = 0; j < WC; ++j)
#pragma unroll
                for (int t = 0; t < 16; ++t) a[i][j][t] = 0.f;
    }
};

// Calls out(row in the block, column in the block, 8 consecutive outputs) for each 8 outputs:
// exchanges between the wavefront's halves make runs of 4 into runs of 8.
template <int WR, int WC, typename Out>
__device__ __forceinline__ void for_outputs(const Acc<WR, WC> &acc, Out out)
{
    const int lane = lane_id(), i = lane & 31, kq = lane >> 5;
#pragma unroll
    for (int br = 0; br < WR; ++br)
#pragma unroll
        for (int bc = 0; bc < WC; ++bc)
#pragma unroll
            for (int g = 0; g < 4; g += 2) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const auto sw = __builtin_amdgcn_permlane32_swap(
                        __float_as_uint(acc.a[br][bc][4 * g + e]), __float_as_uint(acc.a[br][bc][4 * g + 4 + e]),
                        false, false);
                    v[e] = __uint_as_float(sw[0]);
                    v[4 + e] = __uint_as_float(sw[1]);
                }
                out(32 * br + i, 32 * bc + 8 * (g + kq), v);
            }
}

// Stores those of 8 consecutive outputs from column c on that lie below width.
template <typename TY>
__device__ __forceinline__ void store8(TY *__restrict__ row, int c, int width, const float (&v)[8])
{
    if (c + 8 <= width) {
        store_vec<TY, 8>(row, c, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float one[1] = {v[e]};
            if (c + e < width) store_out<TY, 1>(row, c + e, one);
        }
    }
}

struct GroupedArgs {
    int64_t n;
    int32_t E, k, m;
    const int32_t *off;
    const void *X;          // n x k (null where codes are given)
    const int8_t *codes;
    const uint8_t *exps;
    const void *W;          // E x m x k
    const float *bias;      // E x m, nullable
    int32_t act;
    const void *dY;         // n x m
    const void *Y;          // n x m: the forward's outputs, where act' needs them
    void *out;              // Y, dX or dW
    float *db;              // E x m, nullable
    int32_t tiles_c;        // column tiles of a piece of rows (dW: tiles of an output matrix)
    int32_t per;            // rows of a piece
    float *part;            // dW: partial sums (m x k a slot), then those of db (m a slot)
    float *part_db;
};

// Pieces of rows are dealt round the 8 XCDs, the column tiles of a piece one after another on
// one of them: they share the piece's rows in its L2.
__device__ __forceinline__ void tile_of(int tiles_c, int64_t &piece, int &tile)
{
    const int64_t j = blockIdx.x >> 3;
    piece = j / tiles_c * 8 + (blockIdx.x & 7);
    tile = (int)(j % tiles_c);
}

// The forward (DX false) and dX (DX true): TN columns a tile.
template <typename T, typename TY, int TN, bool DX, bool ACT>
__global__ __launch_bounds__(kBlock) void k_grouped_rows(GroupedArgs a)
{
    constexpr int WAVES_C = TN == 128 ? 2 : 1, WAVES_R = 4 / WAVES_C;
    constexpr int WR = kTileR / WAVES_R / 32, WC = TN / WAVES_C / 32;
    __shared__ __align__(16) char sA[kTileR * kX * 2];
    __shared__ __align__(16) char sB[TN * kX * 2];
    int64_t piece;
    int tile;
    tile_of(a.tiles_c, piece, tile);
    Span s;
    if (!find_span(a.off, a.E, a.n, kTileR, piece, s)) return;
    const int wave = threadIdx.x / kWave;
    const int r0 = wave / WAVES_C * (32 * WR), c0 = wave % WAVES_C * (32 * WC);
    const int have = (int)(s.hi - s.lo);
    const int wx = DX ? a.m : a.k;                      // x
    const int wc = DX ? a.k : a.m;                      // outputs of a row
    const int col0 = tile * TN;
    const T *__restrict__ W = static_cast<const T *>(a.W) + (int64_t)s.g * a.m * a.k;
    RowOperand<T, kTileR, ACT> A;
    A.open(static_cast<const T *>(DX ? a.dY : a.X) + s.lo * wx, ACT ? static_cast<const T *>(a.Y) + s.lo * wx : nullptr,
           wx, have, wx, a.act);
    std::conditional_t<DX, ColOperand<T, TN, false, false, false>, RowOperand<T, TN, false>> B;
    if constexpr (DX) B.open(W, nullptr, nullptr, nullptr, col0, a.k, 0);
    else B.open(W + (int64_t)col0 * a.k, nullptr, a.k, a.m - col0 < TN ? a.m - col0 : TN, a.k, 0);
    Acc<WR, WC> acc;
    acc.clear();
    const auto fetch = [&](int x0) {
        A.fetch(x0);
        if constexpr (DX) B.fetch(x0, a.m);
        else B.fetch(x0);
    };
    if (wx > 0) fetch(0);
    for (int x0 = 0; x0 < wx; x0 += kX) {
        __syncthreads();
        A.put(sA);
        B.put(sB);
        __syncthreads();
        if (x0 + kX < wx) fetch(x0 + kX);
#pragma unroll
        for (int st = 0; st < kX / 16; ++st) {
            uint4 fa[WR], fb[WC];
#pragma unroll
            for (int i = 0; i < WR; ++i) fa[i] = row_fragment(sA, r0 + 32 * i, st);
#pragma unroll
            for (int j = 0; j < WC; ++j) {
                if constexpr (DX) fb[j] = col_fragment<TN>(sB, c0 + 32 * j, st);
                else fb[j] = row_fragment(sB, c0 + 32 * j, st);
            }
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int j = 0; j < WC; ++j) acc.a[i][j] = mfma_32x32x16<T>(fb[j], fa[i], acc.a[i][j]);
        }
    }
    TY *__restrict__ out = static_cast<TY *>(a.out) + s.lo * wc;
    const float *__restrict__ bias = !DX && a.bias ? a.bias + (int64_t)s.g * a.m : nullptr;
    for_outputs<WR, WC>(acc, [&](int r, int c, float (&v)[8]) {
        r += r0;
        c += col0 + c0;
        if (r >= have || c >= wc) return;
        if constexpr (!DX) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (bias) v[e] += bias[c + e < wc ? c + e : wc - 1];
                v[e] = apply_act(v[e], a.act);
            }
        }
        store8<TY>(out + (int64_t)r * wc, c, wc, v);
    });
}

// dW and db of one chunk of a group's rows: TM x TN outputs (c by j) of its matrix.
template <typename T, typename TW, int TM, int TN, bool ACT, bool CODES>
__global__ __launch_bounds__(kBlock) void k_grouped_weights(GroupedArgs a)
{
    constexpr int WR = TM / 64, WC = TN / 64;
    __shared__ __align__(16) char sA[TM * kX * 2];
    __shared__ __align__(16) char sB[TN * kX * 2];
    int64_t piece;
    int tile;
    tile_of(a.tiles_c, piece, tile);
    Span s;
    if (!find_span(a.off, a.E, a.n, a.per, piece, s)) return;
    const int wave = threadIdx.x / kWave;
    const int r0 = (wave >> 1) * (32 * WR), c0 = (wave & 1) * (32 * WC);
    const int tiles_k = a.k > 0 ? (a.k + TN - 1) / TN : 1;
    const int row0 = tile / tiles_k * TM, col0 = tile % tiles_k * TN;
    ColOperand<T, TM, ACT, false, true> A;
    A.open(static_cast<const T *>(a.dY), static_cast<const T *>(a.Y), nullptr, nullptr, row0, a.m, a.act);
    ColOperand<T, TN, false, CODES, false> B;
    B.open(static_cast<const T *>(a.X), nullptr, a.codes, a.exps, col0, a.k, 0);
    Acc<WR, WC> acc;
    acc.clear();
    A.fetch(s.lo, s.hi);
    B.fetch(s.lo, s.hi);
    for (int64_t x0 = s.lo; x0 < s.hi; x0 += kX) {
        __syncthreads();
        A.put(sA);
        B.put(sB);
        __syncthreads();
        if (x0 + kX < s.hi) {
            A.fetch(x0 + kX, s.hi);
            B.fetch(x0 + kX, s.hi);
        }
#pragma unroll
        for (int st = 0; st < kX / 16; ++st) {
            uint4 fa[WR], fb[WC];
#pragma unroll
            for (int i = 0; i < WR; ++i) fa[i] = col_fragment<TM>(sA, r0 + 32 * i, st);
#pragma unroll
            for (int j = 0; j < WC; ++j) fb[j] = col_fragment<TN>(sB, c0 + 32 * j, st);
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int j = 0; j < WC; ++j) acc.a[i][j] = mfma_32x32x16<T>(fb[j], fa[i], acc.a[i][j]);
        }
    }
    const int64_t mk = (int64_t)a.m * a.k;
    if (a.out) {
        TW *__restrict__ whole = static_cast<TW *>(a.out) + s.g * mk;
        float *__restrict__ part = a.part + (s.slot + s.local) * mk;
        for_outputs<WR, WC>(acc, [&](int r, int c, float (&v)[8]) {
            r += row0 + r0;
            c += col0 + c0;
            if (r >= a.m || c >= a.k) return;
            if (s.count == 1) store8<TW>(whole + (int64_t)r * a.k, c, a.k, v);
            else store8<float>(part + (int64_t)r * a.k, c, a.k, v);
        });
    }
    if (a.db && col0 == 0) {
        // the threads that share 8 columns add up in order
        constexpr int P = TM / 8, S = kBlock / P;
        static_assert(S * TM * (int)sizeof(float) <= TM * kX * 2, "the sums fit the dY tile");
        float *const sums = reinterpret_cast<float *>(sA);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[(threadIdx.x / P) * TM + (threadIdx.x % P) * 8 + e] = A.sum[e];
        __syncthreads();
        const int c = row0 + (int)threadIdx.x;
        if ((int)threadIdx.x < TM && c < a.m) {
            float t = 0.f;
#pragma unroll
            for (int q = 0; q < S; ++q) t += sums[q * TM + threadIdx.x];
            if (s.count == 1) a.db[(int64_t)s.g * a.m + c] = t;
            else a.part_db[(s.slot + s.local) * a.m + c] = t;
        }
    }
}

// dW and db of the groups of several chunks (sums of their slots in order) and of none
// (zeros).  Group blockIdx.y, 4 consecutive values a thread (dW, then db).
template <typename TW>
__global__ __launch_bounds__(kBlock) void k_reduce_chunks(GroupedArgs a)
{
    const int g = blockIdx.y, lane = lane_id();
    int64_t slot = 0;
    for (int e = lane; e < g; e += kWave) {
        const int64_t lo = offset_at(a.off, e, a.n), hi = offset_at(a.off, e + 1, a.n);
        if (hi - lo > a.per) slot += (hi - lo + a.per - 1) / a.per;
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) slot += __shfl_xor(slot, d);
    const int64_t lo = offset_at(a.off, g, a.n), hi = offset_at(a.off, g + 1, a.n);
    const int64_t count = hi > lo ? (hi - lo + a.per - 1) / a.per : 0;
    if (count == 1) return;
    const int64_t mk = (int64_t)a.m * a.k;
    TW *__restrict__ dW = static_cast<TW *>(a.out);
    const int64_t step = (int64_t)gridDim.x * kBlock;
    if (dW) {
        for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < mk; i += step) {
            float t = 0.f;
            for (int64_t c = 0; c < count; ++c) t += a.part[(slot + c) * mk + i];
            const float one[1] = {t};
            store_out<TW, 1>(dW, g * mk + i, one);
        }
    }
    if (a.db) {
        for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < a.m; i += step) {
            float t = 0.f;
            for (int64_t c = 0; c < count; ++c) t += a.part_db[(slot + c) * a.m + i];
            a.db[(int64_t)g * a.m + i] = t;
        }
    }
}

// ------------------------------------------------------------- the host

// Most pieces of `per` rows that n rows in E groups can have.
int64_t most_pieces(int64_t n, int32_t E, int64_t per) { return n / per + (n < E ? n : E); }

using Kernel = void (*)(GroupedArgs);

template <typename T>
Kernel pick_forward(int y_dtype, bool wide)
{
    if (y_dtype == COGDL_F32) return wide ? k_grouped_rows<T, float, 128, false, false> : k_grouped_rows<T, float, 64, false, false>;
    if (y_dtype == COGDL_BF16) return wide ? k_grouped_rows<T, bf16_t, 128, false, false> : k_grouped_rows<T, bf16_t, 64, false, false>;
    return wide ? k_grouped_rows<T, f16_t, 128, false, false> : k_grouped_rows<T, f16_t, 64, false, false>;
}

template <typename T>
Kernel pick_dx(bool wide, bool act)
{
    if (act) return wide ? k_grouped_rows<T, T, 128, true, true> : k_grouped_rows<T, T, 64, true, true>;
    return wide ? k_grouped_rows<T, T, 128, true, false> : k_grouped_rows<T, T, 64, true, false>;
}

template <typename T, typename TW, bool ACT, bool CODES>
Kernel pick_dw_tile(bool tall, bool wide)
{
    if (tall) return wide ? k_grouped_weights<T, TW, 128, 128, ACT, CODES> : k_grouped_weights<T, TW, 128, 64, ACT, CODES>;
    return wide ? k_grouped_weights<T, TW, 64, 128, ACT, CODES> : k_grouped_weights<T, TW, 64, 64, ACT, CODES>;
}

template <typename T, typename TW>
Kernel pick_dw(bool tall, bool wide, bool act, bool codes)
{
    if (act) return codes ? pick_dw_tile<T, TW, true, true>(tall, wide) : pick_dw_tile<T, TW, true, false>(tall, wide);
    return codes ? pick_dw_tile<T, TW, false, true>(tall, wide) : pick_dw_tile<T, TW, false, false>(tall, wide);
}

// Rows of a chunk of dW: about 1024 workgroups over all tiles, at least 1024 rows each (a
// partial sum is written and read once for each chunk).
struct Chunks {
    int64_t per;
    int64_t slots;     // most partial sums: a group of several chunks has under 2 n_g / per
    int tm, tn, tiles;
};

Chunks chunks_of(int64_t n, int32_t k, int32_t m)
{
    Chunks c;
    c.tm = m > 64 ? 128 : 64;
    c.tn = k > 64 ? 128 : 64;
    const int64_t tk = k > 0 ? ((int64_t)k + c.tn - 1) / c.tn : 1;
    const int64_t tiles = ((int64_t)m + c.tm - 1) / c.tm * tk;
    c.tiles = (int)(tiles < INT32_MAX ? tiles : INT32_MAX);
    int64_t per = n * tiles / 1024;
    per = (per + kX - 1) / kX * kX;
    if (per < 1024) per = 1024;
    if (per > (1 << 30)) per = 1 << 30;
    c.per = per;
    c.slots = n > per ? 2 * (n / per) : 0;
    return c;
}

cogdl_status check_grouped(int64_t n, int32_t E, int32_t k, int32_t m, const int32_t *offsets, int dtype)
{
    if (n < 0 || E < 1 || k < 0 || m < 0) return COGDL_ERR_INVALID;
    if (dtype != COGDL_BF16 && dtype != COGDL_F16) return COGDL_ERR_DTYPE;
    if (n > INT32_MAX || E > COGDL_MAX_GROUPS) return COGDL_ERR_TOO_LARGE;
    if (!offsets) return COGDL_ERR_INVALID;
    return COGDL_OK;
}

// The grid of pieces x tiles, pieces rounded up to whole rounds of the XCDs; 0: too large.
unsigned piece_tiles(int64_t pieces, int64_t tiles)
{
    const int64_t b = (pieces + 7) / 8 * 8 * tiles;
    return b <= INT32_MAX ? (unsigned)b : 0u;
}

}  // namespace
}  // namespace cogdl

using namespace cogdl;

extern "C" {

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
    const bool wide = m > 64;
    const int64_t tiles = ((int64_t)m + (wide ? 127 : 63)) / (wide ? 128 : 64);
    const unsigned grid = piece_tiles(most_pieces(n, E, kTileR), tiles);
    if (m > 0 && grid == 0) return COGDL_ERR_TOO_LARGE;
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
    a.tiles_c = (int32_t)tiles;
    const Kernel kern = dtype == COGDL_BF16 ? pick_forward<bf16_t>((int)y_dtype, wide)
                                            : pick_forward<f16_t>((int)y_dtype, wide);
    COGDL_LAUNCH("grouped_linear", kern, grid, kBlock, stream, a);
    return COGDL_OK;
}

cogdl_status cogdl_grouped_linear_backward_workspace(int64_t n, int32_t E, int32_t k, int32_t m, size_t *bytes)
{
    if (n < 0 || E < 1 || k < 0 || m < 0 || !bytes) return COGDL_ERR_INVALID;
    if (n > INT32_MAX || E > COGDL_MAX_GROUPS) return COGDL_ERR_TOO_LARGE;
    const Chunks c = chunks_of(n, k, m);
    *bytes = (size_t)c.slots * ((size_t)m * k + m) * sizeof(float);
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
    const Chunks c = chunks_of(n, k, m);
    const size_t need = (size_t)c.slots * ((size_t)m * k + m) * sizeof(float);
    const bool weights = (dW && k > 0 && m > 0) || (db && m > 0);
    if (weights && need > 0 && (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < need))
        return COGDL_ERR_INVALID;
    const bool wide = k > 64;
    const int64_t tiles_x = ((int64_t)k + (wide ? 127 : 63)) / (wide ? 128 : 64);
    const unsigned grid_x = piece_tiles(most_pieces(n, E, kTileR), tiles_x);
    // db alone needs one column of tiles; dW's own walk takes them all
    const int64_t tiles_w = dW ? c.tiles : ((int64_t)m + c.tm - 1) / c.tm;
    const unsigned grid_w = piece_tiles(most_pieces(n, E, c.per), tiles_w);
    if ((n > 0 && dX && k > 0 && grid_x == 0) || (n > 0 && weights && grid_w == 0)) return COGDL_ERR_TOO_LARGE;
    GroupedArgs a{};
    a.n = n; a.E = E; a.k = k; a.m = m;
    a.off = offsets;
    a.X = X; a.codes = codes; a.exps = exps;
    a.W = W;
    a.act = (int32_t)act;
    a.dY = dY; a.Y = Y;
    const bool bf = dtype == COGDL_BF16, with_act = act != COGDL_ACT_NONE;
    if (dX && n > 0 && k > 0) {
        a.out = dX;
        a.tiles_c = (int32_t)tiles_x;
        const Kernel kern = bf ? pick_dx<bf16_t>(wide, with_act) : pick_dx<f16_t>(wide, with_act);
        COGDL_LAUNCH("grouped_linear_dx", kern, grid_x, kBlock, stream, a);
    }
    if (!weights) return COGDL_OK;
    a.out = k > 0 ? dW : nullptr;
    a.db = db;
    a.per = (int32_t)c.per;
    a.part = static_cast<float *>(workspace);
    a.part_db = a.part + (size_t)c.slots * m * k;
    if (!dW) { a.k = 0; a.X = a.codes = nullptr; a.part_db = a.part; }
    a.tiles_c = (int32_t)tiles_w;
    if (n > 0) {
        const bool tall = c.tm == 128, wide_w = c.tn == 128, q = a.codes != nullptr;
        Kernel kern;
        if (bf)
            kern = dw_dtype == COGDL_F32 ? pick_dw<bf16_t, float>(tall, wide_w, with_act, q)
                                         : pick_dw<bf16_t, bf16_t>(tall, wide_w, with_act, q);
        else
            kern = dw_dtype == COGDL_F32 ? pick_dw<f16_t, float>(tall, wide_w, with_act, q)
                                         : pick_dw<f16_t, f16_t>(tall, wide_w, with_act, q);
        COGDL_LAUNCH("grouped_linear_dw", kern, grid_w, kBlock, stream, a);
    }
    const int64_t values = a.out ? (int64_t)m * k : m;
    int64_t bx = (values + kBlock - 1) / kBlock;
    const int64_t most = 4096 / E > 0 ? 4096 / E : 1;
    if (bx > most) bx = most;
    const dim3 grid_r((unsigned)bx, (unsigned)E);
    if (dw_dtype == COGDL_F32) COGDL_LAUNCH("grouped_linear_sum", k_reduce_chunks<float>, grid_r, kBlock, stream, a);
    else if (bf) COGDL_LAUNCH("grouped_linear_sum", k_reduce_chunks<bf16_t>, grid_r, kBlock, stream, a);
    else COGDL_LAUNCH("grouped_linear_sum", k_reduce_chunks<f16_t>, grid_r, kBlock, stream, a);
    return COGDL_OK;
}

}  // extern "C"
