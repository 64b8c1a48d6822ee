// The tile engine of the grouped products (grouped_rows.hip, grouped_weights.hip):
// C[r, c] = sum_x A(r, x) B(c, x) for one tile of one group's outputs.
//
// A workgroup owns TM x TN outputs and walks x in chunks of 64.  Both operands' chunks lie in
// LDS, twice: while the matrix cores work on one, the next is on its way, so a chunk costs
// one barrier.  An operand lies in memory with x along its rows ("row" operands: X and W of
// the forward, dZ of dX) or down its rows ("col" operands: W of dX, both of dW).  A row
// operand's matrix fragments are 16-byte LDS reads, a col operand's the LDS reads that
// transpose 4 x 16 elements.  Operands whose rows lie on the 16-byte grid go from memory to
// LDS directly; the others, and those that are computed on the way (an activation's slope,
// a decoded checkpoint), pass through registers.
#pragma once

#include "checkpoint.hpp"
#include "internal.hpp"

namespace cogdl {

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

__device__ __forceinline__ uint2 load8_bytes(const void *p)
{
    const u32x2_b v = *reinterpret_cast<const u32x2_b *>(p);
    return make_uint2(v.x, v.y);
}

// A whole row of under 8 elements, zeros behind it.
template <typename T>
__device__ __forceinline__ uint4 load_short(const T *__restrict__ row, int width)
{
    uint64_t lo = 0, hi = 0;
#pragma unroll 1
    for (int e = 0; e < width; ++e) {
        const uint64_t v = (uint64_t)row[e].bits << (16 * (e & 3));
        if (e < 4) lo |= v;
        else hi |= v;
    }
    return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

__device__ __forceinline__ uint2 load_short(const int8_t *__restrict__ row, int width)
{
    uint64_t r = 0;
#pragma unroll 1
    for (int e = 0; e < width; ++e) r |= (uint64_t)(uint8_t)row[e] << (8 * e);
    return make_uint2((uint32_t)r, (uint32_t)(r >> 32));
}

// v shifted down by `gone` of its 8 elements, zeros from above (8 and more: all zeros).
__device__ __forceinline__ uint4 shift_down(uint4 v, int gone)
{
    if (gone <= 0) return v;
    if (gone >= 8) return make_uint4(0u, 0u, 0u, 0u);
    const uint64_t lo = ((uint64_t)v.y << 32) | v.x, hi = ((uint64_t)v.w << 32) | v.z;
    const int bits = 16 * gone;
    const uint64_t a = bits < 64 ? (lo >> bits) | (hi << (64 - bits)) : hi >> (bits - 64);
    const uint64_t b = bits < 64 ? hi >> bits : 0u;
    return make_uint4((uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32));
}

__device__ __forceinline__ uint2 shift_down(uint2 v, int gone)
{
    const uint64_t w = ((uint64_t)v.y << 32) | v.x;
    const uint64_t r = gone >= 8 ? 0u : gone > 0 ? w >> (8 * gone) : w;
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

__device__ __forceinline__ int row_swizzle(int r) { return (r >> 1) & 7; }            // of 16-byte pieces
template <int C>
__device__ __forceinline__ int col_swizzle(int x) { return C >= 128 ? (x & 3) << 2 : ((x >> 1) & 1) << 2; }

__device__ __forceinline__ int row_tile_at(int r, int p) { return r * (kX * 2) + ((p ^ row_swizzle(r)) << 4); }
template <int C>
__device__ __forceinline__ int col_tile_at(int x, int byte) { return x * (C * 2) + (byte ^ (col_swizzle<C>(x) << 4)); }

// 8 consecutive x (16 s + 8 (lane / 32) ...) of index idx0 + lane % 32 of a tile.
__device__ __forceinline__ uint4 row_fragment(const char *tile, int idx0, int s)
{
    const int lane = lane_id();
    return *reinterpret_cast<const uint4 *>(tile + row_tile_at(idx0 + (lane & 31), 2 * s + (lane >> 5)));
}

template <int C>
__device__ __forceinline__ uint4 col_fragment(const char *tile, int idx0, int s)
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

// 16 bytes a lane from memory to LDS, the wavefront's 1024 bytes in lane order from `to` on.
__device__ __forceinline__ void load_to_lds(const void *from, char *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// ------------------------------------------------------------- operands
// An operand's chunk on its way from memory to LDS: issue() starts the loads of the pieces
// this thread brings (FULL: the chunk's 64 x all exist), finish() writes those that wait in
// registers.  N threads.  Staged pieces at a row's end are read from its last 8 elements and
// shifted down, those behind the last row from the last one and zeroed: no load leaves the
// operand, and none waits for a branch.

enum Source { kDirect, kStaged, kSloped, kCodes };

// R indices (rows of the matrix) x 64 x along the row; indices from `have` on repeat the last
// (their outputs are not stored).  x from `width` on are zero.
template <typename T, int R, int N, int SRC>
struct RowOperand {
    static constexpr bool direct = SRC == kDirect, sloped = SRC == kSloped;
    static constexpr int Q = R * kPieces / N;
    static_assert(R * kPieces % N == 0 && N % (2 * kWave) == 0, "whole pieces a thread, whole swizzles a round");
    const T *base, *ybase;       // (uniform)
    uint32_t off[Q];             // the rows' elements from there
    int width, act;
    int gone;                    // elements of this thread's piece past the row's end
    uint4 v[direct ? 1 : Q], y[sloped ? Q : 1];

    __device__ __forceinline__ static int index(int q) { return ((int)threadIdx.x + q * N) / kPieces; }
    // the piece this thread brings: in direct loads the one whose place is the thread's
    __device__ __forceinline__ static int piece()
    {
        const int p = threadIdx.x % kPieces;
        return direct ? p ^ row_swizzle(index(0)) : p;      // (N / 8 rows a round: a multiple of 16)
    }
    __device__ __forceinline__ void open(const T *p, const T *py, int have, int w, int a)
    {
        base = p;
        ybase = py;
        width = w;
        act = a;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int r = index(q);
            off[q] = (uint32_t)(r < have ? r : have - 1) * (uint32_t)w;
        }
    }
    template <bool FULL>
    __device__ __forceinline__ void issue(int x0, char *tile)
    {
        const int at = x0 + piece() * 8;
        if constexpr (direct && FULL) {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
#pragma unroll
            for (int q = 0; q < Q; ++q) load_to_lds(base + (off[q] + at), tile + (wave * kWave + q * N) * 16);
        } else if constexpr (direct) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                uint4 w = make_uint4(0u, 0u, 0u, 0u);       // (whole pieces: rows on the grid)
                if (at < width) w = load16(base + (off[q] + at));
                *reinterpret_cast<uint4 *>(tile + ((int)threadIdx.x + q * N) * 16) = w;
            }
        } else if (width >= 8) {
            const int from = at + 8 <= width ? at : width - 8;
            gone = at - from;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                v[q] = load16(base + (off[q] + from));
                if constexpr (sloped) y[q] = load16(ybase + (off[q] + from));
            }
        } else {
            gone = at;               // (one piece holds the row)
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                v[q] = load_short(base + off[q], width);
                if constexpr (sloped) y[q] = load_short(ybase + off[q], width);
            }
        }
    }
    __device__ __forceinline__ void finish(int x0, char *tile)
    {
        if constexpr (!direct) {
            const bool tail = x0 + kX > width;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                uint4 w = v[q];
                if constexpr (sloped) {
                    float d[8], o[8];
                    unpack8<T>(w, d);
                    unpack8<T>(y[q], o);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[e] = act_grad(d[e], o[e], act);
                    w = pack8<T>(d);        // the matrix cores take 16 bits
                }
                if (tail) w = shift_down(w, gone);
                *reinterpret_cast<uint4 *>(tile + row_tile_at(index(q), piece())) = w;
            }
        }
    }
    __device__ __forceinline__ static uint4 fragment(const char *tile, int idx0, int s) { return row_fragment(tile, idx0, s); }
};

// 64 x (rows of the matrix, those from `have` on zero) by C indices along the row, from column c0
// (columns past the row's end: zeros, or in direct loads whatever, their outputs are not stored).
// SUM: keeps this thread's share of the sums over x of its 8 columns.
template <typename T, int C, int N, int SRC, bool SUM>
struct ColOperand {
    static constexpr bool direct = SRC == kDirect, sloped = SRC == kSloped, coded = SRC == kCodes;
    static constexpr int P = C / 8;
    static constexpr int Q = kX * P / N;
    static_assert(kX * P % N == 0 && N / P % 4 == 0, "whole pieces a thread, whole swizzles a round");
    const T *base, *ybase;       // (uniform)
    const int8_t *codes;
    const uint8_t *exps;
    int have, width, act, nb;
    int at, from;                // this thread's columns, and where they are read
    bool ragged;                 // the tile reaches past the row's end
    uint4 v[direct || coded ? 1 : Q], y[sloped ? Q : 1];
    uint2 c[coded ? Q : 1];
    uint32_t b[coded ? Q : 1];
    float sum[SUM ? 8 : 1];

    __device__ __forceinline__ static int index(int q) { return ((int)threadIdx.x + q * N) / P; }
    __device__ __forceinline__ static int piece()
    {
        const int p = threadIdx.x % P;
        return direct ? p ^ col_swizzle<C>(index(0)) : p;
    }
    __device__ __forceinline__ void open(const T *p, const T *py, const int8_t *pc, const uint8_t *pe, int c0, int w,
                                         int64_t rows, int a)
    {
        base = p;
        ybase = py;
        codes = pc;
        exps = pe;
        width = w;
        have = (int)rows;
        act = a;
        nb = (w + kCkptBlock - 1) / kCkptBlock;
        at = c0 + piece() * 8;
        from = at + 8 <= w ? at : w >= 8 ? w - 8 : 0;
        ragged = c0 + C > w;
#pragma unroll
        for (int e = 0; e < (SUM ? 8 : 1); ++e) sum[e] = 0.f;
    }
    template <bool FULL>
    __device__ __forceinline__ void issue(int x0, char *tile)
    {
        if constexpr (direct && FULL) {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
            const uint32_t off = (uint32_t)index(0) * (uint32_t)width + (uint32_t)from;
#pragma unroll
            for (int q = 0; q < Q; ++q)
                load_to_lds(base + (int64_t)(x0 + q * (N / P)) * width + off, tile + (wave * kWave + q * N) * 16);
        } else if constexpr (direct) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int64_t x = x0 + index(q);
                uint4 w = make_uint4(0u, 0u, 0u, 0u);
                if (x < have) w = load16(base + x * width + from);
                *reinterpret_cast<uint4 *>(tile + ((int)threadIdx.x + q * N) * 16) = w;
            }
        } else if (width >= 8) {
            const int last = have - 1 - x0;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int i = index(q) < last ? index(q) : last;
                const uint32_t off = (uint32_t)i * (uint32_t)width + (uint32_t)from;
                if constexpr (coded) {
                    c[q] = load8_bytes(codes + (int64_t)x0 * width + off);
                    b[q] = exps[(int64_t)x0 * nb + (uint32_t)(i * nb + (at < width ? at : width - 1) / kCkptBlock)];
                } else {
                    v[q] = load16(base + (int64_t)x0 * width + off);
                    if constexpr (sloped) y[q] = load16(ybase + (int64_t)x0 * width + off);
                }
            }
        } else {
            const int last = have - 1 - x0;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int64_t x = x0 + (index(q) < last ? index(q) : last);
                if constexpr (coded) {
                    c[q] = load_short(codes + x * width, width);
                    b[q] = exps[x];
                } else {
                    v[q] = load_short(base + x * width, width);
                    if constexpr (sloped) y[q] = load_short(ybase + x * width, width);
                }
            }
        }
    }
    __device__ __forceinline__ void finish(int x0, char *tile)
    {
        if constexpr (!direct) {
            const int gone = at - from;
            const bool tail = x0 + kX > have;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                uint4 w;
                if constexpr (coded) {
                    w = decode8<T>(ragged ? shift_down(c[q], gone) : c[q], b[q]);
                } else {
                    w = ragged ? shift_down(v[q], gone) : v[q];
                }
                if constexpr (sloped || SUM) {
                    float d[8];
                    unpack8<T>(w, d);
                    if constexpr (sloped) {
                        float o[8];
                        unpack8<T>(ragged ? shift_down(y[q], gone) : y[q], o);
#pragma unroll
                        for (int e = 0; e < 8; ++e) d[e] = act_grad(d[e], o[e], act);
                        w = pack8<T>(d);    // the matrix cores take 16 bits; the sums do not round
                    }
                    if constexpr (SUM) {
                        if (!tail || x0 + index(q) < have) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum[e] += d[e];
                        }
                    }
                }
                if (tail && x0 + index(q) >= have) w = make_uint4(0u, 0u, 0u, 0u);
                *reinterpret_cast<uint4 *>(tile + col_tile_at<C>(index(q), (threadIdx.x % P) * 16)) = w;
            }
        }
    }
    __device__ __forceinline__ static uint4 fragment(const char *tile, int idx0, int s) { return col_fragment<C>(tile, idx0, s); }
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

// A wavefront's own part of the LDS for its outputs: 32 rows of 32 WC fp32, rows 16 bytes apart
// in the banks.
template <int WC>
struct OutTile {
    static constexpr int kRow = 32 * WC * 4 + 16;
    static constexpr int kBytes = 32 * kRow;
};

// Calls out(row in the block, column in the block, 8 consecutive outputs) for each 8 outputs of a
// wavefront, through its part of the LDS: neighbouring lanes then hold neighbouring columns of
// a row, and a store instruction fills whole lines.  The LDS is free of other use.
template <int WR, int WC, typename Out>
__device__ __forceinline__ void for_outputs(char *lds, int wave, const Acc<WR, WC> &acc, Out out)
{
    constexpr int kLanes = 4 * WC, kRows = kWave / kLanes;      // lanes of a row, rows of a round
    const int lane = lane_id(), i = lane & 31, kq = lane >> 5;
    char *const mine = lds + wave * OutTile<WC>::kBytes;
    const int row = lane / kLanes, col = lane % kLanes * 8;
#pragma unroll
    for (int br = 0; br < WR; ++br) {
#pragma unroll
        for (int bc = 0; bc < WC; ++bc)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4 *>(mine + i * OutTile<WC>::kRow + (32 * bc + 8 * g + 4 * kq) * 4) =
                    make_float4(acc.a[br][bc][4 * g], acc.a[br][bc][4 * g + 1], acc.a[br][bc][4 * g + 2],
                                acc.a[br][bc][4 * g + 3]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int r = row; r < 32; r += kRows) {
            const float4 lo = *reinterpret_cast<const float4 *>(mine + r * OutTile<WC>::kRow + col * 4);
            const float4 hi = *reinterpret_cast<const float4 *>(mine + r * OutTile<WC>::kRow + col * 4 + 16);
            float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            out(32 * br + r, col, v);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// A step's fragments of both operands.
template <int WR, int WC>
struct Fragments {
    uint4 a[WR], b[WC];
    template <int TM, typename A, typename B>
    __device__ __forceinline__ void read(const char *tiles, int r0, int c0, int s)
    {
#pragma unroll
        for (int i = 0; i < WR; ++i) a[i] = A::fragment(tiles, r0 + 32 * i, s);
#pragma unroll
        for (int j = 0; j < WC; ++j) b[j] = B::fragment(tiles + TM * kX * 2, c0 + 32 * j, s);
    }
};

template <typename T, int WR, int WC>
__device__ __forceinline__ void step(const Fragments<WR, WC> &f, Acc<WR, WC> &acc)
{
#pragma unroll
    for (int i = 0; i < WR; ++i)
#pragma unroll
        for (int j = 0; j < WC; ++j) acc.a[i][j] = mfma_32x32x16<T>(f.b[j], f.a[i], acc.a[i][j]);
}

// Every wavefront's loads to LDS have landed (the compiler does not wait for them) and its reads are done.
__device__ __forceinline__ void chunk_done()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
}

// acc += A B over one chunk of 64 x in `now`, whose first step's fragments are in f[0]; the next
// one's loads go to `next` meanwhile (from x1 on: kFullNext its 64 x all exist, kTailNext some,
// kNoNext there is none).  The two never overlap, which the compiler has to know to keep loads in
// flight under the reads.  A step's fragments are read while the matrix cores work on the step
// before, those of the next chunk's first step behind the barrier under this one's last.
enum Next { kNoNext, kFullNext, kTailNext };

template <typename T, int TM, typename A, typename B, int WR, int WC, typename Each>
__device__ __forceinline__ void chunk(const char *__restrict__ now, char *__restrict__ next, A &a, B &b, int x1, Next more,
                                      int r0, int c0, Fragments<WR, WC> (&f)[2], Acc<WR, WC> &acc, Each each)
{
    constexpr int kB = TM * kX * 2, S = kX / 16;
    if (more == kFullNext) {
        a.template issue<true>(x1, next);
        b.template issue<true>(x1, next + kB);
    } else if (more == kTailNext) {
        a.template issue<false>(x1, next);
        b.template issue<false>(x1, next + kB);
    }
#pragma unroll
    for (int s = 0; s + 1 < S; ++s) {
        f[(s + 1) & 1].template read<TM, A, B>(now, r0, c0, s + 1);
        __builtin_amdgcn_sched_barrier(0);       // (the reads start before the step's products, not among the last)
        each(f[s & 1].a);
        step<T>(f[s & 1], acc);
    }
    if (more != kNoNext) {
        a.finish(x1, next);
        b.finish(x1, next + kB);
        chunk_done();
        f[0].template read<TM, A, B>(next, r0, c0, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
    each(f[1].a);
    step<T>(f[1], acc);
}

// acc += A B over x in [0, width): lds holds two pairs of tiles.
template <typename T, int TM, int TN, typename A, typename B, int WR, int WC, typename Each>
__device__ __forceinline__ void multiply(char *lds, A &a, B &b, int width, int r0, int c0, Acc<WR, WC> &acc, Each each)
{
    constexpr int kB = TM * kX * 2, kPair = (TM + TN) * kX * 2;
    if (width <= 0) return;
    if (width >= kX) {
        a.template issue<true>(0, lds);
        b.template issue<true>(0, lds + kB);
    } else {
        a.template issue<false>(0, lds);
        b.template issue<false>(0, lds + kB);
    }
    a.finish(0, lds);
    b.finish(0, lds + kB);
    chunk_done();
    char *now = lds, *next = lds + kPair;
    Fragments<WR, WC> f[2];
    f[0].template read<TM, A, B>(now, r0, c0, 0);
#pragma unroll 1
    for (int x1 = kX; x1 < width + kX; x1 += kX) {
        const Next more = x1 + kX <= width ? kFullNext : x1 < width ? kTailNext : kNoNext;
        chunk<T, TM>(now, next, a, b, x1, more, r0, c0, f, acc, each);
        char *const t = now;
        now = next;
        next = t;
    }
    __syncthreads();
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

// The same into element `row` on of an array of any output type.
__device__ __forceinline__ void store8(void *out, int dtype, int64_t row, int c, int width, const float (&v)[8])
{
    if (dtype == COGDL_BF16) store8(static_cast<bf16_t *>(out) + row, c, width, v);
    else if (dtype == COGDL_F16) store8(static_cast<f16_t *>(out) + row, c, width, v);
    else store8(static_cast<float *>(out) + row, c, width, v);
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
    int32_t out_dtype;
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

// Most pieces of `per` rows that n rows in E groups can have.
inline int64_t most_pieces(int64_t n, int32_t E, int64_t per) { return n / per + (n < E ? n : E); }

// The grid of pieces x tiles, pieces rounded up to whole rounds of the XCDs; 0: too large.
inline unsigned piece_tiles(int64_t pieces, int64_t tiles)
{
    const int64_t b = (pieces + 7) / 8 * 8 * tiles;
    return b <= INT32_MAX ? (unsigned)b : 0u;
}

// Rows a tile spans at most; a row operand's offsets are 32 bits (kMaxTile rows of kMaxWidth).
constexpr int kMaxTile = 256;
constexpr int kMaxWidth = 1 << 23;

// Whether rows of `width` 16-bit elements from p on lie on the 16-byte grid.
inline bool on_grid(const void *p, int width) { return width % 8 == 0 && (uintptr_t)p % 16 == 0; }

using GroupedKernel = void (*)(GroupedArgs);

// The products over rows: the forward, and dX of dY (and Y, with an activation).
cogdl_status grouped_rows_launch(const char *name, GroupedArgs a, bool dx, cogdl_dtype dtype, hipStream_t s);

// dW and db: their work plan for these sizes, and the launches.
struct Chunks {
    int64_t per;       // rows of a chunk
    int64_t slots;     // most partial sums
};
Chunks chunks_of(int64_t n, int32_t E, int32_t k, int32_t m);
cogdl_status grouped_weights_launch(GroupedArgs a, const Chunks &c, cogdl_dtype dtype, hipStream_t s);

}  // namespace cogdl
