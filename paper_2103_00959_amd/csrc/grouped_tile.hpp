// The tile engine of the grouped products (grouped_rows.hip, grouped_weights.hip):
// C[r, c] = sum_x A(r, x) B(c, x) for one tile of one group's outputs.
//
// A workgroup computes TM x TN outputs at a time and walks x in chunks of 64.  Both operands'
// chunks lie in LDS, two of them: while the matrix cores work on one, the next is on its way.
// An operand lies in memory with x along its rows ("row" operands: X and W of the forward, dZ of
// dX) or down its rows ("col" operands: W of dX, both of dW).  A row operand's matrix fragments
// are 16-byte LDS reads, a col operand's the LDS reads that transpose 4 x 16 elements.  Operands
// whose rows all lie on the 4-byte grid (even widths) go from memory to LDS directly; the others,
// and those that are computed on the way (an activation's slope, a decoded checkpoint), pass
// through registers.
//
// Workgroups are resident and take tile after tile: a tile's first chunk is loaded under the last
// products of the tile before, whose stores drain under this one's.  (A workgroup a tile, on one
// group of 32768 rows, 2048 -> 2048: 280 us, 70 a tile and compute unit, of which 17 were waits
// for the start, the first chunk and the stores.)
#pragma once

#include "checkpoint.hpp"
#include "internal.hpp"

namespace cogdl {

constexpr int kX = 64;           // x elements of a chunk

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

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

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ f32x4 mfma_16x16x32(uint4 a, uint4 b, f32x4 c)
{
    if constexpr (Fmt<T>::code == COGDL_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// ---------------------------------------------------------------- groups
// Offsets as the kernels use them: inside [0, n], so that no contents of the device array
// lead outside the operands.
__device__ __forceinline__ int64_t offset_at(const int32_t *__restrict__ off, int e, int64_t n)
{
    const int64_t o = off[e];
    return o < 0 ? 0 : (o < n ? o : n);
}

// A tile of the output: rows [lo, lo + have) of group g, column tile `tile`.  dW: `slot` is where
// its partial sums go, -1 where the rows are all of the group's.
struct Span {
    int g, tile, have, slot;
    int64_t lo;
};

// The groups 64 at a time, a group a lane; every wavefront does the same.
struct Groups {
    const int32_t *off;
    int64_t n;
    int E;
    int base;                    // the window's first group
    int lo, size;                // this lane's group: its first row and its rows

    __device__ __forceinline__ void read(int e)
    {
        lo = size = 0;
        if (e < E) {
            const int64_t o = offset_at(off, e, n), next = offset_at(off, e + 1, n);
            lo = (int)o;
            size = next > o ? (int)(next - o) : 0;
        }
    }
    __device__ __forceinline__ void window(int from)
    {
        base = from;
        read(base + lane_id());
    }
    __device__ __forceinline__ int lo_of(int l) const { return __builtin_amdgcn_readlane(lo, l); }
    __device__ __forceinline__ int size_of(int l) const { return __builtin_amdgcn_readlane(size, l); }
};

// A workgroup's tiles of the products over rows, in order.  Groups are cut into pieces of `per` rows;
// tiles are numbered by piece and column tile, and each of the 8 XCDs takes an equal run of
// them, its workgroups one after another: a group's pieces share its weights in that XCD's L2, a
// piece's tiles its rows.
struct PieceWalk {
    Groups groups;
    int per, tiles;
    int total;                   // the window's pieces
    int64_t first;               // pieces before the window
    int pieces, before;          // this lane's group: its pieces, and those up to and with it
    uint32_t j, step, end;       // the next tile, the way to the one after, the XCD's end

    __device__ __forceinline__ int pieces_of(int rows) const { return (int)(((int64_t)rows + per - 1) / per); }
    __device__ __forceinline__ void window(int from)
    {
        groups.window(from);
        pieces = pieces_of(groups.size);
        before = wave_inclusive_scan(pieces);
        total = __builtin_amdgcn_readlane(before, kWave - 1);
    }
    __device__ __forceinline__ void start(const int32_t *offsets, int E, int64_t n, int rows_a_piece, int col_tiles)
    {
        groups.off = offsets;
        groups.E = E;
        groups.n = n;
        per = rows_a_piece;
        tiles = col_tiles;
        int64_t all = 0;
        if (E > kWave) {
            int more = 0;
            for (int e = kWave + lane_id(); e < E; e += kWave) {
                groups.read(e);
                more += pieces_of(groups.size);
            }
            all = __builtin_amdgcn_readlane(wave_inclusive_scan(more), kWave - 1);
        }
        first = 0;
        window(0);
        all += total;
        const uint32_t xcd = blockIdx.x & 7;
        j = (uint32_t)(all * tiles * xcd / 8) + (blockIdx.x >> 3);
        end = (uint32_t)(all * tiles * (xcd + 1) / 8);
        step = gridDim.x >> 3;
    }
    // The next tile; false when there is none.
    __device__ __forceinline__ bool next(Span &s)
    {
        if (j >= end) return false;
        const int64_t t = j / (uint32_t)tiles;
        s.tile = (int)(j % (uint32_t)tiles);
        j = end - j > step ? j + step : end;
        while (t - first >= total) {
            first += total;
            if (groups.base + kWave >= groups.E) return false;
            window(groups.base + kWave);
        }
        const int w = (int)(t - first);
        const int l = __builtin_ctzll(__ballot(before > w));
        s.g = groups.base + l;
        const int at = (w - (__builtin_amdgcn_readlane(before, l) - __builtin_amdgcn_readlane(pieces, l))) * per;
        const int rows = groups.size_of(l) - at;
        s.lo = (int64_t)groups.lo_of(l) + at;
        s.have = rows < per ? rows : per;
        s.slot = -1;
        return true;
    }
};

// A workgroup's tiles of dW.  Rows [0, n) are cut into slices of `per`, whatever the groups: each
// takes the same time, however uneven those are (with pieces of groups instead, 64 groups of 150
// to 1400 rows, 2048 x 2048, took 587 us, the same rows in even groups 540).  Slices and output
// tiles are numbered slice by slice, each XCD takes an equal run of them; a workgroup's tile of a
// slice has its part of every group in turn.  Groups without rows are in no slice (deal_empty_groups).
// Of a slice's groups only the first and the last can reach out of it: their partial sums go to
// slots 2 i (begun before slice i) and 2 i + 1.
struct SliceWalk {
    Groups groups;
    int per, tiles, slices;
    uint32_t j, step, end;
    int slice, tile;
    int64_t from, to;            // the slice's rows
    uint64_t todo;               // groups of the window that have a part in the slice
    bool past;                   // the window holds a group behind the slice

    __device__ __forceinline__ static int slices_of(int64_t n, int per)
    {
        const int64_t s = (n + per - 1) / per;
        return s > 1 ? (int)s : 1;
    }
    __device__ __forceinline__ void window(int at)
    {
        groups.window(at);
        const int64_t lo = groups.lo, hi = lo + groups.size;
        todo = __ballot(groups.size > 0 && lo < to && hi > from);
        past = __ballot(groups.base + lane_id() >= groups.E || lo >= to) != 0;
    }
    // the groups of the slice: from the one that holds the row before it
    __device__ __forceinline__ void open_slice()
    {
        slice = (int)(j / (uint32_t)tiles);
        tile = (int)(j % (uint32_t)tiles);
        from = (int64_t)slice * per;
        to = from + per < groups.n ? from + per : groups.n;
        int64_t g = 0;
        if (groups.E > kWave && from > 0 && groups.off[0] < from) g = RowCursor::find(groups.off, groups.E, from - 1);
        window((int)(g / kWave * kWave));
    }
    __device__ __forceinline__ void start(const int32_t *offsets, int E, int64_t n, int rows_a_slice, int out_tiles)
    {
        groups.off = offsets;
        groups.E = E;
        groups.n = n;
        per = rows_a_slice;
        tiles = out_tiles;
        slices = slices_of(n, per);
        const uint32_t xcd = blockIdx.x & 7;
        const int64_t all = (int64_t)slices * tiles;
        j = (uint32_t)(all * xcd / 8) + (blockIdx.x >> 3);
        end = (uint32_t)(all * (xcd + 1) / 8);
        step = gridDim.x >> 3;
        todo = 0;
        past = true;
        if (j < end) open_slice();
    }
    __device__ __forceinline__ bool next(Span &s)
    {
        while (todo == 0) {
            if (!past && groups.base + kWave < groups.E) {
                window(groups.base + kWave);
                continue;
            }
            if (j >= end || end - j <= step) {
                j = end;
                return false;
            }
            j += step;
            open_slice();
        }
        const int l = __builtin_ctzll(todo);
        todo &= todo - 1;
        const int64_t lo = groups.lo_of(l), hi = lo + groups.size_of(l);
        s.g = groups.base + l;
        s.tile = tile;
        s.lo = lo > from ? lo : from;
        const int64_t stop = hi < to ? hi : to;
        s.have = (int)(stop - s.lo);
        s.slot = lo < from ? 2 * slice : hi > to ? 2 * slice + 1 : -1;
        return true;
    }
};

// Calls zero(g, piece) for every group g without rows and each of `pieces` pieces of its output, dealt over
// the workgroups one by one whatever the groups' places: E x pieces pairs, a lane looks at one, 64 at a time.
template <typename Zero>
__device__ __forceinline__ void deal_empty_groups(const int32_t *__restrict__ off, int E, int64_t n, int64_t pieces, Zero zero)
{
    Groups groups{off, n, E};
    const int64_t all = E * pieces, step = gridDim.x;
    for (int64_t u0 = blockIdx.x; u0 < all; u0 += kWave * step) {
        const int64_t u = u0 + lane_id() * step;
        const int g = u < all ? (int)(u / pieces) : E;
        groups.read(g);
        uint64_t todo = __ballot(g < E && groups.size == 0);
        while (todo != 0) {
            const int l = __builtin_ctzll(todo);
            todo &= todo - 1;
            const int mine = __builtin_amdgcn_readlane(g, l);
            zero(mine, u0 + l * step - mine * pieces);
        }
    }
}

// -------------------------------------------------------- pieces of memory

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

// The activation of the outputs: apply_act's, but that ReLU leaves NaN as it is (there it becomes 0), so
// that a row gone wrong stays visible, as it does under ELU and in a decoded checkpoint.
__device__ __forceinline__ float output_act(float v, int act)
{
    if (act == COGDL_ACT_RELU) return v <= 0.f ? 0.f : v;
    return apply_act(v, act);
}

// d act'(y) from the activation's output y: ReLU 0 where y <= 0 and 1 elsewhere (NaN among it: a NaN
// of d stays), ELU 1 where y > 0 and y + 1 = exp(v) elsewhere.
__device__ __forceinline__ float act_grad(float d, float y, int act)
{
    if (act == COGDL_ACT_RELU) return y <= 0.f ? 0.f : d;
    return y > 0.f ? d : d * (y + 1.f);
}

// ------------------------------------------------------------- LDS tiles
// A row tile holds R rows of 64 x (128 bytes): the 16-byte pieces of a row are permuted by the
// row, so that the 16 rows that a phase of fragment reads takes cover all banks.  A col tile holds
// 64 x of C elements: the 32-byte granules of a row are permuted by the row, so that the four rows
// a transposing read takes lie on different banks.

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

// Buffers: loads past their end give zeros.  Direct loads: 16 bytes a lane from byte `offset` of
// the buffer to LDS, the wavefront's 1024 bytes in lane order from `to` on.
typedef __amdgpu_buffer_rsrc_t Buffer;

__device__ __forceinline__ Buffer buffer_of(const void *p, int64_t bytes)
{
    const int64_t most = (int64_t)kBufferMaxBytes;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)(uint32_t)(bytes < most ? bytes : most),
                                             kBufferWord3);
}

__device__ __forceinline__ void load_to_lds(Buffer from, uint32_t offset, char *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, (int)offset, 0, 0, 0);
}

__device__ __forceinline__ uint4 load16(Buffer from, uint32_t offset)
{
    const auto w = __builtin_amdgcn_raw_buffer_load_b128(from, (int)offset, 0, 0);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ uint2 load8_bytes(Buffer from, uint32_t offset)
{
    const auto w = __builtin_amdgcn_raw_buffer_load_b64(from, (int)offset, 0, 0);
    return make_uint2(w[0], w[1]);
}

// An offset past every buffer.
constexpr uint32_t kNowhere = (uint32_t)kBufferMaxBytes;

// ------------------------------------------------------------- operands
// An operand's chunks on their way from memory to LDS: issue() starts the loads of the pieces
// this thread brings, finish() writes those that wait in registers.  N threads.  x
// past the end are zero: loads leave the buffer there; a row operand's direct piece that reaches
// past its row's end is trimmed in LDS by trim(), once it has landed; staged pieces at a row's end
// are read from its last 8 elements and shifted down, so that each lies inside or outside.

enum Source { kDirect, kStaged, kSloped, kCodes };

// R indices (rows of the matrix) by x along the row; indices from `have` on are zero, and so are
// x from `width` on.
template <typename T, int R, int N, int SRC>
struct RowOperand {
    static constexpr bool direct = SRC == kDirect, sloped = SRC == kSloped;
    static constexpr int P = kX / 8;
    static constexpr int Q = R * P / N;
    static constexpr int kBytes = R * kX * 2;
    static_assert(R * P % N == 0 && N / P % 16 == 0, "whole pieces a thread, whole swizzles a round");
    const T *base, *ybase;       // (uniform)
    Buffer rows, yrows;
    uint32_t off[Q];             // bytes to the rows (direct: to the piece)
    int have, width, act;
    uint4 v[direct ? 1 : Q], y[sloped ? Q : 1];

    __device__ __forceinline__ static int index(int q) { return ((int)threadIdx.x + q * N) / P; }
    // the piece this thread brings: in direct loads the one whose place is the thread's
    __device__ __forceinline__ static int piece()
    {
        const int p = threadIdx.x % P;
        return direct ? p ^ row_swizzle(index(0)) : p;
    }
    __device__ __forceinline__ void open(const T *p, const T *py, int rows_here, int w, int a)
    {
        base = p;
        ybase = py;
        have = rows_here;
        width = w;
        act = a;
        rows = buffer_of(p, (int64_t)have * w * 2);
        if constexpr (sloped) yrows = buffer_of(py, (int64_t)have * w * 2);
#pragma unroll
        for (int q = 0; q < Q; ++q) off[q] = (uint32_t)index(q) * (uint32_t)w * 2u + (direct ? (uint32_t)piece() * 16u : 0u);
    }
    __device__ __forceinline__ void issue(int x0, char *tile)
    {
        const int at = x0 + piece() * 8;
        if constexpr (direct) {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
#pragma unroll
            for (int q = 0; q < Q; ++q)
                load_to_lds(rows, at < width ? off[q] + (uint32_t)x0 * 2u : kNowhere, tile + (wave * kWave + q * N) * 16);
        } else if (width >= 8) {
            const uint32_t add = (uint32_t)(at + 8 <= width ? at : width - 8) * 2u;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                v[q] = load16(rows, off[q] + add);
                if constexpr (sloped) y[q] = load16(yrows, off[q] + add);
            }
        } else {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int n = index(q) < have ? width : 0;
                v[q] = load_short(base + off[q] / 2u, n);
                if constexpr (sloped) y[q] = load_short(ybase + off[q] / 2u, n);
            }
        }
    }
    __device__ __forceinline__ void finish(int x0, char *tile)
    {
        if constexpr (!direct) {
            const bool tail = x0 + kX > width;
            const int at = x0 + piece() * 8;        // (of rows under 8 wide the first piece holds all)
            const int gone = width >= 8 ? at + 8 - width : at;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                uint4 w = v[q];
                if constexpr (sloped) {
                    float d[8], o[8];
                    unpack8<T>(w, d);
                    unpack8<T>(y[q], o);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[e] = act_grad(d[e], o[e], act);
                    w = pack8<T>(d);        // the matrix cores take 16 bits: ELU's dZ is rounded (see ColOperand)
                }
                if (tail) w = shift_down(w, gone);
                *reinterpret_cast<uint4 *>(tile + row_tile_at(index(q), piece())) = w;
            }
        }
    }
    __device__ __forceinline__ void trim(int x0, char *tile)
    {
        if constexpr (direct) {
            const int keep = width - (x0 + piece() * 8);
            if (x0 + kX <= width || keep <= 0 || keep >= 8) return;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                uint32_t *const w = reinterpret_cast<uint32_t *>(tile + ((int)threadIdx.x + q * N) * 16);
                for (int d = keep / 2; d < 4; ++d) w[d] = 0u;       // (even widths)
            }
        }
    }
    __device__ __forceinline__ static uint4 fragment(const char *tile, int idx0, int s) { return row_fragment(tile, idx0, s); }
};

// x (rows of the matrix, those from `have` on zero) by C indices along the row, from column c0
// (columns past the row's end: zeros, or in direct loads whatever, their outputs are not stored).
// SUM: keeps this thread's share of the sums over x of its 8 columns, where asked to.
template <typename T, int C, int N, int SRC, bool SUM>
struct ColOperand {
    static constexpr bool direct = SRC == kDirect, sloped = SRC == kSloped, coded = SRC == kCodes;
    static constexpr int P = C / 8;
    static constexpr int Q = kX * P / N;
    static constexpr int kBytes = kX * C * 2;
    static_assert(kX * P % N == 0 && N / P % 4 == 0, "whole pieces a thread, whole swizzles a round");
    const T *base, *ybase;       // (uniform)
    const int8_t *codes;
    const uint8_t *exps;
    int have, width, act, nb;
    int at, from;                // this thread's columns, and where they are read
    bool ragged;                 // the tile reaches past the row's end
    bool sums;
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
                                         int64_t rows, int a, bool want_sums)
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
        // (direct pieces stay in place: what they hold past the row's end is no output's)
        from = direct || at + 8 <= w ? at : w >= 8 ? w - 8 : 0;
        ragged = c0 + C > w;
        sums = want_sums;
    }
    __device__ __forceinline__ void clear_sums()
    {
#pragma unroll
        for (int e = 0; e < (SUM ? 8 : 1); ++e) sum[e] = 0.f;
    }
    __device__ __forceinline__ void issue(int x0, char *tile)
    {
        const int64_t first = (int64_t)x0 * width, left = (int64_t)(have - x0) * width;
        const uint32_t off = (uint32_t)index(0) * (uint32_t)width + (uint32_t)from, step = (uint32_t)(N / P) * (uint32_t)width;
        if constexpr (direct) {
            const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
            const Buffer rows = buffer_of(base + first, left * 2);
#pragma unroll
            for (int q = 0; q < Q; ++q) load_to_lds(rows, (off + q * step) * 2u, tile + (wave * kWave + q * N) * 16);
        } else if (width >= 8) {
            if constexpr (coded) {
                const Buffer rows = buffer_of(codes + first, left), bytes = buffer_of(exps + (int64_t)x0 * nb, (int64_t)(have - x0) * nb);
                const uint32_t boff = (uint32_t)index(0) * (uint32_t)nb + (uint32_t)((at < width ? at : width - 1) / kCkptBlock);
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    c[q] = load8_bytes(rows, off + q * step);
                    b[q] = __builtin_amdgcn_raw_buffer_load_b8(bytes, (int)(boff + (uint32_t)(q * (N / P)) * (uint32_t)nb), 0, 0);
                }
            } else {
                const Buffer rows = buffer_of(base + first, left * 2);
#pragma unroll
                for (int q = 0; q < Q; ++q) v[q] = load16(rows, (off + q * step) * 2u);
                if constexpr (sloped) {
                    const Buffer yrows = buffer_of(ybase + first, left * 2);
#pragma unroll
                    for (int q = 0; q < Q; ++q) y[q] = load16(yrows, (off + q * step) * 2u);
                }
            }
        } else {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int64_t x = x0 + index(q);
                const int n = x < have ? width : 0;
                if constexpr (coded) {
                    c[q] = load_short(codes + x * width, n);
                    b[q] = n > 0 ? exps[x] : 0u;
                } else {
                    v[q] = load_short(base + x * width, n);
                    if constexpr (sloped) y[q] = load_short(ybase + x * width, n);
                }
            }
        }
    }
    __device__ __forceinline__ void finish(int x0, char *tile)
    {
        if constexpr (!direct) {
            const int gone = at - from;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                uint4 w;
                if constexpr (coded) {
                    w = decode8<T>(ragged ? shift_down(c[q], gone) : c[q], b[q]);
                } else {
                    w = ragged ? shift_down(v[q], gone) : v[q];
                }
                if constexpr (sloped || SUM) {
                    if (sloped || sums) {
                        float d[8];
                        unpack8<T>(w, d);
                        if constexpr (sloped) {
                            float o[8];
                            unpack8<T>(ragged ? shift_down(y[q], gone) : y[q], o);
#pragma unroll
                            for (int e = 0; e < 8; ++e) d[e] = act_grad(d[e], o[e], act);
                            // The matrix cores take 16 bits.  ReLU's dZ is dY or 0, ELU's is rounded here, by up to
                            // half a step of T a term, as where a layer below hands dZ on in T; a dW in fp32 has that
                            // error too (20000 rows: 8e-4 of its size in bf16, 1e-4 in fp16, against 1e-7 of the other
                            // activations).  The sums do not round.
                            w = pack8<T>(d);
                        }
                        if constexpr (SUM) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum[e] += d[e];
                        }
                    }
                }
                const int x = index(q);
                *reinterpret_cast<uint4 *>(tile + col_tile_at<C>(x, (threadIdx.x % P) * 16)) = w;
            }
        }
    }
    __device__ __forceinline__ void trim(int, char *) {}
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

// A wavefront's own part of the LDS for its outputs: 32 x 32 fp32, the 16-byte pieces of a row
// permuted by the row.
constexpr int kOutBytes = 4096;

// Calls out(column block, row in the block, column in the block, 8 consecutive outputs) for each 8 outputs of a
// wavefront, through its part of the LDS: neighbouring lanes then hold neighbouring columns of
// a row.
template <int WR, int WC, typename Out>
__device__ __forceinline__ void for_outputs(char *mine, const Acc<WR, WC> &acc, Out out)
{
    const int lane = lane_id(), i = lane & 31, kq = lane >> 5;
    const int row = lane >> 2, piece = lane & 3;
#pragma unroll
    for (int br = 0; br < WR; ++br)
#pragma unroll
        for (int bc = 0; bc < WC; ++bc) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4 *>(mine + i * 128 + (((2 * g + kq) ^ (i & 7)) << 4)) =
                    make_float4(acc.a[br][bc][4 * g], acc.a[br][bc][4 * g + 1], acc.a[br][bc][4 * g + 2],
                                acc.a[br][bc][4 * g + 3]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = row + 16 * h;
                const float4 lo = *reinterpret_cast<const float4 *>(mine + r * 128 + (((2 * piece) ^ (r & 7)) << 4));
                const float4 hi = *reinterpret_cast<const float4 *>(mine + r * 128 + (((2 * piece + 1) ^ (r & 7)) << 4));
                float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                out(bc, 32 * br + r, 32 * bc + 8 * piece, v);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
}

// A step's fragments of both operands.
template <int WR, int WC>
struct Fragments {
    uint4 a[WR], b[WC];
    template <typename A, typename B>
    __device__ __forceinline__ void read(const char *tiles, int r0, int c0, int s)
    {
#pragma unroll
        for (int i = 0; i < WR; ++i) a[i] = A::fragment(tiles, r0 + 32 * i, s);
#pragma unroll
        for (int j = 0; j < WC; ++j) b[j] = B::fragment(tiles + A::kBytes, c0 + 32 * j, s);
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

// Starts the chunk from x0 on: first the operand that passes through registers, since a wait for it is one
// for every load before it (dW of an 8-bit checkpoint, 2.4M rows, 256 -> 128: 403 us, in this order 352).
template <typename A, typename B>
__device__ __forceinline__ void issue(int x0, char *to, A &a, B &b)
{
    if constexpr (A::direct) b.issue(x0, to + A::kBytes);
    a.issue(x0, to);
    if constexpr (!A::direct) b.issue(x0, to + A::kBytes);
}

// This wavefront's chunk is in LDS: what waits in registers is written, direct loads have landed.
// (The compiler does not wait for loads to LDS on behalf of other wavefronts.)
template <typename A, typename B>
__device__ __forceinline__ void landed(int x0, char *to, A &a, B &b)
{
    a.finish(x0, to);
    b.finish(x0, to + A::kBytes);
    if constexpr (A::direct || B::direct) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
        asm volatile("" ::: "memory");
        a.trim(x0, to);
        b.trim(x0, to + A::kBytes);
    }
}

// This wavefront's LDS accesses are done, and so are every other wavefront's.
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);              // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// acc += A B over one chunk, which lies in `now` and whose first step's fragments are in f[0].
// `start` starts the loads of what goes to `next`: this tile's chunk x1, if x1 > 0, which is
// finished here, or the next tile's first.  `next` and `now` never overlap, which the compiler has
// to know to keep loads in flight under the reads.  A step's fragments are read while the matrix
// cores work on the step before, those of the next chunk's first step behind the barrier under
// this one's last.  A wavefront whose outputs all lie past the tile's end (not `busy`) leaves the
// matrix cores to the others.
template <typename T, typename A, typename B, int WR, int WC, typename Start, typename Each>
__device__ __forceinline__ void chunk(const char *__restrict__ now, char *__restrict__ next, A &a, B &b, int x1, bool busy,
                                      int r0, int c0, Fragments<WR, WC> (&f)[2], Acc<WR, WC> &acc, Start start, Each each)
{
    constexpr int S = kX / 16;
    start(next);
    if (busy) {
#pragma unroll
        for (int s = 0; s + 1 < S; ++s) {
            f[(s + 1) & 1].template read<A, B>(now, r0, c0, s + 1);
            __builtin_amdgcn_sched_barrier(0);       // (the reads start before the step's products, not among the last)
            each(f[s & 1].a);
            step<T>(f[s & 1], acc);
        }
    }
    // lgkmcnt(0), for f[1]: behind the branch the compiler would wait for the next chunk's reads with it
    __builtin_amdgcn_s_waitcnt(0xc07f);
    if (x1 > 0) {
        landed(x1, next, a, b);
        meet();
        if (busy) f[0].template read<A, B>(next, r0, c0, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (busy) {
        each(f[1].a);
        step<T>(f[1], acc);
    }
}

// The tiles of a workgroup.  open(span) makes the operands a and b those of a tile; each(span, fa)
// sees the first operand's fragments; done(span, acc) takes the products of the tile (its own
// wavefront's, no barrier needed).  lds: two pairs of chunks.  settle() runs between a tile's last
// product and the next tile's first chunk being finished.
template <typename T, typename A, typename B, int WR, int WC, typename Walk, typename Open, typename Busy, typename Each,
          typename Settle, typename Done>
__device__ __forceinline__ void run_tiles(char *lds, Walk &walk, A &a, B &b, int r0, int c0, Open open, Busy busy,
                                          Each each, Settle settle, Done done)
{
    constexpr int kPair = A::kBytes + B::kBytes;
    Span s, ahead;
    if (!walk.next(s)) return;
    char *now = lds, *next = lds + kPair;
    int width = open(s);
    issue(0, now, a, b);
    landed(0, now, a, b);
    Acc<WR, WC> acc;
    Fragments<WR, WC> f[2];
    for (;;) {
        const bool more = walk.next(ahead);
        acc.clear();
        meet();
        f[0].template read<A, B>(now, r0, c0, 0);
        const bool mine = busy(s);
        int x1 = kX, width1 = 0;
#pragma unroll 1
        do {
            const bool last = x1 >= width;
            chunk<T>(now, next, a, b, last ? 0 : x1, mine, r0, c0, f, acc,
                     [&](char *to) {
                         if (last && more) width1 = open(ahead);
                         if (!last || more) issue(last ? 0 : x1, to, a, b);
                     },
                     [&](const uint4 (&fa)[WR]) { each(s, fa); });
            char *const t = now;
            now = next;
            next = t;
            x1 += kX;
        } while (x1 < width + kX);
        settle(s);
        if (more) landed(0, now, a, b);      // (before this tile's stores: waits are in order)
        done(s, acc);
        if (!more) return;
        s = ahead;
        width = width1;
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

// The same into element `row` on of an array of any output type.
__device__ __forceinline__ void store8(void *out, int dtype, int64_t row, int c, int width, const float (&v)[8])
{
    if (dtype == COGDL_BF16) store8(static_cast<bf16_t *>(out) + row, c, width, v);
    else if (dtype == COGDL_F16) store8(static_cast<f16_t *>(out) + row, c, width, v);
    else store8(static_cast<float *>(out) + row, c, width, v);
}

__device__ __forceinline__ void store4(void *out, int dtype, int64_t row, int c, int width, const float (&v)[4])
{
    if (c + 4 <= width) {
        if (dtype == COGDL_BF16) store_vec<bf16_t, 4>(static_cast<bf16_t *>(out), row + c, v);
        else if (dtype == COGDL_F16) store_vec<f16_t, 4>(static_cast<f16_t *>(out), row + c, v);
        else store_vec<float, 4>(static_cast<float *>(out), row + c, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float one[1] = {v[e]};
        if (c + e >= width) continue;
        if (dtype == COGDL_BF16) store_out<bf16_t, 1>(static_cast<bf16_t *>(out), row + c + e, one);
        else if (dtype == COGDL_F16) store_out<f16_t, 1>(static_cast<f16_t *>(out), row + c + e, one);
        else store_out<float, 1>(static_cast<float *>(out), row + c + e, one);
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
    int32_t out_dtype;
    float *db;              // E x m, nullable
    int32_t tiles_c;        // column tiles of a row (dW: tiles of an output matrix)
    int32_t per;            // rows of a slice (dW)
    float *part;            // dW: partial sums (m x k a slot), then those of db (m a slot)
    float *part_db;
};

// Most pieces of `per` rows that n rows in E groups can have.
inline int64_t most_pieces(int64_t n, int32_t E, int64_t per) { return n / per + (n < E ? n : E); }

// The walks number tiles in 31 bits.
inline bool countable(int64_t pieces, int64_t tiles) { return pieces * tiles <= INT32_MAX; }

// Widths: the byte offsets inside a tile of 256 rows (or a chunk of 64) are 32 bits.
constexpr int kMaxWidth = 1 << 22;

// Whether direct loads take rows of `width` 16-bit elements from p on: buffer loads of 16 bytes want
// 4-byte addresses, and count the buffer's end in 4 bytes.
inline bool on_grid(const void *p, int width) { return width % 2 == 0 && (uintptr_t)p % 4 == 0; }

using GroupedKernel = void (*)(GroupedArgs);

// A kernel over `all` tiles: resident workgroups (`most` a compute unit, where given), as many on
// each XCD, no more than there are tiles.
inline cogdl_status launch_tiles(const char *name, GroupedKernel kern, const GroupedArgs &a, int64_t all, int waves, size_t lds,
                                 int most, hipStream_t stream)
{
    const int64_t resident = resident_blocks(reinterpret_cast<const void *>(kern), waves * kWave, lds, most) / 8;
    if (resident < 1) return COGDL_ERR_LAUNCH;
    const int64_t need = (all + 7) / 8;
    COGDL_LAUNCH_SHM(name, kern, dim3((unsigned)(8 * (need < resident ? need : resident))), waves * kWave, lds, stream, a);
    return COGDL_OK;
}

// The LDS of a kernel for tiles of tm x tn: two pairs of chunks, and the outputs' part.
inline size_t lds_of(int waves, int tm, int tn) { return (size_t)2 * (tm + tn) * kX * 2 + (size_t)waves * kOutBytes; }

// The products over rows: the forward, and dX of dY (and Y, with an activation).
cogdl_status grouped_rows_launch(const char *name, GroupedArgs a, bool dx, cogdl_dtype dtype, hipStream_t s);

// dW and db: the rows of a slice for these sizes, the slices' number, and the launches.
struct Slices {
    int64_t per;
    int64_t count;
    int64_t slots() const { return count > 1 ? 2 * count : 0; }     // partial sums
};
Slices slices_of(int64_t n, int32_t E, int32_t k, int32_t m);
cogdl_status grouped_weights_launch(GroupedArgs a, const Slices &c, cogdl_dtype dtype, hipStream_t s);

}  // namespace cogdl
