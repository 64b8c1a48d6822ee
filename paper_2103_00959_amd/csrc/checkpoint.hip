// Activations into 8-bit checkpoints and back (the format: checkpoint.hpp).
//
// A lane holds 8 consecutive features, a block of 32 four adjacent lanes: the block's
// maximum is two DPP steps, and a wavefront reads 64 x 16 (fp32: 32) bytes and writes 64 x 8
// of codes.  Both ways are bound by memory: 2.4M x 256 bf16 351 us there and 361 back (1.86 GB each, 5.3
// and 5.2 TB/s; a large copy 4.9), 169343 x 300 fp32 55 and 49 us (256 MB, 4.6 and 5.2 TB/s).  Small calls
// by their launch: 2708 x 1433 bf16 5 us each.
#include "checkpoint.hpp"
#include "internal.hpp"

namespace cogdl {
namespace {

constexpr int kBlock = 256;

// The 8 values from element i of p on, `have` (1 to 8) of them inside the row of F; zeros past it.
// A row's end is read with its last 8 elements, which are then moved down.
template <typename T>
__device__ __forceinline__ void load_features(const T *__restrict__ p, int64_t i, int have, int F, float (&x)[8])
{
    if (F < 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float one[1] = {0.f};
            if (e < have) load_vec<T, 1>(p, i + e, one);
            x[e] = one[0];
        }
        return;
    }
    const int gone = 8 - have;
    if constexpr (sizeof(T) == 4) {
        float a[4], b[4];
        load_vec<T, 4>(p, i - gone, a);
        load_vec<T, 4>(p, i - gone + 4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
    } else {
        load_vec<T, 8>(p, i - gone, x);
    }
    if (gone == 0) return;
#pragma unroll
    for (int bit = 0; bit < 3; ++bit)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float from = e + (1 << bit) < 8 ? x[e + (1 << bit)] : 0.f;
            x[e] = (gone >> bit) & 1 ? from : x[e];
        }
}

// Pieces of 8 features: nb blocks of 4 pieces a row, the pieces past the row's end empty.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_act_checkpoint(int64_t n, int F, int nb, const T *__restrict__ A,
                                                           int8_t *__restrict__ codes,
                                                           uint8_t *__restrict__ exps)
{
    const int64_t pieces = n * nb * 4;
    const int64_t step = (int64_t)gridDim.x * kBlock;
    for (int64_t t = (int64_t)blockIdx.x * kBlock + threadIdx.x; t < pieces; t += step) {
        const int64_t blk = t >> 2;                  // exponent byte of this piece
        const int64_t row = blk <= UINT32_MAX ? (int64_t)((uint32_t)blk / (uint32_t)nb) : blk / nb;
        const int f = (int)(blk - row * nb) * kCkptBlock + (int)(t & 3) * 8;
        const int left = F - f;
        const int have = left < 0 ? 0 : (left > 8 ? 8 : left);
        const int64_t at = row * F + f;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (have > 0) load_features<T>(A, at, have, F, x);
        uint32_t top = 0;                            // magnitudes order as their bits, NaN above infinity
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = __float_as_uint(x[e]) & 0x7fffffffu;
            top = u > top ? u : top;
        }
        top = group_reduce(top, 4, [](uint32_t u, uint32_t v) { return u > v ? u : v; });
        const int b = ckpt_exponent<T>(top);
        if ((t & 3) == 0) exps[blk] = (uint8_t)b;
        const CkptScale sc = ckpt_encode_scale(b);
        const uint32_t lo = ckpt_encode4(x[0], x[1], x[2], x[3], sc);
        const uint32_t hi = ckpt_encode4(x[4], x[5], x[6], x[7], sc);
        if (have > 0) store_bytes(codes + at, have, lo, hi);
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_act_restore(int64_t n, int F, int nb, const int8_t *__restrict__ codes,
                                                        const uint8_t *__restrict__ exps, T *__restrict__ out)
{
    const int64_t pieces = n * nb * 4;
    const int64_t step = (int64_t)gridDim.x * kBlock;
    for (int64_t t = (int64_t)blockIdx.x * kBlock + threadIdx.x; t < pieces; t += step) {
        const int64_t blk = t >> 2;
        const int64_t row = blk <= UINT32_MAX ? (int64_t)((uint32_t)blk / (uint32_t)nb) : blk / nb;
        const int f = (int)(blk - row * nb) * kCkptBlock + (int)(t & 3) * 8;
        const int left = F - f;
        if (left <= 0) continue;
        const int64_t at = row * F + f;
        const float s = ckpt_scale(exps[blk]);
        float v[8];
        if (left >= 8) {
            const u32x2_b w = *reinterpret_cast<const u32x2_b *>(codes + at);
            float a[4], b[4];
            ckpt_decode4(w.x, s, a);
            ckpt_decode4(w.y, s, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
            store_vec<T, 8>(out, at, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e < left) {
                    const float one[1] = {(float)codes[at + e] * s};
                    store_out<T, 1>(out, at + e, one);
                }
            }
        }
    }
}

// A grid past the resident size (one piece a lane up to 2^24 of them).
unsigned piece_grid(int64_t pieces)
{
    int64_t b = (pieces + kBlock - 1) / kBlock;
    if (b > 65536) b = 65536;
    return (unsigned)b;
}

}  // namespace
}  // namespace cogdl

using namespace cogdl;

extern "C" {

cogdl_status cogdl_act_checkpoint(int64_t n, int32_t F, const void *A, cogdl_dtype a_dtype, int8_t *codes,
                                  uint8_t *exps, hipStream_t stream)
{
    if (n < 0 || F < 1) return COGDL_ERR_INVALID;
    if (!dtype_ok(a_dtype)) return COGDL_ERR_DTYPE;
    if (n > 0 && (!A || !codes || !exps)) return COGDL_ERR_INVALID;
    if (n == 0) return COGDL_OK;
    const int nb = (int)(((int64_t)F + kCkptBlock - 1) / kCkptBlock);
    const unsigned grid = piece_grid(n * nb * 4);
    if (a_dtype == COGDL_F32)
        COGDL_LAUNCH("act_checkpoint", k_act_checkpoint<float>, grid, kBlock, stream, n, F, nb,
                     static_cast<const float *>(A), codes, exps);
    else if (a_dtype == COGDL_BF16)
        COGDL_LAUNCH("act_checkpoint", k_act_checkpoint<bf16_t>, grid, kBlock, stream, n, F, nb,
                     static_cast<const bf16_t *>(A), codes, exps);
    else
        COGDL_LAUNCH("act_checkpoint", k_act_checkpoint<f16_t>, grid, kBlock, stream, n, F, nb,
                     static_cast<const f16_t *>(A), codes, exps);
    return COGDL_OK;
}

cogdl_status cogdl_act_restore(int64_t n, int32_t F, const int8_t *codes, const uint8_t *exps, void *out,
                               cogdl_dtype out_dtype, hipStream_t stream)
{
    if (n < 0 || F < 1) return COGDL_ERR_INVALID;
    if (!dtype_ok(out_dtype)) return COGDL_ERR_DTYPE;
    if (n > 0 && (!out || !codes || !exps)) return COGDL_ERR_INVALID;
    if (n == 0) return COGDL_OK;
    const int nb = (int)(((int64_t)F + kCkptBlock - 1) / kCkptBlock);
    const unsigned grid = piece_grid(n * nb * 4);
    if (out_dtype == COGDL_F32)
        COGDL_LAUNCH("act_restore", k_act_restore<float>, grid, kBlock, stream, n, F, nb, codes, exps,
                     static_cast<float *>(out));
    else if (out_dtype == COGDL_BF16)
        COGDL_LAUNCH("act_restore", k_act_restore<bf16_t>, grid, kBlock, stream, n, F, nb, codes, exps,
                     static_cast<bf16_t *>(out));
    else
        COGDL_LAUNCH("act_restore", k_act_restore<f16_t>, grid, kBlock, stream, n, F, nb, codes, exps,
                     static_cast<f16_t *>(out));
    return COGDL_OK;
}

}  // extern "C"
