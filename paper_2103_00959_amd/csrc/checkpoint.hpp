// The 8-bit checkpoint format, shared by the kernels that write, read and multiply it.
//
// A block of kCkptBlock consecutive features of a row (the last block of a row may be
// shorter) has one exponent byte b and an int8 code per feature; feature x is kept as
// q 2^(b - 127).  With M the block's largest magnitude, b is the biased exponent of M
// less 6, one more where M / 2^(b - 127) would round to 128, so |q| <= 127 and
// |x - q s| <= s / 2 with s <= M / 63.75.  Powers of two keep both ways exact: x / s is
// exact, so codes depend on nothing but x and M, and q s has 7 significant bits and is a
// bf16 (from fp16 activations, an fp16) as it stands: a product reads a checkpoint at no
// rounding of its own.  A block that holds a value that is not finite gets b = 255 and
// codes 0, which decodes to NaN.
#pragma once

#include "common.hpp"

namespace cogdl {

constexpr int kCkptBlock = COGDL_CKPT_BLOCK;
constexpr int kCkptBad = 255;

// Bounds of the exponent byte: steps of the activations' own format at least (fp16
// subnormals are multiples of 2^-24) and decoded values below its overflow at most
// (127 2^121 in bf16 and fp32, 127 2^9 in fp16: larger blocks saturate at 127).
template <typename T> struct CkptRange { static constexpr int lo = 1, hi = 248; };
template <> struct CkptRange<f16_t> { static constexpr int lo = 103, hi = 136; };

// The exponent byte of a block whose largest |x| has these fp32 bits.  Adding 2^16 carries
// into the exponent exactly where M's mantissa is 1.9921875 or more (127.5 / 64).
template <typename T>
__device__ __forceinline__ int ckpt_exponent(uint32_t max_bits)
{
    if (max_bits >= 0x7f800000u) return kCkptBad;
    const int b = (int)((max_bits + 0x10000u) >> 23) - 6;
    return b < CkptRange<T>::lo ? CkptRange<T>::lo : (b > CkptRange<T>::hi ? CkptRange<T>::hi : b);
}

// A block's way from values to codes: 2^(127 - b), and the value of code 127 (a bad block: zeros).
struct CkptScale {
    float inverse, limit;
};

__device__ __forceinline__ CkptScale ckpt_encode_scale(int b)
{
    if (b == kCkptBad) return {0.f, 0.f};
    return {__uint_as_float((uint32_t)(254 - b) << 23), 127.f * __uint_as_float((uint32_t)b << 23)};
}

// 4 codes of 4 features, the first in the low byte.  Adding 1.5 2^23 rounds to a whole number
// (to nearest even), which is then the low bits of the sum; the limit comes first, as a median,
// which also makes zeros of the infinities and NaN of a bad block.
__device__ __forceinline__ uint32_t ckpt_encode4(float a, float b, float c, float d, CkptScale s)
{
    const auto one = [&](float x) {
        return __float_as_uint(fmaf(__builtin_amdgcn_fmed3f(x, -s.limit, s.limit), s.inverse, 12582912.f));
    };
    const uint32_t lo = __builtin_amdgcn_perm(one(b), one(a), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(one(d), one(c), 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// The first `have` (1 to 8) of 8 bytes.
typedef uint32_t u32x2_b __attribute__((ext_vector_type(2), aligned(1)));

__device__ __forceinline__ void store_bytes(int8_t *__restrict__ p, int have, uint32_t lo, uint32_t hi)
{
    if (have >= 8) {
        *reinterpret_cast<u32x2_b *>(p) = u32x2_b{lo, hi};
        return;
    }
    typedef uint32_t u32_b __attribute__((aligned(1)));
    typedef uint16_t u16_b __attribute__((aligned(1)));
    if (have & 4) {
        *reinterpret_cast<u32_b *>(p) = lo;
        p += 4;
        lo = hi;
    }
    if (have & 2) {
        *reinterpret_cast<u16_b *>(p) = (uint16_t)lo;
        p += 2;
        lo >>= 16;
    }
    if (have & 1) *p = (int8_t)lo;
}

// The 4 values of 4 codes (exact: 7 bits times a power of two).
__device__ __forceinline__ void ckpt_decode4(uint32_t codes, float s, float (&v)[4])
{
    v[0] = (float)(int8_t)codes * s;
    v[1] = (float)(int8_t)(codes >> 8) * s;
    v[2] = (float)(int8_t)(codes >> 16) * s;
    v[3] = (float)((int32_t)codes >> 24) * s;
}

// 2^(b - 127), infinite for the bad block, whose codes of 0 then give NaN.
__device__ __forceinline__ float ckpt_scale(uint32_t b) { return __uint_as_float(b << 23); }

}  // namespace cogdl
