// The cache in 4 bits: layout of a page and the conversions to and from bf16.
//
// A (token, kv head) row of 128 values is held as four blocks of 32 four-bit
// floats (sign, two exponent bits, one mantissa bit: magnitudes 0, 0.5, 1, 1.5,
// 2, 3, 4, 6) with one power of two per block:
//   value = code 2^(scale byte - 127).
// A block's exponent e is the smallest with max |x| <= 7 2^e, so that every
// value, the largest one included (6 to 7 units become 6), is within half a step
// of the format at its size; values round to the nearest code, ties to the even
// one.  e is kept in [-100, 100]: what is larger saturates at 6 2^100, what is
// below 2^-102 is held as zero, and no product of a probability with a scale
// leaves the range of fp32.  A block that holds an infinity or a NaN has scale
// byte 255 and codes 0 and reads as NaN (255 << 23 is +inf as a float, and
// inf * 0 is NaN; the matrix instruction takes 255 for NaN itself).
//
// Page of one kv head, 16 tokens (2176 bytes; bf16 8192):
//   K codes  [16 tokens][64 B], dim 2i in the low half of byte i.  A lane that
//     takes 16 bytes has one block of one key: the A operand of the scaled
//     16x16x128 matrix instruction, as it lies in memory.
//   V codes  [4 token quads][16 c][8 t][2 B]: token 4g + 2k + n, dim
//     32 (t/2) + 2c + t%2 in half n of byte [g][c][t][k].  A lane that takes 16
//     bytes has, for each of the eight 16-dim tiles of O^T, its row of V^T for
//     four consecutive tokens: the keys are the contraction of the second
//     product, so they must lie side by side in an operand, which the bf16 cache
//     gets by a transposing read through LDS and this one by its layout.
//   scales   [K, V][4 blocks][16 tokens] bytes, 128 in a row (a cache line).
#pragma once
#include "mw_internal.h"

namespace {
namespace kv4 {

using namespace mw;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int kCodeBytes = kPageSize * kHeadDim / 2;  // of K or V of one (page, kv head)
constexpr int kBlocks = 4;
constexpr int kScaleBytes = 2 * kBlocks * kPageSize;  // of K and V
constexpr int kExpMost = 100;
constexpr int kBias = 127;

__device__ __forceinline__ uint32_t abs2(uint32_t x) { return x & 0x7fff7fffu; }
// Larger of two pairs of bf16 magnitudes: as integers, so that NaN is the largest.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return __builtin_amdgcn_update_dpp(0, x, kCtrl, 0xf, 0xf, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;  // DPP within 16 lanes

// Scale byte of a block whose largest magnitude has the bf16 bits `most`.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    const int power = static_cast<int>(most >> 7);  // biased exponent, 255: not finite
    const int e = power - kBias - 2 + ((most & 0x7f) > 0x60 ? 1 : 0);  // mantissa above 1.75
    const int kept = min(max(e, -kExpMost), kExpMost) + kBias;
    return power == 255 ? 255 : kept;
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
// The scale that a block's values are encoded by: any for one that is not finite, whose codes are 0.
__device__ __forceinline__ float encode_scale(uint32_t byte) { return byte == 255 ? 1.f : scale_of(byte); }

// Two bf16 values to two codes in byte `kByte` of `into`.
template <int kByte>
__device__ __forceinline__ uint32_t encode2(uint32_t into, uint32_t x, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(into, __builtin_bit_cast(bf16x2_t, x), scale, kByte);
}
// The two values of byte `kByte` of `codes`, as two bf16; exact.
template <int kByte>
__device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, static_cast<bf16x2_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte)));
}

// A lane's share of a row of K: dims 8c .. 8c+7, c the lane within 16.  *byte:
// the scale byte of its block (dims 32 (c/4) ..), the same in its four lanes.
__device__ __forceinline__ uint32_t encode_k(uint4 x, uint32_t *byte) {
    uint32_t most = max2(max2(abs2(x.x), abs2(x.y)), max2(abs2(x.z), abs2(x.w)));
    most = max2(most, dpp<kXor1>(most));
    most = max2(most, dpp<kXor2>(most));
    most = max(most & 0xffff, most >> 16);
    *byte = scale_byte(most);
    const float scale = encode_scale(*byte);
    uint32_t codes = encode2<0>(0, x.x, scale);
    codes = encode2<1>(codes, x.y, scale);
    codes = encode2<2>(codes, x.z, scale);
    codes = encode2<3>(codes, x.w, scale);
    return *byte == 255 ? 0 : codes;
}

// The four codes of one dim for tokens 4g .. 4g+3 lie in 16 bits, those of its
// neighbour in the next 16; a conversion takes or gives the two dims of one token
// in a byte.  by_dim: from tokens in bytes 0 .. 3.
__device__ __forceinline__ uint32_t by_dim(uint32_t tokens) {
    const auto gather = [](uint32_t x) {
        x = (x | x >> 4) & 0x00ff00ffu;
        return (x | x >> 8) & 0xffffu;
    };
    return gather(tokens & 0x0f0f0f0fu) | gather(tokens >> 4 & 0x0f0f0f0fu) << 16;
}

// V of token k of a quad: x[b] has dims 32b + 2c, + 1.  Adds its codes (by token)
// and scale bytes, which every lane of the 16 gets, to those of the blocks.
__device__ __forceinline__ void encode_v(const uint32_t (&x)[kBlocks], int k, uint32_t (&codes)[kBlocks],
                                         uint32_t (&bytes)[kBlocks]) {
    // magnitudes of blocks 0, 1 and of blocks 2, 3 side by side, over the 16 lanes
    uint32_t most[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = abs2(x[2 * i]), hi = abs2(x[2 * i + 1]);
        uint32_t m = max2((lo & 0xffff) | hi << 16, lo >> 16 | (hi & 0xffff0000u));
        m = max2(m, dpp<kXor1>(m));
        m = max2(m, dpp<kXor2>(m));
        m = max2(m, dpp<kHalfMirror>(m));
        most[i] = max2(m, dpp<kMirror>(m));
    }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        const uint32_t byte = scale_byte(b & 1 ? most[b >> 1] >> 16 : most[b >> 1] & 0xffff);
        bytes[b] |= byte << (8 * k);
        codes[b] |= byte == 255 ? 0 : encode2<0>(0, x[b], scale_of(byte)) << (8 * k);
    }
}

// The inverse: x[k][b] from the codes of block b, kept by dim, and its tokens' scale
// bytes.  (A conversion takes the exponent of its scale and no other bit of it, so
// a byte is only shifted there.)
__device__ __forceinline__ void decode_v(const uint32_t (&codes)[kBlocks], const uint32_t (&bytes)[kBlocks],
                                         uint32_t (&x)[4][kBlocks]) {
    const auto scale = [](uint32_t bits) { return __builtin_bit_cast(float, bits); };
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        const uint32_t even = codes[b] & 0x0f0f0f0fu, odd = codes[b] >> 4 & 0x0f0f0f0fu;  // tokens 0, 2 and 1, 3
        const uint32_t t02 = even | even >> 12, t13 = odd | odd >> 12;
        x[0][b] = decode2<0>(t02, scale(bytes[b] << 23));
        x[1][b] = decode2<0>(t13, scale(bytes[b] << 15));
        x[2][b] = decode2<1>(t02, scale(bytes[b] << 7));
        x[3][b] = decode2<1>(t13, scale(bytes[b] >> 1));
    }
}
__device__ __forceinline__ uint4 decode_k(uint32_t codes, uint32_t byte) {
    const float scale = scale_of(byte);
    return make_uint4(decode2<0>(codes, scale), decode2<1>(codes, scale), decode2<2>(codes, scale), decode2<3>(codes, scale));
}

// Quantises and stores V of tokens [t0, t1) of quad g of a (page, kv head), token
// t's row at src + t stride, with 16 lanes: whole bytes, those of the quad's other
// tokens as they were.
__device__ __forceinline__ void write_v(const uint16_t *__restrict__ src, int64_t stride, uint8_t *__restrict__ codes_at,
                                        uint8_t *__restrict__ scales_at, int g, int t0, int t1, int c) {
    uint4 *dst = reinterpret_cast<uint4 *>(codes_at + g * 256 + c * 16);
    uint8_t *sc = scales_at + (kBlocks + (c & 3)) * kPageSize + 4 * g;  // lanes 0..3
    const auto load = [&](int t, uint32_t (&x)[kBlocks]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) x[k] = *reinterpret_cast<const uint32_t *>(src + t * stride + 32 * k + 2 * c);
    };
    uint32_t codes[kBlocks] = {0, 0, 0, 0}, bytes[kBlocks] = {0, 0, 0, 0};
    if (t1 - t0 == 4) {
        uint32_t x[4][kBlocks];
#pragma unroll
        for (int t = 0; t < 4; ++t) load(t, x[t]);
#pragma unroll
        for (int t = 0; t < 4; ++t) encode_v(x[t], t, codes, bytes);
        *dst = make_uint4(by_dim(codes[0]), by_dim(codes[1]), by_dim(codes[2]), by_dim(codes[3]));
        if (c < kBlocks) *reinterpret_cast<uint32_t *>(sc) = c == 0 ? bytes[0] : c == 1 ? bytes[1] : c == 2 ? bytes[2] : bytes[3];
        return;
    }
    // a single token of a decode step, or a chunk's first or last ones
    const uint4 old = *dst;
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
        uint32_t x[kBlocks];
        load(t, x);
        encode_v(x, t, codes, bytes);
    }
    const uint32_t half = (1u << 4 * t1) - (1u << 4 * t0);  // the tokens' codes of one dim
    const uint32_t mask = half | half << 16;
    *dst = make_uint4((by_dim(codes[0]) & mask) | (old.x & ~mask), (by_dim(codes[1]) & mask) | (old.y & ~mask),
                      (by_dim(codes[2]) & mask) | (old.z & ~mask), (by_dim(codes[3]) & mask) | (old.w & ~mask));
    if (c < kBlocks) {
        const uint32_t mine = c == 0 ? bytes[0] : c == 1 ? bytes[1] : c == 2 ? bytes[2] : bytes[3];
        for (int t = t0; t < t1; ++t) sc[t] = static_cast<uint8_t>(mine >> (8 * t));
    }
}

}  // namespace kv4
}  // namespace
