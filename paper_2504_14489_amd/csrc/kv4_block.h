// What the attention kernels over the cache in 4 bits share.
#pragma once
#include "decode_block.h"
#include "kv4_format.h"

namespace {
namespace kv4 {

using dk::f32x4;
using dk::wave_max;
using dk::wave_sum;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

// Two bf16 values into half kHalf of hi and lo.
template <int kHalf>
__device__ __forceinline__ void split2(uint32_t two, float unit, i16x2 &hi, i16x2 &lo) {
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2_t, two), unit, kHalf);
    const auto near = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(__builtin_bit_cast(int, hi), unit, kHalf);
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, __builtin_bit_cast(float, two << 16) - near[0],
                                                  __builtin_bit_cast(float, two & 0xffff0000u) - near[1], unit, kHalf);
}

// A query row as two e4m3 operands of the scaled matrix instruction, hi + lo: with
// q 2^-e, e such that the row's largest is in [128, 256), hi is its nearest and lo
// the nearest of the rest.  hi keeps four bits of the eight that bf16 has and the
// rest has four, so the sum is exact down to 2^-9 of the row's largest; below, the
// rest is rounded to its smallest step, 2^-9, and the sum is off by at most 2^-10, 2^-17
// of a row's largest of 128.
// x[4 i + j], j < 4: the lane's dims of operand i, the first 16 bytes of the
// operand and the last; the row's other dims are in the lanes 32 apart and, with
// kQuarters, those 16 apart.  Returns the factor of its scores.
template <bool kQuarters, int N>
__device__ __forceinline__ float split_q(const uint4 (&x)[4 * N], i32x8 (&hi)[N], i32x8 (&lo)[N]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) most = max2(max2(max2(most, abs2(x[i].x)), max2(abs2(x[i].y), abs2(x[i].z))), abs2(x[i].w));
    most = max(most & 0xffff, most >> 16);
    if constexpr (kQuarters) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 16)));
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 32)));
    const int power = static_cast<int>(most >> 7);
    const int e = max(power - 127 - 7, -100);  // rows below 2^-93 keep fewer bits
    const float unit = __builtin_bit_cast(float, static_cast<uint32_t>(127 + e) << 23);
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            i16x2 h{0, 0}, l{0, 0};
            split2<0>(w[2 * j], unit, h, l);
            split2<1>(w[2 * j + 1], unit, h, l);
            hi[i / 4][2 * (i % 4) + j] = __builtin_bit_cast(int, h);
            lo[i / 4][2 * (i % 4) + j] = __builtin_bit_cast(int, l);
        }
    }
    // a row that is not finite: NaN scores
    return power == 255 ? NAN : unit;
}

// Weighted sum of the fragments or pieces of one head in a wave: (m, l) of up to
// 64 of them one per lane, which gives every weight 2^(m - M) and the denominator
// within the wave, then two outputs per lane.  Those without keys have l = 0 and
// contribute nothing.  load_o(j): the lane's two values of the j-th, j < n.  The
// first 8 kBatches of them are requested before (m, l) is looked at: one latency
// instead of two or three.
struct HeadSum {
    float M = -INFINITY, L = 0.f;
    float2 acc = make_float2(0.f, 0.f);
    template <int kBatches = 1, class LoadO>
    __device__ __forceinline__ void add(float2 ml, int n, int lane, const LoadO &load_o) {
        float2 o[8 * kBatches];
        const auto load = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kBatches; ++i)
                if (i == 0 || j0 + 8 * i < n)
#pragma unroll
                    for (int k = 8 * i; k < 8 * i + 8; ++k) o[k] = load_o(min(j0 + k, n - 1));
        };
#pragma unroll
        for (int k = 8; k < 8 * kBatches; ++k) o[k] = make_float2(0.f, 0.f);
        load(0);
        const bool in = lane < n && ml.y != 0.f;
        const float top = fmaxf(M, wave_max(in ? ml.x : -INFINITY));
        const float old = L == 0.f ? 0.f : __builtin_amdgcn_exp2f(M - top);
        const float w = in ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
        M = top;
        L = L * old + wave_sum(in ? w * ml.y : 0.f);
        acc.x *= old;
        acc.y *= old;
        for (int j0 = 0;;) {
#pragma unroll
            for (int k = 0; k < 8 * kBatches; ++k) {
                if (k >= 8 && k % 8 == 0 && j0 + k >= n) break;
                // lanes from n on have weight 0, and j0 + k < 64
                const float wk = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), j0 + k));
                acc.x += wk * o[k].x;
                acc.y += wk * o[k].y;
            }
            j0 += 8 * kBatches;
            if (j0 >= n) break;
            load(j0);
        }
    }
};

// The larger of m and four scores; a NaN wins, which spares the instructions that
// would quiet it (its column comes out as NaN).
__device__ __forceinline__ float max4(float m, f32x4 s) {
    return __builtin_elementwise_maximum(
        __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, s[0]), s[1]),
        __builtin_elementwise_maximum(s[2], s[3]));
}
// x of the four lanes of a column (those 16 and 32 apart) combined by f, in each.
template <class F>
__device__ __forceinline__ float across(float x, const F &f) {
    const auto pair = [&](auto r) {
        const uint32_t lo = r[0], hi = r[1];  // (a bit cast of an element itself takes the first one)
        return f(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
    };
    const uint32_t a = __builtin_bit_cast(uint32_t, x);
    const uint32_t b = __builtin_bit_cast(uint32_t, pair(__builtin_amdgcn_permlane16_swap(a, a, false, false)));
    return pair(__builtin_amdgcn_permlane32_swap(b, b, false, false));
}

}  // namespace kv4
}  // namespace
