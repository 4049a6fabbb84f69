// Queries and keys on their way from the projection: RMS norm of each head,
// position rotation and the append to the cache, in one pass.
//
// With x a head's 128 values, w its weights and t the token's position:
//   y = x w / sqrt(mean(x^2) + eps)
//   (a, b) -> (a cos(t f_i) - b sin(t f_i), b cos(t f_i) + a sin(t f_i))
// over the pairs i < rot_dim / 2 of y: (y_i, y_{i + rot_dim/2}), or neighbours
// (y_2i, y_2i+1).  Dims past rot_dim stay.  Sums, norm and rotation are fp32, one
// rounding to bf16 at the end; the angle t f_i is a product in 64 bits, brought
// to one turn before fp32 sees it (at t = 10^5, f = 1 the fp32 product is off by
// 2^-8 of a radian).
//
// Bound by memory: every row is read and written once, 256 bytes a head.
#include "kv4_format.h"

using namespace mw;

namespace {

using namespace kv4;

struct NormRopeArgs {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;  // elements from a token's row to the next
    const uint16_t *q_weight, *k_weight;   // NULL: no norm
    const double *inv_freq;
    float eps;
    int rot_dim, neighbours, hq;
    uint16_t *q_out;
};
struct Cache {
    uint16_t *k, *v;               // bf16 pages, or
    uint8_t *k4, *v4, *scales;     // those in 4 bits
    const int32_t *bt;
    int bt_stride, num_pages, hkv;
};

__device__ __forceinline__ float lo(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float hi(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    bf16x2_t v;
    v[0] = static_cast<__bf16>(a);
    v[1] = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint32_t, v);
}
template <int kCtrl>
__device__ __forceinline__ float add_dpp(float x) {
    return x + __builtin_bit_cast(float, dpp<kCtrl>(__builtin_bit_cast(uint32_t, x)));
}

// A lane's dims 8c .. 8c+7 of a head row; cs: the token's (cos, sin) by pair.
__device__ __forceinline__ uint4 norm_rope_row(uint4 x, bool norm, uint4 w, float eps, int rot_dim, bool neighbours,
                                               const float2 *cs, int c) {
    float y[8] = {lo(x.x), hi(x.x), lo(x.y), hi(x.y), lo(x.z), hi(x.z), lo(x.w), hi(x.w)};
    if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += y[j] * y[j];
        sum = add_dpp<kXor1>(sum);
        sum = add_dpp<kXor2>(sum);
        sum = add_dpp<kHalfMirror>(sum);
        sum = add_dpp<kMirror>(sum);
        const float r = rsqrtf(sum * (1.f / kHeadDim) + eps);
        const float wf[8] = {lo(w.x), hi(w.x), lo(w.y), hi(w.y), lo(w.z), hi(w.z), lo(w.w), hi(w.w)};
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = y[j] * r * wf[j];
    }
    if (neighbours) {
        if (8 * c < rot_dim) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 t = cs[4 * c + j];
                const float a = y[2 * j], b = y[2 * j + 1];
                y[2 * j] = a * t.x - b * t.y;
                y[2 * j + 1] = b * t.x + a * t.y;
            }
        }
    } else if (rot_dim > 0) {
        const int half = rot_dim / 16;  // lanes of the first half
        const bool first = c < half;
        const int partner = (threadIdx.x & 48) | (first ? c + half : c < 2 * half ? c - half : c);
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = __shfl(y[j], partner);
        if (c < 2 * half) {
            const float2 *at = cs + 8 * (first ? c : c - half);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = y[j] * at[j].x + (first ? -p[j] : p[j]) * at[j].y;
        }
    }
    return make_uint4(pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7]));
}

// One work-group: the (up to four) new tokens of one quad of page slots; grid.z
// slices share its heads.  The quad's angles are computed once, one a thread,
// and lie in LDS; then 16 lanes take a head row at a time.  Quads, because V in 4
// bits is stored by four tokens (kv4_format.h).
template <bool kFourBit>
__global__ void __launch_bounds__(256)
k_norm_rope(NormRopeArgs a, Cache kv, const int32_t *__restrict__ indptr, const int32_t *__restrict__ start_pos) {
    __shared__ float2 s_cs[4][kHeadDim / 2];
    const int b = blockIdx.y, c = threadIdx.x & 15;
    const int row0 = indptr[b], n = indptr[b + 1] - row0, pos0 = start_pos[b];
    if (n <= 0 || pos0 < 0) return;
    const int32_t *btrow = kv.bt + static_cast<size_t>(b) * kv.bt_stride;
    const int quad0 = pos0 / 4, quads = (pos0 + n + 3) / 4 - quad0;
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 wq = a.q_weight ? *reinterpret_cast<const uint4 *>(a.q_weight + 8 * c) : none;
    const uint4 wk = a.k_weight ? *reinterpret_cast<const uint4 *>(a.k_weight + 8 * c) : none;
    const int rows = a.hq + kv.hkv;  // rotated rows of a token
    for (int i = blockIdx.x; i < quads; i += gridDim.x) {
        const int first = (quad0 + i) * 4 - pos0;  // row of the quad's first slot
        const int t0 = max(0, -first), m = min(4, n - first) - t0;
        const int pos = pos0 + first, slot = pos % kPageSize;
        const int page = pos / kPageSize < kv.bt_stride ? btrow[pos / kPageSize] : -1;
        const bool held = page >= 0 && page < kv.num_pages;  // elsewhere only the queries are written
        __syncthreads();  // the last quad's angles are read
        {
            const int t = threadIdx.x >> 6, f = threadIdx.x & 63;
            if (2 * f < a.rot_dim) {
                const double turns = static_cast<double>(pos + t) * a.inv_freq[f] * 0.15915494309189533577;
                float sn, cs;
                sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sn, &cs);
                s_cs[t][f] = make_float2(cs, sn);
            }
        }
        __syncthreads();
        const int v_tasks = kFourBit ? kv.hkv : m * kv.hkv;
        const int tasks = m * rows + v_tasks;
        const int step = gridDim.z * 16;
        for (int task = blockIdx.z * 16 + (threadIdx.x >> 4); task < tasks; task += step) {
            if (task < m * rows) {
                const int h = task / m, t = t0 + task - h * m;
                const int64_t row = static_cast<int64_t>(row0) + first + t;
                if (h < a.hq) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(a.q + row * a.q_stride + h * kHeadDim + 8 * c);
                    const uint4 y = norm_rope_row(x, a.q_weight != nullptr, wq, a.eps, a.rot_dim, a.neighbours != 0, s_cs[t], c);
                    *reinterpret_cast<uint4 *>(a.q_out + (row * a.hq + h) * kHeadDim + 8 * c) = y;
                } else {
                    const int kh = h - a.hq;
                    const uint4 x = *reinterpret_cast<const uint4 *>(a.k + row * a.k_stride + kh * kHeadDim + 8 * c);
                    const uint4 y = norm_rope_row(x, a.k_weight != nullptr, wk, a.eps, a.rot_dim, a.neighbours != 0, s_cs[t], c);
                    if (!held) continue;
                    const size_t at = static_cast<size_t>(page) * kv.hkv + kh;
                    if constexpr (kFourBit) {
                        uint32_t byte;
                        const uint32_t codes = encode_k(y, &byte);
                        *reinterpret_cast<uint32_t *>(kv.k4 + at * kCodeBytes + (slot + t) * (kHeadDim / 2) + 4 * c) = codes;
                        if ((c & 3) == 0)
                            kv.scales[at * kScaleBytes + (c >> 2) * kPageSize + slot + t] = static_cast<uint8_t>(byte);
                    } else {
                        *reinterpret_cast<uint4 *>(kv.k + (at * kPageSize + slot + t) * kHeadDim + 8 * c) = y;
                    }
                }
            } else if (held) {
                const int v_task = task - m * rows;
                if constexpr (kFourBit) {
                    uint32_t vr[4][kBlocks];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const bool in = t >= t0 && t < t0 + m;
                        const int64_t row = static_cast<int64_t>(row0) + first + (in ? t : t0);
                        const uint16_t *src = a.v + row * a.v_stride + v_task * kHeadDim + 2 * c;
#pragma unroll
                        for (int k = 0; k < kBlocks; ++k)
                            vr[t][k] = in ? *reinterpret_cast<const uint32_t *>(src + 32 * k) : 0;
                    }
                    uint32_t codes[kBlocks], bytes[kBlocks];
                    encode_v(vr, codes, bytes);
                    const size_t at = static_cast<size_t>(page) * kv.hkv + v_task;
                    store_v(kv.v4 + at * kCodeBytes, kv.scales + at * kScaleBytes, codes, bytes, slot / 4, t0, t0 + m, c);
                } else {
                    const int vh = v_task / m, t = t0 + v_task - vh * m;
                    const int64_t row = static_cast<int64_t>(row0) + first + t;
                    *reinterpret_cast<uint4 *>(kv.v + ((static_cast<size_t>(page) * kv.hkv + vh) * kPageSize + slot + t) * kHeadDim + 8 * c) =
                        *reinterpret_cast<const uint4 *>(a.v + row * a.v_stride + vh * kHeadDim + 8 * c);
                }
            }
        }
    }
}

}  // namespace

extern "C" mw_status mw_qk_norm_rope_write(const mw_kv_pool *pool, const mw_norm_rope *rope, int32_t batch,
                                           const int32_t *h_new_lens, const int32_t *h_start_pos,
                                           const int32_t *d_qo_indptr, const int32_t *d_start_pos,
                                           const int32_t *d_block_table, int32_t bt_stride, const void *d_q,
                                           int64_t q_stride, const void *d_k, int64_t k_stride, const void *d_v,
                                           int64_t v_stride, void *d_q_out, mw_stream stream, mw_timing *timing) {
    const char *who = "mw_qk_norm_rope_write";
    if (!rope) return fail(MW_ERR_INVALID_ARG, "%s: rope is NULL", who);
    int64_t max_n = 0, total = 0;
    mw_status st = check_rows(pool, batch, h_new_lens, h_start_pos, d_qo_indptr, d_start_pos, d_block_table, bt_stride,
                              &max_n, &total, who);
    if (st != MW_OK) return st;
    const int64_t hq = rope->num_q_heads, hkv = pool->desc.num_kv_heads;
    if (hq < 0) return fail(MW_ERR_INVALID_ARG, "%s: num_q_heads must not be negative", who);
    if (rope->rot_dim < 0 || rope->rot_dim > kHeadDim || rope->rot_dim % 16)
        return fail(MW_ERR_UNSUPPORTED, "%s: rot_dim must be a multiple of 16 in [0, 128]", who);
    if (!(rope->eps >= 0.f) || !(rope->eps < INFINITY))
        return fail(MW_ERR_INVALID_ARG, "%s: eps must be finite and not negative", who);
    if ((rope->d_q_weight && !aligned16(rope->d_q_weight)) || (rope->d_k_weight && !aligned16(rope->d_k_weight)))
        return fail(MW_ERR_INVALID_ARG, "%s: norm weights must be 16-byte aligned", who);
    if (rope->rot_dim > 0 && (!rope->d_inv_freq || (reinterpret_cast<uintptr_t>(rope->d_inv_freq) & 7)))
        return fail(MW_ERR_INVALID_ARG, "%s: d_inv_freq must be 8-byte aligned doubles", who);
    const auto bad = [](const void *p, int64_t stride, int64_t heads) {
        return !p || !aligned16(p) || stride < heads * kHeadDim || stride % 8;
    };
    if (total > 0 && (bad(d_k, k_stride, hkv) || bad(d_v, v_stride, hkv) || (hq > 0 && bad(d_q, q_stride, hq)) ||
                      (hq > 0 && (!d_q_out || !aligned16(d_q_out)))))
        return fail(MW_ERR_INVALID_ARG,
                    "%s: rows must be 16-byte aligned, strides multiples of 8 elements and no less than a token's heads", who);
    if (4 * (hq + 2 * hkv) > INT32_MAX / 2) return fail(MW_ERR_UNSUPPORTED, "%s: too many heads", who);
    hipStream_t s = static_cast<hipStream_t>(stream);
    st = timing_begin(timing, s);
    if (st != MW_OK) return st;
    if (total > 0) {
        // a quad of slots more than n / 4 where a row begins inside one.  The heads of
        // a quad go to as many work-groups as it takes to have four per CU.
        const int64_t quads = (max_n + 3) / 4 + 1;
        const int64_t blocks = quads > 65536 ? 65536 : quads;
        const int64_t per_token = (hq + 2 * hkv + 15) / 16;
        int64_t slices = (1024 + blocks * batch - 1) / (blocks * batch);
        if (slices > per_token) slices = per_token;
        const NormRopeArgs a{static_cast<const uint16_t *>(d_q), static_cast<const uint16_t *>(d_k),
                             static_cast<const uint16_t *>(d_v), q_stride, k_stride, v_stride,
                             static_cast<const uint16_t *>(rope->d_q_weight),
                             static_cast<const uint16_t *>(rope->d_k_weight), rope->d_inv_freq, rope->eps, rope->rot_dim,
                             rope->neighbours, static_cast<int>(hq), static_cast<uint16_t *>(d_q_out)};
        const Cache kv{pool->k, pool->v, pool->k4, pool->v4, pool->scales, d_block_table, bt_stride,
                       pool->desc.num_pages, pool->desc.num_kv_heads};
        hipLaunchKernelGGL(pool->k4 ? k_norm_rope<true> : k_norm_rope<false>,
                           dim3(static_cast<unsigned>(blocks), batch, static_cast<unsigned>(slices)), dim3(256), 0, s, a,
                           kv, d_qo_indptr, d_start_pos);
        st = check_launch("k_norm_rope");
        if (st != MW_OK) return st;
    }
    st = timing_kernel_done(timing, s);
    timing_end(timing);
    return st;
}
