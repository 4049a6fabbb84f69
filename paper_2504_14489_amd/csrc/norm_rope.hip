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
// 2^-8 of a radian), and what that rounding leaves is added to cosine and sine.
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
    int rot_dim, hq;
    uint16_t *q_out;
};
struct Cache {
    uint16_t *k, *v;               // bf16 pages, or
    uint8_t *k4, *v4, *scales;     // those in 4 bits
    const int32_t *bt;
    int bt_stride, num_pages, hkv;
};

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ float lo(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float hi(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    bf16x2_t v;
    v[0] = static_cast<__bf16>(a);
    v[1] = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint32_t, v);
}
constexpr int kRor8 = 0x128;  // DPP: rotate the 16 lanes by 8
template <int kCtrl>
__device__ __forceinline__ float add_dpp(float x) {
    return x + __builtin_bit_cast(float, dpp<kCtrl>(__builtin_bit_cast(uint32_t, x)));
}

// A quad's angles in LDS, by token and pair, and the norm's weights.  Of the
// halves' pairs the first lanes take the sine with its sign turned, from a copy of
// its own.
struct Shared {
    float cos[4][kHeadDim / 2], sin[4][2][kHeadDim / 2];  // [0]: -sin, [1]: sin
    float weight[2][kHeadDim];                            // of queries and keys
};
// Which dims are paired: neighbours, the halves of a whole head (8 lanes apart), or
// the halves of its first rot_dim.
enum Pairing { kNeighbours, kWholeHalves, kHalves };

// Sum of the squares of a row's 128 values, eight of them in each of 16 lanes.
__device__ __forceinline__ float sum_squares(const float (&y)[8]) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += y[j] * y[j];
    sum = add_dpp<kXor1>(sum);
    sum = add_dpp<kXor2>(sum);
    sum = add_dpp<kHalfMirror>(sum);
    return add_dpp<kMirror>(sum);
}

// A lane's dims 8c .. 8c+7 of a head row of token t.
template <Pairing kPairing>
__device__ __forceinline__ uint4 norm_rope_row(uint4 x, bool norm, const float *weight, float eps, int rot_dim,
                                               const Shared &sh, int t, int c) {
    float y[8] = {lo(x.x), hi(x.x), lo(x.y), hi(x.y), lo(x.z), hi(x.z), lo(x.w), hi(x.w)};
    if (norm) {
        float r = rsqrtf(sum_squares(y) * (1.f / kHeadDim) + eps);
        if (__builtin_amdgcn_ballot_w64(!(r > 0x1p-63f && r < 0x1p50f)) != 0) {
            // a row whose squares leave the range of fp32, or lose bits at its lower end
            // next to as small an eps: by a power of two, the root with it
            const float k = r > 0x1p-63f && r < 0x1p50f ? 1.f : r >= 0x1p50f ? 0x1p70f : 0x1p-70f;
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= k;
            r = rsqrtf(sum_squares(y) * (1.f / kHeadDim) + eps * k * k);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = y[j] * r * weight[8 * c + j];
    }
    if constexpr (kPairing == kNeighbours) {
        if (8 * c < rot_dim) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float cs = sh.cos[t][4 * c + j], sn = sh.sin[t][1][4 * c + j];
                const float a = y[2 * j], b = y[2 * j + 1];
                y[2 * j] = a * cs - b * sn;
                y[2 * j + 1] = b * cs + a * sn;
            }
        }
    } else {
        const int half = kPairing == kWholeHalves ? 8 : rot_dim / 16;  // lanes of the first half
        const bool first = c < half;
        float p[8];
        if constexpr (kPairing == kWholeHalves) {
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = __builtin_bit_cast(float, dpp<kRor8>(__builtin_bit_cast(uint32_t, y[j])));
        } else {
            const int partner = (threadIdx.x & 48) | (first ? c + half : c < 2 * half ? c - half : c);
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = __shfl(y[j], partner);
        }
        if (kPairing == kWholeHalves || c < 2 * half) {
            const int pair = 8 * (first ? c : c - half);
            const float *cs = &sh.cos[t][pair], *sn = &sh.sin[t][first ? 0 : 1][pair];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = y[j] * cs[j] + p[j] * sn[j];
        }
    }
    return make_uint4(pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7]));
}

// Head rows of a quad's tokens t0 .. t0 + m, `heads` of each, spread over the
// `step` groups of 16 lanes that share the quad: task i is head i / m of token
// i % m.  The next row's load is in flight while one is worked on: load(h, t),
// store(h, t, x); each_row starts with the group's first row in x and returns its
// place behind these tasks.
__device__ __forceinline__ int head_of(int i, int m) {
    return m == 4 ? i >> 2 : m == 1 ? i : m == 2 ? i >> 1 : static_cast<int>(static_cast<unsigned>(i) / 3u);
}
template <class Load>
__device__ __forceinline__ uint4 row_of(int i, int t0, int m, int heads, const Load &load) {
    const int h = head_of(i, m);
    return i < m * heads ? load(h, t0 + i - h * m) : make_uint4(0, 0, 0, 0);
}
template <class Load, class Store>
__device__ __forceinline__ int each_row(uint4 x, int group, int step, int t0, int m, int heads, const Load &load,
                                        const Store &store) {
    const int tasks = m * heads;
#pragma unroll 1
    for (int i = group; i < tasks; i += step) {
        const uint4 now = x;
        x = row_of(i + step, t0, m, heads, load);
        const int h = head_of(i, m);
        store(h, t0 + i - h * m, now);
    }
    const int next = group - tasks % step;
    return next < 0 ? next + step : next;
}

// One work-group: the (up to four) new tokens of one quad of page slots; grid.z
// slices share its heads.  The quad's angles are computed once, one a thread,
// and lie in LDS; then 16 lanes take a head row at a time.  Quads, because V in 4
// bits is stored by four tokens (kv4_format.h).
// Measured (kernel alone): 4096 tokens of 32 + 2 * 8 heads into bf16, 101 MB, 23 us
// (a copy of as many bytes 21); 10315 of 64 + 2 * 8 into 4 bits, 391 MB, 84 us (a copy
// 80).  Six work-groups per CU: with the registers of five the latter takes 6% longer.
// kPassBy: rows are read and queries stored past the caches.
template <bool kFourBit, Pairing kPairing, bool kPassBy>
__global__ void __launch_bounds__(256, 6)
k_norm_rope(NormRopeArgs a, Cache kv, const int32_t *__restrict__ indptr, const int32_t *__restrict__ start_pos) {
    __shared__ __attribute__((aligned(16))) Shared sh;
    const int b = blockIdx.y, c = threadIdx.x & 15;
    const int row0 = indptr[b], n = indptr[b + 1] - row0, pos0 = start_pos[b];
    if (n <= 0 || pos0 < 0) return;
    const int32_t *btrow = kv.bt + static_cast<size_t>(b) * kv.bt_stride;
    const int quad0 = pos0 / 4, quads = (pos0 + n - 1) / 4 + 1 - quad0;
    {
        const uint16_t *from = threadIdx.x < kHeadDim ? a.q_weight : a.k_weight;
        const int d = threadIdx.x % kHeadDim;
        if (from) sh.weight[threadIdx.x / kHeadDim][d] = lo(from[d]);
    }
    const int f = threadIdx.x & 63;
    const double freq = 2 * f < a.rot_dim ? a.inv_freq[f] * 0.15915494309189533577 : 0.0;  // turns per position
    const int step = gridDim.z * 16;
    for (int i = blockIdx.x; i < quads; i += gridDim.x) {
        const int first = (quad0 + i) * 4 - pos0;  // row of the quad's first slot
        const int t0 = max(0, -first), m = min(4, n - first) - t0;
        const int pos = pos0 + first, slot = pos % kPageSize;
        const int page = pos / kPageSize < kv.bt_stride ? btrow[pos / kPageSize] : -1;
        const bool held = page >= 0 && page < kv.num_pages;  // elsewhere only the queries are written
        const int64_t row = static_cast<int64_t>(row0) + first;
        const uint16_t *q_src = a.q + row * a.q_stride, *k_src = a.k + row * a.k_stride, *v_src = a.v + row * a.v_stride;
        uint16_t *q_dst = a.q_out + row * a.hq * kHeadDim;
        const size_t at = static_cast<size_t>(held ? page : 0) * kv.hkv;
        // offsets within the quad fit 32 bits (the host refuses longer strides)
        const auto source = [&](const uint16_t *from, int stride) __attribute__((always_inline)) {
            return [=](int h, int t) __attribute__((always_inline)) {
                const int off = ((t & 1) ? stride : 0) + ((t & 2) ? 2 * stride : 0) + h * kHeadDim + 8 * c;
                if constexpr (kPassBy)
                    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + off)));
                else
                    return *reinterpret_cast<const uint4 *>(from + off);
            };
        };
        const auto load_q = source(q_src, static_cast<int>(a.q_stride)), load_k = source(k_src, static_cast<int>(a.k_stride));
        int group = blockIdx.z * 16 + (threadIdx.x >> 4);
        const uint4 q_row = row_of(group, t0, m, a.hq, load_q);  // on its way while the angles are computed
        __syncthreads();  // the last quad's angles are read
        if (2 * f < a.rot_dim) {
            const int t = threadIdx.x >> 6;
            const double turns = static_cast<double>(pos + t) * freq;
            // half turns in [-1, 1], and what their rounding to fp32 leaves (up to 2^-25; a sine
            // near 0 would be off by 2^-23) by the first order
            const double half_turns = 2.0 * (turns - rint(turns));
            const float near = static_cast<float>(half_turns);
            const float rest = static_cast<float>(half_turns - near) * 3.14159265f;
            float sn0, cs0;
            sincospif(near, &sn0, &cs0);
            const float cs = fmaf(-sn0, rest, cs0), sn = fmaf(cs0, rest, sn0);
            sh.cos[t][f] = cs;
            sh.sin[t][0][f] = -sn;
            sh.sin[t][1][f] = sn;
        }
        __syncthreads();
        group = each_row(q_row, group, step, t0, m, a.hq, load_q, [&](int h, int t, uint4 v) __attribute__((always_inline)) {
            const uint4 y = norm_rope_row<kPairing>(v, a.q_weight != nullptr, sh.weight[0], a.eps, a.rot_dim, sh, t, c);
            uint16_t *dst = q_dst + (static_cast<int>(__umul24(t, a.hq)) + h) * kHeadDim + 8 * c;
            if constexpr (kPassBy)
                __builtin_nontemporal_store(__builtin_bit_cast(u32x4, y), reinterpret_cast<u32x4 *>(dst));
            else
                *reinterpret_cast<uint4 *>(dst) = y;
        });
        if (!held) continue;
        const uint4 k_row = row_of(group, t0, m, kv.hkv, load_k);
        group = each_row(k_row, group, step, t0, m, kv.hkv, load_k, [&](int h, int t, uint4 v) __attribute__((always_inline)) {
            const uint4 y = norm_rope_row<kPairing>(v, a.k_weight != nullptr, sh.weight[1], a.eps, a.rot_dim, sh, t, c);
            if constexpr (kFourBit) {
                uint32_t byte;
                const uint32_t codes = encode_k(y, &byte);
                *reinterpret_cast<uint32_t *>(kv.k4 + (at + h) * kCodeBytes + (slot + t) * (kHeadDim / 2) + 4 * c) = codes;
                if ((c & 3) == 0)
                    kv.scales[(at + h) * kScaleBytes + (c >> 2) * kPageSize + slot + t] = static_cast<uint8_t>(byte);
            } else {
                *reinterpret_cast<uint4 *>(kv.k + ((at + h) * kPageSize + slot + t) * kHeadDim + 8 * c) = y;
            }
        });
        if constexpr (kFourBit) {
            for (int h = group; h < kv.hkv; h += step)
                write_v(v_src + h * kHeadDim, a.v_stride, kv.v4 + (at + h) * kCodeBytes, kv.scales + (at + h) * kScaleBytes,
                        slot / 4, t0, t0 + m, c);
        } else {
            const auto load_v = source(v_src, static_cast<int>(a.v_stride));
            const uint4 v_row = row_of(group, t0, m, kv.hkv, load_v);
            each_row(v_row, group, step, t0, m, kv.hkv, load_v, [&](int h, int t, uint4 v) __attribute__((always_inline)) {
                *reinterpret_cast<uint4 *>(kv.v + ((at + h) * kPageSize + slot + t) * kHeadDim + 8 * c) = v;
            });
        }
    }
}

// Rows and queries of more bytes than these, half of the last cache, go past the
// caches: queries will not be found there, and would take the place of rows that the
// projection has just written and this kernel still has to read.  Rows written by a
// copy just before, 32 + 2 * 8 heads, us past the caches and through them: 512 tokens
// 10.3 and 10.2, 4096 (84 MB) 20.9 and 20.6, 8192 (168 MB) 40 and 42, 16384 73 and 83;
// the 10315 of 64 + 2 * 8 heads above, behind nothing, 82 and 90.
constexpr int64_t kThroughBytes = int64_t{128} << 20;

using Kernel = void (*)(NormRopeArgs, Cache, const int32_t *, const int32_t *);
template <bool kFourBit, bool kPassBy>
Kernel kernel_of(const mw_norm_rope &rope) {
    return rope.neighbours              ? k_norm_rope<kFourBit, kNeighbours, kPassBy>
           : rope.rot_dim == kHeadDim ? k_norm_rope<kFourBit, kWholeHalves, kPassBy>
                                      : k_norm_rope<kFourBit, kHalves, kPassBy>;
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
    if (hq + 2 * hkv > (1 << 20) || q_stride > (1 << 28) || k_stride > (1 << 28) || v_stride > (1 << 28))
        return fail(MW_ERR_UNSUPPORTED, "%s: at most 2^20 heads and strides of 2^28 elements", who);
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
                             static_cast<int>(hq), static_cast<uint16_t *>(d_q_out)};
        const Cache kv{pool->k, pool->v, pool->k4, pool->v4, pool->scales, d_block_table, bt_stride,
                       pool->desc.num_pages, pool->desc.num_kv_heads};
        const bool past = total * (2 * hq + 2 * hkv) * kHeadDim * 2 > kThroughBytes;
        const Kernel kernel = pool->k4 ? (past ? kernel_of<true, true>(*rope) : kernel_of<true, false>(*rope))
                                       : (past ? kernel_of<false, true>(*rope) : kernel_of<false, false>(*rope));
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks), batch, static_cast<unsigned>(slices)), dim3(256), 0, s, a,
                           kv, d_qo_indptr, d_start_pos);
        st = check_launch("k_norm_rope");
        if (st != MW_OK) return st;
    }
    st = timing_kernel_done(timing, s);
    timing_end(timing);
    return st;
}
