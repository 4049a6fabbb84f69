// The KV pool in 4 bits: append (quantises) and read-back.
//
// Both are bound by memory: a (token, kv head) row is 512 bytes of K and V in bf16
// and 136 in 4 bits.  8100 tokens of 8 kv heads, 42 MB, are appended in 9.5 us and
// read back in 8 (kernels alone; a copy of as many bytes takes 9), 64 single tokens
// in 3.5 and 2.7, a launch and three dependent loads.
#include "decode_block.h"
#include "kv4_format.h"

using namespace mw;

namespace {

using namespace kv4;

// Rows [0, n) of sequence b go to positions pos0 + i; the quads of page slots
// that they touch, 16 lanes to a (quad, kv head).
struct Quad {
    int row, t0, t1;  // row of slot 4g; slots [t0, t1) of the quad are the call's
    int page, g;
};
__device__ __forceinline__ bool find_quad(Quad &q, int quad, int pos0, int n, const int32_t *btrow, int bt_stride,
                                          int num_pages) {
    const int first = quad * 4;  // position
    q.row = first - pos0;
    q.t0 = max(0, -q.row);
    q.t1 = min(4, n - q.row);
    if (first < 0 || first / kPageSize >= bt_stride || q.t0 >= q.t1) return false;
    q.page = btrow[first / kPageSize];
    q.g = (first % kPageSize) / 4;
    return q.page >= 0 && q.page < num_pages;
}

// K of tokens [t0, t1) of quad g, token t's row at src + t stride.
__device__ __forceinline__ void write_k(const uint16_t *__restrict__ src, int64_t stride, uint8_t *__restrict__ codes_at,
                                        uint8_t *__restrict__ scales_at, int g, int t0, int t1, int c) {
    uint32_t *dst = reinterpret_cast<uint32_t *>(codes_at + 4 * g * (kHeadDim / 2) + 4 * c);
    uint8_t *sc = scales_at + (c >> 2) * kPageSize + 4 * g;
    if (t1 - t0 == 4) {
        uint4 x[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) x[t] = *reinterpret_cast<const uint4 *>(src + t * stride + 8 * c);
        uint32_t bytes = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            uint32_t byte;
            dst[t * (kHeadDim / 8)] = encode_k(x[t], &byte);
            bytes |= byte << (8 * t);
        }
        if ((c & 3) == 0) *reinterpret_cast<uint32_t *>(sc) = bytes;
        return;
    }
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
        uint32_t byte;
        dst[t * (kHeadDim / 8)] = encode_k(*reinterpret_cast<const uint4 *>(src + t * stride + 8 * c), &byte);
        if ((c & 3) == 0) sc[t] = static_cast<uint8_t>(byte);
    }
}

__global__ void __launch_bounds__(256)
k_kv4_write(uint8_t *__restrict__ kpool, uint8_t *__restrict__ vpool, uint8_t *__restrict__ scales,
            const uint16_t *__restrict__ knew, const uint16_t *__restrict__ vnew, const int32_t *__restrict__ indptr,
            const int32_t *__restrict__ start_pos, const int32_t *__restrict__ bt, int bt_stride, int num_pages, int hkv) {
    const int b = blockIdx.y, c = threadIdx.x & 15;
    const int row0 = indptr[b], n = indptr[b + 1] - row0, pos0 = start_pos[b];
    const int32_t *btrow = bt + static_cast<size_t>(b) * bt_stride;
    if (n <= 0 || pos0 < 0) return;
    const int quad0 = pos0 / 4;
    const int64_t total = static_cast<int64_t>((pos0 + n - 1) / 4 + 1 - quad0) * hkv;
    for (int64_t idx = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4); idx < total;
         idx += static_cast<int64_t>(gridDim.x) * 16) {
        const int i = static_cast<int>(static_cast<uint32_t>(idx) / static_cast<uint32_t>(hkv));
        const int h = static_cast<int>(static_cast<uint32_t>(idx) - static_cast<uint32_t>(i) * hkv);
        Quad q;
        if (!find_quad(q, quad0 + i, pos0, n, btrow, bt_stride, num_pages)) continue;
        const size_t at = static_cast<size_t>(q.page) * hkv + h;
        const int64_t src = (static_cast<int64_t>(row0) + q.row) * hkv + h;  // of slot t = 0
        uint8_t *sc = scales + at * kScaleBytes;
        write_k(knew + src * kHeadDim, hkv * kHeadDim, kpool + at * kCodeBytes, sc, q.g, q.t0, q.t1, c);
        write_v(vnew + src * kHeadDim, hkv * kHeadDim, vpool + at * kCodeBytes, sc, q.g, q.t0, q.t1, c);
    }
}

__global__ void __launch_bounds__(256)
k_kv4_gather(const uint8_t *__restrict__ kpool, const uint8_t *__restrict__ vpool, const uint8_t *__restrict__ scales,
             uint16_t *__restrict__ kout, uint16_t *__restrict__ vout, const int32_t *__restrict__ indptr,
             const int32_t *__restrict__ start_pos, const int32_t *__restrict__ bt, int bt_stride, int num_pages, int hkv) {
    const int b = blockIdx.y, c = threadIdx.x & 15;
    const int row0 = indptr[b], n = indptr[b + 1] - row0, pos0 = start_pos[b];
    const int32_t *btrow = bt + static_cast<size_t>(b) * bt_stride;
    if (n <= 0 || pos0 < 0) return;
    const int quad0 = pos0 / 4;
    const int64_t total = static_cast<int64_t>((pos0 + n - 1) / 4 + 1 - quad0) * hkv;
    for (int64_t idx = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4); idx < total;
         idx += static_cast<int64_t>(gridDim.x) * 16) {
        const int i = static_cast<int>(static_cast<uint32_t>(idx) / static_cast<uint32_t>(hkv));
        const int h = static_cast<int>(static_cast<uint32_t>(idx) - static_cast<uint32_t>(i) * hkv);
        Quad q;
        const bool there = find_quad(q, quad0 + i, pos0, n, btrow, bt_stride, num_pages);
        if (q.t0 >= q.t1) continue;
        // rows on an absent page read as zeros
        uint4 kr[4];
        uint32_t vr[4][kBlocks];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            kr[t] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < kBlocks; ++k) vr[t][k] = 0;
        }
        if (there) {
            const size_t at = static_cast<size_t>(q.page) * hkv + h;
            const uint8_t *sc = scales + at * kScaleBytes + 4 * q.g;
            const uint32_t kbytes = *reinterpret_cast<const uint32_t *>(sc + (c >> 2) * kPageSize);
            uint32_t kc[4], bytes[kBlocks];
#pragma unroll
            for (int t = 0; t < 4; ++t)
                kc[t] = *reinterpret_cast<const uint32_t *>(kpool + at * kCodeBytes + (4 * q.g + t) * (kHeadDim / 2) + 4 * c);
            const uint4 vc = *reinterpret_cast<const uint4 *>(vpool + at * kCodeBytes + q.g * 256 + c * 16);
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
                bytes[k] = *reinterpret_cast<const uint32_t *>(sc + (kBlocks + k) * kPageSize);
#pragma unroll
            for (int t = 0; t < 4; ++t) kr[t] = decode_k(kc[t], kbytes >> (8 * t) & 255);
            const uint32_t codes[kBlocks] = {vc.x, vc.y, vc.z, vc.w};
            decode_v(codes, bytes, vr);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t < q.t0 || t >= q.t1) continue;
            const size_t dst = (static_cast<size_t>(row0 + q.row + t) * hkv + h) * kHeadDim;
            *reinterpret_cast<uint4 *>(kout + dst + 8 * c) = kr[t];
#pragma unroll
            for (int k = 0; k < kBlocks; ++k) *reinterpret_cast<uint32_t *>(vout + dst + 32 * k + 2 * c) = vr[t][k];
        }
    }
}

// Grid of the two row kernels: 16 (quad, kv head) to a work-group of 256, grid.y
// the sequences.  A quad more than n / 4 where a row begins inside one.
mw_status row_grid(int64_t max_n, int hkv, int32_t batch, dim3 *grid, const char *who) {
    const int64_t items = ((max_n + 3) / 4 + 1) * hkv;
    if (items > INT32_MAX) return fail(MW_ERR_UNSUPPORTED, "%s: too many rows", who);
    int64_t blocks = (items + 15) / 16;
    if (blocks > 4096) blocks = 4096;
    *grid = dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(batch));
    return MW_OK;
}

}  // namespace

extern "C" {

mw_status mw_kv4_pool_write(const mw_kv_pool *pool, int32_t batch, const int32_t *h_new_lens, const int32_t *h_start_pos,
                            const int32_t *d_qo_indptr, const int32_t *d_start_pos, const int32_t *d_block_table,
                            int32_t bt_stride, const void *d_k_new, const void *d_v_new, mw_stream stream,
                            mw_timing *timing) {
    const char *who = "mw_kv4_pool_write";
    int64_t max_n = 0, total = 0;
    mw_status st = check_rows(pool, batch, h_new_lens, h_start_pos, d_qo_indptr, d_start_pos, d_block_table, bt_stride,
                              &max_n, &total, who);
    if (st == MW_OK) st = check_pool_kind(pool, true, who);
    if (st != MW_OK) return st;
    if (total > 0 && (!d_k_new || !d_v_new || !aligned16(d_k_new) || !aligned16(d_v_new)))
        return fail(MW_ERR_INVALID_ARG, "%s: new K/V must be 16-byte aligned", who);
    dim3 grid;
    st = row_grid(max_n, pool->desc.num_kv_heads, batch, &grid, who);
    if (st != MW_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    st = timing_begin(timing, s);
    if (st != MW_OK) return st;
    if (total > 0) {
        hipLaunchKernelGGL(k_kv4_write, grid, dim3(256), 0, s, pool->k4, pool->v4, pool->scales,
                           static_cast<const uint16_t *>(d_k_new), static_cast<const uint16_t *>(d_v_new), d_qo_indptr,
                           d_start_pos, d_block_table, bt_stride, pool->desc.num_pages, pool->desc.num_kv_heads);
        st = check_launch("k_kv4_write");
        if (st != MW_OK) return st;
    }
    st = timing_kernel_done(timing, s);
    timing_end(timing);
    return st;
}

mw_status mw_kv4_pool_gather(const mw_kv_pool *pool, int32_t batch, const int32_t *h_lens, const int32_t *h_start_pos,
                             const int32_t *d_indptr, const int32_t *d_start_pos, const int32_t *d_block_table,
                             int32_t bt_stride, void *d_k_out, void *d_v_out, mw_stream stream, mw_timing *timing) {
    const char *who = "mw_kv4_pool_gather";
    int64_t max_n = 0, total = 0;
    mw_status st = check_rows(pool, batch, h_lens, h_start_pos, d_indptr, d_start_pos, d_block_table, bt_stride, &max_n,
                              &total, who);
    if (st == MW_OK) st = check_pool_kind(pool, true, who);
    if (st != MW_OK) return st;
    if (total > 0 && (!d_k_out || !d_v_out || !aligned16(d_k_out) || !aligned16(d_v_out)))
        return fail(MW_ERR_INVALID_ARG, "%s: outputs must be 16-byte aligned", who);
    dim3 grid;
    st = row_grid(max_n, pool->desc.num_kv_heads, batch, &grid, who);
    if (st != MW_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    st = timing_begin(timing, s);
    if (st != MW_OK) return st;
    if (total > 0) {
        hipLaunchKernelGGL(k_kv4_gather, grid, dim3(256), 0, s, pool->k4, pool->v4, pool->scales,
                           static_cast<uint16_t *>(d_k_out), static_cast<uint16_t *>(d_v_out), d_indptr, d_start_pos,
                           d_block_table, bt_stride, pool->desc.num_pages, pool->desc.num_kv_heads);
        st = check_launch("k_kv4_gather");
        if (st != MW_OK) return st;
    }
    st = timing_kernel_done(timing, s);
    timing_end(timing);
    return st;
}

}  // extern "C"
