// Prefill attention over the cache in 4 bits.
#include <algorithm>

#include "kv4_block.h"

using namespace mw;

namespace {

using namespace dk;
using namespace kv4;

typedef float f32x16 __attribute__((ext_vector_type(16)));

// x of a lane and of the one 32 away combined by f, in both.
template <class F>
__device__ __forceinline__ float across_half(float x, const F &f) {
    const uint32_t a = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const uint32_t lo = r[0], hi = r[1];
    return f(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}

// Takes blocks of V that are not finite out of four tokens' scale bytes, of `tokens`
// (0 or 255 in each byte): their scales become finite, which times a probability of
// 0 gives 0.  Returns them: bit i of byte j is block i of token j.
__device__ __forceinline__ uint32_t take_bad(uint32_t (&bytes)[kBlocks], uint32_t tokens) {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
        const uint32_t x = bytes[i] & tokens;
        const uint32_t full = ((x & 0x7f7f7f7fu) + 0x01010101u) >> 7 & x >> 7 & 0x01010101u;  // 1 where x has 255
        bytes[i] &= ~(full * 255);
        bad |= full << i;
    }
    return bad;
}
// Mask of the first n of four bytes.
__device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << 8 * n) - 1; }

// Unpacks the pages of a batch's sequences, laid end to end, to bf16 pages
// [page][kv head][16][128] and writes the table that names them.  One wave to a
// (page, kv head).
//
// A row never gets anything from a token that it does not see: the attention masks its
// scores, but would multiply V by a probability of 0, and 0 times a V that is not
// finite is NaN.  So such blocks of V of the new tokens are unpacked as zeros and noted
// in `bad`, four bits a token (64 a page), and k_kv4_unseen makes their dims NaN in the
// rows from their token on.
struct ChunkLengths {
    const int32_t *indptr, *prefix;
    int batch, bt_stride;
    __device__ __forceinline__ int pages(int b) const {
        if (b >= batch) return 0;
        const int64_t n = static_cast<int64_t>(indptr[b + 1]) - indptr[b], len = n > 0 ? n + prefix[b] : 0;  // (nothing is read without new tokens)
        const int64_t np = (len + kPageSize - 1) / kPageSize;
        return static_cast<int>(max(int64_t{0}, min(np, static_cast<int64_t>(bt_stride))));
    }
};

__global__ void __launch_bounds__(256)
k_kv4_unpack(const uint8_t *__restrict__ kpool, const uint8_t *__restrict__ vpool, const uint8_t *__restrict__ scales,
             uint16_t *__restrict__ kout, uint16_t *__restrict__ vout, uint16_t *__restrict__ bad,
             int32_t *__restrict__ table, int table_stride, const int32_t *__restrict__ indptr, const int32_t *__restrict__ prefix, const int32_t *__restrict__ bt,
             int bt_stride, int batch, int num_pages, int hkv, int64_t items) {
    const int lane = threadIdx.x & 63;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= items) return;
    const int page_no = static_cast<int>(item / hkv), h = static_cast<int>(item - static_cast<int64_t>(page_no) * hkv);
    const ChunkLengths len{indptr, prefix, batch, bt_stride};
    int running = 0, b = -1, p = 0;
    for (int b0 = 0; b0 < batch; b0 += 64) {
        const int np = len.pages(b0 + lane);
        const int incl = running + lane_scan(np);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(page_no >= incl - np && page_no < incl);
        if (hit) {
            const int src = __builtin_ctzll(hit);
            b = b0 + src;
            p = page_no - __builtin_amdgcn_readlane(incl - np, src);
            break;
        }
        running = __builtin_amdgcn_readlane(incl, 63);
    }
    if (b < 0 || p >= table_stride) return;  // device lengths that disagree with the host's
    const int page = bt[static_cast<size_t>(b) * bt_stride + p];
    const bool ok = page >= 0 && page < num_pages;
    if (h == 0 && lane == 0) table[static_cast<size_t>(b) * table_stride + p] = ok ? page_no : -1;
    if (!ok) return;
    const size_t at = static_cast<size_t>(page) * hkv + h;
    const uint8_t *sc = scales + at * kScaleBytes;
    // K: four lane-contiguous dwords (8 dims) of codes, 16 bytes out each
    const uint32_t *kc = reinterpret_cast<const uint32_t *>(kpool + at * kCodeBytes) + lane;
    uint32_t codes_k[4], byte_k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        codes_k[i] = kc[64 * i];
        byte_k[i] = sc[((lane & 15) >> 2) * kPageSize + 4 * i + (lane >> 4)];
    }
    const int g = lane >> 4, c = lane & 15;
    const uint4 vc = *reinterpret_cast<const uint4 *>(vpool + at * kCodeBytes + lane * 16);
    uint32_t bytes[kBlocks], vr[4][kBlocks];
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) bytes[k] = *reinterpret_cast<const uint32_t *>(sc + (kBlocks + k) * kPageSize + 4 * g);
    uint4 *ko = reinterpret_cast<uint4 *>(kout + static_cast<size_t>(item) * (kPageSize * kHeadDim)) + lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) ko[64 * i] = decode_k(codes_k[i], byte_k[i]);
    const int first = kPageSize * p + 4 * g, r = prefix[b], n = indptr[b + 1] - indptr[b];
    if (kPageSize * (p + 1) > r) {
        const uint32_t w = take_bad(bytes, first_bytes(r + n - first) & ~first_bytes(r - first));
        if (c == 0) bad[4 * item + g] = static_cast<uint16_t>((w & 15) | (w >> 4 & 0xf0) | (w >> 8 & 0xf00) | (w >> 12 & 0xf000));
    }
    const uint32_t codes[kBlocks] = {vc.x, vc.y, vc.z, vc.w};
    decode_v(codes, bytes, vr);
    uint32_t *vo = reinterpret_cast<uint32_t *>(vout + static_cast<size_t>(item) * (kPageSize * kHeadDim)) + c;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) vo[(4 * g + t) * (kHeadDim / 2) + 16 * k] = vr[t][k];
}

// Behind the attention on unpacked pages: for each (sequence, kv head) the first new
// token whose V is not finite in a block of dims, and NaN there in all rows from it on.
// (2.1 to 2.9 us of a call: a launch and three dependent loads.)
__global__ void __launch_bounds__(256)
k_kv4_unseen(uint16_t *__restrict__ out, const uint64_t *__restrict__ bad, const int32_t *__restrict__ table,
             int table_stride, int pages, const int32_t *__restrict__ indptr, const int32_t *__restrict__ prefix, int group) {
    __shared__ int s_first[kBlocks];
    const int h = blockIdx.x, hkv = gridDim.x, b = blockIdx.y;
    const int row0 = indptr[b], n = indptr[b + 1] - row0, r = prefix[b];
    if (n <= 0 || r < 0) return;
    if (threadIdx.x < kBlocks) s_first[threadIdx.x] = n;
    __syncthreads();
    const int end = min((r + n - 1) / kPageSize + 1, table_stride);
    for (int p = r / kPageSize + static_cast<int>(threadIdx.x); p < end; p += 256) {
        const int at = table[static_cast<size_t>(b) * table_stride + p];
        const uint64_t tokens = at >= 0 && at < pages ? bad[static_cast<size_t>(at) * hkv + h] : 0;
        if (tokens == 0) continue;
        for (int i = 0; i < kBlocks; ++i) {
            const uint64_t of_block = tokens >> i & 0x1111111111111111u;
            if (of_block) atomicMin(&s_first[i], kPageSize * p + __builtin_ctzll(of_block) / 4 - r);
        }
    }
    __syncthreads();
    for (int i = 0; i < kBlocks; ++i) {
        // 16 bytes a thread: (row, head) of the group, a quarter of the block's dims
        const int64_t first = static_cast<int64_t>(s_first[i]) * group * 4, last = static_cast<int64_t>(n) * group * 4;
        for (int64_t j = first + threadIdx.x; j < last; j += 256) {
            const int64_t row_head = j >> 2, row = row_head / group;
            const size_t at = ((row0 + row) * hkv + h) * group + (row_head - row * group);
            *reinterpret_cast<uint4 *>(out + at * kHeadDim + 32 * i + 8 * (j & 3)) =
                make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
        }
    }
}

// Workspace of a prefill call: K pages, V pages, which of their blocks are not finite,
// their table, then the workspace of the attention itself.
struct UnpackLayout {
    int64_t pages;
    int64_t table_stride;
    size_t off_v, off_bad, off_table, off_ws;
};
mw_status unpack_layout(int32_t batch, const int32_t *h_new_lens, const int32_t *h_prefix_lens, int64_t hkv,
                        UnpackLayout *u, const char *who) {
    u->pages = 0;
    u->table_stride = 1;
    for (int32_t b = 0; b < batch; ++b) {
        const int64_t np = h_new_lens[b] == 0 ? 0 : (static_cast<int64_t>(h_new_lens[b]) + h_prefix_lens[b] + kPageSize - 1) / kPageSize;
        u->pages += np;
        u->table_stride = np > u->table_stride ? np : u->table_stride;
    }
    if (u->pages > INT32_MAX || u->pages * hkv > static_cast<int64_t>(INT32_MAX) * 4)
        return fail(MW_ERR_UNSUPPORTED, "%s: too many pages", who);
    const size_t pages_bytes = static_cast<size_t>(u->pages) * hkv * (kPageSize * kHeadDim * 2);
    u->off_v = pages_bytes;
    u->off_bad = 2 * pages_bytes;
    u->off_table = u->off_bad + static_cast<size_t>(u->pages) * hkv * 8;
    u->off_ws = (u->off_table + static_cast<size_t>(batch) * u->table_stride * 4 + 255) & ~static_cast<size_t>(255);
    return MW_OK;
}

// ------------------------------------------------------- few rows: straight from the codes
// A chunk of few rows reads each page for few query blocks, so unpacking it to
// bf16 first (write 8192 bytes, read them again) costs more than it saves: 64
// tokens over 8000 of 32/8 heads take 25 us like this and 42 unpacked, 16 tokens 17
// and 42.  A tile takes 1.5 us of a CU with one work-group, 1.1 of each of two; it
// is bound by what each of its four waves does one after the other (scores, conversion
// of V, exponentials, second product), not by memory (reading the same tile over and
// over changes nothing; without the conversions it is 15-20% shorter, without the
// exponentials or half of the second product 10% each).
//
// A work-group is four waves on 128 rows of a (sequence, kv head) (row = position *
// group + head, 32 per wave) and one piece of their keys, 64 at a time:
//   * S^T[key][row] = K Q^T on the scaled 32x32x64 instruction, K from memory as it
//     lies (16 bytes a lane: one block of one key), Q as two e4m3 operands.
//   * V is converted once for the four waves, a page each, into LDS in the order in
//     which the second product takes it, [dim block][16 keys][half][dim][8 keys]:
//     a lane of the page has four consecutive keys of eight dims, and the product's
//     k slots of half h are keys 4h .. 4h+3 and 8+4h .. +3 of the 16, as the score
//     registers hold them, so each dim is one 8-byte store and each operand one
//     16-byte read.  Lanes 16 apart store quads of one half and lanes 8 apart flip
//     their two dims, so that neither store nor read has a bank conflict (with
//     half of the LDS cycles lost to them, long chunks took 2-4% longer).
//   * the causal mask by position; online softmax as in the other kernels.
// K of the next tile and the V codes of the one after it are on their way while a
// tile is worked on; one barrier a tile.  A piece leaves (m, l) and its unnormalised
// output in the workspace and k_kv4_merge adds them up, unless it is the only one.
//
// What a row does not see never reaches it.  Its scores are masked, but a V block that
// is not finite would come through the product, as 0 times NaN, to all rows of the
// wave.  So in the tiles that some row of the block does not see whole (at most the
// last two or three) V holds zeros in its place, and the block is noted beside V:
// it makes its dims NaN in the rows from its position on.
constexpr int kBlockRows = 128;
constexpr int kTileKeys = 64;
constexpr int kMaxPieces = 64;  // (a lane of the merging wave each)
constexpr int kTableTiles = 512;  // tiles of a piece, whose table entries fit the LDS copy

// The work-groups of a call: those of a sequence after the earlier ones', its pieces'
// blocks in turn, kv heads fastest (a die's L2 then has those of one).  What a group
// leaves stands at its number: rows of the largest block each.
struct FewRows {
    float *o;    // [groups][block_rows][128]
    float2 *ml;  // [groups][block_rows]
    int groups, block_rows, piece_tiles, max_pieces;
    // (blocks, pieces at most) of a sequence
    __device__ __forceinline__ int2 of(int n, int r, int group) const {
        if (n <= 0 || r < 0) return make_int2(0, 0);
        const int tiles = (r + n + kTileKeys - 1) / kTileKeys;
        return make_int2((n * group + kBlockRows - 1) / kBlockRows, prefill_pieces(tiles, piece_tiles, max_pieces));
    }
};

// A barrier for what the waves leave each other in LDS.  (__syncthreads would also
// wait for the global loads on their way: 1.5 us a tile, whatever else it does.)
__device__ __forceinline__ void tile_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__global__ void __launch_bounds__(256, 2)
k_kv4_prefill(const uint8_t *__restrict__ kpool, const uint8_t *__restrict__ vpool, const uint8_t *__restrict__ scales,
              const uint16_t *__restrict__ q, uint16_t *__restrict__ out, const int32_t *__restrict__ indptr,
              const int32_t *__restrict__ prefix, const int32_t *__restrict__ bt, int bt_stride, int batch, Divisor hkv,
              Divisor group, int num_pages, float scale_log2, FewRows ws) {
    __shared__ __attribute__((aligned(16))) char s_v[2][kTileKeys * kHeadDim * 2];
    __shared__ __attribute__((aligned(16))) int32_t s_bt[4 * kTableTiles];  // (page, kv head) blocks; -1: absent
    __shared__ uint32_t s_bad[2][kTileKeys / 4];  // bit i of byte j: block i of V of key 4 [.] + j is not finite
    __shared__ int s_absent;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    // 64 sequences at a time are searched for this work-group's
    const int x = blockIdx.x, xb = x / hkv, kvh = x - xb * hkv;
    int b = -1, row0 = 0, n = 0, r = 0, nqb = 1, at_b = 0;
    for (int b0 = 0, running = 0; b0 < batch; b0 += 64) {
        const int at = min(b0 + lane, batch - 1), row = indptr[at], len = indptr[at + 1] - row, pre = prefix[at];
        const int2 of = ws.of(b0 + lane < batch ? len : 0, pre, group);
        const int count = of.x * of.y, incl = running + lane_scan(count);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(xb >= incl - count && xb < incl);
        if (hit) {
            const int src = __builtin_ctzll(hit);
            b = b0 + src;
            at_b = xb - __builtin_amdgcn_readlane(incl - count, src);
            row0 = __builtin_amdgcn_readlane(row, src);
            n = __builtin_amdgcn_readlane(len, src);
            r = __builtin_amdgcn_readlane(pre, src);
            nqb = __builtin_amdgcn_readlane(of.x, src);
            break;
        }
        running = __builtin_amdgcn_readlane(incl, 63);
    }
    if (b < 0) return;
    const int piece = at_b / nqb, blk = at_b - piece * nqb;
    const int rows = n * group, hq = hkv * group;
    const int nt = prefill_block_tiles<int>(r, n, blk, kBlockRows, group);
    // (device lengths that disagree with the host's)
    if (nt <= 0 || nt > ws.piece_tiles * ws.max_pieces || min(kBlockRows, rows - blk * kBlockRows) > ws.block_rows) return;
    const int pieces = prefill_pieces(nt, ws.piece_tiles, ws.max_pieces);
    if (piece >= pieces) return;
    const int t_lo = piece * nt / pieces, t_hi = (piece + 1) * nt / pieces;
    const int len = r + n, np = min((len + kPageSize - 1) / kPageSize, bt_stride);
    const int32_t *btrow = bt + static_cast<size_t>(b) * bt_stride;
    if (threadIdx.x == 0) s_absent = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * (t_hi - t_lo); i += 256) {
        const int p = 4 * t_lo + i;
        const int page = p < np ? btrow[p] : -1;
        const bool there = page >= 0 && page < num_pages;
        s_bt[i] = there ? page * hkv + kvh : -1;
        if (!there) s_absent = 1;
    }

    // this lane's row, and the tiles that some row of the wave sees
    const int first = blk * kBlockRows + 32 * wave;
    const int mine = first + l32;
    const bool valid = mine < rows;
    const int pos = valid ? mine / group : n - 1, head = valid ? mine - pos * group : 0;
    const int seen = r + pos;  // the last key it sees
    const int t_whole = (r + blk * kBlockRows / group + 1) / kTileKeys;  // tiles that every row of the block sees whole
    const int nt_w = first < rows ? (r + min(first + 31, rows - 1) / group) / kTileKeys + 1 : 0;
    i32x8 q_hi[2], q_lo[2];
    float q_scale;
    {
        const uint16_t *qp = q + (static_cast<size_t>(row0 + pos) * hq + kvh * group + head) * kHeadDim + 16 * half;
        uint4 raw[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            raw[i] = first < rows ? *reinterpret_cast<const uint4 *>(qp + 64 * (i >> 2) + 32 * (i >> 1 & 1) + 8 * (i & 1))
                                  : make_uint4(0, 0, 0, 0);
        const float f = split_q<false>(raw, q_hi, q_lo) * scale_log2;
        q_scale = f < 1e-37f ? 1e-37f : f;  // (above 0, or a masked score would be a NaN; of a NaN row, NaN)
    }
    f32x16 oacc[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) oacc[d] = f32x16{};
    // a row may see no key of the piece's first tiles
    float m_run = -__FLT_MAX__, l_run = 0.f;

    // the lane's codes of a tile: K of keys l32 and 32 + l32, blocks half and 2 + half;
    // V of page `wave`, key quad g, dims 32 b + 2 c, + 1
    const int g = (lane >> 5) | (lane >> 3 & 2), c = lane & 15;  // (quads of one half of the slots side by side)
    uint4 kc[4], vc = make_uint4(0, 0, 0, 0);
    uint32_t ks[4], vs[kBlocks] = {0, 0, 0, 0};
    const uint8_t *const k_lane = kpool + (l32 & 15) * 64 + half * 16;
    const uint8_t *const ks_lane = scales + half * kPageSize + (l32 & 15);
    const auto load_k = [&](int t) __attribute__((always_inline)) {
        const int32_t *at = s_bt + 4 * (t - t_lo);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const size_t block = max(at[2 * kb + (l32 >> 4)], 0);
            const uint8_t *src = k_lane + block * kCodeBytes, *sc = ks_lane + block * kScaleBytes;
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                kc[2 * kb + d] = *reinterpret_cast<const uint4 *>(src + 32 * d);
                ks[2 * kb + d] = sc[2 * kPageSize * d];
            }
        }
    };
    const auto load_v = [&](int t) __attribute__((always_inline)) {
        const size_t block = max(__builtin_amdgcn_readfirstlane(s_bt[4 * (t - t_lo) + wave]), 0);
        vc = *reinterpret_cast<const uint4 *>(vpool + block * kCodeBytes + g * 256 + c * 16);
        const uint8_t *sc = scales + block * kScaleBytes + kBlocks * kPageSize + 4 * g;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) vs[i] = *reinterpret_cast<const uint32_t *>(sc + i * kPageSize);
    };
    const auto store_v = [&](int t, int buf) __attribute__((always_inline)) {
        // keys past the sequence or on an absent page are zeros: 0 times the infinite
        // scale of a slack slot would not be 0
        const int there = __builtin_amdgcn_readfirstlane(s_bt[4 * (t - t_lo) + wave]) < 0 ? 0 : len - (t * kTileKeys + wave * kPageSize + 4 * g);
        const uint32_t mask = first_bytes(there);
        const uint32_t codes[kBlocks] = {vc.x, vc.y, vc.z, vc.w};
        uint32_t bytes[kBlocks], v[4][kBlocks];
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) bytes[i] = vs[i] & mask;
        if (t >= t_whole) {
            const uint32_t bad = take_bad(bytes, ~0u);
            if (c == 0) s_bad[buf][4 * wave + g] = bad;
        }
        decode_v(codes, bytes, v);
        char *dst = s_v[buf] + (2 * wave + (g & 1)) * 512 + c * 32 + (g >> 1) * 8;
        const int flip = 16 * (c >> 3);
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            // two dims of four keys each to four keys of two dims
            *reinterpret_cast<uint2 *>(dst + i * 4096 + flip) =
                make_uint2(__builtin_amdgcn_perm(v[1][i], v[0][i], 0x05040100), __builtin_amdgcn_perm(v[3][i], v[2][i], 0x05040100));
            *reinterpret_cast<uint2 *>(dst + i * 4096 + 16 - flip) =
                make_uint2(__builtin_amdgcn_perm(v[1][i], v[0][i], 0x07060302), __builtin_amdgcn_perm(v[3][i], v[2][i], 0x07060302));
        }
    };

    // (the last tile's loads are made again instead of none: with loads that may not
    // have been made the compiler waits for all that may be on their way)
    const int t_end = t_hi - 1;
    __syncthreads();
    const bool absent = s_absent != 0;
    load_v(t_lo);
    load_k(t_lo);
    store_v(t_lo, 0);
    load_v(min(t_lo + 1, t_end));
    tile_barrier();
    int t = t_lo;
    for (const int t_seen = min(t_hi, nt_w); t < t_seen; ++t) {
        f32x16 sc[2];
        {
            if (absent) {  // keys on an absent page are zeros
                const int32_t *at = s_bt + 4 * (t - t_lo);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool there = at[2 * (i >> 1) + (l32 >> 4)] >= 0;
                    kc[i] = sel4(there, kc[i]);
                    ks[i] = there ? ks[i] : kBias;
                }
            }
            const f32x16 zero{};
#pragma unroll
            for (int d = 0; d < 2; ++d)
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb) {
                        const uint4 k = kc[2 * kb + d];
                        const i32x8 a{static_cast<int>(k.x), static_cast<int>(k.y), static_cast<int>(k.z), static_cast<int>(k.w), 0, 0, 0, 0};
                        const int sb = static_cast<int>(ks[2 * kb + d]);
                        sc[kb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, part ? q_lo[d] : q_hi[d], d + part ? sc[kb] : zero,
                                                                                 4, 0, 0, sb, 0, 127);
                    }
        }
        // the loads below go to the registers that the instructions above have read: moved
        // up they would take others, to be waited for and copied at the end of the tile
        __builtin_amdgcn_sched_barrier(0);
        load_k(min(t + 1, t_end));
        store_v(min(t + 1, t_end), (t + 1 - t_lo) & 1);
        __builtin_amdgcn_sched_barrier(0);
        load_v(min(t + 2, t_end));
        {
            const int k0 = t * kTileKeys;
            if (k0 + kTileKeys - 1 > r + first / group) {  // some row of the wave does not see the whole tile
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (k0 + 32 * kb + 8 * (i >> 2) + 4 * half + (i & 3) > seen) sc[kb][i] = -INFINITY;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; i += 2)
                    mx = __builtin_elementwise_maximum(__builtin_elementwise_maximum(mx, sc[kb][i]), sc[kb][i + 1]);
            mx = across_half(mx, [](float a, float b) { return __builtin_elementwise_maximum(a, b); }) * q_scale;
            if (__builtin_amdgcn_ballot_w64(mx > m_run + kRescaleLog2) != 0) {
                const float m_new = fmaxf(m_run, mx);
                const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
                m_run = m_new;
                l_run *= alpha;
#pragma unroll
                for (int d = 0; d < 4; ++d) oacc[d] *= alpha;
            }
            // bf16 for the second product, as in the bf16 cache's kernels (off by 2^-8 of a
            // weight at most); the sum is of the weights before that
            bf16x8 p[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[s >> 1][8 * (s & 1) + i], q_scale, -m_run));
                l_run += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
                p[s] = __builtin_bit_cast(bf16x8, make_uint4(cvt2(w[0], w[1]), cvt2(w[2], w[3]), cvt2(w[4], w[5]), cvt2(w[6], w[7])));
            }
            const char *vb = s_v[(t - t_lo) & 1] + half * 512 + (l32 ^ l32 >> 4) * 16;
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        *reinterpret_cast<const bf16x8 *>(vb + (4 * d + s) * 1024), p[s], oacc[d], 0, 0, 0);
        }
        if (t >= t_whole) {
            const uint32_t bad = s_bad[(t - t_lo) & 1][lane & 15];
            if (__builtin_amdgcn_ballot_w64(bad != 0) != 0) {
                uint32_t mine = 0;  // blocks of V that the row sees
#pragma unroll 1
                for (int i = 0; i < kTileKeys; ++i) {
                    const uint32_t of_key = __builtin_amdgcn_readlane(bad, i >> 2) >> (8 * (i & 3)) & 15;
                    mine |= t * kTileKeys + i <= seen ? of_key : 0;
                }
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) oacc[d][i] = mine >> d & 1 ? NAN : oacc[d][i];
            }
        }
        tile_barrier();
    }
    for (; t < t_hi; ++t) {  // tiles past all of the wave's rows: its page of each only
        store_v(min(t + 1, t_end), (t + 1 - t_lo) & 1);
        load_v(min(t + 2, t_end));
        tile_barrier();
    }
    if (!valid) return;
    l_run = across_half(l_run, [](float a, float b) { return a + b; });
    const size_t at = static_cast<size_t>(row0 + pos) * hq + kvh * group + head;
    if (pieces == 1) {
        const float inv = 1.f / l_run;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<uint2 *>(out + at * kHeadDim + 32 * d + 8 * i + 4 * half) =
                    make_uint2(cvt2(oacc[d][4 * i] * inv, oacc[d][4 * i + 1] * inv),
                               cvt2(oacc[d][4 * i + 2] * inv, oacc[d][4 * i + 3] * inv));
        return;
    }
    const size_t slot = static_cast<size_t>(x) * ws.block_rows + mine - blk * kBlockRows;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4 *>(ws.o + slot * kHeadDim + 32 * d + 8 * i + 4 * half) =
                f32x4{oacc[d][4 * i], oacc[d][4 * i + 1], oacc[d][4 * i + 2], oacc[d][4 * i + 3]};
    if (half == 0) ws.ml[slot] = make_float2(m_run, l_run);
}

// The pieces of every row that has more than one, a wave to a (row, head).
__global__ void __launch_bounds__(256)
k_kv4_merge(uint16_t *__restrict__ out, const int32_t *__restrict__ indptr, const int32_t *__restrict__ prefix, Divisor hkv,
            Divisor group, FewRows ws) {
    const int b = blockIdx.y, row0 = indptr[b], n = indptr[b + 1] - row0, r = prefix[b], hq = hkv * group;
    const int lane = threadIdx.x & 63, at = 4 * blockIdx.x + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pos_kvh = at / group, pos = pos_kvh / hkv, kvh = pos_kvh - pos * hkv;
    if (pos >= n) return;
    const int row = pos * group + at - pos_kvh * group, blk = row / kBlockRows;
    const int nt = prefill_block_tiles<int>(r, n, blk, kBlockRows, group);
    const int pieces = prefill_pieces(nt, ws.piece_tiles, ws.max_pieces);
    if (pieces < 2) return;
    int first = blk;  // the work-group of the block's first piece, then over kv heads
    for (int b0 = 0; b0 < b; b0 += 64) {
        const int seq = min(b0 + lane, b);
        const int2 of = ws.of(seq < b ? indptr[seq + 1] - indptr[seq] : 0, prefix[seq], group);
        first += __builtin_amdgcn_readlane(lane_scan(of.x * of.y), 63);
    }
    first = first * hkv + kvh;
    const int step = ws.of(n, r, group).x * hkv;
    if (first < 0 || first + (pieces - 1) * step >= ws.groups) return;  // (device lengths that disagree with the host's)
    const size_t slot = static_cast<size_t>(first) * ws.block_rows + row - blk * kBlockRows;
    const size_t next = static_cast<size_t>(step) * ws.block_rows;
    HeadSum s;
    s.add(ws.ml[slot + min(lane, pieces - 1) * next], pieces, lane, [&](int p) __attribute__((always_inline)) {
        return reinterpret_cast<const float2 *>(ws.o + (slot + p * next) * kHeadDim)[lane];
    });
    const float inv = 1.f / s.L;
    reinterpret_cast<uint32_t *>(out + (static_cast<size_t>(row0) * hq + at) * kHeadDim)[lane] = cvt2(s.acc.x * inv, s.acc.y * inv);
}

// Whether a call goes straight from the codes, and in which pieces: by the costs
// below, fitted to 82 calls of 1 to 500 tokens over 0 to 30000, of one sequence and
// of batches, of 1 to 32 kv heads, each made all three ways: straight from the codes
// with one work-group to a CU, with two that slow each other down, or unpacked
// first.  The way so chosen took 1% longer than the fastest in the mean and 14% at
// most.  us (one, two, unpacked), 8 kv heads of 4 query heads, as measured now:
//       1 token over 0           6.6    6.6    9.8      64 over 2000      17.3  20.9  27.7
//      16 tokens over 8000      16.5   19.6   42.1      64 over 30000     57    53    83
//     256 tokens over 0         14.9   15.0   14.3     256 over 8000      61    55    57
//     16 sequences of 4 over 4000  50  35    114        4 of 128 over 500 27    31    24
// The costs are those of a whole MI355X whatever CUs the stream has, so that the
// workspace and the results do not depend on it.  On fewer CUs the way straight from the
// codes slows down more than the other, whose unpacking needs few: over 18 calls the one
// chosen took 1% longer than the fastest in the mean (8% at most) on 256 CUs, 3% (18%)
// on 192, 7% (35%) on 128, 17% (81%) on 64 and 37% (175%) on 32, where 256 tokens over 0
// take 42 us and unpacked 15.
constexpr int kCus = 256;
constexpr size_t kRowBytes = kHeadDim * 4 + 8;
constexpr int kFewBlocks = 8;  // (pages read by more blocks are unpacked with profit)
struct FewCost {
    double fixed, tile, byte;  // us of a call, of a tile of the longest piece, of a byte of partials out or in
};
constexpr FewCost kFewCost[2] = {{6.5, 1.5, 0.33e-6}, {5.6, 2.29, 0.27e-6}};
// us of a call (2.1 of them k_kv4_unseen), of a tile of each CU (a sixteenth of the keys
// at least: its pieces), of the first tiles, of a byte of pages read, written and read
constexpr struct {
    double fixed, tile, first, byte;
} kUnpackCost = {11.8, 1.03, 0.68, 0.203e-6};
struct FewPlan {
    int32_t groups;  // work-groups; 0: not straight from the codes
    int32_t block_rows, piece_tiles, max_pieces;
    size_t rows, bytes;  // of workspace
};
FewPlan few_plan(int32_t batch, const int32_t *h_new_lens, const int32_t *h_prefix_lens, int64_t hkv, int64_t group) {
    FewPlan p{};
    int64_t tiles = 0, work = 0, max_n = 0;
    int32_t most = 0;
    const auto blocks_of = [&](int32_t b) -> int64_t { return (h_new_lens[b] * group + kBlockRows - 1) / kBlockRows; };
    const auto tiles_of = [&](int32_t b) -> int32_t {
        return h_new_lens[b] == 0 ? 0 : (h_prefix_lens[b] + h_new_lens[b] + kTileKeys - 1) / kTileKeys;
    };
    for (int32_t b = 0; b < batch; ++b) {
        if (static_cast<int64_t>(h_prefix_lens[b]) + h_new_lens[b] > int64_t{kTableTiles} * kMaxPieces * kTileKeys) return p;
        tiles += tiles_of(b);
        work += blocks_of(b) * tiles_of(b);
        max_n = std::max<int64_t>(max_n, h_new_lens[b]);
        most = std::max(most, tiles_of(b));
    }
    if (max_n == 0 || max_n * group > kFewBlocks * kBlockRows) return p;
    const double tile_bytes = kTileKeys * kHeadDim * 4 + kTileKeys / kPageSize * (2 * kCodeBytes + kScaleBytes);
    double best = kUnpackCost.fixed + kUnpackCost.tile * std::max(static_cast<double>(work * hkv) / kCus, static_cast<double>(most) / 16) +
                  kUnpackCost.first * static_cast<double>(std::min(most, 8)) +
                  kUnpackCost.byte * tile_bytes * static_cast<double>(tiles * hkv);
    const auto groups = [&](int32_t len) {
        int64_t sum = 0;
        for (int32_t b = 0; b < batch; ++b) sum += blocks_of(b) * ((tiles_of(b) + len - 1) / len);
        return sum * hkv;
    };
    for (int per_cu = 1; per_cu <= 2; ++per_cu) {
        const int64_t slots = per_cu * kCus;
        // the shortest pieces that all run at once, or, where many short sequences leave
        // few places for a long one's, in up to four rounds (4 tokens each over 30000 and
        // 59 times over 100: 35 us, in one round 325)
        for (int rounds = 1, last = 0; rounds <= 4; rounds *= 2) {
            int32_t lo = std::max<int32_t>(2, (most + kMaxPieces - 1) / kMaxPieces);
            for (int32_t hi = std::max(lo, std::min(most, kTableTiles)); lo < hi;) {
                const int32_t mid = (lo + hi) / 2;
                if (groups(mid) <= rounds * slots)
                    hi = mid;
                else
                    lo = mid + 1;
            }
            if (lo == last) break;
            last = lo;
            const int64_t n = groups(lo), len = std::min(lo, most);
            if (n > INT32_MAX) break;
            double moved = 0;  // bytes of partials
            for (int32_t b = 0; b < batch && lo < most; ++b)
                if (tiles_of(b) > lo) moved += static_cast<double>(h_new_lens[b]) * hkv * group * ((tiles_of(b) + lo - 1) / lo) * kRowBytes;
            const FewCost &c = kFewCost[per_cu - 1];
            const double in_turn = n <= slots ? len : std::min<double>(len * ((n + slots - 1) / slots), len + static_cast<double>(work * hkv) / slots);
            const double us = c.fixed + c.tile * in_turn + c.byte * 2.0 * moved;
            if (us >= best) continue;
            best = us;
            p.groups = static_cast<int32_t>(n);
            p.block_rows = static_cast<int32_t>(std::min<int64_t>(kBlockRows, max_n * group));
            p.piece_tiles = lo;
            p.max_pieces = (most + lo - 1) / lo;
            p.rows = lo < most ? static_cast<size_t>(n) * p.block_rows : 0;
            p.bytes = p.rows * kRowBytes;
        }
    }
    return p;
}

}  // namespace

extern "C" {

mw_status mw_kv4_prefill_workspace_size(const mw_attn_shape *shape, int32_t batch, const int32_t *h_new_lens,
                                        const int32_t *h_prefix_lens, int32_t num_cus, size_t *bytes) {
    const char *who = "mw_kv4_prefill_workspace_size";
    size_t inner = 0;
    mw_status st = mw_prefill_workspace_size(shape, batch, h_new_lens, h_prefix_lens, num_cus, &inner);
    if (st != MW_OK) return st;
    if (!bytes) return fail(MW_ERR_INVALID_ARG, "%s: bytes is NULL", who);
    const FewPlan few = few_plan(batch, h_new_lens, h_prefix_lens, shape->num_kv_heads, shape->num_q_heads / shape->num_kv_heads);
    if (few.groups > 0) {
        *bytes = few.bytes;
        return MW_OK;
    }
    UnpackLayout u;
    st = unpack_layout(batch, h_new_lens, h_prefix_lens, shape->num_kv_heads, &u, who);
    if (st != MW_OK) return st;
    *bytes = u.pages > 0 ? u.off_ws + inner : 0;
    return MW_OK;
}

mw_status mw_kv4_prefill_attn(const mw_kv_pool *pool, const mw_attn_shape *shape, int32_t batch,
                              const int32_t *h_new_lens, const int32_t *h_prefix_lens, const int32_t *d_qo_indptr,
                              const int32_t *d_prefix_lens, const int32_t *d_block_table, int32_t bt_stride,
                              const void *d_q, void *d_out, void *d_workspace, size_t workspace_bytes, mw_stream stream,
                              mw_timing *timing) {
    const char *who = "mw_kv4_prefill_attn";
    int64_t max_n = 0, total = 0;
    mw_status st = check_rows(pool, batch, h_new_lens, h_prefix_lens, d_qo_indptr, d_prefix_lens, d_block_table,
                              bt_stride, &max_n, &total, who);
    if (st == MW_OK) st = check_pool_kind(pool, true, who);
    if (st == MW_OK && !shape) st = fail(MW_ERR_INVALID_ARG, "%s: bad arguments", who);
    if (st != MW_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t cus = stream_cus(s);
    mw_prefill_args a{pool,          *shape,        batch,         h_new_lens, h_prefix_lens, d_qo_indptr,
                      d_prefix_lens, d_block_table, bt_stride,     d_q,        d_out};
    PrefillPlan pl;
    st = prefill_prepare(&a, cus, true, &pl, who, true, true);
    if (st != MW_OK) return st;
    const FewPlan few = few_plan(batch, h_new_lens, h_prefix_lens, pl.hkv, pl.group);
    if (total == 0) {
        st = timing_begin(timing, s);
        if (st == MW_OK) st = timing_kernel_done(timing, s);
        timing_end(timing);
        return st;
    }
    if (few.groups > 0) {
        if (workspace_bytes < few.bytes || (few.bytes > 0 && (!d_workspace || !aligned16(d_workspace))))
            return fail(MW_ERR_INVALID_ARG, "%s: needs a 16-byte aligned workspace of %zu bytes (got %zu)", who, few.bytes,
                        workspace_bytes);
        float *ws = static_cast<float *>(d_workspace);
        const FewRows rows{ws, reinterpret_cast<float2 *>(ws + few.rows * kHeadDim), few.groups, few.block_rows, few.piece_tiles,
                           few.max_pieces};
        st = timing_begin(timing, s);
        if (st != MW_OK) return st;
        hipLaunchKernelGGL(k_kv4_prefill, dim3(static_cast<unsigned>(few.groups)), dim3(256), 0, s, pool->k4, pool->v4,
                           pool->scales, static_cast<const uint16_t *>(d_q), static_cast<uint16_t *>(d_out), d_qo_indptr,
                           d_prefix_lens, d_block_table, bt_stride, batch, Divisor(pl.hkv), Divisor(pl.group),
                           pool->desc.num_pages, pl.scale_log2, rows);
        st = check_launch("k_kv4_prefill");
        if (st == MW_OK) st = timing_kernel_done(timing, s);
        if (st == MW_OK && few.max_pieces > 1) {
            hipLaunchKernelGGL(k_kv4_merge, dim3(static_cast<unsigned>((max_n * shape->num_q_heads + 3) / 4), batch), dim3(256), 0,
                               s, static_cast<uint16_t *>(d_out), d_qo_indptr, d_prefix_lens, Divisor(pl.hkv),
                               Divisor(pl.group), rows);
            st = check_launch("k_kv4_merge");
            if (st == MW_OK) st = timing_kernel_done(timing, s);
        }
        timing_end(timing);
        return st;
    }
    UnpackLayout u;
    st = unpack_layout(batch, h_new_lens, h_prefix_lens, pl.hkv, &u, who);
    if (st != MW_OK) return st;
    if (!d_workspace || !aligned16(d_workspace) || workspace_bytes < u.off_ws)
        return fail(MW_ERR_INVALID_ARG, "%s: needs a 16-byte aligned workspace of %zu bytes and the attention's (got %zu)",
                    who, u.off_ws, workspace_bytes);
    char *ws = static_cast<char *>(d_workspace);
    // the unpacked pages, which the attention reads
    uint16_t *k = reinterpret_cast<uint16_t *>(ws), *v = reinterpret_cast<uint16_t *>(ws + u.off_v);
    uint16_t *bad = reinterpret_cast<uint16_t *>(ws + u.off_bad);
    int32_t *table = reinterpret_cast<int32_t *>(ws + u.off_table);
    a.d_block_table = table;
    a.bt_stride = static_cast<int32_t>(u.table_stride);
    a.d_workspace = ws + u.off_ws;
    a.workspace_bytes = workspace_bytes - u.off_ws;
    st = prefill_fit_workspace(&a, cus, &pl, a.d_workspace, a.workspace_bytes, who);
    if (st == MW_OK) st = timing_begin(timing, s);
    if (st != MW_OK) return st;
    const int64_t items = u.pages * pool->desc.num_kv_heads;
    hipLaunchKernelGGL(k_kv4_unpack, dim3(static_cast<unsigned>((items + 3) / 4)), dim3(256), 0, s, pool->k4, pool->v4,
                       pool->scales, k, v, bad, table, static_cast<int>(u.table_stride), d_qo_indptr, d_prefix_lens,
                       d_block_table, bt_stride, batch, pool->desc.num_pages, pool->desc.num_kv_heads, items);
    st = check_launch("k_kv4_unpack");
    if (st == MW_OK) st = timing_kernel_done(timing, s);
    if (st == MW_OK) st = prefill_launch(a, PrefillPages{k, v, static_cast<int>(u.pages)}, pl, s, timing);
    if (st != MW_OK) return st;
    hipLaunchKernelGGL(k_kv4_unseen, dim3(static_cast<unsigned>(pl.hkv), batch), dim3(256), 0, s, static_cast<uint16_t *>(d_out),
                       reinterpret_cast<const uint64_t *>(bad), table, static_cast<int>(u.table_stride),
                       static_cast<int>(u.pages), d_qo_indptr, d_prefix_lens, pl.group);
    st = check_launch("k_kv4_unseen");
    if (st == MW_OK) st = timing_kernel_done(timing, s);
    timing_end(timing);
    return st;
}

}  // extern "C"
