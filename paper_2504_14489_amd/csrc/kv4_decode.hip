// Decode attention over the cache in 4 bits.
#include "kv4_block.h"

using namespace mw;

namespace {

using namespace dk;
using namespace kv4;

// The balanced split of decode_block.h (its units, shares, pieces and merge) on
// pages of 2176 bytes instead of 8192: per byte nearly four times the work, so
// the work is what the body is built around.  Nothing of a page passes through
// LDS or is converted but V:
//   * S^T[token][head] = K Q^T on the scaled 16x16x128 matrix instruction, K as
//     it lies in memory with its scale bytes (a page is one 16-byte load a lane),
//     Q^T as the sum of two e4m3 operands (kv4_block.h).
//   * O^T[dim][head] += V^T P^T on the bf16 instruction, V^T a conversion of two
//     codes each (without scales: 32 conversions for two pages) and the scale of
//     (token, block of 32 dims) multiplied into P^T.  A tile of 16 dims has one
//     block, so P^T is needed once per block: with up to four query heads per kv
//     head the columns that they leave empty hold the other blocks (column 4 blk +
//     head), with up to eight two operands hold two blocks each, with sixteen four
//     one each; a tile's columns of other blocks are not used.
// kHeads: 4, 8 or 16, the most query heads of a kv head.
//
// Measured: 32 sequences of 16K to 32K tokens of 8 kv heads, 843 MB, 131.6 us (6.4 TB/s;
// a plain read reaches 6.5), where memory bounds it.  64 of 512 to 4096, 141 MB, 31.7,
// and 128 of 64 to 16K of one kv head with 8 query heads, 29 MB, 14.6: a CU's waves
// issue a page in 0.061 us, and 8 to 10 us pass in a start (lengths, table, pages:
// dependent loads) and an end (pieces, flags, merge) on which nothing else waits.
// One of 4003 tokens, 4.4 MB, takes 9.3 and has little else.  On 192, 128, 64 and 32 CUs
// the first takes 152, 201, 381 and 748 us (0.061 us a page of a CU on the last two) and
// the second 39, 48, 82 and 149.  With 16 query heads a kv head, 32 of 16K to 32K of 8 kv
// heads take 161 us (5.3 TB/s; 252 on 128 CUs) and 64 of 512 to 4096 of one 15.2.
//
// A unit has eight waves, with steps of four pages: sixteen with steps of two (128
// registers, the scores' bookkeeping twice as often) took 41 us for 32 sequences
// of 4096 tokens of 8 kv heads instead of 28, and 16.8 instead of 13 for one of 4003.
constexpr int kStep = 4;  // pages of a wave's step
// What the waves leave for the end of a unit: record 2 wave + i is the wave's
// first (0) or last (1) fragment.
template <int kHeads>
struct Span4Lds {
    static constexpr int kRecords = 2 * kSpanWaves;
    float o[kRecords][kHeads][OSTR];
    float2 ml[kRecords][kHeads];
    Fragment frag[kRecords];
    int done[2];  // the pending segments' pieces are all done
};

// The end of a unit, after the barrier behind its waves' shares: as
// add_up_fragments and finish_segments of the bf16 cache (the same pieces, slots
// and flags), a head at a time per wave, the heads of several runs of fragments,
// and of both segments that are merged, side by side.  (Flags for each head, so that
// no wave waits for another, made the merge of a sequence of 4003 tokens 1 us longer:
// many waves see all flags and merge the same.)
template <int kHeads>
__device__ __forceinline__ void
finish_unit(uint16_t *__restrict__ out, float *__restrict__ ws_o, float2 *__restrict__ ws_ml,
            uint32_t *__restrict__ flags, uint32_t tag, int64_t slots, int hkv, int group, bool aligned, int u, int tid,
            Span4Lds<kHeads> &lds) {
    constexpr int kRecords = Span4Lds<kHeads>::kRecords;
    constexpr uint32_t kFirst = 0x5555;  // the records of first fragments
    static_assert(kRecords == 16);
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const auto write = [&](int b, int kvh, int h, const HeadSum &s) __attribute__((always_inline)) {
        const float inv = 1.f / s.L;
        reinterpret_cast<uint32_t *>(out + (static_cast<size_t>(b) * hkv * group + kvh * group + h) * kHeadDim)[lane] =
            cvt2(s.acc.x * inv, s.acc.y * inv);
    };
    const Fragment fr = lds.frag[lane & (kRecords - 1)];
    const bool mine = lane < kRecords && fr.seg >= 0;
    uint32_t todo = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(mine));
    const uint32_t valid = todo, starts_at = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(mine && fr.starts)),
                   ends_at = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(mine && fr.ends));
    Pending pend{};
    int turn = wave;  // the wave's head of the next run
#pragma unroll 1
    while (todo) {
        // the run: record i and the first fragments of the waves after it
        const int i = __builtin_ctz(todo), w = i >> 1;
        int j = i, n = 1;
        if (!(ends_at >> i & 1)) {
            // up to the first that ends the segment, or the one before the first that is
            // not there
            const int next = (i | 1) + 1;
            const uint32_t later = kFirst & ~((1u << next) - 1);
            const int gap = __builtin_ctz((~valid & later) | 1u << kRecords), end = __builtin_ctz((ends_at & later) | 1u << 31);
            const int last = min(gap - 2, end);
            if (last >= next) {
                j = last;
                n = 2 + (last - next) / 2;
            }
        }
        todo &= ~((2u << j) - 1);
        const bool whole = (starts_at >> i & 1) && (ends_at >> j & 1);
        const int sb = __builtin_amdgcn_readlane(fr.b, i), skvh = __builtin_amdgcn_readlane(fr.kvh, i);
        const int64_t shift = aligned ? 0 : __builtin_amdgcn_readlane(fr.seg, i);  // of the workspace slots
        const int64_t piece = u + shift;
#pragma unroll 1
        for (int h = turn & (kSpanWaves - 1); h < group; h += kSpanWaves) {
            HeadSum s;
            const float2 ml = lds.ml[lane == 0 ? i : min(2 * (w + lane), kRecords - 1)][h];
            s.add(ml, n, lane, [&](int k) __attribute__((always_inline)) {
                return reinterpret_cast<const float2 *>(lds.o[k == 0 ? i : 2 * (w + k)][h])[lane];
            });
            if (whole) {
                write(sb, skvh, h, s);
            } else if (piece < slots) {
                // device-scope stores (through the L2 of this XCD): the piece may be
                // merged by a work-group on another XCD without a cache writeback
                const size_t at = static_cast<size_t>(piece) * group + h;
                __hip_atomic_store(reinterpret_cast<unsigned long long *>(ws_o + at * kHeadDim) + lane,
                                   __builtin_bit_cast(unsigned long long, s.acc), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (lane == 0)
                    __hip_atomic_store(reinterpret_cast<unsigned long long *>(ws_ml + at),
                                       __builtin_bit_cast(unsigned long long, make_float2(s.M, s.L)), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        turn += kSpanWaves - (group & (kSpanWaves - 1));
        if (!whole) {
            const Pending::Piece pc{sb, skvh, __builtin_amdgcn_readlane(fr.nch, i), __builtin_amdgcn_readlane(fr.u0, i) + shift, piece};
            if (pend.n == 0)
                pend.p0 = pc;
            else
                pend.p1 = pc;
            pend.n = pend.n == 0 ? 1 : 2;
        }
    }
    if (pend.n == 0) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's piece stores are complete
    __syncthreads();
    // device lengths that disagree with the host's must not lead outside the
    // workspace
    const auto in_workspace = [&](const Pending::Piece &p) {
        return p.first >= 0 && p.first + p.nch - 1 < slots && p.self < slots;
    };
    const bool ok0 = in_workspace(pend.p0), ok1 = pend.n > 1 && in_workspace(pend.p1);
    if (tid == 0) {
        if (ok0) __hip_atomic_store(flags + pend.p0.self, tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (ok1) __hip_atomic_store(flags + pend.p1.self, tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        lds.done[0] = ok0;
        lds.done[1] = ok1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __syncthreads();
    // both segments' flags in one round of loads, half of the waves each
    const int second = wave / (kSpanWaves / 2);
    if (second ? ok1 : ok0) {
        const Pending::Piece &p = second ? pend.p1 : pend.p0;
        bool all = true;
        for (int j = tid & (kSpanThreads / 2 - 1); j < p.nch; j += kSpanThreads / 2)
            all = all && __hip_atomic_load(flags + p.first + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == tag;
        if (!all) lds.done[second] = 0;
    }
    __syncthreads();
    // the heads of what is done, over the waves
    const int n0 = __builtin_amdgcn_readfirstlane(lds.done[0]) ? group : 0;
    const int n1 = __builtin_amdgcn_readfirstlane(lds.done[1]) ? group : 0;
#pragma unroll 1
    for (int t = wave; t < n0 + n1; t += kSpanWaves) {
        const Pending::Piece p = t < n0 ? pend.p0 : pend.p1;
        const int h = t < n0 ? t : t - n0;
        HeadSum s;
        const unsigned long long *ml_src = reinterpret_cast<const unsigned long long *>(ws_ml) + p.first * group + h;
        const unsigned long long *o_src =
            reinterpret_cast<const unsigned long long *>(ws_o) + (p.first * group + h) * (kHeadDim / 2) + lane;
        const int step = group * (kHeadDim / 2);
#pragma unroll 1
        for (int jb = 0; jb < p.nch; jb += 64) {
            const int n = min(p.nch - jb, 64);
            const float2 ml = __builtin_bit_cast(
                float2, __hip_atomic_load(ml_src + (jb + min(lane, n - 1)) * group, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
            s.add<2>(ml, n, lane, [&](int k) __attribute__((always_inline)) {
                return __builtin_bit_cast(float2, __hip_atomic_load(o_src + static_cast<int64_t>(jb + k) * step, __ATOMIC_RELAXED,
                                                                    __HIP_MEMORY_SCOPE_AGENT));
            });
        }
        write(p.b, p.kvh, h, s);
        // a merged segment's flags are cleared, for a replay of this launch
        if (h == 0)
            for (int j = lane; j < p.nch; j += 64)
                __hip_atomic_store(flags + p.first + j, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

__device__ __forceinline__ bf16x8 v_operand(uint4 a, uint4 b, int t) {
    const uint32_t p = t < 2 ? a.x : t < 4 ? a.y : t < 6 ? a.z : a.w, q = t < 2 ? b.x : t < 4 ? b.y : t < 6 ? b.z : b.w;
    const uint4 r = t & 1 ? make_uint4(decode2<2>(p, 1.f), decode2<3>(p, 1.f), decode2<2>(q, 1.f), decode2<3>(q, 1.f))
                          : make_uint4(decode2<0>(p, 1.f), decode2<1>(p, 1.f), decode2<0>(q, 1.f), decode2<1>(q, 1.f));
    return __builtin_bit_cast(bf16x8, r);
}

template <int kHeads>
__global__ void __launch_bounds__(kSpanThreads)
k_kv4_decode(const uint8_t *__restrict__ kpool, const uint8_t *__restrict__ vpool, const uint8_t *__restrict__ scales,
             const uint16_t *__restrict__ q, uint16_t *__restrict__ out, const int32_t *__restrict__ seq_lens,
             const int32_t *__restrict__ bt, int bt_stride, float *__restrict__ ws_o, float2 *__restrict__ ws_ml,
             uint32_t *__restrict__ flags, uint32_t tag, int64_t slots, int batch, int hkv, int group, int num_pages,
             float scale_log2, int per_unit, int total, int aligned_) {
    constexpr int kOps = kHeads / 4;          // P^T operands: blocks 4 / kOps in each
    constexpr int kPerOp = kBlocks / kOps;    // blocks side by side in the columns
    __shared__ __attribute__((aligned(16))) Span4Lds<kHeads> lds;
    const bool aligned = aligned_ != 0;
    const int u = blockIdx.x, tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int head = col & (kHeads - 1), side = col / kHeads;  // side: which of an operand's blocks
    const int hq = hkv * group, align = aligned ? per_unit : 0;
    SpanShare<kStep> walk{seq_lens, bt, bt_stride, batch, hkv, per_unit, total, aligned, u, wave, lane};
    using Chunk = SpanShare<kStep>::Chunk;
    const bool in_group = head < group;

    i32x8 q_hi[1], q_lo[1];
    float q_scale = 0.f;
    uint4 q_next[4];  // the next fragment's rows, on their way since its chunk is known
    auto load_q = [&](const Chunk &c) __attribute__((always_inline)) {
        const uint16_t *qp = q + (static_cast<size_t>(c.b) * hq + c.kvh * group + (in_group ? head : 0)) * kHeadDim + 16 * grp;
#pragma unroll
        for (int i = 0; i < 4; ++i) q_next[i] = *reinterpret_cast<const uint4 *>(qp + 64 * (i >> 1) + 8 * (i & 1));
    };
    auto take_q = [&]() __attribute__((always_inline)) {
        // (above 0, or a masked score would be a NaN; of a NaN row, NaN)
        const float f = split_q<true>(q_next, q_hi, q_lo) * scale_log2;
        q_scale = f < 1e-37f ? 1e-37f : f;
    };

    // a step's pages: K codes of key lane%16, block lane/16, and that scale byte;
    // V codes of this lane's rows and tokens 4 grp .. +3, and those tokens' scale
    // bytes of the lane's blocks
    uint4 kr[kStep], vr[kStep];
    uint32_t ks[kStep], vs[kStep][kOps];
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
        kr[j] = vr[j] = make_uint4(0, 0, 0, 0);
        ks[j] = 0;
#pragma unroll
        for (int o = 0; o < kOps; ++o) vs[j][o] = 0;
    }
    int step_ok = 0;  // bit j: page j of it exists
    uint32_t at[kStep];
    auto step_pages = [&](const Chunk &c, int tbl, int p) __attribute__((always_inline)) {
        step_ok = 0;
#pragma unroll
        for (int j = 0; j < kStep; ++j) {
            const int page = __builtin_amdgcn_readlane(tbl, min(p + j, c.p_end - 1) - c.p);
            const bool ok = p + j < c.p_end && page >= 0 && page < num_pages;
            step_ok |= ok ? 1 << j : 0;
            at[j] = static_cast<uint32_t>((ok ? page : 0) * hkv + c.kvh);
        }
    };
    auto load_k = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kStep; ++j)
            if (step_ok >> j & 1) {
                kr[j] = load_stream(reinterpret_cast<const uint16_t *>(kpool + static_cast<size_t>(at[j]) * kCodeBytes + col * 64 + grp * 16));
                ks[j] = scales[static_cast<size_t>(at[j]) * kScaleBytes + lane];
            }
    };
    auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kStep; ++j)
            if (step_ok >> j & 1) {
                vr[j] = load_stream(reinterpret_cast<const uint16_t *>(vpool + static_cast<size_t>(at[j]) * kCodeBytes + lane * 16));
                const uint8_t *sc = scales + static_cast<size_t>(at[j]) * kScaleBytes + kBlocks * kPageSize + 4 * grp;
#pragma unroll
                for (int o = 0; o < kOps; ++o)
                    vs[j][o] = *reinterpret_cast<const uint32_t *>(sc + (o * kPerOp + side) * kPageSize);
            }
    };

    f32x4 oacc[8];  // O^T[dim 32 (t/2) + 2 (4grp + i) + t%2][col]
    float m_run = -INFINITY, l_run = 0.f;
    auto reset = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 8; ++t) oacc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run = in_group ? -INFINITY : INFINITY;
        l_run = 0.f;
    };
    // the eight dims 32 blk + 8 grp .. +7 of the lane's block of operand o
    auto outputs = [&](int o, float (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v = oacc[2 * o * kPerOp + e][i];
#pragma unroll
                for (int s = 1; s < kPerOp; ++s) v = side == s ? oacc[2 * (o * kPerOp + s) + e][i] : v;
                x[2 * i + e] = v;
            }
    };
    if (lane < 2) lds.frag[2 * wave + lane].seg = -1;

    Chunk cur = walk.next();
    if (cur.valid) {
        int tbl = walk.table(cur);
        load_q(cur);
        reset();
        int frag_p = cur.p;  // first page of the fragment
        Chunk nxt = walk.next();
        int tbl_n = nxt.valid ? walk.table(nxt) : 0;
        step_pages(cur, tbl, cur.p);
        load_k();
        load_v();
        take_q();
        for (;;) {
            const bool frag_end = !nxt.valid || nxt.b != cur.b || nxt.kvh != cur.kvh;
            // its queries are on their way since the next fragment's chunk is known
            if (frag_end && nxt.valid) load_q(nxt);
            for (int p = cur.p; p < cur.p_end; p += kStep) {
                const int ok = step_ok;
                // a step with a missing page, or past the sequence's end
                const bool edge = ok != (1 << kStep) - 1 || (p + kStep) * kPageSize > cur.len;
                f32x4 sc[kStep];
#pragma unroll
                for (int j = 0; j < kStep; ++j) {
                    const i32x8 a{static_cast<int>(kr[j].x), static_cast<int>(kr[j].y), static_cast<int>(kr[j].z),
                                  static_cast<int>(kr[j].w), 0, 0, 0, 0};
                    const int s = static_cast<int>(ks[j]);
                    // A: four-bit floats with their scales; B: e4m3 with scale 1
                    sc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q_hi[0], f32x4{0.f, 0.f, 0.f, 0.f}, 4, 0, 0, s, 0, 127);
                    sc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q_lo[0], sc[j], 4, 0, 0, s, 0, 127);
                }
                // the next step's K loads go out while this one is computed, its V
                // loads once this one's V is used
                const bool last = p + kStep >= cur.p_end;
                const bool more = !last || nxt.valid;
                if (more) {
                    step_pages(last ? nxt : cur, last ? tbl_n : tbl, last ? nxt.p : p + kStep);
                    load_k();
                }
                if (edge) {
                    // scores of keys on an absent page or past the sequence's end are
                    // masked, and their V scales are zeros (a masked key has p = 0,
                    // but 0 times the infinite scale of a slack slot would not be 0)
#pragma unroll
                    for (int j = 0; j < kStep; ++j) {
                        const int seen = (ok >> j & 1) ? cur.len - (p + j) * kPageSize - 4 * grp : 0;  // of the lane's four
#pragma unroll
                        for (int i = 0; i < 4; ++i) sc[j][i] = i < seen ? sc[j][i] : -INFINITY;
                        const uint32_t mask = seen >= 4 ? ~0u : seen <= 0 ? 0u : (1u << 8 * seen) - 1;
#pragma unroll
                        for (int o = 0; o < kOps; ++o) vs[j][o] &= mask;
                    }
                }
                float mx = -INFINITY;
#pragma unroll
                for (int j = 0; j < kStep; ++j) mx = max4(mx, sc[j]);
                mx = across(mx, [](float a, float b) { return __builtin_elementwise_maximum(a, b); }) * q_scale;
                if (__builtin_amdgcn_ballot_w64(mx > m_run + kRescaleLog2) != 0) {
                    const float m_new = fmaxf(m_run, mx);
                    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
                    m_run = m_new;
                    l_run *= alpha;
#pragma unroll
                    for (int t = 0; t < 8; ++t) oacc[t] *= alpha;
                }
#pragma unroll
                for (int j = 0; j < kStep; ++j) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[j][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j][i], q_scale, -m_run));
                    l_run += (sc[j][0] + sc[j][1]) + (sc[j][2] + sc[j][3]);
                }
                // P^T operands of two pages: k-slot e < 4 is token 4grp + e of the
                // first, e >= 4 token 4grp + e - 4 of the second, as in V's layout.
                // bf16, as in the bf16 cache's kernels (a scale is a power of two, so
                // the rounding is that of p)
#pragma unroll
                for (int j = 0; j < kStep; j += 2)
#pragma unroll
                    for (int o = 0; o < kOps; ++o) {
                        float w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            w[i] = sc[j + i / 4][i % 4] * scale_of(vs[j + i / 4][o] >> (8 * (i % 4)) & 255);
                        const bf16x8 pop = __builtin_bit_cast(
                            bf16x8, make_uint4(cvt2(w[0], w[1]), cvt2(w[2], w[3]), cvt2(w[4], w[5]), cvt2(w[6], w[7])));
#pragma unroll
                        for (int t = 2 * o * kPerOp; t < 2 * (o + 1) * kPerOp; ++t)
                            oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_operand(vr[j], vr[j + 1], t), pop, oacc[t], 0, 0, 0);
                    }
                if (more) load_v();
            }
            if (frag_end) {
                l_run = across(l_run, [](float a, float b) { return a + b; });
                const bool starts = frag_p == 0, ends = cur.p_end == cur.np;
                const bool whole = starts && ends;
                // only the share's first fragment continues an earlier page
                const int rec = 2 * wave + (starts ? 1 : 0);
                const float inv = 1.f / l_run;
                uint16_t *orow = out + (static_cast<size_t>(cur.b) * hq + cur.kvh * group + head) * kHeadDim + 32 * side + 8 * grp;
                float *so = &lds.o[rec][head][32 * side + 8 * grp];
#pragma unroll
                for (int o = 0; o < kOps; ++o) {
                    float x[8];
                    outputs(o, x);
                    if (in_group) {
                        if (whole) {
                            *reinterpret_cast<uint4 *>(orow + 32 * o * kPerOp) =
                                make_uint4(cvt2(x[0] * inv, x[1] * inv), cvt2(x[2] * inv, x[3] * inv),
                                           cvt2(x[4] * inv, x[5] * inv), cvt2(x[6] * inv, x[7] * inv));
                        } else {
                            *reinterpret_cast<f32x4 *>(so + 32 * o * kPerOp) = f32x4{x[0], x[1], x[2], x[3]};
                            *reinterpret_cast<f32x4 *>(so + 32 * o * kPerOp + 4) = f32x4{x[4], x[5], x[6], x[7]};
                        }
                    }
                }
                if (!whole) {
                    if (grp == 0 && side == 0) lds.ml[rec][head] = make_float2(m_run, l_run);
                    const int extent = aligned ? (cur.np + align - 1) / align * align : cur.np;
                    const int f0 = cur.first / per_unit, f1 = (cur.first + extent - 1) / per_unit;
                    if (lane == 0)
                        lds.frag[rec] = Fragment{cur.b * hkv + cur.kvh, cur.b, cur.kvh, starts, ends, f0, f1 - f0 + 1, 0};
                }
                if (!nxt.valid) break;
                take_q();
                reset();
                frag_p = nxt.p;
            }
            cur = nxt;
            tbl = tbl_n;
            nxt = walk.next();
            if (nxt.valid) tbl_n = walk.table(nxt);
        }
    }
    __syncthreads();
    finish_unit<kHeads>(out, ws_o, ws_ml, flags, tag, slots, hkv, group, aligned, u, tid, lds);
}

}  // namespace

extern "C" {

mw_status mw_kv4_decode_attn(const mw_kv_pool *pool, const mw_attn_shape *shape, int32_t batch,
                             const int32_t *h_seq_lens, const int32_t *d_seq_lens, const int32_t *d_block_table,
                             int32_t bt_stride, const void *d_q, void *d_out, void *d_workspace, size_t workspace_bytes,
                             mw_stream stream, mw_timing *timing) {
    const char *who = "mw_kv4_decode_attn";
    if (!shape) return fail(MW_ERR_INVALID_ARG, "%s: bad arguments", who);
    const mw_decode_args a{pool,      *shape, batch, h_seq_lens,  d_seq_lens,      d_block_table,
                           bt_stride, d_q,    d_out, d_workspace, workspace_bytes, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    DecodePlan pl;
    mw_status st = decode_prepare(&a, stream_cus(s), &pl, who, true);
    if (st != MW_OK) return st;
    st = timing_begin(timing, s);
    if (st != MW_OK) return st;
    if (pl.units > 0) {
        char *ws = static_cast<char *>(d_workspace);
        auto kernel = pl.group <= 4 ? k_kv4_decode<4> : pl.group <= 8 ? k_kv4_decode<8> : k_kv4_decode<16>;
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(pl.units)), dim3(kSpanThreads), 0, s, pool->k4, pool->v4,
                           pool->scales, static_cast<const uint16_t *>(d_q), static_cast<uint16_t *>(d_out), d_seq_lens,
                           d_block_table, bt_stride, reinterpret_cast<float *>(ws),
                           reinterpret_cast<float2 *>(ws + pl.off_ml), reinterpret_cast<uint32_t *>(ws + pl.off_meta),
                           next_decode_tag(), pl.slots, batch, pl.hkv, pl.group, pool->desc.num_pages, pl.scale_log2,
                           static_cast<int>(pl.per_unit), static_cast<int>(pl.total), pl.aligned ? 1 : 0);
        st = check_launch("k_kv4_decode");
        if (st != MW_OK) return st;
    }
    st = timing_kernel_done(timing, s);
    timing_end(timing);
    return st;
}

}  // extern "C"
