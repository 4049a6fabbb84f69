// Attention over the cache in 4 bits: decode, and prefill.
#include "decode_block.h"
#include "kv4_format.h"

using namespace mw;

namespace {

using namespace dk;
using namespace kv4;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------ decode
// The balanced split of decode_block.h (its units, shares, pieces and merge) on
// pages of 2176 bytes instead of 8192: per byte nearly four times the work, so
// the work is what the body is built around.  Nothing of a page passes through
// LDS or is converted but V:
//   * S^T[token][head] = K Q^T on the scaled 16x16x128 matrix instruction, K as
//     it lies in memory with its scale bytes (a page is one 16-byte load a lane),
//     Q^T as the sum of two e4m3 operands hi + lo: q 2^-e with e such that a row's
//     largest is in [128, 256), hi its nearest, lo the nearest of the rest.  hi keeps
//     four bits of the eight that bf16 has and the rest has four, so the sum is
//     exact down to 2^-10 of the row's largest, and off by at most 2^-18 of it
//     below.
//   * O^T[dim][head] += V^T P^T on the bf16 instruction, V^T a conversion of two
//     codes each (without scales: 32 conversions for two pages) and the scale of
//     (token, block of 32 dims) multiplied into P^T.  A tile of 16 dims has one
//     block, so P^T is needed once per block: with up to four query heads per kv
//     head the columns that they leave empty hold the other blocks (column 4 blk +
//     head), with up to eight two operands hold two blocks each, with sixteen four
//     one each; a tile's columns of other blocks are not used.
// kHeads: 4, 8 or 16, the most query heads of a kv head.
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

// Two bf16 values into half kHalf of hi and lo.
template <int kHalf>
__device__ __forceinline__ void split2(uint32_t two, float unit, i16x2 &hi, i16x2 &lo) {
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2_t, two), unit, kHalf);
    const auto near = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(__builtin_bit_cast(int, hi), unit, kHalf);
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, __builtin_bit_cast(float, two << 16) - near[0],
                                                  __builtin_bit_cast(float, two & 0xffff0000u) - near[1], unit, kHalf);
}

// hi and lo operands of a Q row and the factor of its scores; x[i]: the lane's
// dims 64 (i / 2) + 16 g + 8 (i % 2) .. +7 of its column's row.
__device__ __forceinline__ float split_q(const uint4 (&x)[4], i32x8 &hi, i32x8 &lo) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max2(max2(max2(most, abs2(x[i].x)), max2(abs2(x[i].y), abs2(x[i].z))), abs2(x[i].w));
    most = max(most & 0xffff, most >> 16);
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 16)));
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 32)));
    const int power = static_cast<int>(most >> 7);
    const int e = max(power - 127 - 7, -100);  // rows below 2^-93 keep fewer bits
    const float unit = __builtin_bit_cast(float, static_cast<uint32_t>(127 + e) << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            i16x2 h{0, 0}, l{0, 0};
            split2<0>(w[2 * j], unit, h, l);
            split2<1>(w[2 * j + 1], unit, h, l);
            hi[2 * i + j] = __builtin_bit_cast(int, h);
            lo[2 * i + j] = __builtin_bit_cast(int, l);
        }
    }
    // a row that is not finite: NaN scores
    return power == 255 ? NAN : unit;
}

// Weighted sum of the fragments or pieces of one head in a wave: (m, l) of up to
// 64 of them one per lane, which gives every weight 2^(m - M) and the denominator
// within the wave, then two outputs per lane.  Those without keys have l = 0 and
// contribute nothing.  load_o(j): the lane's two values of the j-th, j < n.
struct HeadSum {
    float M = -INFINITY, L = 0.f;
    float2 acc = make_float2(0.f, 0.f);
    template <class LoadO>
    __device__ __forceinline__ void add(float2 ml, int n, int lane, const LoadO &load_o) {
        const bool in = lane < n && ml.y != 0.f;
        const float top = fmaxf(M, wave_max(in ? ml.x : -INFINITY));
        const float old = L == 0.f ? 0.f : __builtin_amdgcn_exp2f(M - top);
        const float w = in ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
        M = top;
        L = L * old + wave_sum(in ? w * ml.y : 0.f);
        acc.x *= old;
        acc.y *= old;
#pragma unroll 1
        for (int j0 = 0; j0 < n; j0 += 8) {
            float2 o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = load_o(min(j0 + k, n - 1));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                // lanes from n on have weight 0, and j0 + k < 64
                const float wk = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), j0 + k));
                acc.x += wk * o[k].x;
                acc.y += wk * o[k].y;
            }
        }
    }
};

// The end of a unit, after the barrier behind its waves' shares: as
// add_up_fragments and finish_segments of the bf16 cache (the same pieces, slots
// and flags), a head at a time per wave, the heads of several runs of fragments,
// and of both segments that are merged, side by side.
template <int kHeads>
__device__ __forceinline__ void
finish_unit(uint16_t *__restrict__ out, float *__restrict__ ws_o, float2 *__restrict__ ws_ml,
            uint32_t *__restrict__ flags, uint32_t tag, int64_t slots, int hkv, int group, bool aligned, int u, int tid,
            Span4Lds<kHeads> &lds) {
    constexpr int kRecords = Span4Lds<kHeads>::kRecords;
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
        while (!(ends_at >> j & 1) && (j | 1) + 1 < kRecords && (valid >> ((j | 1) + 1) & 1)) {
            j = (j | 1) + 1;
            ++n;
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
            s.add(ml, n, lane, [&](int k) __attribute__((always_inline)) {
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
    SpanShare walk{seq_lens, bt, bt_stride, batch, hkv, per_unit, total, aligned, u, wave, lane};
    using Chunk = SpanShare::Chunk;
    const bool in_group = head < group;

    i32x8 q_hi, q_lo;
    float q_scale = 0.f;
    uint4 q_next[4];  // the next fragment's rows, on their way since its chunk is known
    auto load_q = [&](const Chunk &c) __attribute__((always_inline)) {
        const uint16_t *qp = q + (static_cast<size_t>(c.b) * hq + c.kvh * group + (in_group ? head : 0)) * kHeadDim + 16 * grp;
#pragma unroll
        for (int i = 0; i < 4; ++i) q_next[i] = *reinterpret_cast<const uint4 *>(qp + 64 * (i >> 1) + 8 * (i & 1));
    };
    auto take_q = [&]() __attribute__((always_inline)) {
        // (above 0, or a masked score would be a NaN; of a NaN row, NaN)
        const float f = split_q(q_next, q_hi, q_lo) * scale_log2;
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
                    sc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q_hi, f32x4{0.f, 0.f, 0.f, 0.f}, 4, 0, 0, s, 0, 127);
                    sc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q_lo, sc[j], 4, 0, 0, s, 0, 127);
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

// ----------------------------------------------------------------- prefill
// Unpacks the pages of a batch's sequences, laid end to end, to bf16 pages
// [page][kv head][16][128] and writes the table that names them.  One wave to a
// (page, kv head).
struct ChunkLengths {
    const int32_t *indptr, *prefix;
    int batch, bt_stride;
    __device__ __forceinline__ int pages(int b) const {
        if (b >= batch) return 0;
        const int64_t len = static_cast<int64_t>(indptr[b + 1]) - indptr[b] + prefix[b];
        const int64_t np = (len + kPageSize - 1) / kPageSize;
        return static_cast<int>(max(int64_t{0}, min(np, static_cast<int64_t>(bt_stride))));
    }
};

__global__ void __launch_bounds__(256)
k_kv4_unpack(const uint8_t *__restrict__ kpool, const uint8_t *__restrict__ vpool, const uint8_t *__restrict__ scales,
             uint16_t *__restrict__ kout, uint16_t *__restrict__ vout, int32_t *__restrict__ table, int table_stride,
             const int32_t *__restrict__ indptr, const int32_t *__restrict__ prefix, const int32_t *__restrict__ bt,
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
    const uint32_t codes[kBlocks] = {vc.x, vc.y, vc.z, vc.w};
    decode_v(codes, bytes, vr);
    uint32_t *vo = reinterpret_cast<uint32_t *>(vout + static_cast<size_t>(item) * (kPageSize * kHeadDim)) + c;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) vo[(4 * g + t) * (kHeadDim / 2) + 16 * k] = vr[t][k];
}

// Workspace of a prefill call: K pages, V pages, their table, then the
// workspace of the attention itself.
struct UnpackLayout {
    int64_t pages;
    int64_t table_stride;
    size_t off_v, off_table, off_ws;
};
mw_status unpack_layout(int32_t batch, const int32_t *h_new_lens, const int32_t *h_prefix_lens, int64_t hkv,
                        UnpackLayout *u, const char *who) {
    u->pages = 0;
    u->table_stride = 1;
    for (int32_t b = 0; b < batch; ++b) {
        const int64_t np = (static_cast<int64_t>(h_new_lens[b]) + h_prefix_lens[b] + kPageSize - 1) / kPageSize;
        u->pages += np;
        u->table_stride = np > u->table_stride ? np : u->table_stride;
    }
    if (u->pages > INT32_MAX || u->pages * hkv > static_cast<int64_t>(INT32_MAX) * 4)
        return fail(MW_ERR_UNSUPPORTED, "%s: too many pages", who);
    const size_t pages_bytes = static_cast<size_t>(u->pages) * hkv * (kPageSize * kHeadDim * 2);
    u->off_v = pages_bytes;
    u->off_table = 2 * pages_bytes;
    u->off_ws = (u->off_table + static_cast<size_t>(batch) * u->table_stride * 4 + 255) & ~static_cast<size_t>(255);
    return MW_OK;
}

}  // namespace

extern "C" {

mw_status mw_kv4_decode_workspace_size(const mw_attn_shape *shape, int32_t batch, const int32_t *h_seq_lens,
                                       size_t *bytes) {
    return mw_decode_workspace_size(shape, batch, h_seq_lens, 0, bytes);
}

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

mw_status mw_kv4_prefill_workspace_size(const mw_attn_shape *shape, int32_t batch, const int32_t *h_new_lens,
                                        const int32_t *h_prefix_lens, int32_t num_cus, size_t *bytes) {
    const char *who = "mw_kv4_prefill_workspace_size";
    size_t inner = 0;
    mw_status st = mw_prefill_workspace_size(shape, batch, h_new_lens, h_prefix_lens, num_cus, &inner);
    if (st != MW_OK) return st;
    if (!bytes) return fail(MW_ERR_INVALID_ARG, "%s: bytes is NULL", who);
    UnpackLayout u;
    st = unpack_layout(batch, h_new_lens, h_prefix_lens, shape->num_kv_heads, &u, who);
    if (st != MW_OK) return st;
    *bytes = u.off_ws + inner;
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
    UnpackLayout u;
    st = unpack_layout(batch, h_new_lens, h_prefix_lens, pool->desc.num_kv_heads, &u, who);
    if (st != MW_OK) return st;
    if (total > 0 && (!d_workspace || !aligned16(d_workspace) || workspace_bytes < u.off_ws))
        return fail(MW_ERR_INVALID_ARG, "%s: needs a 16-byte aligned workspace of %zu bytes and the attention's (got %zu)",
                    who, u.off_ws, workspace_bytes);
    char *ws = static_cast<char *>(d_workspace);
    // the unpacked pages, as the pool that the attention reads
    mw_kv_pool bf16{};
    bf16.desc = pool->desc;
    bf16.desc.num_pages = static_cast<int32_t>(u.pages > 0 ? u.pages : 1);
    bf16.k = reinterpret_cast<uint16_t *>(ws);
    bf16.v = reinterpret_cast<uint16_t *>(ws + u.off_v);
    int32_t *table = reinterpret_cast<int32_t *>(ws + u.off_table);
    const size_t left = total > 0 ? workspace_bytes - u.off_ws : 0;
    const mw_prefill_args a{&bf16,       *shape,        batch, h_new_lens,
                            h_prefix_lens, d_qo_indptr, d_prefix_lens, table,
                            static_cast<int32_t>(u.table_stride), d_q, d_out, ws + u.off_ws, left};
    PrefillPlan pl;
    const int64_t cus = stream_cus(s);
    st = prefill_prepare(&a, cus, true, &pl, who, true);
    if (st == MW_OK) st = prefill_fit_workspace(&a, cus, &pl, ws + u.off_ws, left, who);
    if (st == MW_OK) st = timing_begin(timing, s);
    if (st != MW_OK) return st;
    if (total == 0) return prefill_launch(a, pl, s, timing);
    const int64_t items = u.pages * pool->desc.num_kv_heads;
    hipLaunchKernelGGL(k_kv4_unpack, dim3(static_cast<unsigned>((items + 3) / 4)), dim3(256), 0, s, pool->k4, pool->v4,
                       pool->scales, bf16.k, bf16.v, table, static_cast<int>(u.table_stride), d_qo_indptr, d_prefix_lens,
                       d_block_table, bt_stride, batch, pool->desc.num_pages, pool->desc.num_kv_heads, items);
    st = check_launch("k_kv4_unpack");
    if (st == MW_OK) st = timing_kernel_done(timing, s);
    if (st != MW_OK) return st;
    return prefill_launch(a, pl, s, timing);
}

}  // extern "C"
