"""The KV pool in 4 bits on the GPU: append, read-back, decode and prefill, against the format's definition and the
fp64 oracle on the values that the codes stand for."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_14489_amd import mw
from paper_2504_14489_amd.device import Partition, bits_to_f32
from paper_2504_14489_amd.workloads import f32_to_bf16_bits
from tests import kv4_reference as R
from tests.helpers import say

pytestmark = pytest.mark.gpu

SCALE = 128 ** -0.5


def normal_bits(rng, *shape, gain=1.0):
    return f32_to_bf16_bits((gain * rng.standard_normal(shape)).astype(np.float32))


def rows(lens):
    return R.device(np.concatenate([[0], np.cumsum(lens)]), np.int32)


class Append:
    """A batch of appended rows and the pool's expected bytes after it."""

    def __init__(self, hkv, lens, starts, seed, bits=None, table=None):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.lens, self.starts = np.array(lens, np.int32), np.array(starts, np.int32)
        self.table, pages = R.tables([n + s for n, s in zip(lens, starts)], rng, spare=2)
        if table is not None:
            self.table = table(self.table)
        self.pool = R.Pool4(pages, hkv, seed + 1)
        total = int(sum(lens))
        self.k = normal_bits(rng, total, hkv, 128) if bits is None else bits
        self.v = normal_bits(rng, total, hkv, 128) if bits is None else bits[..., ::-1].copy()
        self.dk, self.dv = R.device(self.k.view(np.int16)), R.device(self.v.view(np.int16))
        self.dtable, self.dstart, self.indptr = R.device(self.table), R.device(self.starts), rows(lens)

    def args(self):
        return (self.lens, self.starts, self.indptr.data_ptr(), self.dstart.data_ptr(), self.dtable.data_ptr(),
                self.table.shape[1])

    def write(self, stream=0):
        mw.mw_kv4_pool_write(self.pool.handle, *self.args(), self.dk.data_ptr(), self.dv.data_ptr(), stream)

    def expect(self):
        """Puts the rows' codes where they belong, in the reference pool."""
        p, row = self.pool, 0
        kc, ks = R.quantise(self.k)
        vc, vs = R.quantise(self.v)
        for b, (n, s) in enumerate(zip(self.lens, self.starts)):
            for i in range(n):
                page = self.table[b, (s + i) // 16]
                if 0 <= page < p.pages:
                    slot = (s + i) % 16
                    p.kc[page, :, slot], p.ks[page, :, slot] = kc[row], ks[row]
                    p.vc[page, :, slot], p.vs[page, :, slot] = vc[row], vs[row]
                row += 1
        return kc, ks, vc, vs

    def check_pool(self):
        torch.cuda.synchronize()
        assert np.array_equal(self.pool.k4.cpu().numpy(), R.pack_k(self.pool.kc))
        assert np.array_equal(self.pool.v4.cpu().numpy(), R.pack_v(self.pool.vc))
        assert np.array_equal(self.pool.scales.cpu().numpy(), R.pack_scales(self.pool.ks, self.pool.vs))

    def check_gather(self):
        ko = torch.full_like(self.dk, 77)
        vo = torch.full_like(self.dv, 77)
        mw.mw_kv4_pool_gather(self.pool.handle, *self.args(), ko.data_ptr(), vo.data_ptr())
        torch.cuda.synchronize()
        row = 0
        for b, (n, s) in enumerate(zip(self.lens, self.starts)):
            for i in range(n):
                page, slot = self.table[b, (s + i) // 16], (s + i) % 16
                there = 0 <= page < self.pool.pages
                for out, code, scale in ((ko, self.pool.kc, self.pool.ks), (vo, self.pool.vc, self.pool.vs)):
                    got = bits_to_f32(R.bits_of(out[row]))
                    want = R.values(code[page, :, slot], scale[page, :, slot]) if there else np.zeros(got.shape)
                    assert np.array_equal(got, want.astype(np.float32), equal_nan=True), (b, i)
                row += 1


@pytest.mark.parametrize("hkv,lens,starts", [
    (1, [1], [0]), (2, [1, 1, 1, 1, 1], [0, 1, 2, 3, 18]), (8, [1] * 9, list(range(5, 14))), (3, [2, 3], [3, 13]),
    (2, [16, 4, 0, 33], [0, 4, 7, 5]), (5, [97, 1, 250], [31, 100, 2]), (1, [0, 0], [0, 3]),
])
def test_append_and_read_back(hkv, lens, starts):
    """Every byte of the pool, those of the other tokens included, and every row read back."""
    say(f"kv4 append hkv={hkv} lens={lens} starts={starts}")
    a = Append(hkv, lens, starts, seed=hkv + len(lens))
    try:
        a.write()
        a.expect()
        a.check_pool()
        a.check_gather()
    finally:
        a.pool.close()


def test_every_bf16_value_rounds_as_defined():
    """All 65536 bit patterns: next to a large, an equal and a small neighbour, infinities and NaN among them, the
    largest and smallest blocks, ties and signed zeros."""
    say("kv4 all bf16 patterns")
    every = np.arange(65536, dtype=np.uint16)
    blocks = []
    for first in (0x3F80, 0x40A0, 0x4110):           # 1, 5, 9: blocks of an exponent of their own beside the value
        rows_ = np.zeros((65536 // 31 + 1) * 32, np.uint16).reshape(-1, 32)
        rows_[:, 0] = first
        flat = np.resize(every, rows_.shape[0] * 31).reshape(-1, 31)
        rows_[:, 1:] = flat                          # 31 neighbouring patterns: of one binade
        blocks.append(rows_)
    alone = np.zeros((65536, 32), np.uint16)         # each alone in a block of zeros
    alone[:, 7] = every
    blocks.append(alone)
    rng = np.random.Generator(np.random.PCG64(3))
    scaled = rng.standard_normal((40000, 32)) * np.exp2(rng.integers(-120, 120, (40000, 1)))
    blocks.append(f32_to_bf16_bits(scaled.astype(np.float32)))
    bits = np.concatenate(blocks)
    bits = np.concatenate([bits, np.zeros((-len(bits) % 8, 32), np.uint16)]).reshape(-1, 2, 128)
    a = Append(2, [len(bits)], [0], seed=4, bits=bits)
    try:
        a.write()
        a.expect()
        a.check_pool()
        ko, vo = torch.empty_like(a.dk), torch.empty_like(a.dv)
        mw.mw_kv4_pool_gather(a.pool.handle, *a.args(), ko.data_ptr(), vo.data_ptr())
        torch.cuda.synchronize()
        for out, x in ((ko, a.k), (vo, a.v)):
            got = bits_to_f32(R.bits_of(out))
            code, scale = R.quantise(x)
            assert np.array_equal(got, R.values(code, scale).astype(np.float32), equal_nan=True)
            assert np.isnan(got).any() and np.isfinite(got).any()
    finally:
        a.pool.close()


def test_append_leaves_what_has_no_page_alone():
    say("kv4 append with pages outside the pool")

    def holes(table):
        table[0, 1], table[1, 0] = -1, 1 << 30
        return table

    a = Append(2, [40, 21], [3, 9], seed=9, table=holes)
    try:
        a.write()
        a.expect()
        a.check_pool()
        a.check_gather()
    finally:
        a.pool.close()


# ------------------------------------------------------------------- decode
class Decode:
    def __init__(self, hq, hkv, lens, seed, gain=1.0, poison=True):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.hq, self.hkv, self.lens = hq, hkv, np.array(lens, np.int32)
        self.table, pages = R.tables(lens, rng, spare=1)
        self.pool = R.Pool4(pages, hkv, seed + 1)
        if poison:  # slack slots of last pages and the spare page
            self.pool.poison_slots(pages - 1, 0)
            for b, n in enumerate(lens):
                if n % 16:
                    self.pool.poison_slots(self.table[b, n // 16], n % 16)
            mw.mw_kv_pool_destroy(self.pool.handle)
            self.pool.upload()
        self.q = normal_bits(rng, len(lens), hq, 128, gain=gain)
        self.dq = R.device(self.q.view(np.int16))
        self.out = torch.full_like(self.dq, 0x7FC0)
        self.dlens, self.dtable = R.device(self.lens), R.device(self.table)
        size = mw.mw_kv4_decode_workspace_size(hq, hkv, 128, self.lens)
        self.ws = torch.full((size + 16,), 0xA5, dtype=torch.uint8, device="cuda")
        self.size = size

    def run(self, stream=0, timing=None):
        mw.mw_kv4_decode_attn(self.pool.handle, self.hq, self.hkv, 128, SCALE, self.lens, self.dlens.data_ptr(),
                              self.dtable.data_ptr(), self.table.shape[1], self.dq.data_ptr(), self.out.data_ptr(),
                              self.ws.data_ptr(), self.size, stream, timing)

    def check(self, what=""):
        torch.cuda.synchronize()
        got = bits_to_f32(R.bits_of(self.out)).astype(np.float64)
        k, v = self.pool.bf16()
        k[~np.isfinite(bits_to_f32(k))] = 0          # poisoned slots, not seen by any query
        v[~np.isfinite(bits_to_f32(v))] = 0
        ref = oracle.decode(self.q, k, v, self.table, self.lens)
        ref_abs = oracle.decode(self.q, k, v & 0x7FFF, self.table, self.lens)
        assert np.isfinite(got).all(), what
        bound = R.attention_bound(self.q, bits_to_f32(k), ref, ref_abs, SCALE)
        worst = float((np.abs(got - ref) / bound).max())
        say(f"  {what} worst error / bound {worst:.3f}")
        assert worst <= 1, (what, worst)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (3, 1), (4, 1), (5, 1), (8, 1), (9, 1), (16, 1), (8, 2), (12, 2),
                                    (32, 8), (64, 8), (32, 32)])
def test_decode_groups(hq, hkv):
    say(f"kv4 decode hq={hq} hkv={hkv}")
    d = Decode(hq, hkv, [1, 15, 16, 17, 63, 64, 65, 300, 1029], seed=hq + hkv)
    try:
        d.run()
        d.check(f"{hq}/{hkv}")
    finally:
        d.pool.close()


@pytest.mark.parametrize("lens", [[1], [4003], [30000], [2] * 200, [1, 9000], [5000, 5000, 5000],
                                  list(range(1, 130)), [16384, 1, 1, 1, 700]])
@pytest.mark.parametrize("cus", [256, 32])
def test_decode_lengths(lens, cus):
    """Splits of every kind (whole segments, padded ones, straddling ranges), on the whole GPU and on few CUs."""
    say(f"kv4 decode lens={lens[:6]}.. cus={cus}")
    d = Decode(8, 2, lens, seed=len(lens) + cus)
    part = Partition(256 - cus, cus) if cus < 256 else None
    try:
        torch.cuda.synchronize()
        d.run(part.decode_stream if part else 0)
        d.check(f"{len(lens)} sequences")
    finally:
        d.pool.close()
        if part:
            part.close()


@pytest.mark.parametrize("gain", [0.0, 1e-30, 4.0, 1e4])
def test_decode_query_sizes(gain):
    """Zero and tiny queries (the mean of V), peaked ones, and scores beyond the exponential's range."""
    say(f"kv4 decode gain={gain}")
    d = Decode(12, 2, [1, 33, 500, 2100], seed=11, gain=gain)
    try:
        d.run()
        d.check(f"gain {gain}")
    finally:
        d.pool.close()


def test_decode_random_batches():
    rng = np.random.Generator(np.random.PCG64(77))
    for it in range(12):
        hkv = int(rng.choice([1, 2, 4, 8]))
        hq = hkv * int(rng.choice([1, 2, 4, 6, 8, 16]))
        lens = [int(x) for x in np.exp(rng.uniform(0, np.log(3000), int(rng.integers(1, 40))))]
        say(f"kv4 decode random {it}: {hq}/{hkv} {lens[:5]}..")
        d = Decode(hq, hkv, lens, seed=100 + it, gain=float(rng.choice([1, 4])))
        try:
            d.run()
            d.check(f"random {it}")
        finally:
            d.pool.close()


def test_decode_not_finite_values_reach_only_who_sees_them():
    """A NaN block of K makes its sequence's head NaN, one of V the 32 dims of it, a NaN query its own head."""
    say("kv4 decode NaN")
    d = Decode(8, 2, [200, 100, 50], seed=21, poison=False)
    p, t = d.pool, d.table
    p.ks[t[0, 3], 1, 5, 2], p.kc[t[0, 3], 1, 5, 64:96] = 255, 0
    p.vs[t[1, 2], 0, 7, 3], p.vc[t[1, 2], 0, 7, 96:128] = 255, 0
    mw.mw_kv_pool_destroy(p.handle)
    p.upload()
    q = d.q.copy()
    q[2, 6, 3] = 0x7FC0
    d.dq.copy_(R.device(q.view(np.int16)))
    try:
        d.run()
        torch.cuda.synchronize()
        got = bits_to_f32(R.bits_of(d.out))
        want = np.zeros(got.shape, bool)
        want[0, 4:8] = True
        want[1, 0:4, 96:128] = True
        want[2, 6] = True
        assert np.array_equal(np.isnan(got), want)
        assert np.isfinite(got[~want]).all()
    finally:
        p.close()


def test_decode_in_a_graph_with_eager_calls_between():
    """Two captured calls that share a workspace, replayed in turn with an eager call on it."""
    say("kv4 decode graph")
    a, b = Decode(32, 8, [4000, 1, 700], seed=31), Decode(32, 8, [5, 2500, 2500], seed=33)
    try:
        stream = torch.cuda.Stream()
        size = max(a.size, b.size)
        a.ws = b.ws = torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda")
        a.size = b.size = size
        a.run(stream.cuda_stream)
        b.run(stream.cuda_stream)
        torch.cuda.synchronize()
        eager = [R.bits_of(a.out), R.bits_of(b.out)]
        graphs = []
        for d in (a, b):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                d.run(stream.cuda_stream)
            graphs.append(g)
        for _ in range(4):
            for d, g, want in ((a, graphs[0], eager[0]), (b, graphs[1], eager[1])):
                d.out.fill_(0)
                torch.cuda.synchronize()
                with torch.cuda.stream(stream):
                    g.replay()
                torch.cuda.synchronize()
                assert np.array_equal(R.bits_of(d.out), want)
                d.run(stream.cuda_stream)
                torch.cuda.synchronize()
                assert np.array_equal(R.bits_of(d.out), want)
        a.check("graph a")
        b.check("graph b")
    finally:
        a.pool.close()
        b.pool.close()


# ------------------------------------------------------------------ prefill
@pytest.mark.parametrize("hq,hkv,new,prefix", [
    (4, 1, [1], [0]), (8, 2, [33], [0]), (8, 2, [1, 5, 0, 64], [17, 0, 40, 1000]), (32, 8, [300], [700]),
    (16, 1, [65, 2], [3, 2000]), (6, 6, [100], [31]), (12, 2, [17, 17, 17], [1, 15, 16]), (8, 1, [1], [4000]),
    (2, 2, [7] * 70, list(range(70))),
])
def test_prefill(hq, hkv, new, prefix):
    say(f"kv4 prefill {hq}/{hkv} new={new[:4]} prefix={prefix[:4]}")
    rng = np.random.Generator(np.random.PCG64(hq + sum(new)))
    table, pages = R.tables([n + r for n, r in zip(new, prefix)], rng, spare=1)
    pool = R.Pool4(pages, hkv, seed=7)
    pool.poison_slots(pages - 1, 0)
    for b, (n, r) in enumerate(zip(new, prefix)):
        if (n + r) % 16:
            pool.poison_slots(table[b, (n + r) // 16], (n + r) % 16)
    mw.mw_kv_pool_destroy(pool.handle)
    pool.upload()
    total = sum(new)
    q = normal_bits(rng, total, hq, 128)
    dq = R.device(np.concatenate([q, q[:2]]).view(np.int16))
    out = torch.full_like(dq, 0x1234)
    dtable, dprefix, indptr = R.device(table), R.device(prefix, np.int32), rows(new)
    size = mw.mw_kv4_prefill_workspace_size(hq, hkv, 128, new, prefix)
    ws = torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    timing = mw.mw_timing_create()
    try:
        for it in range(2):  # the workspace as it was left, then again
            out.fill_(0x1234)
            mw.mw_kv4_prefill_attn(pool.handle, hq, hkv, 128, SCALE, new, prefix, indptr.data_ptr(),
                                   dprefix.data_ptr(), dtable.data_ptr(), table.shape[1], dq.data_ptr(),
                                   out.data_ptr(), ws.data_ptr(), size, 0, timing)
            torch.cuda.synchronize()
            got = R.bits_of(out)
            assert (got[total:] == 0x1234).all()     # rows behind the last sequence
            assert mw.mw_timing_kernels(timing) >= 1
            k, v = pool.bf16()
            k[~np.isfinite(bits_to_f32(k))] = 0
            v[~np.isfinite(bits_to_f32(v))] = 0
            row = 0
            for b, (n, r) in enumerate(zip(new, prefix)):
                if n == 0:
                    continue
                ref = oracle.prefill(q[row:row + n], k, v, table[b], r)
                ref_abs = oracle.prefill(q[row:row + n], k, v & 0x7FFF, table[b], r)
                bound = R.attention_bound(q[row:row + n], bits_to_f32(k), ref, ref_abs, SCALE)
                o = bits_to_f32(got[row:row + n]).astype(np.float64)
                assert np.isfinite(o).all()
                worst = float((np.abs(o - ref) / bound).max())
                assert worst <= 1, (b, worst)
                row += n
    finally:
        mw.mw_timing_destroy(timing)
        pool.close()


class Prefill:
    """A call of few new tokens, its rows behind the last sequence, and its check against the oracle."""

    def __init__(self, hq, hkv, new, prefix, seed, table=None, gain=1.0):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.hq, self.hkv, self.new, self.prefix = hq, hkv, new, prefix
        self.table, pages = R.tables([n + r for n, r in zip(new, prefix)], rng, spare=2)
        self.pool = R.Pool4(pages, hkv, seed + 1)
        self.pool.poison_slots(pages - 1, 0)
        for b, (n, r) in enumerate(zip(new, prefix)):
            if (n + r) % 16:
                self.pool.poison_slots(self.table[b, (n + r) // 16], (n + r) % 16)
        mw.mw_kv_pool_destroy(self.pool.handle)
        self.pool.upload()
        if table is not None:
            self.table = table(self.table, pages)
        self.total = sum(new)
        self.q = normal_bits(rng, self.total, hq, 128, gain=gain)
        self.dq = R.device(np.concatenate([self.q, self.q[:2]]).view(np.int16))
        self.out = torch.full_like(self.dq, 0x1234)
        self.dtable, self.dprefix, self.indptr = R.device(self.table), R.device(prefix, np.int32), rows(new)
        self.size = mw.mw_kv4_prefill_workspace_size(hq, hkv, 128, new, prefix)
        self.ws = torch.full((max(self.size, 16),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, stream=0, timing=None):
        mw.mw_kv4_prefill_attn(self.pool.handle, self.hq, self.hkv, 128, SCALE, self.new, self.prefix,
                               self.indptr.data_ptr(), self.dprefix.data_ptr(), self.dtable.data_ptr(),
                               self.table.shape[1], self.dq.data_ptr(), self.out.data_ptr(), self.ws.data_ptr(),
                               self.size, stream, timing)

    def check(self, absent_reads_zero=False):
        torch.cuda.synchronize()
        got = R.bits_of(self.out)
        assert (got[self.total:] == 0x1234).all()
        k, v = self.pool.bf16()
        k[~np.isfinite(bits_to_f32(k))] = 0
        v[~np.isfinite(bits_to_f32(v))] = 0
        table = self.table
        if absent_reads_zero:  # a page of zeros in the place of every page that is not there
            zero = np.zeros((1,) + k.shape[1:], k.dtype)
            k, v = np.concatenate([k, zero]), np.concatenate([v, zero])
            table = np.where((table < 0) | (table >= self.pool.pages), self.pool.pages, table)
        row = 0
        for b, (n, r) in enumerate(zip(self.new, self.prefix)):
            if n == 0:
                continue
            q = self.q[row:row + n]
            ref = oracle.prefill(q, k, v, table[b], r)
            ref_abs = oracle.prefill(q, k, v & 0x7FFF, table[b], r)
            bound = R.attention_bound(q, bits_to_f32(k), ref, ref_abs, SCALE)
            o = bits_to_f32(got[row:row + n]).astype(np.float64)
            assert np.isfinite(o).all()
            worst = float((np.abs(o - ref) / bound).max())
            assert worst <= 1, (b, worst)
            row += n

    def close(self):
        self.pool.close()


FEW = [  # heads, new and prefix lengths
    (8, 2, [1], [1]), (32, 8, [16], [0]), (4, 1, [63, 64, 65], [1, 0, 63]),
    (32, 8, [1], [8000]), (32, 8, [64], [2500]), (1, 1, [1], [20000]), (16, 1, [64, 63], [1000, 3001]),
    (6, 2, [43, 42, 1], [3000, 2, 0]), (5, 5, [128, 129], [500, 2000]), (8, 2, [33, 1, 0, 130], [4000, 0, 77, 2900]),
    (16, 16, [31], [33]), (32, 2, [3] * 40, list(range(0, 400, 10))), (48, 1, [9], [4500]),
    (32, 8, [4] * 32, [9000] + [100] * 31), (8, 2, [250] + [1, 0, 2] * 30, [2000] * 91), (4, 2, [3] * 130, [1500] + [70] * 129),
]


@pytest.mark.parametrize("hq,hkv,new,prefix", FEW)
def test_prefill_of_few_rows(hq, hkv, new, prefix):
    """One piece, several, and blocks of one call with different counts of them; a row of several tokens' heads."""
    say(f"kv4 few rows {hq}/{hkv} new={new[:4]} prefix={prefix[:4]}")
    p = Prefill(hq, hkv, new, prefix, seed=hq + sum(new) + sum(prefix))
    timing = mw.mw_timing_create()
    try:
        for _ in range(2):
            p.out.fill_(0x1234)
            p.run(timing=timing)
            p.check()
            assert (mw.mw_timing_kernels(timing) == 1) == (p.size == 0)
    finally:
        mw.mw_timing_destroy(timing)
        p.close()


@pytest.mark.parametrize("new", [127, 128, 129, 257])
def test_prefill_either_side_of_the_block_limit(new):
    """Eight query blocks of a kv head go straight from the codes, nine are unpacked first."""
    say(f"kv4 prefill {new} of 8/1")
    p = Prefill(8, 1, [new], [700], seed=new)
    try:
        p.run()
        p.check()
    finally:
        p.close()


@pytest.mark.parametrize("gain", [0.0, 1e-30, 4.0, 1e3])
def test_prefill_query_sizes(gain):
    say(f"kv4 few rows gain={gain}")
    p = Prefill(12, 2, [5, 40], [2100, 33], seed=12, gain=gain)
    try:
        p.run()
        p.check()
    finally:
        p.close()


@pytest.mark.parametrize("new,prefix", [([20, 1], [2000, 600]), ([900], [1100])])
def test_prefill_pages_that_are_not_there_read_as_zeros(new, prefix):
    say(f"kv4 prefill absent pages {new}")

    def gaps(table, pages):
        table = table.copy()
        table[0, 3], table[0, 17], table[0, 40] = -1, pages, pages + 1000
        table[-1, 20:24] = -7
        return table

    p = Prefill(8, 2, new, prefix, seed=5, table=gaps)
    try:
        p.run()
        p.check(absent_reads_zero=True)
    finally:
        p.close()


def test_prefill_not_finite_values_reach_only_who_sees_them():
    """A NaN block of K reaches the rows of its head that see it, one of V their 32 dims, a NaN query its own head."""
    say("kv4 few rows NaN")
    p = Prefill(8, 2, [40, 40], [3000, 3000], seed=31)
    pool, t = p.pool, p.table
    pool.ks[t[0, 188], 1, 9, 2], pool.kc[t[0, 188], 1, 9, 64:96] = 255, 0   # key 3017: rows 17 and later
    pool.vs[t[1, 100], 0, 7, 3], pool.vc[t[1, 100], 0, 7, 96:128] = 255, 0  # before all rows
    mw.mw_kv_pool_destroy(pool.handle)
    pool.upload()
    q = p.q.copy()
    q[45, 6, 3] = 0x7FC0
    p.dq[:80].copy_(R.device(q.view(np.int16)))
    try:
        p.run()
        torch.cuda.synchronize()
        got = bits_to_f32(R.bits_of(p.out))[:80]
        want = np.zeros(got.shape, bool)
        want[17:40, 4:8] = True
        want[40:, 0:4, 96:128] = True
        want[45, 6] = True
        assert np.array_equal(np.isnan(got), want)
        assert np.isfinite(got[~want]).all()
    finally:
        p.close()


def test_prefill_on_a_part_of_the_gpu_is_the_same():
    say("kv4 few rows on 32 CUs")
    p = Prefill(32, 8, [64, 3], [2000, 900], seed=41)
    part = Partition(224, 32)
    try:
        torch.cuda.synchronize()
        p.run()
        torch.cuda.synchronize()
        whole = R.bits_of(p.out)
        p.out.fill_(0x1234)
        torch.cuda.synchronize()
        p.run(part.decode_stream)
        p.check()
        assert np.array_equal(R.bits_of(p.out), whole)
    finally:
        p.close()
        part.close()


def test_prefill_in_a_graph_with_eager_calls_between():
    """Captured calls, straight from the codes and unpacked, that share a workspace with each other and eager calls."""
    say("kv4 prefill graph")
    calls = [Prefill(32, 8, [60], [2000], seed=51), Prefill(8, 1, [300], [500], seed=52), Prefill(4, 4, [9], [3], seed=53)]
    try:
        stream = torch.cuda.Stream()
        size = max(p.size for p in calls)
        ws = torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda")
        graphs, eager = [], []
        for p in calls:
            p.ws, p.size = ws, size
            p.run(stream.cuda_stream)
            torch.cuda.synchronize()
            eager.append(R.bits_of(p.out))
        for p in calls:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                p.run(stream.cuda_stream)
            graphs.append(g)
        for _ in range(3):
            for p, g, want in zip(calls, graphs, eager):
                p.out.fill_(0x1234)
                torch.cuda.synchronize()
                with torch.cuda.stream(stream):
                    g.replay()
                torch.cuda.synchronize()
                assert np.array_equal(R.bits_of(p.out), want)
                p.run(stream.cuda_stream)
                torch.cuda.synchronize()
                assert np.array_equal(R.bits_of(p.out), want)
        for p in calls:
            p.check()
    finally:
        for p in calls:
            p.close()


def test_two_calls_at_a_time():
    """A decode batch and a chunk on two streams, with workspaces of their own: what each gives alone."""
    say("kv4 two streams")
    d, p = Decode(32, 8, [3000, 50, 1700, 900], seed=61), Prefill(32, 8, [40, 7], [3000, 100], seed=62)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    try:
        d.run()
        p.run()
        torch.cuda.synchronize()
        alone = [R.bits_of(d.out), R.bits_of(p.out)]
        for _ in range(8):
            d.out.fill_(0x1234)
            p.out.fill_(0x1234)
            torch.cuda.synchronize()
            for _ in range(4):
                d.run(streams[0].cuda_stream)
                p.run(streams[1].cuda_stream)
            torch.cuda.synchronize()
            assert np.array_equal(R.bits_of(d.out)[:4], alone[0][:4])
            assert np.array_equal(R.bits_of(p.out)[:47], alone[1][:47])
        d.check("decode beside a chunk")
        p.check()
    finally:
        d.pool.close()
        p.close()


def test_a_pool_past_32_bits():
    """Rows on the last pages of a pool whose codes take more than 4 GiB: every call as on a small pool."""
    say("kv4 large pool")
    hq, hkv, lens = 8, 4, [1030, 5]
    rng = np.random.Generator(np.random.PCG64(71))
    table, pages = R.tables(lens, rng)
    far = (1 << 32) // (hkv * 1024) + 100
    k, v = (R.device(normal_bits(rng, sum(lens), hkv, 128).view(np.int16)) for _ in range(2))
    x = R.device(normal_bits(rng, 2, hq + 2 * hkv, 128).view(np.int16))
    q = R.device(normal_bits(rng, 602, hq, 128).view(np.int16))
    freq = R.device(1e4 ** (-np.arange(64, dtype=np.float64) / 64))
    got = []
    for shift in (0, far):
        total = pages + shift
        k4, v4 = (torch.empty(total, hkv, 1024, dtype=torch.uint8, device="cuda") for _ in range(2))
        scales = torch.empty(total, hkv, 128, dtype=torch.uint8, device="cuda")
        assert shift == 0 or k4.numel() > 1 << 32
        for t in (k4, v4, scales):
            t[-pages:].zero_()
        pool = mw.mw_kv4_pool_create(total, 16, hkv, 128, k4.data_ptr(), v4.data_ptr(), scales.data_ptr())
        try:
            bt = table + shift
            dbt, zero, ip = R.device(bt), R.device([0, 0], np.int32), rows(lens)
            place = (np.array(lens, np.int32), np.zeros(2, np.int32), ip.data_ptr(), zero.data_ptr(), dbt.data_ptr(),
                     bt.shape[1])
            mw.mw_kv4_pool_write(pool, *place, k.data_ptr(), v.data_ptr())
            # one token of each again, through the norm and rotation
            last, ones, ip1 = np.array(lens, np.int32) - 1, np.ones(2, np.int32), rows([1, 1])
            dlast, q_out = R.device(last), torch.empty(2, hq, 128, dtype=torch.int16, device="cuda")
            rope = mw.NormRope(num_q_heads=hq, rot_dim=128, neighbours=0, eps=1e-6, d_q_weight=0, d_k_weight=0,
                               d_inv_freq=freq.data_ptr())
            at, stride = x.data_ptr(), (hq + 2 * hkv) * 128
            mw.mw_qk_norm_rope_write(pool, rope, ones, last, ip1.data_ptr(), dlast.data_ptr(), dbt.data_ptr(),
                                     bt.shape[1], at, stride, at + 256 * hq, stride, at + 256 * (hq + hkv), stride,
                                     q_out.data_ptr())
            ko, vo = torch.empty_like(k), torch.empty_like(v)
            mw.mw_kv4_pool_gather(pool, *place, ko.data_ptr(), vo.data_ptr())
            out = [q_out, ko, vo]
            dlens, o = R.device(lens, np.int32), torch.empty(2, hq, 128, dtype=torch.int16, device="cuda")
            n = mw.mw_kv4_decode_workspace_size(hq, hkv, 128, lens)
            ws = torch.empty(n, dtype=torch.uint8, device="cuda")
            mw.mw_kv4_decode_attn(pool, hq, hkv, 128, SCALE, lens, dlens.data_ptr(), dbt.data_ptr(), bt.shape[1],
                                  q.data_ptr(), o.data_ptr(), ws.data_ptr(), n)
            out.append(o)
            for new in ([20, 2], [600, 2]):  # straight from the codes, and unpacked
                prefix = [m - c for m, c in zip(lens, new)]
                ipn, dpre = rows(new), R.device(prefix, np.int32)
                n = mw.mw_kv4_prefill_workspace_size(hq, hkv, 128, new, prefix)
                ws2 = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
                o = torch.empty(sum(new), hq, 128, dtype=torch.int16, device="cuda")
                mw.mw_kv4_prefill_attn(pool, hq, hkv, 128, SCALE, new, prefix, ipn.data_ptr(), dpre.data_ptr(),
                                       dbt.data_ptr(), bt.shape[1], q.data_ptr(), o.data_ptr(), ws2.data_ptr(), n)
                torch.cuda.synchronize()
                out.append(o)
            torch.cuda.synchronize()
            got.append([R.bits_of(t) for t in out])
        finally:
            torch.cuda.synchronize()
            mw.mw_kv_pool_destroy(pool)
        del k4, v4, scales
    for a, b in zip(*got):
        assert np.isfinite(bits_to_f32(a)).all() and a.any() and np.array_equal(a, b)
