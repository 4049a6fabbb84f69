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
            assert mw.mw_timing_kernels(timing) >= 2
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
