"""Norm, rotation and append in one pass on the GPU, against the formulas in fp64; and the pass with the attention of
both kinds of pool behind it, as a layer uses them."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_14489_amd import mw
from paper_2504_14489_amd.device import bits_to_f32
from paper_2504_14489_amd.workloads import f32_to_bf16_bits
from tests import kv4_reference as R
from tests.helpers import say

pytestmark = pytest.mark.gpu

EPS = 1e-6


def formula(x, weight, positions, inv_freq, neighbours, eps=EPS):
    """x [T, heads, 128] fp64 -> the rotated rows."""
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    x = x.copy()
    half = len(inv_freq)
    angle = positions[:, None, None] * inv_freq
    cos, sin = np.cos(angle), np.sin(angle)
    one, two = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if neighbours
                else (slice(0, half), slice(half, 2 * half)))
    a, b = x[..., one].copy(), x[..., two].copy()
    x[..., one], x[..., two] = a * cos - b * sin, b * cos + a * sin
    return x


class Rows:
    """Projection rows of a batch (queries, keys and values of a token side by side) and a pool of either kind."""

    def __init__(self, hq, hkv, lens, starts, four_bit, norm=True, rot=128, neighbours=False, theta=1e4, seed=1,
                 gain=1.0, apart=False):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.hq, self.hkv, self.four_bit, self.neighbours = hq, hkv, four_bit, neighbours
        self.lens, self.starts = np.array(lens, np.int32), np.array(starts, np.int32)
        self.total = int(sum(lens))
        self.positions = np.concatenate([s + np.arange(n) for n, s in zip(lens, starts)] or [[]]).astype(np.float64)
        first = min([s // 16 for s in starts] + [1 << 30])
        self.table, self.pages = R.tables([n + s - 16 * first for n, s in zip(lens, starts)], rng, spare=1)
        # pages before the first written one need not exist
        self.table = np.concatenate([np.full((len(self.table), first), -1, np.int32), self.table], axis=1)
        heads = hq + 2 * hkv
        self.x = f32_to_bf16_bits((gain * rng.standard_normal((self.total, heads, 128))).astype(np.float32))
        self.pad = 8 if apart else 0  # elements between a token's row and the next
        wide = np.zeros((self.total, heads * 128 + self.pad), np.uint16)
        wide[:, :heads * 128] = self.x.reshape(self.total, -1)
        self.rows = R.device(wide.view(np.int16))
        self.w = [f32_to_bf16_bits((1 + 0.2 * rng.standard_normal(128)).astype(np.float32)) if norm else None
                  for _ in range(2)]
        self.dw = [None if w is None else R.device(w.view(np.int16)) for w in self.w]
        self.inv_freq = theta ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1))
        self.dfreq = R.device(self.inv_freq) if rot else None
        if four_bit:
            self.pool = R.Pool4(self.pages, hkv, seed + 1)
            self.handle = self.pool.handle
        else:
            self.k = torch.full((self.pages, hkv, 16, 128), 0x1111, dtype=torch.int16, device="cuda")
            self.v = torch.full_like(self.k, 0x2222)
            self.handle = mw.mw_kv_pool_create(self.pages, 16, hkv, 128, self.k.data_ptr(), self.v.data_ptr())
        self.rope = mw.NormRope(num_q_heads=hq, rot_dim=rot, neighbours=int(neighbours), eps=EPS,
                                d_q_weight=self.dw[0].data_ptr() if norm else 0,
                                d_k_weight=self.dw[1].data_ptr() if norm else 0,
                                d_inv_freq=self.dfreq.data_ptr() if rot else 0)
        self.q_out = torch.full((self.total + 1, max(hq, 1), 128), 0x1234, dtype=torch.int16, device="cuda")
        self.dtable, self.dstart = R.device(self.table), R.device(self.starts)
        self.indptr = R.device(np.concatenate([[0], np.cumsum(lens)]), np.int32)

    def place(self):
        return (self.lens, self.starts, self.indptr.data_ptr(), self.dstart.data_ptr(), self.dtable.data_ptr(),
                self.table.shape[1])

    def run(self, stream=0):
        at, stride = self.rows.data_ptr(), self.rows.shape[1]
        mw.mw_qk_norm_rope_write(self.handle, self.rope, *self.place(), at, stride, at + 256 * self.hq, stride,
                                 at + 256 * (self.hq + self.hkv), stride, self.q_out.data_ptr(), stream)

    def reference(self):
        x = bits_to_f32(self.x).astype(np.float64)
        w = [None if w is None else bits_to_f32(w).astype(np.float64) for w in self.w]
        q = formula(x[:, :self.hq], w[0], self.positions, self.inv_freq, self.neighbours)
        k = formula(x[:, self.hq:self.hq + self.hkv], w[1], self.positions, self.inv_freq, self.neighbours)
        return q, k

    def cache_rows(self):
        """The rows of the call as the pool holds them: K and V [T, hkv, 128] fp64."""
        if self.four_bit:
            k = torch.empty(self.total, self.hkv, 128, dtype=torch.int16, device="cuda")
            v = torch.empty_like(k)
            mw.mw_kv4_pool_gather(self.handle, *self.place(), k.data_ptr(), v.data_ptr())
            torch.cuda.synchronize()
            return [bits_to_f32(R.bits_of(t)).astype(np.float64) for t in (k, v)]
        seq = np.repeat(np.arange(len(self.lens)), self.lens)
        pos = self.positions.astype(np.int64)
        page, slot = self.table[seq, pos // 16], pos % 16
        torch.cuda.synchronize()
        return [bits_to_f32(R.bits_of(t))[page, :, slot].astype(np.float64) for t in (self.k, self.v)]

    def check(self):
        torch.cuda.synchronize()
        got = bits_to_f32(R.bits_of(self.q_out)).astype(np.float64)
        assert (R.bits_of(self.q_out)[self.total:] == 0x1234).all()
        q, k = self.reference()
        # rounding to bf16 is half a step, 2^-8 of the value; sums of 128 squares, rsqrt and two products in fp32 are
        # off by less than 2^-19 of the pair's size, the angle's cosine and sine by 2^-20
        def near(a, want, what):
            if not a.size:
                return
            half = len(self.inv_freq)
            size = np.abs(want).copy()
            if half:
                one, two = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if self.neighbours
                            else (slice(0, half), slice(half, 2 * half)))
                pair = np.hypot(want[..., one], want[..., two])
                size[..., one], size[..., two] = pair, pair
            bound = 2.0**-8 * np.abs(want) + 2.0**-18 * size + 1e-37
            assert (np.abs(a - want) <= bound).all(), (what, float((np.abs(a - want) / bound).max()))

        if self.hq:
            near(got[:self.total], q, "q")
        held = self.cache_rows()
        v = self.x[:, self.hq + self.hkv:]
        if self.four_bit:
            assert np.array_equal(held[1], R.values(*R.quantise(v)))
            # what is held is the quantised form of a bf16 key that is near the formula's: a value may go to the
            # other side of a border only if the key lies within that error of it
            lo, hi = (R.values(*R.quantise(f32_to_bf16_bits((k * f).astype(np.float32)))) for f in (1 - 2**-7, 1 + 2**-7))
            unit = np.exp2(R.quantise(f32_to_bf16_bits(k.astype(np.float32)))[1].astype(np.float64) - 127)
            step = np.repeat(unit, 32, axis=-1) * 2
            low, high = np.minimum(lo, hi), np.maximum(lo, hi)
            assert (held[0] >= low - step).all() and (held[0] <= high + step).all()
            same = held[0] == R.values(*R.quantise(f32_to_bf16_bits(k.astype(np.float32))))
            assert same.mean() >= 0.995, same.mean()  # 2^-10 of values lie that near a bf16 border, fewer a code's
        else:
            near(held[0], k, "k")
            assert np.array_equal(held[1], bits_to_f32(v))

    def close(self):
        torch.cuda.synchronize()
        mw.mw_kv_pool_destroy(self.handle)


@pytest.mark.parametrize("four_bit", [False, True])
@pytest.mark.parametrize("hq,hkv,lens,starts", [
    (4, 1, [1], [0]), (32, 8, [1] * 5, [0, 17, 3, 100, 4094]), (8, 2, [33], [5]), (12, 2, [2, 0, 70], [14, 3, 33]),
    (0, 3, [9], [2]), (64, 8, [130], [1000]), (1, 1, [1, 1], [131071, 1 << 20]),
])
def test_shapes(hq, hkv, lens, starts, four_bit):
    say(f"norm rope {hq}/{hkv} lens={lens} starts={starts} four_bit={four_bit}")
    r = Rows(hq, hkv, lens, starts, four_bit, seed=hq + hkv)
    try:
        r.run()
        r.check()
    finally:
        r.close()


@pytest.mark.parametrize("rot", [0, 16, 48, 64, 112, 128])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rotations(rot, neighbours, norm):
    say(f"norm rope rot={rot} neighbours={neighbours} norm={norm}")
    r = Rows(6, 2, [21, 40], [3, 5000], False, norm=norm, rot=rot, neighbours=neighbours, theta=5e5, seed=rot,
             apart=True)
    try:
        r.run()
        r.check()
    finally:
        r.close()


@pytest.mark.parametrize("gain", [0.0, 1e-4, 1e4])
def test_sizes_of_rows(gain):
    """Zero rows (eps keeps them zero), rows that eps outweighs, and large ones."""
    say(f"norm rope gain={gain}")
    r = Rows(4, 2, [19], [7], False, seed=5, gain=gain)
    try:
        r.run()
        r.check()
    finally:
        r.close()


def test_four_bit_keys_are_the_bf16_ones_quantised():
    """The pass into a 4-bit pool holds, bit for bit, what the pass into bf16 and the 4-bit append hold."""
    say("norm rope four bit against two steps")
    for rot, neighbours in ((128, False), (64, True)):
        wide = Rows(8, 2, [50, 1, 31], [9, 64, 0], False, rot=rot, neighbours=neighbours, seed=8)
        kept = Rows(8, 2, [50, 1, 31], [9, 64, 0], True, rot=rot, neighbours=neighbours, seed=8)
        try:
            wide.run()
            kept.run()
            k, _ = wide.cache_rows()
            want = R.values(*R.quantise(f32_to_bf16_bits(k.astype(np.float32))))
            assert np.array_equal(kept.cache_rows()[0], want)
            assert np.array_equal(R.bits_of(wide.q_out), R.bits_of(kept.q_out))
        finally:
            wide.close()
            kept.close()


def test_other_slots_stay_and_absent_pages_are_skipped():
    say("norm rope slots")
    r = Rows(4, 2, [5, 20], [6, 30], False, seed=12)
    r.table[1, 2] = -1
    r.dtable.copy_(R.device(r.table))
    try:
        r.run()
        torch.cuda.synchronize()
        touched = np.zeros((r.pages, 16), bool)
        for b, (n, s) in enumerate(zip(r.lens, r.starts)):
            for p in range(s, s + n):
                if r.table[b, p // 16] >= 0:
                    touched[r.table[b, p // 16], p % 16] = True
        k = R.bits_of(r.k).transpose(0, 2, 1, 3)
        assert (k[~touched] == 0x1111).all() and (k[touched] != 0x1111).any()
        q, _ = r.reference()
        got = bits_to_f32(R.bits_of(r.q_out))[:r.total]
        assert np.abs(got - q).max() <= 2.0**-7 * np.abs(q).max()   # queries of absent pages too
    finally:
        r.close()


def test_in_place_queries():
    say("norm rope in place")
    a, b = (Rows(8, 2, [37], [11], False, seed=14) for _ in range(2))
    try:
        a.run()
        dense = b.rows.view(-1, 12, 128)[:, :8].contiguous()
        at = b.rows.data_ptr()
        mw.mw_qk_norm_rope_write(b.handle, b.rope, *b.place(), dense.data_ptr(), 1024, at + 256 * 8, 12 * 128,
                                 at + 256 * 10, 12 * 128, dense.data_ptr())
        torch.cuda.synchronize()
        assert np.array_equal(R.bits_of(dense), R.bits_of(a.q_out)[:37])
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    finally:
        a.close()
        b.close()


def attend(pool, four_bit, hq, hkv, q, lens, table, new=None, prefix=None, indptr=None, dstart=None, stream=0):
    """Decode (new None) or prefill through the calls of the pool's kind."""
    out = torch.zeros_like(q)
    dtable = R.device(table)
    if new is None:
        dlens = R.device(lens)
        size = (mw.mw_kv4_decode_workspace_size if four_bit else mw.mw_decode_workspace_size)(hq, hkv, 128, lens)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        args = (pool, hq, hkv, 128, 128**-0.5, lens, dlens.data_ptr(), dtable.data_ptr(), table.shape[1], q.data_ptr(),
                out.data_ptr(), ws.data_ptr(), size)
        if four_bit:
            mw.mw_kv4_decode_attn(*args, stream)
        else:
            mw.mw_decode_attn(*args, 0, stream)
    else:
        size = (mw.mw_kv4_prefill_workspace_size if four_bit else mw.mw_prefill_workspace_size)(hq, hkv, 128, new, prefix)
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        (mw.mw_kv4_prefill_attn if four_bit else mw.mw_prefill_attn_ws)(
            pool, hq, hkv, 128, 128**-0.5, new, prefix, indptr.data_ptr(), dstart.data_ptr(), dtable.data_ptr(),
            table.shape[1], q.data_ptr(), out.data_ptr(), ws.data_ptr(), size, stream)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("four_bit", [False, True])
def test_a_layer_from_projection_to_output(four_bit):
    """A prompt's chunk, a second chunk over it, then single tokens: norm, rotation and append, then attention, each
    step compared with the oracle on what the cache holds."""
    say(f"layer run four_bit={four_bit}")
    hq, hkv = 8, 2
    lens, start = [[70, 33], [30, 64], [1, 1], [1, 1]], [[0, 0], [70, 33], [100, 97], [101, 98]]
    rng = np.random.Generator(np.random.PCG64(5))
    table, pages = R.tables([102, 99], rng)
    if four_bit:
        pool = R.Pool4(pages, hkv, 3)
        handle = pool.handle
    else:
        kp = torch.zeros(pages, hkv, 16, 128, dtype=torch.int16, device="cuda")
        vp = torch.zeros_like(kp)
        handle = mw.mw_kv_pool_create(pages, 16, hkv, 128, kp.data_ptr(), vp.data_ptr())
    try:
        for n, s in zip(lens, start):
            r = Rows(hq, hkv, n, s, four_bit, seed=sum(s) + 1)
            mw.mw_kv_pool_destroy(r.handle)
            r.handle, r.table, r.dtable = handle, table, R.device(table)
            r.run()
            if not four_bit:
                r.k, r.v = kp, vp
            r.check()
            after = np.array(n) + np.array(s)
            q = r.q_out[:r.total]
            if n[0] == 1:
                out = attend(handle, four_bit, hq, hkv, q, after.astype(np.int32), table)
            else:
                out = attend(handle, four_bit, hq, hkv, q, None, table, r.lens, r.starts, r.indptr, r.dstart)
            # the cache as it is held, read back into dense pools for the oracle
            if four_bit:
                held = [torch.zeros(int(after.sum()), hkv, 128, dtype=torch.int16, device="cuda") for _ in range(2)]
                ip = R.device(np.concatenate([[0], np.cumsum(after)]), np.int32)
                zero = R.device([0, 0], np.int32)
                mw.mw_kv4_pool_gather(handle, after.astype(np.int32), np.zeros(2, np.int32), ip.data_ptr(),
                                      zero.data_ptr(), r.dtable.data_ptr(), table.shape[1], held[0].data_ptr(),
                                      held[1].data_ptr())
                torch.cuda.synchronize()
                k = np.zeros((pages, hkv, 16, 128), np.uint16)
                v = np.zeros_like(k)
                at = 0
                for b, m in enumerate(after):
                    for p in range(m):
                        k[table[b, p // 16], :, p % 16] = R.bits_of(held[0][at])
                        v[table[b, p // 16], :, p % 16] = R.bits_of(held[1][at])
                        at += 1
            else:
                k, v = R.bits_of(kp), R.bits_of(vp)
            qb, row = R.bits_of(q), 0
            for b in range(2):
                mine = qb[row:row + n[b]]
                ref = oracle.prefill(mine, k, v, table[b], s[b])
                ref_abs = oracle.prefill(mine, k, v & 0x7FFF, table[b], s[b])
                bound = R.attention_bound(mine, bits_to_f32(k), ref, ref_abs, 128**-0.5)
                got = bits_to_f32(R.bits_of(out[row:row + n[b]]))
                assert (np.abs(got - ref) <= bound).all()
                row += n[b]
    finally:
        torch.cuda.synchronize()
        mw.mw_kv_pool_destroy(handle)


@pytest.mark.parametrize("four_bit", [False, True])
def test_a_decode_step_in_a_graph_with_eager_steps_between(four_bit):
    """Norm, rotation, append and decode attention of one token of each sequence, captured; replayed on other rows,
    against an eager step on them."""
    say(f"layer graph four_bit={four_bit}")
    hq, hkv, starts = 8, 2, [700, 0, 33, 1900]
    r = Rows(hq, hkv, [1] * 4, starts, four_bit, seed=3)
    lens = np.array(starts, np.int32) + 1
    dlens, out = R.device(lens), torch.zeros(4, hq, 128, dtype=torch.int16, device="cuda")
    # the sequences' earlier pages: any page of the pool, read by both sides
    table = np.where(r.table < 0, 0, r.table)
    r.table, r.dtable = table, R.device(table)
    size = (mw.mw_kv4_decode_workspace_size if four_bit else mw.mw_decode_workspace_size)(hq, hkv, 128, lens)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()

    def step():
        at = r.rows.data_ptr()
        stride = r.rows.shape[1]
        mw.mw_qk_norm_rope_write(r.handle, r.rope, *r.place(), at, stride, at + 256 * hq, stride,
                                 at + 256 * (hq + hkv), stride, r.q_out.data_ptr(), stream.cuda_stream)
        args = (r.handle, hq, hkv, 128, 128**-0.5, lens, dlens.data_ptr(), r.dtable.data_ptr(), table.shape[1],
                r.q_out.data_ptr(), out.data_ptr(), ws.data_ptr(), size)
        if four_bit:
            mw.mw_kv4_decode_attn(*args, stream.cuda_stream)
        else:
            mw.mw_decode_attn(*args, 0, stream.cuda_stream)

    try:
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        gen = torch.Generator(device="cuda").manual_seed(9)
        for _ in range(4):
            fresh = torch.randn(r.rows.shape, generator=gen, device="cuda").bfloat16().view(torch.int16)
            r.rows.copy_(fresh)
            out.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()
            torch.cuda.synchronize()
            replayed = R.bits_of(out)
            assert np.isfinite(bits_to_f32(replayed)).all() and replayed.any()
            out.zero_()
            torch.cuda.synchronize()
            step()
            torch.cuda.synchronize()
            assert np.array_equal(R.bits_of(out), replayed)
    finally:
        r.close()


@pytest.mark.parametrize("four_bit", [False, True])
@pytest.mark.parametrize("rot,neighbours", [(128, False), (64, False), (128, True)])
def test_a_call_larger_than_the_caches_as_its_parts(four_bit, rot, neighbours):
    """Rows and queries of more than 128 MB in one call, and as calls of a few sequences each."""
    say(f"norm rope large four_bit={four_bit} rot={rot} neighbours={neighbours}")
    hq, hkv, lens, starts = 64, 4, [1500, 1, 1101, 600, 777], [5, 0, 16, 3, 100]
    whole, parts = (Rows(hq, hkv, lens, starts, four_bit, rot=rot, neighbours=neighbours, seed=17) for _ in range(2))
    assert whole.total * (2 * hq + 2 * hkv) * 256 > 128 << 20
    try:
        whole.run()
        row, stride = 0, parts.rows.shape[1]
        for b in range(len(lens)):
            one = slice(b, b + 1)
            at = parts.rows[row:].data_ptr()
            indptr, start = R.device([0, lens[b]], np.int32), R.device(starts[one], np.int32)
            mw.mw_qk_norm_rope_write(parts.handle, parts.rope, parts.lens[one], parts.starts[one], indptr.data_ptr(),
                                     start.data_ptr(), parts.dtable[b].data_ptr(), parts.table.shape[1], at, stride,
                                     at + 256 * hq, stride, at + 256 * (hq + hkv), stride, parts.q_out[row:].data_ptr())
            row += lens[b]
            torch.cuda.synchronize()
        assert torch.equal(whole.q_out, parts.q_out) and (R.bits_of(whole.q_out[row:]) == 0x1234).all()
        for a, b in zip(whole.cache_rows(), parts.cache_rows()):
            assert np.isfinite(a).all() and np.array_equal(a, b)
    finally:
        whole.close()
        parts.close()
