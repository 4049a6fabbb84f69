"""Attention over the cache in 4 bits where scores are far beyond the exponential's range, by value: queries that the two
8-bit parts hold exactly, so that the scores' own roundings are all that is left to allow for."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_14489_amd.device import bits_to_f32
from paper_2504_14489_amd.workloads import f32_to_bf16_bits
from tests import kv4_reference as R
from tests.helpers import say
from tests.test_gpu_kv4 import SCALE, Decode, Prefill

pytestmark = pytest.mark.gpu


def set_queries(call, numbers):
    call.q = f32_to_bf16_bits(numbers.astype(np.float32))
    assert np.array_equal(bits_to_f32(call.q), numbers.astype(np.float32))  # exact in bf16
    call.dq[:len(numbers)].copy_(R.device(call.q.view(np.int16)))


def rows_of(call):
    """(sequence, query row, keys it sees) of each row of the call."""
    if isinstance(call, Decode):
        return [(b, b, int(n)) for b, n in enumerate(call.lens)]
    out, row = [], 0
    for b, (n, r) in enumerate(zip(call.new, call.prefix)):
        out += [(b, row + i, r + i + 1) for i in range(n)]
        row += n
    return out


def held(call):
    """K and V of the pool, fp64 [pages, hkv, 16, 128], what is not finite as zeros."""
    k, v = (bits_to_f32(x).astype(np.float64) for x in call.pool.bf16())
    return np.where(np.isfinite(k), k, 0), np.where(np.isfinite(v), v, 0)


def made(kind, seed):
    if kind == "decode":
        return Decode(12, 2, [1, 33, 500, 2100], seed=seed)
    return Prefill(12, 2, [5, 40, 1], [2100, 33, 0], seed=seed)


@pytest.mark.parametrize("kind", ["decode", "prefill"])
@pytest.mark.parametrize("gain", [1, 2**7, 2**14, 2**20])
def test_the_key_that_a_query_is_made_of_wins(kind, gain):
    """A head's query is a key of its sequence times a power of two: from a gain of 128 on every other key's weight is
    below 2^-100 and the output is the value of that key, rounded as the output and one probability are (2^-8 each at
    most, half a step, together 2^-7)."""
    say(f"kv4 {kind} winner gain={gain}")
    call = made(kind, 81)
    k, v = held(call)
    rng = np.random.Generator(np.random.PCG64(gain))
    group = call.hq // call.hkv
    q = np.zeros(call.q.shape)
    want = np.zeros(call.q.shape)
    ahead = np.inf
    for b, row, seen in rows_of(call):
        at = np.arange(seen)
        keys, values = k[call.table[b, at // 16], :, at % 16], v[call.table[b, at // 16], :, at % 16]  # [seen, hkv, 128]
        for h in range(call.hq):
            # (one of the longest tenth, so that no other key has the larger product)
            longest = np.argsort((keys[:, h // group]**2).sum(-1))[-max(1, seen // 10):]
            j = int(rng.choice(longest))
            q[row, h] = gain * keys[j, h // group]
            s = SCALE * keys[:, h // group] @ q[row, h] * np.log2(np.e)
            want[row, h] = values[j, h // group]
            if seen > 1:
                ahead = min(ahead, s[j] - np.delete(s, j).max())
    set_queries(call, q)
    try:
        call.run()
        torch.cuda.synchronize()
        got = bits_to_f32(R.bits_of(call.out))[:len(q)].astype(np.float64)
        if gain == 1:
            assert (np.abs(got - oracle_of(call)[0]) <= R.attention_bound(call.q, k, *oracle_of(call), SCALE)).all()
            return
        assert ahead > 100, ahead
        worst = float((np.abs(got - want) / (2.0**-7 * np.abs(want) + 1e-25)).max())
        say(f"  ahead by 2^{ahead:.0f}, worst error / bound {worst:.3f}")
        assert worst <= 1, worst
    finally:
        call.pool.close()


def oracle_of(call):
    """The call's outputs in fp64, and those with |V|."""
    k, v = (f32_to_bf16_bits(x.astype(np.float32)) for x in held(call))
    out = []
    for value in (v, v & 0x7FFF):
        if isinstance(call, Decode):
            out.append(oracle.decode(call.q, k, value, call.table, call.lens))
            continue
        parts, row = [], 0
        for b, (n, r) in enumerate(zip(call.new, call.prefix)):
            parts.append(oracle.prefill(call.q[row:row + n], k, value, call.table[b], r))
            row += n
        out.append(np.concatenate(parts))
    return out


@pytest.mark.parametrize("kind", ["decode", "prefill"])
@pytest.mark.parametrize("gain", [2.0**-6, 1.0, 2.0**3])
def test_whole_queries(kind, gain):
    """Whole numbers up to 255 times a power of two, scores up to several thousand.  With S the largest sum of
    |q k| scale over the keys, the scores are off by S 2^-20 for the fp32 sums of 2 * 128 products and S 2^-21 for the five
    roundings of scale, log2(e), their product, the reference maximum and the exponent: d <= S 2^-19, and every weight
    by a factor within e^(+-2 d).  Output and probabilities are rounded to bf16 (2^-8 each at most), the sums in fp32
    (2^-14).  The bound stays below a tenth of the values'; outputs that are weights of e^-69 and less, where fp64 keeps
    what fp32 cannot, are not told from zero (1e-30)."""
    say(f"kv4 {kind} whole queries gain={gain}")
    call = made(kind, 83)
    rng = np.random.Generator(np.random.PCG64(85))
    q = rng.integers(-255, 256, call.q.shape).astype(np.float64)
    q[..., 0] = 255  # the row's largest: its unit is 1
    set_queries(call, gain * q)
    k, _ = held(call)
    largest = SCALE * gain * (np.abs(q).reshape(-1, 128) @ np.abs(k).reshape(-1, 128).T).max()
    factor = np.expm1(2 * largest * 2.0**-19)
    assert factor < 0.1
    try:
        call.run()
        torch.cuda.synchronize()
        got = bits_to_f32(R.bits_of(call.out))[:len(q)].astype(np.float64)
        ref, ref_abs = oracle_of(call)
        bound = 2.0**-8 * np.abs(ref) + (2.0**-8 + 2.0**-14 + factor) * (1 + 2.0**-7) * ref_abs + 1e-30
        worst = float((np.abs(got - ref) / bound).max())
        say(f"  scores up to {largest:.0f}, worst error / bound {worst:.3f}")
        assert worst <= 1, worst
    finally:
        call.pool.close()
