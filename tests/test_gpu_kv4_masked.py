"""Values that are not finite at positions that a row does not see, in the prefill over the cache in 4 bits: 0 times NaN must
not reach the row through the others of its block."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_14489_amd import mw
from paper_2504_14489_amd.device import bits_to_f32
from tests import kv4_reference as R
from tests.helpers import say
from tests.test_gpu_kv4 import SCALE, Prefill

pytestmark = pytest.mark.gpu

# (heads, new and prefix lengths, bad V blocks as (sequence, position, kv head, block of 32 dims)): blocks of a wave's 32
# rows that span one position to 32, in one key tile and in two; one piece and several; rows behind the bad position in
# the same tile, in the next and in both; the last position; several bad blocks; a chunk that begins inside a page; straight from the codes, and (the last ones)
# unpacked first, where the block may be one of the prefix's
CASES = [
    (2, 2, [100], [0], [(0, 70, 0, 1)]),
    (2, 2, [100], [0], [(0, 70, 0, 1), (0, 64, 1, 3), (0, 99, 1, 0)]),
    (2, 2, [90], [45], [(0, 66, 1, 2), (0, 130, 0, 0)]),
    (4, 2, [60], [50], [(0, 64, 0, 0), (0, 63, 1, 1), (0, 109, 0, 2)]),
    (3, 1, [42], [7], [(0, 20, 0, 0), (0, 21, 0, 1), (0, 48, 0, 2)]),
    (8, 2, [33, 40], [60, 130], [(0, 70, 0, 3), (1, 150, 1, 0), (1, 168, 1, 1)]),
    (8, 2, [70], [3000], [(0, 3001, 0, 0), (0, 3040, 1, 1), (0, 3069, 0, 2)]),
    (2, 2, [120, 5], [2500, 2000], [(0, 2560, 0, 0), (0, 2550, 1, 2), (1, 2004, 0, 3)]),
    (16, 1, [16], [8000], [(0, 8001, 0, 0), (0, 8015, 0, 1)]),
    (32, 8, [1, 20], [5000, 11], [(0, 5000, 7, 2), (1, 12, 0, 1), (1, 30, 3, 0)]),
    (12, 2, [250, 3] + [1] * 30, [100] * 32, [(0, 200, 0, 0), (0, 349, 1, 3), (1, 101, 1, 1), (9, 100, 0, 2)]),
    (2, 2, [1300], [0], [(0, 70, 0, 1), (0, 1000, 0, 1), (0, 1299, 1, 3), (0, 640, 1, 0)]),
    (8, 1, [300, 5, 0, 129], [77, 1000, 40, 15], [(0, 70, 0, 2), (0, 77, 0, 0), (0, 200, 0, 1), (1, 1003, 0, 3), (3, 15, 0, 0), (3, 143, 0, 1)]),
    (32, 8, [2, 700], [5000, 300], [(0, 5001, 7, 2), (1, 310, 3, 0), (1, 420, 3, 0), (1, 999, 0, 1), (1, 200, 5, 3)]),
]


@pytest.mark.parametrize("hq,hkv,new,prefix,bad", CASES)
def test_values_of_later_positions(hq, hkv, new, prefix, bad):
    """Each bad block of V makes its 32 dims NaN in the rows of its heads from its position on; everything else is the
    attention without it.  The codes beside a scale of 255 are the largest ones."""
    say(f"kv4 few rows later values {hq}/{hkv} new={new[:4]} prefix={prefix[:4]}")
    p = Prefill(hq, hkv, new, prefix, seed=hq + sum(new) + len(bad))
    timing = mw.mw_timing_create()
    for b, pos, kvh, blk in bad:
        page = p.table[b, pos // 16]
        p.pool.vs[page, kvh, pos % 16, blk] = 255
        p.pool.vc[page, kvh, pos % 16, 32 * blk:32 * blk + 32] = 7
    mw.mw_kv_pool_destroy(p.pool.handle)
    p.pool.upload()
    try:
        p.run(timing=timing)
        torch.cuda.synchronize()
        # a kernel or two straight from the codes; unpacking, the attention's one or two and what follows them
        few = max(new) * hq // hkv <= 1024
        assert mw.mw_timing_kernels(timing) in ((1,) if p.size == 0 else (2,) if few else (3, 4))
        got = bits_to_f32(R.bits_of(p.out)).astype(np.float64)
        k, v = p.pool.bf16()
        k[~np.isfinite(bits_to_f32(k))] = 0
        v[~np.isfinite(bits_to_f32(v))] = 0
        group, row = hq // hkv, 0
        for b, (n, r) in enumerate(zip(new, prefix)):
            if n == 0:
                continue
            want = np.zeros((n, hq, 128), bool)
            for at, pos, kvh, blk in bad:
                if at == b:
                    want[max(pos - r, 0):, kvh * group:(kvh + 1) * group, 32 * blk:32 * blk + 32] = True
            out, q = got[row:row + n], p.q[row:row + n]
            assert np.array_equal(np.isnan(out), want), (b, np.argwhere(np.isnan(out) != want)[:4])
            ref = oracle.prefill(q, k, v, p.table[b], r)
            bound = R.attention_bound(q, bits_to_f32(k), ref, oracle.prefill(q, k, v & 0x7FFF, p.table[b], r), SCALE)
            assert (np.abs(out - ref)[~want] <= bound[~want]).all(), b
            row += n
    finally:
        mw.mw_timing_destroy(timing)
        p.close()
