"""Rows at the last positions that a 32-bit length can name, 2^31 - 2 and before, through the append and read-back in 4 bits
and the norm and rotation pass into both kinds of pool."""
import numpy as np
import pytest
import torch

from paper_2504_14489_amd import mw
from paper_2504_14489_amd.device import bits_to_f32
from tests import kv4_reference as R
from tests.helpers import say
from tests.test_gpu_kv4 import normal_bits
from tests.test_gpu_norm_rope import Rows

pytestmark = pytest.mark.gpu

LAST = 2**31 - 1  # the most tokens of a sequence


@pytest.mark.parametrize("n", [1, 3, 37])
def test_append_and_read_back(n):
    say(f"kv4 append of {n} rows before position 2^31 - 1")
    hkv, rng = 2, np.random.Generator(np.random.PCG64(n))
    start, stride = LAST - n, 1 << 27
    first = start // 16
    pool = R.Pool4(stride - first + 1, hkv, seed=n)
    table = torch.full((1, stride), -1, dtype=torch.int32, device="cuda")
    pages = rng.permutation(stride - first).astype(np.int32)
    table[0, first:] = R.device(pages)
    k, v = normal_bits(rng, n, hkv, 128), normal_bits(rng, n, hkv, 128)
    dk, dv = R.device(k.view(np.int16)), R.device(v.view(np.int16))
    indptr, dstart = R.device([0, n], np.int32), R.device([start], np.int32)
    where = ([n], [start], indptr.data_ptr(), dstart.data_ptr(), table.data_ptr(), stride)
    ko, vo = torch.full_like(dk, 77), torch.full_like(dv, 77)
    try:
        mw.mw_kv4_pool_write(pool.handle, *where, dk.data_ptr(), dv.data_ptr())
        mw.mw_kv4_pool_gather(pool.handle, *where, ko.data_ptr(), vo.data_ptr())
        torch.cuda.synchronize()
        for rows, out, code, scale in ((k, ko, pool.kc, pool.ks), (v, vo, pool.vc, pool.vs)):
            c, s = R.quantise(rows)
            for i in range(n):
                page, slot = pages[(start + i) // 16 - first], (start + i) % 16
                code[page, :, slot], scale[page, :, slot] = c[i], s[i]
            assert np.array_equal(bits_to_f32(R.bits_of(out)), R.values(c, s).astype(np.float32))
        assert np.array_equal(pool.k4.cpu().numpy(), R.pack_k(pool.kc))
        assert np.array_equal(pool.v4.cpu().numpy(), R.pack_v(pool.vc))
        assert np.array_equal(pool.scales.cpu().numpy(), R.pack_scales(pool.ks, pool.vs))
    finally:
        pool.close()


@pytest.mark.parametrize("four_bit", [False, True])
@pytest.mark.parametrize("n", [1, 21])
def test_norm_rotation_and_append(four_bit, n):
    say(f"norm and rotation of {n} rows before position 2^31 - 1, four_bit={four_bit}")
    r = Rows(4, 2, [n], [LAST - n], four_bit, seed=n)
    assert r.table.shape == (1, 1 << 27)
    try:
        r.run()
        r.check()
    finally:
        torch.cuda.synchronize()
        mw.mw_kv_pool_destroy(r.handle)
