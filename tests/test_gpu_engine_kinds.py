"""The engine, the fused launch and the decode that allocates nothing are for bf16 pools: pools in 4 bits are refused before
anything runs."""
import pytest
import torch

from paper_2504_14489_amd import mw, workloads as W
from paper_2504_14489_amd.device import DeviceWorkload
from paper_2504_14489_amd.engine import Engine
from tests.helpers import say

pytestmark = pytest.mark.gpu


def refused(call, *args, **kw):
    with pytest.raises(mw.MWError) as e:
        call(*args, **kw)
    assert e.value.status == mw.MW_ERR_INVALID_ARG and "4-bit" in e.value.message, e.value


def test_pools_in_4_bits_are_refused():
    say("engine, fused and no-allocation calls on a pool in 4 bits")
    cfg = W.custom_config("kinds", hq=8, hkv=2, pre_chunks=((0, 200),), dec_batch=6, dec_len_lo=100, dec_len_hi=900)
    dw = DeviceWorkload(W.make_workload(cfg, seed=3))
    eng = Engine([64])
    codes = torch.zeros(3, 64, 2, 1024, dtype=torch.uint8, device="cuda")
    four = mw.mw_kv4_pool_create(64, 16, 2, 128, *(t.data_ptr() for t in codes))
    try:
        dec, pre = dw.engine_args()
        dw.o_dec.fill_(7)
        dw.o_pre.fill_(7)
        torch.cuda.synchronize()
        dec4, pre4 = dict(dec, pool=four), dict(pre, pool=four)
        for d, p in ((dec4, pre), (dec, pre4), (dec4, pre4)):
            for graph in (False, True):
                refused(eng.run, d, p, config=0, decode_iters=2, decode_layers=2, prefill_layers=2, layers_per_launch=1,
                        decode_graph=graph)
        refused(mw.mw_fused_attn, pre4, dec4)
        refused(mw.mw_decode_attn_noalloc, four, dw.hq, dw.hkv, dw.d, dw.scale, dw.dec_lens, dec["d_seq_lens"],
                dec["d_block_table"], dec["bt_stride"], dec["d_q"], dec["d_out"])
        torch.cuda.synchronize()
        assert (dw.o_dec == 7).all() and (dw.o_pre == 7).all()
        # and the engine still runs
        eng.run(dec, pre, config=0, decode_iters=2, decode_layers=2, prefill_layers=2, layers_per_launch=1, decode_graph=True)
        assert not (dw.o_dec == 7).all() and not (dw.o_pre == 7).all()
    finally:
        torch.cuda.synchronize()
        mw.mw_kv_pool_destroy(four)
        eng.close()
        dw.close()
