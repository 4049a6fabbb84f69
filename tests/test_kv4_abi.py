"""The 4-bit pool and the norm and rotation pass without a GPU: argument checks, the shared page allocator, workspace
sizes and struct layout.  No call here launches a kernel."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2504_14489_amd import build as B
from paper_2504_14489_amd import mw

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
K, V, S = 0x10000, 0x20000, 0x30000  # aligned addresses that are never dereferenced


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(mw.LIB_PATH):
        B.build()
    return mw.load()


@pytest.fixture()
def pool4():
    p = mw.mw_kv4_pool_create(10, 16, 2, 128, K, V, S)
    yield p
    mw.mw_kv_pool_destroy(p)


@pytest.fixture()
def pool16():
    p = mw.mw_kv_pool_create(10, 16, 2, 128, K, V)
    yield p
    mw.mw_kv_pool_destroy(p)


def refused(status, call, *args, **kw):
    with pytest.raises(mw.MWError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value
    return e.value.message


def test_create(lib):
    refused(mw.MW_ERR_UNSUPPORTED, mw.mw_kv4_pool_create, 10, 8, 2, 128, K, V, S)
    refused(mw.MW_ERR_UNSUPPORTED, mw.mw_kv4_pool_create, 10, 16, 2, 64, K, V, S)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv4_pool_create, 0, 16, 2, 128, K, V, S)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv4_pool_create, 10, 16, 0, 128, K, V, S)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv4_pool_create, 10, 16, 2, 128, K, V, 0)
    for bad in ((K + 8, V, S), (K, V + 4, S), (K, V, S + 1)):
        assert "aligned" in refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv4_pool_create, 10, 16, 2, 128, *bad)


def test_pages_are_dealt_as_in_a_bf16_pool(pool4):
    assert mw.mw_kv_pool_num_free(pool4) == 10
    mw.mw_kv_pool_set_free_order(pool4, [7, 3])
    assert list(mw.mw_kv_pool_alloc(pool4, 2)) == [7, 3]
    refused(mw.MW_ERR_OUT_OF_PAGES, mw.mw_kv_pool_alloc, pool4, 1)
    mw.mw_kv_pool_free(pool4, [3])
    assert mw.mw_kv_pool_num_free(pool4) == 1


def test_each_kind_of_pool_refuses_the_other_calls(pool4, pool16):
    rows = ([4], [0], 0x100, 0x200, 0x300, 2)
    for call in (mw.mw_kv4_pool_write, mw.mw_kv4_pool_gather):
        assert "bf16" in refused(mw.MW_ERR_INVALID_ARG, call, pool16, *rows, 0x400, 0x500)
    assert "4-bit" in refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv_pool_write, pool4, *rows, 0x400, 0x500)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv_pool_gather, pool4, 0x100, 5, 0x400, 0x500)
    dec = (4, 2, 128, 0.1, [5], 0x100, 0x200, 1, 0x300, 0x400, 0x500, 1 << 24)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv4_decode_attn, pool16, *dec)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_decode_attn, pool4, *dec)
    pre = (4, 2, 128, 0.1, [5], [0], 0x100, 0x200, 0x300, 1, 0x400, 0x500)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_prefill_attn, pool4, *pre)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_prefill_attn_ws, pool4, *pre, 0x600, 1 << 24)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv4_prefill_attn, pool16, *pre, 0x600, 1 << 24)


@pytest.mark.parametrize("call", [mw.mw_kv4_pool_write, mw.mw_kv4_pool_gather])
def test_rows(pool4, call):
    ok = dict(new=[4], start=[0])
    refused(mw.MW_ERR_INVALID_ARG, call, None, [4], [0], 0x100, 0x200, 0x300, 2, 0x400, 0x500)
    for new, start in (([5], [28]), ([-1], [0]), ([1], [-1]), ([33], [0]), ([2**31 - 1], [2**31 - 1])):
        refused(mw.MW_ERR_INVALID_ARG, call, pool4, new, start, 0x100, 0x200, 0x300, 2, 0x400, 0x500)
    for k, v in ((0, 0x500), (0x400, 0), (0x408, 0x500), (0x400, 0x501)):
        refused(mw.MW_ERR_INVALID_ARG, call, pool4, ok["new"], ok["start"], 0x100, 0x200, 0x300, 2, k, v)
    for ip, sp, bt, stride in ((0, 0x200, 0x300, 2), (0x100, 0, 0x300, 2), (0x100, 0x200, 0, 2), (0x100, 0x200, 0x300, 0)):
        refused(mw.MW_ERR_INVALID_ARG, call, pool4, [4], [0], ip, sp, bt, stride, 0x400, 0x500)
    refused(mw.MW_ERR_INVALID_ARG, call, pool4, [0] * 65536, [0] * 65536, 0x100, 0x200, 0x300, 2, 0x400, 0x500)
    # nothing to do is no error, whatever the rows' addresses
    call(pool4, [], [], 0, 0, 0, 2, 0, 0)
    call(pool4, [0, 0], [0, 32], 0x100, 0x200, 0x300, 2, 0, 0)


def test_decode(pool4):
    size = mw.mw_kv4_decode_workspace_size(4, 2, 128, [17])
    assert size == mw.mw_decode_workspace_size(4, 2, 128, [17], 0)

    def call(hq=4, hkv=2, d=128, scale=0.1, lens=(17,), dlens=0x100, bt=0x200, stride=2, q=0x300, out=0x400, ws=0x500,
             n=size):
        mw.mw_kv4_decode_attn(pool4, hq, hkv, d, scale, list(lens), dlens, bt, stride, q, out, ws, n)

    for kw in (dict(lens=(33,)), dict(lens=(0,)), dict(scale=0.0), dict(scale=float("nan")), dict(hq=3),
               dict(hkv=4), dict(n=size - 1), dict(q=0x308), dict(out=0x401), dict(ws=0x508), dict(q=0), dict(dlens=0),
               dict(bt=0), dict(ws=0), dict(stride=0)):
        refused(mw.MW_ERR_INVALID_ARG, call, **kw)
    refused(mw.MW_ERR_UNSUPPORTED, call, d=64)
    refused(mw.MW_ERR_UNSUPPORTED, call, hq=34)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv4_decode_workspace_size, 4, 2, 128, [0])
    refused(mw.MW_ERR_UNSUPPORTED, mw.mw_kv4_decode_workspace_size, 34, 2, 128, [5])


def test_prefill(pool4):
    # a chunk of many rows is unpacked: pages of two heads and a table of two rows
    new, prefix = [1000, 3], [0, 40]
    size = mw.mw_kv4_prefill_workspace_size(4, 2, 128, new, prefix)
    assert size >= 2 * 66 * 2 * 4096 + 2 * 63 * 4
    # of few rows over few keys it needs nothing, over many its pieces' sums
    few = mw.mw_kv4_prefill_workspace_size(4, 2, 128, [20, 3], [4000, 40])
    assert mw.mw_kv4_prefill_workspace_size(4, 2, 128, [20, 3], [0, 40]) == 0
    assert few > 0 and few % 520 == 0
    for cus in (0, 32, 256):
        assert mw.mw_kv4_prefill_workspace_size(4, 2, 128, [20, 3], [4000, 40], cus) == few
    # long lengths are sized in 64 bits
    far = mw.mw_kv4_prefill_workspace_size(64, 8, 128, [4096] * 64, [100000] * 64)
    assert far >= 2 * 64 * ((104096 + 15) // 16) * 8 * 4096 > 1 << 32

    def call(hq=4, hkv=2, d=128, scale=0.1, new=new, prefix=prefix, ip=0x100, pl=0x200, bt=0x300, stride=500, q=0x400,
             out=0x500, ws=0x600, n=size):
        mw.mw_kv4_prefill_attn(pool4, hq, hkv, d, scale, new, prefix, ip, pl, bt, stride, q, out, ws, n)

    shapes = ((new, prefix, 2 * 66 * 2 * 4096), ([20, 3], [4000, 40], few - 1))
    for new_, prefix_, short in shapes:
        for kw in (dict(new=[20, 8000]), dict(new=[-1, 3]), dict(prefix=[-1, 40]), dict(scale=0.0), dict(hkv=4),
                   dict(hq=3), dict(ws=0), dict(ws=0x608), dict(n=short), dict(n=0), dict(q=0x408), dict(out=0),
                   dict(ip=0), dict(bt=0), dict(stride=0), dict(stride=2)):
            refused(mw.MW_ERR_INVALID_ARG, call, **(dict(new=new_, prefix=prefix_) | kw))
    refused(mw.MW_ERR_UNSUPPORTED, call, d=64)
    refused(mw.MW_ERR_INVALID_ARG, mw.mw_kv4_prefill_workspace_size, 4, 2, 128, [5], [-3])
    call(new=[0, 0], prefix=[0, 0], ws=0, n=0)    # nothing to do


@pytest.mark.parametrize("kind", ["pool4", "pool16"])
def test_norm_rope(kind, request):
    pool = request.getfixturevalue(kind)

    def call(hq=4, rot=128, eps=1e-6, qw=0x100, kw=0x200, freq=0x300, new=(4,), start=(0,), ip=0x400, sp=0x500,
             bt=0x600, stride=2, q=0x700, qs=512, k=0x800, ks=256, v=0x900, vs=256, out=0xA00):
        rope = mw.NormRope(num_q_heads=hq, rot_dim=rot, neighbours=0, eps=eps, d_q_weight=qw, d_k_weight=kw,
                           d_inv_freq=freq)
        mw.mw_qk_norm_rope_write(pool, rope, list(new), list(start), ip, sp, bt, stride, q, qs, k, ks, v, vs, out)

    for kw_ in (dict(hq=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(qw=0x108),
                dict(kw=0x201), dict(freq=0), dict(freq=0x304), dict(q=0), dict(q=0x708), dict(qs=511), dict(qs=504),
                dict(qs=516), dict(ks=128), dict(vs=-256), dict(k=0), dict(v=0x902), dict(out=0), dict(out=0xA08),
                dict(new=(33,)), dict(start=(-1,)), dict(new=(5,), start=(28,)), dict(ip=0), dict(bt=0), dict(stride=0)):
        refused(mw.MW_ERR_INVALID_ARG, call, **kw_)
    for rot in (-16, 8, 24, 144):
        refused(mw.MW_ERR_UNSUPPORTED, call, rot=rot)
    call(new=(0,), q=0, k=0, v=0, out=0)          # nothing to do
    with pytest.raises(mw.MWError):
        mw._check(mw.load().mw_qk_norm_rope_write(pool, None, 0, None, None, 0, 0, 0, 1, 0, 0, 0, 0, 0, 0, 0, 0, None))


def test_struct_layout(tmp_path):
    fields = [f for f, _ in mw.NormRope._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mw.h"\nint main(void) {\n'
                   'printf("%zu", sizeof(mw_norm_rope));\n'
                   + "".join(f'printf(" %zu", offsetof(mw_norm_rope, {f}));\n' for f in fields) + "return 0; }")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(mw.NormRope)] + [getattr(mw.NormRope, f).offset for f in fields]


def test_reference_rounds_within_half_a_step():
    """The tests' own quantiser keeps every value within half of its step: of the magnitudes' spacing at the value's
    size, one unit at the most."""
    from tests import kv4_reference as R
    rng = np.random.Generator(np.random.PCG64(1))
    x = R.f32_to_bf16_bits((rng.standard_normal((200, 128)) * np.exp2(rng.integers(-90, 90, (200, 1)))).astype(np.float32))
    code, scale = R.quantise(x)
    value = R.bits_to_f32(x).astype(np.float64)
    unit = np.repeat(np.exp2(scale.astype(np.float64) - 127), 32, axis=-1)
    a = np.abs(value) / unit
    step = np.where(a < 2, 0.5, np.where(a < 4, 1, 2))
    assert a.max() <= 7
    assert (np.abs(R.values(code, scale) - value) / unit <= step / 2).all()
