"""The host side of the calls on a pool in 4 bits at their limits, without a GPU: no call here launches a kernel."""
import os
import shutil
import subprocess

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


@pytest.fixture(params=[4, 16])
def pool(request):
    p = mw.mw_kv4_pool_create(10, 16, 2, 128, K, V, S) if request.param == 4 else mw.mw_kv_pool_create(10, 16, 2, 128, K, V)
    p.bits = request.param
    yield p
    mw.mw_kv_pool_destroy(p)


@pytest.mark.parametrize("new,start", [([1], [2**31 - 1]), ([2**31 - 1], [1]), ([4, 3], [0, 2**31 - 3])])
def test_rows_past_the_longest_sequence_are_refused(pool, new, start):
    """A sequence of 2^31 tokens and more has no 32-bit length, however long its table is."""
    place = (new, start, 0x100, 0x200, 0x300, 1 << 28)
    rope = mw.NormRope(num_q_heads=4, rot_dim=0, neighbours=0, eps=0.0, d_q_weight=0, d_k_weight=0, d_inv_freq=0)
    calls = [lambda: mw.mw_qk_norm_rope_write(pool, rope, *place, 0x400, 1024, 0x800, 1024, 0xA00, 1024, 0xC00)]
    if pool.bits == 4:
        calls += [lambda: mw.mw_kv4_pool_write(pool, *place, 0x400, 0x500), lambda: mw.mw_kv4_pool_gather(pool, *place, 0x400, 0x500)]
    else:
        calls += [lambda: mw.mw_kv_pool_write(pool, *place, 0x400, 0x500)]
    for call in calls:
        with pytest.raises(mw.MWError) as e:
            call()
        assert e.value.status == mw.MW_ERR_INVALID_ARG and "32-bit" in e.value.message


@pytest.mark.parametrize("hq,hkv,new,prefix", [(32, 8, [1000], [0]), (8, 1, [300, 2], [77, 4000])])
def test_sequences_without_new_tokens_need_no_workspace(hq, hkv, new, prefix):
    """Beside unpacked ones, whatever their prefix: a row each in the table of pages is all that they add."""
    size = mw.mw_kv4_prefill_workspace_size(hq, hkv, 128, new, prefix)
    assert size > 4 << 20
    longest = max((n + r + 15) // 16 for n, r in zip(new, prefix))
    more = mw.mw_kv4_prefill_workspace_size(hq, hkv, 128, new + [0] * 31, prefix + [30000] * 31)
    assert size <= more <= size + 31 * 4 * longest + 256
    # by themselves they need nothing, and are no reason to refuse a batch
    assert mw.mw_kv4_prefill_workspace_size(hq, hkv, 128, [0] * 4, [30000] * 4) == 0
    far = [2**31 - 100] * 64
    assert mw.mw_kv4_prefill_workspace_size(hq, hkv, 128, [0] * 64, far) == 0
    assert mw.mw_kv4_prefill_workspace_size(hq, hkv, 128, new + [0] * 64, prefix + far) <= size + 64 * 4 * longest + 256


def test_prefill_allocates_nothing(tmp_path):
    """Calls that end on the host (nothing to do, a workspace too small) make as many allocations as those on a bf16 pool,
    which make none of their own: a handle of a pool, of a queue and an array, is two."""
    if not shutil.which("g++"):
        pytest.skip("g++ not found")
    src = tmp_path / "allocations.cpp"
    src.write_text(r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <new>
#include "mw.h"
static long g_count = 0;
void *operator new(std::size_t n) { ++g_count; return std::malloc(n ? n : 1); }
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
alignas(256) static unsigned char fake[4096];  // stands in for device buffers: never dereferenced
int main() {
    const mw_kv_pool_desc desc{64, 16, 2, 128};
    mw_kv_pool *p16, *p4;
    if (mw_kv_pool_create(&desc, fake, fake, &p16) || mw_kv4_pool_create(&desc, fake, fake, fake, &p4)) return 1;
    const mw_attn_shape shape{8, 2, 128, 0.1f};
    int32_t *const d = reinterpret_cast<int32_t *>(fake);
    const int32_t none[2] = {0, 0}, some[2] = {20, 3}, many[2] = {700, 3}, prefix[2] = {4000, 40};
    for (int i = 0; i < 4; ++i) {
        const long a = g_count;
        mw_status st = mw_prefill_attn_ws(p16, &shape, 2, none, prefix, d, d, d, 500, fake, fake, fake, 0, nullptr, nullptr);
        const long b = g_count;
        if (st != MW_OK) return 2;
        std::printf("%ld", b - a);
        for (const int32_t *n : {none, some, many}) {
            const long c = g_count;
            st = mw_kv4_prefill_attn(p4, &shape, 2, n, prefix, d, d, d, 500, fake, fake, fake, 0, nullptr, nullptr);
            if (st != (n == none ? MW_OK : MW_ERR_INVALID_ARG)) return 3;
            std::printf(" %ld", g_count - c);
        }
        std::printf("\n");
    }
}
""")
    exe, where = str(tmp_path / "allocations"), os.path.dirname(mw.LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), str(src), mw.LIB_PATH, "-o", exe,
                    f"-Wl,-rpath,{where}:/opt/rocm/lib", "-Wl,--allow-shlib-undefined", "-rdynamic"], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, (res.returncode, res.stderr)
    # the first call of the process may set up the HIP runtime
    for bf16, *four in [[int(x) for x in line.split()] for line in res.stdout.splitlines()][1:]:
        assert max(four) <= bf16, res.stdout
