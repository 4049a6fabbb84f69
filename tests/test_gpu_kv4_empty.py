"""Sequences without new tokens in a prefill batch over the cache in 4 bits that is unpacked first: none of their pages is."""
import pytest

from tests.helpers import say
from tests.test_gpu_kv4 import Prefill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,prefix", [
    ([300, 0, 0, 200], [100, 5000, 0, 31]), ([0, 0, 257], [16, 3000, 1000]), ([400] + [0] * 70, [33] + list(range(0, 1400, 20))),
    ([0, 1, 0, 500, 0], [700, 700, 700, 0, 2000]),
])
def test_empty_sequences_beside_unpacked_ones(new, prefix):
    """Every row against the oracle, in a workspace of the size call's bytes and not one more."""
    say(f"kv4 prefill with empty sequences new={new[:5]} prefix={prefix[:5]}")
    p = Prefill(8, 1, new, prefix, seed=len(new) + sum(new))
    try:
        assert p.size < 2 * 8192 * sum((n + r + 15) // 16 for n, r in zip(new, prefix) if n) + (8 << 20)
        p.run()
        p.check()
    finally:
        p.close()
