"""Norm and rotation on rows of every size that bf16 has, whose squares leave the range of fp32 on either side."""
import numpy as np
import pytest
import torch

from paper_2504_14489_amd import mw
from paper_2504_14489_amd.device import bits_to_f32
from tests import kv4_reference as R
from tests.helpers import say
from tests.test_gpu_norm_rope import Rows, formula

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-6, 1e30])
@pytest.mark.parametrize("exponents", [(-133, -110), (-80, -60), (-50, -40), (50, 62), (62, 66), (80, 120), (-133, 124)])
@pytest.mark.parametrize("rot,neighbours", [(128, False), (64, False), (128, True)])
def test_rows_of_any_size(exponents, eps, rot, neighbours):
    """Each head row has a power of two of its own.  Bound as for ordinary rows: 2^-8 of the value for the rounding to
    bf16 (half a step), 2^-18 of the pair's size for fp32's sums, root, products, cosine and sine, and half a step of the
    smallest bf16 numbers, 2^-134, for outputs below the normal ones."""
    say(f"norm of rows 2^{exponents} eps={eps} rot={rot} neighbours={neighbours}")
    r = Rows(4, 2, [5, 30], [3, 1000], False, rot=rot, neighbours=neighbours, seed=3)
    try:
        rng = np.random.Generator(np.random.PCG64(5))
        x = rng.standard_normal((35, 8, 128)) * np.exp2(rng.integers(exponents[0], exponents[1] + 1, (35, 8, 1)).astype(float))
        with np.errstate(under="ignore"):
            r.x = R.f32_to_bf16_bits(x.astype(np.float32))
        r.rows.copy_(R.device(r.x.reshape(35, -1).view(np.int16)))
        r.rope.eps = eps
        r.run()
        torch.cuda.synchronize()
        x = bits_to_f32(r.x).astype(np.float64)
        assert np.isfinite(x).all() and (np.abs(x).max(-1) > 0).all()
        half = rot // 2
        one, two = ((slice(0, rot, 2), slice(1, rot, 2)) if neighbours else (slice(0, half), slice(half, rot)))
        eps32 = float(np.float32(eps))
        for rows, weight, got in ((x[:, :4], r.w[0], bits_to_f32(R.bits_of(r.q_out))[:35]), (x[:, 4:6], r.w[1], r.cache_rows()[0])):
            want = formula(rows, bits_to_f32(weight).astype(np.float64), r.positions, r.inv_freq, neighbours, eps32)
            size = np.abs(want)
            size[..., one] = size[..., two] = np.hypot(want[..., one], want[..., two])
            bound = 2.0**-8 * np.abs(want) + 2.0**-18 * size + 2.0**-134
            worst = np.abs(got.astype(np.float64) - want) / bound
            assert worst.max() <= 1, (float(worst.max()), np.argwhere(~(worst <= 1))[:3])
        assert np.array_equal(r.cache_rows()[1], bits_to_f32(r.x[:, 6:]).astype(np.float64))  # values as they were
    finally:
        torch.cuda.synchronize()
        mw.mw_kv_pool_destroy(r.handle)


@pytest.mark.parametrize("position", [1, 37, 1000, 30001])
@pytest.mark.parametrize("neighbours", [False, True])
def test_cosine_and_sine_near_their_zeros(position, neighbours):
    """Pairs (1, 0) become (cos, sin); the angles are whole, half and quarter turns, off by 2^-8 to 2^-22 of a half turn.
    The angle's product in fp64 is off by 2^-51 of it (3 roundings), below 2^-34 for up to 2^14 turns and 2^-11 of the
    smallest value; what is computed in fp32 is off by less than 2^-20 of the value; the output's rounding by 2^-8."""
    say(f"rotation near the zeros at {position}, neighbours={neighbours}")
    r = Rows(4, 2, [1], [position], False, norm=False, neighbours=neighbours, seed=9)
    try:
        rng = np.random.Generator(np.random.PCG64(position))
        off = np.exp2(rng.uniform(-22, -8, 64)) * rng.choice([-1, 1], 64)
        half_turns = rng.integers(1, 2 * position + 1, 64) * 0.5 + off  # up to half a turn a position
        freq = half_turns * np.pi / position
        r.dfreq.copy_(torch.from_numpy(freq))
        x = np.zeros((1, 8, 128))
        x[..., (slice(0, 128, 2) if neighbours else slice(0, 64))] = 1
        r.rows.copy_(R.device(R.f32_to_bf16_bits(x.astype(np.float32)).reshape(1, -1).view(np.int16)))
        r.run()
        torch.cuda.synchronize()
        # the angle as the frequencies give it, in extended precision
        angle = np.longdouble(freq) * np.longdouble(position)
        turn = 2 * np.longdouble("3.14159265358979323846264338327950288")
        angle = angle - np.rint(angle / turn) * turn
        want = np.zeros(128)
        one, two = ((slice(0, 128, 2), slice(1, 128, 2)) if neighbours else (slice(0, 64), slice(64, 128)))
        want[one], want[two] = np.cos(angle), np.sin(angle)
        assert 2.0**-22 < np.abs(want).min() < 2.0**-12
        got = bits_to_f32(R.bits_of(r.q_out))[0].astype(np.float64)
        bound = (2.0**-8 + 2.0**-20) * np.abs(want) + 2.0**-33
        assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
    finally:
        torch.cuda.synchronize()
        mw.mw_kv_pool_destroy(r.handle)
