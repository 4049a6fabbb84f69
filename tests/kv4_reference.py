"""The 4-bit cache's definition in numpy and fp64, and pools built from it: what the kernels are compared with.

A block of 32 dims has the exponent e = smallest integer with max|x| <= 7 * 2^e, kept in [-100, 100]; a value becomes
the nearest of the format's magnitudes times 2^e, ties to the even mantissa, at most 6 * 2^e.
"""
import math

import numpy as np
import torch

from paper_2504_14489_amd import mw
from paper_2504_14489_amd.device import bits_to_f32
from paper_2504_14489_amd.workloads import f32_to_bf16_bits

PAGE, DIM, BLOCKS = 16, 128, 4
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
# between magnitude i and i + 1: the border, and whether the border itself goes up (to the even mantissa)
BORDERS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))


def quantise(bits):
    """bf16 bits [..., 128] -> (codes uint8 [..., 128], scale bytes uint8 [..., 4])."""
    with np.errstate(invalid="ignore"):  # (signalling NaNs)
        x = bits_to_f32(bits).astype(np.float64).reshape(*bits.shape[:-1], BLOCKS, 32)
    finite = np.isfinite(x).all(-1)
    most = np.abs(np.where(finite[..., None], x, 0)).max(-1)
    with np.errstate(divide="ignore"):
        e = np.clip(np.ceil(np.log2(most / 7)), -100, 100)  # a bf16 value over 7 is a power of two or well off one
    unit = np.where(finite, np.exp2(e), 1)[..., None]
    a = np.where(finite[..., None], np.abs(x), 0) / unit
    code = np.zeros(x.shape, np.uint8)
    for border, up in BORDERS:
        code += (a >= border) if up else (a > border)
    code |= np.where(finite[..., None] & np.signbit(x), 8, 0).astype(np.uint8)
    return code.reshape(bits.shape), np.where(finite, e + 127, 255).astype(np.uint8)


def values(code, scale):
    """The numbers held, fp64; NaN where the scale byte is 255."""
    unit = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    number = MAGNITUDES[code & 7] * np.where(code & 8, -1.0, 1.0)
    return (number.reshape(*code.shape[:-1], BLOCKS, 32) * unit[..., None]).reshape(code.shape)


def pack_k(code):
    """[P, hkv, 16, 128] codes -> [P, hkv, 16, 64] bytes."""
    return code[..., 0::2] | (code[..., 1::2] << 4)


def pack_v(code):
    """[P, hkv, 16, 128] codes -> [P, hkv, 4, 16, 8, 2] bytes, one code at a time."""
    out = np.zeros((*code.shape[:2], 4, 16, 8, 2), np.uint8)
    for token in range(PAGE):
        g, k, n = token // 4, token % 4 // 2, token % 2
        for dim in range(DIM):
            t, c = 2 * (dim // 32) + dim % 2, dim % 32 // 2
            out[:, :, g, c, t, k] |= code[:, :, token, dim] << (4 * n)
    return out


def pack_scales(k_scale, v_scale):
    """Two [P, hkv, 16, 4] -> [P, hkv, 2, 4, 16]."""
    return np.stack([np.swapaxes(k_scale, -1, -2), np.swapaxes(v_scale, -1, -2)], axis=2)


def as_bf16(numbers):
    """Held values as bf16 bits (exact: two bits of significand and an exponent in range)."""
    bits = f32_to_bf16_bits(numbers.astype(np.float32))
    fine = np.isfinite(numbers)
    assert np.array_equal(bits_to_f32(bits)[fine].astype(np.float64), numbers[fine])
    return bits


def device(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype))).cuda()


def bits_of(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


class Pool4:
    """A 4-bit pool on the GPU, filled from N(0, 1) rows through the reference, with its values as bf16 pools for the
    oracle.  ``slack`` bytes fill never-used pages (codes and scales): scale 255 reads as NaN."""

    def __init__(self, pages, hkv, seed, gain=1.0):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.hkv, self.pages = hkv, pages
        rows = [f32_to_bf16_bits((gain * rng.standard_normal((pages, hkv, PAGE, DIM))).astype(np.float32))
                for _ in range(2)]
        (self.kc, self.ks), (self.vc, self.vs) = (quantise(x) for x in rows)
        self.upload()

    def upload(self):
        self.k4, self.v4 = device(pack_k(self.kc)), device(pack_v(self.vc))
        self.scales = device(pack_scales(self.ks, self.vs))
        self.handle = mw.mw_kv4_pool_create(self.pages, PAGE, self.hkv, DIM, self.k4.data_ptr(), self.v4.data_ptr(),
                                            self.scales.data_ptr())

    def poison_slots(self, page, first):
        """Slots from `first` on get scale byte 255 and the largest codes."""
        for code, scale in ((self.kc, self.ks), (self.vc, self.vs)):
            code[page, :, first:] = 7
            scale[page, :, first:] = 255

    def bf16(self):
        """K and V values as bf16 pools (uint16 bits)."""
        return as_bf16(values(self.kc, self.ks)), as_bf16(values(self.vc, self.vs))

    def close(self):
        torch.cuda.synchronize()
        mw.mw_kv_pool_destroy(self.handle)


def tables(lengths, rng, spare=1, stride=None):
    """Block tables of sequences of those lengths over one random permutation of pages: (table, pages in all); the
    padding names the last page, which no sequence has."""
    need = [-(-n // PAGE) for n in lengths]
    total = sum(need) + spare
    order = rng.permutation(total - spare).astype(np.int32)
    width = max(need + [1]) if stride is None else stride
    table = np.full((max(len(lengths), 1), width), total - 1, np.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, total


def attention_bound(q_bits, k_rows, ref, ref_abs, scale):
    """Largest |error| of each output value that the kernels' arithmetic allows, given the fp64 result ``ref`` and the
    same with |V| (``ref_abs``):

      output and probabilities rounded to bf16, half a step (2^-8 relative) each: 2^-8 |O| and 2^-8 sum p|v|;
      scores: the two e4m3 parts of a query are off by 2^-18 of its largest value, fp32 accumulation of 2 * 128
      products by 2^-16 of their absolute sum at most, exp2 and the fp32 sum of probabilities by less: the score is off
      by d <= scale 2^-15 max|q| max ||k||_1, every weight by a factor within e^(+-2 d);
      fp32 sums of O and l: 2^-14 of sum p|v| (up to 2^10 roundings in a row at half a step each)."""
    q = np.abs(bits_to_f32(q_bits).astype(np.float64)).max()
    d = scale * 2.0**-15 * q * np.abs(k_rows).sum(-1).max()
    return 2.0**-8 * np.abs(ref) + (2.0**-8 + 2.0**-14 + math.expm1(2 * d)) * ref_abs * (1 + 2.0**-7) + 1e-30
