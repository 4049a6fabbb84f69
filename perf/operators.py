"""The calls on a KV cache held in 4 bits, and on the rows that enter a cache, as measured cases.

A pool in 4 bits keeps every (token, kv head) row of 128 values as four blocks of 32 four-bit floats (sign, two
exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) with one shared power of two each.  The cases:

  write    append bf16 rows to such a pool and read the same rows back
  rope     per-head RMS norm of queries and keys, position rotation and append in one pass, from the rows of a QKV
           projection into a bf16 pool or one in 4 bits
  decode   one query token per sequence over the 4-bit cache
  prefill  a causal chunk over its cached prefix and itself, all keys from the 4-bit cache

Head layouts and lengths are those of the layers in ``paper_2504_14489_amd/workloads.py`` and of the GQA groupings
its tests run; values are N(0, 1) in bf16 with the query gain of those tests.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
DIM = 128
BLOCKS = 4           # blocks of 32 dims with a scale each
BIAS = 127           # a scale byte s stands for 2^(s - 127)
EXP_MOST = 100       # exponents are kept in [-100, 100]
DEVICE = "cuda"
EPS = 1e-6

# (query heads, kv heads) of the library's layers and of the groupings 1 .. 16
HEADS = ((32, 8), (64, 8), (8, 1), (8, 2), (32, 32), (4, 4), (2, 1), (12, 2), (6, 2), (16, 1))


def listed():
    return [
        # one decode step's append: a batch of 64 sequences, one token each; launch latency counts
        dict(name="write_step", kind="write", hq=32, hkv=8, batch=64, n_lo=1, n_hi=1, r_lo=511, r_hi=4095, lens=1),
        # the append of a long chunk over a cached prefix, pages begun in the middle
        dict(name="write_chunk", kind="write", hq=32, hkv=8, batch=2, n_lo=4001, n_hi=4096, r_lo=1003, r_hi=28672,
             lens=2),
        # one decode step's norm, rotation and append into the bf16 pool
        dict(name="rope_step", kind="rope", hq=32, hkv=8, batch=64, n_lo=1, n_hi=1, r_lo=511, r_hi=4095, bits=16,
             norm=True, rot=128, neighbours=False, theta=500000.0, lens=3),
        # a prompt chunk far into a context, into the bf16 pool
        dict(name="rope_chunk", kind="rope", hq=32, hkv=8, batch=1, n_lo=4096, n_hi=4096, r_lo=28672, r_hi=28672,
             bits=16, norm=True, rot=128, neighbours=False, theta=500000.0, lens=4),
        # a ragged batch of prompts into the pool in 4 bits, half of each head rotated, neighbours paired
        dict(name="rope_ragged4", kind="rope", hq=64, hkv=8, batch=12, n_lo=17, n_hi=1500, r_lo=0, r_hi=4000, bits=4,
             norm=True, rot=64, neighbours=True, theta=10000.0, lens=5),
        # one interactive sequence: decode latency
        dict(name="decode_single", kind="decode", hq=32, hkv=8, batch=1, l_lo=4003, l_hi=4003, dist="uniform",
             gain=1.0, lens=6),
        # an ordinary decode batch
        dict(name="decode_8b", kind="decode", hq=32, hkv=8, batch=64, l_lo=512, l_hi=4096, dist="uniform", gain=1.0,
             lens=7),
        # one GPU's share of the 70B-shaped layer at tensor-parallel degree 8
        dict(name="decode_tp8", kind="decode", hq=8, hkv=1, batch=128, l_lo=64, l_hi=16384, dist="lognormal",
             gain=4.0, lens=8),
        # the largest decode: 32 sequences of 16K .. 32K tokens
        dict(name="decode_long", kind="decode", hq=32, hkv=8, batch=32, l_lo=16384, l_hi=32768, dist="uniform",
             gain=1.0, lens=9),
        # a short last chunk over a long conversation
        dict(name="prefill_short", kind="prefill", hq=32, hkv=8, batch=1, n_lo=64, n_hi=64, r_lo=8000, r_hi=8000,
             gain=1.0, lens=10),
        # a batch of prompts of ragged lengths, some over a reused prefix
        dict(name="prefill_ragged", kind="prefill", hq=32, hkv=8, batch=12, n_lo=17, n_hi=1500, r_lo=0, r_hi=4000,
             gain=4.0, lens=11),
        # the largest prefill: 4096 new tokens over a 28672-token cached prefix
        dict(name="prefill_long", kind="prefill", hq=32, hkv=8, batch=1, n_lo=4096, n_hi=4096, r_lo=28672, r_hi=28672,
             gain=1.0, lens=12),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Any kind, grouping, batch and length up to those listed, odd sizes included."""
    kind = rng.choice(["write", "rope", "decode", "decode", "prefill", "prefill"])
    hq, hkv = rng.choice(HEADS)
    case = dict(kind=kind, hq=hq, hkv=hkv)
    if kind == "decode":
        l_hi = _log_int(rng, 1, 32768)
        most = (1 << 30) // (256 * hkv * l_hi)  # at most the longest batch's cache
        case.update(batch=_log_int(rng, 1, max(1, min(256, most))), l_lo=max(1, l_hi // rng.choice([1, 2, 8])),
                    l_hi=l_hi, dist=rng.choice(["uniform", "lognormal"]), gain=rng.choice([1.0, 1.0, 4.0]))
    elif kind == "prefill":
        batch, n_hi = _log_int(rng, 1, 16), _log_int(rng, 1, 4096)
        r_hi = rng.choice([0, _log_int(rng, 1, 28672)])
        # a sixth of the longest chunk's work at most (a drawn batch is padded by its longest member)
        while batch * n_hi * (r_hi + n_hi) * hq > 4096 * 32768 * 32 // 6:
            batch, r_hi = max(1, batch // 2), r_hi // 2
            n_hi = n_hi if batch > 1 or r_hi > 0 else n_hi // 2
        case.update(batch=batch, n_lo=max(1, n_hi // rng.choice([1, 2, 16])), n_hi=n_hi,
                    r_lo=r_hi // rng.choice([1, 2, 16]), r_hi=r_hi, gain=rng.choice([1.0, 1.0, 4.0]))
    else:
        n_hi = _log_int(rng, 1, 4096)
        batch = _log_int(rng, 1, max(1, min(256, 8192 * 8 // (n_hi * hkv), 8192 * 40 // (n_hi * hq))))
        r_hi = rng.choice([0, _log_int(rng, 1, 28672)])
        case.update(batch=batch, n_lo=max(1, n_hi // rng.choice([1, 2, 16])), n_hi=n_hi,
                    r_lo=r_hi // rng.choice([1, 2, 16]), r_hi=r_hi)
        if kind == "rope":
            case.update(bits=rng.choice([16, 4]), norm=rng.choice([True, True, False]), rot=rng.choice([128, 128, 64]),
                        neighbours=rng.choice([False, True]), theta=rng.choice([10000.0, 500000.0]))
    case["lens"] = rng.randint(100, 1 << 20)
    return case


def _lengths(case):
    """(new tokens, prefixes) or (ones, lengths - 1) of a decode batch: part of the case, the same for every seed."""
    rng = random.Random(case["lens"])
    if case["kind"] != "decode":
        pairs = [(rng.randint(case["n_lo"], case["n_hi"]), rng.randint(case["r_lo"], case["r_hi"]))
                 for _ in range(case["batch"])]
        return [n for n, _ in pairs], [r for _, r in pairs]
    lengths = []
    for _ in range(case["batch"]):
        if case["dist"] == "lognormal":
            mid = min(2048, math.sqrt(case["l_lo"] * case["l_hi"]))
            lengths.append(min(case["l_hi"], max(case["l_lo"], int(round(math.exp(rng.gauss(math.log(mid), 0.8)))))))
        else:
            lengths.append(rng.randint(case["l_lo"], case["l_hi"]))
    return [1] * len(lengths), [length - 1 for length in lengths]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


# ------------------------------------------------------- the cache's format
def _quantise(x):
    """(codes, scale bytes) of rows x [..., DIM]: the smallest power of two that keeps a block's largest magnitude
    within 7 of its units, each value rounded to the nearest of the format's (ties to even), 6 the most."""
    blocks = x.float().reshape(*x.shape[:-1], BLOCKS, DIM // BLOCKS)
    part, power = torch.frexp(blocks.abs().amax(-1))
    exponent = (power - 3 + (part > 0.875).int()).clamp(-EXP_MOST, EXP_MOST)
    exponent = torch.where(part == 0, torch.full_like(exponent, -EXP_MOST), exponent)
    a = torch.ldexp(blocks.abs(), -exponent[..., None])
    code = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, 2 + torch.round(a), 4 + torch.round(a / 2)))
    code = code.clamp(max=7).to(torch.uint8) | (torch.signbit(blocks).to(torch.uint8) << 3)
    return code.reshape(x.shape), (exponent + BIAS).to(torch.uint8)


def _values(code, scale):
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    blocks = table[code.long()].reshape(*code.shape[:-1], BLOCKS, DIM // BLOCKS)
    return torch.ldexp(blocks, scale.int()[..., None] - BIAS).reshape(code.shape)


def _pack_k(code):
    """[..., 16 tokens, DIM] -> [..., 16, 64] bytes: dim 2i in the low half of byte i."""
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _pack_v(code):
    """[..., 16 tokens, DIM] -> [..., 4, 16, 8, 2] bytes: token 4g + 2k + n, dim 32b + 2c + e in half n of byte
    [g][c][2b + e][k]."""
    lead = code.shape[:-2]
    at = len(lead)
    v = code.reshape(*lead, 4, 2, 2, 4, 16, 2)  # g k n b c e
    v = v.permute(*range(at), at, at + 4, at + 3, at + 5, at + 1, at + 2).reshape(*lead, 4, 16, 8, 2, 2)
    return (v[..., 0] | (v[..., 1] << 4)).contiguous()


def _page_values(state, pages):
    """K and V [..., hkv, 16, DIM] of pages [...] as the values that their bytes stand for."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEVICE)
    byte = torch.arange(256, device=DEVICE)
    both = torch.stack([table[byte & 15], table[byte >> 4]], dim=-1)
    index = pages.long()
    at = index.dim() + 1
    scale = torch.exp2(state["scales"][index].float() - BIAS)  # [..., hkv, 2, 4, 16]
    scale = scale.movedim(-1, -2)                                # [..., hkv, 2, 16, 4]
    k = both[state["k4"][index].long()].reshape(*index.shape, -1, PAGE, BLOCKS, 32)
    k = (k * scale[..., 0, :, :, None]).reshape(*index.shape, -1, PAGE, DIM)
    v = both[state["v4"][index].long()].reshape(*index.shape, -1, 4, 16, 4, 2, 2, 2)  # g c b e k n
    v = v.permute(*range(at), at, at + 4, at + 5, at + 2, at + 1, at + 3).reshape(*index.shape, -1, PAGE, BLOCKS, 32)
    v = (v * scale[..., 1, :, :, None]).reshape(*index.shape, -1, PAGE, DIM)
    return k, v


# ------------------------------------------------------------------- inputs
def prepare(case, seed):
    """What a serving program has in hand: the pool's arrays, block tables, lengths on host and device, the rows."""
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.bfloat16)

    hq, hkv = case["hq"], case["hkv"]
    new, prefix = _lengths(case)
    attends = case["kind"] in ("decode", "prefill")
    first = [0 if attends else r // PAGE for r in prefix]  # pages before a row that is only appended hold nothing here
    last = [-(-(n + r) // PAGE) for n, r in zip(new, prefix)]
    total = sum(b - a for a, b in zip(first, last)) + 1
    order = torch.randperm(total, generator=gen, device=DEVICE).int()
    table = order[-1].repeat(len(new), max(last))  # padded with the spare page
    at = 0
    for i, (a, b) in enumerate(zip(first, last)):
        table[i, a:b] = order[at:at + b - a]
        at += b - a
    state = dict(case=dict(case), hq=hq, hkv=hkv, new=new, prefix=prefix, table=table.contiguous(), pages=total,
                 h_new=np.array(new, np.int32), h_prefix=np.array(prefix, np.int32), d_prefix=_i32(prefix),
                 d_indptr=_i32([0] + np.cumsum(new).tolist()))
    tokens = sum(new)
    if case.get("bits", 4) == 16:
        state["k"], state["v"] = normal(total, hkv, PAGE, DIM), normal(total, hkv, PAGE, DIM)
    else:
        state["k4"] = torch.empty(total, hkv, PAGE, DIM // 2, dtype=torch.uint8, device=DEVICE)
        state["v4"] = torch.empty(total, hkv, 4, 16, 8, 2, dtype=torch.uint8, device=DEVICE)
        state["scales"] = torch.empty(total, hkv, 2, BLOCKS, PAGE, dtype=torch.uint8, device=DEVICE)
        step = max(1, (1 << 26) // (hkv * PAGE * DIM))
        for i in range(0, total, step):
            part = slice(i, min(total, i + step))
            for which, (name, pack) in enumerate((("k4", _pack_k), ("v4", _pack_v))):
                code, scale = _quantise(normal(part.stop - i, hkv, PAGE, DIM))
                state[name][part] = pack(code)
                state["scales"][part, :, which] = scale.transpose(-1, -2)
    if attends:
        state["q"] = normal(tokens, hq, DIM) * case["gain"]
        state["d_lens"] = _i32([n + r for n, r in zip(new, prefix)])
        state["h_lens"] = np.array([n + r for n, r in zip(new, prefix)], np.int32)
    elif case["kind"] == "write":
        state["k_new"], state["v_new"] = normal(tokens, hkv, DIM), normal(tokens, hkv, DIM)
    else:
        state["rows"] = normal(tokens, hq + 2 * hkv, DIM)  # a projection's rows: queries, keys, values side by side
        if case["norm"]:
            state["q_weight"], state["k_weight"] = 1 + 0.1 * normal(DIM), 1 + 0.1 * normal(DIM)
        rot = case["rot"]
        state["inv_freq"] = case["theta"] ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEVICE) / rot)
    return state


# --------------------------------------------------------------- plain form
def _places(state):
    """Page, slot and position of every new token."""
    new = torch.from_numpy(state["h_new"]).to(DEVICE).long()
    seq = torch.repeat_interleave(torch.arange(len(new), device=DEVICE), new)
    pos = torch.arange(len(seq), device=DEVICE) - state["d_indptr"].long()[seq] + state["d_prefix"].long()[seq]
    return state["table"].long()[seq, pos // PAGE], pos % PAGE, pos


def _plain_write4(state, k_rows, v_rows):
    """Quantises the rows and puts them in their places; the values they then stand for."""
    page, slot, _ = _places(state)
    out = []
    for which, rows in enumerate((k_rows, v_rows)):
        code, scale = _quantise(rows)
        state["scales"][page, :, which, :, slot] = scale
        if which == 0:
            state["k4"][page, :, slot] = _pack_k(code)
        else:
            # the half byte of a token in each of its dims' bytes: the even tokens of the call, then the odd ones
            dims = code.reshape(*code.shape[:-1], BLOCKS, 16, 2).transpose(-3, -2).reshape(*code.shape[:-1], 16, 8)
            for half in (0, 1):
                mine = slot % 2 == half
                at = (page[mine], slice(None), slot[mine] // 4, slice(None), slice(None), slot[mine] % 4 // 2)
                kept = state["v4"][at] & (0xF0 if half == 0 else 0x0F)
                state["v4"][at] = kept | (dims[mine] << (4 * half))
        out.append(_values(code, scale).to(torch.bfloat16))
    return out


def _turn(x, angle, neighbours):
    """Rotates the first 2 * angle.shape[-1] dims of x [T, heads, DIM] by angle [T, half]."""
    half = angle.shape[-1]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if neighbours:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., 2 * half:]], dim=-1)


def _plain_rope(state):
    case, hq, hkv = state["case"], state["hq"], state["hkv"]
    page, slot, pos = _places(state)
    angle = pos.double()[:, None] * state["inv_freq"]
    q, k, v = state["rows"][:, :hq].float(), state["rows"][:, hq:hq + hkv].float(), state["rows"][:, hq + hkv:]
    if case["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * state["q_weight"].float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * state["k_weight"].float()
    q = _turn(q, angle, case["neighbours"]).to(torch.bfloat16)
    k = _turn(k, angle, case["neighbours"]).to(torch.bfloat16)
    if case["bits"] == 4:
        k_held, v_held = _plain_write4(state, k, v)
        return {"q": q, "k": k_held, "v": v_held}
    state["k"][page, :, slot] = k
    state["v"][page, :, slot] = v
    return {"q": q, "k": state["k"], "v": state["v"]}


def _plain_attention(state):
    """softmax(scale q k^T) v, padded to the batch's longest sequences."""
    hq, hkv, group = state["hq"], state["hkv"], state["hq"] // state["hkv"]
    batch, n = len(state["new"]), max(state["new"])
    k, v = _page_values(state, state["table"])                     # [B, W, hkv, 16, DIM]
    k = k.transpose(1, 2).reshape(batch, hkv, -1, DIM)
    v = v.transpose(1, 2).reshape(batch, hkv, -1, DIM)
    new = torch.from_numpy(state["h_new"]).to(DEVICE).long()
    row = torch.arange(n, device=DEVICE)
    there = row < new[:, None]                                     # [B, n]
    q = torch.zeros(batch, n, hq, DIM, device=DEVICE)
    q[there] = state["q"].float()
    q = q.reshape(batch, n, hkv, group, DIM).permute(0, 2, 3, 1, 4).reshape(batch, hkv, group * n, DIM)
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(DIM)).reshape(batch, hkv, group, n, -1)
    seen = state["d_prefix"].long()[:, None] + torch.minimum(row, new[:, None] - 1)
    hidden = torch.arange(k.shape[2], device=DEVICE) > seen[..., None]  # [B, n, L]
    s.masked_fill_(hidden[:, None, None], -math.inf)
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.reshape(batch, hkv, group * n, -1), v).reshape(batch, hkv, group, n, DIM) / total
    return o.permute(0, 3, 1, 2, 4).reshape(batch, n, hq, DIM)[there].to(torch.bfloat16)


# --------------------------------------------------------- the library's calls
# what a handle holds the addresses of
HELD = ("k", "v", "k4", "v4", "scales", "q_weight", "k_weight", "inv_freq")


class _Handles:
    """What a program keeps beside its tensors: the pool's handle, output buffers and workspaces."""

    def __init__(self, state):
        import weakref

        from paper_2504_14489_amd import mw

        self.mw = mw
        self.names = [name for name in HELD if name in state]
        self.held = [state[name].data_ptr() for name in self.names]
        hq, hkv, kind = state["hq"], state["hkv"], state["case"]["kind"]
        if "k" in state:
            self.pool = mw.mw_kv_pool_create(state["pages"], PAGE, hkv, DIM, state["k"].data_ptr(),
                                             state["v"].data_ptr())
        else:
            self.pool = mw.mw_kv4_pool_create(state["pages"], PAGE, hkv, DIM, state["k4"].data_ptr(),
                                              state["v4"].data_ptr(), state["scales"].data_ptr())
        weakref.finalize(self, mw.mw_kv_pool_destroy, self.pool)
        tokens, size = sum(state["new"]), 0
        if kind in ("write", "rope"):
            self.k_held = torch.empty(tokens, hkv, DIM, dtype=torch.bfloat16, device=DEVICE)
            self.v_held = torch.empty_like(self.k_held)
        if kind != "write":
            self.out = torch.empty(tokens, hq, DIM, dtype=torch.bfloat16, device=DEVICE)
        if kind == "decode":
            size = mw.mw_kv4_decode_workspace_size(hq, hkv, DIM, state["h_lens"])
        elif kind == "prefill":
            size = mw.mw_kv4_prefill_workspace_size(hq, hkv, DIM, state["h_new"], state["h_prefix"])
        self.ws = torch.empty(max(size, 16), dtype=torch.uint8, device=DEVICE)
        if kind == "rope":
            case = state["case"]
            self.rope = mw.NormRope(
                num_q_heads=hq, rot_dim=case["rot"], neighbours=int(case["neighbours"]), eps=EPS,
                d_q_weight=state["q_weight"].data_ptr() if case["norm"] else 0,
                d_k_weight=state["k_weight"].data_ptr() if case["norm"] else 0,
                d_inv_freq=state["inv_freq"].data_ptr())


def _own_run(state):
    h = state.get("own")
    if h is None or h.held != [state[name].data_ptr() for name in h.names]:
        state["own"] = h = _Handles(state)
    # torch.cuda.current_stream().cuda_stream without the object (2 us of a call of 9)
    stream = torch._C._cuda_getCurrentRawStream(state["table"].device.index)
    mw, case, hq, hkv, table = h.mw, state["case"], state["hq"], state["hkv"], state["table"]
    where = (state["h_new"], state["h_prefix"], state["d_indptr"].data_ptr(), state["d_prefix"].data_ptr(),
             table.data_ptr(), table.shape[1])
    if case["kind"] == "decode":
        mw.mw_kv4_decode_attn(h.pool, hq, hkv, DIM, 1.0 / math.sqrt(DIM), state["h_lens"], state["d_lens"].data_ptr(),
                              table.data_ptr(), table.shape[1], state["q"].data_ptr(), h.out.data_ptr(),
                              h.ws.data_ptr(), h.ws.numel(), stream)
        return h.out
    if case["kind"] == "prefill":
        mw.mw_kv4_prefill_attn(h.pool, hq, hkv, DIM, 1.0 / math.sqrt(DIM), *where, state["q"].data_ptr(),
                               h.out.data_ptr(), h.ws.data_ptr(), h.ws.numel(), stream)
        return h.out
    if case["kind"] == "write":
        mw.mw_kv4_pool_write(h.pool, *where, state["k_new"].data_ptr(), state["v_new"].data_ptr(), stream)
        mw.mw_kv4_pool_gather(h.pool, *where, h.k_held.data_ptr(), h.v_held.data_ptr(), stream)
        return {"k": h.k_held, "v": h.v_held}
    rows, stride = state["rows"], state["rows"].stride(0)
    mw.mw_qk_norm_rope_write(h.pool, h.rope, *where, rows.data_ptr(), stride, rows[:, hq:].data_ptr(), stride,
                             rows[:, hq + hkv:].data_ptr(), stride, h.out.data_ptr(), stream)
    if case["bits"] == 16:
        return {"q": h.out, "k": state["k"], "v": state["v"]}
    mw.mw_kv4_pool_gather(h.pool, *where, h.k_held.data_ptr(), h.v_held.data_ptr(), stream)
    return {"q": h.out, "k": h.k_held, "v": h.v_held}


def run(state):
    if own:
        return _own_run(state)
    kind = state["case"]["kind"]
    if kind == "write":
        k, v = _plain_write4(state, state["k_new"], state["v_new"])
        return {"k": k, "v": v}
    return _plain_rope(state) if kind == "rope" else _plain_attention(state)


def work(case):
    """Inputs read once, outputs written once; a (token, kv head) row of the 4-bit cache is 68 bytes each for K and
    V, and QK^T and PV count over the visible pairs only."""
    hq, hkv = case["hq"], case["hkv"]
    new, prefix = _lengths(case)
    row, held = 2 * DIM, DIM // 2 + BLOCKS
    nbytes = flops = 0
    for n, r in zip(new, prefix):
        if case["kind"] in ("decode", "prefill"):
            nbytes += 2 * (n + r) * hkv * held + 2 * n * hq * row + 4 * -(-(n + r) // PAGE)
            flops += 4 * DIM * hq * (n * r + n * (n + 1) // 2)
        elif case["kind"] == "write":
            nbytes += 2 * n * hkv * (2 * row + held)
            flops += 2 * n * hkv * DIM * 4
        else:
            nbytes += n * (2 * hq + 2 * hkv) * row
            nbytes += 2 * n * hkv * (row if case["bits"] == 16 else held + row)
            flops += n * (hq + hkv) * DIM * 8
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------ in 64 bits
def _held64(x):
    """The value that the format keeps of each of x [..., DIM], from its definition."""
    blocks = x.double().reshape(*x.shape[:-1], BLOCKS, 32)
    most = blocks.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2(most / 7)).clamp(-EXP_MOST, EXP_MOST))
    a = blocks.abs() / unit
    kept = torch.zeros_like(a)
    for border, upper, step in ((0.25, False, 0.5), (0.75, True, 0.5), (1.25, False, 0.5), (1.75, True, 0.5),
                                (2.5, False, 1.0), (3.5, True, 1.0), (5.0, False, 2.0)):
        kept += step * (a >= border if upper else a > border)
    return (kept * unit * blocks.sign()).reshape(x.shape)


def _rows64(state, page_ids, length):
    """K and V [hkv, length, DIM] of a sequence in 64 bits, each code taken apart by its bits."""
    pages = page_ids.long()[:-(-length // PAGE)]

    def number(code):
        code = code.long()
        top, low = (code >> 1) & 3, code & 1
        size = torch.where(top == 0, 0.5 * low.double(), (1 + 0.5 * low.double()) * torch.exp2(top.double() - 1))
        return torch.where(code >= 8, -size, size)

    token, dim = torch.arange(PAGE, device=DEVICE)[:, None], torch.arange(DIM, device=DEVICE)[None, :]
    k = number((state["k4"][pages][:, :, token, dim // 2].long() >> (4 * (dim % 2))) & 15)
    at = (token // 4, dim % 32 // 2, 2 * (dim // 32) + dim % 2, token % 4 // 2)
    v = number((state["v4"][pages][:, :, at[0], at[1], at[2], at[3]].long() >> (4 * (token % 2))) & 15)
    unit = torch.exp2(state["scales"][pages].double() - BIAS)
    k, v = k * unit[:, :, 0][:, :, dim // 32, token], v * unit[:, :, 1][:, :, dim // 32, token]
    return [x.transpose(0, 1).reshape(state["hkv"], -1, DIM)[:, :length] for x in (k, v)]


def _attend64(state):
    group, out, row = state["hq"] // state["hkv"], [], 0
    for i, (n, r) in enumerate(zip(state["new"], state["prefix"])):
        k, v = _rows64(state, state["table"][i], n + r)
        q = state["q"][row:row + n].double()
        row += n
        heads = []
        keys = torch.arange(n + r, device=DEVICE)
        for h in range(state["hkv"]):
            parts, step = [], max(1, (1 << 26) // (group * (n + r)))
            kt = k[h].t().contiguous()
            for j in range(0, n, step):
                m = min(step, n - j)
                s = (q[j:j + m, h * group:(h + 1) * group].reshape(m * group, DIM) @ kt) / math.sqrt(DIM)
                last = r + j + torch.arange(m, device=DEVICE).repeat_interleave(group)
                s.masked_fill_(keys[None] > last[:, None], -math.inf)
                parts.append((torch.softmax(s, dim=-1) @ v[h]).reshape(m, group, DIM))
            heads.append(torch.cat(parts))
        out.append(torch.cat(heads, dim=1))
    return torch.cat(out)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] in ("decode", "prefill"):
        return _attend64(state)
    if case["kind"] == "write":
        return {"k": _held64(state["k_new"]), "v": _held64(state["v_new"])}
    hq, hkv, rot = state["hq"], state["hkv"], case["rot"]
    rows = state["rows"].double()
    pos = torch.cat([r + torch.arange(n, device=DEVICE) for n, r in zip(state["new"], state["prefix"])]).double()
    unit = torch.polar(torch.ones(len(pos), rot // 2, dtype=torch.float64, device=DEVICE),
                       pos[:, None] * state["inv_freq"])[:, None]
    out = []
    for x, name in ((rows[:, :hq], "q_weight"), (rows[:, hq:hq + hkv], "k_weight")):
        if case["norm"]:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / DIM + EPS) * state[name].double()
        lead = x[..., :rot]
        if case["neighbours"]:
            lead = torch.view_as_real(torch.view_as_complex(lead.reshape(*lead.shape[:-1], -1, 2)) * unit).flatten(-2)
        else:
            turned = torch.complex(lead[..., :rot // 2], lead[..., rot // 2:]) * unit
            lead = torch.cat([turned.real, turned.imag], dim=-1)
        out.append(torch.cat([lead, x[..., rot:]], dim=-1))
    q, k, v = out[0], out[1], rows[:, hq + hkv:]
    if case["bits"] == 4:
        # the row that is kept in 4 bits is the bf16 one
        return {"q": q, "k": _held64(k.to(torch.bfloat16)), "v": _held64(v)}
    pool = {"k": state["k"].double(), "v": state["v"].double()}
    place = [0] + np.cumsum(state["new"]).tolist()
    for i, (n, r) in enumerate(zip(state["new"], state["prefix"])):
        at = r + torch.arange(n, device=DEVICE)
        page = state["table"][i].long()[at // PAGE]
        pool["k"][page, :, at % PAGE] = k[place[i]:place[i] + n]
        pool["v"][page, :, at % PAGE] = v[place[i]:place[i] + n]
    return {"q": q, **pool}
