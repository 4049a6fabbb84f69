"""The library's calls as the measured cases make them: on the stream that is current at each run, and on the tensors that
the state holds then."""
import pytest
import torch

from perf import operators
from tests.helpers import say

pytestmark = pytest.mark.gpu

SMALL = dict(hq=8, hkv=2, batch=3, lens=5)
ROPE = dict(kind="rope", norm=True, rot=128, neighbours=False, theta=1e4, n_lo=1, n_hi=40, r_lo=0, r_hi=50)
CASES = [
    dict(SMALL, kind="write", n_lo=1, n_hi=40, r_lo=0, r_hi=50), dict(SMALL, bits=16, **ROPE), dict(SMALL, bits=4, **ROPE),
    dict(SMALL, kind="decode", l_lo=1, l_hi=900, dist="uniform", gain=1.0),
    dict(SMALL, kind="prefill", n_lo=3, n_hi=30, r_lo=0, r_hi=500, gain=1.0),
    dict(SMALL, kind="prefill", n_lo=200, n_hi=400, r_lo=0, r_hi=500, gain=1.0),
]


def outputs(state):
    out = operators.run(state)
    out = dict(out) if isinstance(out, dict) else {"out": out}
    torch.cuda.synchronize()
    return {k: t.clone() for k, t in out.items()}


def same(a, b):
    return a.keys() == b.keys() and all(torch.equal(a[k], b[k]) for k in a)


@pytest.fixture(autouse=True)
def the_librarys_calls(monkeypatch):
    monkeypatch.setattr(operators, "own", True)


@pytest.mark.parametrize("case", CASES, ids=lambda c: c["kind"])
def test_the_current_stream_at_each_run(case, monkeypatch):
    say(f"measured calls on two streams {case}")
    state = operators.prepare(case, 1)
    first = outputs(state)
    mw, seen = state["own"].mw, []
    for name in ("mw_kv4_pool_write", "mw_kv4_pool_gather", "mw_qk_norm_rope_write", "mw_kv4_decode_attn",
                 "mw_kv4_prefill_attn"):
        def call(*args, _call=getattr(mw, name)):
            seen.append(args[-1])
            _call(*args)
        monkeypatch.setattr(mw, name, call)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        assert same(outputs(state), first)
    assert seen and set(seen) == {stream.cuda_stream}


@pytest.mark.parametrize("case", CASES, ids=lambda c: c["kind"])
def test_tensors_that_were_replaced(case):
    """A state with another's tensors in the place of its own gives what the other gives."""
    say(f"measured calls on replaced tensors {case}")
    state, other = operators.prepare(case, 1), operators.prepare(case, 2)
    fresh = operators.prepare(case, 2)
    first = outputs(state)
    for name, value in other.items():
        if isinstance(value, torch.Tensor):
            state[name] = value
    got, want = outputs(state), outputs(fresh)
    assert same(got, want) and not same(got, first)
