"""Capped scores at caps of any size, from far below the scores to far above them, in all attentions
that take a cap.

Tolerances as in test_prompt_attention, with the cap's share 2^-21 of the cap up to 64, where that is
what the score itself may be off by, and past that 2^-20 of the capped score, however far it is below
the cap.  (Below half of the cap, a product and a series in its square, of factors near one: 2^-22.
Above it, y = cap - 2 cap r with r = 1 / (t + 1), t = e^(2 s / cap): t's exponent of at most 1.5
binades where y is smallest, formed of two roundings, t and r to an ulp each; at s = -cap / 2 that is
2^-23 cap of t's share, 2.2 2^-23 of r's and half of that of the last rounding, 3.3 2^-23 of the cap
where y is 0.46 of it.)  A cap below the scores takes the error of the score itself down with it: at
most 2 cap."""
import math

import numpy as np
import pytest

import paper_2606_01556_amd as tq
from test_kvcache import BF16, KINDS, randn, say, ulp
from test_prompt_attention import Prompts, prompts
from test_shared_prefix import Shared

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CAPS = [1e-40, 1e-30, 1e-3, 0.5, 20.0, 64.0, 65.0, 300.0, 1e4, 1e6, 1e30, 3e38]


@pytest.fixture(autouse=True)
def _wait():
    yield
    torch.cuda.synchronize()


def plain(s, q, scale, cap, weight):
    """(out, lse, their bounds) of the streams' new tokens, causal, in 64 bits."""
    rows, hq, d = q.shape
    heads = s.k.shape[1]
    cap = float(np.float32(cap))
    out, lse, bound, lse_bound = np.zeros((rows, hq, d)), np.full((rows, hq), -np.inf), np.zeros((rows, hq, d)), np.zeros((rows, hq))
    at = 0
    for i, (n, t) in enumerate(zip(s.lens, s.new)):
        k, v = s.k[at:at + n], s.v[at:at + n]
        at += n
        for h in range(hq):
            kh, vh = k[:, h * heads // hq], v[:, h * heads // hq]
            x = q[s.starts[i]:s.starts[i] + t, h].double().numpy()
            z = x @ kh.T * scale
            y = cap * np.tanh(z / cap)
            e = np.minimum(2.0 ** -19 * (np.abs(x) @ np.abs(kh).T) * abs(scale), 2 * cap) + 2.0 ** -22 * np.abs(y)
            e += 2.0 ** -21 * cap if cap <= 64 else 2.0 ** -20 * np.abs(y)
            e += 2.0 ** -18 if s.cache.bits < 16 else 0.0
            seen = np.arange(n)[None] <= n - t + np.arange(t)[:, None]
            y = np.where(seen, y, -np.inf)
            m = y.max(-1, keepdims=True)
            w = np.exp(y - m)
            total = w.sum(-1, keepdims=True)
            w /= total
            mean = (w * e).sum(-1, keepdims=True)
            r = slice(s.starts[i], s.starts[i] + t)
            out[r, h] = w @ vh
            lse[r, h] = (m + np.log(total))[:, 0]
            off = (w * (weight + e + mean)) @ np.abs(vh)
            bound[r, h] = ulp(q.dtype) * np.abs(out[r, h]) + off + n * 2.0 ** -36 * np.abs(vh).max(0) + 2.0 ** -24
            lse_bound[r, h] = mean[:, 0] + 2.0 ** -18 * (1 + np.abs(lse[r, h]))
    return out, lse, bound, lse_bound


def check(got, lse, ref, ref_lse, bound, lse_bound):
    got, lse = got.cpu().double().numpy(), lse.cpu().double().numpy()
    assert np.isfinite(got).all() and np.isfinite(lse).all()
    assert (np.abs(lse - ref_lse) <= lse_bound).all(), (np.abs(lse - ref_lse) - lse_bound).max()
    assert (np.abs(got - ref) <= bound).all(), (np.abs(got - ref) - bound).max()


def rounding(s):
    return 2.0 ** -8 if s.cache.bits == 16 and s.cache.k.dtype == BF16 else 2.0 ** -11


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("cap", CAPS)
def test_prompts(kind, dtype, d, cap):
    """(scores up to about 100)"""
    say("prompts", kind, dtype, d, cap)
    s, q = prompts([150, 70], [150, 6], 1, 2, d, 16, kind, dtype, scale=3.0)
    q[3] = 0
    check(*s.call(q, softcap=cap, return_lse=True), *plain(s, q, d ** -0.5, cap, rounding(s)))


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("cap", CAPS)
def test_one_token(kind, dtype, d, cap):
    say("token", kind, dtype, d, cap)
    for lens in ([1, 40, 300], [3000, 17]):
        s, q = prompts(lens, [1] * len(lens), 1, 4, d, 16, kind, dtype, scale=3.0)
        q[0, 0] = 0
        table, lengths = s.args()
        got = tq.paged_attention(s.cache, q.cuda(), table, lengths, softcap=cap, return_lse=True)
        check(*got, *plain(s, q, d ** -0.5, cap, 2.0 ** -11))


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("cap", CAPS)
def test_shared_prefix(kind, dtype, cap):
    say("prefix", kind, dtype, cap)
    s = Shared([300], [0, 3], [5, 40, 1], 1, 128, 16, kind, dtype)
    q = (3.0 * randn(3, 4, 128, seed=9)).to(dtype)
    whole = object.__new__(Prompts)
    at = np.cumsum([0] + s.lens)
    rows = lambda x: np.concatenate([np.concatenate((x[:at[1]], x[a:b])) for a, b in zip(at[1:], at[2:])])
    whole.cache, whole.k, whole.v = s.cache, rows(s.k), rows(s.v)
    whole.lens, whole.new, whole.starts = [300 + n for n in s.own], [1, 1, 1], [0, 1, 2]
    check(*s.call(q, softcap=cap, return_lse=True), *plain(whole, q, 128 ** -0.5, cap, rounding(s)))


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_a_cap_out_of_reach_is_none(kind, dtype):
    """Scores far below the cap are left as they are, to the last bit of the log-sum-exp's bound."""
    say("none", kind, dtype)
    s, q = prompts([150, 70], [150, 6], 1, 2, 128, 16, kind, dtype, scale=3.0)
    (got, lse), (ref, ref_lse) = (s.call(q, softcap=cap, return_lse=True) for cap in (1e8, 0.0))
    # (scores of at most 128, so off by 2^-17 where they are formed with one more rounding; the
    # logarithm of a value's scale rounds its sum with them elsewhere)
    assert bool(((lse - ref_lse).abs() <= 2.0 ** -16 * (1 + ref_lse.abs())).all())
    _, _, bound, _ = plain(s, q, 128 ** -0.5, 1e8, rounding(s))
    assert (np.abs((got.double() - ref.double()).cpu().numpy()) <= 2 * bound).all()


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("cap", [20.0, 100.0])
def test_a_row_does_not_depend_on_its_neighbours(kind, dtype, cap):
    """Rows whose scores are far below the cap, beside others that are too and beside ones that are not."""
    say("neighbours", kind, dtype, cap)
    s, q = prompts([500, 420], [500, 420], 2, 4, 128, 16, kind, dtype, scale=0.3)
    ref, lse = s.call(q, softcap=cap, return_lse=True)
    q[::3] *= 30.0
    got, got_lse = s.call(q, softcap=cap, return_lse=True)
    keep = torch.arange(920) % 3 != 0
    assert torch.equal(got[keep], ref[keep]) and torch.equal(got_lse[keep], lse[keep])
    assert not torch.equal(got[~keep], ref[~keep])
