"""The operators between the linear layers at the ends of their types: values near
bf16's largest and far below one, weights whose low bits decide, rows past the
largest scale, infinities and NaN in live rows.

Tolerances: as in test_attention_plans, with
  2^-20   of sum_t w_t |v_t| where the scores are at most 8 and their own sums are of
          two products: such a score is off by 2^-22, its exponent, of at most 16
          binades, by 2^-21 (0.7 of that in the weight), exp2 by 2^-23; a weight of
          16 bits would be off by up to 2^-18"""
import math

import numpy as np
import pytest

import paper_2606_01556_amd as tq
from test_attention_plans import Held
from test_kvcache import BF16, F16, KINDS, make_cache, randn, say, stored, ulp

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _wait():
    yield
    torch.cuda.synchronize()


def refill(s, k, v, dtype):
    """The streams' rows replaced by k and v [all tokens, heads, d]."""
    every = torch.cat(s.slots)
    tq.kv_append(s.cache, k.to(dtype).cuda(), v.to(dtype).cuda(), every.cuda())
    (kv, ks), (vv, vs) = stored(s.cache, every)
    s.k = kv if ks is None else kv * ks.astype(np.float64)[..., None]
    s.v = vv if vs is None else vv * vs.astype(np.float64)[..., None]


def run(s, q, **kw):
    out, lse = tq.paged_attention(s.cache, q.cuda(), *s.args(), return_lse=True, **kw)
    return out.cpu().double().numpy(), lse.cpu().double().numpy()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,dtype", KINDS[2:])
def test_sum_with_values_that_are_no_number(kind, dtype, d):
    """The log-sum-exp is the keys' alone: value rows whose scale is NaN, all or one of
    them, far above the others or not, leave it as it is."""
    lens = [1, 40, 3000, 60, 3001, 700, 33]
    s = Held(lens, 2, d, 16, kind, dtype, seed=d)
    k, v = randn(sum(lens), 2, d, seed=1), randn(sum(lens), 2, d, seed=2)
    at = np.cumsum([0] + lens)
    v[at[0]:at[3], :, 5] = math.nan               # all rows of the first three streams
    for i in (3, 4, 5):                           # one row of the others but the last
        row = at[i] + lens[i] // 2
        v[row, :, 9] = math.nan
        if i < 5:
            k[row, :, 0] = 40.0
    refill(s, k, v, dtype)
    q = randn(len(lens), 6, d, seed=3)
    q[..., 0] = 40.0                              # 40 * 40 / d^0.5: 100 and more e-folds above the others
    q = q.to(dtype)
    got, lse = run(s, q)
    with np.errstate(invalid="ignore"):
        ref, ref_lse, bound, lse_bound = s.plain(q, d ** -0.5, 0)
    assert (np.abs(lse - ref_lse) <= lse_bound).all()
    assert np.isnan(got[:6]).all() and (np.abs(got[6] - ref[6]) <= bound[6]).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,dtype", KINDS[2:])
def test_sum_with_infinite_scales(kind, dtype, d):
    """So do value rows whose scale is infinite (which the quantizer does not write): their streams have
    no finite channel, the log-sum-exp is the keys', scored or not, alone or behind a shared prefix."""
    lens = [1, 40, 3000, 60, 700, 33]
    s = Held(lens, 2, d, 16, kind, dtype, seed=d)
    q = randn(len(lens), 6, d, seed=3).to(dtype)
    at = [int(s.slots[i][n // 2]) for i, n in enumerate(lens[:5])]
    s.cache.v_scales[[x // 16 for x in at], :, [x % 16 for x in at]] = math.inf
    s.cache.v_scales[[int(x) // 16 for x in s.slots[3]], :, [int(x) % 16 for x in s.slots[3]]] = math.inf      # (all rows)
    got, lse = run(s, q)
    ref, ref_lse, bound, lse_bound = s.plain(q, d ** -0.5, 0)
    assert (np.abs(lse - ref_lse) <= lse_bound).all()
    assert not np.isfinite(got[:5]).any() and (np.abs(got[5] - ref[5]) <= bound[5]).all()
    # (slopes of zero, and a prefix of no tokens: as without)
    table, lengths = s.args()
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    for out, sums in (run(s, q, slopes=torch.zeros(6, device="cuda")), tq.shared_prefix_attention(
            s.cache, q.cuda(), torch.tensor([0, len(lens)], dtype=torch.int32, device="cuda"), table[:1], none, table, lengths, return_lse=True)):
        out, sums = (x.cpu().double().numpy() if hasattr(x, "cpu") else x for x in (out, sums))
        assert (np.abs(sums - ref_lse) <= lse_bound).all()
        assert not np.isfinite(out[:5]).any() and (np.abs(out[5] - ref[5]) <= bound[5]).all()


@pytest.mark.parametrize("d,lens", [(64, [1, 40, 0, 5000]), (128, [300, 17, 9000]), (256, [200, 3]), (256, [4100, 64]), (64, [70000])])
@pytest.mark.parametrize("exponent", [127, 120, 0, -60, -90])
def test_bf16_values_of_any_size(exponent, d, lens):
    """Values up to bf16's largest, and far below one: the result is as good as at one."""
    say("values of 2^", exponent, d, lens)
    s = Held(lens, 2, d, 16, "bf16", BF16, seed=d)
    v = randn(sum(lens), 2, d, seed=2).clamp(-1.9, 1.9).double()
    v[:, :, 3] = 1.9921875                        # times 2^127: the largest value there is
    v[:, :, 4] = -v[:, :, 3]
    refill(s, randn(sum(lens), 2, d, seed=1), v * 2.0 ** exponent, BF16)
    s.v = s.v * 2.0 ** -exponent
    for scale in (None, 0.0):                     # (0: all weights alike)
        q = randn(len(lens), 8, d, seed=3).to(BF16)
        got, lse = run(s, q, scale=scale)
        ref, ref_lse, bound, lse_bound = s.plain(q, d ** -0.5 if scale is None else scale, 0)
        live = np.isfinite(ref_lse)
        bound[live] += 2.0 ** (-133 - exponent) - 2.0 ** -24     # (no floor but the type's own smallest step)
        assert np.isfinite(got).all()
        over = (np.abs(got * 2.0 ** -exponent - ref) - bound).max()
        assert over <= 0, over
        assert (np.abs(lse - ref_lse)[live] <= lse_bound[live]).all() and np.isinf(lse[~live]).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,dtype", KINDS)
def test_weights_keep_fp32s_bits(kind, dtype, d):
    """Two keys of all but one score, values 1 and -1, beside a larger one of value 0: the
    result is what the two weights differ by."""
    batch, heads, gen = 256, 2, torch.Generator().manual_seed(1)
    s = Held([3] * batch, heads, d, 16, kind, dtype, seed=d)
    k, v = torch.zeros(3 * batch, heads, d), torch.zeros(3 * batch, heads, d)
    k[:, :, 0] = torch.rand(3 * batch, heads, generator=gen)
    k[..., 1] = 1.0
    k[0::3, :, 1] = 1.2
    v[1::3], v[2::3] = 1.0, -1.0
    refill(s, k, v, dtype)
    q = torch.zeros(batch, 8, d)
    q[..., 0] = 2.0 ** -11
    q[..., 1] = 4.0 * torch.rand(batch, 8, generator=gen)
    q = q.to(dtype)
    got, _ = run(s, q, scale=1.0)
    for i in range(batch):
        kk, vv, qq = s.k[3 * i:3 * i + 3], s.v[3 * i:3 * i + 3], q[i].double().numpy()
        for h in range(8):
            x = kk[:, h // 4] @ qq[h]
            w = np.exp(x - x.max())
            w /= w.sum()
            o = w @ vv[:, h // 4]
            bound = ulp(dtype) * np.abs(o) + 2.0 ** -20 * (w @ np.abs(vv[:, h // 4])) + 2.0 ** -24
            over = (np.abs(got[i, h] - o) - bound).max()
            assert over <= 0, (i, h, over)


@pytest.mark.parametrize("kind,top", [("4", 7), ("8", 448)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_past_the_largest_scale(kind, top, d):
    """bf16 rows whose scale, max|x| / top, no fp16 number holds have the scale NaN, as
    rows that are not finite; the largest ones below keep theirs."""
    c = make_cache(2, 16, 2, d, kind)
    x = randn(6, 2, d, seed=d).to(BF16)
    x[1, 0, 7] = top * 65536.0                    # / top: 65536, which rounds to infinity
    x[2, 1, d - 1] = -top * 65536.0
    x[3, 0, 0] = 3.3e38
    x[4, 0, 11] = top * 65536.0 * 0.995           # the next bf16 number below the first: 65280 or less
    assert float(x[4, 0, 11]) / top < 65504 and float(x[1, 0, 7]) / top == 65536
    slots = torch.arange(6).cuda()
    tq.kv_append(c, x.cuda(), x.neg().cuda(), slots)
    dead = torch.zeros(6, 2, dtype=torch.bool)
    dead[1, 0] = dead[2, 1] = dead[3, 0] = True
    for got, want in zip(tq.kv_read(c, slots, bf16=True), (x, x.neg())):
        got, want = got.cpu().double(), want.double()
        alive = int((~got[dead].isnan()).sum())
        assert alive == 0
        step = want.abs().amax(-1, keepdim=True) / top
        # half a code (8 bits: of the largest binade, 32 steps of its scale), the scale's and the result's rounding
        bound = step * (0.5 if kind == "4" else 16.0) + want.abs() * 2.0 ** -7 + step * 2.0 ** -9
        assert ((got - want).abs() <= bound)[~dead].all()


@pytest.mark.parametrize("kind,dtype", KINDS[:2])
@pytest.mark.parametrize("lens", [[40, 9], [5000, 33]])
def test_infinite_values(kind, dtype, lens):
    """A live value that is infinite leaves no finite number in its channel, and all
    others as they were."""
    s = Held(lens, 2, 128, 16, kind, dtype, seed=2)
    k, v = randn(sum(lens), 2, 128, seed=1), randn(sum(lens), 2, 128, seed=2)
    q = randn(2, 8, 128, seed=3).to(dtype)
    refill(s, k, v, dtype)
    clean, clean_lse = run(s, q)
    v[5, 0, 17], v[7, 1, 100], v[lens[0] - 1, 1, 3] = math.inf, -math.inf, math.inf
    refill(s, k, v, dtype)
    got, lse = run(s, q)
    hit = np.zeros(got.shape, bool)
    hit[0, :4, 17] = hit[0, 4:, 100] = hit[0, 4:, 3] = True
    assert not np.isfinite(got[hit]).any() and np.array_equal(got[~hit], clean[~hit])
    assert np.array_equal(lse, clean_lse)


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -110, -2.0 ** -104])
@pytest.mark.parametrize("lens", [[40, 9], [5000, 33]])
def test_scales_next_to_zero(lens, scale):
    """Products q . k far above what a scale next to zero leaves of them: the score is
    their product also there, and zero with a scale of zero."""
    s = Held(lens, 2, 128, 16, "bf16", BF16, seed=2)
    refill(s, 2.0 ** 50 * randn(sum(lens), 2, 128, seed=1), randn(sum(lens), 2, 128, seed=2), BF16)
    q = (2.0 ** 50 * randn(2, 8, 128, seed=3)).to(BF16)
    got, lse = run(s, q, scale=scale)
    ref, ref_lse, bound, lse_bound = s.plain(q, scale, 0)
    over, lse_over = (np.abs(got - ref) - bound).max(), (np.abs(lse - ref_lse) - lse_bound).max()
    assert over <= 0 and lse_over <= 0, (over, lse_over)
