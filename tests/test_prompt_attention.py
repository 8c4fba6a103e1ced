"""Attention of many new tokens over the paged cache against a plain form in 64 bits, with
every mask, cap and bias, at the sizes where tiles of 64 keys and 128 rows begin and end;
its refusals on the CPU.

Tolerances (u = half a unit in the last place of the 16-bit type: 2^-11 for fp16, 2^-8 for
bf16, relative to the result's binade at most).  For weights w that sum to 1 and values v:
  u |o|                          the one rounding of the result
  sum_j w_j |v_j| (p + e_j + ē)  p: the one rounding of a weight, 2^-11 where they enter the
                                 second product in fp16 (all caches but bf16 rows), 2^-8 in
                                 bf16, and with two terms (exact) the squares of these; e_j: what a score may be off by, ē its mean over w (the
                                 divisor's share).  e_j = 2^-19 of scale sum |q k| (products and
                                 sums of up to 256 terms in fp32), plus 2^-21 of the cap (an
                                 exponential and a reciprocal of an ulp or two each), plus 2^-22
                                 of the biased score (its sums and the exponent's), plus, with
                                 codes, 2^-18 (the logarithm of a scale, up to 24 binades, in
                                 fp32)
  n 2^-36 max |v|                fp16 weights of n keys end at 2^-25 where the largest is 2^12 or more
  2^-24                          fp16's smallest results
and ē + 2^-18 (1 + |lse|) for the log-sum-exp."""
import math

import numpy as np
import pytest

import paper_2606_01556_amd as tq
from test_kvcache import BF16, F16, FAKE, KINDS, ROWS, Streams, desc, randn, say, ulp

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _wait():
    yield
    if torch.cuda.is_available():
        torch.cuda.synchronize()


class Prompts(Streams):
    """Streams of which the last `new` tokens are new; the plain form of what they attend to."""
    floor = 2.0 ** -24     # (bf16: its smallest results are far smaller)

    def __init__(self, lens, new, *a, **kw):
        super().__init__(lens, *a, **kw)
        self.new = new
        self.starts = np.concatenate(([0], np.cumsum(new))).astype(np.int32)

    def plain(self, q, scale, window=0, prefix=None, first=None, softcap=0.0, slopes=None, exact=False):
        rows, hq, d = q.shape
        heads = self.k.shape[1]
        group = hq // heads
        on = lambda x: torch.as_tensor(np.asarray(x)).cuda()
        wide = not (self.cache.bits == 16 and self.cache.k.dtype == BF16)
        weight = (2.0 ** -11 if wide else 2.0 ** -8) ** (2 if exact else 1)
        new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")
        out, lse, bound, lse_bound = new(rows, hq, d), new(rows, hq) - math.inf, new(rows, hq, d), new(rows, hq)
        at = 0
        for i, (n, t) in enumerate(zip(self.lens, self.new)):
            k, v = self.k[at:at + n], self.v[at:at + n]
            at += n
            r = slice(int(self.starts[i]), int(self.starts[i]) + t)
            if n == 0 or t == 0:
                continue
            p, j = n - t + torch.arange(t, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
            seen = j <= p
            if prefix is not None:
                seen = seen | (j < int(prefix[i]))
            if window:
                seen = seen & (j > p - window)
            if first is not None:
                seen = seen & (j >= on(first)[r][:, None])
            # [heads, tokens * group, ...]: a kv head's rows
            kh, vh = (on(x).double().transpose(0, 1).contiguous() for x in (k, v))
            x = q[r].cuda().double().view(t, heads, group, d).transpose(0, 1).reshape(heads, -1, d)
            seen = seen.repeat_interleave(group, 0)[None]
            s = torch.matmul(x, kh.transpose(1, 2).contiguous()) * scale
            e = 2.0 ** -19 * torch.matmul(x.abs(), kh.abs().transpose(1, 2).contiguous()) * abs(scale)
            if softcap:
                s = softcap * torch.tanh(s / softcap)
                e = e.clamp(max=2 * softcap) + 2.0 ** -21 * softcap
            if slopes is not None:
                slope = torch.as_tensor(np.asarray(slopes)).double().cuda().view(heads, 1, group).expand(-1, t, -1).reshape(heads, -1, 1)
                s = s - slope * (p - j).abs().repeat_interleave(group, 0)[None]
            e = e + 2.0 ** -22 * s.abs() + (2.0 ** -18 if self.cache.bits < 16 else 0.0)
            s = torch.where(seen, s, -math.inf)
            any_seen = seen.any(-1)
            m = torch.where(any_seen, s.amax(-1), 0.0)
            w = torch.exp(s - m[..., None])
            total = torch.where(any_seen, w.sum(-1), 1.0)
            w = w / total[..., None]
            e = torch.where(w > 0, e, 0.0)
            o = torch.matmul(w, vh)
            mean = (w * e).sum(-1)
            off = torch.matmul(w * (weight + e + mean[..., None]), vh.abs())
            top = vh.abs().amax(1, keepdim=True)
            b = ulp(q.dtype) * o.abs() + off + n * 2.0 ** -36 * top + self.floor
            l = torch.where(any_seen, m + torch.log(total), 0.0)
            back = lambda y: y.view(heads, t, group, *y.shape[2:]).transpose(0, 1).reshape(t, hq, *y.shape[2:])
            out[r], bound[r] = back(o), back(b)
            lse[r], lse_bound[r] = back(torch.where(any_seen, l, -math.inf)), back(mean + 2.0 ** -18 * (1 + l.abs()))
        return [y.cpu().numpy() for y in (out, lse, bound, lse_bound)]

    def call(self, q, **kw):
        cuda = lambda x, t=torch.int32: None if x is None else torch.as_tensor(np.asarray(x)).to(t).cuda()
        kw = dict(kw, prefix=cuda(kw.get("prefix")), first=cuda(kw.get("first")), slopes=cuda(kw.get("slopes"), torch.float32))
        return tq.prompt_attention(self.cache, q.cuda(), cuda(self.starts), *self.args(), **kw)


def held(s, q, scale=None, **kw):
    """The call's results, held to the plain form's bounds."""
    got, lse = s.call(q, scale=scale, return_lse=True, **kw)
    ref, ref_lse, bound, lse_bound = s.plain(q, scale if scale is not None else q.shape[-1] ** -0.5, **kw)
    got, lse = got.cpu().double().numpy(), lse.cpu().double().numpy()
    assert not np.isnan(got).any()
    assert (np.abs(got - ref) <= bound).all(), (np.abs(got - ref) - bound).max()
    empty = np.isinf(ref_lse)
    np.testing.assert_array_equal(lse[empty], ref_lse[empty])
    assert (np.abs(lse - ref_lse)[~empty] <= lse_bound[~empty]).all(), (np.abs(lse - ref_lse) - lse_bound)[~empty].max()
    assert (got[empty] == 0).all()
    return got


def prompts(lens, new, heads, group, d, page, kind, dtype, seed=0, pad=0, scale=1.3, **kw):
    s = Prompts(lens, new, heads, d, page, kind, dtype, seed=seed, **kw)
    return s, (scale * randn(sum(new) + pad, heads * group, d, seed=seed + 9)).to(dtype)


# ------------------------------------------------------------------ refusals, on the CPU
def scores(**over):
    s = dict(scale=1.0, softcap=0.0, slopes=None, window=0, exact=0)
    s.update(over)
    return tq.kvcache._Scores(*s.values())


def test_validation():
    L = tq.lib()

    def call(c=None, q=ROWS, dt=0, t=0, b=1, hq=4, starts=FAKE, pt=FAKE, stride=4, pages=4, ln=FAKE, prefix=None, first=None,
             s=None, out=FAKE, lse=None, scratch=FAKE):
        return L.tq_prompt_attention(c or desc(), q, dt, t, b, hq, starts, pt, stride, pages, ln, prefix, first,
                                     s or scores(), out, lse, scratch, None)

    assert call() == 0 and call(b=0) == 0 and call(scratch=None) == 0
    assert call(dt=1, c=desc(dtype=1)) == 0 and call(dt=1, c=desc(bits=8, k_scales=FAKE, v_scales=FAKE)) == 0
    for missing in (dict(q=None), dict(starts=None), dict(pt=None), dict(ln=None), dict(out=None), dict(t=1, pages=400, scratch=None),
                    dict(c=desc(k=None))):
        assert call(**missing) == 1, missing
    assert L.tq_prompt_attention(desc(), ROWS, 0, 0, 1, 4, FAKE, FAKE, 4, 4, FAKE, None, None, None, FAKE, None, FAKE, None) == 1
    for bad in (dict(t=-1), dict(b=-1), dict(t=1, b=0), dict(b=65536), dict(hq=0), dict(hq=3), dict(hq=65536), dict(pages=0),
                dict(pages=(1 << 26) + 1), dict(stride=-4), dict(t=1 << 29), dict(s=scores(window=-1)), dict(s=scores(scale=math.nan)),
                dict(s=scores(scale=math.inf)), dict(s=scores(softcap=-1.0)), dict(s=scores(softcap=math.inf)),
                dict(s=scores(softcap=math.nan))):
        assert call(**bad) == 2, bad
    assert call(dt=1) == 5 and call(dt=3, c=desc(bits=4, k_scales=FAKE, v_scales=FAKE)) == 5
    for bad in (dict(starts=FAKE + 2), dict(pt=FAKE + 2), dict(ln=FAKE + 1), dict(prefix=FAKE + 2), dict(first=FAKE + 1),
                dict(out=FAKE + 8), dict(lse=FAKE + 2), dict(scratch=FAKE + 4), dict(s=scores(slopes=FAKE + 2))):
        assert call(**bad) == 6, bad
    assert call(c=desc(head_dim=96)) == 7
    size = lambda t, b, pages, window=0, c=None: L.tq_prompt_attention_scratch_bytes(c or desc(), t, b, 4, pages, window)
    assert size(1, 1, 400) > 0 and size(100000, 1, 400) == 0 and size(1, 1, 400, window=-1) == 0
    assert size(-1, 1, 400) == 0 and size(1, 1, 400, c=desc(bits=2)) == 0


# ------------------------------------------------------------------ against 64 bits
EDGES = [([1], [1]), ([64, 65], [64, 65]), ([0, 200, 3], [0, 200, 3]), ([127, 0, 129, 400], [5, 0, 129, 33])]


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,group,page", [(1, 1, 16), (2, 4, 32), (3, 5, 16), (1, 16, 128)])
def test_lengths(kind, dtype, d, heads, group, page):
    for lens, new in EDGES:
        say("lengths", kind, dtype, d, heads, group, page, lens, new)
        held(*prompts(lens, new, heads, group, d, page, kind, dtype))


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 150, 1000])
def test_window(kind, dtype, window):
    say("window", kind, dtype, window)
    s, q = prompts([333, 40, 500], [333, 40, 70], 2, 4, 128, 16, kind, dtype)
    held(s, q, window=window)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_intervals_of_many_tiles(kind, dtype, d):
    """Intervals that begin late and hold every number of whole tiles around those that the kernel
    takes two at a time, in front of tiles that not all rows see."""
    say("intervals", kind, dtype, d)
    s, q = prompts([1100, 700], [300, 700], 2, 4, d, 16, kind, dtype)
    for window in range(200, 800, 45):
        held(s, q, window=window)
    first = np.concatenate([np.full(300, 333), np.repeat([0, 131], [131, 569])])
    held(s, q, first=first)
    first[::5] = 1 << 20
    held(s, q, first=first, window=640)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_masks(kind, dtype, d):
    say("masks", kind, dtype, d)
    lens, new = [200, 131, 90], [200, 131, 20]
    s, q = prompts(lens, new, 2, 3, d, 16, kind, dtype)
    held(s, q, prefix=[77, 0, 90])
    held(s, q, prefix=[500, 64, -3], window=50)
    # documents, and rows that see nothing at all
    first = np.concatenate([np.repeat([0, 30, 95], [30, 65, 105]), np.repeat([0, 64], [64, 67]), np.full(20, 60)])
    held(s, q, first=first)
    first[::7] = 1 << 20
    first[3] = -5
    held(s, q, first=first, prefix=[0, 131, 80])


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_caps_and_biases(kind, dtype, d):
    say("caps", kind, dtype, d)
    s, q = prompts([300, 77], [300, 11], 2, 4, d, 32, kind, dtype, scale=6.0)
    slopes = np.float32(2.0) ** -np.arange(1, 9)
    held(s, q, softcap=20.0)
    held(s, q, softcap=0.5, window=70)
    held(s, q, slopes=slopes)
    held(s, q, softcap=30.0, slopes=-slopes / 64, prefix=[200, 70])
    held(s, q, scale=-0.05, softcap=5.0)
    held(s, q, scale=-0.05)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d,lens,new", [(128, [9000], [3]), (128, [3000, 0, 5000, 700], [1, 0, 5, 2]), (64, [20001], [40]),
                                        (256, [3007], [17]), (128, [2500], [700])])
def test_split_keys(kind, dtype, d, lens, new):
    """Few rows: their keys are split over work-groups and joined."""
    say("split", kind, dtype, d, lens, new)
    s, q = prompts(lens, new, 2, 4, d, 16, kind, dtype, hot=True)
    assert tq.lib().tq_prompt_attention_scratch_bytes(desc(kv_heads=2, head_dim=d, page_size=16), q.shape[0], len(lens), 8,
                                                      s.table.shape[1], 0) > 0
    held(s, q)
    held(s, q, window=1000, softcap=25.0)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens,new", [([1, 90, 333], [1, 90, 20]), ([5000, 40], [3, 1])])
def test_exact(kind, dtype, d, lens, new):
    say("exact", kind, dtype, d, lens)
    s, q = prompts(lens, new, 2, 4, d, 16, kind, dtype)
    got = held(s, q, exact=True)
    held(s, q, exact=True, window=70, softcap=9.0)
    # and so what one token gets by itself, but for the last rounding of each
    last = s.starts[1:] - 1
    alone, _, bound, _ = s.plain(q, d ** -0.5, exact=True)
    one = tq.paged_attention(s.cache, q[torch.from_numpy(last.astype(np.int64))].cuda(), *s.args()).cpu().double().numpy()
    assert (np.abs(got[last] - one) <= 2 * bound[last]).all()


@gpu
@pytest.mark.parametrize("kind,dtype", [("f16", F16), ("bf16", BF16), ("4", F16)])
def test_many_streams(kind, dtype):
    """More streams than a search step looks at, most of them empty; padded rows, and a first row past 0."""
    say("many", kind, dtype)
    rng = np.random.default_rng(0)
    new = [int(x) for x in rng.choice([0, 0, 0, 1, 2, 9, 40], 4500)]
    new[4499] = 33
    lens = [n + (int(rng.integers(0, 30)) if n else 0) for n in new]
    s, q = prompts(lens, new, 1, 2, 64, 16, kind, dtype, pad=7)
    got = held(s, q)
    assert (got[-7:] == 0).all()
    # rows in front of the first stream
    s, q = prompts([50, 60], [50, 60], 1, 2, 64, 16, kind, dtype, pad=300)
    shifted = torch.cat((q[110:], q[:110]))
    ref = s.call(q).cpu()
    s.starts = s.starts + 300
    got = s.call(shifted).cpu()
    assert torch.equal(got[300:], ref[:110]) and (got[:300] == 0).all()


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("lens", [[200, 100], [1500]])
def test_what_is_not_seen_has_no_part(kind, dtype, lens):
    """NaN and infinities in keys and values that a row does not see."""
    say("unseen", kind, dtype, lens)
    new = [n if n < 1000 else 40 for n in lens]
    s, q = prompts(lens, new, 2, 4, 128, 16, kind, dtype)
    first = np.concatenate([np.where(np.arange(n - t, n) >= n - t // 2, n - t // 2, 0) for n, t in zip(lens, new)])
    ref, lse = s.call(q, first=first, return_lse=True)
    bad = {16: [float("nan"), float("inf"), -float("inf")], 8: [float("nan")], 4: [float("nan")]}[s.cache.bits]
    for value in bad:
        # the last document's rows: the others do not see them
        at = [int(x) for i, (n, t) in enumerate(zip(lens, new)) for x in s.slots[i][n - t // 2:]]
        page = s.cache.page_size
        idx = torch.tensor(at).cuda()
        for t in (s.cache.k, s.cache.v) if s.cache.bits == 16 else (s.cache.k_scales, s.cache.v_scales):
            t[idx // page, :, idx % page] = value
        if s.cache.bits == 8:
            for t in (s.cache.k, s.cache.v):
                t.view(torch.uint8)[idx // page, :, idx % page] = 0x7f
        got, got_lse = s.call(q, first=first, return_lse=True)
        clean = np.concatenate([np.arange(n - t, n) < n - t // 2 for n, t in zip(lens, new)])
        assert torch.equal(got[clean], ref[clean]) and torch.equal(got_lse[clean], lse[clean])
        if value != value:
            assert torch.isnan(got[~clean].float()).all()


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("lens,new", [([300], [300]), ([1500], [6])])
def test_values_that_are_no_number(kind, dtype, lens, new):
    """A value that is not finite shows in its channel of the rows that see it, and nowhere else."""
    say("values", kind, dtype, lens)
    s, q = prompts(lens, new, 2, 2, 128, 16, kind, dtype)
    ref, lse = s.call(q, return_lse=True)
    n, t = lens[0], new[0]
    key = n - t // 2 - 1
    slot = int(s.slots[0][key])
    page, place = slot // s.cache.page_size, slot % s.cache.page_size
    sees = np.arange(n - t, n) >= key
    channels = np.zeros(128, bool)
    if s.cache.bits == 16:
        s.cache.v[page, 1, place, 5] = float("nan")
        s.cache.v[page, 1, place, 70] = float("inf")
        channels[[5, 70]] = True
    else:
        s.cache.v_scales[page, 1, place] = float("nan")
        channels[:] = True
    got, got_lse = s.call(q, return_lse=True)
    if s.cache.bits == 16:
        assert torch.equal(got_lse, lse)
    else:
        # With codes the reference is that of score plus log2(value scale), and the key's scale now
        # counts as 2^-24: the same sum is rounded from another reference.  Each of the two is
        # within ē + 2^-18 (1 + |lse|) of the exact one, where ē is 2^-18 for the logarithm (the
        # scores themselves are the same), so they differ by 2^-16 (1 + |lse|) at most.
        assert bool(((got_lse - lse).abs() <= 2.0 ** -16 * (1 + lse.abs())).all())
    hit = np.zeros(tuple(got.shape), bool)
    hit[np.ix_(sees, [2, 3], channels)] = True
    finite = torch.isfinite(got.float()).cpu().numpy()
    np.testing.assert_array_equal(finite, ~hit)
    assert torch.equal(got[torch.from_numpy(~hit)], ref[torch.from_numpy(~hit)])


@gpu
@pytest.mark.parametrize("exponent", [127, 120, 0, -60, -90])
@pytest.mark.parametrize("lens,new", [([300], [300]), ([5000], [3])])
def test_bf16_values_of_any_size(exponent, lens, new):
    say("range", exponent, lens)
    s, q = prompts(lens, new, 1, 4, 64, 16, "bf16", BF16)
    v = torch.where(randn(sum(lens), 1, 64, seed=3) > 0, 1.0, -1.0) * (1.0 + torch.rand(sum(lens), 1, 64, generator=torch.Generator().manual_seed(4)) * 0.99)
    every = torch.cat(s.slots).cuda()
    k, _ = tq.kv_read(s.cache, every)
    v = (v.double() * 2.0 ** exponent).to(BF16)
    v = torch.where(torch.isinf(v), torch.finfo(BF16).max, v.double()).to(BF16)
    tq.kv_append(s.cache, k, v.cuda(), every)
    s.v = v.double().numpy()
    s.floor = 2.0 ** -133
    got = s.call(q).cpu().double().numpy()
    ref, _, bound, _ = s.plain(q, 64 ** -0.5)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bound).all()


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("lens,new", [([40000], [5]), ([3000], [300])])
def test_small_weights_beside_a_large_one(kind, dtype, lens, new):
    """A first key that takes most of the weight leaves the many others their share."""
    say("small", kind, dtype, lens)
    s, q = prompts(lens, new, 1, 4, 64, 16, kind, dtype)
    q = torch.ones_like(q)
    k = 0.01 * randn(sum(lens), 1, 64, seed=5)
    k[0] = 20.0 / 8.0 / 1.0
    v = 1.0 + 0.1 * randn(sum(lens), 1, 64, seed=6)
    v[0] = 0.0
    every = torch.cat(s.slots)
    tq.kv_append(s.cache, k.to(dtype).cuda(), v.to(dtype).cuda(), every.cuda())
    from test_kvcache import stored
    (kv, ks), (vv, vs) = stored(s.cache, every)
    s.k = kv if ks is None else kv * ks.astype(np.float64)[..., None]
    s.v = vv if vs is None else vv * vs.astype(np.float64)[..., None]
    held(s, q)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS[:2])
def test_infinite_keys(kind, dtype):
    """Keys whose score is -infinity have no weight."""
    say("infinite", kind, dtype)
    s, q = prompts([300, 70], [300, 4], 2, 2, 64, 16, kind, dtype)
    q[..., 0] = 1.0
    for at in (0, 1, 130, 299):
        slot = int(s.slots[0][at])
        s.cache.k[slot // 16, :, slot % 16, 0] = -float("inf")
        s.k[at, :, 0] = -1e30
    ref, _, bound, _ = s.plain(q, 0.125)
    got = s.call(q).cpu().double().numpy()
    live = slice(2, None)       # (the first two rows see nothing but such keys)
    assert (np.abs(got - ref)[live] <= np.where(np.isfinite(bound), ulp(dtype) * np.abs(ref) + 0.02, 0)[live]).all()


@gpu
def test_strides_tables_and_limits():
    say("strides")
    s, q = prompts([300, 20, 77], [300, 20, 7], 2, 4, 128, 16, "f16", F16)
    ref = s.call(q)
    big = torch.full((q.shape[0], 24, 160), float("nan"), dtype=F16, device="cuda")
    big[:, 4:12, 16:144] = q.cuda()
    table, lengths = s.args()
    wide = torch.full((3, table.shape[1] + 9), -7, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    starts = torch.from_numpy(s.starts).cuda()
    got = tq.prompt_attention(s.cache, big[:, 4:12, 16:144], starts, wide[:, :table.shape[1]], lengths)
    assert torch.equal(got, ref)
    # lengths past the table, below the new tokens, and starts past the rows: taken into range
    odd = torch.tensor([1 << 30, -5, 3], dtype=torch.int32, device="cuda")
    over = starts.clone()
    over[3] = 1 << 30
    table[table < 0] = 0
    out = tq.prompt_attention(s.cache, q.cuda(), over, table, odd)
    assert (out[300:320] == 0).all() and (out[320:324] == 0).all() and bool((out[324:] != 0).any())
    assert tq.prompt_attention(s.cache, q.cuda()[:0], starts * 0, table, lengths).shape == (0, 8, 128)


@gpu
def test_python_refusals():
    say("refusals")
    s, q = prompts([30, 20], [30, 20], 2, 4, 128, 16, "f16", F16)
    q, starts, (table, lengths) = q.cuda(), torch.from_numpy(s.starts).cuda(), s.args()
    call = lambda c=s.cache, x=q, st=starts, t=table, n=lengths, **kw: tq.prompt_attention(c, x, st, t, n, **kw)
    call()
    for kw, kind in ((dict(x=q.cpu()), ValueError), (dict(x=q.bfloat16()), TypeError), (dict(x=q[:, :3]), ValueError),
                     (dict(x=q[..., :64]), ValueError), (dict(st=starts.long()), TypeError), (dict(st=starts[:1]), ValueError),
                     (dict(st=starts[:2]), ValueError), (dict(t=table[:1]), ValueError), (dict(t=table.t()), ValueError),
                     (dict(n=lengths[:1]), ValueError), (dict(prefix=lengths[:1]), ValueError), (dict(first=lengths), ValueError),
                     (dict(slopes=torch.ones(2, device="cuda")), ValueError), (dict(slopes=torch.ones(8, device="cuda").half()), TypeError),
                     (dict(window=-1), ValueError), (dict(softcap=-2.0), ValueError), (dict(softcap=math.inf), ValueError),
                     (dict(scale=math.nan), tq.TQError), (dict(c=None), TypeError), (dict(st=None), ValueError)):
        with pytest.raises(kind):
            call(**kw)
    assert torch.equal(call(window=1 << 40), call())


@gpu
@pytest.mark.parametrize("lens,new", [([300, 77], [300, 9]), ([5000], [3])])
def test_other_stream_and_graph(lens, new):
    say("graph", lens)
    s, q = prompts(lens, new, 2, 4, 128, 16, "8", F16)
    q, starts, (table, lengths) = q.cuda(), torch.from_numpy(s.starts).cuda(), s.args()
    ref = tq.prompt_attention(s.cache, q, starts, table, lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = tq.prompt_attention(s.cache, q, starts, table, lengths, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, ref)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = tq.prompt_attention(s.cache, q, starts, table, lengths)
        graphs.append((g, out))
    keep = q.clone()
    for i in range(3):
        q.copy_(keep if i != 1 else -keep)
        want = tq.prompt_attention(s.cache, q, starts, table, lengths)
        for g, out in graphs:
            out.zero_()
            g.replay()
        torch.cuda.synchronize()
        for g, out in graphs:
            assert torch.equal(out, want)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS[:3])
@pytest.mark.parametrize("lens,new", [([5000], [3]), ([40, 90], [40, 33])])
def test_rows_of_no_stream(kind, dtype, lens, new):
    """Rows before and behind the streams, whole and with split keys."""
    say("no stream", kind, dtype, lens)
    s, q = prompts(lens, new, 2, 4, 64, 16, kind, dtype, pad=150)
    rows = sum(new)
    ref, lse = s.call(q, return_lse=True)
    assert (ref[rows:] == 0).all() and torch.isinf(lse[rows:]).all()
    s.starts = s.starts + 70
    got, got_lse = s.call(torch.cat((q[-70:], q[:-70])), return_lse=True)
    assert torch.equal(got[70:70 + rows], ref[:rows]) and torch.equal(got_lse[70:70 + rows], lse[:rows])
    rest = torch.cat((got[:70], got[70 + rows:]))
    assert (rest == 0).all() and (torch.cat((got_lse[:70], got_lse[70 + rows:])) == -math.inf).all()


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("page", [512, 32768])
def test_large_pages(kind, dtype, page):
    say("pages", kind, dtype, page)
    s, q = prompts([700, 1, 600], [700, 1, 30], 1, 4, 64, page, kind, dtype)
    held(s, q)
    held(s, q, window=330)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
def test_a_row_does_not_depend_on_its_neighbours(kind, dtype):
    """The same rows beside others, and in another place of the call."""
    say("neighbours", kind, dtype)
    s, q = prompts([500, 420], [500, 420], 2, 4, 128, 16, kind, dtype)
    ref = s.call(q)
    other = q.clone()
    other[::3] *= 9.0
    got = s.call(other)
    keep = torch.arange(920) % 3 != 0
    assert torch.equal(got[keep], ref[keep])


@gpu
@pytest.mark.parametrize("kind", ["f16", "4"])
def test_offsets_past_32_bits(kind):
    """Pages past 4 GiB of the cache's tensors."""
    say("offsets", kind)
    heads, d, page = 8, 256, 64
    pages = (1 << 32) // (heads * page * d * (2 if kind == "f16" else 0.5)) + 40
    cache = tq.empty_kv_cache(int(pages), page, heads, d, 16 if kind == "f16" else 4)
    s = Prompts([300, 80], [300, 5], heads, d, page, "f16" if kind == "f16" else "4", F16)
    for big, small in zip(cache._t, s.cache._t):
        if big is not None:
            big[-s.cache.pages:] = small
    q = randn(305, heads * 2, d, seed=9).half().cuda()
    table, lengths = s.args()
    starts = torch.from_numpy(s.starts).cuda()
    ref = tq.prompt_attention(s.cache, q, starts, table, lengths)
    got = tq.prompt_attention(cache, q, starts, torch.where(table < 0, table, table + (cache.pages - s.cache.pages)), lengths)
    assert torch.equal(got, ref)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS[2:])
@pytest.mark.parametrize("lens,new", [([300, 77], [300, 50]), ([1500], [40])])
def test_scales_that_are_not_finite(kind, dtype, lens, new):
    """Infinite and NaN scales of rows that are not seen (behind a row, in another document, before a
    window) have no part; an infinite scale of a value that is seen leaves no channel finite, and
    the log-sum-exp the keys'."""
    say("scales", kind, dtype, lens)
    s, q = prompts(lens, new, 2, 4, 128, 16, kind, dtype)
    n, t = lens[0], new[0]
    row, page = t // 2, s.cache.page_size               # of stream 0; its key is not seen by those before it
    slot = int(s.slots[0][n - t + row])
    places = [(slot // page, slot % page)]
    rows = np.arange(t)
    for kw, hidden in ((dict(), rows < row), (dict(window=9), (rows < row) | (rows >= row + 9)),
                       (dict(first=np.concatenate((np.where(rows > row, n - t + row + 1, 0), np.zeros(sum(new) - t)))), rows != row)):
        hidden = torch.from_numpy(np.concatenate((hidden, np.ones(sum(new) - t, bool))))
        ref, lse = s.call(q, return_lse=True, **kw)
        for scales, values in ((s.cache.k_scales, False), (s.cache.v_scales, True)):
            keep = scales.clone()
            for value in (math.inf, -math.inf, math.nan):
                for p, at in places:
                    scales[p, :, at] = value
                got, got_lse = s.call(q, return_lse=True, **kw)
                assert torch.equal(got[hidden], ref[hidden]) and torch.equal(got_lse[hidden], lse[hidden]), (value, values)
                if values:
                    assert not torch.isfinite(got[~hidden].float()).any()
                    # (the same sum from another reference, as in test_values_that_are_no_number)
                    assert bool(((got_lse - lse).abs() <= 2.0 ** -16 * (1 + lse.abs())).all())
                scales.copy_(keep)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
def test_streams_in_another_order(kind, dtype):
    """What a row gets does not depend on where in the call its stream stands."""
    say("order", kind, dtype)
    s, q = prompts([500, 420, 9], [500, 400, 9], 2, 4, 128, 16, kind, dtype)
    ref, lse = s.call(q, return_lse=True)
    table, lengths = s.args()
    order = [2, 0, 1]
    rows = np.concatenate([np.arange(s.starts[i], s.starts[i + 1]) for i in order])
    starts = torch.tensor(np.cumsum([0] + [s.new[i] for i in order]), dtype=torch.int32).cuda()
    got, got_lse = tq.prompt_attention(s.cache, q[rows].cuda(), starts, table[order].contiguous(), lengths[order].contiguous(), return_lse=True)
    assert torch.equal(got, ref[rows]) and torch.equal(got_lse, lse[rows])
