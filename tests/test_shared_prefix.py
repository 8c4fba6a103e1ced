"""Attention of one new token with capped and biased scores, and over a prefix that a group of
streams shares, against plain forms in 64 bits; their refusals on the CPU.

Tolerances as in test_prompt_attention; the attention of one token holds a weight to 2^-15
at least, so that keys of a stream's own tokens are within what a prefix's are."""
import math

import numpy as np
import pytest

import paper_2606_01556_amd as tq
from test_kvcache import BF16, F16, FAKE, KINDS, ROWS, Streams, attend, desc, randn, say, ulp
from test_prompt_attention import Prompts, scores

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _wait():
    yield
    if torch.cuda.is_available():
        torch.cuda.synchronize()


def check(got, lse, ref, ref_lse, bound, lse_bound):
    got, lse = got.cpu().double().numpy(), lse.cpu().double().numpy()
    assert not np.isnan(got).any()
    assert (np.abs(got - ref) <= bound).all(), (np.abs(got - ref) - bound).max()
    empty = np.isinf(ref_lse)
    np.testing.assert_array_equal(lse[empty], ref_lse[empty])
    assert (np.abs(lse[~empty] - ref_lse[~empty]) <= lse_bound[~empty]).all()
    assert (got[empty] == 0).all()


# ------------------------------------------------------------------ one token, scored
def test_scored_validation():
    L = tq.lib()

    def call(c=None, q=ROWS, dt=0, b=0, hq=4, pt=FAKE, stride=4, pages=4, ln=FAKE, s=None, out=FAKE, lse=None, scratch=FAKE):
        return L.tq_paged_attention_scored(c or desc(), q, dt, b, hq, pt, stride, pages, ln, s or scores(), out, lse, scratch, None)

    assert call() == 0 and call(s=scores(softcap=30.0, slopes=FAKE, window=5)) == 0
    assert L.tq_paged_attention_scored(desc(), ROWS, 0, 0, 4, FAKE, 4, 4, FAKE, None, FAKE, None, None, None) == 1
    assert call(b=1, pages=400, scratch=None) == 1 and call(q=None) == 1 and call(out=None) == 1
    for bad in (dict(b=-1), dict(hq=3), dict(pages=0), dict(stride=-4), dict(s=scores(window=-1)), dict(s=scores(scale=math.inf)),
                dict(s=scores(softcap=-1.0)), dict(s=scores(softcap=math.nan))):
        assert call(**bad) == 2, bad
    assert call(dt=1) == 5 and call(s=scores(slopes=FAKE + 1)) == 6 and call(lse=FAKE + 2) == 6


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens", [[1, 0, 40, 300], [9000, 33]])
def test_scored_token(kind, dtype, d, lens):
    say("scored", kind, dtype, d, lens)
    new = [min(n, 1) for n in lens]
    for group in (4, 20, 40):
        s = Prompts(lens, new, 2, d, 16, kind, dtype)
        q = (6.0 * randn(len(lens), 2 * group, d, seed=9)).to(dtype)
        slopes = torch.exp2(-8.0 * (torch.arange(2 * group) + 1) / (2 * group))
        live = np.array(lens) > 0
        for kw in (dict(softcap=20.0), dict(slopes=slopes, window=200), dict(softcap=50.0, slopes=-slopes / 64, scale=-0.06)):
            cuda = dict(kw, slopes=kw["slopes"].cuda()) if "slopes" in kw else kw
            got, lse = tq.paged_attention(s.cache, q.cuda(), *s.args(), return_lse=True, **cuda)
            plain = dict(kw)
            scale = plain.pop("scale", d ** -0.5)
            ref, ref_lse, bound, lse_bound = s.plain(q[live], scale, **plain)
            check(got[live], lse[live], ref, ref_lse, bound, lse_bound)
            assert (got[~live] == 0).all() and torch.isinf(lse[~live]).all()


@gpu
def test_scored_with_nothing_is_the_plain_call():
    say("nothing")
    s = Streams([300, 0, 5000], 2, 128, 16, "f16", F16)
    q = randn(3, 8, 128, seed=1).half().cuda()
    table, lengths = s.args()
    ref = tq.paged_attention(s.cache, q, table, lengths)
    assert torch.equal(tq.paged_attention(s.cache, q, table, lengths, softcap=0.0, slopes=None), ref)
    # a slope of zero and a cap far above the scores leave them as they are
    attend(s, q.cpu(), slopes=torch.zeros(8, device="cuda"))
    with pytest.raises(ValueError):
        tq.paged_attention(s.cache, q, table, lengths, softcap=-1.0)
    with pytest.raises(ValueError):
        tq.paged_attention(s.cache, q, table, lengths, slopes=torch.zeros(7, device="cuda"))


# ------------------------------------------------------------------ a shared prefix
class Shared(Prompts):
    """Groups' prefixes and streams' own tokens in one cache: the first `groups` of lens are prefixes."""

    def __init__(self, shared, members, own, *a, **kw):
        super().__init__(list(shared) + list(own), [0] * (len(shared) + len(own)), *a, **kw)
        self.shared, self.members, self.own = list(shared), list(members), list(own)

    def call(self, q, **kw):
        g = len(self.shared)
        table, lengths = self.args()
        return tq.shared_prefix_attention(self.cache, q.cuda(), torch.tensor(self.members, dtype=torch.int32).cuda(), table[:g],
                                          lengths[:g], table[g:], lengths[g:], **kw)

    def plain(self, q, scale, **kw):
        """Every stream as one of its prefix and its own tokens."""
        g, ends = len(self.shared), np.cumsum([0] + self.lens)
        rows = [(self.k[a:b], self.v[a:b]) for a, b in zip(ends, ends[1:])]
        parts = []
        for i, n in enumerate(self.own):
            mine = [j for j in range(g) if self.members[j] <= i < self.members[j + 1]]
            pieces = [rows[j] for j in mine] + [rows[g + i]]
            one = object.__new__(Prompts)
            one.cache, one.k, one.v = self.cache, np.concatenate([p[0] for p in pieces]), np.concatenate([p[1] for p in pieces])
            one.lens, one.new, one.starts = [len(one.k)], [1], np.array([0, 1])
            parts.append(Prompts.plain(one, q[i:i + 1], scale, **kw))
        return [np.concatenate(x) for x in zip(*parts)]


SHARED = [([100], [0, 5], [3, 0, 70, 1, 200]), ([64, 0, 1000], [0, 2, 3, 40], [(i * 37) % 130 for i in range(40)]),
          ([20000], [1, 3], [5, 9, 0, 0, 12]), ([300, 5], [0, 0, 2], [6000, 40])]


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("shape", range(len(SHARED)))
def test_shared_prefix(kind, dtype, d, shape):
    say("shared", kind, dtype, d, SHARED[shape])
    for heads, group in ((2, 4), (1, 7), (1, 33)):
        s = Shared(*SHARED[shape], heads, d, 16, kind, dtype)
        q = (1.3 * randn(len(s.own), heads * group, d, seed=9)).to(dtype)
        check(*s.call(q, return_lse=True), *s.plain(q, d ** -0.5))
        check(*s.call(q, return_lse=True, exact=True), *s.plain(q, d ** -0.5, exact=True))


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
def test_shared_prefix_scores(kind, dtype):
    say("shared scores", kind, dtype)
    s = Shared([500, 90], [0, 4, 9], [1, 40, 300, 0, 17, 64, 65, 1, 2], 2, 128, 32, kind, dtype)
    q = (6.0 * randn(9, 10, 128, seed=9)).to(dtype)
    slopes = torch.exp2(-8.0 * (torch.arange(10) + 1) / 10)
    for kw in (dict(softcap=25.0), dict(slopes=slopes), dict(softcap=10.0, slopes=slopes / 8)):
        cuda = dict(kw, slopes=kw["slopes"].cuda()) if "slopes" in kw else kw
        check(*s.call(q, return_lse=True, **cuda), *s.plain(q, 128 ** -0.5, **kw))
    assert torch.equal(s.call(q, scale=128 ** -0.5), s.call(q))


@gpu
def test_shared_prefix_is_the_streams_by_themselves():
    """The same tokens as one stream each, prefix pages in every stream's table."""
    say("themselves")
    s = Shared([256], [0, 6], [0, 16, 5, 100, 31, 64], 2, 128, 16, "f16", F16)
    q = randn(6, 8, 128, seed=1).half().cuda()
    table, lengths = s.args()
    joined = torch.cat((table[:1].expand(6, -1)[:, :16], table[1:]), 1).contiguous()
    got, lse = s.call(q, return_lse=True)
    ref, ref_lse = tq.paged_attention(s.cache, q, joined, lengths[1:] + 256, return_lse=True)
    # (each is within the bounds of its own tests of the exact one)
    _, _, bound, lse_bound = s.plain(q.cpu(), 128 ** -0.5)
    assert (np.abs((got.double() - ref.double()).cpu().numpy()) <= 2 * bound).all()
    assert (np.abs((lse - ref_lse).cpu().numpy()) <= 2 * lse_bound).all()


def test_shared_prefix_validation():
    L = tq.lib()

    def call(c=None, q=ROWS, dt=0, b=0, hq=4, g=1, m=FAKE, ptab=FAKE, pstride=4, ppages=4, plen=FAKE, pt=FAKE, stride=4, pages=4,
             ln=FAKE, s=None, out=FAKE, lse=None, scratch=FAKE):
        return L.tq_shared_prefix_attention(c or desc(), q, dt, b, hq, g, m, ptab, pstride, ppages, plen, pt, stride, pages, ln,
                                            s or scores(), out, lse, scratch, None)

    assert call() == 0 and call(scratch=None) == 0 and call(s=scores(softcap=3.0, slopes=FAKE)) == 0
    for bad in (dict(q=None), dict(m=None), dict(ptab=None), dict(plen=None), dict(pt=None), dict(ln=None), dict(out=None),
                dict(b=1, scratch=None)):
        assert call(**bad) == 1, bad
    for bad in (dict(b=-1), dict(b=65536), dict(b=65535, hq=1024, pages=1, ppages=1), dict(g=0), dict(g=65536), dict(hq=3), dict(ppages=0), dict(pages=0), dict(pstride=-1),
                dict(stride=-1), dict(s=scores(window=3)), dict(s=scores(softcap=-1.0)), dict(ppages=(1 << 26) + 1)):
        assert call(**bad) == 2, bad
    assert call(dt=1) == 5 and call(c=desc(head_dim=32)) == 7
    for bad in (dict(m=FAKE + 2), dict(ptab=FAKE + 2), dict(plen=FAKE + 2), dict(pt=FAKE + 2), dict(ln=FAKE + 2), dict(out=FAKE + 8),
                dict(lse=FAKE + 1), dict(scratch=FAKE + 8), dict(s=scores(slopes=FAKE + 2))):
        assert call(**bad) == 6, bad
    size = lambda b, g=1, c=None, pages=4: L.tq_shared_prefix_attention_scratch_bytes(c or desc(), b, 4, g, pages, 4)
    assert size(1) > 0 and size(0) == 0 and size(-1) == 0 and size(1, g=0) == 0 and size(1, pages=0) == 0


@gpu
def test_shared_prefix_refusals_and_limits():
    say("refusals")
    s = Shared([100, 50], [0, 2, 4], [3, 0, 70, 1], 2, 128, 16, "f16", F16)
    q = randn(4, 8, 128, seed=1).half().cuda()
    table, lengths = s.args()
    m = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    call = lambda c=s.cache, x=q, mm=m, pt=table[:2], pl=lengths[:2], t=table[2:], n=lengths[2:], **kw: tq.shared_prefix_attention(
        c, x, mm, pt, pl, t, n, **kw)
    ref = call()
    for kw, kind in ((dict(x=q[:3]), ValueError), (dict(x=q.cpu()), ValueError), (dict(mm=m.long()), TypeError), (dict(mm=m[:1]), ValueError),
                     (dict(mm=m[:2]), ValueError), (dict(pl=lengths[:1]), ValueError), (dict(n=lengths[:2]), ValueError),
                     (dict(t=table[:2]), ValueError), (dict(slopes=torch.zeros(2, device="cuda")), ValueError),
                     (dict(softcap=math.nan), ValueError), (dict(scale=math.inf), tq.TQError), (dict(c=1), TypeError)):
        with pytest.raises(kind):
            call(**kw)
    # a strided q, bounds outside the batch, lengths outside the tables
    big = torch.zeros(4, 10, 160, device="cuda", dtype=F16)
    big[:, 1:9, 8:136] = q
    assert torch.equal(call(x=big[:, 1:9, 8:136]), ref)
    assert torch.equal(call(mm=torch.tensor([-3, 2, 1 << 30], dtype=torch.int32, device="cuda")), ref)
    table[table < 0] = 0
    full = call(pl=torch.tensor([1 << 30, -1], dtype=torch.int32, device="cuda"), n=lengths[2:] * 0 - 5)
    assert (full[2:] == 0).all() and (full[:2] != 0).any()
    assert call(x=q[:0], t=table[:0], n=lengths[:0], mm=m * 0).shape == (0, 8, 128)


@gpu
def test_shared_prefix_other_stream_and_graph():
    say("graph")
    s = Shared([700, 90], [0, 4, 9], [1, 40, 300, 0, 17, 64, 65, 1, 2], 2, 128, 32, "8", F16)
    q = randn(9, 8, 128, seed=1).half().cuda()
    table, lengths = s.args()
    m = torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda")
    call = lambda **kw: tq.shared_prefix_attention(s.cache, q, m, table[:2], lengths[:2], table[2:], lengths[2:], **kw)
    ref = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, ref)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call()
        graphs.append((g, out))
    keep = q.clone()
    for i in range(3):
        q.copy_(keep if i != 1 else -keep)
        want = call()
        for g, out in graphs:
            out.zero_()
            g.replay()
        torch.cuda.synchronize()
        for g, out in graphs:
            assert torch.equal(out, want)


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
def test_shared_prefix_of_the_largest_values(d):
    """bf16's largest value everywhere, and weights as large as either half of a row holds them: keys
    just less than 8 binades above the first 32 of each part, which set its reference."""
    say("largest", d)
    n = 511
    s = Shared([n], [0, 1], [n], 1, d, 16, "bf16", BF16)
    every = torch.cat(s.slots).cuda()
    k, v = torch.zeros(2 * n, 1, d), torch.full((2 * n, 1, d), torch.finfo(BF16).max)
    k[:n, 0, 0] = torch.where((torch.arange(n) % 256) < 32, 0.0, 5.46875)     # (parts of 256 keys)
    k[n:, 0, 0] = torch.where(torch.arange(n) < 256, 0.0, 5.46875)            # (eight wavefronts' first steps)
    tq.kv_append(s.cache, k.to(BF16).cuda(), v.to(BF16).cuda(), every)
    q = torch.zeros(1, 1, d)
    q[..., 0] = d ** 0.5
    for exact in (False, True):
        for scale in (d ** -0.5, 0.0):
            got = s.call(q.to(BF16), scale=scale, exact=exact)
            assert bool((got == torch.finfo(BF16).max).all()), got.flatten()[:4]


@gpu
@pytest.mark.parametrize("exponent", [127, 120, 0, -60, -90])
@pytest.mark.parametrize("shape", [0, 2, 3])
def test_shared_prefix_bf16_values_of_any_size(exponent, shape, monkeypatch):
    say("range", exponent, shape)
    s = Shared(*SHARED[shape], 1, 64, 16, "bf16", BF16)
    total = sum(s.lens)
    v = torch.where(randn(total, 1, 64, seed=3) > 0, 1.0, -1.0) * (1.0 + 0.99 * torch.rand(total, 1, 64, generator=torch.Generator().manual_seed(4)))
    v = (v.double() * 2.0 ** exponent).clamp(-torch.finfo(BF16).max, torch.finfo(BF16).max).to(BF16)
    every = torch.cat(s.slots).cuda()
    k, _ = tq.kv_read(s.cache, every)
    tq.kv_append(s.cache, k, v.cuda(), every)
    s.v = v.double().numpy()
    q = (1.3 * randn(len(s.own), 4, 64, seed=9)).to(BF16)
    got = s.call(q).cpu().double().numpy()
    monkeypatch.setattr(Prompts, "floor", 2.0 ** -133)
    ref, _, bound, _ = s.plain(q, 64 ** -0.5)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= bound).all()


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
def test_shared_prefix_values_that_are_no_number(kind, dtype):
    """A value that is not finite shows in its channels of the streams that see it, and nowhere else;
    what lies behind a prefix's or a stream's end has no part."""
    say("no number", kind, dtype)
    s = Shared([100, 300], [0, 2, 4], [3, 70, 0, 20], 2, 128, 16, kind, dtype)
    q = randn(5, 8, 128, seed=1).to(dtype)
    table, lengths = s.args()
    extra = table[2:3], lengths[2:3]               # a stream of no group, of the first one's own tokens
    m = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    call = lambda: tq.shared_prefix_attention(s.cache, q.cuda(), m, table[:2], lengths[:2], torch.cat((table[2:], extra[0])),
                                              torch.cat((lengths[2:], extra[1])), return_lse=True)
    ref, lse = call()
    bits, page = s.cache.bits, s.cache.page_size
    # (a prefix or a stream's own tokens, one of its keys, and the streams that see it)
    for which, key, sees in ((0, 50, [0, 1]), (1, 299, [2, 3]), (3, 69, [1]), (2, 0, [0, 4])):
        slot = int(s.slots[which][key])
        for value in (math.nan, math.inf):
            rows = s.cache.v if bits == 16 else s.cache.v_scales
            keep = rows.clone()
            at = (slot // page, 1, slot % page) + ((5,) if bits == 16 else ())
            rows[at] = value
            got, got_lse = call()
            hit = np.zeros((5, 8, 128), bool)
            hit[np.ix_(sees, [4, 5, 6, 7], [5] if bits == 16 else np.arange(128))] = True
            np.testing.assert_array_equal(torch.isfinite(got.float()).cpu().numpy(), ~hit)
            other = [i for i in range(5) if i not in sees]
            assert torch.equal(got[other], ref[other]) and torch.equal(got_lse[other], lse[other])
            rows.copy_(keep)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("page", [128, 1024])
def test_shared_prefix_many_groups_and_large_pages(kind, dtype, page):
    """More groups than a search step looks at, some of them empty, some without a prefix."""
    say("groups", kind, dtype, page)
    rng = np.random.default_rng(0)
    sizes = [int(x) for x in rng.choice([0, 0, 1, 2, 3], 150)]
    shared = [int(x) for x in rng.choice([0, 1, 40, 130, 200], 150)]
    s = Shared(shared, np.concatenate(([0], np.cumsum(sizes))), [int(x) for x in rng.choice([0, 1, 30, 70], sum(sizes) + 3)], 1, 64, page,
               kind, dtype)
    q = (1.3 * randn(len(s.own), 4, 64, seed=9)).to(dtype)
    check(*s.call(q, return_lse=True), *s.plain(q, 64 ** -0.5))


def test_shared_prefix_scratch_is_what_the_parts_take():
    """Short own ranges are one part each."""
    L = tq.lib()
    for batch, heads, group, d, pages in ((1024, 8, 32, 256, 1), (512, 8, 4, 128, 2), (3, 1, 1, 64, 1)):
        hq = heads * group
        got = L.tq_shared_prefix_attention_scratch_bytes(desc(kv_heads=heads, head_dim=d, page_size=16), batch, hq, 1, 1, pages)
        most = 4 * batch * hq * (d + 2) + 256                                  # the prefix's
        most += 4 * batch * heads * (group * (d + 2) + 4) + 8 * batch * heads   # the streams' and where they are
        assert 0 < got <= most, (got, most)
