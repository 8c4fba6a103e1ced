"""The attention of one new token in each of its two plans (a work-group per short
range; runs of steps and their join), with the plan that a case takes asserted: a
window that cuts tokens off in runs, many streams of which several hold tokens,
head_dim 256 and wide groups in the plan that the other tests of the operator leave
out, a page table far wider than its streams.

Bounds as in test_kvcache, with 2^-15 as what a weight may be off by in every
format (weights enter the products with 16 bits or more)."""
import math

import numpy as np
import pytest

import paper_2606_01556_amd as tq
from test_kvcache import BF16, F16, FAKE, KINDS, Streams, attend, randn, say, ulp

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _wait():
    yield
    if torch.cuda.is_available():
        torch.cuda.synchronize()


class Held(Streams):
    """Streams whose results are held to `off` of sum_t w_t |v_t| in every format."""
    off = 2.0 ** -15

    def plain(self, q, scale, window, start=None):
        b, hq, d = q.shape
        heads = self.k.shape[1]
        group = hq // heads
        out, lse, bound = np.zeros((b, hq, d)), np.full((b, hq), -np.inf), np.zeros((b, hq, d))
        lse_bound = np.zeros((b, hq))
        at = 0
        for i, n in enumerate(self.lens):
            a = max(0, n - window) if window else 0
            k, v = self.k[at + a:at + n], self.v[at + a:at + n]
            at += n
            if a == n:
                continue
            for j in range(heads):
                h = slice(j * group, (j + 1) * group)
                qh, kh, vh = q[i, h].double().numpy(), k[:, j], v[:, j]
                s = qh @ kh.T * scale
                err = 2.0 ** -19 * (np.abs(qh) @ np.abs(kh).T).max(-1) * abs(scale)
                m = s.max(-1)
                w = np.exp(s - m[:, None])
                total = w.sum(-1)
                lse[i, h] = m + np.log(total)
                w /= total[:, None]
                out[i, h] = w @ vh
                bound[i, h] = ulp(q.dtype) * np.abs(out[i, h]) + (self.off + 2 * err)[:, None] * (w @ np.abs(vh)) + 2.0 ** -24
                lse_bound[i, h] = err + 2.0 ** -18 * (1 + np.abs(lse[i, h]))
        return out, lse, bound, lse_bound

    def in_runs(self, hq, window=0):
        """Whether the call is cut into runs (it needs scratch memory then)."""
        c = self.cache
        d = tq.kvcache._CacheDesc(c.pages, c.page_size, c.kv_heads, c.head_dim, c.bits, 0, FAKE, FAKE, FAKE, FAKE)
        return tq.lib().tq_paged_attention_scratch_bytes(d, len(self.lens), hq, self.table.shape[1], window) > 0

    def forget(self, window):
        """Rows before the window hold NaN, their pages are no longer the stream's."""
        page, pages = self.cache.page_size, self.cache.pages
        for i, n in enumerate(self.lens):
            first = max(0, n - window)
            at, off = self.slots[i][:first] // page, self.slots[i][:first] % page
            for x in self.cache._t:
                if x is not None:
                    x.view(torch.uint8).view(pages, self.cache.kv_heads, page, -1)[at, :, off] = 255
            self.table[i, :first // page] = -1


@pytest.mark.parametrize("d,bits,steps", [(64, 16, 32), (64, 8, 32), (64, 4, 32), (128, 16, 16), (128, 8, 32), (128, 4, 32),
                                          (256, 16, 8), (256, 8, 16), (256, 4, 32)])
def test_plans(d, bits, steps):
    """Which calls run in one launch: those whose ranges have so many steps of 32 tokens,
    by the page table or the window; twice as many from 128 ranges on."""
    c = tq.kvcache._CacheDesc(100, 16, 2, d, bits, 0, FAKE, FAKE, FAKE, FAKE)
    size = lambda batch, tokens, window=0: tq.lib().tq_paged_attention_scratch_bytes(c, batch, 8, tokens // 16, window)
    for batch, s in ((1, steps), (63, steps), (64, 2 * steps), (300, 2 * steps)):
        assert size(batch, 32 * s) == 0 < size(batch, 32 * s + 16)
        assert size(batch, 1 << 20, 32 * s - 15) == 0 < size(batch, 1 << 20, 32 * s - 14)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d,heads,group,page", [(64, 2, 4, 16), (64, 1, 20, 32), (128, 2, 4, 64), (128, 1, 17, 16), (256, 2, 3, 16),
                                                (256, 1, 33, 128)])
def test_window_in_runs(kind, dtype, d, heads, group, page):
    """A window that starts within a step and a tile, in ranges that runs cut."""
    lens = [9000, 2600, 40, 0, 4017, 4001, 4002]
    for window in (2500, 4001):
        say("window in runs", kind, dtype, d, heads, group, page, window)
        s = Held(lens, heads, d, page, kind, dtype, seed=window)
        assert s.in_runs(heads * group, window)
        s.forget(window)
        attend(s, randn(len(lens), heads * group, d, seed=5).to(dtype), window=window)


@gpu
@pytest.mark.parametrize("kind,dtype", [("f16", F16), ("bf16", BF16), ("8", F16), ("4", BF16)])
@pytest.mark.parametrize("batch", [63, 64, 65, 200, 513, 4097, 5200])
def test_many_streams_in_runs(kind, dtype, batch):
    """Runs that find their stream among many, full ones of several lengths around empty
    ones."""
    say("many streams in runs", kind, dtype, batch)
    rng = np.random.default_rng(batch)
    lens = rng.choice([0, 0, 0, 1, 3, 33, 40, 150], batch)
    for i in rng.choice(batch, 3, replace=False):
        lens[i] = 2080 + i % 100
    lens[batch // 2:batch // 2 + batch // 8] = 0
    s = Held([int(n) for n in lens], 2, 64, 16, kind, dtype, seed=batch)
    assert s.in_runs(6)
    attend(s, randn(batch, 6, 64, seed=5).to(dtype))


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (3, 16), (2, 17), (1, 32), (2, 40)])
def test_head_dim_256_in_one_launch(kind, dtype, heads, group):
    say("256 in one launch", kind, dtype, heads, group)
    lens = [256, 0, 1, 17, 33, 64, 65, 240, 255, 31]
    s = Held(lens, heads, 256, 16, kind, dtype, seed=group)
    assert not s.in_runs(heads * group)
    attend(s, randn(len(lens), heads * group, 256, seed=5, scale=1.5).to(dtype))
    window = 241
    s = Held([777, 300, 5, 0], heads, 256, 32, kind, dtype, seed=group)
    assert not s.in_runs(heads * group, window) and s.in_runs(heads * group) == (kind != "4")
    s.forget(window)
    attend(s, randn(4, heads * group, 256, seed=6).to(dtype), window=window)
    # ranges that fill half the CUs: twice the steps
    lens = [int(n) for n in np.random.default_rng(3).integers(0, 513, 128 // heads + 1)]
    lens[0] = 512
    s = Held(lens, heads, 256, 16, kind, dtype, seed=group)
    assert not s.in_runs(heads * group)
    attend(s, randn(len(lens), heads * group, 256, seed=7).to(dtype))


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d,group", [(64, 17), (64, 32), (64, 40), (128, 20), (256, 20)])
def test_wide_groups_in_runs(kind, dtype, d, group):
    say("wide groups in runs", kind, dtype, d, group)
    lens = [2100, 7, 0, 5003]
    s = Held(lens, 2, d, 32, kind, dtype, seed=group, hot=True)
    assert s.in_runs(2 * group)
    attend(s, randn(len(lens), 2 * group, d, seed=5).to(dtype))


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_table_wider_than_the_streams(kind, dtype, d):
    """A table for 131072 tokens: the host cannot know that its streams are short."""
    say("wide table", kind, dtype, d)
    lens = [300, 1, 0, 33, 700]
    s = Held(lens, 2, d, 16, kind, dtype, seed=d)
    s.table = np.concatenate([s.table, np.full((len(lens), 8192 - s.table.shape[1]), -1, np.int32)], 1)
    assert s.in_runs(8)
    attend(s, randn(len(lens), 8, d, seed=5).to(dtype))


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
def test_weights_keep_16_bits(kind, dtype):
    """Many keys of nearly one score with values that all but cancel: what is left shows
    what each weight is off by."""
    say("cancelling values", kind, dtype)
    for n in (60, 5000):
        s = Held([n, n], 2, 128, 16, kind, dtype, seed=11)
        k, v = 0.01 * randn(2 * n, 2, 128, seed=12), torch.ones(2 * n, 2, 128)
        v[1::2] = -1.0
        every = torch.cat(s.slots)
        tq.kv_append(s.cache, k.to(dtype).cuda(), v.to(dtype).cuda(), every.cuda())
        from test_kvcache import stored
        (kv, ks), (vv, vs) = stored(s.cache, every)
        s.k = kv if ks is None else kv * ks.astype(np.float64)[..., None]
        s.v = vv if vs is None else vv * vs.astype(np.float64)[..., None]
        attend(s, randn(2, 8, 128, seed=13).to(dtype), scale=math.sqrt(1 / 128))
