"""The example's decoder block.

With a 16-bit cache, tokens that are decoded one by one get the outputs that the same
tokens get as part of a prompt.  The layers' sums differ in the last bits between the
two batch sizes, which moves a 4-bit code of the next layer here and there (by a
seventh of its group's largest value): the bound is 2 % of the outputs (relative
2-norm), and a wrong page, position or mask is off by a share of order 1 of the
attention's part.  With quantized caches the layers behind the attention turn its small
differences into such steps everywhere, so there the attention itself is compared, with
64-bit attention over what the cache's bytes stand for, bounded as in the operator's own
tests."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu

SIZES = dict(hidden=512, mlp=1024, heads=8, kv_heads=2, head_dim=64, rank=16, positions=256)


@pytest.fixture(scope="module")
def example():
    import decode_block
    return decode_block


def inputs(streams, length):
    return torch.randn(streams, length, 512, generator=torch.Generator().manual_seed(3)).half().cuda()


@pytest.mark.parametrize("page_size,head_norms", [(16, True), (32, False)])
def test_decode_continues_the_prompt(example, page_size, head_norms):
    streams, length, tokens = 3, 37, 30
    print("[case] decode", page_size, head_norms, flush=True)
    pages = example.Pages(streams, length + tokens, page_size)
    block = example.Block(**SIZES, head_norms=head_norms, pages=pages.table.numel(), page_size=page_size)
    x = inputs(streams, length)
    y, _ = example.generate(block, pages, x, tokens)
    # the same inputs as one prompt
    full = torch.cat((x, example.rms_norm(y[:, length - 1:-1])), 1)
    whole, _ = example.generate(block, pages, full, 0)
    err = (y[:, length:] - whole[:, length:]).float().norm() / whole[:, length:].float().norm()
    print("[case] relative difference", float(err), flush=True)
    assert err < 0.02


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_decode_attends_to_what_was_written(example, bits, monkeypatch):
    from test_kvcache import stored, ulp
    streams, length, tokens = 3, 37, 30
    print("[case] attention", bits, flush=True)
    pages = example.Pages(streams, length + tokens, 16)
    block = example.Block(**SIZES, bits=bits, pages=pages.table.numel())
    seen, attend = [], example.tq.paged_attention

    def record(cache, q, table, lengths):
        out = attend(cache, q, table, lengths)
        seen.append((q.clone(), lengths.clone(), out))
        return out

    monkeypatch.setattr(example.tq, "paged_attention", record)
    example.generate(block, pages, inputs(streams, length), tokens)
    assert [int(s[1][0]) for s in seen] == list(range(length + 1, length + tokens + 1))
    q, lengths, out = seen[-1]
    n = length + tokens
    for i in range(streams):
        slots = pages.slots(torch.full((n,), i, device="cuda"), torch.arange(n, device="cuda")).cpu()
        (k, ks), (v, vs) = stored(block.cache, slots)
        k, v = (x if s is None else x * s.astype(np.float64)[..., None] for x, s in ((k, ks), (v, vs)))
        for h in range(8):
            kh, vh, qh = k[:, h // 4], v[:, h // 4], q[i, h].cpu().double().numpy()
            s = kh @ qh / 8.0
            w = np.exp(s - s.max())
            w /= w.sum()
            off = 2.0 ** -15 + 2.0 ** -18 * np.abs(kh * qh).sum(-1).max() / 8.0
            bound = ulp(torch.float16) * np.abs(w @ vh) + off * (w @ np.abs(vh)) + 2.0 ** -24
            assert (np.abs(out[i, h].cpu().double().numpy() - w @ vh) <= bound).all()


@pytest.mark.parametrize("bits", [16, 4])
def test_graph_is_the_eager_step(example, bits):
    streams, length, tokens = 4, 20, 12
    print("[case] graph", bits, flush=True)
    pages = example.Pages(streams, length + tokens, 16)
    out = []
    for graph in (False, True):
        block = example.Block(**SIZES, bits=bits, pages=pages.table.numel())
        out.append(example.generate(block, pages, inputs(streams, length), tokens, graph)[0])
    assert torch.equal(*out)
