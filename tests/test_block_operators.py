"""The operators of a block run together as a program would: prompts in chunks or whole,
prefixes shared or held by every stream, steps launched one by one or replayed.

Two ways to the same tokens: the layers' sums and the weights' roundings differ in the last
bits between them, which moves a 4-bit code of the next layer here and there (by a seventh
of its group's largest value): the bound is 2 % of the outputs (relative 2-norm), as in
test_decode_block; a wrong page, position or mask is off by a share of order 1."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu

SIZES = dict(hidden=512, mlp=1024, heads=8, kv_heads=2, head_dim=64, rank=16, positions=512)


@pytest.fixture(scope="module")
def example():
    import decode_block
    return decode_block


def tokens_of(*shape, seed=3):
    return torch.randn(*shape, 512, generator=torch.Generator().manual_seed(seed)).half().cuda()


def near(a, b):
    err = float((a - b).float().norm() / b.float().norm())
    print("[case] relative difference", err, flush=True)
    return err < 0.02


@pytest.mark.parametrize("cut", [1, 17, 64])
def test_chunks_of_a_prompt(example, cut):
    print("[case] chunks", cut, flush=True)
    streams, length = 3, 90
    x = tokens_of(streams, length)
    outs = []
    for cuts in ([length], [cut, length - cut]):
        pages = example.Pages(streams, length, 16)
        block = example.Block(**SIZES, pages=pages.count)
        stream, at, rows = torch.arange(streams, device="cuda"), 0, []
        for n in cuts:
            position = torch.arange(at, at + n, device="cuda")
            slots = pages.slots(stream.repeat_interleave(n), position.repeat(streams))
            starts = torch.arange(0, streams * n + 1, n, dtype=torch.int32, device="cuda")
            lengths = torch.full((streams,), at + n, dtype=torch.int32, device="cuda")
            y = block.prompt(x[:, at:at + n].reshape(-1, 512), position.repeat(streams).to(torch.int32), slots, starts,
                             pages.table, lengths)
            rows.append(y.view(streams, n, 512))
            at += n
        outs.append(torch.cat(rows, 1))
    assert near(outs[1], outs[0])


@pytest.mark.parametrize("graph", [False, True])
def test_shared_prefix_is_every_streams_own(example, graph):
    print("[case] shared", graph, flush=True)
    streams, front, length, tokens = 4, 64, 21, 12
    shared, x = tokens_of(front, seed=5), tokens_of(streams, length)
    outs = []
    for held_once in (True, False):
        own = x if held_once else torch.cat((shared.expand(streams, -1, -1), x), 1)
        pages = example.Pages(streams, own.shape[1] + tokens, 16, shared=front if held_once else 0)
        block = example.Block(**SIZES, pages=pages.count)
        y, _ = example.generate(block, pages, own, tokens, graph, shared if held_once else None)
        outs.append(y[:, -(length + tokens):])
    assert near(outs[0][:, :length + 1], outs[1][:, :length + 1])
    # (each way generates from its own last output, whose differences grow with the tokens)
    assert torch.isfinite(outs[0].float()).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_graph_is_the_eager_step(example, bits):
    print("[case] graph", bits, flush=True)
    streams, front, length, tokens = 4, 32, 20, 8
    out = []
    for graph in (False, True):
        pages = example.Pages(streams, length + tokens, 16, shared=front)
        block = example.Block(**SIZES, bits=bits, pages=pages.count)
        out.append(example.generate(block, pages, tokens_of(streams, length), tokens, graph, tokens_of(front, seed=5))[0])
    assert torch.equal(*out)
