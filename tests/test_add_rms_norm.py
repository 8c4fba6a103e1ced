"""Norm, gate, residual sum and norm between two blocks against a plain form in 64 bits; the
refusals on the CPU.

Tolerances, with u half a unit in the last place of the 16-bit type (2^-11 fp16, 2^-8 bf16,
relative): each result is rounded once, u |y|.  The fp32 arithmetic in front of it: a sum of n
squares by 64 or more lanes with up to 32 terms each and a tree of at most 16 more, 2^-24 each,
a root and a quotient, so 2^-18 of the norm's factor at most; the products and the sum 2^-22 of
|r| + |scale z|.  A norm of the sum takes those over: 2^-18 of its value, and 2^-17 of the
largest term of the sum times the factor (where r and scale z cancel)."""
import math

import pytest

import paper_2606_01556_amd as tq
from test_kvcache import BF16, F16, FAKE, randn, say, ulp

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _wait():
    yield
    if torch.cuda.is_available():
        torch.cuda.synchronize()


def plain(x, residual, weight, post_weight, gate, scale, eps):
    """(sum, its bound, normed, its bound) in 64 bits, without the last rounding's share."""
    z = x.double()
    if post_weight is not None:
        z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt() * post_weight.double()
    if gate is not None:
        z = z * gate.double()
    r = torch.zeros_like(z) if residual is None else residual.double()
    s = r + scale * z
    terms = r.abs() + (scale * z).abs()
    off = 2.0 ** -18 * (scale * z).abs() + 2.0 ** -22 * terms
    if weight is None:
        return s, off, None, None
    factor = weight.double() / (s.square().mean(-1, keepdim=True) + eps).sqrt()
    y = s * factor
    share = off.square().mean(-1, keepdim=True).sqrt() / (s.square().mean(-1, keepdim=True) + eps).sqrt()
    return s, off, y, 2.0 ** -18 * y.abs() + off * factor.abs() + share * y.abs()


def held(x, residual=None, weight=None, post_weight=None, gate=None, scale=1.0, eps=1e-6):
    cuda = lambda t: None if t is None else t.cuda()
    got = tq.add_rms_norm(cuda(x), cuda(residual), cuda(weight), cuda(post_weight), cuda(gate), scale=scale, eps=eps)
    s, s_off, y, y_off = plain(x, residual, weight, post_weight, gate, scale, eps)
    tiny = 2.0 ** -25 if x.dtype == F16 else 2.0 ** -133
    pairs = [(got, s, s_off)] if weight is None else [(got[0], s, s_off), (got[1], y, y_off)]
    for g, want, off in pairs:
        assert g.dtype == x.dtype and g.shape == x.shape
        g = g.cpu().double()
        assert torch.isfinite(g).all()
        assert bool(((g - want).abs() <= ulp(x.dtype) * want.abs() * (1 + 2.0 ** -10) + 2 * off + tiny).all()), ((g - want).abs() - ulp(x.dtype) * want.abs() - 2 * off).max()
    return got


def parts(tokens, n, dtype, seed=0):
    w = lambda i: (1 + 0.2 * randn(n, seed=seed + i)).to(dtype)
    return dict(x=randn(tokens, n, seed=seed + 1).to(dtype), residual=(3 * randn(tokens, n, seed=seed + 2)).to(dtype), weight=w(3),
                post_weight=w(4), gate=randn(tokens, n, seed=seed + 5).to(dtype))


def test_validation():
    L = tq.lib()
    make = lambda **over: tq.kvcache._ResidualNorm(*{**dict(x=FAKE, x_stride=64, residual=FAKE, residual_stride=64, gate=FAKE, gate_stride=64,
                                                            post_weight=FAKE, weight=FAKE, scale=1.0, eps=1e-6), **over}.values())
    call = lambda p=None, t=0, n=64, dt=0, s=FAKE, y=FAKE, **over: L.tq_add_rms_norm(p or make(**over), t, n, dt, s, y, None)
    assert call() == 0 and call(s=None) == 0 and call(y=None, weight=None) == 0 and call(dt=1) == 0
    assert call(residual=None, gate=None, post_weight=None) == 0 and call(gate_stride=0) == 0
    assert L.tq_add_rms_norm(None, 0, 64, 0, FAKE, FAKE, None) == 1
    assert call(x=None) == 1 and call(s=None, y=None) == 1 and call(weight=None) == 1
    for bad in (dict(t=-1), dict(n=0), dict(n=4), dict(n=63), dict(n=32776), dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan),
                dict(scale=math.nan), dict(scale=math.inf)):
        assert call(**bad) == 2, bad
    assert call(dt=2) == 5
    for bad in (dict(x=FAKE + 2), dict(x_stride=4), dict(residual=FAKE + 8), dict(residual_stride=1), dict(gate=FAKE + 2),
                dict(gate_stride=12), dict(post_weight=FAKE + 2), dict(weight=FAKE + 8), dict(s=FAKE + 8), dict(y=FAKE + 2)):
        assert call(**bad) == 6, bad


@gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n", [8, 64, 512, 520, 1000, 1024, 2048, 2056, 4096, 5000, 8192, 8200, 16384, 20000, 32768])
def test_sizes(dtype, n):
    say("sizes", dtype, n)
    for tokens in (1, 3, 5, 66):
        p = parts(tokens, n, dtype)
        held(**p, scale=0.5)
        held(p["x"], p["residual"], p["weight"])


@gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("left_out", range(16))
def test_what_is_left_out(dtype, left_out):
    say("left out", dtype, left_out)
    for n in (72, 4096):
        p = parts(9, n, dtype)
        p = {k: v for i, (k, v) in enumerate(p.items()) if i == 0 or not left_out >> (i - 1) & 1}
        for scale in (1.0, -0.25, 0.0):
            held(**p, scale=scale)
        if "gate" in p:
            held(**dict(p, gate=p["gate"][3]))
        if "weight" in p:
            c = {k: v.cuda() for k, v in p.items()}
            both = tq.add_rms_norm(**c)
            assert torch.equal(tq.add_rms_norm(**c, return_sum=False), both[1])


@gpu
@pytest.mark.parametrize("dtype,exponents", [(F16, [0, 7, -9]), (BF16, [0, 100, 125, -60, -120])])
def test_ranges(dtype, exponents):
    """Squares past fp32's range, and below it with no eps."""
    for e in exponents:
        for n in (64, 4096):
            say("range", dtype, e, n)
            x = torch.where(randn(5, n, seed=1) > 0, 1.0, -1.0) * (1 + 0.9 * torch.rand(5, n, generator=torch.Generator().manual_seed(2)))
            x = (x.double() * 2.0 ** e).to(dtype)
            w = (1 + 0.2 * randn(n, seed=3)).to(dtype)
            held(x, None, w, eps=0.0)
            held(x, None, w, eps=1e-6)
            held(x, (0.5 * randn(5, n, seed=4)).to(dtype), w, w, eps=0.0)
            for eps in (100.0, 1e30):
                held(x, None, w, eps=eps)


@gpu
def test_rows_by_themselves():
    """A row that is not finite leaves the others; zeros give zeros; strides; results over an input."""
    say("rows")
    p = {k: v.cuda() for k, v in parts(7, 264, F16).items()}
    ref = tq.add_rms_norm(**p)
    bad = dict(p, x=p["x"].clone())
    bad["x"][3, 5] = float("nan")
    got = tq.add_rms_norm(**bad)
    keep = [0, 1, 2, 4, 5, 6]
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(got, ref)) and torch.isnan(got[1][3]).all()
    zero = torch.zeros(2, 264, dtype=F16, device="cuda")
    assert all((t == 0).all() for t in tq.add_rms_norm(zero, zero, p["weight"], p["weight"]))
    wide = {k: torch.full((7, 400), float("nan"), dtype=F16, device="cuda") for k in ("x", "residual", "gate")}
    for k, t in wide.items():
        t[:, 16:280] = p[k]
    got = tq.add_rms_norm(**dict(p, **{k: t[:, 16:280] for k, t in wide.items()}))
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    one = {k: p[k][2:3].expand(7, -1) for k in ("x", "residual", "gate")}     # (rows 0 apart)
    got = tq.add_rms_norm(**dict(p, **one))
    assert all(torch.equal(a, b[2:3].expand(7, -1)) for a, b in zip(got, ref))
    # the C call may write over its inputs
    x, r = p["x"].clone(), p["residual"].clone()
    d = tq.kvcache._ResidualNorm(x.data_ptr(), 264, r.data_ptr(), 264, p["gate"].data_ptr(), 264, p["post_weight"].data_ptr(),
                                 p["weight"].data_ptr(), 1.0, 1e-6)
    assert tq.lib().tq_add_rms_norm(d, 7, 264, 0, r.data_ptr(), x.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(r, ref[0]) and torch.equal(x, ref[1])


@gpu
def test_refusals():
    say("refusals")
    p = {k: v.cuda() for k, v in parts(4, 64, F16).items()}
    for over, kind in ((dict(x=p["x"].cpu()), ValueError), (dict(x=p["x"].float()), TypeError), (dict(x=p["x"][0]), ValueError),
                       (dict(x=p["x"][:, :60]), ValueError), (dict(x=p["x"].t()), ValueError), (dict(residual=p["x"][:3]), ValueError),
                       (dict(residual=p["x"].bfloat16()), TypeError), (dict(gate=p["gate"][:, :32]), ValueError),
                       (dict(gate=p["gate"][0, :32]), ValueError), (dict(weight=p["gate"]), ValueError), (dict(post_weight=p["weight"].float()), TypeError),
                       (dict(weight=None, return_sum=False), ValueError), (dict(eps=-1.0), tq.TQError), (dict(scale=math.inf), tq.TQError),
                       (dict(x=None), ValueError)):
        with pytest.raises(kind):
            tq.add_rms_norm(**dict(p, **over))
    assert [t.shape for t in tq.add_rms_norm(p["x"][:0], p["residual"][:0], p["weight"])] == [(0, 64), (0, 64)]


@gpu
@pytest.mark.parametrize("tokens,n", [(1, 4096), (300, 1000)])
def test_other_stream_and_graph(tokens, n):
    say("graph", tokens, n)
    p = {k: v.cuda() for k, v in parts(tokens, n, BF16).items()}
    ref = tq.add_rms_norm(**p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = tq.add_rms_norm(**p, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(other, ref))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = tq.add_rms_norm(**p)
    keep = p["x"].clone()
    for i in range(3):
        p["x"].copy_(keep if i != 1 else -keep)
        want = tq.add_rms_norm(**p)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@gpu
@pytest.mark.parametrize("n", [8, 4096, 8192, 32768])
def test_largest_values(n):
    """Rows of bf16's largest values, whose squares' sum passes fp32's range also of values scaled by 2^-70."""
    say("largest", n)
    sign = torch.where(randn(3, n, seed=1) > 0, 1.0, -1.0).double()
    w = (1 + 0.2 * randn(n, seed=3)).to(BF16)
    for x in (sign * torch.finfo(BF16).max, sign * 2.0 ** 127 * (1 + 0.9 * torch.rand(3, n, generator=torch.Generator().manual_seed(2)))):
        x = x.clamp(-torch.finfo(BF16).max, torch.finfo(BF16).max).to(BF16)
        held(x, None, w, eps=0.0)
        held(x, None, w, eps=1e-6)
        # the norm after a block; the norm of a residual sum
        held(x, randn(3, n, seed=4).to(BF16), w, w)
        y = tq.add_rms_norm((0.4 * x.double()).to(BF16).cuda(), (0.5 * x.double()).to(BF16).cuda(), w.cuda(), return_sum=False)
        _, _, want, off = plain((0.4 * x.double()).to(BF16), (0.5 * x.double()).to(BF16), w, None, None, 1.0, 1e-6)
        assert bool(((y.cpu().double() - want).abs() <= ulp(BF16) * want.abs() * (1 + 2.0 ** -10) + 2 * off).all())
    # an eps as large as a mean whose sum is just past the range
    for eps in (1e33, 1e36, 3e38):
        held((x.double() * 2.0 ** -71).to(BF16), None, w, eps=eps)


@gpu
@pytest.mark.parametrize("n", [8, 4096, 32768])
@pytest.mark.parametrize("exponent", [-126, -129, -133])
def test_smallest_values(n, exponent):
    """Rows down to bf16's smallest values, normed without eps: the factor itself passes fp32's range."""
    say("smallest", n, exponent)
    sign = torch.where(randn(3, n, seed=1) > 0, 1.0, -1.0).double()
    w = (1 + 0.2 * randn(n, seed=3)).to(BF16)
    x = (sign * 2.0 ** exponent * torch.randint(1, 4, (3, n), generator=torch.Generator().manual_seed(2))).to(BF16)
    held(x, None, w, eps=0.0)
    held(x, randn(3, n, seed=4).to(BF16), w, w, eps=0.0)
    held(x, None, w, eps=1e-6)
    held(x, None, w, eps=2.0 ** -140)
