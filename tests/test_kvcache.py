"""The operators between the linear layers (norm and rotation of queries and keys,
the paged key-value cache, the attention of one new token) against plain forms in
64 bits, at the sizes, masks and types where they can go wrong; their refusals on
the CPU.

Tolerances (u = half a unit in the last place of the 16-bit type: 2^-11 for fp16,
2^-8 for bf16, relative to the result's binade at most):
  norm, rotation   u |y| for the one rounding; the fp32 arithmetic in front of it
                   (a sum of 256 squares, a root, a quotient, two products and a
                   difference) is good to 2^-18 of the row's largest value
  cache            bit-exact: the codes and scales are fixed by their definition
  attention        u |o|, plus sum_t w_t |v_t| times what its weights are off by:
                   2^-11 where they enter the second product in fp16, else 2^-15,
                   and the fp32 scores' error, 2^-19 of scale sum |q k| (products
                   and sums of up to 256 terms, one more rounding of the exponent)
"""
import ctypes
import importlib
import math
import os

import numpy as np
import pytest

import paper_2606_01556_amd as tq

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
F16, BF16, F8 = torch.float16, torch.bfloat16, torch.float8_e4m3fn
FAKE = 1 << 20     # 16-byte aligned fake device address; never dereferenced


def say(*a):
    print("[case]", *a, flush=True)


@pytest.fixture(autouse=True)
def _wait():
    yield
    if torch.cuda.is_available():
        torch.cuda.synchronize()


def ulp(dtype):
    return 2.0 ** -11 if dtype == F16 else 2.0 ** -8


def randn(*shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale


# ------------------------------------------------------------------ plain forms (host, 64 bits)
def plain_norm_rope(x, w, pos, table, eps, interleaved):
    y = x.double()
    if w is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    if table is None:
        return y
    row = table.double()[pos.long()][:, None]
    rot = row.shape[-1]
    c, s = row[..., :rot // 2], row[..., rot // 2:]
    out = y.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def e4m3(t):
    """t (float64, |t| <= 448) rounded half to even to e4m3, as values."""
    e = np.floor(np.log2(np.maximum(np.abs(t), 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    return np.round(t / step) * step


def plain_quantize(x, bits):
    """(code values float64, scales float16) of float64 rows x."""
    top = 7.0 if bits == 4 else 448.0
    s = np.minimum((np.abs(x).max(-1).astype(np.float32) / np.float32(top)), np.float32(65504)).astype(np.float16)
    sd = s.astype(np.float64)[..., None]
    t = np.divide(x, sd, out=np.zeros_like(x), where=sd > 0)
    t = np.clip(t, -top, top)
    return (np.round(t) if bits == 4 else e4m3(t)), s


def stored(cache, slots):
    """(code values float64, scales or None) of k and v at slots, by the layout that
    the class documents."""
    out = []
    at, off = slots // cache.page_size, slots % cache.page_size
    for rows, scales in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
        raw = rows.view(torch.uint8) if cache.bits == 8 else rows
        raw = raw.cpu()[at, :, off]
        if cache.bits == 16:
            out.append((raw.double().numpy(), None))
            continue
        if cache.bits == 8:
            val = raw.view(F8).double().numpy()
        else:
            val = tq.tq4_decode(raw.numpy()).astype(np.float64)
        out.append((val, scales.cpu()[at, :, off].numpy()))
    return out


def make_cache(pages, page, heads, d, kind, fill=None):
    bits = {"f16": 16, "bf16": 16, "8": 8, "4": 4}[kind]
    c = tq.empty_kv_cache(pages, page, heads, d, bits, **({"dtype": F16 if kind == "f16" else BF16} if bits == 16 else {}))
    for t in (c.k, c.v, c.k_scales, c.v_scales):
        if t is not None:
            t.view(torch.uint8).fill_(255 if fill is None else fill)     # NaN in every format that has one
    return c


# ------------------------------------------------------------------ refusals, on the CPU
def desc(**over):
    d = dict(pages=4, page_size=16, kv_heads=2, head_dim=128, bits=16, dtype=0, k=FAKE, v=FAKE, k_scales=None,
             v_scales=None)
    d.update(over)
    return tq.kvcache._CacheDesc(*d.values())


ROWS = tq.kvcache._HeadRows(FAKE, 256, 128)
ROPE = dict(q_weight=None, k_weight=None, positions=FAKE, table=FAKE, rotary_dim=128, max_positions=8, interleaved=0,
            eps=1e-6)


def rope(**over):
    return tq.kvcache._NormRope(*{**ROPE, **over}.values())


BAD_CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(bits=8), 1), (dict(bits=4, k_scales=FAKE), 1),
              (dict(pages=0), 7), (dict(page_size=8), 7), (dict(page_size=24), 7), (dict(page_size=65536), 7),
              (dict(kv_heads=0), 7), (dict(kv_heads=1025), 7), (dict(head_dim=96), 7), (dict(bits=2), 7),
              (dict(pages=1 << 30, page_size=32768), 7), (dict(dtype=2), 5), (dict(k=FAKE + 8), 6),
              (dict(bits=8, k_scales=FAKE, v_scales=FAKE + 2), 6)]


@pytest.mark.parametrize("over,code", BAD_CACHES)
def test_cache_validation(over, code):
    L, c = tq.lib(), desc(**over)
    assert L.tq_kv_append(c, ROWS, ROWS, FAKE, 0, 0, None) == code
    assert L.tq_kv_read(c, FAKE, 0, FAKE, FAKE, 0, None) == code
    assert L.tq_qk_norm_rope_append(rope(), c, ROWS, ROWS, ROWS, FAKE, 0, 2, 0, FAKE, None, None) == code
    assert L.tq_paged_attention(c, ROWS, 0, 0, 2, FAKE, 4, 4, FAKE, 1.0, 0, FAKE, None, FAKE, None) == code
    assert L.tq_paged_attention_scratch_bytes(c, 1, 2, 400, 0) == 0


def test_append_and_read_validation():
    L = tq.lib()
    app = lambda c=None, k=ROWS, v=ROWS, s=FAKE, t=0, dt=0: L.tq_kv_append(c or desc(), k, v, s, t, dt, None)
    assert app() == 0 and app(dt=1, c=desc(dtype=1)) == 0 and app(dt=1, c=desc(bits=8, k_scales=FAKE, v_scales=FAKE)) == 0
    assert L.tq_kv_append(None, ROWS, ROWS, FAKE, 0, 0, None) == 1 and app(s=None) == 1
    assert app(k=None) == 1 and app(v=tq.kvcache._HeadRows(None, 0, 0)) == 1
    assert app(t=-1) == 2 and app(t=1 << 29) == 2
    assert app(dt=1) == 5 and app(dt=7, c=desc(bits=8, k_scales=FAKE, v_scales=FAKE)) == 5
    assert app(s=FAKE + 4) == 6
    for bad in ((FAKE + 2, 256, 128), (FAKE, 255, 128), (FAKE, 256, 4)):
        assert app(k=tq.kvcache._HeadRows(*bad)) == 6 and app(v=tq.kvcache._HeadRows(*bad)) == 6
    rd = lambda c=None, s=FAKE, t=0, k=FAKE, v=FAKE, dt=0: L.tq_kv_read(c or desc(), s, t, k, v, dt, None)
    assert rd() == 0 and rd(s=None) == 1 and rd(k=None) == 1 and rd(v=None) == 1
    assert rd(t=-1) == 2 and rd(t=1 << 29) == 2 and rd(dt=1) == 5 and rd(k=FAKE + 8) == 6 and rd(s=FAKE + 4) == 6


def test_norm_rope_validation():
    L = tq.lib()
    call = lambda p=None, q=ROWS, k=ROWS, t=0, hq=4, hkv=2, d=128, dt=0, qo=FAKE, ko=FAKE: L.tq_qk_norm_rope(
        p or rope(), q, k, t, hq, hkv, d, dt, qo, ko, None)
    assert call() == 0 and call(p=rope(rotary_dim=0, positions=None, table=None)) == 0
    assert L.tq_qk_norm_rope(None, ROWS, ROWS, 0, 4, 2, 128, 0, FAKE, FAKE, None) == 1
    assert call(q=None) == 1 and call(k=None) == 1 and call(qo=None) == 1 and call(ko=None) == 1
    assert call(p=rope(positions=None)) == 1 and call(p=rope(table=None)) == 1
    assert call(t=-1) == 2 and call(hq=0) == 2 and call(hkv=0) == 2 and call(d=96) == 2 and call(t=1 << 30) == 2
    for r in (-16, 8, 144, 100):
        assert call(p=rope(rotary_dim=r)) == 2
    assert call(p=rope(max_positions=0)) == 2
    for eps in (-1.0, math.nan, math.inf):
        assert call(p=rope(eps=eps)) == 2
    assert call(dt=2) == 5
    assert call(p=rope(table=FAKE + 4)) == 6 and call(p=rope(positions=FAKE + 2)) == 6
    assert call(p=rope(q_weight=FAKE + 8)) == 6 and call(qo=FAKE + 8) == 6 and call(ko=FAKE + 2) == 6
    both = lambda p=None, c=None, s=FAKE, t=0, hq=4, qo=FAKE, ko=None, dt=0: L.tq_qk_norm_rope_append(
        p or rope(), c or desc(), ROWS, ROWS, ROWS, s, t, hq, dt, qo, ko, None)
    assert both() == 0 and both(s=None) == 1 and both(qo=None) == 1 and both(t=-1) == 2 and both(hq=0) == 2
    assert both(dt=1) == 5 and both(ko=FAKE + 8) == 6 and both(p=rope(rotary_dim=8)) == 2


def test_attention_validation():
    L = tq.lib()

    def call(c=None, q=ROWS, dt=0, b=0, hq=4, pt=FAKE, stride=4, pages=4, ln=FAKE, scale=1.0, window=0, out=FAKE,
             lse=None, scratch=FAKE):
        return L.tq_paged_attention(c or desc(), q, dt, b, hq, pt, stride, pages, ln, scale, window, out, lse, scratch, None)

    assert call() == 0 and call(scratch=None) == 0
    assert call(b=1, pages=400, scratch=None) == 1 and call(q=None) == 1 and call(pt=None) == 1 and call(ln=None) == 1
    assert call(out=None) == 1
    for bad in (dict(b=-1), dict(b=65536), dict(hq=0), dict(hq=3), dict(hq=65536), dict(pages=0), dict(pages=(1 << 26) + 1),
                dict(window=-1), dict(stride=-4), dict(scale=math.nan), dict(scale=math.inf)):
        assert call(**bad) == 2, bad
    assert call(dt=1) == 5 and call(dt=3, c=desc(bits=4, k_scales=FAKE, v_scales=FAKE)) == 5
    assert call(out=FAKE + 8) == 6 and call(lse=FAKE + 2) == 6 and call(scratch=FAKE + 8) == 6 and call(pt=FAKE + 2) == 6
    assert call(b=65535, pages=1 << 20) == 2
    size = lambda *a: L.tq_paged_attention_scratch_bytes(*a)
    assert size(desc(), 1, 3, 400, 0) == 0 and size(None, 1, 4, 400, 0) == 0 and size(desc(), 1, 4, 400, -1) == 0
    assert 0 < size(desc(), 1, 4, 400, 0) < size(desc(), 9, 4, 400, 0)
    # short streams: a work-group holds a range whole
    assert size(desc(), 9, 4, 4, 0) == 0 and size(desc(), 9, 4, 400, 100) == 0


@pytest.mark.parametrize("d", [64, 128, 256])
def test_calls_beyond_a_launch(d):
    """A launch holds 2^32 lanes: calls of more rows are refused before it, attentions of
    more ranges run in fewer work-groups than ranges."""
    L, c = tq.lib(), desc(kv_heads=1024, head_dim=d)
    rows = (1 << 36) // d                       # one more than fit
    row = tq.kvcache._HeadRows(FAKE, 0, 0)
    assert L.tq_kv_append(c, row, row, FAKE, rows // 2048, 0, None) == 2
    assert L.tq_kv_read(c, FAKE, rows // 2048, FAKE, FAKE, 0, None) == 2
    p = rope(rotary_dim=0, positions=None, table=None)
    assert L.tq_qk_norm_rope(p, row, row, rows // 2048, 1024, 1024, d, 0, FAKE, FAKE, None) == 2
    assert L.tq_qk_norm_rope_append(p, c, row, row, row, FAKE, rows // 4096, 2048, 0, FAKE, None, None) == 2
    size = lambda batch: L.tq_paged_attention_scratch_bytes(c, batch, 1024, 1, 0)
    assert size(8191) == 0 < size(8192)


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 4, 128, dtype=F16)
    with pytest.raises(ValueError):
        tq.KVCache(torch.zeros(2, 4, 16, 128, dtype=F16), torch.zeros(2, 4, 16, 128, dtype=F16))
    with pytest.raises(ValueError):
        tq.qk_norm_rope(x, x, None, None)
    for call in (lambda: tq.kv_append(None, x, x, None), lambda: tq.kv_read(None, None),
                 lambda: tq.paged_attention("cache", x, None, None),
                 lambda: tq.qk_norm_rope_append(None, x, x, x, None, None, None)):
        with pytest.raises(TypeError):
            call()
    for bad in (dict(bits=2), dict(head_dim=96), dict(bits=8, dtype=F16), ):
        with pytest.raises(ValueError):
            tq.empty_kv_cache(**{**dict(pages=2, page_size=16, kv_heads=1, head_dim=64, device="cpu"), **bad})


def test_missing_binding_raises(monkeypatch):
    """No fallback: without its built half the binding says what to build."""
    kv = importlib.import_module("paper_2606_01556_amd.kvcache")
    monkeypatch.setattr(kv, "_native", None)
    monkeypatch.setattr(kv, "_HERE", os.path.join(os.path.dirname(kv.__file__), "csrc"))
    with pytest.raises(RuntimeError, match="_tqtorch.so is missing"):
        tq.qk_norm_rope(torch.zeros(1, 2, 64, dtype=F16), torch.zeros(1, 1, 64, dtype=F16), None, None)


@gpu
def test_binding_refuses():
    c16, c4 = tq.empty_kv_cache(4, 16, 2, 128), tq.empty_kv_cache(4, 16, 2, 128, 4)
    new = lambda *s, dtype=F16: torch.zeros(s, dtype=dtype, device="cuda")
    k, slots = new(3, 2, 128), torch.arange(3, device="cuda")
    for a, b in ((c16.k[:, :, :8], c16.v[:, :, :8]), (c16.k, c16.v[:3]), (c16.k.transpose(1, 2), c16.v.transpose(1, 2)),
                 (c16.k.contiguous()[..., :96].contiguous(), c16.v[..., :96].contiguous()), (c16.k[0], c16.v[0]),
                 (c16.k, c16.v.cpu())):
        with pytest.raises(ValueError):
            tq.KVCache(a, b)
    with pytest.raises(TypeError):
        tq.KVCache(c16.k, c16.v.bfloat16())
    with pytest.raises(TypeError):
        tq.KVCache(c16.k.float(), c16.v.float())
    with pytest.raises(ValueError):
        tq.KVCache(c4.k, c4.v)
    with pytest.raises(ValueError):
        tq.KVCache(c4.k, c4.v, c4.k_scales, c4.v_scales[:2])
    with pytest.raises(ValueError):
        tq.KVCache(c16.k, c16.v, c4.k_scales, c4.v_scales)
    with pytest.raises(AttributeError):
        c16.k = c16.v
    moved = tq.empty_kv_cache(4, 16, 2, 128)
    moved.v.data = moved.v.clone()
    with pytest.raises(ValueError):
        tq.kv_append(moved, k, k, slots)
    for bad in (new(3, 3, 128), new(3, 2, 64), new(2, 2, 128), new(3, 2, 256)[..., ::2], new(3, 2 * 132)[:, :264].view(3, 2, 132)[..., 4:],
                k.cpu(), new(3, 256)):
        with pytest.raises(ValueError):
            tq.kv_append(c16, k, bad, slots)
    with pytest.raises(TypeError):
        tq.kv_append(c16, k.bfloat16(), k.bfloat16(), slots)
    with pytest.raises(TypeError):
        tq.kv_append(c4, k, k.bfloat16(), slots)
    for bad in (slots[:2], slots.cpu(), new(6, dtype=torch.int64)[::2], None):
        with pytest.raises(ValueError):
            tq.kv_append(c16, k, k, bad)
    with pytest.raises(TypeError):
        tq.kv_append(c16, k, k, slots.int())
    with pytest.raises(TypeError):
        tq.kv_read(c16, slots, bf16=True)
    pos, table = slots.int(), tq.rope_table(8, 128)
    for args in ((k, new(2, 2, 128), pos, table), (k, k, pos[:2], table), (k, k, None, table), (k, k, pos, table[:, :8].contiguous()),
                 (k, k, pos, table[0]), (k, k, pos, table, new(64)), (k, k, pos, table[::2]), (new(3, 2, 96), new(3, 2, 96), pos, None)):
        with pytest.raises(ValueError):
            tq.qk_norm_rope(*args)
    for args in ((k, k, slots, table), (k, k, pos, table.double()), (k, k.bfloat16(), pos, table), (k, k, pos, table, new(128, dtype=BF16)),
                 (k.float(), k.float(), pos, table)):
        with pytest.raises(TypeError):
            tq.qk_norm_rope(*args)
    q, pt, ln = new(2, 4, 128), new(2, 3, dtype=torch.int32), new(2, dtype=torch.int32)
    for args, kw in (((new(2, 3, 128), pt, ln), {}), ((q, pt[:1], ln), {}), ((q, pt, ln[:1]), {}), ((q, pt[0], ln), {}),
                     ((q, pt.t().contiguous().t(), ln), {}), ((q, pt[:, :0], ln), {}), ((q, pt, ln), {"window": -1}),
                     ((q, pt.cpu(), ln), {}), ((q, pt[:1].expand(2, 3), ln), {})):
        with pytest.raises(ValueError):
            tq.paged_attention(c16, *args, **kw)
    for args in ((q, pt.long(), ln), (q, pt, ln.long()), (q.bfloat16(), pt, ln)):
        with pytest.raises(TypeError):
            tq.paged_attention(c16, *args)
    with pytest.raises(tq.TQError):
        tq.paged_attention(c16, q, pt, ln, scale=math.nan)


# ------------------------------------------------------------------ norm and rotation
def check_turned(got, x, w, pos, table, eps, interleaved):
    ref = plain_norm_rope(x, w, pos, table, eps, interleaved)
    bound = ulp(x.dtype) * ref.abs() + 2.0 ** -18 * ref.abs().amax(-1, keepdim=True) + 2.0 ** -24
    over = ((got.cpu().double() - ref).abs() - bound).max().item()
    assert over <= 0, over


@gpu
@pytest.mark.parametrize("d,rot,norm,interleaved", [
    (128, 128, True, False), (128, 128, False, False), (128, 128, True, True), (128, 64, True, False),
    (128, 48, False, True), (128, 0, True, False), (64, 64, True, False), (64, 32, True, True), (64, 16, False, False),
    (256, 256, True, False), (256, 128, False, True), (256, 240, True, False), (64, 0, False, False)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_norm_rope(d, rot, norm, interleaved, dtype):
    for tokens, hq, hkv in ((1, 1, 1), (3, 5, 1), (67, 8, 3), (33, 32, 8)):
        say("norm_rope", d, rot, norm, interleaved, dtype, tokens, hq, hkv)
        qkv = randn(tokens, hq + 2 * hkv, d, seed=tokens, scale=2.0).to(dtype)
        qkv[0, 0] = 0
        dev = qkv.cuda()
        q, k = dev[:, :hq], dev[:, hq:hq + hkv]
        w = [(1 + 0.3 * randn(d, seed=9 + i)).to(dtype) if norm else None for i in range(2)]
        table = tq.rope_table(301, rot) if rot else None
        pos = torch.arange(tokens, dtype=torch.int32) * 7 % 301
        out = tq.qk_norm_rope(q, k, pos.cuda(), table, *(None if x is None else x.cuda() for x in w), eps=1e-5,
                              interleaved=interleaved)
        for got, x, wt in zip(out, (qkv[:, :hq], qkv[:, hq:hq + hkv]), w):
            assert got.is_contiguous() and got.dtype == dtype and got.shape == x.shape
            check_turned(got, x, wt, pos, None if table is None else table.cpu(), 1e-5, interleaved)
            if not norm and not rot:
                assert torch.equal(got.cpu(), x)


@gpu
def test_norm_rope_one_weight_and_limits():
    """A norm of q alone; positions outside the table go to its ends; no tokens."""
    q, k = (randn(5, 2, 128, seed=i).half().cuda() for i in range(2))
    w, table = (1 + 0.3 * randn(128, seed=2)).half().cuda(), tq.rope_table(10, 128)
    pos = torch.tensor([-3, 0, 9, 10, 1 << 30], dtype=torch.int32, device="cuda")
    got = tq.qk_norm_rope(q, k, pos, table, w)
    same = torch.tensor([0, 0, 9, 9, 9], dtype=torch.int32)
    check_turned(got[0], q.cpu(), w.cpu(), same, table.cpu(), 1e-6, False)
    check_turned(got[1], k.cpu(), None, same, table.cpu(), 1e-6, False)
    none = tq.qk_norm_rope(q[:0], k[:0], pos[:0], table, w)
    assert none[0].shape == (0, 2, 128) and none[1].shape == (0, 2, 128)


def test_rope_table():
    t = tq.rope_table(5, 16, base=100.0, device="cpu").double()
    for p in range(5):
        for i in range(8):
            a = p * 100.0 ** (-2 * i / 16)
            assert abs(t[p, i] - math.cos(a)) < 1e-7 and abs(t[p, 8 + i] - math.sin(a)) < 1e-7


# ------------------------------------------------------------------ the cache
def spread_slots(tokens, pages, page, seed):
    return torch.from_numpy(np.random.default_rng(seed).permutation(pages * page)[:tokens].astype(np.int64))


@gpu
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,dtype", [("f16", F16), ("bf16", BF16), ("8", F16), ("8", BF16), ("4", F16), ("4", BF16)])
def test_append_read(d, kind, dtype):
    for tokens, heads, pages, page in ((1, 1, 1, 16), (37, 3, 5, 16), (130, 8, 3, 64), (70, 2, 1, 256)):
        say("append", d, kind, dtype, tokens, heads, pages, page)
        c = make_cache(pages, page, heads, d, kind)
        kv = randn(tokens, 2 * heads + 1, d, seed=d + tokens, scale=3.0).to(dtype)
        kv[0, 0] = 0                                    # scale 0
        kv[-1, 0, 1:] = 0
        kv[-1, -2] *= 2.0 ** -12                        # small scales
        slots = spread_slots(tokens, pages, page, tokens)
        dev = kv.cuda()
        k, v = dev[:, :heads], dev[:, heads:2 * heads]  # strided views
        before = [t.clone() for t in (c.k.view(torch.uint8), c.v.view(torch.uint8))]
        tq.kv_append(c, k, v, slots.cuda())
        refs = []
        for (val, scale), x in zip(stored(c, slots), (kv[:, :heads], kv[:, heads:2 * heads])):
            x = x.double().numpy()
            if c.bits == 16:
                np.testing.assert_array_equal(val, x)
                refs.append(x)
            else:
                code, s = plain_quantize(x, c.bits)
                np.testing.assert_array_equal(scale.view(np.uint16), s.view(np.uint16))
                np.testing.assert_array_equal(val, code)
                refs.append((code.astype(np.float32) * s.astype(np.float32)[..., None]))
        # nothing else was written
        keep = torch.ones(pages * page, dtype=torch.bool)
        keep[slots] = False
        for old, t in zip(before, (c.k, c.v)):
            now = t.view(torch.uint8)
            o, n = (b.transpose(1, 2).reshape(pages * page, -1).cpu()[keep] for b in (old, now))
            assert torch.equal(o, n)
        for out_bf16 in ([None] if c.bits == 16 else [False, True]):
            out = tq.kv_read(c, slots.cuda(), out_bf16)
            for got, ref in zip(out, refs):
                want = torch.from_numpy(ref).to(got.dtype)
                assert got.shape == want.shape and torch.equal(got.cpu(), want)


@gpu
@pytest.mark.parametrize("kind", ["8", "4"])
def test_quantizer_ties(kind):
    """Rows of scale 1: every code and every tie between two of them."""
    if kind == "4":
        vals = np.arange(-14, 15) / 2.0
    else:
        grid = np.unique(e4m3(np.concatenate([2.0 ** e * (1 + np.arange(8) / 8) for e in range(-6, 9)] + [np.arange(8) * 2.0 ** -9])))
        grid = grid[grid <= 448]
        vals = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2])
        vals = np.concatenate([vals, -vals])
    top = 7.0 if kind == "4" else 448.0
    rows = np.full((-(-len(vals) // 120), 128), 0.0)
    rows[:, 0] = top
    for i, v in enumerate(vals):
        rows[i // 120, 8 + i % 120] = v
    x = torch.from_numpy(rows).half()
    assert np.array_equal(x.double().numpy(), rows)     # all are fp16 values
    x = x[:, None].cuda()
    c = make_cache(2, 64, 1, 128, kind)
    slots = torch.arange(len(rows))
    tq.kv_append(c, x, -x, slots.cuda())
    for (val, scale), sign in zip(stored(c, slots), (1, -1)):
        assert np.all(scale == 1.0)
        np.testing.assert_array_equal(val[:, 0], sign * plain_quantize(rows, c.bits)[0])


@gpu
@pytest.mark.parametrize("kind", ["8", "4"])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_not_finite(kind, dtype, d):
    """A row with an infinity or NaN anywhere reads as NaN, its neighbours as they were
    without it, and an attention that sees it is NaN, through the key or the value."""
    rows, heads, bad = 32, 2, {3: math.inf, 9: -math.inf, 17: math.nan, 30: math.nan}
    k, v = randn(rows, heads, d, seed=1).to(dtype), randn(rows, heads, d, seed=2).to(dtype)
    for side in (0, 1):
        c, clean = (make_cache(3, 16, heads, d, kind) for _ in range(2))
        x = [k.clone(), v.clone()]
        for i, (r, b) in enumerate(bad.items()):
            x[side][r, 1, (i * 37 + 5) % d] = b
        slots = torch.arange(rows).cuda()
        tq.kv_append(c, x[0].cuda(), x[1].cuda(), slots)
        tq.kv_append(clean, k.cuda(), v.cuda(), slots)
        dead = torch.zeros(rows, heads, dtype=torch.bool)
        dead[list(bad), 1] = True
        for s, (got, want) in enumerate(zip(tq.kv_read(c, slots), tq.kv_read(clean, slots))):
            got, want = got.cpu(), want.cpu()
            hit = dead if s == side else torch.zeros_like(dead)
            assert got[hit].isnan().all() and torch.equal(got[~hit], want[~hit])
        q = randn(2, 4, d, seed=3).to(dtype).cuda()
        table = torch.tensor([[0, 1], [1, 0]], dtype=torch.int32).cuda()
        out = tq.paged_attention(c, q, table, torch.tensor([3, 16], dtype=torch.int32).cuda())
        assert out[0].isfinite().all() and out[1, :2].isfinite().all() and out[1, 2:].isnan().all()


@gpu
@pytest.mark.parametrize("kind", ["f16", "8", "4"])
def test_slots_outside(kind):
    """Slots before and past the cache are neither written nor read."""
    c = make_cache(3, 16, 2, 64, kind, fill=0)
    k = randn(6, 2, 64, seed=1).half().cuda()
    slots = torch.tensor([-1, 5, 48, -(1 << 40), 47, 1 << 50], device="cuda")
    tq.kv_append(c, k, k, slots)
    assert all(torch.count_nonzero(t.view(torch.uint8).flatten(2).any(-1)) <= 4 for t in (c.k, c.v))
    a, b = tq.kv_read(c, slots)
    live = torch.tensor([1, 4])
    dead = torch.tensor([0, 2, 3, 5])
    assert torch.equal(a, b) and torch.count_nonzero(a.cpu()[dead]) == 0
    assert ((a.cpu()[live].float() - k.cpu()[live].float()).abs().amax() <= {"f16": 0, "8": 0.25, "4": 0.3}[kind])
    tq.kv_append(c, k[:0], k[:0], slots[:0])
    assert tq.kv_read(c, slots[:0])[0].shape == (0, 2, 64)


@gpu
@pytest.mark.parametrize("kind,dtype", [("f16", F16), ("bf16", BF16), ("8", F16), ("8", BF16), ("4", F16), ("4", BF16)])
@pytest.mark.parametrize("d,rot,interleaved", [(64, 64, False), (128, 128, False), (128, 64, True), (256, 192, False)])
def test_fused_is_the_separate_calls(kind, dtype, d, rot, interleaved):
    tokens, hq, hkv, pages, page = 29, 6, 2, 4, 16
    say("fused", kind, dtype, d, rot, interleaved)
    qkv = randn(tokens, hq + 2 * hkv, d, seed=d).to(dtype).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    table = tq.rope_table(64, rot)
    w = [(1 + 0.3 * randn(d, seed=i)).to(dtype).cuda() for i in range(2)]
    slots = spread_slots(tokens, pages, page, 3)
    slots[4] = -1
    slots = slots.cuda()
    a, b = make_cache(pages, page, hkv, d, kind), make_cache(pages, page, hkv, d, kind)
    q1, k1 = tq.qk_norm_rope(q, k, pos, table, *w, interleaved=interleaved)
    tq.kv_append(a, k1, v, slots)
    q2, k2 = tq.qk_norm_rope_append(b, q, k, v, pos, table, slots, *w, interleaved=interleaved, return_k=True)
    assert torch.equal(q1, q2) and torch.equal(k1, k2)
    for x, y in zip(a._t, b._t):
        assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    c = make_cache(pages, page, hkv, d, kind)
    assert torch.equal(tq.qk_norm_rope_append(c, q, k, v, pos, table, slots, *w, interleaved=interleaved), q1)
    assert torch.equal(c.k.view(torch.uint8), a.k.view(torch.uint8))


# ------------------------------------------------------------------ attention
class Streams:
    """A cache with streams of the given lengths in shuffled pages; every slot that no
    stream holds is NaN (or the largest code, at 4 bits with a NaN scale)."""

    def __init__(self, lens, heads, d, page, kind, src, seed=0, extra=3, hot=False):
        need = [-(-n // page) for n in lens]
        pages = sum(need) + extra
        self.cache = make_cache(pages, page, heads, d, kind)
        order = np.random.default_rng(seed).permutation(pages)
        self.table = np.full((len(lens), max(max(need), 1)), -1, np.int32)    # unused entries: no page
        self.slots, at = [], 0
        for i, (n, p) in enumerate(zip(lens, need)):
            self.table[i, :p] = order[at:at + p]
            at += p
            t = np.arange(n)
            self.slots.append(torch.from_numpy(self.table[i, t // page].astype(np.int64) * page + t % page))
        self.lens = lens
        total = sum(lens)
        if total:
            k = randn(total, heads, d, seed=seed + 1)
            k[..., :3] *= 6.0
            if hot:
                k[::37] *= 8.0                  # a few keys far above the others
            v = randn(total, heads, d, seed=seed + 2)
            every = torch.cat(self.slots)
            tq.kv_append(self.cache, k.to(src).cuda(), v.to(src).cuda(), every.cuda())
            (kv, ks), (vv, vs) = stored(self.cache, every)
            self.k = kv if ks is None else kv * ks.astype(np.float64)[..., None]
            self.v = vv if vs is None else vv * vs.astype(np.float64)[..., None]
        else:
            self.k = self.v = np.zeros((0, heads, d))

    def args(self):
        return torch.from_numpy(self.table).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda()

    def plain(self, q, scale, window, start=None):
        """(out, lse, bound) in 64 bits for q [batch, hq, d]."""
        b, hq, d = q.shape
        heads = self.k.shape[1]
        out, lse, bound = np.zeros((b, hq, d)), np.full((b, hq), -np.inf), np.zeros((b, hq, d))
        lse_bound = np.zeros((b, hq))
        wide = self.cache.k.dtype == F16
        at = 0
        for i, n in enumerate(self.lens):
            a = max(0, n - window) if window else 0
            k, v = self.k[at + a:at + n], self.v[at + a:at + n]
            at += n
            if a == n:
                continue
            for h in range(hq):
                kh, vh, qh = k[:, h * heads // hq], v[:, h * heads // hq], q[i, h].double().numpy()
                s = kh @ qh * scale
                err = 2.0 ** -19 * np.abs(kh * qh).sum(-1).max() * abs(scale)
                m = s.max()
                w = np.exp(s - m)
                lse[i, h] = m + math.log(w.sum())
                w /= w.sum()
                out[i, h] = w @ vh
                off = (2.0 ** -11 if wide else 2.0 ** -15) + 2 * err
                bound[i, h] = ulp(q.dtype) * np.abs(out[i, h]) + off * (w @ np.abs(vh)) + 2.0 ** -24
                lse_bound[i, h] = err + 2.0 ** -18 * (1 + abs(lse[i, h]))
        return out, lse, bound, lse_bound


def attend(s, q, window=0, scale=None, **kw):
    got, lse = tq.paged_attention(s.cache, q.cuda(), *s.args(), window=window, scale=scale, return_lse=True, **kw)
    ref, ref_lse, bound, lse_bound = s.plain(q, scale if scale is not None else q.shape[-1] ** -0.5, window)
    got, lse = got.cpu().double().numpy(), lse.cpu().double().numpy()
    assert not np.isnan(got).any()
    assert (np.abs(got - ref) <= bound).all(), (np.abs(got - ref) - bound).max()
    empty = np.isinf(ref_lse)
    np.testing.assert_array_equal(lse[empty], ref_lse[empty])
    assert (np.abs(lse - ref_lse)[~empty] <= lse_bound[~empty]).all()
    assert (got[empty] == 0).all()
    return got


KINDS = [("f16", F16), ("bf16", BF16), ("8", F16), ("8", BF16), ("4", F16), ("4", BF16)]
LENS = [0, 1, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 255, 257, 300, 0]


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,group,page", [(1, 1, 16), (2, 4, 32), (3, 5, 16), (1, 16, 128), (2, 20, 16)])
def test_attention_lengths(kind, dtype, d, heads, group, page):
    say("attend", kind, dtype, d, heads, group, page)
    s = Streams(LENS, heads, d, page, kind, dtype, seed=d)
    attend(s, randn(len(LENS), heads * group, d, seed=5, scale=1.5).to(dtype))


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("group", [17, 31, 32, 33, 40, 70])
@pytest.mark.parametrize("d,lens", [(64, [0, 40, 300]), (128, [1, 129]), (128, [5000, 0, 33]), (256, [600]), (256, [4100])])
def test_attention_wide_groups(kind, dtype, group, d, lens):
    """More query heads to a key-value head than a product has columns."""
    say("wide", kind, dtype, group, d, lens)
    s = Streams(lens, 2, d, 16, kind, dtype, seed=group)
    attend(s, randn(len(lens), 2 * group, d, seed=5, scale=1.5).to(dtype))


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("window", [1, 2, 16, 17, 100, 250, 5000])
def test_attention_window(kind, dtype, window):
    """Tokens before the window have no effect: their rows hold NaN, their pages are
    no longer the stream's."""
    say("window", kind, dtype, window)
    lens, page = [1, 5, 16, 40, 129, 300, 0, 777], 16
    s = Streams(lens, 2, 128, page, kind, dtype, seed=window)
    # rows before the window: NaN
    for i, n in enumerate(lens):
        first = max(0, n - window)
        for t in range(first):
            p, o = int(s.slots[i][t]) // page, int(s.slots[i][t]) % page
            for x in (s.cache.k, s.cache.v, s.cache.k_scales, s.cache.v_scales):
                if x is not None:
                    x.view(torch.uint8)[p, :, (o if x.dim() == 4 else slice(2 * o, 2 * o + 2))] = 255
        s.table[i, :first // page] = -1
    attend(s, randn(len(lens), 8, 128, seed=5).to(dtype), window=window)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d,lens", [(128, [40000]), (128, [9000, 1, 0, 3333]), (64, [20001, 7]), (256, [6007])])
def test_attention_long(kind, dtype, d, lens):
    """Ranges split over many work-groups and joined; keys far above the others late
    and early, so that the running maximum moves."""
    say("long", kind, dtype, d, lens)
    s = Streams(lens, 2, d, 64, kind, dtype, seed=3, hot=True)
    q = randn(len(lens), 4, d, seed=5).to(dtype)
    a = attend(s, q)
    b = attend(s, q)
    assert np.array_equal(a, b)


@gpu
@pytest.mark.parametrize("kind,dtype", [("f16", F16), ("4", F16)])
def test_attention_many_streams(kind, dtype):
    """More streams than lanes of a wavefront, most of them empty or short."""
    for batch in (63, 64, 65, 200, 513, 4097, 9000):
        say("streams", kind, batch)
        lens = [int(x) for x in np.random.default_rng(batch).choice([0, 0, 1, 3, 40, 150, 400], batch)]
        s = Streams(lens, 1, 64, 16, kind, dtype, seed=batch)
        attend(s, randn(batch, 2, 64, seed=5).to(dtype))
    for batch in (70, 5000):
        s = Streams([0] * batch, 2, 64, 16, kind, dtype)
        attend(s, randn(batch, 4, 64, seed=5).to(dtype))
    # a long stream behind many empty ones
    s = Streams([0] * 4500 + [3000] + [0] * 700, 2, 64, 16, kind, dtype)
    attend(s, randn(5201, 4, 64, seed=5).to(dtype))


@gpu
def test_attention_scores_in_extremes():
    """Scores far apart: one key takes all; a large scale; scores all far below zero."""
    for scale in (1e-6, 0.5, 30.0, -0.25):
        say("scale", scale)
        s = Streams([500, 33], 1, 128, 16, "f16", F16, seed=2)
        q = randn(2, 4, 128, seed=5).half()
        if scale == 0.5:
            q = -q.abs() * 20
        attend(s, q, scale=scale)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("lens", [[60000, 7], [900]])
def test_attention_small_weights(kind, dtype, lens):
    """A first token 17.5 e-folds above the rest: in all channels but one the result is
    that of the many small weights beside it."""
    say("small weights", kind, dtype, lens)
    s = Streams(lens, 2, 128, 16, kind, dtype, seed=7)
    total = sum(lens)
    k = 0.02 * randn(total, 2, 128, seed=8)
    v = 1.0 + 0.1 * randn(total, 2, 128, seed=9)
    at = 0
    for n in lens:
        k[at], v[at] = 0.0, 0.0
        k[at, :, 0], v[at, :, 0] = 14.0, 1.0
        at += n
    every = torch.cat(s.slots)
    tq.kv_append(s.cache, k.to(dtype).cuda(), v.to(dtype).cuda(), every.cuda())
    (kv, ks), (vv, vs) = stored(s.cache, every)
    s.k = kv if ks is None else kv * ks.astype(np.float64)[..., None]
    s.v = vv if vs is None else vv * vs.astype(np.float64)[..., None]
    q = randn(len(lens), 6, 128, seed=10)
    q[..., 0] = 20.0                         # 20 * 14 * 0.0625 = 17.5
    attend(s, q.to(dtype), scale=0.0625)


@gpu
@pytest.mark.parametrize("kind,dtype", KINDS[:2])
def test_attention_infinite_keys(kind, dtype):
    """A key whose score is -infinity has no weight: the result is that over the others,
    wherever they lie; with such keys alone it is no number, as 0 / 0."""
    lens, live = [200, 40, 6000, 20, 33], [range(160, 200), range(3, 40), [5, 5990], range(20), []]
    s = Streams(lens, 2, 128, 16, kind, dtype, seed=6)
    q = randn(5, 8, 128, seed=5)
    q[..., 0] = q[..., 0].abs() + 0.1
    q = q.to(dtype)
    at, keep = 0, []
    rows = s.cache.k.permute(0, 2, 1, 3).reshape(-1, 2, 128).clone()      # by slot
    for n, alive, slots in zip(lens, live, s.slots):
        dead = sorted(set(range(n)) - set(alive))
        rows[slots[dead].cuda(), :, 0] = -math.inf
        keep += [at + t for t in alive]
        at += n
    s.cache.k.copy_(rows.view(s.cache.k.shape[0], 16, 2, 128).permute(0, 2, 1, 3))
    got, lse = tq.paged_attention(s.cache, q.cuda(), *s.args(), return_lse=True)
    s.k, s.v, s.lens = s.k[keep], s.v[keep], [len(a) for a in live]
    ref, ref_lse, bound, lse_bound = s.plain(q, 128 ** -0.5, 0)
    got, lse = got.cpu().double().numpy(), lse.cpu().double().numpy()
    assert (np.abs(got - ref)[:4] <= bound[:4]).all() and np.isnan(got[4]).all()
    assert (np.abs(lse - ref_lse)[:4] <= lse_bound[:4]).all() and (lse[4] == -np.inf).all()


@gpu
def test_attention_strides_and_limits():
    """q as a view of a fused projection, page table rows apart, lengths past the
    table and negative ones, page numbers outside the cache past the length, none."""
    lens = [70, 33, 5]
    s = Streams(lens, 2, 128, 16, "f16", F16, seed=4)
    q = randn(3, 8, 128, seed=5).half()
    want = attend(s, q)
    wide = torch.full((3, 12, 128), float("nan"), dtype=F16, device="cuda")
    wide[:, 2:10] = q.cuda()
    table = torch.full((3, 9), 1 << 30, dtype=torch.int32, device="cuda")
    table[:, :s.table.shape[1]] = s.args()[0]
    got = tq.paged_attention(s.cache, wide[:, 2:10], table[:, :7], s.args()[1])
    assert np.array_equal(got.cpu().double().numpy(), want)
    # lengths are taken into the table: here 5 pages
    more = torch.tensor([10 ** 9, 33, -7], dtype=torch.int32, device="cuda")
    full = s.args()[0].clone()
    full[0] = full[0, 0]
    got, lse = tq.paged_attention(s.cache, q.cuda(), full, more, return_lse=True)
    assert np.array_equal(got[1].cpu().double().numpy(), want[1]) and torch.count_nonzero(got[2]) == 0
    assert torch.isinf(lse[2]).all() and torch.isfinite(got[0]).all()
    none = tq.paged_attention(s.cache, q[:0].cuda(), table[:0, :7], more[:0])
    assert none.shape == (0, 8, 128)


@gpu
def test_other_stream_and_graph():
    """The same bits on another stream, and from a captured graph replayed between
    other work."""
    lens = [3000, 17, 0, 450]
    s = Streams(lens, 2, 128, 16, "8", F16, seed=4)
    q, (table, ln) = randn(4, 8, 128, seed=5).half().cuda(), s.args()
    want = tq.paged_attention(s.cache, q, table, ln)
    k = randn(4, 2, 128, seed=6).half().cuda()
    slots = torch.tensor([int(s.slots[0][5]), int(s.slots[1][3]), -1, int(s.slots[3][449])], device="cuda")
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = tq.paged_attention(s.cache, q, table, ln, stream=other)
    back = tq.kv_read(s.cache, slots, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(got, want)
    assert all(torch.equal(a, b) for a, b in zip(back, tq.kv_read(s.cache, slots)))
    torch.cuda.synchronize()
    q_in, ln_in = q.clone(), ln.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tq.kv_append(s.cache, k, k, slots)
        out = tq.paged_attention(s.cache, q_in, table, ln_in)
    for i in range(4):
        q_in.copy_(q * (1 + i))
        ln_in.copy_(torch.clamp(ln - i, min=0))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, tq.paged_attention(s.cache, q_in, table, ln_in)), i
        torch.ones(1 << 20, device="cuda").sum().item()


@gpu
@pytest.mark.parametrize("kind", ["f16", "4"])
def test_offsets_past_32_bits(kind):
    """Slots whose rows start beyond 2^32 bytes (fp16: beyond 2^32 values)."""
    page, heads, d = 16, 8, 128
    row = {"f16": 256, "4": 64}[kind]
    pages = (9 << 30 if kind == "f16" else 5 << 30) // (page * heads * row)
    c = tq.empty_kv_cache(pages, page, heads, d, 16 if kind == "f16" else 4)
    say("far", kind, pages, c.k.numel())
    s = Streams([40, 200], heads, d, page, kind, F16, seed=8, extra=0)
    q = randn(2, 16, d, seed=5).half().cuda()
    table, ln = s.args()
    want = tq.paged_attention(s.cache, q, table, ln)
    n = s.cache.pages
    far = pages - n
    every = torch.cat(s.slots).cuda()
    k, v = tq.kv_read(s.cache, every)
    if kind == "f16":
        tq.kv_append(c, k, v, every + far * page)
    else:
        for dst, src in zip(c._t, s.cache._t):
            dst[far:] = src
    assert torch.equal(tq.paged_attention(c, q, torch.where(table >= 0, table + far, -1), ln), want)
    back = tq.kv_read(c, every + far * page)
    assert torch.equal(back[0], k) and torch.equal(back[1], v)
