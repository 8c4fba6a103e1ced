"""Performance cases of the operators between the linear layers of a decoder
block: the norm and position rotation of queries and keys, the paged key-value
cache in 16, 8 and 4 bits, and the attention of one new token over it.

Operators (the ``op`` of a case):
  rope    ``qk_norm_rope``: per-head RMS norm (or none) and rotation of q and k,
          which are views of one fused projection's output
  cache   ``kv_append`` of k and v, then ``kv_read`` of the same slots
  write   ``qk_norm_rope_append``: norm, rotation and the cache write in one
          pass, then ``kv_read`` of the slots it wrote
  attend  ``paged_attention``: one new token of every stream over its pages

A cache is a pair of tensors [pages, kv_heads, page_size, row]: the values
themselves (16 bits), float8_e4m3fn codes (8 bits) or int32 TQ4 words of eight
codes (4 bits); the last two with one fp16 scale per slot and head.

The head layouts are those of the LLaMA3-8B, LLaMA3-70B and Qwen3-8B
configurations (32 or 64 query heads, 8 key-value heads of 128), and generic
ones of 64 and 256.
"""
from __future__ import annotations

import math

import torch

own = False

ROPE_BASE = 500000.0
EPS = 1e-6


# ------------------------------------------------------------------ cases
def _rope(name, tokens, hq, hkv, d=128, rot=128, norm=False, interleaved=False, bf16=False):
    return {"name": name, "op": "rope", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rot": rot,
            "norm": norm, "interleaved": interleaved, "bf16": bf16}


def _cache(name, tokens, hkv, bits, d=128, page=16, streams=1, bf16=False):
    return {"name": name, "op": "cache", "tokens": tokens, "hkv": hkv, "bits": bits, "d": d,
            "page": page, "streams": streams, "bf16": bf16}


def _write(name, tokens, hq, hkv, bits, d=128, rot=128, norm=False, interleaved=False, page=16,
           streams=1, bf16=False):
    return {"name": name, "op": "write", "tokens": tokens, "hq": hq, "hkv": hkv, "bits": bits, "d": d,
            "rot": rot, "norm": norm, "interleaved": interleaved, "page": page, "streams": streams,
            "bf16": bf16}


def _attend(name, batch, length, hq, hkv, bits, d=128, page=16, window=0, empty=False, bf16=False):
    return {"name": name, "op": "attend", "batch": batch, "length": length, "hq": hq, "hkv": hkv,
            "bits": bits, "d": d, "page": page, "window": window, "empty": empty, "bf16": bf16}


def listed():
    return [
        # one token of one stream through Qwen3-8B's head norms: a launch and its host work
        _rope("qwen_rope_t1", 1, 32, 8, norm=True, bf16=True),
        # a long prompt of LLaMA3-70B
        _rope("70b_rope_t8192", 8192, 64, 8),
        # an odd prompt into a 4-bit cache
        _cache("70b_cache_t777_4bit", 777, 8, 4),
        # a long prompt into an 8-bit cache with large pages
        _cache("8b_cache_t8192_8bit", 8192, 8, 8, page=64, bf16=True),
        # a decode step of 32 streams: each token goes to its own stream's page
        _write("qwen_write_32_streams_8bit", 32, 32, 8, 8, norm=True, streams=32),
        # a prompt into a 16-bit cache
        _write("8b_write_t2048_16bit", 2048, 32, 8, 16, bf16=True),
        # one stream, shortly after its prompt: the smallest attention
        _attend("8b_attend_1x300_16bit", 1, 300, 32, 8, 16),
        # one stream with a long document
        _attend("70b_attend_1x131072_16bit", 1, 131072, 64, 8, 16),
        # a decode batch of ragged streams
        _attend("qwen_attend_32x8192_16bit", 32, 8192, 32, 8, 16, bf16=True),
        # a large decode batch over an 8-bit cache
        _attend("8b_attend_64x8192_8bit", 64, 8192, 32, 8, 8, page=64),
        # a large decode batch over a 4-bit cache
        _attend("70b_attend_48x16384_4bit", 48, 16384, 64, 8, 4),
        # odd batch, small heads, a sliding window, and a stream that holds nothing yet
        _attend("odd_attend_13x5001_window", 13, 5001, 15, 3, 8, d=64, page=32, window=1000, empty=True,
                bf16=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """The same four operators over head layouts, lengths, page sizes and types."""
    largest = 48 * 16384 * 8 * 128
    while True:
        op = rng.choice(("rope", "cache", "write", "attend", "attend", "attend"))
        d = rng.choice((64, 128, 128, 128, 256))
        hkv = rng.choice((1, 2, 3, 4, 8, 8, 8, 16))
        hq = hkv * rng.choice((1, 2, 4, 4, 5, 7, 8, 8, 16, 20))
        if hq > 96:
            continue
        bf16 = rng.random() < 0.4
        page = rng.choice((16, 16, 32, 64, 128, 256))
        rot = rng.choice((d, d, d, d // 2, 16 * rng.randint(1, d // 16)))
        norm, interleaved = rng.random() < 0.5, rng.random() < 0.3
        if op == "attend":
            batch, length = _log_int(rng, 1, 128), _log_int(rng, 1, 131072)
            if batch * length * hkv * d > largest // 2:
                continue
            window = rng.choice((0, 0, 0, _log_int(rng, 1, 4096)))
            case = _attend("", batch, length, hq, hkv, rng.choice((16, 8, 4)), d, page, window,
                           batch > 1 and rng.random() < 0.3, bf16)
        else:
            tokens = _log_int(rng, 1, 8192)
            if tokens * (hq + hkv) * d > 8192 * 72 * 128:
                continue
            streams = rng.choice((1, tokens)) if tokens <= 256 else rng.randint(1, 8)
            if op == "rope":
                case = _rope("", tokens, hq, hkv, d, rot, norm, interleaved, bf16)
            elif op == "cache":
                case = _cache("", tokens, hkv, rng.choice((16, 8, 4)), d, page, streams, bf16)
            else:
                # (a fused 4-bit write differs from any other order of its sums by a
                # whole code here and there; the operator's own test takes that up)
                case = _write("", tokens, hq, hkv, rng.choice((16, 8)), d, rot, norm, interleaved, page,
                              streams, bf16)
        del case["name"]
        return case


# ------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.bfloat16 if case["bf16"] else torch.float16


def _generator(seed, stream):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + stream)


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _keys(shape, gen):
    """Keys as projections give them: a few channels of every head are far larger
    than the others, in all tokens."""
    heads, d = shape[1], shape[-1]
    big = torch.rand((heads, 1, d), generator=gen, device="cuda") < 0.03
    if len(shape) == 3:
        big = big[:, 0]
    return torch.where(big, 6.0, 0.7) * _normal(shape, gen)


def _token_inputs(case, seed):
    """The fused projection's output, cut into its three views, and the positions,
    the slots, the rotation's table and the norms' weights."""
    t, hkv, d, dtype = case["tokens"], case["hkv"], case["d"], _dtype(case)
    hq = case.get("hq", 0)
    gen = _generator(seed, 0)
    qkv = torch.cat((_normal((t, hq, d), gen), _keys((t, hkv, d), gen), _normal((t, hkv, d), gen)), 1).to(dtype)
    s = {"q": qkv[:, :hq], "k": qkv[:, hq:hq + hkv], "v": qkv[:, hq + hkv:]}
    streams, page = case.get("streams", 1), case.get("page", 16)
    # a stream's new tokens continue it from somewhere; t tokens over the streams
    counts = [t // streams + (i < t % streams) for i in range(streams)]
    host = torch.Generator().manual_seed(seed * 7919 + 1)
    starts = torch.randint(0, 4096, (streams,), generator=host).tolist()
    pos = torch.cat([torch.arange(a, a + n) for a, n in zip(starts, counts)])
    stream = torch.repeat_interleave(torch.arange(streams), torch.tensor(counts))
    pages_each = max((a % page + n + page - 1) // page for a, n in zip(starts, counts))
    pages = streams * pages_each + 3
    order = torch.randperm(pages, generator=host)[:streams * pages_each].view(streams, pages_each)
    first = torch.tensor(starts) // page
    slots = order[stream, pos // page - first[stream]] * page + pos % page
    s["positions"], s["slots"] = pos.to(torch.int32).cuda(), slots.cuda()
    if "rot" in case:
        rot = case["rot"]
        freq = ROPE_BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        angle = torch.arange(int(pos.max()) + 1, dtype=torch.float64)[:, None] * freq[None]
        s["table"] = torch.cat((angle.cos(), angle.sin()), 1).float().cuda()
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"] = (1.0 + 0.2 * _normal((d,), gen)).to(dtype)
            s["k_weight"] = (1.0 + 0.2 * _normal((d,), gen)).to(dtype)
    if "bits" in case:
        bits = case["bits"]
        shape = (pages, hkv, page, d // 8 if bits == 4 else d)
        kind = {16: dtype, 8: torch.float8_e4m3fn, 4: torch.int32}[bits]
        s["cache"] = [torch.zeros(shape, dtype=kind, device="cuda") for _ in range(2)]
        s["cache"] += [None if bits == 16 else torch.zeros(shape[:3], dtype=torch.float16, device="cuda")
                       for _ in range(2)]
    return s


def _lengths(case):
    """Ragged lengths of a batch up to the case's, spread evenly; the last is 0
    where one stream is to hold nothing."""
    n, top = case["batch"], case["length"]
    out = [top] + [max(1, int(top * (0.05 + 0.95 * (i * 0.6180339887 % 1.0)))) for i in range(1, n)]
    if case["empty"]:
        out[-1] = 0
    return out


def _attend_inputs(case, seed):
    b, d, hkv, page, bits = (case[x] for x in ("batch", "d", "hkv", "page", "bits"))
    dtype = _dtype(case)
    gen = _generator(seed, 1)
    host = torch.Generator().manual_seed(seed * 7919 + 2)
    lens = torch.tensor(_lengths(case))[torch.randperm(b, generator=host)]
    need = (lens + page - 1) // page
    pages = int(need.sum()) + 5
    order = torch.randperm(pages, generator=host)
    table = torch.zeros((b, max(int(need.max()), 1)), dtype=torch.int32)
    valid = torch.arange(table.shape[1])[None] < need[:, None]
    table[valid] = order[:int(need.sum())].to(torch.int32)
    shape = (pages, hkv, page, d)
    cache, scales = [], []
    for x in (_keys(shape, gen), _normal(shape, gen)):
        codes, scale = _quantize(x.to(dtype), bits)
        cache.append(codes)
        scales.append(scale)
        del x
    # queries that look for some of what is there: scores spread over several e-folds
    q = (1.3 * _normal((b, case["hq"], d), gen)).to(dtype)
    return {"q": q, "cache": cache + scales, "page_table": table.cuda(),
            "lengths": lens.to(torch.int32).cuda(), "window": case["window"]}


def prepare(case, seed):
    state = _attend_inputs(case, seed) if case["op"] == "attend" else _token_inputs(case, seed)
    state.update(op=case["op"], bf16=case["bf16"], bits=case.get("bits", 16),
                 interleaved=case.get("interleaved", False))
    return state


# ------------------------------------------------------------------ plain forms
def _quantize(x, bits):
    """(codes, scales) of 16-bit x [..., d], one scale for the last axis."""
    if bits == 16:
        return x, None
    top = 448.0 if bits == 8 else 7.0
    f = x.float()
    scale = (f.abs().amax(-1) / top).half()
    s = scale.float()[..., None]
    t = torch.where(s > 0, f / torch.where(s > 0, s, 1.0), 0.0)
    if bits == 8:
        return t.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn), scale
    c = t.round_().clamp_(-7.0, 7.0).to(torch.int32).unflatten(-1, (-1, 8))
    mag, neg = c.abs(), (c < 0).to(torch.int32)
    at = torch.arange(4, device=x.device, dtype=torch.int32)
    low = (mag[..., :4] << (8 * at)) | (neg[..., :4] << (8 * at + 7))
    high = (mag[..., 4:] << (8 * at + 4)) | (neg[..., 4:] << (8 * ((at + 1) % 4) + 3))
    return (low | high).sum(-1, dtype=torch.int32), scale   # (disjoint bits: the sum is their union)


def _values(codes, scales, bits):
    """fp32 values of codes [..., row] with scales [...]."""
    if bits == 16:
        return codes.float()
    if bits == 8:
        return codes.float() * scales.float()[..., None]
    at = torch.arange(4, device=codes.device, dtype=torch.int32)
    w = codes[..., None]
    low = ((w >> (8 * at)) & 7) * (1 - 2 * ((w >> (8 * at + 7)) & 1))
    high = ((w >> (8 * at + 4)) & 7) * (1 - 2 * ((w >> (8 * ((at + 1) % 4) + 3)) & 1))
    return torch.cat((low, high), -1).flatten(-2).float() * scales.float()[..., None]


def _bytes(x):
    """A view whose rows can be indexed whatever the type."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _plain_rotated(x, weight, state):
    """Norm and rotation of x [t, heads, d], rounded to x's type."""
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    row = state["table"][state["positions"].long()][:, None]
    rot = row.shape[-1]
    c, s = row[..., :rot // 2], row[..., rot // 2:]
    if state["interleaved"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)


def _plain_stored(k, v, state):
    """k and v into the slots and back."""
    kc, vc, ks, vs = state["cache"]
    bits, slots, page = state["bits"], state["slots"], state["cache"][0].shape[2]
    at, off = slots // page, slots % page
    out = []
    for x, codes, scales in ((k, kc, ks), (v, vc, vs)):
        c, s = _quantize(x, bits)
        _bytes(codes)[at, :, off] = _bytes(c)
        if s is not None:
            scales[at, :, off] = s
        back = _bytes(codes)[at, :, off].view(codes.dtype)
        out.append(_values(back, None if s is None else scales[at, :, off], bits).to(x.dtype))
    return tuple(out)


def _plain_attend(state):
    q, (kc, vc, ks, vs), table, bits = state["q"], state["cache"], state["page_table"].long(), state["bits"]
    b, hq, d = q.shape
    _, hkv, page, _ = kc.shape

    def rows(codes, scales):
        c = _bytes(codes)[table].view(codes.dtype)
        x = _values(c, None if scales is None else scales[table], bits)
        return x.permute(0, 2, 1, 3, 4).reshape(b, hkv, -1, d)      # [b, hkv, positions, d]

    at = torch.arange(table.shape[1] * page, device=q.device)[None]
    end = state["lengths"].long()[:, None]
    seen = at < end
    if state["window"]:
        seen = seen & (at >= end - state["window"])
    seen = seen[:, None, None]
    k = rows(kc, ks)
    score = (q.float().view(b, hkv, hq // hkv, d) / math.sqrt(d)) @ k.transpose(-1, -2).contiguous()
    del k
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / torch.where(total > 0, total, 1.0), 0.0)
    v = torch.where(seen.transpose(-1, -2), rows(vc, vs), 0.0)
    return (p @ v).reshape(b, hq, d).to(q.dtype)


def run(state):
    op = state["op"]
    if not own:
        if op == "attend":
            return _plain_attend(state)
        if op == "cache":
            return _plain_stored(state["k"], state["v"], state)
        q, k = (_plain_rotated(state[x], state[x + "_weight"], state) for x in "qk")
        return (q, k) if op == "rope" else (q, *_plain_stored(k, state["v"], state))
    import paper_2606_01556_amd as tq
    if op == "rope":
        return tq.qk_norm_rope(state["q"], state["k"], state["positions"], state["table"],
                               state["q_weight"], state["k_weight"], eps=EPS,
                               interleaved=state["interleaved"])
    cache = tq.KVCache(*state["cache"])
    if op == "attend":
        return tq.paged_attention(cache, state["q"], state["page_table"], state["lengths"],
                                  window=state["window"])
    if op == "cache":
        tq.kv_append(cache, state["k"], state["v"], state["slots"])
        return tq.kv_read(cache, state["slots"], bf16=state["bf16"])
    q = tq.qk_norm_rope_append(cache, state["q"], state["k"], state["v"], state["positions"],
                               state["table"], state["slots"], state["q_weight"], state["k_weight"],
                               eps=EPS, interleaved=state["interleaved"])
    return (q, *tq.kv_read(cache, state["slots"], bf16=state["bf16"]))


# ------------------------------------------------------------------ accounting
def _row_bytes(case):
    """Bytes of one slot of one head: a row and its scale."""
    return case["d"] * case["bits"] // 8 + (2 if case["bits"] < 16 else 0)


def _seen(case):
    return sum(min(n, case["window"]) if case["window"] else n for n in _lengths(case))


def work(case):
    """rope: q and k in and out, a table row per token.  cache: k and v in and out,
    their rows written and read.  write: both.  attend: the rows that the streams
    see, the page numbers, q in and the result out."""
    d, hkv, hq = case["d"], case["hkv"], case.get("hq", 0)
    if case["op"] == "attend":
        seen = _seen(case)
        return {"bytes": seen * hkv * 2 * _row_bytes(case) + 4 * (seen // case["page"])
                + 4 * case["batch"] * hq * d, "flops": 4 * seen * hq * d}
    t = case["tokens"]
    nbytes = flops = 0
    if case["op"] in ("rope", "write"):
        nbytes += t * (4 * hq * d + 4 + 4 * case["rot"]) + (4 * d if case["norm"] else 0)
        flops += t * (hq + hkv) * (3 * case["rot"] + (4 * d if case["norm"] else 0))
    if case["op"] == "rope":
        return {"bytes": nbytes + t * 4 * hkv * d, "flops": flops}
    nbytes += t * (2 * hkv * (4 * d + 2 * _row_bytes(case)) + 8)
    return {"bytes": nbytes, "flops": flops + t * 2 * hkv * d * (0 if case["bits"] == 16 else 4)}


# ------------------------------------------------------------------ the definition in 64 bits
def _e4m3_table():
    """The 256 values of e4m3: sign, four exponent bits of bias 7, three of mantissa."""
    out = []
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = math.nan if e == 15 and m == 7 else (m / 8.0 * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7))
        out.append(-v if b >> 7 else v)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _exact_values(codes, scales, bits):
    if bits == 16:
        return codes.double()
    if bits == 8:
        return _e4m3_table()[codes.view(torch.uint8).long()] * scales.double()[..., None]
    out = torch.empty((*codes.shape, 8), dtype=torch.float64, device=codes.device)
    for i in range(8):
        first, sign = (8 * i, 8 * i + 7) if i < 4 else (8 * (i - 4) + 4, (8 * (i - 4) + 11) % 32)
        out[..., i] = ((codes >> first).bitwise_and(7)).double()
        out[..., i] *= torch.where((codes >> sign).bitwise_and(1) == 1, -1.0, 1.0)
    return out.flatten(-2) * scales.double()[..., None]


def _exact_rotated(x, weight, case, s):
    y = x.double()
    if weight is not None:
        y = y / (y.pow(2).sum(-1, keepdim=True) / case["d"] + EPS).sqrt() * weight.double()
    rot = case["rot"]
    half = rot // 2
    row = s["table"].double().index_select(0, s["positions"].long())
    out = y.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
        c, sn = row[:, i, None], row[:, half + i, None]
        out[..., a] = y[..., a] * c - y[..., b] * sn
        out[..., b] = y[..., b] * c + y[..., a] * sn
    return out


def _exact_stored(x, bits):
    """What the cache stands for after x [t, heads, d] was written."""
    if bits == 16:
        return x
    top = 448.0 if bits == 8 else 7.0
    s = (x.abs().amax(-1, keepdim=True) / top).float().half().double()
    t = torch.where(s > 0, x / s.clamp_min(1e-30), 0.0)
    if bits == 4:
        return t.round().clamp(-7, 7) * s
    t = t.clamp(-448, 448)
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp_min(2.0 ** -6))) - 3)
    return (t / step).round() * step * s


def exact(case, seed):
    bits = case.get("bits", 16)
    if case["op"] == "attend":
        s = _attend_inputs(case, seed)
        kc, vc, ks, vs = s["cache"]
        hkv, d, page = case["hkv"], case["d"], case["page"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for i, n in enumerate(s["lengths"].tolist()):
            a = max(0, n - case["window"]) if case["window"] else 0
            if a == n:
                continue
            t = torch.arange(a, n, device="cuda")
            at, off = s["page_table"][i].long()[t // page], t % page
            k, v = (_exact_values(c.view(torch.uint8)[at, :, off].view(c.dtype) if bits == 8 else c[at, :, off],
                                  None if w is None else w[at, :, off], bits).transpose(0, 1).contiguous()
                    for c, w in ((kc, ks), (vc, vs)))                   # [hkv, n, d]
            q = s["q"][i].double().view(hkv, -1, d)
            logit = torch.matmul(k, q.transpose(1, 2).contiguous()) * d ** -0.5    # [hkv, n, g]
            w = torch.exp(logit - logit.amax(1, keepdim=True))
            w = (w / w.sum(1, keepdim=True)).transpose(1, 2).contiguous()
            out[i] = torch.matmul(w, v).reshape(-1, d)
        return out
    s = _token_inputs(case, seed)
    if case["op"] == "cache":
        return tuple(_exact_stored(s[x].double(), bits) for x in "kv")
    q, k = (_exact_rotated(s[x], s[x + "_weight"], case, s) for x in "qk")
    if case["op"] == "rope":
        return q, k
    # the cache takes k in the model's type
    k = k.to(_dtype(case)).double()
    return q, _exact_stored(k, bits), _exact_stored(s["v"].double(), bits)
