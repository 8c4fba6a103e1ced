"""Performance cases of what a decoder block with quantized layers needs beside the norm,
rotation, cache and attention of one token: the attention of many new tokens over the
paged cache with its masks, caps and biases, the attention of a batch that shares a
prefix, and the norms at a block's ends with its residual sum.

Operators (the ``op`` of a case):
  prompt  ``prompt_attention``: the new tokens of every stream (a prompt, a chunk of one, a
          few tokens to verify) over the stream's pages, causal, with a window, a prefix
          that all tokens see, documents that do not see each other, scores capped by a
          tanh, a bias by distance
  token   ``paged_attention`` of one new token with capped or biased scores
  prefix  ``shared_prefix_attention``: one new token of every stream over a prefix that a
          group of streams shares and the stream's own pages
  norm    ``add_rms_norm``: the norm after a block, its gate, the residual sum and the norm
          before the next block

A cache is a pair of tensors [pages, kv_heads, page_size, row]: the values themselves (16
bits), float8_e4m3fn codes (8 bits) or int32 TQ4 words of eight codes (4 bits); the last
two with one fp16 scale per slot and head.

The head layouts and hidden sizes are those of the LLaMA3-8B, LLaMA3-70B and Qwen3-8B
configurations (32 or 64 query heads, 8 key-value heads of 128; 4096 or 8192), and generic
ones.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
LOW = -math.inf


# ------------------------------------------------------------------ cases
def _prompt(name, streams, new, before, hq, hkv, bits, d=128, page=16, window=0, prefix=False, documents=0, cap=0.0,
            slopes=False, pad=0, lse=False, bf16=False):
    return {"name": name, "op": "prompt", "streams": streams, "new": new, "before": before, "hq": hq, "hkv": hkv,
            "bits": bits, "d": d, "page": page, "window": window, "prefix": prefix, "documents": documents, "cap": cap,
            "slopes": slopes, "pad": pad, "lse": lse, "bf16": bf16}


def _token(name, streams, length, hq, hkv, bits, d=128, page=16, window=0, cap=0.0, slopes=False, empty=False, bf16=False):
    return {"name": name, "op": "token", "streams": streams, "length": length, "hq": hq, "hkv": hkv, "bits": bits,
            "d": d, "page": page, "window": window, "cap": cap, "slopes": slopes, "empty": empty, "bf16": bf16}


def _prefix(name, groups, streams, shared, length, hq, hkv, bits, d=128, page=16, cap=0.0, slopes=False, empty=False,
            bf16=False):
    return {"name": name, "op": "prefix", "groups": groups, "streams": streams, "shared": shared, "length": length,
            "hq": hq, "hkv": hkv, "bits": bits, "d": d, "page": page, "cap": cap, "slopes": slopes, "empty": empty,
            "bf16": bf16}


def _norm(name, tokens, n, after=False, gate="", scale=1.0, before=True, bf16=False):
    return {"name": name, "op": "norm", "tokens": tokens, "n": n, "after": after, "gate": gate, "scale": scale,
            "before": before, "bf16": bf16}


def listed():
    return [
        # a long prompt of LLaMA3-8B
        _prompt("8b_prompt_1x8192", 1, 8192, 0, 32, 8, 16),
        # a batch of ragged prompts
        _prompt("qwen_prompts_32x700", 32, 700, 0, 32, 8, 16, bf16=True),
        # a chunk of a long document behind what the 8-bit cache holds of it
        _prompt("70b_chunk_2048_behind_30720_8bit", 1, 2048, 30720, 64, 8, 8, page=64, bf16=True),
        # large heads with capped scores and a sliding window
        _prompt("capped_window_2x4096_d256", 2, 4096, 0, 16, 8, 16, d=256, page=32, window=1024, cap=50.0, bf16=True),
        # packed documents with a bias by distance, small heads, odd sizes, a 4-bit cache
        _prompt("documents_3x1777_4bit", 3, 1777, 0, 15, 3, 4, d=64, documents=5, slopes=True, pad=5),
        # a few proposed tokens of every stream to verify
        _prompt("qwen_verify_16x5_behind_8192", 16, 5, 8192, 32, 8, 16, lse=True, bf16=True),
        # one stream shortly after its prompt, with a bias by distance: the smallest attention
        _token("8b_token_1x300_slopes", 1, 300, 32, 8, 16, slopes=True),
        # a decode batch of ragged streams with capped scores
        _token("capped_token_32x8192_8bit", 32, 8192, 32, 8, 8, page=64, cap=30.0, bf16=True),
        # a decode batch behind one long instruction
        _prefix("8b_prefix_64x16384", 1, 64, 16384, 1024, 32, 8, 16),
        # three odd groups, short tails, one stream with nothing of its own, a 4-bit cache
        _prefix("70b_prefix_3_groups_21x2500_4bit", 3, 21, 2500, 131, 64, 8, 4, empty=True, bf16=True),
        # one token between two blocks: a launch and its host work
        _norm("8b_norm_t1", 1, 4096),
        # a long prompt between two blocks, norms on both sides, a gate and a residual scale
        _norm("70b_norm_t8192_both", 8192, 8192, after=True, gate="token", scale=0.5, bf16=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """The same operators over head layouts, lengths, page sizes, masks and types."""
    largest = 4 * 64 * 128 * 2048 * 31744
    while True:
        op = rng.choice(("prompt", "prompt", "prompt", "token", "prefix", "norm"))
        bf16 = rng.random() < 0.5
        if op == "norm":
            n, tokens = 8 * _log_int(rng, 8, 2048), _log_int(rng, 1, 8192)
            if n * tokens > 8192 * 8192:
                continue
            case = _norm("", tokens, n, rng.random() < 0.5, rng.choice(("", "channel", "token")),
                         rng.choice((1.0, 1.0, 0.22, -0.5)), rng.random() < 0.8, bf16)
            del case["name"]
            return case
        d = rng.choice((64, 128, 128, 128, 256))
        hkv = rng.choice((1, 2, 3, 4, 8, 8, 8, 16))
        hq = hkv * rng.choice((1, 2, 4, 4, 5, 7, 8, 8, 16))
        if hq > 96:
            continue
        bits, page = rng.choice((16, 16, 8, 4)), rng.choice((16, 16, 32, 64, 256))
        cap, slopes = rng.choice((0.0, 0.0, 20.0, 50.0)), rng.random() < 0.25
        window = rng.choice((0, 0, 0, _log_int(rng, 1, 4096)))
        if op == "prompt":
            streams, new = _log_int(rng, 1, 32), _log_int(rng, 1, 8192)
            before = rng.choice((0, 0, _log_int(rng, 1, 32768)))
            documents = rng.randint(2, 9) if before == 0 and rng.random() < 0.25 else 0
            case = _prompt("", streams, new, before, hq, hkv, bits, d, page, window, rng.random() < 0.25, documents, cap,
                           slopes, rng.choice((0, 0, rng.randint(1, 40))), bf16=bf16)
            held = streams * (new + before) * hkv * d
            cost = 4 * streams * new * (before + new) * hq * d
        elif op == "token":
            streams, length = _log_int(rng, 1, 128), _log_int(rng, 1, 65536)
            if cap == 0.0:
                slopes = True
            case = _token("", streams, length, hq, hkv, bits, d, page, window, cap, slopes, streams > 1 and rng.random() < 0.3,
                          bf16)
            held, cost = streams * length * hkv * d, 0
        else:
            groups, shared, length = rng.randint(1, 4), _log_int(rng, 1, 32768), _log_int(rng, 1, 2048)
            streams = groups * _log_int(rng, 1, 40) + rng.randint(0, 2)
            case = _prefix("", groups, streams, shared, length, hq, hkv, bits, d, page, cap, slopes, rng.random() < 0.3, bf16)
            held, cost = (groups * shared + streams * length) * hkv * d, 4 * streams * (shared + length) * hq * d
        if held > 32 * 8192 * 8 * 128 or cost > largest // 2:
            continue
        del case["name"]
        return case


# ------------------------------------------------------------------ sizes
def _spread(top, count, share):
    """`count` sizes up to `top`, spread evenly from `share` of it on; the first is `top`."""
    return [top] + [max(1, int(top * (share + (1 - share) * (i * 0.6180339887 % 1.0)))) for i in range(1, count)]


def _sizes(case):
    """Of every stream the new tokens and the tokens in the cache (for ``prefix``: its own)."""
    s = case["streams"]
    if case["op"] == "prompt":
        new = _spread(case["new"], s, 0.2)
        before = [0] * s if case["before"] == 0 else _spread(case["before"], s, 0.05)
        return new, [a + b for a, b in zip(new, before)]
    held = _spread(case["length"], s, 0.05)
    if case["empty"] and s > 1:
        held[-1] = 0
    return [1] * s, held


def _members(case):
    """Bounds of the groups' streams: as even as they go."""
    g, s = case["groups"], case["streams"]
    return [s * i // g for i in range(g + 1)]


def _shared(case):
    return _spread(case["shared"], case["groups"], 0.3)


# ------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.bfloat16 if case["bf16"] else torch.float16


def _generator(seed, stream):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + stream)


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _pages(lengths, page, host, order):
    """A page table of streams of these lengths, from the front of `order`; what is left of it."""
    need = [-(-n // page) for n in lengths]
    table = torch.zeros((len(lengths), max(max(need), 1)), dtype=torch.int32)
    for i, n in enumerate(need):
        table[i, :n] = order[:n].to(torch.int32)
        order = order[n:]
    return table.cuda(), order


def _attention_inputs(case, seed):
    hq, hkv, d, page, bits = (case[x] for x in ("hq", "hkv", "d", "page", "bits"))
    dtype, gen = _dtype(case), _generator(seed, 1)
    host = torch.Generator().manual_seed(seed * 7919 + 2)
    new, held = _sizes(case)
    shared = _shared(case) if case["op"] == "prefix" else []
    pages = sum(-(-n // page) for n in held + shared) + 5
    order = torch.randperm(pages, generator=host)
    table, order = _pages(held, page, host, order)
    s = {"op": case["op"], "bits": bits, "page_table": table, "held": held, "new": new,
         "lengths": torch.tensor(held, dtype=torch.int32).cuda(), "window": case.get("window", 0), "cap": case["cap"],
         "lse": case.get("lse", False)}
    if shared:
        s["prefix_table"], order = _pages(shared, page, host, order)
        s["shared"], s["members_list"] = shared, _members(case)
        s["prefix_lengths"] = torch.tensor(shared, dtype=torch.int32).cuda()
        s["members"] = torch.tensor(s["members_list"], dtype=torch.int32).cuda()
    # keys as projections give them: a few channels of every head far larger than the others
    shape = (pages, hkv, page, d)
    big = torch.rand((hkv, 1, d), generator=gen, device="cuda") < 0.03
    s["cache"] = [None] * 4
    for i, spread in enumerate((torch.where(big, 6.0, 0.7), 1.0)):
        s["cache"][i], s["cache"][2 + i] = _quantize((spread * _normal(shape, gen)).to(dtype), bits)
    rows = sum(new) + case.get("pad", 0)
    # scores spread over several e-folds, and past the cap where there is one
    s["q"] = ((8.0 if case["cap"] else 1.3) * _normal((rows, hq, d), gen)).to(dtype)
    s["slopes"] = s["prefix"] = s["first"] = None
    if case["slopes"]:
        s["slopes"] = torch.exp2(-8.0 * (torch.arange(hq, dtype=torch.float32) + 1) / hq).cuda()
    if case["op"] != "prompt":
        return s
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["starts"], s["starts_list"] = torch.tensor(starts, dtype=torch.int32).cuda(), starts
    if case["prefix"]:
        s["prefix_list"] = [int(n * x) for n, x in zip(held, torch.rand(len(held), generator=host).tolist())]
        s["prefix"] = torch.tensor(s["prefix_list"], dtype=torch.int32).cuda()
    if case["documents"]:
        # (a token sees its own document; a few see nothing at all)
        first = torch.zeros(rows, dtype=torch.int32)
        for a, n in zip(starts, new):
            cuts = torch.sort(torch.randint(0, n, (case["documents"] - 1,), generator=host)).values
            at = torch.arange(n)
            first[a:a + n] = torch.cat((torch.zeros(1, dtype=cuts.dtype), cuts))[torch.searchsorted(cuts, at, right=True)].to(torch.int32)
            nothing = torch.rand(n, generator=host) < 0.01
            first[a:a + n] = torch.where(nothing, n, first[a:a + n])
        s["first"] = first.cuda()
    return s


def _norm_inputs(case, seed):
    t, n, dtype, gen = case["tokens"], case["n"], _dtype(case), _generator(seed, 0)
    # the residual stream has a few channels far above the others
    loud = torch.where(torch.rand((n,), generator=gen, device="cuda") < 0.01, 30.0, 2.0)
    s = {"op": "norm", "x": _normal((t, n), gen).to(dtype), "residual": (loud * _normal((t, n), gen)).to(dtype),
         "scale": case["scale"], "weight": None, "post_weight": None, "gate": None}
    if case["before"]:
        s["weight"] = (1.0 + 0.2 * _normal((n,), gen)).to(dtype)
    if case["after"]:
        s["post_weight"] = (1.0 + 0.2 * _normal((n,), gen)).to(dtype)
    if case["gate"]:
        s["gate"] = _normal((t, n) if case["gate"] == "token" else (n,), gen).to(dtype)
    return s


def prepare(case, seed):
    return _norm_inputs(case, seed) if case["op"] == "norm" else _attention_inputs(case, seed)


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


def _plain_rows(state, table, i, length):
    """k and v of a stream's `length` tokens: fp32 [hkv, length, d]."""
    kc, vc, ks, vs = state["cache"]
    page = kc.shape[2]
    at = table[i, :-(-length // page)].long()
    out = []
    for codes, scales in ((kc, ks), (vc, vs)):
        c = (codes.view(torch.uint8) if state["bits"] == 8 else codes)[at].view(codes.dtype)
        x = _values(c, None if scales is None else scales[at], state["bits"])
        out.append(x.transpose(0, 1).flatten(1, 2)[:, :length].contiguous())
    return out


def _plain_scores(state, q, k, seen, distance):
    """Base-e scores [hkv, tokens, group, keys] of q [tokens, hq, d]; seen and distance [tokens, keys]."""
    (t, hq, d), hkv = q.shape, k.shape[0]
    x = (q.float() / math.sqrt(d)).view(t, hkv, hq // hkv, d).transpose(0, 1).reshape(hkv, -1, d)
    s = torch.matmul(x, k.transpose(1, 2).contiguous()).view(hkv, t, hq // hkv, -1)
    if state["cap"]:
        s = torch.tanh(s.div_(state["cap"])).mul_(state["cap"])
    if state["slopes"] is not None:
        s = s - state["slopes"].view(hkv, 1, -1, 1) * distance[None, :, None]
    return s if seen is None else s.masked_fill_(~seen[None, :, None], LOW)


def _plain_softmax(s):
    """Weights of scores, zero where nothing is seen, and the log-sum-exp."""
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top > LOW, top, 0.0))
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), LOW)[..., 0]
    return p.div_(torch.where(total > 0, total, 1.0)), lse


def _plain_stream(state, i, q, first, out, lse):
    """The attention of stream i's new tokens q [tokens, hq, d] into out and lse."""
    n, held, window = q.shape[0], state["held"][i], state["window"]
    if n == 0 or held == 0:
        return
    k, v = _plain_rows(state, state["page_table"], i, held)
    hkv = k.shape[0]
    key = torch.arange(held, device=q.device)
    step = max(1, 2 ** 28 // (q.shape[1] * held))       # (scores of 1 GiB at a time)
    for a in range(0, n, step):
        b = min(n, a + step)
        at = held - n + torch.arange(a, b, device=q.device)[:, None]
        seen = key <= at
        if state["prefix"] is not None:
            seen = seen | (key < state["prefix_list"][i])
        if window:
            seen = seen & (key > at - window)
        if first is not None:
            seen = seen & (key >= first[a:b, None])
        p, l = _plain_softmax(_plain_scores(state, q[a:b], k, seen, (at - key).abs().float()))
        y = torch.matmul(p.flatten(1, 2), v).view(hkv, b - a, -1, v.shape[-1])
        out[a:b] = y.transpose(0, 1).reshape(b - a, -1, v.shape[-1])
        lse[a:b] = l.transpose(0, 1).reshape(b - a, -1)


def _plain_attention(state):
    q = state["q"]
    out = torch.zeros(q.shape, dtype=torch.float32, device=q.device)
    lse = torch.full(q.shape[:2], LOW, dtype=torch.float32, device=q.device)
    at = 0
    for i, n in enumerate(state["new"]):
        rows = slice(at, at + n)
        _plain_stream(state, i, q[rows], None if state["first"] is None else state["first"][rows], out[rows], lse[rows])
        at += n
    out = out.to(q.dtype)
    return (out, lse) if state["lse"] else out


def _plain_prefix(state):
    q, bounds = state["q"], state["members_list"]
    (_, hq, d), out = q.shape, torch.zeros(q.shape, dtype=torch.float32, device=q.device)
    for g, shared in enumerate(state["shared"]):
        k, v = _plain_rows(state, state["prefix_table"], g, shared)
        key = torch.arange(shared, device=q.device)
        for i in range(bounds[g], bounds[g + 1]):
            held = state["held"][i]
            far = (shared + held - 1 - key)[None].float()
            s = _plain_scores(state, q[i:i + 1], k, None, far)
            if held:
                ki, vi = _plain_rows(state, state["page_table"], i, held)
                near = (held - 1 - torch.arange(held, device=q.device))[None].float()
                s = torch.cat((s, _plain_scores(state, q[i:i + 1], ki, None, near)), -1)
            p, _ = _plain_softmax(s)
            p = p[:, 0]
            y = torch.matmul(p[..., :shared].contiguous(), v)
            if held:
                y = y + torch.matmul(p[..., shared:].contiguous(), vi)
            out[i] = y.reshape(hq, d)
    return out.to(q.dtype)


def _plain_norm(state):
    dtype = state["x"].dtype
    z = state["x"].float()
    if state["post_weight"] is not None:
        z = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + EPS) * state["post_weight"].float()
    if state["gate"] is not None:
        z = z * state["gate"].float()
    r = state["residual"].float() + state["scale"] * z
    if state["weight"] is None:
        return r.to(dtype)
    y = r * torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS) * state["weight"].float()
    return r.to(dtype), y.to(dtype)


def run(state):
    op = state["op"]
    if not own:
        return {"norm": _plain_norm, "prefix": _plain_prefix, "prompt": _plain_attention, "token": _plain_attention}[op](state)
    import paper_2606_01556_amd as tq
    if op == "norm":
        return tq.add_rms_norm(state["x"], state["residual"], state["weight"], post_weight=state["post_weight"],
                               gate=state["gate"], scale=state["scale"], eps=EPS)
    cache = tq.KVCache(*state["cache"])
    if op == "token":
        return tq.paged_attention(cache, state["q"], state["page_table"], state["lengths"], window=state["window"],
                                  softcap=state["cap"], slopes=state["slopes"])
    if op == "prefix":
        return tq.shared_prefix_attention(cache, state["q"], state["members"], state["prefix_table"],
                                          state["prefix_lengths"], state["page_table"], state["lengths"],
                                          softcap=state["cap"], slopes=state["slopes"])
    return tq.prompt_attention(cache, state["q"], state["starts"], state["page_table"], state["lengths"],
                               window=state["window"], prefix=state["prefix"], first=state["first"], softcap=state["cap"],
                               slopes=state["slopes"], return_lse=state["lse"])


# ------------------------------------------------------------------ accounting
def _causal_pairs(n, held, window):
    """Pairs of n new tokens and the keys each sees, of `held` tokens, and the keys that any of them sees."""
    before = held - n
    if not window:
        return n * before + n * (n + 1) // 2, held
    short = min(max(window - before - 1, 0), n)            # tokens that see all keys up to themselves
    return short * before + short * (short + 1) // 2 + (n - short) * window, min(held, window + n - 1)


def work(case):
    """norm: the values in and out, at one addition and a few products each.  Attention: the
    rows that any of a stream's tokens sees, once, the page numbers, q in and the result
    out; two products per pair of a token and a key that it sees.  (Documents and
    prefixes: pairs as the causal mask alone would leave them, over the documents' number;
    what a prefix adds is not counted.)"""
    if case["op"] == "norm":
        t, n = case["tokens"], case["n"]
        arrays = 3 * t + (t if case["before"] else 0) + (t if case["gate"] == "token" else 0)
        rows = (1 if case["before"] else 0) + (1 if case["after"] else 0) + (1 if case["gate"] == "channel" else 0)
        return {"bytes": 2 * n * (arrays + rows), "flops": t * n * (2 + 4 * case["before"] + 4 * case["after"] + (case["gate"] != ""))}
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    new, held = _sizes(case)
    pairs = seen = 0
    for n, h in zip(new, held):
        p, s = _causal_pairs(n, h, case.get("window", 0)) if h else (0, 0)
        pairs, seen = pairs + p // max(case.get("documents", 0), 1), seen + s
    if case["op"] == "prefix":
        bounds = _members(case)
        for g, n in enumerate(_shared(case)):
            pairs, seen = pairs + n * (bounds[g + 1] - bounds[g]), seen + n
    row = 2 * (d * case["bits"] // 8 + (2 if case["bits"] < 16 else 0))
    rows = sum(new)
    return {"bytes": seen * hkv * row + 4 * (seen // page) + 4 * rows * hq * d + (4 * rows * hq if case.get("lse") else 0),
            "flops": 4 * pairs * hq * d}


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
        bit, sign = (8 * i, 8 * i + 7) if i < 4 else (8 * (i - 4) + 4, (8 * (i - 4) + 11) % 32)
        out[..., i] = ((codes >> bit).bitwise_and(7)).double()
        out[..., i] *= torch.where((codes >> sign).bitwise_and(1) == 1, -1.0, 1.0)
    return out.flatten(-2) * scales.double()[..., None]


def _exact_head(s, table, i, tokens, h):
    """Rows `tokens` (positions) of stream i's pages for key-value head h: k, v [n, d]."""
    kc, vc, ks, vs = s["cache"]
    page, bits = kc.shape[2], s["bits"]
    at, off = table[i].long()[tokens // page], tokens % page
    return [_exact_values((c.view(torch.uint8)[at, h, off].view(c.dtype) if bits == 8 else c[at, h, off]),
                          None if w is None else w[at, h, off], bits) for c, w in ((kc, ks), (vc, vs))]


def _exact_weights(s, q, k, head, distance, seen):
    """softmax over the seen keys for one query head's rows q [t, d]; the log-sum-exp."""
    x = torch.mm(q.double(), k.t().contiguous()) * q.shape[-1] ** -0.5
    if s["cap"]:
        x = s["cap"] * (1.0 - 2.0 / (torch.exp(2.0 * x / s["cap"]) + 1.0))
    if s["slopes"] is not None:
        x = x - s["slopes"][head].double() * distance
    x = torch.where(seen, x, LOW)
    lse = torch.logsumexp(x, -1)
    return torch.where(seen, torch.exp(x - torch.where(lse > LOW, lse, 0.0)[:, None]), 0.0), lse


def exact(case, seed):
    if case["op"] == "norm":
        s = _norm_inputs(case, seed)
        z, n = s["x"].double(), case["n"]
        if s["post_weight"] is not None:
            z = z / (z.pow(2).sum(-1, keepdim=True) / n + EPS).sqrt() * s["post_weight"].double()
        if s["gate"] is not None:
            z = z * s["gate"].double()
        r = s["residual"].double() + z * case["scale"]
        if s["weight"] is None:
            return r
        return r, r / (r.pow(2).sum(-1, keepdim=True) / n + EPS).sqrt() * s["weight"].double()
    s = _attention_inputs(case, seed)
    q, d, group = s["q"], case["d"], case["hq"] // case["hkv"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:2], LOW, dtype=torch.float64, device=q.device)
    row = 0
    for i, (n, held) in enumerate(zip(s["new"], s["held"])):
        own_keys = torch.arange(held, device=q.device)
        front = 0
        if case["op"] == "prefix":
            g = max(j for j in range(case["groups"]) if s["members_list"][j] <= i)
            front = s["shared"][g]
        if held + front == 0:
            row += n
            continue
        keys = torch.arange(front + held, device=q.device)[None]
        for h in range(case["hkv"]):
            k, v = _exact_head(s, s["page_table"], i, own_keys, h)
            if front:
                k0, v0 = _exact_head(s, s["prefix_table"], g, torch.arange(front, device=q.device), h)
                k, v = torch.cat((k0, k)), torch.cat((v0, v))
            part = max(1, 2 ** 27 // (front + held))
            for a in range(0, n, part):
                b = min(n, a + part)
                at = (front + held - n + torch.arange(a, b, device=q.device))[:, None]
                low = torch.zeros_like(at)
                if case.get("window"):
                    low = torch.clamp(at - case["window"] + 1, min=0)
                if s["first"] is not None:
                    low = torch.maximum(low, s["first"][row + a:row + b, None].long())
                end = at + 1
                if s["prefix"] is not None:
                    end = torch.clamp(end, min=s["prefix_list"][i])
                seen = (keys >= low) & (keys < end)
                far = torch.abs(at - keys).double()
                for head in range(h * group, (h + 1) * group):
                    w, l = _exact_weights(s, q[row + a:row + b, head], k, head, far, seen)
                    out[row + a:row + b, head] = torch.mm(w, v)
                    lse[row + a:row + b, head] = l
        row += n
    return (out, lse) if s["lse"] else out
