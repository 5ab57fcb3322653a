"""Operators of a decoder that serves requests, and their plain forms: attention over packed prompts with grouped heads
(``FtPrompt.forward``), a paged key / value cache held in 4 bits (``FtCache.append`` with the position rotation, ``FtCache.read``)
and attention of single tokens over it (``FtCache.attend``).

All of them are forward passes.  A cache page holds, for every key / value head, the key codes ``[token][D / 2 bytes]``, the value
codes ``[token / 8][D / 4][token % 8][4 codes in 16 bits]`` and the parameters ``[token / 8][key scale, key minimum, value scale,
value minimum][token % 8]`` in the model's type; a code c stands for scale * c + minimum.
"""
import math
import random

import torch

own = False

DTYPES = {"fp16": (0, torch.float16), "bf16": (1, torch.bfloat16)}


def _prompt(batch, longest, shortest, heads, kv_heads, head_dim, dtype, prefix=0):
    return {"path": "prompt", "batch": batch, "longest": longest, "shortest": shortest, "prefix": prefix, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype}


def _append(batch, longest, shortest, heads, kv_heads, head_dim, dtype, prefix, page_size, rotary_dim, interleaved=False):
    return {"path": "append", "batch": batch, "longest": longest, "shortest": shortest, "prefix": prefix, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "page_size": page_size, "rotary_dim": rotary_dim,
            "interleaved": interleaved}


def _attend(batch, longest, shortest, heads, kv_heads, head_dim, dtype, page_size):
    return {"path": "attend", "batch": batch, "longest": longest, "shortest": shortest, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": dtype, "page_size": page_size}


def _read(batch, longest, shortest, heads, kv_heads, head_dim, dtype, page_size):
    return {"path": "read", "batch": batch, "longest": longest, "shortest": shortest, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": dtype, "page_size": page_size}


def listed():
    named = {
        # one short question
        "prompt_tiny": _prompt(1, 19, 19, 8, 2, 64, "fp16"),
        # a batch of requests of every length, empty ones among them, a key head for every query head
        "prompt_ragged": _prompt(24, 1531, 0, 12, 12, 64, "fp16"),
        # one long prompt: the sizes of the benchmark's longest sequence
        "prompt_long": _prompt(1, 16384, 16384, 32, 4, 128, "bf16"),
        # chunks of prompts whose earlier part lies in the cache already
        "prompt_chunks": _prompt(6, 509, 60, 16, 4, 128, "fp16", prefix=3000),
        # a decoding step's new tokens
        "append_step": _append(32, 1, 1, 32, 8, 128, "bf16", 2048, 16, 128),
        # packed prompts of a prefill, part of the head rotated in neighbouring pairs
        "append_prompts": _append(5, 8192, 700, 32, 8, 128, "fp16", 0, 64, 64, interleaved=True),
        # one sequence at the start of an answer
        "attend_single": _attend(1, 333, 333, 16, 2, 64, "fp16", 16),
        # a batch of dialogues in full swing
        "attend_batch": _attend(32, 4096, 100, 32, 8, 128, "bf16", 16),
        # one very long document: few rows, a long axis
        "attend_long": _attend(1, 131072, 131072, 32, 4, 128, "fp16", 64),
        # a large batch of long dialogues: the cache's bytes are all that counts
        "attend_large": _attend(96, 24000, 6000, 32, 8, 128, "bf16", 32),
        # cached prefixes read back for the next chunk of their prompts
        "read_prefixes": _read(6, 8000, 500, 32, 8, 128, "bf16", 16),
        # a short prefix
        "read_short": _read(2, 211, 100, 16, 2, 64, "fp16", 32),
    }
    return [dict(case, name=name) for name, case in named.items()]


def _lengths(case, longest, shortest, salt):
    """Lengths of the sequences: the longest, and others between the limits, spread over their logarithm; zeros where the shortest is 0."""
    rng = random.Random("%s %d %d %d" % (salt, case["batch"], longest, shortest))
    n = [longest]
    while len(n) < case["batch"]:
        x = int(math.exp(rng.uniform(math.log(max(1, shortest)), math.log(max(1, longest) + 1))))
        n.append(0 if shortest == 0 and rng.random() < 0.1 else max(shortest, min(longest, x)))
    rng.shuffle(n)
    return n


def _sizes(case):
    """(new tokens, tokens before them) of every sequence."""
    n = _lengths(case, case["longest"], case["shortest"], "n")
    prefix = case.get("prefix", 0)
    return n, _lengths(case, prefix, prefix // 5, "p") if prefix else [0] * case["batch"]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm: any value, odd ones among them."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _cost(case):
    """What bounds the plain form: padded scores or padded cached elements, relative to the largest listed case."""
    n, before = _sizes(case)
    most = max(a + b for a, b in zip(n, before))
    if case["path"] == "prompt":
        return case["batch"] * case["heads"] * max(n) * most / (32 * 16384.0 ** 2)
    if case["path"] == "append":
        return sum(n) * (case["heads"] + 4 * case["kv_heads"]) * case["head_dim"] / (16384 * 64 * 128.0)
    return case["batch"] * most * case["kv_heads"] * case["head_dim"] / (96 * 24000 * 8 * 128.0)


def draw(rng):
    """One more case of the same ranges."""
    while True:
        path = rng.choice(["prompt"] * 4 + ["append"] * 2 + ["attend"] * 4 + ["read"])
        dtype, head_dim, page_size = rng.choice(["fp16", "bf16"]), rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 12])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
        if heads > 64:
            continue
        spread = rng.choice([0.0, 0.1, 0.5, 1.0])
        limits = lambda longest: (longest, int(longest * spread))  # noqa: E731
        if path == "prompt":
            prefix = _log(rng, 10, 8000) if rng.random() < 0.25 else 0
            c = _prompt(_log(rng, 1, 32), *limits(_log(rng, 1, 2000 if prefix else 16384)), heads, kv_heads, head_dim, dtype, prefix)
        elif path == "append":
            c = _append(_log(rng, 1, 128), *limits(1 if rng.random() < 0.4 else _log(rng, 2, 16384)), heads, kv_heads, head_dim, dtype,
                        _log(rng, 1, 8000) if rng.random() < 0.6 else 0, page_size, rng.choice([head_dim, head_dim, head_dim // 2, 32]),
                        rng.random() < 0.4)
        elif path == "attend":
            c = _attend(_log(rng, 1, 128), *limits(_log(rng, 1, 131072)), heads, kv_heads, head_dim, dtype, page_size)
        else:
            c = _read(_log(rng, 1, 16), *limits(_log(rng, 1, 16384)), heads, kv_heads, head_dim, dtype, page_size)
        if _cost(c) <= 1.0 and (path == "attend" or _cost(c) <= 0.5 or path == "prompt"):
            return c


def work(case):
    """Operands once, results once; the products' multiplications and additions over the pairs that the mask leaves."""
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    n, before = _sizes(case)
    total, cached = sum(n), hk * (d + 8)
    if case["path"] == "prompt":
        keys = total + sum(before)
        pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(n, before))
        return {"bytes": 2 * d * (2 * h * total + 2 * hk * keys), "flops": 4.0 * d * h * pairs}
    if case["path"] == "append":
        # the tokens' rows once in and once out, their place in the cache written and read back
        return {"bytes": total * (2 * d * (2 * h + 3 * hk) + 4 * case["rotary_dim"] + 2 * cached + 4 * hk * d),
                "flops": total * (h + hk) * 3.0 * case["rotary_dim"] + total * hk * d * 12.0}
    if case["path"] == "attend":
        return {"bytes": total * cached + 4 * case["batch"] * h * d, "flops": 4.0 * d * h * total}
    return {"bytes": total * (cached + 4 * hk * d), "flops": 4.0 * total * hk * d}


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _bounds(n):
    return _ints([sum(n[:i]) for i in range(len(n) + 1)])


def _rotation(positions, rotary_dim):
    """cos then sin of position * 10000^(-2i / rotary_dim), taken in 64 bits."""
    at = torch.arange(positions, device="cuda", dtype=torch.float64)
    speed = 10000.0 ** (-torch.arange(0, rotary_dim, 2, device="cuda", dtype=torch.float64) / rotary_dim)
    angle = at[:, None] * speed
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    code, dtype = DTYPES[case["dtype"]]
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    n, before = _sizes(case)
    total, whole = sum(n), [a + b for a, b in zip(n, before)]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dtype)  # noqa: E731
    s = {"case": case, "cu": _bounds(n), "longest": max(n), "longest_whole": max(whole)}
    if case["path"] == "prompt":
        if case["prefix"]:
            # the chunk's queries, and the keys and values of prefix and chunk
            s |= {"q": normal(total, h, d), "k": normal(sum(whole), hk, d), "v": normal(sum(whole), hk, d), "cu_k": _bounds(whole)}
        else:
            # views of the fused projection's output
            qkv = normal(total, h + 2 * hk, d)
            s |= {"q": qkv[:, :h], "k": qkv[:, h:h + hk], "v": qkv[:, h + hk:], "cu_k": s["cu"]}
        s["o"] = torch.empty((total, h, d), dtype=dtype, device="cuda")
        if own:
            from paper_2504_02211_amd import ftprompt
            s["ctx"] = ftprompt.FtPrompt(h, hk, d, code)
        return s
    ps = case["page_size"]
    per_seq = [(m + ps - 1) // ps for m in whole]
    pages = sum(per_seq) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    width = max(1, max(per_seq))
    cut = _bounds(per_seq)
    at = cut[:-1, None] + torch.arange(width, device="cuda", dtype=torch.int32)
    s["table"] = torch.where(at < cut[1:, None], order[at.clamp(max=pages - 1).long()], 0).contiguous()
    # codes of any value; minima and scales as groups of standard-normal elements have them
    pool = torch.randint(-2 ** 63, 2 ** 63 - 1, (pages * hk * ps * (d + 8) // 8,), generator=g, device="cuda", dtype=torch.int64)
    s["pool"] = pool.view(torch.uint8)
    scale = torch.rand((pages, hk, ps // 8, 2, 8), generator=g, device="cuda") * 0.15 + 0.25
    low = -scale * (torch.rand(scale.shape, generator=g, device="cuda") * 2 + 6.5)
    _parts(s)[2].copy_(torch.stack([scale, low], dim=4).flatten(3, 4).to(dtype).view(torch.uint8).unflatten(-1, (8, 2)))
    s["starts"], s["lengths"], s["batch"] = _ints(before), _ints(whole), case["batch"]
    if case["path"] == "append":
        qkv = normal(total, h + 2 * hk, d)
        s |= {"q": qkv[:, :h], "k": qkv[:, h:h + hk], "v": qkv[:, h + hk:]}
        s["rotation"] = _rotation(max(whole), case["rotary_dim"])
        s |= {"q_rot": torch.empty((total, h, d), dtype=dtype, device="cuda"), "k_rot": torch.empty((total, hk, d), dtype=dtype, device="cuda")}
    if case["path"] == "attend":
        s |= {"q": normal(case["batch"], h, d), "o": torch.empty((case["batch"], h, d), dtype=dtype, device="cuda")}
    else:
        s |= {"k_seen": torch.empty((total, hk, d), dtype=dtype, device="cuda"), "v_seen": torch.empty((total, hk, d), dtype=dtype, device="cuda")}
    if own:
        from paper_2504_02211_amd import ftcache
        s["ctx"] = ftcache.FtCache(h, hk, d, pages, ps, code, rotary_dim=case.get("rotary_dim", 0),
                                   interleaved=case.get("interleaved", False), max_batch=case["batch"])
    return s


def _parts(s):
    """Key codes [page, head, token, D / 2], value codes [page, head, token / 8, D / 4, token % 8, 2], parameters
    [page, head, token / 8, 4, token % 8, 2]: bytes, as views of the pool."""
    c = s["case"]
    ps, d = c["page_size"], c["head_dim"]
    pages = s["pool"].view(-1, c["kv_heads"], ps * (d + 8))
    return (pages[:, :, :ps * d // 2].unflatten(-1, (ps, d // 2)),
            pages[:, :, ps * d // 2:ps * d].unflatten(-1, (ps // 8, d // 4, 8, 2)),
            pages[:, :, ps * d:].unflatten(-1, (ps // 8, 4, 8, 2)))


def _cached(s):
    """Keys and values of every sequence in 32 bits, [batch, head, token, D]: pages gathered, codes unpacked, scaled and shifted."""
    dtype = DTYPES[s["case"]["dtype"]][1]
    d = s["case"]["head_dim"]
    k, v, par = (x[s["table"].long().clamp(min=0)] for x in _parts(s))       # [batch, page, head, ...]
    par = par.contiguous().view(dtype).squeeze(-1).float().transpose(4, 5).transpose(1, 2).flatten(2, 4)     # [batch, head, token, 4]
    k = torch.stack([k & 15, k >> 4], dim=-1).flatten(-2).transpose(1, 2).flatten(2, 3).float()
    v = torch.stack([v & 15, v >> 4], dim=-1).flatten(-2).transpose(4, 5).flatten(5).flatten(3, 4)
    v = v.transpose(1, 2).flatten(2, 3).float()
    assert k.shape[-1] == v.shape[-1] == d
    return k.mul_(par[..., 0:1]).add_(par[..., 1:2]), v.mul_(par[..., 2:3]).add_(par[..., 3:4])


def _of_tokens(s):
    """(sequence, place in its sequence) of every packed token."""
    cu = s["cu"].long()
    t = torch.arange(s["q"].shape[0] if "q" in s else s["k_seen"].shape[0], device="cuda")
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, t - cu[b]


def _padded(x, cu, longest):
    """Packed rows [token, head, D] as [batch, head, place, D] in 32 bits; places behind a sequence hold some other row."""
    at = cu[:-1, None].long() + torch.arange(max(1, longest), device="cuda")
    return x[at.clamp(max=x.shape[0] - 1)].float().transpose(1, 2)


def _softmax_product(scores, seen, v):
    """softmax over the seen keys times v; rows that see none are 0."""
    scores.masked_fill_(~seen, -math.inf)
    most = scores.amax(dim=-1, keepdim=True)
    scores.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    total = scores.sum(dim=-1, keepdim=True)
    out = torch.matmul(scores, v)
    return torch.where(total == 0, 0.0, out / total)


def _plain_prompt(s):
    c, cu, cu_k = s["case"], s["cu"].long(), s["cu_k"].long()
    h, hk, d = c["heads"], c["kv_heads"], c["head_dim"]
    q = _padded(s["q"], s["cu"], s["longest"])
    k, v = (_padded(s[x], s["cu_k"], s["longest_whole"]) for x in "kv")
    batch, nq, nk = q.shape[0], q.shape[2], k.shape[2]
    scores = torch.matmul(q.reshape(batch, hk, (h // hk) * nq, d), k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
    lens, lens_k = (cu[1:] - cu[:-1])[:, None], (cu_k[1:] - cu_k[:-1])[:, None]
    last = lens_k - lens + torch.arange(nq, device="cuda")                      # the last key that a query sees
    seen = torch.arange(nk, device="cuda") <= last[:, :, None]
    out = _softmax_product(scores.view(batch, hk, h // hk, nq, nk), seen[:, None, None], v.unsqueeze(2))
    b, at = _of_tokens(s)
    return out.reshape(batch, h, nq, d)[b, :, at].to(s["q"].dtype)


def _rotated(x, cos, sin, rotary_dim, interleaved):
    y = x.float()
    a, b = (y[..., 0:rotary_dim:2], y[..., 1:rotary_dim:2]) if interleaved else (y[..., :rotary_dim // 2], y[..., rotary_dim // 2:rotary_dim])
    first, second = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([first, second], dim=-1).flatten(-2) if interleaved else torch.cat([first, second], dim=-1)
    return torch.cat([turned, y[..., rotary_dim:]], dim=-1).to(x.dtype)


def _coded(x):
    """Codes of x [token, head, D] in the groups of one token and head, with their scales and minima (in x's type)."""
    y = x.float()
    low, high = y.amin(dim=-1, keepdim=True), y.amax(dim=-1, keepdim=True)
    scale = (high / 15 - low / 15).to(x.dtype)
    half = scale.float() * 0.5
    codes = ((y * 0.5 - low * 0.5) / torch.where(half == 0, 1.0, half)).round().clamp(0, 15)
    return torch.where(half == 0, 0.0, codes).to(torch.uint8), scale, low.to(x.dtype)


def _plain_append(s):
    c = s["case"]
    ps = c["page_size"]
    b, at = _of_tokens(s)
    place = s["starts"].long()[b] + at
    page, row = s["table"][b, place // ps].long(), place % ps
    cos, sin = s["rotation"][place].unsqueeze(1).chunk(2, dim=-1)
    q, k = (_rotated(s[x], cos, sin, c["rotary_dim"], c["interleaved"]) for x in "qk")
    (kc, ks, kl), (vc, vs, vl) = _coded(k), _coded(s["v"])
    kp, vp, par = _parts(s)
    kp[page, :, row] = kc[..., 0::2] | kc[..., 1::2] << 4
    vp[page, :, row // 8, :, row % 8] = (vc[..., 0::2] | vc[..., 1::2] << 4).unflatten(-1, (-1, 2))
    par[page, :, row // 8, :, row % 8] = torch.cat([ks, kl, vs, vl], dim=-1).view(torch.uint8).unflatten(-1, (4, 2))
    return {"q_rot": q, "k_rot": k, **_plain_read(s)}


def _plain_read(s):
    c = s["case"]
    ps, d = c["page_size"], c["head_dim"]
    dtype = DTYPES[c["dtype"]][1]
    b, at = _of_tokens(s)
    place = s["starts"].long()[b] + at
    page, row = s["table"][b, place // ps].long(), place % ps
    kp, vp, par = _parts(s)
    k, v = kp[page, :, row], vp[page, :, row // 8, :, row % 8].flatten(-2)       # [token, head, D / 2]
    par = par[page, :, row // 8, :, row % 8].contiguous().view(dtype).squeeze(-1).float()
    k, v = (torch.stack([x & 15, x >> 4], dim=-1).flatten(-2).float() for x in (k, v))
    return {"k_seen": (k * par[..., 0:1] + par[..., 1:2]).to(dtype), "v_seen": (v * par[..., 2:3] + par[..., 3:4]).to(dtype)}


def _plain_attend(s):
    c = s["case"]
    h, hk, d = c["heads"], c["kv_heads"], c["head_dim"]
    k, v = _cached(s)
    q = s["q"].float().view(-1, hk, h // hk, d)
    seen = torch.arange(k.shape[2], device="cuda") < s["lengths"][:, None]
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
    return _softmax_product(scores, seen[:, None, None], v).reshape(-1, h, d).to(s["q"].dtype)


def run(s):
    path = s["case"]["path"]
    if not own:
        return {"prompt": _plain_prompt, "append": _plain_append, "read": _plain_read, "attend": _plain_attend}[path](s)
    stream = torch.cuda.current_stream().cuda_stream
    if path == "prompt":
        s["ctx"].forward(s["q"], s["k"], s["v"], s["o"], s["cu"], s["cu_k"], stream)
        return s["o"]
    if path == "attend":
        s["ctx"].attend(s["pool"], s["q"], s["o"], s["lengths"], s["table"], stream)
        return s["o"]
    out = {}
    if path == "append":
        s["ctx"].append(s["pool"], s["q"], s["k"], s["v"], s["rotation"], s["cu"], s["starts"], s["table"], s["q_rot"], s["k_rot"], stream)
        out = {"q_rot": s["q_rot"], "k_rot": s["k_rot"]}
    s["ctx"].read(s["pool"], s["k_seen"], s["v_seen"], s["cu"], s["starts"], s["table"], stream)
    return {**out, "k_seen": s["k_seen"], "v_seen": s["v_seen"]}


def _element(s, b, first, count, value):
    """Cached elements [token, head, D] of sequence b in 64 bits, each from its address in the pool."""
    c = s["case"]
    hk, d, ps, dtype = c["kv_heads"], c["head_dim"], c["page_size"], DTYPES[c["dtype"]][1]
    place = torch.arange(first, first + count, device="cuda")
    head, e = torch.arange(hk, device="cuda")[:, None], torch.arange(d, device="cuda")
    row = (place % ps)[:, None, None]
    base = (s["table"][b].long()[place // ps][:, None, None] * hk + head) * (ps * (d + 8))
    at = ps * d // 2 + (row // 8) * 4 * d + (e // 4) * 16 + (row % 8) * 2 + (e % 4) // 2 if value else row * (d // 2) + e // 2
    codes = (s["pool"][base + at] >> (e % 2 * 4).to(torch.uint8)) & 15
    numbers = s["pool"].view(dtype)
    at = (base + ps * d) // 2 + (row // 8) * 32 + row % 8 + (16 if value else 0)
    return codes.double() * numbers[at].double() + numbers[at + 8].double()


def _exact_rows(q, k, v, visible, scale):
    """q [row, group, D], k, v [key, D], visible [row]: how many keys each row sees."""
    p = torch.tensordot(q, k, dims=([2], [1])) * scale
    p[(torch.arange(k.shape[0], device="cuda") >= visible[:, None])[:, None].expand_as(p)] = -math.inf
    p = torch.softmax(p, dim=-1)
    p[visible <= 0] = 0.0
    return torch.tensordot(p, v, dims=([2], [0]))


def _quantised(x, dtype):
    """What a cache in 4 bits holds of x [token, head, D] (64 bits, values of dtype)."""
    low = x.min(dim=-1, keepdim=True).values
    scale = ((x.max(dim=-1, keepdim=True).values - low) / 15.0).to(dtype).double()
    steps = torch.clamp(torch.round((x - low) / scale), 0, 15)
    return torch.where(scale > 0, steps * scale, torch.zeros_like(x)) + low


def exact(case, seed):
    s = prepare(case, seed)
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    dtype = DTYPES[case["dtype"]][1]
    group, scale = h // hk, d ** -0.5
    n, before = _sizes(case)
    starts = [sum(n[:i]) for i in range(len(n))]
    if case["path"] == "prompt":
        out = torch.zeros((sum(n), h, d), dtype=torch.float64, device="cuda")
        at_k = 0
        for b, m in enumerate(n):
            keys = m + before[b]
            for head in range(hk):
                k, v = (s[x][at_k:at_k + keys, head].double() for x in "kv")
                for i in range(0, m, 2048):
                    rows = slice(starts[b] + i, starts[b] + min(m, i + 2048))
                    heads = slice(head * group, (head + 1) * group)
                    visible = before[b] + 1 + torch.arange(i, min(m, i + 2048), device="cuda")
                    out[rows, heads] = _exact_rows(s["q"][rows, heads].double(), k, v, visible, scale)
            at_k += keys
        return out
    if case["path"] == "attend":
        out = torch.zeros((case["batch"], h, d), dtype=torch.float64, device="cuda")
        for b, m in enumerate(n):
            if m:
                k, v = _element(s, b, 0, m, False), _element(s, b, 0, m, True)
                for head in range(hk):
                    heads = slice(head * group, (head + 1) * group)
                    seen = torch.tensor([m], device="cuda")
                    out[b, heads] = _exact_rows(s["q"][b:b + 1, heads].double(), k[:, head], v[:, head], seen, scale)[0]
        return out
    if case["path"] == "read":
        empty = torch.zeros((0, hk, d), dtype=torch.float64, device="cuda")
        return {x: torch.cat([_element(s, b, before[b], m, x == "v_seen") if m else empty for b, m in enumerate(n)]) for x in ("k_seen", "v_seen")}
    place = torch.cat([torch.arange(p, p + m, device="cuda") for m, p in zip(n, before)])
    r = case["rotary_dim"]
    turn = torch.polar(torch.ones(()).double().to("cuda"), torch.zeros(()).double().to("cuda"))
    turn = turn * torch.complex(s["rotation"][place][:, :r // 2].double(), s["rotation"][place][:, r // 2:].double())[:, None]
    out = {}
    for x in "qk":
        y = s[x].double()
        pairs = y[..., :r].unflatten(-1, (-1, 2)) if case["interleaved"] else y[..., :r].unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
        out[x + "_rot"] = torch.cat([z, y[..., r:]], dim=-1)
    return {**out, "k_seen": _quantised(out["k_rot"].to(dtype).double(), dtype), "v_seen": _quantised(s["v"].double(), dtype)}
