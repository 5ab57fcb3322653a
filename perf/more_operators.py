"""More operators of a decoder that serves requests, and their plain forms: the linear layer on 8-bit integers with a scale for each token
and each output channel (``FtInt8.forward``), linear attention with a decay for each head over packed prompts (``FtDecay.forward``) and
for single tokens (``FtDecay.step``), and the choice of the next token from its logits and a given random number (``FtSample.choose``).

All of them are forward passes.  The codes of a row x are rint(x * (127 / max|x|)), its scale is max|x| / 127; weights are given as codes and
scales.  Linear attention keeps one matrix per sequence and head, S = exp(log_decay) S + k v^T for every token, which gives scale * q S.
"""
import math
import random

import torch

own = False

DTYPES = {"fp16": (0, torch.float16), "bf16": (1, torch.bfloat16), "fp32": (2, torch.float32)}


def _linear(m, n, k, dtype):
    return {"path": "linear", "m": m, "n": n, "k": k, "dtype": dtype}


def _prompt(batch, longest, shortest, heads, kv_heads, head_dim, dtype, continued=False):
    return {"path": "prompt", "batch": batch, "longest": longest, "shortest": shortest, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": dtype, "continued": continued}


def _step(batch, heads, kv_heads, head_dim, dtype):
    return {"path": "step", "batch": batch, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype}


def _choose(rows, vocab, dtype, temperature, top_k, top_p, min_p, masked=0.0):
    return {"path": "choose", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature, "top_k": top_k, "top_p": top_p,
            "min_p": min_p, "masked": masked}


def listed():
    named = {
        # one token through a feed-forward layer: the weights' bytes are all that counts
        "linear_token": _linear(1, 16384, 4096, "bf16"),
        # a decoding step of a batch, back from the feed-forward layer's width
        "linear_step": _linear(96, 4096, 16384, "bf16"),
        # packed prompts on sizes that no tile divides
        "linear_odd": _linear(1531, 2500, 1000, "fp16"),
        # a long prompt: the benchmark's linear layer
        "linear_prompt": _linear(16384, 16384, 4096, "fp16"),
        # one short question
        "decay_tiny": _prompt(1, 19, 19, 8, 8, 64, "fp16"),
        # a batch of requests of every length, empty ones among them, chunks of prompts whose earlier part the states hold
        "decay_ragged": _prompt(24, 1531, 0, 12, 12, 64, "fp16", continued=True),
        # one long prompt: the sizes of the benchmark's longest sequence
        "decay_long": _prompt(1, 16384, 16384, 32, 8, 128, "bf16"),
        # one token of one sequence
        "decay_token": _step(1, 16, 16, 64, "fp16"),
        # a decoding step of a batch
        "decay_step": _step(96, 32, 8, 128, "bf16"),
        # one sequence's next token, all rules in force
        "choose_one": _choose(1, 32000, "fp16", True, True, True, True),
        # a batch without truncation, tokens masked by a grammar
        "choose_masked": _choose(48, 50001, "fp32", True, False, False, False, masked=0.3),
        # a large batch over a large vocabulary, nucleus and floor, every row with values of its own
        "choose_batch": _choose(256, 131072, "bf16", True, False, True, True),
    }
    return [dict(case, name=name) for name, case in named.items()]


def _lengths(case):
    """Lengths of the sequences: the longest, and others between the limits, spread over their logarithm; zeros where the shortest is 0."""
    longest, shortest = case["longest"], case["shortest"]
    rng = random.Random("%d %d %d" % (case["batch"], longest, shortest))
    n = [longest]
    while len(n) < case["batch"]:
        x = int(math.exp(rng.uniform(math.log(max(1, shortest)), math.log(max(1, longest) + 1))))
        n.append(0 if shortest == 0 and rng.random() < 0.1 else max(shortest, min(longest, x)))
    rng.shuffle(n)
    return n


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm: any value, odd ones among them."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _cost(case):
    """What bounds the plain form, relative to the largest listed case of its path."""
    if case["path"] == "linear":
        return case["m"] * case["n"] * case["k"] / (16384.0 * 16384 * 4096)
    if case["path"] == "prompt":
        return case["batch"] * case["heads"] * case["longest"] ** 2 / (32 * 16384.0 ** 2)
    if case["path"] == "step":
        return case["batch"] * case["heads"] * case["head_dim"] ** 2 / (96 * 32 * 128.0 ** 2)
    return case["rows"] * case["vocab"] / (256 * 131072.0)


def draw(rng):
    """One more case of the same ranges."""
    while True:
        path = rng.choice(["linear"] * 4 + ["prompt"] * 3 + ["step"] * 2 + ["choose"] * 4)
        kv_heads, head_dim = rng.choice([1, 2, 3, 4, 8, 12, 16]), rng.choice([64, 128])
        heads = kv_heads * rng.choice([1, 1, 1, 2, 3, 4, 5, 8])
        if heads > 64:
            continue
        if path == "linear":
            # half of the widths are multiples of 64, as layers have them
            n, k = (64 * _log(rng, 1, 256) if rng.random() < 0.5 else _log(rng, 16, 16384) for _ in range(2))
            c = _linear(_log(rng, 1, 16384), n, k, rng.choice(["fp16", "bf16"]))
        elif path == "prompt":
            longest = _log(rng, 1, 16384)
            c = _prompt(_log(rng, 1, 32), longest, int(longest * rng.choice([0.0, 0.1, 0.5, 1.0])), heads, kv_heads, head_dim,
                        rng.choice(["fp16", "bf16"]), rng.random() < 0.5)
        elif path == "step":
            c = _step(_log(rng, 1, 512), heads, kv_heads, head_dim, rng.choice(["fp16", "bf16"]))
        else:
            c = _choose(_log(rng, 1, 512), _log(rng, 100, 262144), rng.choice(["fp16", "bf16", "fp32"]),
                        *(rng.random() < share for share in (0.8, 0.5, 0.5, 0.3)), masked=rng.choice([0.0, 0.0, 0.3, 0.95]))
        if _cost(c) <= 1.0:
            return c


def work(case):
    """Operands once, results once; multiplications and additions of the products, of the recurrence for linear attention."""
    if case["path"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 2 * m * k + n * k + 4 * n + 2 * m * n, "flops": 2.0 * m * n * k}
    if case["path"] == "choose":
        # a maximum, a weight and its place in a sum for every logit
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": case["rows"] * (case["vocab"] * size + 28), "flops": 4.0 * case["rows"] * case["vocab"]}
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    n = _lengths(case) if case["path"] == "prompt" else [1] * case["batch"]
    states = len(n) * h * d * d * 4
    read = case["path"] == "step" or case["continued"]
    return {"bytes": 2 * sum(n) * d * (2 * h + 2 * hk) + states * (2 if read else 1), "flops": 4.0 * sum(n) * h * d * d}


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _codes(x):
    """Codes of the rows of x in 8 bits, as numbers in 32, and their scales."""
    y = x.float()
    most = y.abs().amax(dim=1)
    inverse = torch.where(most == 0, 0.0, 127.0 / most)
    return (y * inverse[:, None]).round_(), most / 127.0


def _prepare_linear(case, g):
    code, dtype = DTYPES[case["dtype"]]
    m, n, k = case["m"], case["n"], case["k"]
    x = torch.randn((m, k), generator=g, device="cuda")
    # some channels of the activations are larger than the others
    x *= torch.where(torch.rand(k, generator=g, device="cuda") < 0.01, 8.0, 1.0)
    codes, scales = _codes(torch.randn((n, k), generator=g, device="cuda") * k ** -0.5)
    s = {"case": case, "x": x.to(dtype), "codes": codes.to(torch.int8), "scales": scales, "y": torch.empty((m, n), dtype=dtype, device="cuda")}
    if own:
        from paper_2504_02211_amd import ftint8
        s["ctx"] = ftint8.FtInt8(n, k, code, max_tokens=m)
        # rows of codes as the layer reads them: filled up with zeros
        s["codes"] = torch.nn.functional.pad(s["codes"], (0, s["ctx"].k_padded - k)).contiguous()
    return s


def _prepare_attention(case, g):
    code, dtype = DTYPES[case["dtype"]]
    h, hk, d, prompt = case["heads"], case["kv_heads"], case["head_dim"], case["path"] == "prompt"
    n = _lengths(case) if prompt else [1] * case["batch"]
    total, batch = sum(n), len(n)
    # views of the fused projection's output
    qkv = torch.randn((total, h + 2 * hk, d), generator=g, device="cuda").to(dtype)
    s = {"case": case, "q": qkv[:, :h], "k": qkv[:, h:h + hk], "v": qkv[:, h + hk:], "o": torch.empty((total, h, d), dtype=dtype, device="cuda")}
    # heads that forget after some tokens, and heads that remember thousands
    half_life = 2.0 ** torch.linspace(1, 12, h, device="cuda", dtype=torch.float64)
    s["log_decay"] = (-math.log(2.0) / half_life).float()
    # sequences have their states where a slot of the pool was free
    s["slots"] = torch.randperm(batch + 3, generator=g, device="cuda")[:batch].to(torch.int32)
    s["states"] = torch.randn((batch + 3, h, d, d), generator=g, device="cuda")
    if prompt:
        s["cu"] = _ints([sum(n[:i]) for i in range(batch + 1)])
        s["longest"] = max(n)
        # tokens before these: a sequence without any begins with zeros
        s["starts"] = torch.randint(1, 1000, (batch,), generator=g, device="cuda", dtype=torch.int32) * case["continued"]
    if own:
        from paper_2504_02211_amd import ftdecay
        s["ctx"] = ftdecay.FtDecay(h, hk, d, code)
    return s


def _prepare_choose(case, g):
    code, dtype = DTYPES[case["dtype"]]
    rows, vocab = case["rows"], case["vocab"]
    uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    # rows from sure to undecided
    logits = torch.randn((rows, vocab), generator=g, device="cuda") * (1.0 + 3.0 * uniform(rows, 1))
    if case["masked"]:
        logits[uniform(rows, vocab) < case["masked"]] = -math.inf
    s = {"case": case, "logits": logits.to(dtype), "uniform": uniform(rows), "tokens": torch.empty(rows, dtype=torch.int32, device="cuda"),
         "probability": torch.empty(rows, dtype=torch.float32, device="cuda")}
    # one request in eight asks for the likeliest token, or for no cut
    some = lambda: uniform(rows) < 0.125  # noqa: E731
    s["temperature"] = torch.where(some(), 0.0, 0.3 + uniform(rows)) if case["temperature"] else None
    s["top_k"] = torch.where(some(), 0, (2.0 ** (uniform(rows) * 10)).int()) if case["top_k"] else None
    s["top_p"] = torch.where(some(), 1.0, 0.5 + 0.5 * uniform(rows)) if case["top_p"] else None
    s["min_p"] = torch.where(some(), 0.0, 0.1 * uniform(rows)) if case["min_p"] else None
    if own:
        from paper_2504_02211_amd import ftsample
        s["ctx"] = ftsample.FtSample(vocab, code, max_rows=rows)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"linear": _prepare_linear, "choose": _prepare_choose}.get(case["path"], _prepare_attention)(case, g)


def _plain_linear(s):
    # (sums of up to 16384 products of two codes leave the 24 bits that whole numbers have in 32)
    codes, scales = _codes(s["x"])
    sums = torch.matmul(codes.double(), s["codes"].double().t())
    return sums.mul_(scales.double()[:, None]).mul_(s["scales"].double()).to(s["x"].dtype)


def _of_states(s):
    c = s["case"]
    return c["kv_heads"], c["heads"] // c["kv_heads"], c["head_dim"], c["head_dim"] ** -0.5, s["slots"].long()


def _plain_step(s):
    hk, group, d, scale, slots = _of_states(s)
    q, k, v = (s[x].float() for x in "qkv")
    k, v = k.repeat_interleave(group, dim=1), v.repeat_interleave(group, dim=1)
    state = s["states"][slots] * s["log_decay"].exp()[:, None, None] + k[..., :, None] * v[..., None, :]
    s["states"][slots] = state
    return {"o": (torch.matmul(q[:, :, None], state)[:, :, 0] * scale).to(s["q"].dtype), "states": s["states"]}


def _plain_prompt(s):
    hk, group, d, scale, slots = _of_states(s)
    cu, g = s["cu"].long(), s["log_decay"]
    lens, batch, h, longest = cu[1:] - cu[:-1], len(slots), hk * group, max(1, s["longest"])
    place = torch.arange(longest, device="cuda")
    at = (cu[:-1, None] + place).clamp(max=s["q"].shape[0] - 1)
    q, k, v = (s[x][at].float().transpose(1, 2) for x in "qkv")                  # [batch, head, place, D]
    here = (place < lens[:, None])[:, None, :, None]
    k, v = torch.where(here, k, 0.0), torch.where(here, v, 0.0)
    first = torch.where((s["starts"] > 0)[:, None, None, None], s["states"][slots], 0.0)
    # the tokens' own weights, decayed over the places between
    weights = torch.matmul(q.reshape(batch, hk, group * longest, d), k.transpose(-1, -2)).view(batch, h, longest, longest)
    between = (place[:, None] - place).float()
    weights.mul_((between.clamp(min=0) * g[:, None, None]).exp_())
    weights.masked_fill_(between < 0, 0.0)
    out = torch.matmul(weights.view(batch, hk, group * longest, longest), v).view(batch, h, longest, d)
    # and what the state has of earlier ones
    out += torch.matmul(q, first) * ((place + 1) * g[:, None]).exp()[:, :, None]
    left = (lens[:, None] - 1 - place).clamp(min=0)[:, None] * g[:, None]        # [batch, head, place]
    k, v = k.repeat_interleave(group, dim=1), v.repeat_interleave(group, dim=1)
    last = torch.matmul((k * left.exp()[..., None]).transpose(-1, -2), v) + first * (lens[:, None] * g).exp()[..., None, None]
    s["states"][slots] = last
    b = torch.searchsorted(cu, torch.arange(s["q"].shape[0], device="cuda"), right=True) - 1
    return {"o": (out[b, :, torch.arange(len(b), device="cuda") - cu[b]] * scale).to(s["q"].dtype), "states": s["states"]}


def _plain_choose(s):
    c, x = s["case"], s["logits"].float()
    rows, vocab = x.shape
    value = lambda name, otherwise: otherwise if s[name] is None else s[name][:, None].double()  # noqa: E731
    temperature = value("temperature", 1.0)
    greedy = torch.as_tensor(temperature, device="cuda") <= 0
    x, order = x.sort(dim=1, descending=True, stable=True)
    # (weights and their sums in 64 bits: the random number may lie next to a border)
    weight = ((x.double() - x[:, :1].double()) / torch.where(greedy, 1.0, temperature)).exp_()
    weight = torch.where(x == -math.inf, 0.0, weight)
    rank = torch.arange(vocab, device="cuda")
    most = torch.where(greedy, 1, vocab).expand(rows, 1)
    if s["top_k"] is not None:
        most = torch.where((s["top_k"] > 0)[:, None], torch.minimum(most, s["top_k"][:, None]), most)
    weight = torch.where(rank < most, weight, 0.0)
    if s["top_p"] is not None:
        total = weight.cumsum(dim=1)
        before = torch.cat([torch.zeros_like(total[:, :1]), total[:, :-1]], dim=1)
        weight = torch.where((before < value("top_p", 1.0) * total[:, -1:]) | (rank == 0) | (value("top_p", 1.0) >= 1), weight, 0.0)
    if s["min_p"] is not None:
        weight = torch.where((weight >= value("min_p", 0.0)) | (rank == 0), weight, 0.0)
    kept = torch.zeros_like(weight).scatter_(1, order, weight)
    upto = kept.cumsum(dim=1)
    total = upto[:, -1:]
    token = (upto <= s["uniform"][:, None].double() * total).sum(dim=1, keepdim=True)
    chance = torch.where(total > 0, kept.gather(1, token.clamp(max=vocab - 1)) / total, 0.0)
    return {"tokens": torch.where(total > 0, token, -1).int()[:, 0], "probability": chance.float()[:, 0]}


def run(s):
    path = s["case"]["path"]
    if not own:
        return {"linear": _plain_linear, "prompt": _plain_prompt, "step": _plain_step, "choose": _plain_choose}[path](s)
    stream = torch.cuda.current_stream().cuda_stream
    if path == "linear":
        s["ctx"].forward(s["x"], s["codes"], s["scales"], s["y"], stream)
        return s["y"]
    if path == "choose":
        s["ctx"].choose(s["logits"], s["uniform"], s["tokens"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["probability"], stream)
        return {"tokens": s["tokens"], "probability": s["probability"]}
    if path == "prompt":
        s["ctx"].forward(s["q"], s["k"], s["v"], s["o"], s["log_decay"], s["states"], s["cu"], s["starts"], s["slots"], stream)
    else:
        s["ctx"].step(s["q"], s["k"], s["v"], s["o"], s["log_decay"], s["states"], s["slots"], stream)
    return {"o": s["o"], "states": s["states"]}


def _exact_linear(s):
    x = s["x"].double()
    unit = (x.abs().max(dim=1, keepdim=True).values.float() / 127.0).double()
    whole = torch.round(s["x"].float() * (127.0 / s["x"].float().abs().max(dim=1, keepdim=True).values)).double()
    w = s["codes"][:, :s["case"]["k"]].double() * s["scales"].double()[:, None]
    return torch.nn.functional.linear(whole * torch.where(unit > 0, unit, 0.0), w)


def _exact_sequence(q, k, v, state, decay, scale):
    """q, k, v [head, token, D] in 64 bits, state [head, D, D], decay [head]: by pieces of 128 tokens, each from the state before it."""
    out = []
    for i in range(0, q.shape[1], 128):
        qi, ki, vi = (x[:, i:i + 128] for x in (q, k, v))
        m = qi.shape[1]
        powers = decay[:, None] ** torch.arange(m + 1, device="cuda").double()
        lower = torch.zeros((len(decay), m, m), dtype=torch.float64, device="cuda")
        for j in range(m):
            lower[:, j:, j] = powers[:, :m - j]
        out.append(scale * (torch.bmm(torch.bmm(qi, ki.transpose(1, 2).contiguous()) * lower, vi) + torch.bmm(qi * powers[:, 1:, None], state)))
        state = state * powers[:, m, None, None] + torch.bmm((ki * powers[:, :m].flip(1)[:, :, None]).transpose(1, 2).contiguous(), vi)
    return torch.cat(out, dim=1), state


def _exact_attention(s):
    c = s["case"]
    h, d, group = c["heads"], c["head_dim"], c["heads"] // c["kv_heads"]
    n = _lengths(c) if c["path"] == "prompt" else [1] * c["batch"]
    decay, slots = torch.exp(s["log_decay"].double()), s["slots"].tolist()
    fresh = [x == 0 for x in s["starts"].tolist()] if c["path"] == "prompt" else [False] * len(n)
    if c["path"] == "step":
        k, v = (s[x].double()[:, torch.arange(h, device="cuda") // group] for x in "kv")
        states = s["states"].double()
        states[slots] = states[slots] * decay[:, None, None] + torch.einsum("bhi,bhj->bhij", k, v)
        return {"o": (s["q"].double().unsqueeze(-1) * states[slots]).sum(dim=2) * d ** -0.5, "states": states}
    states, out, at = s["states"].double(), torch.zeros(s["o"].shape, dtype=torch.float64, device="cuda"), 0
    for b, m in enumerate(n):
        state = torch.zeros_like(states[slots[b]]) if fresh[b] else states[slots[b]].clone()
        if m:
            q, k, v = (s[x][at:at + m].double().transpose(0, 1) for x in "qkv")
            k, v = (x[torch.arange(h, device="cuda") // group] for x in (k, v))
            o, state = _exact_sequence(q, k, v, state, decay, d ** -0.5)
            out[at:at + m] = o.transpose(0, 1)
        states[slots[b]] = state
        at += m
    return {"o": out, "states": states}


def _exact_choose(s):
    """Row after row: the kept tokens found one rule after the other, in the order of their ranks."""
    tokens, chances = [], []
    for r in range(s["logits"].shape[0]):
        x = s["logits"][r].double()
        at = lambda name, otherwise: otherwise if s[name] is None else s[name][r].item()  # noqa: E731
        temperature, k, p, floor = at("temperature", 1.0), at("top_k", 0), at("top_p", 1.0), at("min_p", 0.0)
        if not bool((x > -math.inf).any()):
            tokens.append(-1)
            chances.append(0.0)
            continue
        kept = torch.argsort(-x, stable=True)
        kept = kept[x[kept] > -math.inf]
        if temperature <= 0:
            kept, temperature = kept[:1], 1.0
        if k > 0:
            kept = kept[:k]
        w = torch.exp((x[kept] - x[kept[0]]) / temperature)
        if p < 1:
            upto = torch.cumsum(w, 0)
            count = max(1, int((upto - w < p * upto[-1]).sum()))
            kept, w = kept[:count], w[:count]
        count = max(1, int((w >= floor).sum()))
        kept, w = kept[:count], w[:count]
        kept, places = torch.sort(kept)
        w = w[places]
        upto = torch.cumsum(w, 0)
        chosen = int(torch.searchsorted(upto, s["uniform"][r].double() * upto[-1], right=True))
        tokens.append(int(kept[chosen]))
        chances.append((w[chosen] / upto[-1]).item())
    return {"tokens": torch.tensor(tokens, dtype=torch.int32), "probability": torch.tensor(chances, dtype=torch.float64)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "choose": _exact_choose}.get(case["path"], _exact_attention)(s)
