"""A small decoder on the serving operators: layers on 8-bit integers around linear attention, logits, the next token; prompts first, then steps.

Every stage is compared with its formula in 64 bits on what the stage before it really gave, and a captured step with the eager one, bit for bit.
"""
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftdecay, ftint8, ftsample

pytestmark = pytest.mark.gpu

HEADS, KV, D, WIDTH, VOCAB, BATCH = 4, 2, 64, 200, 3001, 3


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Decoder:
    def __init__(self, dtype, code, tokens):
        g = torch.Generator(device="cuda").manual_seed(11)
        self.dtype, self.g = dtype, g
        normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.table = normal(VOCAB, WIDTH).to(dtype)
        self.attention = ftdecay.FtDecay(HEADS, KV, D, code)
        self.sample = ftsample.FtSample(VOCAB, ftsample.F32, max_rows=BATCH)
        self.layers = {}
        for name, n, k, out in (("qkv", (HEADS + 2 * KV) * D, WIDTH, code), ("back", WIDTH, HEADS * D, code), ("logits", VOCAB, WIDTH, ftint8.F32)):
            layer = ftint8.FtInt8(n, k, code, out, max_tokens=tokens)
            w, scales = torch.empty((n, layer.k_padded), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
            layer.encode((normal(n, k) * k ** -0.5).to(dtype), w, scales, torch.cuda.current_stream().cuda_stream)
            self.layers[name] = layer, w, scales
        self.log_decay = torch.tensor([-0.5, -0.1, -0.02, -0.002], device="cuda")
        self.states = torch.full((BATCH + 2, HEADS, D, D), float("nan"), device="cuda")
        self.slots, self.top_k, self.top_p = ints([3, 0, 2]), ints([50, 0, 7]), torch.tensor([0.9, 0.95, 1.0], device="cuda")

    def layer(self, name, x, stream):
        layer, w, scales = self.layers[name]
        y = torch.empty((x.shape[0], layer.config.n), dtype=torch.float32 if name == "logits" else self.dtype, device="cuda")
        layer.forward(x, w, scales, y, stream)
        return y

    def tokens(self, ids, cu, starts):
        """Hidden rows of packed tokens; cu None: one token of every sequence."""
        stream = torch.cuda.current_stream().cuda_stream
        x = self.table[ids]
        qkv = self.layer("qkv", x, stream).view(-1, HEADS + 2 * KV, D)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
        o = torch.empty((len(ids), HEADS, D), dtype=self.dtype, device="cuda")
        if cu is None:
            self.attention.step(q, k, v, o, self.log_decay, self.states, self.slots, stream)
        else:
            self.attention.forward(q, k, v, o, self.log_decay, self.states, cu, starts, self.slots, stream)
        y = self.layer("back", o.view(-1, HEADS * D), stream)
        return dict(x=x, q=q, k=k, v=v, o=o, y=y)

    def choose(self, rows, uniform):
        stream = torch.cuda.current_stream().cuda_stream
        logits = self.layer("logits", rows, stream)
        tokens = torch.empty(BATCH, dtype=torch.int32, device="cuda")
        self.sample.choose(logits, uniform, tokens, top_k=self.top_k, top_p=self.top_p, stream=stream)
        return logits, tokens

    def check_layer(self, name, x, y):
        """Tokens are off by up to half a code of their scale in each element, the result by its rounding."""
        layer, w, scales = self.layers[name]
        weights = w[:, :layer.config.k].double() * scales.double()[:, None]
        most = x.double().abs().amax(1, keepdim=True) / 127
        near = (0.5 + 2.0 ** -15) * most * weights.abs().sum(1)
        want = x.double() @ weights.T
        assert ((y.double() - want).abs() <= near + (want.abs() + near) * (torch.finfo(y.dtype).eps / 2 + 2.0 ** -22)).all()


@pytest.mark.parametrize("dtype,code", [(torch.float16, 0), (torch.bfloat16, 1)])
def test_prompts_then_steps(dtype, code):
    lengths, steps = [70, 1, 33], 4
    d = Decoder(dtype, code, sum(lengths))
    cu = ints([0, 70, 71, 104])
    ids = torch.randint(0, VOCAB, (sum(lengths),), generator=d.g, device="cuda")
    uniform = torch.rand((steps + 1, BATCH), generator=d.g, device="cuda")
    first = d.tokens(ids, cu, None)
    logits, new = d.choose(first["y"][cu[1:].long() - 1], uniform[0])
    history = [{k: v.clone() for k, v in first.items()}]
    for name, x, y in (("qkv", first["x"], torch.cat([first["q"], first["k"], first["v"]], 1).flatten(1)), ("back", first["o"].flatten(1), first["y"]),
                       ("logits", first["y"][cu[1:].long() - 1], logits)):
        d.check_layer(name, x, y)
    # steps: eager, and the same step captured and replayed from the same states
    held_ids, held_uniform, held = new.long().clone(), uniform[1].clone(), d.states.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = d.tokens(held_ids, None, None)
        captured_logits, captured_new = d.choose(captured["y"], held_uniform)
    d.states.copy_(held)
    for step in range(steps):
        held_ids.copy_(new), held_uniform.copy_(uniform[step + 1])
        before = d.states.clone()
        one = d.tokens(new.long(), None, None)
        logits, new = d.choose(one["y"], uniform[step + 1])
        after = d.states.clone()
        d.states.copy_(before)
        graph.replay()
        assert torch.equal(captured["y"], one["y"]) and torch.equal(captured_logits, logits) and torch.equal(captured_new, new)
        assert torch.equal(d.states[d.slots.long()], after[d.slots.long()])
        d.check_layer("logits", one["y"], logits)
        history.append({k: v.clone() for k, v in one.items()})
        assert ((new >= 0) & (new < VOCAB)).all()
    assert d.states[[1, 4]].isnan().all()
    # every sequence's attention from its first token to its last, by the formula, on the queries, keys and values that the layers gave
    for b, n in enumerate(lengths):
        rows = slice(int(cu[b]), int(cu[b]) + n)
        q, k, v, o = (torch.cat([history[0][x][rows]] + [h[x][b:b + 1] for h in history[1:]]).double().transpose(0, 1) for x in "qkvo")
        k, v = k.repeat_interleave(HEADS // KV, 0), v.repeat_interleave(HEADS // KV, 0)
        t = torch.arange(n + steps, device="cuda").double()
        decay = torch.exp((t[:, None] - t).clamp(min=0) * d.log_decay.double()[:, None, None]).tril()
        form = lambda q, k, v: torch.bmm(torch.bmm(q, k.transpose(1, 2).contiguous()) * decay, v) * D ** -0.5  # noqa: E731
        want, size = form(q, k, v), form(q.abs(), k.abs(), v.abs())
        # 2^-14 of the terms' magnitudes (as tests/test_gpu_decay.py derives) and the result's rounding
        assert ((o - want).abs() <= 2.0 ** -14 * size + want.abs() * torch.finfo(dtype).eps / 2 + 2.0 ** -24).all()
