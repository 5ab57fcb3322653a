"""Linear attention with a decay for each head (ftdecay_*) against its recurrence in 64 bits on the host, token after token.

Errors are counted relative to A, the result with all its terms taken by magnitude (scale * sum of decay^(t - j) |q| . |k_j| |v_j|, and the initial state's).
Products of two 16-bit elements are exact in 32 bits.  What is rounded before a product, weights q . k * decay and states, enters it as two words of bf16: off by at
most 2^-18, and the product of two lower words that is left out by as much: 2^-16 for both sides of a sum.  Powers of the decay, 2^(n x) with n x in 32 bits, are
off by |n x| 2^-24, below 2^-17 while they are not smaller than 2^-126; 32-bit sums of T terms, taken in pieces of up to 128 and then piece by piece, by
(128 + T / 64) 2^-24 at worst: 2^-16 for the lengths here.  In all 2^-14 A.  States enter no product in fewer bits than 32 (or three words): the powers and sums, 2^-15 A.
A result is then rounded to its type: half a step.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftdecay

pytestmark = pytest.mark.gpu

TYPES = {ftdecay.F16: torch.float16, ftdecay.BF16: torch.bfloat16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def stream():
    return torch.cuda.current_stream().cuda_stream


def recurrence(q, k, v, state, decay, scale):
    """q [token, heads, D], k, v [token, kv_heads, D], state [heads, D, D], decay [heads], all float64: (o, state)."""
    group = q.shape[1] // k.shape[1]
    o = torch.zeros_like(q)
    for t in range(q.shape[0]):
        kt, vt = k[t].repeat_interleave(group, 0), v[t].repeat_interleave(group, 0)
        state = decay[:, None, None] * state + kt[:, :, None] * vt[:, None, :]
        o[t] = scale * (q[t][:, :, None] * state).sum(1)
    return o, state


def bound(name, got, want, size, dtype=None):
    tol = 2.0 ** -15 * size if dtype is None else 2.0 ** -14 * size + float(torch.finfo(TYPES[dtype]).eps) / 2 * want.abs() + (2.0 ** -24 if dtype == ftdecay.F16 else 0)
    off = (got.double().cpu() - want).abs() - tol
    assert not got.isnan().any() and float(off.max() if off.numel() else 0) <= 0, (name, float(off.max()))


def decays(heads):
    return -np.log(2.0) / 2.0 ** torch.linspace(0, 12, heads, dtype=torch.float64)


class Case:
    def __init__(self, lengths, heads, kv_heads, d, dtype, starts=None, slots=None, n_slots=None, log_decay=None, scale=0.0, seed=0, behind=0):
        g = torch.Generator().manual_seed(seed + sum(lengths) + heads + d)
        self.lengths, self.heads, self.kv_heads, self.d, self.dtype = lengths, heads, kv_heads, d, dtype
        self.total, self.batch = sum(lengths) + behind, len(lengths)
        self.qkv = torch.randn((self.total, heads + 2 * kv_heads, d), generator=g).to(TYPES[dtype])
        self.log_decay = (decays(heads) if log_decay is None else log_decay).float()
        self.slots = slots
        self.states = torch.randn((n_slots or self.batch, heads, d, d), generator=g) * 3
        self.starts = starts
        self.scale = scale
        self.ctx = ftdecay.FtDecay(heads, kv_heads, d, dtype, scale)

    def split(self, qkv):
        h, hk = self.heads, self.kv_heads
        return qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]

    def want(self, magnitudes=False):
        q, k, v = (x.double() for x in self.split(self.qkv))
        states = self.states.double()
        if magnitudes:
            q, k, v, states = q.abs(), k.abs(), v.abs(), states.abs()
        decay = torch.exp(torch.nan_to_num(self.log_decay.double(), nan=0.0, neginf=-np.inf).clamp(max=0.0))
        out, new, at = torch.zeros((self.total, self.heads, self.d), dtype=torch.float64), states.clone(), 0
        for b, n in enumerate(self.lengths):
            slot = self.slots[b] if self.slots is not None else b
            there = 0 <= slot < states.shape[0]
            state = states[slot] if there and self.starts is not None and self.starts[b] > 0 else torch.zeros_like(states[0])
            out[at:at + n], state = recurrence(q[at:at + n], k[at:at + n], v[at:at + n], state, decay, self.scale if self.scale > 0 else self.d ** -0.5)
            if there:
                new[slot] = state
            at += n
        return out, new

    def run(self, strm=None):
        qkv = self.qkv.cuda()
        q, k, v = self.split(qkv)
        o = torch.full((self.total, self.heads, self.d), 55.0, dtype=TYPES[self.dtype], device="cuda")
        states = self.states.cuda()
        cu = ints(np.concatenate([[0], np.cumsum(self.lengths)]).tolist())
        self.ctx.forward(q, k, v, o, self.log_decay.cuda(), states, cu, None if self.starts is None else ints(self.starts),
                         None if self.slots is None else ints(self.slots), stream() if strm is None else strm)
        return o, states

    def check(self):
        o, states = self.run()
        (want, new), (size, state_size) = self.want(), self.want(True)
        n = sum(self.lengths)
        bound("o", o[:n], want[:n], size[:n], self.dtype)
        bound("states", states, new, state_size)
        assert (o[n:] == 55).all()
        return o, states


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths,heads,kv_heads", [([1], 1, 1), ([0, 2, 0], 2, 1), ([19], 8, 8), ([63, 64, 65], 3, 3), ([127, 1, 128, 129], 4, 2), ([31, 32, 33], 5, 1), ([300], 2, 2),
                                                    ([5, 0, 191, 192, 1, 193], 6, 2)])
def test_packed_prompts(lengths, heads, kv_heads, d, dtype):
    Case(lengths, heads, kv_heads, d, dtype).check()
    Case(lengths, heads, kv_heads, d, dtype, starts=[(i + 1) % 3 for i in range(len(lengths))], seed=1).check()


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("d,lengths,heads", [(64, [2100, 900], 2), (128, [1700], 1), (128, [1025, 0, 511, 513], 2), (64, [193, 385, 384, 191, 1537], 3)])
def test_long_prompts(d, lengths, heads, dtype):
    c = Case(lengths, heads, heads, d, dtype, starts=[1] * len(lengths))
    _, states = c.check()
    # on random operands roundings do not add up: three words and 32-bit sums stay within a few times 2^-24
    new = c.want()[1]
    assert float((states.double().cpu() - new).norm() / new.norm()) < 2e-6


def test_one_very_long_prompt():
    """Chunks of pieces of one sequence, joined: against the recurrence of its last tokens from the state that 64 bits give for those before."""
    n, d = 9001, 64
    c = Case([n], 1, 1, d, ftdecay.BF16, log_decay=torch.tensor([-1e-4], dtype=torch.float64))
    o, states = c.run()
    q, k, v = (x[:, 0].double() for x in c.split(c.qkv))
    decay = float(np.exp(np.float64(c.log_decay[0])))

    def state(q, k, v):
        return (k * (decay ** torch.arange(n - 1, -1, -1).double())[:, None]).T @ v
    bound("states", states[0, 0], state(q, k, v), state(q.abs(), k.abs(), v.abs()))
    for t in (0, 63, 64, 4095, 4096, 7777, n - 1):
        w = decay ** torch.arange(t, -1, -1).double()
        row = lambda q, k, v: d ** -0.5 * ((k[:t + 1] @ q[t]) * w) @ v[:t + 1]  # noqa: E731
        bound("o", o[t, 0], row(q, k, v), row(q.abs(), k.abs(), v.abs()), ftdecay.BF16)


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
def test_slots_and_rows_behind_the_last_sequence(dtype):
    """States anywhere in a pool; sequences without a state; slots that no sequence has stay as they were."""
    c = Case([70, 3, 0, 129, 20], 2, 2, 64, dtype, starts=[1, 0, 1, 7, -3], slots=[6, 2, 4, -1, 99], n_slots=8, behind=9)
    _, states = c.check()
    assert torch.equal(states[[0, 1, 3, 5, 7]].cpu(), c.states[[0, 1, 3, 5, 7]])


def test_an_empty_sequence_that_begins_leaves_zeros():
    c = Case([0, 0], 2, 2, 64, ftdecay.F16, starts=[0, 1])
    _, states = c.run()
    assert (states[0] == 0).all() and torch.equal(states[1].cpu(), c.states[1])


def test_without_states():
    c = Case([100, 30], 2, 1, 64, ftdecay.BF16)
    o, _ = c.run()
    alone = torch.empty_like(o)
    q, k, v = c.split(c.qkv.cuda())
    c.ctx.forward(q, k, v, alone, c.log_decay.cuda(), None, ints([0, 100, 130]), ints([5, 0]), stream=stream())
    assert torch.equal(o, alone)


@pytest.mark.parametrize("d", [64, 128])
def test_decays_at_the_ends(d):
    """No decay, a decay that leaves nothing, and what counts as one of them."""
    log_decay = torch.tensor([0.0, -np.inf, 3.0, np.nan, -1e-9, -200.0, -1e30, -5.0], dtype=torch.float64)
    c = Case([200, 1, 66], 8, 8, d, ftdecay.F16, starts=[1, 1, 0], log_decay=log_decay)
    c.check()
    o, _ = c.run()
    assert torch.equal(o[:, 2], o[:, 2]) and not o.isnan().any()


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("size", [1e-3, 60.0])
def test_small_and_large_operands(dtype, size):
    """Weights and states beyond the range of fp16, and far below 1.  (Results of fp16 beyond its largest number are infinite.)"""
    c = Case([150, 70], 2, 1, 64, dtype, starts=[1, 0], scale=1.0 if size < 1 else 1e-6)
    c.qkv = (c.qkv.float() * size).to(TYPES[dtype])
    c.check()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("d,at", [(64, 70), (128, 100), (64, 127), (128, 640)])
def test_what_later_tokens_hold_has_no_influence(bad, dtype, d, at):
    """Results of earlier tokens are the same bits, whatever the later ones' keys, values and queries are."""
    c = Case([at + 60, 40], 2, 2, d, dtype, starts=[1, 1])
    want, states = c.run()
    for part in range(3):
        c2 = Case([at + 60, 40], 2, 2, d, dtype, starts=[1, 1])
        c2.split(c2.qkv)[part][at + 1, 0, 3] = bad
        c2.split(c2.qkv)[part][at + 30, 1] = bad
        got, new = c2.run()
        assert torch.equal(got[:at + 1], want[:at + 1]) and torch.equal(got[at + 60:], want[at + 60:]) and torch.equal(new[1], states[1])
        assert torch.equal(got[:at + 30, 1], want[:at + 30, 1])
        if part == 0:
            assert got[at + 1, 0].isnan().any() or got[at + 1, 0].isinf().any()
            assert torch.equal(got[at + 2:at + 30], want[at + 2:at + 30]) and torch.equal(new, states)
        if part == 2:
            assert not got[at + 1:at + 60, 0, 3].isfinite().any() and not new[0, 0, :, 3].isfinite().any()
            assert torch.equal(got[:at + 60, 0, 4:], want[:at + 60, 0, 4:]) and torch.equal(new[0, 0, :, 4:], states[0, 0, :, 4:])


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 4, 64), (6, 2, 128), (1, 1, 128)])
@pytest.mark.parametrize("batch", [1, 3, 70])
def test_single_tokens(batch, heads, kv_heads, d, dtype):
    """Three steps of a batch, each against the recurrence."""
    c = Case([1] * batch, heads, kv_heads, d, dtype, starts=[1] * batch, slots=[(7 * b + 2) % (batch + 2) for b in range(batch)] if (batch + 2) % 7 else None, n_slots=batch + 2)
    states, slots = c.states.cuda(), None if c.slots is None else ints(c.slots)
    for step in range(3):
        want, new = c.want()
        size, state_size = c.want(True)
        q, k, v = c.split(c.qkv.cuda())
        o = torch.empty((batch, heads, d), dtype=TYPES[dtype], device="cuda")
        c.ctx.step(q, k, v, o, c.log_decay.cuda(), states, slots, stream())
        bound("o", o, want, size, dtype)
        bound("states", states, new, state_size)
        c.states = states.cpu()
        c.qkv = torch.randn(c.qkv.shape, generator=torch.Generator().manual_seed(step)).to(c.qkv.dtype)


def test_single_tokens_without_a_state():
    c = Case([1] * 4, 2, 2, 64, ftdecay.F16, starts=[1] * 4, slots=[3, -1, 5, 0], n_slots=5)
    want, new = c.want()
    size, state_size = c.want(True)
    q, k, v = c.split(c.qkv.cuda())
    o, states = torch.empty((4, 2, 64), dtype=torch.float16, device="cuda"), c.states.cuda()
    c.ctx.step(q, k, v, o, c.log_decay.cuda(), states, ints(c.slots), stream())
    bound("o", o, want, size, ftdecay.F16)
    bound("states", states, new, state_size)


@pytest.mark.parametrize("d", [64, 128])
def test_a_prompt_in_chunks_and_steps(d):
    """A prompt, then chunks of it, then single tokens: states carry over."""
    whole = Case([230], 2, 1, d, ftdecay.BF16)
    want, new = whole.want()
    size, state_size = whole.want(True)
    q, k, v = whole.split(whole.qkv.cuda())
    o, states, g = torch.empty((230, 2, d), dtype=torch.bfloat16, device="cuda"), whole.states.cuda(), whole.log_decay.cuda()
    at = 0
    for n in (90, 1, 64, 70):
        part = slice(at, at + n)
        whole.ctx.forward(q[part], k[part], v[part], o[part], g, states, ints([0, n]), ints([at]), stream=stream())
        at += n
    for t in range(at, 230):
        whole.ctx.step(q[t:t + 1], k[t:t + 1], v[t:t + 1], o[t:t + 1], g, states, stream=stream())
    bound("o", o, want, size, ftdecay.BF16)
    bound("states", states, new, state_size)


@pytest.mark.parametrize("lengths,d", [([150, 3], 64), ([700, 40], 128)])
def test_results_in_place_of_queries_and_twice_the_same(lengths, d):
    c = Case(lengths, 3, 1, d, ftdecay.F16, starts=[1, 1])
    want, states = c.run()
    again, states2 = c.run()
    assert torch.equal(want, again) and torch.equal(states, states2)
    qkv, new = c.qkv.cuda(), c.states.cuda()
    q, k, v = c.split(qkv)
    q = q.contiguous()
    c.ctx.forward(q, k, v, q, c.log_decay.cuda(), new, ints([0, lengths[0], sum(lengths)]), ints([1, 1]), stream=stream())
    assert torch.equal(q, want) and torch.equal(new, states)
    rows = qkv[:5].contiguous()
    q, k, v = c.split(rows)
    o, a, b = torch.empty((5, 3, d), dtype=torch.float16, device="cuda"), torch.ones((5, 3, d, d), device="cuda"), torch.ones((5, 3, d, d), device="cuda")
    c.ctx.step(q, k, v, o, c.log_decay.cuda(), a, stream=stream())
    c.ctx.step(q, k, v, q, c.log_decay.cuda(), b, stream=stream())
    assert torch.equal(q, o) and torch.equal(a, b)


def test_bounds_beyond_the_total():
    c = Case([50, 50], 2, 2, 64, ftdecay.F16)
    want, _ = c.run()
    q, k, v = c.split(c.qkv.cuda())
    o, states = torch.zeros((100, 2, 64), dtype=torch.float16, device="cuda"), c.states.cuda()
    c.ctx.forward(q, k, v, o, c.log_decay.cuda(), states, ints([0, 50, 2 ** 31 - 1]), stream=stream())
    assert torch.equal(o, want)
    c.ctx.forward(q, k, v, o, c.log_decay.cuda(), states, ints([-5, 50, 20]), stream=stream())
    assert torch.equal(o, want) and (states[1] == 0).all()


@pytest.mark.parametrize("lengths", [[70, 9], [1, 1], [1500, 300]])
def test_on_another_stream_and_in_a_graph(lengths):
    c = Case(lengths, 4, 2, 64, ftdecay.BF16, starts=[1, 1])
    want, new = c.run()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        got, states = c.run(other.cuda_stream)
    other.synchronize()
    assert torch.equal(got, want) and torch.equal(states, new)
    qkv, states, cu, starts, g = c.qkv.cuda(), c.states.cuda(), ints([0, lengths[0], sum(lengths)]), ints([1, 1]), c.log_decay.cuda()
    q, k, v = c.split(qkv)
    o = torch.empty((sum(lengths), 4, 64), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.ctx.forward(q, k, v, o, g, states, cu, starts, stream=stream())
        if lengths == [1, 1]:
            c.ctx.step(q, k, v, o, g, states, stream=stream())
    for seed in range(3):
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(seed)))
        states.copy_(c.states)
        graph.replay()
        got, kept = o.clone(), states.clone()
        states.copy_(c.states)
        c.ctx.forward(q, k, v, o, g, states, cu, starts, stream=stream())
        if lengths == [1, 1]:
            c.ctx.step(q, k, v, o, g, states, stream=stream())
        assert torch.equal(got, o) and torch.equal(kept, states)
