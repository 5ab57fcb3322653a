"""Linear attention with a decay where values are small: near fp16's least numbers, decayed far within a chunk of 64 tokens, or beside larger ones.

A state is a number of 32 bits, so that its error is counted relative to its own terms, as test_gpu_decay.py derives it (2^-15 of them), however small they are.  Values decayed to the
end of a chunk are two words in fp16, of values lifted by 2^e, e = 15 where a slab's largest is below 2, one less for each octave above.  The upper word leaves at most 2^-12 of the lifted value, the
lower one, of 2^11 times that, at most 2^-12 of it again, or half of fp16's least number, 2^-25: 2^-24 of the value, or 2^-(36 + e).  So 2^-15 of a term holds where it is above
2^-(21 + e); where a test goes below, what the words leave is added to its bound.
"""
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftdecay
from test_gpu_decay import TYPES, Case, bound, ints, stream
from test_gpu_decay_many import recurrence

pytestmark = pytest.mark.gpu


def check(values, log_decay, dtype, first=None, lengths=None, outputs=True, left=None):
    """values: [total, heads, D]; queries and keys are random.  left: what a value of each token may be off by in the last state, [total, heads]."""
    g = torch.Generator().manual_seed(3)
    total, heads, d = values.shape
    lengths = lengths or [total]
    qkv = torch.cat([torch.randn((total, 2 * heads, d), generator=g).to(TYPES[dtype]), values.to(TYPES[dtype])], 1).cuda()
    q, k, v = qkv[:, :heads], qkv[:, heads:2 * heads], qkv[:, 2 * heads:]
    states = torch.zeros((len(lengths), heads, d, d)) if first is None else first
    begin, o = states.cuda(), torch.empty((total, heads, d), dtype=TYPES[dtype], device="cuda")
    states, cu, decay = begin.clone(), torch.tensor([0] + lengths).cumsum(0), torch.tensor(log_decay).float().cuda()
    ctx = ftdecay.FtDecay(heads, heads, d, dtype)
    ctx.forward(q, k, v, o, decay, states, ints(cu.tolist()), ints([1] * len(lengths)), stream=stream())
    want, new = recurrence(qkv.double(), heads, heads, cu.cuda(), begin.double(), torch.exp(decay.double()), d ** -0.5)
    size, state_size = recurrence(qkv.double().abs(), heads, heads, cu.cuda(), begin.double().abs(), torch.exp(decay.double()), d ** -0.5)
    if left is not None:
        state_size += 2.0 ** 15 * (k.double().abs() * left.cuda()[..., None]).sum(0)[None, :, :, None]
    bound("states", states, new.cpu(), state_size.cpu())
    if outputs:
        bound("o", o, want.cpu(), size.cpu(), dtype)
    return states


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", [[2, 3, 64], [193, 65, 400]])
@pytest.mark.parametrize("size", [2.0 ** -24, 2.0 ** -21, 2.0 ** -17, 2.0 ** -12])
def test_values_near_the_least_numbers(size, lengths, d, dtype):
    g = torch.Generator().manual_seed(d)
    values = torch.randint(-3, 4, (sum(lengths), 3, d), generator=g) * size
    check(values, [-0.7, -0.03, -0.001], dtype, lengths=lengths)


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens", [30, 64, 100])
def test_values_that_are_remembered_faintly(tokens, d, dtype):
    """Two tokens with values, then none: the state is what their decay leaves, 2^-16 and 2^-31 of them within a chunk."""
    g = torch.Generator().manual_seed(d + tokens)
    values = torch.zeros((tokens, 2, d))
    values[:2] = torch.randn((2, 2, d), generator=g)
    assert values.abs().max() < 8
    half, left = 0.69314718056 / (min(tokens, 64) - 1), torch.zeros((tokens, 2), dtype=torch.float64)
    # values below 8 are lifted by 2^13 at least; what the words leave decays with the chunk behind them
    left[:2] = 2.0 ** -(36 + 13) * torch.exp(-half * torch.tensor([16.0, 31.0]).double() * max(0, tokens - 64)) * (dtype == ftdecay.F16)
    check(values, [-16 * half, -31 * half], dtype, left=left)


@pytest.mark.parametrize("d", [64, 128])
def test_small_columns_beside_larger_ones(d):
    """Values of up to 4000 (lifted by 2^4) among those of 2^-14: the words leave 2^-40, below 2^-15 of terms above 2^-25.  (Sums of 150 of these have terms of 2^-14.)"""
    g = torch.Generator().manual_seed(d)
    values = torch.randn((150, 2, d), generator=g) * 2.0 ** -14
    values[:, :, 5] = 4000 * torch.randn((150, 2), generator=g).clamp(-1, 1)
    check(values, [-0.05, -0.001], ftdecay.F16, outputs=False)


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("d", [64, 128])
def test_states_with_no_room_above(d, dtype):
    """States up to near the largest number, with small values: nothing is lifted beyond it."""
    g = torch.Generator().manual_seed(d)
    values = torch.randn((130, 2, d), generator=g) * 2.0 ** -20
    first = (torch.rand((2, 2, d, d), generator=g) - 0.5) * 2.0 ** torch.tensor([127.0, 104.0])[:, None, None, None]
    states = check(values, [-0.01, -0.3], dtype, first=first, lengths=[70, 60], outputs=False)
    assert states.isfinite().all()


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("d", [64, 128])
def test_what_counts_as_no_decay(d, dtype):
    """A log_decay above 0, or NaN, gives the results and states of 0, bit for bit: prompts, divided ones among them, and single tokens."""
    lengths, odd = [200, 1, 66, 300], [3.0, float("nan"), float("inf"), 1e-30, -0.1]
    runs = []
    for log_decay in (odd, [0.0, 0.0, 0.0, 0.0, -0.1]):
        c = Case(lengths, 5, 5, d, dtype, starts=[1, 1, 0, 1], log_decay=torch.tensor(log_decay, dtype=torch.float64))
        o, states = c.run()
        q, k, v = c.split(c.qkv[:4].cuda())
        one = torch.empty((4, 5, d), dtype=TYPES[dtype], device="cuda")
        c.ctx.step(q, k, v, one, c.log_decay.cuda(), states, stream=stream())
        runs.append((o, states, one))
    assert all(torch.equal(x, y) and not x.isnan().any() for x, y in zip(*runs))
