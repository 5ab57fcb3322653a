"""Linear attention with a decay over more workgroups than the chip holds at a time (ftdecay_forward): continued prompts that are divided into segments.

Which segments run together is not known, and a segment may begin when the last one of its sequence has stored its state long ago.  Against the recurrence in 64 bits,
for all sequences at once on the GPU, with the tolerances that test_gpu_decay.py derives.
"""
import pytest

torch = pytest.importorskip("torch")

from paper_2504_02211_amd import ftdecay
from test_gpu_decay import TYPES, bound, decays, ints, stream

pytestmark = pytest.mark.gpu


def recurrence(qkv, heads, kv_heads, cu, states, decay, scale):
    """Packed rows [total, heads + 2 kv_heads, D], states [batch, heads, D, D], all float64: (o, states)."""
    d, group = qkv.shape[2], heads // kv_heads
    n, states, o = cu[1:] - cu[:-1], states.clone(), torch.zeros((qkv.shape[0], heads, qkv.shape[2]), dtype=torch.float64, device="cuda")
    for t in range(int(n.max())):
        on = (n > t).nonzero()[:, 0]
        rows = qkv[cu[on] + t]
        q, k, v = rows[:, :heads], rows[:, heads:heads + kv_heads].repeat_interleave(group, 1), rows[:, heads + kv_heads:].repeat_interleave(group, 1)
        new = states[on] * decay[:, None, None] + k[..., :, None] * v[..., None, :]
        o[cu[on] + t] = scale * (q[..., :, None] * new).sum(2)
        states[on] = new
    assert d == states.shape[2]
    return o, states


def check(lengths, heads, kv_heads, d, dtype, starts, seed):
    g = torch.Generator().manual_seed(seed)
    batch, total = len(lengths), sum(lengths)
    qkv = torch.randn((total, heads + 2 * kv_heads, d), generator=g).to(TYPES[dtype]).cuda()
    slots = torch.randperm(batch + 2, generator=g)[:batch]
    first = (torch.randn((batch + 2, heads, d, d), generator=g) * 3).cuda()
    log_decay = decays(heads).float().cuda()
    cu = torch.tensor([0] + lengths).cumsum(0)
    states, o = first.clone(), torch.full((total, heads, d), 55.0, dtype=TYPES[dtype], device="cuda")
    ctx = ftdecay.FtDecay(heads, kv_heads, d, dtype)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    ctx.forward(q, k, v, o, log_decay, states, ints(cu.tolist()), ints(starts), ints(slots.tolist()), stream())
    cu, slots = cu.cuda(), slots.cuda()
    begin = torch.where(torch.tensor(starts, device="cuda")[:, None, None, None] > 0, first[slots], 0.0).double()
    decay = torch.exp(log_decay.double())
    want, new = recurrence(qkv.double(), heads, kv_heads, cu, begin, decay, d ** -0.5)
    size, state_size = recurrence(qkv.double().abs(), heads, kv_heads, cu, begin.abs(), decay, d ** -0.5)
    bound("o", o, want.cpu(), size.cpu(), dtype)
    bound("states", states[slots], new.cpu(), state_size.cpu())
    free = [x for x in range(batch + 2) if x not in slots.tolist()]
    assert torch.equal(states[free], first[free])
    # whatever runs together, the same bits
    again, o2 = first.clone(), torch.empty_like(o)
    ctx.forward(q, k, v, o2, log_decay, again, ints(cu.tolist()), ints(starts), ints(slots.tolist()), stream())
    assert torch.equal(o, o2) and torch.equal(states, again)


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (2, 2), (3, 3), (6, 3), (8, 1)])
def test_continued_prompts_of_a_segment_and_a_token(heads, kv_heads, d, dtype):
    """Segments of 192 tokens, and as many of one token: 960 workgroups and more."""
    check([193] * (480 // heads), heads, kv_heads, d, dtype, [1] * (480 // heads), heads + d)


@pytest.mark.parametrize("dtype", [ftdecay.F16, ftdecay.BF16])
@pytest.mark.parametrize("heads,kv_heads,d", [(8, 8, 64), (4, 4, 128), (6, 2, 64)])
def test_continued_prompts_among_empty_ones(heads, kv_heads, d, dtype):
    """Some prompts are divided, hundreds have a token or none, some begin."""
    g = torch.Generator().manual_seed(heads)
    divided, others = 480 // heads, 2400 // heads
    lengths = torch.tensor([193] * (divided // 2) + [200, 385] * (divided // 8) + [0, 1] * (others // 2))
    lengths = lengths[torch.randperm(len(lengths), generator=g)].tolist()
    check(lengths, heads, kv_heads, d, dtype, [(i % 4 > 0) * (i + 1) for i in range(len(lengths))], heads + d)
