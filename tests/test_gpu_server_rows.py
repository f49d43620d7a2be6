"""Idle rows of a serving batch: a slot outside the pool means the same to a
prompt and to a step, and no other sequence sees it."""
import sys

import pytest
import torch

from paper_1906_11367_amd import boxconv as bc
from paper_1906_11367_amd.recurrent import RecurrentServer

pytestmark = pytest.mark.gpu

D, C, M, S = 32, 24, 40, 6


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def server(bias=True):
    s = RecurrentServer((rand(1, 2 * D, C) / 5).cuda(), (rand(2, M, D) / 5).cuda(), S,
                        b_in=rand(3, 2 * D).cuda(), b_out=rand(4, M).cuda() if bias else None)
    s.state.copy_(rand(5, S, D))
    return s


def slots(*v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


@pytest.mark.parametrize("layout", [bc.BC_TOKENS, bc.BC_MAPS])
@pytest.mark.parametrize("fresh", [True, False])
@pytest.mark.parametrize("lengths", [None, [9, 20, 0, 33, 5]])
def test_prompts_of_a_batch_with_idle_rows(layout, fresh, lengths):
    """Rows 1, 2 and 4 idle, below the pool and past it.  Every other row of the
    batch and of the pool is, bit for bit, that of the batch without them."""
    print("idle rows", layout, fresh, lengths, flush=True)
    sys.stdout.flush()
    N, T, live, idle = 5, 33, [0, 3], [1, 2, 4]
    x = rand(6, N, T, C).to(torch.bfloat16).cuda()
    x[idle] = float("nan")
    x = x if layout == bc.BC_TOKENS else x.transpose(1, 2).contiguous()
    ln = None if lengths is None else slots(*lengths)
    a, b = server(), server()
    before = a.state.clone()
    z = a.prefill(x, slots(4, -1, S, S - 1, 2 ** 30), ln, layout, fresh)
    want = b.prefill(x[live].contiguous(), slots(4, S - 1), None if ln is None else ln[live], layout, fresh)
    assert torch.equal(z[live], want)
    assert torch.equal(a.state[[4, S - 1]], b.state[[4, S - 1]])
    assert torch.equal(a.state[:4], before[:4])
    assert not torch.equal(a.state[S - 1], before[S - 1])
    # an idle row's z: that of a zero state, as a step's
    zi = z[idle] if layout == bc.BC_TOKENS else z[idle].transpose(1, 2)
    one = a.step(rand(7, 1, C).to(torch.bfloat16).cuda(), slots(-1))
    assert torch.equal(zi, one.expand_as(zi))
    # and the next batch's idle rows start from it again
    z = a.prefill(x, slots(S, 0, -5, S, S), ln, layout, fresh=False)
    assert torch.equal(z[0], z[2])


def test_an_idle_batch_and_wide_slots():
    s = server()
    before = s.state.clone()
    x = rand(8, 2, 7, C).to(torch.bfloat16).cuda()
    s.prefill(x, slots(-1, -1), fresh=False)
    s.prefill(x, slots(-2 ** 62, 2 ** 62, dtype=torch.int64))
    assert torch.equal(s.state, before)
    t = server()
    s.prefill(x, slots(5, 0, dtype=torch.int64))
    t.prefill(x, slots(5, 0))
    assert torch.equal(s.state, t.state)


def test_a_pool_that_is_set():
    """A pool put in place of the first (of another size too) is the one that
    prompts and steps read and write."""
    s, x = server(), rand(9, 1, 5, C).to(torch.bfloat16).cuda()
    saved = rand(10, S + 3, D).cuda()
    s.state = saved
    assert torch.equal(s.state, saved)
    s.prefill(x, slots(S + 2), fresh=False)
    s.step(x[:, 0].contiguous(), slots(S + 1))
    assert torch.equal(s.state[:S + 1], saved[:S + 1])
    assert not torch.equal(s.state[S + 1], saved[S + 1]) and not torch.equal(s.state[S + 2], saved[S + 2])


@pytest.mark.parametrize("bad", [dict(slots=slots_) for slots_ in ((0,), (0, 1, 2))] + [dict(lengths=(3,))])
def test_refusals(bad):
    s, x = server(), rand(11, 2, 7, C).to(torch.bfloat16).cuda()
    with pytest.raises(bc.BoxConvError, match="prefill: (slots|lengths)"):
        s.prefill(x, slots(*bad.get("slots", (0, 1))), None if "lengths" not in bad else slots(*bad["lengths"]))
