"""The gates' coefficients alone: of a sequence of one step, the last state is 1 - a
where x = 1 and h0 = 0, and a where x = 0 and h0 = 1, with no rounding of its own.

Bar (units of 2^-24 of the value): the exponential 2 (an ulp) and its correction 1,
the sum 1, the reciprocal 2 (an ulp), the product 1: 7, and 8 with what is of
second order.  bf16 storage does without the correction: the rounding of
|gate| / ln 2 (half an ulp of at most 1.4427 |gate|, times ln 2: |gate| units) and
of the constant 1 / ln 2 (1.33e-8 |gate|: 0.23 |gate| units) come on top."""
import numpy as np
import pytest
import torch

from paper_1906_11367_amd import boxconv as bc

UNIT = 2.0 ** -24
GATES = np.concatenate([s * np.concatenate([np.linspace(0.0, 85.0, 4001), np.logspace(-8, 0, 95)]) for s in (1, -1)])


def bar(gate, dtype):
    return (8.0 + (1.25 * np.abs(gate) if dtype == torch.bfloat16 else 0.0)) * UNIT


def exact(gate):
    """a and 1 - a."""
    return 1.0 / (1.0 + np.exp(-gate)), 1.0 / (1.0 + np.exp(gate))


def test_the_bar_tells_a_corrected_exponential_from_another():
    """1 - a in 32 bits from an exponential whose argument is a rounded product,
    everything else exact: past the bar for fp32, within that for bf16."""
    gate = np.float32(GATES[GATES > 40]).astype(np.float64)
    t = (np.float32(gate) * np.float32(-1.44269504)).astype(np.float32).astype(np.float64)
    off = np.abs(np.exp2(t) / (1 + np.exp2(t)) / exact(gate)[1] - 1.0)
    assert (off > 3 * bar(gate, torch.float32)).any()
    assert (off <= bar(gate, torch.bfloat16)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("how", ["tokens", "maps", "step"])
def test_coefficients(how, dtype):
    gate = torch.from_numpy(GATES).to(dtype).cuda()
    C = gate.numel()
    g64 = gate.double().cpu().numpy()
    for x0, h0, want in ((0.0, 1.0, exact(g64)[0]), (1.0, 0.0, exact(g64)[1])):
        shape = (1, 1, C) if how == "tokens" else (1, C, 1) if how == "maps" else (1, C)
        x, y = torch.full(shape, x0, dtype=dtype, device="cuda"), torch.empty(shape, dtype=dtype, device="cuda")
        h = torch.full((1, C), h0, device="cuda")
        if how == "step":
            bc.gated_scan_step(gate.view(shape), x, h, y)
        else:
            bc.gated_scan_fwd(gate.view(shape), x, y, h0=h, h_last=h, layout=bc.BC_TOKENS if how == "tokens" else bc.BC_MAPS)
        off = np.abs(h[0].double().cpu().numpy() / want - 1.0)
        worst = np.argmax(off - bar(g64, dtype))
        print(how, dtype, "units", (off / UNIT).max(), flush=True)
        assert (off <= bar(g64, dtype)).all(), (g64[worst], off[worst] / UNIT)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_coefficients_below_the_normal_range(dtype):
    """Where a or 1 - a is below 2^-126 it may be zero, and is never more than that off."""
    gate = torch.tensor([86.0, 88.0, 90.0, 100.0, 104.0, 120.0, 200.0, 3e38, float("inf")], device="cuda").to(dtype)
    for s in (1, -1):
        g = s * gate
        h = torch.zeros((1, len(gate)), device="cuda")
        bc.gated_scan_step(g[None], torch.ones_like(g)[None], h, torch.empty_like(g)[None])
        with np.errstate(over="ignore"):
            want = exact(g.double().cpu().numpy())[1]
        assert (np.abs(h[0].double().cpu().numpy() - want) <= 2.0 ** -126 + bar(200.0, dtype) * want).all()
