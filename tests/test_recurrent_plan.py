"""The type of x that a RecurrentPlan takes."""
import os

import pytest
import torch

from paper_1906_11367_amd import boxconv as bc
from paper_1906_11367_amd.recurrent import RecurrentPlan

pytestmark = pytest.mark.skipif(not os.path.exists(bc.LIB_PATH), reason="libboxconv.so not built")

f32, bf16 = torch.float32, torch.bfloat16
N, C, T, D, M = 2, 4, 6, 4, 5


@pytest.mark.parametrize("mix,x_dtype,takes,refuses", [
    ("f32", None, [f32], [bf16, torch.int32]), ("f32", f32, [f32], [bf16]), ("bf16", None, [f32, bf16], [torch.float64]),
    ("bf16", f32, [f32], [bf16]), ("bf16", bf16, [bf16], [f32])])
def test_the_plans_type_is_the_type_of_x(mix, x_dtype, takes, refuses):
    """On the CPU: an x of a type that is taken gets as far as the device check."""
    plan = RecurrentPlan(N, C, T, D, M, mix_dtype=mix, x_dtype=x_dtype, device="cpu")
    w_in, w_out, gz = torch.zeros(2 * D, C), torch.zeros(M, D), torch.zeros(N, M, T)
    for dt, says in [(d, "must be on the GPU") for d in takes] + [(d, "x has dtype") for d in refuses]:
        x = torch.zeros((N, C, T), dtype=dt)
        with pytest.raises(bc.BoxConvError, match=says):
            plan.forward(x, w_in, w_out)
        with pytest.raises(bc.BoxConvError, match=says):
            plan.backward(x, w_in, w_out, gz)


@pytest.mark.parametrize("mix,x_dtype", [("f32", bf16), ("bf16", torch.float64), ("bf16", torch.int32)])
def test_types_no_mix_takes(mix, x_dtype):
    with pytest.raises(ValueError, match="x must be"):
        RecurrentPlan(N, C, T, D, M, mix_dtype=mix, x_dtype=x_dtype, device="cpu")


@pytest.mark.gpu
def test_bf16_x_trains_as_its_values_in_fp32():
    """A bf16 mix rounds x to the same bits; its sums may run in another order, by
    which a value here and there may round to the neighbouring bf16, 2^-8 away."""
    N, C, T, D, M = 2, 40, 200, 24, 16
    rand = lambda seed, *shape: torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()
    x = rand(1, N, C, T).to(bf16)
    w_in, w_out, gz = rand(2, 2 * D, C) / C ** 0.5, rand(3, M, D) / D ** 0.5, rand(4, N, M, T)
    results = []
    for dt in (bf16, f32):
        plan = RecurrentPlan(N, C, T, D, M, mix_dtype="bf16", x_dtype=dt)
        results.append([*plan.forward(x.to(dt), w_in, w_out), *plan.backward(x.to(dt), w_in, w_out, gz)])
    for name, a, b in zip("z h_last dx dw_in dw_out dh0".split(), *results):
        assert torch.isfinite(a).all() and b.norm() > 0, name
        assert (a - b).norm() <= 2.0 ** -8 * b.norm(), name
