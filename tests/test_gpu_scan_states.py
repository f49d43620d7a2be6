"""The states that the forward of the gated scan keeps for its backward."""
import os

import pytest
import torch

from paper_1906_11367_amd import boxconv as bc


@pytest.mark.skipif(not os.path.exists(bc.LIB_PATH), reason="libboxconv.so not built")
def test_room_for_a_state_every_128_steps():
    n = bc.load_library().bc_gated_scan_states_bytes
    for N, T, C in ((1, 1, 1), (2, 128, 9), (3, 129, 64), (8, 4096, 2048), (1, 1 << 30, 5)):
        assert n(N, T, C, bc.BC_TOKENS) == 4 * N * C * ((T + 127) // 128)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [257, 700, 2049])
def test_every_kept_state_is_read(T, dtype):
    """A NaN in the state before steps [128 i, 128 (i + 1)) of channel c reaches
    those steps' coefficient gradients (delta_t h_{t-1}), and nothing else."""
    N, C, c = 2, 70, 33
    g = torch.Generator().manual_seed(T)
    gate, x, gy = (torch.rand((N, T, C), generator=g).add(0.1).to(dtype).cuda() for _ in range(3))
    y, want_gate, want_x, gg, gx = (torch.empty_like(x) for _ in range(5))
    states = bc.gated_scan_states(N, T, C, dtype)
    spans = (T + 127) // 128
    assert states.numel() == N * spans * C
    bc.gated_scan_fwd(gate, x, y, states=states, form=bc.BC_GATE_VALUE)
    bc.gated_scan_bwd(gate, x, states, gy, want_gate, want_x, form=bc.BC_GATE_VALUE)
    for i in range(spans):
        bad = states.clone()
        bad.view(N, spans, C)[1, i, c] = float("nan")
        bc.gated_scan_bwd(gate, x, bad, gy, gg, gx, form=bc.BC_GATE_VALUE)
        hit = torch.zeros((N, T, C), dtype=torch.bool, device="cuda")
        hit[1, 128 * i:128 * (i + 1), c] = True
        assert torch.isnan(gg[hit]).all() and torch.equal(gg[~hit], want_gate[~hit]) and torch.equal(gx, want_x), i
