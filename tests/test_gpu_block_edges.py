"""Calls of the feed-forward blocks at the ends of what their sizes and arguments allow."""
import pytest
import torch

from paper_2305_02299_amd import StructuredLinear
from paper_2305_02299_amd import binding as B_

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_layer_without_outputs(dtype):
    """d_out of 0: there is no gradient to take in, dx is zero, and the bias's gradient has no element, wherever it is said to stand."""
    B, d_in = 5, 24
    x, W, dy = (torch.ones(s, device="cuda", dtype=dtype) for s in ((B, d_in), (1, d_in), (B, 1)))
    dx, dW, db = torch.full((B, d_in), 7.0, device="cuda", dtype=dtype), torch.full((1, d_in), 7.0, device="cuda", dtype=dtype), torch.full((4,), 7.0, device="cuda")
    ws = torch.empty(max(B_.srigl_structured_bwd_workspace_bytes(B, d_in, 0, 0, B_._dtype_code(x)), 16), dtype=torch.uint8, device="cuda")
    B_.srigl_structured_linear_bwd(dy, x, B, d_in, W, None, 0, db, None, 0, dx, dW, db, ws)
    assert not dx.any() and (dW == 7).all() and (db == 7).all()


@pytest.mark.parametrize("ablate", [0.0, 0.4, 1.0])
def test_dense_rows_of_their_own(ablate):
    """structured() takes the weights as they stand, and what becomes of its rows is nothing to the condensed layer."""
    import synth_inputs as si
    from gpu_util import dev
    from paper_2305_02299_amd import condense_layer
    L = si.make_layer(96, 40, 12, 80, ablate_frac=min(ablate, 0.4), seed=3)
    mask = L.mask * 0 if ablate == 1.0 else L.mask
    layer, x = condense_layer(dev(L.W), dev(mask), L.K, dev(L.bias)), dev(L.x)
    before = layer.dense_rows().clone()
    layer.W_c.mul_(2)
    rows = layer.structured()
    assert rows.Wd.shape == (layer.n_active, 96) and torch.equal(rows.Wd, 2 * before[:layer.n_active])
    rows.Wd.zero_()
    assert torch.equal(layer.dense_rows(), before) and torch.equal(layer.structured().Wd, 2 * before[:layer.n_active])
    assert layer.structured().forward(x).shape == (80, 40)


def test_a_result_in_the_memory_of_the_bias_or_the_list():
    """Refused before anything is launched: what is there stays."""
    room = torch.arange(200, device="cuda", dtype=torch.float32)
    bias, x, W = room[50:80], torch.ones(2, 8, device="cuda"), torch.ones(30, 8, device="cuda")
    for first in (0, 30, 79):
        with pytest.raises(ValueError):
            StructuredLinear(8, 30, W, None, bias).forward(x, y=room[first:first + 60].view(2, 30))
    assert torch.equal(room, torch.arange(200, device="cuda", dtype=torch.float32))
    y = room[80:140].view(2, 30)   # right behind it
    assert (StructuredLinear(8, 30, W, None, bias).forward(x, y=y) == 8 + bias).all()
    active = torch.arange(64, device="cuda", dtype=torch.int32)[:20]
    layer = StructuredLinear(8, 30, W[:20], active)
    with pytest.raises(ValueError):
        layer.forward(x[:1], y=_over(active, 30))
    assert active.tolist() == list(range(20))


def _over(t, n):
    """A float [1, n] that begins where t does"""
    return torch.empty(0, dtype=torch.float32, device="cuda").set_(t.view(torch.float32).untyped_storage(), 0, (1, n))
