"""Calls of the feed-forward blocks at the ends of what their sizes and arguments allow."""
import pytest
import torch

from paper_2305_02299_amd import GatedLinear, StructuredLinear
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


# ---- more workgroups than one dimension of a grid holds (2^32 threads) ----
def _same_everywhere(got, want, rows=1 << 25):
    """got [n, ...] against want(first, behind), in pieces"""
    return all(torch.equal(got[k:k + rows], want(k, min(k + rows, got.shape[0]))) for k in range(0, got.shape[0], rows))


@pytest.mark.parametrize("gated", [False, True])
def test_neurons_by_the_hundred_million(gated):
    n, d_in = (1 << 28) + 37, 8
    W = torch.empty(n, d_in, device="cuda", dtype=torch.bfloat16).random_(-2, 3)
    x = torch.tensor([[1, 2, 0, -1, 3, 1, -2, 1], [0, 1, 1, 2, -1, 0, 1, 3]], device="cuda", dtype=torch.bfloat16)
    want = lambda a, b: (W[a:b].float() @ x.float().T).bfloat16()  # noqa: E731  (whole numbers: exact)
    if not gated:
        y = StructuredLinear(d_in, n, W).forward(x)
        for r in range(2):
            assert _same_everywhere(y[r], lambda a, b: want(a, b)[:, r])
        return
    h, g, u = GatedLinear(d_in, n, W, W, act=B_.ACT_NONE).forward(x, save=True)
    for r in range(2):
        assert _same_everywhere(g[r], lambda a, b: want(a, b)[:, r]) and torch.equal(g[r], u[r])
        assert _same_everywhere(h[r], lambda a, b: want(a, b)[:, r] * want(a, b)[:, r])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_by_the_thousand_million(dtype):
    """2^30 rows, the most that a call takes, of one neuron."""
    B, d_in = 1 << 30, 8
    x = torch.empty(B, d_in, device="cuda", dtype=dtype).random_(-2, 3)
    W = torch.tensor([[1, -2, 0, 1, 3, 1, -2, 2]], device="cuda", dtype=dtype)
    y = StructuredLinear(d_in, 1, W).forward(x)
    assert _same_everywhere(y, lambda a, b: (x[a:b].float() @ W.float().T).to(dtype))


def test_bias_sums_of_the_most_neurons():
    n, d_in = 1 << 29, 1
    dh, g, u = (torch.empty(1, n, device="cuda", dtype=torch.bfloat16).random_(-3, 4) for _ in range(3))
    x, W = torch.ones(1, d_in, device="cuda", dtype=torch.bfloat16), torch.empty(1, 1, device="cuda", dtype=torch.bfloat16)
    dbg, dbu = (torch.full((n,), 77.0, device="cuda") for _ in range(2))
    ws = torch.empty(B_.srigl_gated_bwd_workspace_bytes(1, d_in, n, B_.BF16), dtype=torch.uint8, device="cuda")
    B_.srigl_gated_linear_bwd(dh, x, 1, d_in, W, W, n, g, u, None, None, None, dbg, dbu, ws, B_.ACT_NONE)
    assert torch.equal(dbg, (dh * u)[0].float()) and torch.equal(dbu, (dh * g)[0].float())


# ---- neighbours ablated together ----
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,d_in", [(1, 72), (16, 200), (17, 72), (64, 136), (40, 2056), (300, 4096)])
@pytest.mark.parametrize("kind", ["first", "last", "one in the middle", "both ends", "blocks", "every 300th", "all but one"])
def test_runs_of_ablated_neurons(kind, B, d_in, out):
    """Every column of every row, from runs of any length, with a residual in place and without: whole numbers, exact."""
    d_out = 9001
    gen = torch.Generator().manual_seed(B)
    stored = {"first": torch.arange(33), "last": torch.arange(d_out - 5, d_out), "one in the middle": torch.tensor([4500]), "both ends": torch.tensor([0, d_out - 1]),
              "blocks": torch.cat([torch.arange(256, 512), torch.arange(1024, 1040), torch.arange(8960, 8992)]), "every 300th": torch.arange(7, d_out, 300),
              "all but one": torch.cat([torch.arange(2000), torch.arange(2001, d_out)])}[kind]
    W, x, bias, residual = (torch.randint(-2, 3, s, generator=gen).float() for s in ((len(stored), d_in), (B, d_in), (d_out,), (B, d_out)))
    t = torch.bfloat16
    layer = StructuredLinear(d_in, d_out, W.to(t).cuda(), stored.int().cuda(), bias.cuda())
    want = bias.expand(B, d_out).clone()
    want[:, stored] += x @ W.T
    want = want.clamp(min=0)
    assert torch.equal(layer.forward(x.to(t).cuda(), act=B_.ACT_RELU, out_dtype=out).cpu(), want.to(out))
    y = residual.to(out).cuda()
    got, z = layer.forward(x.to(t).cuda(), act=B_.ACT_RELU, residual=y, y=y, save=True)
    assert torch.equal(y.cpu(), (want + residual).to(out)) and torch.equal(z.cpu(), (x @ W.T + bias[stored]).to(t))


@pytest.mark.parametrize("B,d_in", [(1, 64), (16, 64), (40, 4096)])
def test_a_run_of_millions_is_shared_out(B, d_in):
    """One neuron of 4 million: a tenth of a second is two hundred times what the columns take and a fifth of what one thread took for a row's."""
    d_out = (1 << 22) + 5
    bias = torch.empty(d_out, device="cuda").random_(-3, 4)
    layer = StructuredLinear(d_in, d_out, torch.ones(1, d_in, device="cuda", dtype=torch.bfloat16), torch.tensor([d_out // 3], device="cuda", dtype=torch.int32), bias)
    x = torch.ones(B, d_in, device="cuda", dtype=torch.bfloat16)
    y = layer.forward(x, act=B_.ACT_RELU)
    want = bias.clone()
    want[d_out // 3] += d_in
    assert torch.equal(y, want.clamp(min=0).bfloat16().expand(B, d_out))
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    layer.forward(x, act=B_.ACT_RELU)
    end.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(end) < 100
