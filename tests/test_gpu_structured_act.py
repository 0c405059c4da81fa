"""The structured-only layer with bias, activation and residual, and its gradients, against the operators in 64 bits."""
import pytest
import torch

from block_util import (ACTS, TYPES, at_offset, evaluation, half_step, linear, normal, places, products_bound, rounded, slope, sum_gate, untouched, value, whole, within)
from paper_2305_02299_amd import SriglError, StructuredLinear
from paper_2305_02299_amd import binding as B_

pytestmark = pytest.mark.gpu

# (batch, d_in, d_out): one of everything, whole tiles, a little more and less than tiles and stages, rows that begin anywhere, long sums, few and many rows
SIZES = [(1, 1, 1), (1, 8, 3), (2, 64, 64), (3, 65, 66), (1, 768, 1000), (4, 4096, 130), (7, 300, 513), (16, 72, 257), (37, 1001, 777), (64, 128, 128), (65, 136, 129),
         (130, 520, 260), (200, 33, 40), (257, 264, 390), (300, 1024, 520), (33, 2056, 96)]
# (large enough for the largest tiles in one of the three products each, whole stages of K and not)
LARGE = [(1500, 264, 9000), (1100, 8200, 264), (200, 4104, 5000), (2048, 256, 8192), (1024, 8192, 256)]


def _layer(gen, d_in, d_out, ablated, t, make, biased=True):
    active, stored = places(gen, d_out, ablated)
    W, bias = make((len(stored), d_in), t), make((d_out,), torch.float32) if biased else None
    return W, bias, active, stored


def _cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


@pytest.mark.parametrize("ablated", [0.0, 0.3, 0.97])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES + LARGE)
def test_whole_numbers_come_out_exactly(size, dtype, ablated):
    """Sums of small whole numbers are exact in fp32 in any order: every bit of the result and of the gradients is known."""
    B, d_in, d_out = size
    gen, t = torch.Generator().manual_seed(B + 7 * d_in + 31 * d_out), TYPES[dtype]
    make = lambda shape, tt: whole(gen, shape, 2, tt)  # noqa: E731
    W, bias, active, stored = _layer(gen, d_in, d_out, ablated, t, make)
    x = make((B, d_in), t)
    layer = StructuredLinear(d_in, d_out, *_cuda(W, active, bias))
    for out in {t, torch.float32}:
        residual = make((B, d_out), out)
        want, _, z, _ = linear(x, W, stored, bias, d_out, "relu", residual)
        y, got_z = layer.forward(x.cuda(), act=B_.ACT_RELU, residual=residual.cuda(), out_dtype=out, save=True)
        assert y.dtype == out and torch.equal(y.cpu(), want.to(out)) and torch.equal(got_z.cpu(), z.to(t))
        dy = make((B, d_out), out)
        dz = dy.double()[:, stored] * (got_z.cpu() > 0)
        dbias = dy.double().sum(0) * (bias > 0)
        dbias[stored] = dz.sum(0)
        dx, dWd, db = layer.backward(dy.cuda(), x.cuda(), got_z, act=B_.ACT_RELU)
        assert torch.equal(dx.cpu(), (dz @ W.double()).to(t)) and torch.equal(dWd.cpu(), (dz.T @ x.double()).to(t))
        assert torch.equal(db.cpu(), dbias.float())


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("size,ablated", [((1, 768, 257), 0.0), ((5, 200, 90), 0.5), ((37, 1001, 777), 0.1), ((130, 520, 260), 0.0), ((300, 1024, 520), 0.2)])
def test_activations_against_64_bits(size, ablated, dtype, out, act):
    B, d_in, d_out = size
    gen, t, o = torch.Generator().manual_seed(B + d_in), TYPES[dtype], TYPES[out]
    make = lambda shape, tt: normal(gen, shape, 1.0 if len(shape) == 1 else d_in ** -0.5, tt)  # noqa: E731
    W, bias, active, stored = _layer(gen, d_in, d_out, ablated, t, make)
    x, residual = normal(gen, (B, d_in), 2.0, t), normal(gen, (B, d_out), 1.0, o)
    layer = StructuredLinear(d_in, d_out, *_cuda(W, active, bias))
    want, off, z, z_off = linear(x, W, stored, bias, d_out, act, residual)
    y, got_z = layer.forward(x.cuda(), act=ACTS[act], residual=residual.cuda(), out_dtype=o, save=True)
    within(y, want, rounded(want, off, o), "y")
    within(got_z, z, rounded(z, z_off, t), "z")
    # gradients, of the pre-activations as they were saved
    dy, zs = normal(gen, (B, d_out), 0.1, o), got_z.cpu().double()
    dz = dy.double()[:, stored] * slope(zs, act)
    dz_off = dy.double()[:, stored].abs() * evaluation(zs) + 2.0 ** -24 * dz.abs()
    dx, dWd, db = layer.backward(dy.cuda(), x.cuda(), got_z if act != "none" else None, act=ACTS[act])
    want = dz @ W.double()
    within(dx, want, rounded(want, products_bound(dz, dz_off, W, t, len(stored)), t), "dx")
    want = dz.T @ x.double()
    within(dWd, want, rounded(want, products_bound(dz.T, dz_off.T, x, t, B), t), "dWd")
    want = dy.double().sum(0) * slope(bias.double(), act)
    bound = sum_gate(B) * dy.double().abs().sum(0) * 1.13 + dy.double().abs().sum(0) * evaluation(bias.double())
    want[stored], bound[stored] = dz.sum(0), sum_gate(B) * dz.abs().sum(0) + dz_off.sum(0)
    within(db, want, bound + 2.0 ** -24 * want.abs(), "dbias")


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_gradients_against_differences(act):
    """Central differences of the forward formula in 64 bits: the slope of a weighted sum of y along random directions of x, Wd and the bias."""
    gen = torch.Generator().manual_seed(5)
    B, d_in, d_out = 9, 40, 24
    active, stored = places(gen, d_out, 0.25)
    W, bias, x, dy = (normal(gen, s) for s in ((len(stored), d_in), (d_out,), (B, d_in), (B, d_out)))
    layer = StructuredLinear(d_in, d_out, *_cuda(W, active, bias))
    _, z = layer.forward(x.cuda(), act=ACTS[act], save=True)
    grads = [g.cpu().double() for g in layer.backward(dy.cuda(), x.cuda(), z, act=ACTS[act])]

    def loss(x, W, bias):
        every = bias.expand(B, d_out).clone()
        every[:, stored] = x @ W.T + bias[stored]
        return (value(every, act) * dy.double()).sum()

    at = [v.double() for v in (x, W, bias)]
    for k in range(3):
        for _ in range(4):
            step = torch.randn(at[k].shape, generator=gen, dtype=torch.float64) * 1e-6
            up, down = (loss(*[v + sign * step if i == k else v for i, v in enumerate(at)]) for sign in (1, -1))
            # 1e-9: the square of the step times the third derivative, and 2^-53 of a sum of a few hundred; 1e-5 of the sizes: fp32 sums
            assert abs((up - down) / 2 - (grads[k] * step).sum()) <= 1e-9 + 1e-5 * (grads[k].abs() * step.abs()).sum()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_any_address_and_nothing_beside_it(dtype, shift):
    """Operands and results that begin at any element: the same values, and not an element in front of or behind the results is written."""
    gen, t = torch.Generator().manual_seed(shift), TYPES[dtype]
    B, d_in, d_out = 70, 136, 200
    make = lambda shape, tt: whole(gen, shape, 2, tt)  # noqa: E731
    W, bias, active, stored = _layer(gen, d_in, d_out, 0.2, t, make)
    n = len(stored)
    x, dy, residual = (make(s, t) for s in ((B, d_in), (B, d_out), (B, d_out)))
    put = lambda v: at_offset(v, shift)[0]  # noqa: E731
    (y, y_room), (z, z_room), (dx, dx_room), (dW, dW_room), (db, db_room) = (at_offset(torch.zeros(s, dtype=tt), shift) for s, tt in (
        ((B, d_out), t), ((B, n), t), ((B, d_in), t), ((n, d_in), t), ((d_out,), torch.float32)))
    code = B_.F32 if dtype == "f32" else B_.BF16
    ws = torch.empty(B_.srigl_structured_act_workspace_bytes(B, d_in, n, code), dtype=torch.uint8, device="cuda")
    xs, Ws, bs, acts = put(x), put(W), put(bias), put(active)
    B_.srigl_structured_linear_fwd_act(xs, B, d_in, Ws, acts, n, bs, put(residual), d_out, y, z, B_.ACT_RELU, ws)
    want, _, wz, _ = linear(x, W, stored, bias, d_out, "relu", residual)
    assert torch.equal(y.cpu(), want.to(t)) and torch.equal(z.cpu(), wz.to(t))
    ws = torch.empty(B_.srigl_structured_bwd_workspace_bytes(B, d_in, n, d_out, code), dtype=torch.uint8, device="cuda")
    B_.srigl_structured_linear_bwd(put(dy), xs, B, d_in, Ws, acts, n, bs, z, d_out, dx, dW, db, ws, B_.ACT_RELU)
    dz = dy.double()[:, stored] * (z.cpu() > 0)
    assert torch.equal(dx.cpu(), (dz @ W.double()).to(t)) and torch.equal(dW.cpu(), (dz.T @ x.double()).to(t))
    for room, m in ((y_room, B * d_out), (z_room, B * n), (dx_room, B * d_in), (dW_room, n * d_in), (db_room, d_out)):
        assert untouched(room, shift, m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_residual_in_place_and_gradients_one_by_one(dtype):
    gen, t = torch.Generator().manual_seed(3), TYPES[dtype]
    for ablated in (0.0, 0.4):
        W, bias, active, stored = _layer(gen, 96, 150, ablated, t, lambda s, tt: whole(gen, s, 2, tt))
        x, residual, dy = (whole(gen, s, 2, t).cuda() for s in ((33, 96), (33, 150), (33, 150)))
        layer = StructuredLinear(96, 150, *_cuda(W, active, bias))
        want = layer.forward(x, act=B_.ACT_GELU, residual=residual)
        y = residual.clone()
        assert layer.forward(x, act=B_.ACT_GELU, residual=y, y=y) is y and torch.equal(y, want)
        every = layer.backward(dy, x)
        none, dWd, db = layer.backward(dy, x, need_dx=False)
        assert none is None and torch.equal(dWd, every[1]) and torch.equal(db, every[2])
        plain = StructuredLinear(96, 150, *_cuda(W, active, None))
        dx, dWd, none = plain.backward(dy, x)
        assert none is None and torch.equal(dx, every[0]) and torch.equal(dWd, every[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_stored_no_rows_no_columns(dtype):
    t = TYPES[dtype]
    bias = torch.tensor([1.0, -2.0, 0.5], device="cuda")
    x, dy = torch.ones(4, 16, device="cuda", dtype=t), torch.ones(4, 3, device="cuda", dtype=t)
    # every neuron ablated: act(bias) and its slope
    layer = StructuredLinear(16, 3, torch.empty(0, 16, device="cuda", dtype=t), torch.empty(0, device="cuda", dtype=torch.int32), bias)
    assert torch.equal(layer.forward(x, act=B_.ACT_RELU, residual=dy).cpu(), torch.tensor([2.0, 1.0, 1.5]).expand(4, 3).to(t))
    dx, dWd, db = layer.backward(dy, x, torch.empty(4, 0, device="cuda", dtype=t), act=B_.ACT_RELU)
    assert not dx.any() and dx.shape == (4, 16) and dWd.shape == (0, 16) and db.tolist() == [4.0, 0.0, 4.0]
    # no rows: the weights' and the bias's gradients are zeros
    layer = StructuredLinear(16, 3, torch.ones(3, 16, device="cuda", dtype=t), None, bias)
    y, z = layer.forward(x[:0], save=True)
    assert y.shape == (0, 3) and z.shape == (0, 3)
    dx, dWd, db = layer.backward(dy[:0], x[:0], z)
    assert dx.shape == (0, 16) and not dWd.any() and not db.any()
    # no columns
    layer = StructuredLinear(0, 3, torch.empty(3, 0, device="cuda", dtype=t), None, bias)
    assert torch.equal(layer.forward(x[:, :0].contiguous()).cpu(), bias.cpu().expand(4, 3).to(t))
    dx, dWd, db = layer.backward(dy, x[:, :0].contiguous())
    assert dx.shape == (4, 0) and dWd.shape == (3, 0) and db.tolist() == [4.0, 4.0, 4.0]


@pytest.mark.parametrize("d_in,d_out,B", [(100, 70, 40), (256, 300, 200), (1001, 90, 3)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_stays_where_it_belongs(dtype, B, d_in, d_out):
    gen, t = torch.Generator().manual_seed(8), TYPES[dtype]
    x, W = whole(gen, (B, d_in), 2, t), whole(gen, (d_out, d_in), 2, t)
    x[1, d_in - 1], W[d_out - 1, 0] = float("inf"), float("nan")
    W[:, d_in - 1] = 1.0
    layer = StructuredLinear(d_in, d_out, W.cuda())
    y = layer.forward(x.cuda(), act=B_.ACT_RELU).cpu()
    assert y[:, -1].isnan().all() and (y[1, :-1] == float("inf")).all()
    clean = torch.ones(B, d_out, dtype=torch.bool)
    clean[1], clean[:, -1] = False, False
    assert y[clean].isfinite().all()
    dy = whole(gen, (B, d_out), 2, t)
    dy[:, -1] = 0.0   # 0 times the NaN row of W is NaN in its column, and only there
    dx, dWd, _ = layer.backward(dy.cuda(), x.cuda())
    assert dx[:, 0].isnan().all() and dx[:, 1:].isfinite().all()
    assert dWd[:, :-1].isfinite().all() and not dWd[:, -1].isfinite().any()


def test_update_takes_the_weight_gradient():
    """A training step of a masked layer: forward, backward, connectivity update, from the gradient as it comes."""
    gen = torch.Generator().manual_seed(2)
    d_in, d_out, K, B = 96, 64, 12, 50
    mask = torch.zeros(d_out, d_in, dtype=torch.uint8)
    mask.scatter_(1, torch.rand(d_out, d_in, generator=gen).topk(K, dim=1).indices, 1)
    W = (normal(gen, (d_out, d_in)) * mask).cuda()
    x, dy, mask = normal(gen, (B, d_in)).cuda(), normal(gen, (B, d_out)).cuda(), mask.cuda()
    layer = StructuredLinear(d_in, d_out, W)
    _, z = layer.forward(x, act=B_.ACT_GELU, save=True)
    _, grad, _ = layer.backward(dy, x, z, act=B_.ACT_GELU, need_dx=False)
    outs = []
    for g in (grad, (dy.double() * slope(z.double(), "gelu")).T.contiguous().cpu() @ x.double().cpu()):
        mask_out, W_out, report = torch.empty_like(mask), torch.empty_like(W), torch.empty(4, dtype=torch.int64, device="cuda")
        ws = torch.empty(B_.srigl_mask_update_workspace_bytes(d_out, d_in), dtype=torch.uint8, device="cuda")
        B_.srigl_mask_update(W, mask, g.float().cuda(), d_out, d_in, K, 200, 30, d_out * K, mask_out, W_out, ws, report)
        outs.append((mask_out.cpu(), W_out.cpu(), report.cpu()))
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and outs[0][2][1] > 0


@pytest.mark.parametrize("B,d_in,d_out", [(70000, 8, 5), (3, 16, 70001), (300, 40, 30000), (100, 0, 70), (129, 8, 1)])
@pytest.mark.parametrize("ablated", [0.0, 0.4])
def test_more_rows_or_neurons_than_a_grid_has_lines(B, d_in, d_out, ablated):
    gen = torch.Generator().manual_seed(B)
    W, bias, active, stored = _layer(gen, d_in, d_out, ablated, torch.bfloat16, lambda s, tt: whole(gen, s, 1, tt))
    x, dy = whole(gen, (B, d_in), 1, torch.bfloat16), whole(gen, (B, d_out), 1, torch.bfloat16)
    layer = StructuredLinear(d_in, d_out, *_cuda(W, active, bias))
    want, _, z, _ = linear(x, W, stored, bias, d_out, "relu")
    y, got_z = layer.forward(x.cuda(), act=B_.ACT_RELU, save=True)
    assert torch.equal(y.cpu(), want.bfloat16()) and torch.equal(got_z.cpu(), z.bfloat16())
    dx, dWd, db = layer.backward(dy.cuda(), x.cuda(), got_z, act=B_.ACT_RELU)
    dz = dy.double()[:, stored] * (got_z.cpu() > 0)
    dbias = dy.double().sum(0) * (bias > 0)
    dbias[stored] = dz.sum(0)
    assert torch.equal(dx.cpu(), (dz @ W.double()).bfloat16()) and torch.equal(dWd.cpu(), (dz.T @ x.double()).bfloat16()) and torch.equal(db.cpu(), dbias.float())


@pytest.mark.parametrize("spread", [1, 300, 3000])
def test_neurons_far_apart(spread):
    """Stored neurons in runs with long gaps: a workgroup's columns fit its LDS or do not."""
    gen = torch.Generator().manual_seed(spread)
    d_out, n = 20000, 700
    stored = torch.cat([torch.arange(k, k + n // 7) for k in torch.arange(7) * (n // 7 + spread - 1) + 11])
    active, W, x, bias = stored.int(), whole(gen, (n, 72), 2, torch.bfloat16), whole(gen, (40, 72), 2, torch.bfloat16), whole(gen, (d_out,), 2)
    dy = whole(gen, (40, d_out), 2, torch.bfloat16)
    layer = StructuredLinear(72, d_out, *_cuda(W, active, bias))
    want, _, z, _ = linear(x, W, stored, bias, d_out, "relu")
    for rows in (40, 5):
        y, got_z = layer.forward(x[:rows].cuda(), act=B_.ACT_RELU, save=True)
        assert torch.equal(y.cpu(), want[:rows].bfloat16()) and torch.equal(got_z.cpu(), z[:rows].bfloat16())
        dx, dWd, db = layer.backward(dy[:rows].cuda(), x[:rows].cuda(), got_z, act=B_.ACT_RELU)
        dz = dy[:rows].double()[:, stored] * (z[:rows] > 0)
        dbias = dy[:rows].double().sum(0) * (bias > 0)
        dbias[stored] = dz.sum(0)
        assert torch.equal(dx.cpu(), (dz @ W.double()).bfloat16()) and torch.equal(dWd.cpu(), (dz.T @ x[:rows].double()).bfloat16()) and torch.equal(db.cpu(), dbias.float())


@pytest.mark.parametrize("B,d_in,d_out", [(3, 264, 100), (100, 264, 300), (70, 137, 90)])
def test_fp32_from_end_to_end_of_its_range(B, d_in, d_out):
    """Powers of two from 2^-40 to 2^100: products and sums of one sign keep their relative error, and sums beyond the range are infinite as in fp32."""
    gen = torch.Generator().manual_seed(4)
    x, W = torch.rand(B, d_in, generator=gen) + 0.5, torch.rand(d_out, d_in, generator=gen) + 0.5
    scale = 2.0 ** torch.randint(-40, 100, (B, 1), generator=gen).float()
    y = StructuredLinear(d_in, d_out, W.cuda()).forward((x * scale).cuda())
    want = (x * scale).double() @ W.double().T
    within(y, want, sum_gate(d_in) * want, "y")
    dx, dWd, _ = StructuredLinear(d_in, d_out, W.cuda()).backward((torch.ones(B, d_out) * scale).cuda(), x.cuda())
    want = (torch.ones(B, d_out) * scale).double() @ W.double()
    within(dx, want, sum_gate(d_out) * want, "dx")
    x[0], W[0] = 3e38, 1.0
    y = StructuredLinear(d_in, d_out, W.cuda()).forward(x.cuda()).cpu()
    assert (y[0] == float("inf")).all() and y[1:].isfinite().all()
    x[0, 1:], W[0, 1:] = 0.0, 0.0
    y = StructuredLinear(d_in, d_out, W.cuda()).forward(x.cuda()).cpu()
    assert y[0, 0] == x[0, 0] and y[1:].isfinite().all()


def test_same_bits_every_time():
    gen = torch.Generator().manual_seed(6)
    for t, B, d_in, d_out in ((torch.float32, 200, 520, 300), (torch.bfloat16, 77, 1001, 400), (torch.bfloat16, 300, 768, 3000)):
        W, bias, active, stored = _layer(gen, d_in, d_out, 0.2, t, lambda s, tt: normal(gen, s, 0.1, tt))
        x, dy = normal(gen, (B, d_in), 1.0, t).cuda(), normal(gen, (B, d_out), 1.0, t).cuda()
        layer, runs = StructuredLinear(d_in, d_out, *_cuda(W, active, bias)), []
        for _ in range(3):
            y, z = layer.forward(x, act=B_.ACT_SILU, save=True)
            runs.append([y, z, *layer.backward(dy, x, z, act=B_.ACT_SILU)])
        assert all(torch.equal(a, b) for other in runs[1:] for a, b in zip(runs[0], other))


def test_condensed_layer_as_dense_rows():
    """A condensed layer's structured() runs the same layer, with what stands behind the product."""
    import numpy as np
    import synth_inputs as si
    from gpu_util import TOL_F32, dev, gate, host, oracle_condensed
    from paper_2305_02299_amd import condense_layer
    import oracle
    L = si.make_layer(200, 130, 20, 9, ablate_frac=0.3, seed=7)
    layer = condense_layer(dev(L.W), dev(L.mask), L.K, dev(L.bias)).structured()
    W_c, idx, active = oracle_condensed(L)
    y_ref, S = oracle.fwd(L.x, W_c, idx, active, L.bias, 130, want_scale=True)
    gate(host(layer.forward(dev(L.x))), y_ref, S, TOL_F32)
    np.testing.assert_array_equal(host(layer.forward(dev(L.x), act=B_.ACT_RELU)), np.maximum(host(layer.forward(dev(L.x))), 0))


def test_refused_tensors():
    x, W = torch.zeros(4, 16, device="cuda"), torch.zeros(8, 16, device="cuda")
    layer = StructuredLinear(16, 8, W)
    y = torch.zeros(4, 8, device="cuda")
    for wrong in (lambda: layer.forward(x[:, :8]), lambda: layer.forward(x[:, ::2].contiguous()), lambda: layer.forward(x.cpu()), lambda: layer.forward(x.bfloat16()),
                  lambda: layer.forward(x, residual=y[:2]), lambda: layer.forward(x, residual=y.bfloat16()), lambda: layer.forward(x, y=y[:, :4]),
                  lambda: layer.forward(x, out_dtype=torch.bfloat16), lambda: layer.forward(x, y=y.t()), lambda: layer.backward(y[:3], x), lambda: layer.backward(y, x, y[:, :4].contiguous()),
                  lambda: layer.backward(y, x, y.bfloat16()), lambda: layer.backward(y.bfloat16(), x), lambda: StructuredLinear(16, 9, W).forward(x),
                  lambda: StructuredLinear(16, 8, W, None, torch.zeros(7, device="cuda")).forward(x), lambda: StructuredLinear(16, 8, W, None, torch.zeros(8, device="cuda").bfloat16()).forward(x),
                  lambda: StructuredLinear(16, 8, W, torch.zeros(8, device="cuda")).forward(x), lambda: StructuredLinear(16, 8, W.t().contiguous().t()).forward(x),
                  lambda: layer.forward(x, act=4), lambda: layer.forward(x, act=-1), lambda: layer.backward(y, x, None, act=B_.ACT_GELU),
                  lambda: StructuredLinear(16, 9, W).backward(torch.zeros(4, 9, device="cuda"), x)):
        with pytest.raises((SriglError, TypeError, AssertionError, ValueError)):
            wrong()
    assert half_step(torch.bfloat16) == 2.0 ** -8


def test_refused_results():
    """A result in the memory of an input, or of another type than asked for; the residual itself is a place for it."""
    gen = torch.Generator().manual_seed(5)
    memory = normal(gen, (3, 20, 64), 1.0, torch.float32).cuda()
    x, W, residual = memory[0], normal(gen, (64, 64), 0.1, torch.float32).cuda(), memory[1]
    layer = StructuredLinear(64, 64, W)
    want = layer.forward(x, residual=residual)
    for kw in (dict(y=x), dict(y=W[:20]), dict(y=memory.view(-1)[20 * 64 - 64:2 * 20 * 64 - 64].view(20, 64)),
               dict(y=memory.view(-1)[2 * 20 * 64 - 64:3 * 20 * 64 - 64].view(20, 64), residual=residual)):
        with pytest.raises(ValueError):
            layer.forward(x, **kw)
    half = StructuredLinear(64, 64, W.bfloat16())
    with pytest.raises(AssertionError):
        half.forward(x.bfloat16(), out_dtype=torch.float32, y=torch.empty(20, 64, dtype=torch.bfloat16, device="cuda"))
    y = memory[2]
    assert layer.forward(x, residual=residual, y=y) is not None and torch.equal(y, want)
    assert torch.equal(layer.forward(x, residual=residual, y=residual), want) and torch.equal(residual, want)
