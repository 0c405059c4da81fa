"""fp32 products on the bf16 matrix units: each value as three bf16 parts, six products of parts to a product.

A sum with one term that is not zero shows what becomes of a product.  Where the product has 24 bits, nothing may be missing: one factor a power of two and the other of 24 bits takes all three parts of the other
one times the leading part of the first, 1 + i 2^-11 times 1 + j 2^-11 (1 + (i + j) 2^-11 + i j 2^-22, i and j below 8) the second parts' product too.  Every operand is both the one that has one value in a line
and the one that is full, so that every place of the parts in the matrix units' registers counts."""
import pytest
import torch

from paper_2305_02299_amd import GatedLinear, StructuredLinear
from paper_2305_02299_amd import binding as B_

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,d_in,n", [(78, 64, 66), (116, 2396, 40), (1767, 156, 3201), (898, 644, 2197), (71, 21, 23)])
@pytest.mark.parametrize("terms", [1, 3, 16])
def test_products_of_any_mantissas(terms, B, d_in, n):
    """Sums of a few products of one sign and size.  2^-24 of each product may be left out.  Terms in the same 16 of K meet in one rounding but for the much smaller ones of the other parts; whichever way
    the units round, the sum is off by a step of 2^-23 behind each 16 of K that has terms, of a running sum that is at most the result: (1 + 2 groups) 2^-24, and a thirtieth for the roundings of the sums of
    the smaller parts (below 2^-6 of the sum, six of them)."""
    gen = torch.Generator().manual_seed(B + terms)
    x, W = torch.zeros(B, d_in), torch.zeros(n, d_in)
    first = min(d_in - terms, 32)
    groups = (first + terms - 1) // 16 - first // 16 + 1   # one but for 16 terms of 21
    x[:, first:first + terms] = (torch.randint(2 ** 23, 2 ** 24, (B, 1), generator=gen).double() * 2.0 ** -23).float()
    W[:, first:first + terms] = (torch.randint(2 ** 23, 2 ** 24, (n, 1), generator=gen).double() * 2.0 ** -23).float()
    # the mantissas of which most is left out when the parts are cut off
    x[:3, first:first + terms] = W[:3, first:first + terms] = 1 + 2.0 ** -7 - 2.0 ** -23
    want = terms * (x[:, first:first + 1].double() @ W[:, first:first + 1].double().T)
    off = (StructuredLinear(d_in, n, W.cuda()).forward(x.cuda()).cpu().double() - want).abs() / want
    assert off.max() <= 31 / 30 * (1 + 2 * groups) * 2.0 ** -24, float(off.max()) * 2.0 ** 24


KINDS = [("full", "power"), ("power", "full"), ("middle", "middle")]   # of the operand with all its values, of the one with a value a line


def _values(gen, shape, kind):
    sign = torch.randint(0, 2, shape, generator=gen) * 2.0 - 1
    scale = sign * 2.0 ** torch.randint(-3, 4, shape, generator=gen)
    if kind == "power":
        return scale
    if kind == "middle":
        return scale * (1 + torch.randint(1, 8, shape, generator=gen) * 2.0 ** -11)
    return scale * (torch.randint(2 ** 23, 2 ** 24, shape, generator=gen) * 2.0 ** -23)


def _single(gen, lines, K, kind):
    """lines x K with one value a line; the places and the values"""
    at, v = torch.randint(0, K, (lines,), generator=gen), _values(gen, (lines,), kind)
    m = torch.zeros(lines, K)
    m[torch.arange(lines), at] = v
    return m, at, v


def _operands(gen, M, N, K, full, single, of_n):
    """A [M, K], B [N, K] and A B^T, exact in fp32; of_n: B is the operand with one value a line"""
    dense, (sparse, at, v) = _values(gen, (M if of_n else N, K), full), _single(gen, N if of_n else M, K, single)
    product = dense[:, at].double() * v.double()
    assert torch.equal(product.float().double(), product)
    return (dense, sparse, product.float()) if of_n else (sparse, dense, product.float().T)


# (batch, d_in, neurons; the tile that the library takes: S 64 x 64, M 128 x 128, H 256 x 128, S2 and M2 with two stages of the ring; odd d_in: rows that begin anywhere, through registers)
@pytest.mark.parametrize("B,d_in,n", [(78, 100, 90), (80, 2120, 20), (453, 480, 462), (898, 644, 2197), (2372, 96, 2660), (1767, 156, 3201), (71, 21, 23), (453, 481, 462), (1372, 21, 4675)],
                         ids=["S2", "S parts", "S", "M", "M2", "H", "S any", "S any deep", "M any"])
@pytest.mark.parametrize("full,single", KINDS)
def test_every_part_counts_forward(full, single, B, d_in, n):
    gen = torch.Generator().manual_seed(B)
    for of_n in (True, False):
        x, W, want = _operands(gen, B, n, d_in, full, single, of_n)
        assert torch.equal(StructuredLinear(d_in, n, W.cuda()).forward(x.cuda()).cpu(), want)


@pytest.mark.parametrize("B,d_in,n", [(81, 100, 90), (116, 2396, 22), (463, 704, 321), (828, 1148, 1766), (1550, 96, 3352), (1231, 216, 3104), (71, 21, 24), (1690, 45, 2291)],
                         ids=["S2", "S parts", "S", "M", "M2", "H", "S any", "M any"])
@pytest.mark.parametrize("full,single", KINDS)
def test_every_part_counts_gated(full, single, B, d_in, n):
    gen = torch.Generator().manual_seed(B)
    for of_n in (True, False):
        x, Wg, want = _operands(gen, B, n, d_in, full, single, of_n)
        other = torch.zeros(n, d_in)   # (the other matrix takes a column of x as it is)
        other[:, d_in // 2] = 1.0
        for first in (True, False):
            h, g, u = GatedLinear(d_in, n, *((Wg.cuda(), other.cuda()) if first else (other.cuda(), Wg.cuda())), act=B_.ACT_NONE).forward(x.cuda(), save=True)
            mine, its = (g, u) if first else (u, g)
            assert torch.equal(mine.cpu(), want) and torch.equal(its.cpu(), x[:, d_in // 2:d_in // 2 + 1].expand(B, n))
            assert torch.equal(h.cpu(), (g.cpu().double() * u.cpu().double()).float())


BACKWARD = [(78, 100, 90), (453, 480, 462), (506, 416, 482), (1241, 932, 910), (1739, 2312, 747), (402, 3012, 2260), (1954, 2180, 1878), (2113, 1856, 2265), (71, 21, 23), (1513, 453, 994)]
BACKWARD_IDS = ["S2", "S", "S2 parts", "M2", "M", "H", "S2 and M2", "M and M2", "S any", "M any"]


@pytest.mark.parametrize("B,d_in,n", BACKWARD, ids=BACKWARD_IDS)
@pytest.mark.parametrize("full,single", KINDS)
def test_every_part_counts_in_gradients(full, single, B, d_in, n):
    gen = torch.Generator().manual_seed(B)
    for of_n in (True, False):
        # dx = dy W: K is the neurons
        dy, Wt, want = _operands(gen, B, d_in, n, full, single, of_n)
        x = torch.zeros(B, d_in)
        dx, dW, _ = StructuredLinear(d_in, n, Wt.T.contiguous().cuda()).backward(dy.cuda(), x.cuda())
        assert torch.equal(dx.cpu(), want) and not dW.any()
        # dW = dy^T x: K is the batch
        dyt, xt, want = _operands(gen, n, d_in, B, full, single, of_n)
        layer = StructuredLinear(d_in, n, torch.zeros(n, d_in).cuda())
        dx, dW, _ = layer.backward(dyt.T.contiguous().cuda(), xt.T.contiguous().cuda())
        assert torch.equal(dW.cpu(), want) and not dx.any()
        assert torch.equal(layer.backward(dyt.T.contiguous().cuda(), xt.T.contiguous().cuda(), need_dx=False)[1], dW)


@pytest.mark.parametrize("B,d_in,n", [(81, 100, 90), (463, 704, 321), (459, 436, 504), (1019, 944, 589), (828, 1148, 1766), (402, 1432, 2388), (1051, 2352, 1667), (71, 21, 24), (1977, 325, 490)],
                         ids=["S2", "S", "S2 parts", "M2", "M", "H", "M2 and S2", "S any", "M any"])
@pytest.mark.parametrize("full,single", KINDS)
def test_every_part_counts_in_gated_gradients(full, single, B, d_in, n):
    """Without an activation dg = dh u and du = dh g: with one of g and u 1 and the other 0, one of them is dh and the other 0."""
    gen = torch.Generator().manual_seed(B)
    ones, zeros = torch.ones(B, n).cuda(), torch.zeros(B, n).cuda()
    for of_n in (True, False):
        dh, Wt, want = _operands(gen, B, d_in, n, full, single, of_n)
        W, other = Wt.T.contiguous().cuda(), torch.ones(n, d_in).cuda()
        for first in (True, False):
            block = GatedLinear(d_in, n, *((W, other) if first else (other, W)), act=B_.ACT_NONE)
            dx = block.backward(dh.cuda(), torch.zeros(B, d_in).cuda(), *((zeros, ones) if first else (ones, zeros)))[0]
            assert torch.equal(dx.cpu(), want)
        dht, xt, want = _operands(gen, n, d_in, B, full, single, of_n)
        block = GatedLinear(d_in, n, other, other, act=B_.ACT_NONE)
        for first in (True, False):
            _, dWg, dWu, _, _ = block.backward(dht.T.contiguous().cuda(), xt.T.contiguous().cuda(), *((zeros, ones) if first else (ones, zeros)))
            mine, its = (dWg, dWu) if first else (dWu, dWg)
            assert torch.equal(mine.cpu(), want) and not its.any()


@pytest.mark.parametrize("B,d_in,d_out", [(100, 264, 300), (70, 137, 90), (520, 768, 2048)])
def test_weight_gradients_from_end_to_end_of_the_range(B, d_in, d_out):
    """Full mantissas from 2^-40 to 2^40, every neuron of its own size and every sum of one sign: each keeps its relative error."""
    gen = torch.Generator().manual_seed(d_in)
    x, W = torch.rand(B, d_in, generator=gen) + 0.5, torch.rand(d_out, d_in, generator=gen) + 0.5
    dy = (torch.rand(B, d_out, generator=gen) + 0.5) * 2.0 ** torch.randint(-40, 41, (1, d_out), generator=gen).float()
    dx, dWd, _ = StructuredLinear(d_in, d_out, W.cuda()).backward(dy.cuda(), x.cuda())
    for got, want, K in ((dx, dy.double() @ W.double(), d_out), (dWd, dy.double().T @ x.double(), B)):
        assert ((got.cpu().double() - want).abs() <= min((K + 8) * 2.0 ** -24, 1e-5) * want).all()


def test_values_that_round_beyond_the_range_of_bf16():
    """3.4e38 is finite in fp32 and rounds to infinity in bf16: its tile is computed by the fp32 units."""
    x, W = torch.zeros(100, 64), torch.zeros(70, 64)
    x[:, 3], W[:, 3] = 3.4e38, 0.5
    x[7, 3] = -3.4e38
    y = StructuredLinear(64, 70, W.cuda()).forward(x.cuda()).cpu()
    assert torch.equal(y, (x[:, 3:4] * 0.5).expand(100, 70))
