"""What the C calls of the feed-forward blocks refuse, and the scratch they ask for: host arithmetic, before anything reaches a GPU."""
import pytest

from paper_2305_02299_amd import binding as B_

lib, P = B_.lib, 4096   # P: some address; nothing is read


def _fwd(x=P, xt=0, B=4, d_in=16, W=P, wt=0, active=None, n=8, bias=None, res=None, d_out=8, y=P, yt=0, z=None, act=0, ws=None, wb=0):
    return lib.srigl_structured_linear_fwd_act(x, xt, B, d_in, W, wt, active, n, bias, res, d_out, y, yt, z, act, ws, wb, None)


def _bwd(dy=P, dt=0, x=P, xt=0, B=4, d_in=16, W=P, wt=0, active=None, n=8, bias=None, z=P, d_out=8, act=0, dx=P, dW=P, db=P, ws=P, wb=1 << 40):
    return lib.srigl_structured_linear_bwd(dy, dt, x, xt, B, d_in, W, wt, active, n, bias, z, d_out, act, dx, dW, db, ws, wb, None)


def _gated(x=P, xt=0, B=4, d_in=16, Wg=P, Wu=P, wt=0, n=8, bg=None, bu=None, act=3, h=P, g=None, u=None, ws=None, wb=0):
    return lib.srigl_gated_linear_fwd(x, xt, B, d_in, Wg, Wu, wt, n, bg, bu, act, h, g, u, ws, wb, None)


def _gated_bwd(dh=P, x=P, xt=0, B=4, d_in=16, Wg=P, Wu=P, wt=0, n=8, g=P, u=P, act=3, dx=P, dWg=P, dWu=P, dbg=None, dbu=None, ws=P, wb=1 << 40):
    return lib.srigl_gated_linear_bwd(dh, x, xt, B, d_in, Wg, Wu, wt, n, g, u, act, dx, dWg, dWu, dbg, dbu, ws, wb, None)


INVALID, CAPACITY, UNSUPPORTED = B_.ERR_INVALID_ARG, B_.ERR_CAPACITY, B_.ERR_UNSUPPORTED


@pytest.mark.parametrize("call,size", [(_fwd, "B"), (_fwd, "d_in"), (_fwd, "n"), (_fwd, "d_out"), (_bwd, "B"), (_bwd, "d_in"), (_bwd, "n"), (_bwd, "d_out"),
                                       (_gated, "B"), (_gated, "d_in"), (_gated, "n"), (_gated_bwd, "B"), (_gated_bwd, "d_in"), (_gated_bwd, "n")])
def test_sizes(call, size):
    assert call(**{size: -1}) == INVALID and call(**{size: -2 ** 31}) == INVALID
    more = {"n": 2 ** 30 + 1, "d_out": 2 ** 30 + 1, "active": P} if size in ("n", "d_out") and call in (_fwd, _bwd) else {size: 2 ** 30 + 1}
    assert call(**more) == UNSUPPORTED


@pytest.mark.parametrize("call", [_fwd, _bwd, _gated, _gated_bwd])
def test_types_and_activations(call):
    for wrong in (-1, 4, 2 ** 31 - 1):
        assert call(act=wrong) == INVALID
    assert call(xt=2) == INVALID and call(wt=-1) == INVALID and call(xt=1) == UNSUPPORTED and call(wt=1) == UNSUPPORTED


def test_mixed_result_types():
    assert _fwd(yt=1) == UNSUPPORTED and _fwd(yt=5) == INVALID and _bwd(dt=1) == UNSUPPORTED and _bwd(dt=5) == INVALID


def test_missing_arguments():
    assert all(_fwd(**{k: None}) == INVALID for k in ("x", "W", "y")) and _fwd(n=7) == INVALID and _fwd(n=9) == INVALID
    assert all(_bwd(**{k: None}) == INVALID for k in ("dy", "x", "W")) and _bwd(z=None, act=2) == INVALID and _bwd(n=7) == INVALID
    assert all(_gated(**{k: None}) == INVALID for k in ("x", "Wg", "Wu", "h")) and _gated(g=P) == INVALID and _gated(u=P) == INVALID
    assert all(_gated_bwd(**{k: None}) == INVALID for k in ("dh", "x", "Wg", "Wu", "g", "u"))


def test_addresses_between_elements():
    for k in ("x", "W", "bias", "res", "y", "z"):
        assert _fwd(**{k: P + 2}) == INVALID and _fwd(xt=1, wt=1, yt=1, **{k: P + 1}) == INVALID
    for k in ("dy", "x", "W", "bias", "z", "dx", "dW", "db"):
        assert _bwd(**{k: P + 2}) == INVALID
    for k in ("x", "Wg", "Wu", "bg", "bu", "h"):
        assert _gated(**{k: P + 2}) == INVALID
    for k in ("dh", "x", "Wg", "Wu", "g", "u", "dx", "dWg", "dWu", "dbg", "dbu", "ws"):
        assert _gated_bwd(**{k: P + 2}) == INVALID
    assert _bwd(ws=P + 8) == INVALID


def test_scratch_too_small():
    for call, need in ((_bwd, B_.srigl_structured_bwd_workspace_bytes(4, 16, 8, 8, B_.F32)), (_gated_bwd, B_.srigl_gated_bwd_workspace_bytes(4, 16, 8, B_.F32))):
        assert need >= 4 * 8 * 4 and call(wb=need - 1) == CAPACITY and call(ws=None, wb=need) == CAPACITY


def test_nothing_to_do():
    assert _fwd(B=0) == B_.OK and _fwd(d_out=0, n=0) == B_.OK and _gated(B=0) == B_.OK and _gated(n=0) == B_.OK
    assert _bwd(dx=None, dW=None, db=None, ws=None, wb=0) == B_.OK and _gated_bwd(dx=None, dWg=None, dWu=None, ws=None, wb=0) == B_.OK


def test_scratch_of_no_size():
    for args in ((-1, 8, 8), (8, -1, 8), (8, 8, -1), (2 ** 30 + 1, 8, 8), (8, 2 ** 30 + 1, 8)):
        assert B_.srigl_structured_act_workspace_bytes(*args, B_.F32) == B_.srigl_gated_workspace_bytes(*args, B_.F32) == B_.srigl_gated_bwd_workspace_bytes(*args, B_.F32) == 0
        assert B_.srigl_structured_bwd_workspace_bytes(*args, max(args[2], 8), B_.F32) == 0
    # more than 32 bits of it
    assert B_.srigl_gated_bwd_workspace_bytes(2 ** 20, 4096, 2 ** 14, B_.BF16) > 2 ** 35


def test_silu_is_not_for_the_condensed_calls():
    assert lib.srigl_condensed_linear_fwd_act(P, 0, 4, 16, P, 0, P, None, 8, 2, None, 8, P, None, None, B_.ACT_SILU, 0, None, None) == INVALID
