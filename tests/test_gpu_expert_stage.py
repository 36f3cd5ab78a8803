"""The expert stage as the example runs it: gate, routing, moves and 4-bit layers together against 64 bits, and the
moves' gradients through autograd.  GPU only."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import expert_stage as ex  # noqa: E402
import paper_2512_19342_b200 as bls  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,D,E,H,O,k", [(1, 64, 8, 96, 64, 2), (37, 128, 4, 200, 72, 3), (500, 256, 16, 384, 128, 2), (2000, 64, 5, 128, 64, 1)])
def test_stage_against_64_bits(n, D, E, H, O, k):
    """Reference: the same choice of experts, then every row through its experts' weights in 64 bits with the activations rounded
    to bfloat16 where the stage stores them.  A value within fp32 round-off of a rounding boundary may round the other way, one unit of
    2^-8 of a hidden value at most, and so may each answer: per row the error stays under 2^-7 of the largest output plus the same
    share of a hidden value times a row of weights, which 2e-2 of the largest output covers."""
    g = torch.Generator(device="cuda").manual_seed(n)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    gate = (rnd(E, D) / D ** 0.5).to(torch.bfloat16)
    up_b, down_b = 0.1 * rnd(E, H), 0.1 * rnd(E, O)
    stage = ex.ExpertStage(gate, rnd(E, H, D) / D ** 0.5, up_b, rnd(E, O, H) / H ** 0.5, down_b, k, n)
    x = rnd(n, D).to(torch.bfloat16)
    out = stage(x)
    logits = torch.empty(n, E, device="cuda")
    stage.gate.forward(x, logits)
    assert stage.gate.status() == bls.bls_w4_status() == bls.BLS_OK
    top, expert = logits.topk(k, dim=1)
    w = torch.softmax(top, 1).double()
    up, down = (torch.empty(E, q.N, q.K, device="cuda") for q in (stage.up, stage.down))
    bls.bls_w4_dequantize(stage.up, up)
    bls.bls_w4_dequantize(stage.down, down)
    want = torch.zeros(n, O, device="cuda", dtype=torch.float64)
    for i in range(k):
        for e in range(E):
            rows = torch.nonzero(expert[:, i] == e)[:, 0]
            h = torch.relu(x[rows].double() @ up[e].double().t() + up_b[e].double()).to(torch.bfloat16).double()
            a = (h @ down[e].double().t() + down_b[e].double()).to(torch.bfloat16).double()
            want[rows] += w[rows, i:i + 1] * a
    err = (out.double() - want).abs().amax(1) / want.abs().amax(1)
    assert float(err.max()) <= 2e-2


def test_moves_through_autograd():
    """fp32: the moves' gradients against the same function in 64 bits.  A result of c fp32 roundings on its longest path is off by at
    most c 2^-24 times the sum of its terms' magnitudes: k + 2 for sums over a token's slots, D + 2 for dot products of rows."""
    n, k, E, D = 50, 3, 6, 40
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    expert = torch.randint(-1, E, (n, k), device="cuda", generator=g, dtype=torch.int32)
    routes = ex.Routes(expert, E)
    x, w, scale = rnd(n, D).requires_grad_(), rnd(n, k).requires_grad_(), rnd(n * k, D)
    out = ex.combine(ex.dispatch(x, routes) * scale, w, routes)
    dout = rnd(n, D)
    out.backward(dout)
    place = routes.place
    xd, wd = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    keep, at = place >= 0, place.clamp(min=0).long()
    want = (torch.where(keep[..., None], xd[:, None, :] * scale.double()[at], 0.0) * wd[..., None]).sum(1)
    want.backward(dout.double())
    aw, asc, ad = wd.detach().abs(), torch.where(keep[..., None], scale.double()[at], 0.0).abs(), dout.double().abs()
    sizes = ((xd.detach().abs()[:, None, :] * asc * aw[..., None]).sum(1), (asc * aw[..., None]).sum(1) * ad,
             (xd.detach().abs()[:, None, :] * asc * ad[:, None, :]).sum(2))
    for got, ref, size, c in ((out, want, sizes[0], k + 2), (x.grad, xd.grad, sizes[1], k + 2), (w.grad, wd.grad, sizes[2], D + 2)):
        assert bool(((got.detach().double() - ref.detach()).abs() <= c * 2.0 ** -24 * size + 2.0 ** -149).all())


def test_example_runs(capsys):
    ex.main()
    assert "probabilities" in capsys.readouterr().out
