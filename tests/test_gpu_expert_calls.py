"""How the expert stage's calls treat their memory, streams and threads, beside what they compute.  GPU only."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import expert_stage as ex  # noqa: E402
import paper_2512_19342_b200 as bls  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("rows", [3, 200])
def test_weights_whose_memory_moves(rows):
    """Doubled scales double every answer exactly, wherever they lie; a scale tensor that no longer fits is refused."""
    g = gen(rows)
    t = bls.bls_w4_quantize(torch.randn(200, 300, device="cuda", generator=g), 64, False)
    x = torch.randn(rows, 300, device="cuda", generator=g).to(BF16)
    y0, y1, w0, w1 = torch.empty(rows, 200, device="cuda"), torch.empty(rows, 200, device="cuda"), *(torch.empty(200, 300, device="cuda") for _ in range(2))
    bls.bls_w4_linear(t, x, y0)
    bls.bls_w4_dequantize(t, w0)
    before = t.scale.data_ptr()
    t.scale.data = t.scale * 2
    t.q.data, t.zero.data = t.q.clone(), t.zero.clone()
    assert t.scale.data_ptr() != before
    bls.bls_w4_linear(t, x, y1)
    bls.bls_w4_dequantize(t, w1)
    assert torch.equal(y1, 2 * y0) and torch.equal(w1, 2 * w0)
    t.scale.data = t.scale[:, :2].clone()
    with pytest.raises(ValueError):
        bls.bls_w4_linear(t, x, y1)
    with pytest.raises(ValueError):
        bls.bls_w4_dequantize(t, w1)


def test_second_derivatives_are_refused():
    """d out / d x depends on w: a graph of the gradient that leaves this out must not come back."""
    n, k, E, D = 20, 2, 4, 24
    g = gen(5)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    routes = ex.Routes(torch.randint(0, E, (n, k), device="cuda", generator=g, dtype=torch.int32), E)
    x, w = rnd(n, D).requires_grad_(), rnd(n, k).requires_grad_()
    out = ex.combine(ex.dispatch(x, routes), w, routes).sum()
    with pytest.raises(RuntimeError, match="first derivatives"):
        torch.autograd.grad(out, (x, w), create_graph=True)
    only = ex.dispatch(x, routes).sum()
    with pytest.raises(RuntimeError, match="first derivatives"):
        torch.autograd.grad(only, x, create_graph=True)
    again = ex.combine(ex.dispatch(x, routes), w, routes).sum()
    dx, dw = torch.autograd.grad(again, (x, w))
    # fp32 sums: k terms for dx, D products for dw, two more roundings each
    assert bool(((dx - w.sum(1, keepdim=True)).abs() <= 2 * (k + 2) * 2.0 ** -24 * w.abs().sum(1, keepdim=True)).all())
    assert bool(((dw - x.sum(1, keepdim=True)).abs() <= 2 * (D + 2) * 2.0 ** -24 * x.abs().sum(1, keepdim=True)).all())
