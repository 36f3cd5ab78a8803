"""The expert stage as a whole, and the plain forms of its operators, against bounds for every single value.  GPU only.

A result summed in fp32 is within c 2^-24 sum|terms| of the exact one (c = 2 K + groups + 12 for products of K inputs, whose additions may
truncate; see tests/test_gpu_experts.py) and is then rounded once.  Where a bound on a value before rounding is known, the rounded
value lies between the rounded ends of its interval, so a hidden value only counts as uncertain where it is next to a rounding boundary."""
import importlib.util
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

import expert_stage as ex  # noqa: E402
import paper_2512_19342_b200 as bls  # noqa: E402

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def product(lo, hi, w, bias, groups):
    """Ends of what a layer may answer to inputs between lo and hi, before rounding."""
    mid, half = (lo + hi) / 2, (hi - lo) / 2
    terms = torch.maximum(lo.abs(), hi.abs()) @ w.abs().t() + bias.abs()
    slack = half @ w.abs().t() + (2 * w.shape[1] + groups + 12) * 2.0 ** -24 * terms
    y = mid @ w.t() + bias
    return y - slack, y + slack


def stored(lo, hi):
    return lo.to(BF16).double(), hi.to(BF16).double()


@pytest.mark.parametrize("n,D,E,H,O,k", [(1, 64, 8, 96, 64, 2), (37, 128, 4, 200, 72, 3), (300, 256, 16, 384, 128, 4), (2000, 64, 5, 128, 64, 1)])
def test_every_value_of_the_stage(n, D, E, H, O, k):
    g = torch.Generator(device="cuda").manual_seed(n + k)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    stage = ex.ExpertStage((rnd(E, D) / D ** 0.5).to(BF16), rnd(E, H, D) / D ** 0.5, 0.1 * rnd(E, H), rnd(E, O, H) / H ** 0.5, 0.1 * rnd(E, O), k, n)
    x = rnd(n, D).to(BF16)
    out = stage(x).double()
    logits = torch.empty(n, E, device="cuda")
    stage.gate.forward(x, logits)
    top, expert = logits.topk(k, dim=1)
    w = torch.softmax(top, 1).double()
    up, down = (torch.empty(E, q.N, q.K, device="cuda") for q in (stage.up, stage.down))
    bls.bls_w4_dequantize(stage.up, up)                       # fp32: (q - z) s has at most 12 bits
    bls.bls_w4_dequantize(stage.down, down)
    low, high, size = (torch.zeros(n, O, device="cuda", dtype=torch.float64) for _ in range(3))
    last = torch.zeros_like(low)                              # what the expert of the smallest weight adds
    for i in range(k):
        for e in range(E):
            rows = torch.nonzero(expert[:, i] == e)[:, 0]
            xd = x[rows].double()
            h = product(xd, xd, up[e].double(), stage.up_bias[e].double(), D // 64 + 1)
            h = stored(*(v.clamp(min=0) for v in h))
            a = stored(*product(*h, down[e].double(), stage.down_bias[e].double(), H // 64 + 1))
            low[rows] += w[rows, i:i + 1] * a[0]
            high[rows] += w[rows, i:i + 1] * a[1]
            size[rows] += w[rows, i:i + 1] * torch.maximum(a[0].abs(), a[1].abs())
            if i == k - 1:
                last[rows] = w[rows, i:i + 1] * (a[0] + a[1]) / 2
    slack = (k + 1) * 2.0 ** -24 * size
    low, high = stored(low - slack, high + slack)
    assert bool(((out >= low) & (out <= high)).all())
    less = out - last                                         # the bounds are narrow enough to miss that expert in every row
    assert bool(((less < low) | (less > high)).any(1).all())


def plain_forms():
    spec = importlib.util.spec_from_file_location("operators_cases", os.path.join(ROOT, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def both(case, seed):
    m = plain_forms()
    s = m.prepare(case, seed)
    got = []
    for own in (False, True):
        m.own = own
        got.append(m.run(s))
    return m, s, *got


@pytest.mark.parametrize("n,k,E,left_out", [(1, 8, 64, 0.0), (77, 3, 9, 0.5), (3000, 6, 256, 0.03)])
def test_plain_route(n, k, E, left_out):
    _, _, plain, own = both(dict(op="route", n=n, k=k, E=E, left_out=left_out), 7)
    assert all(torch.equal(plain[name], own[name]) for name in plain)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,k,D", [(50, 1, 333), (200, 5, 256)])
def test_plain_moves(n, k, D, dtype):
    """Copies and single products are equal; a sum of c terms in two orders differs by 2 c roundings and two roundings to the output's type."""
    _, s, plain, own = both(dict(op="move", n=n, k=k, D=D, dtype=dtype, left_out=0.1, train=True), 8)
    assert torch.equal(plain["xs"], own["xs"]) and torch.equal(plain["dye"], own["dye"])
    here, at = (s["place"] >= 0)[..., None], s["place"].clamp(min=0).long()
    ye, dxs = (torch.where(here, s[v][at].double().abs(), 0.0) for v in ("ye", "dxs"))
    u = torch.finfo(s["x"].dtype).eps / 2
    tiny = torch.finfo(s["x"].dtype).smallest_normal * u
    for name, terms, c, unit in (("out", (ye * s["w"].double()[..., None]).sum(1), k + 1, u), ("dx", dxs.sum(1), k + 1, u),
                                 ("dw", (ye * s["dout"].double().abs()[:, None, :]).sum(2), D + 1, 0.0)):
        a, b = plain[name].double(), own[name].double()
        bound = 2 * c * 2.0 ** -24 * terms * (1 + unit) + 2 * unit * torch.maximum(a.abs(), b.abs()) + 2 * tiny
        assert bool(((a - b).abs() <= bound).all()), name


@pytest.mark.parametrize("case", [
    dict(op="linear", rows=3, N=300, K=517, group=32, zero=True, dtype="f16", act=1, bias=True),
    dict(op="linear", rows=40, N=264, K=1032, group=64, zero=False, dtype="bf16", act=0, bias=False),
    dict(op="experts", rows=60, E=9, active=4, N=200, K=384, group=128, zero=True, dtype="bf16", act=0, bias=True),
    dict(op="experts", rows=700, E=6, active=6, N=136, K=250, group=32, zero=False, dtype="f16", act=1, bias=True),
], ids=lambda c: f"{c['op']}-{c['rows']}")
def test_plain_products(case):
    m, s, plain, own = both(case, 9)
    N, K, group = case["N"], case["K"], case["group"]
    w = m._unpack(s["q"], s["scale"], s["zero"], N, K, group).double().abs()
    x = s["x"].double().abs()
    off = s["offsets"].long() if s["offsets"] is not None else torch.tensor([0, case["rows"]], device="cuda")
    terms = torch.zeros(case["rows"], N, dtype=torch.float64, device="cuda")
    for e in range(len(off) - 1):
        terms[off[e]:off[e + 1]] = x[off[e]:off[e + 1]] @ w[e].t() + (0 if s["bias"] is None else s["bias"][e].double().abs())
    u = torch.finfo(s["x"].dtype).eps / 2
    a, b = plain["y"].double(), own["y"].double()
    # the plain form rounds in a product's additions too: 2 K at most, as the kernel's
    slack = 2 * (2 * K + K // group + 12) * 2.0 ** -24 * terms
    assert bool(((a - b).abs() <= slack * (1 + u) + 2 * u * torch.maximum(a.abs(), b.abs()) + 2.0 ** -24).all())
