"""The expert stage behind the lookup: lookup -> interaction -> mixture of 4-bit experts -> top MLP.

``ExpertStage`` is the serving form: a gate (a linear layer) picks k of E experts for every row, rows are
sorted by expert and moved there, every expert answers with two linear layers whose weights are held in 4 bits,
and the answers come back as a weighted sum.  ``dispatch`` and ``combine`` are the two moves with their
gradients, for whoever trains a stage of their own around them.

    python examples/expert_stage.py        # one small loop on cuda:0
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2512_19342_b200 as bls  # noqa: E402


class Routes:
    """Where the slots of one batch go: order, place and offsets of bls_moe_route."""

    def __init__(self, expert: torch.Tensor, n_experts: int):
        n, k = expert.shape
        self.order = expert.new_empty(n * k)
        self.place = torch.empty_like(expert)
        self.offsets = expert.new_empty(n_experts + 1)
        bls.bls_moe_route(expert, n_experts, self.order, self.place, self.offsets)


def _first_derivative_only():
    """The kernels' results are constants to autograd: where a graph of the gradients is asked for, terms would be missing from it.
    (once_differentiable does not see this where only saved tensors need gradients.)"""
    if torch.is_grad_enabled():
        raise RuntimeError("dispatch and combine have first derivatives only: no create_graph")


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, routes):
        ctx.routes = routes
        y = x.new_empty(routes.place.numel(), x.shape[1])
        bls.bls_moe_dispatch(x, routes.place, routes.offsets, y)
        return y

    @staticmethod
    def backward(ctx, dy):
        _first_derivative_only()
        dx = dy.new_empty(ctx.routes.place.shape[0], dy.shape[1])
        bls.bls_moe_combine(dy.contiguous(), ctx.routes.place, None, dx)
        return dx, None


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, w, routes):
        ctx.save_for_backward(y, w)
        ctx.routes = routes
        out = y.new_empty(routes.place.shape[0], y.shape[1])
        bls.bls_moe_combine(y, routes.place, w, out)
        return out

    @staticmethod
    def backward(ctx, dout):
        _first_derivative_only()
        y, w = ctx.saved_tensors
        dy, dw = torch.empty_like(y), torch.empty_like(w)
        bls.bls_moe_combine_grad(dout.contiguous(), y, ctx.routes.place, ctx.routes.offsets, w, dy, dw)
        return dy, dw, None


def dispatch(x: torch.Tensor, routes: Routes) -> torch.Tensor:
    """Rows of x [n][D] at their sorted places [n * k][D]; differentiable once in x."""
    return _Dispatch.apply(x, routes)


def combine(y: torch.Tensor, w: torch.Tensor, routes: Routes) -> torch.Tensor:
    """Weighted sums [n][D] of the sorted rows y [n * k][D], w fp32 [n][k]; differentiable once in y and w."""
    return _Combine.apply(y, w, routes)


class ExpertStage:
    """gate bf16 [E][D]; up [E][H][D], down [E][O][H] of any type: they are put in 4 bits with a scale per `group` inputs."""

    def __init__(self, gate, up, up_bias, down, down_bias, k, max_rows, group=64):
        self.E, self.k = gate.shape[0], k
        self.gate = bls.Mlp([gate], [torch.zeros(self.E, device=gate.device)], 0, max_rows)
        self.up, self.down = (bls.bls_w4_quantize(w, group, symmetric=False) for w in (up, down))
        self.up_bias, self.down_bias = up_bias, down_bias

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        n = x.shape[0]
        logits = torch.empty(n, self.E, device=x.device)
        self.gate.forward(x, logits)
        top, expert = logits.topk(self.k, dim=1)
        routes = Routes(expert.to(torch.int32), self.E)
        w = torch.softmax(top, dim=1)
        rows = dispatch(x, routes)
        hidden = x.new_empty(rows.shape[0], self.up.N)
        bls.bls_w4_linear(self.up, rows, hidden, offsets=routes.offsets, bias=self.up_bias, act=1)
        answers = x.new_empty(rows.shape[0], self.down.N)
        bls.bls_w4_linear(self.down, hidden, answers, offsets=routes.offsets, bias=self.down_bias)
        return combine(answers, w, routes)


def main():
    import bls_inputs as bi
    import numpy as np

    torch.cuda.set_device(0)
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    w = bi.workload(3, 0.01, 0.02)                       # 26 tables, 8 ranks, 64-wide vectors, scaled down
    tables = [torch.from_numpy(bi.table_values(t)).cuda() for t in w.tables]
    P, T, b, D = w.P, w.T, w.local_batch, w.tables[0].dim
    B = P * b
    inputs = [bi.make_iteration(w, t) for t in range(4)]
    cap = max(int(np.diff(off[::T * b].astype(np.int64)).max()) for _, off in inputs) + 16
    plan = bls.bls_plan(tables, w.partition, P, b, 1, cap)
    width = (D + T * (T + 1) // 2 + 63) // 64 * 64       # interaction output, padded
    E, H, O = 16, 512, 256
    stage = ExpertStage((rnd(E, width) / width ** 0.5).to(torch.bfloat16), rnd(E, H, width) / width ** 0.5, 0.1 * rnd(E, H),
                        rnd(E, O, H) / H ** 0.5, 0.1 * rnd(E, O), 2, B)
    top = bls.Mlp([(rnd(8, O) / O ** 0.5).to(torch.bfloat16)], [torch.zeros(8, device="cuda")], 2, B)
    dense = torch.relu(rnd(B, D)).to(torch.bfloat16)     # stands for the bottom MLP's output
    r = torch.empty(B, width, dtype=torch.bfloat16, device="cuda")
    p = torch.empty(B, 8, device="cuda")
    done = 0

    def finish(pooled):
        bls.bls_interact(dense, 0.1 * pooled, r)
        top.forward(stage(r), p)

    for ids, off in inputs:
        out, _ = bls.bls_step(plan, 1, torch.from_numpy(ids).cuda(), torch.from_numpy(off).cuda())
        if out is not None:
            finish(out)
            done += 1
    while True:
        out, _ = bls.bls_drain(plan)
        if out is None:
            break
        finish(out)
        done += 1
    assert bls.bls_status(plan)[0] == top.status() == stage.gate.status() == bls.bls_w4_status() == bls.BLS_OK
    print(f"{done} batches of {B} samples through {E} experts, 2 each; probabilities of the first sample: "
          + " ".join(f"{float(v):.3f}" for v in p[0]))


if __name__ == "__main__":
    main()
