"""How the expert stage's calls treat their memory, streams and threads, beside what they compute.  GPU only."""
import os
import sys
import threading

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import expert_stage as ex  # noqa: E402
import paper_2512_19342_b200 as bls  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Step:
    """Routing, moves, a product and the gradient of one batch large enough that routing and the product need scratch memory: 8000
    slots, and rows of x that do not start at 16-byte boundaries."""
    n, k, E, D, N = 2000, 4, 16, 257, 136

    def __init__(self, seed):
        g = gen(seed)
        self.expert = torch.randint(-1, self.E, (self.n, self.k), device="cuda", generator=g, dtype=torch.int32)
        self.w4 = bls.bls_w4_quantize(torch.randn(self.E, self.N, self.D, device="cuda", generator=g), 32, False)
        self.x = torch.randn(self.n, self.D, device="cuda", generator=g).to(BF16)
        self.w = torch.rand(self.n, self.k, device="cuda", generator=g)
        R = self.n * self.k
        self.routes = [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((R,), (self.n, self.k), (self.E + 1,))]
        self.rows, self.y = (torch.zeros(R, d, dtype=BF16, device="cuda") for d in (self.D, self.N))
        self.out, self.dy, self.dw = torch.zeros(self.n, self.N, dtype=BF16, device="cuda"), torch.zeros_like(self.y), torch.zeros_like(self.w)
        assert R > 4096 and R > 8 * self.E and self.D % 8

    def __call__(self, stream=None, between=lambda: None):
        _, place, offsets = self.routes
        bls.bls_moe_route(self.expert, self.E, *self.routes, stream=stream)
        between()
        bls.bls_moe_dispatch(self.x, place, offsets, self.rows, stream=stream)
        bls.bls_w4_linear(self.w4, self.rows, self.y, offsets=offsets, stream=stream)
        between()
        bls.bls_moe_combine(self.y, place, self.w, self.out, stream=stream)
        bls.bls_moe_combine_grad(self.out, self.y, place, offsets, self.w, self.dy, self.dw, stream=stream)

    def results(self):
        return [t.clone() for t in (*self.routes, self.rows, self.y, self.out, self.dy, self.dw)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_scratch_memory_belongs_to_the_call_s_stream():
    """A call returns before its kernels run.  Memory that the caller takes then, on another stream, and clears must not be the call's own."""
    step, s = Step(1), torch.cuda.Stream()
    sizes = [1 << p for p in range(9, 23)] + [step.n * step.k * 264 * 2]

    def clear():
        for n in sizes:
            torch.zeros(n, dtype=torch.uint8, device="cuda")

    step()
    want = step.results()
    step(s, clear)                                            # the allocator has memory for all of it from here on, and asks the driver for none
    torch.cuda.synchronize()
    held = False
    for _ in range(3):
        for t in (*step.routes, step.rows, step.y, step.out, step.dy, step.dw):
            t.fill_(-3)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(400_000_000)                    # 0.2 s
        step(s, clear)
        clear()
        held = held or not s.query()                          # everything was enqueued while the stream was held up
        torch.cuda.synchronize()
        assert same(step.results(), want)
    assert bls.bls_w4_status() == bls.BLS_OK
    if not held:
        pytest.skip("the host was too slow to enqueue the calls within 0.2 s")


def test_scratch_memory_in_a_cuda_graph():
    step = Step(2)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (3, 4):
        step.expert.copy_(Step(seed).expert)
        junk = [torch.full((1 << p,), 255, dtype=torch.uint8, device="cuda") for p in range(9, 23)]
        graph.replay()
        got = step.results()
        step()
        assert same(step.results(), got)
        del junk
    assert bls.bls_w4_status() == bls.BLS_OK


def test_calls_from_several_threads():
    """Each thread on a stream of its own; the answers are those of one thread alone."""
    steps = [Step(10 + i) for i in range(4)]
    want = []
    for step in steps:
        step()
        torch.cuda.synchronize()
        want.append(step.results())
    bad, start = [], threading.Barrier(len(steps))

    def work(step, ref):
        s = torch.cuda.Stream()
        start.wait()
        for _ in range(20):
            with torch.cuda.stream(s):
                step()
                ok = same(step.results(), ref)
            if not ok:
                bad.append(step)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=a) for a in zip(steps, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad and bls.bls_w4_status() == bls.BLS_OK


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
