"""The expert stage on the GPU (slots sorted by expert, rows moved there and back with the gradients, products
with 4-bit weights, quantisation) against plain 64-bit references, through the public calls.  GPU only.

Tolerances are bounds, not fits.  With u = the unit roundoff of the output type (2^-24, 2^-8, 2^-11 for fp32, bf16 and
f16: half the spacing at 1, plus half the spacing of its subnormals) a result that is summed in fp32 and rounded once is off by at most
u |result| + c 2^-24 sum|terms|, c = the number of roundings on the longest path of the sum.  The matrix
instructions may truncate instead of rounding, so products with weights count every addition twice."""
import ctypes as C
import zlib

import numpy as np
import pytest
import torch

import paper_2512_19342_b200 as bls

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
UNIT = {t: torch.finfo(t).eps / 2 for t in (F32, BF16, F16)}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -134, F16: 2.0 ** -25}


def close(got, want, terms, c):
    """|got - want| within one rounding to got's type plus c fp32 roundings of a sum whose terms' magnitudes add up to `terms`."""
    u = UNIT[got.dtype]
    slack = c * 2.0 ** -24 * terms
    bound = u * (want.abs() + slack) + slack + TINY[got.dtype]
    off = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all()
    assert bool((off <= bound).all()), float((off / bound).max())


def gen(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def experts(g, n, k, E, left_out):
    e = torch.randint(0, E, (n, k), device="cuda", generator=g, dtype=torch.int32)      # the same expert twice is allowed
    out = torch.rand(n, k, device="cuda", generator=g) < left_out
    odd = torch.where(torch.rand(n, k, device="cuda", generator=g) < 0.5, -1, E + 5).to(torch.int32)
    return torch.where(out, odd, e)


def route_by_numpy(expert, E):
    flat = expert.cpu().numpy().reshape(-1)
    kept = np.nonzero((flat >= 0) & (flat < E))[0]
    by = kept[np.argsort(flat[kept], kind="stable")]
    order = np.full(flat.size, -1, np.int32)
    order[:by.size] = by
    place = np.full(flat.size, -1, np.int32)
    place[by] = np.arange(by.size)
    offsets = np.searchsorted(flat[by], np.arange(E + 1)).astype(np.int32)
    return order, place.reshape(tuple(expert.shape)), offsets


def route(expert, E, stream=None):
    n, k = expert.shape
    o = [torch.full(s, -77, dtype=torch.int32, device="cuda") for s in ((n * k,), (n, k), (E + 1,))]
    bls.bls_moe_route(expert, E, *o, stream=stream)
    return o


@pytest.mark.parametrize("n,k,E,left_out", [
    (0, 2, 5, 0.0), (1, 1, 1, 0.0), (1, 1, 1, 1.0), (1, 8, 64, 0.0), (3, 5, 1000, 0.2), (31, 1, 2, 0.5), (33, 3, 7, 0.0),
    (129, 8, 1024, 0.1), (1000, 4, 32, 0.0), (5000, 1, 3, 0.9), (4097, 6, 257, 0.03), (20000, 8, 256, 0.02), (70001, 8, 64, 0.0),
    (2049, 1, 1, 0.0), (1500, 1024, 16, 0.5), (300000, 2, 1024, 0.01), (9000, 7, 33, 1.0),
])
def test_route_is_the_stable_sort(n, k, E, left_out):
    e = experts(gen(n, k, E), n, k, E, left_out)
    for _ in range(2):                                   # the same twice: no state is kept, nothing depends on timing
        got = route(e, E)
        for a, b in zip(got, route_by_numpy(e, E)):
            assert np.array_equal(a.cpu().numpy(), b)


def test_route_of_one_expert_and_of_sorted_and_reversed_experts():
    for e in (torch.zeros(10000, 2), torch.arange(20000).reshape(10000, 2) // 100, torch.arange(19999, -1, -1).reshape(10000, 2) // 100):
        e = e.to(torch.int32).cuda()
        got = route(e, 200)
        for a, b in zip(got, route_by_numpy(e, 200)):
            assert np.array_equal(a.cpu().numpy(), b)


def pitched(t, pad, shift=0):
    """The same matrix with rows `pad` elements further apart, starting `shift` elements into its memory."""
    buf = torch.full((t.shape[0] * (t.shape[1] + pad) + shift,), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[shift:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    v.copy_(t)
    return v


MOVES = [
    # n, k, E, D, left_out, pad, shift
    (1, 1, 1, 1, 0.0, 0, 0), (1, 8, 64, 128, 0.0, 0, 0), (16, 4, 8, 1024, 0.1, 0, 0), (7, 3, 5, 33, 0.3, 0, 0),
    (130, 2, 4, 264, 0.2, 8, 0), (65, 6, 16, 100, 0.1, 4, 1), (513, 4, 8, 1531, 0.0, 1, 3), (33, 17, 40, 72, 0.5, 0, 8),
    (40, 2, 3, 4096, 0.0, 0, 0), (9, 1, 4, 9000, 0.0, 0, 0), (3, 2, 4, 20000, 0.2, 0, 0), (50, 2, 4, 64, 1.0, 0, 0),
]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,k,E,D,left_out,pad,shift", MOVES)
def test_moves_and_their_gradients(dtype, n, k, E, D, left_out, pad, shift):
    g = gen(n, k, E, D)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    e = experts(g, n, k, E, left_out)
    if n > 2:
        e[n // 2] = -1                                   # a token without any expert
    _, place, offsets = route(e, E)
    total, R = int(offsets[-1]), n * k
    x, ye, dout, dxs = (pitched(rnd(r, D).to(dtype), pad, shift) for r in (n, R, n, R))
    ye[total:] = float("nan")                           # rows of nobody are not read
    dxs[total:] = float("nan")
    w = rnd(n, k)
    w[place < 0] = float("nan")                          # nor is the weight of a slot without a place
    keep = (place >= 0)
    at = place.clamp(min=0).long()

    xs = pitched(torch.full((R, D), 7.0, device="cuda").to(dtype), pad, shift)
    bls.bls_moe_dispatch(x, place, offsets, xs)
    want = torch.zeros(R, D, dtype=dtype, device="cuda")
    want[at[keep]] = x[:, None, :].expand(n, k, D)[keep]
    assert torch.equal(xs, want)

    out = pitched(torch.zeros(n, D, device="cuda").to(dtype), pad, shift)
    bls.bls_moe_combine(ye, place, w, out)
    t = torch.where(keep[..., None], ye[at].double() * w[..., None].double(), 0.0)
    close(out, t.sum(1), t.abs().sum(1), k + 1)
    assert torch.all(out[~keep.any(1)] == 0)

    dx = torch.empty(n, D, dtype=dtype, device="cuda")
    bls.bls_moe_combine(dxs, place, None, dx)
    t = torch.where(keep[..., None], dxs[at].double(), 0.0)
    close(dx, t.sum(1), t.abs().sum(1), k + 1)

    for weights in (w, None):
        dye = pitched(torch.full((R, D), 7.0, device="cuda").to(dtype), pad, shift)
        dw = torch.full((n, k), 7.0, device="cuda")
        bls.bls_moe_combine_grad(dout, ye, place, offsets, weights, dye, dw)
        wt = w.double() if weights is not None else torch.ones(n, k, device="cuda", dtype=torch.float64)
        t = wt[..., None] * dout[:, None, :].double()
        want = torch.zeros(R, D, dtype=torch.float64, device="cuda")
        want[at[keep]] = t[keep]
        close(dye, want, want.abs(), 1)
        assert torch.all(dye[total:] == 0)
        t = torch.where(keep[..., None], ye[at].double() * dout[:, None, :].double(), 0.0)
        close(dw, t.sum(2), t.abs().sum(2), D + 1)
        assert torch.all(dw[~keep] == 0)
        only = pitched(torch.full((R, D), 7.0, device="cuda").to(dtype), pad, shift)
        bls.bls_moe_combine_grad(dout, None, place, offsets, weights, only)          # without dw, y is not needed
        assert torch.equal(only, dye)


def test_gradients_against_differences():
    """loss = <dout, combine(y, w)> is linear in y and in w: a central difference of step h is the derivative up to the rounding of
    the two fp32 evaluations, at most (k + 2) 2^-24 sum|terms| / h each."""
    n, k, E, D = 6, 3, 4, 20
    g = gen("differences")
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    e = experts(g, n, k, E, 0.2)
    _, place, offsets = route(e, E)
    y, w, dout = rnd(n * k, D), rnd(n, k), rnd(n, D)
    dy, dw = torch.empty_like(y), torch.empty_like(w)
    bls.bls_moe_combine_grad(dout, y, place, offsets, w, dy, dw)

    def loss(y, w):
        out = torch.empty(n, D, device="cuda")
        bls.bls_moe_combine(y, place, w, out)
        return float((out.double() * dout.double()).sum())

    h = 0.25
    at, keep = place.clamp(min=0).long(), place >= 0
    size = float(torch.where(keep[..., None], (y[at].abs() + h) * (w.abs()[..., None] + h) * dout.abs()[:, None, :], 0.0).double().sum())
    tol = 2 * (k + 2) * 2.0 ** -24 * size / (2 * h) + 2.0 ** -20
    for t in range(n):
        for i in range(k):
            d = torch.zeros_like(w)
            d[t, i] = h
            assert abs((loss(y, w + d) - loss(y, w - d)) / (2 * h) - float(dw[t, i])) <= tol
    for r in range(0, n * k, 3):
        for c in range(0, D, 7):
            d = torch.zeros_like(y)
            d[r, c] = h
            assert abs((loss(y + d, w) - loss(y - d, w)) / (2 * h) - float(dy[r, c])) <= tol
    x, dxs = rnd(n, D), rnd(n * k, D)

    def loss_x(x):
        xs = torch.empty(n * k, D, device="cuda")
        bls.bls_moe_dispatch(x, place, offsets, xs)
        return float((xs.double() * dxs.double()).sum())

    dx = torch.empty_like(x)
    bls.bls_moe_combine(dxs, place, None, dx)
    for t in range(n):
        d = torch.zeros_like(x)
        d[t, 3 * t] = h
        tol = 2 * (k + 2) * 2.0 ** -24 * float((dxs.abs().sum() + 1) * (x.abs().max() + h)) / (2 * h)
        assert abs((loss_x(x + d) - loss_x(x - d)) / (2 * h) - float(dx[t, 3 * t])) <= tol


def test_moves_past_two_to_the_31_elements():
    n, k, E, D = 4200, 8, 4, 65536                       # 33 600 rows x 65 536: 2.2e9 elements
    g = gen("far")
    e = experts(g, n, k, E, 0.01)
    _, place, offsets = route(e, E)
    total = int(offsets[-1])
    x = torch.randn(n, D, device="cuda", generator=g).to(BF16)
    xs = torch.empty(n * k, D, dtype=BF16, device="cuda")
    bls.bls_moe_dispatch(x, place, offsets, xs)
    keep, at = place >= 0, place.clamp(min=0).long()
    for t in (0, 1, n // 2, n - 1):
        for i in range(k):
            if keep[t, i]:
                assert torch.equal(xs[at[t, i]], x[t])
    assert torch.all(xs[total:] == 0) and total < n * k
    out = torch.empty_like(x)
    bls.bls_moe_combine(xs, place, None, out)            # count * x, rounded once: exact in fp32 up to k = 8
    want = (x.float() * keep.sum(1, keepdim=True).float()).to(BF16)
    assert torch.equal(out, want)
    dw = torch.empty(n, k, device="cuda")
    bls.bls_moe_combine_grad(x, xs, place, offsets, None, xs.new_empty(xs.shape), dw)
    sq = (x.double() ** 2).sum(1, keepdim=True)
    close(dw, torch.where(keep, sq, 0.0), torch.where(keep, sq, 0.0), D + 1)


# ---------------------------------------------------------------------------------------- 4-bit weights

def padded(t):
    return (t + 127) // 128 * 128


def quantize_by_numpy(w, group, symmetric):
    """q [E][N][Kp], scale and zero [E][N][groups] by the documented rule (fp32 quotients)."""
    w = w.float().cpu().numpy()
    E, N, K = w.shape
    f = np.zeros((E, N, padded(K)), np.float32)
    f[:, :, :K] = w
    f = f.reshape(E, N, -1, group)
    with np.errstate(all="ignore"):
        lo, hi = np.minimum(f.min(3), 0), np.maximum(f.max(3), 0)
        s = (np.maximum(hi, -lo) / np.float32(7)) if symmetric else (hi - lo) / np.float32(15)
        s = torch.from_numpy(s.astype(np.float32)).to(BF16)
        s[torch.from_numpy(~np.isfinite(f).all(3))] = float("nan")
        s32 = s.float().numpy()
        ok = (s32 > 0) & np.isfinite(s32)
        z = np.full(s32.shape, 8, np.float32) if symmetric else np.where(ok, np.clip(np.rint(-lo / s32), 0, 15), 0)
        q = np.where(ok[..., None], np.rint(f / s32[..., None]), 0)
        q = np.clip(q + z[..., None], 0, 15)
    return q.reshape(E, N, -1).astype(np.int64), s, z.astype(np.int64)


def stored_q(q, E, N, K):
    """Reads q[e][n][k] out of the storage, element by element by its address."""
    flat = q.cpu().numpy().reshape(E, -1)
    kt = padded(K) // 128
    n, k = np.arange(N)[:, None], np.arange(padded(K))[None, :]
    r, i = n % 128, k % 8
    t, b = k % 128 // 8 % 4, k % 128 // 32
    j = i // 2 + 4 * (i % 2)
    at = ((n // 128) * kt + k // 128) * 8192 + r * 64 + (t ^ ((r >> 1) & 3)) * 16 + 4 * b + j // 2
    return (flat[:, at] >> (4 * (j % 2)))[..., :] & 15


W4_SHAPES = [(1, 1, 1), (1, 128, 128), (2, 100, 31), (1, 129, 257), (3, 300, 640), (1, 17, 96), (2, 256, 1000)]


@pytest.mark.parametrize("symmetric", [True, False], ids=["symmetric", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("E,N,K", W4_SHAPES)
def test_quantize_and_back(E, N, K, dtype, group, symmetric):
    w = (torch.randn(E, N, K, device="cuda", generator=gen(E, N, K)) * 0.3).to(dtype)
    w[0, 0, :] = 0                                        # a group of zeros
    if N > 3:
        w[0, 1, :] = w[0, 1, :].abs()                     # one sign only
        w[0, 2, :] *= 1e-4
    t = bls.bls_w4_quantize(w, group, symmetric)
    q, s, z = quantize_by_numpy(w, group, symmetric)
    assert np.array_equal(stored_q(t.q, E, N, K), q)
    assert torch.equal(t.scale[:, :, :N].transpose(1, 2).cpu(), s)
    assert torch.all(t.scale[:, :, N:] == 0)
    if not symmetric:
        assert np.array_equal(t.zero[:, :, :N].transpose(1, 2).cpu().numpy(), z)
    exact = (q.reshape(E, N, -1, group) - z[..., None]) * s.double().numpy()[..., None]
    exact = torch.from_numpy(exact.reshape(E, N, -1)[:, :, :K])
    for out in (F32, BF16, F16):
        back = torch.full((E, N, K + 3), float("nan"), dtype=out, device="cuda")
        bls.bls_w4_dequantize(t, back[:, :, :K])
        assert torch.equal(back[:, :, :K].cpu(), exact.float().to(out))
        assert torch.isnan(back[:, :, K:]).all()
    # half a step, a quarter more where the rounded scale or zero point cuts the range short
    step = torch.from_numpy(np.repeat(s.double().numpy(), group, axis=2)[:, :, :K])
    off = (exact - w.double().cpu()).abs()
    assert bool((off <= 0.75 * step + 1e-30).all()) if symmetric else bool((off <= 1.25 * step + 1e-30).all())
    pitch = torch.full((E, N, K + 5), float("nan"), dtype=dtype, device="cuda")
    pitch[:, :, :K] = w
    t2 = bls.bls_w4_quantize(pitch[:, :, :K], group, symmetric)
    assert torch.equal(t2.q, t.q) and torch.equal(t2.scale, t.scale)


def test_quantize_marks_groups_that_are_not_finite():
    w = torch.randn(40, 128, device="cuda", generator=gen("nan"))
    w[3, 5], w[4, 40], w[5, 127] = float("nan"), float("inf"), -float("inf")
    for symmetric in (True, False):
        t = bls.bls_w4_quantize(w, 32, symmetric)
        back = torch.empty_like(w)
        bls.bls_w4_dequantize(t, back)
        bad = torch.isnan(back)
        want = torch.zeros_like(bad)
        want[3, 0:32] = want[4, 32:64] = want[5, 96:128] = True
        assert torch.equal(bad, want)


def weights(g, E, N, K, group, symmetric):
    """A W4 and its weights in 64 bits."""
    w = torch.randn(E, N, K, device="cuda", generator=g)
    t = bls.bls_w4_quantize(w, group, symmetric)
    back = torch.empty_like(w)
    bls.bls_w4_dequantize(t, back)
    return t, back.double()


def check_linear(t, w, x, offsets, bias, act, y_dtype, y=None, **kw):
    rows, K = x.shape
    E, N = w.shape[:2]
    if y is None:
        y = torch.full((rows, N), float("nan"), dtype=y_dtype, device="cuda")
    bls.bls_w4_linear(t, x, y, offsets=offsets, bias=bias, act=act, **kw)
    ends = [0, rows] if offsets is None else offsets.tolist()
    assert bls.bls_w4_status() == bls.BLS_OK
    want = torch.zeros(rows, N, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        want[a:b] = x[a:b].double() @ w[e].t()
        size[a:b] = x[a:b].double().abs() @ w[e].abs().t()
        if bias is not None:
            want[a:b] += bias[e].double()
            size[a:b] += bias[e].double().abs()
    live = ends[-1]
    want = want.clamp(min=0) if act == 1 else torch.sigmoid(want) if act == 2 else want
    extra = 8.0 if act == 2 else 0.0                      # the logistic function itself: a few fp32 roundings of a value up to 1
    if live:
        close(y[:live], want[:live], size[:live] + extra, 2 * K + t.K // t.group + 12)
    assert torch.all(y[live:] == 0)
    return y


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 127, 130, 300])
@pytest.mark.parametrize("N,K,group,symmetric,dtype", [
    (256, 512, 128, True, BF16), (300, 640, 64, False, BF16), (129, 257, 32, False, F16), (1, 1, 32, True, BF16),
    (100, 31, 128, False, F16), (17, 1031, 64, True, F16), (520, 136, 32, True, BF16),
])
def test_linear_matches_the_definition(rows, N, K, group, symmetric, dtype):
    g = gen(rows, N, K)
    t, w = weights(g, 1, N, K, group, symmetric)
    x = torch.randn(rows, K, device="cuda", generator=g).to(dtype)
    bias = torch.randn(1, N, device="cuda", generator=g)
    act = rows % 3
    check_linear(t, w, x, None, bias if rows % 2 else None, act, dtype)
    check_linear(t, w, x, None, bias, 0, F32)
    y = pitched(torch.zeros(rows, N, device="cuda").to(dtype), 5, 3)      # other pitches and bases on both sides
    check_linear(t, w, pitched(x, 3, 1), None, bias, act, dtype, y=y)
    check_linear(t, w, pitched(x, 8, 8), None, None, 0, F16 if dtype == BF16 else BF16)


@pytest.mark.parametrize("counts", [
    [1, 0, 0, 0, 0, 0, 0, 1], [0, 0, 0, 0], [3, 5, 0, 8, 1], [40, 0, 1, 129, 64], [0, 0, 300], [128, 128, 256], [1] * 40,
    [17, 0, 200, 33, 2, 0, 70, 0, 0, 9],
], ids=str)
@pytest.mark.parametrize("tail", [0, 13])
@pytest.mark.parametrize("N,K,group,symmetric,dtype", [(256, 384, 64, False, BF16), (133, 200, 32, True, F16), (96, 1003, 128, False, BF16)])
def test_linear_by_experts(counts, tail, N, K, group, symmetric, dtype):
    E, rows = len(counts), sum(counts) + tail
    g = gen(str(counts), tail, N)
    t, w = weights(g, E, N, K, group, symmetric)
    x = torch.randn(rows, K, device="cuda", generator=g).to(dtype)
    x[rows - tail:] = float("nan")                        # rows of no expert are not read into anybody's answer
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    bias = torch.randn(E, N, device="cuda", generator=g)
    check_linear(t, w, x, offsets, bias, 1, dtype)
    check_linear(t, w, x, offsets, None, 0, F32)


def test_linear_is_exact_on_whole_numbers():
    """Scale 1, integer x: every product and sum is a small integer, so the answer has no rounding at all; a permutation
    matrix shows that no row or input is misplaced."""
    for rows in (1, 20, 200):
        for dtype in (BF16, F16):
            N = K = 384
            g = gen("exact", rows)
            q = torch.randint(-7, 8, (1, N, K), device="cuda", generator=g).float()
            q[:, :, ::32] = 7.0                           # every group reaches 7: the scale is exactly 1
            t = bls.bls_w4_quantize(q, 32)
            x = torch.randint(-3, 4, (rows, K), device="cuda", generator=g).to(dtype)
            y = torch.empty(rows, N, device="cuda")
            bls.bls_w4_linear(t, x, y)
            assert torch.equal(y.double(), x.double() @ q[0].double().t())
            perm = torch.randperm(N, device="cuda", generator=g)
            p = torch.zeros(N, K, device="cuda")
            p[torch.arange(N, device="cuda"), perm] = 7.0
            x = torch.randn(rows, K, device="cuda", generator=g).to(dtype)
            bls.bls_w4_linear(bls.bls_w4_quantize(p, 32), x, y)
            assert torch.equal(y, 7.0 * x.float()[:, perm])


def test_linear_keeps_infinities_and_nans_in_their_rows():
    for rows in (5, 200):
        g = gen("inf", rows)
        t, w = weights(g, 1, 200, 300, 64, True)
        x = torch.randn(rows, 300, device="cuda", generator=g).to(BF16)
        y0, y1 = (torch.empty(rows, 200, dtype=BF16, device="cuda") for _ in range(2))
        bls.bls_w4_linear(t, x, y0)
        x[1, 7], x[3, 299] = float("nan"), float("inf")
        bls.bls_w4_linear(t, x, y1)
        assert torch.isnan(y1[1]).all() and not torch.isfinite(y1[3].float()).any()
        rest = [r for r in range(rows) if r not in (1, 3)]
        assert torch.equal(y1[rest], y0[rest])
        bls.bls_w4_linear(t, x, y1, act=1)
        assert torch.isnan(y1[1]).all()                   # ReLU keeps a NaN


def test_same_inputs_same_bits():
    g = gen("again")
    for rows, N, K in ((3, 512, 2048), (40, 256, 1024), (700, 384, 640)):
        t, _ = weights(g, 1, N, K, 64, False)
        x = torch.randn(rows, K, device="cuda", generator=g).to(BF16)
        ys = [torch.empty(rows, N, dtype=BF16, device="cuda") for _ in range(4)]
        for y in ys:
            bls.bls_w4_linear(t, x, y)
        assert all(torch.equal(ys[0], y) for y in ys[1:])


def test_on_another_stream():
    """Everything runs on the stream that is given, after what was enqueued there, and its scratch memory belongs to that stream."""
    s = torch.cuda.Stream()
    n, k, E, D = 600, 4, 16, 256
    g = gen("stream")
    e = experts(g, n, k, E, 0.1)
    t, w = weights(g, E, 192, D, 32, True)
    x = torch.randn(n, D, device="cuda", generator=g).to(BF16)
    wt = torch.rand(n, k, device="cuda", generator=g)
    torch.cuda.synchronize()
    res = []
    for stream in (None, s, s):
        o = [torch.empty(v, dtype=torch.int32, device="cuda") for v in ((n * k,), (n, k), (E + 1,))]
        xs, y = (torch.empty(n * k, d, dtype=BF16, device="cuda") for d in (D, 192))
        out, dy, dw = torch.empty(n, 192, dtype=BF16, device="cuda"), torch.empty_like(y), torch.empty_like(wt)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            late = x.clone() if stream is not None else None
            if late is not None:
                torch.cuda._sleep(2_000_000)
                late.copy_(x)
        src = x if late is None else late
        bls.bls_moe_route(e, E, *o, stream=stream)
        bls.bls_moe_dispatch(src, o[1], o[2], xs, stream=stream)
        bls.bls_w4_linear(t, xs, y, offsets=o[2], stream=stream)
        bls.bls_moe_combine(y, o[1], wt, out, stream=stream)
        bls.bls_moe_combine_grad(out, y, o[1], o[2], wt, dy, dw, stream=stream)
        torch.cuda.synchronize()
        res.append([*o, xs, y, out, dy, dw])
    for other in res[1:]:
        for a, b in zip(res[0], other):
            assert torch.equal(a, b)


def test_in_a_cuda_graph():
    n, k, E, D = 300, 2, 8, 128
    g = gen("graph")
    t, _ = weights(g, E, 128, D, 64, False)
    e, x, wt = experts(g, n, k, E, 0.0), torch.randn(n, D, device="cuda", generator=g).to(BF16), torch.rand(n, k, device="cuda", generator=g)
    o = [torch.empty(v, dtype=torch.int32, device="cuda") for v in ((n * k,), (n, k), (E + 1,))]
    xs, y, out = torch.empty(n * k, D, dtype=BF16, device="cuda"), torch.empty(n * k, 128, dtype=BF16, device="cuda"), torch.empty(n, 128, dtype=BF16, device="cuda")

    def step():
        bls.bls_moe_route(e, E, *o)
        bls.bls_moe_dispatch(x, o[1], o[2], xs)
        bls.bls_w4_linear(t, xs, y, offsets=o[2])
        bls.bls_moe_combine(y, o[1], wt, out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2):
        e.copy_(experts(gen("graph", seed), n, k, E, 0.2))
        graph.replay()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
    assert bls.bls_w4_status() == bls.BLS_OK


# ---------------------------------------------------------------------------------------- refusals

def test_calls_refuse_bad_arguments():
    lib = bls.lib()
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    f = lambda *s: torch.zeros(*s, device="cuda")
    place, off = i32(4, 2), i32(9)
    for call in (
        lambda: bls.bls_moe_route(i32(4), 8, i32(8), place, off),                        # not [tokens][k]
        lambda: bls.bls_moe_route(f(4, 2), 8, i32(8), place, off),                       # not whole numbers
        lambda: bls.bls_moe_route(i32(4, 4)[:, ::2], 8, i32(8), place, off),             # strided IDs
        lambda: bls.bls_moe_route(i32(4, 2), 8, i32(7), place, off),                     # order too short
        lambda: bls.bls_moe_route(i32(4, 2), 8, i32(8), place, i32(8)),                  # offsets too short
        lambda: bls.bls_moe_route(torch.zeros(4, 2, dtype=torch.int32), 8, i32(8), place, off),      # not on the GPU
        lambda: bls.bls_moe_dispatch(f(4, 16), place, off, f(8, 15)),                    # another width
        lambda: bls.bls_moe_dispatch(f(4, 16), place, off, f(8, 16).half()),             # another type
        lambda: bls.bls_moe_dispatch(f(5, 16), place, off, f(8, 16)),                    # another number of tokens
        lambda: bls.bls_moe_dispatch(f(4, 32)[:, ::2], place, off, f(8, 16)),            # columns apart
        lambda: bls.bls_moe_combine(f(8, 16), place, f(4, 3), f(4, 16)),                 # weights of another shape
        lambda: bls.bls_moe_combine(f(8, 16), place, f(4, 2).half(), f(4, 16)),          # weights are fp32
        lambda: bls.bls_moe_combine_grad(f(4, 16), None, place, off, None, f(8, 16), f(4, 2)),       # dw needs y
        lambda: bls.bls_moe_combine_grad(f(4, 16), f(7, 16), place, off, None, f(8, 16), f(4, 2)),   # y and dy differ
        lambda: bls.bls_w4_quantize(f(16, 16), 48),
        lambda: bls.bls_w4_quantize(f(16, 32)[:, ::2], 32),
        lambda: bls.bls_w4_quantize(torch.zeros(16, 16, device="cuda", dtype=torch.float64), 32),
    ):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(bls.BlsError) as err:
        bls.bls_moe_route(i32(4, 2), 1025, i32(8), place, i32(1026))
    assert err.value.code == bls.BLS_EINVAL
    with pytest.raises(bls.BlsError):
        bls.bls_moe_route(i32(1, 1025), 8, i32(1025), i32(1, 1025), off)
    t = bls.bls_w4_quantize(f(2, 40, 64), 32)
    x, y = f(5, 64).half(), f(5, 40)
    o3 = i32(3)
    for call in (
        lambda: bls.bls_w4_linear(t, x, y),                                              # two matrices, no offsets
        lambda: bls.bls_w4_linear(t, x.float(), y, offsets=o3),                          # fp32 x
        lambda: bls.bls_w4_linear(t, f(5, 63).half(), y, offsets=o3),
        lambda: bls.bls_w4_linear(t, x, f(5, 41), offsets=o3),
        lambda: bls.bls_w4_linear(t, x, f(6, 40), offsets=o3),
        lambda: bls.bls_w4_linear(t, x, y, offsets=i32(2)),
        lambda: bls.bls_w4_linear(t, x, y, offsets=o3, bias=f(1, 40)),
        lambda: bls.bls_w4_dequantize(t, f(2, 40, 63)),
        lambda: bls.W4(t.q, t.scale[:, :1], None, 40, 64, 32),
        lambda: bls.W4(t.q.float(), t.scale, None, 40, 64, 32),
        lambda: bls.W4(t.q, t.scale, None, 40, 64, 16),
    ):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(bls.BlsError):
        bls.bls_w4_linear(t, x, y, offsets=o3, act=3)
    n = C.c_size_t(0)
    assert lib.bls_moe_bytes(-1, 2, 8, C.byref(n)) == bls.BLS_EINVAL
    assert lib.bls_moe_bytes(1 << 30, 2, 8, C.byref(n)) == bls.BLS_EINVAL
    assert lib.bls_w4_bytes(1, 8, 0, None, 8, 5, C.byref(n)) == bls.BLS_EINVAL
    assert bls.bls_w4_sizes(2, 129, 130, 64) == (2 * 2 * 2 * 8192, 2 * 2 * 2 * 2 * 128)
    # a misaligned q and a missing status word are refused by the library itself
    p = t._args
    args = lambda q, st: (q, p[1], None, 2, 40, 64, 32, x.data_ptr(), 2, 64, 5, o3.data_ptr(), None, 0, y.data_ptr(), 0, 40, None, 0, st, None)
    assert lib.bls_w4_linear(*args(p[0] + 8, o3.data_ptr())) == bls.BLS_EINVAL
    assert lib.bls_w4_linear(*args(p[0], None)) == bls.BLS_EINVAL
    assert torch.ones(4, device="cuda").sum().item() == 4.0


def test_empty_calls():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    o = route(i32(0, 3), 4)
    assert torch.equal(o[2], i32(5))
    f = lambda *s: torch.ones(*s, device="cuda")
    bls.bls_moe_dispatch(f(0, 8), o[1], o[2], f(0, 8))
    y = f(6, 8)
    bls.bls_moe_dispatch(f(0, 8), o[1], o[2], y)                                         # room for rows that nobody sends
    assert torch.all(y == 0)
    bls.bls_moe_combine(f(0, 8), o[1], f(0, 3), f(0, 8))
    bls.bls_moe_combine_grad(f(0, 8), f(0, 8), o[1], o[2], None, f(0, 8), f(0, 3))
    t = bls.bls_w4_quantize(f(16, 32), 32)
    bls.bls_w4_linear(t, f(0, 32).half(), f(0, 16))
    torch.cuda.synchronize()


def test_places_past_the_rows_are_left_out():
    """A caller's y may have fewer rows than slots (a capacity): slots placed past it are dropped everywhere."""
    n, k, E, D, cap = 40, 2, 4, 24, 50
    g = gen("cap")
    e = experts(g, n, k, E, 0.0)
    _, place, offsets = route(e, E)
    x = torch.randn(n, D, device="cuda", generator=g)
    xs = torch.empty(cap, D, device="cuda")
    bls.bls_moe_dispatch(x, place, offsets, xs)
    full = torch.empty(n * k, D, device="cuda")
    bls.bls_moe_dispatch(x, place, offsets, full)
    assert torch.equal(xs, full[:cap])
    out = torch.empty(n, D, device="cuda")
    bls.bls_moe_combine(xs, place, None, out)
    kept = (place >= 0) & (place < cap)
    close(out, x.double() * kept.sum(1, keepdim=True), x.double().abs() * k, k)
    dw = torch.empty(n, k, device="cuda")
    bls.bls_moe_combine_grad(x, xs, place, offsets, None, torch.empty_like(xs), dw)
    assert torch.all(dw[~kept] == 0)


@pytest.mark.parametrize("rows,N,K,group,symmetric,dtype", [
    (300, 25000, 264, 64, False, BF16), (513, 20000, 130, 32, True, F16), (1000, 12800, 128, 128, True, BF16), (256, 38000, 96, 32, False, BF16),
])
def test_linear_of_many_outputs(rows, N, K, group, symmetric, dtype):
    """Enough tiles for those of 256 rows: whole ones, and ends inside the first and the second half."""
    g = gen(rows, N, K)
    t, w = weights(g, 1, N, K, group, symmetric)
    x = torch.randn(rows, K, device="cuda", generator=g).to(dtype)
    check_linear(t, w, x, None, torch.randn(1, N, device="cuda", generator=g), 1, dtype)


def test_linear_by_experts_of_many_rows():
    counts = [0, 1000, 1, 0, 127, 129, 257, 0, 2000, 640, 500, 384, 0]
    E, N, K = len(counts), 1700, 200
    g = gen("many rows")
    t, w = weights(g, E, N, K, 64, False)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    x = torch.randn(sum(counts) + 70, K, device="cuda", generator=g).to(BF16)
    bias = torch.randn(E, N, device="cuda", generator=g)
    check_linear(t, w, x, offsets, bias, 0, BF16)
    check_linear(t, w, x, offsets, bias, 2, F32)


@pytest.mark.parametrize("rows", [5, 8, 20, 150])
def test_linear_of_one_matrix_with_offsets_and_of_long_rows(rows):
    """One matrix that answers a part of the rows; K of several turns of a block's warps, and of slices of unequal length."""
    g = gen("one", rows)
    for K, N in ((200, 136), (5000, 90), (4224, 264)):
        t, w = weights(g, 1, N, K, 32, False)
        x = torch.randn(rows, K, device="cuda", generator=g).to(BF16)
        for live in (0, 1, rows - 1, rows):
            off = torch.tensor([0, live], dtype=torch.int32, device="cuda")
            check_linear(t, w, x, off, torch.randn(1, N, device="cuda", generator=g), 1, BF16)
        check_linear(t, w, x, None, None, 0, F32)


@pytest.mark.parametrize("rows", [3, 40, 1500, 9000])
def test_linear_by_a_thousand_experts(rows):
    """More matrices than rows (the ones that have rows are looked up), and more than a block has threads."""
    E, N, K = 1024, 24, 64
    g = gen("thousand", rows)
    t, w = weights(g, E, N, K, 64, True)
    e = torch.sort(torch.randint(0, E, (rows,), device="cuda", generator=g)).values
    offsets = torch.searchsorted(e, torch.arange(E + 1, device="cuda")).to(torch.int32)
    x = torch.randn(rows, K, device="cuda", generator=g).to(F16)
    y = torch.empty(rows, N, device="cuda")
    bls.bls_w4_linear(t, x, y, offsets=offsets)
    assert bls.bls_w4_status() == bls.BLS_OK
    want = torch.einsum("rk,rnk->rn", x.double(), w[e])
    size = torch.einsum("rk,rnk->rn", x.double().abs(), w[e].abs())
    close(y, want, size, 2 * K + 13)


def test_offsets_outside_the_rows_are_cut():
    """A broken offsets array (negative, past the rows, falling) cannot lead outside x and y: whatever rows it names, the guard rows
    after y stay untouched."""
    g = gen("broken")
    t, _ = weights(g, 4, 72, 96, 32, True)
    for rows in (6, 300):
        x = torch.randn(rows, 96, device="cuda", generator=g).to(BF16)
        buf = torch.full((rows + 8, 72), 7.0, device="cuda", dtype=BF16)
        for off in ([-5, 2, 3, 4, rows], [0, rows + 50, rows + 60, 3, 5], [4, 3, 2, 1, 0], [0, 0, 0, 0, 2 ** 31 - 1]):
            bls.bls_w4_linear(t, x, buf[:rows], offsets=torch.tensor(off, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert torch.all(buf[rows:] == 7.0)
    assert bls.bls_w4_status() == bls.BLS_OK
