"""Products with 4-bit weights on whole numbers, compared for equality.  Weights are (q - z) 2^p with any q and z of
0..15 and p in -1..2, inputs are whole numbers up to 3, so every product, group sum, scaled sum and answer is a multiple of 1/2 below
2^23 and nothing is rounded anywhere, in whatever order it is added.  One dropped or doubled input, a zero point off by
one, a scale of another group or a slice that ends in the wrong place changes the answer.  GPU only."""
import pytest
import torch

import paper_2512_19342_b200 as bls

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def whole(g, E, N, K, group, zero):
    """A W4 put together element by element from the documented storage, and its weights in 64 bits."""
    nt, kt = -(-N // 128), -(-K // 128)
    rnd = lambda lo, hi, *s: torch.randint(lo, hi, s, device="cuda", generator=g)
    q = rnd(0, 16, E, N, K)
    n, k = torch.arange(N, device="cuda")[:, None], torch.arange(K, device="cuda")[None, :]
    i, t, b = k % 8, k % 128 // 8 % 4, k % 128 // 32
    j = i // 2 + 4 * (i % 2)
    at = ((n // 128) * kt + k // 128) * 8192 + n % 128 * 64 + (t ^ (n % 128 // 2 % 4)) * 16 + 4 * b + j // 2
    flat = rnd(0, 16, E, nt * kt * 8192) * 17                 # what pads the last tiles may hold anything
    flat[:, at.reshape(-1)] = 0
    for half in (0, 1):
        some = (j % 2 == half).expand_as(at)
        flat[:, at[some]] |= q[:, some] << (4 * half)
    groups = kt * 128 // group
    scale = torch.zeros(E, groups, nt * 128, device="cuda", dtype=BF16)
    live = -(-K // group)
    scale[:, :live, :N] = 2.0 ** rnd(-1, 3, E, live, N).to(BF16)
    z = rnd(0, 16, E, groups, nt * 128).to(torch.uint8) if zero else None
    zk = 8 if z is None else z[:, k[0] // group, :N].transpose(1, 2).long()
    w = (q - zk).double() * scale[:, k[0] // group, :N].transpose(1, 2).double()
    return bls.W4(flat.to(torch.uint8).reshape(E, nt, kt, 128, 64), scale, z, N, K, group), w


def check(t, w, x, offsets, bias, act):
    y = torch.full((x.shape[0], t.N), float("nan"), device="cuda")
    bls.bls_w4_linear(t, x, y, offsets=offsets, bias=bias, act=act)
    want = torch.zeros(x.shape[0], t.N, dtype=torch.float64, device="cuda")
    ends = [0, x.shape[0]] if offsets is None else offsets.tolist()
    for e in range(t.E):
        a, b = ends[e], ends[e + 1]
        want[a:b] = x[a:b].double() @ w[e].t() + (0 if bias is None else bias[e].double())
    assert float(want.abs().max()) < 2 ** 23
    first = ends[0]                                           # rows in front of the first matrix are nobody's, and not written
    assert torch.equal(y[first:].double(), (want.clamp(min=0) if act else want)[first:]) and torch.isnan(y[:first]).all()


@pytest.mark.parametrize("rows", [1, 8, 9, 13, 64, 65, 200])
@pytest.mark.parametrize("N,K,dtype", [(136, 800, BF16), (300, 1152, F16), (264, 4224, BF16), (90, 5000, F16)])
@pytest.mark.parametrize("group,zero", [(32, True), (64, True), (128, True), (32, False), (128, False)])
def test_one_matrix(rows, N, K, dtype, group, zero):
    """From 9 rows on K is split over the CTAs of a cluster: 3, 4 and 8 slices, with a shorter or an empty last one."""
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + K + group)
    t, w = whole(g, 1, N, K, group, zero)
    x = torch.randint(-3, 4, (rows, K), device="cuda", generator=g).to(dtype)
    bias = torch.randint(-9, 10, (1, N), device="cuda", generator=g).float()
    check(t, w, x, None, bias, 1)
    check(t, w, x, torch.tensor([rows // 3, rows], dtype=torch.int32, device="cuda"), None, 0)


@pytest.mark.parametrize("counts", [[1, 0, 2, 0, 5], [0, 30, 1, 0, 9], [70, 0, 0, 129, 3], [64, 64, 64, 64, 64]], ids=str)
@pytest.mark.parametrize("group,zero", [(32, True), (64, False), (128, True)])
def test_experts(counts, group, zero):
    g = torch.Generator(device="cuda").manual_seed(sum(counts) + group)
    t, w = whole(g, len(counts), 200, 1100, group, zero)
    x = torch.randint(-3, 4, (sum(counts) + 3, 1100), device="cuda", generator=g).to(BF16)
    ends = torch.tensor([0] + counts, device="cuda").cumsum(0).to(torch.int32)
    check(t, w, x, ends, torch.randint(-9, 10, (len(counts), 200), device="cuda", generator=g).float(), 1)


@pytest.mark.parametrize("rows,N", [(257, 15000), (384, 15000), (600, 10000), (1000, 7700)])
@pytest.mark.parametrize("group,zero", [(32, True), (64, True), (128, False)])
def test_tiles_of_256_rows(rows, N, group, zero):
    g = torch.Generator(device="cuda").manual_seed(rows + group)
    t, w = whole(g, 1, N, 520, group, zero)
    x = torch.randint(-3, 4, (rows, 520), device="cuda", generator=g).to(F16 if zero else BF16)
    check(t, w, x, None, None, 0)
