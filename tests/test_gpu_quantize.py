"""The scales of 4-bit weights against the quotients in 64 bits, and the quantiser against its plain torch form.  GPU only.

A scale is (hi - lo) / 15 or max|w| / 7 rounded once, to bfloat16's 8 bits with ties to even, so it is compared for equality.  The
difference of two fp32 numbers of similar size and its quotient in 64 bits are off by less than 2^-52 relatively; a
quotient that is no tie stays 2^-33 away from one."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2512_19342_b200 as bls

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GROUP = 32


def rounded(v):
    """float64 -> 8 significant bits, or a multiple of 2^-133 where that is coarser; ties to even."""
    m, e = np.frexp(v)
    bits = np.minimum(e + 133, 8)                            # negative: nothing is left of m
    return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)


def scales(w, symmetric):
    """Scales of w [N][K] by the library and by definition, [N][K / GROUP] in float64."""
    t = bls.bls_w4_quantize(w, GROUP, symmetric)
    got = t.scale[0, :w.shape[1] // GROUP, :w.shape[0]].t().double().cpu().numpy()
    g = w.float().reshape(w.shape[0], -1, GROUP)
    if symmetric:
        return got, rounded(g.abs().amax(2).double().cpu().numpy() / 7)
    lo, hi = g.amin(2).clamp(max=0).double().cpu().numpy(), g.amax(2).clamp(min=0).double().cpu().numpy()
    return got, rounded((hi - lo) / 15)


@pytest.mark.parametrize("symmetric", [True, False], ids=["symmetric", "zeros"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
def test_scales_of_many_groups(dtype, symmetric):
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        got, want = scales(torch.randn(8192, 2560, device="cuda", generator=g).to(dtype), symmetric)
        assert np.array_equal(got, want)


def group_of(rows):
    """[rows][GROUP] fp32 with the given values in front and zeros behind."""
    w = np.zeros((len(rows), GROUP), np.float32)
    for i, r in enumerate(rows):
        w[i, :len(r)] = r
        assert np.all(w[i, :len(r)].astype(np.float64) == r)
    return torch.from_numpy(w).cuda()


def test_scales_next_to_ties():
    """hi - lo a little above and below 15 ties: fp32 rounds it onto 15 times the tie, where only what was rounded off decides."""
    rows = []
    for odd in range(257, 512, 2):                           # a tie has nine bits, the last of them set
        for at in (0, -70, 60):
            tie = float(np.ldexp(15.0 * odd, at))            # 12 or 13 bits
            ulp = float(np.spacing(np.float32(tie)))
            rows += [(tie, 0.0), (tie, -ulp / 4), (tie, -ulp / 2 ** 20), (tie - ulp, -ulp * 0.75), (0.0, -tie), (ulp / 4, -tie),
                     (ulp * 0.75, ulp - tie), (tie + ulp, 0.0), (tie - ulp, 0.0)]
    got, want = scales(group_of(rows), False)
    assert np.array_equal(got, want)
    rows = [(float(np.ldexp(7.0 * odd, at)) + d * float(np.spacing(np.float32(np.ldexp(7.0 * odd, at)))),)
            for odd in range(257, 512, 2) for at in (0, -70, 60) for d in (-1, 0, 1)]
    got, want = scales(group_of(rows), True)
    assert np.array_equal(got, want)


def test_scales_of_tiny_weights():
    """Quotients below bfloat16's normal range: scales are multiples of 2^-133, spans multiples of 2^-149."""
    g = np.random.default_rng(5)
    spans = np.concatenate([g.integers(1, 15 << 24, 2000), [15 * (2 * i + 1) * 2 ** 15 + d for i in range(60) for d in (-1, 0, 1)]])
    rows = [(np.ldexp(float(s - s // 3), -149), -np.ldexp(float(s // 3), -149)) for s in spans if s < 1 << 24]
    got, want = scales(group_of(rows), False)
    assert np.array_equal(got, want)
    spans = np.concatenate([g.integers(1, 1 << 24, 2000), [7 * (2 * i + 1) * 2 ** 15 + d for i in range(30) for d in (-1, 0, 1)]])
    got, want = scales(group_of([(np.ldexp(float(s), -149),) for s in spans]), True)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("symmetric", [True, False], ids=["symmetric", "zeros"])
def test_weights_of_every_magnitude(symmetric):
    """Groups from the smallest to the largest numbers, around the end of the normal range above all: the stored weights are those of the
    fp32 quotients by the scale, which numpy divides the same way."""
    g = np.random.default_rng(6)
    size = np.concatenate([np.exp2(g.uniform(-149, 126, 3000)), np.exp2(g.uniform(-130, -120, 3000))])
    w = (g.uniform(-1, 1, (size.size, GROUP)) * size[:, None]).astype(np.float32)
    t = bls.bls_w4_quantize(torch.from_numpy(w).cuda(), GROUP, symmetric)
    s = t.scale[0, 0, :size.size].float().cpu().numpy()
    safe = np.where(s > 0, s, np.float32(1))
    z = np.full(size.size, 8, np.float32) if symmetric else np.where(s > 0, np.clip(np.rint(np.maximum(-w.min(1), 0) / safe), 0, 15), 0)
    q = np.clip(np.where(s[:, None] > 0, np.rint(w / safe[:, None]), 0) + z[:, None], 0, 15)
    back = torch.empty(size.size, GROUP, device="cuda")
    bls.bls_w4_dequantize(t, back)
    assert np.array_equal(back.cpu().numpy(), (q - z[:, None]).astype(np.float32) * s[:, None])


def test_scales_of_spans_past_the_range():
    """hi - lo passes fp32's range, the scale does not: the group is held, each weight to within half a step and half a zero point's step."""
    big = float(np.ldexp(255.0, 120))
    rows = [(big, -big), (big, -big / 2, big / 3, -big / 5, 1.0), (big / 4, -big), (big * 0.75, -big * 0.75, 0.25 * big)]
    w = group_of([[float(np.float32(v)) for v in r] for r in rows])
    got, want = scales(w, False)
    assert np.array_equal(got, want)
    t = bls.bls_w4_quantize(w, GROUP, False)
    q = torch.empty_like(w)
    bls.bls_w4_dequantize(t, q)
    fine = torch.isfinite(q)
    assert bool((fine | (w.abs() >= 0.9 * big)).all())       # (q - z) s of the largest weight may itself pass the range
    off = (q.double() - w.double()).abs()
    assert bool((off <= 1.25 * torch.from_numpy(want).cuda())[fine].all())


def plain_forms():
    spec = importlib.util.spec_from_file_location("operators_cases", os.path.join(ROOT, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("zero", [False, True])
def test_the_plain_form_gives_the_same_bits(dtype, zero):
    """Both take fp32 quotients by the same scales, so all weights and scales are equal."""
    m = plain_forms()
    for seed in range(12):
        s = m.prepare(dict(op="quantize", E=2, N=1000, K=1023, group=GROUP, zero=zero, dtype=dtype), seed)
        m.own = False
        plain = m.run(s)
        m.own = True
        own = m.run(s)
        assert torch.equal(own["scale"], plain["scale"]) and torch.equal(own["w"], plain["w"])
