"""How the expert stage's calls treat their memory, streams and threads, beside what they compute.  GPU only."""
import pytest
import torch

import paper_2512_19342_b200 as bls

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
