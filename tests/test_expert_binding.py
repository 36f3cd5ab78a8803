"""What the expert stage's Python calls check and keep, without a GPU: stand-in tensors that only have an address, and a
stand-in library that notes its calls.  Nothing is launched."""
import pytest
import torch

import paper_2512_19342_b200 as bls
from paper_2512_19342_b200 import binding

I32, F32, BF16, U8 = torch.int32, torch.float32, torch.bfloat16, torch.uint8


class Stub:
    """A contiguous CUDA tensor as far as the checks look."""
    is_cuda = True

    def __init__(self, shape, dtype=F32, device=0, at=1 << 20):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, at
        self.move(device)

    def move(self, device, at=None):
        self.device, self.at = torch.device("cuda", device), at or self.at

    def get_device(self):
        return self.device.index

    def data_ptr(self):
        return self.at

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self, d=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s) if d is None else s[d]


def stub_w4(E=2, N=40, K=64, group=32, zero=True, device=0):
    t = [Stub((E, 1, 1, 128, 64), U8, device, 1 << 12), Stub((E, 4, 128), BF16, device, 1 << 13),
         Stub((E, 4, 128), U8, device, 1 << 14) if zero else None]
    return bls.W4(*t, N, K, group), t


def test_w4_holds_what_it_was_made_of():
    w4, (q, scale, zero) = stub_w4()
    for name, v in (("q", q), ("scale", scale), ("zero", zero), ("E", 2), ("N", 40), ("K", 64), ("group", 32)):
        assert getattr(w4, name) is v or getattr(w4, name) == v
        with pytest.raises(AttributeError):
            setattr(w4, name, v)
    assert stub_w4(zero=False)[0].zero is None


def test_w4_follows_its_tensors():
    """Memory that moved is read where it is now; memory that no longer fits is refused."""
    w4, (q, scale, zero) = stub_w4()
    assert w4._args == (1 << 12, 1 << 13, 1 << 14, 2, 40, 64, 32)
    scale.move(0, 1 << 16)
    zero.move(0, 1 << 17)
    assert w4._args == (1 << 12, 1 << 16, 1 << 17, 2, 40, 64, 32)
    scale.move(0, 1 << 18)
    scale.shape = torch.Size((2, 4, 64))
    with pytest.raises(ValueError):
        w4._args
