"""What the expert stage's Python calls check and keep, without a GPU: stand-in tensors that only have an address, and a
stand-in library that notes its calls.  Nothing is launched."""
import threading
import time

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


class Notes:
    """Stands for the library: notes the calls, and the device that was current in each."""

    def __init__(self):
        self.calls, self.current = [], 0

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args, self.current))
            return 0
        return call


@pytest.fixture
def notes(monkeypatch):
    n = Notes()

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.back, n.current = n.current, self.index

        def __exit__(self, *_):
            n.current = self.back

    monkeypatch.setattr(binding, "lib", lambda: n)
    monkeypatch.setattr(binding, "_current_device", lambda: n.current, raising=False)
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(binding, "_w4_status_word", {d: (None, 7) for d in range(2)})
    return n


class Stream:
    def __init__(self, device_index):
        self.device_index, self.cuda_stream = device_index, 2000 + device_index


def calls(device):
    """Every call on stand-in tensors of one device: (name, function of a list of tensors and a stream, the tensors)."""
    i, f = (lambda *s: Stub(s, I32, device)), (lambda *s: Stub(s, F32, device))
    w4, parts = stub_w4(device=device)
    x16 = Stub((5, 64), BF16, device)
    return [
        ("bls_moe_route", lambda t, s: bls.bls_moe_route(t[0], 8, *t[1:], stream=s), [i(4, 2), i(8), i(4, 2), i(9)]),
        ("bls_moe_dispatch", lambda t, s: bls.bls_moe_dispatch(*t, stream=s), [f(4, 16), i(4, 2), i(9), f(8, 16)]),
        ("bls_moe_combine", lambda t, s: bls.bls_moe_combine(*t, stream=s), [f(8, 16), i(4, 2), f(4, 2), f(4, 16)]),
        ("bls_moe_combine_grad", lambda t, s: bls.bls_moe_combine_grad(*t, stream=s),
         [f(4, 16), f(8, 16), i(4, 2), i(9), f(4, 2), f(8, 16), f(4, 2)]),
        ("bls_w4_linear", lambda t, s: bls.bls_w4_linear(w4, *t[:4], 0, s), [x16, f(5, 40), i(3), f(2, 40), *parts]),
        ("bls_w4_dequantize", lambda t, s: bls.bls_w4_dequantize(w4, t[0], s), [f(2, 40, 64), *parts]),
    ]


def test_tensors_of_another_gpu_are_refused(notes):
    for n in range(len(calls(0))):
        for at in range(len(calls(0)[n][2])):
            name, call, tensors = calls(0)[n]
            tensors[at].move(1, 1 << 24)                      # one tensor, another GPU's memory
            with pytest.raises(ValueError):
                call(tensors, None)
        name, call, tensors = calls(0)[n]
        with pytest.raises(ValueError):
            call(tensors, Stream(1))
    name, call, (x, *rest) = calls(0)[4]
    for t in rest[3:]:
        t.move(1, 1 << 24)                                    # weights that moved to another GPU as a whole
    with pytest.raises(ValueError):
        call([x, *rest], None)
    with pytest.raises(ValueError):
        bls.bls_w4_quantize(Stub((40, 64), F32, 0), 32, stream=Stream(1))
    assert notes.calls == []
    with pytest.raises(ValueError):
        t = [Stub((2, 1, 1, 128, 64), U8, 0), Stub((2, 4, 128), BF16, 1)]
        bls.W4(*t, None, 40, 64, 32)


@pytest.mark.parametrize("device", [0, 1])
@pytest.mark.parametrize("current", [0, 1])
def test_calls_run_on_their_tensors_gpu(notes, device, current):
    """The tensors' device is the current one during the call, and the stream is that device's."""
    notes.current = current
    for stream, handle in ((None, 1000 + device), (Stream(device), 2000 + device)):
        for name, call, tensors in calls(device):
            notes.calls.clear()
            call(tensors, stream)
            (called, args, at), = notes.calls
            assert called == name and args[-1] == handle and at == device and notes.current == current


def test_one_status_word_however_many_threads_ask(monkeypatch):
    """A launch holds the word's address, so a second word must never replace the first."""
    made = []

    def zeros(*_, **__):
        made.append(threading.current_thread())
        time.sleep(0.05)                                      # the others arrive meanwhile
        return Stub((1,), I32, 0, (1 << 20) + 256 * len(made))

    monkeypatch.setattr(binding, "_w4_status_word", {})
    monkeypatch.setattr(torch, "zeros", zeros)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *_: None)
    start, got = threading.Barrier(8), []

    def ask():
        start.wait()
        got.append(binding._status_word(0))

    threads = [threading.Thread(target=ask) for _ in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(made) == 1 and len(got) == 8 and all(w is got[0] for w in got)


def test_a_time_out_is_reported_once(monkeypatch):
    word = torch.zeros(1, dtype=torch.int32)
    monkeypatch.setattr(binding, "_w4_status_word", {0: (word, 7)})
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *_: None)
    assert bls.bls_w4_status("cuda:0") == bls.BLS_OK
    for _ in range(2):
        word.fill_(8)                                         # what a wait that gives up leaves there
        assert bls.bls_w4_status("cuda:0") == bls.BLS_ETIMEOUT
        assert bls.bls_w4_status("cuda:0") == bls.BLS_OK
