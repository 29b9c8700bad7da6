"""The operators on matrices and scores take all tensors from one device, and the stream and work space of that device.  Tensors here are stand-ins
that say where they are; nothing is launched."""
import pytest
import torch


class Elsewhere:
    """A contiguous tensor of a device of that number (-1: the host), as far as the argument checks look at it."""

    def __init__(self, device, *shape, dtype=torch.float32):
        self.number, self.shape, self.dtype = device, torch.Size(shape), dtype

    is_cuda = property(lambda self: self.number >= 0)
    device = property(lambda self: torch.device("cuda", self.number) if self.number >= 0 else torch.device("cpu"))

    def get_device(self):
        return self.number

    def stride(self):
        return (self.shape[1], 1) if len(self.shape) == 2 else (1,)

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def H(monkeypatch):
    import paper_2401_15207_amd as H
    from paper_2401_15207_amd import binding
    asked = []
    monkeypatch.setattr(binding.torch._C, "_cuda_getCurrentRawStream", lambda number: asked.append(number) or 0, raising=False)
    monkeypatch.setattr(H, "asked", asked, raising=False)
    return H


def test_matrices_of_two_devices(H):
    a, b, ws = Elsewhere(0, 300, 300), Elsewhere(1, 300, 300), Elsewhere(0, 1 << 24, dtype=torch.uint8)
    opt = dict(kind="muon", lr=1e-3, momentum=0.9)
    for src, dst in (([a], [b]), ([a, b], [a, a]), ([a, a], [a, b])):
        with pytest.raises(ValueError, match="cuda:"):
            H.kernel_orthogonalize(src, dst, workspace=ws)
    for arrays in (([a], [b], [a]), ([a], [a], [b]), ([a], [a], [a], [Elsewhere(1, 300, 300, dtype=torch.bfloat16)]), ([a, b], [a, b], [a, b])):
        with pytest.raises(ValueError, match="cuda:"):
            H.kernel_muon(opt, *arrays, workspace=ws)
    for bad in (Elsewhere(1, 1 << 24, dtype=torch.uint8), Elsewhere(-1, 1 << 24, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="workspace"):
            H.kernel_orthogonalize([a], [a], workspace=bad)
        with pytest.raises(ValueError, match="workspace"):
            H.kernel_muon(opt, [a], [a], [a], workspace=bad)


def test_the_stream_is_that_of_the_tensors_device(H):
    """Refused for their work space after the stream was asked for, so that nothing is launched."""
    b, small = Elsewhere(1, 300, 300), Elsewhere(1, 64, dtype=torch.uint8)
    for call in (lambda: H.kernel_orthogonalize([b], [b], workspace=small), lambda: H.kernel_muon(dict(kind="muon", lr=1e-3, momentum=0.9), [b], [b], [b], workspace=small)):
        H.asked.clear()
        with pytest.raises(H.HiftError):
            call()
        assert H.asked == [1]


def test_scores_of_two_devices(H):
    x, rows = Elsewhere(0, 4, 50), lambda device, dtype=torch.float32: Elsewhere(device, 4, dtype=dtype)
    i32 = torch.int32
    for args in ((x, 50, rows(1, i32), 1.0, rows(0), None, None), (x, 50, rows(0, i32), 1.0, rows(1), None, None), (x, 50, None, 1.0, None, rows(-1), None)):
        with pytest.raises(ValueError):
            H.kernel_token_logprob(*args)
    stats = Elsewhere(0, 4, 2)
    for d, dx in ((rows(1), x), (rows(0), Elsewhere(1, 4, 50))):
        with pytest.raises(ValueError):
            H.kernel_token_logprob_bwd(x, 50, rows(0, i32), 1.0, stats, rows(0), d, None, dx)


def test_nothing_to_do(H):
    H.kernel_orthogonalize([], [])
    H.kernel_muon(dict(kind="muon", lr=1e-3, momentum=0.9), [], [], [])
    with pytest.raises(H.HiftError):
        H.kernel_muon(dict(kind="adamw", lr=1e-3), [], [], [])
