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


class Pages(Elsewhere):
    """Pages of keys or values on a device of that number."""

    def __init__(self, device, *shape, dtype=torch.bfloat16):
        super().__init__(device, *shape, dtype=dtype)

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        steps = [torch.Size(self.shape[k + 1:]).numel() for k in range(len(self.shape))]
        return tuple(steps) if i is None else steps[i]

    def __getitem__(self, i):
        return Pages(self.number, *self.shape[1:], dtype=self.dtype)


def cache_on(H, device, pages=None, lengths=None, v=None):
    i32 = torch.int32
    return H.PagedCache(Pages(device, 8, 2, 16, 64), v or Pages(device, 8, 2, 16, 64), pages or Pages(device, 3, 4, dtype=i32), lengths or Elsewhere(device, 3, dtype=i32))


def test_caches_of_two_devices(H):
    i32 = torch.int32
    for more in (dict(v=Pages(1, 8, 2, 16, 64)), dict(pages=Pages(1, 3, 4, dtype=i32)), dict(lengths=Elsewhere(1, 3, dtype=i32)), dict(lengths=Elsewhere(0, 2, dtype=i32)),
                 dict(pages=Pages(0, 3, 4, dtype=torch.int64))):
        with pytest.raises(ValueError):
            cache_on(H, 0, **more)
    cache = cache_on(H, 0)
    with pytest.raises(ValueError):
        cache.lengths = Elsewhere(1, 3, dtype=i32)
    bf = torch.bfloat16
    rows, starts, cs = lambda d, w: Elsewhere(d, 5, w, dtype=bf), lambda d, n=4: Elsewhere(d, n, dtype=i32), Elsewhere(0, 9, 32, 2)
    for call in (lambda: H.kernel_cache_append(cache, starts(0), rows(1, 512), 4), lambda: H.kernel_cache_append(cache, starts(1), rows(0, 512), 4),
                 lambda: H.kernel_cache_append(cache, starts(0), rows(0, 512), 4, rows(1, 256)), lambda: H.kernel_cache_append(cache, starts(0), rows(0, 512), 4, None, Elsewhere(1, 9, 32, 2)),
                 lambda: H.kernel_cache_append(cache, starts(0, 5), rows(0, 512), 4), lambda: H.kernel_attention_paged(cache, starts(0), rows(1, 256), 4, rows(0, 256), 5, 50),
                 lambda: H.kernel_attention_paged(cache, starts(0), rows(0, 256), 4, rows(1, 256), 5, 50),
                 lambda: H.kernel_attention_paged(cache, starts(0), rows(0, 256), 4, rows(0, 256), 5, 50, lse=Elsewhere(1, 5, 4)),
                 lambda: H.kernel_attention_paged(cache, starts(0), rows(0, 256), 4, rows(0, 256), 5, 50, workspace=Elsewhere(1, 1 << 20, dtype=torch.uint8)),
                 lambda: H.kernel_attention_paged(cache, starts(0), Elsewhere(0, 5, 256), 4, rows(0, 256), 5, 50),
                 lambda: H.kernel_rotary(rows(0, 256), 4, 64, rows(1, 256), cs, seq=9), lambda: H.kernel_rotary(rows(0, 256), 4, 64, rows(0, 256), Elsewhere(1, 9, 32, 2), seq=9),
                 lambda: H.kernel_rotary(rows(0, 256), 4, 64, rows(0, 256), cs, positions=Elsewhere(1, 5, dtype=i32))):
        with pytest.raises(ValueError):
            call()


def test_other_tensors_in_a_caches_place(H):
    """The cache says to the library what it holds now."""
    i32 = torch.int32
    cache = cache_on(H, 0)
    cache.pages = Pages(0, 5, 7, dtype=i32)
    assert (cache.c.sequences, cache.c.max_pages, cache.c.pages_ld) == (5, 7, 7)
    with pytest.raises(ValueError, match="lengths"):
        H.kernel_cache_append(cache, Elsewhere(0, 6, dtype=i32), Elsewhere(0, 5, 512, dtype=torch.bfloat16), 4)
    cache.lengths = Elsewhere(0, 5, dtype=i32)
    assert cache.c.lengths == 1 << 20


def test_logits_of_two_devices(H):
    x, i32, i64 = Elsewhere(0, 4, 50), torch.int32, torch.int64
    tokens, at = lambda d: Elsewhere(d, 9, dtype=i32), lambda d: Elsewhere(d, 4, dtype=i64)
    for kw in (dict(out=Elsewhere(1, 4, 50)), dict(tokens=tokens(1), begin=at(0), end=at(0)), dict(tokens=tokens(0), begin=at(1), end=at(0)), dict(tokens=tokens(0), begin=at(0)),
               dict(bias=Elsewhere(1, 1, 50)), dict(bias=Elsewhere(0, 2, 50)), dict(allowed=Elsewhere(1, 1, 2, dtype=i32)), dict(allowed=Elsewhere(0, 1, 1, dtype=i32)),
               dict(allowed=Elsewhere(0, 1, 2, dtype=i64))):
        out = kw.pop("out", x)
        with pytest.raises(ValueError):
            H.kernel_adjust_logits(x, 50, out, **kw)
        with pytest.raises(ValueError):
            H.kernel_adjust_logits_bwd(x, 50, Elsewhere(0, 4, 50), out if out is not x else Elsewhere(-1, 4, 50), **kw)


def test_the_new_operators_ask_for_their_tensors_stream(H):
    """Refused by the library after the stream was asked for, so that nothing is launched."""
    bf, i32 = torch.bfloat16, torch.int32
    cache, starts = cache_on(H, 1), Elsewhere(1, 4, dtype=i32)
    rows = lambda w: Elsewhere(1, 5, w, dtype=bf)
    for call in (lambda: H.kernel_rotary(rows(256), 4, 64, rows(256), Elsewhere(1, 9, 32, 2), seq=10), lambda: H.kernel_cache_append(cache, starts, rows(512), 3),
                 lambda: H.kernel_attention_paged(cache, starts, rows(256), 4, rows(256), 5, 50, scale=-1.0), lambda: H.kernel_adjust_logits(Elsewhere(1, 4, 50), 50, Elsewhere(1, 4, 50), repetition=0.0),
                 lambda: H.kernel_rotary_table(dict(rot=64), Elsewhere(1, 9, 32, 2), first=-1)):
        H.asked.clear()
        with pytest.raises(H.HiftError):
            call()
        assert H.asked == [1]
