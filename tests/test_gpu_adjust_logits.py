"""Adjusted logits and the gradient through them on the GPU, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2401_15207_amd as H

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def words(let):
    """Truth values [rows, V] as the mask's words."""
    rows, v = let.shape
    pad = torch.zeros(rows, -v % 32, dtype=torch.bool)
    bits = torch.cat([let.cpu(), pad], 1).view(rows, -1, 32).long()
    w = (bits << torch.arange(32)).sum(2)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32).cuda()


def definition(x, counts, by, bias, let, d=None):
    """Result and the sizes of what is added up for it."""
    x, counts = x.double(), counts.double()
    r = by.get("repetition", 1.0)
    factor = torch.where(counts > 0, torch.where(x > 0, 1.0 / r, r), 1.0)
    if d is not None:
        z = d.double() * factor
        return z if let is None else torch.where(let, z, 0.0), z.abs()
    p, f = by.get("presence", 0.0), by.get("frequency", 0.0)
    z = x * factor - p * (counts > 0) - f * counts
    size = (x * factor).abs() + abs(p) + abs(f) * counts
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    return z if let is None else torch.where(let, z, -math.inf), size


def counts_of(tokens, begin, end, v):
    out = []
    for b, e in zip(begin.tolist(), end.tolist()):
        t = tokens[max(b, 0):max(e, 0)].long()
        out.append(torch.bincount(t[(t >= 0) & (t < v)], minlength=v))
    return torch.stack(out)


def close(got, want, size, dtype):
    inf = torch.isinf(want)
    assert torch.equal(got.double()[inf], want[inf])
    # fp32: the reciprocal, its product, the product with the count and three sums, each off by at most 2^-24 of the sizes; then the type's rounding
    tol = 6 * 2.0 ** -24 * size + HALF_STEP[dtype] * (want.abs() + 6 * 2.0 ** -24 * size) + 1e-37
    far = (got.double() - want).abs()
    assert (far <= tol)[~inf].all(), f"off by up to {(far / tol)[~inf].max().item():.2f} of the tolerance"


def make(rows, v, dtype, history, ld=None, offset=0, seed=0):
    g = torch.Generator().manual_seed(seed + rows + v)
    flat = torch.randn(rows * (ld or v) + offset + 64, generator=g).mul_(3).to("cuda", DT[dtype])
    x = flat[offset:offset + rows * (ld or v)].view(rows, -1)
    lens = torch.randint(0, history + 1, (rows,), generator=g)
    end = lens.cumsum(0)
    tokens = (torch.rand(int(end[-1]), generator=g) ** 3 * (v + 1)).long().sub(1).to(torch.int32)   # -1 and all ids
    return x, tokens.cuda(), (end - lens).cuda(), end.cuda(), g


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,v,ld,offset,history", [(1, 1, None, 0, 3), (3, 7, 9, 1, 5), (2, 33, None, 3, 40), (5, 2047, 2051, 0, 300), (4, 8200, 8200, 8, 2000),
                                                      (3, 50265, None, 0, 1500), (70, 5003, 5008, 5, 64), (600, 1000, None, 0, 10)])
@pytest.mark.parametrize("mask", ["none", "one", "rows"])
def test_forward_and_backward(dtype, rows, v, ld, offset, history, mask):
    x, tokens, begin, end, g = make(rows, v, dtype, history, ld, offset)
    let = None if mask == "none" else torch.rand(1 if mask == "one" else rows, v, generator=g) < 0.6
    if let is not None and mask == "rows":
        let[0] = False          # a row of which nothing is left
    allowed = None if let is None else words(let)
    let = None if let is None else let.cuda().expand(rows, v)
    bias = torch.randn(1 if mask == "one" else rows, v, generator=g).cuda() if mask != "none" else None
    by = dict(repetition=1.3, presence=0.4, frequency=0.15)
    out = torch.full((rows, v + 2), -7.0, device="cuda", dtype=DT[dtype])
    H.kernel_adjust_logits(x, v, out, tokens, begin, end, bias=bias, allowed=allowed, **by)
    counts = counts_of(tokens, begin, end, v)
    want, size = definition(x[:, :v], counts, by, bias, let)
    close(out[:, :v], want, size, DT[dtype])
    assert (out[:, v:] == -7.0).all()
    # backwards: into rows of another distance, and in the place of what comes in
    d = torch.randn(rows, v, generator=g).to("cuda", DT[dtype])
    dx = torch.full((rows, v + 1), -7.0, device="cuda", dtype=DT[dtype])
    H.kernel_adjust_logits_bwd(x, v, d, dx, tokens, begin, end, bias=bias, allowed=allowed, **by)
    want, size = definition(x[:, :v], counts, by, None, let, d)
    close(dx[:, :v], want, size, DT[dtype])
    assert (dx[:, v:] == -7.0).all()
    H.kernel_adjust_logits_bwd(x, v, d, d, tokens, begin, end, allowed=allowed, **by)
    assert torch.equal(d, dx[:, :v])
    # forward in place: the same bits, behind the vocabulary nothing changes
    behind = x[:, v:].clone()
    H.kernel_adjust_logits(x, v, x, tokens, begin, end, bias=bias, allowed=allowed, **by)
    assert torch.equal(x[:, :v], out[:, :v]) and torch.equal(x[:, v:], behind)


@pytest.mark.parametrize("by", [dict(repetition=0.5), dict(presence=-1.0), dict(frequency=0.25), dict(repetition=2.0, presence=1.0, frequency=-0.5)])
def test_each_penalty_by_hand(by):
    x = torch.tensor([[1.0, -2.0, 0.0, 3.0]], device="cuda")
    tokens = torch.tensor([1, 3, 3, 3, 9, -5], device="cuda", dtype=torch.int32)
    begin, end = torch.tensor([0], device="cuda"), torch.tensor([6], device="cuda")
    out = torch.empty_like(x)
    H.kernel_adjust_logits(x, 4, out, tokens, begin, end, **by)
    r, p, f = by.get("repetition", 1.0), by.get("presence", 0.0), by.get("frequency", 0.0)
    assert out.tolist() == [[1.0, -2.0 * r - p - f, 0.0, 3.0 / r - p - 3 * f]]


def test_nothing_to_do_copies():
    x = torch.randn(3, 1001, device="cuda").bfloat16()
    out = torch.empty_like(x)
    H.kernel_adjust_logits(x, 1001, out)
    assert torch.equal(out, x)
    empty = torch.empty(0, 5, device="cuda")
    H.kernel_adjust_logits(empty, 5, empty)


def test_histories_that_overlap_and_leave_the_list():
    """Positions of one text have seen what precedes them; bounds outside the list are kept in it, an end before its begin is nothing."""
    v = 300
    g = torch.Generator().manual_seed(5)
    tokens = torch.randint(0, v, (64,), generator=g, dtype=torch.int32).cuda()
    x = torch.randn(67, v, generator=g).cuda()
    begin = torch.tensor([0] * 64 + [-10, 40, 60], device="cuda")
    end = torch.tensor([i + 1 for i in range(64)] + [5, 20, 2 ** 40], device="cuda")
    out = torch.empty_like(x)
    by = dict(repetition=1.2, frequency=0.5)
    H.kernel_adjust_logits(x, v, out, tokens, begin, end, **by)
    e = end.clamp(max=64)
    counts = counts_of(tokens, begin.clamp(min=0), torch.maximum(e, begin.clamp(min=0)), v)
    want, size = definition(x, counts, by, None, None)
    close(out, want, size, torch.float32)


def test_infinities_and_nan():
    inf, nan = math.inf, math.nan
    x = torch.tensor([[-inf, inf, nan, -inf, inf, nan, 1.0, -3.4e38]], device="cuda")
    tokens = torch.tensor([0, 1, 2, 7], device="cuda", dtype=torch.int32)
    begin, end = torch.tensor([0], device="cuda"), torch.tensor([4], device="cuda")
    out = torch.empty_like(x)
    H.kernel_adjust_logits(x, 8, out, tokens, begin, end, repetition=1.5, presence=0.5)
    assert out[0].isnan().tolist() == [False, False, True, False, False, True, False, False]
    assert out[0, [0, 1, 3, 4, 6, 7]].tolist() == [-inf, inf, -inf, inf, 1.0, -inf]
    # masked: -inf whatever was there
    H.kernel_adjust_logits(x, 8, out, tokens, begin, end, repetition=1.5, allowed=torch.zeros(1, 1, device="cuda", dtype=torch.int32))
    assert (out == -inf).all()
    H.kernel_adjust_logits_bwd(x, 8, torch.full_like(x, nan), out, tokens, begin, end, repetition=1.5, allowed=torch.zeros(1, 1, device="cuda", dtype=torch.int32))
    assert (out == 0).all()


def test_gradient_by_differences():
    """d_logits of a weighted sum of the results, by central differences of the definition away from its kink at 0."""
    v = 50
    g = torch.Generator().manual_seed(9)
    x = torch.randn(2, v, generator=g).cuda()
    x = torch.where(x.abs() < 0.05, 0.1, x)
    tokens = torch.randint(0, v, (30,), generator=g, dtype=torch.int32).cuda()
    begin, end = torch.tensor([0, 10], device="cuda"), torch.tensor([20, 30], device="cuda")
    w = torch.randn(2, v, generator=g).cuda()
    by = dict(repetition=1.7, presence=0.3, frequency=0.2)
    d = torch.empty_like(x)
    H.kernel_adjust_logits_bwd(x, v, w, d, tokens, begin, end, **by)
    counts = counts_of(tokens, begin, end, v)
    for j in range(v):
        up, down = x.double().clone(), x.double().clone()
        up[:, j] += 1e-3
        down[:, j] -= 1e-3
        slope = ((definition(up, counts, by, None, None)[0] - definition(down, counts, by, None, None)[0]) * w.double()).sum(1) / 2e-3
        assert (slope - d[:, j].double()).abs().max().item() <= 1e-9 + 3 * 2.0 ** -24 * 1.7 * w.abs().max().item()


def test_scores_of_adjusted_logits():
    """As a sampler uses it: the mask's rows go on into the log probabilities, a row without any allowed token too, and the gradient comes back through both."""
    rows, v = 6, 777
    g = torch.Generator().manual_seed(2)
    x = torch.randn(rows, v, generator=g).mul(2).cuda()
    let = torch.rand(rows, v, generator=g) < 0.3
    let[4] = False
    let[:4, 11] = True
    tokens = torch.randint(0, v, (200,), generator=g, dtype=torch.int32).cuda()
    begin, end = torch.arange(rows).cuda() * 20, torch.arange(rows).cuda() * 20 + 100
    out, dz, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    by = dict(repetition=1.4, presence=0.2, frequency=0.1)
    H.kernel_adjust_logits(x, v, out, tokens, begin, end, allowed=words(let), **by)
    target = torch.tensor([11, 11, 11, 11, 11, -1], device="cuda", dtype=torch.int32)
    logp, entropy, stats = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    H.kernel_token_logprob(out, v, target, 1.0, logp, entropy, stats)
    assert logp[4].item() == -math.inf and entropy[4].item() == 0.0
    H.kernel_token_logprob_bwd(out, v, target, 1.0, stats, entropy, torch.ones(rows, device="cuda"), None, dz)
    H.kernel_adjust_logits_bwd(x, v, dz, dx, tokens, begin, end, allowed=words(let), **by)
    counts = counts_of(tokens, begin, end, v)
    leaf = x.double().requires_grad_()
    r = by["repetition"]
    z = torch.where(counts > 0, torch.where(leaf > 0, leaf / r, leaf * r) - by["presence"], leaf) - by["frequency"] * counts.double()
    z = z.masked_fill(~let.cuda(), -math.inf)[:4]
    want = torch.log_softmax(z, 1)[:, 11]
    want.sum().backward()
    assert (logp[:4].double() - want.detach()).abs().max().item() <= 2.0 ** -18
    # probabilities from fp32 logits of size up to 12: exponents off by 12 * 6 * 2^-24, times the factor of the penalty
    assert (dx[:4].double() - leaf.grad[:4]).abs().max().item() <= r * (12 * 8 + 16) * 2.0 ** -24
    assert (dx[4:][~let[4:].cuda()] == 0).all()


def test_replayed_from_a_graph():
    v = 5003
    x, tokens, begin, end, g = make(9, v, "bf16", 100)
    out = torch.empty_like(x)
    H.kernel_adjust_logits(x, v, out, tokens, begin, end, repetition=1.3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.kernel_adjust_logits(x, v, out, tokens, begin, end, repetition=1.3)
    for k in range(3):
        x.copy_(torch.randn(9, v, generator=g).bfloat16())
        end[0] = int(begin[0]) + k
        want = torch.empty_like(x)
        H.kernel_adjust_logits(x, v, want, tokens, begin, end, repetition=1.3)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_one_row_in_place_by_views_of_other_widths():
    """A single row has no distance to the next."""
    x = torch.randn(1, 300, generator=torch.Generator().manual_seed(3)).cuda()
    tokens, begin, end = torch.tensor([5, 7, 7], device="cuda", dtype=torch.int32), torch.zeros(1, device="cuda", dtype=torch.int64), torch.full((1,), 3, device="cuda", dtype=torch.int64)
    by = dict(tokens=tokens, begin=begin, end=end, repetition=2.0)
    want, grad, d = torch.empty(1, 290, device="cuda"), torch.empty(1, 290, device="cuda"), torch.randn(1, 300, generator=torch.Generator().manual_seed(4)).cuda()
    H.kernel_adjust_logits(x, 290, want, frequency=0.5, **by)
    H.kernel_adjust_logits_bwd(x, 290, d, grad, **by)
    H.kernel_adjust_logits_bwd(x, 290, d, d[:, :290], **by)
    H.kernel_adjust_logits(x, 290, x[:, :290], frequency=0.5, **by)
    assert torch.equal(x[:, :290], want) and torch.equal(d[:, :290], grad)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("v,ld", [(50000, 50000), (50001, 50004)])
def test_large_matrices_as_their_halves(dtype, v, ld):
    """A call that goes past the caches gives the bits of two that do not."""
    rows, g = 400 if dtype == "bf16" else 200, torch.Generator(device="cuda").manual_seed(9)
    x, d = (torch.randn(rows, ld, device="cuda", generator=g).to(DT[dtype]) for _ in range(2))
    tokens = torch.randint(0, v, (rows * 64,), device="cuda", generator=g, dtype=torch.int32)
    begin = torch.arange(rows, device="cuda") * 64
    end, bias = begin + 64, torch.randn(1, v, device="cuda", generator=g)
    allowed = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, (v + 31) // 32), device="cuda", generator=g).to(torch.int32)
    half = rows // 2
    assert rows * v * 2 * x.element_size() >= 2 ** 26 > half * v * 2 * x.element_size()
    out, grad, outs, grads = (torch.full_like(x, -7.0) for _ in range(4))
    for to, dto, parts in ((out, grad, [slice(0, rows)]), (outs, grads, [slice(0, half), slice(half, rows)])):
        for r in parts:
            by = dict(tokens=tokens, begin=begin[r], end=end[r], repetition=1.5, allowed=allowed[r])
            H.kernel_adjust_logits(x[r], v, to[r], presence=0.5, frequency=0.25, bias=bias, **by)
            H.kernel_adjust_logits_bwd(x[r], v, d[r], dto[r], **by)
    assert torch.equal(out, outs) and torch.equal(grad, grads)
    seen = torch.zeros(rows, v, dtype=torch.bool, device="cuda").scatter_(1, tokens.view(rows, 64).long(), True)
    let = (allowed[:, torch.arange(v, device="cuda") // 32] >> (torch.arange(v, device="cuda") % 32)[None, :].to(torch.int32)) & 1 != 0
    assert torch.equal(torch.isinf(out[:, :v]), ~let) and torch.equal(grad[:, :v][let & ~seen], d[:, :v][let & ~seen])
