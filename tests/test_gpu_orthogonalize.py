"""Newton-Schulz orthogonalisation and the update with it, against the definitions in 64 bits.

Tolerances.  A factor holds 22 bits of what matters of it and sums are in fp32: a step perturbs X by about 3 products' roundings of 2^-22.  A
perturbation grows with the singular values it lies in, at most 3.4445 a step and not at all from about 0.7 on.  `well`: singular values
above 0.05 of the norm need two steps to get there, so 15 2^-22 3.4445^2 = 4.3e-5 of the result, in the 2-norm.  `any`: whatever
the matrix, 5 2^-21 3.4445^5 sqrt(short side) absolutely.  bf16 results: 2^-8 on top (their rounding is 2^-9 at most)."""
import math

import pytest

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
WELL = 15 * 2.0 ** -22 * COEF[0] ** 2


def reference(u, steps=5, coef=COEF, eps=1e-7):
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    x = x / max(x.norm().item(), eps)
    for _ in range(steps):
        s = x @ x.t().contiguous()
        x = coef[0] * x + (coef[1] * s + coef[2] * (s @ s)) @ x
    return x.t() if tall else x


def conditioned(r, c, seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(r, c, generator=g, device="cuda") * 1e-4


def rel(a, b):
    return ((a.double() - b).norm() / b.norm()).item()


LISTS = {
    "one entry": [(1, 1)], "rows and columns": [(1, 7), (9, 1), (1, 300)], "small": [(64, 64), (5, 3), (33, 65)],
    "odd": [(129, 257), (77, 300), (130, 128), (255, 31)], "layer": [(256, 256), (256, 256), (1024, 256), (256, 1024)],
    "many": [(8 + 3 * i, 40) for i in range(19)], "in LDS": [(64, 256), (96, 128), (600, 20), (33, 33), (1, 9), (128, 90)], "long": [(16, 5000), (3001, 20)],
}


@pytest.mark.parametrize("src,dst", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_lists(name, src, dst):
    import torch
    import paper_2401_15207_amd as H
    dts = {"fp32": torch.float32, "bf16": torch.bfloat16}
    u = [conditioned(r, c, i).to(dts[src]) for i, (r, c) in enumerate(LISTS[name])]
    # (rows further apart than they are long, and not on 16 bytes)
    out = [torch.full((r, c + 3), 7.0, device="cuda", dtype=dts[dst])[:, 1:c + 1] for r, c in LISTS[name]]
    H.kernel_orthogonalize(u, out)
    for a, b in zip(u, out):
        want = reference(a)
        spread = torch.linalg.svdvals(a.double())
        grown = max(1.0, min(5.0, math.log(0.7 / max((spread[-1] / a.double().norm()).item(), 1e-9)) / math.log(COEF[0])))
        assert rel(b, want) <= 15 * 2.0 ** -22 * COEF[0] ** grown + (2.0 ** -8 if dst == "bf16" else 0.0), (name, tuple(a.shape))
        wide = torch.as_strided(b, (b.shape[0], b.shape[1] + 3), b.stride(), b.storage_offset() - 1)
        assert (wide[:, 0] == 7.0).all() and (wide[:, -2:] == 7.0).all()
    # the same call gives the same bits
    again = [torch.full_like(b, 7.0) for b in out]
    H.kernel_orthogonalize(u, again)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("r,c", [(1000, 333), (512, 1536), (1024, 1024), (700, 2300)])
def test_larger(r, c):
    import torch
    import paper_2401_15207_amd as H
    g = torch.Generator(device="cuda")
    g.manual_seed(r + c)
    q, _ = torch.linalg.qr(torch.randn(max(r, c), min(r, c), generator=g, device="cuda", dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(min(r, c), min(r, c), generator=g, device="cuda", dtype=torch.float64))
    s = torch.linspace(0.2, 1.0, min(r, c), device="cuda", dtype=torch.float64)
    u = (q * s) @ v.t().contiguous()
    u = (u if r >= c else u.t()).float().contiguous()
    # values of the norm's 1 / sqrt(short side): up to five steps to 0.7
    grown = min(5.0, math.log(0.7 * math.sqrt(min(r, c)) / 0.2) / math.log(COEF[0]))
    out = torch.empty_like(u)
    H.kernel_orthogonalize([u], [out])
    assert rel(out, reference(u)) <= 15 * 2.0 ** -22 * COEF[0] ** grown
    # of low rank, with noise 10^5 times smaller
    u = (torch.randn(r, 3, generator=g, device="cuda") @ torch.randn(3, c, generator=g, device="cuda")) + 1e-5 * torch.randn(r, c, generator=g, device="cuda")
    H.kernel_orthogonalize([u], [out])
    assert (out.double() - reference(u)).norm().item() <= 5 * 2.0 ** -21 * COEF[0] ** 5 * math.sqrt(min(r, c))


@pytest.mark.parametrize("shapes", [[(512, 700), (700, 512), (1100, 600)], [(1500, 3000), (2900, 1400), (2048, 2048), (600, 520)]])
def test_results_in_bf16(shapes):
    """Large matrices take fewer products for a result in bf16, each within 2^-9 of the 2-norm (as its rounding is) whatever the spectrum."""
    import torch
    import paper_2401_15207_amd as H
    g = torch.Generator(device="cuda")
    g.manual_seed(len(shapes))
    for noise in (1.0, 1e-3, 1e-5):
        u = [torch.randn(r, 9, generator=g, device="cuda") @ torch.randn(9, c, generator=g, device="cuda") + noise * torch.randn(r, c, generator=g, device="cuda")
             for r, c in shapes]
        out, exact = [torch.empty(s, device="cuda", dtype=torch.bfloat16) for s in shapes], [torch.empty(s, device="cuda") for s in shapes]
        H.kernel_orthogonalize(u, out)
        H.kernel_orthogonalize(u, exact)
        again = [torch.empty_like(x) for x in out]
        H.kernel_orthogonalize(u, again)
        for a, b, c, x in zip(u, out, exact, again):
            want = reference(a)
            assert rel(b, want) <= 2.0 ** -9 + 2.0 ** -9, (noise, tuple(a.shape))
            # (fp32 results keep all of them; roundings of 22 bits, amplified by low rank)
            assert (c.double() - want).norm().item() <= 5 * 2.0 ** -21 * COEF[0] ** 5 * math.sqrt(min(a.shape))
            assert torch.equal(b, x)


@pytest.mark.parametrize("shapes", [[(2048, 9000)], [(8700, 2000)], [(2304, 2200), (2048, 9100)], [(4096, 4200)]])
def test_last_rounds_of_large_tiles(shapes):
    import torch
    import paper_2401_15207_amd as H
    u = [conditioned(r, c, 40 + i) for i, (r, c) in enumerate(shapes)]
    want = [reference(x) for x in u]
    # random matrices: singular values within a factor that `any` covers; smallest over norm at least 1e-3, so five steps' growth of a rounding at most
    for dt, tol in ((torch.float32, 15 * 2.0 ** -22 * COEF[0] ** 5), (torch.bfloat16, 2.0 ** -8 + 2.0 ** -9)):
        outs = [[torch.empty(x.shape, device="cuda", dtype=dt) for x in u] for _ in range(2)]
        for o in outs:
            H.kernel_orthogonalize(u, o)
        for a, b, w in zip(outs[0], outs[1], want):
            assert rel(a, w) <= tol
            assert torch.equal(a, b)     # whoever adds a tile's sums


def test_update_of_large_matrices():
    import torch
    import paper_2401_15207_amd as H
    shapes = [(1400, 2900), (2900, 1400), (520, 600)]
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    w, gr, m = ([torch.randn(s, generator=g, device="cuda") * size for s in shapes] for size in (0.02, 1e-4, 1e-3))
    opt = dict(kind="muon", lr=1e-2, momentum=0.95, weight_decay=0.0)
    for copies in (True, False):
        w1, m1 = [x.clone() for x in w], [x.clone() for x in m]
        cc = [torch.empty(s, device="cuda", dtype=torch.bfloat16) for s in shapes] if copies else None
        H.kernel_muon(opt, w1, gr, m1, cc)
        for i, s in enumerate(shapes):
            m64 = 0.95 * m[i].double() + gr[i].double()
            o = reference(gr[i].double() + 0.95 * m64) * 1e-2 * 0.2 * math.sqrt(max(s))
            # an fp32 model's update keeps all products, a bf16 model's is within 2^-9 of the step
            assert (w1[i].double() - (w[i].double() - o)).norm().item() <= (2.0 ** -9 if copies else 15 * 2.0 ** -22 * COEF[0] ** 5) * o.norm().item() + 2.0 ** -23 * w[i].norm().item()
            assert rel(m1[i], m64) <= 2.0 ** -23
            assert not copies or torch.equal(cc[i], w1[i].to(torch.bfloat16))


def test_other_steps_and_coefficients():
    import torch
    import paper_2401_15207_amd as H
    u = conditioned(90, 200, 3)
    out = torch.empty_like(u)
    for steps, coef in ((1, COEF), (12, (1.875, -1.25, 0.375)), (3, (1.5, -0.5, 0.0)), (4, (2.0, -1.5, 0.5))):
        H.kernel_orthogonalize([u], [out], steps=steps, coefficients=coef)
        want = reference(u, steps, coef)
        assert rel(out, want) <= 15 * 2.0 ** -22 * COEF[0] ** 5, (steps, coef)
    assert abs(torch.linalg.svdvals(reference(u, 12, (1.875, -1.25, 0.375)))[-1].item() - 1.0) < 1e-6


def test_scale_zeros_and_numbers_that_are_none():
    import torch
    import paper_2401_15207_amd as H
    u = conditioned(70, 130, 5)
    base, out = torch.empty_like(u), torch.empty_like(u)
    H.kernel_orthogonalize([u], [base], eps=1e-30)
    for power in (-80, -30, 40, 100):                # the norm takes any power of two out: the same bits
        H.kernel_orthogonalize([u * 2.0 ** power], [out], eps=1e-30)
        assert torch.equal(out, base), power
    H.kernel_orthogonalize([u * 1e-20], [out])       # below eps: the linear part alone, three times a
    want = reference(u * 1e-20)
    assert rel(out, want) <= WELL
    H.kernel_orthogonalize([torch.zeros_like(u)], [out])
    assert (out == 0).all()
    for bad in (math.nan, math.inf):
        v = u.clone()
        v[3, 4] = bad
        other = torch.empty_like(u)
        H.kernel_orthogonalize([v, u], [out, other], eps=1e-30)
        assert torch.isnan(out).all() and torch.equal(other, base)     # its neighbour in the list is not touched by it


def test_transposed_in_place_repeated_and_in_a_graph():
    import torch
    import paper_2401_15207_amd as H
    u, stream = conditioned(150, 400, 9), torch.cuda.Stream()
    want = reference(u)
    a, b = torch.empty_like(u), torch.empty(400, 150, device="cuda")
    H.kernel_orthogonalize([u, u.t().contiguous()], [a, b])
    assert rel(a, want) <= 4 * WELL and rel(b.t(), want) <= 4 * WELL
    v = u.clone()
    H.kernel_orthogonalize([v], [v])
    assert torch.equal(v, a)
    ws = torch.full((H.kernel_orthogonalize_bytes([(150, 400)]),), 255, device="cuda", dtype=torch.uint8)    # NaN wherever it is not written first
    c, src = torch.empty_like(u), u.clone()
    torch.cuda.synchronize()
    H.kernel_orthogonalize([src], [c], workspace=ws, stream=stream)
    stream.synchronize()
    assert torch.equal(c, a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        H.kernel_orthogonalize([src], [c], workspace=ws)
    for _ in range(3):
        c.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, a)


def test_update():
    import torch
    import paper_2401_15207_amd as H
    shapes = [(96, 96), (40, 131), (300, 64), (1, 20)]
    opt = dict(kind="muon", lr=2e-3, momentum=0.9, weight_decay=0.1)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    w = [torch.randn(s, generator=g, device="cuda") * 0.02 for s in shapes]
    m = [torch.zeros(s, device="cuda") for s in shapes]
    cc = [torch.empty(s, device="cuda", dtype=torch.bfloat16) for s in shapes]
    w64, m64 = [x.double() for x in w], [x.double() for x in m]
    for step in range(3):
        gr = [torch.randn(s, generator=g, device="cuda") * 1e-4 for s in shapes]
        H.kernel_muon(opt, w, gr, m, cc)
        for i, s in enumerate(shapes):
            m64[i] = 0.9 * m64[i] + gr[i].double()
            o = reference(gr[i].double() + 0.9 * m64[i])
            w64[i] = (1 - 2e-3 * 0.1) * w64[i] - 2e-3 * 0.2 * math.sqrt(max(s)) * o
            assert rel(m[i], m64[i]) <= (step + 1) * 2.0 ** -23
            # each step's orthogonal part within 15 2^-22 a^4 of itself, its size against the weights' 0.02: 0.02 sqrt(max s) / sqrt(count / n) at most
            step_size = 2e-3 * 0.2 * math.sqrt(max(s)) * o.norm().item()
            assert (w[i].double() - w64[i]).norm().item() <= (step + 1) * (15 * 2.0 ** -22 * COEF[0] ** 4 * step_size + 2.0 ** -23 * w64[i].norm().item())
            assert torch.equal(cc[i], w[i].to(torch.bfloat16))
    before = [x.clone() for x in w]
    H.kernel_muon(dict(opt, lr=0.0), w, gr, m)      # no copies, and a rate of zero
    assert all(torch.equal(a, b) for a, b in zip(before, w))


def test_refusals():
    import torch
    import paper_2401_15207_amd as H
    u, out = torch.randn(8, 9, device="cuda"), torch.empty(8, 9, device="cuda")
    for bad in (dict(steps=0), dict(steps=17), dict(eps=0.0), dict(eps=math.inf), dict(coefficients=(1e3, 0.0, 0.0)), dict(coefficients=(math.nan, 1.0, 0.0)),
                dict(steps=16, coefficients=(3.0, 3.0, 3.0)), dict(steps=2, coefficients=(0.0, 0.0, 1.0))):
        with pytest.raises(H.HiftError):
            H.kernel_orthogonalize([u], [out], **bad)
    large = torch.randn(300, 300, device="cuda")     # (smaller ones need no work space)
    with pytest.raises(H.HiftError):
        H.kernel_orthogonalize([large], [large.clone()], workspace=torch.empty(64, device="cuda"))
    for a, b in (([u], []), ([u], [out[:7]]), ([u.t()], [out.t()]), ([u.double()], [out]), ([u], [out.cpu()]), ([u, u.bfloat16()], [out, out])):
        with pytest.raises(ValueError):
            H.kernel_orthogonalize(a, b)
    H.kernel_orthogonalize([], [])
    H.kernel_orthogonalize([u[:0], u], [out[:0], out])
    assert torch.isfinite(out).all()
    opt = dict(kind="muon", lr=1e-3, momentum=0.9)
    for bad in (dict(opt, kind="adamw"), dict(opt, momentum=1.0), dict(opt, momentum=-0.1)):
        with pytest.raises(H.HiftError):
            H.kernel_muon(bad, [u], [u.clone()], [out])
    for args in (([u], [u[:7]], [out]), ([u], [u.bfloat16()], [out]), ([u], [u], []), ([u], [u], [out], [out]), ([u[:, :5]], [u[:, :5]], [out[:, :5]])):
        with pytest.raises(ValueError):
            H.kernel_muon(opt, *args)
