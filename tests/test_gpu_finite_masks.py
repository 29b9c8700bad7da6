"""Log probabilities, entropies, alternatives and gradients of rows whose masked entries are large finite numbers, against 64 bits.

Tolerances.  Every row here has its entries of weight either within 50 of 0 or at one and the same value far from it, so that a probability depends
on differences that are formed exactly or within 2^-24 of themselves: 2^-22 (|m| + |z - m| + 16) for a log probability, |m| counted up to 4096
(rows whose largest z is farther from 0 subtract it before anything else is rounded), where those with |z - m| of thousands and more are
compared as fp32 numbers (they round to -inf beyond that range).  Gradients: as relatively exact as the log probability is absolutely, one
rounding of the type on top."""
import math

import pytest

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "fp32"]
MASKS = ["lowest", -1e30, -1e10, -1e9, -65504.0]
PLACES = ["last", "first", "both ends", "run", "nearly all", "all but one", "half", "thread"]
SIZES = [(7, 64, 0), (5, 4099, 0), (3, 50265, 0), (2, 32000, 0), (300, 777, 1)]


def types():
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}


def value_of(mask, dt):
    import torch
    return torch.finfo(dt).min if mask == "lowest" else mask


def masked_columns(place, vocab, g):
    import torch
    on = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    if place in ("last", "both ends"):
        on[-1] = True
    if place in ("first", "both ends"):
        on[:2] = True
    if place == "run":
        on[vocab // 3:vocab // 3 + max(1, vocab // 4)] = True
    elif place == "nearly all":
        on[:] = True
        on[torch.randint(0, vocab, (max(1, min(100, vocab // 10)),), generator=g, device="cuda")] = False
    elif place == "all but one":
        on[:] = True
        on[vocab // 2] = False
    elif place == "half":
        on = torch.rand(vocab, generator=g, device="cuda") < 0.5
    elif place == "thread":      # every other run of 16 entries, so that some threads see nothing else
        on = torch.arange(vocab, device="cuda") // 16 % 2 == 0
    return on


def check(x, vocab, targets, scale, top):
    """Forward and gradient of logits x [rows, >= vocab] against 64 bits."""
    import torch
    import paper_2401_15207_amd as H
    rows, dt = x.shape[0], x.dtype
    f = dict(device="cuda", dtype=torch.float32)
    logp, ent, stats = torch.full((rows,), 77.0, **f), torch.full((rows,), 77.0, **f), torch.full((rows, 2), 77.0, **f)
    top_logp, top_ids = torch.full((rows, top), 77.0, **f), torch.full((rows, top), -77, device="cuda", dtype=torch.int32)
    H.kernel_token_logprob(x, vocab, targets, scale, logp, ent, stats, top_logp, top_ids)
    s = torch.tensor(scale, dtype=torch.float32).double().item()
    z = x[:, :vocab].double() * s
    m = z.max(1, keepdim=True).values
    lp = z - m - (z - m).exp().sum(1, keepdim=True).log()
    p = lp.exp()
    entropy = torch.special.entr(p).sum(1)
    tol = 2.0 ** -22 * (torch.where(m.abs() <= 4096.0, m.abs(), 0.0) + (z - m).abs().clamp(max=1e4) + 16.0)

    def close(got, want, slack):
        far = want < -1e4                # rounded to fp32, and a few roundings off at most
        edge = want < -3.0e38
        ok = torch.where(far, (got.double() - want).abs() <= 2.0 ** -21 * want.abs(), (got.double() - want).abs() <= slack)
        return (ok | (edge & (got < -3.0e38))).all()

    has = targets >= 0
    at = targets.clamp(min=0).long().unsqueeze(1)
    assert (logp[~has] == 0).all()
    assert close(logp[has], lp.gather(1, at)[:, 0][has], tol.gather(1, at)[:, 0][has]), (logp, lp.gather(1, at)[:, 0])
    assert ((ent.double() - entropy).abs() <= 2.0 ** -22 * (2 * entropy + 66.0) + torch.where(m.abs() <= 4096.0, 2.0 ** -22 * m.abs(), 0.0)[:, 0]).all(), (ent, entropy)
    ids = torch.sort(x[:, :vocab].double(), dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(top_ids.long(), ids)
    assert close(top_logp, lp.gather(1, ids), tol.gather(1, ids))

    g = torch.Generator(device="cuda")
    g.manual_seed(rows + vocab)
    dl, dh = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    gl = torch.where(has, dl.double(), 0.0).unsqueeze(1)
    lp0 = torch.where(p > 0, lp, 0.0)
    want = s * (-p * (gl + dh.double().unsqueeze(1) * torch.where(p > 0, lp0 + entropy.unsqueeze(1), 0.0)))
    want.scatter_add_(1, at, gl * s)
    size = s * p * (gl.abs() + dh.double().abs().unsqueeze(1) * (lp0.abs() + entropy.unsqueeze(1) + 1.0))
    slack = 3 * size * torch.where(p > 0, tol, 0.0) + (2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -22) * want.abs() + 2.0 ** -23 * gl.abs() * s + 1e-37
    dx = torch.full_like(x, 5.0)
    H.kernel_token_logprob_bwd(x, vocab, targets, scale, stats, ent, dl, dh, dx)
    assert ((dx[:, :vocab].double() - want).abs() <= slack).all()
    assert (dx[:, vocab:] == 5.0).all()
    y = x.clone()
    H.kernel_token_logprob_bwd(y, vocab, targets, scale, stats, ent, dl, dh, y)
    assert torch.equal(y[:, :vocab], dx[:, :vocab])
    return logp, ent


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("place", PLACES)
def test_some_entries(place, mask, dtype):
    import torch
    dt = types()[dtype]
    for i, (rows, vocab, pad) in enumerate(SIZES):
        for scale in (1.0, 1.0 / 0.7):
            g = torch.Generator(device="cuda")
            g.manual_seed(rows * 1009 + vocab)
            x = torch.randn(rows, vocab + pad, generator=g, device="cuda") * 3.0
            on = masked_columns(place, vocab, g)
            x[:, :vocab][:, on] = value_of(mask, dt)
            targets = torch.randint(-1, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
            check(x.to(dt), vocab, targets, scale, min(8, vocab))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mask", [*MASKS, 1e9, 1e10, 1e30, 3e38])
def test_whole_rows_of_one_value(mask, dtype):
    """Probabilities 1 / V; also with the last entry far lower, and next to ordinary rows."""
    import torch
    dt = types()[dtype]
    for rows, vocab, pad in SIZES:
        for scale in (0.5, 1.0, 1.3, 2.0):
            g = torch.Generator(device="cuda")
            g.manual_seed(rows + vocab)
            x = torch.randn(rows, vocab + pad, generator=g, device="cuda") * 3.0
            x[::2, :vocab] = value_of(mask, dt)
            targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
            logp, ent = check(x.to(dt), vocab, targets, scale, min(5, vocab))
            assert ((logp[::2] + math.log(vocab)).abs() <= 1e-5).all() and ((ent[::2] - math.log(vocab)).abs() <= 1e-5).all()
            x[:, vocab - 1] = torch.finfo(dt).min
            x[:, 0] = -math.inf
            check(x.to(dt), vocab, targets.clamp(max=vocab - 2).clamp(min=1), scale, min(5, vocab))


def test_large_rows_that_differ_by_little():
    """Logits far from 0 whose differences are whole numbers: exact in fp32 at a scale that is a power of two."""
    import torch
    for offset, step in ((2.0 ** 11, 0.125), (-2.0 ** 11, 0.125), (2.0 ** 20, 0.25), (-2.0 ** 20, 0.25), (2.0 ** 23, 1.0), (-2.0 ** 23, 1.0), (-2.0 ** 24, 2.0), (2.0 ** 25, 4.0), (-2.0 ** 40, 2.0 ** 17)):
        for scale in (0.5, 1.0):
            g = torch.Generator(device="cuda")
            g.manual_seed(3)
            x = offset + step * torch.randint(0, 9, (6, 3001), generator=g, device="cuda").float()
            targets = torch.randint(0, 3001, (6,), generator=g, device="cuda", dtype=torch.int32)
            check(x, 3001, targets, scale, 4)
