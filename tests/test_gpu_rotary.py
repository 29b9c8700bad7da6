"""Rotary positions on the GPU: the table of angles and the rotation of heads, both directions, against the definitions in 64 bits."""
import math

import pytest
import torch

import paper_2401_15207_amd as H

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def rates(rot, base=10000.0, scaling="plain", factor=1.0, trained=1.0, slow=0.0, fast=1.0):
    out = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "base" else base
        r = b ** (-2.0 * i / rot)
        if scaling == "linear":
            r = r / factor
        if scaling == "parts":
            k = min(1.0, max(0.0, (trained * r / (2 * math.pi) - slow) / (fast - slow)))
            r = k * r + (1 - k) * r / factor
        out.append(r)
    return torch.tensor(out, dtype=torch.float64)


def table(rows, rot, device="cuda"):
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * rates(rot)
    return torch.stack([angle.cos(), angle.sin()], 2).float().to(device)


def turned(x, cs, layout, backward=False):
    """x [rows, heads, head_dim] and cs [rows, rot / 2, 2]: the result and the sizes of what is added up for it, in 64 bits."""
    x, cs = x.double(), cs.double()
    half = cs.shape[1]
    at = torch.arange(half, device=x.device)
    one, two = (at, at + half) if layout == "halves" else (2 * at, 2 * at + 1)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1] * (-1 if backward else 1)
    y, size = x.clone(), x.abs()
    y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., two] * c + x[..., one] * s
    size[..., one] = (x[..., one] * c).abs() + (x[..., two] * s).abs()
    size[..., two] = (x[..., two] * c).abs() + (x[..., one] * s).abs()
    return y, size


def close(got, want, size, dtype):
    """Two products and a sum in fp32 (three roundings of at most 2^-24 of the sizes) and one rounding to the type."""
    far = (got.double() - want).abs()
    tol = 3 * 2.0 ** -24 * size + HALF_STEP[dtype] * (want.abs() + 3 * 2.0 ** -24 * size) + 1e-37
    assert (far <= tol).all(), f"off by up to {(far / tol).max().item():.2f} of the tolerance"


@pytest.mark.parametrize("scaling", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                     dict(scaling="parts", factor=16.0, trained=4096.0, slow=1.0, fast=32.0)])
@pytest.mark.parametrize("rot,count,first,amplitude", [(128, 300, 0, 1.0), (64, 1, 1000003, 1.25), (6, 77, 5, 1.0), (256, 33, 131072, 0.5)])
def test_table(scaling, rot, count, first, amplitude):
    out = torch.full((count + 1, rot // 2, 2), -7.0, device="cuda")
    H.kernel_rotary_table(dict(scaling, rot=rot, base=10000.0, amplitude=amplitude), out[:count], first=first)
    angle = (torch.arange(count, dtype=torch.float64) + first)[:, None] * rates(rot, **scaling)
    want = amplitude * torch.stack([angle.cos(), angle.sin()], 2)
    # rounding to fp32, and the angle: its rate is off by a few 2^-53, which the position multiplies (both here and there)
    tol = amplitude * (2.0 ** -24 + (first + count) * 2.0 ** -49)
    assert (out[:count].cpu().double() - want).abs().max().item() <= tol
    assert (out[count] == -7.0).all()


def test_table_of_two_columns():
    out = torch.empty(50, 1, 2, device="cuda")
    H.kernel_rotary_table(dict(rot=2), out)
    at = torch.arange(50, dtype=torch.float64)
    assert (out.cpu().double()[:, 0] - torch.stack([at.cos(), at.sin()], 1)).abs().max().item() <= 2.0 ** -24 + 50 * 2.0 ** -49


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("rows,heads,head_dim,rot,pad", [(1, 1, 2, 2, 0), (3, 5, 16, 16, 0), (7, 4, 128, 64, 8), (5, 3, 80, 20, 5), (130, 40, 128, 128, 64),
                                                         (9, 2, 34, 10, 1), (2100, 33, 64, 64, 0), (600, 12, 256, 256, 0)])
def test_rotation(dtype, layout, backward, rows, heads, head_dim, rot, pad):
    g = torch.Generator().manual_seed(rows + rot)
    width = heads * head_dim
    x = torch.randn(rows, width + pad, generator=g).to("cuda", DT[dtype])
    cs = table(64, rot)
    positions = torch.randint(0, 64, (rows,), generator=g, dtype=torch.int32).cuda()
    y = torch.full((rows, width + 3), -7.0, device="cuda", dtype=DT[dtype])
    H.kernel_rotary(x, heads, head_dim, y, cs, positions=positions, layout=layout, backward=backward)
    want, size = turned(x[:, :width].reshape(rows, heads, head_dim), cs[positions.long()], layout, backward)
    close(y[:, :width].reshape(rows, heads, head_dim), want, size, DT[dtype])
    assert (y[:, width:] == -7.0).all()
    if rot < head_dim:
        keep = slice(rot, head_dim)
        assert torch.equal(y[:, :width].reshape(rows, heads, head_dim)[..., keep], x[:, :width].reshape(rows, heads, head_dim)[..., keep])
    # in place, the same bits, and nothing else of the rows is touched
    z = x.clone()
    H.kernel_rotary(z, heads, head_dim, z, cs, positions=positions, layout=layout, backward=backward)
    assert torch.equal(z[:, :width], y[:, :width]) and torch.equal(z[:, width:], x[:, width:])


def test_positions_follow_the_sequence_and_are_kept_in_the_table():
    x, cs = torch.randn(10, 32, device="cuda"), table(4, 32)
    y, z = torch.empty_like(x), torch.empty_like(x)
    H.kernel_rotary(x, 1, 32, y, cs, seq=4)
    H.kernel_rotary(x, 1, 32, z, cs, positions=torch.arange(10, device="cuda", dtype=torch.int32) % 4)
    assert torch.equal(y, z)
    H.kernel_rotary(x, 1, 32, y, cs, positions=torch.full((10,), 2 ** 31 - 1, device="cuda", dtype=torch.int32))
    H.kernel_rotary(x, 1, 32, z, cs, positions=torch.full((10,), 3, device="cuda", dtype=torch.int32))
    assert torch.equal(y, z)
    H.kernel_rotary(x, 1, 32, y, cs, positions=torch.full((10,), -2 ** 31, device="cuda", dtype=torch.int32))
    assert torch.equal(y, x)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_gradient(layout):
    """The gradient of sum(w * rotated(x)): by differences, and rotating forth and back with amplitude a gives a^2 x."""
    rows, heads, hd, rot = 6, 3, 24, 16
    g = torch.Generator().manual_seed(3)
    x, w = (torch.randn(rows, heads * hd, generator=g).cuda() for _ in range(2))
    cs = torch.empty(rows, rot // 2, 2, device="cuda")
    H.kernel_rotary_table(dict(rot=rot, amplitude=1.5), cs, first=11)
    d, y = torch.empty_like(x), torch.empty_like(x)
    H.kernel_rotary(w, heads, hd, d, cs, seq=rows, layout=layout, backward=True)
    H.kernel_rotary(x, heads, hd, y, cs, seq=rows, layout=layout)

    def value(v):
        out, _ = turned(v.view(rows, heads, hd), cs, layout)
        return (out.view(rows, -1) * w.double()).sum().item()

    for at in [(0, 0), (1, 7), (2, 8), (3, 15), (4, 16), (5, 71), (2, 33)]:
        up, down = x.double().clone(), x.double().clone()
        up[at] += 1e-3
        down[at] -= 1e-3
        # linear in x: the difference is exact up to 64-bit rounding; the kernel's value has three roundings of sizes up to 3 |w|
        assert abs((value(up) - value(down)) / 2e-3 - d[at].item()) <= 1e-9 + 2.0 ** -22 * 3 * w.abs().max().item()
    back = torch.empty_like(x)
    H.kernel_rotary(y, heads, hd, back, cs, seq=rows, layout=layout, backward=True)
    want = x.view(rows, heads, hd).double().clone()
    want[..., :rot] *= 1.5 ** 2
    assert (back.view(rows, heads, hd).double() - want).abs().max().item() <= 12 * 2.0 ** -24 * 2.25 * x.abs().max().item() * 2


def test_agrees_with_the_attention_backward_kernels_angles():
    """A row turned by the table and back is what hift_kernel_attention_bwd's un-rotation undoes: halves, one angle per position."""
    x = torch.randn(64, 2 * 128, device="cuda").bfloat16()
    cs = table(64, 128)
    y, z = torch.empty_like(x), torch.empty_like(x)
    H.kernel_rotary(x, 2, 128, y, cs, seq=64)
    H.kernel_rotary(y, 2, 128, z, cs, seq=64, backward=True)
    # two roundings to bf16 of numbers up to sqrt(2) of the row's largest pair
    assert (z.float() - x.float()).abs().max().item() <= 3 * 2.0 ** -8 * x.float().abs().max().item() * math.sqrt(2)


def test_zero_rows_and_another_stream():
    cs = table(8, 32)
    empty = torch.empty(0, 64, device="cuda")
    H.kernel_rotary(empty, 2, 32, empty, cs, seq=8)
    H.kernel_rotary_table(dict(rot=32), torch.empty(0, 16, 2, device="cuda"))
    x = torch.randn(8, 64, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    H.kernel_rotary(x, 2, 32, y, cs, seq=8)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    H.kernel_rotary(x, 2, 32, z, cs, seq=8, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(y, z)
