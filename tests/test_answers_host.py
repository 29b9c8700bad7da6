"""Refusals of the operators that write answers: on the CPU, with addresses that nothing reads."""
import ctypes as C

import pytest
import torch

import paper_2401_15207_amd as H
from paper_2401_15207_amd import binding as B

A = 1 << 20   # an address, 16-byte aligned; every call here is refused before anything is launched
EINVAL = -1


def table_call(first=0, count=4, cos_sin=A, **r):
    r = dict(dict(rot=64, base=10000.0, amplitude=1.0), **r)
    rot = B.Rotary(r["rot"], r.get("kind", 0), r["base"], r.get("factor", 1.0), r.get("trained", 1.0), r.get("slow", 0.0), r.get("fast", 1.0), r["amplitude"])
    return B.lib.hift_kernel_rotary_table(C.byref(rot), first, count, cos_sin, None)


@pytest.mark.parametrize("bad", [dict(rot=0), dict(rot=3), dict(rot=258), dict(rot=-2), dict(kind=4), dict(kind=-1), dict(base=0.0), dict(base=float("nan")),
                                 dict(base=float("inf")), dict(amplitude=0.0), dict(amplitude=float("nan")), dict(kind=1, factor=0.0), dict(kind=2, rot=2),
                                 dict(kind=2, factor=float("inf")), dict(kind=3, trained=0.0), dict(kind=3, slow=2.0, fast=2.0), dict(kind=3, fast=float("nan")),
                                 dict(first=-1), dict(count=-1), dict(first=2 ** 30, count=1), dict(first=2 ** 62, count=2 ** 62), dict(cos_sin=None), dict(cos_sin=A + 4),
                                 dict(base=0.5), dict(base=1e19), dict(kind=1, factor=0.5), dict(kind=1, factor=1e10)])
def test_table_refusals(bad):
    assert table_call(**bad) == EINVAL and B.lib.hift_last_error()


def test_table_of_nothing():
    assert table_call(count=0, cos_sin=None) == 0


def rotary_call(**o):
    a = dict(dict(dtype=1, layout=0, backward=0, rows=4, heads=2, head_dim=64, rot=64, x=A, ldx=128, y=2 * A, ldy=128, positions=None, seq=4, cos_sin=A, table_rows=4), **o)
    return B.lib.hift_kernel_rotary(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(layout=2), dict(rows=-1), dict(rows=2 ** 31), dict(heads=-1), dict(head_dim=0), dict(heads=2 ** 20, head_dim=64, ldx=2 ** 26, ldy=2 ** 26),
                                 dict(rot=0), dict(rot=63), dict(rot=66), dict(rot=-2), dict(ldx=127), dict(ldy=127), dict(x=None), dict(y=None), dict(x=A + 1), dict(y=A + 1),
                                 dict(positions=A + 2), dict(seq=0), dict(seq=5), dict(cos_sin=None), dict(cos_sin=A + 4), dict(table_rows=0), dict(table_rows=2 ** 31),
                                 dict(y=A, ldy=136), dict(dtype=0, x=A + 2)])
def test_rotary_refusals(bad):
    assert rotary_call(**bad) == EINVAL and B.lib.hift_last_error()


def test_rotary_of_nothing():
    assert rotary_call(rows=0, x=None, y=None) == 0
    assert rotary_call(heads=0, x=None, y=None) == 0


def cache_of(**o):
    a = dict(dict(dtype=1, kv_heads=2, head_dim=64, page=16, n_pages=8, sequences=3, max_pages=4, page_stride=2048, pages_ld=4, k=A, v=A, pages=A, lengths=A), **o)
    return B.Cache(*a.values())


BAD_CACHE = [dict(dtype=2), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136), dict(dtype=0, head_dim=6), dict(page=0), dict(page=8),
             dict(page=24), dict(page=2 ** 17), dict(page=-16), dict(n_pages=-1), dict(sequences=-1), dict(max_pages=-1), dict(max_pages=2 ** 27), dict(page_stride=2047),
             dict(page_stride=2052), dict(pages_ld=3), dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2), dict(pages=None), dict(lengths=None)]
BAD_ROWS = [dict(rows=-1), dict(rows=2 ** 30 + 1), dict(max_new=-1), dict(starts=None), dict(heads=0), dict(heads=5), dict(heads=65538), dict(rows=2 ** 30, max_new=2 ** 30)]


def append_call(cache=None, **o):
    a = dict(dict(rows=8, starts=A, max_new=4, heads=4, layout=0, rot=64, cos_sin=A, table_rows=4, qkv=A, ld=512, q_out=2 * A, ldq=256), **o)
    return B.lib.hift_kernel_cache_append(C.byref(cache or cache_of()), *a.values(), None)


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_append_refuses_caches(bad):
    assert append_call(cache_of(**bad)) == EINVAL and B.lib.hift_last_error()


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(layout=3), dict(rot=1), dict(rot=66), dict(cos_sin=None), dict(cos_sin=A + 4), dict(table_rows=0), dict(qkv=None), dict(ld=511),
                                            dict(ld=516), dict(ldq=255), dict(ldq=260), dict(qkv=A + 8), dict(q_out=A + 8), dict(q_out=A)])
def test_append_refusals(bad):
    assert append_call(**bad) == EINVAL and B.lib.hift_last_error()


def test_append_of_nothing():
    assert append_call(rows=0, starts=None, qkv=None) == 0
    assert append_call(cache_of(sequences=0, pages=None, lengths=None), starts=None) == 0
    assert append_call(max_new=0, starts=None) == 0


def attend_call(cache=None, **o):
    a = dict(dict(rows=8, starts=A, max_new=4, max_length=5000, heads=4, window=0, scale=0.125, q=A, ldq=256, out=2 * A, ldo=256, lse=None, workspace=A, nbytes=2 ** 40), **o)
    return B.lib.hift_kernel_attention_paged(C.byref(cache or cache_of(max_pages=4096, pages_ld=4096)), *a.values(), None)


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_attention_refuses_caches(bad):
    assert attend_call(cache_of(**bad)) == EINVAL and B.lib.hift_last_error()


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(max_length=-1), dict(window=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None),
                                            dict(out=None), dict(q=A + 8), dict(out=A + 8), dict(ldq=255), dict(ldo=255), dict(ldq=260), dict(ldo=260), dict(out=A, ldo=512),
                                            dict(lse=A + 2), dict(workspace=None), dict(workspace=A + 8), dict(nbytes=16)])
def test_attention_refusals(bad):
    assert attend_call(**bad) == EINVAL and B.lib.hift_last_error()


def test_attention_of_nothing():
    assert attend_call(rows=0, starts=None, q=None, out=None) == 0
    assert attend_call(cache_of(sequences=0, pages=None, lengths=None), starts=None) == 0


def test_workspace_sizes():
    n = C.c_size_t()
    c = cache_of(max_pages=4096, pages_ld=4096)
    call = B.lib.hift_kernel_attention_paged_bytes
    assert call(C.byref(c), 3, 1, 60000, 4, 0, C.byref(n)) == 0 and n.value > 0
    most = n.value
    # a window reads less, and a short bound nothing that is worth splitting
    assert call(C.byref(c), 3, 1, 60000, 4, 128, C.byref(n)) == 0 and n.value < most
    assert call(C.byref(c), 3, 1, 100, 4, 0, C.byref(n)) == 0 and n.value == 0
    assert call(C.byref(c), 0, 1, 60000, 4, 0, C.byref(n)) == 0 and n.value == 0
    assert call(C.byref(c), 3, 1, 60000, 4, 0, None) == EINVAL


def adjust_call(backward=False, by=None, **o):
    d = dict(dict(tokens=A, n_tokens=10, begin=A, end=A, repetition=1.0, presence=0.0, frequency=0.0, bias=A, ld_bias=0, allowed=A, ld_allowed=0), **(by if isinstance(by, dict) else {}))
    b = None if by == "null" else C.byref(B.Adjust(*d.values()))
    a = dict(dict(dtype=1, rows=4, vocab=100, ld=100, logits=A), **{k: v for k, v in o.items() if k in ("dtype", "rows", "vocab", "ld", "logits")})
    if backward:
        e = dict(dict(ldg=100, g=2 * A, ldd=100, d=3 * A), **{k: v for k, v in o.items() if k in ("ldg", "g", "ldd", "d")})
        return B.lib.hift_kernel_adjust_logits_bwd(*a.values(), b, *e.values(), None)
    e = dict(dict(ldo=100, out=2 * A), **{k: v for k, v in o.items() if k in ("ldo", "out")})
    return B.lib.hift_kernel_adjust_logits(*a.values(), b, *e.values(), None)


SHAPES = [dict(dtype=2), dict(rows=-1), dict(rows=2 ** 23), dict(vocab=0), dict(vocab=2 ** 30 + 1, ld=2 ** 31), dict(ld=99), dict(logits=None), dict(logits=A + 1),
          dict(rows=2 ** 22, vocab=2 ** 27, ld=2 ** 27, ldo=2 ** 27, ldg=2 ** 27, ldd=2 ** 27)]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", SHAPES)
def test_adjust_refuses_shapes(backward, bad):
    assert adjust_call(backward, **bad) == EINVAL and B.lib.hift_last_error()


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", [dict(repetition=0.0), dict(repetition=-1.0), dict(repetition=float("nan")), dict(repetition=float("inf")), dict(repetition=2.0 ** 61),
                                 dict(presence=float("inf")), dict(frequency=float("nan")), dict(n_tokens=-1), dict(begin=None), dict(end=None), dict(ld_bias=99), dict(ld_bias=-1),
                                 dict(ld_allowed=3), dict(tokens=A + 2), dict(bias=A + 2), dict(allowed=A + 1), dict(begin=A + 4), dict(end=A + 4)])
def test_adjust_refuses_what_it_adjusts_by(backward, bad):
    assert adjust_call(backward, by=bad) == EINVAL and B.lib.hift_last_error()


def test_adjust_refusals():
    for bad in (dict(ldo=99), dict(out=None), dict(out=A + 1), dict(out=A, ldo=101), dict(by="null")):
        assert adjust_call(**bad) == EINVAL, bad
    for bad in (dict(ldg=99), dict(ldd=99), dict(g=None), dict(d=None), dict(g=A + 1), dict(d=A + 1), dict(d=A), dict(d=2 * A, ldd=101), dict(by="null")):
        assert adjust_call(True, **bad) == EINVAL, bad
    assert adjust_call(rows=0, logits=None, out=None) == 0 and adjust_call(True, rows=0, logits=None, g=None, d=None) == 0


def test_binding_refuses_host_tensors():
    x, cs = torch.zeros(4, 64), torch.zeros(4, 16, 2)
    for call in (lambda: H.kernel_rotary(x, 2, 32, x, cs, seq=4), lambda: H.kernel_rotary_table(dict(rot=32), cs),
                 lambda: H.PagedCache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)),
                 lambda: H.kernel_adjust_logits(x, 64, x), lambda: H.kernel_adjust_logits_bwd(x, 64, x, x)):
        with pytest.raises(ValueError):
            call()
