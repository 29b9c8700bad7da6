"""Work space of the attention over a paged cache: what suffices for the longest keys suffices for shorter ones and for any window."""
import ctypes as C

import pytest

from tests.test_answers_host import A, B, attend_call, cache_of


def bytes_of(cache, rows, max_new, max_length, heads, window):
    n = C.c_size_t()
    assert B.lib.hift_kernel_attention_paged_bytes(C.byref(cache), rows, max_new, max_length, heads, window, C.byref(n)) == 0
    return n.value


# (dtype, sequences, new tokens of each, heads, kv_heads, head_dim): both kernels, parts of every size and whole keys
SHAPES = [(1, 1, 128, 32, 8, 128), (1, 4, 16, 32, 8, 128), (1, 1, 455, 8, 8, 64), (1, 1, 20, 8, 8, 128), (1, 1, 512, 32, 32, 128), (1, 8, 64, 32, 32, 128),
          (1, 64, 1, 32, 8, 128), (1, 1, 1, 8, 1, 128), (1, 16, 20, 8, 8, 16), (0, 1, 2048, 12, 12, 128), (0, 36, 30, 32, 16, 64), (0, 3, 77, 8, 2, 80), (0, 1, 1, 4, 4, 80),
          (0, 45, 38, 64, 32, 32)]
# both sides of every multiple of 64 keys, and far apart
LENGTHS = sorted({0, 1, 20000, 65536, 2 ** 40, *(64 * i + j for i in range(1, 140) for j in (0, 1)), *range(64, 9000, 173)})


@pytest.mark.parametrize("dtype,sequences,new,heads,kv,hd", SHAPES)
def test_more_keys_never_need_less(dtype, sequences, new, heads, kv, hd):
    c = cache_of(dtype=dtype, kv_heads=kv, head_dim=hd, page_stride=kv * 16 * hd, sequences=sequences, max_pages=2048, pages_ld=2048)
    rows = sequences * new
    for window in (0, 1, 700, 3702):
        needs = [bytes_of(c, rows, new, n, heads, window) for n in LENGTHS]
        assert needs == sorted(needs)
    for length in (300, 4000, 4380, 9001, 32768):
        needs = [bytes_of(c, rows, new, length, heads, w) for w in LENGTHS[1:] if w < 2 ** 31]
        assert needs == sorted(needs) and needs[-1] <= bytes_of(c, rows, new, length, heads, 0)
    # pages for longer sequences, too
    needs = []
    for pages in range(0, 1000, 7):
        c.max_pages = pages
        needs.append(bytes_of(c, rows, new, 2 ** 30, heads, 0))
    assert needs == sorted(needs)


def test_a_buffer_for_the_longest_bound_is_taken_at_a_shorter_one():
    """One buffer for a cache's lifetime; what is a byte too small is refused."""
    c = cache_of(kv_heads=8, head_dim=128, page_stride=8 * 16 * 128, sequences=1, max_pages=2048, pages_ld=2048)
    most = bytes_of(c, 128, 128, 32768, 32, 0)
    a = dict(rows=128, max_new=128, heads=32, ldq=4096, ldo=4096)
    for length in range(64, 32768, 1237):
        for window in (0, 100, 3702):
            need = bytes_of(c, 128, 128, length, 32, window)
            assert need <= most
            if need:
                assert attend_call(c, max_length=length, window=window, nbytes=need - 1, **a) == -1 and b"workspace" in B.lib.hift_last_error()
