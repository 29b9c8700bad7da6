"""Attention over a paged cache with the caller's own work space on the GPU."""
import pytest
import torch

import paper_2401_15207_amd as H
from tests.test_gpu_paged import Made

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,heads,kv,hd", [([(3925, 455)], 8, 8, 64), ([(4200, 128)], 32, 8, 128), ([(4000, 16), (37, 16), (4380, 16), (0, 16)], 32, 8, 128), ([(5000, 1)], 8, 1, 80)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_buffer_for_all_bounds_and_windows(dtype, tokens, heads, kv, hd):
    """Asked for once, without a window and for the longest keys; taken by every shorter bound and window, with the result of a buffer of the call's own."""
    m = Made(tokens, heads, kv, hd, 16, dtype, seed=3)
    n = H.kernel_attention_paged_bytes(m.cache, m.rows, heads, m.max_new, 16384)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    for bound in (0, 1000, 4096, 4200, m.max_length, 16384):
        for window in (0, 100, 3702):
            ws.fill_(0xFF)
            out, lse = m.attend(window=window, max_length=bound, workspace=ws) if bound else m.attend(window=window, workspace=ws)
            want, want_lse = m.attend(window=window, max_length=bound or None)
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
    m.check(out, lse, window=window)


def test_a_window_that_asks_for_more_than_none_did():
    """455 new tokens over 3925, window 3702: the keys' parts are cut by the window, and a buffer asked for without it has to do."""
    m = Made([(3925, 455)], 8, 8, 64, 16, "bf16", seed=4)
    whole, part = (H.kernel_attention_paged_bytes(m.cache, m.rows, 8, m.max_new, m.max_length, window=w) for w in (0, 3702))
    assert 0 < part <= whole
    out, lse = m.attend(window=3702, workspace=torch.empty(whole, dtype=torch.uint8, device="cuda"))
    m.check(out, lse, window=3702)
