"""Argument checks of the score entry points that need no GPU: calls without rows launch nothing."""
import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2401_15207_amd as H
    return H.lib


@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_longer_than_the_kernels_count(lib, dtype):
    """Positions in a row are counted in 32 bits with a launch's stride on top: 2^30 entries at most."""
    forward = lambda V: lib.hift_kernel_token_logprob(dtype, 0, V, V, None, None, 1.0, 0, None, None, None, None, None, None)  # noqa: E731
    backward = lambda V: lib.hift_kernel_token_logprob_bwd(dtype, 0, V, V, None, None, 1.0, None, None, None, None, V, None, None)  # noqa: E731
    for call in (forward, backward):
        assert call(2 ** 30) == 0 and call(1) == 0
        for V in (2 ** 30 + 1, 2 ** 31 - 1, 0, -1):
            assert call(V) == -1, V
        assert b"entries" in lib.hift_last_error()


def test_rows_and_shapes(lib):
    assert lib.hift_kernel_token_logprob(0, 0, 8, 7, None, None, 1.0, 0, None, None, None, None, None, None) == -1      # rows overlap
    assert lib.hift_kernel_token_logprob(0, -1, 8, 8, None, None, 1.0, 0, None, None, None, None, None, None) == -1
    assert lib.hift_kernel_token_logprob(2, 0, 8, 8, None, None, 1.0, 0, None, None, None, None, None, None) == -1      # type
