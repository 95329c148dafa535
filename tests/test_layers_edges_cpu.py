"""Layer operators without a GPU: refusals of the C entry points that protect memory, and the
build where torch is missing."""
import pytest

from paper_2607_11985_gb300 import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_11985_gb300 import build
    build.build()


A = 1 << 20    # an address that is never read: every call below is refused


@pytest.mark.parametrize("dtype,e", [(0, 4), (1, 2), (2, 2)])
def test_misaligned_bias_gradients_are_refused(dtype, e):
    """Outputs lie on 16-byte boundaries: the sums of a bias gradient are stored in packs."""
    def linear(gb):
        return B.lib().vqc_linear_backward(dtype, dtype, 4, 8, 8, A, 8, A, 8, A, 8, A, 2, A, A, gb, A, 1 << 30, None)

    def gated(gb, gbu):
        return B.lib().vqc_gated_backward(dtype, 4, 8, 8, A, 8, A, 8, A, A, 8, A, 3, A, A, A, gb, gbu, A, 1 << 30, None)
    for off in (e, 8):
        assert linear(A + off) == 1 and "vqc_linear_backward: misaligned" in B.vqc_last_error()
        assert gated(A + off, A) == 1 and gated(A, A + off) == 1
        assert "vqc_gated_backward: misaligned" in B.vqc_last_error()
