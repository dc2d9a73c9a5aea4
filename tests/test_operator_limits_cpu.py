"""The largest sizes that the library accepts, without a GPU: the checks come before any device work, so the addresses
here are never read."""
from paper_2509_21301_amd import nova

FAKE = 1 << 20
LIB = nova.lib


def test_logit_rows_fit_a_grid():
    """A row of the joining kernel is a workgroup of 512 threads, and a grid has fewer than 2^32 threads."""
    def call(rows):
        return LIB.nova_logprobs(FAKE, 1, 152064, rows, 152064, None, 0, None, FAKE, 4, FAKE, FAKE, FAKE, 0, None)
    assert call(1 << 23) == nova.EUNSUPPORTED
    assert call((1 << 23) - 1) == nova.ENOSPACE                       # accepted, but for its workspace
    assert ((1 << 23) - 1) * 512 < 1 << 32
