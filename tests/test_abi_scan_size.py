"""The recurrence's limit on B T H together, where the product does not fit 64 bits, without a GPU."""
import pytest

from paper_1805_08899_amd import binding as eb

A = 0x10000  # a fake, aligned, never dereferenced device address
BIG = 1 << 60


@pytest.mark.parametrize("B,T,H", [(1 << 24, 1 << 24, 1 << 20), (1 << 24, 1 << 24, 1 << 16), (1 << 24, 1 << 20, 1 << 20), (1 << 24, 1 << 24, (1 << 20) - (1 << 16)),
                                   (1 << 24, 1 << 16, 2), (1 << 20, 1 << 20, 2), (1 << 22, 1 << 22, 1 << 20), (1 << 24, 1 << 24, 1)])
def test_products_above_the_limit(B, T, H):
    d = eb.make_scan_desc(B, T, H)
    # G and dh are NULL: where the size is taken, the call still stops at a host check
    assert eb.echo_scan_fwd(d, None, A, A, A, A, A, A, BIG) == eb.ECHO_ERR_SHAPE
    assert eb.echo_scan_bwd(d, None, A, A, A, A, A, A, A, BIG) == eb.ECHO_ERR_SHAPE
    assert eb.echo_scan_states_bytes(d) == eb.echo_scan_fwd_workspace_bytes(d) == eb.echo_scan_bwd_workspace_bytes(d) == 0


@pytest.mark.parametrize("B,T,H", [(1 << 24, 1 << 16, 1), (1 << 4, 1 << 16, 1 << 20), (1 << 16, 1 << 24, 1), (1 << 20, 1, 1 << 20)])
def test_products_at_the_limit(B, T, H):
    d = eb.make_scan_desc(B, T, H)
    assert eb.echo_scan_fwd(d, None, A, A, A, A, A, A, BIG) == eb.ECHO_ERR_NULL
    assert eb.echo_scan_states_bytes(d) == B * -(-T // eb.ECHO_SCAN_CHUNK) * H * 4
