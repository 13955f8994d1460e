"""Calls of the serving operators that would read or write beyond the storage described to them: decided on the host,
nothing enqueued, no device pointer read."""
import pytest

from paper_2504_06419_amd import spire
from tests.test_serving_abi_cpu import INVALID, OK, lattn, latent, msg


@pytest.mark.parametrize("blocks", [-1, 0, 1])
def test_more_sequences_than_a_contiguous_cache_has(blocks):
    view = latent(page_size=0, block_table=None, capacity=64, num_blocks=blocks)
    assert lattn(lat=view, B=2, wb=0) == INVALID and "num_blocks" in msg()


def test_as_many_sequences_as_a_contiguous_cache_has():
    """Accepted up to the next check: the workspace's, or without a device the device's."""
    assert lattn(lat=latent(page_size=0, block_table=None, capacity=64, num_blocks=2), B=2, ws=None) == 3
    assert lattn(lat=latent(page_size=0, block_table=None, capacity=64, num_blocks=0), B=0) == OK
    assert spire.load().spire_version() == 1
