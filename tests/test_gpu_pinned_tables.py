"""A pinned table outlives the calls that read it."""
import pytest
import torch

from paper_2410_22697_amd import RowFormat, block_mean, pack_rows, unpack_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("read", ["unpack", "mean"])
def test_a_pinned_table_dropped_after_the_call(read):
    """Its memory is not handed out again before the stream has read it."""
    fmt = RowFormat(64, 8)
    n = 4096
    packed = pack_rows(torch.randn(n, 64, device="cuda"), fmt)
    indptr, indices = torch.arange(n + 1, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda").flip(0).contiguous()

    def call(table):
        return unpack_rows(table, fmt) if read == "unpack" else block_mean(table, indptr, indices, fmt=fmt)
    want = call(packed)
    pinned = torch.empty(packed.shape, dtype=torch.uint8, pin_memory=True)
    pinned.copy_(packed)
    torch.cuda.synchronize()
    at = pinned.data_ptr()
    torch.cuda._sleep(200_000_000)  # the call's work waits behind this
    got = call(pinned)
    del pinned
    again = torch.empty(packed.shape, dtype=torch.uint8, pin_memory=True)
    assert again.data_ptr() != at
    again.fill_(0)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
