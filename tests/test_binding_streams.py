"""The stream a call is enqueued on belongs to the device of its tensors (without a GPU)."""
from types import SimpleNamespace

import pytest

import paper_2508_12851_amd as P
from paper_2508_12851_amd import binding as B


def test_a_stream_of_another_device_is_refused():
    assert B._stream_on(0, SimpleNamespace(device_index=0, cuda_stream=0x1000)) == 0x1000
    assert B._stream_on(1, SimpleNamespace(device_index=1, cuda_stream=0)) is None       # the default stream
    with pytest.raises(P.PrismError, match="device 1"):
        B._stream_on(0, SimpleNamespace(device_index=1, cuda_stream=0x1000))
