"""Which memory the operators may be given, as far as the host decides it: strides that overlap, memory that outputs share, sizes beyond 32 bits.  No call
here reaches a launch."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2501_19324_amd import binding, ops
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return ops._load()


@pytest.fixture
def on_host(lib, monkeypatch):
    """The binding on tensors in host memory: for calls that are refused."""
    from paper_2501_19324_amd import ops
    monkeypatch.setattr(ops, "_stream", lambda t: 0)
    return ops


def refused(call, ops):
    with pytest.raises(ops._b.RsdError) as e:
        call()
    return e.value.code == ops._b.RSD_EINVAL


@pytest.mark.parametrize("shape,strides", [((48, 64), (0, 1)), ((48, 64), (1, 1)), ((2, 64), (63, 1)), ((5, 1), (0, 1))], ids=str)
def test_weights_whose_rows_overlap_are_refused(on_host, shape, strides):
    """A row stride below the row's length was once taken for that length: a read behind the tensor's memory."""
    import torch
    w = torch.zeros(4096).as_strided(shape, strides)
    assert refused(lambda: on_host.rsd_w4_pack(w), on_host)
