"""What the Python binding makes of its arguments before the library sees them: addresses, strides of parts of larger
tensors.  No GPU: a recorder stands in for the library."""
import enum

import pytest
import torch


@pytest.fixture(scope="module")
def oc():
    from paper_2607_23844_b200 import build
    build.build()
    from paper_2607_23844_b200 import omnicache
    return omnicache


@pytest.fixture
def calls(oc, monkeypatch):
    """(a context, the arguments of every call that it made)"""
    made = []

    class Recorder:
        def __getattr__(self, name):
            def call(*args):
                made.append((name, args))
                return oc.OK
            return call
    monkeypatch.setattr(oc, "_lib", Recorder())
    ctx = object.__new__(oc.Context)
    ctx._h = None
    return ctx, made


class Address(enum.IntEnum):
    BUFFER = 0x7000


def test_addresses_may_be_any_int(oc):
    for p in (oc._ptr, oc._ptr_strided):
        assert p(None) is None and p(64) == 64 and p(Address.BUFFER) == 0x7000
    t = torch.zeros(4, 6)
    assert oc._ptr(t) == t.data_ptr()
    with pytest.raises(AssertionError):
        oc._ptr(t[:, :3])
