"""The layers' binding refuses tensors that are not on the calls' device, the
workspace among them, before the library sees a pointer (CPU only: tensors
of the meta device and the host stand in for two devices)."""
import pytest

from paper_2205_14465_amd import binding as B


def test_workspace():
    import torch
    with pytest.raises(ValueError):
        B._ws(torch.empty(64, dtype=torch.uint8))  # host memory
    with pytest.raises(ValueError):
        B._ws(torch.empty(64, 2, dtype=torch.uint8, device="meta")[:, 0])  # its bytes do not follow each other
    assert B._ws(None) == (None, 0)


def test_one_device():
    import torch
    a, b = torch.empty(3, device="meta"), torch.empty(3)
    with pytest.raises(ValueError):
        B._Call("bytecomp_layernorm_forward", (), (a, None, b))
    with pytest.raises(ValueError):
        B._Call("bytecomp_orthogonalize", (), ([a, a], [a, b], None))
    B._Call("bytecomp_orthogonalize", (), ([a, a], [a, a], None))
