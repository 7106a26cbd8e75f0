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


def up(n):
    return (n + 63) // 64 * 64


@pytest.mark.parametrize("shapes", [[(1, 1)], [(512, 4608)], [(4096, 1024)], [(4781, 188)], [(70, 6011)], [(1600, 6400)],
                                    [(512, 4608)] * 3 + [(2048, 512)], [(64, 100000)], [(17, 5000), (5, 0), (1100, 1100)],
                                    [(3, 5)] * 200])
def test_orthogonalize_workspace_is_what_the_header_says(shapes):
    """12 bytes an element and 12 for each of min(rows, cols)^2, sides as whole
    64s, 3 KB a matrix, and where a tile can be cut along an axis of 1024 or more at
    most 512 slots of 16 KB and their counters in all; no less than the factors alone."""
    size = B.bytecomp_orthogonalize_workspace_size(shapes)
    factors = sum(12 * up(r) * up(c) + 12 * up(min(r, c)) ** 2 for r, c in shapes if r and c)
    cut = any(max(r, c) >= 1024 for r, c in shapes if r and c)
    assert size <= factors + 3072 * len(shapes) + (512 * (16384 + 4) + 256 if cut else 0), (size, factors)
    assert size >= sum(12 * r * c + 12 * min(r, c) ** 2 for r, c in shapes)
