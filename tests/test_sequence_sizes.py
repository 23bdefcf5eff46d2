"""Workspace sizes are kept by device: the norm's gradients take as many parts of dweight
as the current one has room for."""
import ctypes

from paper_1905_05233_amd import _native as N
from paper_1905_05233_amd import sequence_ops as S


def test_sizes_are_asked_for_on_each_device(monkeypatch):
    asked = []

    class Lib:
        def query(self, *args):
            asked.append(args[:-1])
            ctypes.cast(args[-1], ctypes.POINTER(ctypes.c_size_t))[0] = 100 * len(asked)
            return N.WG_OK

    monkeypatch.setattr(S, "_sizes", {})
    monkeypatch.setattr(N, "lib", Lib)
    assert [S._size("query", dev, 5, 7) for dev in (0, 1, 0, 1)] == [100, 200, 100, 200]
    assert S._size("query", 1, 5, 8) == 300
    assert asked == [(5, 7), (5, 7), (5, 8)]
