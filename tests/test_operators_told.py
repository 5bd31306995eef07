"""Tensors of a call are told that it writes them when it has been made, not when their places are read."""
import pytest


def test_places_are_read_first_and_writes_told_later():
    import torch
    from paper_2312_08728_amd import _tensors as T
    f = torch.float32
    m, v, y = torch.zeros(5, 7), torch.zeros(5), torch.zeros(5, 7)
    args = ((m, v, None, y), (f, f, f, f), ((5, 7), (5,), (5, 7), (5, 7)), b"mVMM", -1)
    assert T.operands(*args, False) == T.operands(*args, 0 == 1) and (m._version, v._version, y._version) == (0, 0, 0)
    assert T.told(args[0], args[3]) is None and (m._version, v._version, y._version) == (0, 1, 1)
    T.operands(*args, True)
    assert (m._version, v._version, y._version) == (0, 2, 2)
    with torch.inference_mode():
        kept = torch.zeros(3)
    T.told((kept,), b"V")                                            # (has no count)
    for bad in (lambda: T.told([m], b"M"), lambda: T.told((m,), b"MM"), lambda: T.told((m,)), lambda: T.told((m,), "M"), lambda: T.operands(*args, False, False)):
        with pytest.raises(TypeError):
            bad()
    assert (m._version, v._version, y._version) == (0, 2, 2)
