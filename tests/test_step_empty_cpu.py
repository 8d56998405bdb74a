"""Steps without a token: every call of a step takes the empty tensors that a program then has (whose address is 0) and launches nothing."""
import torch


def test_rotary_without_tokens():
    import paper_2608_08081_b200 as iq
    from paper_2608_08081_b200 import binding as lib

    shape, rot = iq.Shape(1, 4, 2, 128, 128), iq.iq_make_rotary(128)
    q, k, pos = torch.empty((0, 4, 128), dtype=torch.float16), torch.empty((0, 2, 128), dtype=torch.float16), torch.empty(0, dtype=torch.int32)
    assert q.data_ptr() == 0
    import ctypes

    def call(q, k, n):
        return lib._lib.iq_apply_rotary(ctypes.byref(shape.c()), ctypes.byref(rot.c()), q, 512, 128, q, 512, 128, k, 256, 128, k, 256, 128, None, n, None)

    assert call(q.data_ptr(), k.data_ptr(), 0) == 0 and call(None, None, 0) == 0
    assert call(None, None, 1) == -1 and call(None, None, -1) == -2
    assert lib._lib.iq_apply_rotary(ctypes.byref(shape.c()), None, None, 0, 0, None, 0, 0, None, 0, 0, None, 0, 0, None, 0, None) == -1
