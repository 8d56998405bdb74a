"""The workspace of iq_tree_attention is checked against the size for the device of the call. Nothing is launched: every call that passes
the check is refused for its window."""
import types

import pytest
import torch


@pytest.fixture
def binding():
    from paper_2608_08081_b200 import binding as m
    return m


def test_the_size_is_that_of_the_current_device(binding, monkeypatch):
    """Two devices of different sizes, the smaller one first: a workspace that is large enough there is not on the other."""
    need, device = {0: 1000, 1: 3000}, [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device[0])
    monkeypatch.setattr(binding, "iq_tree_workspace_bytes", lambda shape, T: need[device[0]])
    shape = binding.Shape(1, 2, 1, 128, 128)
    cb = binding.iq_lloyd_max_codebook(128, 3, "int8")
    cache = binding.Cache(torch.zeros((1, 1, 128, 48), dtype=torch.uint8), torch.zeros((1, 1, 128)), torch.zeros((1, 1, 128, 48), dtype=torch.uint8),
                          torch.zeros((1, 1, 128)))
    rot, ctx = torch.zeros(256), torch.zeros(1, dtype=torch.int32)
    stream = types.SimpleNamespace(cuda_stream=0)

    def call(nbytes, T):
        q = torch.zeros((1, T, 2, 128), dtype=torch.float16)
        binding.iq_tree_attention(shape, rot, cb, q, cache, ctx, None, None, torch.zeros(nbytes, dtype=torch.uint8), torch.zeros_like(q), window=-1,
                                  stream=stream)

    def passes(nbytes, T):
        with pytest.raises(binding.IQError) as e:
            call(nbytes, T)
        assert e.value.code == -2

    def refused(nbytes, T):
        with pytest.raises(AssertionError):
            call(nbytes, T)

    passes(1000, 4)
    refused(999, 4)
    device[0] = 1
    refused(1000, 4)
    refused(2999, 4)
    passes(3000, 4)
    device[0] = 0
    passes(1000, 4)
    need[0] = 2000
    passes(2000, 5)
    refused(1999, 5)
