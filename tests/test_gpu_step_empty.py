"""A step without a token, through the binding: every call takes the empty tensors that a program then has, and writes nothing."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.mark.parametrize("d", [128, 256])
def test_a_step_without_tokens(iq, d):
    B, H, hk, dev = 3, 8, 2, "cuda"
    shape, cb = iq.Shape(B, H, hk, d, 256), iq.iq_lloyd_max_codebook(d, 3)
    rot = torch.empty(iq.iq_rotation_floats(d, hk), dtype=torch.float32, device=dev)
    iq.iq_make_rotation(d, hk, 5, None, rot)
    cache = iq.new_cache(shape)
    for x in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
        x.fill_(3)
    before = [x.clone() for x in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales)]
    status = torch.zeros(4, dtype=torch.int32, device=dev)
    lens, n_new = torch.tensor([5, 0, 9], dtype=torch.int32, device=dev), torch.zeros(B, dtype=torch.int32, device=dev)
    start = torch.full((B + 1,), 7, dtype=torch.int32, device=dev)
    positions, sequences = (torch.empty(0, dtype=torch.int32, device=dev) for _ in range(2))
    slots = torch.empty(0, dtype=torch.int64, device=dev)
    q, k, v = torch.empty((0, H, d), dtype=torch.float16, device=dev), *(torch.empty((0, hk, d), dtype=torch.float16, device=dev) for _ in range(2))
    assert q.data_ptr() == 0
    ws = torch.empty(iq.iq_chunk_workspace_bytes(shape), dtype=torch.uint8, device=dev)
    iq.iq_plan_tokens(shape, lens, n_new, start, positions, sequences, slots, status_dev=status)
    assert start.tolist() == [0] * (B + 1)
    iq.iq_apply_rotary(shape, iq.iq_make_rotary(d), q, k, positions)
    iq.iq_apply_rotary(shape, iq.iq_make_rotary(d), q, None, positions, torch.empty_like(q))
    iq.iq_apply_rotary(shape, iq.iq_make_rotary(d), None, k[None], positions)
    iq.iq_quantize_append_packed(shape, rot, cb, k, v, lens, start, 4, cache, status)
    iq.iq_chunk_attention(shape, rot, cb, q, cache, lens, ws, torch.empty_like(q), token_start=start, status_dev=status)
    iq.iq_cross_attention(shape, rot, cb, q, cache, lens, ws, torch.empty_like(q), token_start=start, status_dev=status)
    padded = q.view(B, 0, H, d)
    iq.iq_chunk_attention(shape, rot, cb, padded, cache, lens, ws, torch.empty_like(padded), status_dev=status)
    assert status.tolist() == [0, 0, 0, 0]
    for x, y in zip(before, (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales)):
        assert torch.equal(x, y)
