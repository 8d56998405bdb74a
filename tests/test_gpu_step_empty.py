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


def test_rotary_of_padded_tokens_without_places(iq):
    """[B][0] in one piece and as a view of wider rows."""
    shape, rot = iq.Shape(1, 2, 1, 128, 128), iq.iq_make_rotary(128)
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    iq.iq_apply_rotary(shape, rot, torch.empty((4, 0, 2, 128), dtype=torch.float16, device="cuda"), None, pos)
    iq.iq_apply_rotary(shape, rot, torch.empty((4, 9, 2, 128), dtype=torch.float16, device="cuda")[:, :0], None, pos)


@pytest.mark.parametrize("T", [1, 4])
@pytest.mark.parametrize("d", [128, 256])
def test_rotary_of_views(iq, T, d):
    """[B][T] tokens evenly spaced in a larger tensor: the last token of every sequence, one head of many, in place and into another."""
    B, H, hk = 5, 4, 2
    shape, rot = iq.Shape(1, H, hk, d, 128), iq.iq_make_rotary(d)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    wide_q = torch.randn((B, 7, H, d), generator=gen, device="cuda").half()
    pos = torch.arange(100, 100 + B * T, dtype=torch.int32, device="cuda")
    q = wide_q[:, -1:] if T == 1 else wide_q.flatten(0, 1)[:B * T].unflatten(0, (B, T))
    want = q.clone(memory_format=torch.contiguous_format)
    iq.iq_apply_rotary(shape, rot, want, None, pos)
    out = torch.zeros_like(want)
    iq.iq_apply_rotary(shape, rot, q, None, pos, out)
    assert torch.equal(out, want)
    before = wide_q.clone()
    iq.iq_apply_rotary(shape, rot, q, None, pos)
    assert torch.equal(q, want)
    changed = (wide_q != before).flatten(2).any(-1)
    assert int(changed.sum()) == B * T
    # one head: its stride, and that of a single token, may be no multiple of 8
    one = iq.Shape(1, 1, 1, d, 128)
    x = torch.randn((3, 1, d), generator=gen, device="cuda").half()
    odd = torch.as_strided(x, (3, 1, d), (d, 5, 1))
    y = torch.zeros_like(x)
    iq.iq_apply_rotary(one, rot, odd, None, pos[:3].contiguous(), y)
    iq.iq_apply_rotary(one, rot, x, None, pos[:3].contiguous())
    assert torch.equal(x, y)
    single = torch.as_strided(x[:1].clone(), (1, 1, d), (3, 5, 1))
    z = torch.zeros((1, 1, d), dtype=torch.float16, device="cuda")
    iq.iq_apply_rotary(one, rot, single, None, pos[:1].contiguous(), z)


def test_views_that_are_not_evenly_spaced_are_refused(iq):
    shape, rot = iq.Shape(1, 2, 1, 128, 128), iq.iq_make_rotary(128)
    wide = torch.zeros((3, 5, 2, 128), dtype=torch.float16, device="cuda")
    with pytest.raises(AssertionError):
        iq.iq_apply_rotary(shape, rot, wide[:, :2], None, torch.zeros(6, dtype=torch.int32, device="cuda"))
