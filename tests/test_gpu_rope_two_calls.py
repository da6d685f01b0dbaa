"""Rotary positions of q and k whose strides differ take two launches: neither happens if one is refused, and neither reads what the
other has written."""
import pytest

pytestmark = pytest.mark.gpu


def test_nothing_is_rotated_when_the_second_tensor_is_refused():
    import torch
    from paper_2603_17051_b200 import binding as A
    rope = A.astro_rope_create(64, 64, "halves", (32,))
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    q = normal(2, 9, 4, 64)
    pos = torch.arange(5, 14, dtype=torch.int32, device="cuda").view(1, 9, 1)
    before = q.clone()
    off = normal(2 * 9 * 2 * 64 + 4)[4:].view(2, 9, 2, 64)                     # keys that start 8 bytes off
    uneven = normal(2, 9, 2, 68)[..., :64]                                     # rows 136 bytes apart
    shared = torch.empty(2, 9, 1, 64, dtype=torch.bfloat16, device="cuda").expand(2, 9, 2, 64)   # heads on top of each other
    k = normal(2, 9, 2, 64)
    for keys, kw, status in ((off, dict(k_out=k), 3), (off, dict(k_out=off), 3), (uneven, dict(k_out=k), 3), (k, dict(k_out=shared), 2),
                             (k, dict(k_out=uneven), 3)):
        with pytest.raises(A.AstroError) as e:
            A.astro_rope_apply(rope, q, keys, pos, q_out=q, **kw)
        assert e.value.status == status
    torch.cuda.synchronize()
    assert torch.equal(q, before)
    qo, ko = A.astro_rope_apply(rope, q, k, pos)
    A.astro_rope_apply(rope, q, k, pos, q_out=q, k_out=k)                       # both in place, two launches
    assert torch.equal(q, qo) and torch.equal(k, ko)


def test_an_output_on_top_of_the_other_input_is_refused():
    import torch
    from paper_2603_17051_b200 import binding as A
    rope = A.astro_rope_create(64, 64, "halves", (32,))
    room = torch.randn(2, 9, 4, 64, device="cuda").bfloat16()
    q, k = torch.randn(2, 9, 4, 64, device="cuda").bfloat16(), room[:, :, :2]
    pos = torch.arange(9, dtype=torch.int32, device="cuda").view(1, 9, 1)
    for kw in (dict(q_out=room), dict(q_out=room, k_out=room[:, :, :2]), dict(k_out=q[:, :, :2])):
        with pytest.raises(A.AstroError) as e:
            A.astro_rope_apply(rope, q, k, pos, **kw)
        assert e.value.status == 2
