"""A device-side wait that runs out for some lanes of a warp and completes for the others: the warp must leave together."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_warp_gets_one_answer_from_a_wait():
    import torch
    from paper_2603_17051_b200 import binding as A
    assert A.astro_last_device_status() == 0
    A.astro_selftest_wait_timeout()                           # one lane on a barrier nothing completes, the others on a complete one
    with pytest.raises(A.AstroError) as e:
        A.astro_last_device_status()
    assert e.value.status == 8 and "detail 0x1)" in str(e.value)   # bit 1 would say that lanes went on by themselves
    torch.cuda.synchronize()
    assert A.astro_last_device_status() == 0
