"""What a forked cache says it has seen."""
import pytest

from test_gpu_block_select import ring

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("frames,seen", [(None, 3), ([2], 3), ([0, 1, 2, 0, 1], 5), ([1, 1, 1, 1], 4), ([0, 2, 1], 3)])
def test_frames_seen_of_a_fork_covers_repeats(frames, seen):
    """The source's count, or the number of frames held where that is larger: a saved record must always be restorable."""
    from paper_2603_17051_b200 import binding as A
    src, _, _, held = ring(A, 1, 2, 64, 20, 1, 5, 0, 3, 9)
    assert held == 3 and A.astro_kvcache_query(src)[2] == 3
    dst = A.astro_kvcache_create(2, 2, 64, 20, 1, 5)
    A.astro_kvcache_fork(dst, src, frames=frames)
    sink, win, got = A.astro_kvcache_query(dst)
    assert got == seen and sink + win == (3 if frames is None else len(frames))
    A.astro_kvcache_set_state(dst, A.astro_kvcache_get_state(dst))
