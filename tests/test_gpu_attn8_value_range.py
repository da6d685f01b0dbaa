"""Attention over a cache in 8 bits where one value row is far larger than all others, in one element: the other elements are made
of the other rows alone, whatever the number of queries, and are held to the bounds of attn_bounds.py like all."""
import pytest

from attn_bounds import check, head

pytestmark = pytest.mark.gpu


def modules():
    import torch
    from paper_2603_17051_b200 import binding as A
    return torch, A


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [1, 3, 8, 9, 16, 40])
@pytest.mark.parametrize("held", [32, 47, 3000])
@pytest.mark.parametrize("power", [16, 22, 26, 34, 60, 100])
def test_one_row_far_larger_in_one_element(D, n_q, held, power):
    torch, A = modules()
    H = 2
    g = torch.Generator(device="cuda").manual_seed(power + held)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    cache = A.astro_kvcache8_create(1, H, D, 1, 0, held)
    k, v = make(1, held, H, D), make(1, held, H, D)
    for at, element in ((5, 3), (held - 2, D - 1)):              # among a warp's first keys, among another's last
        v[0, at] = 0.0
        v[0, at, :, element] = 2.0 ** power
    A.astro_kvcache8_append(cache, k, v, held)
    k8, v8 = (x.double() for x in A.astro_kvcache8_read(cache, dtype=torch.float32))
    q, kc, vc = make(1, n_q, H, D), make(1, 3, H, D), make(1, 3, H, D)
    for own in (False, True):                                     # with the chunk's keys, whose values are ordinary, and without
        o, lse = A.astro_chunk_attn8_fwd(cache, q, kc if own else None, vc if own else None, D ** -0.5)
        A.astro_last_device_status()
        for h in range(H):
            kk, vv = (torch.cat([x[0, :, h]] + ([y[0, :, h].double()] if own else [])) for x, y in ((k8, kc), (v8, vc)))
            want = head(q[0, :, h].double(), kk, vv, D ** -0.5)
            check(o[0, :, h], want["o"], "O")
            check(lse[0, h], want["lse"], "LSE")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [1, 12])
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
def test_rows_of_sizes_90_powers_of_two_apart(D, n_q, order):
    """Every key fills one element; the elements' sizes go up along the keys, down, or stand side by side within every step."""
    torch, A = modules()
    n = 4000
    g = torch.Generator(device="cuda").manual_seed(n_q)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    k, q = make(1, n, 1, D), make(1, n_q, 1, D)
    i = torch.arange(n, device="cuda")
    e = {"up": i * D // n, "down": (n - 1 - i) * D // n, "mixed": i * 37 % D}[order]
    v = torch.zeros(n, D, device="cuda")
    v[i, e] = torch.exp2((90 * e // D - 45).float()) * (1 + torch.rand(n, generator=g, device="cuda"))
    cache = A.astro_kvcache8_create(1, 1, D, 1, 0, n)
    A.astro_kvcache8_append(cache, k, v.bfloat16().view(1, n, 1, D), n)
    k8, v8 = (x.double() for x in A.astro_kvcache8_read(cache, dtype=torch.float32))
    o, lse = A.astro_chunk_attn8_fwd(cache, q, None, None, D ** -0.5)
    A.astro_last_device_status()
    want = head(q[0, :, 0].double(), k8[0, :, 0], v8[0, :, 0], D ** -0.5)
    value, bound = want["o"]
    check(o[0, :, 0], (value, bound - 1e-7), "O")                 # small elements too are held to their own size
    check(lse[0, 0], want["lse"], "LSE")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [1, 12])
@pytest.mark.parametrize("power", [-118, -100, 115])
def test_values_that_are_all_tiny_or_all_huge(D, n_q, power):
    torch, A = modules()
    n = 700
    g = torch.Generator(device="cuda").manual_seed(n_q)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    q, k, v = make(1, n_q, 1, D), make(1, n, 1, D), make(1, n, 1, D) * 2.0 ** power
    cache = A.astro_kvcache8_create(1, 1, D, 1, 0, n)
    A.astro_kvcache8_append(cache, k, v, n)
    k8, v8 = (x.double() for x in A.astro_kvcache8_read(cache, dtype=torch.float32))
    o, lse = A.astro_chunk_attn8_fwd(cache, q, None, None, D ** -0.5)
    A.astro_last_device_status()
    # in units of 2^power, where the bound's 1e-7 can be taken from it again (1e-7 + 1e-35 is 1e-7 in 64 bits); bf16 has steps of 2^-133
    value, bound = head(q[0, :, 0].double(), k8[0, :, 0], v8[0, :, 0] * 2.0 ** -power, D ** -0.5)["o"]
    check(o[0, :, 0].double() * 2.0 ** -power, (value, bound - 1e-7 + 2.0 ** (-133 - power)), "O")
