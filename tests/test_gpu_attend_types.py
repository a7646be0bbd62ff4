"""Attention at the ends of what its types hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2503_05330_b200 import binding  # noqa: E402
import model_ref as ref  # noqa: E402
from test_gpu_attend import DEV, make_cache  # noqa: E402

MOST = torch.finfo(torch.bfloat16).max


def clamped(x, scale):
    """What 8-bit caches hold, as bfloat16 takes it: nothing is larger than its largest number."""
    return ref.cache_values(x, scale).clamp(-MOST, MOST)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 5])
def test_largest_numbers_in_a_refused_draft(T, d, sign):
    """The largest bfloat16 is stored as 256 * 2^120, which bfloat16 does not hold: it stays a number, and reaches only the queries that see it."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T + d)
    P, heads, group, lens = 3, 2, 2, [0, 126, 150]
    paths = make_cache(P, 200, heads, d, torch.float8_e4m3fn, gen)
    i32 = dict(device=DEV, dtype=torch.int32)
    new = [torch.randn((P, T, heads, d), device=DEV, generator=gen).to(torch.bfloat16) for _ in range(2)]
    new[1][:, T - 1, 1, 7] = sign * MOST
    binding.sdms_kv_append(paths, *new, torch.tensor(lens, **i32))
    for p, at in enumerate(lens):
        assert int(paths.v_scale[p, 1, at + T - 1]) == 247
    q = torch.randn((P, T, heads * group, d), device=DEV, generator=gen).to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    attention = binding.PathAttention(1, P, T, heads * group, heads, d, torch.bfloat16)
    attention(q, out, paths, torch.tensor(lens, **i32))
    assert not attention.timed_out()
    expect, tol = ref.attend(q, clamped(paths.k, paths.k_scale), clamped(paths.v, paths.v_scale), lens, None, d ** -0.5)
    assert bool(torch.isfinite(out).all()) and bool(((out.double() - expect).abs() <= tol).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("code,scale", [(0x78, 247), (0xf8, 247), (0x7e, 247), (0xfe, 248), (0x7e, 254), (0x01, 254), (0x77, 247)])
def test_values_beyond_bfloat16_count_as_its_largest(code, scale, d):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(code + scale)
    paths = make_cache(2, 150, 1, d, torch.float8_e4m3fn, gen)
    for x, s in ((paths.k, paths.k_scale), (paths.v, paths.v_scale)):
        x.view(torch.uint8)[1, 40, 0] = 0
        x.view(torch.uint8)[1, 40, 0, 3] = code
        s[1, 0, 40] = scale
    q = torch.randn((2, 1, 2, d), device=DEV, generator=gen).to(torch.bfloat16)
    q[..., 3] = 2.0 ** -122                                  # at most 2^6 times the element that is so large
    out = torch.full_like(q, 7.0)
    binding.PathAttention(1, 2, 1, 2, 1, d, torch.bfloat16)(q, out, paths, torch.tensor([100, 100], device=DEV, dtype=torch.int32))
    expect, tol = ref.attend(q, clamped(paths.k, paths.k_scale), clamped(paths.v, paths.v_scale), [100, 100], None, d ** -0.5)
    assert bool(torch.isfinite(out).all()) and bool(((out.double() - expect).abs() <= tol).all())
