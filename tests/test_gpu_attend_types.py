"""Attention at the ends of what its types hold."""
import math

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


@pytest.mark.parametrize("T,group", [(1, 1), (1, 24), (5, 40)])
def test_many_small_weights_behind_a_large_one(T, group):
    """One key 18 ahead of 16000 others in fp16: each of those weighs 2^-26 of it, all of them together 2^-12."""
    P, n, d, lead = 148, 16000, 64, 18.0
    k = torch.zeros((P, n, 1, d), device=DEV, dtype=torch.float16)
    v = torch.ones_like(k)
    k[:, 0, 0, 0] = 12
    v[:, 0] = 0
    q = torch.zeros((P, T, group, d), device=DEV, dtype=torch.float16)
    q[..., 0] = lead / 12 * 8
    out = torch.empty_like(q)
    attention = binding.PathAttention(1, P, T, group, 1, d, torch.float16)
    mask = torch.zeros((P, T), device=DEV, dtype=torch.int64)      # the new tokens are not looked at
    attention(q, out, binding.KvCache(k, v), torch.full((P,), n - T, device=DEV, dtype=torch.int32), None, mask, scale=0.125)
    assert not attention.timed_out()
    small = math.exp(-lead) * (n - T - 1)
    expect = small / (1 + small)
    # a weight is rounded to 2^-25 of what a 16-bit number can be here, 2^6 times the largest weight; the output to half a step; exponents by 2^-21
    tol = (n - T - 1) * 2.0 ** -31 + expect * (2.0 ** -11 + 2.0 ** -20)
    assert bool(((out.double() - expect).abs() <= tol).all()), (float(out.min()), float(out.max()), expect, tol)
