"""Attention where its warps, tiles and types come to their ends."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2503_05330_b200 import binding  # noqa: E402,F401
import model_ref as ref  # noqa: E402,F401
from test_gpu_attend import DEV, KINDS, check, make_cache  # noqa: E402,F401


@pytest.mark.parametrize("kind,q_type", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,T,group,keys", [(5, 13, 2, 500), (7, 5, 4, 2000), (10, 16, 1, 129), (23, 7, 1, 128), (3, 64, 1, 300), (193, 1, 1, 40000), (7, 32, 1, 700)])
def test_rows_that_leave_warps_of_the_second_half_without_one(kind, q_type, d, N, T, group, keys):
    """129 to 224 rows: of the second 128 some warps' 32 have nobody, and those warps run ahead of the others.  The same bits every time."""
    att, args = check(1, N, T, group, 1, d, kind, q_type, 0, None, prefix_cap=keys + 3, prefix_lens=[keys], seed=N + T)
    first = args[1].clone()
    for _ in range(100):
        args[1].fill_(7.0)
        att(*args)
        assert torch.equal(args[1], first)
    assert not att.timed_out()


@pytest.mark.parametrize("kind,q_type", KINDS)
def test_own_rows_that_leave_warps_without_one(kind, q_type):
    att, args = check(1, 6, 33, 4, 1, 128, kind, q_type, 300, [0, 90, 128, 200, 267, 100], seed=70)          # 132 rows a path
    first = args[1].clone()
    for _ in range(100):
        args[1].fill_(7.0)
        att(*args)
        assert torch.equal(args[1], first)


def spoiled_attention(d, T, lens, prefix_len, spoil, mask=None, seed=90):
    """8-bit caches that `spoil` has been at: (output, expected, tolerance)."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    P, group, heads = len(lens), 2, 2
    paths = make_cache(P, 300, heads, d, torch.float8_e4m3fn, gen)
    prefix = make_cache(1, 200, heads, d, torch.float8_e4m3fn, gen)
    spoil(paths, prefix)
    q = torch.randn((P, T, heads * group, d), device=DEV, generator=gen).to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    i32 = dict(device=DEV, dtype=torch.int32)
    attention = binding.PathAttention(1, P, T, heads * group, heads, d, torch.bfloat16)
    attention(q, out, paths, torch.tensor(lens, **i32), None, mask, prefix, torch.tensor([prefix_len], **i32))
    assert not attention.timed_out()
    expect, tol = ref.attend(q, ref.cache_values(paths.k, paths.k_scale), ref.cache_values(paths.v, paths.v_scale), lens, None, d ** -0.5,
                             ref.cache_values(prefix.k, prefix.k_scale), ref.cache_values(prefix.v, prefix.v_scale), [prefix_len], mask)
    return out, expect, tol


@pytest.mark.parametrize("scale", [0, 120, 134, 135, 254])
@pytest.mark.parametrize("code", [0x7f, 0xff])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", ["k", "v", "k_prefix", "v_prefix"])
def test_codes_that_are_not_numbers(where, d, code, scale):
    """float8_e4m3fn's own NaN, under whatever scale: in K no query that sees the key has an answer, in V one element has none."""
    token, head, element = 77, 1, d - 3

    def spoil(paths, prefix):
        c, row = (prefix, 0) if "prefix" in where else (paths, 1)
        x, s = (c.k, c.k_scale) if where[0] == "k" else (c.v, c.v_scale)
        x.view(torch.uint8)[row, token, head, element] = code
        if scale == 254:                                     # (the other elements of such a vector are zero: they are numbers that no sum holds)
            x.view(torch.uint8)[row, token, head, :element] = 0
            x.view(torch.uint8)[row, token, head, element + 1:] = 0
        s[row, head, token] = scale
    out, expect, tol = spoiled_attention(d, 1, [100, 130, 140], 199, spoil)
    want = torch.isnan(expect)
    rows = [0, 1, 2] if "prefix" in where else [1]
    assert bool(want[rows, :, 2:, element].all()) and int(want.sum()) == len(rows) * 2 * (d if where[0] == "k" else 1)
    assert torch.equal(torch.isnan(out), want)
    assert bool(((out.double() - expect).abs() <= tol)[~want].all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,tree", [(2, False), (9, False), (9, True), (64, False)])
@pytest.mark.parametrize("where", ["k", "v"])
def test_codes_that_are_not_numbers_in_new_tokens(where, T, tree, d):
    """What a query does not see does it no harm; for those that see it nothing is left."""
    lens = [0, 127, 128 - T // 2]
    mask = None
    if tree:
        mask = torch.tensor([[1 << t | (t % 2) for t in range(T)]] * 3, device=DEV)

    def spoil(paths, prefix):
        c = paths.k if where == "k" else paths.v
        for p, at in enumerate(lens):
            for u, code in ((T - 1, 0x7f), (T // 2, 0xff)):
                c.view(torch.uint8)[p, at + u, u % 2, (u * 11 + 5) % d] = code
    out, expect, tol = spoiled_attention(d, T, lens, 150, spoil, mask)
    reached = torch.isnan(expect).any(-1)
    assert reached.any() and not reached.all()
    assert bool(torch.isnan(out[reached]).all())
    assert bool(((out.double() - expect).abs() <= tol)[~reached].all())


def test_codes_that_are_not_numbers_behind_the_last_key():
    def spoil(paths, prefix):
        for p, n in enumerate((4, 133, 260)):
            for x in (paths.k, paths.v):
                x.view(torch.uint8)[p, n:] = 0x7f
        for x in (prefix.k, prefix.v):
            x.view(torch.uint8)[:, 100:] = 0xff
    out, expect, tol = spoiled_attention(128, 3, [1, 130, 257], 100, spoil)
    assert bool(torch.isfinite(expect).all()) and bool(((out.double() - expect).abs() <= tol).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [121, 140])
def test_codes_that_are_not_numbers_wherever_a_tile_has_them(d, scale):
    """A path for every token of a tile, its code at another element each time: all tokens, elements and places of a word come up."""
    P = 2 * 128
    gen = torch.Generator(device=DEV)
    gen.manual_seed(d + scale)
    paths = make_cache(P, 256, 1, d, torch.float8_e4m3fn, gen)
    p = torch.arange(P, device=DEV)
    token, element = p % 128 + 128 * (p % 2), (p * 5 + p // 128 * 3) % d
    assert len(set((token % 128).tolist())) == 128 and len(set(element.tolist())) == d
    paths.v.view(torch.uint8)[p, token, 0, element] = torch.where(p % 3 == 0, 0xff, 0x7f).to(torch.uint8)
    paths.v_scale[p, 0, token] = scale
    q = torch.randn((P, 1, 2, d), device=DEV, generator=gen).to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    lens = torch.full((P,), 255, device=DEV, dtype=torch.int32)
    binding.PathAttention(1, P, 1, 2, 1, d, torch.bfloat16)(q, out, paths, lens)
    expect, tol = ref.attend(q, ref.cache_values(paths.k, paths.k_scale), ref.cache_values(paths.v, paths.v_scale), [255] * P, None, d ** -0.5)
    want = torch.isnan(expect)
    assert int(want.sum()) == 2 * P
    assert torch.equal(torch.isnan(out), want)
    assert bool(((out.double() - expect).abs() <= tol)[~want].all())
