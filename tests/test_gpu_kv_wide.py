"""Appending with the kernel that whole prompts and wide batches take: many tokens a CTA, scales written head by head."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2503_05330_b200 import binding  # noqa: E402
import model_ref as ref  # noqa: E402
from test_gpu_kv import DEV, TYPES, bits, cache, parts  # noqa: E402


def expected(c, new, lens, counts):
    """The cache's parts after the call."""
    out = [x.clone() for x in parts(c)]
    T, cap = new[0].shape[1], c.shape[1]
    for i in range(2):
        value, s = ref.quantised(new[i]) if c.k_scale is not None else (None, None)
        codes = value.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8) if value is not None else bits(new[i])
        for r in range(c.shape[0]):
            at = max(lens[r], 0)
            n = min(T if counts is None else min(max(counts[r], 0), T), max(cap - at, 0))
            out[i][r, at:at + n] = codes[r, :n]
            if s is not None:
                out[2 + i][r, :, at:at + n] = s[r, :n].T
    return out


# (rows, heads, head, tokens): at least 4.85 million of 16 bytes a side and call; heads that divide a CTA's vectors and those that do not
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,heads,d,T", [(44, 3, 128, 1300), (56, 5, 64, 1111), (20, 8, 128, 1001), (150, 7, 64, 290), (3, 1, 128, 60001)])
@pytest.mark.parametrize("heads_first,slack", [(False, 0), (True, 3)])
def test_append(dtype, rows, heads, d, T, heads_first, slack):
    assert T * heads * (d // 8) * rows * 2 >= 148 * 2048 * 16
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T)
    cap = T + 40
    c = cache(rows, cap, heads, d, dtype, heads_first, slack)
    new = []
    for _ in range(2):
        x = torch.randn((rows, T, heads, d), device=DEV, generator=gen)
        if dtype != torch.float16:
            x *= torch.exp2(torch.randint(-20, 20, (rows, T, heads, 1), device=DEV, generator=gen).float())
        x = x.to(c.new_dtype)
        x[1, 7, heads - 1, 3] = float("inf")
        new.append(x)
    # whole rows, none, one token, ends inside a CTA's part and next to its ends, more than there are; lengths that leave room for some, for one and for none
    per_cta = 4096 // (heads * (d // 8))
    some = [T, 0, 1, T - 1, per_cta, per_cta + 1, per_cta - 1, 2 * per_cta + 3, T // 2, T + 5, -3, T]
    places = [0, 40, 17, 41, 0, cap - 1, cap, cap + 9, -2, cap - per_cta - 2, 5, 33]
    counts, lens = [some[r % 12] for r in range(rows)], [places[(r * 5 + r // 12) % 12] for r in range(rows)]
    i32 = dict(device=DEV, dtype=torch.int32)
    want = expected(c, new, lens, counts)
    binding.sdms_kv_append(c, *new, torch.tensor(lens, **i32), torch.tensor(counts, **i32))
    for a, b in zip(parts(c), want):
        assert torch.equal(a, b)
    want = expected(c, new, lens, None)
    binding.sdms_kv_append(c, *new, torch.tensor(lens, **i32))
    for a, b in zip(parts(c), want):
        assert torch.equal(a, b)
