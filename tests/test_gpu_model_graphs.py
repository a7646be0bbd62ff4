"""The operators of the model's side captured into graphs, and tensors that they refuse."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from harness import t32  # noqa: E402
from paper_2503_05330_b200 import binding, synth  # noqa: E402

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_selection_whose_chunks_know_of_one_another(dtype):
    """2560 chunks: a word a row is cleared in front of the launches, in the graph as well, whatever an earlier call left in it."""
    G, N, V = 32, 16, 40003
    P = G * N
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    logits = (torch.randn((P, V), device=DEV, generator=gen) * 3).to(dtype)
    scores = torch.randn((P,), device=DEV, generator=gen) - 5
    select, other = binding.BeamSelect(G, N, V, dtype), binding.BeamSelect(G, N, V, dtype)
    outs = [[torch.empty(P, device=DEV, dtype=t) for t in (torch.int32, torch.int32, torch.float32)] for _ in range(2)]
    select(logits, scores, *outs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        select(logits, scores, *outs[0])
    for turn in range(4):
        # every turn lower than the one before: what that one left would hide all of this one's
        logits.copy_((torch.randn((P, V), device=DEV, generator=gen) * 3 - 40 * turn).to(dtype))
        for x in outs[0]:
            x.fill_(-9)
        graph.replay()
        other(logits, scores, *outs[1])
        for a, b in zip(*outs):
            assert torch.equal(a, b), turn
    assert int(outs[0][0].min()) >= 0


@pytest.mark.parametrize("G,N,L,kw", [(1, 16, 1024, {}), (2, 64, 2048, {}), (3, 5, 77, dict(epsilon=1))])
def test_histories_and_index(G, N, L, kw):
    """sdms_reorder replayed with other parents each time, next to a context that is called."""
    P, V, D, k_max = G * N, 50, 4, 3
    tokens, lps = synth.small_random(P, L, V, 900 + L)
    n = (L // 3 + (np.arange(P) * 7) % (L // 4)).astype(np.int32)
    w = int(n.max())
    a, b = (binding.Sdms(G, N, L, V, k_max, D, **kw) for _ in range(2))
    for x in (a, b):
        x.append(t32(np.ascontiguousarray(tokens[:, :w], np.int32), DEV), torch.from_numpy(np.ascontiguousarray(lps[:, :w], np.float32)).to(DEV), t32(n, DEV))
    parents = torch.arange(P, device=DEV, dtype=torch.int32)
    a.reorder(parents)                                       # (nobody moves; the kernels are loaded)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.reorder(parents)
    rng = np.random.default_rng(3)
    for turn in range(3):
        want = np.arange(P)
        for g in range(G):
            order = rng.permutation(N)
            want[g * N + order[:N // 2]] = g * N + rng.choice(order[N // 2:], N // 2)
        parents.copy_(t32(want.astype(np.int32), DEV))
        graph.replay()
        b.reorder(parents)
        for x, y in zip(a.history(), b.history()):
            if x.ndim == 1:
                lens = x
                assert np.array_equal(x, y)
        for x, y in zip(a.history()[:2], b.history()[:2]):
            for p in range(P):
                assert np.array_equal(x[p, :lens[p]], y[p, :lens[p]])
        for k in range(1, k_max + 1):
            if kw and k == 1:
                continue
            for x, y in zip(a.build_drafts(k), b.build_drafts(k)):
                assert torch.equal(x, y)
    assert a.status() == 0 and b.status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("rows,T", [(8, 5), (44, 1300)])
def test_caches(dtype, rows, T):
    """Append and reorder replayed: lengths, counts and parents are read when the graph runs."""
    heads, d, cap = 3, 128, T + 60
    gen = torch.Generator(device=DEV)
    gen.manual_seed(rows)
    a, b = (binding.KvCache.empty(rows, cap, heads, d, dtype) for _ in range(2))
    held = [x for c in (a, b) for x in (c.k, c.v, c.k_scale, c.v_scale) if x is not None]
    for x in held:
        x.view(torch.uint8).fill_(0x31)
    new = [torch.empty((rows, T, heads, d), device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    lens, counts, parents = (torch.zeros(rows, device=DEV, dtype=torch.int32) for _ in range(3))

    def step(c):
        binding.sdms_kv_append(c, *new, lens, counts)
        binding.sdms_kv_reorder(c, parents, lens, rows // 4)
    step(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for turn in range(3):
        for x in new:
            x.normal_(generator=gen)
        lens.random_(0, cap, generator=gen)
        counts.random_(-1, T + 2, generator=gen)
        at = torch.arange(rows, device=DEV, dtype=torch.int32)
        parents.copy_(torch.where(at % (rows // 4) > turn, at - at % (rows // 4), at))
        graph.replay()
        step(b)
        half = len(held) // 2
        for x, y in zip(held[:half], held[half:]):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), turn


def test_caches_that_are_refused():
    def t(shape, dtype=torch.bfloat16, device=DEV):
        return torch.zeros(shape, device=device, dtype=dtype)
    shape = (2, 10, 3, 64)
    k, v, code, scale = t(shape), t(shape), t(shape, torch.float8_e4m3fn), t((2, 3, 10), torch.uint8)
    assert binding.KvCache(k, v).shape == shape and binding.KvCache(code, code.clone(), scale, scale.clone()).new_dtype == torch.bfloat16
    for args in [
        (k, v[:1]), (k, v.half()), (k, v.cpu()), (t(shape, torch.float64), t(shape, torch.float64)), (k[0], v[0]),
        (k, t((2, 3, 10, 64)).permute(0, 2, 1, 3)),                                 # K and V laid out differently
        (t((2, 10, 3, 128))[..., ::2], t((2, 10, 3, 128))[..., ::2]),               # gaps inside a head
        (k, v, scale, scale), (code, code), (code, code, scale, None), (code, code, None, scale),
        (code, code, scale[:, :, :9], scale[:, :, :9]), (code, code, scale.int(), scale.int()), (code, code, scale.cpu(), scale.cpu()),
        (code, code, t((2, 10, 3), torch.uint8).permute(0, 2, 1), t((2, 10, 3), torch.uint8).permute(0, 2, 1)),
    ]:
        with pytest.raises(ValueError):
            binding.KvCache(*args)
    lens, new = t((2,), torch.int32), t((2, 1, 3, 64))
    for cache in (binding.KvCache(t(shape, torch.float32), t(shape, torch.float32)),                                     # no cache's type
                  binding.KvCache(t((2, 10, 3, 32)), t((2, 10, 3, 32))),                                                 # nor a head's size
                  binding.KvCache(t((2, 10, 3, 68))[..., :64], t((2, 10, 3, 68))[..., :64]),                             # strides of 8 bytes
                  binding.KvCache(*(t((1, 10, 3, 64)).expand(shape) for _ in range(2))),                                 # rows in one place
                  binding.KvCache(*(t((2 * 10 * 3 * 64 + 8,))[4:-4].view(shape) for _ in range(2)))):                    # not where 16 bytes begin
        with pytest.raises(binding.SdmsError):
            d = cache.shape[3]
            binding.sdms_kv_append(cache, t((2, 1, 3, d), cache.new_dtype), t((2, 1, 3, d), cache.new_dtype), lens)
    good = binding.KvCache(k, v)
    for args in [(new.half(), new, lens), (new, new[:1], lens), (new, new, lens.long()), (new, new, lens[:1]), (new, new, lens.cpu()), (new, new, lens, lens.float()),
                 (t((2, 1, 3, 128))[..., ::2], new, lens)]:
        with pytest.raises(ValueError):
            binding.sdms_kv_append(good, *args)
    with pytest.raises(binding.SdmsError):
        binding.sdms_kv_append(good, t((2, 0, 3, 64)), t((2, 0, 3, 64)), lens)                                           # no tokens at all
    for args in [(lens.long(), lens, 2), (lens[:1], lens, 2), (lens, lens.cpu(), 2)]:
        with pytest.raises(ValueError):
            binding.sdms_kv_reorder(good, *args)
    with pytest.raises(binding.SdmsError):
        binding.sdms_kv_reorder(good, lens, lens, 3)
    torch.cuda.synchronize()


def test_calls_of_attention_that_are_refused():
    def t(shape, dtype=torch.bfloat16, device=DEV):
        return torch.zeros(shape, device=device, dtype=dtype)
    att = binding.PathAttention(1, 2, 3, 4, 2, 64, torch.bfloat16)
    paths = binding.KvCache.empty(2, 20, 2, 64, torch.bfloat16)
    q, out, lens = t((2, 3, 4, 64)), t((2, 3, 4, 64)), t((2,), torch.int32)
    att(q, out, paths, lens)
    for args, kw in [((q[:, :2], out, paths, lens), {}), ((q, out.half(), paths, lens), {}), ((q.cpu(), out, paths, lens), {}), ((q, out, paths, None), {}),
                     ((q, out, paths, lens.long()), {}), ((q, out, None, None), dict(prefix=paths)), ((q, out, paths, lens), dict(mask=t((2, 3), torch.int32))),
                     ((q, out, paths, lens), dict(mask=t((2, 2), torch.int64))), ((q, out, paths, lens), dict(counts=t((3,), torch.int32))),
                     ((t((2, 3, 4, 128))[..., ::2], out, paths, lens), {}), ((q, t((2, 3, 4, 128))[..., ::2], paths, lens), {})]:
        with pytest.raises(ValueError):
            att(*args, **kw)
    for args, kw in [((q, out, None, None), {}), ((q, out, paths, lens), dict(scale=0.0)), ((q, out, paths, lens), dict(scale=float("nan"))),
                     ((q, out, binding.KvCache.empty(3, 20, 2, 64, torch.bfloat16), lens), {}), ((q, out, binding.KvCache.empty(2, 20, 1, 64, torch.bfloat16), lens), {}),
                     ((q, out, binding.KvCache.empty(2, 20, 2, 64, torch.float16), lens), {}), ((t((2, 3, 4, 68))[..., :64], out, paths, lens), {}),
                     ((q, t((2, 3, 1, 64)).expand(2, 3, 4, 64), paths, lens), {})]:
        with pytest.raises(binding.SdmsError):
            att(*args, **kw)
    att(q, out, paths, lens)                                 # and the next call is as the first
    assert not att.timed_out()
