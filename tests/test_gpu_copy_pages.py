"""Pages copied within a cache and from one to another, bit for bit."""
import numpy as np
import pytest
import torch

from lr_workloads import Model
from paper_2506_19830_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["bf16", "fp8", "fp4"]


def cache_of(kind, model, pages, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    h, d = model.n_kv_heads, model.head_dim
    u8 = lambda *shape: torch.randint(0, 256, shape, dtype=torch.uint8, device=DEV, generator=g)  # noqa: E731
    if kind == "bf16":
        return B.Bf16Cache(*(u8(pages, h, 16, d * 2).view(torch.bfloat16) for _ in range(2)))
    if kind == "fp8":
        return B.Fp8Cache(u8(pages, h, 16, d), u8(pages, h, 16, d), u8(pages, h, 16), u8(pages, h, 16))
    return B.Fp4Cache(u8(pages, h, 16, d // 2), u8(pages, h, 16, d // 2), u8(pages, h, 16, d // 32), u8(pages, h, 16, d // 32))


def pools(cache):
    names = ("k", "v") if isinstance(cache, B.Bf16Cache) else ("k", "v", "k_scale", "v_scale")
    return [getattr(cache, n).view(torch.uint8) for n in names]


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("h,d", [(1, 64), (3, 64), (8, 128), (1, 128), (50, 128)])
@pytest.mark.parametrize("n,layers", [(1, 1), (7, 3), (40, 1), (3, 70)])
def test_pages_are_copied(kind, h, d, n, layers):
    model, pages = Model(h, h, d, 8), 2 * n + 5
    if layers == 70 and h == 50:
        pages = 7
    rng = np.random.default_rng(n + h)
    ctx = B.Context(model, 0)
    caches = [cache_of(kind, model, pages, s) for s in range(layers)]
    order = rng.permutation(pages)
    n = min(n, pages // 2)
    src, dst = order[:n], order[n:2 * n]
    before = [[p.clone() for p in pools(c)] for c in caches]
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    ctx.lr_copy_pages(caches, caches, i32(src.tolist()), i32(dst.tolist()), status)
    origin = np.arange(pages)
    origin[dst] = src
    at = torch.from_numpy(origin).to(DEV)
    for c, was in zip(caches, before):
        for p, w in zip(pools(c), was):
            assert torch.equal(p, w[at])
    assert status.tolist() == [0, 0] and ctx.launch_count == (layers + 31) // 32
    ctx.close()


@pytest.mark.parametrize("kind", KINDS)
def test_pages_are_taken_out_and_put_back(kind):
    """Through a cache of another size, with the same page twice as a source; one onto itself."""
    model = Model(4, 2, 128, 8)
    ctx, big, small = B.Context(model, 0), cache_of(kind, model, 20, 1), cache_of(kind, model, 4, 2)
    before = [p.clone() for p in pools(big)]
    ctx.lr_copy_pages(big, small, i32([19, 7, 7, 0]), i32([0, 1, 3, 2]))
    for p, w in zip(pools(small), before):
        assert torch.equal(p, w[[19, 7, 0, 7]])
    for p in pools(big):
        p.zero_()
    ctx.lr_copy_pages(small, big, i32([0, 1, 2]), i32([19, 7, 0]))
    ctx.lr_copy_pages(big, big, i32([7]), i32([7]))
    for p, w in zip(pools(big), before):
        want = torch.zeros_like(w)
        want[[19, 7, 0]] = w[[19, 7, 0]]
        assert torch.equal(p, want)
    ctx.close()


def test_pages_that_are_not_there_are_left_out_and_reported():
    model = Model(4, 2, 64, 8)
    ctx, a, b = B.Context(model, 0), cache_of("fp4", model, 6, 1), cache_of("fp4", model, 4, 2)
    was = [p.clone() for p in pools(b)]
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    ctx.lr_copy_pages(a, b, i32([-1, 5, 3, -7]), i32([0, -2, 1, -1]), status)  # negative: left out
    assert status.tolist() == [0, 0]
    for p, w, s in zip(pools(b), was, pools(a)):
        w[1] = s[3]
        assert torch.equal(p, w)
    for src, dst in ((6, 0), (1, 4), ((1 << 31) - 1, 2), (0, (1 << 31) - 1)):
        status.zero_()
        ctx.lr_copy_pages(a, b, i32([2, src]), i32([3, dst]), status)
        assert status.tolist() == [-5, 1]
        ctx.lr_copy_pages(a, b, i32([2, src]), i32([3, dst]))
        for p, w, s in zip(pools(b), was, pools(a)):
            w[3] = s[2]
            assert torch.equal(p, w)
    ctx.close()


def test_refusals():
    model = Model(4, 2, 64, 8)
    ctx, L = B.Context(model, 0), B.lib()
    a, b, other = cache_of("fp4", model, 6, 1), cache_of("fp8", model, 6, 2), cache_of("fp4", Model(4, 4, 64, 8), 6, 3)
    one = i32([1])
    for src, dst, s, d in ((a, other, one, one), (other, a, one, one), ([a, a], a, one, one), (a, a, one.long(), one), (a, a, one, i32([1, 2])), (a, a, one.cpu(), one),
                           (a, a, i32([1, 2, 3, 4])[::2], i32([1, 2]))):
        with pytest.raises(ValueError):
            ctx.lr_copy_pages(src, dst, s, d)
    for src, dst in ((a, b), ([a, b], [a, b])):
        with pytest.raises(B.LrError) as e:
            ctx.lr_copy_pages(src, dst, one, one)
        assert e.value.status == -1 and "one kind" in str(e.value)
    at = one.data_ptr()
    for args in ((None, a.any, a.any, 1, at, at, 1), (ctx.handle, None, a.any, 1, at, at, 1), (ctx.handle, a.any, None, 1, at, at, 1), (ctx.handle, a.any, a.any, -1, at, at, 1),
                 (ctx.handle, a.any, a.any, 1, None, at, 1), (ctx.handle, a.any, a.any, 1, at, None, 1), (ctx.handle, a.any, a.any, 1, at, at, -1), (ctx.handle, a.any, a.any, 1, at + 2, at, 1)):
        assert L.lr_copy_pages(*args, None, None) == -1
    ctx.lr_copy_pages(a, a, one[:0], one[:0])
    ctx.lr_copy_pages([], [], one, one)
    assert ctx.launch_count == 0
    ctx.close()


def test_a_cache_whose_bytes_pass_32_bits_and_a_graph():
    model, pages = Model(8, 8, 128, 8), 140_000  # 4.6 GB a pool
    ctx = B.Context(model, 0)
    k, v = (torch.zeros((pages, 8, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cache = B.Bf16Cache(k, v)
    k[pages - 1], v[pages - 2] = 3.0, 5.0
    src, dst = i32([pages - 1, 4]), i32([4, pages - 2])
    ctx.lr_copy_pages(cache, cache, src[:1], dst[:1])
    assert bool((k[4] == 3.0).all()) and bool((v[4] == 0.0).all())
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        ctx.lr_copy_pages(cache, cache, src[1:], dst[1:])
    assert bool((v[pages - 2] == 5.0).all())
    graph.replay()
    torch.cuda.synchronize()
    assert bool((k[pages - 2] == 3.0).all()) and bool((v[pages - 2] == 0.0).all())
    del graph
    ctx.close()
