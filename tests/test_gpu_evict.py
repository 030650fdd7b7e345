"""Eviction by gathered weight against sorting on the CPU: the kept places exactly,
the moved rows bit for bit, everything else in the cache as it was."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]


def kept64(w, n, budget, first, recent):
    """The places that stay of n with weights w (numpy, 64 bits)."""
    if n <= budget:
        return list(range(n))
    middle = range(first, n - recent)
    order = sorted(middle, key=lambda j: (-(math.inf if np.isnan(w[j]) else w[j]), not np.isnan(w[j]), j))
    take = order[:budget - first - recent]
    return sorted(list(range(first)) + take + list(range(n - recent, n)))


def setup(lengths, page, max_pages, heads, d, dtype, seed, max_to=0, kind="spread"):
    """(k, v, w, table, to) on the CPU: shuffled pages, -1 where unused."""
    g = torch.Generator().manual_seed(seed)
    B = len(lengths)
    need = [-(-max(n, 0) // page) for n in lengths]
    pages = sum(need) + B * max_to + 3
    order = torch.randperm(pages, generator=g).int()
    table, at = torch.full((B, max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :min(n, max_pages)] = order[at:at + min(n, max_pages)]
        at += n
    to = order[at:at + B * max_to].view(B, max_to).contiguous()
    k, v = (torch.randn((pages, heads, page, d), generator=g).to(dtype) for _ in range(2))
    w = torch.randn((pages, heads, page), generator=g)
    w = {"spread": lambda: w.exp(), "ties": lambda: (w * 2).round(), "equal": lambda: torch.zeros_like(w),
         "wild": lambda: torch.where(w > 1.5, math.nan, torch.where(w < -1.5, -math.inf,
                                                                    torch.where(w.abs() < 0.3, -0.0, w)))}[kind]()
    return k, v, w, table, to


def evicted(k, v, w, table, to, lengths, budget, first, recent):
    """(k, v, w, kept, left) by the definition; to None: in place."""
    page, heads = k.shape[2], k.shape[1]
    out = [x.clone() for x in (k, v, w)]
    kept = torch.full((len(lengths), heads, budget), -1, dtype=torch.int32)
    left = torch.full((len(lengths),), -1, dtype=torch.int32)
    room = table.shape[1] * page
    valid = lambda p: 0 <= p < k.shape[0]
    for b, n in enumerate(lengths):
        if n < 0 or n > min(room, 65536):
            continue
        left[b] = min(n, budget)
        j = np.arange(n)
        for h in range(heads):
            p = table[b, j // page].numpy()
            ok = (p >= 0) & (p < k.shape[0])
            wj = np.where(ok, w[np.where(ok, p, 0), h, j % page].double().numpy(), -math.inf)
            stay = kept64(wj, n, budget, first, recent)
            if not ok.all():     # places without a page weigh less than -inf
                order = sorted(range(first, n - recent), key=lambda i: (
                    not ok[i], -(math.inf if np.isnan(wj[i]) else wj[i]), not np.isnan(wj[i]), i))
                if n > budget:
                    stay = sorted(list(range(first)) + order[:budget - first - recent]
                                  + list(range(n - recent, n)))
            kept[b, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
            for i, s in enumerate(stay):
                q = int((table if to is None else to)[b, i // page])
                if not ok[s] or not valid(q):
                    continue
                for x, y in zip(out, (k, v, w)):
                    x[q, h, i % page] = y[p[s], h, s % page]
    return (*out, kept, left)


def same(a, b):
    """Equal bits (NaN payloads and zeros' signs too)."""
    kind = {torch.float32: torch.int32, torch.bfloat16: torch.int16}.get(a.dtype, a.dtype)
    return torch.equal(a.cpu().contiguous().view(kind), b.cpu().contiguous().view(kind))


def run(splat, case, budget, first, recent, lengths, moves, **kw):
    k, v, w, table, to = (x.cuda() for x in case)
    kept, left = splat.cache_evict(k, v, w, table, torch.tensor(lengths, dtype=torch.int32).cuda(), budget,
                                   first=first, recent=recent, to=to if moves else None, **kw)
    torch.cuda.synchronize()
    return k, v, w, kept, left


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,d,page", [(1, 64, 1), (3, 128, 16), (2, 64, 128)])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "wild"])
@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (1, 1, 0), (70, 0, 0), (70, 4, 20), (70, 30, 40),
                                                 (300, 1, 77)])
@pytest.mark.parametrize("moves", [False, True])
def test_evict(gpu_lib, moves, budget, first, recent, kind, heads, d, page, dtype):
    splat = gpu_lib
    lengths = [0, 1, budget, budget + 1, 331, 64]
    print(f"[gpu] evict {budget} {first} {recent} {kind} heads={heads} d={d} page={page} {dtype} {moves}", flush=True)
    case = setup(lengths, page, -(-400 // page), heads, d, dtype, budget + d, -(-budget // page), kind)
    want = evicted(*case[:4], case[4] if moves else None, lengths, budget, first, recent)
    for got, x in zip(run(splat, case, budget, first, recent, lengths, moves), want):
        assert same(got, x)


@pytest.mark.parametrize("n,budget", [(4096, 1000), (4097, 4096), (16384, 9000), (16385, 100), (65536, 65535),
                                      (65536, 33)])
@pytest.mark.parametrize("moves", [False, True])
def test_long(gpu_lib, moves, n, budget):
    """Each size of the kernel that selects, at and past its room."""
    splat = gpu_lib
    case = setup([n, n // 2], 256, -(-n // 256), 1, 64, torch.bfloat16, n, -(-budget // 256), "ties")
    want = evicted(*case[:4], case[4] if moves else None, [n, n // 2], budget, 5, 7)
    for got, x in zip(run(splat, case, budget, 5, 7, [n, n // 2], moves), want):
        assert same(got, x)


@pytest.mark.parametrize("moves", [False, True])
def test_bad_lengths_and_pages(gpu_lib, moves):
    splat = gpu_lib
    lengths = [-1, 200, 201, 2 ** 31 - 1, 150, -2 ** 31]
    case = setup([200] * 6, 8, 25, 2, 64, torch.float32, 3, 8)
    case[3][1, 2], case[3][1, 20], case[3][4, 3], case[4][4, 1], case[4][1, 7] = -1, 10 ** 6, -7, 5000, -1
    for budget, first, recent in ((60, 20, 30), (60, 0, 0), (62, 0, 50)):
        want = evicted(*case[:4], case[4] if moves else None, lengths, budget, first, recent)
        for got, x in zip(run(splat, case, budget, first, recent, lengths, moves), want):
            assert same(got, x)


def test_shared_pages_stay(gpu_lib):
    """Sequences with a common beginning move to pages of their own: what they share
    stays as it was."""
    splat = gpu_lib
    case = setup([120, 120], 16, 8, 2, 64, torch.bfloat16, 3, 3)
    case[3][1, :5] = case[3][0, :5]
    want = evicted(*case, [120, 100], 48, 4, 8)
    got = run(splat, case, 48, 4, 8, [120, 100], True)
    for x, y in zip(got, want):
        assert same(x, y)


def test_given_outputs_streams_and_graphs(gpu_lib):
    splat = gpu_lib
    lengths = [300, 77, 512]
    case = setup(lengths, 16, 32, 2, 64, torch.bfloat16, 9, 7)
    k, v, w, table, to = (x.cuda() for x in case)
    n = torch.tensor(lengths, dtype=torch.int32).cuda()
    kept = torch.empty((3, 2, 100), dtype=torch.int32, device="cuda")
    left = torch.empty(3, dtype=torch.int32, device="cuda")
    call = lambda: splat.cache_evict(k, v, w, table, n, 100, first=2, recent=9, to=to, kept=kept, left=left)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert r[0] is kept or r[0].data_ptr() == kept.data_ptr()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for r in range(4):
        w.copy_(torch.randn(w.shape, generator=torch.Generator().manual_seed(r)))
        n.copy_(torch.tensor([300 - 50 * r, 77 + r, 512], dtype=torch.int32))
        want = evicted(k.cpu(), v.cpu(), w.cpu(), case[3], case[4], n.tolist(), 100, 2, 9)
        kept.zero_(), left.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((k, v, w, kept, left), want):
            assert same(x, y)


def test_refusals(gpu_lib):
    splat = gpu_lib
    k, v, w, table, to = (x.cuda() for x in setup([40, 40], 8, 5, 2, 64, torch.float32, 1, 2))
    n = torch.tensor([40, 40], dtype=torch.int32).cuda()
    before = [x.clone() for x in (k, v, w)]
    call = lambda **kw: splat.cache_evict(**{**dict(k_cache=k, v_cache=v, weights=w, table=table, lengths=n,
                                                    budget=16, to=to), **kw})
    ints = torch.zeros(64, dtype=torch.int32, device="cuda")
    bad = [lambda: call(budget=0), lambda: call(budget=-1), lambda: call(budget=65537), lambda: call(budget=2 ** 32 + 16),
           lambda: call(first=-1), lambda: call(recent=-2), lambda: call(first=10, recent=7), lambda: call(budget=17),
           lambda: call(first=2 ** 32), lambda: call(to=to[:1]), lambda: call(to=to.long()), lambda: call(to=to[:, :1]),
           lambda: call(to=to[:, :0]), lambda: call(table=table[:1]), lambda: call(lengths=n.long()),
           lambda: call(lengths=n[:1]), lambda: call(weights=w.double()), lambda: call(weights=w[:, :1]),
           lambda: call(v_cache=k), lambda: call(v_cache=v.bfloat16()), lambda: call(left=n),
           lambda: call(kept=torch.empty((2, 2, 15), dtype=torch.int32, device="cuda")),
           lambda: call(left=torch.empty(3, dtype=torch.int32, device="cuda")), lambda: call(left=ints[:2], kept=ints.view(2, 2, 16)),
           lambda: call(weights=k.view(-1)[:w.numel()].view(w.shape)), lambda: call(weights=w.transpose(0, 1)),
           lambda: call(k_cache=k.cpu()), lambda: call(k_cache=k.half(), v_cache=v.half()),
           lambda: call(k_cache=k[..., :32].contiguous(), v_cache=v[..., :32].contiguous()), lambda: call(budget=1.5)]
    for i, f in enumerate(bad):
        with pytest.raises((splat.SplatError, TypeError, ValueError)) as e:
            f()
        if isinstance(e.value, splat.SplatError):
            assert e.value.name in ("INVALID_ARG", "UNSUPPORTED"), (i, e.value)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((k, v, w), before))
