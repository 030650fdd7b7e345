"""The measured operators of serving long and mixed sequences from the paged cache:
prompts that arrive in chunks, caches kept within a budget, tokens with a place in
time and in a picture.

``chunk``   sparse_mhsa_chunk: the new tokens of each sequence, already in the
            paged cache, attend to it under the mask; returns O and the rows'
            log-sum-exp
``weigh``   cache_weights: adds the attention weight that each cached key took from
            a step's queries to what it has gathered; returns the weights
``evict``   cache_evict: keeps a budget of each head's keys, those that gathered
            the most, and moves them to a sequence's new pages; returns the caches,
            the weights, the kept places and the new lengths
``axes``    rotary with several axes: Q and K of video tokens (or, `inverse`, their
            gradients) turned by time, row and column
``append``  cache_append of such tokens: positions apart from the cache's places;
            returns Q and both caches

Values are N(0, 1), which with scale = 1/sqrt(d) gives scores of standard
deviation 1, as attention inputs after a normalisation layer have.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_MASKS = {"causal": (), "sliding": ("w", "n_global"), "window_global": ("w", "n_global"),
          "strided_local": ("local", "stride"), "blocked": ("block",), "dilated": ("w", "dilation")}


def _paged(op, kind, B, H, Hkv, T, L, d, dtype, page, shortest, **params):
    return dict(op=op, kind=kind, B=B, H=H, Hkv=Hkv, T=T, L=L, d=d, dtype=dtype, page=page,
                shortest=shortest, **params)


def _weigh(kind, B, H, Hkv, T, L, d, dtype, page, shortest, decay, **params):
    return _paged("weigh", kind, B, H, Hkv, T, L, d, dtype, page, shortest, decay=decay, **params)


def _evict(B, Hkv, L, d, dtype, page, shortest, budget, first, recent):
    return dict(op="evict", B=B, Hkv=Hkv, L=L, d=d, dtype=dtype, page=page, shortest=shortest,
                budget=budget, first=first, recent=recent)


def _axes(B, H, Hkv, L, d, dtype, t, y, x, cyclic, restart, interleaved, inverse):
    return dict(op="axes", B=B, H=H, Hkv=Hkv, L=L, d=d, dtype=dtype, t=t, y=y, x=x, cyclic=cyclic,
                restart=restart, interleaved=interleaved, inverse=inverse, max_len=8192)


def _append(B, H, Hkv, T, L, d, dtype, page, t, y, x, cyclic, restart, interleaved):
    return dict(op="append", B=B, H=H, Hkv=Hkv, T=T, L=L, d=d, dtype=dtype, page=page, t=t, y=y, x=x,
                cyclic=cyclic, restart=restart, interleaved=interleaved, max_len=8192)


def listed():
    return [
        # a few drafted tokens of one user checked at once: launch and latency
        dict(_paged("chunk", "window_global", 1, 16, 16, 8, 4096, 64, "bf16", 16, 4096, w=512, n_global=64),
             name="chunk_T8_window512_global64_B1_bf16"),
        # the same for a running batch over shared heads, every earlier key
        dict(_paged("chunk", "causal", 16, 32, 8, 5, 8192, 128, "bf16", 64, 1000),
             name="chunk_T5_causal_B16_d128_bf16"),
        # a scheduler's step of prompts over 1024 tokens of each sequence, ragged
        dict(_paged("chunk", "causal", 4, 32, 8, 1024, 8192, 128, "bf16", 64, 2048),
             name="chunk_T1024_causal_L8192_d128_bf16"),
        # the second half of long documents under the window + global mask
        dict(_paged("chunk", "window_global", 4, 16, 16, 2048, 4096, 64, "bf16", 16, 4096, w=512,
                    n_global=64), name="chunk_T2048_window512_global64_bf16"),
        # a short ragged chunk of a model held in fp32, sliding window with first tokens
        dict(_paged("chunk", "sliding", 2, 12, 12, 300, 2048, 64, "f32", 16, 700, w=255, n_global=4),
             name="chunk_T300_sliding256_f32"),
        # the keys' weights after a token of a running batch
        dict(_weigh("causal", 32, 32, 8, 1, 8192, 128, "bf16", 64, 1000, 1.0),
             name="weigh_T1_causal_B32_d128_bf16"),
        # ... and after a chunk of prompts, older weight fading
        dict(_weigh("causal", 4, 16, 4, 512, 4096, 64, "bf16", 16, 600, 0.98),
             name="weigh_T512_causal_B4_bf16"),
        # one user's cache of a small model brought back to its budget
        dict(_evict(1, 16, 4096, 64, "bf16", 16, 4096, 2048, 4, 256), name="evict_4096_to_2048_B1_bf16"),
        # a running batch, half of the long sequences' keys go
        dict(_evict(16, 8, 8192, 128, "bf16", 64, 2000, 4096, 64, 512), name="evict_8192_to_4096_B16_d128_bf16"),
        # Q and K of a training batch of video tokens from their projections
        dict(_axes(2, 16, 16, 4096, 64, "bf16", 8, 12, 12, False, False, False, False),
             name="axes_8_12_12_L4096_bf16"),
        # gradients of a ragged fp32 layer, axes in turn, each with frequencies of its own
        dict(_axes(2, 12, 4, 1000, 128, "f32", 24, 20, 20, True, True, True, True),
             name="axes_cyclic_24_20_20_inverse_L1000_d128_f32"),
        # a ragged step of picture tokens into the cache, places apart from positions
        dict(_append(8, 32, 8, 500, 4096, 128, "bf16", 64, 16, 24, 24, True, False, False),
             name="append_axes_T500_d128_bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_mask(rng, L):
    kind = rng.choice(["causal", "causal", "sliding", "sliding", "window_global", "strided_local",
                       "blocked", "dilated"])
    if kind in ("sliding", "window_global"):
        return kind, dict(w=_log_int(rng, 4, 512), n_global=_log_int(rng, 1, 64))
    if kind == "strided_local":
        return kind, dict(local=_log_int(rng, 4, 256), stride=_log_int(rng, 16, 512))
    if kind == "blocked":
        return kind, dict(block=_log_int(rng, 8, 512))
    if kind == "dilated":
        return kind, dict(w=_log_int(rng, 8, 256), dilation=rng.randint(2, 4))
    return kind, {}


def draw(rng):
    """A case of the ranges above: any operator, mask family, dtype, head layout
    and page, lengths and chunks from one token on, bounded by the largest listed."""
    op = rng.choice(["chunk", "chunk", "chunk", "weigh", "weigh", "evict", "evict", "axes", "append"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32", "f32"])
    d = rng.choice([64, 64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12, 16])
    H = Hkv * rng.choice([1, 1, 2, 3, 4, 8])
    page = rng.choice([1, 8, 16, 64, 256])
    inter, cyclic, restart = (rng.random() < 0.5 for _ in range(3))
    t, y, x = rng.choice([s for s in ((8, 12, 12), (16, 8, 8), (4, 2, 2), (11, 11, 10), (16, 24, 24),
                                      (24, 20, 20), (44, 10, 10)) if 2 * sum(s) <= d])
    if op in ("axes", "append"):
        L = _log_int(rng, 1, 4096)
        B = max(1, min(rng.randint(1, 8), (1 << 24) // (L * (H + 2 * Hkv) * d)))
        if op == "axes":
            return _axes(B, H, Hkv, L, d, dtype, t, y, x, cyclic, restart, inter, rng.random() < 0.5)
        T = _log_int(rng, 1, min(L, 700))
        return _append(B, H, Hkv, T, L, d, dtype, page, t, y, x, cyclic, restart, inter)
    L = _log_int(rng, 16, 8192)
    shortest = rng.choice([0, 1, L // 3, L])
    if op == "evict":
        B = max(1, min(_log_int(rng, 1, 32), (1 << 27) // (L * Hkv * d)))
        budget = rng.randint(max(1, L // 16), L)
        first = rng.randint(0, min(64, budget // 4))
        return _evict(B, Hkv, L, d, dtype, page, shortest, budget, first, rng.randint(0, budget // 2))
    T = _log_int(rng, 1, min(L, 1024))
    kind, p = _draw_mask(rng, L)
    B = max(1, min(_log_int(rng, 1, 32), (1 << 27) // (L * Hkv * d)))
    most = 1.5e10 if dtype == "f32" else 2.0e11
    while B > 1 and 4.0 * B * H * T * L * d > most:
        B -= 1
    while 4.0 * B * H * T * L * d > most:
        T = (T + 1) // 2
    if op == "weigh":
        return _weigh(kind, B, H, Hkv, T, L, d, dtype, page, shortest, rng.choice([1.0, 0.9]), **p)
    return _paged("chunk", kind, B, H, Hkv, T, L, d, dtype, page, shortest, **p)


# ---- masks, lengths, positions: what the case says, on any device
def _mask_rows(case, i):
    """[.., L]: the mask's rows i, from the pattern's definition."""
    L, kind = case["L"], case["kind"]
    i, j = i[..., None], torch.arange(L, device=i.device)
    if kind == "sliding":            # w earlier keys, and the first n_global
        return ((j <= i) & (j >= i - case["w"])) | ((j < case["n_global"]) & (i >= case["n_global"]))
    if kind == "window_global":
        return ((i - j).abs() <= case["w"]) | (i < case["n_global"]) | (j < case["n_global"])
    if kind == "strided_local":
        s = case["stride"]
        return ((j > i - case["local"]) | (j % s == s - 1)) & (j <= i)
    if kind == "blocked":
        bi, bj = i // case["block"], j // case["block"]
        return (bi == bj) | (bj == bi - 1)
    if kind == "dilated":
        g = case["dilation"]
        return ((j - i) % g == 0) & ((j - i).abs() <= g * case["w"])
    return j <= i


def _lengths(case):
    """A batch's lengths, from `shortest` to L."""
    B, lo, hi = case["B"], case["shortest"], case["L"]
    return torch.tensor([hi if b == 0 else lo + (hi - lo) * (B - 1 - b) // max(1, B - 1)
                         for b in range(B)])


def _counts(case):
    """New tokens of each sequence: ragged where T > 1, at most its length."""
    B, T = case["B"], case["T"]
    n = torch.tensor([T - (b * T) // (2 * B) for b in range(B)])
    return torch.minimum(n, _lengths(case)) if "shortest" in case else n


def _rows(case):
    """(mask rows of the new tokens [B, T] clamped, which of them count)."""
    n, c = _lengths(case), _counts(case)
    t = torch.arange(case["T"])[None, :]
    return ((n - c)[:, None] + t).clamp(0, case["L"] - 1), t < c[:, None]


def _seen(case, device):
    """[B, T, L]: the keys that each new token attends to, in the cache."""
    rows, counts = (x.to(device) for x in _rows(case))
    n = _lengths(case).to(device)
    below = torch.arange(case["L"], device=device)[None, :] < n[:, None]
    return _mask_rows(case, rows) & below[:, None] & counts[..., None]


def _pairs_and_keys(case):
    """(query-key pairs a head, keys that some query of their sequence sees)."""
    rows, counts = _rows(case)
    pairs = keys = 0
    for b, n in enumerate(_lengths(case).tolist()):
        m = _mask_rows(case, rows[b][counts[b]])[:, :n]
        pairs, keys = pairs + int(m.sum()), keys + int(m.any(0).sum())
    return pairs, keys


def _starts(case):
    """Where an append's tokens begin in their caches."""
    B, room = case["B"], case["L"] - case["T"]
    return torch.tensor([(room * b) // B for b in range(B)])


def _table(lengths, page, max_pages, g, spare=3):
    """A shuffled page table: (table [B, max_pages], -1 where unused; pages)."""
    need = [-(-int(n) // page) for n in lengths]
    order = torch.randperm(sum(need) + spare, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(need), max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order


def _places(case, table, lengths):
    """(pages, offsets) [B, L] of each sequence's places, page 0 where none."""
    j = torch.arange(case["L"], device=table.device)
    return table.long().clamp(min=0)[:, j // case["page"]], (j % case["page"]).expand(table.shape[0], -1)


def _pair_axes(case):
    """Axis of each pair, and its number among the axis's pairs."""
    left, owner = [case["t"], case["y"], case["x"]], []
    if case["cyclic"]:               # the axes take turns while they have pairs left
        while sum(left):
            for a in range(3):
                if left[a]:
                    owner.append(a)
                    left[a] -= 1
    else:
        owner = [a for a in range(3) for _ in range(left[a])]
    return owner, [owner[:k].count(a) for k, a in enumerate(owner)]


def _frequencies(case, device):
    """Angle per position of each pair, 64 bits: one ladder over all pairs, or one
    over each axis's."""
    owner, number = _pair_axes(case)
    size = [case["t"], case["y"], case["x"]]
    if case["restart"]:
        e = [k / size[a] for a, k in zip(owner, number)]
    else:
        e = [k / len(owner) for k in range(len(owner))]
    return 10000.0 ** -torch.tensor(e, dtype=torch.float64, device=device)


def _grid_positions(B, T, max_len, g):
    """[3, B, T]: frames of a picture of 8 .. 64 rows and columns, one after the
    other from some time on."""
    rows, cols = (int(x) for x in torch.randint(8, 65, (2,), generator=g, device="cuda"))
    n = torch.randint(0, rows * cols, (B, 1), generator=g, device="cuda") + torch.arange(T, device="cuda")
    time = torch.randint(0, max_len // 2, (B, 1), generator=g, device="cuda") + n // (rows * cols)
    return torch.stack((time, n // cols % rows, n % cols)).int()


# ---- inputs
def _randn(shape, dtype, g):
    return torch.randn(shape, generator=g, device="cuda").to(_DTYPES[dtype])


def _log_sums(case, st):
    """The rows' log-sum-exp, which the attention before leaves, [B, H, T] fp32."""
    out = torch.full((case["B"], case["H"], case["T"]), -math.inf, device="cuda")
    seen = _seen(case, "cuda")
    pages, offs = _places(case, st["table"], st["lengths"])
    G = case["H"] // case["Hkv"]
    for b in range(case["B"]):
        k = st["kc"][pages[b], :, offs[b]].transpose(0, 1).float()
        q = st["q"][b].float().view(case["Hkv"], G * case["T"], case["d"])
        s = (q @ k.transpose(-1, -2) * st["scale"]).view(case["H"], case["T"], case["L"])
        out[b] = torch.logsumexp(s.masked_fill_(~seen[b], -math.inf), -1)
    return out


def _inputs(case, seed):
    g = torch.Generator("cuda").manual_seed(int(seed))
    dt, d, op, B, Hkv = case["dtype"], case["d"], case["op"], case["B"], case["Hkv"]
    st = dict(case=case, scale=1.0 / math.sqrt(d))
    if op in ("axes", "append"):
        # [B, T, H, d], as a projection leaves them, seen as [B, H, T, d]
        T = case["L"] if op == "axes" else case["T"]
        st["q"] = _randn((B, T, case["H"], d), dt, g).transpose(1, 2)
        st["k"] = _randn((B, T, Hkv, d), dt, g).transpose(1, 2)
        st["positions"] = _grid_positions(B, T, case["max_len"], g)
    if op == "axes":
        return st
    page = case["page"]
    if op == "append":
        st["v"] = _randn((B, case["T"], Hkv, d), dt, g).transpose(1, 2)
        start, count = _starts(case), _counts(case)
        lengths = start + count
        st["start"], st["count"] = start.int().cuda(), count.int().cuda()
    else:
        lengths = _lengths(case)
    most = -(-case["L"] // page)
    kept = lengths.clamp(max=case["budget"]) if op == "evict" else lengths[:0]
    spare = 3 + sum(-(-int(n) // page) for n in kept)
    st["table"], order = _table(lengths, page, most, g, spare)
    st["lengths"] = lengths.int().cuda()
    st["kc"], st["vc"] = (_randn((order.numel(), Hkv, page, d), dt, g) for _ in range(2))
    if op == "evict":
        # weights as attention gathers them: most keys little, a few much
        st["w"] = torch.randn((order.numel(), Hkv, page), generator=g, device="cuda").mul_(2).exp_()
        st["to"] = torch.full((B, -(-case["budget"] // page)), -1, dtype=torch.int32, device="cuda")
        at = order.numel() - spare
        for b, n in enumerate(kept.tolist()):
            need = -(-n // page)
            st["to"][b, :need] = order[at:at + need]
            at += need
        return st
    if op in ("chunk", "weigh"):
        st["q"] = _randn((B, case["H"], case["T"], d), dt, g)
        st["count"] = _counts(case).int().cuda()
    if op == "weigh":
        st["lse"] = _log_sums(case, st)
        st["w"] = torch.randn((order.numel(), Hkv, page), generator=g, device="cuda").mul_(2).exp_()
        st["out"] = torch.zeros_like(st["w"])
    return st


def _acsr_of(case, splat):
    L, p = case["L"], {k: case[k] for k in _MASKS[case["kind"]]}
    if case["kind"] == "causal":
        pat = splat.Pattern.from_terms(L, [dict(hi_i=1)])
    elif case["kind"] == "sliding":
        terms = [dict(lo_i=1, lo_c=-p["w"], hi_i=1)]
        if p["n_global"] < L:
            terms.append(dict(row_lo=p["n_global"], hi_c=p["n_global"] - 1))
        pat = splat.Pattern.from_terms(L, terms)
    else:
        pat = splat.Pattern.named(case["kind"], p, L)
    return splat.Acsr(pat)


def prepare(case, seed):
    """A step's inputs, and what a program keeps from call to call: the mask's and
    the rotation's handles; for the plain form the mask, the places of the cache's
    tokens and the angles' cosines and sines."""
    st = _inputs(case, seed)
    op = case["op"]
    if own:
        import paper_2407_16847_amd as splat
        if op in ("chunk", "weigh"):
            st["acsr"] = _acsr_of(case, splat)
        elif op != "evict":
            st["rot"] = splat.Rotary(case["max_len"], 2 * (case["t"] + case["y"] + case["x"]),
                                     interleaved=case["interleaved"],
                                     axes=(case["t"], case["y"], case["x"]), cyclic=case["cyclic"],
                                     restart=case["restart"])
        return st
    if op in ("chunk", "weigh"):
        st["seen"] = _seen(case, "cuda")
    if op in ("chunk", "weigh", "evict"):
        st["pages"], st["offs"] = _places(case, st["table"], st["lengths"])
        return st
    a = (torch.arange(case["max_len"], device="cuda", dtype=torch.float64)[:, None]
         * _frequencies(case, "cuda")[None, :])
    st["cos"], st["sin"] = a.cos().float(), a.sin().float()
    st["owner"] = torch.tensor(_pair_axes(case)[0], device="cuda")
    if op == "append":
        t = torch.arange(case["T"], device="cuda")[None, :]
        b, t = (t < st["count"][:, None]).nonzero(as_tuple=True)
        st["b"], st["t"], st["place"] = b, t, st["start"].long()[b] + t
    return st


# ---- the plain forms
def _scores(st):
    """Masked scores [B, Hkv, G T, L] of the new tokens, in 32 bits, and V."""
    c = st["case"]
    B, H, Hkv, T, d = (c[x] for x in ("B", "H", "Hkv", "T", "d"))
    k = st["kc"][st["pages"], :, st["offs"]].permute(0, 2, 3, 1).float()
    q = st["q"].float().view(B, Hkv, (H // Hkv) * T, d)
    s = (q @ k).mul_(st["scale"])
    s.view(B, H, T, -1).masked_fill_(~st["seen"][:, None], -math.inf)
    return s


def _plain_chunk(st):
    c = st["case"]
    s = _scores(st)
    m = s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (m + total.log()).view(c["B"], c["H"], c["T"])
    v = st["vc"][st["pages"], :, st["offs"]].transpose(1, 2).float()
    v = v * (torch.arange(c["L"], device="cuda") < st["lengths"][:, None])[:, None, :, None]
    o = (p @ v) / total.clamp(min=torch.finfo(torch.float32).tiny)
    return o.view(st["q"].shape).to(st["q"].dtype), lse


def _plain_weigh(st):
    c = st["case"]
    s = _scores(st).view(c["B"], c["Hkv"], -1, c["T"], c["L"])
    lse = st["lse"].view(c["B"], c["Hkv"], -1, c["T"], 1).clamp(min=torch.finfo(torch.float32).min)
    add = s.sub_(lse).exp_().sum((2, 3))
    j = torch.arange(c["L"], device="cuda")
    old = st["w"][st["pages"], :, st["offs"]].transpose(1, 2)
    fade = torch.where(st["count"] > 0, c["decay"], 1.0)[:, None, None]
    before = (j < (st["lengths"] - st["count"])[:, None])[:, None]
    new = torch.where(before, old * fade, 0.0) + add
    b, j = (j < st["lengths"][:, None]).nonzero(as_tuple=True)
    st["out"][st["pages"][b, j], :, st["offs"][b, j]] = new[b, :, j]
    return st["out"]


def _plain_evict(st):
    c = st["case"]
    B, Hkv, L, budget, page = (c[x] for x in ("B", "Hkv", "L", "budget", "page"))
    j, n = torch.arange(L, device="cuda"), st["lengths"].long()[:, None]
    w = st["w"][st["pages"], :, st["offs"]].transpose(1, 2)
    always = (j < c["first"]) | (j >= n - c["recent"])
    w = w.masked_fill(always[:, None], math.inf).masked_fill((j >= n)[:, None], -math.inf)
    best = w.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    left = n.clamp(max=budget)
    best = best.masked_fill(torch.arange(best.shape[-1], device="cuda") >= left[:, None], L)
    best = best.sort(dim=-1).values
    kept = torch.where(best < L, best, -1)
    b, h, i = (kept >= 0).nonzero(as_tuple=True)
    src = kept[b, h, i]
    sp, so = st["pages"][b, src], st["offs"][b, src]
    dp, do = st["to"].long()[b, i // page], i % page
    for x in (st["kc"], st["vc"], st["w"]):
        x[dp, h, do] = x[sp, h, so]
    return st["kc"], st["vc"], st["w"], kept.int(), left[:, 0].int()


def _rotate(c, x, cos, sin, inverse):
    """x [.., d] in 32 bits, cos and sin [.., pairs] broadcast against it."""
    R = 2 * cos.shape[-1]
    sin = -sin if inverse else sin
    r, rest = x[..., :R], x[..., R:]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :R // 2], r[..., R // 2:])
    u, v = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((u, v), -1).flatten(-2) if c["interleaved"] else torch.cat((u, v), -1)
    return torch.cat((y, rest), -1)


def _plain_axes(st):
    c = st["case"]
    at = st["positions"].long()[st["owner"]].permute(1, 2, 0)     # [B, T, pairs]
    pair = torch.arange(at.shape[-1], device="cuda")
    cos, sin = st["cos"][at, pair][:, None], st["sin"][at, pair][:, None]
    return tuple(_rotate(c, x.float(), cos, sin, c.get("inverse", False)).to(x.dtype)
                 for x in (st["q"], st["k"]))


def _plain_append(st):
    c, b, t, place = st["case"], st["b"], st["t"], st["place"]
    q, k = _plain_axes(st)
    pages, offs = st["table"].long()[b, place // c["page"]], place % c["page"]
    st["kc"][pages, :, offs] = k[b, :, t]
    st["vc"][pages, :, offs] = st["v"][b, :, t]
    fresh = torch.arange(c["T"], device="cuda")[None, :] < st["count"][:, None]
    return q * fresh[:, None, :, None], st["kc"], st["vc"]


def run(st):
    c = st["case"]
    op = c["op"]
    if not own:
        return {"chunk": _plain_chunk, "weigh": _plain_weigh, "evict": _plain_evict,
                "axes": _plain_axes, "append": _plain_append}[op](st)
    import paper_2407_16847_amd as splat
    if op == "chunk":
        return splat.sparse_mhsa_chunk(st["acsr"], st["q"], st["kc"], st["vc"], st["table"],
                                       st["lengths"], st["scale"], counts=st["count"])
    if op == "weigh":
        return splat.cache_weights(st["acsr"], st["q"], st["lse"], st["kc"], st["table"], st["lengths"],
                                   st["w"], st["scale"], counts=st["count"], decay=c["decay"],
                                   out=st["out"])
    if op == "evict":
        kept, left = splat.cache_evict(st["kc"], st["vc"], st["w"], st["table"], st["lengths"],
                                       c["budget"], first=c["first"], recent=c["recent"], to=st["to"])
        return st["kc"], st["vc"], st["w"], kept, left
    if op == "axes":
        return splat.rotary(st["rot"], st["q"], st["k"], positions=st["positions"], inverse=c["inverse"])
    q = splat.cache_append(st["kc"], st["vc"], st["table"], st["start"], st["k"], st["v"],
                           counts=st["count"], rot=st["rot"], Q=st["q"], positions=st["positions"])
    return q, st["kc"], st["vc"]


def work(case):
    """Each input read once and each output written once.  chunk, weigh: the keys
    that some new token sees (and their values), four and two flops a feature of
    each query-key pair.  evict: all weights in, the kept rows in and out."""
    e, d, op, B, Hkv = _BYTES[case["dtype"]], case["d"], case["op"], case["B"], case["Hkv"]
    if op in ("axes", "append"):
        pairs, H = case["t"] + case["y"] + case["x"], case["H"]
        n = B * case["L"] if op == "axes" else int(_counts(case).sum())
        heads = H + Hkv + (Hkv if op == "append" else 0)
        return {"bytes": 2 * n * heads * d * e + n * (12 + 8 * pairs), "flops": 6.0 * n * (H + Hkv) * pairs}
    if op == "evict":
        n = _lengths(case)
        kept = int(n.clamp(max=case["budget"]).sum()) * Hkv
        return {"bytes": kept * (4 * d * e + 4 + 4) + 4 * int(n.sum()) * Hkv, "flops": 0.0}
    pairs, keys = _pairs_and_keys(case)
    rows = int(_counts(case).sum()) * case["H"]
    if op == "weigh":
        return {"bytes": keys * Hkv * d * e + rows * (d * e + 4) + 8 * int(_lengths(case).sum()) * Hkv,
                "flops": 2.0 * pairs * case["H"] * d}
    return {"bytes": 2 * keys * Hkv * d * e + rows * (2 * d * e + 4), "flops": 4.0 * pairs * case["H"] * d}


# ---- from the definitions, in 64 bits
def _sequence(case, st, b):
    """(length, new tokens, their mask rows [t, n], page and offset of each key)."""
    n, c = int(_lengths(case)[b]), int(_counts(case)[b])
    m = _mask_rows(case, torch.arange(n - c, n, device="cuda"))[:, :n]
    j = torch.arange(n, device="cuda")
    return n, c, m, st["table"][b].long()[j // case["page"]], j % case["page"]


def _exact_chunk(case, st):
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        n, c, m, pages, offs = _sequence(case, st, b)
        for h in range(case["H"] if c else 0):
            hk = h // (case["H"] // case["Hkv"])
            k, v = (st[x][pages, hk, offs].double() for x in ("kc", "vc"))
            s = (st["q"][b, h, :c].double() @ k.t() * st["scale"]).masked_fill(~m, -math.inf)
            lse[b, h, :c] = torch.logsumexp(s, -1)
            o[b, h, :c] = torch.softmax(s, -1).masked_fill(~m.any(-1)[:, None], 0.0) @ v
    return o, lse


def _exact_weigh(case, st):
    out = st["out"].double()
    G = case["H"] // case["Hkv"]
    for b in range(case["B"]):
        n, c, m, pages, offs = _sequence(case, st, b)
        for hk in range(case["Hkv"] if n else 0):
            k = st["kc"][pages, hk, offs].double()
            w = st["w"][pages, hk, offs].double() * (case["decay"] if c else 1.0)
            w[n - c:] = 0.0
            for h in range(hk * G, hk * G + G):
                s = st["q"][b, h, :c].double() @ k.t() * st["scale"]
                p = (s - st["lse"][b, h, :c, None].double()).exp()
                w = w + torch.where(m, p, 0.0).sum(0)
            out[pages, hk, offs] = w
    return out


def _exact_evict(case, st):
    """Kept places by sorting each head's (weight, place) pairs on their own."""
    B, Hkv, page, budget = case["B"], case["Hkv"], case["page"], case["budget"]
    kc, vc, w = (st[x].double() for x in ("kc", "vc", "w"))
    kept = torch.full((B, Hkv, min(budget, case["L"])), -1, dtype=torch.int32, device="cuda")
    left = torch.zeros(B, dtype=torch.int32, device="cuda")
    for b, n in enumerate(_lengths(case).tolist()):
        left[b] = min(n, budget)
        j = torch.arange(n, device="cuda")
        pages, offs = st["table"][b].long()[j // page], j % page
        i = torch.arange(min(n, budget), device="cuda")
        to = st["to"][b].long()[i // page], i % page
        for h in range(Hkv if n else 0):
            middle = j[case["first"]:max(case["first"], n - case["recent"])]
            order = torch.argsort(-w[pages, h, offs][middle], stable=True)
            room = max(0, min(n, budget) - (n - middle.numel()))
            chosen = torch.ones(n, dtype=torch.bool, device="cuda")
            chosen[middle[order[room:]]] = False
            keep = j[chosen]
            kept[b, h, :keep.numel()] = keep.int()
            for x in (kc, vc, w):
                x[to[0], h, to[1]] = x[pages[keep], h, offs[keep]]
    return kc, vc, w, kept, left


def _exact_turn(case, x, positions, inverse):
    """x [B, H, T, d] in 64 bits: each pair times e^(i angle), as complex numbers."""
    owner, _ = _pair_axes(case)
    R = 2 * len(owner)
    pos = torch.stack([positions[a] for a in owner], -1).double()[:, None]
    angle = pos * _frequencies(case, x.device)
    turn = torch.polar(torch.ones_like(angle), -angle if inverse else angle)
    y = x.clone()
    first, second = ((slice(0, R, 2), slice(1, R, 2)) if case["interleaved"]
                     else (slice(0, R // 2), slice(R // 2, R)))
    z = torch.complex(x[..., first], x[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_append(case, st):
    page = case["page"]
    q, k = (_exact_turn(case, st[x].double(), st["positions"], False) for x in ("q", "k"))
    v, kc, vc = st["v"].double(), st["kc"].double(), st["vc"].double()
    for b, n in enumerate(_counts(case).tolist()):
        q[b, :, n:] = 0.0
        place = int(_starts(case)[b]) + torch.arange(n, device="cuda")
        pages, offs = st["table"][b].long()[place // page], place % page
        kc[pages, :, offs] = k[b, :, :n].transpose(0, 1)
        vc[pages, :, offs] = v[b, :, :n].transpose(0, 1)
    return q, kc, vc


def exact(case, seed):
    """What `run` returns, in 64 bits."""
    st = _inputs(case, seed)
    op = case["op"]
    if op == "axes":
        return tuple(_exact_turn(case, st[x].double(), st["positions"], case["inverse"]) for x in ("q", "k"))
    return {"chunk": _exact_chunk, "weigh": _exact_weigh, "evict": _exact_evict,
            "append": _exact_append}[op](case, st)
