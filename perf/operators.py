"""The measured operators of a layer's training and serving around the masked
attention, over the range of masks, sizes and types they are used on.

``train``   sparse_mhsa_fwd_lse and sparse_mhsa_bwd: one training pass through
            the attention; returns O, the rows' log-sum-exp, dQ, dK and dV
``rotary``  rotary: the position rotation of a layer's Q and K (or, `inverse`,
            of their gradients)
``append``  cache_append: a step's K and V rotated into a paged cache, Q rotated
            beside them; returns Q and both caches
``decode``  sparse_mhsa_decode: one query token a sequence, the mask's row of its
            position over the paged cache

Values are N(0, 1), which with scale = 1/sqrt(d) gives scores of standard
deviation 1, as attention inputs after a normalisation layer have.
"""
import math

import torch

own = False

_PARAMS = {"window": ("w",), "blocked": ("block",), "strided_local": ("local", "stride"),
           "dilated": ("w", "dilation"), "window_global": ("w", "n_global"), "full": (),
           "window_rows": ("w", "row_lo", "row_hi")}
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _train(kind, B, H, L, d, dtype, **params):
    return dict(op="train", kind=kind, B=B, H=H, L=L, d=d, dtype=dtype, **params)


def _rotary(B, H, Hkv, L, d, dtype, rot_dim, interleaved, inverse, max_len, positions, factor, lo=0.0,
            hi=0.0, original=0):
    return dict(op="rotary", B=B, H=H, Hkv=Hkv, L=L, d=d, dtype=dtype, rot_dim=rot_dim,
                interleaved=interleaved, inverse=inverse, max_len=max_len, positions=positions,
                factor=factor, lo=lo, hi=hi, original=original)


def _append(B, H, Hkv, T, d, dtype, page, max_len, rot_dim, interleaved):
    return dict(op="append", B=B, H=H, Hkv=Hkv, T=T, d=d, dtype=dtype, page=page, max_len=max_len,
                rot_dim=rot_dim, interleaved=interleaved)


def _decode(kind, B, H, Hkv, L, d, dtype, page, shortest, **params):
    return dict(op="decode", kind=kind, B=B, H=H, Hkv=Hkv, L=L, d=d, dtype=dtype, page=page,
                shortest=shortest, **params)


def listed():
    return [
        # the smallest training call: one head of a short sequence in fp32, a
        # unit of a small model; launches and latency are all of it
        dict(_train("window", 1, 1, 256, 64, "f32", w=16), name="train_window16_L256_f32"),
        # an ordinary encoder layer with block-local attention, short sequence
        dict(_train("blocked", 2, 8, 1024, 64, "bf16", block=64), name="train_blocked64_L1024_bf16"),
        # causal strided + local mask (sparse-transformer decoder)
        dict(_train("strided_local", 2, 12, 2048, 64, "bf16", local=128, stride=128),
             name="train_strided128_L2048_bf16"),
        # wide heads, dilated window, long sequence
        dict(_train("dilated", 1, 16, 4096, 128, "bf16", w=256, dilation=2),
             name="train_dilated2_L4096_d128_bf16"),
        # window + global tokens (long-document encoder), a batch of long sequences
        dict(_train("window_global", 4, 16, 4096, 64, "bf16", w=512, n_global=64),
             name="train_window512_global64_L4096_bf16"),
        # a long-document layer held in fp32 throughout
        dict(_train("window_global", 1, 12, 2048, 64, "f32", w=256, n_global=32),
             name="train_window256_global32_L2048_f32"),
        # Q and K of a training batch straight from their projections
        dict(_rotary(4, 16, 16, 4096, 64, "bf16", 64, False, False, 4096, False, 1.0),
             name="rotary_half_L4096_bf16"),
        # the gradients of a ragged layer: wide heads, half of them rotated, far
        # positions, scaled by parts
        dict(_rotary(2, 12, 4, 1000, 128, "f32", 64, True, True, 65536, True, 8.0, 1.0, 4.0, 8192),
             name="rotary_interleaved64_inverse_L1000_d128_f32"),
        # a ragged prefill of several sequences into the cache
        dict(_append(8, 32, 8, 1000, 128, "bf16", 64, 8192, 128, False), name="append_T1000_d128_bf16"),
        # one token a sequence of a running batch; launch and latency
        dict(_append(32, 16, 16, 1, 64, "bf16", 16, 4096, 64, False), name="append_T1_bf16"),
        # the answer to one user: one sequence, a row of the window + global mask
        dict(_decode("window_global", 1, 16, 16, 4096, 64, "bf16", 16, 4000, w=512, n_global=64),
             name="decode_window512_global64_B1_bf16"),
        # a running batch of long sequences over shared heads, every earlier key
        dict(_decode("full", 32, 32, 8, 8192, 128, "bf16", 64, 1000), name="decode_full_B32_d128_bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_mask(rng, L):
    kind = rng.choice(["window", "blocked", "strided_local", "dilated", "window_global",
                       "window_global", "full", "window_rows"])
    if kind == "full" and L > 2048:
        kind = "window_global"
    p = {}
    if kind == "window":
        p = dict(w=_log_int(rng, 2, 1024))
    elif kind == "blocked":
        p = dict(block=_log_int(rng, 8, 512))
    elif kind == "strided_local":
        p = dict(local=_log_int(rng, 4, 256), stride=_log_int(rng, 16, 512))
    elif kind == "dilated":
        p = dict(w=_log_int(rng, 8, 256), dilation=rng.randint(2, 4))
    elif kind == "window_global":
        p = dict(w=_log_int(rng, 8, 512), n_global=_log_int(rng, 1, 128))
    elif kind == "window_rows":      # the rows outside have no key
        lo = rng.randint(0, L // 3)
        p = dict(w=_log_int(rng, 2, 512), row_lo=lo, row_hi=rng.randint((lo + L + 1) // 2, L))
    return kind, p


def draw(rng):
    """A case of the ranges above: any operator, mask family, dtype and head
    width, lengths from 1 on, bounded by the largest listed cases."""
    op = rng.choice(["train", "train", "train", "train", "rotary", "append", "decode", "decode"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32", "f32"])
    d = rng.choice([64, 64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12, 16])
    H = Hkv * rng.choice([1, 1, 2, 4, 8])
    inter = rng.random() < 0.5
    rot_dim = rng.choice([x for x in (16, 32, 64, 96, 128) if x <= d])
    if op == "train":
        L = _log_int(rng, 1, 4352)
        B = rng.randint(1, 4)
        kind, p = _draw_mask(rng, L)
        case = _train(kind, B, Hkv, L, d, dtype, **p)
        nnz = _nnz(case)
        most = (6.0e9 if dtype == "f32" else 7.0e10) / (4.0 * d * max(1, nnz))
        room = min(most, 64 * (4096 / L) ** 2, 64)
        while case["B"] * case["H"] > max(1, room):
            if case["B"] > 1:
                case["B"] -= 1
            else:
                case["H"] = max(1, case["H"] // 2)
        return case
    if op == "rotary":
        L = _log_int(rng, 1, 4352)
        B = max(1, min(rng.randint(1, 8), (1 << 25) // (L * (H + Hkv) * d)))
        far = rng.random() < 0.5
        parts = rng.random() < 0.5
        return _rotary(B, H, Hkv, L, d, dtype, rot_dim, inter, rng.random() < 0.5, 65536 if far else 4352,
                       far, rng.choice([1.0, 2.0, 8.0]), 1.0 if parts else 0.0, 4.0 if parts else 0.0,
                       8192 if parts else 0)
    if op == "append":
        T = _log_int(rng, 1, 1500)
        B = max(1, min(_log_int(rng, 1, 48), 8192 // T, (1 << 25) // (T * (H + 2 * Hkv) * d)))
        return _append(B, H, Hkv, T, d, dtype, rng.choice([1, 8, 16, 64, 256]), 4096, rot_dim, inter)
    L = _log_int(rng, 64, 16384)
    kind, p = _draw_mask(rng, L)
    if kind == "window_rows":       # the longest sequence's row has keys
        p["row_hi"] = L
    B = max(1, min(_log_int(rng, 1, 48), (1 << 27) // (L * Hkv * d)))
    return _decode(kind, B, H, Hkv, L, d, dtype, rng.choice([1, 8, 16, 64, 256]),
                   rng.choice([0, 1, L // 2, L]), **p)


# ---- masks, lengths, positions: what the case says, on any device
def _mask_rows(case, i):
    """[len(i), L]: the mask's rows i, from the pattern's definition."""
    L, kind = case["L"], case["kind"]
    i, j = i[:, None], torch.arange(L, device=i.device)[None, :]
    if kind == "window":
        return (i - j).abs() <= case["w"]
    if kind == "blocked":
        bi, bj = i // case["block"], j // case["block"]
        return (bi == bj) | (bj == bi - 1)
    if kind == "strided_local":
        s = case["stride"]
        return ((j > i - case["local"]) | (j % s == s - 1)) & (j <= i)
    if kind == "dilated":
        g = case["dilation"]
        return ((j - i) % g == 0) & ((j - i).abs() <= g * case["w"])
    if kind == "window_global":
        G = case["n_global"]
        return ((i - j).abs() <= case["w"]) | (i < G) | (j < G)
    if kind == "window_rows":
        return ((i - j).abs() <= case["w"]) & (i >= case["row_lo"]) & (i < case["row_hi"])
    return (i >= 0) & (j >= 0)


def _nnz(case):
    """Non-zeros per head."""
    return int(_mask_rows(case, torch.arange(case["L"])).sum())


def _lengths(case):
    """A decode batch's lengths, from `shortest` to L."""
    B, lo, hi = case["B"], case["shortest"], case["L"]
    return torch.tensor([hi if b == 0 else lo + (hi - lo) * (B - 1 - b) // max(1, B - 1)
                         for b in range(B)])


def _keys(case):
    """Keys that a decode batch reads: the rows' columns below the lengths."""
    n = _lengths(case)
    m = _mask_rows(case, (n - 1).clamp(min=0)) & (torch.arange(case["L"])[None, :] < n[:, None])
    return int(m.sum())


def _counts(case):
    """Tokens that an append adds to each sequence: ragged where T > 1."""
    B, T = case["B"], case["T"]
    return torch.tensor([T - (b * T) // (2 * B) for b in range(B)])


def _starts(case):
    B, room = case["B"], case["max_len"] - case["T"]
    return torch.tensor([(room * b) // B for b in range(B)])


def _table(lengths, page, max_pages, g):
    """A shuffled page table: (table [B, max_pages], -1 where unused; pages)."""
    need = [-(-int(n) // page) for n in lengths]
    order = torch.randperm(sum(need) + 3, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(need), max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order.numel()


def _frequencies(case, device):
    """Angle per position of each pair, 64 bits."""
    R = case["rot_dim"]
    f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device=device) / R)
    factor, lo, hi = case.get("factor", 1.0), case.get("lo", 0.0), case.get("hi", 0.0)
    if hi > lo:      # pairs that turn often in the original length keep their frequency
        keep = ((case["original"] * f / (2 * math.pi) - lo) / (hi - lo)).clamp(0, 1)
        return f * keep + f / factor * (1 - keep)
    return f / factor


def _rotary_of(case, splat):
    kw = {}
    if case.get("hi", 0.0) > case.get("lo", 0.0):
        kw = dict(ramp=(case["lo"], case["hi"]), original_len=case["original"])
    return splat.Rotary(case["max_len"], case["rot_dim"], interleaved=case["interleaved"],
                        factor=case.get("factor", 1.0), **kw)


def _acsr_of(case, splat, grad):
    p = {k: case[k] for k in _PARAMS[case["kind"]]}
    if case["kind"] == "window_rows":
        pat = splat.Pattern.from_terms(case["L"], [dict(row_lo=p["row_lo"], row_hi=p["row_hi"], lo_i=1,
                                                        lo_c=-p["w"], hi_i=1, hi_c=p["w"])])
    else:
        pat = splat.Pattern.named(case["kind"], p, case["L"])
    return splat.Acsr(pat, grad=grad)


# ---- inputs
def _randn(shape, dtype, g):
    return torch.randn(shape, generator=g, device="cuda").to(_DTYPES[dtype])


def _inputs(case, seed):
    g = torch.Generator("cuda").manual_seed(int(seed))
    dt, d, op = case["dtype"], case["d"], case["op"]
    st = dict(case=case, scale=1.0 / math.sqrt(d))
    if op == "train":
        shape = (case["B"], case["H"], case["L"], d)
        st.update(zip(("q", "k", "v", "do"), [_randn(shape, dt, g) for _ in range(4)]))
    elif op == "rotary":
        # [B, L, H, d], as a projection leaves them, seen as [B, H, L, d]
        B, L = case["B"], case["L"]
        st["q"] = _randn((B, L, case["H"], d), dt, g).transpose(1, 2)
        st["k"] = _randn((B, L, case["Hkv"], d), dt, g).transpose(1, 2)
        st["positions"] = (torch.randint(0, case["max_len"], (B, L), generator=g, device="cuda",
                                         dtype=torch.int32) if case["positions"] else None)
    elif op == "append":
        B, T, page = case["B"], case["T"], case["page"]
        st["q"] = _randn((B, T, case["H"], d), dt, g).transpose(1, 2)
        st["k"] = _randn((B, T, case["Hkv"], d), dt, g).transpose(1, 2)
        st["v"] = _randn((B, T, case["Hkv"], d), dt, g).transpose(1, 2)
        start, count = _starts(case), _counts(case)
        st["table"], pages = _table(start + count, page, -(-case["max_len"] // page), g)
        st["kc"] = _randn((pages, case["Hkv"], page, d), dt, g)
        st["vc"] = _randn((pages, case["Hkv"], page, d), dt, g)
        st["start"], st["count"] = start.int().cuda(), count.int().cuda()
    else:
        page, lengths = case["page"], _lengths(case)
        st["q"] = _randn((case["B"], case["H"], 1, d), dt, g)
        st["table"], pages = _table(lengths, page, -(-case["L"] // page), g)
        st["kc"] = _randn((pages, case["Hkv"], page, d), dt, g)
        st["vc"] = _randn((pages, case["Hkv"], page, d), dt, g)
        st["lengths"] = lengths.int().cuda()
    return st


def prepare(case, seed):
    """A layer's inputs, and what a program keeps from call to call: the mask's
    and the rotation's handles; for the plain form the mask, the angles' cosines
    and sines and the places of the new tokens."""
    st = _inputs(case, seed)
    op = case["op"]
    if own:
        import paper_2407_16847_amd as splat
        if op in ("train", "decode"):
            st["acsr"] = _acsr_of(case, splat, op == "train")
        else:
            st["rot"] = _rotary_of(case, splat)
        return st
    if op == "train":
        st["mask"] = _mask_rows(case, torch.arange(case["L"], device="cuda"))
    elif op == "decode":
        n = st["lengths"].long()
        st["mask"] = (_mask_rows(case, (n - 1).clamp(min=0))
                      & (torch.arange(case["L"], device="cuda")[None, :] < n[:, None]))
    else:
        a = (torch.arange(case["max_len"], device="cuda", dtype=torch.float64)[:, None]
             * _frequencies(case, "cuda")[None, :])
        st["cos"], st["sin"] = a.cos().float(), a.sin().float()
        if op == "append":
            t = torch.arange(case["T"], device="cuda")[None, :]
            b, t = (t < st["count"][:, None]).nonzero(as_tuple=True)
            st["b"], st["t"], st["pos"] = b, t, st["start"].long()[b] + t
    return st


# ---- the plain forms
def _rotate(x, cos, sin, R, interleaved, inverse):
    """x [.., d] in 32 bits, cos and sin [.., R/2] broadcast against it."""
    sin = -sin if inverse else sin
    r, rest = x[..., :R], x[..., R:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :R // 2], r[..., R // 2:])
    u, v = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((y, rest), -1)


def _plain_train(st):
    q, k, v, do = (st[x].float() for x in ("q", "k", "v", "do"))
    dt, scale = st["q"].dtype, st["scale"]
    s = (q @ k.transpose(-1, -2) * scale).masked_fill_(~st["mask"], -math.inf)
    m = s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p = (s - m).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (m + total.log()).squeeze(-1)
    p /= total.clamp(min=torch.finfo(torch.float32).tiny)
    o = p @ v
    dv = p.transpose(-1, -2) @ do
    dp = do @ v.transpose(-1, -2)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
    return o.to(dt), lse, (ds @ k).to(dt), (ds.transpose(-1, -2) @ q).to(dt), dv.to(dt)


def _plain_rotary(st):
    c = st["case"]
    if st["positions"] is None:
        cos, sin = st["cos"][: c["L"]][None, None], st["sin"][: c["L"]][None, None]
    else:
        at = st["positions"].long()
        cos, sin = st["cos"][at][:, None], st["sin"][at][:, None]
    return tuple(_rotate(x.float(), cos, sin, c["rot_dim"], c["interleaved"], c["inverse"]).to(x.dtype)
                 for x in (st["q"], st["k"]))


def _plain_append(st):
    c, b, t, pos = st["case"], st["b"], st["t"], st["pos"]
    dt = st["q"].dtype
    at = st["start"].long()[:, None] + torch.arange(c["T"], device="cuda")[None, :]
    cos, sin = st["cos"][at][:, None], st["sin"][at][:, None]
    q, k = (_rotate(x.float(), cos, sin, c["rot_dim"], c["interleaved"], False).to(dt)
            for x in (st["q"], st["k"]))
    pages, offs = st["table"].long()[b, pos // c["page"]], pos % c["page"]
    st["kc"][pages, :, offs] = k[b, :, t]
    st["vc"][pages, :, offs] = st["v"][b, :, t]
    fresh = torch.arange(c["T"], device="cuda")[None, :] < st["count"][:, None]
    return q * fresh[:, None, :, None], st["kc"], st["vc"]


def _plain_decode(st):
    c = st["case"]
    B, H, Hkv, L, d = (c[x] for x in ("B", "H", "Hkv", "L", "d"))
    table = st["table"].long().clamp(min=0)
    k, v = (x[table].transpose(1, 2).reshape(B, Hkv, -1, d)[:, :, :L].float() for x in (st["kc"], st["vc"]))
    q = st["q"].float().view(B, Hkv, H // Hkv, d)
    s = (q @ k.transpose(-1, -2) * st["scale"]).masked_fill_(~st["mask"][:, None, None], -math.inf)
    p = (s - s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)).exp_()
    p /= p.sum(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).tiny)
    return (p @ v).view(B, H, 1, d).to(st["q"].dtype)


def run(st):
    op = st["case"]["op"]
    if not own:
        return {"train": _plain_train, "rotary": _plain_rotary, "append": _plain_append,
                "decode": _plain_decode}[op](st)
    import paper_2407_16847_amd as splat
    if op == "train":
        a, q, k, v, scale = (st[x] for x in ("acsr", "q", "k", "v", "scale"))
        o, lse = splat.sparse_mhsa_fwd_lse(a, q, k, v, scale)
        return (o, lse, *splat.sparse_mhsa_bwd(a, q, k, v, o, lse, st["do"], scale))
    if op == "rotary":
        return splat.rotary(st["rot"], st["q"], st["k"], positions=st["positions"],
                            inverse=st["case"]["inverse"])
    if op == "append":
        q = splat.cache_append(st["kc"], st["vc"], st["table"], st["start"], st["k"], st["v"],
                               counts=st["count"], rot=st["rot"], Q=st["q"])
        return q, st["kc"], st["vc"]
    return splat.sparse_mhsa_decode(st["acsr"], st["q"], st["kc"], st["vc"], st["table"], st["lengths"],
                                    st["scale"])


def work(case):
    """Each input read once and each output written once.  train: five products
    of 2 d flops a non-zero in the backward pass and two in the forward.
    decode: K and V of the keys of each sequence's row."""
    e, d, op = _BYTES[case["dtype"]], case["d"], case["op"]
    if op == "train":
        heads, nnz = case["B"] * case["H"], _nnz(case)
        dense = heads * case["L"] * d
        # Q, K, V, dO in; O, dQ, dK, dV out; the log-sum-exp
        return {"bytes": dense * 8 * e + 4 * heads * case["L"], "flops": 14.0 * nnz * heads * d}
    if op == "rotary":
        n = case["B"] * case["L"] * (case["H"] + case["Hkv"])
        angles = (case["B"] if case["positions"] else 1) * case["L"] * case["rot_dim"] // 2 * 8
        return {"bytes": 2 * n * d * e + angles, "flops": 3.0 * n * case["rot_dim"]}
    if op == "append":
        n = int(_counts(case).sum())
        heads = case["H"] + 2 * case["Hkv"]
        return {"bytes": 2 * n * heads * d * e + n * case["rot_dim"] // 2 * 8,
                "flops": 3.0 * n * (case["H"] + case["Hkv"]) * case["rot_dim"]}
    keys = _keys(case)
    return {"bytes": 2 * keys * case["Hkv"] * d * e + 2 * case["B"] * case["H"] * d * e,
            "flops": 4.0 * keys * case["H"] * d}


# ---- from the definitions, in 64 bits
def _exact_rotate(case, x, pos, inverse):
    """x [B, H, T, d] in 64 bits at positions pos [B, T]: each pair times
    e^(i angle), as complex numbers."""
    R = case["rot_dim"]
    angle = pos.double()[:, None, :, None] * _frequencies(case, x.device)
    turn = torch.polar(torch.ones_like(angle), -angle if inverse else angle)
    y = x.clone()
    first, second = ((slice(0, R, 2), slice(1, R, 2)) if case["interleaved"]
                     else (slice(0, R // 2), slice(R // 2, R)))
    z = torch.complex(x[..., first], x[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_train(case, st):
    scale, outs = st["scale"], []
    mask = _mask_rows(case, torch.arange(case["L"], device="cuda"))
    some = mask.any(-1)
    for b in range(case["B"]):
        for h in range(case["H"]):
            q, k, v, do = (st[x][b, h].double() for x in ("q", "k", "v", "do"))
            s = ((q @ k.t()) * scale).masked_fill(~mask, -math.inf)
            lse = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1).masked_fill(~some[:, None], 0.0)
            g = do @ v.t()
            ds = p * (g - (p * g).sum(-1, keepdim=True))
            outs.append((p @ v, lse, scale * (ds @ k), scale * (ds.t() @ q), p.t() @ do))
    return tuple(torch.stack(x).unflatten(0, (case["B"], case["H"])) for x in zip(*outs))


def _exact_append(case, st):
    page = case["page"]
    pos = st["start"].long()[:, None] + torch.arange(case["T"], device="cuda")
    q, k = (_exact_rotate(case, st[x].double(), pos, False) for x in ("q", "k"))
    v, kc, vc = st["v"].double(), st["kc"].double(), st["vc"].double()
    for b, n in enumerate(st["count"].tolist()):
        q[b, :, n:] = 0.0
        pages, offs = st["table"][b].long()[pos[b, :n] // page], pos[b, :n] % page
        kc[pages, :, offs] = k[b, :, :n].transpose(0, 1)
        vc[pages, :, offs] = v[b, :, :n].transpose(0, 1)
    return q, kc, vc


def _exact_decode(case, st):
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    G = case["H"] // case["Hkv"]
    for b, n in enumerate(st["lengths"].tolist()):
        if n == 0:
            continue
        cols = _mask_rows(case, torch.tensor([n - 1], device="cuda"))[0, :n].nonzero()[:, 0]
        if cols.numel() == 0:
            continue
        pages, offs = st["table"][b].long()[cols // case["page"]], cols % case["page"]
        k, v = (st[x][pages, :, offs].double().transpose(0, 1).repeat_interleave(G, 0) for x in ("kc", "vc"))
        s = (k @ st["q"][b, :, 0].double()[:, :, None])[:, :, 0] * st["scale"]
        o[b, :, 0] = (torch.softmax(s, -1)[:, None, :] @ v)[:, 0]
    return o


def exact(case, seed):
    """What `run` returns, in 64 bits."""
    st = _inputs(case, seed)
    if case["op"] == "train":
        return _exact_train(case, st)
    if case["op"] == "rotary":
        pos = st["positions"]
        if pos is None:
            pos = torch.arange(case["L"], device="cuda").expand(case["B"], -1)
        return tuple(_exact_rotate(case, st[x].double(), pos, case["inverse"]) for x in ("q", "k"))
    if case["op"] == "append":
        return _exact_append(case, st)
    return _exact_decode(case, st)
