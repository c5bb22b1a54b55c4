"""The attention half of a served layer over a cache held in 4 bits, as cases that can be timed and compared.

  rotate   norms of queries and keys for each head, and the position rotation, in one pass (tempo_qk_rotate)
  append   the same for a batch whose keys and values go into the paged 4-bit cache, and the appended rows read back
           (tempo_kv_append, tempo_kv_read)
  attend   attention over the paged cache: one query token per sequence, a few (drafted tokens) or a prompt's chunk
           (tempo_attend)

A cached group of 32 elements is 4-bit codes c, a scale s of four significant bits and a zero point z: value s * (c - z).
Where `own` is false, run() computes the plain form with elementary torch operations."""
import torch

own = False

EPS = 1e-6
DEV = "cuda"
GROUP = 32


# ---- cases --------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token of one sequence: latency
        dict(name="rotate 1 x 64+4", op="rotate", T=1, Hq=64, Hkv=4, D=128, rot=128, pairs="half", norm=True),
        # a ragged batch of narrow heads of which a part is rotated, neighbouring elements as pairs, no norm
        dict(name="rotate 333 x 12+2 part", op="rotate", T=333, Hq=12, Hkv=2, D=64, rot=32, pairs="next", norm=False),
        # a prompt
        dict(name="rotate 8192 x 64+4", op="rotate", T=8192, Hq=64, Hkv=4, D=128, rot=128, pairs="half", norm=True),
        # a small decode batch: latency
        dict(name="append 7 x 32+8", op="append", T=7, Hq=32, Hkv=8, D=128, rot=128, pairs="half", norm=True, page=64),
        # a prompt's chunk into small pages, narrow heads without a norm
        dict(name="append 701 x 14+2 narrow", op="append", T=701, Hq=14, Hkv=2, D=64, rot=64, pairs="half", norm=False, page=16),
        # a long prompt
        dict(name="append 4096 x 64+4", op="append", T=4096, Hq=64, Hkv=4, D=128, rot=128, pairs="half", norm=True, page=64),
        # one sequence being decoded: latency
        dict(name="attend 1 x 1500", op="attend", B=1, L=1500, n=1, Hq=64, Hkv=4, D=128, page=64),
        # a decode batch of ragged lengths
        dict(name="attend 64 x 8192", op="attend", B=64, L=8192, n=1, Hq=64, Hkv=4, D=128, page=64),
        # two very long sequences
        dict(name="attend 2 x 131072", op="attend", B=2, L=131072, n=1, Hq=32, Hkv=8, D=128, page=128),
        # narrow heads, a key head for each query head, small pages
        dict(name="attend 37 x 2999 narrow", op="attend", B=37, L=2999, n=1, Hq=8, Hkv=8, D=64, page=16),
        # drafted tokens being verified
        dict(name="attend 16 x 4096 draft", op="attend", B=16, L=4096, n=4, Hq=32, Hkv=8, D=128, page=64),
        # the last chunk of two prompts
        dict(name="attend 2 x 6144 prompt", op="attend", B=2, L=6144, n=2048, Hq=64, Hkv=4, D=128, page=64),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(("rotate", "append", "attend", "attend"))
    while True:
        Hkv = rng.choice((1, 2, 3, 4, 8))
        c = dict(op=op, Hq=Hkv * rng.choice((1, 2, 3, 4, 6, 7, 8, 16)), Hkv=Hkv, D=rng.choice((64, 128)))
        if op == "rotate":
            c.update(T=_log(rng, 1, 8192), D=8 * rng.randint(4, 32))
        elif op == "append":
            c.update(T=_log(rng, 1, 4096), page=rng.choice((16, 32, 64, 128)))
        if op != "attend":
            c["rot"] = c["D"] if rng.random() < 0.6 else 2 * rng.randint(4, c["D"] // 2)
            c["pairs"] = rng.choice(("half", "next"))
            c["norm"] = rng.random() < 0.6
            if c["T"] * (c["Hq"] + 2 * Hkv) * c["D"] <= 8192 * 72 * 128:
                return c
            continue
        c.update(B=_log(rng, 1, 64), L=_log(rng, 1, 131072), page=rng.choice((16, 32, 64, 128)))
        kind = rng.choice(("one", "one", "few", "many"))
        c["n"] = min(c["L"], {"one": 1, "few": rng.randint(2, 9), "many": _log(rng, 16, 2048)}[kind])
        if c["B"] * c["L"] * Hkv * c["D"] <= 64 * 8192 * 4 * 128 and c["B"] * c["n"] * c["Hq"] * c["L"] <= 2 ** 30:
            return c


def _lengths(case):
    """Tokens in the cache and new query tokens of each sequence: the longest first, the shortest a quarter (a half)."""
    B = case["B"]
    return ([max(1, case["L"] - 3 * case["L"] * b // (4 * B)) for b in range(B)],
            [max(1, case["n"] - case["n"] * b // (2 * B)) if case["n"] > 16 else case["n"] for b in range(B)])


def _spans(case):
    """(length, queries) of each sequence; a sequence has no more queries than tokens."""
    return [(l, min(l, n)) for l, n in zip(*_lengths(case))]


# ---- inputs -------------------------------------------------------------------------------------------------------

def _heads(g, T, H, D):
    """Keys or queries as a projection gives them: a few loud channels, tokens of unlike size."""
    loud = torch.where(torch.rand(H, D, generator=g, device=DEV) < 0.02, 5.0, 1.0)
    size = 0.5 + torch.rand(T, 1, 1, generator=g, device=DEV)
    return torch.randn(T, H, D, generator=g, device=DEV).mul_(loud).mul_(size)


def _table(case, g):
    """cos and sin of every position's angles, and this batch's positions (one run of a longer sequence)."""
    half = case["rot"] // 2
    n_pos = 32768
    freq = 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    ang = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * freq
    first = int(torch.randint(0, n_pos - case["T"], (1,), generator=g, device=DEV))
    pos = torch.arange(first, first + case["T"], device=DEV, dtype=torch.int32)
    return torch.cat([torch.cos(ang), torch.sin(ang)], dim=1).float(), pos


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if case["op"] == "attend":
        return _prepare_attend(case, g, s)
    T = case["T"]
    # one row of queries, keys and values for each token, as one projection writes it
    qkv = torch.cat([_heads(g, T, Hq, D), _heads(g, T, Hkv, D), torch.randn(T, Hkv, D, generator=g, device=DEV)], 1)
    s["q"], s["k"], s["v"] = qkv.to(torch.bfloat16).split([Hq, Hkv, Hkv], dim=1)
    for w in ("q_w", "k_w"):
        s[w] = (1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16) if case["norm"] else None
    s["cos_sin"], s["positions"] = _table(case, g)
    s["q_out"] = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV)
    if case["op"] == "rotate":
        s["k_out"] = torch.zeros(T, Hkv, D, dtype=torch.bfloat16, device=DEV)
        return s
    n_pages = (T + case["page"] - 1) // case["page"] + 3
    where = torch.randperm(n_pages, generator=g, device=DEV)
    t = torch.arange(T, device=DEV)
    s["slots"] = (where[t // case["page"]] * case["page"] + t % case["page"]).to(torch.int32)
    if own:
        from paper_2608_13057_b200 import binding as B
        s["shape"] = B.make_cache(n_pages, case["page"], Hkv, D)
        s["cache"] = torch.zeros(B.tempo_cache_bytes(s["shape"]), dtype=torch.uint8, device=DEV)
        s["k_back"] = torch.zeros(T, Hkv, D, dtype=torch.float16, device=DEV)
        s["v_back"] = torch.zeros(T, Hkv, D, dtype=torch.float16, device=DEV)
    return s


def _prepare_attend(case, g, s):
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    spans = _spans(case)
    per = [(l + page - 1) // page for l, _ in spans]
    n_pages = sum(per) + 3
    where = torch.randperm(n_pages, generator=g, device=DEV)
    s["page_table"] = torch.zeros(len(spans), max(per), dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(per):
        s["page_table"][b, :n] = where[at : at + n]
        at += n
    s["lens"] = torch.tensor([l for l, _ in spans], dtype=torch.int32, device=DEV)
    starts = [0]
    for _, n in spans:
        starts.append(starts[-1] + n)
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["max_q"] = max(n for _, n in spans)
    s["scale"] = D ** -0.5
    s["q"] = (1.5 * torch.randn(starts[-1], Hq, D, generator=g, device=DEV)).to(torch.bfloat16)
    s["out"] = torch.zeros(starts[-1], Hq, D, dtype=torch.bfloat16, device=DEV)
    # the cache, filled page by page with rotated keys and values
    k = _heads(g, n_pages * page, Hkv, D).to(torch.bfloat16)
    v = torch.randn(n_pages * page, Hkv, D, generator=g, device=DEV).to(torch.bfloat16)
    if own:
        from paper_2608_13057_b200 import binding as B
        s["shape"] = B.make_cache(n_pages, page, Hkv, D)
        s["cache"] = torch.zeros(B.tempo_cache_bytes(s["shape"]), dtype=torch.uint8, device=DEV)
        B.tempo_kv_append(s["shape"], k, v, torch.arange(n_pages * page, dtype=torch.int32, device=DEV), s["cache"], s["status"])
        s["workspace"] = torch.zeros(B.tempo_attend_workspace_bytes(s["shape"], Hq), dtype=torch.uint8, device=DEV)
    else:
        s["cached_k"], s["cached_v"] = _pack(*_quantise(k)), _pack(*_quantise(v))
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s["op"]](s)


def _own_rotate(s):
    from paper_2608_13057_b200 import binding as B
    B.tempo_qk_rotate(s["q"], s["k"], s["positions"], s["cos_sin"], s["q_out"], s["k_out"], s["status"], q_w=s["q_w"], k_w=s["k_w"],
                      eps=EPS, interleaved=s["pairs"] == "next")
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_append(s):
    from paper_2608_13057_b200 import binding as B
    B.tempo_kv_append(s["shape"], s["k"], s["v"], s["slots"], s["cache"], s["status"], k_w=s["k_w"], positions=s["positions"],
                      cos_sin=s["cos_sin"], q=s["q"], q_w=s["q_w"], q_out=s["q_out"], eps=EPS, interleaved=s["pairs"] == "next")
    B.tempo_kv_read(s["shape"], s["cache"], s["slots"], s["k_back"], s["v_back"], s["status"])
    return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}


def _own_attend(s):
    from paper_2608_13057_b200 import binding as B
    B.tempo_attend(s["shape"], s["q"], s["cache"], s["page_table"], s["lens"], s["out"], s["status"], s["workspace"],
                   scale=s["scale"], q_start=s["q_start"], max_q=s["max_q"])
    return {"out": s["out"]}


_own = {"rotate": _own_rotate, "append": _own_append, "attend": _own_attend}


def _rotated(s, x, w):
    """norm(x) * w for each head and the rotation, in x's type."""
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(dim=2, keepdim=True) + EPS) * w.to(x.dtype)
    rot, half = s["rot"], s["rot"] // 2
    cs = s["cos_sin"][s["positions"].long()].to(x.dtype)[:, None, :]
    cos, sin = cs[..., :half], cs[..., half:]
    turned = x.clone()
    a = slice(0, half) if s["pairs"] == "half" else slice(0, rot, 2)
    b = slice(half, rot) if s["pairs"] == "half" else slice(1, rot, 2)
    turned[..., a] = x[..., a] * cos - x[..., b] * sin
    turned[..., b] = x[..., b] * cos + x[..., a] * sin
    return turned


def _plain_rotate(s):
    return {"q": _rotated(s, s["q"].float(), s["q_w"]).to(torch.bfloat16), "k": _rotated(s, s["k"].float(), s["k_w"]).to(torch.bfloat16)}


def _quantise(x):
    """Codes, scales and zero points of groups of 32 neighbouring elements, in 64 bits: a value next to a border has one code."""
    x = x.double().unflatten(2, (-1, GROUP))
    low = x.amin(dim=3, keepdim=True).clamp_(max=0.0)
    step = (x.amax(dim=3, keepdim=True).clamp_(min=0.0) - low) / 15.0
    unit = torch.exp2((torch.frexp(step).exponent - 4).clamp(min=-17).double())      # four significant bits, rounded up
    scale = (torch.ceil(step / unit) * unit).clamp_(max=768.0)
    safe = torch.where(scale > 0.0, scale, 1.0)
    zero = torch.round(-low / safe).clamp_(max=15.0)
    codes = torch.clamp(torch.round(x / safe) + zero, 0.0, 15.0)
    return codes, scale, zero


def _values(codes, scale, zero):
    return (scale * (codes - zero)).flatten(2)


def _pack(codes, scale, zero):
    c = codes.to(torch.uint8).flatten(2)
    return c[..., 0::2] | (c[..., 1::2] << 4), scale.squeeze(3).to(torch.float16), zero.squeeze(3).to(torch.uint8)


def _plain_append(s):
    k = _rotated(s, s["k"].double(), s["k_w"])
    return {"q": _rotated(s, s["q"].float(), s["q_w"]).to(torch.bfloat16),
            "k": _values(*_quantise(k)).to(torch.float16), "v": _values(*_quantise(s["v"])).to(torch.float16)}


def _cached(packed, slot):
    """The cache's rows `slot` [B, L] as 32-bit values [B, heads, L, D]."""
    codes, scale, zero = (t[slot] for t in packed)
    c = torch.stack([codes & 15, codes >> 4], dim=4).flatten(3).unflatten(3, (-1, GROUP)).float()
    x = scale.float()[..., None] * (c - zero.float()[..., None])
    return x.flatten(3).transpose(1, 2)


def _plain_attend(s):
    B, page, Hkv, D, n = s["B"], s["page"], s["Hkv"], s["D"], s["max_q"]
    g = s["Hq"] // Hkv
    t = torch.arange(int(s["page_table"].shape[1]) * page, device=DEV)
    slot = s["page_table"].long()[:, t // page] * page + t % page                    # [B, L]
    k, v = _cached(s["cached_k"], slot), _cached(s["cached_v"], slot)
    first, lens = s["q_start"].long()[:-1], s["lens"].long()
    count = s["q_start"].long()[1:] - first
    i = torch.arange(n, device=DEV)
    at = (first[:, None] + i).clamp(max=s["q"].shape[0] - 1)                         # [B, n], rows of q
    q = s["q"][at].float().view(B, n, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * g, D)
    seen = t <= (lens[:, None] - count[:, None] + i)[:, :, None]                     # [B, n, L]
    seen = seen & (t < lens[:, None, None]) & (i < count[:, None])[:, :, None]
    p = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    p.masked_fill_(~seen.repeat_interleave(g, dim=1)[:, None], float("-inf"))
    top = p.amax(dim=3, keepdim=True)
    p = p.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0.0, total, 1.0)
    o = o.view(B, Hkv, n, g, D).permute(0, 2, 1, 3, 4).reshape(B, n, s["Hq"], D)
    return {"out": o[i < count[:, None]].to(torch.bfloat16)}


_plain = {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    row = D // 2 + D // 16                                                           # bytes of a cached row of one head
    if case["op"] == "attend":
        spans = _spans(case)
        pairs = sum(n * l - n * (n - 1) // 2 for l, n in spans)
        return {"bytes": sum(l for l, _ in spans) * Hkv * 2 * row + 4 * D * Hq * sum(n for _, n in spans),
                "flops": 4.0 * D * Hq * pairs}
    T = case["T"]
    table = T * (4 * case["rot"] + 4) + (4 * D if case["norm"] else 0)
    if case["op"] == "rotate":
        return {"bytes": T * (Hq + Hkv) * D * 4 + table, "flops": 8 * T * (Hq + Hkv) * D}
    # q turned, k and v into the cache and out of it again as 16-bit values
    return {"bytes": T * Hq * D * 4 + T * Hkv * 2 * (2 * D + row + row + 2 * D) + table + 4 * T, "flops": 8 * T * (Hq + 2 * Hkv) * D}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    return {"rotate": _exact_rotate, "append": _exact_append, "attend": _exact_attend}[case["op"]](s)


def _exact_turn(s, x, w):
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.pow(2).sum(2, keepdim=True) / x.shape[2] + EPS) * w.double()
    half = s["rot"] // 2
    cs = s["cos_sin"].double()[s["positions"].long()]
    unit = torch.complex(cs[:, :half], cs[:, half:])[:, None, :]
    part, rest = x[..., : s["rot"]], x[..., s["rot"] :]
    if s["pairs"] == "half":
        z = torch.complex(part[..., :half].contiguous(), part[..., half:].contiguous()) * unit
        return torch.cat([z.real, z.imag, rest], dim=2)
    z = torch.view_as_complex(part.unflatten(2, (half, 2)).contiguous()) * unit
    return torch.cat([torch.view_as_real(z).flatten(2), rest], dim=2)


def _exact_cache(x):
    """The values that a 4-bit group stands for, by a search over all scales that can be written."""
    m = torch.arange(8, 16, device=DEV, dtype=torch.float64)
    scales = torch.cat([torch.arange(0, 8, device=DEV, dtype=torch.float64) * 2.0 ** -17]
                       + [m * 2.0 ** e for e in range(-17, 7)])
    scales = scales[scales <= 768.0]
    x = x.double().reshape(x.shape[0], x.shape[1], -1, GROUP)
    low, high = x.amin(3).clamp(max=0.0), x.amax(3).clamp(min=0.0)
    at = torch.searchsorted(scales * 15.0, (high - low).contiguous()).clamp(max=scales.numel() - 1)   # first 15 s >= range
    s = scales[at][..., None]
    z = torch.where(s > 0, torch.round(-low[..., None] / s), 0.0).clamp(max=15.0)
    c = torch.where(s > 0, torch.round(x / s), 0.0) + z
    return (s * (c.clamp(0.0, 15.0) - z)).reshape(x.shape[0], x.shape[1], -1)


def _exact_rotate(s):
    return {"q": _exact_turn(s, s["q"], s["q_w"]), "k": _exact_turn(s, s["k"], s["k_w"])}


def _exact_append(s):
    return {"q": _exact_turn(s, s["q"], s["q_w"]), "k": _exact_cache(_exact_turn(s, s["k"], s["k_w"])), "v": _exact_cache(s["v"])}


def _exact_attend(s):
    Hkv, D, page = s["Hkv"], s["D"], s["page"]
    g = s["Hq"] // Hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)

    def row(packed, at, h):
        codes, scale, zero = (t[at, h] for t in packed)
        c = torch.empty(at.numel(), D, dtype=torch.float64, device=DEV)
        c[:, 0::2], c[:, 1::2] = (codes % 16).double(), (codes // 16).double()
        return scale.double().repeat_interleave(GROUP, 1) * (c - zero.double().repeat_interleave(GROUP, 1))

    for b, (length, count) in enumerate(_spans(s)):
        t = torch.arange(length, device=DEV)
        at = s["page_table"][b, t // page].long() * page + t % page
        q0 = int(s["q_start"][b])
        hidden = t[None, :] > (length - count + torch.arange(count, device=DEV))[:, None]
        for h in range(Hkv):
            k, v = row(s["cached_k"], at, h), row(s["cached_v"], at, h)
            q = s["q"][q0 : q0 + count, h * g : (h + 1) * g].double()
            for part in torch.arange(count, device=DEV).split(max(1, 2 ** 27 // (g * length))):
                logits = torch.einsum("ngd,ld->ngl", q[part], k) * s["scale"]
                p = torch.softmax(logits.masked_fill_(hidden[part][:, None], float("-inf")), dim=2)
                out[q0 + part, h * g : (h + 1) * g] = torch.einsum("ngl,ld->ngd", p, v)
    return {"out": out}
