"""The operators around and instead of the four-step expert block, as cases that can be timed and compared.

  norm    the norm before a block (tempo_norm_in), and the norm after it fused with the block's gate, its residual
          scale, the residual sum and the next block's norm (tempo_norm_out)
  route   the router: logits, scores, the k best experts of every token and their weights (tempo_route)
  layer   a whole mixture-of-experts layer for a few tokens: the router, then every chosen expert's SwiGLU FFN and the
          weighted sum over a token's experts in one kernel (tempo_route + tempo_few_ffn / tempo_few_ffn_bf16)

Where `own` is false, run() computes the plain form with elementary torch operations in 32 bits."""
import torch

own = False

EPS = 1e-6
DEV = "cuda"


# ---- cases --------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token of one sequence being decoded: the latency of the fused norm is what counts
        dict(name="norm out 1x4096", op="norm", side="out", T=1, d=4096, kind="rms", stream="bf16", gate="none", pad=0),
        # a decode batch with a 32-bit residual stream inside a wider buffer, a gate for each token, layer norms
        dict(name="norm out 203x4096 f32", op="norm", side="out", T=203, d=4096, kind="layer", stream="f32", gate="token", pad=64),
        # a width that no vector load divides
        dict(name="norm in 515x1021", op="norm", side="in", T=515, d=1021, kind="rms", stream="bf16", gate="none", pad=0),
        # a prefill batch of the widest block, a learned scale for each channel of the block's output
        dict(name="norm out 8192x7168", op="norm", side="out", T=8192, d=7168, kind="rms", stream="bf16", gate="channel", pad=0),
        # one token through the router: latency
        dict(name="route 1 of 128", op="route", T=1, E=128, k=8, d=4096, score="softmax", bias=False),
        # a ragged batch over a number of experts that is no power of two
        dict(name="route 333 of 60", op="route", T=333, E=60, k=4, d=2048, score="softmax", bias=False),
        # a prefill batch: many experts, sigmoid scores, a bias that steers the choice and not the weight
        dict(name="route 8192 of 256", op="route", T=8192, E=256, k=8, d=7168, score="sigmoid", bias=True),
        # a small layer: what the launches and the waits cost
        dict(name="layer 5 bf16 small", op="layer", T=5, E=8, local=8, k=2, d=256, f=512, weights="bf16"),
        # one token, every expert on this GPU
        dict(name="layer 1 of 128 fp8", op="layer", T=1, E=128, local=128, k=8, d=4096, f=1536, weights="fp8"),
        # a ragged batch through bf16 experts whose width is an odd number of 128-column blocks
        dict(name="layer 11 of 64 bf16", op="layer", T=11, E=64, local=64, k=6, d=2048, f=1408, weights="bf16"),
        # one of eight ranks, the largest few-token batch
        dict(name="layer 64 rank fp8", op="layer", T=64, E=128, local=16, k=8, d=4096, f=1536, weights="fp8"),
        # one of eight ranks of the widest experts
        dict(name="layer 24 rank fp8 wide", op="layer", T=24, E=256, local=32, k=8, d=7168, f=2048, weights="fp8"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(("norm", "route", "layer"))
    if op == "norm":
        d = _log(rng, 128, 7168)
        d = d if rng.random() < 0.25 else max(8, d // 8 * 8)
        return dict(op="norm", side=rng.choice(("in", "out")), T=_log(rng, 1, 8192), d=d, kind=rng.choice(("rms", "layer")),
                    stream=rng.choice(("bf16", "f32")) if d < 3500 else "bf16", gate=rng.choice(("none", "token", "channel")),
                    pad=rng.choice((0, 0, 8, 64, 3)))
    if op == "route":
        E = _log(rng, 4, 256)
        score = rng.choice(("softmax", "sigmoid"))          # a bias steers sigmoid scores
        return dict(op="route", T=_log(rng, 1, 8192), E=E, k=rng.randint(1, min(10, E)), d=128 * _log(rng, 2, 56),
                    score=score, bias=score == "sigmoid" and rng.random() < 0.5)
    while True:
        E = _log(rng, 4, 256)
        local = rng.choice((E, max(1, E // 2), max(1, E // 8)))
        c = dict(op="layer", T=_log(rng, 1, 64), E=E, local=local, k=rng.randint(1, min(8, E)), d=128 * _log(rng, 2, 56),
                 f=128 * _log(rng, 2, 16), weights=rng.choice(("fp8", "bf16")))
        one = 3 * c["d"] * c["f"] * (1 if c["weights"] == "fp8" else 2)
        if local * one <= 2.4e9 and _active(c) * one <= 7e8:
            return c


def _active(case):
    """Expected number of this rank's experts that at least one of the T tokens chooses (choices as good as uniform)."""
    return case["local"] * (1.0 - (1.0 - case["k"] / case["E"]) ** case["T"])


# ---- inputs -------------------------------------------------------------------------------------------------------

def _grid(g, shape, std, step, most):
    """Normal draws on a grid fine enough to keep their distribution and coarse enough that a dot product of two such
    vectors is exact in 32 bits in any order: equal logits on every path, so the chosen experts can be compared."""
    v = torch.randn(shape, generator=g, device=DEV) * std
    return (torch.round(v / step) * step).clamp_(-most, most).to(torch.bfloat16)


def _router_inputs(case, g):
    T, E, d = case["T"], case["E"], case["d"]
    s = dict(x=_grid(g, (T, d), 1.0, 2.0 ** -5, 7.96875), w_router=_grid(g, (E, d), 0.02, 2.0 ** -11, 255 * 2.0 ** -11))
    s["bias"] = torch.randn(E, generator=g, device=DEV) * 0.05 if case.get("bias") else None
    s["ids"] = torch.zeros(T, case["k"], dtype=torch.int32, device=DEV)
    s["w"] = torch.zeros(T, case["k"], dtype=torch.float32, device=DEV)
    s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def _fp8_matrix(g, n, k):
    """One expert's matrix: N(0, 0.02), e4m3 codes with a power-of-two scale for each 128x128 block."""
    w = torch.randn((n // 128, 128, k // 128, 128), generator=g, device=DEV).mul_(0.02)
    amax = w.abs().amax(dim=(1, 3))
    scale = torch.exp2(torch.ceil(torch.log2(amax / 448.0)))
    q = (w / scale[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).reshape(n, k), scale


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case)
    T, d = case["T"], case["d"]
    if case["op"] == "norm":
        dt = torch.float32 if case["stream"] == "f32" else torch.bfloat16
        pad = case["pad"]
        loud = torch.where(torch.rand(d, generator=g, device=DEV) < 0.01, 12.0, 1.5)   # a few loud channels
        s["r"] = (torch.randn(T, d + pad, generator=g, device=DEV)).mul_(torch.cat([loud, loud.new_ones(pad)])).to(dt)[:, :d]
        s["w"] = (1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
        s["b"] = (0.1 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) if case["kind"] == "layer" else None
        s["x"] = torch.zeros(T, d, dtype=torch.bfloat16, device=DEV)
        if case["side"] == "out":
            s["y"] = (0.5 * torch.randn(T, d, generator=g, device=DEV)).to(torch.bfloat16)
            s["post_w"] = (1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
            s["post_b"] = (0.1 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) if case["kind"] == "layer" else None
            s["gate"] = {"none": lambda: None,
                         "token": lambda: torch.sigmoid(torch.randn(T, 1, generator=g, device=DEV)),
                         "channel": lambda: 0.3 * torch.randn(1, d, generator=g, device=DEV)}[case["gate"]]()
            s["r_out"] = torch.zeros(T, d + pad, dtype=dt, device=DEV)[:, :d]
        return s
    s.update(_router_inputs(case, g))
    if case["op"] == "route":
        if own:
            s["shape"] = _shape(case)
        return s
    G, f = case["local"], case["f"]
    s["replica_map"] = torch.full((case["E"], 1), -1, dtype=torch.int32, device=DEV)
    s["replica_map"][:G, 0] = torch.arange(G, dtype=torch.int32, device=DEV)
    s["out"] = torch.zeros(T, d, dtype=torch.bfloat16, device=DEV)
    if case["weights"] == "fp8":
        s["w13"] = torch.empty(G, 2 * f, d, dtype=torch.uint8, device=DEV)
        s["s13"] = torch.empty(G, 2 * f // 128, d // 128, device=DEV)
        s["w2"] = torch.empty(G, d, f, dtype=torch.uint8, device=DEV)
        s["s2"] = torch.empty(G, d // 128, f // 128, device=DEV)
        for e in range(G):
            s["w13"][e], s["s13"][e] = _fp8_matrix(g, 2 * f, d)
            s["w2"][e], s["s2"][e] = _fp8_matrix(g, d, f)
    else:
        s["w13"] = torch.empty(G, 2 * f, d, dtype=torch.bfloat16, device=DEV)
        s["w2"] = torch.empty(G, d, f, dtype=torch.bfloat16, device=DEV)
        for e in range(G):
            s["w13"][e] = torch.randn(2 * f, d, generator=g, device=DEV) * 0.02
            s["w2"][e] = torch.randn(d, f, generator=g, device=DEV) * 0.02
    if own:
        # what a program that serves these weights keeps: the packed blob (laid out once, the same one that the four-step
        # block reads) and the workspace
        from paper_2608_13057_b200 import binding as B
        s["shape"] = _shape(case)
        if case["weights"] == "fp8":
            s["packed"] = torch.empty(B.tempo_packed_weight_bytes(s["shape"]), dtype=torch.uint8, device=DEV)
            B.tempo_pack_weights(s["shape"], s["w13"], s["s13"], s["w2"], s["s2"], s["packed"], s["status"])
        else:
            s["packed"] = torch.empty(B.tempo_packed_weight_bytes_bf16(s["shape"]), dtype=torch.uint8, device=DEV)
            B.tempo_pack_weights_bf16(s["shape"], s["w13"], s["w2"], s["packed"])
        s["workspace"] = torch.zeros(B.tempo_few_workspace_bytes(s["shape"]), dtype=torch.uint8, device=DEV)
    return s


def _shape(case):
    from paper_2608_13057_b200 import binding as B
    return B.make_shape(case["T"], case["k"], case["E"], case.get("local", 1), 1, case["d"], case.get("f", 128), 128)


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s["op"]](s)


def _own_norm(s):
    from paper_2608_13057_b200 import binding as B
    kind = B.NORM_LAYER if s["kind"] == "layer" else B.NORM_RMS
    if s["side"] == "in":
        B.tempo_norm_in(s["r"], s["w"], s["x"], b=s["b"], kind=kind, eps=EPS)
        return {"x": s["x"]}
    B.tempo_norm_out(s["y"], s["r"], s["r_out"], post_w=s["post_w"], post_b=s["post_b"], gate=s["gate"], next_w=s["w"],
                     next_b=s["b"], x_out=s["x"], kind=kind, eps=EPS, r_scale=0.75, y_scale=1.25)
    return {"r": s["r_out"], "x": s["x"]}


def _own_route(s):
    from paper_2608_13057_b200 import binding as B
    score = B.ROUTE_SIGMOID if s.get("score") == "sigmoid" else B.ROUTE_SOFTMAX
    B.tempo_route(s["shape"], s["x"], s["w_router"], s["bias"], None, s["ids"], s["w"], s["status"], score=score,
                  renormalise=True, scale=1.0)
    return {"ids": s["ids"], "w": s["w"]}


def _own_layer(s):
    from paper_2608_13057_b200 import binding as B
    r = _own_route(s)
    ffn = B.tempo_few_ffn if s["weights"] == "fp8" else B.tempo_few_ffn_bf16
    ffn(s["shape"], s["x"], s["ids"], s["w"], None, s["replica_map"], s["packed"], s["out"], s["status"], s["workspace"])
    return {**r, "out": s["out"]}


_own = {"norm": _own_norm, "route": _own_route, "layer": _own_layer}


def _norm32(v, w, b, kind):
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS) * w.float()
    return v if b is None else v + b.float()


def _plain_norm(s):
    r = s["r"].float()
    if s["side"] == "in":
        return {"x": _norm32(r, s["w"], s["b"], s["kind"]).to(torch.bfloat16)}
    y = _norm32(s["y"].float(), s["post_w"], s["post_b"], s["kind"])
    if s["gate"] is not None:
        y = y * s["gate"]
    r = 0.75 * r + 1.25 * y
    return {"r": r.to(s["r"].dtype), "x": _norm32(r, s["w"], s["b"], s["kind"]).to(torch.bfloat16)}


def _plain_route(s):
    logits = s["x"].float() @ s["w_router"].float().t()
    if s.get("score") == "sigmoid":
        scores = 1.0 / (1.0 + torch.exp(-logits))
    else:
        scores = torch.exp(logits - logits.amax(dim=1, keepdim=True))
        scores = scores / scores.sum(dim=1, keepdim=True)
    key = logits if s["bias"] is None else scores + s["bias"]
    ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, : s["k"]]   # ties: the lowest index first
    w = torch.gather(scores, 1, ids)
    return {"ids": ids.to(torch.int32), "w": w / w.sum(dim=1, keepdim=True)}


def _dequant(s, which, at=None):
    q = s["w" + which] if at is None else s["w" + which][at]
    if s["weights"] == "bf16":
        return q.float()
    sc = s["s" + which] if at is None else s["s" + which][at]
    G, n, k = q.shape
    return (q.view(torch.float8_e4m3fn).float().view(G, n // 128, 128, k // 128, 128) * sc[:, :, None, :, None]).view(G, n, k)


def _plain_layer(s):
    r = _plain_route(s)
    T, k, f, G = s["T"], s["k"], s["f"], s["local"]
    x = s["x"].float()
    slot = s["replica_map"][:, 0][r["ids"].long()].long()                       # [T, k], -1: not on this rank
    if T * k <= G:                                                              # an expert's weights for each pair
        at = slot.clamp(min=0).reshape(-1)
        gu = torch.bmm(_dequant(s, "13", at), x.repeat_interleave(k, dim=0)[:, :, None])[:, :, 0]
        h = gu[:, :f] / (1.0 + torch.exp(-gu[:, :f])) * gu[:, f:]
        y = torch.bmm(_dequant(s, "2", at), h[:, :, None])[:, :, 0]
        out = (y.view(T, k, -1) * torch.where(slot >= 0, r["w"], 0.0)[:, :, None]).sum(dim=1)
    else:                                                                       # every expert for every token
        gu = torch.matmul(x[None], _dequant(s, "13").transpose(1, 2))
        h = gu[:, :, :f] / (1.0 + torch.exp(-gu[:, :, :f])) * gu[:, :, f:]
        y = torch.matmul(h, _dequant(s, "2").transpose(1, 2))                   # [G, T, d]
        c = (torch.arange(G, device=DEV)[:, None, None] == slot[None]).float() * r["w"][None]
        out = (y * c.sum(dim=2)[:, :, None]).sum(dim=0)
    return {**r, "out": out.to(torch.bfloat16)}


_plain = {"norm": _plain_norm, "route": _plain_route, "layer": _plain_layer}


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    T, d = case["T"], case["d"]
    if case["op"] == "norm":
        rb = 4 if case["stream"] == "f32" else 2
        affine = 2 * d * (2 if case["kind"] == "layer" else 1)
        if case["side"] == "in":
            return {"bytes": T * d * (rb + 2) + affine, "flops": 4 * T * d}
        gate = {"none": 0, "token": 4 * T, "channel": 4 * d}[case["gate"]]
        return {"bytes": T * d * (2 * rb + 4) + 2 * affine + gate, "flops": 11 * T * d}
    E, k = case["E"], case["k"]
    route = {"bytes": 2 * T * d + 2 * E * d + (4 * E if case.get("bias") else 0) + 8 * T * k, "flops": 2 * T * E * d}
    if case["op"] == "route":
        return route
    f = case["f"]
    one = 3 * d * f + 4 * 3 * (d // 128) * (f // 128) if case["weights"] == "fp8" else 6 * d * f
    return {"bytes": route["bytes"] + _active(case) * one + 2 * T * d,
            "flops": route["flops"] + 6.0 * T * k * case["local"] / E * d * f}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    ids, w = _exact_route(s)
    if case["op"] == "route":
        return {"ids": ids.to(torch.int32), "w": w}
    x = s["x"].double()
    out = torch.zeros(case["T"], case["d"], dtype=torch.float64, device=DEV)
    for e in range(case["local"]):                                              # slot e holds expert e on this rank
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if t.numel() == 0:
            continue
        up_gate, down = s["w13"][e], s["w2"][e]
        if case["weights"] == "fp8":
            up_gate = up_gate.view(torch.float8_e4m3fn).double() * s["s13"][e].double().repeat_interleave(128, 0).repeat_interleave(128, 1)
            down = down.view(torch.float8_e4m3fn).double() * s["s2"][e].double().repeat_interleave(128, 0).repeat_interleave(128, 1)
        gate, up = (x[t] @ up_gate.double().t()).chunk(2, dim=1)
        y = (gate * torch.sigmoid(gate) * up) @ down.double().t()
        out.index_add_(0, t, y * w[t, j][:, None])
    return {"ids": ids.to(torch.int32), "w": w, "out": out}


def _exact_route(s):
    logits = torch.einsum("td,ed->te", s["x"].double(), s["w_router"].double())
    p = torch.sigmoid(logits) if s.get("score") == "sigmoid" else torch.softmax(logits, dim=1)
    key = logits if s["bias"] is None else p + s["bias"].double()
    left = key.clone()
    ids = []
    for _ in range(s["k"]):
        top = left.max(dim=1, keepdim=True).values
        first = torch.where(left == top, torch.arange(s["E"], device=DEV), s["E"]).min(dim=1).values
        ids.append(first)
        left.scatter_(1, first[:, None], float("-inf"))
    ids = torch.stack(ids, dim=1)
    w = p.gather(1, ids)
    return ids, w / w.sum(dim=1, keepdim=True)


def _exact_norm(s):
    def norm(v, w, b):
        if s["kind"] == "layer":
            mean = v.sum(1, keepdim=True) / s["d"]
            v = v - mean
        out = v / torch.sqrt(v.pow(2).sum(1, keepdim=True) / s["d"] + EPS) * w.double()
        return out + (0 if b is None else b.double())

    r = s["r"].double()
    if s["side"] == "in":
        return {"x": norm(r, s["w"], s["b"])}
    y = norm(s["y"].double(), s["post_w"], s["post_b"])
    if s["gate"] is not None:
        y = y * s["gate"].double()
    r = r * 0.75 + y * 1.25
    return {"r": r, "x": norm(r, s["w"], s["b"])}
