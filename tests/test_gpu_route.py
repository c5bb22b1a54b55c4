"""tempo_route against the definition in 64 bits.

Inputs lie on a grid on which every dot product is exact in 32 bits in any order (products are multiples of 2^-16, sums
stay below 2^7), so the chosen experts are compared exactly.  Weights: the argument of an exponential is off by at most
2^-20 (logits below 16), the exponential by 2^-22 of itself, and a quotient of two such by 2^-19 in all; 2^-18 is granted."""
import pytest
import torch

pytestmark = pytest.mark.gpu

RTOL = 2.0 ** -18


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


def grid(g, shape, std, step, most):
    v = torch.randn(shape, generator=g) * std
    return (torch.round(v / step) * step).clamp(-most, most).to(torch.bfloat16)


def inputs(T, E, d, seed):
    g = torch.Generator().manual_seed(seed)
    return (grid(g, (T, d), 1.0, 2.0 ** -5, 7.96875), grid(g, (E, d), 0.02, 2.0 ** -11, 255 * 2.0 ** -11),
            torch.randn(E, generator=g) * 0.05)


def definition(logits, bias, k, score, renormalise, scale):
    logits = logits.double()
    fine = torch.isfinite(logits)
    l = torch.where(fine, logits, float("-inf"))
    p = torch.sigmoid(l) if score else torch.nan_to_num(torch.softmax(l, 1), nan=0.0)
    key = l if bias is None else torch.where(fine, p + bias.double(), float("-inf"))
    key = torch.where(torch.isnan(key) | (key == float("inf")), torch.tensor(float("-inf"), dtype=torch.float64), key)
    ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :k]
    w = p.gather(1, ids)
    if bias is not None:
        w = torch.where(torch.isfinite(bias)[ids], w, 0.0)
    if renormalise:
        s = w.sum(1, keepdim=True)
        w = torch.where(s > 0, w / s, 0.0)
    return ids.int(), w * scale


def run(B, x, wr, bias, k, score, renormalise=True, scale=1.0, n_valid=None):
    T, d = x.shape
    E = wr.shape[0]
    shape = B.make_shape(T, k, E, 1, 1, d, 128, 128)
    ids = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), -7.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    nv = None if n_valid is None else torch.tensor([n_valid], dtype=torch.int32, device="cuda")
    B.tempo_route(shape, x.cuda(), wr.cuda(), None if bias is None else bias.cuda(), nv, ids, w, st, score=score,
                  renormalise=renormalise, scale=scale)
    torch.cuda.synchronize()
    return ids.cpu(), w.cpu(), int(st.item())


def check(got, ref):
    assert torch.equal(got[0], ref[0])
    assert ((got[1].double() - ref[1]).abs() <= RTOL * ref[1].abs()).all()


CASES = [  # T, E, d, k, score, bias, renormalise, scale
    (1, 128, 4096, 8, 0, False, True, 1.0),
    (1, 1, 128, 1, 0, False, True, 1.0),
    (1, 2, 128, 2, 1, True, False, 2.5),
    (2, 17, 256, 3, 1, False, True, 1.0),
    (5, 60, 2048, 4, 0, False, False, 1.0),
    (9, 33, 384, 32, 0, False, True, 1.0),
    (64, 256, 7168, 8, 1, True, True, 2.5),
    (127, 64, 1024, 6, 0, False, False, 16.0),
    (129, 160, 5120, 6, 0, False, True, 1.0),
    (200, 257, 512, 8, 1, True, True, 1.0),              # more than 256 experts: 64-token tiles, two weight boxes
    (131, 512, 1024, 10, 0, False, True, 1.0),
    (3, 300, 128, 5, 1, False, True, 1.0),
    (1000, 128, 640, 8, 0, False, True, 1.0),
    (2500, 96, 512, 2, 1, True, True, 1.0),
]


@pytest.mark.parametrize("T,E,d,k,score,with_bias,renorm,scale", CASES)
def test_route_matches_the_definition(B, T, E, d, k, score, with_bias, renorm, scale):
    x, wr, bias = inputs(T, E, d, T * 31 + E)
    logits = x.double() @ wr.double().t()
    if not with_bias:
        bias = None
    ids, w, st = run(B, x, wr, bias, k, score, renorm, scale)
    ref_ids, ref_w = definition(logits, bias, k, score, renorm, scale)
    assert st == 0
    if with_bias:
        # score + bias is a 32-bit sum: experts whose sums are within its rounding may change places
        key = torch.sigmoid(logits) + bias.double()
        near = (key.gather(1, ids.long()) - key.gather(1, ref_ids.long())).abs() <= 2.0 ** -21
        assert near.all() and (ids == ref_ids).float().mean() > 0.999
        same = (ids == ref_ids).all(1)
        check((ids[same], w[same]), (ref_ids[same], ref_w[same]))
    else:
        check((ids, w), (ref_ids, ref_w))
    assert all(len(set(r)) == k for r in ids.tolist())


def test_ties_go_to_the_lowest_expert(B):
    x = torch.ones(3, 128).bfloat16()
    wr = torch.zeros(70, 128).bfloat16()
    wr[[5, 40, 69]] = 0.25
    wr[[6, 38]] = -0.0
    ids, w, st = run(B, x, wr, None, 6, 0)
    assert ids[0].tolist() == [5, 40, 69, 0, 1, 2] and torch.equal(ids[0], ids[2]) and st == 0


def test_non_finite_logits_and_excluded_experts(B):
    x, wr, _ = inputs(6, 40, 256, 5)
    x[1, 0] = float("nan")                                # every logit of token 1
    wr[7, 3] = float("inf")                               # expert 7 for every token (x[:, 3] may be 0: NaN then)
    logits = x.double() @ wr.double().t()
    ids, w, st = run(B, x, wr, None, 4, 0)
    ref = definition(logits, None, 4, 0, True, 1.0)
    assert st == B.STATUS_BAD_LOGIT
    assert ids[1].tolist() == [0, 1, 2, 3] and (w[1] == 0).all()
    keep = [0, 2, 3, 4, 5]
    check((ids[keep], w[keep]), (ref[0][keep], ref[1][keep]))
    assert not (ids[keep] == 7).any()
    # a bias of -inf takes an expert out; with every expert out the lowest ids come with weight 0
    x, wr, bias = inputs(6, 40, 256, 6)
    bias[::2] = float("-inf")
    ids, w, st = run(B, x, wr, bias, 8, 1)
    assert st == 0 and (ids % 2 == 1).all() and torch.allclose(w.sum(1), torch.ones(6))
    bias[:] = float("-inf")
    bias[30] = 0.0
    ids, w, st = run(B, x, wr, bias, 3, 1)
    assert st == 0 and ids[0].tolist() == [30, 0, 1] and (w[:, 0] == 1).all() and (w[:, 1:] == 0).all()
    bias[:] = torch.finfo(torch.float32).min              # the type's lowest value is an ordinary bias: ties by index
    ids, w, st = run(B, x, wr, bias, 3, 1)
    assert st == 0 and ids[0].tolist() == [0, 1, 2] and (w > 0).all()


@pytest.mark.parametrize("n_valid", [0, 1, 77, 128, 150])
def test_padding_rows(B, n_valid):
    x, wr, _ = inputs(150, 64, 512, 9)
    ids, w, st = run(B, x, wr, None, 4, 0, n_valid=n_valid)
    ref = definition((x.double() @ wr.double().t())[:n_valid], None, 4, 0, True, 1.0)
    check((ids[:n_valid], w[:n_valid]), ref)
    assert (ids[n_valid:] == -1).all() and (w[n_valid:] == 0).all() and st == 0


def test_same_bits_every_time(B):
    g = torch.Generator().manual_seed(3)
    x, wr = torch.randn(300, 2048, generator=g).bfloat16(), (torch.randn(200, 2048, generator=g) * 0.02).bfloat16()
    first = run(B, x, wr, None, 8, 0)
    for _ in range(5):
        again = run(B, x, wr, None, 8, 0)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_refusals(B):
    x, wr, bias = inputs(4, 16, 128, 1)
    ok = B.make_shape(4, 2, 16, 1, 1, 128, 128, 128)
    ids, w = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    xc, wc = x.cuda(), wr.cuda()
    for f in (
        lambda: B.tempo_route(ok, x, wc, None, None, ids, w, st),
        lambda: B.tempo_route(ok, xc.float(), wc, None, None, ids, w, st),
        lambda: B.tempo_route(ok, xc, wc, None, None, ids, w, st, score=2),
        lambda: B.tempo_route(ok, xc, wc, None, None, None, w, st),
        lambda: B.tempo_route(B.make_shape(4, 20, 16, 1, 1, 128, 128, 128), xc, wc, None, None, ids, w, st),
        lambda: B.tempo_route(B.make_shape(4, 2, 513, 1, 1, 128, 128, 128), xc, wc, None, None, ids, w, st),
        lambda: B.tempo_route(B.make_shape(4, 2, 16, 1, 1, 100, 128, 128), xc, wc, None, None, ids, w, st),
        lambda: B.tempo_route(ok, torch.zeros(4 * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(4, 128), wc, None, None,
                              ids, w, st),
    ):
        with pytest.raises(B.TempoError):
            f()
