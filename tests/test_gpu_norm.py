"""tempo_norm_in / tempo_norm_out against the formula in 64 bits.

Tolerances (derived, per element): a bf16 store is off by at most 2^-8 of the value (half a unit in the eighth bit), an f32
store by 2^-24; the 32-bit arithmetic before it by at most E32 = 2^-20 of the sum of the magnitudes that enter the element
(a row sum of up to 16384 terms is a tree of shuffles over sums of at most 128 terms, so some 140 roundings of 2^-24 at
worst, 9 with the usual cancellation of signs: 16 are granted), where subtracting a mean counts the row's largest value
over its deviation."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

E32 = 16 * 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


def norm64(v, w, b, kind, eps):
    """-> (normed row times w plus b, bound of the 32-bit error of each element)"""
    v = v.double()
    big = v.abs().amax(1, keepdim=True)
    if kind:
        v = v - v.mean(1, keepdim=True)
    s = torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    w = w.double()
    n = v / s * w
    err = E32 * ((v.abs() + (big if kind else 0)) / s * w.abs() + (0 if b is None else b.double().abs()))
    return n + (0 if b is None else b.double()), err


def check(got, ref, err):
    ulp = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -23
    got, ref = got.double().cpu(), ref.cpu()
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got))
    d = (got - ref).abs()[fine]
    tol = (ulp * (ref.abs() + err.cpu()) + err.cpu() + 2.0 ** -133)[fine]
    assert (d <= tol).all(), float((d / tol).max())


def strided(T, d, pad, dtype, fill, shift=0):
    """[T, d] view of a wider buffer (rows `pad` apart, base shifted by `shift` elements) and the buffer around it."""
    whole = torch.full((T * (d + pad) + shift + 8,), fill, dtype=dtype, device="cuda")
    return whole[shift:].as_strided((T, d), (d + pad, 1)), whole


CASES = [  # T, d, pad, shift, kind, stream f32, param f32, gate
    (1, 4096, 0, 0, 0, False, False, "none"),
    (1, 1, 0, 0, 0, False, True, "channel"),
    (3, 1, 5, 1, 1, True, False, "none"),
    (2, 7, 0, 0, 1, False, False, "token"),
    (5, 31, 3, 1, 0, True, True, "full"),
    (7, 33, 0, 0, 0, False, False, "channel_bf16"),
    (4, 130, 2, 0, 1, False, True, "channel"),
    (9, 1021, 0, 0, 0, False, False, "token"),
    (6, 1024, 8, 3, 1, False, False, "full"),          # base off by 3 elements: scalar loads
    (6, 1024, 4, 4, 1, False, False, "channel"),       # 8-byte vectors
    (6, 1022, 0, 2, 0, True, False, "column"),         # 4-byte vectors; a gate whose columns are strided
    (700, 512, 0, 0, 0, False, False, "channel"),
    (700, 2050, 0, 0, 1, True, False, "token"),
    (311, 7168, 64, 0, 0, False, False, "channel"),
    (311, 7168, 0, 0, 1, True, True, "full_bf16"),
    (2, 8200, 0, 0, 1, False, False, "none"),
    (2, 16384, 0, 0, 0, True, False, "channel"),
    (2, 16383, 0, 0, 1, False, False, "one"),
    (300, 16384, 0, 0, 0, False, True, "token"),
]


@pytest.mark.parametrize("T,d,pad,shift,kind,f32,pf32,gate", CASES)
def test_norms_match_the_formula(B, T, d, pad, shift, kind, f32, pf32, gate):
    g = torch.Generator(device="cuda").manual_seed(T * 7919 + d)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    dt, pt = (torch.float32 if f32 else torch.bfloat16), (torch.float32 if pf32 else torch.bfloat16)
    y, _ = strided(T, d, pad, torch.bfloat16, 3.0, shift)
    r, _ = strided(T, d, pad, dt, 5.0, shift)
    ro, ro_all = strided(T, d, pad, dt, -77.0, shift)
    x, x_all = strided(T, d, pad, torch.bfloat16, -77.0, shift)
    y.copy_(rnd(T, d) * 0.5 + 0.25)
    r.copy_(rnd(T, d) * 3 + 1)
    pw, pb, w, b = ((1 + 0.2 * rnd(d)).to(pt), (0.1 * rnd(d)).to(pt), (1 + 0.2 * rnd(d)).to(pt), (0.1 * rnd(d)).to(pt))
    gt = {"none": lambda: None, "channel": lambda: rnd(d), "channel_bf16": lambda: rnd(1, d).bfloat16(),
          "token": lambda: rnd(T, 1), "full": lambda: rnd(T, d), "full_bf16": lambda: rnd(T, d).bfloat16(),
          "one": lambda: rnd(1, 1), "column": lambda: rnd(d, 3)[:, 1]}[gate]()
    eps = 1e-5
    B.tempo_norm_out(y, r, ro, pw, pb, gt, w, b, x, kind=kind, eps=eps, r_scale=0.75, y_scale=1.25)
    x1 = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    B.tempo_norm_in(r, w, x1, b=b, kind=kind, eps=eps)
    torch.cuda.synchronize()
    n, e = norm64(r, w, b, kind, eps)
    check(x1, n, e)
    n, e = norm64(y, pw, pb, kind, eps)
    if gt is not None:
        n, e = n * gt.double(), e * gt.double().abs()
    ref = 0.75 * r.double() + 1.25 * n
    err = 1.25 * e + E32 * (1.25 * n.abs() + 0.75 * r.double().abs())
    check(ro, ref, err)
    n, e = norm64(ref, w, b, kind, eps)
    s = torch.sqrt((((ref - ref.mean(1, keepdim=True)) if kind else ref) ** 2).mean(1, keepdim=True) + eps)
    # r' enters the second norm with its own 32-bit error, in the element and through the row's sums
    check(x, n, e + (2 * err + err.amax(1, keepdim=True)) / s * w.double().abs() * (1 + ref.abs().amax(1, keepdim=True) / s))
    for whole, rows in ((ro_all, ro), (x_all, x)):               # nothing between the rows or behind them is written
        keep = torch.ones_like(whole, dtype=torch.bool)
        keep[shift:].as_strided((T, d), (d + pad, 1)).fill_(False)
        assert (whole[keep] == -77.0).all()


@pytest.mark.parametrize("T,d,kind,place", [
    (9, 1, 0, (1, 2, 3, 5)), (11, 7, 1, (7, 0, 6, 1)), (8, 8, 0, (4, 4, 3, 2)), (8, 9, 1, (0, 1, 2, 3)), (16, 255, 0, (5, 6, 7, 0)),
    (16, 256, 1, (3, 3, 3, 3)), (16, 257, 0, (1, 1, 1, 1)), (350, 2056, 1, (2, 4, 6, 0)), (350, 2311, 0, (0, 0, 0, 0)),
    (700, 1030, 1, (6, 1, 4, 7)), (310, 8193, 0, (1, 0, 7, 2)), (3, 12345, 1, (4, 7, 2, 5))])
def test_operands_at_alignments_of_their_own(B, T, d, kind, place):
    """Rows of bf16 that begin anywhere between two 16-byte boundaries, each operand elsewhere, and the in-place form."""
    g = torch.Generator(device="cuda").manual_seed(T * 31 + d)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    bf = torch.bfloat16
    (y, y_all), (r, r_all), (ro, ro_all), (x, x_all) = (strided(T, d, pad, bf, float("nan"), s) for pad, s in zip((0, 3, 1, 2), place))
    y.copy_(rnd(T, d) * 0.5 + 0.25)
    r.copy_(rnd(T, d) * 3 + 1)
    off = torch.empty(d + 1, device="cuda")
    pw, w, gt = (1 + 0.2 * rnd(d)), off[1:], rnd(1, d)             # one weight that no 16-byte load reaches
    w.copy_(1 + 0.2 * rnd(d))
    eps = 1e-5
    outside = []
    for whole, rows, pad, s in ((ro_all, ro, 1, place[2]), (x_all, x, 2, place[3]), (r_all, r, 3, place[1]), (y_all, y, 0, place[0])):
        keep = torch.ones_like(whole, dtype=torch.bool)
        keep[s:].as_strided((T, d), (d + pad, 1)).fill_(False)
        outside.append((whole, keep))
    B.tempo_norm_out(y, r, ro, pw, None, gt, w, None, x, kind=kind, eps=eps, r_scale=0.75, y_scale=1.25)
    n, e = norm64(y, pw, None, kind, eps)
    n, e = n * gt.double(), e * gt.double().abs()
    ref = 0.75 * r.double() + 1.25 * n
    err = 1.25 * e + E32 * (1.25 * n.abs() + 0.75 * r.double().abs())
    check(ro, ref, err)
    n, e = norm64(ref, w, None, kind, eps)
    s = torch.sqrt((((ref - ref.mean(1, keepdim=True)) if kind else ref) ** 2).mean(1, keepdim=True) + eps)
    check(x, n, e + (2 * err + err.amax(1, keepdim=True)) / s * w.double().abs() * (1 + ref.abs().amax(1, keepdim=True) / s))
    first, second = ro.clone(), x.clone()
    B.tempo_norm_in(r, w, x, kind=kind, eps=eps)
    n, e = norm64(r, w, None, kind, eps)
    check(x, n, e)
    B.tempo_norm_out(y, r, r, pw, None, gt, w, None, y, kind=kind, eps=eps, r_scale=0.75, y_scale=1.25)
    torch.cuda.synchronize()
    assert torch.equal(r, first) and torch.equal(y, second)
    for whole, keep in outside:                                    # nothing around or between the rows is written
        assert torch.isnan(whole[keep]).all()


def test_optional_operands(B):
    T, d = 5, 640
    y, r = torch.randn(T, d, device="cuda").bfloat16(), torch.randn(T, d, device="cuda").bfloat16()
    ro = torch.empty_like(r)
    B.tempo_norm_out(y, r, ro, y_scale=2.0)                       # no post norm, no next norm: a residual sum
    check(ro, r.double() + 2 * y.double(), E32 * (r.double().abs() + 2 * y.double().abs()))


def test_in_place_n_valid_and_zero_rows(B):
    T, d = 6, 1000
    y, r = torch.randn(T, d, device="cuda").bfloat16(), torch.randn(T, d, device="cuda")
    y[1], r[1] = 0, 0                                             # a row of zeros: eps keeps it finite
    w = torch.ones(d, device="cuda")
    a, c = torch.empty_like(r), torch.empty_like(y)
    B.tempo_norm_out(y, r, a, post_w=w, next_w=w, x_out=c)
    y2, r2 = y.clone(), r.clone()
    nv = torch.tensor([4], dtype=torch.int32, device="cuda")
    B.tempo_norm_out(y2, r2, r2, post_w=w, next_w=w, x_out=y2, n_valid=nv)
    torch.cuda.synchronize()
    assert torch.equal(r2[:4], a[:4]) and torch.equal(y2[:4], c[:4])          # r' over r, x' over y
    assert torch.equal(r2[4:], r[4:]) and torch.equal(y2[4:], y[4:])          # padding rows untouched
    assert (a[1] == 0).all() and (c[1] == 0).all()
    nv.zero_()
    B.tempo_norm_in(r2, w, y2, n_valid=nv)
    torch.cuda.synchronize()
    assert torch.equal(y2[:4], c[:4])


def test_non_finite_values_stay_in_their_row(B):
    T, d = 4, 512
    r = torch.randn(T, d, device="cuda").bfloat16()
    ref = torch.empty_like(r)
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    B.tempo_norm_in(r, w, ref)
    r[1, 3], r[2, 9] = float("nan"), float("inf")
    x = torch.empty_like(r)
    B.tempo_norm_in(r, w, x)
    torch.cuda.synchronize()
    assert torch.equal(x[0], ref[0]) and torch.equal(x[3], ref[3])
    assert torch.isnan(x[1]).all() and torch.isnan(x[2, 9])


def test_large_offsets(B):
    """Row offsets beyond 2^31 elements."""
    T, d, pitch = 3, 256, 1_200_000_000
    if torch.cuda.mem_get_info()[0] < 12e9:
        pytest.skip("needs 12 GB")
    whole = torch.empty(2 * pitch + d, dtype=torch.bfloat16, device="cuda")
    r = whole.as_strided((T, d), (pitch, 1))
    r.copy_(torch.randn(T, d, device="cuda"))
    w = torch.ones(d, device="cuda")
    x, x2 = torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    B.tempo_norm_in(r, w, x)
    B.tempo_norm_in(r.contiguous(), w, x2)
    torch.cuda.synchronize()
    assert torch.equal(x, x2)


def test_side_stream_and_graph(B):
    T, d = 65, 2048
    r, w = torch.randn(T, d, device="cuda").bfloat16(), torch.ones(d, device="cuda")
    a, c = torch.empty_like(r), torch.zeros_like(r)
    B.tempo_norm_in(r, w, a)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        big = torch.randn(4096, 4096, device="cuda")
        r2 = r * 0
        for _ in range(20):
            big = big @ big * 1e-3
        r2.copy_(r)
        B.tempo_norm_in(r2, w, c)
    st.synchronize()
    assert torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    c.zero_()
    with torch.cuda.graph(graph):
        B.tempo_norm_in(r, w, c)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, c)


def test_refusals(B):
    T, d = 4, 64
    y = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    r, w = torch.zeros(T, d, device="cuda"), torch.ones(d, device="cuda")
    x = torch.zeros_like(y)
    bad = [
        lambda: B.tempo_norm_in(r.cpu(), w, x),
        lambda: B.tempo_norm_in(r.half(), w, x),
        lambda: B.tempo_norm_in(r, w, x.float()),
        lambda: B.tempo_norm_in(r, w[:32], x),
        lambda: B.tempo_norm_in(r, w, x[:3]),
        lambda: B.tempo_norm_in(r.t().contiguous().t(), w, x),
        lambda: B.tempo_norm_in(r[:1].expand(T, d), w, x),
        lambda: B.tempo_norm_in(r, w, x, b=w.bfloat16()),
        lambda: B.tempo_norm_in(r, w, x, kind=7),
        lambda: B.tempo_norm_in(r[:0], w, x[:0]),
        lambda: B.tempo_norm_in(torch.zeros(1, 16385, device="cuda"), torch.ones(16385, device="cuda"),
                                torch.zeros(1, 16385, dtype=torch.bfloat16, device="cuda")),
        lambda: B.tempo_norm_out(y, r, r.bfloat16()),
        lambda: B.tempo_norm_out(y, r, r, x_out=x),
        lambda: B.tempo_norm_out(y, r, r, post_b=w),
        lambda: B.tempo_norm_out(y, r, r, gate=torch.ones(3, 1, device="cuda")),
        lambda: B.tempo_norm_out(y, r, r, gate=torch.ones(T, 1, device="cuda").half()),
        lambda: B.tempo_norm_out(y, r, r, gate=torch.ones(T, 1)),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(B.TempoError):
            f()
            pytest.fail(f"case {i} was accepted")
