"""The norm kernel that takes several rows per CTA (aligned bf16 rows in batches), after a block: one parameter between the
first norm and the sum, alone or with a gate, in place and with padding rows.  Tolerances as in test_gpu_norm."""
import pytest
import torch

from tests.test_gpu_norm import E32, check, norm64, strided

pytestmark = pytest.mark.gpu
bf = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


def operands(T, d, pad, pt, gate, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    y, r = strided(T, d, pad, bf, 3.0)[0], strided(T, d, pad, bf, 5.0)[0]
    y.copy_(rnd(T, d) * 0.5 + 0.25)
    r.copy_(rnd(T, d) * 3 + 1)
    pw, w, b = (1 + 0.2 * rnd(d)).to(pt), (1 + 0.2 * rnd(d)).to(pt), (0.1 * rnd(d)).to(pt)
    gt = {"none": lambda: None, "channel": lambda: rnd(d), "channel_bf16": lambda: rnd(1, d).bfloat16(), "token": lambda: rnd(T, 1),
          "one": lambda: rnd(1, 1)}[gate]()
    return y, r, pw, w, b, gt


CASES = [  # T, d, pad, kind, parameters f32, gate
    (700, 512, 0, 0, False, "none"),
    (3001, 512, 64, 1, True, "channel"),
    (700, 1032, 0, 1, False, "channel"),
    (3001, 1032, 8, 0, True, "token"),
    (700, 4096, 0, 0, False, "channel_bf16"),
    (3001, 4096, 0, 0, False, "none"),
    (700, 7168, 64, 1, True, "token"),
    (3001, 7168, 0, 0, False, "channel"),
    (300, 16384, 0, 0, True, "channel_bf16"),
    (1481, 2048, 0, 1, False, "one"),
]


@pytest.mark.parametrize("T,d,pad,kind,pf32,gate", CASES)
def test_one_parameter_after_the_first_norm(B, T, d, pad, kind, pf32, gate):
    eps = 1e-5
    y, r, pw, w, b, gt = operands(T, d, pad, torch.float32 if pf32 else bf, gate, T + d)
    (ro, ro_all), (x, x_all) = strided(T, d, pad, bf, -77.0), strided(T, d, pad, bf, -77.0)
    call = lambda y, r, ro, x, **kw: B.tempo_norm_out(y, r, ro, post_w=pw, gate=gt, next_w=w, next_b=b, x_out=x, kind=kind, eps=eps,
                                                     r_scale=0.75, y_scale=1.25, **kw)
    call(y, r, ro, x)
    n, e = norm64(y, pw, None, kind, eps)
    if gt is not None:
        n, e = n * gt.double(), e * gt.double().abs()
    ref = 0.75 * r.double() + 1.25 * n
    err = 1.25 * e + E32 * (1.25 * n.abs() + 0.75 * r.double().abs())
    check(ro, ref, err)
    n, e = norm64(ref, w, b, kind, eps)
    s = torch.sqrt((((ref - ref.mean(1, keepdim=True)) if kind else ref) ** 2).mean(1, keepdim=True) + eps)
    check(x, n, e + (2 * err + err.amax(1, keepdim=True)) / s * w.double().abs() * (1 + ref.abs().amax(1, keepdim=True) / s))
    for whole in (ro_all, x_all):                                  # nothing between the rows or behind them is written
        keep = torch.ones_like(whole, dtype=torch.bool)
        keep.as_strided((T, d), (d + pad, 1)).fill_(False)
        assert (whole[keep] == -77.0).all()
    only = torch.full_like(ro, -77.0)                              # without the next norm
    call_only = B.tempo_norm_out(y, r, only, post_w=pw, gate=gt, kind=kind, eps=eps, r_scale=0.75, y_scale=1.25)
    assert call_only is None
    torch.cuda.synchronize()
    assert torch.equal(only, ro)
    # in place (r' over r, x' over y), and only the first rows: the others are neither read nor written
    for nv in (0, 1, T // 2 + 3, T):
        y2, r2 = y.clone(), r.clone()
        y2[nv:], r2[nv:] = float("nan"), float("nan")
        call(y2, r2, r2, y2, n_valid=torch.tensor([nv], dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert torch.equal(r2[:nv], ro[:nv]) and torch.equal(y2[:nv], x[:nv])
        assert torch.isnan(r2[nv:]).all() and torch.isnan(y2[nv:]).all()


@pytest.mark.parametrize("T,d", [(700, 512), (3001, 1032), (311, 16384)])
def test_before_a_block_with_padding_rows(B, T, d):
    _, r, _, w, b, _ = operands(T, d, 0, bf, "none", d)
    x = torch.empty(T, d, dtype=bf, device="cuda")
    B.tempo_norm_in(r, w, x, b=b, eps=1e-5)
    check(x, *norm64(r, w, b, 0, 1e-5))
    nv = T // 3 + 1
    part = torch.full_like(x, -77.0)
    r[nv:] = float("nan")
    B.tempo_norm_in(r, w, part, b=b, eps=1e-5, n_valid=torch.tensor([nv], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(part[:nv], x[:nv]) and (part[nv:] == -77).all()
