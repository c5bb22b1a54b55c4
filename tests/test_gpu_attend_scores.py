"""tempo_attend with scores far beyond the integers that 32-bit floats hold: the softmax is that of the largest scores."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attend import Case
from tests.test_gpu_attend_many import Followed

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", params=["little work", "much work"])
def B(request):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13057_b200 import binding
    return binding if request.param == "little work" else Followed(binding)


@pytest.mark.parametrize("loud,scale", [(1e4, None), (1e6, None), (1e8, None), (1e10, 0.3), (1e20, 1.0), (3e38, None), (3e38, 9e29), (1e-3, 1e12),
                                        (1.0, 1e29), (1e10, -0.7)])
@pytest.mark.parametrize("n,Hq,Hkv,D", [(1, 8, 2, 64), (4, 16, 2, 128), (100, 6, 2, 64), (130, 12, 1, 128)])
def test_the_largest_scores_win(B, loud, scale, n, Hq, Hkv, D):
    """Keys are one direction times a size that the cache holds exactly, queries that direction times +-loud: every product and sum is
    exact, and scores differ by a fifteenth of the largest at least or not at all.  The output is the mean of the values of the
    largest ones that a query sees."""
    L = 300
    c = Case(B, [(L, n)], Hq, Hkv, D, 16)
    g = torch.Generator(device=DEV).manual_seed(n)
    size = torch.randint(1, 16, (L, Hkv, 1), generator=g, device=DEV).float() * 15 / 8                  # 15 times a scale
    size = torch.where(torch.rand(L, Hkv, 1, generator=g, device=DEV) < 0.5, size, -size)
    k = (size * torch.ones(D, device=DEV)).to(torch.bfloat16)
    v = torch.randn(L, Hkv, D, generator=g, device=DEV).to(torch.bfloat16)
    t = torch.arange(L, device=DEV)
    B.tempo_kv_append(c.shape, k, v, (c.table[0][t // 16] * 16 + t % 16).to(torch.int32), c.cache, c.status)
    sign = torch.where(torch.rand(n, Hq, 1, generator=g, device=DEV) < 0.5, -1.0, 1.0)
    c.q = (sign * torch.full((D,), loud, device=DEV)).to(torch.bfloat16)
    c.scale = D ** -0.5 if scale is None else scale
    out = c.run()
    want = torch.zeros(n, Hq, D, dtype=torch.float64, device=DEV)
    size, value = size[:, :, 0].double(), R.cached(v)
    for i in range(n):
        for h in range(Hq):
            to = L - n + i + 1
            s = size[:to, h * Hkv // Hq] * float(sign[i, h, 0]) * (1.0 if c.scale > 0 else -1.0)
            want[i, h] = value[:to, h * Hkv // Hq][s == s.max()].mean(0)
    # the mean's rounding to bf16, its equal weights' to fp16, and its sums in 32 bits
    tol = want.abs() * (2.0 ** -8 + 2.0 ** -11) + 2.0 ** -20 * value.abs().amax()
    assert torch.equal(R.cached(k).double(), k.double())
    assert ((out.double() - want).abs() <= tol).all(), float(((out.double() - want).abs() / tol).nan_to_num(1e9).max())
    assert int(c.status) == 0


@pytest.mark.parametrize("n", [1, 5, 200])
def test_rows_of_huge_and_ordinary_scores_side_by_side(B, n):
    c = Case(B, [(700, n), (90, min(n, 90))], 16, 2, 128, 16)
    ordinary = c.run()
    c.check(ordinary)
    huge = torch.zeros(16, dtype=torch.bool, device=DEV)
    huge[1::3] = True
    c.q[:, huge] = (c.q[:, huge].float() * 1e12).to(torch.bfloat16)
    out = c.run()
    assert torch.equal(out[:, ~huge], ordinary[:, ~huge]) and out.isfinite().all()
    # of random scores one wins: its token's value
    for b, (l, m) in enumerate(c.spans):
        rows = slice(c.starts[b], c.starts[b] + m)
        kv = torch.arange(16, device=DEV) // 8
        s = torch.einsum("nhd,lhd->nhl", c.q[rows].double(), c.k[b][:, kv])
        off = torch.einsum("nhd,lhd->nhl", c.q[rows].double().abs(), c.k[b][:, kv].abs()).amax(2) * (128 + 8) * 2.0 ** -24
        hidden = torch.arange(l, device=DEV)[None, :] > l - m + torch.arange(m, device=DEV)[:, None]
        s = s.masked_fill(hidden[:, None], float("-inf"))
        top = s.topk(2, dim=2).values
        clear = huge[None] & (top[..., 0] - top[..., 1] > 4 * off)      # apart by more than the scores' roundings
        assert clear.any()
        at = s.argmax(2)
        want = c.v[b][at, kv[None].expand(m, 16)]
        err = (out[rows].double() - want).abs()
        assert (err <= want.abs() * (2.0 ** -8 + 2.0 ** -11) + 2.0 ** -20 * want.abs().amax()).all(2)[clear].all()
    assert int(c.status) == 0
