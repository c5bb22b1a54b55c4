"""Sigmoid scores below the smallest 32-bit value: their renormalised weights still have one.

Logits are exact in 32 bits (two products).  A weight is exp(l - m) over the sum of such: 2^-18 of itself as in test_gpu_route,
and where a score is below 2^-100 of the largest, 2^-100 absolutely."""
import pytest
import torch

from tests.test_gpu_route import RTOL, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


@pytest.mark.parametrize("T,E", [(3, 24), (600, 64), (2500, 160), (70, 300)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_renormalised_weights_of_very_negative_logits(B, T, E, with_bias):
    k, d = 6, 128
    g = torch.Generator().manual_seed(T + E)
    x, wr = torch.zeros(T, d), torch.zeros(E, d)
    base = torch.tensor([0.0, -64.0, -72.0, -88.0, -96.0, -104.0, -176.0, -1024.0])
    x[:, 0] = base[torch.arange(T) % 8]
    x[:, 1] = 1.0
    wr[:, 0] = 1.0
    wr[:, 1] = -torch.randperm(E, generator=g).float() / 16
    bias = torch.where(torch.arange(E) % 2 == 0, 1.0, float("-inf")) if with_bias else None
    x, wr = x.bfloat16(), wr.bfloat16()
    logits = x.double() @ wr.double().t()
    ids, w, st = run(B, x, wr, bias, k, 1, True, 2.0)
    assert st == 0 and not torch.isnan(w).any()
    l = logits.gather(1, ids.long())
    ref = torch.softmax(torch.nn.functional.logsigmoid(l), 1) * 2.0   # scores over their sum, in logarithms
    assert ((w.double() - ref).abs() <= RTOL * ref + 2.0 ** -100).all()
    if not with_bias:
        assert torch.equal(ids.long(), torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k])
    else:
        assert (ids % 2 == 0).all()
    ids2, w2, _ = run(B, x, wr, bias, k, 1, False, 2.0)               # as they are: below 2^-126 or so they are zero
    assert torch.equal(ids, ids2)
    p = torch.sigmoid(l) * 2.0
    assert ((w2.double() - p).abs() <= RTOL * p + 2.0 ** -125).all()
