"""An H beyond 32 bits from a finite x makes its own token's output NaN, with either weight type, and no other token's."""
import pytest
import torch

from tests.test_gpu_few import Layer, batch, plain_map

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


class PositiveLayer(Layer):
    """Positive weights: with a positive x no infinite H is hidden by a difference of two infinities."""

    def __init__(self, B, G, d, f, bf16):
        super().__init__(B, G, d, f, bf16, seed=8)
        g = torch.Generator().manual_seed(9)
        w13, w2 = torch.rand(G, 2 * f, d, generator=g) * 0.05 + 0.01, torch.rand(G, d, f, generator=g) * 0.05 + 0.01
        if bf16:
            a, b = w13.bfloat16(), w2.bfloat16()
            B.tempo_pack_weights_bf16(self.shape0, a.cuda(), b.cuda(), self.packed)
            self.w13, self.w2 = a.double(), b.double()
        else:
            (qa, sa, self.w13), (qb, sb, self.w2) = self._quantise(w13, g), self._quantise(w2, g)
            B.tempo_pack_weights(self.shape0, qa.cuda(), sa.cuda(), qb.cuda(), sb.cuda(), self.packed, self.status)
        torch.cuda.synchronize()


@pytest.mark.parametrize("bf16", [False, True], ids=["fp8", "bf16"])
@pytest.mark.parametrize("T", [5, 37])
def test_overflow_of_h(B, bf16, T):
    L = PositiveLayer(B, 4, 256, 256, bf16)
    x, ids, w = batch(T, 2, 4, 256, seed=1)
    x = x.abs()
    m = plain_map(4, 4)
    clean, st = L.run(x, ids, w, m)
    assert st == 0
    L.check(clean, *L.definition(x, ids, w, m))
    x[2] *= 2.0 ** 80                                     # gate and up near 2^80: their product is beyond 2^128
    x[T - 1] *= 2.0 ** 75
    got, _ = L.run(x, ids, w, m)
    assert torch.isnan(got[2]).all() and torch.isnan(got[T - 1]).all()
    keep = [t for t in range(T) if t not in (2, T - 1)]
    assert torch.equal(got[keep], clean[keep])
