"""tempo_route on batches large enough for two tokens per warp, for one CTA per tile of tokens, and with softmax scores under a
bias.  Inputs and tolerances as in test_gpu_route; a biased softmax score is off by 2^-19 of the score (its exponential 2^-22,
the sum of at most 512 such terms 2^-20, the quotient and the argument the rest) and 2^-23 of a sum below 2, so two keys that
stand in the other order than the definition's differ by 2^-19 of both scores and 2^-22 at most."""
import pytest
import torch

from tests.test_gpu_route import check, definition, inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


CASES = [  # T, E, d, k, score, bias, renormalise, scale, n_valid
    (2500, 160, 512, 8, 0, False, True, 1.0, None),
    (2500, 256, 384, 8, 1, True, True, 2.5, None),
    (5003, 256, 256, 8, 0, False, False, 1.0, None),
    (5003, 129, 128, 3, 1, False, True, 1.0, 4933),       # the rows of the last tile and a part of the one before are padding
    (5003, 160, 256, 8, 0, True, True, 1.0, 2500),
    (9601, 256, 128, 6, 0, False, True, 1.0, None),       # 76 tiles: no split of the reduction
    (9601, 64, 128, 4, 1, False, True, 1.0, 9599),
    (5003, 300, 128, 5, 0, False, True, 1.0, None),       # 79 tiles of 64 tokens
    (5003, 512, 128, 32, 1, True, True, 1.0, 4999),
    (1, 128, 1024, 8, 0, True, True, 1.0, None),          # softmax scores with a bias
    (7, 40, 256, 4, 0, True, False, 2.0, None),
    (150, 256, 512, 8, 0, True, True, 1.0, 77),
    (131, 500, 256, 10, 0, True, False, 1.0, None),
]


@pytest.mark.parametrize("T,E,d,k,score,with_bias,renorm,scale,n_valid", CASES)
def test_route_matches_the_definition(B, T, E, d, k, score, with_bias, renorm, scale, n_valid):
    x, wr, bias = inputs(T, E, d, T * 7 + E)
    bias = bias if with_bias else None
    ids, w, st = run(B, x, wr, bias, k, score, renorm, scale, n_valid)
    assert st == 0
    n = T if n_valid is None else n_valid
    assert (ids[n:] == -1).all() and (w[n:] == 0).all()
    ids, w = ids[:n], w[:n]
    logits = (x.double() @ wr.double().t())[:n]
    ref_ids, ref_w = definition(logits, bias, k, score, renorm, scale)
    if with_bias:
        p = torch.sigmoid(logits) if score else torch.softmax(logits, 1)
        key = p + bias.double()
        at = lambda v, i: v.gather(1, i.long())
        near = (at(key, ids) - at(key, ref_ids)).abs() <= 2.0 ** -19 * (at(p, ids) + at(p, ref_ids)) + 2.0 ** -22
        assert near.all() and (ids == ref_ids).float().mean() > 0.995
        same = (ids == ref_ids).all(1)
        check((ids[same], w[same]), (ref_ids[same], ref_w[same]))
    else:
        check((ids, w), (ref_ids, ref_w))
    s = ids.sort(1).values
    assert (s[:, 1:] > s[:, :-1]).all()                             # k different experts


def test_ties_and_non_finite_tokens_in_a_batch(B):
    """Two tokens share a warp: what one of them needs must not touch the other."""
    T, E, d, k = 2500, 200, 128, 8
    x, wr, _ = inputs(T, E, d, 3)
    wr[100:] = wr[:100]                                             # every expert twice: ties everywhere
    ref, ref_w = definition(x.double() @ wr.double().t(), None, k, 0, True, 1.0)
    ids, w, st = run(B, x, wr, None, k, 0)
    assert st == 0
    check((ids, w), (ref, ref_w))
    bad = torch.arange(0, T, 17)
    x[bad, 5] = float("nan")
    ids, w, st = run(B, x, wr, None, k, 0)
    assert st == B.STATUS_BAD_LOGIT
    keep = torch.ones(T, dtype=torch.bool)
    keep[bad] = False
    check((ids[keep], w[keep]), (ref[keep], ref_w[keep]))
    assert (ids[bad] == torch.arange(k, dtype=torch.int32)).all() and (w[bad] == 0).all()
