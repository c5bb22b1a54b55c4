"""The hint max_q where a caller leaves it out, without a GPU: one query without starts, else what the sizes allow."""
import pytest
import torch

from tests.test_attention_refusals import B  # noqa: F401


@pytest.fixture
def passed(B, monkeypatch):  # noqa: F811
    calls = []

    class Marshal:
        attend = staticmethod(lambda *a: calls.append(a[10]) or 0)
        kv_append = staticmethod(lambda *a: 0)
    monkeypatch.setattr(B, "_marshal", Marshal)
    return calls


@pytest.mark.parametrize("T,n_seq,starts,given,want", [(5, 5, False, None, 1), (5, 5, True, None, 1), (300, 2, True, None, 299), (64, 16, True, None, 49),
                                                       (3, 9, True, None, 1), (300, 2, True, 1, 1), (5, 5, False, 7, 7)])
def test_what_is_passed_on(B, passed, T, n_seq, starts, given, want):  # noqa: F811
    from paper_2608_13057_b200 import layer
    a = layer.Attention(4, 16, 4, 2, 64, 400, device="cpu")
    i = torch.zeros(max(T, n_seq + 1), dtype=torch.int32)
    table = torch.zeros(n_seq, 3, dtype=torch.int32)
    q = torch.zeros(T, 4, 64, dtype=torch.bfloat16)
    kw = dict(q_start=i if starts else None)
    if given is not None:
        kw["max_q"] = given
    B.tempo_attend(a.shape, q, a.cache, table, i, q, a.status, a.workspace, **kw)
    a.forward(torch.zeros(T, 512, dtype=torch.bfloat16), i, i, table, i, q, **kw)
    assert passed == [want, want]


def test_what_is_no_tensor_is_refused_as_before(B):  # noqa: F811
    s, i, u = B.make_cache(4, 16, 2, 64), torch.zeros(3, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    for q, table in ((x, None), (3, i[None]), (None, None), (x, i[0]), (x, i[None])):
        with pytest.raises(B.TempoError):
            B.tempo_attend(s, q, u, table, i, x, i, u, q_start=i)
