"""What tempo_attend_padded and the layer refuse, and what the layer passes on, without a GPU."""
import ctypes

import pytest
import torch

from tests.test_attention_refusals import NULL, ONE, Attention, B  # noqa: F401


def test_a_count_at_an_odd_address(B):
    shape = B.make_cache(4, 16, 2, 64)
    a = Attention(B=3, T=3, Hq=4, max_q=1, max_pages=2, ld_q=256, hd_q=64, ld_out=256, hd_out=64, scale=0.125)

    def attend(n_valid, q=ONE):
        return B._lib.tempo_attend_padded(ctypes.byref(a), ctypes.byref(shape), q, ONE, ONE, ONE, NULL, n_valid, ONE, ONE, ONE, NULL)
    assert attend(ctypes.c_void_p(258)) == -5 and attend(ONE, q=NULL) == -1 and attend(NULL, q=ctypes.c_void_p(264)) == -5


def test_the_layer_passes_its_count_to_both(B, monkeypatch):
    from paper_2608_13057_b200 import layer
    calls = []
    for name in ("tempo_kv_append", "tempo_attend"):
        monkeypatch.setattr(B, name, lambda *a, **kw: calls.append(kw))
    a = layer.Attention(4, 16, 4, 2, 64, 10, device="cpu")
    qkv, i = torch.zeros(8, 8 * 64, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.int32)
    n = torch.zeros(1, dtype=torch.int32)
    a.forward(qkv, i, i, i[None], i, torch.zeros(8, 256, dtype=torch.bfloat16), n_valid=n)
    assert [kw["n_valid"] is n for kw in calls] == [True, True]
