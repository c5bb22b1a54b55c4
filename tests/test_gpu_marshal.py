"""Counts and status words without an element are refused: they have no address, and a count without one would mean that every
row is live.  Operands on another device than the current one (fakes without memory) are refused too."""
import pytest
import torch

from tests.test_marshal_operands import CALLS, fakes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


def test_empty_counts_and_status_words(B):
    T, d, E, k = 4, 128, 8, 2
    i32 = dict(dtype=torch.int32, device="cuda")
    none, one = torch.zeros(0, **i32), torch.zeros(1, **i32)
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    w, wr = torch.ones(d, device="cuda"), torch.zeros(E, d, dtype=torch.bfloat16, device="cuda")
    ids, tw = torch.zeros(T, k, **i32), torch.zeros(T, k, device="cuda")
    s = B.make_shape(T, k, E, 2, 1, d, 128, 128)
    rmap = torch.full((E, 1), -1, **i32)
    out = torch.full((T, d), 5.0, dtype=torch.bfloat16, device="cuda")
    buffers = {}
    for bf16 in (False, True):
        size = B.tempo_packed_weight_bytes_bf16(s) if bf16 else B.tempo_packed_weight_bytes(s)
        buffers[bf16] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(B.tempo_few_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    few = lambda bf16, nv, st: (B.tempo_few_ffn_bf16 if bf16 else B.tempo_few_ffn)(s, x, ids, tw, nv, rmap, buffers[bf16], out, st, ws)
    calls = {
        "norm in, count": lambda: B.tempo_norm_in(x, w, out, n_valid=none),
        "norm out, count": lambda: B.tempo_norm_out(x, x, out, n_valid=none),
        "route, count": lambda: B.tempo_route(s, x, wr, None, none, ids, tw, one),
        "route, status": lambda: B.tempo_route(s, x, wr, None, None, ids, tw, none),
        "few, count": lambda: few(False, none, one),
        "few, status": lambda: few(False, None, none),
        "few bf16, count": lambda: few(True, none, one),
        "few bf16, status": lambda: few(True, None, none),
    }
    accepted = []
    for name, call in calls.items():
        try:
            call()
            accepted.append(name)
        except B.TempoError as e:
            assert "expected at least 1 elements" in str(e), (name, str(e))
    torch.cuda.synchronize()
    assert not accepted and (out == 5).all()


@pytest.mark.parametrize("name", list(CALLS))
def test_operands_on_another_device_than_the_current_one(B, name):
    operands, call = CALLS[name]
    with pytest.raises(B.TempoError, match="operands on cuda:1, but the current device is cuda:0"):
        call(B, B.make_shape(4, 2, 8, 2, 1, 128, 128, 128), fakes(*operands))
