"""tempo_attend with n_valid: rows from it on are neither read nor written, whatever the starts and lengths say of them."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attend import Case
from tests.test_gpu_attend_many import Followed
from tests.test_gpu_attention_layer import Model

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", params=["little work", "much work"])
def B(request):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13057_b200 import binding
    return binding if request.param == "little work" else Followed(binding)


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _run(c, n_valid, q=None, out=None, q_start="own", max_q=None):
    q = c.q if q is None else q
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device=DEV) if out is None else out
    c.B.tempo_attend(c.shape, q, c.cache, c.table, c.lens, out, c.status, c.work, scale=c.scale, n_valid=n_valid,
                     q_start=c.q_start if q_start == "own" else q_start, max_q=c.max_q if max_q is None else max_q)
    return out


@pytest.mark.parametrize("spans,Hq,Hkv,D,page", [
    ([(9, 3), (300, 5), (64, 1), (33, 0), (40, 2)], 32, 8, 128, 64), ([(200, 200), (77, 1), (500, 130)], 4, 2, 64, 32),
    ([(777, 130), (50, 50), (1000, 1)], 6, 1, 128, 64), ([(4, 9), (0, 3), (10, 10)], 6, 2, 64, 16), ([(600, 257), (90, 20)], 16, 1, 128, 128)])
def test_rows_behind_it_of_any_sequence(B, spans, Hq, Hkv, D, page):
    c = Case(B, spans, Hq, Hkv, D, page)
    T = c.starts[-1]
    whole = _run(c, None)
    c.check(whole)
    for valid in {0, 1, 2, T // 3, T // 2 + 1, T - 1, T, T + 7, -4}:
        live = min(max(valid, 0), T)
        q = c.q.clone()
        q[live:] = float("nan")
        out = _run(c, _i32(valid), q=q)
        assert (out[live:] == 5.0).all(), valid
        for b, (l, n) in enumerate(c.spans):
            m = min(n, live - c.starts[b])
            if m <= 0:
                continue
            rows = slice(c.starts[b], c.starts[b] + m)
            if l == 0:
                assert (out[rows] == 0).all()
                continue
            want, spread, off = (x[:m] for x in R.attend(c.q[c.starts[b]:c.starts[b] + n], c.k[b], c.v[b], c.scale, l - n))
            err, tol = (out[rows].double() - want).abs(), R.attend_tolerance(want, spread, off, l)
            assert (err <= tol).all(), (valid, b)
    assert int(c.status) == 0 and not c.work[:640].any()


def test_a_decode_batch_whose_padding_has_lengths(B):
    c = Case(B, [(300, 1), (41, 1), (900, 1), (64, 1)], 8, 2, 128, 16)
    first, out = _run(c, None, q_start=None), torch.full(c.q.shape, 5.0, dtype=torch.bfloat16, device=DEV)
    n_valid = _i32(2)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run(c, n_valid, out=out, q_start=None)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            _run(c, n_valid, out=out, q_start=None)
    for valid in (2, 0, 3, 4, 1):
        n_valid.fill_(valid)
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        # not by bits: where items are cut goes by the lengths of all that have queries
        c.check(torch.cat([out[:valid], first[valid:]]))
        assert (out[valid:] == 5.0).all()
    assert int(c.status) == 0


@pytest.mark.parametrize("starts", [False, True])
def test_the_layers_padding_rows_are_not_those_of_an_earlier_batch(starts):
    m = Model(8, 2, 64, 16, 64, 4, 400)
    m.step([100, 250, 30, 60])
    a = m.layer
    table = m.table
    keep = a.cache.clone()
    outs = []
    for seed in (0, 1):
        a.cache.copy_(keep)
        g = torch.Generator(device=DEV).manual_seed(9)
        a.q.copy_(torch.randn(a.q.shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))   # an earlier batch's
        qkv = torch.randn(4, (a.Hq + 2 * a.Hkv) * a.D, generator=g, device=DEV).to(torch.bfloat16)
        lens = _i32(101, 251, 31, 61)
        pos = lens - 1
        slots = (table[torch.arange(4, device=DEV), pos.long() // 16] * 16 + pos % 16).to(torch.int32)
        out = torch.full((4, a.Hq, a.D), 7.0, dtype=torch.bfloat16, device=DEV)
        a.forward(qkv, pos, slots, table, lens, out, q_start=_i32(0, 1, 2, 3, 4) if starts else None, n_valid=_i32(2))
        assert (out[2:] == 7.0).all() and out[:2].isfinite().all() and not (out[:2] == 7.0).all(2).any()
        outs.append(out)
    assert torch.equal(*outs) and int(a.status) == 0
