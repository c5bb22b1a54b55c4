"""tempo_attend calls that take longer than the limit of a device-side wait: a warp may have nothing to do for as long, while the others work."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
LIMIT_MS = 50.0


@pytest.mark.parametrize("D", [64, 128])
def test_half_full_items_over_a_very_long_sequence(D):
    """64 rows, one of an item's two row tiles, over 2^30 tokens that share one page, and a short sequence of two row tiles behind them.
    Weights are equal (keys of zeros) and so are values of all tokens, small integers: every sum is exact."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13057_b200 import binding as B
    Hq, page, L = 64, 256, 2 ** 30
    shape = B.make_cache(2, page, 1, D)
    cache = torch.zeros(B.tempo_cache_bytes(shape), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    v = torch.randint(-7, 9, (D,), device=DEV).float()
    v[0::32], v[1::32] = -7, 8                                          # groups of scale 1
    v = v.to(torch.bfloat16).expand(page, 1, D)
    slots = torch.arange(page, 2 * page, dtype=torch.int32, device=DEV)
    B.tempo_kv_append(shape, torch.zeros_like(v), v.contiguous(), slots, cache, status)
    table = torch.ones(2, L // page, dtype=torch.int32, device=DEV)
    lens = torch.tensor([L, 10000], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 1, 4], dtype=torch.int32, device=DEV)
    q = torch.randn(4, Hq, D, device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(q)
    work = torch.zeros(B.tempo_attend_workspace_bytes(shape, Hq), dtype=torch.uint8, device=DEV)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    B.tempo_attend(shape, q, cache, table, lens, out, status, work, q_start=starts, max_q=3)
    end.record()
    torch.cuda.synchronize()
    assert int(status) == 0
    assert torch.equal(out, v[0].expand(4, Hq, D)) and not work[:640].any()
    assert begin.elapsed_time(end) > LIMIT_MS                           # or the test is of nothing
