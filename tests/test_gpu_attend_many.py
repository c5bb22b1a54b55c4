"""tempo_attend's calls of several queries again, in batches of so many rows that none of them counts as little work: q and out are
followed by rows of no sequence.  And a batch of which one part counts as that and the other does not."""
import pytest
import torch

from tests.test_gpu_attend import (Case, test_a_missing_page_anywhere_in_a_tile, test_another_stream_and_a_graph,  # noqa: F401
                                   test_bad_pages_lengths_and_values, test_large_scores_and_far_apart_sizes,
                                   test_more_tiles_than_are_numbered, test_rows_outside_the_sequences_and_strides, test_scales,
                                   test_several_queries_per_sequence)

pytestmark = pytest.mark.gpu
ROWS_TIMES_HEADS = 5 << 20


class Followed:
    """The binding, with tempo_attend called on buffers of many more rows in the same order."""

    def __init__(self, binding):
        self.binding = binding

    def __getattr__(self, name):
        return getattr(self.binding, name)

    def tempo_attend(self, shape, q, cache, page_table, lens, out, *args, **kw):
        T, H, D = q.shape
        rows = ROWS_TIMES_HEADS // H + T
        longer = []
        for t in (q, out):
            ld, hd, _ = t.stride()
            longer.append(torch.empty_strided((rows, H, D), (ld, ld * rows if hd > ld else hd, 1), dtype=t.dtype, device=t.device))
        for t, big in zip((q, out), longer):
            heads = H if t.stride(1) else 1                              # one that all heads share is written once
            big[:T, :heads].copy_(t[:, :heads])
        if kw.get("q_start") is None:
            kw["q_start"] = torch.arange(lens.shape[0] + 1, dtype=torch.int32, device=q.device)
        self.binding.tempo_attend(shape, longer[0], cache, page_table, lens, longer[1], *args, **kw)
        out.copy_(longer[1][:T])


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13057_b200 import binding
    return Followed(binding)


@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
def test_little_and_much_in_one_batch(B, D, page):
    # 4 Mi pairs over 260 rows of 64 heads: 252 tokens
    c = Case(B.binding, [(600, 100), (251, 90), (252, 50), (253, 8), (1500, 7), (0, 4), (40, 1)], 64, 4, D, page)
    assert c.q.shape[0] == 260
    for _ in range(2):
        c.check(c.run())
    assert int(c.status) == 0 and not c.work[:640].any()


@pytest.mark.parametrize("spans,Hq,Hkv,D", [([(30000, 16)], 64, 8, 128), ([(150000, 9)], 16, 1, 64), ([(40000, 40), (9000, 30)], 16, 1, 128)])
def test_items_of_many_parts(B, spans, Hq, Hkv, D):
    """Few items of many tokens: the parts of one are joined in groups."""
    c = Case(B.binding, spans, Hq, Hkv, D, 256)
    out = c.run()
    c.check(out)
    assert torch.equal(out, c.run())
    assert int(c.status) == 0 and not c.work[:2048].any()
