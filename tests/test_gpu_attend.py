"""tempo_attend against the formula in 64 bits, over caches filled by tempo_kv_append."""
import pytest
import torch

from tests import attention_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13057_b200 import binding
    return binding


class Case:
    """Sequences of (tokens, queries), their pages in any order among pages of garbage."""

    def __init__(self, B, spans, Hq, Hkv, D, page, seed=0, spare=2, loud=1.0, fill=0xFF):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed + 17 * len(spans) + D)
        per = [max(1, -(-l // page)) for l, _ in spans]
        n_pages = sum(per) + spare
        self.B, self.spans, self.page = B, spans, page
        self.shape = B.make_cache(n_pages, page, Hkv, D)
        # whatever lies behind a sequence's last token must not matter: NaN scales among it
        self.cache = torch.full((B.tempo_cache_bytes(self.shape),), fill, dtype=torch.uint8, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        where = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        self.table = torch.full((len(spans), max(per) + 1), 2 ** 30, dtype=torch.int32, device=DEV)
        at = 0
        self.k, self.v = [], []
        for b, (l, _) in enumerate(spans):
            self.table[b, :per[b]] = where[at:at + per[b]]
            at += per[b]
            k, v = (torch.randn(l, Hkv, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
            t = torch.arange(l, device=DEV)
            if l:
                slots = (self.table[b][t // page] * page + t % page).to(torch.int32)
                B.tempo_kv_append(self.shape, k, v, slots, self.cache, self.status)
            self.k.append(R.cached(k) if l else k.double()), self.v.append(R.cached(v) if l else v.double())
        starts = [0]
        for _, n in spans:
            starts.append(starts[-1] + n)
        self.starts = starts
        self.q_start = torch.tensor(starts, dtype=torch.int32, device=DEV)
        self.lens = torch.tensor([l for l, _ in spans], dtype=torch.int32, device=DEV)
        self.q = (loud * torch.randn(max(starts[-1], 1), Hq, D, generator=g, device=DEV)).to(torch.bfloat16)
        self.max_q = max(1, max(n for _, n in spans))
        self.scale = D ** -0.5
        self.work = torch.zeros(B.tempo_attend_workspace_bytes(self.shape, Hq), dtype=torch.uint8, device=DEV)

    def run(self, q=None, out=None, q_start="own", max_q=None):
        q = self.q if q is None else q
        out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device=DEV) if out is None else out
        self.B.tempo_attend(self.shape, q, self.cache, self.table, self.lens, out, self.status, self.work, scale=self.scale,
                            q_start=self.q_start if q_start == "own" else q_start, max_q=self.max_q if max_q is None else max_q)
        return out

    def check(self, out, q=None):
        q = self.q if q is None else q
        for b, (l, n) in enumerate(self.spans):
            rows = slice(self.starts[b], self.starts[b] + n)
            if n == 0:
                continue
            if l == 0:
                assert (out[rows] == 0).all()
                continue
            want, spread, off = R.attend(q[rows], self.k[b], self.v[b], self.scale, l - n)
            err, tol = (out[rows].double() - want).abs(), R.attend_tolerance(want, spread, off, l)
            assert (err <= tol).all(), (b, l, n, float((err / tol).max()))


ONE = [
    ([(1, 1)], 1, 1, 64, 16), ([(1, 1)], 64, 4, 128, 64), ([(31, 1), (32, 1), (33, 1)], 8, 2, 128, 16),
    ([(1500, 1)], 64, 4, 128, 64), ([(17, 1), (0, 1), (2999, 1), (16, 1), (1, 1)], 8, 8, 64, 16), ([(5000, 1)], 16, 1, 128, 256),
    ([(4097, 1), (100, 1)], 40, 2, 64, 32), ([(100 + 37 * b, 1) for b in range(70)], 12, 4, 128, 128),
    ([(20000, 1), (3, 1)], 8, 8, 128, 64), ([(64, 1)] * 300, 7, 1, 64, 64),
]


@pytest.mark.parametrize("spans,Hq,Hkv,D,page", ONE)
def test_one_query_per_sequence(B, spans, Hq, Hkv, D, page):
    c = Case(B, spans, Hq, Hkv, D, page)
    out = c.run()
    c.check(out)
    assert torch.equal(out, c.run(q_start=None))                        # the same call without the starts, and again
    assert int(c.status) == 0 and not c.work[:640].any()


MANY = [
    ([(4, 4)], 8, 2, 128, 16), ([(9, 3), (300, 5), (64, 1), (33, 0), (40, 2)], 32, 8, 128, 64), ([(200, 200)], 4, 2, 64, 32),
    ([(777, 130), (50, 50), (1000, 1)], 6, 1, 128, 64), ([(2, 5), (0, 3), (10, 10)], 6, 2, 64, 16), ([(600, 257)], 16, 1, 128, 128),
    ([(1100, 300), (4000, 40)], 14, 2, 64, 16), ([(515, 515)], 3, 3, 128, 64), ([(2300, 512)], 8, 1, 128, 256), ([(40, 17)] * 9, 48, 3, 64, 16),
]


@pytest.mark.parametrize("spans,Hq,Hkv,D,page", MANY)
def test_several_queries_per_sequence(B, spans, Hq, Hkv, D, page):
    c = Case(B, spans, Hq, Hkv, D, page)
    c.check(c.run())
    c.check(c.run(max_q=1))                                             # a hint, no more
    assert int(c.status) == 0 and not c.work[:640].any()


@pytest.mark.parametrize("n", [1, 6, 140])
def test_large_scores_and_far_apart_sizes(B, n):
    """Scores in the hundreds (the maximum moves, most weights vanish), queries of tiny and huge size side by side."""
    c = Case(B, [(900, n), (130, min(n, 130))], 16, 2, 128, 16, loud=40.0)
    c.q[:, ::2] *= 2.0 ** -30
    c.q[:, 1] = 0
    c.check(c.run())


@pytest.mark.parametrize("n", [1, 3, 150])
def test_rows_outside_the_sequences_and_strides(B, n):
    """Padding rows before and behind the sequences stay; q and out inside wider rows, q shared by the heads."""
    Hq, Hkv, D = 6, 2, 64
    c = Case(B, [(400, n), (200, n)], Hq, Hkv, D, 32)
    T = 2 * n + 9
    wide = torch.randn(T, Hq + 5, D, device=DEV).to(torch.bfloat16)
    wide[4:4 + 2 * n, 2:2 + Hq] = c.q
    c.q_start += 4
    out = torch.full((Hq, T, D), 5.0, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    c.run(q=wide[:, 2:2 + Hq], out=out)
    c.check(out[4:])
    assert (out[:4] == 5.0).all() and (out[4 + 2 * n:] == 5.0).all()
    one = c.q[:, :1].expand(-1, Hq, -1)
    out2 = torch.zeros_like(c.q)
    c.q_start -= 4
    c.run(q=one, out=out2)
    c.check(out2, q=one)


@pytest.mark.parametrize("n", [1, 2, 140])
def test_bad_pages_lengths_and_values(B, n):
    c = Case(B, [(300, n), (300, n), (300, n), (300, n)], 4, 2, 128, 16, fill=0)
    good = c.run()
    c.table[1, 3] = 10 ** 6                                            # tokens 48 to 63 are nowhere
    c.lens[2] = 10 ** 6                                                # counts as the table's end
    c.table[2] = c.table[2, :19].repeat(2)[:c.table.shape[1]]
    out = c.run()
    assert int(c.status) == B.STATUS_BAD_INDEX
    assert out[n:2 * n].isnan().all()
    c.check(torch.cat([out[:n], good[n:3 * n], out[3 * n:]]))          # not by bits: where items are cut goes by all the lengths
    assert not out[2 * n:3 * n].isnan().any()
    # a marked token: whoever sees it, of its head
    c = Case(B, [(300, n), (300, n)], 4, 2, 128, 16)
    good = c.run()
    at = 300 - max(1, n // 2)                                           # the first query that sees it is number n - n // 2
    slot = (c.table[0, at // 16] * 16 + at % 16).view(1).to(torch.int32)
    k = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    v[0, 1, 5] = float("nan")
    B.tempo_kv_append(c.shape, k, v, slot, c.cache, c.status)
    out = c.run()
    first = at - (300 - n)
    assert out[first:n, 2:].isnan().all() and not out[:, :2].isnan().any()
    assert torch.equal(out[:first], good[:first]) and torch.equal(out[n:], good[n:])
    # queries that are not finite
    c.q[0, 1, 7] = float("inf")
    c.q[0, 0, 7] = float("nan")
    out = c.run()
    assert out[0, :2].isnan().all() and torch.equal(out[1:first, :2], good[1:first, :2])


def test_starts_that_fall_or_leave_the_rows(B):
    c = Case(B, [(100, 2), (100, 2), (100, 2)], 4, 2, 64, 16)
    c.q_start.copy_(torch.tensor([0, 4, 2, 99], device=DEV))            # four queries, none, and the last four of six
    out = c.run(max_q=4)
    assert int(c.status) == B.STATUS_BAD_INDEX and not out.isnan().any()


def test_another_stream_and_a_graph(B):
    c = Case(B, [(3000, 1), (500, 1), (40, 1)], 16, 4, 128, 64)
    d = Case(B, [(700, 300)], 8, 2, 128, 64)
    want, want_d = c.run(), d.run()
    out, out_d = torch.zeros_like(want), torch.zeros_like(want_d)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            c.run(out=out)
    d.run(out=out_d)                                                    # beside it, with a workspace of its own
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(out_d, want_d)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            c.run(out=out)
            d.run(out=out_d)
    for _ in range(4):
        out.zero_(), out_d.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out_d, want_d)
    c.lens -= 30                                                        # lengths are the device's: the captured call follows
    g.replay()
    torch.cuda.synchronize()
    c.spans = [(l - 30, n) for l, n in c.spans]
    c.k, c.v = [k[:-30] for k in c.k], [v[:-30] for v in c.v]
    c.check(out)


@pytest.mark.parametrize("n", [1, 100])
def test_a_missing_page_anywhere_in_a_tile(B, n):
    c = Case(B, [(300, n)], 4, 2, 64, 16)
    c.run()
    for page in range(10):
        table = c.table.clone()
        c.table[0, page] = -1
        out = c.run()
        first = max(0, page * 16 - (300 - n))                          # the first query that sees a token of it
        assert out[first:].isnan().all() and not out[:first].isnan().any()
        c.table.copy_(table)
    assert int(c.status) == B.STATUS_BAD_INDEX


def test_pages_beyond_4_gib_of_the_cache(B):
    D, Hkv, page, n = 128, 8, 256, 300
    shape = B.make_cache(4 * 2 ** 30 // (9 * D * page // 8 * Hkv) + 40, page, Hkv, D)
    assert B.tempo_cache_bytes(shape) > 2 ** 32
    c = Case(B, [(700, 1), (400, n)], 16, Hkv, D, page)
    c.shape, c.cache = shape, torch.zeros(B.tempo_cache_bytes(shape), dtype=torch.uint8, device=DEV)
    c.table[:] = shape.n_pages - 1 - torch.arange(c.table.numel(), dtype=torch.int32, device=DEV).view(c.table.shape)
    for b, (l, _) in enumerate(c.spans):
        k, v = (torch.randn(l, Hkv, D, device=DEV).to(torch.bfloat16) for _ in range(2))
        t = torch.arange(l, device=DEV)
        B.tempo_kv_append(shape, k, v, (c.table[b][t // page] * page + t % page).to(torch.int32), c.cache, c.status)
        c.k[b], c.v[b] = R.cached(k), R.cached(v)
    c.check(c.run())
    assert int(c.status) == 0


def test_one_row_at_any_pitch(B):
    c = Case(B, [(77, 1)], 4, 2, 64, 16)
    want = c.run()
    row = torch.zeros(2, 4 * 64 + 3, dtype=torch.bfloat16, device=DEV)
    row[0, :256] = c.q.flatten()
    q = row[:1, :256].unflatten(1, (4, 64))
    out = torch.zeros(3, 261, dtype=torch.bfloat16, device=DEV)
    assert torch.equal(c.run(q=q, out=out[:1, :256].unflatten(1, (4, 64)))[0], want[0])
    assert not out[1:].any() and not out[0, 256:].any()


@pytest.mark.parametrize("max_q", [1, 4])
def test_more_tiles_than_are_numbered(B, max_q):
    """A sequence that would need more is left out and told; the others are served."""
    c = Case(B, [(90, 3), (2000, 2000)], 4, 2, 64, 256)
    good = c.run()
    c.table = c.table[:, :1].repeat(1, 2 ** 20)                         # 2^28 tokens, all in one page
    c.lens[1] = 2 ** 28
    out = c.run(max_q=max_q)
    assert int(c.status) == B.STATUS_CAPACITY and (out[3:] == 5.0).all()
    c.check(torch.cat([out[:3], good[3:]]))


def test_as_many_sequences_as_there_may_be(B):
    spans = [(1 + 13 * b % 97, 1) for b in range(1020)] + [(90, 90), (5, 0), (333, 20), (64, 64)]
    c = Case(B, spans, 4, 1, 64, 16)
    c.check(c.run())
    assert int(c.status) == 0


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 3.0])
def test_scales(B, scale):
    c = Case(B, [(200, 70), (45, 2)], 4, 2, 64, 16)
    c.scale = scale
    c.check(c.run())
