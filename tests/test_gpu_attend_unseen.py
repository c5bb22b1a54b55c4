"""tempo_attend: what lies in tokens that a query does not see says nothing in its output, whatever its bytes.  Page 0, which stands in
for pages that are not in the cache, is no sequence's here and was never written."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_attend import Case
from tests.test_gpu_attend_many import Followed

pytestmark = pytest.mark.gpu
DEV = "cuda"
FILLS = [0xFF, 0xF8, 0xF7, 0xC5, 0x7B]        # value scales that are NaN, infinite, beyond what is ever stored; an ordinary one


@pytest.fixture(scope="module", params=["little work", "much work"])
def B(request):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13057_b200 import binding
    return binding if request.param == "little work" else Followed(binding)


def _without_page_0(c, fill):
    """Page 0's tokens go to a spare page; it holds `fill` from then on."""
    pages = c.cache.view(c.shape.n_pages, -1)
    used = set(c.table[c.table < 2 ** 30].tolist())
    spare = max(set(range(c.shape.n_pages)) - used)
    if 0 in used:
        pages[spare] = pages[0]
        c.table[c.table == 0] = spare
    pages[0] = fill


@pytest.mark.parametrize("fill", FILLS)
@pytest.mark.parametrize("L,n,Hq,Hkv,D,page", [(300, 20, 4, 2, 64, 16), (290, 3, 4, 2, 128, 16), (258, 4, 32, 4, 128, 64), (300, 100, 4, 2, 64, 16),
                                               (300, 200, 12, 2, 128, 32), (300, 90, 6, 1, 128, 128)])
def test_a_missing_page_that_some_queries_do_not_see(B, fill, L, n, Hq, Hkv, D, page):
    c = Case(B, [(L, n), (70, 2)], Hq, Hkv, D, page, fill=fill)
    _without_page_0(c, fill)
    good = c.run()
    c.check(good)
    tried = 0
    for at in range((L - n) // page, -(-L // page)):
        table = c.table.clone()
        c.table[0, at] = -1
        out = c.run()
        c.table.copy_(table)
        first = min(n, max(0, at * page - (L - n)))                   # the first query that sees a token of it
        assert out[first:n].isnan().all()
        assert torch.equal(out[:first], good[:first]) and torch.equal(out[n:], good[n:]), (at, first)
        tried += first > 0
    assert tried > 0 and int(c.status) == B.STATUS_BAD_INDEX


@pytest.mark.parametrize("fill", FILLS)
@pytest.mark.parametrize("n,Hq,Hkv,D,page", [(7, 4, 2, 64, 16), (8, 32, 4, 128, 64), (150, 12, 2, 128, 32), (33, 6, 6, 64, 256)])
def test_tokens_that_were_not_appended(B, fill, n, Hq, Hkv, D, page):
    """The newest tokens of a sequence are counted in its length, and their keys and values were never written."""
    c = Case(B, [(300, n), (90, 1)], Hq, Hkv, D, page, fill=fill)
    good = c.run()
    for missing in {1, 2, n // 2, n - 1}:
        cache = c.cache.clone()
        c.cache.fill_(fill)
        for b, (l, _) in enumerate(c.spans):                            # all again, without the last `missing` of the first sequence
            t = torch.arange(l, device=DEV)
            slots = (c.table[b][t // page] * page + t % page).to(torch.int32)
            if b == 0:
                slots[l - missing:] = -1
            g = torch.Generator(device=DEV).manual_seed(b)
            k, v = (torch.randn(l, Hkv, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
            B.tempo_kv_append(c.shape, k, v, slots, c.cache, c.status)
            c.k[b], c.v[b] = R.cached(k), R.cached(v)
        out = c.run()
        seen = n - missing                                              # queries that see none of them
        for b, rows in ((0, slice(0, seen)), (1, slice(n, n + 1))):
            l = 300 if b == 0 else 90
            want, spread, off = R.attend(c.q[c.starts[b]:c.starts[b] + (n if b == 0 else 1)], c.k[b], c.v[b], c.scale, l - (n if b == 0 else 1))
            err, tol = (out[rows].double() - want[:rows.stop - rows.start]).abs(), R.attend_tolerance(want, spread, off, l)[:rows.stop - rows.start]
            assert (err <= tol).all(), (missing, b)
        c.cache.copy_(cache)
    assert torch.equal(c.run(), good) and int(c.status) == 0
