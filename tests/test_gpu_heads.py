"""tempo_qk_rotate, tempo_kv_append and tempo_kv_read against the formulas in 64 bits."""
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


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _table(g, rot, n_pos=97):
    a = _rand(g, n_pos, rot // 2) * 50
    return torch.cat([a.cos(), a.sin()], 1)


def _status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def _close(got, want, amp):
    """bf16 rounding (2^-8 of the value) and about 32 roundings of 2^-24 of the two products of a turned pair."""
    tol = want.abs() * 2.0 ** -8 + amp * 2.0 ** -18
    assert ((got.to(torch.float64) - want).abs() <= tol).all(), float(((got.to(torch.float64) - want).abs() - tol).max())


def _amp(x, w):
    """Largest element of each normed head, which bounds what a turned pair adds up."""
    return R.turn(x, w, None, None).abs().amax(2, keepdim=True)


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,pairs,norm", [
    (1, 64, 4, 128, 128, "half", "bf16"), (1, 1, 1, 8, 0, "half", None), (3, 5, 2, 64, 64, "next", "f32"),
    (17, 3, 3, 96, 96, "half", "bf16"), (5, 2, 1, 96, 24, "next", None), (33, 7, 1, 256, 64, "half", "f32"),
    (2, 1, 1, 24, 22, "half", "bf16"), (9, 4, 2, 40, 10, "next", "bf16"), (130, 16, 2, 128, 6, "half", None),
    (1031, 12, 2, 64, 32, "next", "bf16"), (4, 2, 2, 200, 200, "half", "bf16"), (11, 0, 3, 128, 128, "half", "bf16"),
    (11, 3, 0, 72, 72, "half", "bf16"), (2, 9, 1, 16, 2, "next", None)])
def test_rotate(B, T, Hq, Hkv, D, rot, pairs, norm):
    g = _gen(T * 1000 + D + rot)
    q, k = (_rand(g, T, H, D).to(torch.bfloat16) if H else None for H in (Hq, Hkv))
    dt = torch.float32 if norm == "f32" else torch.bfloat16
    q_w, k_w = ((1 + 0.3 * _rand(g, D)).to(dt) if norm else None for _ in range(2))
    cs = _table(g, rot) if rot else None
    pos = torch.randint(0, 97, (T,), generator=g, device=DEV, dtype=torch.int32) if rot else None
    qo, ko = (None if x is None else torch.full_like(x, 7.0) for x in (q, k))
    st = _status()
    B.tempo_qk_rotate(q, k, pos, cs, qo, ko, st, q_w=q_w, k_w=k_w, interleaved=pairs == "next")
    for x, w, got in ((q, q_w, qo), (k, k_w, ko)):
        if x is not None:
            _close(got, R.turn(x, w, pos, cs, interleaved=pairs == "next"), _amp(x, w))
    assert int(st) == 0


@pytest.mark.parametrize("pairs", ["half", "next"])
@pytest.mark.parametrize("D,rot,layout", [(128, 128, "qkv"), (128, 20, "qkv"), (64, 64, "odd"), (96, 26, "odd"), (128, 128, "heads first")])
def test_rotate_in_place_of_strided_rows(B, D, rot, pairs, layout):
    """q and k as parts of one projection's row, at odd addresses, and with the heads outermost; nothing else is written."""
    T, Hq, Hkv = 37, 6, 2
    g = _gen(D + rot)
    if layout == "heads first":
        buf = _rand(g, Hq + Hkv + 1, T, D).to(torch.bfloat16)
        view = buf.transpose(0, 1)
    else:
        pad = 3 if layout == "odd" else 0
        buf = _rand(g, T, (Hq + Hkv + 1) * D + 2 * pad).to(torch.bfloat16)
        view = buf[:, pad:pad + (Hq + Hkv + 1) * D].unflatten(1, (-1, D))
    before = buf.clone()
    q, k, v = view[:, :Hq], view[:, Hq:Hq + Hkv], view[:, Hq + Hkv:]
    w = (1 + 0.3 * _rand(g, D + 1))[1:]
    cs = _table(g, rot)
    pos = torch.randint(0, 97, (T,), generator=g, device=DEV, dtype=torch.int32)
    want = [R.turn(x, w, pos, cs, interleaved=pairs == "next") for x in (q, k)]
    amp = [_amp(x, w) for x in (q, k)]
    n_valid = torch.tensor([30], dtype=torch.int32, device=DEV)
    B.tempo_qk_rotate(q, k, pos, cs, q, k, _status(), q_w=w, k_w=w, interleaved=pairs == "next", n_valid=n_valid)
    for x, y, a in zip((q, k), want, amp):
        _close(x[:30], y[:30], a[:30])
        assert torch.equal(x[30:], (before.transpose(0, 1) if layout == "heads first" else before[:, pad:pad + (Hq + Hkv + 1) * D].unflatten(1, (-1, D)))
                           [30:, (0 if x is q else Hq):(Hq if x is q else Hq + Hkv)])
    q.zero_(), k.zero_()
    was = before.clone()
    (was.transpose(0, 1) if layout == "heads first" else was[:, pad:pad + (Hq + Hkv + 1) * D].unflatten(1, (-1, D)))[:, :Hq + Hkv] = 0
    assert torch.equal(buf, was)


def test_rotate_positions_outside_the_table_and_broadcast_rows(B):
    g = _gen(3)
    row = _rand(g, 1, 2, 64).to(torch.bfloat16)
    q = row.expand(5, 2, 64)                                            # one row read five times
    cs = _table(g, 64, 10)
    pos = torch.tensor([-1, 0, 9, 10, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    out, st = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device=DEV), _status()
    B.tempo_qk_rotate(q, None, pos, cs, out, None, st)
    _close(out, R.turn(q, None, pos, cs), _amp(q, None))
    assert int(st) == B.STATUS_BAD_INDEX


def _cache(B, n_pages, page, Hkv, D, fill=0xA5):
    shape = B.make_cache(n_pages, page, Hkv, D)
    return shape, torch.full((B.tempo_cache_bytes(shape),), fill, dtype=torch.uint8, device=DEV)


def _read(B, shape, cache, slots):
    out = [torch.full((len(slots), shape.Hkv, shape.D), 3.0, dtype=torch.float16, device=DEV) for _ in range(2)]
    st = _status()
    B.tempo_kv_read(shape, cache, slots, *out, st)
    return out, int(st)


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,pairs,norm,page", [
    (1, 4, 1, 128, 128, "half", True, 64), (7, 32, 8, 128, 128, "half", True, 16), (701, 14, 2, 64, 64, "half", False, 16),
    (300, 0, 3, 64, 16, "next", True, 128), (333, 2, 1, 128, 50, "half", True, 32), (64, 6, 6, 128, 0, "half", True, 256),
    (515, 8, 4, 128, 128, "next", True, 64)])
def test_append_and_read_back(B, T, Hq, Hkv, D, rot, pairs, norm, page):
    g = _gen(T + D)
    qkv = (_rand(g, T, Hq + 2 * Hkv, D) * torch.where(torch.rand(Hq + 2 * Hkv, D, generator=g, device=DEV) < 0.03, 9.0, 1.0)).to(torch.bfloat16)
    q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
    q_w, k_w = ((1 + 0.3 * _rand(g, D)) if norm else None for _ in range(2))
    cs = _table(g, rot) if rot else None
    pos = torch.randint(0, 97, (T,), generator=g, device=DEV, dtype=torch.int32) if rot else None
    n_pages = T // page + 3
    slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:T].to(torch.int32)
    shape, cache = _cache(B, n_pages, page, Hkv, D)
    before = _read(B, shape, cache, torch.arange(n_pages * page, device=DEV, dtype=torch.int32))[0]
    qo = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV) if Hq else None
    st = _status()
    B.tempo_kv_append(shape, k, v, slots, cache, st, k_w=k_w, positions=pos, cos_sin=cs, q=q if Hq else None, q_w=q_w, q_out=qo,
                      interleaved=pairs == "next")
    (kb, vb), bad = _read(B, shape, cache, slots)
    assert int(st) == 0 and bad == 0
    assert torch.equal(kb.to(torch.float64), R.cached(R.turn(k, k_w, pos, cs, interleaved=pairs == "next")))
    assert torch.equal(vb.to(torch.float64), R.cached(v))
    if Hq:
        _close(qo, R.turn(q, q_w, pos, cs, interleaved=pairs == "next"), _amp(q, q_w))
    # tokens that were not appended are as before
    rest = torch.ones(n_pages * page, dtype=torch.bool, device=DEV)
    rest[slots.long()] = False
    at = torch.nonzero(rest)[:, 0].to(torch.int32)
    for x, y in zip(_read(B, shape, cache, at)[0], before):
        assert torch.equal(x, y[rest])


def _bf16_bits(*bits):
    return torch.tensor([b - 65536 if b > 32767 else b for b in bits], dtype=torch.int16, device=DEV).view(torch.bfloat16)


@pytest.mark.parametrize("D", [64, 128])
def test_append_of_values_next_to_borders(B, D):
    """Without norm or rotation every quotient is exact: halves between two codes, groups of one sign, zeros, huge and tiny values."""
    rows = []
    for s in (1.0, 0.1015625, 12.0, 768.0, 2.0 ** -17, 3 * 2.0 ** -17):
        rows.append(torch.arange(32, device=DEV) * 0.5 * s)                    # 0 to 15.5 s: halves
        rows.append((torch.arange(32, device=DEV) - 15) * 0.5 * s)
        rows.append(-(torch.arange(32, device=DEV) % 16) * s)
        rows.append(15 * s + torch.zeros(32, device=DEV))
    rows.append(torch.zeros(32, device=DEV))
    rows.append(torch.full((32,), -0.0, device=DEV))
    rows.append(torch.tensor([15.0] + [-2.0 ** -120] * 31, device=DEV))        # a hair beyond a scale's span
    rows.append(torch.tensor([3e38, -3e38] + [1000.0] * 30, device=DEV))       # beyond the largest scale
    rows.append(torch.full((32,), 2.0 ** -130, device=DEV))
    rows.append(_bf16_bits(*range(0x3F80, 0x3FA0)).float())
    x = torch.stack(rows).to(torch.bfloat16)
    n = x.shape[0] // (D // 32) * (D // 32)
    x = x[:n].reshape(-1, 1, D)
    T = x.shape[0]
    shape, cache = _cache(B, 2, 32, 1, D)
    slots = torch.arange(T, device=DEV, dtype=torch.int32)
    st = _status()
    B.tempo_kv_append(shape, x, x.flip(0).contiguous(), slots, cache, st)
    (k, v), _ = _read(B, shape, cache, slots)
    assert int(st) == 0
    assert torch.equal(k.to(torch.float64), R.cached(x)) and torch.equal(v.to(torch.float64), R.cached(x.flip(0)))


def test_append_skips_marks_and_reports(B):
    g = _gen(5)
    D, Hkv = 64, 2
    k, v = (_rand(g, 8, Hkv, D).to(torch.bfloat16) for _ in range(2))
    k[1, 0, 3] = float("nan")
    v[2, 1, 40] = float("inf")
    shape, cache = _cache(B, 1, 16, Hkv, D, fill=0)
    slots = torch.tensor([0, 1, 2, -1, 16, 5, 6, 7], dtype=torch.int32, device=DEV)
    n_valid = torch.tensor([7], dtype=torch.int32, device=DEV)
    st = _status()
    B.tempo_kv_append(shape, k, v, slots, cache, st, n_valid=n_valid)
    assert int(st) == B.STATUS_BAD_INDEX | B.STATUS_BAD_VALUE
    (kb, vb), st = _read(B, shape, cache, torch.tensor([0, 1, 2, 5, 6, 7, 3, -1, 16], dtype=torch.int32, device=DEV))
    assert st == B.STATUS_BAD_INDEX
    want_v = v.clone()
    want_v[2, 1, 40] = 0
    want_k, want_v = R.cached(k.nan_to_num(0.0)), R.cached(want_v)
    at = [0, 1, 2, 5, 6]
    assert torch.equal(vb[:5].to(torch.float64), want_v[at])
    marked = torch.zeros(9, Hkv, dtype=torch.bool, device=DEV)
    marked[1, 0] = marked[2, 1] = True
    assert kb[marked].isnan().all() and not kb[~marked].isnan().any()
    assert torch.equal(kb[:5].to(torch.float64)[~marked[:5]], want_k[at][~marked[:5]])
    assert (kb[5:] == 0).all() and (vb[5:] == 0).all()                   # not live, never written, no slot, beyond the cache


def test_offsets_beyond_32_bits(B):
    """A cache of more than 4 GiB: the last page's rows come back, the first page's stay."""
    D, Hkv, page = 128, 8, 256
    n_pages = 4 * 2 ** 30 // (9 * D * page // 8 * Hkv) + 40
    shape = B.make_cache(n_pages, page, Hkv, D)
    assert B.tempo_cache_bytes(shape) > 2 ** 32
    cache = torch.zeros(B.tempo_cache_bytes(shape), dtype=torch.uint8, device=DEV)
    g = _gen(9)
    k, v = (_rand(g, 4, Hkv, D).to(torch.bfloat16) for _ in range(2))
    slots = torch.tensor([n_pages * page - 1, n_pages * page - 2, (n_pages - 30) * page, 3], dtype=torch.int32, device=DEV)
    B.tempo_kv_append(shape, k, v, slots, cache, _status())
    (kb, vb), _ = _read(B, shape, cache, slots)
    assert torch.equal(kb.to(torch.float64), R.cached(k)) and torch.equal(vb.to(torch.float64), R.cached(v))
    assert int((cache != 0).sum()) <= 4 * Hkv * 2 * 72


@pytest.mark.parametrize("D,norm,pairs", [(128, True, "half"), (64, False, "next"), (128, False, "half")])
def test_codes_of_many_keys_are_the_formulas(B, D, norm, pairs):
    """A few of a million elements lie so near a border that 32 bits would not tell on which side."""
    g = _gen(D + norm)
    T, Hkv = 4000, 8
    k = (_rand(g, T, Hkv, D) * (0.01 + 4 * torch.rand(T, Hkv, 1, generator=g, device=DEV))).to(torch.bfloat16)
    v = _rand(g, T, Hkv, D).to(torch.bfloat16)
    w = (1 + 0.3 * _rand(g, D)).to(torch.bfloat16) if norm else None
    cs = _table(g, D)
    pos = torch.randint(0, 97, (T,), generator=g, device=DEV, dtype=torch.int32)
    shape, cache = _cache(B, T // 16, 16, Hkv, D)
    slots = torch.randperm(T, generator=g, device=DEV).to(torch.int32)
    B.tempo_kv_append(shape, k, v, slots, cache, _status(), k_w=w, positions=pos, cos_sin=cs, interleaved=pairs == "next")
    (kb, vb), _ = _read(B, shape, cache, slots)
    assert torch.equal(kb.to(torch.float64), R.cached(R.turn(k, w, pos, cs, interleaved=pairs == "next")))
    assert torch.equal(vb.to(torch.float64), R.cached(v))
