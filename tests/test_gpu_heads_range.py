"""Heads whose squares leave the range of 32-bit floats, and angle tables that are not of unit length: tempo_qk_rotate and
tempo_kv_append against the formulas in 64 bits."""
import pytest
import torch

from tests import attention_ref as R
from tests.test_gpu_heads import B, _cache, _gen, _rand, _read, _status, _table  # noqa: F401

pytestmark = pytest.mark.gpu
DEV = "cuda"
HUGE = [1.0, 1e18, 3e18, 2e19, 1e20, 1e30, 3e38]
TINY = [1.0, 1e-16, 1e-18, 1e-19, 1e-20, 1e-22, 1e-30, 1e-38, 2e-40]


def _sized(g, T, H, D, sizes):
    """Heads of unlike size beside one another; one in four has but one element of its size, the others of it much smaller."""
    at = torch.randint(0, len(sizes), (T, H, 1), generator=g, device=DEV)
    x = _rand(g, T, H, D).double().clamp(-1, 1) * torch.tensor(sizes, dtype=torch.float64, device=DEV)[at]
    alone = torch.rand(T, H, 1, generator=g, device=DEV) < 0.25
    x = torch.where(alone & (torch.arange(D, device=DEV) != 5), x * 1e-9, x)
    return x.to(torch.bfloat16)


def _f32(eps):
    return torch.tensor(eps, dtype=torch.float32).double().item()


def _near(got, want, x, w, eps):
    """NaN where the formula has it (a head of zeros without eps: 0 / 0).  Elsewhere the rounding to bf16 (2^-8 of the value, 2^-134 for
    the least ones), 32 roundings of 2^-24 of the two products of a turned pair (of 2^-149 where they are below the normal range,
    times the inverse root)."""
    assert torch.equal(got.isnan(), want.isnan())
    x = x.double()
    r = ((x ** 2).mean(2, keepdim=True) + eps).rsqrt()
    amp = (x * r * w.double()).abs().amax(2, keepdim=True)
    tol = want.abs() * 2.0 ** -8 + amp * 2.0 ** -18 + 2.0 ** -133 + r * 2.0 ** -144
    err = (got.double() - want).abs()
    assert ((err <= tol) | want.isnan()).all(), float((err / tol).nan_to_num(0.0).max())


@pytest.mark.parametrize("sizes,eps", [(HUGE, 1e-6), (HUGE, 0.0), (TINY, 0.0), (TINY, 1e-38), (TINY, 1e-30), (TINY + HUGE, 1e-6)])
@pytest.mark.parametrize("D,rot,pairs", [(128, 128, "half"), (64, 32, "next"), (128, 90, "half"), (200, 50, "next"), (64, 0, "half")])
def test_rotate_normed_heads_of_any_size(B, sizes, eps, D, rot, pairs):
    g = _gen(D + rot)
    for T, H in ((3, 5), (300, 24)):                                    # one head of a lane group, and four again and again
        x = _sized(g, T, H, D, sizes)
        w = 1 + 0.3 * _rand(g, D)
        cs = _table(g, rot) if rot else None
        pos = torch.randint(0, 97, (T,), generator=g, device=DEV, dtype=torch.int32) if rot else None
        out, st = torch.zeros_like(x), _status()
        B.tempo_qk_rotate(x, None, pos, cs, out, None, st, q_w=w, eps=eps, interleaved=pairs == "next")
        _near(out, R.turn(x, w, pos, cs, eps=_f32(eps), interleaved=pairs == "next"), x, w, _f32(eps))
        assert int(st) == 0


@pytest.mark.parametrize("sizes,eps", [(HUGE, 1e-6), (HUGE, 0.0), (TINY, 0.0), (TINY, 1e-38), (TINY + HUGE, 1e-6)])
@pytest.mark.parametrize("D,rot,pairs", [(128, 128, "half"), (64, 64, "half"), (64, 32, "next"), (128, 90, "half"), (128, 0, "half")])
def test_append_normed_keys_of_any_size(B, sizes, eps, D, rot, pairs):
    """A key's codes do not go by the heads that share its warp: 8 key heads of unlike size, and each by itself."""
    g = _gen(7 * D + rot)
    T, Hkv, page = 400, 8, 16
    k = _sized(g, T, Hkv, D, sizes)
    k[(k == 0).all(2)] = 1.0                                            # 0 / 0 is another test's
    v = _rand(g, T, Hkv, D).to(torch.bfloat16)
    w = 1 + 0.3 * _rand(g, D)
    cs = _table(g, rot) if rot else None
    pos = torch.randint(0, 97, (T,), generator=g, device=DEV, dtype=torch.int32) if rot else None
    slots = torch.arange(T, device=DEV, dtype=torch.int32)
    turned = R.turn(k, w, pos, cs, eps=_f32(eps), interleaved=pairs == "next")
    want = R.cached(turned)
    shape, cache = _cache(B, T // page, page, Hkv, D)
    st = _status()
    B.tempo_kv_append(shape, k, v, slots, cache, st, k_w=w, positions=pos, cos_sin=cs, eps=eps, interleaved=pairs == "next")
    (kb, vb), _ = _read(B, shape, cache, slots)
    assert int(st) == 0
    assert torch.equal(kb.double(), want) and torch.equal(vb.double(), R.cached(v))
    shape, cache = _cache(B, T // page, page, 1, D)
    for h in range(Hkv):
        B.tempo_kv_append(shape, k[:, h:h + 1], v[:, h:h + 1], slots, cache, st, k_w=w, positions=pos, cos_sin=cs, eps=eps,
                          interleaved=pairs == "next")
        assert torch.equal(_read(B, shape, cache, slots)[0][0], kb[:, h:h + 1])


def test_append_keys_and_weights_so_small_that_their_product_vanishes(B):
    """Products below 32-bit floats' range: a group of them has a scale (the least one) in 64 bits, a group of zeros has none."""
    D, T = 64, 12
    k = torch.zeros(T, 1, D, dtype=torch.bfloat16, device=DEV)
    k[::2] = 9e-41
    k[1] = 1.0
    w = torch.full((D,), 1e-10, device=DEV)
    shape, cache = _cache(B, 1, 16, 1, D, fill=0)
    slots, st = torch.arange(T, device=DEV, dtype=torch.int32), _status()
    B.tempo_kv_append(shape, k, k, slots, cache, st, k_w=w)
    scales = cache[8 * D:8 * D + 2 * T * (D // 32)].view(T, D // 32, 2)[:, :, 0]
    want = (k[:, 0].view(T, D // 32, 32) != 0).any(2)
    assert torch.equal(scales != 0, want) and (scales[::2] == 1).all() and int(st) == 0


@pytest.mark.parametrize("size", [1.35, 50.0, 0.02])
@pytest.mark.parametrize("D,rot,norm,pairs", [(128, 128, True, "half"), (64, 64, False, "next"), (128, 96, True, "next"), (64, 50, True, "half")])
def test_codes_with_tables_of_other_lengths(B, size, D, rot, norm, pairs):
    """cos and sin multiplied by a factor, as a caller may do to scale the scores of long contexts."""
    g = _gen(D + rot + norm)
    T, Hkv = 4000, 8
    k = (_rand(g, T, Hkv, D) * (0.01 + 4 * torch.rand(T, Hkv, 1, generator=g, device=DEV))).to(torch.bfloat16)
    v = _rand(g, T, Hkv, D).to(torch.bfloat16)
    w = (1 + 0.3 * _rand(g, D)).to(torch.bfloat16) if norm else None
    cs = _table(g, rot) * size
    pos = torch.randint(0, 97, (T,), generator=g, device=DEV, dtype=torch.int32)
    shape, cache = _cache(B, T // 16, 16, Hkv, D)
    slots = torch.randperm(T, generator=g, device=DEV).to(torch.int32)
    st = _status()
    B.tempo_kv_append(shape, k, v, slots, cache, st, k_w=w, positions=pos, cos_sin=cs, interleaved=pairs == "next")
    (kb, vb), _ = _read(B, shape, cache, slots)
    assert torch.equal(kb.double(), R.cached(R.turn(k, w, pos, cs, interleaved=pairs == "next")))
    assert torch.equal(vb.double(), R.cached(v)) and int(st) == 0


@pytest.mark.parametrize("size", [1.0, 30.0, 1000.0])
@pytest.mark.parametrize("D,rot,norm,pairs", [(128, 128, True, "half"), (128, 128, False, "half"), (64, 64, False, "next"), (64, 60, False, "next"),
                                              (64, 50, False, "half")])
def test_codes_where_the_products_of_a_pair_cancel(B, size, D, rot, norm, pairs):
    """Equal elements turned by an eighth of a circle: half of the results are small, and off by what their products are."""
    g = _gen(D + rot + norm)
    T, Hkv = 4000, 4
    one = _rand(g, T, Hkv, rot // 2).to(torch.bfloat16)
    k = _rand(g, T, Hkv, D).to(torch.bfloat16)
    k[:, :, :rot] = one.repeat_interleave(2, 2) if pairs == "next" else torch.cat([one, one], 2)
    if pairs == "next":                                                 # both results of a pair share a group: the sums are made small too
        k[:, :, 1:rot:2] *= torch.where(torch.rand(T, Hkv, 1, generator=g, device=DEV) < 0.5, 1.0, -1.0).to(torch.bfloat16)
    w = torch.full((D,), 1.25, device=DEV) if norm else None
    a = torch.pi / 4 + 0.003 * _rand(g, 97, rot // 2).double()
    cs = (size * torch.cat([a.cos(), a.sin()], 1)).float()
    pos = torch.randint(0, 97, (T,), generator=g, device=DEV, dtype=torch.int32)
    shape, cache = _cache(B, T // 16, 16, Hkv, D)
    slots = torch.randperm(T, generator=g, device=DEV).to(torch.int32)
    st = _status()
    B.tempo_kv_append(shape, k, k, slots, cache, st, k_w=w, positions=pos, cos_sin=cs, interleaved=pairs == "next")
    (kb, vb), _ = _read(B, shape, cache, slots)
    assert torch.equal(kb.double(), R.cached(R.turn(k, w, pos, cs, interleaved=pairs == "next")))
    assert torch.equal(vb.double(), R.cached(k)) and int(st) == 0
