"""What the entries of the attention half refuse, without a GPU: nothing is launched."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2608_13057_b200 import build
    build.build()
    from paper_2608_13057_b200 import binding
    return binding


def test_cpu_tensors_and_other_objects_are_refused(B):
    s = B.make_cache(4, 16, 2, 64)
    x, i = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    u, w = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(3, 64)
    for f in (lambda: B.tempo_qk_rotate(x, x, i, w, x, x, i), lambda: B.tempo_qk_rotate(None, None, None, None, None, None, i),
              lambda: B.tempo_kv_append(s, x, x, i, u, i), lambda: B.tempo_kv_append(s, None, x, i, u, i),
              lambda: B.tempo_kv_read(s, u, i, x.half(), x.half(), i), lambda: B.tempo_kv_read(s, 3, i, x.half(), x.half(), i),
              lambda: B.tempo_attend(s, x, u, i[None], i, x, i, u), lambda: B.tempo_attend(s, x, u, None, None, x, i, u)):
        with pytest.raises(B.TempoError):
            f()


def test_the_module_itself_checks_its_argument_counts(B):
    from paper_2608_13057_b200 import _marshal
    for name in ("qk_rotate", "kv_append", "kv_read", "attend"):
        with pytest.raises(TypeError):
            getattr(_marshal, name)(1, 2, 3)


def test_sizes(B):
    assert B.tempo_cache_bytes(B.make_cache(3, 64, 4, 128)) == 3 * 64 * 4 * 2 * (128 // 2 + 128 // 16)
    assert B.tempo_cache_bytes(B.make_cache(5, 16, 1, 64)) == 5 * 16 * 2 * (32 + 4)
    out = ctypes.c_size_t(0)
    for shape, rc in ((B.make_cache(0, 64, 4, 128), -2), (B.make_cache(3, 64, 0, 128), -2), (B.make_cache(3, 48, 4, 128), -3),
                      (B.make_cache(3, 8, 4, 128), -3), (B.make_cache(3, 512, 4, 128), -3), (B.make_cache(3, 64, 4, 96), -3),
                      (B.make_cache(2 ** 30, 64, 4, 128), -3), (B.make_cache(2 ** 22, 256, 64, 128), -3)):
        assert B._lib.tempo_cache_bytes(ctypes.byref(shape), ctypes.byref(out)) == rc
    assert B._lib.tempo_cache_bytes(ctypes.byref(B.make_cache(1, 16, 1, 64)), None) == -1
    assert B.tempo_attend_workspace_bytes(B.make_cache(3, 64, 4, 128), 64) % 256 == 0
    with pytest.raises(B.TempoError):
        B.tempo_attend_workspace_bytes(B.make_cache(3, 64, 4, 128), 30)


class Heads(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("T", "Hq", "Hkv", "D", "rot", "interleaved", "n_pos", "w_f32")]
                + [(n, ctypes.c_int64) for n in ("ld_q", "hd_q", "ld_k", "hd_k", "ld_v", "hd_v", "ld_q_out", "hd_q_out", "ld_k_out", "hd_k_out")]
                + [("eps", ctypes.c_float)])


class Attention(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "T", "Hq", "max_q", "max_pages")]
                + [(n, ctypes.c_int64) for n in ("ld_q", "hd_q", "ld_out", "hd_out")] + [("scale", ctypes.c_float)])


ONE, NULL = ctypes.c_void_p(256), ctypes.c_void_p(0)      # never dereferenced: every call below is refused before a launch


def heads(**kw):
    D = kw.get("D", 64)
    a = dict(T=3, Hq=4, Hkv=2, D=64, rot=64, n_pos=9)
    a.update({f"ld_{x}": 4 * D for x in ("q", "k", "v", "q_out", "k_out")})
    a.update({f"hd_{x}": D for x in ("q", "k", "v", "q_out", "k_out")})
    a.update(kw)
    return Heads(**a)


def test_rotate_and_append_report_what_the_host_can_see(B):
    lib = B._lib

    def rotate(q=ONE, k=ONE, w=ONE, pos=ONE, table=ONE, out=ONE, status=ONE, **kw):
        return lib.tempo_qk_rotate(ctypes.byref(heads(**kw)), q, k, w, w, pos, table, NULL, out, out, status, NULL)
    assert lib.tempo_qk_rotate(None, *[ONE] * 11) == -1
    for bad in (dict(T=0), dict(Hq=-1), dict(Hq=0, Hkv=0), dict(D=60), dict(rot=66), dict(rot=5), dict(n_pos=0), dict(ld_q=-1),
                dict(hd_q_out=32), dict(ld_k_out=0), dict(ld_q_out=64 * 4 - 1), dict(D=0)):
        assert rotate(**bad) == -2, bad
    assert rotate(D=264, rot=0) == -3 and rotate(interleaved=2) == -3
    for bad in (dict(q=NULL), dict(k=NULL), dict(pos=NULL), dict(table=NULL), dict(out=NULL), dict(status=NULL)):
        assert rotate(**bad) == -1, bad
    assert rotate(q=ctypes.c_void_p(257)) == -5 and rotate(table=ctypes.c_void_p(258)) == -5 and rotate(w=ctypes.c_void_p(258), w_f32=1) == -5

    def append(shape=B.make_cache(4, 16, 2, 64), k=ONE, v=ONE, slots=ONE, cache=ONE, **kw):
        return lib.tempo_kv_append(ctypes.byref(heads(**kw)), ctypes.byref(shape), ONE, k, v, ONE, ONE, ONE, ONE, slots, NULL, ONE, cache, ONE, NULL)
    for bad in (dict(k=NULL), dict(v=NULL), dict(slots=NULL), dict(cache=NULL)):
        assert append(**bad) == -1, bad
    assert append(Hkv=0) == -2 and append(Hkv=3) == -2 and append(D=128, rot=64) == -2 and append(shape=B.make_cache(4, 20, 2, 64)) == -3
    assert append(cache=ctypes.c_void_p(264)) == -5 and append(ld_v=-1) == -2

    def read(shape=B.make_cache(4, 16, 2, 64), cache=ONE, n=3, k=ONE):
        return lib.tempo_kv_read(ctypes.byref(shape), cache, ONE, ctypes.c_int32(n), k, ONE, ONE, NULL)
    assert read(n=0) == -2 and read(cache=NULL) == -1 and read(k=NULL) == -1 and read(k=ctypes.c_void_p(264)) == -5
    assert read(shape=B.make_cache(4, 16, 2, 32)) == -3


def test_attend_reports_what_the_host_can_see(B):
    lib = B._lib

    def attend(shape=B.make_cache(4, 16, 2, 64), q=ONE, table=ONE, starts=NULL, out=ONE, work=ONE, **kw):
        a = dict(B=3, T=3, Hq=4, max_q=1, max_pages=2, ld_q=256, hd_q=64, ld_out=256, hd_out=64, scale=0.125)
        a.update(kw)
        return lib.tempo_attend(ctypes.byref(Attention(**a)), ctypes.byref(shape), q, ONE, table, ONE, starts, out, ONE, work, NULL)
    for bad in (dict(q=NULL), dict(table=NULL), dict(out=NULL), dict(work=NULL)):
        assert attend(**bad) == -1, bad
    for bad in (dict(B=0), dict(T=0), dict(Hq=3), dict(Hq=0), dict(max_q=0), dict(max_pages=0), dict(T=5), dict(ld_out=128), dict(hd_out=0), dict(ld_q=-8)):
        assert attend(**bad) == -2, bad
    for bad in (dict(B=1025, T=1025), dict(max_pages=2 ** 30), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attend(**bad) == -3, bad
    for bad in (dict(q=ctypes.c_void_p(264)), dict(ld_q=260), dict(hd_out=68, ld_out=300), dict(work=ctypes.c_void_p(384)), dict(table=ctypes.c_void_p(258))):
        assert attend(**bad) == -5, bad
    assert attend(shape=B.make_cache(4, 16, 2, 256)) == -3


def test_the_layer_refuses_what_does_not_fit(B, monkeypatch):
    from paper_2608_13057_b200 import layer
    calls = []
    for name in ("tempo_kv_append", "tempo_attend"):
        monkeypatch.setattr(B, name, lambda *a, name=name, **kw: calls.append((name, a, kw)))
    a = layer.Attention(4, 16, 4, 2, 64, 10, device="cpu")
    qkv, i = torch.zeros(8, 8 * 64, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.int32)
    out = torch.zeros(8, 256, dtype=torch.bfloat16)
    assert a.forward(qkv, i, i, i[None], i, out, q_start=i, max_q=8) is out
    (n0, a0, k0), (n1, a1, k1) = calls
    assert n0 == "tempo_kv_append" and n1 == "tempo_attend" and "positions" not in k0 and k1["max_q"] == 8
    assert k0["q"].shape == (8, 4, 64) and a0[1].shape == a0[2].shape == (8, 2, 64) and k0["q_out"].data_ptr() == a1[1].data_ptr()
    assert a0[2].storage_offset() == 6 * 64 and a1[5].shape == (8, 4, 64)
    with pytest.raises(B.TempoError, match="11"):
        a.forward(torch.zeros(11, 512, dtype=torch.bfloat16), i, i, i[None], i, out)
    with pytest.raises(B.TempoError):
        layer.Attention(4, 16, 5, 2, 64, 10, device="cpu")
