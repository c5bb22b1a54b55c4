"""The extension module that marshals the short calls refuses what it cannot pass on, without a GPU: nothing is launched."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2608_13057_b200 import build
    build.build()
    from paper_2608_13057_b200 import binding
    return binding


def test_cpu_tensors_and_other_objects_are_refused(B):
    r, w, x = torch.zeros(4, 8), torch.ones(8), torch.zeros(4, 8, dtype=torch.bfloat16)
    s = B.make_shape(4, 2, 8, 2, 1, 128, 128, 128)
    for f in (lambda: B.tempo_norm_in(r, w, x), lambda: B.tempo_norm_in(5, w, x), lambda: B.tempo_norm_in(None, w, x),
              lambda: B.tempo_norm_out(x, r, r), lambda: B.tempo_norm_out(x, r, r, gate=torch.ones(1)),
              lambda: B.tempo_route(s, x, x, None, None, r, r, r), lambda: B.tempo_few_ffn(s, x, r, r, None, r, r, x, r, r),
              lambda: B.tempo_few_ffn_bf16(s, "x", r, r, None, r, r, x, r, r)):
        with pytest.raises(B.TempoError):
            f()


def test_the_module_itself_checks_its_argument_counts(B):
    from paper_2608_13057_b200 import _marshal
    for name in ("bind", "norm_in", "norm_out", "route", "few"):
        with pytest.raises(TypeError):
            getattr(_marshal, name)(1, 2, 3)


def test_c_entries_report_what_the_host_can_see(B):
    """NULL pointers and shapes outside the documented limits, straight through the C ABI."""
    import ctypes
    lib, null = B._lib, ctypes.c_void_p(0)
    s = B.make_shape(4, 2, 8, 2, 1, 128, 128, 128)
    one = ctypes.c_void_p(256)                           # never dereferenced: every call below is refused before a launch
    route = lambda shape, score=0, x=one, ids=one: lib.tempo_route(
        ctypes.byref(shape), ctypes.c_int32(score), ctypes.c_int32(1), ctypes.c_float(1.0), x, one, null, null, ids, one, one, null)
    assert route(s, x=null) == -1 and route(s, ids=null) == -1
    assert route(s, score=2) == -3
    assert route(B.make_shape(4, 9, 8, 2, 1, 128, 128, 128)) == -2          # k > E
    assert route(B.make_shape(4, 2, 513, 2, 1, 128, 128, 128)) == -3
    assert route(s, x=ctypes.c_void_p(264)) == -5
    few = lambda shape, x=one, packed=one, ws=one: lib.tempo_few_ffn(
        ctypes.byref(shape), x, one, one, null, one, packed, one, one, ws, null)
    assert few(s, x=null) == -1 and few(s, ws=null) == -1
    assert few(B.make_shape(65, 2, 8, 2, 1, 128, 128, 128)) == -3
    assert few(B.make_shape(64, 17, 20, 2, 1, 128, 128, 128)) == -3         # more than 1024 pairs
    assert few(s, packed=ctypes.c_void_p(512 + 16)) == -5 and few(s, ws=ctypes.c_void_p(512 + 16)) == -5

    class Norm(ctypes.Structure):
        _fields_ = ([(n, ctypes.c_int32) for n in ("T", "d", "kind", "stream_f32", "param_f32", "gate_f32")]
                    + [(n, ctypes.c_int64) for n in ("ld_y", "ld_r", "ld_r_out", "ld_x", "gate_row", "gate_col")]
                    + [(n, ctypes.c_float) for n in ("eps", "r_scale", "y_scale")])

    def norm(T=2, d=64, kind=0, ld=64, r=one, w=one):
        a = Norm(T=T, d=d, kind=kind, ld_r=ld, ld_x=ld)
        return lib.tempo_norm_in(ctypes.byref(a), r, w, null, null, one, null)
    assert norm(T=0) == -2 and norm(d=0) == -2 and norm(ld=63) == -2 and norm(kind=5) == -3
    assert norm(d=16385, ld=16385) == -3 and norm(r=null) == -1 and norm(w=null) == -1
    assert norm(w=ctypes.c_void_p(257)) == -5
    assert b"aligned" in lib.tempo_status_string(-5)
