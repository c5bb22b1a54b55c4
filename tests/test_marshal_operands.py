"""The extension module that marshals the short calls, without a GPU: operands on several devices are refused before an address
is taken, and an argument that cannot be converted raises its own error.  Tensors of two GPUs are fakes without memory."""
import ctypes
from unittest import mock

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode


@pytest.fixture(scope="module")
def B():
    from paper_2608_13057_b200 import build
    build.build()
    from paper_2608_13057_b200 import binding
    return binding


def fakes(*names):
    """The named operands of a small call as fake tensors on the first GPU; those in `names` on the second."""
    bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
    sizes = dict(r=((4, 128), bf), w=((128,), bf), x=((4, 128), bf), y=((4, 128), bf), ro=((4, 128), bf), gate=((4, 1), f32),
                 n_valid=((1,), i32), wr=((8, 128), bf), bias=((8,), f32), ids=((4, 2), i32), tw=((4, 2), f32), st=((1,), i32),
                 rmap=((8, 1), i32), packed=((1 << 20,), u8), ws=((1 << 24,), u8))
    # a fake tensor brings up its GPU where there is one, and a second GPU need not be there
    with mock.patch("torch._subclasses.fake_tensor.init_gpu_context"), FakeTensorMode():
        return {n: torch.empty(s, dtype=t, device="cuda:1" if n in names else "cuda:0") for n, (s, t) in sizes.items()}


CALLS = {
    "norm_in": (("r", "w", "x", "n_valid"), lambda B, s, o: B.tempo_norm_in(o["r"], o["w"], o["x"], b=o["w"], n_valid=o["n_valid"])),
    "norm_out": (("y", "r", "ro", "w", "gate", "x", "n_valid"), lambda B, s, o: B.tempo_norm_out(
        o["y"], o["r"], o["ro"], post_w=o["w"], gate=o["gate"], next_w=o["w"], x_out=o["x"], n_valid=o["n_valid"])),
    "route": (("x", "wr", "bias", "n_valid", "ids", "tw", "st"), lambda B, s, o: B.tempo_route(
        s, o["x"], o["wr"], o["bias"], o["n_valid"], o["ids"], o["tw"], o["st"])),
    "few": (("x", "ids", "tw", "n_valid", "rmap", "packed", "ro", "st", "ws"), lambda B, s, o: B.tempo_few_ffn(
        s, o["x"], o["ids"], o["tw"], o["n_valid"], o["rmap"], o["packed"], o["ro"], o["st"], o["ws"])),
    "few bf16": (("x", "ids", "tw", "n_valid", "rmap", "packed", "ro", "st", "ws"), lambda B, s, o: B.tempo_few_ffn_bf16(
        s, o["x"], o["ids"], o["tw"], o["n_valid"], o["rmap"], o["packed"], o["ro"], o["st"], o["ws"])),
}


@pytest.mark.parametrize("name,operand", [(n, o) for n, (operands, _) in CALLS.items() for o in operands])
def test_operands_on_two_devices(B, name, operand):
    s = B.make_shape(4, 2, 8, 2, 1, 128, 128, 128)
    with pytest.raises(B.TempoError, match="cuda:0 and cuda:1|cuda:1 and cuda:0"):
        CALLS[name][1](B, s, fakes(operand))


class Unsure:
    def __bool__(self):
        raise ZeroDivisionError("neither")


def test_arguments_that_cannot_be_converted_raise_their_own_error(B):
    from paper_2608_13057_b200 import _marshal
    s, o = B.make_shape(4, 2, 8, 2, 1, 128, 128, 128), fakes()
    with pytest.raises(ZeroDivisionError):
        B.tempo_route(s, o["x"], o["wr"], None, None, o["ids"], o["tw"], o["st"], renormalise=Unsure())
    with pytest.raises(ZeroDivisionError):
        _marshal.few(Unsure(), ctypes.addressof(s), *(o[n] for n in ("x", "ids", "tw", "n_valid", "rmap", "packed", "ro", "st", "ws")))
    with pytest.raises(TypeError):
        B.tempo_norm_in(o["r"], o["w"], o["x"], eps="small")
    for kind in (2 ** 32, -2 ** 31 - 1, 2 ** 80):                   # 2^32 is not NORM_RMS
        with pytest.raises((B.TempoError, OverflowError), match="32-bit|too large"):
            B.tempo_norm_in(o["r"], o["w"], o["x"], kind=kind)
        with pytest.raises((B.TempoError, OverflowError), match="32-bit|too large"):
            B.tempo_route(s, o["x"], o["wr"], None, None, o["ids"], o["tw"], o["st"], score=kind)
