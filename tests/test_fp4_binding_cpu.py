"""Argument checks of the binding's 4-bit calls, answered on the host.

A tensor is checked against the current device; here that is the CPU (ordinal -1), so that tensors in host memory come as far as
the checks behind that one.  A call that passes them all ends in the library at the missing GPU.
"""
import pytest
import torch

from paper_1711_04713_b200 import binding as B
from paper_1711_04713_b200 import build

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that pass the checks would run on host memory")

ROWS, INNER = 6, 70           # rows of 70 elements, pitch 80 (fixed point) and 96 (4 bits)


def _bind(device, stream):
    samples = (torch.empty(3, 5)[1:, 1:4], torch.empty(4, dtype=torch.bfloat16))
    B._native.bind(build.LIB_PATH, B.AdaptionError, device, stream, torch.float32, torch.float16, torch.bfloat16, torch.Tensor,
                   exchange["api"], samples)


exchange = {"api": None}


@pytest.fixture(params=["exchange", "attributes"], autouse=True)
def host_is_the_device(request):
    """Both ways in which the binding reads tensors."""
    build.build_library()
    B.load()
    api = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)
    exchange["api"] = api if request.param == "exchange" else None
    _bind(lambda: -1, lambda device: 0)
    yield
    exchange["api"] = api
    _bind(*B._stream_getters())


def status(call, *args):
    with pytest.raises(B.AdaptionError) as e:
        call(*args)
    return e.value.status


def fixed(n_bits=16, **planes):
    q = B.QTensor.empty(ROWS, INNER, n_bits, 3, 80, device="cpu")
    for name, t in planes.items():
        setattr(q, name, t)
    return q


def four_bit(rows=ROWS, **buffers):
    q = B.Fp4Tensor.empty(rows, INNER, 16, device="cpu")
    for name, t in buffers.items():
        setattr(q, name, t)
    return q


def plane(n=ROWS * 80, dtype=torch.uint8):
    return torch.zeros(n, dtype=dtype)


def quantize_status(x, out=None, rows=ROWS):
    return status(B.adaption_fp4_quantize, x, rows, INNER, four_bit() if out is None else out)


def test_planes_of_a_fixed_point_tensor_have_to_hold_its_rows():
    assert quantize_status(fixed()) == B.ERR_CUDA
    assert quantize_status(fixed(8)) == B.ERR_CUDA
    assert quantize_status(fixed(lo=plane(dtype=torch.int8), hi=plane())) == B.ERR_CUDA       # (any type of a byte)
    assert quantize_status(fixed(lo=plane().view(ROWS, 80))) == B.ERR_CUDA
    assert quantize_status(fixed(lo=plane(2 * 80), hi=plane(2 * 80)), rows=2) == B.ERR_CUDA    # those of the call
    for bad in (dict(lo=plane(ROWS * 80 - 1)), dict(hi=plane(ROWS * 80 - 1)), dict(lo=plane(1)), dict(hi=plane(0)), dict(lo=None), dict(hi=None),
                dict(lo=plane(2 * ROWS * 80)[::2]), dict(hi=plane(2 * ROWS * 80)[::2]), dict(lo=plane(1).expand(ROWS * 80)),
                dict(hi=plane(80).expand(ROWS, 80)), dict(lo=plane(ROWS * 80, torch.int16)), dict(hi=plane(ROWS * 40, torch.int16)),
                dict(c_stride=96), dict(c_stride=1 << 62), dict(c_stride=-80)):
        assert quantize_status(fixed(**bad)) == B.ERR_INVALID_ARG, bad
    assert quantize_status(fixed(8, lo=plane(ROWS * 80 - 1))) == B.ERR_INVALID_ARG
    assert quantize_status(fixed(8, hi=plane(1))) == B.ERR_CUDA                                # (a plane that eight bits do not use)


def test_buffers_have_to_hold_their_bytes_one_after_the_other():
    x, y, st = torch.zeros(ROWS, INNER), torch.zeros(ROWS, 5), B.new_stats("cpu")
    w, good = four_bit(5), four_bit()
    need = B.fp4_act_ip_workspace_bytes(ROWS, INNER, 5, 16)

    def views(n):
        return plane(1).expand(n), plane(1).expand(2, n), plane(2 * n)[::2], plane(2 * n).view(n, 2)[:, 0], plane(n).view(2, n // 2).t()

    def calls(q=good, stats=st, ws=plane(need)):
        return [status(B.adaption_fp4_quantize, x, ROWS, INNER, q, False, stats), status(B.adaption_fp4_dequantize, q, ROWS, INNER, x),
                status(B.adaption_fp4_ip_fwd, ROWS, INNER, 5, q, w, None, False, y, stats),
                status(B.adaption_fp4_act_ip_fwd, ROWS, INNER, 5, x, 0, w, None, False, y, stats, ws),
                status(B.adaption_fp4_act_ip_fwd, ROWS, INNER, ROWS, x, 0, q, None, False, torch.zeros(ROWS, ROWS), stats, plane(2 * need))]

    assert calls() == [B.ERR_CUDA] * 5
    assert calls(ws=plane(need).view(2, need // 2)) == [B.ERR_CUDA] * 5
    for ws in views(need):
        assert calls(ws=ws)[3] == B.ERR_INVALID_ARG
    for name in ("codes", "scales"):
        for t in views(getattr(good, name).numel()):
            got = calls(q=four_bit(**{name: t}))
            assert got[:3] + got[4:] == [B.ERR_INVALID_ARG] * 4, (name, t.shape, t.stride())
    for stats in views(B.STATS_BYTES):
        got = calls(stats=stats)
        assert [got[0]] + got[2:] == [B.ERR_INVALID_ARG] * 4
