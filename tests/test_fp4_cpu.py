"""Microscaled 4-bit operators without a GPU: the oracle's pins, host helpers, and refusals before any launch."""
import ctypes
import subprocess
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import microscale as ms
from paper_1711_04713_b200 import binding as B
from paper_1711_04713_b200 import build

FAKE = 4096          # never dereferenced: the calls below fail validation first, or have nothing to do


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load()


# --------------------------------------------------------------------------- the oracle
def test_oracle_handworked_values():
    # amax 6: floor(log2 6) - 2 = 0, step 1; amax 7.99 keeps it, and 7 and more are clipped to 6
    x = np.zeros((1, 32))
    x[0, :12] = [6, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -7.99, -0.2]
    code, byte, counts = ms.quantize(x, 32)
    assert byte.tolist() == [[127]]
    assert code[0, :12].tolist() == [7, 0, 1, 2, 2, 4, 4, 6, 6, 7, 15, 8]
    assert counts == (22, 0, 1)
    # blocks of 16: amax 6 * 1.75 = 10.5 -> scale 1.75 exactly; 10.5 / 1.75 = 6, 1.75 / 1.75 = 1
    x = np.zeros((1, 16))
    x[0, :3] = [10.5, 1.75, -0.4375]
    code, byte, counts = ms.quantize(x, 16)
    assert ms.E4M3[byte[0, 0]] == 1.75 and code[0, :3].tolist() == [7, 2, 8] and counts == (14, 0, 0)
    # the same in units of 2^-5
    code5, byte5, _ = ms.quantize(x / 32, 16, -5)
    assert byte5.tolist() == byte.tolist() and code5.tolist() == code.tolist()
    # zero, tiny and huge blocks
    for v, want in ((0.0, 0), (2.0 ** -149, 0), (2.0 ** -124, 1), (2.0 ** -125, 0), (ms.FLT_MAX, 252), (np.inf, 252), (np.nan, 0)):
        assert ms.quantize(np.full((1, 32), v), 32)[1].tolist() == [[want]], v
    assert ms.quantize(np.full((1, 16), 1e30), 16)[1].tolist() == [[126]]       # 448
    assert ms.E4M3[126] == 448 and ms.E4M3[1] == 2.0 ** -9 and ms.E4M3[8] == 2.0 ** -6


def test_oracle_codes_are_nearest_in_rational_arithmetic():
    rng = np.random.default_rng(3)
    grid = [Fraction(v) for v in (0, Fraction(1, 2), 1, Fraction(3, 2), 2, 3, 4, 6)]
    for block in (16, 32):
        x = (rng.standard_normal((6, 64)) * 2.0 ** rng.integers(-20, 20, (6, 1))).astype(np.float32)
        code, byte, _ = ms.quantize(x, block, -3 if block == 16 else 0)
        for r in range(6):
            for i in range(64):
                s = Fraction(float(ms.E4M3[byte[r, i // block]])) / 8 if block == 16 else Fraction(2) ** (int(byte[r, i // block]) - 127)
                if s == 0:
                    assert code[r, i] & 7 == 0
                    continue
                d = [abs(abs(Fraction(float(x[r, i]))) / s - g) for g in grid]
                best = [k for k in range(8) if d[k] == min(d)]
                want = best[0] if len(best) == 1 else next(k for k in best if k % 2 == 0)
                assert (code[r, i] & 7) == want and (code[r, i] >> 3) == (x[r, i] < 0)


def test_rounding_the_quotient_to_32_bits_first_keeps_the_code():
    """What the kernel relies on: x / step rounded to a float and then to E2M1 gives the same code as the exact quotient,
    at every border between two codes and its neighbours, for every scale."""
    f32 = np.float32
    mids = ((ms.E2M1[1:] + ms.E2M1[:-1]) / 2)
    for s in ms.E4M3[1:]:
        for exp in (-63, -9, 0, 63):
            step = np.ldexp(s, exp)
            x = (mids * step).astype(f32)
            assert np.all(x.astype(np.float64) == mids * step)               # the border is a float
            for v in (np.nextafter(x, f32(0)), x, np.nextafter(x, f32(np.inf))):
                q = v / f32(step)
                assert q.dtype == f32
                assert np.array_equal(ms.nearest(q.astype(np.float64), ms.E2M1), ms.nearest(v.astype(np.float64) / step, ms.E2M1))
    # the scale: amax / 6 in 32 bits against the borders of E4M3
    mids = (ms.E4M3[1:] + ms.E4M3[:-1]) / 2
    x = (6 * mids).astype(f32)
    for v in (np.nextafter(x, f32(0)), x, np.nextafter(x, f32(np.inf))):
        assert np.array_equal(ms.nearest((v / f32(6)).astype(np.float64), ms.E4M3), ms.nearest(v.astype(np.float64) / 6, ms.E4M3))


def test_oracle_storage_round_trip():
    rng = np.random.default_rng(0)
    for rows, inner, block in ((1, 1, 16), (130, 200, 32), (300, 77, 16)):
        code = rng.integers(0, 16, (rows, inner)).astype(np.uint8)
        pitch = (inner + 31) // 32 * 32
        assert np.array_equal(ms.unpack_codes(ms.pack_codes(code, pitch), inner), code)
        used, fill = ms.scale_places(rows, inner, block)
        every = np.concatenate([used.ravel(), fill.ravel()])
        assert len(set(every.tolist())) == every.size and every.max() < B.fp4_scale_bytes(rows, inner, block)
        assert used[0, 0] == 0 and (rows < 2 or used[1, 0] == 16) and (rows < 33 or used[32, 0] == 4)


# --------------------------------------------------------------------------- host helpers
def test_layouts_and_helpers(lib):
    assert ctypes.sizeof(B.adaption_fp4tensor) == 32 and ctypes.sizeof(B.adaption_matrix) == 24
    for rows, inner, block in ((1, 1, 16), (128, 64, 16), (129, 65, 16), (1000, 4096, 32), (5, 129, 32)):
        want = -(-rows // 128) * -(-(-(-inner // block)) // 4) * 512
        assert lib.adaption_fp4_scale_bytes(rows, inner, block) == B.fp4_scale_bytes(rows, inner, block) == want
    for bad in ((0, 5, 16), (5, 0, 16), (5, 5, 8), (-1, 5, 32)):
        assert lib.adaption_fp4_scale_bytes(*bad) == 0
    for bad in ((0, 5, 16), (5, 0, 16), (5, 5, 8), (5, 5, 0), (5, 5, -16), (-1, 5, 32)):
        assert B.fp4_scale_bytes(*bad) == 0
        with pytest.raises(B.AdaptionError):
            B.Fp4Tensor.empty(max(bad[0], 1), max(bad[1], 1), bad[2] if bad[2] not in (16, 32) else 24, device="cpu")
    assert B.adaption_fp4_choose_exp(0.0) == -63
    assert B.adaption_fp4_choose_exp(2688.0) == 0 and B.adaption_fp4_choose_exp(np.nextafter(np.float32(2688), np.float32(1e9))) == 1
    assert B.adaption_fp4_choose_exp(2688.0 * 2.0 ** -9) == -9
    assert B.adaption_fp4_choose_exp(float("inf")) == 63
    for v in (-1.0, float("nan")):
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_choose_exp(v)
    # with the chosen exponent no scale is clipped
    for v in (1e-3, 1.0, 5.3, 1234.5):
        e = B.adaption_fp4_choose_exp(v)
        assert v / 6 <= 448 * 2.0 ** e < 2 * 448 * 2.0 ** e and v / 6 > 448 * 2.0 ** (e - 1)


def _fp4(block=16, exp=0, stride=64, codes=FAKE, scales=FAKE):
    return B.adaption_fp4tensor(codes, scales, stride, block, exp)


def _mat(stride=64, dtype=0, data=FAKE):
    return B.adaption_matrix(data, stride, dtype, 0)


BAD_FP4 = [(dict(block=8), B.ERR_INVALID_ARG), (dict(block=32, exp=1), B.ERR_INVALID_ARG), (dict(exp=64), B.ERR_INVALID_ARG),
           (dict(exp=-64), B.ERR_INVALID_ARG), (dict(stride=48), B.ERR_INVALID_ARG), (dict(stride=32), B.ERR_INVALID_ARG),
           (dict(codes=None), B.ERR_INVALID_ARG), (dict(scales=None), B.ERR_INVALID_ARG),
           (dict(codes=FAKE + 8), B.ERR_ALIGNMENT), (dict(scales=FAKE + 4), B.ERR_ALIGNMENT)]
BAD_MATRIX = [(dict(dtype=3), B.ERR_INVALID_ARG), (dict(dtype=-1), B.ERR_INVALID_ARG), (dict(stride=59), B.ERR_INVALID_ARG),
              (dict(data=None), B.ERR_INVALID_ARG), (dict(data=FAKE + 2), B.ERR_ALIGNMENT),
              (dict(data=FAKE + 1, dtype=1), B.ERR_ALIGNMENT)]


@pytest.mark.parametrize("bad,rc", BAD_FP4)
def test_bad_4bit_tensors_are_refused(lib, bad, rc):
    f, g, m = _fp4(**bad), _fp4(), _mat()
    assert lib.adaption_fp4_quantize(m, None, 3, 60, 0, f, None, None) == rc
    assert lib.adaption_fp4_dequantize(f, 3, 60, m, None) == rc
    want = rc if bad.get("block") != 32 else B.ERR_INVALID_ARG
    assert lib.adaption_fp4_ip_fwd(3, 60, 60, f, g, None, 0, m, FAKE, None) == want
    assert lib.adaption_fp4_ip_fwd(3, 60, 60, g, f, None, 0, m, FAKE, None) == rc
    assert lib.adaption_fp4_act_ip_fwd(3, 60, 60, m, 0, f, None, 0, m, FAKE, FAKE, 1 << 20, None) == rc


@pytest.mark.parametrize("bad,rc", BAD_MATRIX)
def test_bad_matrices_are_refused(lib, bad, rc):
    f, m, ok = _fp4(), _mat(**bad), _mat()
    assert lib.adaption_fp4_quantize(m, None, 3, 60, 0, f, None, None) == rc
    assert lib.adaption_fp4_dequantize(f, 3, 60, m, None) == rc
    assert lib.adaption_fp4_ip_fwd(3, 60, 60, f, f, None, 0, m, FAKE, None) == rc
    assert lib.adaption_fp4_act_ip_fwd(3, 60, 60, m, 0, f, None, 0, ok, FAKE, FAKE, 1 << 20, None) == rc
    assert lib.adaption_fp4_act_ip_fwd(3, 60, 60, ok, 0, f, None, 0, m, FAKE, FAKE, 1 << 20, None) == rc


def test_other_refusals_and_empty_calls(lib):
    f, m = _fp4(), _mat()
    q = B.adaption_qtensor(FAKE, FAKE, None, B.adaption_qfmt(16, 3), 64)
    both, neither = _mat(), _mat(data=None)
    assert lib.adaption_fp4_quantize(both, ctypes.byref(q), 3, 60, 0, f, None, None) == B.ERR_INVALID_ARG
    assert lib.adaption_fp4_quantize(neither, None, 3, 60, 0, f, None, None) == B.ERR_INVALID_ARG
    bad_q = B.adaption_qtensor(FAKE, FAKE, None, B.adaption_qfmt(17, 3), 64)
    assert lib.adaption_fp4_quantize(neither, ctypes.byref(bad_q), 3, 60, 0, f, None, None) == B.ERR_INVALID_ARG
    long = _fp4(stride=(1 << 24) + 32)
    assert lib.adaption_fp4_quantize(_mat(stride=1 << 25), None, 3, (1 << 24) + 1, 0, long, None, None) == B.ERR_UNSUPPORTED
    assert lib.adaption_fp4_dequantize(long, 3, (1 << 24) + 1, _mat(stride=1 << 25), None) == B.ERR_UNSUPPORTED
    ip, act = lib.adaption_fp4_ip_fwd, lib.adaption_fp4_act_ip_fwd
    assert ip(3, 60, 60, _fp4(block=32), f, None, 0, m, FAKE, None) == B.ERR_INVALID_ARG          # two block lengths
    assert ip(3, 60, 60, f, f, None, 0, m, None, None) == B.ERR_INVALID_ARG                        # no counters
    assert ip(3, 60, 60, f, f, FAKE + 2, 0, m, FAKE, None) == B.ERR_ALIGNMENT
    for B_, K, O in ((-1, 60, 60), (3, 0, 60), (3, 60, 0)):
        assert ip(B_, K, O, f, f, None, 0, m, FAKE, None) == B.ERR_INVALID_ARG
        assert act(B_, K, O, m, 0, f, None, 0, m, FAKE, FAKE, 1 << 20, None) == B.ERR_INVALID_ARG
    assert ip(3, (1 << 24) + 1, 60, long, long, None, 0, m, FAKE, None) == B.ERR_K_TOO_LARGE
    assert ip(3, 60, (1 << 30) + 1, f, f, None, 0, _mat(stride=1 << 31), FAKE, None) == B.ERR_UNSUPPORTED
    need = B.fp4_act_ip_workspace_bytes(3, 60, 60, 16)
    assert need > 0
    assert act(3, 60, 60, m, 0, f, None, 0, m, FAKE, FAKE, need - 1, None) == B.ERR_WORKSPACE
    assert act(3, 60, 60, m, 0, f, None, 0, m, FAKE, None, 0, None) == B.ERR_WORKSPACE
    assert act(3, 60, 60, m, 0, f, None, 0, m, FAKE, FAKE + 8, need, None) == B.ERR_ALIGNMENT
    assert act(3, 60, 60, m, 64, f, None, 0, m, FAKE, FAKE, need, None) == B.ERR_INVALID_ARG
    assert act(3, 60, 60, m, 1, _fp4(block=32), None, 0, m, FAKE, FAKE, need, None) == B.ERR_INVALID_ARG
    # nothing to do: accepted without touching memory
    assert lib.adaption_fp4_quantize(m, None, 0, 60, 0, f, None, None) == B.OK
    assert lib.adaption_fp4_dequantize(f, 0, 60, m, None) == B.OK
    assert ip(0, 60, 60, f, f, None, 0, m, FAKE, None) == B.OK
    assert act(0, 60, 60, m, 0, f, None, 0, m, FAKE, None, 0, None) == B.OK


def test_descriptors_check_their_buffers():
    good = B.Fp4Tensor.empty(130, 70, 16, device="cpu")
    assert good.c_stride == 96 and good.codes.numel() == 130 * 48 and good.scales.numel() == 2 * 2 * 512
    for kw in (dict(block=8), dict(c_stride=80), dict(c_stride=64), dict(inner=0), dict(outer=131), dict(outer=300),
               dict(codes=good.codes[1:]), dict(scales=good.scales[:-1]), dict(codes=good.codes.view(torch.int8)),
               dict(codes=torch.empty(2 * good.codes.numel(), dtype=torch.uint8)[::2])):
        a = dict(outer=good.outer, inner=good.inner, c_stride=good.c_stride, block=16, exp=0, codes=good.codes, scales=good.scales)
        with pytest.raises(B.AdaptionError):
            B.Fp4Tensor(**{**a, **kw})


def test_tensors_off_the_current_device_are_refused(lib):
    """Without a GPU every tensor is off it: the binding answers before the library is entered."""
    if torch.cuda.is_available():
        pytest.skip("tested with a device in tests/test_gpu_fp4.py")
    x, q = torch.zeros(4, 64), B.Fp4Tensor.empty(4, 64, 16, device="cpu")
    st = torch.zeros(40, dtype=torch.uint8)
    for call in (lambda: B.adaption_fp4_quantize(x, 4, 64, q), lambda: B.adaption_fp4_dequantize(q, 4, 64, x),
                 lambda: B.adaption_fp4_ip_fwd(4, 64, 4, q, q, None, False, torch.zeros(4, 4), st)):
        with pytest.raises((B.AdaptionError, RuntimeError, AssertionError)):
            call()


@pytest.mark.parametrize("off", [1, 2, 4])
def test_counters_off_their_alignment_are_refused(lib, off):
    """The kernels add 64-bit counters atomically."""
    f, m = _fp4(), _mat()
    assert lib.adaption_fp4_quantize(m, None, 3, 60, 0, f, FAKE + off, None) == B.ERR_ALIGNMENT
    assert lib.adaption_fp4_ip_fwd(3, 60, 60, f, f, None, 0, m, FAKE + off, None) == B.ERR_ALIGNMENT
    assert lib.adaption_fp4_act_ip_fwd(3, 60, 60, m, 0, f, None, 0, m, FAKE + off, FAKE, 1 << 20, None) == B.ERR_ALIGNMENT


def test_a_question_that_failed_is_asked_again(tmp_path):
    """How the cost model keeps the number of clusters that a device runs at a time: its guess stands for one call only."""
    source, program = tmp_path / "ask.cpp", tmp_path / "ask"
    source.write_text("""
#include "remember.cuh"
#include <cstdio>
int main() {
  std::atomic<int> slot{0};
  int asked = 0, answer = 0;
  const auto ask = [&]() { ++asked; return answer; };
  const auto get = [&]() { return adaption::remembered(slot, 9, ask); };
  std::printf("%d", get());
  answer = -3;
  std::printf(" %d", get());
  answer = 33;
  std::printf(" %d", get());
  answer = 0;
  std::printf(" %d %d\\n", get(), asked);
}
""")
    subprocess.check_call(["g++", "-std=c++17", "-I", build.CSRC, str(source), "-o", str(program)])
    assert subprocess.check_output([str(program)]).split() == [b"9", b"9", b"33", b"33", b"3"]
