"""Microscaled 4-bit operators on the GPU against their definition in 64 bits.

Codes, scales and values are fixed bit for bit.  Products are exact and summed in 32 bits: every addition
rounds (or cuts off) at most one unit in the last place, 2^-23, of a partial sum, none of which exceeds
S = sum |x w| (+ |bias|); a row has at most one addition per scale block and per share of the reduction, two
scalings that are exact, and one rounding to the output type, half a step.
"""
import threading

import numpy as np
import pytest
import torch

from oracle import microscale as ms
from paper_1711_04713_b200 import binding as B
from tests.util import Guards, dev, stats_tuple, to_qtensor

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def _defaults():
    B.adaption_debug_set("reset")
    yield
    B.adaption_debug_set("reset")


def guarded(g, outer, inner, block, exp=0, c_stride=None, fill=0xA5):
    cs = B.pad_to(inner, 32) if c_stride is None else c_stride
    codes = g.alloc(outer * cs // 2, torch.uint8, fill)
    scales = g.alloc(B.fp4_scale_bytes(outer, inner, block), torch.uint8, fill)
    return B.Fp4Tensor(outer, inner, cs, block, exp, codes, scales)


def logical(t):
    """codes [outer][inner], scale bytes [outer][blocks], the padding of the codes, the rest of the row's scale tiles."""
    data = t.codes.cpu().numpy()[:t.outer * t.c_stride // 2].reshape(t.outer, -1)
    every = ms.unpack_codes(data, t.c_stride)
    used, fill = ms.scale_places(t.outer, t.inner, t.block)
    plane = t.scales.cpu().numpy()
    return every[:, :t.inner], plane[used], every[:, t.inner:], plane[fill]


def stored(code, byte, block, exp=0, c_stride=None, fill=0, rows=None):
    """Device tensor of given codes and scale bytes; scale bytes of rows that do not exist hold `fill`."""
    outer, inner = code.shape
    cs = B.pad_to(inner, 32) if c_stride is None else c_stride
    used, rest = ms.scale_places(outer, inner, block)
    plane = np.full(B.fp4_scale_bytes(outer, inner, block), fill, np.uint8)
    plane[used] = byte
    plane[rest] = 0
    return B.Fp4Tensor(outer, inner, cs, block, exp, dev(ms.pack_codes(code, cs).ravel()), dev(plane))


def real_input(rng, outer, inner, dtype, pad=0, shift=0):
    """A real-valued (outer, inner) tensor whose rows are `pad` elements apart, `shift` elements off a 16-byte boundary."""
    x = rng.standard_normal((outer, inner)) * 2.0 ** rng.integers(-3, 4, (outer, 1)) * np.exp(rng.standard_normal((1, inner)))
    x[rng.random(x.shape) < 0.1] = 0.0
    flat = torch.zeros(outer * (inner + pad) + shift + 8, dtype=DT[dtype], device="cuda")
    t = flat[shift:shift + outer * (inner + pad)].view(outer, inner + pad)[:, :inner]
    t.copy_(torch.from_numpy(x).to(DT[dtype]))
    return t


# --------------------------------------------------------------------------- quantizer
SHAPES = [(1, 1), (1, 16), (3, 31), (5, 33), (2, 4096), (129, 200), (130, 64), (257, 95), (40, 1003), (1000, 8)]


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantize(shape, dtype, block):
    outer, inner = shape
    rng = np.random.default_rng(outer * 7 + inner)
    for k, (pad, shift, relu, extra) in enumerate([(0, 0, False, 0), (8, 0, True, 0), (3, 0, False, 32), (0, 1, True, 0), (1, 3, False, 64)]):
        x = real_input(rng, outer, inner, dtype, pad, shift)
        ref = x.double().cpu().numpy()
        exp = B.adaption_fp4_choose_exp(float(np.abs(ref).max())) if block == 16 else 0
        if k == 4 and block == 16:
            exp += 3                     # small scales: E4M3 denormals and blocks whose step is 0
        elif k == 3 and block == 16:
            exp -= 9                     # scales clipped at 448
        g = Guards()
        q = guarded(g, outer, inner, block, exp, B.pad_to(inner, 32) + extra)
        st = B.new_stats()
        B.adaption_fp4_quantize(x, outer, inner, q, relu, st)
        code, byte, counts = ms.quantize(ref, block, exp, relu)
        got, got_byte, pad_codes, pad_scales = logical(q)
        assert np.array_equal(got_byte, byte), (k, np.argwhere(got_byte != byte)[:4])
        assert np.array_equal(got, code), (k, np.argwhere(got != code)[:4])
        assert not pad_codes.any() and not pad_scales.any()
        assert stats_tuple(st) == counts
        # scale bytes of rows that do not exist stay as they were
        untouched = np.ones(q.scales.numel(), bool)
        for places in ms.scale_places(outer, inner, block):
            untouched[places.ravel()] = False
        assert (q.scales.cpu().numpy()[untouched] == 0xA5).all()
        g.check()


@pytest.mark.parametrize("block", [16, 32])
def test_quantize_special_values(block):
    vals = [np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 2.0 ** -126, 3e38, -3.4e38, 448.0, 6.0, 7.0, -7.0, 5.0, 0.25]
    rows = [vals + [0.0] * 16, [0.0] * 32, [np.nan] * 32, [np.inf] * 32, [1e-45] * 32, vals[3:8] + [0.0] * 27,
            [m * s for s in (1.0, 1.875) for m in (0.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, -0.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -6)]]
    x = np.array(rows, np.float32)
    for exp in ((0,) if block == 32 else (0, -63, 63, -9)):
        for relu in (False, True):
            q = B.Fp4Tensor.empty(*x.shape, block, exp)
            B.adaption_fp4_quantize(dev(x), *x.shape, q, relu)
            code, byte, _ = ms.quantize(x, block, exp, relu)
            got, got_byte, _, _ = logical(q)
            assert np.array_equal(got_byte, byte) and np.array_equal(got, code), (exp, relu)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("n_bits", [16, 9, 8, 4, 1])
def test_quantize_from_fixed_point(n_bits, block):
    rng = np.random.default_rng(n_bits)
    for outer, inner, pitch in ((1, 5, 16), (130, 77, 80), (33, 300, 352)):
        f = int(rng.integers(0, n_bits))
        v = rng.integers(-(1 << (n_bits - 1)), 1 << (n_bits - 1), (outer, inner))
        xq = to_qtensor(v, n_bits, f, pitch)
        exp = B.adaption_fp4_choose_exp(float(np.abs(v).max() * 2.0 ** -f)) if block == 16 else 0
        for relu in (False, True):
            q = B.Fp4Tensor.empty(outer, inner, block, exp)
            st = B.new_stats()
            B.adaption_fp4_quantize(xq, outer, inner, q, relu, st)
            code, byte, counts = ms.quantize(v * 2.0 ** -f, block, exp, relu)
            got, got_byte, pc, ps = logical(q)
            assert np.array_equal(got_byte, byte) and np.array_equal(got, code)
            assert not pc.any() and not ps.any() and stats_tuple(st) == counts


def test_quantize_large_and_every_float16():
    # every finite half as the maximum of a block of its own: every rounding of a scale, many of codes
    bits = np.arange(1 << 16, dtype=np.uint16).view(np.float16)
    h = bits[np.isfinite(bits)].astype(np.float32)
    x = np.zeros((h.size, 16), np.float32)
    x[:, 0] = h
    x[:, 1:] = h[:, None] * np.linspace(0, 1, 16)[1:].astype(np.float32)
    for exp in (0, -9, 5):
        q = B.Fp4Tensor.empty(h.size, 16, 16, exp)
        B.adaption_fp4_quantize(dev(x), h.size, 16, q)
        code, byte, _ = ms.quantize(x, 16, exp)
        got, got_byte, _, _ = logical(q)
        assert np.array_equal(got_byte, byte) and np.array_equal(got, code)


@pytest.mark.parametrize("source", ["f32", "f16", "bf16", "fixed"])
def test_quantize_next_to_every_border(source):
    """For each step of E4M3: the numbers between two codes, and those next to them in the source's type, of both signs."""
    frac = 15 - 12                                   # (16-bit fixed point holds 6 * 448)
    rows = []
    for s in ms.E4M3[1:]:
        m = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.01]) * s
        if source == "fixed":
            if s * 2 ** frac != np.floor(s * 2 ** frac):
                continue                             # (the maximum, 6 steps, has to be a number of the source)
            at = np.floor(m * 2 ** frac)
            near = [(at + k) / 2 ** frac for k in (-1, 0, 1, 2)]
        elif source == "bf16":
            bits = (m.astype(np.float32).view(np.uint32) >> 16).astype(np.int64)
            near = [((bits + k) << 16).astype(np.uint32).view(np.float32).astype(np.float64) for k in (-1, 0, 1, 2)]
        else:
            t = m.astype(np.float32 if source == "f32" else np.float16)
            near = [np.nextafter(t, t.dtype.type(0)).astype(np.float64), t.astype(np.float64),
                    np.nextafter(t, t.dtype.type(np.inf)).astype(np.float64)]
        near = np.concatenate(near)
        near = near[near <= 6 * s]
        near = np.concatenate([near, -near])
        for k in range(0, near.size, 15):
            part = near[k:k + 15]
            rows.append(np.concatenate([[6 * s], part, np.zeros(15 - part.size)]))
    x = np.array(rows)
    if source == "fixed":
        whole = np.rint(x * 2 ** frac).astype(np.int64)
        data, x = to_qtensor(whole, 16, frac, 16), whole / 2 ** frac       # (an integer holds no negative zero)
    else:
        data = dev(x.astype(np.float32)).to(DT[source])
        assert np.array_equal(data.double().cpu().numpy(), x)
    q = B.Fp4Tensor.empty(*x.shape, 16, 0)
    st = B.new_stats()
    B.adaption_fp4_quantize(data, *x.shape, q, False, st)
    code, byte, counts = ms.quantize(x, 16, 0)
    got, got_byte, _, _ = logical(q)
    assert np.array_equal(got_byte, byte) and np.array_equal(got, code)
    assert stats_tuple(st) == counts


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_quantize_special_values_of_16_bits(dtype, block):
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -133
    vals = [np.nan, np.inf, -np.inf, 0.0, -0.0, tiny, -tiny, 3 * tiny, 60000.0, -60000.0, 448.0, 6.0, 7.0, -7.0, 5.0, 0.25]
    x = np.array([vals + [0.0] * 16, [0.0] * 32, [np.nan] * 32, [np.inf] * 32, [tiny] * 32, vals[3:8] + [0.0] * 27, [-np.inf] + [1.0] * 31,
                  [1.0] * 17 + [np.nan] + [-1.0] * 14])
    data = torch.from_numpy(x).to(DT[dtype]).cuda()
    x = data.double().cpu().numpy()
    for exp in ((0,) if block == 32 else (0, -63, 63, -9)):
        for relu in (False, True):
            q = B.Fp4Tensor.empty(*x.shape, block, exp)
            B.adaption_fp4_quantize(data, *x.shape, q, relu)
            code, byte, _ = ms.quantize(x, block, exp, relu)
            got, got_byte, _, _ = logical(q)
            assert np.array_equal(got_byte, byte) and np.array_equal(got, code), (exp, relu)


# --------------------------------------------------------------------------- values
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_dequantize(dtype, block):
    rng = np.random.default_rng(block)
    for outer, inner, pad, shift, exp, wide in ((1, 1, 0, 0, 0, 0), (16, 256, 0, 0, 0, 0), (130, 77, 3, 0, -9, 0), (3, 1003, 8, 0, 5, 64),
                                                (257, 40, 0, 1, -3, 0)):
        blocks = -(-inner // block)
        top = 256 if block == 32 else 128
        byte = ((np.arange(outer * blocks) * 7) % top).astype(np.uint8).reshape(outer, blocks)
        code = rng.integers(0, 16, (outer, inner)).astype(np.uint8)
        exp = exp if block == 16 else 0
        t = stored(code, byte, block, exp, B.pad_to(inner, 32) + wide)
        flat = torch.full((outer * (inner + pad) + shift,), 7.0, dtype=DT[dtype], device="cuda")
        full = flat[shift:].view(outer, inner + pad)
        B.adaption_fp4_dequantize(t, outer, inner, full[:, :inner])
        with np.errstate(all="ignore"):
            want = torch.from_numpy(ms.values(code, byte, block, exp)).to(DT[dtype])
        assert torch.equal(torch.nan_to_num(full[:, :inner].cpu(), nan=-77.0), torch.nan_to_num(want, nan=-77.0))
        assert bool((full[:, inner:] == 7).all()) and bool((flat[:shift] == 7).all())


# --------------------------------------------------------------------------- inner product
def operand(rng, rows, inner, block, exp=0, spread=3):
    code = rng.integers(0, 16, (rows, inner)).astype(np.uint8)
    blocks = -(-inner // block)
    mid = 127 if block == 32 else 56
    byte = rng.integers(mid - spread, mid + spread + 1, (rows, blocks)).astype(np.uint8)
    # scale bytes of rows that do not exist hold NaN
    return stored(code, byte, block, exp, fill=0xFF), ms.values(code, byte, block, exp)


def check_product(y, xv, wv, bias, relu, block, dtype, cols=None):
    want = ms.inner_product(xv, wv, bias, relu)
    S = np.abs(xv) @ np.abs(wv).T + (0 if bias is None else np.abs(bias))
    adds = -(-xv.shape[1] // block) + 8 + 1
    bound = adds * 2.0 ** -23 * S
    got = y.double().cpu().numpy()
    if dtype != "f32":
        eps = torch.finfo(DT[dtype]).eps / 2
        bound = bound + (np.abs(want) + bound) * eps + torch.finfo(DT[dtype]).smallest_normal * eps
    err = np.abs(got - want)
    assert np.all(err <= bound), (float((err / np.maximum(bound, 1e-300)).max()), np.argwhere(err > bound)[:5].tolist())


def choose(kernel):
    """One cluster of CTAs or of pairs of CTAs per tile, or the persistent kernel over pairs, wherever the call would run."""
    if kernel != "chosen":
        B.adaption_debug_set("pair", {"cluster": 0, "pairs": 1, "persistent": 1}[kernel])
        B.adaption_debug_set("cluster", {"cluster": 2, "pairs": 2, "persistent": 1}[kernel])


IP_SHAPES = [(1, 1, 1), (1, 64, 128), (1, 4096, 300), (5, 300, 130), (16, 257, 129), (17, 1000, 64), (64, 2048, 256), (100, 33, 500),
             (128, 512, 128), (129, 640, 140), (200, 1411, 257), (256, 768, 200), (257, 256, 128), (300, 900, 384), (520, 320, 1000)]


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("shape", IP_SHAPES)
def test_inner_product(shape, block, kernel):
    choose(kernel)
    Bn, K, O = shape
    rng = np.random.default_rng(Bn + K + O)
    ex, ew = (-3, 2) if block == 16 else (0, 0)
    x, xv = operand(rng, Bn, K, block, ex)
    w, wv = operand(rng, O, K, block, ew)
    bias = (rng.standard_normal(O) * 3).astype(np.float32)
    for dtype, relu, b, pad in (("f32", False, None, 0), ("bf16", True, bias, 0), ("f16", False, bias, 3), ("f32", True, bias, 5)):
        if dtype == "f16" and K > 700:
            continue                      # (sums beyond the type's range)
        full = torch.full((Bn, O + pad), 7.0, dtype=DT[dtype], device="cuda")
        y, st = full[:, :O], B.new_stats()
        B.adaption_fp4_ip_fwd(Bn, K, O, x, w, None if b is None else dev(b), relu, y, st)
        check_product(y, xv, wv, b, relu, block, dtype)
        assert bool((full[:, O:] == 7).all())
        s = B.read_stats(st)
        assert s.status == 0 and s.zeros == int((y == 0).sum())


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
@pytest.mark.parametrize("block", [16, 32])
def test_inner_product_of_exact_sums(block, kernel):
    """Steps of 1 (and of 2 and 1/2): every partial sum is a multiple of 1/16 below 2^20, so the result is exact, and
    any element taken from a wrong place, or with a wrong scale, shows."""
    choose(kernel)
    one = 127 if block == 32 else 56
    for Bn, K, O in ((3, 64, 128), (20, 700, 300), (130, 1056, 256), (270, 2000, 130)):
        rng = np.random.default_rng(K)
        ops = []
        for rows in (Bn, O):
            code = rng.integers(0, 16, (rows, K)).astype(np.uint8)
            blocks = -(-K // block)
            byte = one + rng.integers(-1, 2, (rows, blocks)) * (1 if block == 32 else 8)
            ops.append((stored(code, byte.astype(np.uint8), block, fill=0xFF), ms.values(code, byte, block)))
        y = torch.empty(Bn, O, device="cuda")
        B.adaption_fp4_ip_fwd(Bn, K, O, ops[0][0], ops[1][0], None, False, y, B.new_stats())
        assert np.array_equal(y.double().cpu().numpy(), ms.inner_product(ops[0][1], ops[1][1]))


@pytest.mark.parametrize("kernel,sizes", [("cluster", range(1, 9)), ("pairs", (2, 4, 6, 8))])
def test_every_number_of_shares(kernel, sizes):
    """A reduction cut into 1 to 8 shares, some of them empty, some CTAs without columns of their own."""
    rng = np.random.default_rng(9)
    for Bn, K, O in ((1, 700, 200), (18, 2300, 130), (130, 1500, 300)):
        x, xv = operand(rng, Bn, K, 16)
        w, wv = operand(rng, O, K, 16)
        for size in sizes:
            choose(kernel)
            B.adaption_debug_set("cluster_size", size)
            y, st = torch.full((Bn, O), 7.0, device="cuda"), B.new_stats()
            B.adaption_fp4_ip_fwd(Bn, K, O, x, w, None, False, y, st)
            check_product(y, xv, wv, None, False, 16, "f32")
            assert B.read_stats(st).status == 0


@pytest.mark.parametrize("block", [16, 32])
def test_inner_product_of_more_tiles_than_the_gpu_has_pairs(block):
    """85 tiles of 256 x 256: some pairs of CTAs work on a second one; every type, rows of outputs on 32-byte and 16-byte
    boundaries and off them."""
    Bn = 1100
    for K, O, pad, dtype in ((300, 4112, 0, "f32"), (1300, 4112, 0, "bf16"), (64, 4104, 0, "f16"), (2900, 4101, 0, "f32"), (520, 4112, 1, "bf16"),
                             (200, 4110, 2, "f16"), (600, 4100, 4, "bf16")):
        rng = np.random.default_rng(K)
        x, xv = operand(rng, Bn, K, block, -1 if block == 16 else 0)
        w, wv = operand(rng, O, K, block)
        bias = rng.standard_normal(O).astype(np.float32)
        full = torch.full((Bn, O + pad), 7.0, dtype=DT[dtype], device="cuda")
        y, st = full[:, :O], B.new_stats()
        B.adaption_fp4_ip_fwd(Bn, K, O, x, w, dev(bias), True, y, st)
        check_product(y, xv, wv, bias, True, block, dtype)
        assert bool((full[:, O:] == 7).all())
        s = B.read_stats(st)
        assert s.status == 0 and s.zeros == int((y == 0).sum())


@pytest.mark.parametrize("fused", [0, 1, 2])
@pytest.mark.parametrize("block", [16, 32])
def test_product_of_real_activations(block, fused):
    """Activations quantized in a launch of their own, or by the product where it chooses to, or wherever it can."""
    B.adaption_debug_set("fused", fused)
    for Bn, K, O, dtype, pad, shift in ((1, 4096, 300, "bf16", 0, 0), (7, 333, 200, "f32", 2, 1), (64, 1024, 256, "f16", 8, 0), (140, 77, 130, "bf16", 1, 0),
                                        (16, 640, 1000, "f32", 0, 0), (17, 8200, 140, "bf16", 0, 0)):
        rng = np.random.default_rng(Bn * K)
        x = real_input(rng, Bn, K, dtype, pad, shift)
        ref = x.double().cpu().numpy()
        exp = B.adaption_fp4_choose_exp(float(np.abs(ref).max())) if block == 16 else 0
        w, wv = operand(rng, O, K, block, -2 if block == 16 else 0)
        code, byte, _ = ms.quantize(ref, block, exp)
        xv = ms.values(code, byte, block, exp)
        bias = rng.standard_normal(O).astype(np.float32)
        g = Guards()
        ws = g.alloc(B.fp4_act_ip_workspace_bytes(Bn, K, O, block), torch.uint8, 0xFF)
        y, st = torch.empty(Bn, O, device="cuda"), B.new_stats()
        B.adaption_fp4_act_ip_fwd(Bn, K, O, x, exp, w, dev(bias), True, y, st, ws)
        check_product(y, xv, wv, bias, True, block, "f32")
        g.check()
        # the same bits as the two calls
        q = B.Fp4Tensor.empty(Bn, K, block, exp)
        B.adaption_fp4_quantize(x, Bn, K, q)
        y2 = torch.empty_like(y)
        B.adaption_fp4_ip_fwd(Bn, K, O, q, w, dev(bias), True, y2, st)
        assert torch.equal(y, y2)
        s = B.read_stats(st)
        assert s.status == 0 and s.zeros == 2 * int((y == 0).sum())


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("shape", [(1, 25088, 1000), (3, 4096, 4096), (4, 2048, 8000), (5, 300, 128), (8, 8192, 2048), (4, 12800, 2048), (9, 4096, 1000)])
def test_product_of_few_real_rows_is_the_two_calls(shape, block):
    """The reduction is shared the same way wherever the activations are quantized, so the sums have the same bits."""
    Bn, K, O = shape
    rng = np.random.default_rng(K + O)
    x = real_input(rng, Bn, K, "bf16")
    exp = -6 if block == 16 else 0
    w, _ = operand(rng, O, K, block, 0, 12)          # (scales far enough apart that sums round)
    q, st = B.Fp4Tensor.empty(Bn, K, block, exp), B.new_stats()
    want = torch.empty(Bn, O, device="cuda")
    B.adaption_fp4_quantize(x, Bn, K, q)
    B.adaption_fp4_ip_fwd(Bn, K, O, q, w, None, False, want, st)
    ws = torch.empty(B.fp4_act_ip_workspace_bytes(Bn, K, O, block), dtype=torch.uint8, device="cuda")
    for fused in (0, 1, 2):
        B.adaption_debug_set("fused", fused)
        y = torch.empty_like(want)
        B.adaption_fp4_act_ip_fwd(Bn, K, O, x, exp, w, None, False, y, st, ws)
        assert torch.equal(y, want), fused
    assert B.read_stats(st).status == 0


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
def test_infinite_and_nan_results_stay_in_their_places(kernel):
    """A NaN scale of one row or one channel reaches that row or channel alone; ReLU keeps NaN; fp16 results beyond its range are infinite."""
    choose(kernel)
    rng = np.random.default_rng(1)
    code = rng.integers(1, 8, (40, 96)).astype(np.uint8)
    byte = np.full((40, 3), 127, np.uint8)
    bx = byte.copy()
    bx[7, 1] = 255
    x, w = stored(code, bx, 32), stored(code, byte, 32)
    for relu in (False, True):
        y = torch.empty(40, 40, device="cuda")
        B.adaption_fp4_ip_fwd(40, 96, 40, x, w, None, relu, y, B.new_stats())
        bad = torch.isnan(y).cpu()
        assert bool(bad[7].all()) and not bool(bad[:7].any()) and not bool(bad[8:].any())
    big = stored(code, np.full((40, 3), 140, np.uint8), 32)
    y = torch.empty(40, 40, dtype=torch.float16, device="cuda")
    B.adaption_fp4_ip_fwd(40, 96, 40, big, w, None, False, y, B.new_stats())
    assert bool(torch.isinf(y).all())


# --------------------------------------------------------------------------- streams, graphs, repetition, refusals
def _layer(Bn, K, O, block, seed):
    rng = np.random.default_rng(seed)
    w = torch.from_numpy((rng.standard_normal((O, K)) * np.sqrt(2.0 / K)).astype(np.float32)).cuda()
    exp = B.adaption_fp4_choose_exp(float(w.abs().max())) if block == 16 else 0
    q = B.Fp4Tensor.empty(O, K, block, exp)
    B.adaption_fp4_quantize(w, O, K, q)
    return q, dev(rng.normal(0, 0.1, O).astype(np.float32))


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("Bn", [1, 48])
def test_activations_of_special_values(Bn, block):
    """NaN counts as 0 and infinities as the largest finite number, in the product as in the quantizer; so do blocks out of E4M3's range."""
    rng = np.random.default_rng(Bn)
    x = rng.standard_normal((Bn, 300)).astype(np.float32)
    x[:, ::37] = np.nan
    x[0, 64:80] = 0.0
    x[-1, 100] = np.inf
    x[-1, 260] = -np.inf
    x[0, 5] = 1e30
    x[0, 32:48] *= 1e-30
    w, wv = operand(rng, 40, 300, block, -2 if block == 16 else 0)
    exp = -7 if block == 16 else 0
    code, byte, _ = ms.quantize(x, block, exp)
    xv = ms.values(code, byte, block, exp)
    for fused in (0, 2):
        B.adaption_debug_set("fused", fused)
        y = torch.empty(Bn, 40, device="cuda")
        ws = torch.empty(B.fp4_act_ip_workspace_bytes(Bn, 300, 40, block), dtype=torch.uint8, device="cuda")
        B.adaption_fp4_act_ip_fwd(Bn, 300, 40, dev(x), exp, w, None, False, y, B.new_stats(), ws)
        got, want = y.double().cpu().numpy(), ms.inner_product(xv, wv)
        # (sums with the largest finite number may overflow 32 bits)
        big = np.abs(xv) @ np.abs(wv).T > 1e37
        check_product(y[~torch.from_numpy(big.any(1))], xv[~big.any(1)], wv, None, False, block, "f32")
        assert not np.isnan(got[:, :][~big]).any() and want.shape == got.shape


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("Bn", [1, 48])
def test_a_classifier_end_to_end_in_a_graph_on_its_own_stream(Bn, block):
    """The use the calls are made for: a stack of inner products whose activations stay real between them, captured once
    and replayed on new inputs; the same bits as the same calls made one by one, and near the layers in 64 bits."""
    sizes = [1000, 512, 300, 10]
    layers = [_layer(Bn, k, o, block, 10 + i) for i, (k, o) in enumerate(zip(sizes, sizes[1:]))]
    exps = [-8, -8, -8] if block == 16 else [0, 0, 0]
    x = torch.zeros(Bn, sizes[0], dtype=torch.bfloat16, device="cuda")
    acts = [torch.empty(Bn, o, dtype=torch.bfloat16 if o != 10 else torch.float32, device="cuda") for o in sizes[1:]]
    st = B.new_stats()
    ws = torch.empty(max(B.fp4_act_ip_workspace_bytes(Bn, k, o, block) for k, o in zip(sizes, sizes[1:])), dtype=torch.uint8, device="cuda")

    def step():
        h = x
        for i, (k, o) in enumerate(zip(sizes, sizes[1:])):
            B.adaption_fp4_act_ip_fwd(Bn, k, o, h, exps[i], layers[i][0], layers[i][1], i < 2, acts[i], st, ws)
            h = acts[i]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in (1, 2, 3):
        rng = np.random.default_rng(seed)
        with torch.cuda.stream(side):
            x.copy_(torch.from_numpy(np.maximum(rng.standard_normal((Bn, sizes[0])), 0)).to(torch.bfloat16))
            graph.replay()
        side.synchronize()
        replayed = [a.clone() for a in acts]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(acts, replayed))
        h = x.double().cpu().numpy()
        for i in range(3):
            code, byte, _ = ms.quantize(h, block, exps[i])
            wc, wb, _, _ = logical(layers[i][0])
            xv, wv = ms.values(code, byte, block, exps[i]), ms.values(wc, wb, block, layers[i][0].exp)
            check_product(acts[i], xv, wv, layers[i][1].cpu().numpy(), i < 2, block, "bf16" if i < 2 else "f32")
            h = acts[i].double().cpu().numpy()
    assert B.read_stats(st).status == 0


def test_repeated_and_concurrent_calls_give_the_same_bits():
    rng = np.random.default_rng(5)
    x, _ = operand(rng, 40, 3000, 16)
    w, _ = operand(rng, 500, 3000, 16)
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty(40, 500, device="cuda") for _ in range(6)]
    st = B.new_stats()
    torch.cuda.synchronize()
    for i, y in enumerate(outs):
        with torch.cuda.stream(streams[i % 3]):
            B.adaption_fp4_ip_fwd(40, 3000, 500, x, w, None, False, y, st)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0], y) for y in outs[1:])


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
def test_a_tensor_times_itself(kernel):
    choose(kernel)
    rng = np.random.default_rng(8)
    for rows, K in ((5, 96), (300, 1000)):
        x, xv = operand(rng, rows, K, 16)
        y, st = torch.empty(rows, rows, device="cuda"), B.new_stats()
        B.adaption_fp4_ip_fwd(rows, K, rows, x, x, None, False, y, st)
        check_product(y, xv, xv, None, False, 16, "f32")


def test_products_of_two_streams_with_layers_beside_them():
    """Products in clusters, and the layers' clusters, all of which hold TMEM while they wait for one another."""
    rng = np.random.default_rng(18)
    x, xv = operand(rng, 40, 4096, 16)
    w, wv = operand(rng, 640, 4096, 16)
    B_, K, O = 16, 1024, 512
    xq = to_qtensor(rng.integers(-2000, 2000, (B_, K)), 16, 8, K)
    wq = to_qtensor(rng.integers(-2000, 2000, (O, K)), 16, 8, K)
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs, layers, st = [], [], B.new_stats()
    work = [torch.empty(B_ * O * 8, dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for i in range(30):
        with torch.cuda.stream(streams[i % 3]):
            if i % 2:
                outs.append(torch.empty(40, 640, device="cuda"))
                B.adaption_fp4_ip_fwd(40, 4096, 640, x, w, None, False, outs[-1], st)
            else:
                layers.append(B.QTensor.empty(B_, O, 16, 4))
                B.adaption_lp_ip_fwd(B_, K, O, xq, wq, None, 0, False, B.MODE_REQUANT, B.ALGO_AUTO, layers[-1], st, work[i % 3])
    torch.cuda.synchronize()
    check_product(outs[0], xv, wv, None, False, 16, "f32")
    assert all(torch.equal(outs[0], y) for y in outs[1:])
    assert all(torch.equal(layers[0].lo, y.lo) and torch.equal(layers[0].hi, y.hi) for y in layers[1:])
    assert B.read_stats(st).status == 0


def test_quantizer_and_values_of_more_rows_than_one_launch_takes():
    """Rows of 8 elements, more than 2^32 bytes of x and of y: the first rows, those around the second launch's first one, the last."""
    inner, pitch, rows = 8, 36, (1 << 26) + 1000                    # (two pieces of a row of codes: 2^26 rows a launch)
    rng = np.random.default_rng(6)
    x = torch.zeros(rows, pitch, dtype=torch.bfloat16, device="cuda")
    q = B.Fp4Tensor.empty(rows, inner, 16, -5)
    q.codes.fill_(0xA5)
    places = [0, (1 << 26) - 256, rows - rows % 128 - 256]
    parts = [torch.from_numpy(rng.standard_normal((400, inner))).to(torch.bfloat16).cuda() for _ in places]
    for at, part in zip(places, parts):
        x[at:at + 400, :inner] = part[:rows - at]
    B.adaption_fp4_quantize(x[:, :inner], rows, inner, q)
    y = torch.empty(rows, pitch, dtype=torch.bfloat16, device="cuda")
    B.adaption_fp4_dequantize(q, rows, inner, y[:, :inner])
    for at in places:
        n = min(400, rows - at)
        ref = x[at:at + n, :inner].double().cpu().numpy()
        code, byte, _ = ms.quantize(ref, 16, -5)
        here = B.Fp4Tensor(n, inner, 32, 16, -5, q.codes[at * 16:(at + n) * 16], q.scales[at // 128 * 512:])
        got, got_byte, pad, _ = logical(here)
        assert np.array_equal(got, code) and np.array_equal(got_byte, byte) and not pad.any()
        assert np.array_equal(y[at:at + n, :inner].double().cpu().numpy(), ms.values(code, byte, 16, -5))
    assert int((q.codes.view(-1, 16)[1000:(1 << 26) - 256] != 0).sum()) == 0


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
def test_outputs_beyond_32_bits_of_offset(kernel):
    """y of more than 2^32 bytes: its first and last rows and channels."""
    choose(kernel)
    Bn, K, O = 1040, 64, (1 << 20) + 5
    rng = np.random.default_rng(9)
    x, xv = operand(rng, Bn, K, 32)
    # weights of a few kinds of rows, so that the reference is small
    code = rng.integers(0, 16, (256, K)).astype(np.uint8)
    byte = rng.integers(120, 130, (256, K // 32)).astype(np.uint8)
    kinds, wv = stored(code, byte, 32), ms.values(code, byte, 32)
    times = -(-O // 256)
    w = B.Fp4Tensor(O, K, K, 32, 0, kinds.codes.repeat(times)[:O * K // 2].contiguous(), kinds.scales.repeat(times))
    y, st = torch.empty(Bn, O, device="cuda"), B.new_stats()
    B.adaption_fp4_ip_fwd(Bn, K, O, x, w, None, False, y, st)
    last = (O - 1) // 256 * 256
    check_product(y[:, :256], xv, wv, None, False, 32, "f32")
    check_product(y[:, last:], xv, wv[:O - last], None, False, 32, "f32")
    for r in (0, 517, Bn - 1):
        assert torch.equal(y[r], y[r, :256].repeat(times)[:O])
    assert B.read_stats(st).status == 0


def test_calls_from_two_host_threads():
    """Two host threads, each with its own stream, buffers and sizes, call at the same time and both get the definition's results."""
    errors = []

    def work(seed, Bn, K, O, block):
        try:
            torch.cuda.set_device(0)
            rng = np.random.default_rng(seed)
            with torch.cuda.stream(torch.cuda.Stream()):
                w, wv = operand(rng, O, K, block, -2 if block == 16 else 0)
                x = real_input(rng, Bn, K, "bf16")
                ref = x.double().cpu().numpy()
                exp = B.adaption_fp4_choose_exp(float(np.abs(ref).max())) if block == 16 else 0
                code, byte, _ = ms.quantize(ref, block, exp)
                ws = torch.empty(B.fp4_act_ip_workspace_bytes(Bn, K, O, block), dtype=torch.uint8, device="cuda")
                for _ in range(20):
                    y, st = torch.empty(Bn, O, device="cuda"), B.new_stats()
                    B.adaption_fp4_act_ip_fwd(Bn, K, O, x, exp, w, None, False, y, st, ws)
                check_product(y, ms.values(code, byte, block, exp), wv, None, False, block, "f32")
        except Exception as exc:                              # noqa: BLE001 - reported to the main thread
            errors.append(exc)

    threads = [threading.Thread(target=work, args=a) for a in ((1, 3, 2000, 300, 16), (2, 200, 640, 520, 32))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


def test_leaves_that_want_gradients_are_read():
    x = torch.randn(4, 64, device="cuda", requires_grad=True)
    q, r = B.Fp4Tensor.empty(4, 64, 32), B.Fp4Tensor.empty(4, 64, 32)
    B.adaption_fp4_quantize(x, 4, 64, q)
    B.adaption_fp4_quantize(torch.nn.Parameter(x.detach().clone()), 4, 64, r)
    code, byte, _ = ms.quantize(x.detach().double().cpu().numpy(), 32)
    for t in (q, r):
        got, got_byte, _, _ = logical(t)
        assert np.array_equal(got, code) and np.array_equal(got_byte, byte)


def test_refusals_of_the_binding():
    q = B.Fp4Tensor.empty(4, 64, 16)
    x, y, st = torch.zeros(4, 64, device="cuda"), torch.zeros(4, 4, device="cuda"), B.new_stats()
    bad_x = [x.double(), x[:, ::2], x.t(), x[:3], x.view(2, 128), x.view(-1), x.cpu(), torch.zeros(4, 128, device="cuda")[:, ::2]]
    for t in bad_x:
        with pytest.raises(B.AdaptionError) as e:
            B.adaption_fp4_quantize(t, 4, 64, q)
        assert e.value.status == B.ERR_INVALID_ARG
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_dequantize(q, 4, 64, t)
    with pytest.raises(B.AdaptionError):
        B.adaption_fp4_quantize(torch.zeros(1, 64, device="cuda").expand(4, 64), 4, 64, q)      # rows on top of one another
    with pytest.raises(B.AdaptionError):
        B.adaption_fp4_quantize(x, 4, 64, B.Fp4Tensor.empty(4, 64, 16, device="cpu"))
    with pytest.raises(B.AdaptionError):
        B.adaption_fp4_quantize(x[:, :32], 4, 32, q)                                             # a tensor of another row length
    with pytest.raises(B.AdaptionError):
        B.adaption_fp4_quantize(torch.zeros(5, 64, device="cuda"), 5, 64, q)                     # more rows than it has
    for plane in ("lo", "hi"):
        fixed = B.QTensor.empty(4, 64, 16, 8)
        setattr(fixed, plane, getattr(fixed, plane).cpu())
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_quantize(fixed, 4, 64, q)
    for bias in (torch.zeros(4, device="cuda", dtype=torch.float64), torch.zeros(3, device="cuda"), torch.zeros(8, device="cuda")[::2], torch.zeros(4)):
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_ip_fwd(4, 64, 4, q, q, bias, False, y, st)
    for args in ((4, 64, 4, q, q, None, False, y.cpu(), st), (4, 64, 4, q, q, None, False, y, st.cpu()), (4, 64, 5, q, q, None, False, y, st),
                 (4, 64, 4, q, B.Fp4Tensor.empty(4, 64, 32), None, False, y, st)):
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_ip_fwd(*args)
    for name, short in (("codes", q.codes[:-1]), ("scales", q.scales[:-1]), ("codes", q.codes.cpu())):
        other = B.Fp4Tensor.empty(4, 64, 16)
        setattr(other, name, short)
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_quantize(x, 4, 64, other)
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_ip_fwd(4, 64, 4, q, other, None, False, y, st)
    for stats in (st[:-1], torch.zeros(1, dtype=torch.uint8, device="cuda")):
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_ip_fwd(4, 64, 4, q, q, None, False, y, stats)
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_quantize(x, 4, 64, q, False, stats)
    wide = B.Fp4Tensor(1, 64, (1 << 25) + 32, 16, 0, torch.zeros((1 << 24) + 16, dtype=torch.uint8, device="cuda"), q.scales)
    with pytest.raises(B.AdaptionError) as e:
        B.adaption_fp4_quantize(x[:1], 1, 64, wide)
    assert e.value.status == B.ERR_UNSUPPORTED
    need = B.fp4_act_ip_workspace_bytes(4, 64, 4, 16)
    for ws in (None, torch.empty(need - 1, dtype=torch.uint8, device="cuda"), torch.empty(need, dtype=torch.uint8)):
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_act_ip_fwd(4, 64, 4, x, 0, q, None, False, y, st, ws)
    # a single row may have any pitch, and no rows are no work
    one = torch.zeros(1, 64, device="cuda").as_strided((1, 64), (1, 1))
    B.adaption_fp4_quantize(one, 1, 64, B.Fp4Tensor.empty(1, 64, 16))
    B.adaption_fp4_ip_fwd(0, 64, 4, B.Fp4Tensor.empty(0, 64, 16), q, None, False, torch.empty(0, 4, device="cuda"), st)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
@pytest.mark.parametrize("Bn", [4, 300])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(Bn, kernel):
    choose(kernel)
    rng = np.random.default_rng(2)
    x, xv = operand(rng, Bn, 2048, 16)
    w, wv = operand(rng, 256, 2048, 16)
    y, st = torch.empty(Bn, 256, device="cuda"), B.new_stats()
    B.adaption_debug_set("timeout_us", 3000)
    B.adaption_debug_set("stall_at", 0)
    B.adaption_fp4_ip_fwd(Bn, 2048, 256, x, w, None, False, y, st)
    torch.cuda.synchronize()
    assert B.read_stats(st).status == B.ERR_TIMEOUT
    B.adaption_debug_set("reset")
    choose(kernel)
    st = B.new_stats()
    B.adaption_fp4_ip_fwd(Bn, 2048, 256, x, w, None, False, y, st)
    check_product(y, xv, wv, None, False, 16, "f32")
    assert B.read_stats(st).status == 0
