"""Microscaled 4-bit products at the ends of their ranges, next to the calls in front of them, and where their waits run out.

Tolerances are those of tests/test_gpu_fp4.py, and for sums near the smallest floats one of these more for every addition: an
addition in 32 bits loses at most half a step of its result, and, should the adder have no denormal numbers, a result below 2^-126.
"""
import numpy as np
import pytest
import torch

from oracle import microscale as ms
from paper_1711_04713_b200 import binding as B
from tests.test_gpu_fp4 import DT, check_product, choose, operand, real_input, stored
from tests.util import dev, to_qtensor

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _defaults():
    B.adaption_debug_set("reset")
    yield
    B.adaption_debug_set("reset")


def workspace(Bn, K, O, block):
    return torch.empty(B.fp4_act_ip_workspace_bytes(Bn, K, O, block), dtype=torch.uint8, device="cuda")


# --------------------------------------------------------------------------- special values
@pytest.mark.parametrize("fused", [0, 2])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("Bn", [1, 4, 48])
def test_infinities_among_the_activations_are_the_largest_finite_number(Bn, block, fused):
    """Weights small enough that the sums stay finite, so that every output of every row is compared."""
    B.adaption_debug_set("fused", fused)
    K, O, exp = 300, 40, -7 if block == 16 else 0
    rng = np.random.default_rng(Bn)
    x = rng.standard_normal((Bn, K)).astype(np.float32)
    x[:, ::37] = np.nan
    x[-1, 100], x[-1, 260], x[0, 5], x[0, 70] = np.inf, -np.inf, 1e30, -3e38
    x[0, 32:48] *= 1e-30
    code = rng.integers(0, 16, (O, K)).astype(np.uint8)
    mid = 127 - 40 if block == 32 else 56
    byte = rng.integers(mid - 3, mid + 4, (O, -(-K // block))).astype(np.uint8)
    w, wv = stored(code, byte, block, -40 if block == 16 else 0), ms.values(code, byte, block, -40 if block == 16 else 0)
    xcode, xbyte, _ = ms.quantize(x, block, exp)
    xv = ms.values(xcode, xbyte, block, exp)
    assert np.isinf(x).any(1).any() and (np.abs(xv) @ np.abs(wv).T).max() < 2.0 ** 120
    y, two, st = torch.empty(Bn, O, device="cuda"), torch.empty(Bn, O, device="cuda"), B.new_stats()
    B.adaption_fp4_act_ip_fwd(Bn, K, O, dev(x), exp, w, None, False, y, st, workspace(Bn, K, O, block))
    q = B.Fp4Tensor.empty(Bn, K, block, exp)
    B.adaption_fp4_quantize(dev(x), Bn, K, q)
    B.adaption_fp4_ip_fwd(Bn, K, O, q, w, None, False, two, st)
    check_product(y, xv, wv, None, False, block, "f32")
    assert torch.equal(y, two) and B.read_stats(st).status == 0


# --------------------------------------------------------------------------- ends of the scales' range
def check_with_flush(y, xv, wv, block, dtype):
    """check_product, but of a sum that may lose 2^-126 with every addition."""
    want = ms.inner_product(xv, wv)
    adds = -(-xv.shape[1] // block) + 8 + 1
    bound = adds * (2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T) + 2.0 ** -126)
    if dtype != "f32":
        eps = torch.finfo(DT[dtype]).eps / 2
        bound = bound + (np.abs(want) + bound) * eps + torch.finfo(DT[dtype]).smallest_normal * eps
    err = np.abs(y.double().cpu().numpy() - want)
    assert np.all(err <= bound), (float((err / bound).max()), np.argwhere(err > bound)[:5].tolist())


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
@pytest.mark.parametrize("bytes_x,bytes_w", [((0, 20), (234, 254)), ((234, 254), (0, 20)), ((0, 20), (0, 20)), ((55, 70), (55, 70)),
                                             ((0, 8), (118, 134)), ((180, 184), (180, 184))])
def test_scales_of_two_at_the_ends_of_their_range(bytes_x, bytes_w, kernel):
    choose(kernel)
    rng = np.random.default_rng(bytes_x[0] + bytes_w[1])
    for Bn, K, O in ((5, 96, 130), (140, 300, 200)):
        ops = []
        for rows, (lo, hi) in ((Bn, bytes_x), (O, bytes_w)):
            code = rng.integers(0, 16, (rows, K)).astype(np.uint8)
            byte = rng.integers(lo, hi + 1, (rows, -(-K // 32))).astype(np.uint8)
            ops.append((stored(code, byte, 32, fill=0xFF), ms.values(code, byte, 32)))
        (x, xv), (w, wv) = ops
        assert (np.abs(xv) @ np.abs(wv).T).max() < 2.0 ** 127
        for dtype in ("f32", "bf16"):
            y, st = torch.full((Bn, O), 7.0, dtype=DT[dtype], device="cuda"), B.new_stats()
            B.adaption_fp4_ip_fwd(Bn, K, O, x, w, None, False, y, st)
            check_with_flush(y, xv, wv, 32, dtype)
            s = B.read_stats(st)
            assert s.status == 0 and s.zeros == int((y == 0).sum())


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
@pytest.mark.parametrize("ex,ew", [(63, -63), (-63, 63), (-63, -63), (63, 63), (63, 40)])
def test_exponents_at_the_ends_of_their_range(ex, ew, kernel):
    """Steps of every number of E4M3.  The sum is formed without the exponents and scaled once, so nothing is lost before the result, which
    is infinite beyond the floats."""
    choose(kernel)
    rng = np.random.default_rng(100 + ex)
    for Bn, K, O in ((5, 96, 130), (140, 300, 200)):
        ops = []
        for rows, e in ((Bn, ex), (O, ew)):
            code = rng.integers(0, 16, (rows, K)).astype(np.uint8)
            byte = rng.integers(0, 127, (rows, -(-K // 16))).astype(np.uint8)
            ops.append((stored(code, byte, 16, e, fill=0xFF), ms.values(code, byte, 16, e)))
        (x, xv), (w, wv) = ops
        y, st = torch.full((Bn, O), 7.0, device="cuda"), B.new_stats()
        B.adaption_fp4_ip_fwd(Bn, K, O, x, w, None, False, y, st)
        want, S = ms.inner_product(xv, wv), np.abs(xv) @ np.abs(wv).T
        bound = (-(-K // 16) + 9) * 2.0 ** -23 * S + 2.0 ** -150
        got = y.double().cpu().numpy()
        inside, beyond = np.abs(want) + bound < ms.FLT_MAX, np.abs(want) - bound > 2.0 ** 128
        assert np.all(np.abs(got - want)[inside] <= bound[inside])
        assert np.array_equal(got[beyond], np.sign(want[beyond]) * np.inf) and (ex + ew < 126 or beyond.any())
        assert B.read_stats(st).status == 0


@pytest.mark.parametrize("kernel", ["cluster", "pairs", "persistent"])
def test_sums_beyond_the_floats_are_infinite(kernel):
    choose(kernel)
    rng = np.random.default_rng(3)
    code = rng.integers(1, 8, (40, 96)).astype(np.uint8)
    t = stored(code, np.full((40, 3), 254, np.uint8), 32)
    for dtype in DT:
        y = torch.empty(40, 40, dtype=DT[dtype], device="cuda")
        B.adaption_fp4_ip_fwd(40, 96, 40, t, t, None, False, y, B.new_stats())
        assert bool((y == float("inf")).all())


# --------------------------------------------------------------------------- sizes
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("shape", [(600, 1024, 2048), (2048, 520, 1500), (1100, 300, 4112)])
def test_many_rows_of_real_activations(shape, block):
    """Prompts: the quantizer and the kernel over pairs, or wide tiles of clusters."""
    Bn, K, O = shape
    rng = np.random.default_rng(Bn)
    x = real_input(rng, Bn, K, "bf16")
    ref = x.double().cpu().numpy()
    exp = B.adaption_fp4_choose_exp(float(np.abs(ref).max())) if block == 16 else 0
    w, wv = operand(rng, O, K, block, -2 if block == 16 else 0)
    bias = rng.standard_normal(O).astype(np.float32)
    code, byte, _ = ms.quantize(ref, block, exp)
    ws, q, st = workspace(Bn, K, O, block), B.Fp4Tensor.empty(Bn, K, block, exp), B.new_stats()
    B.adaption_fp4_quantize(x, Bn, K, q)
    for kernel in ("chosen", "persistent"):
        choose(kernel)
        y, two = (torch.empty(Bn, O, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        B.adaption_fp4_act_ip_fwd(Bn, K, O, x, exp, w, dev(bias), True, y, st, ws)
        B.adaption_fp4_ip_fwd(Bn, K, O, q, w, dev(bias), True, two, st)
        check_product(y, ms.values(code, byte, block, exp), wv, bias, True, block, "bf16")
        assert torch.equal(y, two)
    assert B.read_stats(st).status == 0


@pytest.mark.parametrize("shape", [(8, 2048, 28672), (3, 4096, 11008), (1, 512, 130000)])
def test_few_rows_onto_wide_outputs_are_the_two_calls(shape):
    Bn, K, O = shape
    rng = np.random.default_rng(O)
    x = real_input(rng, Bn, K, "bf16")
    ref = x.double().cpu().numpy()
    exp = B.adaption_fp4_choose_exp(float(np.abs(ref).max()))
    code, byte, _ = ms.quantize(ref, 16, exp)
    w, wv = operand(rng, O, K, 16, -2)
    q, st, two = B.Fp4Tensor.empty(Bn, K, 16, exp), B.new_stats(), torch.empty(Bn, O, device="cuda")
    B.adaption_fp4_quantize(x, Bn, K, q)
    B.adaption_fp4_ip_fwd(Bn, K, O, q, w, None, False, two, st)
    check_product(two, ms.values(code, byte, 16, exp), wv, None, False, 16, "f32")
    for fused in (0, 1, 2):
        B.adaption_debug_set("fused", fused)
        y = torch.empty_like(two)
        B.adaption_fp4_act_ip_fwd(Bn, K, O, x, exp, w, None, False, y, st, workspace(Bn, K, O, 16))
        assert torch.equal(y, two), fused
    assert B.read_stats(st).status == 0


# --------------------------------------------------------------------------- order of calls
@pytest.mark.parametrize("by", ["quantizer", "copies"])
@pytest.mark.parametrize("shape", [(16, 4096, 4096), (5, 12800, 2048), (300, 1024, 4096), (4, 4096, 4096)])
def test_weights_rewritten_right_before_the_product(shape, by):
    """A product's first copies of its weights may run beside the quantizer of its activations: never beside what writes the weights."""
    Bn, K, O = shape
    g = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn(Bn, K, device="cuda", generator=g).to(torch.bfloat16)
    real = [torch.randn(O, K, device="cuda", generator=g) for _ in range(2)]
    kept = [B.Fp4Tensor.empty(O, K, 16, -8) for _ in range(2)]
    w, ws, st = B.Fp4Tensor.empty(O, K, 16, -8), workspace(Bn, K, O, 16), B.new_stats()
    outs = [torch.empty(Bn, O, device="cuda") for _ in range(8)]

    def write(k):
        if by == "quantizer":
            B.adaption_fp4_quantize(real[k], O, K, w)
        else:
            w.scales.copy_(kept[k].scales)
            w.codes.copy_(kept[k].codes)

    def step(k, y):
        write(k)
        B.adaption_fp4_act_ip_fwd(Bn, K, O, x, -8, w, None, False, y, st, ws)

    B.adaption_debug_set("pdl", 0)
    for k in range(2):
        B.adaption_fp4_quantize(real[k], O, K, kept[k])
    want = [torch.empty(Bn, O, device="cuda") for _ in range(2)]
    for k in range(2):
        step(k, want[k])
        torch.cuda.synchronize()
    assert not torch.equal(want[0], want[1])
    B.adaption_debug_set("reset")
    for i, y in enumerate(outs):
        step(i % 2, y)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(outs))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for i, y in enumerate(outs):
            step(i % 2, y)
    for _ in range(3):
        for y in outs:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(outs))
    assert B.read_stats(st).status == 0


def test_concurrent_products_are_right():
    rng = np.random.default_rng(5)
    x, xv = operand(rng, 40, 3000, 16)
    w, wv = operand(rng, 500, 3000, 16)
    streams, st = [torch.cuda.Stream() for _ in range(3)], B.new_stats()
    outs = [torch.empty(40, 500, device="cuda") for _ in range(9)]
    torch.cuda.synchronize()
    for i, y in enumerate(outs):
        with torch.cuda.stream(streams[i % 3]):
            B.adaption_fp4_ip_fwd(40, 3000, 500, x, w, None, False, y, st)
    torch.cuda.synchronize()
    check_product(outs[0], xv, wv, None, False, 16, "f32")
    assert all(torch.equal(outs[0], y) for y in outs[1:])
    s = B.read_stats(st)
    assert s.status == 0 and s.zeros == 9 * int((outs[0] == 0).sum())


# --------------------------------------------------------------------------- waits that run out
def _stalled(call, stall_at, settings):
    """The status that the call reports when the copies of every block stop before their stall_at-th stage."""
    for name, value in settings.items():
        B.adaption_debug_set(name, value)
    st = B.new_stats()
    B.adaption_debug_set("timeout_us", 3000)
    B.adaption_debug_set("stall_at", stall_at)
    call(st)
    torch.cuda.synchronize()
    B.adaption_debug_set("reset")
    for name, value in settings.items():
        B.adaption_debug_set(name, value)
    return B.read_stats(st).status


@pytest.mark.parametrize("stall_at", [0, 2])
@pytest.mark.parametrize("settings", [{"pair": 0, "cluster": 2, "cluster_size": 1}, {"pair": 0, "cluster": 2, "cluster_size": 2},
                                      {"pair": 1, "cluster": 2, "cluster_size": 2}, {"pair": 1, "cluster": 2, "cluster_size": 4}, {"pair": 1}])
@pytest.mark.parametrize("Bn", [4, 300])
def test_stalls_of_4_bit_products(Bn, settings, stall_at):
    rng = np.random.default_rng(2)
    K, O = 2048, 256                                   # eight k-blocks, four a share where there are two
    x, xv = operand(rng, Bn, K, 16)
    w, wv = operand(rng, O, K, 16)
    y = torch.empty(Bn, O, device="cuda")

    def call(st):
        B.adaption_fp4_ip_fwd(Bn, K, O, x, w, None, False, y, st)

    assert _stalled(call, stall_at, settings) == B.ERR_TIMEOUT
    st = B.new_stats()
    call(st)
    check_product(y, xv, wv, None, False, 16, "f32")
    assert B.read_stats(st).status == 0


@pytest.mark.parametrize("stall_at", [0, 2])
@pytest.mark.parametrize("Bn,fused,size", [(1, 2, 1), (4, 2, 2), (40, 2, 2), (4, 0, 2), (40, 0, 2), (300, 1, 0)])
def test_stalls_of_products_on_real_activations(Bn, fused, size, stall_at):
    """Quantized by the product's idle warps, which then wait for the ring, or in a launch of their own."""
    rng = np.random.default_rng(4)
    K, O = {0: 1024, 1: 8192, 2: 2048}[size], 256      # (8192: more k-blocks than the ring has stages)
    x = real_input(rng, Bn, K, "bf16")
    code, byte, _ = ms.quantize(x.double().cpu().numpy(), 16, -5)
    w, wv = operand(rng, O, K, 16)
    y, ws = torch.empty(Bn, O, device="cuda"), workspace(Bn, K, O, 16)
    settings = {"fused": fused, "pair": 0 if size else 1, "cluster": 2 if size else 1, "cluster_size": size}

    def call(st):
        B.adaption_fp4_act_ip_fwd(Bn, K, O, x, -5, w, None, False, y, st, ws)

    assert _stalled(call, stall_at, settings) == B.ERR_TIMEOUT
    st = B.new_stats()
    call(st)
    check_product(y, ms.values(code, byte, 16, -5), wv, None, False, 16, "f32")
    assert B.read_stats(st).status == 0


def test_a_stall_in_a_pairs_second_tile():
    """85 tiles on fewer pairs, two k-blocks each: the first tiles are stored, a second one stops between its k-blocks."""
    Bn, K, O = 1100, 300, 4112
    rng = np.random.default_rng(6)
    x, xv = operand(rng, Bn, K, 16)
    w, wv = operand(rng, O, K, 16)
    y = torch.empty(Bn, O, device="cuda")

    def call(st):
        B.adaption_fp4_ip_fwd(Bn, K, O, x, w, None, False, y, st)

    assert _stalled(call, 3, {"pair": 1}) == B.ERR_TIMEOUT
    st = B.new_stats()
    call(st)
    check_product(y, xv, wv, None, False, 16, "f32")
    assert B.read_stats(st).status == 0


# --------------------------------------------------------------------------- refusals
def test_buffers_that_are_too_short_are_refused():
    """(All answered on the host.)"""
    q, st = B.Fp4Tensor.empty(6, 70, 16), B.new_stats()
    one = torch.zeros(1, dtype=torch.uint8, device="cuda")
    x, y = torch.zeros(6, 70, device="cuda"), torch.zeros(6, 6, device="cuda")
    for plane in ("lo", "hi"):
        for short in (one.expand(480), one, torch.zeros(479, dtype=torch.uint8, device="cuda"), torch.zeros(960, dtype=torch.uint8, device="cuda")[::2]):
            fixed = to_qtensor(np.zeros((6, 70), np.int64), 16, 3, 80)
            setattr(fixed, plane, short)
            with pytest.raises(B.AdaptionError) as e:
                B.adaption_fp4_quantize(fixed, 6, 70, q)
            assert e.value.status == B.ERR_INVALID_ARG
    need = B.fp4_act_ip_workspace_bytes(6, 70, 6, 16)
    for ws in (one.expand(need), torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(B.AdaptionError) as e:
            B.adaption_fp4_act_ip_fwd(6, 70, 6, x, 0, q, None, False, y, st, ws)
        assert e.value.status == B.ERR_INVALID_ARG
    for name in ("codes", "scales"):
        other = B.Fp4Tensor.empty(6, 70, 16)
        setattr(other, name, one.expand(getattr(other, name).numel()))
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_quantize(x, 6, 70, other)
        with pytest.raises(B.AdaptionError):
            B.adaption_fp4_ip_fwd(6, 70, 6, q, other, None, False, y, st)
    wide = torch.zeros(B.STATS_BYTES + 8, dtype=torch.uint8, device="cuda")
    for off in (1, 4):
        with pytest.raises(B.AdaptionError) as e:
            B.adaption_fp4_ip_fwd(6, 70, 6, q, q, None, False, y, wide[off:off + B.STATS_BYTES])
        assert e.value.status == B.ERR_ALIGNMENT
