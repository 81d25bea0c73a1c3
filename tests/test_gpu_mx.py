"""GPU parity: microscaled tensors and the layer on them against the oracle.

Codes, scales and values are bit-exact.  A product sums K exact products of two exactly represented operands in binary32, in an
order (and with an alignment of addends) that the hardware chooses: each addition loses at most one unit in the last place
of a running sum of at most B = sum_k |x w|, so |y - exact| <= K 2^-23 B, plus 2^-8 |y| (half a step) in bfloat16.  Gradients: the
same over the N or M terms, plus six roundings for the transform of 32, whose outputs are at most sum |.| / sqrt(32) of
the block."""
import numpy as np
import pytest
import torch

from oracle import mx

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def rows(shape, seed, dtype=BF16, spread=3.0):
    """Normal rows whose blocks differ in size by powers of e."""
    rng = np.random.default_rng(seed)
    a = rng.standard_normal(shape) * np.exp(rng.uniform(-spread, spread, (shape[0], shape[1] // 32))).repeat(32, axis=1)
    return torch.from_numpy(a.astype(np.float32)).to(dtype)


def oracle_of(x, bits, g=1):
    codes, scales = mx.quantize(x.float().numpy(), bits, g)
    return codes, scales, mx.values(codes, scales, bits)


def check_product(y, xv, wv):
    exact = xv @ wv.T
    lim = xv.shape[1] * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T) + (2.0 ** -8 * np.abs(exact) if y.dtype == BF16 else 0.0)
    err = np.abs(y.cpu().double().numpy() - exact)
    assert np.all(err <= lim + 1e-37), f"worst element at {np.max(err / (lim + 1e-37)):.3f} of the bound"


def status():
    import paper_2502_05003_b200 as quest
    torch.cuda.synchronize()
    assert quest.quest_device_status() == 0


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("g", [1, 32])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K", [(1, 32), (3, 96), (33, 160), (130, 128), (128, 2048), (5, 5504), (2, 16384)])
def test_codes_scales_and_values(M, K, dtype, g, bits):
    import paper_2502_05003_b200 as quest
    x = rows((M, K), M + K, dtype)
    codes, scales, values = oracle_of(x, bits, g)
    qc, qs = quest.quest_quantize_mx(x.cuda(), bits, g)
    assert np.array_equal(qc.cpu().numpy(), mx.pack(codes, bits))
    assert np.array_equal(qs.cpu().numpy(), mx.tile(scales))
    for out in (BF16, F32):
        v = quest.quest_dequantize_mx(qc, qs, bits, out)
        assert v.dtype == out and np.array_equal(v.cpu().double().numpy(), values)


@pytest.mark.parametrize("bits", [4, 8])
def test_edges_of_the_number_range(bits):
    import paper_2502_05003_b200 as quest
    x = torch.zeros((2, 320))
    x[0, 32], x[0, 64], x[0, 96], x[0, 130] = 1e-45, 3.4e38, float("nan"), float("-inf")
    x[0, 160:192] = torch.linspace(-8, 8, 32)             # ties and saturation
    x[0, 192:224] = torch.arange(32) * 0.25 - 4
    x[0, 224:256] = torch.tensor(2.0 ** -126) * torch.arange(32)
    x[0, 256:288] = -0.0
    x[1] = float("nan")
    codes, scales, values = oracle_of(x, bits)
    qc, qs = quest.quest_quantize_mx(x.cuda(), bits)
    assert np.array_equal(qc.cpu().numpy(), mx.pack(codes, bits)) and np.array_equal(qs.cpu().numpy(), mx.tile(scales))
    v = quest.quest_dequantize_mx(qc, qs, bits, F32).cpu().double().numpy()
    assert np.array_equal(v, values, equal_nan=True)


def test_every_scale_and_every_code_reads_back():
    import paper_2502_05003_b200 as quest
    for bits, n in ((4, 16), (8, 256)):
        codes = np.tile(np.arange(n, dtype=np.uint8), 256 * 256 // n).reshape(256, 256)
        scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 8, axis=1)
        v = quest.quest_dequantize_mx(torch.from_numpy(mx.pack(codes, bits)).cuda(), torch.from_numpy(mx.tile(scales)).cuda(), bits, F32)
        # values past the largest binary32 number (scales that the quantizer does not reach) read as infinities
        with np.errstate(over="ignore"):
            want = mx.values(codes, scales, bits).astype(np.float32)
        assert np.array_equal(v.cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,N,K", [(33, 8, 128), (40, 130, 256), (64, 64, 384), (129, 300, 512), (256, 256, 640), (257, 513, 1152),
                                   (300, 1000, 2048), (777, 256, 5504)])
def test_products_of_many_rows(M, N, K, bits):
    import paper_2502_05003_b200 as quest
    x, w = rows((M, K), 1), rows((N, K), 2)
    xc, xs, xv = oracle_of(x, bits)
    wc, ws, wv = oracle_of(w, 4)
    t = [torch.from_numpy(a).cuda() for a in (mx.pack(xc, bits), mx.tile(xs), mx.pack(wc, 4), mx.tile(ws))]
    for out in (F32, BF16):
        check_product(quest.quest_gemm_mx(t[0], t[1], bits, t[2], t[3], K, out), xv, wv)
    status()


@pytest.mark.parametrize("K", [32, 64, 96, 160, 288, 416, 1376])
def test_four_bit_products_of_every_row_length(K):
    import paper_2502_05003_b200 as quest
    x, w = rows((70, K), 3), rows((90, K), 4)
    for M in (5, 70):
        r = quest.quest_linear_fwd_mx(x[:M].cuda(), w.cuda(), 4, 1, F32)
        check_product(r["y"], oracle_of(x[:M], 4)[2], oracle_of(w, 4)[2])
    status()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("g", [1, 32])
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 24, 25, 32, 33])
def test_few_rows_from_values_and_from_codes(M, g, bits):
    import paper_2502_05003_b200 as quest
    N, K = (200 if M % 2 else 77), (384 if bits == 8 else 416)
    for dtype in (BF16, F32):
        x, w = rows((M, K), M, dtype), rows((N, K), 5)
        xv, (wc, ws, wv) = oracle_of(x, bits, g)[2], oracle_of(w, 4, g)
        cached = {"wq": torch.from_numpy(mx.pack(wc, 4)).cuda(), "sw": torch.from_numpy(mx.tile(ws)).cuda()}
        for out in (F32, BF16):
            fused = quest.quest_linear_fwd_mx(x.cuda(), None, bits, g, out, w_cached=cached, want_codes=False)
            assert (fused["xq"] is None) == (M <= 8 and M * K <= 4096)
            check_product(fused["y"], xv, wv)
            stored = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), bits, g, out)
            assert torch.equal(stored["wq"], cached["wq"]) and torch.equal(stored["sw"], cached["sw"])
            assert torch.equal(stored["y"], fused["y"])            # the same products in the same order
            assert torch.equal(quest.quest_gemm_mx(stored["xq"], stored["sx"], bits, cached["wq"], cached["sw"], K, out), fused["y"])
    status()


def test_wide_weights_take_several_rows_a_cta():
    import paper_2502_05003_b200 as quest
    x = rows((20, 256), 7)
    for N in (4800, 9600, 14500):
        w = rows((N, 256), N)
        codes, scales = quest.quest_quantize_mx(w.cuda(), 4)
        y = quest.quest_linear_fwd_mx(x.cuda(), None, 8, 1, F32, w_cached={"wq": codes, "sw": scales}, want_codes=False)["y"]
        wv = quest.quest_dequantize_mx(codes, scales, 4, F32).cpu().double().numpy()
        check_product(y, oracle_of(x, 8)[2], wv)
    status()


@pytest.mark.parametrize("M", [4, 200])
def test_strided_and_misaligned_rows_and_outputs(M):
    import paper_2502_05003_b200 as quest
    K, N = 256, 130
    x, w = rows((M, K), 8), rows((N, K), 9)
    r = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), 8, 32, F32)
    wide = torch.zeros((M, K + 24), dtype=BF16, device="cuda")
    wide[:, 8:8 + K] = x.cuda()
    odd = torch.zeros((M, K + 1), dtype=BF16, device="cuda")
    odd[:, 1:] = x.cuda()
    for xs in (wide[:, 8:8 + K], odd[:, 1:], x.cuda().t().contiguous().t()):
        assert torch.equal(quest.quest_linear_fwd_mx(xs, w.cuda(), 8, 32, F32)["y"], r["y"])
    c, s = quest.quest_quantize_mx(wide[:, 8:8 + K], 8, 32)
    assert torch.equal(c, r["xq"]) and torch.equal(s, r["sx"])
    for dtype, shape, cols in ((F32, (M + 2, N + 7), slice(3, 3 + N)), (F32, (M + 2, N + 2), slice(0, N)), (BF16, (M + 2, N + 5), slice(5, 5 + N)),
                               (BF16, (M + 2, N + 6), slice(0, N))):
        room = torch.full(shape, 7.0, dtype=dtype, device="cuda")
        y = room[1:M + 1, cols]
        got = quest.quest_gemm_mx(r["xq"], r["sx"], 8, r["wq"], r["sw"], K, y=y)
        assert got is y and torch.equal(y, r["y"].to(dtype))
        y.fill_(7.0)
        assert bool((room == 7.0).all())                  # nothing beside y was touched
    status()


@pytest.mark.parametrize("M", [3, 100])
@pytest.mark.parametrize("bits", [4, 8])
def test_blocks_that_are_not_finite_reach_their_rows_only(M, bits):
    import paper_2502_05003_b200 as quest
    x, w = rows((M, 512), 10), rows((70, 512), 11)
    clean = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), bits, 1, F32)["y"]
    x[1, 100], w[7, 300], w[8, 511] = float("nan"), float("inf"), float("nan")
    y = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), bits, 1, F32)["y"]
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[1], bad[:, 7], bad[:, 8] = True, True, True
    assert bool(y[bad].isnan().all()) and torch.equal(y[~bad], clean[~bad])
    y = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), bits, 1, F32, want_codes=False)["y"]
    assert bool(y[bad].isnan().all()) and torch.equal(y[~bad], clean[~bad])
    status()


@pytest.mark.parametrize("M", [2, 90])
def test_extreme_scales(M):
    import paper_2502_05003_b200 as quest
    rng = np.random.default_rng(12)
    for ex, ew in ((60, 60), (-60, -40), (100, -100), (-110, 110), (0, 120), (118, -20)):
        x = torch.from_numpy((rng.standard_normal((M, 256)).clip(-3, 3) * 2.0 ** ex).astype(np.float32))
        w = torch.from_numpy((rng.standard_normal((48, 256)).clip(-3, 3) * 2.0 ** ew).astype(np.float32))
        r = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), 8, 1, F32)
        check_product(r["y"], oracle_of(x, 8)[2], oracle_of(w, 4)[2])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M", [2, 20, 90])
def test_products_under_every_scale(M, bits):
    import paper_2502_05003_b200 as quest
    # scales that meet at 2^-8 .. 2^8 together, from both ends of their range; scale 255 is left out
    rng = np.random.default_rng(27)
    for sw in (0, 1, 2, 60, 127, 200, 253, 254):
        xc = rng.integers(0, 16 if bits == 4 else 256, (M, 256)).astype(np.uint8)
        xc[(xc & 127) == 127] = 0                              # E4M3 has two codes for NaN
        wc, ws = rng.integers(0, 16, (40, 256)).astype(np.uint8), np.full((40, 8), sw, np.uint8)
        xs = np.clip(254 - sw + rng.integers(-8, 9, (M, 8)), 0, 254).astype(np.uint8)
        t = [torch.from_numpy(a).cuda() for a in (mx.pack(xc, bits), mx.tile(xs), mx.pack(wc, 4), mx.tile(ws))]
        y = quest.quest_gemm_mx(t[0], t[1], bits, t[2], t[3], 256, F32)
        check_product(y, mx.values(xc, xs, bits), mx.values(wc, ws, 4))
    status()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("g", [1, 32])
@pytest.mark.parametrize("M,N,K", [(8, 8, 128), (64, 40, 256), (264, 520, 384), (1000, 72, 1024), (48, 1032, 2048)])
def test_gradients(M, N, K, g, bits):
    import paper_2502_05003_b200 as quest
    x, w = rows((M, K), 13, spread=1.0), rows((N, K), 14, spread=1.0)
    dy = torch.from_numpy(np.random.default_rng(15).standard_normal((M, N)).astype(np.float32)).to(BF16)
    r = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), bits, g)
    dx, dw, bx, bw = mx.backward(dy.double().numpy(), oracle_of(x, bits, g)[2], oracle_of(w, 4, g)[2], g)
    for out in (F32, BF16):
        d = quest.quest_linear_bwd_mx(dy.cuda(), r, bits, g, K, out)
        for got, want, bound, terms in ((d["dx"], dx, bx, N), (d["dw"], dw, bw, M)):
            assert got.dtype == out
            lim = (terms + 6) * 2.0 ** -23 * bound + (2.0 ** -8 * np.abs(want) if out == BF16 else 0.0)
            assert np.all(np.abs(got.cpu().double().numpy() - want) <= lim + 1e-37)
        only = quest.quest_linear_bwd_mx(dy.cuda(), {"wq": r["wq"], "sw": r["sw"]}, bits, g, K, out, want_dw=False)
        assert only["dw"] is None and torch.equal(only["dx"], d["dx"])
        only = quest.quest_linear_bwd_mx(dy.cuda(), {"xq": r["xq"], "sx": r["sx"]}, bits, g, K, out, want_dx=False)
        assert only["dx"] is None and torch.equal(only["dw"], d["dw"])
    status()


@pytest.mark.parametrize("K", [32, 96, 1376])
def test_gradients_of_four_bit_rows_of_every_length(K):
    import paper_2502_05003_b200 as quest
    x, w = rows((48, K), 16, spread=1.0), rows((56, K), 17, spread=1.0)
    dy = rows((48, 56 // 8 * 32), 18, spread=0.1)[:, :56].contiguous()
    for g in (1, 32):
        r = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), 4, g)
        dx, dw, bx, bw = mx.backward(dy.double().numpy(), oracle_of(x, 4, g)[2], oracle_of(w, 4, g)[2], g)
        d = quest.quest_linear_bwd_mx(dy.cuda(), r, 4, g, K)
        assert np.all(np.abs(d["dx"].cpu().double().numpy() - dx) <= (56 + 6) * 2.0 ** -23 * bx + 1e-37)
        assert np.all(np.abs(d["dw"].cpu().double().numpy() - dw) <= (48 + 6) * 2.0 ** -23 * bw + 1e-37)
    status()


def test_long_tensors_pass_32_bit_offsets():
    import paper_2502_05003_b200 as quest
    # 2^31 bytes of codes and more: the last rows are those of a small tensor of the same content
    M, K = 140000, 16384
    x = torch.zeros((M, K), dtype=BF16, device="cuda")
    tail = rows((130, K), 19).cuda()
    x[-130:] = tail
    codes, scales = quest.quest_quantize_mx(x, 8)
    del x
    tc, _ = quest.quest_quantize_mx(tail, 8)
    assert torch.equal(codes[-130:], tc) and not bool(codes[:1000].any())
    w = rows((40, K), 20).cuda()
    wq, sw = quest.quest_quantize_mx(w, 4)
    y = quest.quest_gemm_mx(codes, scales, 8, wq, sw, K, F32)
    small = quest.quest_linear_fwd_mx(tail, None, 8, 1, F32, w_cached={"wq": wq, "sw": sw})["y"]
    assert torch.equal(y[-130:], small)
    v = quest.quest_dequantize_mx(codes, scales, 8)
    assert torch.equal(v[-130:], quest.quest_dequantize_mx(tc, quest.quest_quantize_mx(tail, 8)[1], 8))
    status()


def test_other_streams_and_captured_graphs():
    import paper_2502_05003_b200 as quest
    x, w = rows((48, 512), 21).cuda(), rows((96, 512), 22).cuda()
    dy = rows((48, 96), 23).cuda()
    want = quest.quest_linear_fwd_mx(x, w, 8, 32)
    grads = quest.quest_linear_bwd_mx(dy, want, 8, 32, 512)
    few = quest.quest_linear_fwd_mx(x[:5], None, 8, 32, w_cached=want, want_codes=False)["y"]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = quest.quest_linear_fwd_mx(x, w, 8, 32)
    side.synchronize()
    assert torch.equal(again["y"], want["y"]) and torch.equal(again["xq"], want["xq"])
    static, graph = x.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = quest.quest_linear_fwd_mx(static, w, 8, 32)
        d = quest.quest_linear_bwd_mx(dy, r, 8, 32, 512)
        f = quest.quest_linear_fwd_mx(static[:5], None, 8, 32, w_cached=r, want_codes=False)["y"]
    for _ in range(3):
        static.zero_()
        graph.replay()
        static.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r["y"], want["y"]) and torch.equal(d["dx"], grads["dx"]) and torch.equal(d["dw"], grads["dw"]) and torch.equal(f, few)
    status()


def test_empty_calls():
    import paper_2502_05003_b200 as quest
    w = rows((16, 128), 24).cuda()
    x = torch.empty((0, 128), dtype=BF16, device="cuda")
    c, s = quest.quest_quantize_mx(x, 8)
    assert c.shape == (0, 128) and s.numel() == 0
    assert quest.quest_dequantize_mx(c, s, 8).shape == (0, 128)
    wq, sw = quest.quest_quantize_mx(w, 4)
    wx, sx = quest.quest_quantize_mx(w, 8)
    r = quest.quest_linear_fwd_mx(x, w, 8)
    assert r["y"].shape == (0, 16) and torch.equal(r["wq"], wq) and torch.equal(r["sw"], sw)
    r = quest.quest_linear_fwd_mx(w, x, 8)
    assert r["y"].shape == (16, 0) and torch.equal(r["xq"], wx) and torch.equal(r["sx"], sx)
    assert quest.quest_gemm_mx(wx, sx, 8, r["wq"], r["sw"], 128).shape == (16, 0)


def test_refusals():
    import paper_2502_05003_b200 as quest
    x, w = rows((40, 256), 25).cuda(), rows((16, 256), 26).cuda()
    r = quest.quest_linear_fwd_mx(x, w, 8)
    refused = [
        (lambda: quest.quest_quantize_mx(x, 5), ValueError), (lambda: quest.quest_quantize_mx(x, 4, 16), quest.QuestError),
        (lambda: quest.quest_quantize_mx(x.half(), 4), TypeError), (lambda: quest.quest_quantize_mx(x.cpu(), 4), ValueError),
        (lambda: quest.quest_quantize_mx(x[:, :40], 4), quest.QuestError), (lambda: quest.quest_quantize_mx(x[:, ::2], 4), ValueError),
        (lambda: quest.quest_quantize_mx(x[0], 4), ValueError), (lambda: quest.quest_quantize_mx(x[:, 1:33], 4), quest.QuestError),
        (lambda: quest.quest_quantize_mx(x, 8, codes=r["xq"][:39].contiguous()), ValueError),
        (lambda: quest.quest_quantize_mx(x, 8, scales=r["sx"].float()), ValueError),
        (lambda: quest.quest_dequantize_mx(r["xq"], r["sx"][:-1], 8), ValueError), (lambda: quest.quest_dequantize_mx(r["xq"].int(), r["sx"], 8), ValueError),
        (lambda: quest.quest_dequantize_mx(r["xq"], r["sx"], 8, torch.float16), TypeError),
        (lambda: quest.quest_gemm_mx(r["xq"], r["sx"], 8, r["wq"][:, :64].contiguous(), r["sw"], 256), ValueError),
        (lambda: quest.quest_gemm_mx(r["xq"], r["sx"], 4, r["wq"], r["sw"], 256), ValueError),
        (lambda: quest.quest_gemm_mx(r["xq"], r["sx"][:8], 8, r["wq"], r["sw"], 256), ValueError),
        (lambda: quest.quest_gemm_mx(r["xq"], r["sx"], 8, r["wq"], r["sw"], 256, y=torch.empty((40, 15), device="cuda")), ValueError),
        (lambda: quest.quest_linear_fwd_mx(x[:, :160], w[:, :160], 8), quest.QuestError),       # 8-bit rows: groups of 128
        (lambda: quest.quest_linear_fwd_mx(x, w[:, :128], 8), ValueError), (lambda: quest.quest_linear_fwd_mx(x, w, 8, 2), quest.QuestError),
        (lambda: quest.quest_linear_fwd_mx(x, w, 8, out_dtype=torch.float16), TypeError),
        (lambda: quest.quest_linear_fwd_mx(x, None, 8, w_cached={"wq": r["wq"], "sw": r["sw"][:4]}), ValueError),
        (lambda: quest.quest_linear_bwd_mx(x[:, :16].float().contiguous(), r, 8, 1, 256), ValueError),
        (lambda: quest.quest_linear_bwd_mx(x[:39, :16].contiguous(), r, 8, 1, 256), ValueError),
        (lambda: quest.quest_linear_bwd_mx(x[:, :16].contiguous(), {"wq": r["wq"], "sw": r["sw"]}, 8, 1, 256), ValueError),
        (lambda: quest.quest_linear_bwd_mx(x[:, :16].contiguous(), r, 8, 8, 256), quest.QuestError),
        (lambda: quest.quest_linear_bwd_mx(x[:, :16].contiguous(), r, 8, 1, 256, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), quest.QuestError),
    ]
    for i, (call, error) in enumerate(refused):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
    status()
