"""GPU parity: RMS norm with the residual's addition, its MX output and its gradient, against the binary64 oracle.

h is exact (one binary32 sum, one rounding).  rstd: a row's squares are added in at most D = 100 steps on any path of the sum (up to 64
in a thread, 13 between threads, the products' roundings beside them), all positive, so the sum is within D 2^-24, rstd within half of
that and four roundings of its own: R = 54 x 2^-24.  y: two more roundings, and half a step of its type.  Gradients: with
n and g within (R and) two roundings, mean(g n) is within E = (D + 8) 2^-24 of mean|g n|; dx = dres + rstd (g - n mean) adds
four roundings of its terms' magnitudes.  The rstd that the gradient takes is given, so R does not enter.  dw: rows are added one
by one inside a CTA, then its partial sums: at most rows + 40 steps."""
import numpy as np
import pytest
import torch

from oracle import mx, norm

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
R, E = 54 * U, 108 * U
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def tensor(shape, seed, dtype, scale=1.0):
    return (torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)) * scale).to(dtype)


def f64(t):
    return t.cpu().double().numpy()


def check_forward(r, x, residual, weight, eps, out):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    if residual is None:
        assert r["h"] is None
    else:
        assert torch.equal(r["h"].cpu(), h)
    rstd, y = norm.forward(f64(h), f64(weight), eps)
    assert np.all(np.abs(f64(r["rstd"]) - rstd) <= R * rstd)
    if out is not None:
        assert r["y"].dtype == out
        assert np.all(np.abs(f64(r["y"]) - y) <= (R + 2 * U + HALF[out]) * np.abs(y) + 1e-38)
    return y


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (5, 100), (2, 1025), (7, 2048), (3, 4097), (4, 5504), (2, 8192), (1, 16384),
                                       (3, 16383), (2100, 64), (2049, 520), (2050, 1032), (2048, 2048), (2047, 2056)])
def test_forward(rows, cols, dtype):
    import paper_2502_05003_b200 as quest
    x, res, w = tensor((rows, cols), 1, dtype, 3.0), tensor((rows, cols), 2, dtype), 1 + tensor((cols,), 3, dtype, 0.2)
    for residual in (None, res):
        for out in (BF16, F32):
            r = quest.quest_rmsnorm_fwd(x.cuda(), w.cuda(), 1e-5, None if residual is None else residual.cuda(), out_dtype=out)
            check_forward(r, x, residual, w, 1e-5, out)
    other = F32 if dtype == BF16 else BF16                     # a weight of another type
    r = quest.quest_rmsnorm_fwd(x.cuda(), w.to(other).cuda(), 0.5)
    check_forward(r, x, None, w.to(other), 0.5, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("g", [1, 32])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 96), (1, 2048), (130, 160), (5, 4096), (3, 5504), (2, 16384), (2100, 256), (2050, 1024), (2049, 2048)])
def test_mx_output_is_that_of_the_quantizer(rows, cols, g, bits, dtype):
    import paper_2502_05003_b200 as quest
    x, res, w = tensor((rows, cols), 4, dtype), tensor((rows, cols), 5, dtype), 1 + tensor((cols,), 6, dtype, 0.2)
    r = quest.quest_rmsnorm_fwd(x.cuda(), w.cuda(), 1e-5, res.cuda(), mx_bits=bits, had_block=g)
    y = check_forward(r, x, res, w, 1e-5, None)
    assert "y" not in r and r["yq"].shape == (rows, cols * bits // 8)
    # the binary32 rows that were rounded, from their definition: (h rstd) w, each product rounded
    rounded = (r["h"].float() * r["rstd"][:, None]) * w.cuda().float()
    codes, scales = quest.quest_quantize_mx(rounded, bits, g)
    assert torch.equal(r["yq"], codes) and torch.equal(r["sy"], scales)
    # and from the oracle: within half a step of its block's scale
    v = f64(quest.quest_dequantize_mx(r["yq"], r["sy"], bits, F32))
    turned = mx.inverse(y, g)
    block = np.abs(turned).reshape(rows, -1, 32).max(2).repeat(32, axis=1)
    # over the block's largest element, which lies in [4, 8) or [256, 512) steps of the scale: half a step is at most 1 of 4 or
    # 16 of 256, but what saturates is off by up to 8 - 6 of 8 or 512 - 448 of 512
    step = 2.0 ** -2 if bits == 4 else 2.0 ** -3
    assert np.all(np.abs(v - turned) <= (step + 64 * U) * block + 1e-37)


def test_rows_of_zeros_infinities_and_nan():
    import paper_2502_05003_b200 as quest
    for cols in (256, 101):
        x = tensor((6, cols), 7, F32)
        x[1], x[2, 5], x[3, 9], x[4] = 0.0, float("inf"), float("nan"), 1e30
        w = torch.ones(cols)
        r = quest.quest_rmsnorm_fwd(x.cuda(), w.cuda(), 1e-5)
        y = r["y"].cpu()
        clean = quest.quest_rmsnorm_fwd(x[[0, 5]].cuda(), w.cuda(), 1e-5)["y"].cpu()
        assert torch.equal(y[[0, 5]], clean)
        assert not bool(y[1].any()) and bool(y[2, 5].isnan()) and bool(y[3].isnan().all())
        assert not bool(y[4].any())                        # the squares overflow binary32: rstd is 0
        if cols % 32 == 0:
            m = quest.quest_rmsnorm_fwd(x.cuda(), w.cuda(), 1e-5, mx_bits=8)
            v = quest.quest_dequantize_mx(m["yq"], m["sy"], 8, F32).cpu()
            assert not bool(v[1].any()) and bool(v[3].isnan().all()) and bool(v[[0, 5]].isfinite().all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (5, 100), (2, 1025), (700, 2048), (3, 4097), (40, 5504), (2, 8192), (9, 16384), (3, 16383),
                                       (1300, 63), (777, 520)])
def test_gradient(rows, cols, dtype):
    import paper_2502_05003_b200 as quest
    h, w = tensor((rows, cols), 8, dtype, 2.0), 1 + tensor((cols,), 9, dtype, 0.2)
    dy, dres = tensor((rows, cols), 10, dtype), tensor((rows, cols), 11, dtype)
    rstd = quest.quest_rmsnorm_fwd(h.cuda(), w.cuda(), 1e-5)["rstd"]
    for res in (None, dres):
        d = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd, None if res is None else res.cuda())
        s = f64(rstd)
        dx, dw = norm.backward(f64(dy), f64(h), f64(w), s, None if res is None else f64(res))
        n, g = f64(h) * s[:, None], f64(dy) * f64(w)
        lim = s[:, None] * (6 * U * np.abs(g) + (E + 6 * U) * np.abs(n) * np.abs(g * n).mean(1, keepdims=True)) + HALF[dtype] * np.abs(dx)
        if res is not None:
            lim = lim + 2 * U * np.abs(f64(res))
        assert np.all(np.abs(f64(d["dx"]) - dx) <= lim + 1e-37)
        assert d["dw"].dtype == F32
        assert np.all(np.abs(f64(d["dw"]) - dw) <= (rows + 40) * U * np.abs(f64(dy) * n).sum(0) + 1e-37)
        again = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd, None if res is None else res.cuda())
        assert torch.equal(again["dx"], d["dx"]) and torch.equal(again["dw"], d["dw"])
    only = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd, dres.cuda(), want_dw=False)
    assert only["dw"] is None and torch.equal(only["dx"], d["dx"])
    only = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd, want_dx=False)
    assert only["dx"] is None and torch.equal(only["dw"], d["dw"])


def test_gradient_against_differences_of_the_forward_call():
    import paper_2502_05003_b200 as quest
    # binary32 forward calls at h +- e along a direction: their difference carries 2 x 2^-24-sized roundings of y over 2 e
    h, w, dy = tensor((4, 96), 12, F32), 1 + tensor((96,), 13, F32, 0.2), tensor((4, 96), 14, F32)
    step, e = tensor((4, 96), 15, F32), 2.0 ** -7
    rstd = quest.quest_rmsnorm_fwd(h.cuda(), w.cuda(), 1e-5)["rstd"]
    d = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd)
    up, down = (f64(quest.quest_rmsnorm_fwd((h + s * e * step).cuda(), w.cuda(), 1e-5)["y"]) for s in (1, -1))
    difference = np.sum(f64(dy) * (up - down)) / (2 * e)
    curve = 30 * e ** 2 * np.sum(np.abs(f64(dy) * f64(w)))     # third derivatives of unit-size rows along unit-size steps
    noise = np.sum(np.abs(f64(dy)) * (np.abs(up) + np.abs(down))) * (R + 4 * U) / (2 * e)
    assert abs(difference - np.sum(f64(d["dx"]) * f64(step))) <= curve + noise


def test_strided_and_misaligned_rows():
    import paper_2502_05003_b200 as quest
    x, res, w = tensor((9, 256), 16, BF16), tensor((9, 256), 17, BF16), 1 + tensor((256,), 18, BF16, 0.2)
    r = quest.quest_rmsnorm_fwd(x.cuda(), w.cuda(), 1e-5, res.cuda())
    d = quest.quest_rmsnorm_bwd(res.cuda(), x.cuda(), w.cuda(), r["rstd"], x.cuda())
    for pitch, at in ((264, 8), (257, 1), (300, 2)):
        def put(t):
            room = torch.full((9, pitch), 5.0, dtype=BF16, device="cuda")
            room[:, at:at + 256] = t.cuda()
            return room[:, at:at + 256] if at + 256 <= pitch else None
        s = quest.quest_rmsnorm_fwd(put(x), w.cuda(), 1e-5, put(res))
        assert torch.equal(s["h"], r["h"])
        check_forward(s, x, res, w, 1e-5, BF16)
        e = quest.quest_rmsnorm_bwd(put(res), put(x), w.cuda(), r["rstd"], put(x))
        assert torch.allclose(e["dx"].float(), d["dx"].float(), rtol=2 ** -7, atol=1e-6) and torch.allclose(e["dw"], d["dw"], rtol=1e-5, atol=1e-5)
    odd = torch.zeros(257, dtype=BF16, device="cuda")
    odd[1:] = w.cuda()
    check_forward(quest.quest_rmsnorm_fwd(x.cuda(), odd[1:], 1e-5, res.cuda()), x, res, w, 1e-5, BF16)


def test_kept_buffers_empty_calls_other_streams_and_graphs():
    import paper_2502_05003_b200 as quest
    x, res, w = tensor((30, 512), 19, BF16).cuda(), tensor((30, 512), 20, BF16).cuda(), (1 + tensor((512,), 21, BF16, 0.2)).cuda()
    out = {k: torch.full(s, 3.0, dtype=d, device="cuda") for k, s, d in (("h", (31, 512), BF16), ("rstd", (31,), F32), ("y", (31, 512), BF16))}
    want = quest.quest_rmsnorm_fwd(x, w, 1e-5, res)
    r = quest.quest_rmsnorm_fwd(x, w, 1e-5, res, out=out)
    for k in ("h", "rstd", "y"):
        assert r[k] is out[k] and torch.equal(out[k][:30], want[k]) and bool((out[k][30:] == 3.0).all())
    e = quest.quest_rmsnorm_fwd(x[:0], w, 1e-5)
    assert e["y"].shape == (0, 512) and e["h"] is None
    d = quest.quest_rmsnorm_bwd(x[:0], x[:0], w, want["rstd"])
    assert d["dx"].shape == (0, 512) and not bool(d["dw"].any())
    grads = quest.quest_rmsnorm_bwd(res, want["h"], w, want["rstd"], x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s = quest.quest_rmsnorm_fwd(x, w, 1e-5, res)
    side.synchronize()
    assert torch.equal(s["y"], want["y"])
    graph, static = torch.cuda.CUDAGraph(), x.clone()
    with torch.cuda.graph(graph):
        f = quest.quest_rmsnorm_fwd(static, w, 1e-5, res)
        b = quest.quest_rmsnorm_bwd(res, f["h"], w, f["rstd"], x)
    for _ in range(2):
        static.zero_()
        graph.replay()
        static.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(f["y"], want["y"]) and torch.equal(b["dx"], grads["dx"]) and torch.equal(b["dw"], grads["dw"])


def test_norm_layer_and_gradients_together():
    import paper_2502_05003_b200 as quest
    # one step of a block's half: stream + norm -> layer; back through both.  The norm's codes are the layer's activations.
    T, H, N = 136, 256, 192
    x, res, w = tensor((T, H), 22, BF16).cuda(), tensor((T, H), 23, BF16).cuda(), (1 + tensor((H,), 24, BF16, 0.2)).cuda()
    weights, dy = tensor((N, H), 25, BF16, 0.1).cuda(), tensor((T, N), 26, BF16).cuda()
    wq, sw = quest.quest_quantize_mx(weights, 4, 32)
    r = quest.quest_rmsnorm_fwd(x, w, 1e-5, res, mx_bits=8, had_block=32)
    y = quest.quest_gemm_mx(r["yq"], r["sy"], 8, wq, sw, H)
    plain = quest.quest_rmsnorm_fwd(x, w, 1e-5, res, out_dtype=F32)
    layer = quest.quest_linear_fwd_mx(plain["y"], None, 8, 32, BF16, w_cached={"wq": wq, "sw": sw})
    assert torch.equal(layer["xq"], r["yq"]) and torch.equal(layer["sx"], r["sy"]) and torch.equal(layer["y"], y)
    d = quest.quest_linear_bwd_mx(dy, {"xq": r["yq"], "sx": r["sy"], "wq": wq, "sw": sw}, 8, 32, H, BF16)
    b = quest.quest_rmsnorm_bwd(d["dx"], r["h"], w, r["rstd"], x)
    dx, dw = norm.backward(f64(d["dx"]), f64(r["h"]), f64(w), f64(r["rstd"]), f64(x))
    assert np.linalg.norm(f64(b["dx"]) - dx) <= 2.0 ** -8 * np.linalg.norm(dx)
    assert np.linalg.norm(f64(b["dw"]) - dw) <= 1e-5 * np.linalg.norm(dw)
    # and the norm in front of the layers that the framework had: the same rows, quantized by their own calls
    own = quest.quest_linear_fwd(plain["y"].to(BF16), weights, 4, 128)
    rel = (own["y"].float() - y.float()).norm() / y.float().norm()
    assert float(rel) < 0.5                                 # two 4-bit roundings of the same product
    # few rows: a decoding step
    few = quest.quest_rmsnorm_fwd(x[:3], w, 1e-5, res[:3], mx_bits=8, had_block=32)
    assert torch.equal(few["yq"], r["yq"][:3])
    assert quest.quest_gemm_mx(few["yq"], few["sy"], 8, wq, sw, H).shape == (3, N)


def test_refusals():
    import paper_2502_05003_b200 as quest
    x, w = tensor((4, 256), 27, BF16).cuda(), torch.ones(256, dtype=BF16, device="cuda")
    rstd = torch.ones(4, device="cuda")
    refused = [
        (lambda: quest.quest_rmsnorm_fwd(x, w[:255]), ValueError), (lambda: quest.quest_rmsnorm_fwd(x, w.half()), TypeError),
        (lambda: quest.quest_rmsnorm_fwd(x.half(), w), TypeError), (lambda: quest.quest_rmsnorm_fwd(x.cpu(), w), ValueError),
        (lambda: quest.quest_rmsnorm_fwd(x, w, -1.0), quest.QuestError), (lambda: quest.quest_rmsnorm_fwd(x, w, float("nan")), quest.QuestError),
        (lambda: quest.quest_rmsnorm_fwd(x, w, float("inf")), quest.QuestError), (lambda: quest.quest_rmsnorm_fwd(x[0], w), ValueError),
        (lambda: quest.quest_rmsnorm_fwd(x[:, ::2], w[:128]), ValueError), (lambda: quest.quest_rmsnorm_fwd(x, w, residual=x[:3]), ValueError),
        (lambda: quest.quest_rmsnorm_fwd(x, w, residual=x.float()), TypeError), (lambda: quest.quest_rmsnorm_fwd(x, w, mx_bits=5), ValueError),
        (lambda: quest.quest_rmsnorm_fwd(x, w, mx_bits=8, had_block=3), quest.QuestError),
        (lambda: quest.quest_rmsnorm_fwd(x[:, :40], w[:40], mx_bits=8), quest.QuestError),
        (lambda: quest.quest_rmsnorm_fwd(x[:, 1:33], w[:32], mx_bits=8), quest.QuestError),
        (lambda: quest.quest_rmsnorm_fwd(x, w, out_dtype=torch.float16), TypeError),
        (lambda: quest.quest_rmsnorm_fwd(x, w, out={"y": torch.empty((3, 256), dtype=BF16, device="cuda")}), ValueError),
        (lambda: quest.quest_rmsnorm_fwd(torch.empty((1, 16400), dtype=BF16, device="cuda"), torch.empty(16400, dtype=BF16, device="cuda")), quest.QuestError),
        (lambda: quest.quest_rmsnorm_bwd(x, x.float(), w, rstd), TypeError), (lambda: quest.quest_rmsnorm_bwd(x, x[:3], w, rstd), ValueError),
        (lambda: quest.quest_rmsnorm_bwd(x, x, w, rstd[:3]), ValueError), (lambda: quest.quest_rmsnorm_bwd(x, x, w, rstd.double()), ValueError),
        (lambda: quest.quest_rmsnorm_bwd(x, x, w, rstd, x[:2]), ValueError),
        (lambda: quest.quest_rmsnorm_bwd(x, x, w, rstd, want_dx=False, want_dw=False), quest.QuestError),
        (lambda: quest.quest_rmsnorm_bwd(x, x, w, rstd, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), quest.QuestError),
    ]
    for i, (call, error) in enumerate(refused):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
