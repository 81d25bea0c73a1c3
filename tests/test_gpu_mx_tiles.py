"""GPU parity of the microscaled products over the tilings they are computed in, against the oracle: sides of the tensor cores'
tiles exchanged with 32, 64 and 128 rows of x, K in one, two, four and eight parts, several tiles of x, and pairs of CTAs with tiles of 128
and 256 columns.

A product sums K exact products in binary32, in an order and with an alignment of addends that the hardware chooses, and up to
eight parts after that: each addition loses at most one unit in the last place of a running sum of at most
B = sum_k |x w|, so |y - exact| <= (K + 8) 2^-23 B, plus 2^-8 |y| (half a step) in bfloat16."""
import numpy as np
import pytest
import torch

from oracle import mx

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

# rows of x, rows of w, K for 8 and 4 bits; what is taken on 148 SMs
FEW_TO_128 = [
    (1, 1, 8192, 16384),          # 32 rows, eight parts
    (32, 300, 4096, 8192),
    (7, 129, 8320, 8224),         # K that ends inside the last part
    (31, 2100, 2048, 4096),       # four parts
    (20, 5504, 2048, 4128),
    (17, 9600, 2688, 5152),       # two parts
    (12, 4737, 256, 288),         # one
    (3, 7105, 128, 32),
    (33, 77, 2048, 4128),         # 64 rows, four parts
    (64, 5000, 3200, 6400),       # two
    (49, 1000, 384, 416),         # one
    (65, 257, 2176, 4224),        # 128 rows, four parts
    (128, 8300, 3328, 6176),      # two
    (100, 19100, 128, 64),        # one, and more tiles than SMs
    (129, 128, 2048, 4128),       # two tiles of x and more
    (300, 515, 3200, 6176),
    (777, 1100, 128, 96),
]
PAIRS = [(129, 40, 384, 416), (300, 127, 2048, 4128), (600, 4100, 640, 160), (1300, 2300, 1152, 416), (1281, 2305, 128, 32)]


def draw(n, k, seed, spread=2.0):
    rng = np.random.default_rng(seed)
    a = rng.standard_normal((n, k)) * np.exp(rng.uniform(-spread, spread, (n, k // 32))).repeat(32, axis=1)
    return torch.from_numpy(a.astype(np.float32)).to(BF16).cuda()


def exact(quest, xc, xs, bits, wc, ws):
    # (that read-back is exact is tested beside the oracle)
    xv, wv = quest.quest_dequantize_mx(xc, xs, bits, F32).double(), quest.quest_dequantize_mx(wc, ws, 4, F32).double()
    return xv @ wv.T, xv.abs() @ wv.abs().T


def check(y, want, size, K):
    lim = (K + 8) * 2.0 ** -23 * size + (2.0 ** -8 * want.abs() if y.dtype == BF16 else 0.0)
    err = (y.double() - want).abs()
    assert bool((err <= lim + 1e-37).all()), f"worst element at {(err / (lim + 1e-37)).max().item():.3f} of the bound"


def status():
    import paper_2502_05003_b200 as quest
    torch.cuda.synchronize()
    assert quest.quest_device_status() == 0


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K8,K4", FEW_TO_128 + PAIRS)
def test_products(M, N, K8, K4, bits):
    import paper_2502_05003_b200 as quest
    K = K8 if bits == 8 else K4
    xc, xs = quest.quest_quantize_mx(draw(M, K, M), bits)
    wc, ws = quest.quest_quantize_mx(draw(N, K, N), 4)
    want, size = exact(quest, xc, xs, bits, wc, ws)
    for out, pad, skip in ((F32, 0, 0), (BF16, 0, 0), (F32, 5, 1), (BF16, 3, 1), (BF16, 8, 8)):
        # a row before and behind, columns on both sides: none is touched
        room = torch.full((M + 2, skip + N + pad), 7.0, dtype=out, device="cuda")
        y = room[1:M + 1, skip:skip + N]
        assert quest.quest_gemm_mx(xc, xs, bits, wc, ws, K, y=y) is y
        check(y, want, size, K)
        first = y.clone()
        y.fill_(7.0)
        assert bool((room == 7.0).all())
        quest.quest_gemm_mx(xc, xs, bits, wc, ws, K, y=y)
        assert torch.equal(y, first)                            # the same sums in the same order
    status()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K8,K4", [c for c in FEW_TO_128 + PAIRS if c[1] <= 2305 and c[0] > 1])
def test_the_layer_takes_the_same_product(M, N, K8, K4, bits):
    import paper_2502_05003_b200 as quest
    K = K8 if bits == 8 else K4
    x, w = draw(M, K, M), draw(N, K, N)
    r = quest.quest_linear_fwd_mx(x, w, bits, 32, F32)
    wide = torch.zeros((M, K + 16), dtype=BF16, device="cuda")
    wide[:, 8:8 + K] = x
    for other in (quest.quest_linear_fwd_mx(x, None, bits, 32, F32, w_cached=r, want_codes=False),
                  quest.quest_linear_fwd_mx(wide[:, 8:8 + K], w, bits, 32, F32)):
        assert torch.equal(other["y"], r["y"])
    assert torch.equal(quest.quest_gemm_mx(r["xq"], r["sx"], bits, r["wq"], r["sw"], K, F32), r["y"])
    want, size = exact(quest, r["xq"], r["sx"], bits, r["wq"], r["sw"])
    check(r["y"], want, size, K)
    status()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", [(9, 200, 8192), (30, 70, 4096), (40, 300, 4096), (120, 70, 4096), (120, 300, 512), (200, 200, 4096), (200, 70, 512)])
def test_blocks_that_are_not_finite_reach_their_rows_only(M, N, K, bits):
    import paper_2502_05003_b200 as quest
    x, w = draw(M, K, 1), draw(N, K, 2)
    clean = quest.quest_linear_fwd_mx(x, w, bits, 1, F32)["y"]
    x[1, 100], x[M - 1, K - 1], w[7, 300], w[N - 1, K - 1] = float("nan"), float("-inf"), float("inf"), float("nan")
    y = quest.quest_linear_fwd_mx(x, w, bits, 1, F32)["y"]
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[1], bad[M - 1], bad[:, 7], bad[:, N - 1] = True, True, True, True
    assert bool(y[bad].isnan().all()) and torch.equal(y[~bad], clean[~bad])
    status()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N", [(20, 200), (60, 200), (110, 200), (200, 200), (200, 40)])
def test_every_scale(M, N, bits):
    import paper_2502_05003_b200 as quest
    # scales that meet at 2^-8 .. 2^8 together, from both ends of their range; K in parts but for the last
    K, rng = 8192, np.random.default_rng(27)
    for sw in (0, 1, 60, 127, 200, 254):
        xc = rng.integers(0, 16 if bits == 4 else 256, (M, K)).astype(np.uint8)
        xc[(xc & 127) == 127] = 0                              # E4M3 has two codes for NaN
        wc, ws = rng.integers(0, 16, (N, K)).astype(np.uint8), np.full((N, K // 32), sw, np.uint8)
        xs = np.clip(254 - sw + rng.integers(-8, 9, (M, K // 32)), 0, 254).astype(np.uint8)
        t = [torch.from_numpy(a).cuda() for a in (mx.pack(xc, bits), mx.tile(xs), mx.pack(wc, 4), mx.tile(ws))]
        y = quest.quest_gemm_mx(t[0], t[1], bits, t[2], t[3], K, F32)
        xv, wv = torch.from_numpy(mx.values(xc, xs, bits)).cuda().double(), torch.from_numpy(mx.values(wc, ws, 4)).cuda().double()
        check(y, xv @ wv.T, xv.abs() @ wv.abs().T, K)
    status()


def test_two_streams_and_a_captured_graph():
    import paper_2502_05003_b200 as quest
    calls = [(24, 300, 8192, 8), (24, 5504, 2048, 8), (100, 300, 4096, 4), (200, 200, 4096, 8), (200, 40, 512, 4)]
    data = []
    for i, (M, N, K, bits) in enumerate(calls):
        wc, ws = quest.quest_quantize_mx(draw(N, K, 50 + i), 4)
        data.append((draw(M, K, i), wc, ws, bits))
    run = lambda: [quest.quest_linear_fwd_mx(x, None, bits, 32, F32, w_cached={"wq": wc, "sw": ws})["y"] for x, wc, ws, bits in data]
    want = run()
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for s in side:
            with torch.cuda.stream(s):
                got.append(run())
    torch.cuda.synchronize()
    for ys in got:
        for a, b in zip(ys, want):
            assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ys = run()
    keep = [x.clone() for x, *_ in data]
    for _ in range(3):
        for x, *_ in data:
            x.zero_()
        graph.replay()
        assert all(not bool(y.any()) for y in ys)
        for (x, *_), k in zip(data, keep):
            x.copy_(k)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(ys, want):
            assert torch.equal(a, b)
    status()
