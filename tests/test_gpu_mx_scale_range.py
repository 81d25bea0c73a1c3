"""GPU parity of the microscaled products where scales are large, small or meaningless: pairs of scales whose product passes the
largest binary32 number over sums that do not, and the scale bytes of blocks and rows that only fill up a tile, which may hold
anything but 255 (blocks) and anything (rows).  Every kernel of the products is reached: few rows, exchanged tiles, pairs of CTAs.

Bound as in test_gpu_mx.py: |y - exact| <= K 2^-23 sum_k |x w|, plus 2^-8 |y| in bfloat16."""
import numpy as np
import pytest
import torch

from oracle import mx
from tests.test_gpu_mx import BF16, F32, check_product, status
from tests.test_gpu_mx_tiles import check, draw, exact

pytestmark = pytest.mark.gpu

# rows of x, rows of w: few rows (one and several groups of eight), exchanged tiles of 64 and 128 rows, pairs of CTAs
SIZES = [(1, 8), (8, 40), (20, 77), (32, 40), (40, 130), (100, 200), (129, 40), (300, 100)]


def device(*arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def filled(scales, blocks, rows, seed):
    """The tiles of `scales` with other bytes in the places that only fill them up."""
    rng = np.random.default_rng(seed)
    n, have = scales.shape
    room = rng.integers(0, 256, (-(-n // 128) * 128, -(-have // 4) * 4)).astype(np.uint8) if rows is None else \
        np.full((-(-n // 128) * 128, -(-have // 4) * 4), rows, np.uint8)
    room[:n] = blocks
    room[:n, :have] = scales
    return mx.tile(room)


@pytest.mark.parametrize("K", [32, 96, 288, 416, 2080])
@pytest.mark.parametrize("M,N", SIZES)
def test_bytes_that_fill_up_a_tile_of_scales(M, N, K):
    import paper_2502_05003_b200 as quest
    rng = np.random.default_rng(K)
    xc, wc = rng.integers(0, 16, (M, K)).astype(np.uint8), rng.integers(0, 16, (N, K)).astype(np.uint8)
    xs, ws = rng.integers(120, 135, (M, K // 32)).astype(np.uint8), rng.integers(120, 135, (N, K // 32)).astype(np.uint8)
    xv, wv = mx.values(xc, xs, 4), mx.values(wc, ws, 4)
    xq, wq, sx, sw = device(mx.pack(xc, 4), mx.pack(wc, 4), mx.tile(xs), mx.tile(ws))
    want = quest.quest_gemm_mx(xq, sx, 4, wq, sw, K, F32)
    check_product(want, xv, wv)
    for blocks, rows in ((200, 0), (254, 254), (0, 255), (254, None)):
        fx, fw = device(filled(xs, blocks, rows, 1), filled(ws, blocks, rows, 2))
        assert torch.equal(quest.quest_gemm_mx(xq, fx, 4, wq, fw, K, F32), want)
    # a layer over weights that were laid out by the caller
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).cuda()
    y = quest.quest_linear_fwd_mx(x, None, 4, 32, F32, w_cached={"wq": wq, "sw": sw}, want_codes=False)["y"]
    assert torch.equal(quest.quest_linear_fwd_mx(x, None, 4, 32, F32, w_cached={"wq": wq, "sw": fw}, want_codes=False)["y"], y)
    status()


@pytest.mark.parametrize("M,N", SIZES)
def test_rows_that_fill_up_a_tile_beside_eight_bit_rows(M, N):
    import paper_2502_05003_b200 as quest
    rng, K = np.random.default_rng(3), 384
    xc, wc = rng.integers(0, 127, (M, K)).astype(np.uint8), rng.integers(0, 16, (N, K)).astype(np.uint8)
    xs, ws = rng.integers(120, 135, (M, K // 32)).astype(np.uint8), rng.integers(120, 135, (N, K // 32)).astype(np.uint8)
    xq, wq, sx, sw = device(xc, mx.pack(wc, 4), mx.tile(xs), mx.tile(ws))
    want = quest.quest_gemm_mx(xq, sx, 8, wq, sw, K, F32)
    check_product(want, mx.values(xc, xs, 8), mx.values(wc, ws, 4))
    for rows in (254, 255, None):
        fx, fw = device(filled(xs, 0, rows, 1), filled(ws, 0, rows, 2))
        assert torch.equal(quest.quest_gemm_mx(xq, fx, 8, wq, fw, K, F32), want)
    status()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,N", SIZES)
def test_scales_past_the_largest_number_over_sums_that_are_not(M, N, bits):
    import paper_2502_05003_b200 as quest
    rng, K = np.random.default_rng(5), 512
    one = {4: 2, 8: 0x38}[bits]                                # the code of 1.0
    for big_x, big_w in ((254, 254), (254, 130), (130, 254), (191, 191), (192, 190), (254, 128), (200, 182)):
        xc, wc = rng.integers(0, 8, (M, K)).astype(np.uint8) | one, rng.integers(0, 16, (N, K)).astype(np.uint8)
        xs, ws = np.full((M, K // 32), 127, np.uint8), np.full((N, K // 32), 127, np.uint8)
        # block 1: elements of x where w has none and the other way round; block 6: x alone; block 9: w alone
        xs[:, [1, 6, 9]], ws[:, [1, 6, 9]] = big_x, big_w
        xc[:, 32:64:2] = 0
        wc[:, 33:64:2] = 0
        wc[:, 192:224] = 0
        xc[:, 288:320] = 0
        xq, wq, sx, sw = device(mx.pack(xc, bits), mx.pack(wc, 4), mx.tile(xs), mx.tile(ws))
        # what those blocks add is 0, whatever their scales
        xv = np.delete(mx.values(xc, xs, bits).reshape(M, -1, 32), [1, 6, 9], axis=1).reshape(M, -1)
        wv = np.delete(mx.values(wc, ws, 4).reshape(N, -1, 32), [1, 6, 9], axis=1).reshape(N, -1)
        for out in (F32, BF16):
            check_product(quest.quest_gemm_mx(xq, sx, bits, wq, sw, K, out), xv, wv)
    status()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,N", SIZES)
def test_finite_sums_under_scales_whose_product_is_not(M, N, bits):
    import paper_2502_05003_b200 as quest
    rng, K, half = np.random.default_rng(6), 256, {4: 1, 8: 0x30}[bits]
    xc, wc = np.zeros((M, K), np.uint8), np.zeros((N, K), np.uint8)
    xs, ws = np.full((M, K // 32), 127, np.uint8), np.full((N, K // 32), 127, np.uint8)
    xc[:, 128:], wc[:, 128:] = rng.integers(0, 8, (M, 128)), rng.integers(0, 16, (N, 128))
    for ex, ew in ((191, 191), (254, 128), (128, 254)):
        # block 2: one product of 2^126, 0.25 under scales of 2^128 together, then two that cancel
        xs[:, 2], ws[:, 2] = ex, ew
        xc[:, 64:66], wc[:, 64], wc[:, 65] = half, 1, 0
        for _ in range(2):
            xq, wq, sx, sw = device(mx.pack(xc, bits), mx.pack(wc, 4), mx.tile(xs), mx.tile(ws))
            check_product(quest.quest_gemm_mx(xq, sx, bits, wq, sw, K, F32), mx.values(xc, xs, bits), mx.values(wc, ws, 4))
            wc[:, 65] = 9
    status()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N", SIZES)
def test_an_outlier_that_meets_zero_weights(M, N, dtype, bits):
    import paper_2502_05003_b200 as quest
    rng, K = np.random.default_rng(7), 256
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).to(dtype)
    w = torch.from_numpy(rng.standard_normal((N, K)).astype(np.float32)).to(dtype)
    x[:, 37] = 1e38
    w[:, 32:64] *= 4096.0
    w[:, 37] = 0.0
    xv = mx.values(*mx.quantize(x.float().numpy(), bits), bits)
    wv = mx.values(*mx.quantize(w.float().numpy(), 4), 4)
    for codes in (True, False):
        y = quest.quest_linear_fwd_mx(x.cuda(), w.cuda(), bits, 1, F32, want_codes=codes)["y"]
        check_product(y, xv, wv)
    status()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K8,K4", [(1, 300, 4096, 4064), (1, 7104, 1280, 1312), (8, 300, 512, 480), (8, 5504, 4096, 4064), (9, 2400, 3584, 3616), (13, 130, 2432, 2464),
                                       (24, 2368, 256, 288), (24, 3552, 1280, 1312), (32, 2368, 1024, 992), (32, 3552, 1024, 992), (100, 300, 512, 544),
                                       (300, 100, 512, 544)])
def test_large_rows_that_meet_small_weights(M, N, K8, K4, bits):
    import paper_2502_05003_b200 as quest
    K = K8 if bits == 8 else K4
    x, w = draw(M, K, M + K), draw(N, K, N)
    for block, e in {1: 66, 2: 70, 7: 90, K // 32 - 1: 110}.items():        # (twice on one block would be infinite)
        x[:, 32 * block:32 * block + 32] *= 2.0 ** e
        w[:, 32 * block:32 * block + 32] *= 2.0 ** -e
    (xc, xs), (wc, ws) = quest.quest_quantize_mx(x, bits), quest.quest_quantize_mx(w, 4)
    y = quest.quest_gemm_mx(xc, xs, bits, wc, ws, K, F32)
    check(y, *exact(quest, xc, xs, bits, wc, ws), K)
    layer = quest.quest_linear_fwd_mx(x, None, bits, 1, F32, w_cached={"wq": wc, "sw": ws}, want_codes=False)["y"]
    assert torch.equal(layer, y)
    status()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,N", SIZES)
def test_products_below_the_smallest_normal_number(M, N, bits):
    import paper_2502_05003_b200 as quest
    K, one = 128, {4: 2, 8: 0x38}[bits]
    xc, wc = np.zeros((M, K), np.uint8), np.zeros((N, K), np.uint8)
    xc[:, 0], wc[:, 0] = one, 2
    for e in (-126, -130, -140, -149):
        for ex in (e // 2, -127, 0):
            if e - ex < -127:
                continue
            xs, ws = np.full((M, 4), 127 + ex, np.uint8), np.full((N, 4), 127 + e - ex, np.uint8)
            xq, wq, sx, sw = device(mx.pack(xc, bits), mx.pack(wc, 4), mx.tile(xs), mx.tile(ws))
            assert bool((quest.quest_gemm_mx(xq, sx, bits, wq, sw, K, F32).double() == 2.0 ** e).all())
    # sums of many under scales of 2^-150 together
    rng = np.random.default_rng(9)
    xc, wc = rng.integers(1, 8 if bits == 4 else 127, (M, K)).astype(np.uint8), rng.integers(1, 8, (N, K)).astype(np.uint8)
    xs, ws = np.full((M, 4), 127 - 64, np.uint8), np.full((N, 4), 127 - 86, np.uint8)
    xq, wq, sx, sw = device(mx.pack(xc, bits), mx.pack(wc, 4), mx.tile(xs), mx.tile(ws))
    y = quest.quest_gemm_mx(xq, sx, bits, wq, sw, K, F32).cpu().double().numpy()
    want = mx.values(xc, xs, bits) @ mx.values(wc, ws, 4).T
    # no addition of K loses more than a unit in the last place of a normal number, or a step of 2^-149
    assert np.all(np.abs(y - want) <= K * 2.0 ** -23 * want + K * 2.0 ** -149)
    status()
