"""Host-side argument checks of the microscaled layer and of the norm: the documented status codes, before anything is launched."""
import ctypes

import pytest

FAKE, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)       # never dereferenced: every case fails a check first
F = ctypes.c_float
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_2502_05003_b200 import build, _lib
    build.build()
    return _lib.load()


def test_sizes(lib):
    assert lib.quest_mx_scales_bytes(1, 32) == 512 and lib.quest_mx_scales_bytes(128, 128) == 512
    assert lib.quest_mx_scales_bytes(129, 160) == 4 * 512 and lib.quest_mx_scales_bytes(0, 32) == 0
    for rows, cols in ((-1, 32), (1, 0), (1, 33), (1, 16416), ((1 << 24) + 1, 32)):
        assert lib.quest_mx_scales_bytes(rows, cols) == 0
    assert lib.quest_bwd_mx_workspace_bytes(8, 8, 64) > lib.quest_bwd_workspace_bytes(8, 8, 64) > 0
    assert lib.quest_bwd_mx_workspace_bytes(7, 8, 64) == 0
    assert lib.quest_rmsnorm_bwd_workspace_bytes(3, 10) >= 120 and lib.quest_rmsnorm_bwd_workspace_bytes(0, 10) >= 40
    assert lib.quest_rmsnorm_bwd_workspace_bytes(1, 16385) == 0 and lib.quest_rmsnorm_bwd_workspace_bytes(1, 0) == 0
    assert b"eps" in lib.quest_status_string(14)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(dtype=2), 5), (dict(bits=5), 3), (dict(bits=0), 3),
    (dict(cols=48), 2), (dict(cols=0), 2), (dict(cols=16416), 2), (dict(rows=-1), 2), (dict(rows=1 << 25), 2), (dict(ld=96), 2),
    (dict(g=2), 4), (dict(g=0), 4), (dict(x=ODD), 6), (dict(ld=129), 6), (dict(codes=ODD), 6), (dict(rows=0), 0)])
def test_quantize(lib, change, status):
    a = dict(x=FAKE, dtype=1, rows=4, cols=128, ld=128, bits=4, g=32, codes=FAKE, scales=FAKE) | change
    assert lib.quest_quantize_mx(a["x"], a["dtype"], a["rows"], a["cols"], a["ld"], a["bits"], a["g"], a["codes"], a["scales"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(out=None), 1), (dict(dtype=3), 5), (dict(bits=3), 3), (dict(cols=40), 2),
    (dict(rows=-2), 2), (dict(codes=ODD), 6), (dict(out=ODD), 6), (dict(rows=0), 0)])
def test_dequantize(lib, change, status):
    a = dict(codes=FAKE, scales=FAKE, rows=4, cols=128, bits=8, out=FAKE, dtype=0) | change
    assert lib.quest_dequantize_mx(a["codes"], a["scales"], a["rows"], a["cols"], a["bits"], a["out"], a["dtype"], None) == status


PRODUCT = [(dict(bits=6), 3), (dict(M=-1), 2), (dict(N=1 << 25), 2), (dict(K=40), 2), (dict(K=160), 2), (dict(K=0), 2), (dict(ydt=2), 5),
           (dict(wq=None), 1), (dict(sw=None), 1), (dict(y=None), 1), (dict(ldy=63), 2), (dict(wq=ctypes.c_void_p(0x10010)), 6),
           (dict(sw=ODD), 6), (dict(y=ctypes.c_void_p(0x10002)), 6), (dict(M=0), 0), (dict(N=0), 0), (dict(M=0, K=160), 2)]


@pytest.mark.parametrize("change,status", PRODUCT + [(dict(xq=None), 1), (dict(sx=None), 1), (dict(xq=ODD), 6), (dict(sx=ODD), 6)])
def test_gemm(lib, change, status):
    a = dict(xq=FAKE, sx=FAKE, bits=8, wq=FAKE, sw=FAKE, M=40, N=64, K=128, y=FAKE, ydt=0, ldy=64) | change
    assert lib.quest_gemm_mx(a["xq"], a["sx"], a["bits"], a["wq"], a["sw"], a["M"], a["N"], a["K"], a["y"], a["ydt"], a["ldy"], None) == status


@pytest.mark.parametrize("change,status", PRODUCT + [
    (dict(x=None), 1), (dict(w=None), 1), (dict(xdt=4), 5), (dict(wdt=4), 5), (dict(g=16), 4), (dict(cached=2), 2), (dict(ldx=64), 2),
    (dict(ldw=64), 2), (dict(x=ODD), 6), (dict(w=ODD), 6), (dict(xq=None), 1), (dict(sx=None), 1), (dict(xq=None, sx=None), 1),
    (dict(xq=None, M=4), 1), (dict(xq=ODD), 6)])
def test_linear(lib, change, status):
    a = dict(x=FAKE, xdt=1, ldx=128, w=FAKE, wdt=1, ldw=128, xq=FAKE, sx=FAKE, bits=8, g=32, wq=FAKE, sw=FAKE, M=40, N=64, K=128, y=FAKE,
             ydt=0, ldy=64, cached=0) | change
    if a["K"] == 160:
        a["ldx"] = a["ldw"] = 160
    if a["M"] == 0 or a["N"] == 0:
        a |= dict(cached=1, xq=None, sx=None)              # nothing to quantize either
    assert lib.quest_linear_fwd_mx(a["x"], a["xdt"], a["ldx"], a["w"], a["wdt"], a["ldw"], a["M"], a["N"], a["K"], a["bits"], a["g"], a["y"],
                                   a["ydt"], a["ldy"], a["xq"], a["sx"], a["wq"], a["sw"], a["cached"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(dy=None), 1), (dict(xq=None), 1), (dict(sw=None), 1), (dict(dx=None, dw=None), 1), (dict(bits=1), 3), (dict(M=12), 2), (dict(N=0), 2),
    (dict(K=48), 2), (dict(g=4), 4), (dict(odt=5), 5), (dict(dy=ODD), 6), (dict(xq=ODD), 6), (dict(wq=ODD), 6), (dict(dx=ODD), 6), (dict(dw=ODD), 6),
    (dict(ws=None), 8), (dict(ws=ODD), 8), (dict(n=1000), 8)])
def test_backward(lib, change, status):
    a = dict(dy=FAKE, M=16, N=8, K=128, bits=8, g=1, xq=FAKE, sx=FAKE, wq=FAKE, sw=FAKE, dx=FAKE, dw=FAKE, odt=0, ws=FAKE, n=1 << 24) | change
    assert lib.quest_linear_bwd_mx(a["dy"], a["M"], a["N"], a["K"], a["bits"], a["g"], a["xq"], a["sx"], a["wq"], a["sw"], a["dx"], a["dw"],
                                   a["odt"], a["ws"], a["n"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(x=None), 1), (dict(w=None), 1), (dict(h=None), 1), (dict(y=None), 1), (dict(bits=8, yq=None), 1), (dict(bits=4, sy=None), 1), (dict(dt=2), 5),
    (dict(wdt=-1), 5), (dict(ydt=9), 5), (dict(bits=2), 3), (dict(rows=-1), 2), (dict(cols=0), 2), (dict(cols=16385, ldx=16385, ldr=16385), 2),
    (dict(ldx=100), 2), (dict(ldr=100), 2), (dict(bits=8, cols=40), 2), (dict(bits=8, g=8), 4), (dict(eps=-1.0), 14), (dict(eps=NAN), 14),
    (dict(eps=INF), 14), (dict(x=ctypes.c_void_p(0x10001)), 6), (dict(rstd=ctypes.c_void_p(0x10002)), 6), (dict(bits=8, x=ODD), 6),
    (dict(bits=8, yq=ODD), 6), (dict(bits=4, h=ODD), 6), (dict(bits=4, ldx=129), 6), (dict(rows=0), 0)])
def test_norm(lib, change, status):
    a = dict(x=FAKE, r=FAKE, dt=1, ldx=128, ldr=128, w=FAKE, wdt=1, rows=4, cols=128, eps=1e-5, h=FAKE, rstd=FAKE, y=FAKE, ydt=1, bits=0, g=1,
             yq=FAKE, sy=FAKE) | change
    assert lib.quest_rmsnorm_fwd(a["x"], a["r"], a["dt"], a["ldx"], a["ldr"], a["w"], a["wdt"], a["rows"], a["cols"], F(a["eps"]), a["h"], a["rstd"],
                                 a["y"], a["ydt"], a["bits"], a["g"], a["yq"], a["sy"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(dy=None), 1), (dict(h=None), 1), (dict(w=None), 1), (dict(rstd=None), 1), (dict(dx=None, dw=None), 1), (dict(dt=2), 5), (dict(wdt=2), 5),
    (dict(rows=-1), 2), (dict(cols=0), 2), (dict(lddy=7), 2), (dict(ldh=7), 2), (dict(lddr=7), 2), (dict(dy=ctypes.c_void_p(0x10001)), 6),
    (dict(dx=ctypes.c_void_p(0x10001)), 6), (dict(dw=ctypes.c_void_p(0x10002)), 6), (dict(ws=None), 8), (dict(ws=ODD), 8), (dict(n=10), 8)])
def test_norm_backward(lib, change, status):
    a = dict(dy=FAKE, h=FAKE, r=FAKE, dt=1, lddy=8, ldh=8, lddr=8, w=FAKE, wdt=1, rstd=FAKE, rows=4, cols=8, dx=FAKE, dw=FAKE, ws=FAKE, n=1 << 20) | change
    assert lib.quest_rmsnorm_bwd(a["dy"], a["h"], a["r"], a["dt"], a["lddy"], a["ldh"], a["lddr"], a["w"], a["wdt"], a["rstd"], a["rows"], a["cols"],
                                 a["dx"], a["dw"], a["ws"], a["n"], None) == status
