"""GPU parity of the norm's gradient where its kernels walk over many rows: short rows that a warp takes each, and long ones of which
every CTA takes several, against the binary64 oracle.  Bounds as in test_gpu_rmsnorm.py; what is compared per column has
as many rows' terms, added one by one inside a CTA or warp and then over at most 1024 partial sums: rows + 40 steps."""
import numpy as np
import pytest
import torch

from oracle import norm
from tests.test_gpu_rmsnorm import BF16, E, F32, HALF, U, f64, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,cols", [
    # a warp to a row: one and two chunks a lane, some lanes without one, several rows to a warp, and a last round that is part empty
    (BF16, 1024, 8), (BF16, 2100, 256), (BF16, 1025, 264), (BF16, 2100, 512), (BF16, 9001, 128), (BF16, 9001, 504),
    (F32, 1024, 8), (F32, 5000, 128), (F32, 1025, 136), (F32, 5000, 256), (F32, 9001, 72),
    # a CTA to a row, several rows to a CTA: every chunk count, whole chunks and single elements
    (BF16, 1023, 512), (BF16, 1500, 520), (BF16, 1700, 2048), (BF16, 700, 4096), (BF16, 700, 5504), (BF16, 400, 8200), (BF16, 400, 12296),
    (BF16, 400, 16384),
    (F32, 1023, 256), (F32, 1500, 264), (F32, 1700, 1024), (F32, 700, 2048), (F32, 700, 4096), (F32, 700, 5504), (F32, 400, 8192), (F32, 400, 16384),
    (BF16, 900, 1023), (BF16, 700, 4095), (BF16, 400, 8191), (BF16, 400, 16383),
    (F32, 900, 1023), (F32, 700, 4095), (F32, 400, 8191), (F32, 400, 16383)])
def test_gradient(dtype, rows, cols):
    import paper_2502_05003_b200 as quest
    h, w = tensor((rows, cols), 8, dtype, 2.0), 1 + tensor((cols,), 9, dtype, 0.2)
    dy, dres = tensor((rows, cols), 10, dtype), tensor((rows, cols), 11, dtype)
    rstd = quest.quest_rmsnorm_fwd(h.cuda(), w.cuda(), 1e-5)["rstd"]
    s, n = f64(rstd), f64(h) * f64(rstd)[:, None]
    g = f64(dy) * f64(w)
    for res in (None, dres):
        d = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd, None if res is None else res.cuda())
        dx, dw = norm.backward(f64(dy), f64(h), f64(w), s, None if res is None else f64(res))
        lim = s[:, None] * (6 * U * np.abs(g) + (E + 6 * U) * np.abs(n) * np.abs(g * n).mean(1, keepdims=True)) + HALF[dtype] * np.abs(dx)
        if res is not None:
            lim = lim + 2 * U * np.abs(f64(res))
        assert np.all(np.abs(f64(d["dx"]) - dx) <= lim + 1e-37)
        assert np.all(np.abs(f64(d["dw"]) - dw) <= (rows + 40) * U * np.abs(f64(dy) * n).sum(0) + 1e-37)
        again = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd, None if res is None else res.cuda())
        assert torch.equal(again["dx"], d["dx"]) and torch.equal(again["dw"], d["dw"])
    only = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd, dres.cuda(), want_dw=False)
    assert only["dw"] is None and torch.equal(only["dx"], d["dx"])
    only = quest.quest_rmsnorm_bwd(dy.cuda(), h.cuda(), w.cuda(), rstd, want_dx=False)
    assert only["dx"] is None and torch.equal(only["dw"], d["dw"])
