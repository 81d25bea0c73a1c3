"""GPU: the norm and its gradient with outputs in the place of inputs give the bits that they give beside them, also in a chain of
layers, where each launch starts while the one before it still writes what it will read."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SHAPES = [(1, 8), (3, 7), (5, 4097), (7, 2048), (300, 512), (2100, 512), (2050, 1032), (777, 5504), (40, 16384)]


def tensor(shape, seed, dtype):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, dtype):
    import paper_2502_05003_b200 as quest
    x, res, w = tensor((rows, cols), 1, dtype), tensor((rows, cols), 2, dtype), tensor((cols,), 3, dtype)
    want, plain = quest.quest_rmsnorm_fwd(x, w, 1e-5, res), quest.quest_rmsnorm_fwd(x, w, 1e-5)
    for h, y in (("x", None), ("res", None), (None, "x"), (None, "res"), ("x", "res"), ("res", "x")):
        t = {"x": x.clone(), "res": res.clone()}
        r = quest.quest_rmsnorm_fwd(t["x"], w, 1e-5, t["res"], out={k: t[v] for k, v in (("h", h), ("y", y)) if v})
        assert (h is None or r["h"] is t[h]) and (y is None or r["y"] is t[y])
        for key in ("h", "y", "rstd"):
            assert torch.equal(r[key], want[key])
    t = x.clone()
    r = quest.quest_rmsnorm_fwd(t, w, 1e-5, out={"y": t})
    assert torch.equal(t, plain["y"]) and torch.equal(r["rstd"], plain["rstd"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_gradient(rows, cols, dtype):
    import paper_2502_05003_b200 as quest
    dy, h, dres, w = (tensor(s, i, dtype) for i, s in enumerate(((rows, cols), (rows, cols), (rows, cols), (cols,))))
    rstd = quest.quest_rmsnorm_fwd(h, w)["rstd"]
    want = quest.quest_rmsnorm_bwd(dy, h, w, rstd, dres)
    for place in range(3):
        t = [dy.clone(), h.clone(), dres.clone()]
        r = quest.quest_rmsnorm_bwd(t[0], t[1], w, rstd, t[2], out={"dx": t[place]})
        assert r["dx"] is t[place] and torch.equal(r["dx"], want["dx"]) and torch.equal(r["dw"], want["dw"])


@pytest.mark.parametrize("rows,cols", [(16, 2048), (2100, 512), (1000, 2048)])
def test_a_chain_of_layers(rows, cols):
    import paper_2502_05003_b200 as quest
    res, ws = tensor((rows, cols), 1, BF16), [tensor((cols,), 10 + i, BF16) for i in range(12)]
    stream, y = res.clone(), tensor((rows, cols), 2, BF16)
    a, b = stream, y
    for w in ws:
        r = quest.quest_rmsnorm_fwd(b, w, 1e-5, a, mx_bits=None)
        a, b = r["h"], r["y"]
    torch.cuda.synchronize()
    for _ in range(3):
        p, q = stream.clone(), y.clone()
        codes = []
        for w in ws:
            quest.quest_rmsnorm_fwd(q, w, 1e-5, p, out={"h": p, "y": q})
            codes.append(quest.quest_rmsnorm_fwd(q, w, 1e-5, mx_bits=8)["yq"])
        assert torch.equal(p, a) and torch.equal(q, b)
        assert torch.equal(codes[-1], quest.quest_rmsnorm_fwd(b, ws[-1], 1e-5, mx_bits=8)["yq"])
