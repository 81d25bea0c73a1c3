"""GPU: a lone row has no next one, so its distance to it matters to no call (torch calls such a row contiguous whatever its pitch)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def pitched(cols, pitch, seed, dtype=BF16):
    a = torch.from_numpy(np.random.default_rng(seed).standard_normal((3, pitch))).to(dtype).cuda()
    return a[:1, :cols], a[:1, :cols].clone()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pitch", [2051, 2052, 2056])
def test_products(pitch, dtype):
    import paper_2502_05003_b200 as quest
    (x, xd), (w, wd) = pitched(2048, pitch, 1, dtype), pitched(2048, pitch, 2, dtype)
    assert x.stride(0) == pitch and x.is_contiguous()
    for bits in (4, 8):
        for a, b in zip(quest.quest_quantize_mx(x, bits, 32), quest.quest_quantize_mx(xd, bits, 32)):
            assert torch.equal(a, b)
        want = quest.quest_linear_fwd_mx(xd, wd, bits, 32, F32)
        for codes in (True, False):
            got = quest.quest_linear_fwd_mx(x, w, bits, 32, F32, want_codes=codes)
            assert torch.equal(got["y"], want["y"]) and torch.equal(got["wq"], want["wq"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pitch", [2051, 2052, 2056])
def test_norm(pitch, dtype):
    import paper_2502_05003_b200 as quest
    (x, xd), (r, rd), (dy, dyd) = (pitched(2048, pitch, s, dtype) for s in (1, 2, 3))
    w = torch.rand(2048, device="cuda").to(dtype)
    for bits in (None, 4, 8):
        got, want = quest.quest_rmsnorm_fwd(x, w, 1e-5, r, mx_bits=bits), quest.quest_rmsnorm_fwd(xd, w, 1e-5, rd, mx_bits=bits)
        for key in ("h", "rstd", "y") if bits is None else ("h", "rstd", "yq", "sy"):
            assert torch.equal(got[key], want[key])
    got, want = quest.quest_rmsnorm_bwd(dy, x, w, got["rstd"], r), quest.quest_rmsnorm_bwd(dyd, xd, w, got["rstd"], rd)
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dw"], want["dw"])
