"""Products into a view of a wider buffer: what stands behind the columns of y stays as it was.  Rows of y that do not end on a
16-byte boundary cannot leave by tile stores, which write whole 16-byte pieces."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,N,pitch", [(torch.float32, 130, 136), (torch.float32, 129, 132), (torch.bfloat16, 130, 136), (torch.bfloat16, 133, 144),
                                           (torch.float32, 132, 140), (torch.bfloat16, 136, 144)])
@pytest.mark.parametrize("bits", [2, 4, 8])
def test_lowbit_gemm(bits, dtype, N, pitch):
    import paper_2502_05003_b200 as quest
    gen = torch.Generator(device="cuda").manual_seed(bits)
    x, w = torch.randn((200, 256), generator=gen, device="cuda"), torch.randn((N, 256), generator=gen, device="cuda")
    xq, sx, _ = quest.quest_quantize(x, bits, 128)
    wq, sw, _ = quest.quest_quantize(w, bits, 128)
    want, _ = quest.quest_lowbit_gemm(xq, sx, bits, wq, sw, bits, 256, out_dtype=dtype)
    room = torch.full((200, pitch), 7.0, dtype=dtype, device="cuda")
    quest.quest_lowbit_gemm(xq, sx, bits, wq, sw, bits, 256, y=room[:, :N])
    assert torch.equal(room[:, :N], want) and bool((room[:, N:] == 7.0).all())
    room.fill_(7.0)
    wide = quest.quest_linear_fwd_weight_only(x.bfloat16(), w.bfloat16(), bits, 128, out_dtype=dtype)["y"]
    quest.quest_linear_fwd_weight_only(x.bfloat16(), w.bfloat16(), bits, 128, out={"y": room[:, :N]})
    assert torch.equal(room[:, :N], wide) and bool((room[:, N:] == 7.0).all())
