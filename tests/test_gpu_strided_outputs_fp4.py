"""The FP4 form of the product into a view of a wider buffer: what stands behind the columns of y stays as it was."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,N,pitch", [(torch.float32, 130, 136), (torch.float32, 129, 132), (torch.bfloat16, 130, 136), (torch.bfloat16, 133, 144),
                                           (torch.float32, 132, 140), (torch.bfloat16, 136, 144)])
@pytest.mark.parametrize("M", [5, 200, 600])
def test_lowbit_gemm_fp4(M, dtype, N, pitch):
    import paper_2502_05003_b200 as quest
    from paper_2502_05003_b200 import _lib
    gen = torch.Generator(device="cuda").manual_seed(M)
    x, w = torch.randn((M, 256), generator=gen, device="cuda"), torch.randn((N, 256), generator=gen, device="cuda")
    (xq, sx, _), (wq, sw, _) = quest.quest_quantize_fp4(x, 128), quest.quest_quantize_fp4(w, 128)
    want, _ = quest.quest_lowbit_gemm_fp4(xq, sx, wq, sw, 256, out_dtype=dtype)
    room = torch.full((M, pitch), 7.0, dtype=dtype, device="cuda")
    # the row stride of y is an argument of the C ABI only
    _lib.check(_lib.load().quest_lowbit_gemm_fp4(xq.data_ptr(), sx.data_ptr(), wq.data_ptr(), sw.data_ptr(), M, N, 256, room.data_ptr(),
                                                 0 if dtype == torch.float32 else 1, pitch, None, None, 0, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(room[:, :N], want) and bool((room[:, N:] == 7.0).all())
