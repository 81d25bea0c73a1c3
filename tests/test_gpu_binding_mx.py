"""The CPython binding and the ctypes path of the microscaled layer and the norm: same results, same keys, same errors."""
import pytest
import torch

from tests.test_gpu_binding import both, same

pytestmark = pytest.mark.gpu


def test_results_and_errors_are_those_of_the_ctypes_path(monkeypatch):
    import paper_2502_05003_b200 as q
    gen = torch.Generator(device="cuda").manual_seed(5)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda").bfloat16()
    x, w, dy = randn(72, 256), randn(48, 256), randn(72, 48)
    fwd = q.quest_linear_fwd_mx(x, w, 8, 32)
    cached = {"wq": fwd["wq"], "sw": fwd["sw"]}
    weight = randn(256)
    h = q.quest_rmsnorm_fwd(x, weight, 1e-5, x.flip(0))
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    calls = [
        lambda: q.quest_quantize_mx(x, 4), lambda: q.quest_quantize_mx(x.float(), 8, 32), lambda: q.quest_quantize_mx(x[:, 8:136], 4),
        lambda: q.quest_quantize_mx(x, 8, codes=u8(72, 256), scales=u8(2048)), lambda: q.quest_quantize_mx(x, 8, codes=u8(72, 255)),
        lambda: q.quest_quantize_mx(x, 8, scales=u8(10)), lambda: q.quest_quantize_mx(x, 6), lambda: q.quest_quantize_mx(x, 4, 2),
        lambda: q.quest_quantize_mx(x[:, :40], 4), lambda: q.quest_quantize_mx(x[:, ::2], 4), lambda: q.quest_quantize_mx(x.cpu(), 4),
        lambda: q.quest_quantize_mx(x.half(), 4), lambda: q.quest_quantize_mx(x[:0], 4), lambda: q.quest_quantize_mx(x[:1], 4),
        lambda: q.quest_dequantize_mx(fwd["xq"], fwd["sx"], 8), lambda: q.quest_dequantize_mx(fwd["wq"], fwd["sw"], 4, torch.float32),
        lambda: q.quest_dequantize_mx(fwd["xq"], fwd["sx"], 8, out=torch.empty((72, 256), device="cuda")),
        lambda: q.quest_dequantize_mx(fwd["xq"], fwd["sx"][:100], 8), lambda: q.quest_dequantize_mx(fwd["xq"][:, ::2], fwd["sx"], 8),
        lambda: q.quest_dequantize_mx(fwd["xq"], fwd["sx"], 8, torch.float16), lambda: q.quest_dequantize_mx(fwd["xq"][:0], fwd["sx"], 8),
        lambda: q.quest_gemm_mx(fwd["xq"], fwd["sx"], 8, fwd["wq"], fwd["sw"], 256),
        lambda: q.quest_gemm_mx(fwd["xq"], fwd["sx"], 8, fwd["wq"], fwd["sw"], 256, y=torch.zeros((72, 50), device="cuda")[:, :48]),
        lambda: q.quest_gemm_mx(fwd["xq"], fwd["sx"], 8, fwd["wq"], fwd["sw"], 256, y=torch.zeros((72, 47), device="cuda")),
        lambda: q.quest_gemm_mx(fwd["xq"], fwd["sx"], 4, fwd["wq"], fwd["sw"], 256), lambda: q.quest_gemm_mx(fwd["xq"], fwd["sx"], 8, fwd["wq"], fwd["sw"], 128),
        lambda: q.quest_linear_fwd_mx(x, w, 4), lambda: q.quest_linear_fwd_mx(x, w.float(), 8, 32, torch.float32),
        lambda: q.quest_linear_fwd_mx(x, None, 8, 32, w_cached=cached), lambda: q.quest_linear_fwd_mx(x[:3], None, 8, 32, w_cached=cached, want_codes=False),
        lambda: q.quest_linear_fwd_mx(x[:20], None, 8, 32, w_cached=cached, want_codes=False, saved={"other": 1}),
        lambda: q.quest_linear_fwd_mx(x[:, 1:129], w[:, :128], 4), lambda: q.quest_linear_fwd_mx(x.t().contiguous().t(), w, 8),
        lambda: q.quest_linear_fwd_mx(x, w[:, :128], 8), lambda: q.quest_linear_fwd_mx(x, None, 8, w_cached={"wq": fwd["wq"][:, :3].contiguous(), "sw": fwd["sw"]}),
        lambda: q.quest_linear_fwd_mx(x, w, 8, saved={"xq": u8(72, 256), "sx": u8(5)}), lambda: q.quest_linear_fwd_mx(x, w, 8, 5),
        lambda: q.quest_linear_fwd_mx(x, w, 7), lambda: q.quest_linear_fwd_mx(x[:0], w, 8), lambda: q.quest_linear_fwd_mx(x, w[:0], 8),
        lambda: q.quest_linear_bwd_mx(dy, fwd, 8, 32, 256), lambda: q.quest_linear_bwd_mx(dy, fwd, 8, 32, 256, torch.bfloat16, want_dx=False),
        lambda: q.quest_linear_bwd_mx(dy, cached, 8, 32, 256, want_dw=False), lambda: q.quest_linear_bwd_mx(dy, cached, 8, 32, 256),
        lambda: q.quest_linear_bwd_mx(dy, fwd, 8, 32, 256, dx=torch.empty((72, 256), device="cuda").bfloat16(), want_dw=False),
        lambda: q.quest_linear_bwd_mx(dy[:7], fwd, 8, 32, 256), lambda: q.quest_linear_bwd_mx(dy.float(), fwd, 8, 32, 256),
        lambda: q.quest_linear_bwd_mx(dy, fwd, 8, 32, 256, want_dx=False, want_dw=False), lambda: q.quest_linear_bwd_mx(dy, fwd, 8, 4, 256),
        lambda: q.quest_linear_bwd_mx(dy, fwd, 8, 32, 256, workspace=u8(256)),
        lambda: q.quest_rmsnorm_fwd(x, weight), lambda: q.quest_rmsnorm_fwd(x, weight.float(), 1e-3, x.flip(0), torch.float32),
        lambda: q.quest_rmsnorm_fwd(x, weight, mx_bits=8), lambda: q.quest_rmsnorm_fwd(x, weight, mx_bits=4, had_block=32, want_rstd=False),
        lambda: q.quest_rmsnorm_fwd(x[:, 1:100], weight[1:100]), lambda: q.quest_rmsnorm_fwd(x, weight, out={"y": torch.zeros((80, 256), device="cuda"), "z": 1}),
        lambda: q.quest_rmsnorm_fwd(x, weight[:7]), lambda: q.quest_rmsnorm_fwd(x, weight, -1.0), lambda: q.quest_rmsnorm_fwd(x, weight, mx_bits=2),
        lambda: q.quest_rmsnorm_fwd(x, weight, residual=x.float()), lambda: q.quest_rmsnorm_fwd(x, weight, mx_bits=8, had_block=4),
        lambda: q.quest_rmsnorm_fwd(x[:, :40], weight[:40], mx_bits=8), lambda: q.quest_rmsnorm_fwd(x[:0], weight),
        lambda: q.quest_rmsnorm_fwd(x, weight, out={"rstd": torch.empty(3, device="cuda")}), lambda: q.quest_rmsnorm_fwd(x, weight, out_dtype=torch.float16),
        lambda: q.quest_rmsnorm_bwd(x, h["h"], weight, h["rstd"]), lambda: q.quest_rmsnorm_bwd(x, h["h"], weight, h["rstd"], x, want_dw=False),
        lambda: q.quest_rmsnorm_bwd(x, h["h"], weight, h["rstd"], want_dx=False, out={"dw": torch.zeros(300, device="cuda")}),
        lambda: q.quest_rmsnorm_bwd(x, h["h"].float(), weight, h["rstd"]), lambda: q.quest_rmsnorm_bwd(x, h["h"], weight, h["rstd"][:9]),
        lambda: q.quest_rmsnorm_bwd(x, h["h"], weight, h["rstd"], workspace=u8(256)), lambda: q.quest_rmsnorm_bwd(x[:0], x[:0], weight, h["rstd"]),
        lambda: q.quest_rmsnorm_bwd(x, h["h"], weight, h["rstd"], want_dx=False, want_dw=False),
    ]
    failed = []
    for i, call in enumerate(calls):
        fast, slow = both(monkeypatch, call)
        try:
            same(fast, slow)
        except AssertionError as e:
            failed.append((i, fast, slow, e))
    assert not failed, failed
