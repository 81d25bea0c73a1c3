"""GPU parity of the microscaled products on both sides of every limit of the kernel of few rows: one and several groups of 16 rows
of w to a CTA, one to four groups of eight rows of x, one and two rounds of its warps over K, x quantized inside or given as codes.
The kernel that ran is asked for by name, so that a limit that moves leaves no case behind.

Bound as in test_gpu_mx_tiles.py."""
import re

import pytest
import torch

from tests.test_gpu_mx_tiles import BF16, F32, check, draw, exact, status

pytestmark = pytest.mark.gpu

# rows of x, rows of w, K for 8 and 4 bits; groups of 16 rows of w and of 8 rows of x that a CTA takes, or None: another kernel
CASES = [
    (1, 77, 2048, 2016, 1, 1),
    (1, 300, 4096, 4064, 1, 1),          # two rounds over K, fused
    (1, 300, 4224, 4128, None, None),
    (1, 4736, 256, 288, 1, 1),
    (1, 4737, 256, 288, 3, 1),           # three groups of w, fused
    (1, 5504, 2048, 2016, 3, 1),
    (1, 7104, 4096, 4064, 3, 1),
    (1, 7105, 256, 288, None, None),
    (3, 5000, 1280, 1312, 3, 1),
    (8, 4737, 512, 480, 3, 1),
    (8, 7104, 512, 32, 3, 1),
    (8, 5504, 640, 672, 3, 1),           # from codes
    (8, 77, 2176, 2080, 1, 1),           # two rounds over K, from codes
    (7, 4801, 4096, 4064, 3, 1),
    (8, 300, 4224, 4128, None, None),
    (9, 2368, 512, 544, 1, 2),
    (9, 2369, 512, 544, 2, 2),
    (9, 2400, 3584, 3616, 2, 2),         # two rounds
    (13, 130, 2432, 2464, 1, 2),
    (16, 4736, 2048, 2016, 2, 2),
    (16, 4737, 512, 544, None, None),
    (16, 300, 2176, 2080, None, None),
    (17, 2369, 1792, 1824, 2, 3),
    (24, 2368, 256, 288, 1, 3),
    (24, 3552, 1280, 1312, 2, 3),
    (24, 3553, 256, 288, None, None),
    (25, 2369, 1280, 1184, 2, 4),
    (32, 2368, 1024, 992, 1, 4),
    (32, 3552, 1024, 992, 2, 4),
    (32, 300, 1152, 1056, None, None),
    (33, 300, 256, 288, None, None),
]


def kernels(call):
    """What the call returns, and the names of the product kernels that it ran with their template arguments."""
    torch.cuda.synchronize()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA], acc_events=True) as p:
        result = call()
        torch.cuda.synchronize()
    found = [re.search(r"(mx_few_rows|mx_thin|mx_gemm)_kernel<([^>]*)>", e.name) for e in p.events()]
    return result, [(m.group(1), [re.sub(r"^\(\w+\)", "", a.strip()) for a in m.group(2).split(",")]) for m in found if m]


def few(bits, groups_x, groups_w, fused):
    """Template arguments of the kernel of few rows; a truth value reads "true" or "1"."""
    return [[("mx_few_rows", [str(bits), str(groups_x), str(groups_w), word])] for word in (("true", "1") if fused else ("false", "0"))]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K8,K4,groups_w,groups_x", CASES)
def test_few_rows(M, N, K8, K4, groups_w, groups_x, bits):
    import paper_2502_05003_b200 as quest
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the limits are those of 148 SMs")
    K = K8 if bits == 8 else K4
    x = draw(M, K, M + K)
    xc, xs = quest.quest_quantize_mx(x, bits)
    wc, ws = quest.quest_quantize_mx(draw(N, K, N), 4)
    want, size = exact(quest, xc, xs, bits, wc, ws)
    for out, pad, skip in ((F32, 5, 1), (BF16, 8, 8)):
        # a row before and behind, columns on both sides: none is touched
        room = torch.full((M + 2, skip + N + pad), 7.0, dtype=out, device="cuda")
        y = room[1:M + 1, skip:skip + N]
        _, ran = kernels(lambda: quest.quest_gemm_mx(xc, xs, bits, wc, ws, K, y=y))
        if groups_w is None:
            assert [name for name, _ in ran] == ["mx_thin"], ran
        else:
            assert ran in few(bits, groups_x, groups_w, False), ran
        check(y, want, size, K)
        given = y.clone()
        y.fill_(7.0)
        assert bool((room == 7.0).all())
        # from values: the same codes, and the same sums in the same order
        _, ran = kernels(lambda: quest.quest_linear_fwd_mx(x, None, bits, 1, y=y, w_cached={"wq": wc, "sw": ws}, want_codes=False))
        assert torch.equal(y, given)
        y.fill_(7.0)
        assert bool((room == 7.0).all())
        if groups_w is not None:
            assert ran in few(bits, groups_x, groups_w, M <= 8 and M * K <= 4096), ran
    status()
