"""The gradients of the microscaled layer take codes and scales of the shapes that their arguments say, by the binding as by ctypes."""
import pytest
import torch

from tests.test_gpu_binding import both

pytestmark = pytest.mark.gpu


def test_codes_of_other_shapes_are_refused(monkeypatch):
    import paper_2502_05003_b200 as quest
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((72, 256), (48, 256), (72, 48)))
    eight, four = quest.quest_linear_fwd_mx(x, w, 8, 32), quest.quest_linear_fwd_mx(x, w, 4, 32)
    flat = dict(eight, xq=eight["xq"].reshape(-1), wq=eight["wq"].reshape(-1))
    turned = dict(eight, wq=eight["wq"].view(96, 64))
    signed = dict(eight, xq=eight["xq"].view(torch.int8))
    refused = [
        lambda **k: quest.quest_linear_bwd_mx(dy, eight, 4, 32, 256, **k),          # 8-bit codes read as 4-bit ones
        lambda **k: quest.quest_linear_bwd_mx(dy, four, 8, 32, 128, **k),
        lambda **k: quest.quest_linear_bwd_mx(dy, eight, 8, 32, 128, **k),          # shorter rows than those of the forward call
        lambda **k: quest.quest_linear_bwd_mx(dy[:64], eight, 8, 32, 256, **k),     # fewer rows than those of the forward call
        lambda **k: quest.quest_linear_bwd_mx(dy, flat, 8, 32, 256, **k),
        lambda **k: quest.quest_linear_bwd_mx(dy, turned, 8, 32, 256, **k),
        lambda **k: quest.quest_linear_bwd_mx(dy, signed, 8, 32, 256, **k),
        lambda **k: quest.quest_linear_bwd_mx(dy[:, :40].contiguous(), eight, 8, 32, 256, **k),
    ]
    for i, call in enumerate(refused):
        asked = []
        for want_dx, want_dw in ((True, True), (True, False), (False, True)):
            fast, slow = both(monkeypatch, lambda: call(want_dx=want_dx, want_dw=want_dw))
            assert type(fast) is type(slow) and (not isinstance(fast, tuple) or fast == slow), (i, want_dx, want_dw, fast, slow)
            asked.append(isinstance(fast, tuple) and fast[0] is ValueError)
        assert asked[0] and any(asked[1:]), i
