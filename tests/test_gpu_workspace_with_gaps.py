"""A workspace whose elements do not lie one behind the other has less memory than elements: refused before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("make", [lambda n: torch.empty(1, dtype=torch.uint8, device="cuda").expand(n), lambda n: torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2],
                                  lambda n: torch.empty((n, 1), dtype=torch.float32, device="cuda").expand(n, 2)])
def test_refused(make):
    import paper_2502_05003_b200 as quest
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((64, 256), (48, 256), (64, 48)))
    fwd = quest.quest_linear_fwd_mx(x, w, 8, 32)
    with pytest.raises(ValueError, match="workspace"):
        quest.quest_linear_bwd_mx(dy, fwd, 8, 32, 256, workspace=make(quest.quest_bwd_mx_workspace_bytes(64, 48, 256)))
    rstd = torch.ones(64, device="cuda")
    with pytest.raises(ValueError, match="workspace"):
        quest.quest_rmsnorm_bwd(x, x, x[0], rstd, workspace=make(quest.quest_rmsnorm_bwd_workspace_bytes(64, 256)))
