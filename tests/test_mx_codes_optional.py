"""Where x may be quantized inside the microscaled product: the library answers, and both bindings ask it."""
import ctypes
import os

import pytest

FAKE = ctypes.c_void_p(0x10000)                                   # never dereferenced: no call gets past the checks
HERE = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2502_05003_b200 import build, _lib
    build.build()
    return _lib.load()


@pytest.mark.parametrize("M,N,K,answer", [(1, 2048, 2048, 1), (1, 7104, 4096, 1), (1, 7105, 4096, 0), (1, 2048, 4128, 0), (8, 7104, 512, 1), (8, 8, 544, 0),
                                          (9, 8, 32, 0), (2, 8, 2048, 1), (2, 8, 2080, 0), (-1, 8, 32, 0), (1, 8, 40, 0)])
def test_the_rule_and_the_call_agree(lib, M, N, K, answer):
    import torch
    assert lib.quest_mx_codes_optional(M, N, K) == answer
    # without codes the call is refused (a null pointer) where the answer is 0; where it is 1 what it misses is the device
    if M > 0 and K % 32 == 0 and not torch.cuda.is_available():
        status = lib.quest_linear_fwd_mx(FAKE, 1, K, None, 1, K, M, N, K, 4, 1, FAKE, 1, N, None, None, FAKE, FAKE, 1, None)
        assert (status == 1) == (answer == 0)


def test_the_bindings_ask(lib):
    for name in ("__init__.py", "csrc/quest_binding.cpp"):
        with open(os.path.join(HERE, "paper_2502_05003_b200", name)) as f:
            text = f.read()
        assert "quest_mx_codes_optional(M, N, K)" in text and "7104)" not in text and "> 7104" not in text
