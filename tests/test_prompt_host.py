"""What macko_prompt_attention refuses before anything is launched."""
import ctypes

import pytest

M = pytest.importorskip("paper_2511_13061_amd")
kv = pytest.importorskip("paper_2511_13061_amd.kv")

INVALID, UNSUPPORTED = -1, -3
A = 1 << 20          # an address that is aligned and never followed


def prompt(**change):
    a = kv._CPrompt(3, 4, 2, 64, 0, 1, A, 256, 64, A, 128, 64, A, 128, 64, A, 256, 64, None, A, 0, 3, 0.125)
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(heads=0), INVALID), (dict(heads=3), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=48), UNSUPPORTED),
    (dict(head_dim=288), UNSUPPORTED), (dict(type=2), INVALID), (dict(batch=-1), INVALID), (dict(q=None), INVALID), (dict(k=A + 1), INVALID), (dict(v=None), INVALID),
    (dict(out=A + 1), INVALID), (dict(q_token=-1), INVALID), (dict(k_token=2 ** 40), INVALID), (dict(start=A + 2), INVALID), (dict(sums=A + 2), INVALID), (dict(window=-1), INVALID),
    (dict(longest=-1), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(tokens=2 ** 31), UNSUPPORTED), (dict(tokens=2 ** 29), UNSUPPORTED),
    (dict(heads=2 ** 17), UNSUPPORTED), (dict(heads=65536, kv_heads=1), UNSUPPORTED)])
def test_prompts_that_are_refused(change, status):
    assert M.load_library().macko_prompt_attention(ctypes.byref(prompt(**change)), None) == status


def test_prompts_of_nothing():
    lib = M.load_library()
    assert lib.macko_prompt_attention(None, None) == INVALID
    assert lib.macko_prompt_attention(ctypes.byref(prompt(tokens=0)), None) == 0 and lib.macko_prompt_attention(ctypes.byref(prompt(batch=0)), None) == 0
