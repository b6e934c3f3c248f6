"""The settings that name a kernel of the attention over the cache and its parts, as far as they show without a GPU: in the workspace."""
import ctypes

import pytest

M = pytest.importorskip("paper_2511_13061_amd")
kv = pytest.importorskip("paper_2511_13061_amd.kv")

HEADS, DIM = 32, 128


@pytest.fixture(autouse=True)
def settings():
    yield
    for name in ("attention_kernel", "attention_parts"):
        M.set_tuning(name, 0)


def size(tokens, longest, **more):
    cache = kv._CCache(None, 4096, 64, 8, DIM)
    a = kv._CAttention(tokens, HEADS, 0, 1, None, 0, 0, None, 0, 0, None, None, 0, 0, None, None, tokens, 0, longest, 0.1)
    for name, value in more.items():
        setattr(a, name, value)
    return M.load_library().macko_kv_attention_workspace(ctypes.byref(cache), ctypes.byref(a))


@pytest.mark.parametrize("kernel", [0, 1, 2])
@pytest.mark.parametrize("tokens", [1, 40, 1000])
@pytest.mark.parametrize("parts,longest,made", [(1, 100000, 1), (2, 100000, 2), (7, 12800, 7), (256, 983040, 256), (256, 10 ** 6, 253), (256, 1000, 8), (5, 128, 1), (3, 129, 2)])
def test_parts_by_name(parts, longest, made, tokens, kernel):
    M.set_tuning("attention_kernel", kernel)
    M.set_tuning("attention_parts", parts)
    got = size(tokens, longest)
    assert got == (0 if made == 1 else tokens * HEADS * 4 * (made * (DIM + 2) + 1))


def test_calls_of_very_many_rows_have_one_part():
    M.set_tuning("attention_parts", 9)
    assert size(2 ** 19, 10 ** 6) == 0 and size(2 ** 19 - 1, 10 ** 6) > 0


def test_parts_by_estimate():
    assert size(1, 131072) > 0 and size(1, 100) == 0
    M.set_tuning("attention_kernel", 1)
    few = size(200, 4096)
    M.set_tuning("attention_kernel", 2)
    assert size(1, 131072) > 0 and size(200, 4096) >= 0 and few >= 0


@pytest.mark.parametrize("name,most", [("attention_kernel", 2), ("attention_parts", 256)])
def test_settings_that_are_refused(name, most):
    for value in (-1, most + 1, 2 ** 40):
        with pytest.raises(M.MackoError):
            M.set_tuning(name, value)
    M.set_tuning(name, most)
    assert M.get_tuning(name) == most
