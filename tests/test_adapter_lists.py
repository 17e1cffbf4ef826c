"""Adapter lists that do not belong to a context are refused before the library
reads them: it takes one entry for every layer of the model.  No call here
touches a GPU, or reaches the library."""
import types

import pytest

from paper_2604_20919_amd import sdverify as sv


@pytest.fixture
def ctx(monkeypatch):
    """A context of three layers on GPU 0, as far as the binding knows."""
    def reached(*a):
        raise AssertionError("the library was called")
    monkeypatch.setattr(sv, "lib", lambda: types.SimpleNamespace(sd_adapters_set=reached))
    monkeypatch.setitem(sv._contexts, 4096, sv._Context(3, 0))
    return 4096


def _lora(index=0):
    t = types.SimpleNamespace(device=types.SimpleNamespace(index=index))
    return types.SimpleNamespace(a=t, b=t, scale=None, desc=sv.sd_lora())


@pytest.mark.parametrize("layers", [[], [{}], [{}, {}], [{}] * 4])
def test_lists_of_other_lengths(ctx, layers):
    with pytest.raises(ValueError, match="layers"):
        sv.sd_adapters_set(ctx, layers)


def test_adapters_on_another_gpu(ctx):
    with pytest.raises(ValueError, match="GPU 0"):
        sv.sd_adapters_set(ctx, [{"o": _lora()}, {}, {"down": _lora(1)}])


def test_names_and_contexts_that_are_not_there(ctx):
    with pytest.raises(ValueError, match="gate"):
        sv.sd_adapters_set(ctx, [{"gate": _lora()}, {}, {}])
    for layers in (None, [{}] * 3):
        with pytest.raises(ValueError, match="context"):
            sv.sd_adapters_set(4097, layers)
