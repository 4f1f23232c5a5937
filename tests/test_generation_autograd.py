"""append and attend have no backward: with tensors that require a gradient, and gradients enabled, they say so."""
import warnings

import pytest

torch = pytest.importorskip("torch")

from tests.test_generation_calls import append, attend, cache, lib, rows  # noqa: E402,F401


@pytest.mark.parametrize("call,name,heads", [(append, "k", 2), (append, "v", 2), (append, "q", 4), (attend, "q", 4)])
def test_a_warning_where_a_gradient_would_be_lost(lib, call, name, heads):  # noqa: F811
    with pytest.warns(UserWarning, match="no backward"):
        call(cache(), **{name: rows(heads, grad=True)})
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        call(cache())
        with torch.no_grad():
            call(cache(), **{name: rows(heads, grad=True)})
        call(cache(), **{name: rows(heads, grad=True).detach()})


def test_a_warning_for_pages_that_require_a_gradient(lib):  # noqa: F811
    kv = cache()
    kv.v.requires_grad_()
    with pytest.warns(UserWarning, match="no backward"):
        attend(kv)


def test_the_warning_names_the_callers_line(lib):  # noqa: F811
    kv = cache()
    with pytest.warns(UserWarning) as seen:
        attend(kv, q=rows(4, grad=True))
        append(kv, q=rows(4, grad=True))
    assert all(w.filename.endswith("test_generation_calls.py") for w in seen)
