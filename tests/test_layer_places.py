"""Results of layers that lie where something else does: refused before anything is launched."""
import pytest

from test_layer_refusals import BASE, calls, handle, lib  # noqa: F401


@pytest.mark.parametrize("change,words,which", [
    (dict(y=64, r=64, ldr=24, ldy=16), "other rows", 1), (dict(y=64, r=64, ldr=16, ldy=24), "other rows", 1),
    (dict(y=64, w=64), "overlap", 1), (dict(z=64, w=64), "overlap", 2), (dict(dx=64, w=64), "overlap", 2), (dict(dx=64, dw=64), "overlap", 2), (dict(z=64, dw=64), "overlap", 2),
    (dict(dw=64, db=64), "overlap", 2), (dict(act=2, slope=1024, dw=64, dslope=64), "overlap", 2), (dict(act=2, slope=1024, dx=64, dslope=64), "overlap", 2),
])
def test_results_at_other_places(lib, handle, change, words, which):  # noqa: F811
    for k, (status, message) in enumerate(calls(lib, handle, **change)):
        if which >> k & 1:
            assert status < 0 and words in message, (k, status, message)


@pytest.mark.parametrize("change", [
    dict(y=64, r=64, ldr=24, ldy=24), dict(y=64, r=64, ldr=24, ldy=16, n=1), dict(dy=64, dx=64, lddx=16), dict(w=64, dw=64, dx=128), dict(z=64, dy=64), dict(act=2, slope=1024, dslope=1024, dw=64),
])
def test_places_that_are_allowed(lib, handle, change):  # noqa: F811
    """Such calls pass the checks, and then find no device."""
    for k, (status, message) in enumerate(calls(lib, handle, **change)):
        assert status != 0 and "cuda" in message.lower(), (k, status, message)


def test_no_rows_and_nothing_wanted(lib, handle):  # noqa: F811
    """Null pointers are at no place."""
    assert BASE["n"] > 0
    (_, _), (status, message) = calls(lib, handle, act=0, z=None, n=6)
    assert status != 0 and "cuda" in message.lower(), message
