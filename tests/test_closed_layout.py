"""Handles that stand on a layout refuse to be used once it is closed."""
import ctypes

import pytest


@pytest.mark.parametrize("kind", ["Grads", "TopK"])
def test_handle_on_a_closed_layout(kind):
    """The library reads the layout through the handle, and closing has freed it."""
    from paper_2008_05823_amd import saef as S
    layout, user = object.__new__(S.Layout), object.__new__(getattr(S, kind))
    layout._h, user._h, user.layout = ctypes.c_void_p(64), ctypes.c_void_p(128), layout
    try:
        assert user.handle.value == 128
        layout._h = None  # as close() leaves it
        with pytest.raises(ValueError, match="layout destroyed"):
            user.handle
    finally:  # (no such handles: nothing to free)
        layout._h = user._h = None
