"""Arguments of the paged calls that would have been taken for others (no GPU)."""
import pytest

from paper_2501_06807_amd import _lib as L


@pytest.mark.parametrize("kw", [dict(window=2 ** 32 + 5, sinks=0), dict(window=5, sinks=2 ** 32), dict(window=2 ** 31, sinks=0),
                                dict(window=0, sinks=-2 ** 31 - 1)])
def test_windows_and_sinks_beyond_32_bits(kw):
    """Their lower 32 bits would be a window of another size."""
    with pytest.raises(ValueError):
        L._attn_cfg(0.1, **kw)


def test_windows_and_sinks_that_fit():
    c = L._attn_cfg(0.25, 2 ** 31 - 1, 7)
    assert (c.sm_scale, c.window, c.sinks) == (0.25, 2 ** 31 - 1, 7)
    assert L._attn_cfg(0.1, -1, -1).window == -1  # (the library refuses these)
