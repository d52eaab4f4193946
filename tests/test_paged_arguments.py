"""Arguments of the paged calls that would have been taken for others (no GPU)."""
import pytest
from test_paged_refusals import FAKE, cache, dims, ref, rope

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


@pytest.mark.parametrize("qs,os_,same", [
    (None, L.MpcStrides(8192, 4096, 512, 128), True),  # the contiguous ones, written out: two layers, two sequences, eight heads
    (None, L.MpcStrides(8192, 4096, 128, 1024), False),  # tokens before heads
    (L.MpcStrides(8192, 4096, 128, 1024), None, False),
    (L.MpcStrides(8192, 4096, 128, 1024), L.MpcStrides(8192, 4096, 128, 1024), True),
    (None, L.MpcStrides(16384, 8192, 1024, 128), False),
])
def test_queries_in_place_are_rotated_where_they_lie(qs, os_, same):
    """Written in another order, a row would be overwritten before it is read. (k_out is k here: a call that passes is refused
    for that, and launches nothing.)"""
    s = L.lib().mpc_paged_append(ref(dims()), ref(cache()), 4, None, ref(rope()), None, FAKE, None, FAKE, None, FAKE, ref(qs), FAKE,
                                 ref(os_), FAKE, None, None)
    assert s == L.MPC_EINVAL and ("k_out" if same else "q_out") in L.lib().mpc_last_error().decode()


def test_strides_of_axes_of_one_entry_are_not_compared():
    s = L.lib().mpc_paged_append(ref(dims(batch=1, n_layers=1)), ref(cache()), 1, None, ref(rope()), None, FAKE, None, FAKE, None, FAKE,
                                 None, FAKE, ref(L.MpcStrides(7, 0, 128, 1)), FAKE, None, None)
    assert s == L.MPC_EINVAL and "k_out" in L.lib().mpc_last_error().decode()
