"""The tests of many query rows to a group once more, over tables with so much room that these are taken in units of 128 (mpc_shared_attn
chooses its units by the rows and the table's room, not by the lengths)."""
import pytest

import test_gpu_shared_attn as attn
import test_gpu_shared_infinite as infinite
import test_gpu_shared_precision as precision
import test_gpu_shared_wide as wide
from test_gpu_shared_attn import behind, test_many_rows_behind_long_prompts, test_one_workspace_for_every_call, test_windows_and_sinks as test_windows  # noqa: F401
from test_gpu_shared_infinite import test_as_the_paged_attention_has_them, test_infinities_that_every_row_sees  # noqa: F401
from test_gpu_shared_precision import test_weights_in_two_parts  # noqa: F401
from test_gpu_shared_wide import (test_captured_calls_of_batches_on_both_sides_of_a_waves_lanes, test_nan_in_a_shared_row, test_page_sizes,  # noqa: F401
                                  test_pages_that_are_missing, test_queries_that_are_not_finite_stay_by_themselves, test_scales_of_a_page_that_rows_do_not_see,
                                  test_scales_of_the_scores, test_sequences_shorter_than_the_shared_rows, test_strides_layers_and_heads,
                                  test_windows_and_sinks)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room(monkeypatch):
    """Tables of 2^18 rows, most entries of which name no page."""
    def roomy(M, fmt, dtype, lens, first, shared, L=1, Hkv=2, d=64, page=16, seed=3, cap=None):
        import torch
        kv = behind(M, fmt, dtype, lens, first, shared, L, Hkv, d, page, seed, cap)
        table = torch.full((kv.B, (1 << 18) // page), -1, dtype=torch.int32, device="cuda")
        table[:, : kv.table.shape[1]] = kv.table
        return M.PagedKV(kv.k_pages, kv.v_pages, table, kv.lens, k_scale=kv.k_scale, v_scale=kv.v_scale, k_tail=kv.k_tail, v_tail=kv.v_tail,
                         dtype=kv.dtype)

    for module in (attn, wide, infinite, precision):
        monkeypatch.setattr(module, "behind", roomy)
