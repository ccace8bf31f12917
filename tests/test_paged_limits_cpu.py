"""Numbers of tokens so large that their product with the heads leaves 64 bits are refused like other large ones (before anything is
launched)."""
import pytest

import test_paged4_cpu as four
import test_paged_cpu as full
from paper_2605_09649_b200 import binding

HUGE = [(1 << 29) + 1, (1 << 62) + 1, (1 << 62) + (1 << 61) + 2, (1 << 63) - 1]


@pytest.mark.parametrize("n", HUGE)
def test_huge_numbers_of_tokens_are_refused(n):
    four.refused("trimkv_paged4_append", four.append_args(n=n), binding.E_ARG)
    four.refused("trimkv_paged4_read", four.read_args(n=n), binding.E_ARG)
    four.refused("trimkv_paged4_attention", four.attention_args(t=n), binding.E_ARG)
    full.refused("trimkv_paged_append", full.append_args(n=n), binding.E_ARG)
    full.refused("trimkv_paged_attention", full.attention_args(t=n), binding.E_ARG)
    full.refused("trimkv_paged_sparse_attention", full.attention_args(sparse=True, t=n), binding.E_ARG)
