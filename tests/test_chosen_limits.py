"""The choice of pages and the attention over them at the ends of what the calls take, as test_chosen_pages.py has the others."""
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import binding as B
from test_chosen_pages import MB, UNSUPPORTED, cache, refused, status


@pytest.mark.parametrize("seqs,new", [(2100, 127), (1 << 18, 2)])
def test_a_joining_launch_that_is_too_large_is_refused_before_the_attention(seqs, new):
    """Few tokens in many sequences of up to `new`: pieces of 64 pages are joined by a workgroup of 512 threads for each of their heads, 2^32 threads and more"""
    c = cache(num_seqs=seqs, page_table=1 << 40, length=1 << 41)
    assert status(lambda: B.lora_cache_chosen_workspace(c, 32, 127, new, 64)) == UNSUPPORTED
    assert refused("attend", c, num_heads=32, num_tokens=127, max_new=new, budget=64, ldq=1 << 13, ldo=1 << 13, q=1 << 42, o=1 << 43, d_chosen=1 << 44, workspace=1 << 45,
                   d_indptr=3 * MB) == UNSUPPORTED


def test_no_sequence_has_more_than_all_tokens():
    assert B.lora_cache_chosen_workspace(cache(num_seqs=1), 16, 127, 1 << 20, 64) > 0
