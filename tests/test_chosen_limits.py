"""The choice of pages and the attention over them at the ends of what the calls take, as test_chosen_pages.py has the others."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import binding as B
from test_attention import BF16, F32, gpu, rounded
from test_chosen_pages import MB, UNSUPPORTED, Long, cache, check_choice, refused, run_choose, status


@pytest.mark.parametrize("seqs,new", [(2100, 127), (1 << 18, 2)])
def test_a_joining_launch_that_is_too_large_is_refused_before_the_attention(seqs, new):
    """Few tokens in many sequences of up to `new`: pieces of 64 pages are joined by a workgroup of 512 threads for each of their heads, 2^32 threads and more"""
    c = cache(num_seqs=seqs, page_table=1 << 40, length=1 << 41)
    assert status(lambda: B.lora_cache_chosen_workspace(c, 32, 127, new, 64)) == UNSUPPORTED
    assert refused("attend", c, num_heads=32, num_tokens=127, max_new=new, budget=64, ldq=1 << 13, ldo=1 << 13, q=1 << 42, o=1 << 43, d_chosen=1 << 44, workspace=1 << 45,
                   d_indptr=3 * MB) == UNSUPPORTED


def test_no_sequence_has_more_than_all_tokens():
    assert B.lora_cache_chosen_workspace(cache(num_seqs=1), 16, 127, 1 << 20, 64) > 0


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hkv,D", [(4, 2, 64), (8, 1, 128), (2, 2, 256), (20, 1, 80)])
@pytest.mark.parametrize("lengths,budget", [([32 * 257, 32 * 256, 32 * 300 + 1], 3), ([32 * 480, 77, 32 * 400 - 5], 130), ([32 * 300, 32 * 479 + 1, 32 * 260], 300)])
@pytest.mark.parametrize("pages", [40, 5000])
def test_some_hundred_pages_in_one_launch(dtype, H, Hkv, D, lengths, budget, pages):
    """More pages than one wavefront chooses among, and too few for pieces: keys in LDS, the last page chosen by all; many equal ones where a few pages are named often"""
    rng = np.random.default_rng(budget + D)
    pool = Long(lengths, Hkv, D, 32, pages, D)
    q = rounded(rng.standard_normal((len(lengths), H, D)), dtype)
    assert B.lora_cache_choose_workspace(pool.cache, len(lengths), 1) == 0
    got = run_choose(pool, q, [1] * len(lengths), dtype, pool.bounds, pool.steps, budget, 1, 1, ptr=None)
    check_choice(pool, q, [1] * len(lengths), lengths, pool.bounds, pool.steps, budget, 1, 1, got)


@gpu
@pytest.mark.parametrize("dtype,H,Hkv,D,max_pages,new,budget", [(F32, 2, 2, 64, 12288, 66, 40), (BF16, 2, 2, 64, 12289, 66, 40), (BF16, 4, 4, 128, 12288, 33, 200), (F32, 4, 4, 256, 12300, 33, 9),
                                                                (BF16, 18, 1, 64, 1000, 130, 64), (F32, 40, 2, 33, 700, 65, 333)])
def test_more_workgroups_than_compute_units(dtype, H, Hkv, D, max_pages, new, budget):
    """One launch: keys in LDS up to 12288 pages, past them in the workspace"""
    rng = np.random.default_rng(max_pages)
    lengths, count = [32 * max_pages, 32 * 700 - 3], [new, new]
    pool = Long(lengths, Hkv, D, 32, 3000, new)
    q = rounded(rng.standard_normal((2 * new, H, D)), dtype)
    assert 2 * new * Hkv > 256 and (B.lora_cache_choose_workspace(pool.cache, 2 * new, new) > 0) == (max_pages > 12288)
    got = run_choose(pool, q, count, dtype, pool.bounds, pool.steps, budget, 1, 1)
    check_choice(pool, q, count, lengths, pool.bounds, pool.steps, budget, 1, 1, got)
