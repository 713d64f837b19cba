"""Resizes of pages at the ends of what the call takes, as test_pages.py has the others."""
import pytest

torch = pytest.importorskip("torch")

from paper_2411_00915_amd import binding as B
from test_pages import BAD, DEV, UNSUPPORTED, desc, gpu, status


@pytest.mark.parametrize("field", ["d_token_seq", "d_token_position", "d_token_slot"])
def test_a_last_launch_that_is_too_large_is_refused_before_the_first(field):
    """2^14 sequences of 4200 pieces of 1024 tokens: 4.4e9 threads.  Where no token's number is wanted, and with fewer rows, launches are of the table's size"""
    big = dict(page_table=1 << 40, num_seqs=1 << 14, table_stride=4200, max_length=4200 * 1024, page_tokens=1024)
    p = B.Pages(desc(**big))
    need = B.lora_pages_workspace(p)
    rows = 4200 * 1024
    none = dict(d_token_seq=None, d_token_position=None, d_token_slot=None)
    fine = dict(d_wanted=1 << 41, d_granted=None, d_indptr=None, d_copies=1 << 42, workspace=1 << 43, workspace_bytes=need)
    resize = lambda **f: status(lambda: B.lora_pages_resize(p, **{**fine, **none, **f}, stream=1))  # noqa: E731
    assert resize(num_tokens=rows, **{field: 1 << 44}) == UNSUPPORTED
    assert resize(num_tokens=2 ** 30, **{field: 1 << 44}) == UNSUPPORTED
    assert resize(num_tokens=4096 * 1024, **{field: 1 << 44}) == UNSUPPORTED


def test_a_list_of_copies_in_the_cache_itself_is_refused():
    """Five pairs, 40 bytes, around both ends of 100 pages of 8 heads, and of their weights"""
    size = 100 * 8 * B.lora_cache_page_bytes(64, 128)
    for weight in (None, 64 << 20):
        c = B.Cache(B.CacheDesc(16 << 20, weight, 2 << 20, 3 << 20, 100, 4, 10, 640, 64, 8, 128))
        places = [(16 << 20, size)] + ([(weight, 100 * 8 * 64 * 4)] if weight else [])
        for at, n in places:
            for copies in (at - 36, at, at + n // 2, at + n - 4):
                assert status(lambda: B.lora_cache_copy(c, 5, copies, 1)) == BAD, (at, copies)


@gpu
def test_no_sequences_have_no_tokens():
    """Offsets have one more number than there are sequences; also in a graph"""
    p = B.Pages(desc(num_seqs=0, page_table=0, length=0, users=0))
    out = torch.full((2,), 7, dtype=torch.int32, device=DEV)
    call = lambda: B.lora_pages_resize(p, None, 5, None, out, None, None, None, None, None, 0)  # noqa: E731
    call()
    torch.cuda.synchronize()
    assert out.tolist() == [0, 7]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for value in (3, -1):
        out.fill_(value)
        graph.replay()
        torch.cuda.synchronize()
        assert out.tolist() == [0, value]
