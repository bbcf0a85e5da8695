"""Reordering and eviction where the table or the counts are not what they should be, or the pages do not suffice: nothing is changed but the status."""
import numpy as np
import pytest

from test_gpu_bounded_cache import FLAG_PAGE, check_evict, check_reorder, state, unchanged
from test_gpu_serving import make_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("gpu-marked test run without a CUDA device")
    return torch


@pytest.fixture(scope="module")
def rm(torch):
    import paper_2607_16784_b200 as pkg
    return pkg


def refused(torch, rm, cache, seqs, parents, flag=FLAG_PAGE):
    before = state(cache)
    rm.kv_reorder(cache, seqs, parents)
    assert cache.status_flags() == flag
    cache.status.zero_()
    unchanged(torch, cache, before)


@pytest.mark.parametrize("bad", [99, -1, -7])
@pytest.mark.parametrize("parents", [[0, 1, 2], [1, 0, 2], [0, 1, 0], [0, -1, 1], [-1, 0, -1]])
def test_reorder_refuses_an_entry_that_is_no_page(torch, rm, bad, parents):
    """In a row of any number of children, one among them; in the middle of it, and its part-filled end."""
    for entry in (0, 1, 2):
        cache = make_cache(torch, rm, [40, 33, 5], page=16, slots=3, extra=6)
        cache.pages[0, entry] = bad
        refused(torch, rm, cache, [0, 1, 2], parents)


@pytest.mark.parametrize("parents", [[0, -1, 2], [-1, 0, 2], [0, 0, 2], [1, 1, 1], [2, 2, 0], [0, -1, 0]])
def test_reorder_refuses_a_page_with_more_holders_than_counts(torch, rm, parents):
    """A page of count 1 in two rows of the call: without the count of the one that ends, the other's children would read a page that counts as free, or for fewer."""
    cache = make_cache(torch, rm, [48, 48, 20], page=16, slots=3, extra=6)
    cache.pages[1, 1] = cache.pages[0, 1]
    refused(torch, rm, cache, [0, 1, 2], parents)
    cache.refs[cache.pages[0, 1].item()] = 2                                  # with both counted the call goes through
    check_reorder(torch, rm, cache, [0, 1, 2], parents)


@pytest.mark.parametrize("parents", [[0, 1], [0, 0], [1, 1], [-1, 0], [1, 0]])
@pytest.mark.parametrize("entry", [0, 1])
def test_reorder_refuses_a_page_that_counts_as_free(torch, rm, parents, entry):
    """A whole page and a part-filled one, whatever becomes of their sequence."""
    cache = make_cache(torch, rm, [20, 16], page=16, slots=2, extra=4)
    cache.refs[cache.pages[0, entry].item()] = 0
    refused(torch, rm, cache, [0, 1], parents)


def test_reorder_takes_back_what_it_counted(torch, rm):
    """Searches whose beams share a prompt, widened and narrowed in a pool of ten pages: sequences with several children and with none, pages with many holders."""
    rng = np.random.default_rng(7)
    full = served = 0
    for trial in range(20):
        slots, everyone = 12, list(range(12))
        cache = rm.KVCache(10, 16, 2, 16, slots, 8, layers=2)
        cache.k.copy_(torch.randint(0, 256, cache.k.shape, device="cuda", dtype=torch.uint8))
        ws = cache.workspace()
        rm.kv_reserve(cache, [0], [int(rng.integers(33, 48))], workspace=ws)
        assert check_reorder(torch, rm, cache, everyone, [0] * 3 + [-1] * 9, ws)       # two shared pages, three of their own
        for step in range(6):
            alive = [i for i, n in enumerate(cache.length.tolist()) if n]
            wide = int(rng.integers(1, 13))
            ok = check_reorder(torch, rm, cache, everyone, [int(rng.choice(alive)) for _ in range(wide)] + [-1] * (slots - wide), ws)
            full, served = full + (not ok), served + ok
        rm.kv_free(cache, everyone)
        assert not cache.refs.any() and cache.status_flags() == 0
    assert full > 20 and served > 20


def test_reorder_into_pages_that_the_call_gives_back(torch, rm):
    """In a full pool: a copy fits where a sequence ends, and nothing is changed where none does."""
    cache = make_cache(torch, rm, [20, 17], page=16, extra=0, slots=3)
    assert not check_reorder(torch, rm, cache, [0, 1, 2], [0, 1, 0])
    assert check_reorder(torch, rm, cache, [0, 1, 2], [0, 0, 0])
    assert int((cache.refs == 0).sum()) == 0 and int(cache.refs.max()) == 3


def test_evict_leaves_a_sequence_whose_page_counts_as_free(torch, rm):
    """Such a page may be handed out in the same call to another sequence: neither is the sequence cut, nor its counts changed."""
    for entry in (0, 3, 9):
        cache = make_cache(torch, rm, [160, 160, 160], page=16, slots=3, extra=16)
        cache.refs[cache.pages[1, entry].item()] = 0
        check_evict(torch, rm, cache, [0, 1, 2], 50, served=[0, 2], flags=FLAG_PAGE)
