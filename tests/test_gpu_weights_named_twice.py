"""The attention weight of cached keys where a call names a sequence twice."""
import numpy as np
import pytest

from test_gpu_serving import make_cache

pytestmark = pytest.mark.gpu

FLAG_SEQUENCE = 32


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


@pytest.mark.parametrize("dim,heads", [(64, 2), (256, 1)])
@pytest.mark.parametrize("new,count", [(1, 3), (1, 140), (1, 300), (40, 3), (40, 140), (20, 300)])
def test_weights_of_a_sequence_named_twice(torch, rm, dim, heads, new, count):
    """The first of them counts, the others are reported and receive nothing, wherever in the call they are."""
    rng = np.random.default_rng(count + new)
    cache = make_cache(torch, rm, [int(n) for n in rng.integers(new, 90, count)], page=16, heads=heads, dim=dim)
    order = [int(s) for s in rng.permutation(count)]
    q = torch.randn(count * new, 2 * heads, dim, device="cuda").half()
    offset = lambda n: torch.arange(0, n * new + 1, new, dtype=torch.int32, device="cuda")
    _, lse = rm.kv_attention(cache, order, q, offset(count))
    start = torch.rand(cache.key_weights().shape, device="cuda")
    for fresh in (False, True):
        for twice in ([(count - 1, 0)], [(1, 0)], [(i, i // 2) for i in range(1, count, 3)]):        # (place, the place whose sequence it names too)
            seqs = list(order)
            for at, like in twice:
                seqs[at] = seqs[like]
            first = [i for i in range(count) if seqs[i] not in seqs[:i]]
            rows = torch.cat([torch.arange(i * new, (i + 1) * new) for i in first]).cuda()
            # each row's lse is of another sequence where it was renamed: shares then add up to something else, and are compared all the same
            want, got = start.clone(), start.clone()
            n = len(first)
            rm.kv_weights(cache, [seqs[i] for i in first], q[rows], lse[rows], want, offset(n), fresh=fresh)
            assert cache.status_flags() == 0
            rm.kv_weights(cache, seqs, q, lse, got, offset(count), fresh=fresh)
            assert cache.status_flags() == FLAG_SEQUENCE
            cache.status.zero_()
            assert torch.equal(got.view(torch.int32), want.view(torch.int32))
    rm.kv_weights(cache, order, q, lse, start, offset(count))
    assert cache.status_flags() == 0


def test_weights_of_a_sequence_named_twice_among_many_slots(torch, rm):
    """More slots than are kept track of one by one."""
    slots = 700000
    cache = rm.KVCache(4, 16, 1, 16, slots, 1)
    spread = [3, 3 + 65536, 3 + 131072, 3 + 420864, 699999, 3 + 16384, 3 + 32768]
    used = torch.tensor(spread, device="cuda")
    cache.pages[used[:4], 0] = torch.arange(4, dtype=torch.int32, device="cuda")
    cache.refs.fill_(1)
    cache.length[used[:4]] = 9
    cache.k.copy_(torch.randint(0, 100, cache.k.shape, device="cuda", dtype=torch.uint8))
    for new in (1, 9):
        n = len(spread)
        q, lse = torch.randn(n * new, 2, 16, device="cuda").half(), torch.zeros(n * new, 2, device="cuda")
        offset = torch.arange(0, n * new + 1, new, dtype=torch.int32, device="cuda")
        want, got = cache.key_weights(), cache.key_weights()
        rm.kv_weights(cache, spread, q, lse, want, offset, fresh=True)
        assert cache.status_flags() == 0
        rm.kv_weights(cache, spread + [spread[1]], torch.cat([q, q[:new]]), torch.cat([lse, lse[:new]]), got, torch.cat([offset, offset[-1:] + new]), fresh=True)
        assert cache.status_flags() == FLAG_SEQUENCE
        cache.status.zero_()
        assert torch.equal(got, want) and float(want.sum()) > 0
