"""Reordering of cached sequences and eviction from the cache, against their definitions on lists: tables, counts, codes, scales and weights are
compared exactly."""
import numpy as np
import pytest

import bounded_plain as bp
import serving_plain as sp
from test_gpu_serving import make_cache

pytestmark = pytest.mark.gpu

FLAG_PAGE, FLAG_SEQUENCE, FLAG_FULL = 16, 32, 128


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


PARTS = ("refs", "pages", "length", "k", "v", "k_scale", "v_scale")


def state(cache):
    return [getattr(cache, n).clone() for n in PARTS]


def unchanged(torch, cache, before):
    for name, t in zip(PARTS, before):
        assert torch.equal(getattr(cache, name).view(torch.uint8), t.view(torch.uint8)), name


# --------------------------------------------------------------------------------------------------------------- reorder
def check_reorder(torch, rm, cache, seqs, parents, ws=None):
    before = dict(zip(PARTS, state(cache)))
    refs, table, length = before["refs"].tolist(), before["pages"].tolist(), before["length"].tolist()
    pairs = bp.reorder(refs, table, length, cache.page_tokens, seqs, parents)
    rm.kv_reorder(cache, seqs, parents, workspace=ws)
    if pairs is None:
        assert cache.status_flags() == FLAG_FULL
        cache.status.zero_()
        unchanged(torch, cache, list(before.values()))
        return False
    assert cache.status_flags() == 0
    assert cache.refs.tolist() == refs and cache.pages.tolist() == table and cache.length.tolist() == length
    for name in ("k", "v", "k_scale", "v_scale"):
        want = before[name].clone()
        for a, b in pairs:
            want[:, b] = before[name][:, a]
        assert torch.equal(getattr(cache, name).view(torch.uint8), want.view(torch.uint8)), name
    return True


@pytest.mark.parametrize("layout,page", [("hnd", 16), ("nhd", 32), ("hnd", 128)])
def test_reorder_by_hand(torch, rm, layout, page):
    lengths = [2 * page + 3, page, 0, 1, 3 * page - 1, page + 1]
    for parents in ([0, 1, 2, 3, 4, 5], [1, 0, 3, 2, 5, 4], [0] * 6, [5, 5, 5, 0, 0, 1], [-1, 0, 0, -1, 4, 4], [-1] * 6, [2] * 6, [4, 1, 1, 1, 1, 4]):
        cache = make_cache(torch, rm, lengths, page=page, layout=layout, layers=2, extra=9, slots=8)
        assert check_reorder(torch, rm, cache, [0, 1, 2, 3, 4, 5], parents)
        assert check_reorder(torch, rm, cache, [5, 3, 1], [2, 2, 0])         # again, on some of them, with pages that are shared by now
        assert check_reorder(torch, rm, cache, [7, 4, 0], [1, 1, 1])
        rm.kv_free(cache, list(range(8)))
        assert not cache.refs.any() and cache.status_flags() == 0


def test_reorder_random_walk(torch, rm):
    """Steps of a search: some beams die, some fork, all get new tokens, pages run short."""
    rng = np.random.default_rng(2)
    page, slots = 16, 24
    cache = rm.KVCache(60, page, 2, 16, slots, 8, layers=2)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=gen, device="cuda", dtype=torch.uint8))
    ws = cache.workspace()
    rm.kv_reserve(cache, [0, 8, 16], [40, 23, 50], workspace=ws)
    full = served = 0
    for step in range(80):
        group = int(rng.integers(0, 3)) * 8
        seqs = [int(s) for s in group + rng.permutation(8)]
        length = cache.length.tolist()
        alive = [i for i, s in enumerate(seqs) if length[s]]
        ok = check_reorder(torch, rm, cache, seqs, [int(rng.choice(alive)) if rng.random() < 0.9 else -1 for _ in seqs] if alive else [0] * 8, ws)
        full, served = full + (not ok), served + ok
        length = cache.length.tolist()
        if not any(length[group:group + 8]):
            rm.kv_reserve(cache, [group], [int(rng.integers(1, 60))], workspace=ws)
        grow = [s for s in range(slots) if 0 < length[s] < 100]
        rm.kv_reserve(cache, grow, [length[s] + int(rng.integers(1, 4)) for s in grow], workspace=ws)
        cache.status.zero_()                                                  # (reserve may run out)
        if max(length) > 90:
            rm.kv_free(cache, list(range(group, group + 8)))
            rm.kv_reserve(cache, [group], [int(rng.integers(1, 30))], workspace=ws)
            cache.status.zero_()
    assert served > 40


@pytest.mark.parametrize("n", [33, 1500, 8192])
def test_reorder_many_sequences(torch, rm, n):
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in rng.integers(0, 70, n)]
    cache = make_cache(torch, rm, lengths, page=16, heads=1, dim=16, extra=n)
    assert check_reorder(torch, rm, cache, [int(s) for s in rng.permutation(n)], [int(p) for p in rng.integers(-1, n, n)])


def test_reorder_long_rows(torch, rm):
    cache = make_cache(torch, rm, [16 * 5000 + 1, 3, 16 * 7000 + 5], page=16, heads=1, dim=16)
    assert check_reorder(torch, rm, cache, [0, 1, 2], [2, 0, 2])
    assert check_reorder(torch, rm, cache, [0, 1, 2], [1, 1, 1])


def test_reorder_is_all_or_nothing(torch, rm):
    cache = make_cache(torch, rm, [20, 33, 5], page=16, extra=1, slots=4)
    check_reorder(torch, rm, cache, [0, 1, 2], [0, 0, 0])                     # 1 gives three pages back: two copies fit
    cache = make_cache(torch, rm, [20, 5, 5], page=16, extra=0, slots=6)
    before = state(cache)
    assert not check_reorder(torch, rm, cache, [0, 1, 2, 3, 4, 5], [0, 1, 2, 0, 1, 2])
    for seqs, parents, flag in (([0, 0], [0, 1], FLAG_SEQUENCE), ([0, 6], [0, 0], FLAG_SEQUENCE), ([0, -1], [0, 0], FLAG_SEQUENCE), ([0, 1], [0, 2], FLAG_SEQUENCE),
                                ([0, 1], [-2, 0], FLAG_SEQUENCE)):
        rm.kv_reorder(cache, seqs, parents)
        assert cache.status_flags() == flag
        cache.status.zero_()
        unchanged(torch, cache, before)
    for bad in (99, -1, -7):                                                  # a table entry that is no page
        cache = make_cache(torch, rm, [40, 33], page=16, slots=3, extra=6)
        cache.pages[0, 1] = bad
        before = state(cache)
        rm.kv_reorder(cache, [0, 1, 2], [0, 1, 0])
        assert cache.status_flags() == FLAG_PAGE
        unchanged(torch, cache, before)
    cache = make_cache(torch, rm, [40, 33], page=16, slots=3, extra=6)
    cache.refs[cache.pages[1, 0].item()] = 0                                  # fewer references than holders
    before = state(cache)
    rm.kv_reorder(cache, [0, 1, 2], [0, 0, 0])
    assert cache.status_flags() == FLAG_PAGE
    unchanged(torch, cache, before)
    cache.length[0] = 16 * 900
    before = state(cache)
    cache.status.zero_()
    rm.kv_reorder(cache, [0, 1], [1, 1])
    assert cache.status_flags() == FLAG_SEQUENCE
    unchanged(torch, cache, before)


# ----------------------------------------------------------------------------------------------------------------- evict
def evicted(cache, before, weight, slots, keep, first, recent):
    """Codes, scales and weights [layers, slot -> ...] that the definition gives for the sequences that are cut."""
    page, out = cache.page_tokens, {}
    table, length = before["pages"].cpu().numpy(), before["length"].cpu().numpy()
    host = {n: before[n].cpu().numpy() for n in ("k", "v", "k_scale", "v_scale")}
    w = weight.cpu().numpy()
    for s in slots:
        n = int(length[s])
        if n <= keep:
            continue
        for layer in range(cache.layers):
            for h in range(cache.kv_heads):
                at = bp.kept(w[layer, s, h], n, keep, first, recent)
                ids, inside = table[s, at // page], at % page
                got = [w[layer, s, h, at]]
                for name in ("k", "v"):
                    codes = host[name][layer][ids, h, inside] if cache.layout == "hnd" else host[name][layer][ids, inside, h]
                    got += bp.packed(codes, host[name + "_scale"][layer][ids, h], cache.fmt, page)
                out[layer, s, h] = got
    return out


def check_evict(torch, rm, cache, seqs, keep, first=0, recent=0, weight=None, seed=0, apart=True, served=None, flags=0, ws=None):
    """served: the sequences of the call that are, None: all."""
    if weight is None:
        gen = torch.Generator(device="cuda").manual_seed(seed)
        weight = torch.rand(cache.key_weights().shape, generator=gen, device="cuda")
    served = seqs if served is None else served
    before = dict(zip(PARTS, state(cache)))
    want = evicted(cache, before, weight, served, keep, first, recent)
    kept_weight = weight.clone()
    out = torch.full_like(weight, 7.0) if apart else weight
    assert rm.kv_evict(cache, seqs, weight, keep, first=first, recent=recent, weight_out=out if apart else None, workspace=ws) is out
    assert cache.status_flags() == flags
    cache.status.zero_()
    page, now = cache.page_tokens, -(-keep // cache.page_tokens)
    old_refs, old_table, old_length = (before[n].tolist() for n in ("refs", "pages", "length"))
    cut = [s for s in served if old_length[s] > keep]
    free = iter([p for p, r in enumerate(old_refs) if r == 0])
    refs, table = list(old_refs), [list(r) for r in old_table]
    for s in cut:
        for e in range(-(-old_length[s] // page)):
            if e >= now:
                refs[table[s][e]] -= 1
                table[s][e] = -1
            elif old_refs[table[s][e]] > 1:
                refs[table[s][e]] -= 1
                table[s][e] = next(free)
                refs[table[s][e]] = 1
    assert cache.refs.tolist() == refs and cache.pages.tolist() == table
    assert cache.length.tolist() == [keep if s in cut else n for s, n in enumerate(old_length)]
    expect = {n: before[n].clone().cpu() for n in ("k", "v", "k_scale", "v_scale")}
    weights = (torch.full_like(weight, 7.0) if apart else kept_weight).cpu()
    for (layer, s, h), (w, k, ks, v, vs) in want.items():
        weights[layer, s, h, :keep] = torch.from_numpy(w)
        weights[layer, s, h, keep:old_length[s]] = 0.0
        for e in range(now):
            n = min(page, keep - e * page)
            for name, codes, scales in (("k", k, ks), ("v", v, vs)):
                to = expect[name][layer, table[s][e]]
                (to[h] if cache.layout == "hnd" else to[:, h])[:n] = torch.from_numpy(codes[e * page:e * page + n])
                expect[name + "_scale"][layer, table[s][e], h] = float(scales[e])
    for name, t in expect.items():
        assert torch.equal(getattr(cache, name).cpu().view(torch.uint8), t.view(torch.uint8)), name
    assert torch.equal(out.cpu().view(torch.int32), weights.view(torch.int32))
    if apart:
        assert torch.equal(weight.view(torch.int32), kept_weight.view(torch.int32))


@pytest.mark.parametrize("fmt,layout", [("e4m3", "hnd"), ("int8", "hnd"), ("e4m3", "nhd"), ("int8", "nhd")])
@pytest.mark.parametrize("page,dim,heads", [(16, 64, 3), (32, 128, 2), (128, 256, 1), (64, 96, 2), (16, 16, 5), (16, 208, 2), (128, 128, 1), (32, 240, 1), (64, 48, 2)])
def test_evict(torch, rm, fmt, layout, page, dim, heads):
    for keep, first, recent in ((100, 0, 0), (129, 4, 30), (1, 0, 1), (3 * page, 1, page), (257, 257, 0), (200, 0, 200)):
        cache = make_cache(torch, rm, [700, 0, keep, keep + 1, 90, 301], page=page, heads=heads, dim=dim, fmt=fmt, layout=layout, layers=2, seed=keep)
        check_evict(torch, rm, cache, [0, 1, 2, 3, 4, 5], keep, first, recent, seed=keep, apart=keep != 100)
        check_evict(torch, rm, cache, [5, 0], max(1, keep // 2), 0, min(recent, keep // 4), seed=1)      # and again


@pytest.mark.parametrize("kind", ["zeros", "few", "steps", "signs", "nan", "lowest", "up", "down"])
def test_evict_weights_that_tie(torch, rm, kind):
    cache = make_cache(torch, rm, [1000, 77, 530], page=16, heads=2, dim=32, layers=2)
    w = cache.key_weights()
    gen = torch.Generator(device="cuda").manual_seed(1)
    if kind == "few":
        w.copy_((torch.rand(w.shape, generator=gen, device="cuda") < 0.05).float())
    elif kind == "steps":
        w.copy_(torch.randint(0, 7, w.shape, generator=gen, device="cuda").float())
    elif kind == "signs":
        w.copy_(torch.randint(-2, 3, w.shape, generator=gen, device="cuda").float() * 0.0 + torch.randint(-2, 3, w.shape, generator=gen, device="cuda"))
        w[..., ::3] *= -0.0
    elif kind == "nan":
        w.copy_(torch.randn(w.shape, generator=gen, device="cuda"))
        w[..., ::2] = float("nan")
        w[..., 1::4] = -float("inf")
        w[..., 3::40] = float("inf")
    elif kind == "lowest":
        w.fill_(torch.finfo(torch.float32).min)
        w[..., 5::50] = 1e-42
    elif kind in ("up", "down"):
        w.copy_(torch.arange(w.shape[-1], device="cuda").float().expand(w.shape) * (1e-3 if kind == "up" else -1e-3))
    check_evict(torch, rm, cache, [0, 1, 2], 300, 2, 10, weight=w)
    check_evict(torch, rm, cache, [0, 1, 2], 64, 0, 0, weight=w, apart=False)


def test_evict_any_scales(torch, rm):
    """Scales that are no powers of two, far apart, zero; pages of zeros."""
    for fmt in ("e4m3", "int8"):
        cache = make_cache(torch, rm, [400, 250], page=16, heads=2, dim=32, fmt=fmt, garbage=False)
        rng = np.random.default_rng(3)
        for t in (cache.k_scale, cache.v_scale):
            t.copy_(torch.from_numpy((10.0 ** rng.uniform(-6, 3, size=tuple(t.shape))).astype(np.float32)).cuda())
        cache.k_scale[0, cache.pages[0, 3].item()] = 0.0
        cache.v_scale[0, cache.pages[0, 4].item()] = 2.0 ** -100
        cache.v[0, cache.pages[1, :5].long()] = 0
        check_evict(torch, rm, cache, [0, 1], 120, 0, 20)


@pytest.mark.parametrize("length,keep", [(40000, 3000), (70001, 69000), (3000, 1)])
def test_evict_long_sequences(torch, rm, length, keep):
    cache = make_cache(torch, rm, [length], page=128, heads=1, dim=16)
    check_evict(torch, rm, cache, [0], keep, min(4, keep - 1), min(keep // 2, 500))


def test_evict_shared_pages(torch, rm):
    """Pages that another sequence holds are replaced, for both where both are cut; the other sequence keeps what it reads."""
    cache = make_cache(torch, rm, [300, 200, 0, 0], page=16, heads=2, dim=32, layers=2, extra=60)
    rm.kv_fork(cache, [0, 0], [2, 3])
    other = [cache.k[:, cache.pages[3, :19].long()].clone(), cache.pages[3].clone()]
    check_evict(torch, rm, cache, [0, 2, 1], 150, 0, 40)
    assert torch.equal(cache.k[:, cache.pages[3, :19].long()], other[0]) and torch.equal(cache.pages[3], other[1])
    check_evict(torch, rm, cache, [3, 0], 70, 0, 0)
    rm.kv_free(cache, [0, 1, 2, 3])
    assert not cache.refs.any()


def test_evict_runs_out_in_order(torch, rm):
    cache = make_cache(torch, rm, [160, 160, 160, 0, 0], page=16, extra=16)
    rm.kv_fork(cache, [0, 1], [3, 4])                                         # whole pages: nothing is copied
    check_evict(torch, rm, cache, [0, 1, 2], 144, served=[0, 2], flags=FLAG_FULL)    # nine pages each of sixteen; the third needs none
    check_evict(torch, rm, cache, [1, 4, 0], 100, flags=FLAG_FULL, served=[1, 0])    # the pool as it is now: seven for the first, the second goes without


def test_evict_reports_and_skips(torch, rm):
    cache = make_cache(torch, rm, [160, 160, 160], page=16, slots=6)
    check_evict(torch, rm, cache, [0, 9, 0, -1, 1], 100, served=[0, 1], flags=FLAG_SEQUENCE)
    cache.pages[2, 3] = 999
    check_evict(torch, rm, cache, [2, 0], 50, served=[0], flags=FLAG_PAGE)
    cache.length[2] = -4
    check_evict(torch, rm, cache, [2, 1], 20, served=[1], flags=FLAG_SEQUENCE)


def test_evict_offsets_past_32_bits(torch, rm):
    """A pool of more than 2^32 bytes, the sequence in its last pages."""
    page_bytes = 128 * 8 * 256
    pages = (1 << 32) // page_bytes + 40
    if torch.cuda.mem_get_info()[0] < 5 * pages * page_bytes:
        pytest.skip("not enough memory")
    cache = rm.KVCache(pages, 128, 8, 256, 1, 16)
    small = make_cache(torch, rm, [1500], page=128, heads=8, dim=256, extra=0)
    last = pages - 1 - torch.arange(12, device="cuda", dtype=torch.int32)
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(cache, name)[:, last.long()] = getattr(small, name)[:, small.pages[0, :12].long()]
    cache.pages[0, :12], cache.length[0] = last, 1500
    cache.refs[last.long()] = 1
    weight = torch.rand(cache.key_weights().shape, device="cuda")
    keep = small.key_weights()
    keep[..., :1500] = weight[..., :1500]
    rm.kv_evict(cache, [0], weight, 600, recent=50)
    rm.kv_evict(small, [0], keep, 600, recent=50)
    for name in ("k", "v", "k_scale", "v_scale"):
        got, want = getattr(cache, name)[:, cache.pages[0, :5].long()], getattr(small, name)[:, small.pages[0, :5].long()]
        if name in ("k", "v"):
            got, want = (torch.cat([x[:, :4].reshape(-1), x[:, 4, :, :88].reshape(-1)]) for x in (got, want))
        assert torch.equal(got, want)
    assert torch.equal(weight[..., :600], keep[..., :600]) and cache.status_flags() == 0


def test_bounded_cache_on_streams_and_in_graphs(torch, rm):
    cache = make_cache(torch, rm, [300, 200, 100, 50], page=16, extra=60)
    ws, weight = cache.workspace(), torch.rand(cache.key_weights().shape, device="cuda")
    seqs, parents = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1, 2, 3], [0, 0, 1, 2]))
    start = state(cache)
    def step(**kw):
        rm.kv_reorder(cache, seqs, parents, workspace=ws, **kw)
        rm.kv_evict(cache, seqs, weight, 70, recent=10, workspace=ws, **kw)
    def back():
        for name, t in zip(PARTS, start):
            getattr(cache, name).copy_(t)
    first = weight.clone()
    step()
    want, want_weight = state(cache), weight.clone()
    assert cache.status_flags() == 0
    back(); weight.copy_(first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step(stream=side)
    side.synchronize()
    unchanged(torch, cache, want)
    graph = torch.cuda.CUDAGraph()
    back(); weight.copy_(first)
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        back(); weight.copy_(first)
        graph.replay()
        unchanged(torch, cache, want)
        assert torch.equal(weight, want_weight)


def test_bounded_cache_refusals(torch, rm):
    cache = make_cache(torch, rm, [40, 20], page=16)
    w = cache.key_weights()
    for bad in (dict(weight=w[..., :-1]), dict(weight=w.double()), dict(weight=w.cpu()), dict(weight_out=w[:, :1]), dict(keep=-1), dict(first=-1), dict(recent=-2)):
        with pytest.raises(ValueError):
            rm.kv_evict(cache, [0], **dict(dict(weight=w, keep=10), **bad))
    for bad in (dict(keep=0), dict(first=6, recent=5), dict(seqs=[0, 1, 0])):
        with pytest.raises(rm.RoomieError, match="invalid argument"):
            rm.kv_evict(cache, **dict(dict(seqs=[0], weight=w, keep=10), **bad))
    with pytest.raises(ValueError):
        rm.kv_reorder(cache, [0, 1], [0])
    with pytest.raises(rm.RoomieError, match="invalid argument"):
        rm.kv_reorder(cache, [0, 1, 0], [0, 1, 2])
    with pytest.raises(rm.RoomieError, match="workspace"):
        rm.kv_reorder(cache, [0, 1], [0, 1], workspace=torch.empty(512, dtype=torch.uint8, device="cuda"))
    rm.kv_reorder(cache, [], [])
    rm.kv_evict(cache, [], w, 10)
