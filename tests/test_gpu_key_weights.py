"""The attention weight that cached keys have received, against its definition in 64 bits.

Error bound of one row's share p = exp(x), x = scale q.k - lse (v = 2^-24): x is off by scale (dim + 4) v sum |q k|, by scale 2^-25 max |q| sum |k|
where elements of q below 2^-14 of its largest are rounded, and by 4 v (|scale q.k| + |lse|) from its own arithmetic in powers of two;
exp2 by 2^-22; a sum of n rows by n v of it.  Then the addition to what is there: v."""
import numpy as np
import pytest

from test_gpu_serving import cached, make_cache

pytestmark = pytest.mark.gpu

V = 2.0 ** -24
FLAG_PAGE, FLAG_SEQUENCE = 16, 32


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


def shares(q, k, lse, start, scale, window):
    """One sequence: q [n, q_heads, d], k [length, kv_heads, d], lse [n, q_heads].  (sum, bound) [kv_heads, length]."""
    n, hq, d = q.shape
    length, h, _ = k.shape
    g = hq // h
    pos = start + np.arange(n)[:, None]
    key = np.arange(length)[None, :]
    seen = (key <= pos) & ((key > pos - window) if window else True)
    total, bound = np.zeros((h, length)), np.zeros((h, length))
    for j in range(hq):
        kk = k[:, j // g]
        s = scale * (q[:, j] @ kk.T)
        x = np.where(seen, s - np.where(np.isneginf(lse[:, j]), 0, lse[:, j])[:, None], -np.inf)
        p = np.exp(x)
        off = scale * (d + 4) * V * (np.abs(q[:, j]) @ np.abs(kk).T) + scale * 2.0 ** -25 * np.abs(q[:, j]).max(-1)[:, None] * np.abs(kk).sum(-1)[None, :]
        off = off + 4 * V * (np.abs(s) + np.where(np.isfinite(lse[:, j]), np.abs(lse[:, j]), 0)[:, None]) + 2.0 ** -22 + n * g * V
        total[j // g] += p.sum(0)
        bound[j // g] += (p * np.expm1(off)).sum(0)
    return total, bound


def check(torch, rm, cache, seqs, news, q_heads, dtype="bf16", window=0, scale=None, fresh=False, layer=0, seed=1, view="whole", offsets=True, size=1.0, weight=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    rows, d = sum(news), cache.head_dim
    q = (torch.randn((rows, q_heads, d), generator=gen, device="cuda") * size).to(kind)
    if view == "slice":
        wide = torch.full((rows, q_heads + 2, d), 9.0, dtype=kind, device="cuda")
        wide[:, 1:1 + q_heads] = q
        q = wide[:, 1:1 + q_heads]
    elif view == "odd":
        odd = torch.zeros(rows * q_heads * (d + 1) + 1, dtype=kind, device="cuda")[1:].view(rows, q_heads, d + 1)[..., :d]
        odd.copy_(q)
        q = odd
    offset = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda") if offsets else None
    _, lse = rm.kv_attention(cache, seqs, q, offset, layer=layer, scale=scale, window=window)
    if weight is None:
        weight = torch.rand(cache.key_weights().shape, generator=gen, device="cuda")
    before = weight.clone()
    again = weight.clone()
    assert rm.kv_weights(cache, seqs, q, lse, weight, offset, layer=layer, scale=scale, window=window, fresh=fresh) is weight
    rm.kv_weights(cache, seqs, q, lse, again, offset, layer=layer, scale=scale, window=window, fresh=fresh)
    assert torch.equal(weight.view(torch.int32), again.view(torch.int32))          # the same bits
    want, bound = before.double().cpu().numpy(), np.zeros(tuple(weight.shape))
    at = 0
    for s, n in zip(seqs, news):
        length = int(cache.length[s])
        if n and length:
            got, off = shares(q[at:at + n].double().cpu().numpy(), cached(cache, layer, s, "k"), lse[at:at + n].double().cpu().numpy(), length - n, d ** -0.5 if scale is None else scale, window)
            old = 0 if fresh else max(0, length - n)
            got[:, :old] += want[layer, s, :, :old]
            want[layer, s, :, :length] = got
            bound[layer, s, :, :length] = off + V * np.abs(got) + 1e-37
        at += n
    err = np.abs(weight.double().cpu().numpy() - want)
    assert np.all(err <= bound), (float((err - bound).max()), np.argwhere(err > bound)[:5], int((err > bound).sum()))
    return q, lse, weight


@pytest.mark.parametrize("fmt,layout", [("e4m3", "hnd"), ("int8", "hnd"), ("e4m3", "nhd"), ("int8", "nhd")])
@pytest.mark.parametrize("page,dim", [(16, 64), (32, 128), (64, 256), (128, 96), (16, 16), (64, 80), (32, 176)])
def test_weights_of_single_tokens(torch, rm, fmt, layout, page, dim):
    cache = make_cache(torch, rm, [1, 700, 33, 0, 16, 129], page=page, heads=2, dim=dim, fmt=fmt, layout=layout, layers=2)
    for group, dtype, view in ((1, "bf16", "whole"), (4, "f16", "slice"), (5, "bf16", "odd"), (16, "bf16", "whole"), (20, "f16", "whole")):
        check(torch, rm, cache, [0, 1, 2, 3, 4, 5], [1] * 6, 2 * group, dtype, layer=group % 2, view=view, offsets=group != 4, fresh=group == 5)


@pytest.mark.parametrize("window", [0, 1, 17, 64, 200])
@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("news", [(3, 5, 2, 0, 1), (40, 20, 33, 0, 16), (300, 129, 33, 0, 2), (1, 400, 1, 0, 1)])
def test_weights_of_chunks(torch, rm, window, fresh, news):
    for dim, group, fmt in ((64, 4, "e4m3"), (128, 2, "int8"), (256, 1, "e4m3")):
        cache = make_cache(torch, rm, [500, 400, 33, 20, 16], page=32, heads=2, dim=dim, fmt=fmt)
        check(torch, rm, cache, [0, 1, 2, 3, 4], list(news), 2 * group, window=window, fresh=fresh)


@pytest.mark.parametrize("dim", [64, 128, 256, 96])
@pytest.mark.parametrize("page,layout,fmt", [(16, "hnd", "e4m3"), (128, "nhd", "int8")])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_weights_of_long_chunks(torch, rm, dim, page, layout, fmt, dtype):
    cache = make_cache(torch, rm, [1100, 257, 640, 2], page=page, heads=2, dim=dim, fmt=fmt, layout=layout)
    check(torch, rm, cache, [2, 0, 3, 1], [640, 513, 2, 100], 8, dtype, view="slice", fresh=True)
    check(torch, rm, cache, [1, 0], [257, 40], 2, dtype, view="odd", window=100)


@pytest.mark.parametrize("group", [1, 3, 7, 20, 32, 33, 48, 70])
@pytest.mark.parametrize("view", ["whole", "odd"])
@pytest.mark.parametrize("window", [0, 30])
def test_weights_of_any_group(torch, rm, group, view, window):
    """Blocks of rows hold whole tokens of a group, or a part of a large one."""
    cache = make_cache(torch, rm, [300, 40, 129], page=16, heads=2, dim=64)
    check(torch, rm, cache, [0, 1, 2], [60, 40, 1], 2 * group, "f16", window=window, view=view)


def test_weights_of_broadcast_queries(torch, rm):
    """Strides of zero, of tokens and of heads."""
    cache = make_cache(torch, rm, [200], page=16, heads=2, dim=64)
    q = torch.randn(40, 8, 64, device="cuda").half()
    for view in (q[:1].expand(40, 8, 64), q[:, :1].expand(40, 8, 64)):
        whole = view.contiguous()
        _, lse = rm.kv_attention(cache, [0], whole, [0, 40])
        got, want = cache.key_weights(), cache.key_weights()
        rm.kv_weights(cache, [0], view, lse, got, [0, 40])
        rm.kv_weights(cache, [0], whole, lse, want, [0, 40])
        assert torch.equal(got, want) and float(want.sum()) > 0


@pytest.mark.parametrize("news,count", [(1, 300), (3, 150), (40, 50)])
def test_weights_of_many_sequences(torch, rm, news, count):
    rng = np.random.default_rng(count)
    lengths = [int(x) for x in rng.integers(0, 200, count)]
    cache = make_cache(torch, rm, lengths, page=16, heads=2, dim=64)
    order = [int(s) for s in rng.permutation(count)]
    check(torch, rm, cache, order, [min(int(rng.integers(0, news + 1)), lengths[s]) for s in order], 8)


@pytest.mark.parametrize("seqs,length,new", [(1, 40000, 1), (3, 130, 1), (2, 9000, 40), (1, 3000, 2000)])
def test_weights_of_long_sequences(torch, rm, seqs, length, new):
    cache = make_cache(torch, rm, [length - 7 * i for i in range(seqs)], page=64, heads=1, dim=64)
    check(torch, rm, cache, list(range(seqs)), [new] * seqs, 4, fresh=new > 1)


def test_weights_add_up(torch, rm):
    """Each row gives 1 in all: over a whole prompt token by token, and over the same prompt at once."""
    cache = make_cache(torch, rm, [200], page=16, heads=2, dim=64)
    q, lse, once = check(torch, rm, cache, [0], [200], 8, fresh=True)
    steps = torch.full_like(once, 5.0)
    for n in range(1, 201):                                                    # what is there when a token arrives does not count
        cache.length[0] = n
        rm.kv_weights(cache, [0], q[n - 1:n], lse[n - 1:n], steps)
    for w in (once, steps):
        assert abs(float(w[0, 0, 0, :200].double().sum()) - 800) < 800 * 2e-5 and abs(float(w[0, 0, 1, :200].double().sum()) - 800) < 800 * 2e-5
    assert torch.allclose(once[..., :200], steps[..., :200], rtol=1e-4, atol=1e-6)
    assert steps[..., 200:].eq(5.0).all()


def test_weights_more_rows_than_tokens_and_an_endless_window(torch, rm):
    cache = make_cache(torch, rm, [5, 40, 0], page=16, heads=2, dim=64)
    for news in ([9, 1, 3], [70, 64, 2]):
        for window in (0, 3, (1 << 31) - 1):
            check(torch, rm, cache, [0, 1, 2], news, 4, window=window)


def test_weights_of_extremes(torch, rm):
    """Keys that take everything, scales of any size, large queries."""
    cache = make_cache(torch, rm, [300, 70], page=16, heads=2, dim=64)
    for news in ([1, 1], [30, 20]):
        check(torch, rm, cache, [0, 1], news, 8, size=30.0)
        check(torch, rm, cache, [0, 1], news, 8, "f16", scale=1e-4)
        check(torch, rm, cache, [0, 1], news, 8, scale=2.0)
    cache = make_cache(torch, rm, [300, 70], page=16, heads=2, dim=64, garbage=False)
    rng = np.random.default_rng(0)
    cache.k_scale.copy_(torch.from_numpy((10.0 ** rng.uniform(-8, -1, size=tuple(cache.k_scale.shape))).astype(np.float32)).cuda())
    cache.k_scale[0, cache.pages[0, 2].item()] = 0.0
    cache.k_scale[0, cache.pages[0, 3].item()] = 2.0 ** -100
    for news in ([1, 1], [30, 20]):
        check(torch, rm, cache, [0, 1], news, 8, "f16")


@pytest.mark.parametrize("new", [1, 4, 40, 150])
def test_weights_of_nan(torch, rm, new):
    """A NaN in a query reaches the keys that its row sees, one in a key that key."""
    cache = make_cache(torch, rm, [300], page=16, heads=2, dim=64)
    q, lse, clean = check(torch, rm, cache, [0], [new], 8, window=20)
    bad = q.clone()
    bad[new - 1, 1, 3] = float("nan")                                           # the last row, of the first key head
    weight = torch.zeros_like(clean)
    rm.kv_weights(cache, [0], bad, lse, weight, [0, new], window=20)
    seen = torch.zeros(2, 300, dtype=torch.bool, device="cuda")
    seen[0, 280:] = True
    assert torch.equal(torch.isnan(weight[0, 0, :, :300]), seen)
    cache.k[0, cache.pages[0, 18].item(), 1, 2, 5] = 0x7F                        # key 290 of the second key head
    weight = torch.zeros_like(clean)
    rm.kv_weights(cache, [0], q, lse, weight, [0, new], window=20)
    seen[0], seen[1, 280:] = False, False
    seen[1, 290] = True
    assert torch.equal(torch.isnan(weight[0, 0, :, :300]), seen)


@pytest.mark.parametrize("new", [1, 40])
def test_weights_report_and_skip(torch, rm, new):
    cache = make_cache(torch, rm, [200, 100, 60], page=16, heads=2, dim=64, slots=4)
    q, lse, good = check(torch, rm, cache, [0, 1, 2], [new] * 3, 4, fresh=True, weight=cache.key_weights())
    offset = torch.tensor([0, new, 2 * new, 3 * new], dtype=torch.int32, device="cuda")
    cache.pages[1, 2] = 12345
    weight = cache.key_weights()
    rm.kv_weights(cache, [0, 1, 2], q, lse, weight, offset, fresh=True)
    assert cache.status_flags() == FLAG_PAGE
    want = good.clone()
    want[0, 1, :, 32:48] = 0
    assert torch.equal(weight, want)
    for seqs, off, flag in (([0, 9, -1], offset, FLAG_SEQUENCE), ([0, 1, 2], torch.tensor([0, new, new - 1, 9999], dtype=torch.int32, device="cuda"), FLAG_SEQUENCE)):
        cache.status.zero_()
        weight = cache.key_weights()
        rm.kv_weights(cache, seqs, q, lse, weight, off, fresh=True)
        assert cache.status_flags() & flag
        assert torch.equal(weight[0, 0], good[0, 0]) and not weight[0, 2:].any()
    cache.status.zero_()
    cache.length[2] = -3
    weight = cache.key_weights()
    rm.kv_weights(cache, [2, 0], q[:2 * new], lse[:2 * new], weight, offset[:3], fresh=True)
    assert cache.status_flags() == FLAG_SEQUENCE and not weight[0, 1:].any()


@pytest.mark.parametrize("new", [1, 40])
def test_weights_past_32_bits(torch, rm, new):
    """The last layer's weights start behind 2^32 bytes, its codes too."""
    layers, slots, width = 9, 512, 2048
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    cache = rm.KVCache(8300, 16, 1, 256, slots, width, layers=130)
    small = make_cache(torch, rm, [300], page=16, heads=1, dim=256, extra=0)
    last = 8299 - torch.arange(19, device="cuda", dtype=torch.int32)
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(cache, name)[129, last.long()] = getattr(small, name)[0, small.pages[0, :19].long()]
    cache.pages[511, :19], cache.length[511] = last, 300
    q = torch.randn(new, 4, 256, device="cuda").half()
    _, lse = rm.kv_attention(small, [0], q, [0, new])
    weight, few = cache.key_weights(), small.key_weights()
    assert weight.numel() > 1 << 30
    rm.kv_weights(cache, [511], q, lse, weight, [0, new], layer=129)
    rm.kv_weights(small, [0], q, lse, few, [0, new])
    assert torch.equal(weight[129, 511, 0, :300], few[0, 0, 0, :300]) and float(few.sum()) > 0
    weight[129, 511, 0, :300] = 0
    assert not weight.any()


@pytest.mark.parametrize("new", [1, 40])
def test_weights_on_streams_and_in_graphs(torch, rm, new):
    cache = make_cache(torch, rm, [300, 200], page=16, heads=2, dim=64)
    q, lse, want = check(torch, rm, cache, [0, 1], [new, new], 8, weight=cache.key_weights())
    seqs, offset = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1], [0, new, 2 * new]))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    weight = cache.key_weights()
    side.wait_stream(torch.cuda.current_stream())
    rm.kv_weights(cache, seqs, q, lse, weight, offset, stream=side)
    side.synchronize()
    assert torch.equal(weight, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rm.kv_weights(cache, seqs, q, lse, weight, offset)
    for _ in range(3):
        weight.zero_()
        graph.replay()
        assert torch.equal(weight, want)


def test_weights_refusals(torch, rm):
    cache = make_cache(torch, rm, [40, 20], page=16, heads=2, dim=64)
    q, lse, w = torch.zeros(2, 4, 64, device="cuda").half(), torch.zeros(2, 4, device="cuda"), cache.key_weights()
    for bad in (dict(q=q[..., :32]), dict(q=q[:, :3]), dict(lse=lse[:1]), dict(lse=lse.double()), dict(lse=lse.t().contiguous().t()), dict(weight=w[..., :-1]), dict(weight=w.half()),
                dict(seqs=[0]), dict(q_offset=[0, 1]), dict(q=q.cpu()), dict(lse=lse.cpu()), dict(weight=w.cpu())):
        with pytest.raises(ValueError):
            rm.kv_weights(**dict(dict(cache=cache, seqs=[0, 1], q=q, lse=lse, weight=w), **bad))
    for bad in (dict(q=q.float()), dict(scale=0.0), dict(scale=float("nan")), dict(window=1 << 31), dict(layer=1)):
        with pytest.raises(rm.RoomieError, match="invalid argument"):
            rm.kv_weights(**dict(dict(cache=cache, seqs=[0, 1], q=q, lse=lse, weight=w), **bad))
    rm.kv_weights(cache, [], q[:0], lse[:0], w)
    assert not w.any()
