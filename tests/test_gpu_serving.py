"""The serving operators against their definitions in 64 bits, at the sizes and masks where they can go wrong.

Error bounds (u = half a unit in the last place of the output type: 2^-24, 2^-11, 2^-8 for float32, float16, bfloat16):
rope       each result is two products and a sum of float32 numbers whose cosine and sine are off by at most the phase's
           2^-25 turns (1.9e-7) and two units (2.4e-7): 7e-7 (|x1| + |x2|) amplitude, plus u |y|.
append     a value is turned in float32 and rounded once: half a step of the code, and 7e-7 of the pair.
attention  S: (dim + 4) 2^-24 sum |q k| absolute, as a relative error of p, twice (numerator and total); exp2 on |S| up to 2^7:
           2^-16 and its own 2^-22; p to 11 bits: 2^-11 p |v|; sums 2^-16 p |v|; then u |o|."""
import numpy as np
import pytest

import serving_plain as sp

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
FLAG_PAGE, FLAG_SEQUENCE, FLAG_NONFINITE, FLAG_FULL = 16, 32, 64, 128


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


def dtype_of(torch, name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def host(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------------------------ rope
def rope_bound(x, frequency, interleaved, y, dtype, amplitude):
    half = len(frequency)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    pair = np.abs(x[..., a]) + np.abs(x[..., b])
    bound = U[dtype] * np.abs(y) + 1e-30
    bound[..., a] += 7e-7 * pair * amplitude
    bound[..., b] += 7e-7 * pair * amplitude
    if dtype == "f16":
        bound += 2.0 ** -25                                        # half of float16's least step
    return bound


@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (96, 32), (80, 80), (256, 256), (64, 2), (6, 4), (2, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rope(torch, rm, dim, rot, interleaved, dtype):
    rng = np.random.default_rng(dim * 7 + rot)
    for tokens, heads, view in ((1, 1, "whole"), (33, 3, "whole"), (19, 5, "slice"), (7, 2, "odd")):
        amplitude = 1.0 if tokens > 1 else 1.25
        table = rm.RopeTable(rot, interleaved=interleaved, amplitude=amplitude)
        f = rm.rope_frequencies(rot)
        assert np.array_equal(table.frequency.cpu().numpy().view(np.uint64), f)
        x = torch.from_numpy(rng.normal(size=(tokens, heads, dim))).to(dtype_of(torch, dtype)).cuda()
        if view == "slice":                                        # heads out of a wider projection
            wide = torch.full((tokens, heads + 3, dim), 7.0, dtype=x.dtype, device="cuda")
            wide[:, 2:2 + heads] = x
            x = wide[:, 2:2 + heads]
        elif view == "odd":                                        # rows that start at odd elements
            flat = torch.zeros(tokens * heads * (dim + 1) + 1, dtype=x.dtype, device="cuda")[1:]
            odd = flat.view(tokens, heads, dim + 1)[..., :dim]
            odd.copy_(x)
            x = odd
        pos = rng.integers(0, 1 << 20, tokens)
        pos[0], pos[-1] = 0, (1 << 31) - 1
        p = torch.from_numpy(pos.astype(np.int32)).cuda()
        for inverse in (False, True):
            want = sp.rotate(host(x), pos, f, interleaved, amplitude, inverse)
            bound = rope_bound(host(x), f, interleaved, want, dtype, amplitude)
            got = rm.rope(x, p, table, inverse=inverse)
            assert np.all(np.abs(host(got) - want) <= bound)
            mine = x.clone() if view == "whole" else x
            keep = x.clone()
            assert torch.equal(rm.rope(mine, p, table, inverse=inverse, out=mine), got)       # in place: the same bits
            mine.copy_(keep)


def test_rope_gradient_is_the_transpose_and_the_difference(torch, rm):
    """<rope(x), g> = <x, rope^T(g)>; and a step h along one element changes <rope(x), g> by h times that gradient."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    for interleaved in (False, True):
        table = rm.RopeTable(16, interleaved=interleaved, amplitude=0.75)
        x, g = (torch.randn((5, 3, 24), generator=gen, device="cuda") for _ in range(2))
        p = torch.tensor([0, 1, 77, 4096, 100003], dtype=torch.int32, device="cuda")
        grad = rm.rope(g, p, table, inverse=True)
        dot = lambda a, b: float((a.double() * b.double()).sum())
        # both sums have 360 products of numbers off by at most 7e-7 * 2 * 4 (|x| < 5)
        assert abs(dot(rm.rope(x, p, table), g) - dot(x, grad)) < 360 * 5.6e-6 * 5
        base = rm.rope(x, p, table)
        for at in ((0, 0, 0), (1, 2, 9), (2, 1, 15), (4, 0, 23), (3, 2, 16)):
            h = 0.5
            y = x.clone()
            y[at] += h
            slope = dot(rm.rope(y, p, table).double() - base.double(), g) / h
            assert abs(slope - float(grad[at])) < 2 * 8e-6 * 5 / h


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rope_is_differentiable(torch, rm, interleaved, dtype):
    """The gradient that autograd finds is the turn back, of ordinary, broadcast and strided inputs and of gradients with zero strides; a second
    derivative; and where no gradient can pass the call says so."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    table = rm.RopeTable(32, interleaved=interleaved, amplitude=1.5)
    new = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(dtype_of(torch, dtype))
    p = torch.tensor([3, 0, 70001, 12], dtype=torch.int32, device="cuda")
    for inverse in (False, True):
        x, g = new(4, 5, 48).requires_grad_(), new(4, 5, 48)
        y = rm.rope(x, p, table, inverse=inverse)
        assert torch.equal(y, rm.rope(x.detach(), p, table, inverse=inverse))
        y.backward(g)
        assert torch.equal(x.grad, rm.rope(g, p, table, inverse=not inverse))
    one = new(4, 1, 48).requires_grad_()                               # one head shared by all
    rm.rope(one.expand(4, 5, 48), p, table).backward(g)
    turned = host(rm.rope(g, p, table, inverse=True))
    assert np.all(np.abs(host(one.grad)[:, 0] - turned.sum(1)) <= 6 * U[dtype] * np.abs(turned).sum(1) + 1e-30)
    x = new(4, 5, 48).requires_grad_()
    rm.rope(x, p.tolist(), table).sum().backward()                     # a gradient with strides of zero
    assert torch.equal(x.grad, rm.rope(torch.ones_like(x), p, table, inverse=True))
    w = new(4, 5, 48).requires_grad_()                                 # of (w . turn back g) by g: the turn of w
    grad, = torch.autograd.grad(rm.rope(x, p, table), x, w, create_graph=True)
    again, = torch.autograd.grad(grad, w, g)
    assert torch.equal(again, rm.rope(g, p, table))
    with pytest.raises(ValueError, match="gradient"):
        rm.rope(x, p, table, out=torch.empty_like(g))
    with torch.no_grad():
        assert not rm.rope(x, p, table, out=torch.empty_like(g)).requires_grad and not rm.rope(x, p, table).requires_grad


def test_rope_stretched_frequencies(torch, rm):
    """By parts: slow frequencies divided, fast ones kept, a mix between; without a context all divided."""
    plain, all_slow = rm.rope_frequencies(64), rm.rope_frequencies(64, factor=8.0)
    # both are whole numbers: each is off by half a unit of 2^-64 at most, and by 2^-52 of itself from the double it came from
    assert np.all(np.abs(all_slow.astype(float) - plain.astype(float) / 8) <= 0.5 + 0.5 / 8 + 2.0 ** -51 * all_slow.astype(float))
    parts = rm.rope_frequencies(64, factor=8.0, context=4096, low_turns=1, high_turns=4)
    f = 10000.0 ** (-np.arange(0, 64, 2) / 64) / (2 * np.pi)
    keep = np.clip((f * 4096 - 1) / 3, 0, 1)
    assert np.allclose(parts.astype(float), (f * (keep + (1 - keep) / 8)) * 2.0 ** 64, rtol=1e-12)
    assert 0 < (keep == 1).sum() < 32 and (keep == 0).sum() > 0 and ((keep > 0) & (keep < 1)).any()


def test_rope_refusals(torch, rm):
    x = torch.zeros((4, 2, 16), device="cuda")
    p = torch.zeros(4, dtype=torch.int32, device="cuda")
    table = rm.RopeTable(16)
    with pytest.raises(rm.RoomieError):
        rm.rope_frequencies(7)
    with pytest.raises(rm.RoomieError):
        rm.rope_frequencies(8, factor=0.5)
    with pytest.raises(rm.RoomieError):                                 # wider than the head
        rm.rope(x, p, rm.RopeTable(32))
    with pytest.raises(ValueError):
        rm.rope(x, p[:3], table)
    with pytest.raises(ValueError):
        rm.rope(x, p.long(), table)
    with pytest.raises(ValueError):
        rm.rope(x.double(), p, table)
    with pytest.raises(ValueError):
        rm.rope(x.transpose(1, 2), p, table)
    with pytest.raises(ValueError):
        rm.rope(x, p, table, out=torch.zeros((4, 2, 16), dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        rm.rope(x.cpu(), p, table)
    assert rm.rope(x[:0], p[:0], table).shape == (0, 2, 16)


# ----------------------------------------------------------------------------------------------------------------- cache
def make_cache(torch, rm, lengths, *, page=16, heads=2, dim=64, fmt="e4m3", layout="hnd", layers=1, seed=0, extra=5, shuffle=True,
               slots=None, garbage=True):
    """A cache whose sequences hold random pages; codes everywhere, NaN codes and wild scales where no token is."""
    rng = np.random.default_rng(seed)
    need = sum(-(-n // page) for n in lengths)
    pages = need + extra
    width = max([1] + [-(-n // page) for n in lengths]) + 1
    cache = rm.KVCache(pages, page, heads, dim, slots or len(lengths), width, layers=layers, fmt=fmt, layout=layout)
    order = rng.permutation(pages) if shuffle else np.arange(pages)
    table = np.full((cache.max_seqs, width), -1, np.int32)
    refs = np.zeros(pages, np.int32)
    at = 0
    for s, n in enumerate(lengths):
        for e in range(-(-n // page)):
            table[s, e] = order[at]
            refs[order[at]] = 1
            at += 1
    def codes():
        x = rng.normal(size=(layers, pages, heads, page, dim))
        c = np.clip(np.rint(x * 30), -127, 127).astype(np.int8).view(np.uint8) if fmt == "int8" else \
            torch.from_numpy((x * 90).clip(-448, 448)).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        return c.copy()
    k, v = codes(), codes()
    ks, vs = (2.0 ** rng.integers(-7, -4, size=(layers, pages, heads)).astype(np.float32) for _ in range(2))
    if garbage:                                                     # what no token owns must never be seen
        for s, n in enumerate(lengths):
            if n % page:
                last = table[s, n // page]
                k[:, last, :, n % page:] = 0x7F
                v[:, last, :, n % page:] = 0xFF if fmt == "e4m3" else 0x80
        for p in np.nonzero(refs == 0)[0]:
            k[:, p], v[:, p], ks[:, p], vs[:, p] = 0x7F, 0x7F, np.nan, np.inf
    shape = (lambda c: c) if layout == "hnd" else (lambda c: np.ascontiguousarray(c.transpose(0, 1, 3, 2, 4)))
    for name, a in (("k", shape(k)), ("v", shape(v)), ("k_scale", ks.astype(np.float32)), ("v_scale", vs.astype(np.float32)),
                    ("refs", refs), ("pages", table)):
        getattr(cache, name).copy_(torch.from_numpy(a).cuda())
    cache.length.zero_()
    cache.length[:len(lengths)] = torch.tensor(lengths, dtype=torch.int32)
    return cache


def cached(cache, layer, slot, name):
    """Values [length, heads, dim] of one sequence, float64."""
    codes = getattr(cache, name)[layer].cpu().numpy()
    scale = getattr(cache, name + "_scale")[layer].cpu().numpy().astype(np.float64)
    n = int(cache.length[slot])
    table = cache.pages[slot].cpu().numpy()
    if n == 0:
        return np.zeros((0, cache.kv_heads, cache.head_dim))
    ids = table[:-(-n // cache.page_tokens)]
    x = sp.values(codes[ids], cache.fmt)
    if cache.layout == "hnd":
        x = x.transpose(0, 2, 1, 3)
    return (x * scale[ids][:, None, :, None]).reshape(-1, cache.kv_heads, cache.head_dim)[:n]


# ------------------------------------------------------------------------------------------------------------- attention
def check_attention(torch, rm, cache, seqs, news, q_heads, dtype="bf16", window=0, scale=None, seed=1, offsets=True, view="whole",
                    layer=0, magnitude=1.0, workspace=None):
    rng = np.random.default_rng(seed)
    rows, d = sum(news), cache.head_dim
    q = torch.from_numpy(rng.normal(size=(rows, q_heads, d)) * magnitude).to(dtype_of(torch, dtype)).cuda()
    out = None
    if view == "slice":
        wide = torch.zeros((rows, q_heads + 2, d), dtype=q.dtype, device="cuda")
        wide[:, 1:1 + q_heads] = q
        q = wide[:, 1:1 + q_heads]
        out = torch.zeros((q_heads, rows, d), dtype=q.dtype, device="cuda").transpose(0, 1)
    elif view == "odd":
        flat = torch.zeros(rows * q_heads * (d + 1) + 1, dtype=q.dtype, device="cuda")[1:].view(rows, q_heads, d + 1)
        flat[..., :d] = q
        q = flat[..., :d]
        out = torch.zeros(rows * q_heads * (d + 1) + 1, dtype=q.dtype, device="cuda")[1:].view(rows, q_heads, d + 1)[..., :d]
    offset = torch.tensor(np.concatenate([[0], np.cumsum(news)]).tolist(), dtype=torch.int32, device="cuda") if offsets else None
    ids = torch.tensor(seqs, dtype=torch.int32, device="cuda")
    got, lse = rm.kv_attention(cache, ids, q, offset, layer=layer, window=window, scale=scale, out=out, workspace=workspace)
    scale = d ** -0.5 if scale is None else scale
    gq, go, gl = host(q), host(got), host(lse)
    at = 0
    for s, n in zip(seqs, news):
        k, v = cached(cache, layer, s, "k"), cached(cache, layer, s, "v")
        want, want_lse, weight = sp.attend(gq[at:at + n], k, v, len(k) - n, scale, window)
        empty = np.isinf(want_lse)
        assert np.array_equal(np.isinf(gl[at:at + n]), empty) and np.all(go[at:at + n][empty] == 0)
        g = cache.kv_heads
        mass = scale * np.abs(gq[at:at + n]).max(initial=0) * np.abs(k).sum(-1).max(initial=0) if len(k) else 0.0
        logit = (d + 4) * 2.0 ** -24 * mass + 2.0 ** -22
        top = np.abs(want_lse[~empty]).max(initial=0)
        p_err = 2 * (logit + 2.0 ** -22 + (top + mass) * 2.0 ** -23)
        bound = (2.0 ** -11 + 2.0 ** -16 + p_err) * weight + U[dtype] * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 1e-30)
        err = np.abs(go[at:at + n] - want)
        assert np.all(err <= bound), (s, n, float((err - bound).max()))
        assert np.all(np.abs(gl[at:at + n] - want_lse)[~empty] <= p_err + 2.0 ** -20 * np.maximum(1, top))
        at += n
    assert cache.status_flags() == 0
    return got, lse


LENGTHS = [1, 15, 16, 17, 31, 33, 127, 128, 129, 0, 300, 511]


@pytest.mark.parametrize("fmt,layout", [("e4m3", "hnd"), ("int8", "hnd"), ("e4m3", "nhd"), ("int8", "nhd")])
@pytest.mark.parametrize("page,dim", [(16, 64), (32, 128), (64, 256), (128, 96), (16, 16), (64, 80), (32, 176)])
def test_attention_single_tokens(torch, rm, fmt, layout, page, dim):
    cache = make_cache(torch, rm, LENGTHS, page=page, dim=dim, fmt=fmt, layout=layout, seed=page + dim)
    workspace = cache.workspace()
    for q_heads, dtype, view in ((2, "bf16", "whole"), (8, "f16", "slice"), (14, "bf16", "odd"), (32, "f16", "whole")):
        check_attention(torch, rm, cache, list(range(len(LENGTHS))), [1] * len(LENGTHS), q_heads, dtype, offsets=False, view=view,
                        workspace=workspace)


@pytest.mark.parametrize("window", [0, 1, 17, 64, 200])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attention_chunks(torch, rm, fmt, window):
    """Several new tokens a sequence, none, all of them, and more rows than the sequence has tokens (leading rows see nothing)."""
    lengths = [5, 40, 257, 64, 0, 130, 3, 190]
    news = [5, 3, 129, 64, 2, 0, 7, 1]
    for dim, q_heads, dtype in ((64, 6, "bf16"), (128, 8, "f16")):
        cache = make_cache(torch, rm, lengths, page=32, dim=dim, fmt=fmt, seed=window)
        check_attention(torch, rm, cache, list(range(8)), news, q_heads, dtype, window=window)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("fmt,layout", [("e4m3", "hnd"), ("int8", "nhd")])
def test_attention_long_chunks(torch, rm, dim, page, fmt, layout):
    """Prompt chunks of hundreds of rows, ragged, over longer contexts: whole and cut row and key tiles."""
    lengths, news = [700, 333, 129, 513], [300, 333, 128, 1]
    for q_heads, window, dtype, view in ((2, 0, "bf16", "whole"), (8, 0, "f16", "slice"), (10, 150, "bf16", "odd")):
        cache = make_cache(torch, rm, lengths, page=page, dim=dim, fmt=fmt, layout=layout, seed=page + dim)
        check_attention(torch, rm, cache, [0, 1, 2, 3], news, q_heads, dtype, window=window, view=view)


@pytest.mark.parametrize("dim,kv_heads,group", [(64, 4, 8), (128, 2, 4), (256, 2, 2), (96, 1, 5), (176, 2, 1)])
def test_attention_prompts_repeat_bit_for_bit(torch, rm, dim, kv_heads, group):
    """Ragged prompt chunks whose rows' maxima move while products are on their way (keys of growing size): the values are right, and
    the same call gives the same bits every time."""
    lengths, news = [1527, 900, 271], [413, 547, 188]
    cache = make_cache(torch, rm, lengths, page=32, dim=dim, heads=kv_heads, seed=dim)
    table = cache.pages.cpu().numpy()
    for s, n in enumerate(lengths):                                  # later pages' keys are larger: up to 2^3 of the first ones
        for e in range(-(-n // 32)):
            cache.k_scale[:, table[s, e]] *= 2.0 ** (3 * e * 32 // n)
    ws = cache.workspace()
    first = check_attention(torch, rm, cache, [0, 1, 2], news, kv_heads * group, "bf16", workspace=ws, magnitude=0.5)
    rows = torch.tensor(np.concatenate([[0], np.cumsum(news)]).tolist(), dtype=torch.int32, device="cuda")
    q = torch.from_numpy(np.random.default_rng(1).normal(size=(sum(news), kv_heads * group, dim)) * 0.5).to(torch.bfloat16).cuda()
    for _ in range(40):
        out, lse = rm.kv_attention(cache, [0, 1, 2], q, rows, workspace=ws)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("dim,kv_heads,group", [(64, 4, 8), (128, 4, 8), (256, 3, 4)])
def test_attention_prompts_of_many_short_segments(torch, rm, dim, kv_heads, group):
    """Three or four (sequence, head, tile) segments of one to three steps for each block of the prompt kernel: where one ends and the
    next begins, the next one's logits take the columns that the last products of the one before read."""
    rng = np.random.default_rng(dim)
    lengths = [int(x) for x in rng.integers(20, 300, 160)]
    news = [int(min(n, x)) for n, x in zip(lengths, rng.integers(9, 30, 160))]
    cache = make_cache(torch, rm, lengths, page=16, dim=dim, heads=kv_heads, seed=dim)
    ws = cache.workspace()
    first = check_attention(torch, rm, cache, list(range(160)), news, kv_heads * group, "bf16", workspace=ws)
    rows = torch.tensor(np.concatenate([[0], np.cumsum(news)]).tolist(), dtype=torch.int32, device="cuda")
    q = torch.from_numpy(np.random.default_rng(1).normal(size=(sum(news), kv_heads * group, dim))).to(torch.bfloat16).cuda()
    ids = torch.arange(160, dtype=torch.int32, device="cuda")
    for _ in range(40):
        out, lse = rm.kv_attention(cache, ids, q, rows, workspace=ws)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


def test_attention_split_key_axis_and_order(torch, rm):
    """Few rows over long contexts: the key axis is split over blocks and joined; the same call gives the same bits, and a batch's
    result does not depend on what was in the workspace's sums."""
    lengths = [9001, 4100, 77]
    cache = make_cache(torch, rm, lengths, page=64, dim=128, heads=1, seed=5)
    ws = cache.workspace()
    a = check_attention(torch, rm, cache, [0, 1, 2], [1, 1, 1], 4, "f16", workspace=ws)
    for _ in range(3):
        b = check_attention(torch, rm, cache, [0, 1, 2], [1, 1, 1], 4, "f16", workspace=ws)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check_attention(torch, rm, cache, [2, 0], [1, 1], 16, "bf16", workspace=ws)          # table rows in another order
    check_attention(torch, rm, cache, [1, 0], [3, 2], 4, "bf16", workspace=ws)


@pytest.mark.parametrize("most_new,count", [(1, 300), (3, 150), (40, 50)])
def test_attention_many_sequences(torch, rm, most_new, count):
    """More sequences than a block has threads (or warps), of very different lengths, some empty, some without new rows."""
    rng = np.random.default_rng(count)
    lengths = [int(x) for x in np.where(rng.random(count) < 0.1, 0, np.exp(rng.uniform(0, np.log(900), count)).astype(int))]
    news = [1] * count if most_new == 1 else [int(x) for x in rng.integers(0, most_new + 1, count)]
    cache = make_cache(torch, rm, lengths, page=16, dim=64, heads=1, seed=count)
    ws = cache.workspace()
    order = [int(s) for s in rng.permutation(count)]
    for _ in range(2):
        check_attention(torch, rm, cache, order, [news[s] for s in order], 4, "f16", workspace=ws, offsets=most_new > 1)


@pytest.mark.parametrize("seqs,length", [(1, 40000), (1, 700), (2, 130), (7, 2600), (40, 390)])
def test_attention_cuts_of_the_key_axis(torch, rm, seqs, length):
    """Items left whole, cut into equal parts, cut at any unit and joined in one and in two levels."""
    cache = make_cache(torch, rm, [max(1, length - 37 * s) for s in range(seqs)], page=64, dim=128, heads=1, seed=seqs)
    ws = cache.workspace()
    for q_heads in (8, 16):
        for window in (0, length // 2):
            check_attention(torch, rm, cache, list(range(seqs)), [1] * seqs, q_heads, "f16", workspace=ws, window=window)


def test_append_many_sequences(torch, rm):
    """More sequences than a block has threads; some bring nothing."""
    rng = np.random.default_rng(8)
    count = 700
    lengths = [int(x) for x in rng.integers(1, 40, count)]
    news = [int(min(n, x)) for n, x in zip(lengths, rng.integers(0, 4, count))]
    cache = make_cache(torch, rm, lengths, page=16, dim=16, heads=1, seed=3, garbage=False)
    check_append(torch, rm, cache, list(range(count)), news, rope=rm.RopeTable(16), q_heads=2)
    assert cache.status_flags() == 0


def test_append_many_queries(torch, rm):
    """Enough query bytes for a launch of their own, in place and not, rows of no sequence passed on."""
    cache = make_cache(torch, rm, [1500, 700], page=64, dim=128, heads=2, seed=6, garbage=False)
    check_append(torch, rm, cache, [0, 1], [1400, 650], rope=rm.RopeTable(128), q_heads=16)
    table, ids = rm.RopeTable(128, amplitude=2.0), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    k, q = torch.randn((2060, 2, 128), device="cuda").half(), torch.randn((2060, 16, 128), device="cuda").half()
    rows = torch.tensor([5, 1400, 2050], dtype=torch.int32, device="cuda")                # five rows before, ten behind
    want = rm.kv_append(cache, ids, k, k, rows, rope=table, q=q)
    assert torch.equal(want[:5], q[:5]) and torch.equal(want[2050:], q[2050:]) and not torch.equal(want[5], q[5])
    assert rm.kv_append(cache, ids, k, k, rows, rope=table, q=q, q_out=q) is q and torch.equal(q, want)


def test_append_without_rope_fills_q_out(torch, rm):
    """Where nothing turns the queries, q_out is their copy; without q there is nothing to write."""
    cache = make_cache(torch, rm, [20, 30], page=16, dim=32, garbage=False)
    k, q = torch.randn((2, 2, 32), device="cuda").half(), torch.randn((2, 4, 32), device="cuda").half()
    assert rm.kv_append(cache, [0, 1], k, k, q=q) is q and rm.kv_append(cache, [0, 1], k, k) is None
    wide = torch.zeros((2, 6, 32), device="cuda").half()
    out = wide[:, 1:5]
    assert rm.kv_append(cache, [0, 1], k, k, q=q, q_out=out) is out and torch.equal(out, q) and not wide[:, 0].any() and not wide[:, 5].any()
    assert rm.kv_append(cache, [0, 1], k, k, q=q, q_out=q) is q and torch.equal(out, q)
    for bad in (dict(q_out=out), dict(q=q, q_out=out[:1]), dict(q=q, q_out=out.float()), dict(q=q[:1], q_out=out[:1])):
        with pytest.raises(ValueError):
            rm.kv_append(cache, [0, 1], k, k, **bad)


def test_append_is_one_launch(torch, rm):
    """However many queries there are."""
    table = rm.RopeTable(128)
    for rows in (2, 2000):
        cache = make_cache(torch, rm, [rows // 2, rows // 2], page=64, dim=128, heads=2, garbage=False)
        k, q = torch.randn((rows, 2, 128), device="cuda").half(), torch.randn((rows, 16, 128), device="cuda").half()
        with rm.record_launches() as launches:
            rm.kv_append(cache, [0, 1], k, k, [0, rows // 2, rows], rope=table, q=q)
        assert [r["name"] for r in launches] == ["kv_append"]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("turned", [64, 6])
def test_append_passes_rows_of_no_sequence_on(torch, rm, interleaved, turned):
    """Bit for bit, infinities, NaN and negative zeros too."""
    dim = 64
    cache = make_cache(torch, rm, [20], page=16, dim=dim, heads=1, seed=2, garbage=False)
    table, ids = rm.RopeTable(turned, interleaved=interleaved), torch.tensor([0], dtype=torch.int32, device="cuda")
    k, q = torch.ones((6, 1, dim), device="cuda").half(), torch.randn((6, 4, dim), device="cuda").half()
    q[0, :, ::3], q[5, :, 1::3], q[5, 0, 0], q[0, 1, 2] = float("inf"), -float("inf"), float("nan"), -0.0
    got = rm.kv_append(cache, ids, k, k, torch.tensor([1, 4], dtype=torch.int32, device="cuda"), rope=table, q=q)
    for row in (0, 4, 5):
        assert torch.equal(got[row].view(torch.int16), q[row].view(torch.int16))
    assert torch.isfinite(got[1:4]).all() and cache.status_flags() == 0


def test_attention_extremes(torch, rm):
    """Large and tiny queries (float16 operands are normalised a row), peaked and flat softmax, zero queries, a given scale."""
    cache = make_cache(torch, rm, [200, 90], page=32, dim=64, seed=9)
    for magnitude, scale in ((1e4, 1e-5), (1e-6, 1e5), (3.0, None), (0.0, None), (1e30, 1e-31)):
        check_attention(torch, rm, cache, [0, 1], [1, 1], 4, "bf16", magnitude=magnitude, scale=scale)
    # one row of a query infinite: that row alone is lost
    q = torch.ones((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    q[0, 1, 3] = float("inf")
    out, _ = rm.kv_attention(cache, [0, 1], q)
    assert not torch.isfinite(out[0, 1]).any() and torch.isfinite(out[0, [0, 2, 3]]).all() and torch.isfinite(out[1]).all()


def test_attention_any_scales_and_layers(torch, rm):
    """Scales that are no powers of two and spread over orders of magnitude; a layer other than the first; strided pools."""
    cache = make_cache(torch, rm, [170, 45], page=16, dim=64, layers=3, seed=11, garbage=False)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(torch.rand(t.shape, generator=gen, device="cuda") * 0.03 * 10.0 ** torch.randint(-3, 1, t.shape, generator=gen, device="cuda"))
    for layer in (0, 2):
        check_attention(torch, rm, cache, [0, 1], [1, 1], 4, "f16", layer=layer)
    both = torch.zeros((3, cache.num_pages, 2) + tuple(cache.k.shape[2:]), dtype=torch.uint8, device="cuda")
    both[:, :, 0], both[:, :, 1] = cache.k, cache.v                     # keys and values of a page side by side
    strided = rm.KVCache.from_tensors(both[:, :, 0], both[:, :, 1], cache.k_scale, cache.v_scale, cache.refs, cache.pages, cache.length)
    check_attention(torch, rm, strided, [0, 1], [2, 1], 4, "f16", layer=2)


def test_attention_offsets_past_32_bits(torch, rm):
    """A pool of more than 2^32 bytes of keys: pages near its end are found."""
    page, heads, dim = 128, 8, 128
    num = (1 << 32) // (page * heads * dim) + 64
    if torch.cuda.mem_get_info()[0] < 3 * (1 << 32):
        pytest.skip("needs 13 GB of device memory")
    k = torch.zeros((1, num, heads, page, dim), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    small = make_cache(torch, rm, [250, 100], page=page, heads=heads, dim=dim, seed=2, extra=0, shuffle=False)
    first = num - small.num_pages
    k[:, first:], v[:, first:] = small.k, small.v
    ks, vs = (torch.ones((1, num, heads), device="cuda") for _ in range(2))
    ks[:, first:], vs[:, first:] = small.k_scale, small.v_scale
    refs = torch.zeros(num, dtype=torch.int32, device="cuda")
    refs[first:] = small.refs
    table = torch.where(small.pages >= 0, small.pages + first, small.pages)
    big = rm.KVCache.from_tensors(k, v, ks, vs, refs, table, small.length)
    q = torch.randn((2, 16, dim), device="cuda").to(torch.bfloat16)
    want, got = rm.kv_attention(small, [0, 1], q), rm.kv_attention(big, [0, 1], q)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    rows = torch.tensor([0, 120, 200], dtype=torch.int32, device="cuda")
    q = torch.randn((200, 16, dim), device="cuda").to(torch.bfloat16)
    want, got = (rm.kv_attention(c, [0, 1], q, rows) for c in (small, big))
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    ws = big.workspace()
    rm.kv_copy(big, [first], big, [first - 1])
    assert torch.equal(big.k[0, first - 1], small.k[0, 0]) and torch.equal(big.v[0, first - 1], small.v[0, 0])
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    rm.kv_compact(big, used_out=used, workspace=ws)
    assert int(used) == small.num_pages and torch.equal(big.k[:, :small.num_pages], small.k) and big.status_flags() == 0


@pytest.mark.parametrize("page,dim,layout", [(16, 64, "hnd"), (16, 128, "nhd"), (32, 256, "hnd"), (64, 128, "hnd"), (128, 64, "nhd")])
@pytest.mark.parametrize("news", [(1, 1, 1), (3, 5, 2), (547, 70, 129)])
def test_attention_reads_nothing_before_the_windows(torch, rm, page, dim, layout, news):
    """What lies before every row's window may be anything: NaN codes, pages given up (-1), NaN and infinite scales of the pages before.
    The results are those of the whole cache, bit for bit, and nothing is reported."""
    lengths, window = [900, 333, 701], 150
    cache = make_cache(torch, rm, lengths, page=page, dim=dim, layout=layout, seed=page + dim)
    ids = torch.arange(3, dtype=torch.int32, device="cuda")
    rows = torch.tensor(np.concatenate([[0], np.cumsum(news)]).tolist(), dtype=torch.int32, device="cuda")
    q = torch.from_numpy(np.random.default_rng(2).normal(size=(sum(news), 8, dim))).to(torch.bfloat16).cuda()
    ws = cache.workspace()
    check_attention(torch, rm, cache, [0, 1, 2], list(news), 8, "bf16", window=window, workspace=ws)
    want, want_lse = rm.kv_attention(cache, ids, q, rows, window=window, workspace=ws)
    table = cache.pages.cpu().numpy()
    for s, (n, new) in enumerate(zip(lengths, news)):
        first = max(0, n - new - window + 1)                           # the first key that the first row sees
        for e in range(-(-first // page)):
            ends = min(first - e * page, page)                         # keys of this page before it
            at = int(table[s, e])
            for codes, nan in ((cache.k, 0x7F), (cache.v, 0xFF)):
                (codes[0, at, :, :ends] if layout == "hnd" else codes[0, at, :ends]).fill_(nan)
            if ends == page and e % 3 and (e + 1) * page + page <= first:
                cache.k_scale[0, at], cache.v_scale[0, at] = (float("nan"), float("inf")) if e % 3 == 1 else (float("-inf"), float("nan"))
            elif ends == page:                                         # every third, and the last one
                cache.pages[s, e] = -1
    got, lse = rm.kv_attention(cache, ids, q, rows, window=window, workspace=ws)
    assert cache.status_flags() == 0
    assert torch.equal(got, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("page", [16, 128])
def test_attention_reads_nothing_that_no_row_of_a_tile_sees(torch, rm, page):
    """A NaN in the last token's value reaches rows of that token's tile only: the first 512 rows end before it, in the same 128 keys."""
    cache = make_cache(torch, rm, [880], page=page, dim=128, heads=1, seed=4)
    rows = torch.tensor([0, 530], dtype=torch.int32, device="cuda")
    q = torch.randn((530, 1, 128), device="cuda").to(torch.bfloat16)
    want, want_lse = rm.kv_attention(cache, [0], q, rows)
    cache.v[0, int(cache.pages[0, 879 // page]), 0, 879 % page] = 0x7F
    got, lse = rm.kv_attention(cache, [0], q, rows)
    assert torch.equal(got[:512], want[:512]) and torch.equal(lse[:512], want_lse[:512]) and torch.isnan(got[529]).all()


def flat_cache(torch, rm, lengths, *, page=16, dim=64, heads=1, fmt="e4m3", value_scales=(1.0,), seed=0):
    """Keys of zeros, so that all logits are equal; the value scales of a sequence's pages in turn, for each head another first."""
    cache = make_cache(torch, rm, lengths, page=page, dim=dim, heads=heads, fmt=fmt, seed=seed)
    cache.k.zero_()
    cache.k_scale.fill_(1.0)
    table = cache.pages.cpu().numpy()
    for s, n in enumerate(lengths):
        for e in range(-(-n // page)):
            for h in range(heads):
                cache.v_scale[0, int(table[s, e]), h] = value_scales[(e + h) % len(value_scales)]
    return cache


@pytest.mark.parametrize("at", [0, 31, 700, 1899])
@pytest.mark.parametrize("news", [1, 3, 40])
@pytest.mark.parametrize("dtype,fmt", [("f16", "e4m3"), ("bf16", "int8")])
def test_attention_one_leading_key_and_a_flat_tail(torch, rm, at, news, dtype, fmt):
    """One key whose weight is 2^19.4 times each other's, with a value of nothing: the result is the sum of the many small weights, each of
    them to 11 bits all the same.  Work enough (64 sequences, on the same pages) that a key axis is not cut."""
    length, seqs, heads, dim = 2048, 64, 8, 64
    cache = flat_cache(torch, rm, [length] + [0] * (seqs - 1), page=64, dim=dim, heads=heads, fmt=fmt, value_scales=(0.0107,), seed=3)
    cache.pages[1:], cache.length[1:] = cache.pages[0].clone(), length
    cache.v.bitwise_and_(0x7F)                                          # no sums that cancel
    cache.v.masked_fill_(cache.v == 0x7F, 0x40)
    p = int(cache.pages[0, at // 64])
    cache.k[0, p, :, at % 64], cache.v[0, p, :, at % 64] = 0x38 if fmt == "e4m3" else 1, 0        # 1 in each dimension
    q = torch.full((seqs * news, 2 * heads, dim), 19.4 * float(np.log(2.0)) / dim, device="cuda").to(dtype_of(torch, dtype))
    rows = torch.arange(0, seqs * news + 1, news, dtype=torch.int32, device="cuda")
    got, lse = rm.kv_attention(cache, torch.arange(seqs, dtype=torch.int32, device="cuda"), q, rows, scale=1.0)
    k, v = cached(cache, 0, 0, "k"), cached(cache, 0, 0, "v")
    for t in sorted({0, news // 2, news - 1}):
        want, want_lse, weight = sp.attend(host(q[t:t + 1]), k, v, length - news + t, 1.0, 0)
        # weights to 11 bits, their sums, and the largest logit (13.4; 68 2^-24 of it each) as in the head of this file
        p_err = 2 * (68 * 2.0 ** -24 * 13.5 + 2.0 ** -22 + 14 * 2.0 ** -23)
        bound = (2.0 ** -11 + 2.0 ** -16 + p_err) * weight + U[dtype] * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0)
        for s in (0, 5, seqs - 1):
            assert np.all(np.abs(host(got[s * news + t]) - want[0]) <= bound[0])
            assert np.all(np.abs(host(lse[s * news + t]) - want_lse[0]) <= p_err + 2.0 ** -20 * 14)


@pytest.mark.parametrize("at", [1867, 1899, 1919])
@pytest.mark.parametrize("news", [1, 40])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attention_a_key_that_leads_late(torch, rm, at, news, fmt):
    """The maximum moves by 2^28 and more at once, in a step's first and later keys: weights that are already taken move with it."""
    length, seqs, heads, dim = 2048, 64, 8, 64
    cache = flat_cache(torch, rm, [length] + [0] * (seqs - 1), page=64, dim=dim, heads=heads, fmt=fmt, value_scales=(2.0 ** -6,), seed=3)
    cache.pages[1:], cache.length[1:] = cache.pages[0].clone(), length
    cache.k_scale.fill_(1.0 if fmt == "e4m3" else 0.125)
    low, middle, top = (0, 0x2C, 0x3B) if fmt == "e4m3" else (0, 3, 11)                            # 0, 0.375 and 1.375
    half = [int(p) for p in cache.pages[0, :length // 64]]
    cache.k.fill_(middle)
    cache.k[0, half[0], :, :32] = low                                   # what the first keys set stays, 2^7.5 are not enough to move it
    cache.v.zero_()
    where, inside = half[at // 64], at % 64
    cache.v[0, where, :, :] = 0x38 if fmt == "e4m3" else 1              # only the keys around the leading one have a value, it has none
    cache.k[0, where, :, inside], cache.v[0, where, :, inside] = top, 0
    q = torch.full((seqs * news, 2 * heads, dim), 20 * float(np.log(2.0)) / dim, device="cuda").to(torch.bfloat16)
    rows = torch.arange(0, seqs * news + 1, news, dtype=torch.int32, device="cuda")
    got, lse = rm.kv_attention(cache, torch.arange(seqs, dtype=torch.int32, device="cuda"), q, rows, scale=1.0)
    k, v = cached(cache, 0, 0, "k"), cached(cache, 0, 0, "v")
    for t in sorted({0, news - 1}):
        want, want_lse, weight = sp.attend(host(q[t:t + 1]), k, v, length - news + t, 1.0, 0)
        p_err = 2 * (68 * 2.0 ** -24 * 20 + 2.0 ** -22 + 20 * 2.0 ** -23)             # as in the head of this file: the largest logit is 19.1
        bound = (2.0 ** -11 + 2.0 ** -16 + p_err) * weight + U["bf16"] * np.abs(want) + 1e-30
        for s in (0, seqs - 1):
            assert np.all(np.abs(host(got[s * news + t]) - want[0]) <= bound[0])
            assert np.all(np.abs(host(lse[s * news + t]) - want_lse[0]) <= p_err + 2.0 ** -20 * 20)


def check_scaled(torch, rm, cache, seqs, news, q_heads, window=0, workspace=None):
    """As check_attention, with what lies under a weight's 11 bits: 2^-32 of the row's largest weight (probability times value scale) for
    each key, times its code.  Where page scales differ by 2^20 and more that is what a small result beside large ones is left with."""
    rng = np.random.default_rng(1)
    rows, d = sum(news), cache.head_dim
    q = torch.from_numpy(rng.normal(size=(rows, q_heads, d))).to(torch.bfloat16).cuda()
    offset = torch.tensor(np.concatenate([[0], np.cumsum(news)]).tolist(), dtype=torch.int32, device="cuda")
    got, lse = rm.kv_attention(cache, torch.tensor(seqs, dtype=torch.int32, device="cuda"), q, offset, window=window, workspace=workspace)
    gq, go, gl, group, scale = host(q), host(got), host(lse), q_heads // cache.kv_heads, d ** -0.5
    at = 0
    for s, n in zip(seqs, news):
        k, v = cached(cache, 0, s, "k"), cached(cache, 0, s, "v")
        ids = cache.pages[s].cpu().numpy()[:-(-len(k) // cache.page_tokens)]
        page_scale = np.maximum(cache.v_scale[0].cpu().numpy().astype(np.float64)[ids], 2.0 ** -100)
        vs = np.repeat(page_scale, cache.page_tokens, 0)[:len(k)]                                    # [length, kv_heads]
        codes = np.abs(v) / vs[..., None]
        want, want_lse, weight = sp.attend(gq[at:at + n], k, v, len(k) - n, scale, window)
        mass = scale * np.abs(gq[at:at + n]).max() * np.abs(k).sum(-1).max()
        p_err = 2 * ((d + 4) * 2.0 ** -24 * mass + 2.0 ** -22 + 2.0 ** -22 + (np.abs(want_lse).max() + mass) * 2.0 ** -23)
        for t in range(n):
            pos = len(k) - n + t
            lo, hi = max(0, pos - window + 1) if window else 0, pos + 1
            for j in range(q_heads):
                g = j // group
                p = np.exp(scale * (k[lo:hi, g] @ gq[at + t, j]) - want_lse[t, j])
                floor = 2.0 ** -32 * (p * vs[lo:hi, g]).max() * codes[lo:hi, g].sum(0)
                bound = (2.0 ** -11 + 2.0 ** -16 + p_err) * weight[t, j] + floor + U["bf16"] * np.abs(want[t, j]) + 1e-30
                # 127 * 2^122 is past float32: where the values' magnitudes add up to its end, infinity is right as well
                past = np.maximum(np.abs(want[t, j]), weight[t, j]) + bound > 3.3895e38
                assert np.all((np.abs(go[at + t, j] - want[t, j]) <= bound) | (past & (go[at + t, j] * np.sign(want[t, j]) > 3.3e38))), (s, t, j)
        assert np.all(np.abs(gl[at:at + n] - want_lse) <= p_err + 2.0 ** -20 * np.maximum(1, np.abs(want_lse).max()))
        at += n
    assert cache.status_flags() == 0
    return got, lse


@pytest.mark.parametrize("scales", [(2.0 ** 30, 2.0 ** -100), (2.0 ** -100, 1.0, 0.0, 2.0 ** 30), (0.0, 0.0, 0.0, 2.0 ** -6), (2.0 ** 122, 0.01, 2.0 ** -100),
                                    (0.0, 2.0 ** 122), (2.0 ** -100,), (3.0e-31, 7.0e-20, 5.0e-3, 11.0, 6.0e25), (2.0 ** 127,), (1.5 * 2.0 ** 126, 1.0)])
@pytest.mark.parametrize("news", [(1, 1, 1), (2, 5, 3), (70, 45, 129)])
@pytest.mark.parametrize("fmt,dim", [("e4m3", 128), ("int8", 64), ("e4m3", 256)])
def test_attention_of_widely_different_value_scales(torch, rm, scales, news, fmt, dim):
    """Every key counts in the softmax total, whatever its page's value scale is: pages of zeros (append gives them 2^-100) and scale 0
    beside large ones, equal and different logits."""
    lengths = [2300, 150, 400]
    cache = flat_cache(torch, rm, lengths, dim=dim, heads=2, fmt=fmt, value_scales=scales, seed=dim)
    if max(scales) >= 2.0 ** 126:                                       # values stay within float32
        cache.v.bitwise_and_(0x83 if fmt == "int8" else 0x9F)
        cache.v.masked_fill_(cache.v == (0x80 if fmt == "e4m3" else 0x83), 0)
        if fmt == "int8":
            cache.v.bitwise_and_(0x01)
    check_scaled(torch, rm, cache, [0, 1, 2], list(news), 4)
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache.k.copy_(torch.randint(0, 0x38 if fmt == "e4m3" else 40, cache.k.shape, generator=gen, device="cuda", dtype=torch.uint8))
    check_scaled(torch, rm, cache, [0, 1, 2], list(news), 4)
    check_scaled(torch, rm, cache, [2, 0], [news[2], news[0]], 4, window=333)
    ws = cache.workspace()                                              # the same bits again
    rows = torch.tensor([0, news[1], news[1] + news[0]], dtype=torch.int32, device="cuda")
    q = torch.randn((news[1] + news[0], 16, dim), generator=gen, device="cuda").to(torch.bfloat16)
    a, b = (rm.kv_attention(cache, [1, 0], q, rows, workspace=ws) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("most", [(1 << 31) - 1, (1 << 31) - 100, 1 << 30])
@pytest.mark.parametrize("idle", [0, 40])
def test_attention_more_rows_than_tokens_and_an_endless_window(torch, rm, most, idle):
    """A window as wide as its type beside rows that lie before the sequence: as without a window, in both kernels (idle sequences decide
    which one runs)."""
    lengths, news = [200, 450] + [5] * idle, [210, 453] + [0] * idle
    cache = make_cache(torch, rm, lengths, page=16, dim=64, heads=1, seed=7)
    order = list(range(2 + idle))
    want = check_attention(torch, rm, cache, order, news, 1, "bf16")
    got = check_attention(torch, rm, cache, order, news, 1, "bf16", window=most)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("news", [1, 4, 40, 300])
def test_attention_of_a_nan_query_is_nan(torch, rm, news):
    """One query head of one row is NaN: that row is NaN, whether its keys are cut into parts or not, and the others are right (not the same
    bits: when the reference of a row's weights moves depends on the rows beside it)."""
    gen = torch.Generator(device="cuda").manual_seed(news)
    for length in (330, 9000):
        cache = make_cache(torch, rm, [length], page=64, dim=128, heads=1, seed=8)
        rows = torch.tensor([0, news], dtype=torch.int32, device="cuda")
        q = torch.randn((news, 2, 128), generator=gen, device="cuda").to(torch.bfloat16)
        gq, k, v = host(q), cached(cache, 0, 0, "k"), cached(cache, 0, 0, "v")
        want, want_lse, weight = sp.attend(gq, k, v, length - news, 128 ** -0.5, 0)
        q[news // 2, 1, 5] = float("nan")
        got, lse = (host(t) for t in rm.kv_attention(cache, [0], q, rows))
        lost = np.zeros((news, 2), bool)
        lost[news // 2, 1] = True
        assert np.isnan(got[lost]).all() and np.isnan(lse[lost]).all()
        mass = 128 ** -0.5 * np.abs(gq).max() * np.abs(k).sum(-1).max()                               # as in check_attention
        p_err = 2 * (132 * 2.0 ** -24 * mass + 2.0 ** -22 + 2.0 ** -22 + (np.abs(want_lse).max() + mass) * 2.0 ** -23)
        bound = (2.0 ** -11 + 2.0 ** -16 + p_err) * weight + U["bf16"] * np.abs(want) + 1e-30
        assert np.all(np.abs(got - want)[~lost] <= bound[~lost])
        assert np.all(np.abs(lse - want_lse)[~lost] <= p_err + 2.0 ** -20 * np.maximum(1, np.abs(want_lse).max()))


def test_attention_bad_tables_are_reported(torch, rm):
    """Page ids, lengths and offsets that do not exist set status bits and read nothing."""
    def fresh():
        return make_cache(torch, rm, [60, 40, 20], page=16, dim=64)
    q = torch.randn((3, 2, 64), device="cuda").to(torch.bfloat16)
    cache = fresh()
    want = rm.kv_attention(cache, [0, 1, 2], q)[0]
    for entry in (-1, 10 ** 6, cache.num_pages):
        cache = fresh()
        cache.pages[1, 0] = entry
        out, _ = rm.kv_attention(cache, [0, 1, 2], q)
        assert cache.status_flags() == FLAG_PAGE and torch.equal(out[[0, 2]], want[[0, 2]]) and torch.isfinite(out).all()
    for slot, length in ((1, 10 ** 6), (1, -5)):
        cache = fresh()
        cache.length[slot] = length
        out, lse = rm.kv_attention(cache, [0, 1, 2], q)
        assert cache.status_flags() == FLAG_SEQUENCE and torch.equal(out[[0, 2]], want[[0, 2]]) and (out[1] == 0).all()
    cache = fresh()
    out, _ = rm.kv_attention(cache, [0, 9, 2], q)
    assert cache.status_flags() == FLAG_SEQUENCE and torch.equal(out[[0, 2]], want[[0, 2]])
    with pytest.raises(rm.RoomieError, match="KV_SEQUENCE"):
        cache.check()
    cache = fresh()
    rm.kv_attention(cache, [0, 1, 2], q, torch.tensor([0, 2, 1, 9], dtype=torch.int32, device="cuda"))
    assert cache.status_flags() == FLAG_SEQUENCE


def test_attention_refusals(torch, rm):
    cache = make_cache(torch, rm, [60, 40], page=16, dim=64)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q=q[:, :3]), dict(q=q[..., :32]), dict(q=q[:1]), dict(q_offset=[0, 1]), dict(lse=torch.zeros(2, device="cuda")),
                dict(out=q.half())):
        with pytest.raises(ValueError):
            rm.kv_attention(cache, [0, 1], **dict(dict(q=q), **bad))
    for bad in (dict(q=q.float()), dict(scale=-1.0), dict(scale=float("nan")), dict(layer=1),
                dict(workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(rm.RoomieError):
            rm.kv_attention(cache, [0, 1], **dict(dict(q=q), **bad))
    assert rm.kv_attention(cache, torch.zeros(0, dtype=torch.int32, device="cuda"), q[:0])[0].shape == (0, 4, 64)
    for bad in (dict(page_tokens=8), dict(head_dim=72), dict(head_dim=272)):
        with pytest.raises(ValueError):
            rm.KVCache(**dict(dict(num_pages=4, page_tokens=16, kv_heads=1, head_dim=64, max_seqs=2, max_pages=2), **bad))


# ---------------------------------------------------------------------------------------------------------------- append
def check_append(torch, rm, cache, seqs, news, *, dtype="bf16", rope=None, q_heads=0, seed=0, view="whole", layer=0, magnitude=1.0):
    """Appends random rows; compares scales, new codes and rescaled earlier codes with the definition."""
    rng = np.random.default_rng(seed)
    rows, h, d, t = sum(news), cache.kv_heads, cache.head_dim, cache.page_tokens
    make = lambda heads: torch.from_numpy(rng.normal(size=(rows, heads, d)) * magnitude).to(dtype_of(torch, dtype)).cuda()
    k, v = make(h), make(h)
    q = make(q_heads) if q_heads else None
    if view == "slice":                                             # one projection's output, split
        packed = torch.cat([q, k, v], 1) if q is not None else torch.cat([k, v], 1)
        q, k, v = (packed[:, :q_heads], packed[:, q_heads:q_heads + h], packed[:, q_heads + h:]) if q is not None else (None, packed[:, :h], packed[:, h:])
    elif view == "odd":
        def odd(x):
            y = torch.zeros(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
            return y.copy_(x)
        k, v = odd(k), odd(v)
    before = {n: (getattr(cache, n)[layer].cpu().numpy().copy(), getattr(cache, n + "_scale")[layer].cpu().numpy().astype(np.float64)) for n in "kv"}
    offset = torch.tensor(np.concatenate([[0], np.cumsum(news)]).tolist(), dtype=torch.int32, device="cuda")
    got_q = rm.kv_append(cache, torch.tensor(seqs, dtype=torch.int32, device="cuda"), k, v, offset, layer=layer, rope=rope, q=q)
    table, lengths = cache.pages.cpu().numpy(), cache.length.cpu().numpy()
    written = {n: np.zeros(before[n][0].shape, bool) for n in "kv"}
    at = 0
    for s, n in zip(seqs, news):
        start = int(lengths[s]) - n
        pos = np.arange(start, start + n)
        x = {"k": host(k[at:at + n]), "v": host(v[at:at + n])}
        slack = {n_: np.zeros(x[n_].shape) for n_ in "kv"}
        if rope is not None:
            f = rope.frequency.cpu().numpy().view(np.uint64)
            turned = sp.rotate(x["k"], pos, f, rope.interleaved, rope.amplitude)
            slack["k"] = rope_bound(x["k"], f, rope.interleaved, turned, "f32", rope.amplitude)
            x["k"] = turned
            if q is not None:
                want = sp.rotate(host(q[at:at + n]), pos, f, rope.interleaved, rope.amplitude)
                bound = rope_bound(host(q[at:at + n]), f, rope.interleaved, want, dtype, rope.amplitude)
                assert np.all(np.abs(host(got_q[at:at + n]) - want) <= bound)
        for name in "kv":
            codes, scales = getattr(cache, name)[layer].cpu().numpy(), getattr(cache, name + "_scale")[layer].cpu().numpy()
            old, old_scale = before[name]
            if cache.layout == "nhd":
                codes, old = codes.transpose(0, 2, 1, 3), old.transpose(0, 2, 1, 3)
            mark = written[name] if cache.layout == "hnd" else written[name].transpose(0, 2, 1, 3)
            for p in range(start // t, -(-(start + n) // t) if n else start // t):
                lo, hi = max(start, p * t), min(start + n, (p + 1) * t)
                held, page = lo - p * t, table[s, p]
                new = x[name][lo - start:hi - start]
                for head in range(h):
                    amax = np.abs(new[:, head]).max()
                    floor = old_scale[page, head] if held else 0.0
                    want = max(sp.scale_of(amax, cache.fmt), floor)
                    near = {max(sp.scale_of(amax * f, cache.fmt), floor) for f in (1 - 2e-6, 1 + 2e-6)} if slack[name].any() else {want}
                    have = float(scales[page, head])
                    assert have in near, (name, head, have, want)
                    values = sp.values(codes[page, head, held:held + hi - lo], cache.fmt)
                    exact = new[:, head] / have
                    room = 0.5 * sp.step_of(exact, cache.fmt) * (1 + 1e-9) + slack[name][lo - start:hi - start, head] / have
                    # the halfway point to the next binade's codes and the format's end
                    assert np.all(np.abs(values - np.clip(exact, -sp.TOP[cache.fmt], sp.TOP[cache.fmt])) <= room * 1.0000001)
                    kept = sp.values(old[page, head, :held], cache.fmt) * (old_scale[page, head] / have)
                    now = sp.values(codes[page, head, :held], cache.fmt)
                    assert np.all(np.abs(now - kept) <= (0.5 * sp.step_of(kept, cache.fmt) if have != old_scale[page, head] else 0))
                mark[page, :, :held + hi - lo] = True
        at += n
    for name in "kv":                                               # nothing else moved
        now = getattr(cache, name)[layer].cpu().numpy()
        assert np.array_equal(now[~written[name]], before[name][0][~written[name]])
    return got_q


@pytest.mark.parametrize("fmt,layout", [("e4m3", "hnd"), ("int8", "nhd"), ("e4m3", "nhd"), ("int8", "hnd")])
@pytest.mark.parametrize("page,dim,heads", [(16, 64, 2), (32, 128, 8), (128, 256, 1), (64, 96, 5), (16, 16, 16)])
def test_append(torch, rm, fmt, layout, page, dim, heads):
    lengths = [1, 16, 17, 150, 64, 40, 260, 31]
    news = [1, 16, 1, 150, 3, 7, 200, 0]
    for dtype, rope, view, q_heads in (("bf16", "half", "slice", 2 * heads), ("f16", None, "whole", 0), ("f32", "pairs", "whole", heads),
                                       ("bf16", "part", "odd", 0)):
        cache = make_cache(torch, rm, lengths, page=page, dim=dim, heads=heads, fmt=fmt, layout=layout, seed=dim, garbage=False)
        table = None if rope is None else rm.RopeTable(dim if rope != "part" else dim // 2, interleaved=rope == "pairs")
        check_append(torch, rm, cache, list(range(8)), news, dtype=dtype, rope=table, view=view, q_heads=q_heads, seed=page)
        assert cache.status_flags() == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_token_by_token(torch, rm, fmt):
    """A page filled one token at a time, magnitudes growing by up to thousands: its scale grows and the earlier codes follow."""
    cache = make_cache(torch, rm, [40, 40], page=16, dim=32, fmt=fmt, seed=3, garbage=False)
    for n, magnitude in zip(range(1, 41), [1e-3, 1e-3, 0.0, 2e-3, 1.0, 0.5, 30.0, 1e3] * 5):
        cache.length.fill_(n)
        check_append(torch, rm, cache, [0, 1], [1, 1], dtype="f32", seed=n, magnitude=magnitude)
    assert cache.status_flags() == 0


def test_append_extremes(torch, rm):
    """Zeros, the type's largest and least values, infinities and NaN."""
    for fmt, top in (("e4m3", 448.0), ("int8", 127.0)):
        cache = make_cache(torch, rm, [4, 4], page=16, dim=16, heads=1, fmt=fmt, garbage=False)
        k = torch.zeros((8, 1, 16), device="cuda")
        v = k.clone()
        k[0], k[1, 0, 0], k[2, 0, 1] = 0.0, 3.0e38, -3.0e38
        v[4:] = 1e-38
        rm.kv_append(cache, [0, 1], k, v, [0, 4, 8])
        assert cache.status_flags() == 0
        got = cached(cache, 0, 0, "k")
        assert np.all(got[0] == 0) and abs(got[1, 0, 0] / 3.0e38 - 1) < 2.0 ** -3.9 and abs(got[2, 0, 1] / -3.0e38 - 1) < 2.0 ** -3.9
        assert np.all(np.abs(cached(cache, 0, 1, "v")) <= 2.0 ** -100)
        k[1, 0, 0], v[5, 0, 3] = float("inf"), float("nan")
        rm.kv_append(cache, [0, 1], k, v, [0, 4, 8])
        assert cache.status_flags() == FLAG_NONFINITE
        codes = cache.k[0, cache.pages[0, 0], 0, 1, 0]
        assert sp.values(codes.cpu().numpy().reshape(1), fmt)[0] > 0.5 * top and np.isfinite(cached(cache, 0, 1, "v")).all()


def test_append_reports_and_skips(torch, rm):
    cache = make_cache(torch, rm, [20, 30], page=16, dim=32)
    k = torch.randn((2, 2, 32), device="cuda")
    def unchanged(flag, seqs=(0, 1), offset=None):
        before = cache.k.clone(), cache.v.clone()
        rm.kv_append(cache, list(seqs), k, k, offset)
        assert cache.status_flags() == flag
        cache.status.zero_()
        return torch.equal(before[0], cache.k) and torch.equal(before[1], cache.v)
    cache.refs[cache.pages[0, 1].long()] = 2                         # shared pages are not written
    cache.refs[cache.pages[1, 1].long()] = 0
    assert unchanged(FLAG_PAGE)
    cache.refs.fill_(1)
    cache.pages[:, 1] = cache.num_pages
    assert unchanged(FLAG_PAGE)
    assert unchanged(FLAG_SEQUENCE, seqs=(-1, 2))
    cache.length.fill_(1)
    assert unchanged(FLAG_SEQUENCE, offset=[0, 2, 2])                # two new tokens in a sequence of one
    cache.length.fill_(10 ** 8)
    assert unchanged(FLAG_SEQUENCE)


def test_append_refusals(torch, rm):
    cache = make_cache(torch, rm, [20, 30], page=16, dim=32)
    k = torch.zeros((2, 2, 32), device="cuda")
    for bad in (dict(k=k[:, :1]), dict(v=k.half()), dict(q_offset=[0, 1]), dict(k=k[:1], v=k[:1]),
                dict(q=k.half(), rope=rm.RopeTable(32)), dict(q=k[:1], rope=rm.RopeTable(32))):
        with pytest.raises(ValueError):
            rm.kv_append(cache, [0, 1], **dict(dict(k=k, v=k), **bad))
    for bad in (dict(layer=1), dict(rope=rm.RopeTable(64))):
        with pytest.raises(rm.RoomieError):
            rm.kv_append(cache, [0, 1], **dict(dict(k=k, v=k), **bad))


# ----------------------------------------------------------------------------------------------------------------- pages
class Both:
    """A cache and its model on lists; page contents are told apart by a byte pattern of their own."""

    def __init__(self, torch, rm, num_pages, page, seqs, width, layers=2, heads=3, dim=16, layout="hnd", seed=0):
        self.torch, self.rm = torch, rm
        self.cache = rm.KVCache(num_pages, page, heads, dim, seqs, width, layers=layers, layout=layout)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for t in (self.cache.k, self.cache.v):
            t.copy_(torch.randint(0, 256, t.shape, generator=gen, device="cuda", dtype=torch.uint8))
        for t in (self.cache.k_scale, self.cache.v_scale):
            t.copy_(torch.rand(t.shape, generator=gen, device="cuda"))
        self.data = [t.clone() for t in (self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale)]
        self.plain = sp.Pages(num_pages, page, seqs, width)
        self.ws = self.cache.workspace()

    def same(self, flags=0):
        c = self.cache
        assert c.refs.tolist() == self.plain.refs and c.length.tolist() == self.plain.length and c.pages.tolist() == self.plain.table
        for t, want in zip((c.k, c.v, c.k_scale, c.v_scale), self.data):
            assert self.torch.equal(t, want)
        assert c.status_flags() == flags
        c.status.zero_()

    def move(self, pairs):
        for t in self.data:
            old = t.clone()
            for a, b in pairs:
                t[:, b] = old[:, a]

    def reserve(self, seqs, want, flags=0):
        self.rm.kv_reserve(self.cache, seqs, want, workspace=self.ws)
        self.plain.reserve(seqs, want)
        self.same(flags)

    def fork(self, parents, children, flags=0):
        self.rm.kv_fork(self.cache, parents, children, workspace=self.ws)
        self.move(self.plain.fork(parents, children))
        self.same(flags)

    def free(self, seqs):
        self.rm.kv_free(self.cache, seqs)
        self.plain.free(seqs)
        self.same()

    def compact(self):
        used = self.torch.zeros(1, dtype=self.torch.int32, device="cuda")
        refs, pages = self.torch.full_like(self.cache.refs, 99), self.torch.full_like(self.cache.pages, 99)
        k = self.cache.k.clone()
        self.rm.kv_compact(self.cache, refs_out=refs, pages_out=pages, used_out=used, workspace=self.ws)     # beside the old table
        assert self.cache.refs.tolist() == self.plain.refs and self.cache.pages.tolist() == self.plain.table
        self.cache.k.copy_(k)
        self.rm.kv_compact(self.cache, used_out=used, workspace=self.ws)
        pairs, n = self.plain.compact()
        self.move(pairs)
        self.same()
        assert int(used) == n and self.torch.equal(refs, self.cache.refs) and self.torch.equal(pages, self.cache.pages)
        assert all(r > 0 for r in self.plain.refs[:n]) and not any(self.plain.refs[n:])


@pytest.mark.parametrize("layout,page", [("hnd", 16), ("nhd", 32)])
def test_pages_by_hand(torch, rm, layout, page):
    b = Both(torch, rm, 12, page, 8, 4, layout=layout)
    b.reserve([0, 3], [page + 1, 2 * page])               # pages 0, 1 and 2, 3
    b.reserve([0, 1], [page + 2, 1])                      # no page, one page
    b.fork([0, 3, 0], [5, 6, 7])                          # part-filled last pages copied, a whole one shared
    b.free([3])                                           # its pages live on in 6
    b.free([6, 0])
    b.compact()
    b.fork([2], [3])                                      # an empty parent: an empty child
    b.free([1, 5, 7])
    assert sum(b.plain.refs) == 0
    b.compact()


def test_pages_random_walk(torch, rm):
    rng = np.random.default_rng(4)
    b = Both(torch, rm, 70, 16, 24, 6, seed=1)
    for step in range(60):
        empty = [s for s in range(24) if b.plain.length[s] == 0]
        full = [s for s in range(24) if b.plain.length[s]]
        room = sum(r == 0 for r in b.plain.refs)
        kind = rng.integers(0, 4)
        if kind == 0 and empty and room > 12:
            seqs = [int(s) for s in rng.permutation(empty)[:rng.integers(1, 3)]]
            b.reserve(seqs, [int(rng.integers(1, 6 * 16)) for _ in seqs])
        elif kind == 1 and empty and full and room > 4:
            n = min(len(empty), int(rng.integers(1, 4)))
            b.fork([int(rng.choice(full)) for _ in range(n)], [int(s) for s in rng.permutation(empty)[:n]])
        elif kind == 2 and full:
            b.free([int(s) for s in rng.permutation(full)[:rng.integers(1, 4)]])
        elif kind == 3:
            b.compact()


def test_pages_large_pools(torch, rm):
    """More pages and requests than one trip of a block looks at."""
    b = Both(torch, rm, 40001, 16, 3000, 16, layers=1, heads=1, dim=16)
    rng = np.random.default_rng(0)
    b.reserve(list(range(0, 2600)), [int(x) for x in rng.integers(1, 257, 2600)])
    b.free([int(s) for s in rng.permutation(2600)[:1300]])
    full = [s for s in range(3000) if b.plain.length[s]]
    empty = [s for s in range(3000) if not b.plain.length[s]]
    b.fork(full[:1100], empty[:1100])
    b.compact()
    b.free(full)


def test_pages_run_out_in_order(torch, rm):
    """Requests are served in order while the free pages cover them and those before; the others change nothing."""
    b = Both(torch, rm, 6, 16, 8, 4)
    b.reserve([0, 1, 2, 3], [33, 48, 16, 0], flags=FLAG_FULL)        # 3 pages, 3 pages, none left for one more; zero needs none
    b.free([1])
    b.reserve([1], [10])
    b.fork([0, 1, 0, 1], [4, 5, 6, 7], flags=FLAG_FULL)              # two pages are left


def test_pages_asked_for_add_up_past_32_bits(torch, rm):
    """1024 requests of 2^22 pages each, together 2^32, and a small one behind them: none is served."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 17 GB of device memory for the page table")
    cache = rm.KVCache(8, 16, 1, 16, 1026, 1 << 22)
    rm.kv_reserve(cache, list(range(1025)), [16 << 22] * 1024 + [16])
    assert cache.status_flags() == FLAG_FULL
    assert not cache.refs.any() and not cache.length.any() and (cache.pages[:, 0] == -1).all()


def test_pages_refusals_on_the_device(torch, rm):
    b = Both(torch, rm, 10, 16, 6, 3)
    b.reserve([0, 1], [20, 30])
    c = b.cache
    def refused(call, flag=FLAG_SEQUENCE):
        call()
        b.same(flag)
    refused(lambda: rm.kv_reserve(c, [0], [5], workspace=b.ws))              # fewer than it has
    refused(lambda: rm.kv_reserve(c, [7, -1], [5, 5], workspace=b.ws))       # no such sequence
    refused(lambda: rm.kv_reserve(c, [2], [49], workspace=b.ws))             # wider than the table
    refused(lambda: rm.kv_fork(c, [0], [1], workspace=b.ws))                 # the child is not empty
    refused(lambda: rm.kv_fork(c, [0], [0], workspace=b.ws))
    refused(lambda: rm.kv_fork(c, [9], [2], workspace=b.ws))
    refused(lambda: rm.kv_free(c, [6, -3]))
    rm.kv_fork(c, [0, 1], [2, 2], workspace=b.ws)                            # a child named twice: the first request has it
    b.move(b.plain.fork([0], [2]))
    b.same(FLAG_SEQUENCE)
    rm.kv_reserve(c, [3, 3], [20, 40], workspace=b.ws)
    b.plain.reserve([3], [20])
    b.same(FLAG_SEQUENCE)
    rm.kv_free(c, [3, 3])                                                    # freed once
    b.plain.free([3])
    b.same()
    refused(lambda: rm.kv_copy(c, [0, 99], c, [-1, 5]), FLAG_PAGE)
    for bad in (lambda: rm.kv_fork(c, [0], [2, 3]), lambda: rm.kv_reserve(c, [0], [1, 2]), lambda: rm.kv_copy(c, [0], c, [1, 2]),
                lambda: rm.kv_compact(c, refs_out=c.refs[:3])):
        with pytest.raises(ValueError):
            bad()
    other = rm.KVCache(4, 32, 3, 16, 1, 1, layers=2)
    small = torch.zeros(64, dtype=torch.uint8, device="cuda")
    for bad in (lambda: rm.kv_copy(c, [0], other, [0]), lambda: rm.kv_compact(c, workspace=small),
                lambda: rm.kv_fork(c, [0] * 7, [1] * 7, workspace=b.ws)):
        with pytest.raises(rm.RoomieError):
            bad()


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_copy_between_caches(torch, rm, layout):
    a = Both(torch, rm, 9, 16, 2, 2, heads=5, dim=48, layout=layout)
    other = rm.KVCache(20, 16, 5, 48, 2, 2, layers=2, layout=layout)
    rm.kv_copy(a.cache, [8, 0, 3], other, [0, 19, 7])
    for name in ("k", "v", "k_scale", "v_scale"):
        src, dst = getattr(a.cache, name), getattr(other, name)
        assert torch.equal(dst[:, [0, 19, 7]], src[:, [8, 0, 3]])
        fresh = getattr(rm.KVCache(20, 16, 5, 48, 2, 2, layers=2, layout=layout), name)
        rest = [p for p in range(20) if p not in (0, 19, 7)]
        assert torch.equal(dst[:, rest], fresh[:, rest])


# ------------------------------------------------------------------------------------------------- streams, one step, record
def test_other_streams_and_graphs(torch, rm):
    """The calls run on the stream they are given, and a step captured in a CUDA graph replays."""
    cache = make_cache(torch, rm, [300, 90], page=32, dim=64, seed=1, garbage=False)
    ws, ids = cache.workspace(), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    table = rm.RopeTable(64)
    k, q = (torch.randn((2, h, 64), device="cuda").to(torch.bfloat16) for h in (2, 4))

    def step(stream=None):
        turned = rm.kv_append(cache, ids, k, k, rope=table, q=q, stream=stream)
        return rm.kv_attention(cache, ids, turned, workspace=ws, stream=stream)[0]
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    q.mul_(0.5)
    graph.replay()
    assert torch.equal(out, step())


def test_tensors_of_another_device_are_refused(torch, rm, monkeypatch):
    """Every call looks at the current device before it launches anything (here it is told of another one)."""
    cache = make_cache(torch, rm, [30, 20], page=16, dim=32, garbage=False)
    ws, table, ids = cache.workspace(), rm.RopeTable(32), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    k, out = torch.zeros((2, 2, 32), device="cuda").half(), torch.zeros((2, 2, 32), device="cuda").half()
    lse = torch.zeros((2, 2), device="cuda")
    before = [t.clone() for t in (cache.k, cache.v, cache.refs, cache.pages, cache.length)]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 7)
    for call in (lambda: rm.rope(k, ids, table, out=out), lambda: rm.kv_append(cache, ids, k, k, rope=table, q=k, q_out=out),
                 lambda: rm.kv_attention(cache, ids, k, out=out, lse=lse, workspace=ws), lambda: rm.kv_reserve(cache, ids, ids, workspace=ws),
                 lambda: rm.kv_fork(cache, ids, ids, workspace=ws), lambda: rm.kv_free(cache, ids), lambda: rm.kv_copy(cache, ids, cache, ids),
                 lambda: rm.kv_compact(cache, workspace=ws)):
        with pytest.raises(ValueError, match="current CUDA device"):
            call()
    monkeypatch.undo()
    assert all(torch.equal(a, b) for a, b in zip(before, (cache.k, cache.v, cache.refs, cache.pages, cache.length)))


def test_serving_step_and_its_profile(torch, rm):
    """Reserve, append, attend, fork and free as one path; its launches become a profile that the model scores."""
    import roomie_synth as rs
    d, kv, heads = 64, 2, 8
    cache = rm.KVCache(40, 16, kv, d, 4, 8)
    ws, table = cache.workspace(), rm.RopeTable(d)
    gen = torch.Generator(device="cuda").manual_seed(0)
    fresh = lambda n, h: torch.randn((n, h, d), generator=gen, device="cuda").to(torch.bfloat16)
    with rm.record_launches() as launches:
        rm.kv_reserve(cache, [0, 1], [37, 20], workspace=ws)
        rows = torch.tensor([0, 37, 57], dtype=torch.int32, device="cuda")
        k, v, q = fresh(57, kv), fresh(57, kv), fresh(57, heads)
        q = rm.kv_append(cache, [0, 1], k, v, rows, rope=table, q=q)
        rm.kv_attention(cache, [0, 1], q, rows, workspace=ws)
        rm.kv_fork(cache, [0], [2], workspace=ws)
        for n in range(1, 6):
            rm.kv_reserve(cache, [0, 1, 2], [37 + n, 20 + n, 37 + n], workspace=ws)
            q = rm.kv_append(cache, [0, 1, 2], fresh(3, kv), fresh(3, kv), rope=table, q=fresh(3, heads))
            out, _ = rm.kv_attention(cache, [0, 1, 2], q, workspace=ws)
        want = np.concatenate([sp.attend(host(q[i:i + 1]), cached(cache, 0, i, "k"), cached(cache, 0, i, "v"),
                                         int(cache.length[i]) - 1, d ** -0.5, 0)[0] for i in range(3)])
        assert np.abs(host(out) - want).max() < 2.0 ** -7
        rm.kv_free(cache, [0, 1, 2])
    assert cache.refs.sum() == 0 and cache.status_flags() == 0
    names = [r["name"] for r in launches]
    assert names[:4] == ["kv_reserve", "kv_append", "kv_attention", "kv_fork_plan"] and names[-1] == "kv_free"
    assert all(r["grid_blocks"] and r["block_threads"] and r["regs_per_thread"] and r["dur_us"] > 0 for r in launches)
    grid, threads, regs, smem, dur, gap = rm.profile_columns(launches)
    synth = rs.make_library(1)
    cat = lambda a, b: np.concatenate([a, b])
    offsets = cat(synth.offsets, [synth.offsets[-1] + len(launches)]).astype(np.uint32)
    lib = rm.library_build(cat(synth.grid_blocks, grid), cat(synth.block_threads, threads), cat(synth.regs_per_thread, regs),
                           cat(synth.smem_per_block, smem), cat(synth.dur_us, dur), cat(synth.gap_us, gap), offsets, synth.spec)
    P, _ = rm.pair_matrix(lib, n_align=8)
    assert lib.status_flags() == 0 and torch.isfinite(P).all() and P.shape == (17, 17)
    with rm.record_launches(2) as few:                               # more launches than the record holds
        for _ in range(4):
            rm.kv_free(cache, [0])
    assert len(few) == 2


def test_example_runs(torch, rm):
    """The example's steps: shared pages after the fork, half of them given back, finite results, a GPU for the model."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_step.py")
    spec = importlib.util.spec_from_file_location("serving_step", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    launches, out, gpu = example.main(["--seqs", "3", "--prompt", "130", "--steps", "4", "--beams", "2"])
    assert torch.isfinite(out).all() and out.shape == (6, 32, 128) and 0 <= gpu < 16
    assert {"kv_reserve", "kv_append", "kv_attention", "kv_fork_plan", "kv_fork_move", "kv_free", "kv_compact_plan",
            "kv_compact_move"} <= {r["name"] for r in launches}
