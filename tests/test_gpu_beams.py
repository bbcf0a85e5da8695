"""Beam search's selection against its definition in 64 bits, in plain numpy.

Picks are compared exactly wherever neighbouring candidates are further apart than what the sums of exponentials may be off: of n logits a
thread adds at most 64 and a block 256 such sums in float32, and each exponential is off by 2^-22 and its argument by 2^-24 of at most 128:
2^-17 + 2^-22 + 320 2^-24 of the sum at the very most, 3e-5 (SLACK; within a row the order is exact).  Scores: the same, and their own rounding."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

SLACK = 3e-5
KINDS = ["f32", "f16", "bf16"]


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


def definition(x, scores, num, ended, pad):
    """x [requests, beams, vocab] float64.  All candidates' (value, row, token), best first, for each request."""
    out = []
    for r in range(x.shape[0]):
        found = []
        for b in range(x.shape[1]):
            s = float(scores[r, b])
            if not np.isfinite(s):
                continue
            if ended is not None and ended[r, b]:
                found.append((s, r * x.shape[1] + b, pad))
                continue
            row = x[r, b]
            if np.isnan(row).any() or not np.isfinite(row.max()):
                continue
            lse = row.max() + np.log(np.exp(row - row.max()).sum())
            top = np.lexsort((np.arange(row.size), -row))[:num]
            found += [(s + (row[t] - lse), r * x.shape[1] + b, int(t)) for t in top if row[t] > -np.inf]
        found.sort(key=lambda f: (-f[0], f[1], f[2]))
        out.append(found)
    return out


def check(torch, rm, logits, scores, num, ended=None, pad=0, workspace=None):
    got = rm.beam_select(logits, scores, num, ended=ended, pad=pad, workspace=workspace)
    again = rm.beam_select(logits, scores, num, ended=ended, pad=pad)
    assert all(torch.equal(a, b) for a, b in zip(got, again))      # the same bits each time
    value, parent, token = (t.cpu().numpy() for t in got)
    want = definition(logits.double().cpu().numpy(), scores.cpu().numpy(), num, None if ended is None else ended.cpu().numpy(), pad)
    for r, found in enumerate(want):
        n = min(num, len(found))
        assert np.all(parent[r, n:] == -1) and np.all(token[r, n:] == -1) and np.all(value[r, n:] == -np.inf)
        where = {(p, t): v for v, p, t in found}
        mine = list(zip(parent[r, :n].tolist(), token[r, :n].tolist()))
        assert len(set(mine)) == n
        for i, (v, p, t) in enumerate(found[:n]):
            assert mine[i] in where and abs(value[r, i] - v) <= SLACK + 2.0 ** -24 * abs(v), (r, i)
            if mine[i] != (p, t):                                  # only where the two are as good as equal, and of different rows
                assert abs(where[mine[i]] - v) <= 2 * SLACK and mine[i][0] != p, (r, i, mine[i], found[:n])
    return got


def logits_of(torch, rng, requests, beams, vocab, dtype, view="whole", spread=3.0):
    x = torch.from_numpy(rng.normal(size=(requests, beams, vocab)) * spread).to(dtype_of(torch, dtype)).cuda()
    if view == "padded":                                           # a vocabulary padded to a multiple, and a larger batch
        wide = torch.full((requests, beams + 1, vocab + 13), 50.0, dtype=x.dtype, device="cuda")
        wide[:, :beams, :vocab] = x
        return wide[:, :beams, :vocab]
    if view == "odd":
        flat = torch.full((requests * beams * vocab + 3,), 50.0, dtype=x.dtype, device="cuda")[3:]
        flat = flat.view(requests, beams, vocab)
        flat.copy_(x)
        return flat
    return x


@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 255, 1000, 4096, 4097, 8191, 32768, 50257])
@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("view", ["whole", "padded", "odd"])
def test_beams(torch, rm, vocab, dtype, view):
    rng = np.random.default_rng(vocab)
    for requests, beams, num in ((1, 1, 1), (3, 4, 8), (2, 3, 32), (1, 5, 33), (2, 2, 128)):
        scores = torch.from_numpy(-20 * rng.random((requests, beams))).float().cuda()
        check(torch, rm, logits_of(torch, rng, requests, beams, vocab, dtype, view), scores, num)


@pytest.mark.parametrize("requests,beams,vocab,num", [(40, 8, 20011, 16), (300, 1, 4099, 1), (2, 256, 1500, 128), (1, 64, 131072, 64), (1, 1, 1 << 20, 5)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beams_of_other_shapes(torch, rm, requests, beams, vocab, num, dtype):
    rng = np.random.default_rng(num)
    scores = torch.from_numpy(-rng.random((requests, beams))).float().cuda()
    check(torch, rm, logits_of(torch, rng, requests, beams, vocab, dtype), scores, num)


@pytest.mark.parametrize("dtype", KINDS)
def test_beams_ended_and_masked(torch, rm, dtype):
    """Ended beams, beams without a score, forbidden words, rows that hold nothing, NaN or +infinity, fewer candidates than asked for."""
    rng = np.random.default_rng(9)
    x = logits_of(torch, rng, 6, 4, 777, dtype)
    inf = float("inf")
    scores = torch.from_numpy(-3 * rng.random((6, 4))).float().cuda()
    ended = torch.zeros(6, 4, dtype=torch.bool, device="cuda")
    ended[0, 1] = ended[1] = True                                  # request 1: all
    x[0, 2, 5:700] = -inf
    x[2] = -inf                                                    # request 2: two words in all
    x[2, 1, 40], x[2, 3, 776] = 1.0, 2.0
    x[3, 0, 3], x[3, 1, 700], x[3, 2] = float("nan"), inf, -inf    # request 3: one row of four
    scores[4] = torch.tensor([-inf, inf, float("nan"), -1.0])
    x[5] = -inf                                                    # request 5: nothing
    x[0, 1, 7] = float("nan")                                      # of an ended beam: not read
    got = check(torch, rm, x, scores, 9, ended, pad=776)
    assert got[1][5].eq(-1).all() and got[2][1][:4].eq(776).all() and got[1][1][4:].eq(-1).all() and got[1][4][0] == 19
    check(torch, rm, x, scores, 1, ended, pad=0)
    check(torch, rm, x, scores, 128, ended.to(torch.uint8), pad=5)
    only = torch.zeros(6, 4, dtype=torch.bool, device="cuda")
    only[3], only[4, 0] = True, True                               # ended beams without a finite score stay out
    check(torch, rm, x, scores, 3, only)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("num", [1, 8, 40, 128])
def test_beams_ties(torch, rm, dtype, num):
    """Equal logits go by token, equal rows by beam - wherever in memory they start - and orders that run through a block's threads."""
    vocab = 33333                                                  # odd: the rows' alignment differs
    scores = torch.tensor([[-1.0, -1.0, -1.0]], device="cuda")
    flat = torch.zeros(1, 3, vocab, dtype=dtype_of(torch, dtype), device="cuda")
    got = check(torch, rm, flat, scores, num)
    assert got[1].eq(0).all() and torch.equal(got[2][0].cpu(), torch.arange(num, dtype=torch.int32))
    row = torch.randn(vocab, generator=torch.Generator().manual_seed(1)).to(flat.dtype).cuda()
    same = row.expand(1, 3, vocab)                                 # one row for all beams
    got, apart = check(torch, rm, same, scores, num), check(torch, rm, same.contiguous(), scores, num)
    assert all(torch.equal(a, b) for a, b in zip(got, apart))
    want = definition(same.double().cpu().numpy(), scores.cpu().numpy(), num, None, 0)[0][:num]
    assert list(zip(got[1][0].tolist(), got[2][0].tolist())) == [w[1:] for w in want]
    steps = (torch.arange(vocab, device="cuda").float() * (2.0 ** -9)).to(flat.dtype).expand(1, 3, vocab)
    check(torch, rm, steps, scores, num)
    check(torch, rm, steps.flip(2), scores, num)
    few = torch.full((1, 3, vocab), -30000.0, device="cuda")       # a mask that is not infinite
    few[0, 1, [7, 20000, 33332]] = torch.tensor([1.0, 3.0, 2.0], device="cuda")
    check(torch, rm, few.to(flat.dtype), scores, num)
    block = torch.full((1, 3, vocab), -5.0, device="cuda")         # all the large ones with a few threads, each with as many
    block[0, 0, 512:4096 + 512] = torch.randn(4096, generator=torch.Generator().manual_seed(2)).cuda()
    block[0, 2, 0:vocab:64] = 2.0
    check(torch, rm, block.to(flat.dtype), scores, num)


def test_beams_of_extreme_logits(torch, rm):
    rng = np.random.default_rng(4)
    scores = torch.zeros(1, 2, device="cuda")
    x = torch.from_numpy(rng.normal(size=(1, 2, 3000))).float().cuda()
    for size in (1e-30, 1e4, 1e30):                                # 1e30: all the weight on one word; differences overflow
        y = x * size
        got = rm.beam_select(y, scores, 2)
        want = definition(y.double().cpu().numpy(), np.zeros((1, 2)), 2, None, 0)[0]
        if size > 1e20:
            assert {tuple(z) for z in zip(got[1][0].tolist(), got[2][0].tolist())} == {z[1:] for z in want[:2]} and not got[0].any()
        elif size < 1:
            assert abs(float(got[0][0, 0]) + np.log(3000)) < 1e-5
        else:
            check(torch, rm, y, scores, 6)
    least = torch.finfo(torch.float32).min
    y = torch.full((1, 2, 100), least, device="cuda")              # the type's lowest value as a mask
    y[0, 1, 9] = 0.5
    got = rm.beam_select(y, scores, 2)
    assert got[1][0].tolist() == [1, 0] and got[2][0].tolist() == [9, 0]


def test_beams_offsets_past_32_bits(torch, rm):
    free = torch.cuda.mem_get_info()[0]
    rows, vocab = 17, 1 << 24
    stride = (1 << 32) // 16 + (1 << 20)                           # the last row starts behind 2^32 elements
    if free < 2 * 18 * stride + (8 << 30):
        pytest.skip("not enough memory")
    flat = torch.zeros(rows * stride + vocab, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((1, rows, 5000), (rows * stride, stride, 1))
    x[0, 16, 4321] = 9.0
    got = rm.beam_select(x, torch.zeros(1, rows, device="cuda"), 2)
    assert got[1][0, 0] == 16 and got[2][0, 0] == 4321 and got[1][0, 1] == 0 and got[2][0, 1] == 0


def test_beams_on_streams_and_in_graphs(torch, rm):
    rng = np.random.default_rng(5)
    x, scores = logits_of(torch, rng, 4, 4, 9001, "bf16"), torch.zeros(4, 4, device="cuda")
    work = rm.beam_workspace(4, 4, 9001, 8, torch.bfloat16)
    out = tuple(torch.empty(4, 8, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert rm.beam_select(x, scores, 8, out=out, workspace=work, stream=side) is out
    side.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for g in graphs:                                               # two graphs with one workspace
        with torch.cuda.graph(g):
            outs.append(rm.beam_select(x, scores, 8, workspace=work))
    for _ in range(3):
        x.copy_(logits_of(torch, rng, 4, 4, 9001, "bf16"))
        for g in graphs:
            g.replay()
        want = rm.beam_select(x, scores, 8)
        assert all(torch.equal(a, w) and torch.equal(b, w) for a, b, w in zip(*outs, want))


def test_beam_refusals(torch, rm):
    x, s = torch.zeros(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    for bad in (dict(logits=x[0]), dict(logits=x.double()), dict(logits=x.cpu()), dict(logits=x.transpose(1, 2)), dict(scores=s[:1]), dict(scores=s.double()),
                dict(scores=s.t().contiguous().t()), dict(ended=s), dict(ended=torch.zeros(2, 4, dtype=torch.bool, device="cuda")), dict(scores=s.cpu()),
                dict(out=(s, s, s)), dict(num=0), dict(num=129), dict(num=4, out=tuple(torch.zeros(2, 5, device="cuda") for _ in range(3)))):
        with pytest.raises(ValueError):
            rm.beam_select(**dict(dict(logits=x, scores=s, num=4), **bad))
    with pytest.raises(rm.RoomieError, match="invalid argument"):
        rm.beam_select(x, s, 4, pad=1 << 31)
    with pytest.raises(rm.RoomieError, match="workspace"):
        rm.beam_select(x, s, 4, workspace=torch.empty(128, dtype=torch.uint8, device="cuda"))
    for bad in ((1, 257, 10, 1), (1, 0, 10, 1), (1, 1, 0, 1), (1, 1, (1 << 24) + 1, 1), (70000, 1, 10, 1), (0, 1, 10, 1)):
        with pytest.raises(ValueError):
            rm.beam_workspace(*bad)
    got = rm.beam_select(x[:0], s[:0], 4)
    assert all(tuple(t.shape) == (0, 4) for t in got)


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("num", [1, 32, 33, 128])
def test_beams_of_one_number_in_large_parts(torch, rm, dtype, num):
    """Rows whose every piece may hold a candidate, enough of them for parts of eight pieces a thread: the same answer each time."""
    requests, beams, vocab = 10, 3, 33333
    x = torch.zeros(requests, beams, vocab, dtype=dtype_of(torch, dtype), device="cuda")
    scores = torch.zeros(requests, beams, device="cuda")
    for _ in range(20):
        got = rm.beam_select(x, scores, num)
        assert torch.equal(got[1].cpu(), (torch.arange(requests, dtype=torch.int32) * beams).unsqueeze(1).expand(-1, num))
        assert torch.equal(got[2].cpu(), torch.arange(num, dtype=torch.int32).expand(requests, num))
        assert (got[0].cpu().double() + math.log(vocab)).abs().max() <= 1e-5      # eps / 2 of 10.4 is 6e-7; sums of ones are exact
    rising = (torch.arange(vocab, device="cuda") // 64).to(x.dtype).expand(requests, beams, vocab)
    check(torch, rm, rising, scores, num)
