"""Beam search's selection where different logits give the same score in 64 bits: those go by (beam, token) too.

All candidates are ranked by their value in 64 bits, score + ((logit - largest) - log of the sum).  The kernel's sum of exponentials may be off by 3e-5 (SLACK, as in
test_gpu_beams.py), so the inputs are such that no value comes closer than that to the border between two numbers of 64 bits: asserted where it is not plain."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

SLACK = 3e-5
KINDS = ["f32", "f16", "bf16"]
LEAST = float(np.finfo(np.float32).min)


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


def ranked(logits, scores, num, ended=None, pad=0):
    """(value, row, token) of the best of each request, all candidates compared by value, then beam, then token."""
    x, s = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    out = []
    for r in range(x.shape[0]):
        value, row, token = [], [], []
        for b in range(x.shape[1]):
            if not np.isfinite(s[r, b]):
                continue
            if ended is not None and bool(ended[r, b]):
                v, t = np.array([s[r, b]]), np.array([pad])
            else:
                y = x[r, b]
                t = np.nonzero(y > -np.inf)[0]
                if t.size == 0:
                    continue
                v = s[r, b] + ((y[t] - y.max()) - math.log(np.exp(y[t] - y.max()).sum()))
            value.append(v)
            row.append(np.full(t.size, r * x.shape[1] + b))
            token.append(t)
        value, row, token = (np.concatenate(a) if a else np.zeros(0) for a in (value, row, token))
        best = np.lexsort((token, row, -value))[:num]
        out.append([(value[i], int(row[i]), int(token[i])) for i in best])
    return out


def check(torch, rm, logits, scores, num, ended=None, pad=0):
    got = rm.beam_select(logits, scores, num, ended=ended, pad=pad)
    again = rm.beam_select(logits, scores, num, ended=ended, pad=pad)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for r, want in enumerate(ranked(logits, scores, num, ended, pad)):
        n = len(want)
        assert list(zip(got[1][r].tolist(), got[2][r].tolist())) == [w[1:] for w in want] + [(-1, -1)] * (num - n), r
        assert all(abs(float(v) - w[0]) <= SLACK + 2.0 ** -24 * abs(w[0]) for v, w in zip(got[0][r].tolist(), want))
    return got


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("vocab", [40, 5000, 40001])
@pytest.mark.parametrize("num", [1, 8, 40, 128])
def test_a_score_that_swallows_the_logits(torch, rm, dtype, vocab, num):
    """A beam held back by the lowest score: all its words are worth the same, so the lowest tokens are its best, wherever its largest logits are."""
    gen = torch.Generator().manual_seed(vocab)
    least = torch.tensor([[LEAST]], device="cuda")
    rising = (torch.arange(vocab) * 2.0 ** -8).to(dtype_of(torch, dtype)).cuda().view(1, 1, vocab)
    check(torch, rm, rising, least, num)
    got = check(torch, rm, torch.randn((1, 1, vocab), generator=gen).to(dtype_of(torch, dtype)).cuda(), least, num)
    assert got[2][0, :min(num, vocab)].tolist() == list(range(min(num, vocab)))
    x = torch.randn((3, 5, vocab), generator=gen).to(dtype_of(torch, dtype)).cuda()
    x[:, :, :vocab // 3] = -math.inf                               # the words that are forbidden do not count
    scores = torch.full((3, 5), LEAST, device="cuda")
    check(torch, rm, x, scores, num)
    x[0, 0, :] = -math.inf                                         # one word, or two, that outrank them
    x[0, 0, vocab - 3] = 1.0
    scores[0, 0] = scores[1, 3] = -1.0
    x[1, 3, :] = -math.inf
    x[1, 3, [2, vocab - 1]] = 0.5
    ended = torch.zeros((3, 5), dtype=torch.bool, device="cuda")
    ended[0, 2] = ended[2, 0] = ended[2, 3] = True                 # an ended beam among them is one candidate, in its place
    check(torch, rm, x, scores, num)
    check(torch, rm, x, scores, num, ended, pad=vocab - 1)


@pytest.mark.parametrize("num", [1, 6, 100])
def test_logits_that_the_sum_swallows(torch, rm, num):
    """Float32 logits near 1e-30 beside the logarithm of their number."""
    gen = torch.Generator().manual_seed(1)
    x = (torch.randn((2, 3, 3000), generator=gen) * 1e-30).cuda()
    got = check(torch, rm, x, torch.zeros(2, 3, device="cuda"), num)
    assert got[2][0].tolist() == list(range(num)) and got[1][1].eq(3).all()


@pytest.mark.parametrize("dtype", KINDS)
@pytest.mark.parametrize("num", [3, 50, 128])
def test_steps_of_a_score(torch, rm, dtype, num):
    """At a score of -2^50 values are a quarter apart: of the words' logits, 2^-6 apart, about sixteen give the same value."""
    rng = np.random.default_rng(num)
    vocab = 20000
    x = rng.integers(0, 512, (2, 4, vocab)) * 2.0 ** -6
    top = x.max(-1, keepdims=True)
    inner = x - top - np.log(np.exp(x - top).sum(-1, keepdims=True))
    border = np.abs((inner * 4) % 1.0 - 0.5) / 4                   # distance to the nearest border between two values
    assert border.min() > SLACK
    logits = torch.from_numpy(x).to(dtype_of(torch, dtype)).cuda()
    if dtype == "bf16":                                            # eight bits hold the logits from 4 up in steps of 2^-5 and more
        inner = logits.double().cpu().numpy()
        inner = inner - top - np.log(np.exp(inner - top).sum(-1, keepdims=True))
        assert (np.abs((inner * 4) % 1.0 - 0.5) / 4).min() > SLACK
    check(torch, rm, logits, torch.full((2, 4), -2.0 ** 50, device="cuda"), num)


@pytest.mark.parametrize("num,vocab", [(128, 50), (128, 300), (64, 131072)])
def test_many_beams_of_one_value(torch, rm, num, vocab):
    x = torch.randn((1, 64, vocab), generator=torch.Generator().manual_seed(vocab)).bfloat16().cuda()
    got = check(torch, rm, x, torch.full((1, 64), LEAST, device="cuda"), num)
    assert got[1][0].tolist() == [i // vocab for i in range(num)] and got[2][0].tolist() == [i % vocab for i in range(num)]


@pytest.mark.parametrize("beams,vocab,num", [(64, 131072, 64), (256, 33000, 128)])
def test_beams_in_rising_order(torch, rm, beams, vocab, num):
    """The best candidates are those that are looked at last: the most trips over the lists."""
    x = torch.randn((1, beams, vocab), generator=torch.Generator().manual_seed(beams)).bfloat16().cuda()
    scores = torch.linspace(-40.0, 0.0, beams, device="cuda").view(1, beams)
    got = rm.beam_select(x, scores, num)
    want = torch.log_softmax(x.double(), -1)[0] + scores.double()[0, :, None]
    order = torch.sort(want.flatten(), descending=True, stable=True)
    assert (order.values[:num].cpu() - got[0][0].cpu().double()).abs().max() < SLACK + 2.0 ** -24 * 60
    mine = want.flatten()[(got[1][0].long() * vocab + got[2][0].long())]
    assert (mine - order.values[:num]).abs().max() < 2 * SLACK and len(set(zip(got[1][0].tolist(), got[2][0].tolist()))) == num


@pytest.mark.parametrize("beams,vocab,num", [(256, 33000, 128), (200, 40000, 100), (256, 50, 128)])
def test_beams_of_one_value_in_rising_order(torch, rm, beams, vocab, num):
    """So far apart that the logits do not count: the last beam's lowest tokens, then those of the beam before it."""
    x = torch.randn((2, beams, vocab), generator=torch.Generator().manual_seed(beams)).half().cuda()
    scores = (torch.arange(-beams, 0).float() * 2.0 ** 90).expand(2, beams).contiguous().cuda()
    check(torch, rm, x, scores, num)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_updated_in_place(torch, rm, dtype):
    """scores_out may be scores where as many are wanted as there are beams."""
    gen = torch.Generator().manual_seed(3)
    x = (torch.randn((9, 4, 7001), generator=gen) * 3).to(dtype_of(torch, dtype)).cuda()
    scores = (-torch.rand((9, 4), generator=gen)).cuda()
    ended = (torch.rand((9, 4), generator=gen) < 0.3).cuda()
    for start in (scores, torch.full_like(scores, LEAST)):
        for which in (None, ended):
            want = rm.beam_select(x, start, 4, ended=which)
            same, parent, token = start.clone(), torch.empty_like(want[1]), torch.empty_like(want[2])
            rm.beam_select(x, same, 4, ended=which, out=(same, parent, token))
            assert all(torch.equal(a, b) for a, b in zip((same, parent, token), want))
