"""A beam search over a bounded cache, all its operators together, each step against the definitions: what the cache holds is read back and followed by
hand.  Error bounds are those of the operators' own tests (attention: 2^-6 of a weighted mean of values of at most about 4)."""
import numpy as np
import pytest

import bounded_plain as bp
import norm_plain as npl
import serving_plain as sp
from test_gpu_key_weights import shares
from test_gpu_serving import cached

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


@pytest.mark.parametrize("fmt,layout,page,dim", [("e4m3", "hnd", 16, 64), ("int8", "nhd", 32, 128), ("e4m3", "hnd", 16, 96)])
def test_search_step_by_step(torch, rm, fmt, layout, page, dim):
    kv, group, beams, prompt, keep, vocab = 2, 4, 3, 70, 40, 500
    heads, scale = kv * group, dim ** -0.5
    rng = np.random.default_rng(page)
    new = lambda *s: torch.from_numpy(rng.normal(size=s)).to(torch.bfloat16).cuda()
    cache = rm.KVCache(40, page, kv, dim, beams, 6, fmt=fmt, layout=layout)
    ws, weight, table, f = cache.workspace(), cache.key_weights(), rm.RopeTable(dim), rm.rope_frequencies(dim)
    slots, follow = [0, 1, 2], np.zeros((beams, kv, 0))
    wq, wk = (torch.from_numpy(rng.uniform(0.5, 1.5, dim)).float().cuda() for _ in range(2))
    scores = torch.tensor([[0.0, -np.inf, -np.inf]], device="cuda")
    host = lambda t: t.double().cpu().numpy()

    def tokens_in(which, positions, news, lengths, fresh):
        """Appends, attends, weighs; checks each; `which`: sequences, one run of rows each."""
        rows = sum(news)
        q0, k0, v = new(rows, heads, dim), new(rows, kv, dim), new(rows, kv, dim)
        p = torch.tensor(positions, dtype=torch.int32, device="cuda")
        q, k = rm.qk_norm_rope(q0, k0, p, table, wq, wk)
        for got, x, w in ((q, q0, wq), (k, k0, wk)):
            want, _ = npl.forward(host(x), host(w), np.array(positions), f, False, 1.0, 1e-6)
            assert np.all(np.abs(host(got) - want) <= 2.0 ** -8 * np.abs(want) + 1e-4)
        offset = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda")
        rm.kv_reserve(cache, which, lengths, workspace=ws)
        rm.kv_append(cache, which, k, v, offset)
        out, lse = rm.kv_attention(cache, which, q, offset, workspace=ws)
        before = host(weight)[0]
        rm.kv_weights(cache, which, q, lse, weight, offset, fresh=fresh)
        at, after = 0, host(weight)[0]
        for s, n, length in zip(which, news, lengths):
            keys, values = cached(cache, 0, s, "k"), cached(cache, 0, s, "v")
            want, want_lse, _ = sp.attend(host(q[at:at + n]), keys, values, length - n, scale, 0)
            assert np.all(np.abs(host(out[at:at + n]) - want) < 2.0 ** -5) and np.all(np.abs(host(lse[at:at + n]) - want_lse) < 2.0 ** -12)
            got, bound = shares(host(q[at:at + n]), keys, host(lse[at:at + n]), length - n, scale, 0)
            if not fresh:
                got[:, :length - n] += before[s, :, :length - n]
            assert np.all(np.abs(after[s, :, :length] - got) <= bound + 2.0 ** -23 * got)
            at += n
        assert cache.status_flags() == 0

    def cut(which):
        held = {(s, n): cached(cache, 0, s, n) for s in which for n in ("k", "v")}
        before, lengths = host(weight)[0], cache.length.tolist()
        rm.kv_evict(cache, which, weight, keep, first=2, recent=10, workspace=ws)
        assert cache.length.tolist() == [min(n, keep) if s in which else n for s, n in enumerate(lengths)] and cache.status_flags() == 0
        for s in which:
            for h in range(kv):
                at = bp.kept(before[s, h], lengths[s], keep, 2, 10) if lengths[s] > keep else np.arange(lengths[s])
                assert np.array_equal(host(weight)[0, s, h, :len(at)], before[s, h, at])
                for n in ("k", "v"):
                    got, want = cached(cache, 0, s, n)[:, h], held[s, n][at, h]
                    # a code moved to another power of two is off by half a step at most, or not at all
                    assert np.all(np.abs(got - want) <= (2.0 ** -4 * np.abs(want) + 2.0 ** -9 if fmt == "e4m3" else np.abs(got).max() / 127))

    tokens_in([0], list(range(prompt)), [prompt], [prompt], True)
    cut([0])
    length = keep
    rm.kv_reorder(cache, slots, [0, 0, 0], workspace=ws)
    weight.copy_(weight[:, [0, 0, 0]])
    for n in range(12):
        held = [(cached(cache, 0, s, "k"), cached(cache, 0, s, "v")) for s in slots]
        logits = torch.from_numpy(rng.normal(size=(1, beams, vocab)) * 3).to(torch.bfloat16).cuda()
        x = host(logits)[0]
        c = host(scores)[0][:, None] + x - np.log(np.exp(x).sum(-1, keepdims=True))
        scores, parent, token = rm.beam_select(logits, scores, beams)
        order = np.lexsort((np.arange(c.size), -c.ravel()))[:beams]
        assert parent[0].tolist() == (order // vocab).tolist() and token[0].tolist() == (order % vocab).tolist()
        assert np.all(np.abs(host(scores)[0] - c.ravel()[order]) < 1e-4)
        rm.kv_reorder(cache, slots, parent, workspace=ws)
        weight.copy_(weight[:, parent[0].long()])
        for s, p in zip(slots, parent[0].tolist()):
            assert all(np.array_equal(cached(cache, 0, s, name), old) for name, old in zip(("k", "v"), held[p]))
        if length >= keep + 5:
            cut(slots)
            length = keep
        length += 1
        tokens_in(slots, [prompt + n] * beams, [1] * beams, [length] * beams, False)
    rm.kv_free(cache, slots)
    assert not cache.refs.any()


def test_example_of_a_search(torch, rm):
    import importlib.util
    import os
    spec = importlib.util.spec_from_file_location("serving_step_example", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    launches, tokens, gpu = example.main(["--seqs", "2", "--beams", "3", "--prompt", "90", "--steps", "12", "--keep", "48"])
    assert tuple(tokens.shape) == (2, 3, 12) and tokens.min() >= 0 and tokens.max() < 4096 and gpu >= -1
    names = {r["name"] for r in launches}
    assert {"qk_norm_rope", "beam_rows", "beam_pick", "kv_reorder_plan", "kv_reorder_move", "kv_weights", "kv_evict_plan", "kv_evict"} <= names
    again = example.search(2, 3, 90, 12, 48)
    assert torch.equal(again[1], tokens)                            # the same search again
