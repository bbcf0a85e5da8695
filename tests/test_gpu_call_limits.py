"""Calls that the binding has to refuse."""
import pytest

from test_gpu_serving import make_cache

pytestmark = pytest.mark.gpu

PAST = 1 << 32


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


def test_numbers_past_32_bits(torch, rm):
    """They do not wrap to a call with another number."""
    cache = make_cache(torch, rm, [40, 20], page=16, heads=2, dim=64, layers=2)
    names = ("k", "v", "k_scale", "v_scale", "refs", "pages", "length")
    before = {n: getattr(cache, n).clone() for n in names}
    w = torch.rand(cache.key_weights().shape, device="cuda")
    old = w.clone()
    q, kv, lse = torch.zeros(2, 4, 64, device="cuda").half(), torch.ones(2, 2, 64, device="cuda").half(), torch.zeros(2, 4, device="cuda")
    logits, scores = torch.zeros(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    calls = [lambda: rm.rope_frequencies(PAST + 8), lambda: rm.kv_evict(cache, [0], w, PAST + 10), lambda: rm.kv_evict(cache, [0], w, 30, first=PAST), lambda: rm.kv_evict(cache, [0], w, 30, recent=PAST + 3),
             lambda: rm.beam_select(logits, scores, 4, pad=PAST + 5), lambda: rm.beam_select(logits, scores, PAST + 4), lambda: rm.beam_workspace(2, 3, 50, PAST + 4),
             lambda: rm.beam_workspace(PAST + 2, 3, 50, 4), lambda: rm.beam_workspace(2, PAST + 3, 50, 4), lambda: rm.beam_workspace(2, 3, PAST + 50, 4)]
    for layer in (PAST, PAST + 1, -PAST):
        calls += [lambda layer=layer: rm.kv_weights(cache, [0, 1], q, lse, w, layer=layer), lambda layer=layer: rm.kv_append(cache, [0, 1], kv, kv, layer=layer),
                  lambda layer=layer: rm.kv_attention(cache, [0, 1], q, layer=layer)]
    for window in (PAST, PAST + 1, -PAST + 1):
        calls += [lambda window=window: rm.kv_weights(cache, [0, 1], q, lse, w, window=window), lambda window=window: rm.kv_attention(cache, [0, 1], q, window=window)]
    for call in calls:
        with pytest.raises(ValueError, match="32 bits|limits"):
            call()
    assert cache.status_flags() == 0 and torch.equal(w, old)
    for n in names:
        assert torch.equal(getattr(cache, n).view(torch.uint8), before[n].view(torch.uint8)), n


def test_forward_mode_is_refused(torch, rm):
    """A tangent that would be lost is an error; beside tensors without one the calls go on."""
    import torch.autograd.forward_ad as fw
    q, k = torch.randn(3, 4, 64, device="cuda"), torch.randn(3, 2, 64, device="cuda")
    w, positions, table = torch.rand(64, device="cuda") + 0.5, torch.arange(3, dtype=torch.int32, device="cuda"), rm.RopeTable(64)
    want, turned = rm.qk_norm_rope(q, k, positions, table, w, w), rm.rope(q, positions, table)
    with fw.dual_level():
        dual = lambda t: fw.make_dual(t, torch.ones_like(t))
        for args in ((dual(q), k, positions, table, w, w), (q, dual(k), positions, table, w, w), (q, k, positions, table, dual(w), None), (q, k, positions, None, None, dual(w)),
                     (dual(q.clone().requires_grad_()), k, positions, table, w, w)):
            with pytest.raises(RuntimeError, match="forward"):
                rm.qk_norm_rope(*args)
        for x in (dual(q), dual(q.clone().requires_grad_())):
            with pytest.raises(RuntimeError, match="forward"):
                rm.rope(x, positions, table)
        with torch.no_grad(), pytest.raises(RuntimeError, match="forward"):
            rm.rope(dual(q), positions, table)
        assert all(torch.equal(a, b) for a, b in zip(rm.qk_norm_rope(q, k, positions, table, w, w), want)) and torch.equal(rm.rope(q, positions, table), turned)
    assert all(torch.equal(a, b) for a, b in zip(rm.qk_norm_rope(q, k, positions, table, w, w), want))
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda x: rm.qk_norm_rope(x, k, positions, table, w, w)[0], (q,), (torch.ones_like(q),))
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda x: rm.rope(x, positions, table), (q,), (torch.ones_like(q),))
