"""Norms of queries and keys with rotary positions, and their gradients, against their definition in 64 bits.

Error bounds (u: half a unit in the last place of the type, 2^-24, 2^-11, 2^-8 for float32, float16, bfloat16; v = 2^-24):
y    r has half of the relative error of a sum of dim squares, (dim + 4) v / 2, and its own 2 v; two products: (dim / 2 + 8) v of x r w;
     the rotation 7e-7 of a pair's sum (its phase's 2^-25 turns and two units of cosine and sine); then u |y|.
dx   the turned gradient has 7e-7 of a pair's sum; the mean and r (dim + 16) v each: ((2 dim + 32) v + 7e-7) of the magnitudes of the two terms;
     then u |dx|.
dw   the same of each term, and a sum of as many float32 numbers as there are rows: rows v more; then u |dw|."""
import numpy as np
import pytest

import norm_plain as npl

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 2.0 ** -140, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}       # half of the least step, and of what products in between may lose
V = 2.0 ** -24


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


def rows(torch, rng, tokens, heads, dim, dtype, view, size=1.0):
    x = torch.from_numpy(rng.normal(size=(tokens, heads, dim)) * size).to(dtype_of(torch, dtype)).cuda()
    if view == "slice":                                            # heads out of a wider projection
        wide = torch.full((tokens, heads + 3, dim), 7.0, dtype=x.dtype, device="cuda")
        wide[:, 2:2 + heads] = x
        return wide[:, 2:2 + heads]
    if view == "odd":                                              # rows that start at odd elements
        flat = torch.zeros(tokens * heads * (dim + 1) + 1, dtype=x.dtype, device="cuda")[1:]
        odd = flat.view(tokens, heads, dim + 1)[..., :dim]
        odd.copy_(x)
        return odd
    return x


def check(torch, rm, *, tokens, q_heads, kv_heads, dim, rot, interleaved=False, dtype="bf16", weights="f32", view="whole", amplitude=1.0, eps=1e-6,
          size=1.0, grad=True, seed=0):
    rng = np.random.default_rng(seed + dim * 7 + rot)
    table = rm.RopeTable(rot, interleaved=interleaved, amplitude=amplitude) if rot else None
    f = rm.rope_frequencies(rot) if rot else None
    pos = rng.integers(0, 1 << 20, tokens)
    if tokens:
        pos[0], pos[-1] = 0, (1 << 31) - 1
    p = torch.from_numpy(pos.astype(np.int32)).cuda() if rot else None
    x = [rows(torch, rng, tokens, h, dim, dtype, view, size) for h in (q_heads, kv_heads)]
    g = [rows(torch, rng, tokens, h, dim, dtype, view) for h in (q_heads, kv_heads)]
    w = [torch.from_numpy(rng.normal(size=dim) + 1).to(dtype_of(torch, weights)).cuda() if weights else None for _ in x]
    out = rm.qk_norm_rope(x[0], x[1], p, table, w[0], w[1], eps=eps)
    wide = [host(t) if t is not None else np.ones(dim) for t in w]
    for i in range(2):
        want, plain = npl.forward(host(x[i]), wide[i], pos, f, interleaved, amplitude, eps)
        bound = ((dim / 2 + 8) * V + (7e-7 if rot else 0)) * npl.pair_sums(plain, f, interleaved, amplitude) + U[dtype] * np.abs(want) + LEAST[dtype]
        assert out[i].shape == x[i].shape and out[i].is_contiguous()
        assert np.all(np.abs(host(out[i]) - want) <= bound), (dim, rot, i)
    mine = [t.clone() if view == "whole" else t for t in x]
    keep = [t.clone() for t in x]
    back = rm.qk_norm_rope(mine[0], mine[1], p, table, w[0], w[1], eps=eps, q_out=mine[0], k_out=mine[1])   # in place: the same bits
    assert all(b is m and torch.equal(b, o) for b, m, o in zip(back, mine, out))
    for m, k in zip(mine, keep):
        m.copy_(k)
    if not grad:
        return
    leaves = [t.detach().requires_grad_() for t in x + [t for t in w if t is not None]]
    got = rm.qk_norm_rope(leaves[0], leaves[1], p, table, *(leaves[2:] or [None, None]), eps=eps)
    assert torch.equal(got[0], out[0]) and torch.equal(got[1], out[1])
    grads = torch.autograd.grad(got, leaves, g)
    again = torch.autograd.grad(rm.qk_norm_rope(leaves[0], leaves[1], p, table, *(leaves[2:] or [None, None]), eps=eps), leaves, g)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))    # the same bits each time
    for i in range(2):
        dx, dw, size_x, size_w = npl.gradients(host(x[i]), wide[i], host(g[i]), pos, f, interleaved, amplitude, eps)
        rel = (2 * dim + 32) * V + (7e-7 if rot else 0)
        assert np.all(np.abs(host(grads[i]) - dx) <= rel * size_x + U[dtype] * np.abs(dx) + LEAST[dtype]), (dim, rot, i)
        if weights:
            n = tokens * (q_heads, kv_heads)[i]
            assert np.all(np.abs(host(grads[2 + i]) - dw) <= (rel + n * V) * size_w + U[weights] * np.abs(dw) + LEAST[weights]), (dim, rot, i)


@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (96, 32), (80, 80), (80, 40), (256, 256), (256, 64), (72, 36), (112, 112), (64, 0), (24, 8), (6, 4), (2, 2), (1, 0), (255, 254)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,weights", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", None)])
def test_norm(torch, rm, dim, rot, interleaved, dtype, weights):
    for tokens, q_heads, kv_heads, view in ((1, 1, 1, "whole"), (33, 6, 3, "whole"), (19, 5, 2, "slice"), (7, 2, 1, "odd")):
        check(torch, rm, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dim=dim, rot=rot, interleaved=interleaved, dtype=dtype, weights=weights, view=view,
              amplitude=1.0 if tokens > 1 else 1.25)


@pytest.mark.parametrize("tokens,q_heads,kv_heads", [(4097, 8, 2), (600, 64, 8), (3, 300, 1), (20011, 1, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_many_rows(torch, rm, tokens, q_heads, kv_heads, dtype):
    check(torch, rm, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dim=64, rot=64, dtype=dtype)


def test_norm_of_extremes(torch, rm):
    """Rows of zeros, of the least and of the largest numbers (their squares leave float32); an infinity or NaN stays in its row."""
    check(torch, rm, tokens=9, q_heads=3, kv_heads=2, dim=64, rot=64, dtype="f32", size=1e30, eps=1e-5)
    check(torch, rm, tokens=9, q_heads=3, kv_heads=2, dim=64, rot=32, dtype="bf16", size=1e37, grad=False)
    check(torch, rm, tokens=9, q_heads=3, kv_heads=2, dim=64, rot=64, dtype="f32", size=1e-18)
    check(torch, rm, tokens=5, q_heads=3, kv_heads=2, dim=80, rot=0, dtype="f16", size=0.0, weights="f16")
    table, p = rm.RopeTable(64), torch.arange(6, dtype=torch.int32, device="cuda")
    x = torch.randn(6, 2, 64, device="cuda")
    clean = rm.qk_norm_rope(x, None, p, table)[0]
    for bad in (float("nan"), float("inf")):
        y = x.clone()
        y[2, 1, 5] = bad
        got = rm.qk_norm_rope(y, None, p, table)[0]
        assert torch.isnan(got[2, 1, 5]) and (bad != bad or (got[2, 1] != got[2, 1])[[5, 37]].all())
        got[2, 1] = clean[2, 1]
        assert torch.equal(got, clean)


def test_norm_gradient_is_the_difference(torch, rm):
    """A step h along one element of x or w changes <y, g> by h times the gradient there: central differences of the kernel's own results in
    float32, each of 96 products off by at most 1e-5 of at most 40, over 2 h; and the third derivative's h^2 / 6 of at most 60."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda")
    table, p = rm.RopeTable(16, interleaved=True, amplitude=0.75), torch.tensor([0, 77, 100003], dtype=torch.int32, device="cuda")
    q, k, wq, wk, gq, gk = new(3, 2, 24), new(3, 1, 24), new(24), new(24), new(3, 2, 24), new(3, 1, 24)
    leaves = [t.requires_grad_() for t in (q, k, wq, wk)]
    run = lambda a: rm.qk_norm_rope(a[0], a[1], p, table, a[2], a[3])
    grads = torch.autograd.grad(run(leaves), leaves, (gq, gk))
    value = lambda a: sum(float((y.double() * g.double()).sum()) for y, g in zip(run(a), (gq, gk)))
    h = 0.0625
    for i, at in ((0, (0, 0, 3)), (0, (2, 1, 20)), (1, (1, 0, 9)), (1, (2, 0, 15)), (2, (0,)), (2, (17,)), (3, (23,)), (3, (8,))):
        sides = []
        for sign in (1, -1):
            moved = [t.detach().clone() for t in leaves]
            moved[i][at] += sign * h
            sides.append(value(moved))
        assert abs((sides[0] - sides[1]) / (2 * h) - float(grads[i][at])) < 96 * 40 * 1e-5 / (2 * h) / 10 + 60 * h * h / 6


def test_norm_gradients_of_shared_and_strided_inputs(torch, rm):
    gen = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda")
    table, p = rm.RopeTable(32), torch.tensor([3, 0, 70001, 12], dtype=torch.int32, device="cuda")
    one, k, w = new(4, 1, 48).requires_grad_(), new(4, 2, 48), new(48)
    g = new(4, 5, 48)
    rm.qk_norm_rope(one.expand(4, 5, 48), k, p, table, w, w)[0].backward(g)     # one head shared by five; k's result is not used
    full = one.detach().expand(4, 5, 48).clone().requires_grad_()
    rm.qk_norm_rope(full, None, p, table, w)[0].backward(g)
    assert torch.allclose(one.grad, full.grad.sum(1, keepdim=True), rtol=0, atol=float(8 * V * full.grad.abs().sum(1).max()))
    both = w.clone().requires_grad_()                                            # one weight for queries and keys
    q = new(4, 3, 48)
    y, z = rm.qk_norm_rope(q, k, p.tolist(), table, both, both)
    (y.sum() + z.sum()).backward()                                               # gradients with strides of zero
    apart = [w.clone().requires_grad_() for _ in range(2)]
    y, z = rm.qk_norm_rope(q, k, p, table, *apart)
    torch.autograd.backward((y, z), (torch.ones_like(y), torch.ones_like(z)))
    assert torch.equal(both.grad, apart[0].grad + apart[1].grad)
    x = new(4, 3, 48).requires_grad_()
    y = rm.qk_norm_rope(x, None, p, table)[0]
    y.backward(new(4, 48, 3).transpose(1, 2))                                    # a gradient whose last dimension is strided
    assert torch.isfinite(x.grad).all()
    with pytest.raises(RuntimeError):                                            # one derivative, no second
        gx, = torch.autograd.grad(rm.qk_norm_rope(x, None, p, table)[0].sum(), x, create_graph=True)
        torch.autograd.grad(gx.sum(), x)
    with pytest.raises(ValueError, match="gradient"):
        rm.qk_norm_rope(x, None, p, table, q_out=torch.empty_like(x))
    with torch.no_grad():
        assert not rm.qk_norm_rope(x, k, p, table, q_out=torch.empty_like(x))[0].requires_grad
    empty = torch.zeros(0, 3, 48, device="cuda", requires_grad=True)
    wg = w.clone().requires_grad_()
    rm.qk_norm_rope(empty, None, torch.zeros(0, dtype=torch.int32, device="cuda"), table, wg)[0].sum().backward()
    assert empty.grad.shape == empty.shape and not wg.grad.any()


def test_norm_on_other_streams_and_in_graphs(torch, rm):
    """A captured forward and backward pass replays with new inputs; the stream argument orders the call."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    table, p = rm.RopeTable(64), torch.arange(50, dtype=torch.int32, device="cuda")
    q, k, w, g = new(50, 4, 64), new(50, 2, 64), new(64), new(50, 4, 64)
    def step():
        a, b, c = q.detach().requires_grad_(), k.detach().requires_grad_(), w.detach().requires_grad_()
        y = rm.qk_norm_rope(a, b, p, table, c, c)
        return y + torch.autograd.grad(y, (a, b, c), (g, g[:, :2]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        q.copy_(new(50, 4, 64)); g.copy_(new(50, 4, 64))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
    torch.cuda.synchronize()
    with torch.no_grad():
        other = rm.qk_norm_rope(q, k, p, table, w, w, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(other, rm.qk_norm_rope(q, k, p, table, w, w)))


def test_norm_refusals(torch, rm):
    table, p = rm.RopeTable(64), torch.arange(4, dtype=torch.int32, device="cuda")
    q, k, w = torch.zeros(4, 4, 64, device="cuda"), torch.zeros(4, 2, 64, device="cuda"), torch.ones(64, device="cuda")
    for bad in (dict(q=q[0]), dict(k=k[:3]), dict(k=k[..., :32]), dict(k=k.half()), dict(q=q.double(), k=None), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(positions=p[:3]), dict(positions=p.long()), dict(q_weight=w[:32]), dict(q_weight=w.double()), dict(k_weight=w.half()), dict(k=None),
                dict(q_out=torch.empty(4, 4, 32, device="cuda")), dict(k_out=k.half()), dict(k=None, k_weight=None, k_out=k), dict(q=q.cpu()), dict(q_weight=w.cpu())):
        a = dict(dict(q=q, k=k, positions=p, table=table, q_weight=w, k_weight=w), **bad)
        if a["q_weight"] is not None and "k_weight" in bad:
            a["k_weight"] = bad["k_weight"]
        with pytest.raises(ValueError):
            rm.qk_norm_rope(**a)
    for bad in (dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(table=rm.RopeTable(66)), dict(q_out=q[:, :1].expand(4, 4, 64))):
        with pytest.raises(rm.RoomieError, match="invalid argument"):
            rm.qk_norm_rope(q, k, p, **dict(dict(table=table), **bad))
    with pytest.raises(rm.RoomieError, match="invalid argument"):
        rm.qk_norm_rope(torch.zeros(4, 1, 264, device="cuda"), None, None, None)
