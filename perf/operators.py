"""The serving operators' measured cases: rotary positions, appending to the 8-bit paged cache, attention over it, and the
page operations (fork, free, compact).

`own` false: the operators in elementary torch operations, in 32 bits.  `own` true: the package's entry points."""
import math
import random

import numpy as np
import torch

own = False

E4M3_MAX, INT8_MAX = 448.0, 127.0
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoding step's queries and keys (32 + 8 heads) of 48 sequences: launch latency is what counts
        dict(name="rope step", op="rope", tokens=48, heads=40, dim=128, rot=128, layout="half", factor=1.0, dtype="bf16", inverse=False, far=32768),
        # prompts of 16384 tokens, frequencies scaled for a context four times the trained one
        dict(name="rope prompt", op="rope", tokens=16384, heads=40, dim=128, rot=128, layout="half", factor=4.0, dtype="bf16", inverse=False, far=131072),
        # the gradient: float32, two thirds of an odd-sized head rotated in neighbouring pairs, a ragged token count
        dict(name="rope gradient", op="rope", tokens=6007, heads=12, dim=96, rot=64, layout="pairs", factor=1.0, dtype="f32", inverse=True, far=8192),
        # one new token for each of 64 sequences, rotated and quantised into pages that are part full
        dict(name="append step", op="append", seqs=64, new=1, ctx=4096, mix=1, q_heads=32, kv_heads=8, dim=128, page=16, fmt="e4m3", layout="hnd", rope=True, dtype="bf16"),
        # ragged prompts of up to 4096 tokens for five sequences
        dict(name="append prompts", op="append", seqs=5, new=4096, ctx=4096, mix=2, q_heads=32, kv_heads=8, dim=128, page=64, fmt="e4m3", layout="hnd", rope=True, dtype="bf16"),
        # three short conversations of a small model: launch latency
        dict(name="attention short", op="attention", seqs=3, new=1, ctx=300, mix=3, q_heads=8, kv_heads=2, dim=64, page=16, fmt="e4m3", layout="hnd", window=0, dtype="bf16"),
        # the ordinary decoding step: 64 sequences of mixed length, one slot of the batch empty
        dict(name="attention step", op="attention", seqs=64, new=1, ctx=4096, mix=4, q_heads=32, kv_heads=8, dim=128, page=16, fmt="e4m3", layout="hnd", window=0, dtype="bf16"),
        # two long documents: few rows, the key axis has to be split
        dict(name="attention long", op="attention", seqs=2, new=1, ctx=131072, mix=5, q_heads=64, kv_heads=8, dim=128, page=64, fmt="e4m3", layout="hnd", window=0, dtype="f16"),
        # chunks of up to 1024 prompt tokens over contexts of up to 8192: matrix products
        dict(name="attention prompts", op="attention", seqs=4, new=1024, ctx=8192, mix=6, q_heads=32, kv_heads=8, dim=128, page=64, fmt="e4m3", layout="hnd", window=0, dtype="bf16"),
        # a full card's step: 64 sequences of up to 16384 tokens in int8
        dict(name="attention large", op="attention", seqs=64, new=1, ctx=16384, mix=7, q_heads=32, kv_heads=8, dim=128, page=32, fmt="int8", layout="hnd", window=0, dtype="bf16"),
        # a search step: the losing continuations are freed, the winners forked (their part-filled pages copied)
        dict(name="fork and free", op="fork", layers=8, seqs=8, beams=4, ctx=2048, mix=8, kv_heads=8, dim=128, page=16, fmt="e4m3", layout="hnd"),
        # the pool is packed into its lower end after sequences left: the memory behind it can be given back
        dict(name="compact", op="compact", layers=16, seqs=48, ctx=2048, mix=9, kv_heads=8, dim=128, page=32, fmt="e4m3", layout="hnd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cache_shape(rng):
    kv = rng.choice([1, 2, 4, 8])
    return dict(kv_heads=kv, dim=rng.choice([64, 96, 128, 128, 256]), page=rng.choice([16, 32, 64, 128]),
                fmt=rng.choice(["e4m3", "e4m3", "int8"]), layout=rng.choice(["hnd", "hnd", "nhd"]), mix=rng.randrange(1, 1 << 20))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention", "fork", "compact"])
    if op == "rope":
        dim = rng.choice([64, 80, 96, 128, 256])
        rot = rng.choice([dim, dim, dim // 2])
        return dict(op=op, tokens=_log(rng, 1, 8000), heads=_log(rng, 1, 64), dim=dim, rot=rot, layout=rng.choice(["half", "pairs"]),
                    factor=rng.choice([1.0, 1.0, 4.0, 32.0]), dtype=rng.choice(["bf16", "f16", "f32"]), inverse=rng.random() < 0.3,
                    far=_log(rng, 2048, 262144))
    c = _cache_shape(rng)
    if op == "append":
        new = 1 if rng.random() < 0.4 else _log(rng, 2, 3000)
        c |= dict(op=op, seqs=_log(rng, 1, 256) if new == 1 else _log(rng, 1, 6), new=new, ctx=new + _log(rng, 1, 2000),
                  dtype=rng.choice(["bf16", "f16"]), rope=c["fmt"] == "e4m3" and rng.random() < 0.7)
        return c | dict(q_heads=c["kv_heads"] * rng.choice([1, 2, 4, 8]))
    if op == "attention":
        kind = rng.choice(["step", "step", "few", "prompt"])
        ctx = _log(rng, 1, 60000)
        seqs = _log(rng, 1, max(1, min(256, 400000 // ctx)))
        new = 1 if kind == "step" else _log(rng, 2, 16) if kind == "few" else _log(rng, 17, 900)
        if kind == "few":
            seqs = max(1, min(seqs, 200000 // ctx))
        if kind == "prompt":
            ctx, seqs = max(1, min(ctx, 8000)), min(seqs, 2)
        group = rng.choice([1, 2, 4, 5, 8, 16])
        if kind != "prompt" and seqs * ctx * c["kv_heads"] * c["dim"] > 1 << 29:
            c["kv_heads"] = 1
        if kind == "prompt":
            group = min(group, 32 // c["kv_heads"])
        return c | dict(op=op, seqs=seqs, new=new, ctx=max(ctx, new), q_heads=c["kv_heads"] * group,
                        window=rng.choice([0, 0, _log(rng, 16, 4096)]), dtype=rng.choice(["bf16", "bf16", "f16"]))
    layers = _log(rng, 1, 12)
    if op == "fork":
        return c | dict(op=op, layers=layers, seqs=_log(rng, 1, 16), beams=_log(rng, 1, 6), ctx=_log(rng, 8, 1500))
    return c | dict(op=op, layers=layers, seqs=_log(rng, 2, 40), ctx=_log(rng, 40, 1500))


def _lengths(c):
    """[(tokens in the cache, new ones among them)] of the case's sequences, by the case alone."""
    r = random.Random(c["mix"])
    got = []
    for s in range(c["seqs"]):
        new = c.get("new", 0)
        if new > 1:
            new = max(1, int(new * r.uniform(0.5, 1.0))) if s else new
        ctx = c["ctx"] if s == 0 else max(new, int(c["ctx"] * r.uniform(0.3, 1.0)))
        got.append((ctx, new))
    if c["op"] == "attention" and c["seqs"] >= 16:
        got[r.randrange(1, c["seqs"])] = (0, 1)  # a batch slot without a sequence: its row sees nothing
    return got


# --------------------------------------------------------------------------------------------------------- inputs
def _frequencies(rot, factor, context=8192):
    """Turns per position in units of 2^-64 turns; for a factor above 1 the slow ones are divided by it (by parts: those that make
    fewer than one turn over the trained context wholly, those with more than four not at all)."""
    f = 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot) / (2.0 * math.pi)
    keep = np.clip((f * context - 1.0) / (4.0 - 1.0), 0.0, 1.0)
    f = f * (keep + (1.0 - keep) / factor)
    return torch.from_numpy(np.array([int(round(x * 2.0 ** 64)) % (1 << 64) for x in f], dtype=np.uint64).view(np.int64).copy()).cuda()


def _codes(shape, fmt, gen):
    """Cache codes as they come about: values of a normal distribution over a scale that leaves the largest near the format's end."""
    out = torch.empty(shape, dtype=torch.uint8, device="cuda")
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - at)
        x = torch.randn(n, generator=gen, device="cuda")
        if fmt == "e4m3":
            flat[at:at + n] = (x * 90.0).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            flat[at:at + n] = (x * 30.0).clamp(-INT8_MAX, INT8_MAX).round().to(torch.int8).view(torch.uint8)
    return out


def _pool(c, num_pages, layers, gen):
    h, t, d = c["kv_heads"], c["page"], c["dim"]
    shape = (layers, num_pages, h, t, d) if c["layout"] == "hnd" else (layers, num_pages, t, h, d)
    unit = 2.0 ** -6 if c["fmt"] == "e4m3" else 2.0 ** -5
    scale = lambda: unit * 2.0 ** torch.randint(-1, 2, (layers, num_pages, h), generator=gen, device="cuda").float()
    return dict(k=_codes(shape, c["fmt"], gen), v=_codes(shape, c["fmt"], gen), k_scale=scale(), v_scale=scale())


def _tables(lengths, page, num_pages, order, rows=None):
    """Page tables (-1 past the end) and reference counts: sequence after sequence takes the next pages of `order`."""
    used = [-(-n // page) for n in lengths]
    width = max(1, max(used))
    table = torch.full((rows or len(lengths), width), -1, dtype=torch.int32)
    refs = torch.zeros(num_pages, dtype=torch.int32)
    at = 0
    for s, n in enumerate(used):
        table[s, :n] = order[at:at + n]
        refs[order[at:at + n].long()] = 1
        at += n
    return table, refs


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    op = case["op"]
    s = dict(case=case, op=op)
    if op == "rope":
        shape = (case["tokens"], case["heads"], case["dim"])
        s["x"] = torch.randn(shape, generator=gen, device="cuda").to(DTYPES[case["dtype"]])
        s["positions"] = torch.randint(0, case["far"], (case["tokens"],), generator=gen, device="cuda", dtype=torch.int32)
        s["frequency"] = _frequencies(case["rot"], case["factor"])
        if own:
            import paper_2607_16784_b200 as rm
            s["table"] = rm.RopeTable.from_tensor(s["frequency"], interleaved=case["layout"] == "pairs")
        return s

    sizes = _lengths(case)
    length = [n for n, _ in sizes]
    page = case["page"]
    need = sum(-(-n // page) for n in length)
    if op == "fork":
        need += case["seqs"] * case["beams"]
    num_pages = need + need // 8 + 3 if op != "compact" else int(need * 1.5) + 5
    order = torch.randperm(num_pages, generator=host).to(torch.int32)
    layers = case.get("layers", 1)
    s |= _pool(case, num_pages, layers, gen)
    slots = case["seqs"] * (1 + case["beams"]) if op == "fork" else case["seqs"]
    table, refs = _tables(length, page, num_pages, order, slots)
    s |= dict(pages=table.cuda(), refs=refs.cuda(), widest=table.shape[1])
    s["length"] = torch.tensor(length + [0] * (slots - len(length)), dtype=torch.int32, device="cuda")
    if op in ("append", "attention"):
        news = [n for _, n in sizes]
        rows = sum(news)
        s |= dict(rows=rows, most=max(news), seqs=torch.arange(case["seqs"], dtype=torch.int32, device="cuda"))
        s["q_offset"] = torch.tensor(np.concatenate([[0], np.cumsum(news)]).tolist(), dtype=torch.int32, device="cuda")
        dtype = DTYPES[case["dtype"]]
        s["q"] = torch.randn((rows, case["q_heads"], case["dim"]), generator=gen, device="cuda").to(dtype)
        if op == "append":
            s["new_k"] = torch.randn((rows, case["kv_heads"], case["dim"]), generator=gen, device="cuda").mul_(1.5).to(dtype)
            s["new_v"] = torch.randn((rows, case["kv_heads"], case["dim"]), generator=gen, device="cuda").to(dtype)
            s["frequency"] = _frequencies(case["dim"], 1.0)
    elif op == "fork":
        n, b = case["seqs"], case["beams"]
        s["parents"] = torch.arange(n, dtype=torch.int32).repeat_interleave(b).cuda()
        s["children"] = torch.arange(n, n + n * b, dtype=torch.int32, device="cuda")
        _plain_fork(s)  # the continuations of the step before: each pass frees them and forks anew
    if own:
        import paper_2607_16784_b200 as rm
        s["cache"] = rm.KVCache.from_tensors(s["k"], s["v"], s["k_scale"], s["v_scale"], s["refs"], s["pages"], s["length"],
                                             fmt=case["fmt"], layout=case["layout"])
        s["workspace"] = s["cache"].workspace()
        if op == "append":
            s["table"] = rm.RopeTable.from_tensor(s["frequency"], interleaved=False) if case["rope"] else None
        if op == "compact":
            s["refs_out"], s["pages_out"] = torch.empty_like(s["refs"]), torch.empty_like(s["pages"])
    return s


# ----------------------------------------------------------------------------------------------------- plain forms
def _plain_rotate(x, phase, layout, amplitude=1.0, inverse=False):
    """x [tokens, heads, dim] in 32 bits; phase [tokens, r / 2] in turns."""
    half = phase.shape[1]
    angle = phase * (2.0 * math.pi)
    cos, sin = torch.cos(angle)[:, None, :] * amplitude, torch.sin(angle)[:, None, :] * amplitude
    if inverse:
        sin = -sin
    y = x.clone()
    a, b = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _plain_phase(positions, frequency):
    """Turns in [-1/2, 1/2): the product wraps at whole turns."""
    return ((positions.long()[:, None] * frequency[None, :]) >> 32).float() * 2.0 ** -32


def _plain_values(codes, fmt):
    return codes.view(torch.float8_e4m3fn).float() if fmt == "e4m3" else codes.view(torch.int8).float()


def _plain_scale(amax, top):
    """The least power of two s with amax / s <= top, within 2^-100 .. 2^120."""
    mantissa, exponent = torch.frexp(amax)
    share, bits = math.frexp(top)
    e = torch.where(amax > 0, exponent - bits + (mantissa > share).int(), -100)
    return torch.ldexp(torch.ones_like(amax), e.clamp(-100, 120))


def _plain_quantise(x, fmt):
    if fmt == "e4m3":
        return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
    return x.clamp(-INT8_MAX, INT8_MAX).round().to(torch.int8).view(torch.uint8)


def _plain_append(s):
    case = s["case"]
    page, fmt, hnd = case["page"], case["fmt"], case["layout"] == "hnd"
    top = E4M3_MAX if fmt == "e4m3" else INT8_MAX
    row = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(s["q_offset"][1:].long(), row, right=True)
    count = (s["q_offset"][1:] - s["q_offset"][:-1]).long()
    start = s["length"].long() - count
    position = start[seq] + row - s["q_offset"][:-1].long()[seq]
    k, v, q = s["new_k"].float(), s["new_v"].float(), s["q"]
    if case["rope"]:
        phase = _plain_phase(position, s["frequency"])
        k = _plain_rotate(k, phase, "half")
        q = _plain_rotate(q.float(), phase, "half").to(s["q"].dtype)
    at, inside = s["pages"].long()[seq, position // page], position % page
    first = s["pages"].long().gather(1, (start // page).clamp(max=s["widest"] - 1)[:, None])[:, 0]  # the page a sequence's first new token goes to
    held = start % page
    token = torch.arange(page, device="cuda")
    for name, x in (("k", k), ("v", v)):
        pool, scale = s[name][0], s[name + "_scale"][0]
        amax = torch.zeros_like(scale).scatter_reduce_(0, at[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
        old = scale[first]
        touched = torch.zeros(scale.shape[0], dtype=torch.bool, device="cuda")
        touched[at] = True
        fresh = _plain_scale(amax, top)
        keep = torch.zeros_like(scale)
        keep[first] = torch.where((held > 0)[:, None], old, 0.0)
        fresh = torch.maximum(fresh, keep)
        ratio = (old / fresh[first]) if hnd else (old / fresh[first])[:, None, :]
        before = pool[first]
        again = _plain_quantise(_plain_values(before, fmt) * (ratio[:, :, None, None] if hnd else ratio[..., None]), fmt)
        earlier = (token[None, :] < held[:, None])
        earlier = earlier[:, None, :, None] if hnd else earlier[:, :, None, None]
        pool[first] = torch.where(earlier, again, before)
        scale.copy_(torch.where(touched[:, None], fresh, scale))
        codes = _plain_quantise(x / fresh[at][..., None], fmt)
        if hnd:
            pool[at, :, inside] = codes
        else:
            pool[at, inside] = codes
    return q


def _plain_attention(s):
    case = s["case"]
    hq, h, d, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    b, g, most = case["seqs"], hq // h, s["most"]
    at = s["pages"].long().clamp(min=0)
    tokens = at.shape[1] * page

    def gathered(name):
        x = _plain_values(s[name][0][at], case["fmt"])
        sc = s[name + "_scale"][0][at]
        if case["layout"] == "hnd":
            return (x * sc[..., None, None]).permute(0, 2, 1, 3, 4).reshape(b, h, tokens, d)
        return (x * sc[:, :, None, :, None]).permute(0, 3, 1, 2, 4).reshape(b, h, tokens, d)

    count = (s["q_offset"][1:] - s["q_offset"][:-1]).long()
    step = torch.arange(most, device="cuda")
    there = step[None, :] < count[:, None]
    row = (s["q_offset"][:-1].long()[:, None] + step[None, :]).clamp(max=s["rows"] - 1)
    q = s["q"][row].float().reshape(b, most, h, g, d).permute(0, 2, 1, 3, 4).reshape(b, h, most * g, d)
    length = s["length"].long()
    position = (length - count)[:, None] + step[None, :]
    key = torch.arange(tokens, device="cuda")
    seen = (key[None, None, :] <= position[..., None]) & (key[None, None, :] < length[:, None, None]) & there[..., None]
    if case["window"]:
        seen &= key[None, None, :] > position[..., None] - case["window"]
    seen = seen[:, None, :, None, :].expand(b, 1, most, g, tokens).reshape(b, 1, most * g, tokens)
    logit = (q @ gathered("k").transpose(2, 3)).mul_(1.0 / math.sqrt(d)).masked_fill_(~seen, -math.inf)
    top = logit.amax(-1, keepdim=True)
    p = logit.sub_(torch.where(top.isinf(), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ gathered("v")) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).reshape(b, h, most, g).permute(0, 2, 1, 3).reshape(b, most, hq)
    o = o.reshape(b, h, most, g, d).permute(0, 2, 1, 3, 4).reshape(b, most, hq, d)
    out = torch.empty((s["rows"], hq, d), dtype=s["q"].dtype, device="cuda")
    out_lse = torch.empty((s["rows"], hq), dtype=torch.float32, device="cuda")
    put = torch.where(there, row, s["rows"]).reshape(-1)  # rows that are not there go to a row behind the last
    out = torch.cat([out, out[:1]]).index_copy_(0, put, o.reshape(b * most, hq, d).to(out.dtype))[: s["rows"]]
    out_lse = torch.cat([out_lse, out_lse[:1]]).index_copy_(0, put, lse.reshape(b * most, hq))[: s["rows"]]
    return out, out_lse


def _plain_free(s, which):
    which = which.long()
    rows = s["pages"][which]
    held = -(-s["length"][which].long() // s["case"]["page"])
    there = torch.arange(rows.shape[1], device="cuda")[None, :] < held[:, None]
    s["refs"].index_add_(0, rows.long().clamp(min=0).reshape(-1), -there.int().reshape(-1))
    s["pages"][which] = -1
    s["length"][which] = 0


def _plain_fork(s):
    page = s["case"]["page"]
    parent, child = s["parents"].long(), s["children"].long()
    length = s["length"][parent].long()
    part = length % page != 0
    held = -(-length // page)
    free = torch.argsort((s["refs"] != 0).int(), stable=True)  # the free pages, lowest first
    fresh = free[(torch.cumsum(part.long(), 0) - 1).clamp(min=0)]
    rows = s["pages"][parent]
    step = torch.arange(rows.shape[1], device="cuda")
    last = (held - 1).clamp(min=0)
    old = rows.long().gather(1, last[:, None])[:, 0]
    shared = step[None, :] < (held - part.long())[:, None]
    s["refs"].index_add_(0, rows.long().clamp(min=0).reshape(-1), shared.int().reshape(-1))
    s["refs"][fresh[part]] = 1
    rows.scatter_(1, last[:, None], torch.where(part, fresh, old)[:, None].int())
    for name in ("k", "v", "k_scale", "v_scale"):
        s[name][:, fresh[part]] = s[name][:, old[part]]
    s["pages"][child] = rows
    s["length"][child] = length.int()


def _plain_compact(s):
    refs, pages = s["refs"], s["pages"]
    used = refs > 0
    index = torch.arange(refs.numel(), device="cuda")
    total = used.sum()
    source = (used & (index >= total)).nonzero()[:, 0]
    hole = (~used & (index < total)).nonzero()[:, 0]
    place = index.clone()
    place[source] = hole
    for name in ("k", "v", "k_scale", "v_scale"):
        s[name][:, hole] = s[name][:, source]
    refs_out = refs.clone()
    refs_out[hole] = refs[source]
    refs_out[source] = 0
    pages_out = torch.where(pages >= 0, place[pages.long().clamp(min=0)].int(), pages)
    return refs_out, pages_out


def _codes_out(s, name):
    return s[name].view(torch.float8_e4m3fn) if s["case"]["fmt"] == "e4m3" else s[name].view(torch.int8)


def run(state):
    s, case = state, state["case"]
    if own:
        import paper_2607_16784_b200 as rm
    if s["op"] == "rope":
        if own:
            return rm.rope(s["x"], s["positions"], s["table"], inverse=case["inverse"])
        return _plain_rotate(s["x"].float(), _plain_phase(s["positions"], s["frequency"]), case["layout"], 1.0, case["inverse"]).to(s["x"].dtype)
    if s["op"] == "append":
        q = rm.kv_append(s["cache"], s["seqs"], s["new_k"], s["new_v"], s["q_offset"], rope=s["table"], q=s["q"]) if own else _plain_append(s)
        return dict(q=q, k=_codes_out(s, "k"), v=_codes_out(s, "v"), k_scale=s["k_scale"], v_scale=s["v_scale"])
    if s["op"] == "attention":
        if own:
            out, lse = rm.kv_attention(s["cache"], s["seqs"], s["q"], s["q_offset"], window=case["window"], workspace=s["workspace"])
        else:
            out, lse = _plain_attention(s)
        return dict(out=out, lse=lse)
    if s["op"] == "fork":
        if own:
            rm.kv_free(s["cache"], s["children"])
            rm.kv_fork(s["cache"], s["parents"], s["children"], workspace=s["workspace"])
        else:
            _plain_free(s, s["children"])
            _plain_fork(s)
        refs, pages = s["refs"], s["pages"]
    else:
        if own:
            refs, pages = s["refs_out"], s["pages_out"]
            rm.kv_compact(s["cache"], refs_out=refs, pages_out=pages, workspace=s["workspace"])
        else:
            refs, pages = _plain_compact(s)
    return dict(refs=refs, pages=pages, length=s["length"], k=_codes_out(s, "k"), v=_codes_out(s, "v"), k_scale=s["k_scale"], v_scale=s["v_scale"])


# ------------------------------------------------------------------------------------------------- the least of work
def work(case):
    op = case["op"]
    if op == "rope":
        n = case["tokens"] * case["heads"]
        return dict(bytes=2.0 * n * case["dim"] * SIZES[case["dtype"]] + 4.0 * case["tokens"], flops=3.0 * n * case["rot"])
    h, d, page = case["kv_heads"], case["dim"], case["page"]
    sizes = _lengths(case)
    if op == "append":
        rows, e = sum(n for _, n in sizes), SIZES[case["dtype"]]
        moved = rows * d * (2 * h * e + 2 * h + (2 * case["q_heads"] * e if case["rope"] else 0))
        return dict(bytes=float(moved + rows * 4), flops=rows * d * (4.0 * h + 3.0 * (h + case["q_heads"]) * case["rope"]))
    if op == "attention":
        tokens = pairs = 0
        for length, new in sizes:
            start, window = length - new, case["window"]
            lowest = max(0, start - window + 1) if window else 0
            tokens += max(0, length - lowest)
            pairs += sum(min(p + 1, window) if window else p + 1 for p in range(max(0, start), length))
        rows = sum(n for _, n in sizes)
        moved = tokens * h * 2 * d + 8 * h * -(-tokens // page) + rows * case["q_heads"] * (2 * d * SIZES[case["dtype"]] + 4)
        return dict(bytes=float(moved), flops=4.0 * d * case["q_heads"] * pairs)
    one = case["layers"] * 2 * h * (page * d + 4)  # a page's bytes over all layers
    entries = sum(-(-n // page) for n, _ in sizes)
    if op == "fork":
        moved = sum(case["beams"] for n, _ in sizes if n % page)
        return dict(bytes=2.0 * one * moved + 12.0 * entries * (1 + case["beams"]), flops=1.0 * entries)
    total = int(entries * 1.5) + 5
    moved = entries * (total - entries) / total  # of a random third's holes: as many as used pages lie behind the new end
    return dict(bytes=2.0 * one * moved + 8.0 * (entries + total), flops=1.0 * total)


# --------------------------------------------------------------------------------------------- values in 64 bits
def _exact_values(codes, fmt):
    if fmt == "int8":
        c = codes.long()
        return torch.where(c > 127, c - 256, c).double()
    bits = np.arange(256)
    e, m = (bits >> 3) & 15, bits & 7
    value = np.where(e > 0, (1.0 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    return torch.from_numpy(np.where(bits > 127, -value, value)).cuda()[codes.long()]


def _exact_turn(x, turns, layout, inverse):
    """x [..., heads, dim], turns [..., r / 2]; each pair as a complex number."""
    half = turns.shape[-1]
    w = torch.polar(torch.ones_like(turns), 2.0 * math.pi * (-turns if inverse else turns))[..., None, :]
    y = x.clone()
    if layout == "half":
        z = torch.complex(x[..., :half], x[..., half:2 * half]) * w
        y[..., :half], y[..., half:2 * half] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :2 * half].unflatten(-1, (half, 2)).contiguous()) * w
        y[..., :2 * half] = torch.view_as_real(z).flatten(-2)
    return y


def _exact_turns(positions, frequency):
    """Fractions of a turn in 64 bits: the high and low halves of the frequency apart."""
    high, low = (frequency >> 32) & 0xFFFFFFFF, frequency & 0xFFFFFFFF
    p = positions.long()[:, None]
    return ((p * high) % (1 << 32)).double() * 2.0 ** -32 + (p * low).double() * 2.0 ** -64


def _exact_round(y, fmt):
    if fmt == "int8":
        return y.round().clamp(-127, 127)
    exponent = (torch.frexp(y.abs())[1] - 1).clamp(min=-6).double()
    unit = torch.exp2(exponent - 3.0)
    return ((y / unit).round() * unit).clamp(-448.0, 448.0)


def _exact_append(s):
    case, page, hnd = s["case"], s["case"]["page"], s["case"]["layout"] == "hnd"
    top = 448.0 if case["fmt"] == "e4m3" else 127.0
    offset, length = s["q_offset"].tolist(), s["length"].tolist()
    pages = s["pages"].long().cpu()
    got = {}
    q_out = s["q"].double() if not case["rope"] else None
    turned = []
    for name, fresh in (("k", s["new_k"]), ("v", s["new_v"])):
        pool, scale = _exact_values(s[name][0], case["fmt"]), s[name + "_scale"][0].double()
        pool = pool if hnd else pool.transpose(1, 2)
        for i in range(case["seqs"]):
            lo, hi = offset[i], offset[i + 1]
            start = length[i] - (hi - lo)
            x = fresh[lo:hi].double()
            if case["rope"]:
                turns = _exact_turns(torch.arange(start, length[i], device="cuda"), s["frequency"])
                if name == "k":
                    x = _exact_turn(x, turns, "half", False)
                    turned.append(_exact_turn(s["q"][lo:hi].double(), turns, "half", False))
            # whole pages: the sequence's first new page may hold earlier tokens
            first = start // page
            n = -(-length[i] // page) - first
            at = pages[i, first:first + n].cuda()
            held = start - first * page
            block = torch.zeros((n * page,) + x.shape[1:], dtype=torch.float64, device="cuda")
            block[held:held + hi - lo] = x
            block = block.unflatten(0, (n, page)).transpose(1, 2)  # [pages, heads, tokens, dim]
            amax = block.abs().amax((2, 3))
            exponent = torch.ceil(torch.log2(torch.where(amax > 0, amax / top, 2.0 ** -100))).clamp(-100, 120)
            unit = torch.exp2(exponent)
            if held:
                unit[0] = torch.maximum(unit[0], scale[at[0]])
                block[0, :, :held] = pool[at[0], :, :held] * scale[at[0]][:, None, None]
            codes = _exact_round(block / unit[..., None, None], case["fmt"])
            new = torch.zeros((n * page,), dtype=torch.bool, device="cuda")
            new[:held + hi - lo] = True
            new = new.unflatten(0, (n, page))[:, None, :, None]
            pool[at] = torch.where(new, codes, pool[at])
            scale[at] = unit
        got[name], got[name + "_scale"] = (pool if hnd else pool.transpose(1, 2))[None], scale[None]
        if case["fmt"] == "int8":
            got[name] = got[name].to(torch.int8)
    got["q"] = q_out if q_out is not None else torch.cat(turned)
    return got


def _exact_attention(s):
    case = s["case"]
    h, page, d = case["kv_heads"], case["page"], case["dim"]
    g = case["q_heads"] // h
    offset, length = s["q_offset"].tolist(), s["length"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for i in range(case["seqs"]):
        lo, hi, n = offset[i], offset[i + 1], length[i]
        if n == 0:
            continue
        at = s["pages"][i, :-(-n // page)].long()
        for head in range(h):
            take = (lambda name: s[name][0][at, head]) if case["layout"] == "hnd" else (lambda name: s[name][0][at, :, head])
            k, v = (( _exact_values(take(name), case["fmt"]) * s[name + "_scale"][0][at, head].double()[:, None, None]).reshape(-1, d)[:n] for name in ("k", "v"))
            q = s["q"][lo:hi, head * g:(head + 1) * g].double()
            logit = torch.einsum("rgd,td->rgt", q, k) / math.sqrt(d)
            position = torch.arange(n - (hi - lo), n, device="cuda")[:, None]
            key = torch.arange(n, device="cuda")[None, :]
            hidden = key > position
            if case["window"]:
                hidden |= key <= position - case["window"]
            logit.masked_fill_(hidden[:, None, :], -math.inf)
            empty = hidden.all(-1)
            lse[lo:hi, head * g:(head + 1) * g] = torch.logsumexp(logit, -1)
            p = torch.softmax(logit, -1)
            p[empty] = 0.0
            out[lo:hi, head * g:(head + 1) * g] = torch.einsum("rgt,td->rgd", p, v)
    return dict(out=out, lse=lse)


def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None  # whole numbers and copies: the plain form's values are the values
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_turn(s["x"].double(), _exact_turns(s["positions"], s["frequency"]), case["layout"], case["inverse"])
    return _exact_append(s) if case["op"] == "append" else _exact_attention(s)
