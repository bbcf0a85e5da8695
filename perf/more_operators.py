"""More of the serving operators' measured cases: normed and rotated queries and keys with their gradients, beam search's selection and the
reordering of the cached sequences, the attention weight that cached keys have received, and eviction by it.

`own` false: the operators in elementary torch operations, in 32 bits (64 where the order of near values matters).  `own` true: the
package's entry points."""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoding step's queries and keys of 48 sequences: launch latency is what counts
        dict(name="norm step", op="norm", tokens=48, q_heads=32, kv_heads=8, dim=128, rot=128, layout="half", dtype="bf16", grad=False, far=32768),
        # prompts of 16384 tokens
        dict(name="norm prompt", op="norm", tokens=16384, q_heads=32, kv_heads=8, dim=128, rot=128, layout="half", dtype="bf16", grad=False, far=131072),
        # a training step over a ragged number of tokens: forward, and the gradients of both inputs and both weights
        dict(name="norm gradient", op="norm", tokens=8191, q_heads=16, kv_heads=4, dim=96, rot=64, layout="pairs", dtype="bf16", grad=True, far=8192),
        # four requests with four beams each: latency
        dict(name="beam step", op="beam", requests=4, beams=4, vocab=32000, num=8, dtype="bf16", ended=0.0, mix=1),
        # odd sizes, float32 logits, some beams already ended, some words forbidden
        dict(name="beam ragged", op="beam", requests=7, beams=5, vocab=50257, num=10, dtype="f32", ended=0.2, mix=2),
        # a full batch over a large vocabulary
        dict(name="beam large", op="beam", requests=64, beams=4, vocab=128256, num=8, dtype="bf16", ended=0.0, mix=3),
        # the cache follows the winners: eight requests with four beams that share their prompt
        dict(name="reorder step", op="reorder", layers=8, requests=8, beams=4, prompt=1024, own_tokens=100, kv_heads=8, dim=128, page=16, fmt="e4m3", layout="hnd", mix=4),
        # many beams of many layers
        dict(name="reorder large", op="reorder", layers=16, requests=32, beams=8, prompt=2048, own_tokens=200, kv_heads=8, dim=128, page=32, fmt="e4m3", layout="hnd", mix=5),
        # each decoding step's share of the weights: 64 sequences of mixed length
        dict(name="weights step", op="weights", seqs=64, new=1, ctx=4096, q_heads=32, kv_heads=8, dim=128, page=16, fmt="e4m3", layout="hnd", window=0, fresh=False, dtype="bf16", mix=6),
        # the last 64 queries of a prompt weigh all of its keys
        dict(name="weights window", op="weights", seqs=4, new=64, ctx=16384, q_heads=32, kv_heads=8, dim=128, page=64, fmt="e4m3", layout="hnd", window=0, fresh=True, dtype="bf16", mix=7),
        # eight short conversations are held to 1024 tokens, four layers
        dict(name="evict step", op="evict", layers=4, seqs=8, ctx=1280, keep=1024, first=4, recent=128, kv_heads=8, dim=128, page=16, fmt="e4m3", layout="hnd", mix=8),
        # prompts of up to 8192 tokens are cut to 2048, sixteen layers
        dict(name="evict prompts", op="evict", layers=16, seqs=16, ctx=8192, keep=2048, first=4, recent=256, kv_heads=8, dim=128, page=32, fmt="e4m3", layout="hnd", mix=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "beam", "beam", "reorder", "weights", "weights", "evict"])
    kv = rng.choice([1, 2, 4, 8])
    if op == "norm":
        dim = rng.choice([64, 80, 96, 128, 256])
        grad = rng.random() < 0.5
        return dict(op=op, tokens=_log(rng, 1, 3000 if grad else 8000), q_heads=kv * rng.choice([1, 2, 4]), kv_heads=kv, dim=dim, rot=rng.choice([dim, dim, dim // 2]),
                    layout=rng.choice(["half", "pairs"]), dtype=rng.choice(["bf16", "f16", "f32"]), grad=grad, far=_log(rng, 2048, 262144))
    if op == "beam":
        requests, beams = _log(rng, 1, 32), rng.choice([1, 2, 3, 4, 6, 8])
        vocab = _log(rng, 1000, 200000)
        while requests * beams * vocab > 16 << 20:
            requests = max(1, requests // 2)
            beams = max(1, beams - 1)
        return dict(op=op, requests=requests, beams=beams, vocab=vocab, num=rng.choice([beams, 2 * beams]), dtype=rng.choice(["bf16", "f16", "f32"]),
                    ended=rng.choice([0.0, 0.0, 0.3]), mix=rng.randrange(1, 1 << 20))
    c = dict(op=op, kv_heads=kv, dim=rng.choice([64, 96, 128, 128, 256]), page=rng.choice([16, 32, 64, 128]), fmt=rng.choice(["e4m3", "e4m3", "int8"]),
             layout=rng.choice(["hnd", "hnd", "nhd"]), mix=rng.randrange(1, 1 << 20))
    if op == "reorder":
        return c | dict(layers=_log(rng, 1, 8), requests=_log(rng, 1, 16), beams=rng.choice([2, 3, 4, 8]), prompt=_log(rng, 1, 2000), own_tokens=_log(rng, 1, 300))
    if op == "weights":
        new = 1 if rng.random() < 0.5 else _log(rng, 2, 128)
        ctx = max(new, _log(rng, 1, 16000))
        seqs = _log(rng, 1, max(1, min(64, (200000 if new == 1 else 20000) // ctx)))
        return c | dict(seqs=seqs, new=new, ctx=ctx, q_heads=kv * rng.choice([1, 2, 4, 5, 8] if new == 1 else [1, 2, 4]), window=rng.choice([0, 0, _log(rng, 16, 4096)]),
                        fresh=new > 1, dtype=rng.choice(["bf16", "bf16", "f16"]))
    ctx = _log(rng, 64, 6000)
    keep = max(2, int(ctx * rng.uniform(0.2, 0.9)))
    return c | dict(layers=_log(rng, 1, 8), seqs=_log(rng, 1, max(1, min(24, 40000 // ctx))), ctx=ctx, keep=keep, first=rng.choice([0, 1, min(4, keep // 8)]), recent=int(keep * rng.uniform(0.0, 0.5)))


def _lengths(c):
    """Tokens in the cache of each of the case's sequences, by the case alone."""
    r = random.Random(c["mix"])
    if c["op"] == "reorder":
        return [c["prompt"] + max(1, int(c["own_tokens"] * r.uniform(0.3, 1.0))) for _ in range(c["requests"])]
    return [c["ctx"] if s == 0 else max(c.get("new", 1), int(c["ctx"] * r.uniform(0.3, 1.0))) for s in range(c["seqs"])]


def _parents(c):
    """Where each beam of a reordering comes from: the best beams have several continuations, others none."""
    r = random.Random(c["mix"] + 1)
    b = c["beams"]
    return [q * b + (i if i == 0 else min(b - 1, int(b * r.random() ** 2))) for q in range(c["requests"]) for i in range(b)]


# --------------------------------------------------------------------------------------------------------- inputs
def _frequencies(rot):
    """Turns per position in units of 2^-64 turns."""
    f = 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot) / (2.0 * math.pi)
    return torch.from_numpy(np.array([int(round(x * 2.0 ** 64)) % (1 << 64) for x in f], dtype=np.uint64).view(np.int64).copy()).cuda()


def _codes(shape, fmt, gen):
    """Cache codes as they come about: values of a normal distribution over a scale that leaves the largest near the format's end."""
    out = torch.empty(shape, dtype=torch.uint8, device="cuda")
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - at)
        x = torch.randn(n, generator=gen, device="cuda")
        if fmt == "e4m3":
            flat[at:at + n] = (x * 90.0).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            flat[at:at + n] = (x * 30.0).clamp(-127.0, 127.0).round().to(torch.int8).view(torch.uint8)
    return out


def _pool(c, num_pages, layers, gen):
    h, t, d = c["kv_heads"], c["page"], c["dim"]
    shape = (layers, num_pages, h, t, d) if c["layout"] == "hnd" else (layers, num_pages, t, h, d)
    unit = 2.0 ** -6 if c["fmt"] == "e4m3" else 2.0 ** -5
    scale = lambda: unit * 2.0 ** torch.randint(-1, 2, (layers, num_pages, h), generator=gen, device="cuda").float()
    return dict(k=_codes(shape, c["fmt"], gen), v=_codes(shape, c["fmt"], gen), k_scale=scale(), v_scale=scale())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    op = case["op"]
    s = dict(case=case, op=op)
    if own:
        import paper_2607_16784_b200 as rm
    if op == "norm":
        dtype, n, d = DTYPES[case["dtype"]], case["tokens"], case["dim"]
        new = lambda heads, size: torch.randn((n, heads, d), generator=gen, device="cuda").mul_(size).to(dtype)
        s["q"], s["k"] = new(case["q_heads"], 3.0), new(case["kv_heads"], 3.0)
        s["wq"], s["wk"] = (1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
        s["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device="cuda", dtype=torch.int32)
        s["frequency"] = _frequencies(case["rot"])
        if case["grad"]:
            s["gq"], s["gk"] = new(case["q_heads"], 1.0), new(case["kv_heads"], 1.0)
        if own:
            s["table"] = rm.RopeTable.from_tensor(s["frequency"], interleaved=case["layout"] == "pairs")
            if case["grad"]:
                for name in ("q", "k", "wq", "wk"):
                    s[name].requires_grad_()
        return s
    if op == "beam":
        r, b, v = case["requests"], case["beams"], case["vocab"]
        logits = torch.randn((r, b, v), generator=gen, device="cuda").mul_(2.5)
        lead = torch.randint(0, v, (r, b, 24), generator=gen, device="cuda")  # a few likely words
        logits.scatter_add_(2, lead, torch.rand((r, b, 24), generator=gen, device="cuda") * 12.0)
        logits[..., v - v // 50:] = -math.inf                                 # words that are forbidden here
        s["logits"] = logits.to(DTYPES[case["dtype"]])
        s["scores"] = -torch.rand((r, b), generator=gen, device="cuda") * 20.0
        s["ended"] = torch.rand((r, b), generator=gen, device="cuda") < case["ended"] if case["ended"] else None
        if own:
            s["workspace"] = rm.beam_workspace(r, b, v, case["num"], s["logits"].dtype)
        return s

    page, lengths, layers = case["page"], _lengths(case), case.get("layers", 1)
    used = lambda n: -(-n // page)
    if op == "reorder":
        b = case["beams"]
        whole = case["prompt"] // page                                        # pages that the beams of a request share
        lengths = [n for n in lengths for _ in range(b)]
        need = sum(used(n) - whole for n in lengths) + case["requests"] * whole
    else:
        need = sum(used(n) for n in lengths)
    num_pages = need + need // 8 + 3 + (len(lengths) if op == "reorder" else 0)
    order = torch.randperm(num_pages, generator=host).to(torch.int32)
    width = max(used(n) for n in lengths)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    refs = torch.zeros(num_pages, dtype=torch.int32)
    at = 0
    for i, n in enumerate(lengths):
        shared = 0
        if op == "reorder" and i % b:
            shared = whole
            table[i, :whole] = table[i - i % b, :whole]
        table[i, shared:used(n)] = order[at:at + used(n) - shared]
        at += used(n) - shared
    refs.index_add_(0, table[table >= 0].long(), torch.ones(int((table >= 0).sum()), dtype=torch.int32))
    s |= _pool(case, num_pages, layers, gen)
    s |= dict(pages=table.cuda(), refs=refs.cuda(), widest=width)
    s["length"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["seqs"] = torch.arange(len(lengths), dtype=torch.int32, device="cuda")
    if op == "reorder":
        s["parents"] = torch.tensor(_parents(case), dtype=torch.int32, device="cuda")
    else:
        shape = (layers, len(lengths), case["kv_heads"], width * page)
        s["weight"] = torch.rand(shape, generator=gen, device="cuda").pow_(4.0)  # few keys have received much
    if op == "evict":
        s["weight_out"] = torch.zeros_like(s["weight"])
        s["want"] = s["length"].clone()
    if op == "weights":
        rows, hq, d = case["seqs"] * case["new"], case["q_heads"], case["dim"]
        s["rows"] = rows
        s["q_offset"] = torch.arange(0, rows + 1, case["new"], dtype=torch.int32, device="cuda")
        s["q"] = torch.randn((rows, hq, d), generator=gen, device="cuda").to(DTYPES[case["dtype"]])
        s["lse"] = torch.empty((rows, hq), dtype=torch.float32, device="cuda")
        for i in range(case["seqs"]):                                            # what attention over these keys returned
            logit = _plain_logits(s, i)
            s["lse"][i * case["new"]:(i + 1) * case["new"]] = torch.logsumexp(logit, -1).permute(1, 0, 2).reshape(case["new"], hq)
    if own:
        s["cache"] = rm.KVCache.from_tensors(s["k"], s["v"], s["k_scale"], s["v_scale"], s["refs"], s["pages"], s["length"], fmt=case["fmt"], layout=case["layout"])
        s["workspace"] = s["cache"].workspace()
    return s


# ----------------------------------------------------------------------------------------------------- plain forms
def _plain_angles(s):
    """Cosines and sines [tokens, 1, r / 2]: the product of position and frequency wraps at whole turns."""
    angle = ((s["positions"].long()[:, None] * s["frequency"][None, :]) >> 32).float() * (2.0 ** -32 * 2.0 * math.pi)
    return torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]


def _plain_turn(x, cos, sin, layout):
    half = cos.shape[-1]
    a, b = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    y = x.clone()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _plain_norm(s):
    layout, got = s["case"]["layout"], {}
    cos, sin = _plain_angles(s)
    for n in ("q", "k"):
        x, w = s[n].float(), s["w" + n]
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        got[n] = _plain_turn(x * r * w, cos, sin, layout).to(s[n].dtype)
        if s["case"]["grad"]:
            g = _plain_turn(s["g" + n].float(), cos, -sin, layout)
            unit, gw = x * r, g * w
            got["dw" + n] = (g * unit).sum((0, 1))
            got["d" + n] = (r * (gw - unit * (gw * unit).mean(-1, keepdim=True))).to(s[n].dtype)
    return got


def _plain_beam(s):
    case = s["case"]
    r, b, v, num = case["requests"], case["beams"], case["vocab"], case["num"]
    out = [torch.empty((r, num), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
    for i in range(r):
        x = s["logits"][i].double()
        top = x.amax(-1, keepdim=True)
        c = s["scores"][i].double()[:, None] + (x - top - (x - top).exp().sum(-1, keepdim=True).log())
        if s["ended"] is not None:                     # an ended beam goes on as it is, with the padding word 0
            stay = torch.full_like(c, -math.inf)
            stay[:, 0] = s["scores"][i].double()
            c = torch.where(s["ended"][i][:, None], stay, c)
        value, index = torch.sort(c.reshape(-1), descending=True, stable=True)
        value, index = value[:num], index[:num]
        none = value == -math.inf
        out[0][i] = value.float()
        out[1][i] = torch.where(none, -1, i * b + index // v).int()
        out[2][i] = torch.where(none, -1, index % v).int()
    return out


def _plain_values(codes, fmt):
    return codes.view(torch.float8_e4m3fn).float() if fmt == "e4m3" else codes.view(torch.int8).float()


def _plain_keys(s, i, name="k", layer=0):
    """[kv_heads, tokens, dim] of one sequence, values in 32 bits."""
    case = s["case"]
    n = _lengths(case)[i]
    at = s["pages"][i, :-(-n // case["page"])].long()
    x = _plain_values(s[name][layer][at], case["fmt"])
    x = x if case["layout"] == "hnd" else x.transpose(1, 2)
    x = x * s[name + "_scale"][layer][at][..., None, None]
    return x.transpose(0, 1).reshape(case["kv_heads"], -1, case["dim"])[:, :n]


def _plain_logits(s, i):
    """[kv_heads, rows, group, keys] of one sequence, -inf where a row does not see a key."""
    case = s["case"]
    h, new, d = case["kv_heads"], case["new"], case["dim"]
    keys = _plain_keys(s, i)
    n = keys.shape[1]
    q = s["q"][i * new:(i + 1) * new].float().reshape(new, h, -1, d).permute(1, 0, 2, 3)
    logit = (q.reshape(h, -1, d) @ keys.transpose(1, 2)).mul_(1.0 / math.sqrt(d)).reshape(h, new, -1, n)
    position = torch.arange(n - new, n, device="cuda")[:, None]
    key = torch.arange(n, device="cuda")[None, :]
    seen = key <= position
    if case["window"]:
        seen = seen & (key > position - case["window"])
    return logit.masked_fill_(~seen[:, None, :], -math.inf)


def _plain_weights(s):
    case = s["case"]
    new, h = case["new"], case["kv_heads"]
    for i in range(case["seqs"]):
        logit = _plain_logits(s, i)
        n = logit.shape[-1]
        lse = s["lse"][i * new:(i + 1) * new].reshape(new, h, -1).transpose(0, 1)
        got = (logit - lse[..., None]).exp_().sum((1, 2))
        if not case["fresh"]:                          # the call's own tokens have received nothing before
            got[:, :n - new] += s["weight"][0, i, :, :n - new]
        s["weight"][0, i, :, :n] = got
    return s["weight"]


def _plain_reorder(s):
    page, n = s["case"]["page"], s["seqs"].numel()
    parent = s["parents"].long()
    rows, length, step = s["pages"], s["length"].long(), torch.arange(s["widest"], device="cuda")
    held, part = -(-length // page), length % page != 0
    count = torch.bincount(parent, minlength=n)
    first = torch.full((n,), n, device="cuda").scatter_reduce_(0, parent, torch.arange(n, device="cuda"), "amin")
    there = step[None, :] < held[:, None]
    last = there & (step[None, :] == held[:, None] - 1) & part[:, None]
    change = torch.where(last, (count > 0).long()[:, None], count[:, None]) - 1
    s["refs"].index_add_(0, rows.long().clamp(min=0).reshape(-1), (change * there).int().reshape(-1))
    copied = part[parent] & (first[parent] != torch.arange(n, device="cuda"))
    free = torch.argsort((s["refs"] != 0).int(), stable=True)          # the free pages, lowest first
    fresh = free[(torch.cumsum(copied.long(), 0) - 1).clamp(min=0)]
    s["refs"][fresh[copied]] = 1
    new = rows[parent]
    end = (held[parent] - 1).clamp(min=0)
    old = new.long().gather(1, end[:, None])[:, 0]
    new.scatter_(1, end[:, None], torch.where(copied, fresh, old)[:, None].int())
    for name in ("k", "v", "k_scale", "v_scale"):
        s[name][:, fresh[copied]] = s[name][:, old[copied]]
    s["pages"].copy_(new)
    s["length"].copy_(length[parent].int())


def _plain_scale(amax, top):
    """The least power of two s with amax / s <= top, from 2^-100 on."""
    mantissa, exponent = torch.frexp(amax)
    share, bits = math.frexp(top)
    e = torch.where(amax > 0, exponent - bits + (mantissa > share).int(), -100)
    return torch.ldexp(torch.ones_like(amax), e.clamp(min=-100))


def _plain_evict(s):
    """Then room for the tokens that follow: every sequence gets its old length again."""
    case = s["case"]
    page, fmt, hnd, keep, first, recent = case["page"], case["fmt"], case["layout"] == "hnd", case["keep"], case["first"], case["recent"]
    top = 448.0 if fmt == "e4m3" else 127.0
    for i, n in enumerate(_lengths(case)):
        if n <= keep:
            continue
        weight = s["weight"][:, i, :, :n].clone()
        weight[..., :first] = math.inf
        weight[..., n - recent:] = math.inf
        order = torch.sort(weight, dim=-1, descending=True, stable=True)[1][..., :keep]
        kept = torch.sort(order, dim=-1)[0]                                                  # [layers, heads, keep]
        s["weight_out"][:, i, :, :keep] = s["weight"][:, i, :, :n].gather(2, kept)
        s["weight_out"][:, i, :, keep:n] = 0.0
        held, now = -(-n // page), -(-keep // page)
        ids = s["pages"][i, :held].long()
        fill = torch.arange(now * page, device="cuda") < keep
        for name in ("k", "v"):
            codes = s[name][:, ids] if hnd else s[name][:, ids].transpose(2, 3)              # [layers, pages, heads, tokens, dim]
            codes = codes.transpose(1, 2).flatten(2, 3)
            kind = codes.gather(2, kept[..., None].expand(-1, -1, -1, case["dim"]))
            scale = s[name + "_scale"][:, ids].transpose(1, 2).gather(2, kept // page)       # [layers, heads, keep]
            value = _plain_values(kind, fmt) * scale[..., None]
            pad = now * page - keep
            amax = torch.nn.functional.pad(value.abs().amax(-1), (0, pad)).unflatten(2, (now, page)).amax(-1)
            fresh = _plain_scale(amax, top)                                                  # [layers, heads, pages]
            value = value / fresh.repeat_interleave(page, 2)[..., :keep, None]
            if fmt == "e4m3":
                kind = value.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
            else:
                kind = value.clamp(-127.0, 127.0).round().to(torch.int8).view(torch.uint8)
            codes[:, :, :now * page][:, :, fill] = kind
            back = codes[:, :, :now * page].unflatten(2, (now, page)).transpose(1, 2)
            s[name][:, ids[:now]] = back if hnd else back.transpose(2, 3)
            s[name + "_scale"][:, ids[:now]] = fresh.transpose(1, 2)
        s["refs"][ids[now:]] -= 1
        s["pages"][i, now:] = -1
        s["length"][i] = keep
    free = torch.argsort((s["refs"] != 0).int(), stable=True)
    at = 0
    for i, n in enumerate(_lengths(case)):
        if n > keep:
            now, held = -(-keep // page), -(-n // page)
            s["pages"][i, now:held] = free[at:at + held - now].int()
            s["refs"][free[at:at + held - now]] = 1
            s["length"][i] = n
            at += held - now


def _codes_out(s, name):
    return s[name].view(torch.float8_e4m3fn) if s["case"]["fmt"] == "e4m3" else s[name].view(torch.int8)


def run(state):
    s, case, op = state, state["case"], state["op"]
    if own:
        import paper_2607_16784_b200 as rm
    if op == "norm":
        if not own:
            return _plain_norm(s)
        q, k = rm.qk_norm_rope(s["q"], s["k"], s["positions"], s["table"], s["wq"], s["wk"], eps=EPS)
        got = dict(q=q, k=k)
        if case["grad"]:
            grads = torch.autograd.grad((q, k), (s["q"], s["k"], s["wq"], s["wk"]), (s["gq"], s["gk"]))
            got = dict(q=q.detach(), dwq=grads[2], dq=grads[0], k=k.detach(), dwk=grads[3], dk=grads[1])
        return got
    if op == "beam":
        got = rm.beam_select(s["logits"], s["scores"], case["num"], ended=s["ended"], workspace=s["workspace"]) if own else _plain_beam(s)
        return dict(scores=got[0], parent=got[1], token=got[2])
    if op == "weights":
        if not own:
            return _plain_weights(s)
        return rm.kv_weights(s["cache"], s["seqs"], s["q"], s["lse"], s["weight"], s["q_offset"], window=case["window"], fresh=case["fresh"])
    if op == "reorder":
        if own:
            rm.kv_reorder(s["cache"], s["seqs"], s["parents"], workspace=s["workspace"])
        else:
            _plain_reorder(s)
        extra = {}
    else:
        if own:
            rm.kv_evict(s["cache"], s["seqs"], s["weight"], case["keep"], first=case["first"], recent=case["recent"], weight_out=s["weight_out"], workspace=s["workspace"])
            rm.kv_reserve(s["cache"], s["seqs"], s["want"], workspace=s["workspace"])
        else:
            _plain_evict(s)
        extra = dict(weight=s["weight_out"])
    return dict(refs=s["refs"], pages=s["pages"], length=s["length"], k=_codes_out(s, "k"), v=_codes_out(s, "v"), k_scale=s["k_scale"], v_scale=s["v_scale"]) | extra


# ------------------------------------------------------------------------------------------------- the least of work
def work(case):
    op = case["op"]
    if op == "norm":
        n, e = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["dim"], SIZES[case["dtype"]]
        return dict(bytes=(4.0 if case["grad"] else 2.0) * n * e + 4.0 * case["tokens"], flops=(20.0 if case["grad"] else 7.0) * n)
    if op == "beam":
        n = case["requests"] * case["beams"] * case["vocab"] * (1.0 - case["ended"])
        return dict(bytes=n * SIZES[case["dtype"]], flops=4.0 * n)
    h, d, page, lengths = case["kv_heads"], case["dim"], case["page"], _lengths(case)
    if op == "weights":
        new, window, keys, pairs = case["new"], case["window"], 0, 0
        for n in lengths:
            keys += n - (max(0, n - new - window + 1) if window else 0)
            pairs += sum(min(p + 1, window) if window else p + 1 for p in range(n - new, n))
        rows = case["seqs"] * new * case["q_heads"]
        moved = h * (keys * d + sum(lengths) * 4.0 * (1 if case["fresh"] else 2)) + rows * (d * SIZES[case["dtype"]] + 4)
        return dict(bytes=float(moved), flops=2.0 * d * case["q_heads"] * pairs)
    layers = case["layers"]
    if op == "reorder":
        b, parents = case["beams"], _parents(case)
        copied = sum((lengths[i // b] % page != 0) and parents.index(p) != i for i, p in enumerate(parents))
        entries = sum(-(-n // page) * b for n in lengths)
        return dict(bytes=layers * 2.0 * h * 2.0 * (page * d + 4) * copied + 8.0 * entries, flops=1.0 * entries)
    over = [n for n in lengths if n > case["keep"]]
    kept = len(over) * case["keep"]
    return dict(bytes=layers * h * (kept * 2.0 * 2.0 * d + 4.0 * sum(over) + 4.0 * sum(over)), flops=layers * h * d * 4.0 * kept)


# --------------------------------------------------------------------------------------------- values in 64 bits
def _exact_values(codes, fmt):
    if fmt == "int8":
        c = codes.long()
        return torch.where(c > 127, c - 256, c).double()
    bits = np.arange(256)
    e, m = (bits >> 3) & 15, bits & 7
    value = np.where(e > 0, (1.0 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    return torch.from_numpy(np.where(bits > 127, -value, value)).cuda()[codes.long()]


def _exact_norm(s):
    """Each pair as a complex number, the gradients through torch's own rules in 64 bits."""
    case = s["case"]
    high, low = (s["frequency"] >> 32) & 0xFFFFFFFF, s["frequency"] & 0xFFFFFFFF
    p = s["positions"].long()[:, None]
    turns = ((p * high) % (1 << 32)).double() * 2.0 ** -32 + (p * low).double() * 2.0 ** -64
    w = torch.polar(torch.ones_like(turns), 2.0 * math.pi * turns)[:, None, :]
    half, got = turns.shape[-1], {}
    for n in ("q", "k"):
        x = s[n].detach().double().requires_grad_(case["grad"])
        weight = s["w" + n].detach().double().requires_grad_(case["grad"])
        y = x / (x.pow(2).sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * weight
        if case["layout"] == "half":
            z = torch.complex(y[..., :half], y[..., half:2 * half]) * w
            y = torch.cat([z.real, z.imag, y[..., 2 * half:]], -1)
        else:
            z = torch.view_as_complex(y[..., :2 * half].unflatten(-1, (half, 2)).contiguous()) * w
            y = torch.cat([torch.view_as_real(z).flatten(-2), y[..., 2 * half:]], -1)
        got[n] = y.detach()
        if case["grad"]:
            grads = torch.autograd.grad(y, (x, weight), s["g" + n].double())
            got["dw" + n], got["d" + n] = grads[1], grads[0]
    return got


def _exact_beam(s):
    """The best of each row first, then the best of those."""
    case = s["case"]
    b, num = case["beams"], case["num"]
    out = [[], [], []]
    for i in range(case["requests"]):
        found = []
        for j in range(b):
            score = float(s["scores"][i, j])
            if s["ended"] is not None and bool(s["ended"][i, j]):
                found.append((-score, j, 0))
                continue
            x = s["logits"][i, j].double()
            lse = float(torch.logsumexp(x, 0))
            least = float(torch.topk(x, min(num, x.numel()))[0][-1])
            for t in (x >= least).nonzero()[:, 0].tolist():
                if float(x[t]) > -math.inf:
                    found.append((-(score + (float(x[t]) - lse)), j, t))
        found = sorted(found)[:num]
        out[0].append([-f[0] for f in found] + [-math.inf] * (num - len(found)))
        out[1].append([i * b + f[1] for f in found] + [-1] * (num - len(found)))
        out[2].append([f[2] for f in found] + [-1] * (num - len(found)))
    kinds = (torch.float64, torch.int32, torch.int32)
    return dict(zip(("scores", "parent", "token"), (torch.tensor(o, dtype=t, device="cuda") for o, t in zip(out, kinds))))


def _exact_weights(s):
    case = s["case"]
    h, page, d, new = case["kv_heads"], case["page"], case["dim"], case["new"]
    g = case["q_heads"] // h
    out = s["weight"].double()
    for i, n in enumerate(_lengths(case)):
        at = s["pages"][i, :-(-n // page)].long()
        position = torch.arange(n - new, n, device="cuda")[:, None]
        key = torch.arange(n, device="cuda")[None, :]
        hidden = key > position
        if case["window"]:
            hidden |= key <= position - case["window"]
        for head in range(h):
            codes = s["k"][0][at, head] if case["layout"] == "hnd" else s["k"][0][at, :, head]
            k = (_exact_values(codes, case["fmt"]) * s["k_scale"][0][at, head].double()[:, None, None]).reshape(-1, d)[:n]
            total = torch.zeros(n, dtype=torch.float64, device="cuda")
            for j in range(head * g, head * g + g):
                p = torch.exp(s["q"][i * new:(i + 1) * new, j].double() @ k.T / math.sqrt(d) - s["lse"][i * new:(i + 1) * new, j].double()[:, None])
                total += torch.where(hidden, 0.0, p).sum(0)
            old = 0 if case["fresh"] else n - new
            total[:old] += out[0, i, head, :old]
            out[0, i, head, :n] = total
    return out


def exact(case, seed):
    if case["op"] in ("reorder", "evict"):
        return None  # whole numbers, copies and codes moved by powers of two: the plain form's values are the values
    s = prepare(case, seed)
    return _exact_norm(s) if case["op"] == "norm" else _exact_beam(s) if case["op"] == "beam" else _exact_weights(s)
