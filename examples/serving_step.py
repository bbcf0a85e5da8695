"""A language model's decoding steps over a paged 8-bit cache, and what they mean to the other residents of a GPU.

    python examples/serving_step.py [--seqs 8] [--prompt 500] [--steps 12] [--beams 2] [--keep 0]

One attention layer's worth of the model's serving operators runs as it would be used: prompts are reserved, rotated, quantised into the
cache and attended to; some sequences are forked and decode on their own; the losers are freed and the pool is compacted.  With --keep the
continuations are a beam search over a bounded cache: queries and keys are normed, keys gather the attention weight that they receive, every sequence is cut
to its heaviest tokens now and then, and the cache follows the search's picks.  The launches
are recorded on the way (the cache operators' own: a model's projections and other products come from other libraries).  Their
configurations and isolated durations become one more profile beside a library of synthetic residents,
the pairwise interference of all of them is evaluated, and the model is placed on the GPU of a small cluster where it is disturbed and
disturbs least."""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_16784_b200 as rm  # noqa: E402
import roomie_synth as rs  # noqa: E402


def serve(seqs, prompt, steps, beams, q_heads=32, kv_heads=8, head_dim=128, page_tokens=32, seed=0):
    """Runs the steps; returns (cache, the last step's attention output, used pages before and after compaction)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda rows, heads: torch.randn((rows, heads, head_dim), generator=gen, device="cuda").to(torch.bfloat16)
    ids = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")
    total = seqs * beams
    width = -(-(prompt + steps) // page_tokens)
    cache = rm.KVCache(total * width + 8, page_tokens, kv_heads, head_dim, total, width)
    workspace, table = cache.workspace(), rm.RopeTable(head_dim)

    def step(slots, lengths, news):
        offset = ids(np.concatenate([[0], np.cumsum(news)]))
        rows = int(np.sum(news))
        rm.kv_reserve(cache, slots, ids(lengths), workspace=workspace)
        q = rm.kv_append(cache, slots, new(rows, kv_heads), new(rows, kv_heads), offset, rope=table, q=new(rows, q_heads))
        return rm.kv_attention(cache, slots, q, offset, workspace=workspace)[0]

    lengths = np.maximum(1, prompt - 17 * np.arange(seqs))                       # ragged prompts
    first = ids(np.arange(seqs))
    out = step(first, lengths, lengths)
    if beams > 1:                                                                # continuations share their prompts' whole pages
        rm.kv_fork(cache, ids(np.tile(np.arange(seqs), beams - 1)), ids(np.arange(seqs, total)), workspace=workspace)
    every, lengths = ids(np.arange(total)), np.tile(lengths, beams)
    for n in range(1, steps + 1):
        out = step(every, lengths + n, np.ones(total, dtype=np.int64))
    used = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2)]
    rm.kv_compact(cache, used_out=used[0], workspace=workspace)
    rm.kv_free(cache, ids(np.arange(0, total, 2)))                               # half of them end
    rm.kv_compact(cache, used_out=used[1], workspace=workspace)
    cache.check()
    return cache, out, int(used[0]), int(used[1])


def search(requests, beams, prompt, steps, keep, q_heads=32, kv_heads=8, head_dim=128, page_tokens=32, vocab=4096, every=8, seed=0):
    """A beam search by one layer of random weights (its projections are torch products) over a cache whose sequences are cut to `keep` tokens every
    `every` steps.  Returns (cache, tokens [requests, beams, steps], scores, the keys' weights)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    ids = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")
    hidden, total, wide = 256, requests * beams, q_heads + 2 * kv_heads
    embed = rand(vocab, hidden).to(torch.bfloat16)
    project = (rand(hidden, wide * head_dim) * hidden ** -0.5).to(torch.bfloat16)
    read_out = (rand(q_heads * head_dim, vocab) * 0.2).to(torch.bfloat16)
    q_weight, k_weight = 1 + 0.1 * rand(head_dim), 1 + 0.1 * rand(head_dim)
    width = -(-max(prompt, keep + every) // page_tokens)
    # a cut replaces the pages that beams share, out of those that are free before it: as many again as the sequences hold
    cache = rm.KVCache(2 * total * width, page_tokens, kv_heads, head_dim, total, width)
    workspace, table, weight = cache.workspace(), rm.RopeTable(head_dim), cache.key_weights()

    def step(slots, words, positions, lengths, offset, fresh):
        """Appends the words, whose positions are not what the cache's lengths say once tokens have left; returns the attention's rows."""
        x = (embed[words] @ project).view(-1, wide, head_dim)
        q, k = rm.qk_norm_rope(x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], positions, table, q_weight, k_weight)
        rm.kv_reserve(cache, slots, lengths, workspace=workspace)
        rm.kv_append(cache, slots, k, x[:, q_heads + kv_heads:], offset)
        out, lse = rm.kv_attention(cache, slots, q, offset, workspace=workspace)
        rm.kv_weights(cache, slots, q, lse, weight, offset, fresh=fresh)
        return out

    first, slots = ids(np.arange(requests) * beams), ids(np.arange(total))
    out = step(first, torch.randint(0, vocab, (requests * prompt,), generator=gen, device="cuda"), ids(np.tile(np.arange(prompt), requests)),
               ids([prompt] * requests), ids(np.arange(requests + 1) * prompt), True)[prompt - 1::prompt]
    rm.kv_evict(cache, first, weight, keep, first=4, recent=keep // 4, workspace=workspace)
    length = min(prompt, keep)
    parent = first.repeat_interleave(beams)                                      # every beam begins as its request's prompt
    rm.kv_reorder(cache, slots, parent, workspace=workspace)
    weight = weight[:, parent.long()].contiguous()
    out = out.repeat_interleave(beams, 0)
    scores = torch.full((requests, beams), -np.inf, device="cuda")
    scores[:, 0] = 0.0
    ended = torch.zeros((requests, beams), dtype=torch.bool, device="cuda")
    tokens = torch.zeros((total, 0), dtype=torch.int32, device="cuda")
    for n in range(steps):
        logits = (out.reshape(total, -1) @ read_out).view(requests, beams, vocab)
        scores, parent, token = rm.beam_select(logits, scores, beams, ended=ended)               # token 0 ends a beam
        at = parent.flatten().long()
        rm.kv_reorder(cache, slots, parent, workspace=workspace)
        weight = weight[:, at].contiguous()
        tokens = torch.cat([tokens[at], token.view(-1, 1)], 1)
        ended = token == 0
        if length >= keep + every - 1:
            rm.kv_evict(cache, slots, weight, keep, first=4, recent=keep // 4, workspace=workspace)
            length = keep
        length += 1
        out = step(slots, token.flatten().long(), ids([prompt + n] * total), ids([length] * total), None, False)
    cache.check()
    return cache, tokens.view(requests, beams, -1), scores, weight


def place_beside(launches, num_gpus=16, residents=3, seed=0):
    """The recorded launches as a profile among synthetic residents: (slowdown of the model, slowdown it causes) for each of them, and
    the GPU chosen for it."""
    synth = rs.make_library(1)
    columns = rm.profile_columns(launches)
    cat = [np.concatenate([a, b]) for a, b in zip((synth.grid_blocks, synth.block_threads, synth.regs_per_thread, synth.smem_per_block,
                                                   synth.dur_us, synth.gap_us), columns)]
    offsets = np.concatenate([synth.offsets, [synth.offsets[-1] + len(launches)]]).astype(np.uint32)
    b200 = rm.GpuSpec(148, 65536, 228 * 1024, 2048, 32)
    lib = rm.library_build(*cat, offsets, b200)
    P, _ = rm.pair_matrix(lib, mode=rm.TIMELINE, n_align=8, start_filter=1)
    lib.check()
    model = lib.num_profiles - 1
    rng = np.random.default_rng(seed)
    ids = np.full((num_gpus, residents + 1), -1, dtype=np.int32)
    count = rng.integers(0, residents + 1, num_gpus).astype(np.uint32)
    for g in range(num_gpus):
        ids[g, :count[g]] = rng.integers(0, model, count[g])
    state = rm.ClusterState(num_gpus, residents + 1, ids, np.zeros(ids.size, dtype=np.uint32), count)
    gpu, mean, _ = rm.place(P, state, np.array([model], dtype=np.int32), np.zeros(1, dtype=np.uint32), lam=10.0)
    M = P.cpu().numpy()
    return M[model, :model], M[:model, model], int(gpu[0]), float(mean[0])


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("seqs", 8), ("prompt", 500), ("steps", 12), ("beams", 2), ("keep", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args(argv)
    if a.keep:
        search(a.seqs, a.beams, a.prompt, 1, a.keep)                             # kernels loaded, allocator warm
        with rm.record_launches() as launches:
            cache, out, scores, _ = search(a.seqs, a.beams, a.prompt, a.steps, a.keep)
        before = after = int((cache.refs > 0).sum())
    else:
        serve(a.seqs, a.prompt, 1, a.beams)
        with rm.record_launches() as launches:
            cache, out, before, after = serve(a.seqs, a.prompt, a.steps, a.beams)
    by_name = {}
    for r in launches:
        by_name.setdefault(r["name"], []).append(r)
    if a.keep:
        print(f"{a.seqs} requests x {a.beams} beams over {a.keep} tokens: {len(launches)} launches; {after} pages in use; best scores {scores[:, 0].tolist()}")
    else:
        print(f"{a.seqs} sequences x {a.beams} continuations: {len(launches)} launches; {before} pages in use, {after} after half of them ended")
    for name, rs_ in by_name.items():
        last = rs_[-1]
        print(f"  {name:18s} {len(rs_):4d} launches  {sum(r['dur_us'] for r in rs_):9.1f} us  last: {last['grid_blocks']} x {last['block_threads']} "
              f"threads, {last['regs_per_thread']} registers, {last['smem_per_block']} bytes shared")
    suffers, causes, gpu, mean = place_beside(launches)
    print(f"slowdown beside each of {len(suffers)} synthetic residents: suffers {suffers.min():.3f} .. {suffers.max():.3f}, "
          f"causes {causes.min():.3f} .. {causes.max():.3f}; placed on GPU {gpu} (mean drop there {mean:.3f})")
    return launches, out, gpu


if __name__ == "__main__":
    main()
