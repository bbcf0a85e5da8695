"""A language model's decoding steps over a paged 8-bit cache, and what they mean to the other residents of a GPU.

    python examples/serving_step.py [--seqs 8] [--prompt 500] [--steps 12] [--beams 2]

One attention layer's worth of the model's serving operators runs as it would be used: prompts are reserved, rotated, quantised into the
cache and attended to; some sequences are forked and decode on their own; the losers are freed and the pool is compacted.  The launches
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
    for name, default in (("seqs", 8), ("prompt", 500), ("steps", 12), ("beams", 2)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args(argv)
    serve(a.seqs, a.prompt, 1, a.beams)                                          # kernels loaded, allocator warm
    with rm.record_launches() as launches:
        cache, out, before, after = serve(a.seqs, a.prompt, a.steps, a.beams)
    by_name = {}
    for r in launches:
        by_name.setdefault(r["name"], []).append(r)
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
