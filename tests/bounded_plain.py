"""Reordering and eviction from their definitions, in plain numpy on the host."""
import numpy as np

import serving_plain as sp


def reorder(refs, table, length, page, seqs, parents):
    """Lists refs, table, length in place; returns the copied pages [(from, to)], or None where the call changes nothing for want of pages."""
    old_table, old_length = [list(r) for r in table], list(length)
    new_refs = list(refs)
    for s in seqs:
        for e in range(-(-old_length[s] // page)):
            new_refs[old_table[s][e]] -= 1
    taken, copies = set(), []
    for i, p in enumerate(parents):
        if p < 0:
            continue
        n = old_length[seqs[p]]
        for e in range(-(-n // page)):
            if e == n // page and p in taken:
                copies.append((i, old_table[seqs[p]][e]))
            else:
                new_refs[old_table[seqs[p]][e]] += 1
        taken.add(p)
    free = [q for q, r in enumerate(new_refs) if r == 0]
    if len(free) < len(copies):
        return None
    pairs, fresh = [], {}
    for (i, a), b in zip(copies, free):
        pairs.append((a, b))
        new_refs[b] = 1
        fresh[i] = b
    for i, p in enumerate(parents):
        n = old_length[seqs[p]] if p >= 0 else 0
        row = list(old_table[seqs[p]]) if p >= 0 else []
        held = -(-n // page)
        if i in fresh:
            row[held - 1] = fresh[i]
        for e in range(max(held, -(-old_length[seqs[i]] // page))):
            table[seqs[i]][e] = row[e] if e < held else -1
        length[seqs[i]] = n
    refs[:] = new_refs
    return pairs


def kept(weight, length, keep, first, recent):
    """Positions that one head keeps, in order."""
    w = np.where(np.isnan(weight[:length]), -np.inf, weight[:length].astype(np.float64))
    lowest = np.isnan(weight[:length])                               # below -infinity
    middle = np.arange(first, length - recent)
    order = middle[np.lexsort((middle, lowest[middle], -w[middle]))]
    return np.sort(np.concatenate([np.arange(first), order[:keep - first - recent], np.arange(length - recent, length)])).astype(int)


def to_codes(x, fmt):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x.astype(np.float32)))
    if fmt == "e4m3":
        return t.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    return t.clamp(-127.0, 127.0).round().to(torch.int8).view(torch.uint8).numpy()


def packed(codes, scales, fmt, page):
    """Codes [n, dim] of one head with each token's scale, to pages: (codes, the pages' scales).  Float32, as the definition says."""
    out, units = codes.copy(), []
    value = sp.values(codes, fmt).astype(np.float32) * scales[:, None].astype(np.float32)
    for at in range(0, len(codes), page):
        unit = sp.scale_of(float(np.abs(value[at:at + page]).max()), fmt)
        units.append(unit)
        for t in range(at, min(at + page, len(codes))):
            if scales[t] != unit:
                out[t] = to_codes(value[t] / np.float32(unit), fmt)
    return out, np.array(units, dtype=np.float32)
