"""The host side of the operators of a search step and a bounded cache: size queries and refusals answer without a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2607_16784_b200 as rm
from paper_2607_16784_b200 import roomie, serving

dll = roomie._dll
FAKE = 0x7F0000000000                                                  # never dereferenced


def rows(data=FAKE, kind=2, token=4 * 128, head=128):
    return serving._pack_rows(data or 0, kind, token, head)


def table(rot=128, frequency=FAKE):
    return serving._RopeTable(rot, 0, 1.0, frequency)


def test_norm_refusals():
    def call(t=table(), eps=1e-6, tokens=4, dim=128, positions=FAKE, kind=0, hq=4, q=rows(), wq=FAKE, qo=rows(FAKE + (1 << 20)), hk=2, k=rows(FAKE + (1 << 21)), wk=None,
             ko=rows(FAKE + (1 << 22))):
        return dll.roomie_qk_norm_rope(C.byref(t) if t is not None else None, eps, tokens, dim, positions, kind, hq, q, wq, qo, hk, k, wk, ko, None)
    for bad in (dict(t=table(0)), dict(t=table(7)), dict(t=table(130)), dict(t=table(frequency=None)), dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(dim=0), dict(dim=257, t=None), dict(dim=64), dict(positions=None), dict(kind=3), dict(kind=-1), dict(wq=FAKE + 2), dict(wq=FAKE + 1, kind=2),
                dict(q=None), dict(q=rows(None)), dict(q=rows(kind=5)), dict(q=rows(FAKE + 1)), dict(qo=None), dict(qo=rows(FAKE + (1 << 20), kind=1)), dict(k=rows(kind=1)),
                dict(k=None), dict(ko=rows(FAKE + (1 << 22), token=0)), dict(ko=rows(FAKE + (1 << 22), head=64)), dict(qo=rows(token=1024)), dict(qo=rows(head=256)),
                dict(tokens=1 << 29)):
        assert call(**bad) == -1, bad
    assert call(tokens=0) == 0 and call(hq=0, hk=0) == 0 and call(tokens=0, t=None, positions=None) == 0


def test_norm_gradient_refusals():
    room = dll.roomie_qk_norm_rope_workspace_bytes(128)
    assert room > 0 and dll.roomie_qk_norm_rope_workspace_bytes(0) == 0 and dll.roomie_qk_norm_rope_workspace_bytes(257) == 0
    far = [rows(FAKE + (i << 20)) for i in range(6)]
    def call(q=far[0], gq=far[1], dq=far[2], dwq=FAKE, k=far[3], gk=far[4], dk=far[5], dwk=None, ws=FAKE, room=room, hk=2, kind=0):
        return dll.roomie_qk_norm_rope_grad(C.byref(table()), 1e-6, 4, 128, FAKE, kind, 4, q, FAKE, gq, dq, dwq, hk, k, None, gk, dk, dwk, ws, room, None)
    for bad in (dict(q=None), dict(gq=None), dict(dq=None), dict(gq=rows(kind=1)), dict(dk=rows(kind=0)), dict(dq=rows(token=0)), dict(dk=rows(head=1)), dict(dwq=FAKE + 2),
                dict(dwk=FAKE + 1, kind=1), dict(ws=None), dict(ws=FAKE + 2), dict(kind=7)):
        assert call(**bad) == -1, bad
    assert call(room=room - 1) == -4


def test_beam_sizes_and_refusals():
    size = dll.roomie_beam_workspace_bytes
    assert size(4, 4, 32000, 8, 2) > 0 and size(4, 4, 32000, 8, 2) % 256 == 0 and size(4, 4, 32000, 16, 2) > size(4, 4, 32000, 8, 2)
    for bad in ((0, 4, 100, 8, 2), (4, 0, 100, 8, 2), (4, 257, 100, 8, 2), (4, 4, 0, 8, 2), (4, 4, (1 << 24) + 1, 8, 2), (4, 4, 100, 0, 2), (4, 4, 100, 129, 2),
                (4, 4, 100, 8, 3), (16384, 4, 100, 8, 2)):
        assert size(*bad) == 0, bad
    need = size(4, 4, 100, 8, 2)
    def call(logits=FAKE, kind=2, requests=4, beams=4, vocab=100, scores=FAKE, pad=0, num=8, out=(FAKE, FAKE, FAKE), ws=FAKE, room=need):
        return dll.roomie_beam_select(logits, kind, 400, 100, requests, beams, vocab, scores, None, pad, num, *out, ws, room, None)
    for bad in (dict(logits=None), dict(logits=FAKE + 1), dict(kind=4), dict(beams=0), dict(vocab=0), dict(scores=None), dict(pad=1 << 31), dict(num=0), dict(num=129),
                dict(out=(None, FAKE, FAKE)), dict(out=(FAKE, None, FAKE)), dict(out=(FAKE, FAKE, None)), dict(ws=None), dict(ws=FAKE + 64)):
        assert call(**bad) == -1, bad
    assert call(room=need - 1) == -4 and call(requests=0) == 0


def cache(**kw):
    d = dict(layers=2, num_pages=100, page_tokens=32, kv_heads=4, head_dim=128, format=0, layout=0, max_seqs=8, max_pages=16,
             k=FAKE, v=FAKE + (1 << 30), layer_stride=100 * 4 * 32 * 128, page_stride=4 * 32 * 128, k_scale=FAKE, v_scale=FAKE,
             refs=FAKE, pages=FAKE, length=FAKE, status=FAKE)
    d.update(kw)
    return serving._KVCache(**d)


def room(**kw):
    return dll.roomie_kv_workspace_bytes(C.byref(cache(**kw)))


def test_reorder_refusals():
    def call(c=cache(), seqs=FAKE, parents=FAKE, n=2, ws=FAKE, size=room()):
        return dll.roomie_kv_reorder(C.byref(c), seqs, parents, n, ws, size, None)
    for bad in (dict(c=cache(head_dim=24)), dict(c=cache(refs=None)), dict(seqs=None), dict(parents=None), dict(n=9), dict(ws=None), dict(ws=FAKE + 8)):
        assert call(**bad) == -1, bad
    big = dict(max_seqs=10000)
    assert call(c=cache(**big), n=8193, size=room(**big)) == -1
    assert call(size=room() - 1) == -4 and call(n=0, seqs=None) == 0


def test_evict_refusals():
    def call(c=cache(), seqs=FAKE, n=2, weight=FAKE, keep=100, first=4, recent=50, out=FAKE, ws=FAKE, size=room()):
        return dll.roomie_kv_evict(C.byref(c), seqs, n, weight, keep, first, recent, out, ws, size, None)
    for bad in (dict(c=cache(page_tokens=48)), dict(seqs=None), dict(weight=None), dict(out=None), dict(weight=FAKE + 2), dict(out=FAKE + 1), dict(n=9), dict(keep=0),
                dict(keep=1 << 31), dict(keep=53), dict(first=0xffffffff, recent=0xffffffff), dict(ws=None), dict(ws=FAKE + 8)):
        assert call(**bad) == -1, bad
    wide = dict(max_pages=(1 << 15) + 1)
    assert call(c=cache(**wide), size=room(**wide)) == -1
    assert call(size=room() - 1) == -4 and call(n=0) == 0


def test_weights_refusals():
    def call(c=cache(), layer=0, seqs=FAKE, n=2, offset=None, count=2, heads=8, q=rows(), lse=FAKE, scale=0.1, window=0, weight=FAKE):
        return dll.roomie_kv_weights(C.byref(c), layer, seqs, n, offset, count, heads, q, lse, scale, window, 0, weight, None)
    for bad in (dict(c=cache(head_dim=24)), dict(layer=5), dict(seqs=None), dict(count=3), dict(heads=0), dict(heads=6), dict(q=rows(kind=0)), dict(q=None),
                dict(lse=None), dict(lse=FAKE + 2), dict(weight=None), dict(weight=FAKE + 1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                dict(scale=float("nan")), dict(window=1 << 31)):
        assert call(**bad) == -1, bad
    assert call(n=0, count=0) == 0 and call(count=0) == 0
