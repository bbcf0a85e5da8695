"""The serving operators' host side: size queries, frequencies and refusals answer without a GPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2607_16784_b200 as rm
from paper_2607_16784_b200 import roomie, serving

dll = roomie._dll
FAKE = 0x7F0000000000                                                  # never dereferenced


def cache(**kw):
    d = dict(layers=2, num_pages=100, page_tokens=32, kv_heads=4, head_dim=128, format=0, layout=0, max_seqs=8, max_pages=16,
             k=FAKE, v=FAKE + (1 << 30), layer_stride=100 * 4 * 32 * 128, page_stride=4 * 32 * 128, k_scale=FAKE, v_scale=FAKE,
             refs=FAKE, pages=FAKE, length=FAKE, status=FAKE)
    d.update(kw)
    return serving._KVCache(**d)


def rows(data=FAKE, kind=2, token=4 * 128, head=128):
    return serving._pack_rows(data or 0, kind, token, head)


def table(rot=128, frequency=FAKE):
    return serving._RopeTable(rot, 0, 1.0, frequency)


def size(**kw):
    return dll.roomie_kv_workspace_bytes(C.byref(cache(**kw)))


def test_workspace_bytes():
    assert size() > 0 and size() % 256 == 0
    assert size(num_pages=100000) >= size() + 4 * 4 * 99000 and size(max_seqs=1000) > size()
    assert dll.roomie_kv_workspace_bytes(None) == 0
    for bad in (dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=256), dict(head_dim=0), dict(head_dim=100), dict(head_dim=272),
                dict(format=2), dict(layout=2), dict(num_pages=0), dict(kv_heads=0), dict(layers=0), dict(max_seqs=0), dict(max_pages=0),
                dict(k=None), dict(v=None), dict(k_scale=None), dict(refs=None), dict(pages=None), dict(length=None), dict(status=None),
                dict(k=FAKE + 8), dict(page_stride=4 * 32 * 128 + 8), dict(page_stride=4 * 32 * 127), dict(layer_stride=64)):
        assert size(**bad) == 0, bad


def test_frequencies():
    """base^(-2i/r) / 2 pi turns a position in 2^-64 turns, exact to a double's rounding; the three ways of stretching."""
    for rot, base in ((2, 10000.0), (128, 10000.0), (96, 500000.0), (64, 1.5)):
        got = rm.rope_frequencies(rot, base)
        want = [base ** (-2.0 * i / rot) / (2 * math.pi) * 2.0 ** 64 for i in range(rot // 2)]
        assert all(abs(int(g) - w) <= 0.5 + abs(w) * 2.0 ** -50 for g, w in zip(got, want))
        assert np.all(got[:-1] >= got[1:]) and got[0] < 1 << 62
    fast, slow = 0.5, 3.0                                              # turns over the context: all above, all below the limits
    assert np.array_equal(rm.rope_frequencies(8, 2.0, factor=4.0, context=1e9), rm.rope_frequencies(8, 2.0))
    assert np.array_equal(rm.rope_frequencies(8, 2.0, factor=4.0, context=1e-3), rm.rope_frequencies(8, 2.0, factor=4.0))
    for bad in (dict(rotary_dim=0), dict(rotary_dim=5), dict(base=1.0), dict(base=float("inf")), dict(base=float("nan")), dict(factor=0.9),
                dict(factor=float("nan")), dict(context=-1.0), dict(context=100, low_turns=slow, high_turns=fast)):
        with pytest.raises(rm.RoomieError, match="invalid argument"):
            rm.rope_frequencies(**dict(dict(rotary_dim=8), **bad))
    assert dll.roomie_rope_frequencies(8, 10000.0, 1.0, 0.0, 0.0, 0.0, None) == -1


def test_rope_refusals():
    def call(t=table(), x=rows(), y=rows(FAKE + (1 << 20)), tokens=4, heads=4, dim=128, positions=FAKE):
        return dll.roomie_rope(C.byref(t) if t is not None else None, x, y, tokens, heads, dim, positions, 0, None)
    for bad in (dict(t=None), dict(t=table(0)), dict(t=table(7)), dict(t=table(130)), dict(t=table(frequency=None)), dict(t=table(frequency=FAKE + 4)),
                dict(x=None), dict(x=rows(None)), dict(x=rows(kind=3)), dict(x=rows(FAKE + 1)), dict(y=rows(kind=1)), dict(positions=None), dict(dim=64),
                dict(dim=2048), dict(y=rows(token=1024)), dict(y=rows(head=256))):
        assert call(**bad) == -1, bad
    assert call(tokens=0) == 0 and call(heads=0) == 0                  # nothing to do: nothing is launched


def test_append_refusals():
    def call(c=cache(), layer=0, seqs=FAKE, n=2, offset=None, count=2, k=rows(), v=rows(), t=None, q_heads=0, q=None, q_out=None):
        return dll.roomie_kv_append(C.byref(c), layer, seqs, n, offset, count, k, v, C.byref(t) if t else None, q_heads, q, q_out, None)
    for bad in (dict(c=cache(format=9)), dict(layer=2), dict(seqs=None), dict(count=3), dict(k=None), dict(v=rows(kind=0)), dict(t=table(130)),
                dict(q=rows(), q_heads=8), dict(q=rows(), q_out=rows(), q_heads=8), dict(t=table(), q=rows(), q_out=rows(), q_heads=0),
                dict(t=table(), q=rows(kind=1), q_out=rows(kind=1), q_heads=8), dict(t=table(), q=rows(), q_out=rows(token=1), q_heads=8)):
        assert call(**bad) == -1, bad
    assert call(n=0, count=0) == 0 and call(count=0) == 0


def test_attention_refusals():
    need = size()
    def call(c=cache(), layer=0, seqs=FAKE, n=2, offset=None, count=2, heads=8, q=rows(), scale=0.1, window=0, out=rows(), ws=FAKE, room=need):
        return dll.roomie_kv_attention(C.byref(c), layer, seqs, n, offset, count, heads, q, scale, window, out, None, ws, room, None)
    for bad in (dict(c=cache(head_dim=24)), dict(layer=5), dict(seqs=None), dict(count=3), dict(heads=0), dict(heads=6), dict(q=rows(kind=0), out=rows(kind=0)),
                dict(out=rows(kind=1)), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(window=1 << 31),
                dict(q=None), dict(out=rows(None)), dict(ws=None), dict(ws=FAKE + 128)):
        assert call(**bad) == -1, bad
    assert call(room=need - 1) == -4
    assert call(n=0, count=0) == 0


def test_page_refusals():
    need = size()
    c, ref = cache(), None
    ref = C.byref(c)
    assert dll.roomie_kv_reserve(ref, None, FAKE, 1, FAKE, need, None) == -1
    assert dll.roomie_kv_reserve(ref, FAKE, FAKE, 9, FAKE, need, None) == -1          # more requests than sequences
    assert dll.roomie_kv_reserve(ref, FAKE, FAKE, 1, FAKE, need - 1, None) == -4
    assert dll.roomie_kv_reserve(ref, FAKE, FAKE, 0, None, 0, None) == 0
    assert dll.roomie_kv_fork(ref, FAKE, None, 1, FAKE, need, None) == -1
    assert dll.roomie_kv_fork(ref, FAKE, FAKE, 1, FAKE + 16, need, None) == -1
    assert dll.roomie_kv_fork(ref, FAKE, FAKE, 0, None, 0, None) == 0
    assert dll.roomie_kv_free(ref, None, 1, None) == -1 and dll.roomie_kv_free(ref, None, 0, None) == 0
    for other in (dict(layers=1), dict(page_tokens=16), dict(kv_heads=2), dict(head_dim=64), dict(format=1), dict(layout=1)):
        assert dll.roomie_kv_copy(ref, FAKE, C.byref(cache(**other)), FAKE, 1, None) == -1, other
    assert dll.roomie_kv_copy(ref, FAKE, C.byref(cache(num_pages=7)), None, 1, None) == -1
    assert dll.roomie_kv_copy(ref, None, ref, None, 0, None) == 0
    assert dll.roomie_kv_compact(ref, None, FAKE, None, FAKE, need, None) == -1
    assert dll.roomie_kv_compact(ref, FAKE, FAKE, None, FAKE, need - 256, None) == -4


def test_tensors_of_a_call_live_on_the_current_device(monkeypatch):
    class Tensor:
        def __init__(self, device):
            self.device = device
        def get_device(self):
            return self.device
    monkeypatch.setattr(serving.torch.cuda, "current_device", lambda: 1)
    serving._here(1, Tensor(1), None, Tensor(1))
    for bad in ((0,), (0, Tensor(1)), (1, Tensor(1), Tensor(0)), (1, None, Tensor(-1))):
        with pytest.raises(ValueError, match="current CUDA device"):
            serving._here(*bad)


def test_binding_needs_no_private_name(monkeypatch):
    """Without torch's short way to a stream the binding is imported all the same and asks the public one."""
    import importlib.util
    from types import SimpleNamespace
    if hasattr(serving.torch._C, "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(serving.torch._C, "_cuda_getCurrentRawStream")
    spec = importlib.util.spec_from_file_location(serving.__name__ + "_again", serving.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)
    monkeypatch.setattr(again.torch.cuda, "current_stream", lambda device: SimpleNamespace(cuda_stream=40 + device))
    assert again._stream(SimpleNamespace(get_device=lambda: 2)) == 42


def test_outputs_whose_rows_share_elements_are_refused():
    """Strides of 0 and below a row's length, of rope's, append's and attention's outputs; one token or one head has no such stride."""
    c, t, need = cache(), table(), size()
    def turn(out, tokens=4, heads=4):
        return dll.roomie_rope(C.byref(t), rows(), out, tokens, heads, 128, FAKE, 0, None)
    def append(out, heads=8):
        return dll.roomie_kv_append(C.byref(c), 0, FAKE, 2, None, 2, rows(), rows(), C.byref(t), heads, rows(FAKE + 4096), out, None)
    def attend(out, heads=8):
        return dll.roomie_kv_attention(C.byref(c), 0, FAKE, 2, None, 2, heads, rows(), 0.1, 0, out, None, FAKE, need, None)
    for call in (turn, append, attend):
        for bad in (dict(token=0), dict(head=0), dict(token=127), dict(head=64), dict(token=-100), dict(token=0, head=0)):
            assert call(rows(FAKE + (1 << 20), **bad)) == -1, (call, bad)
    assert turn(rows(FAKE, token=0, head=0)) == -1                     # in place on a broadcast input: it would be turned several times
    if not torch.cuda.is_available():                                  # accepted: only the launch finds no device
        for good in (turn(rows(FAKE + (1 << 20), token=0), tokens=1), turn(rows(FAKE + (1 << 20), head=0), heads=1),
                     turn(rows(FAKE + (1 << 20), token=-512, head=128)), turn(rows(FAKE + (1 << 20), token=128, head=512))):
            assert good == -3


def test_record_without_launches():
    count = C.c_uint32(7)
    assert dll.roomie_record_enable(0) == 0
    assert dll.roomie_record_read(None, 0, C.byref(count)) == 0 and count.value == 0
    assert dll.roomie_record_read(None, 1, C.byref(count)) == -1 and dll.roomie_record_read(None, 0, None) == -1
    assert dll.roomie_record_enable((1 << 20) + 1) == -1


def test_profile_columns_are_a_kernel_table():
    launches = [dict(name="a", grid_blocks=148, block_threads=640, regs_per_thread=96, smem_per_block=200000, dur_us=400.5, gap_us=1.5),
                dict(name="b", grid_blocks=1, block_threads=1024, regs_per_thread=32, smem_per_block=0, dur_us=3.0, gap_us=0.0)]
    grid, threads, regs, smem, dur, gap = rm.profile_columns(launches)
    assert grid.tolist() == [148, 1] and threads.dtype == np.uint32 and smem.tolist() == [200000, 0]
    assert dur.dtype == np.float32 and dur.tolist() == [400.5, 3.0] and gap.tolist() == [1.5, 0.0]
    assert all(len(x) == 0 for x in rm.profile_columns([]))


def test_structures_match_the_header():
    """Sizes of the packed structures, from the field types of the C header."""
    assert len(rows()) == 32 and C.sizeof(serving._RopeTable) == 24 and C.sizeof(serving._Launch) == 56
    assert C.sizeof(serving._KVCache) == 9 * 4 + 4 + 10 * 8
