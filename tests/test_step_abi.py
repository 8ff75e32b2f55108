"""Argument checks of the training-step operators without a GPU: every refusal comes before the device is used."""
import ctypes

import pytest

from paper_2503_19050_amd import mist

P = 4096  # a non-null address that no refused call reads


def _embed(**over):
    d = mist.EmbedDesc()
    for k, v in dict(dict(batch=2, seq=3, hidden=8, rows=5, vocab_begin=0, ids_stride=3, act_batch_stride=24, act_stride=8,
                          table_stride=8, pos_stride=8, ids_bytes=8, act_type=1, table_type=0, scale=1.0), **over).items():
        setattr(d, k, v)
    return d


BAD = [dict(batch=-1), dict(seq=-1), dict(batch=1 << 20, seq=1 << 20), dict(hidden=0), dict(hidden=1 << 25), dict(rows=0),
       dict(rows=1 << 31), dict(vocab_begin=-1), dict(vocab_begin=1 << 31), dict(ids_bytes=2), dict(act_type=3),
       dict(table_type=-1), dict(scale=float("inf")), dict(scale=float("nan")), dict(table_stride=7), dict(ids_stride=-1),
       dict(act_stride=1 << 41), dict(pos_stride=-8)]


@pytest.mark.parametrize("over", BAD, ids=str)
def test_embedding_descriptors_are_refused(over):
    L = mist.load()
    d = _embed(**over)
    need = ctypes.c_size_t()
    assert L.mist_embed_workspace(ctypes.byref(d), ctypes.byref(need)) == -1 and L.mist_last_error()
    assert L.mist_embed_forward(ctypes.byref(d), P, P, None, P, None) == -1
    assert L.mist_embed_backward(ctypes.byref(d), P, P, P, None, 0, P, 1 << 40, None) == -1


def test_embedding_buffers_are_refused():
    L = mist.load()
    d = _embed()
    r = ctypes.byref
    for args in ((None, P, None, P), (P, None, None, P), (P, P, None, None), (P + 4, P, None, P), (P, P + 2, None, P),
                 (P, P, P + 1, P), (P, P, None, P + 1)):
        assert L.mist_embed_forward(r(d), *args, None) == -1
    assert L.mist_embed_forward(None, P, P, None, P, None) == -1
    for over in (dict(act_stride=7), dict(act_batch_stride=23), dict(act_batch_stride=0), dict(act_stride=0)):
        assert L.mist_embed_forward(r(_embed(**over)), P, P, None, P, None) == -1 and b"overlap" in L.mist_last_error()
    assert L.mist_embed_forward(r(_embed(pos_stride=4)), P, P, P, P, None) == -1
    need = ctypes.c_size_t()
    assert L.mist_embed_workspace(r(d), r(need)) == 0  # a short input may need none
    d = _embed(seq=3000, ids_stride=3000, act_batch_stride=24000)
    assert L.mist_embed_workspace(r(d), r(need)) == 0 and need.value > 0
    assert L.mist_embed_workspace(r(d), None) == -1 and L.mist_embed_workspace(None, r(need)) == -1
    for args in ((None, P, P, None, 0, P), (P, None, P, None, 0, P), (P, P, None, None, 0, P), (P, P, P, None, 0, None),
                 (P, P, P, None, 2, P), (P, P, P, None, 0, P + 128), (P, P, P, P + 2, 0, P)):
        assert L.mist_embed_backward(r(d), *args, need.value, None) == -1
    assert L.mist_embed_backward(r(d), P, P, P, None, 0, P, need.value - 1, None) == -5


def test_nothing_to_look_up():
    assert mist.load().mist_embed_forward(ctypes.byref(_embed(batch=0)), None, None, None, None, None) == 0


def test_tensor_lists_are_refused():
    L = mist.load()
    out = ctypes.c_void_p(1)
    ptrs, sizes = (ctypes.c_void_p * 2)(P, P + 2), (ctypes.c_int64 * 2)(4, 4)

    def create(ptrs=ptrs, sizes=sizes, n=2, type_=1, alloc=None, out=ctypes.byref(out)):
        return L.mist_tensors_create(ptrs, sizes, n, type_, alloc, out)

    assert create(out=None) == -1
    for bad in (dict(n=-1), dict(type_=5), dict(type_=0), dict(ptrs=None), dict(sizes=None),
                dict(ptrs=(ctypes.c_void_p * 2)(P, None)), dict(sizes=(ctypes.c_int64 * 2)(4, -1)),
                dict(sizes=(ctypes.c_int64 * 2)(1 << 41, 1 << 41)), dict(alloc=ctypes.byref(mist.Allocator()))):
        assert create(**bad) == -1 and L.mist_last_error() and not out.value, bad
    assert L.mist_tensors_destroy(None) == 0


def test_null_arguments():
    L = mist.load()
    c, a = mist.ClipDesc(0, 1.0, 1.0), mist.AdamDesc(0.1, 0.9, 0.99, 1e-8, 0.0)
    r = ctypes.byref
    need = ctypes.c_size_t()
    assert L.mist_norm_workspace(None, r(need)) == -1
    assert L.mist_grad_norm(None, r(c), 0, 1, P, P, 8, None) == -1
    assert L.mist_grad_finish(None, P, None) == -1 and L.mist_grad_finish(r(c), None, None) == -1
    assert L.mist_grad_finish(r(c), P + 4, None) == -1
    for bad in (mist.ClipDesc(2, 1.0, 1.0), mist.ClipDesc(0, 0.0, 1.0), mist.ClipDesc(0, float("nan"), 1.0),
                mist.ClipDesc(0, 1.0, 0.0), mist.ClipDesc(0, 1.0, float("nan"))):
        assert L.mist_grad_finish(r(bad), P, None) == -1
    assert L.mist_grad_clip(None, P, None, None) == -1
    assert L.mist_adam_step(None, None, None, None, None, P, r(a), None) == -1
