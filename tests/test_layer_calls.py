"""Calls of the loss, the norms around a block and the kept activations that end on the host, without a GPU: nothing to do, and refusals."""
import ctypes

import pytest

from paper_2503_19050_amd import mist

r = ctypes.byref
A = [k << 22 for k in range(1, 32)]  # addresses of tensors that do not overlap


def test_no_sequences_have_no_gates():
    """Without sequences there are no rows of gates' gradients: nothing is launched, so no device is missed."""
    L = mist.load()
    d = mist.BlockDesc(0, 3, 16, 16, 16, 16, 16, 16, 0, 1, 0, 1, 1e-5, 1.0, 1.0)
    g = mist.BlockGrads(None, None, None, None, None, None, None, None, A[8], 16, 16, 16, 16, 16, 0)
    need = ctypes.c_size_t()
    assert L.mist_block_workspace(r(d), r(g), r(need)) == 0
    assert L.mist_block_backward(r(d), None, None, None, None, None, None, A[9], r(g), A[10], need.value, None) == 0


def clash(call, args, sizes, outs, may=()):
    """Every pair of arguments with an output among them, at one place and at the last byte of the other's: refused, but for the pairs in may."""
    L = mist.load()
    names = list(args)
    for o in outs:
        for other in names:
            if o == other or (o, other) in may or (other, o) in may:
                continue
            for at in (args[other], args[other] + sizes[other] - 16, args[other] - sizes[o] + (256 if o == "ws" else 16)):
                assert call(**dict(args, **{o: at})) == -1, (o, other)
                assert b"overlap" in L.mist_last_error(), (o, other, L.mist_last_error())


def test_token_outputs_that_share_memory():
    """Rows of 64 fp32 logits for 2 x 8 tokens: 4096 bytes, 64 for a float a token, 256 for its statistics."""
    L = mist.load()
    d = mist.TokenDesc(2, 8, 64, 0, 8, 512, 64, 512, 64, 8, 0, 4, 1.0)
    names = ["logits", "targets", "logp", "lse", "entropy", "top_ids", "top_logp", "stats", "weights", "dlogp", "dentropy", "dlogits"]
    at = dict(zip(names, A))
    size = dict.fromkeys(names, 64)
    size.update(logits=4096, dlogits=4096, targets=128, top_ids=256, top_logp=256, stats=256)
    pick = lambda *n: ({k: at[k] for k in n}, {k: size[k] for k in n})  # noqa: E731
    n = ("logits", "targets", "logp", "lse", "entropy", "top_ids", "top_logp")
    clash(lambda **a: L.mist_token_logprob(r(d), *(a[k] for k in n), None), *pick(*n), n[2:])
    n2 = ("logits", "targets", "stats", "top_ids", "top_logp")
    clash(lambda **a: L.mist_token_part(r(d), *(a[k] for k in n2), None), *pick(*n2), n2[2:])
    n3 = ("logits", "targets", "lse", "dlogp", "entropy", "dentropy", "dlogits")
    clash(lambda **a: L.mist_token_grad(r(d), *(a[k] for k in n3), None), *pick(*n3), ("dlogits",), [("dlogits", "logits")])
    n4 = ("logits", "targets", "weights", "logp", "dlogits")
    clash(lambda **a: L.mist_token_loss(r(d), a["logits"], a["targets"], a["weights"], 1.0, a["logp"], a["dlogits"], None), *pick(*n4), ("logp", "dlogits"), [("dlogits", "logits")])
    at.update(all_stats=A[20], all_ids=A[21], all_z=A[22])
    size.update(all_stats=768, all_ids=768, all_z=768)
    n5 = ("all_stats", "all_ids", "all_z", "targets", "logp", "lse", "entropy", "top_ids", "top_logp")
    clash(lambda **a: L.mist_token_join(r(d), 3, *(a[k] for k in n5), None), *pick(*n5), n5[4:])
    in_place = mist.TokenDesc(2, 8, 64, 0, 8, 512, 64, 512, 64, 8, 0, 0, 1.0)
    assert L.mist_token_loss(r(in_place), A[0], A[1], None, 1.0, A[0] + 4032, A[0], None) == -1


def test_block_outputs_that_share_memory():
    """2 x 8 rows of 64 bf16 values: 2048 bytes, with an fp32 residual 4096; weights of fp32: 256, gates by sequence 512."""
    L = mist.load()
    d = mist.BlockDesc(2, 8, 64, 64, 64, 64, 64, 64, 0, 1, 0, 0, 1e-5, 1.0, 1.0)
    n = ("x", "block", "weight", "bias", "post_weight", "post_bias", "gate", "y", "h", "stats")
    at = dict(zip(n, A))
    size = dict.fromkeys(n, 256)
    size.update(x=4096, y=4096, block=2048, h=2048, gate=512)
    clash(lambda **a: L.mist_block_forward(r(d), *(a[k] for k in n), None), at, size, n[7:], [("y", "x")])
    g = ("dh", "dy", "dx", "dblock", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate")
    f = ("y", "block", "stats", "weight", "post_weight", "post_bias", "gate")
    need = ctypes.c_size_t()
    places = dict(zip(g + f + ("ws",), A))
    assert L.mist_block_workspace(r(d), r(mist.BlockGrads(*(places[k] for k in g), 64, 64, 64, 64, 64, 0)), r(need)) == 0
    size = dict.fromkeys(places, 256)
    size.update(dh=2048, dblock=2048, block=2048, dy=4096, dx=4096, y=4096, gate=512, dgate=512, ws=need.value)

    def back(**a):
        grads = mist.BlockGrads(*(a[k] for k in g), 64, 64, 64, 64, 64, 0)
        return L.mist_block_backward(r(d), *(a[k] for k in f), r(grads), a["ws"] // 256 * 256, need.value, None)

    clash(back, places, size, g[2:] + ("ws",), [("dx", "dy"), ("dblock", "dh"), ("dblock", "block")])


def test_gates_beside_their_gradients():
    """Columns of one buffer at one stride that meet."""
    L = mist.load()
    d = mist.BlockDesc(2, 8, 64, 64, 64, 64, 64, 128, 0, 1, 0, 0, 1e-5, 1.0, 1.0)
    grads = lambda dgate: mist.BlockGrads(A[0], A[1], A[2], A[3], None, None, None, None, dgate, 64, 64, 64, 64, 128, 0)  # noqa: E731
    back = lambda dgate, d=d: L.mist_block_backward(r(d), A[4], A[5], A[6], A[7], None, None, A[8], r(grads(dgate)), A[9], 1 << 20, None)  # noqa: E731
    assert back(A[8] + 252) == -1 and b"overlap" in L.mist_last_error()
    assert back(A[8] - 252) == -1 and b"overlap" in L.mist_last_error()


def test_calls_without_targets():
    torch = mist._torch()
    x = torch.zeros(2, 3, 8)
    for call in (lambda: mist.token_part(x, None, vocab_begin=0), lambda: mist.token_loss(x, None)):
        with pytest.raises(mist.MistError, match="targets") as e:
            call()
        assert e.value.status == mist.E_INVALID


@pytest.mark.parametrize("grad", [False, True])
def test_tangents_are_not_dropped(grad):
    torch = mist._torch()
    t = torch.zeros(2, 3, dtype=torch.int64)
    with torch.autograd.forward_ad.dual_level(), torch.set_grad_enabled(grad):
        plain = torch.zeros(2, 3, 8)
        x = torch.autograd.forward_ad.make_dual(plain, torch.ones(2, 3, 8))
        for call in (lambda: mist.token_logprob(x, t), lambda: mist.token_loss(x, t), lambda: mist.token_part(x, t, vocab_begin=0), lambda: mist.block_norm(x, weight=plain[0, 0]),
                     lambda: mist.block_norm(plain, weight=x[0, 0]), lambda: mist.checkpoint_store(x), lambda: mist.mlp_act(plain, x)):
            with pytest.raises(mist.MistError, match="tangent"):
                call()
        with pytest.raises(mist.MistError, match="GPU"):   # without one they go on to the next check
            mist.token_logprob(plain, t)


def test_what_the_norm_is_of():
    L = mist.load()
    for bad in (2, -1):
        d = mist.BlockDesc(2, 3, 16, 16, 16, 16, 16, 0, 0, 1, 0, 1, 1e-5, 1.0, 1.0, bad)
        assert L.mist_block_forward(r(d), *A[:3], None, None, None, None, *A[3:6], None) == -1 and b"of_sum" in L.mist_last_error()
