"""CPU-only checks of the C-ABI of the gated delta rule, layer norm and dropout: what is refused before any work, workspaces, the oracle itself."""
import ctypes as C
import math

import pytest
import torch

import block_oracle as oracle
from paper_2311_09445_amd import per, sequence as seq


class Rows(C.Structure):
    _fields_ = [("d", C.c_void_p), ("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class States(C.Structure):
    _fields_ = [("d", C.c_void_p), ("batch", C.c_int64), ("head", C.c_int64)]


class Delta(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "dtype", "batch", "length", "heads", "q_heads", "k_heads", "v_heads", "dk", "dv")] + [("scale", C.c_float)]


class Block(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "dtype", "batch", "length", "heads", "dim")] + [("eps", C.c_float), ("p", C.c_float)] + \
               [("seed", C.c_uint64), ("offset", C.c_uint64)]


def delta(**kw):
    c = Delta(C.sizeof(Delta), 1, 2, 8, 4, 4, 2, 1, 64, 64, 0.125)
    for k, v in kw.items():
        setattr(c, k, v)
    return C.byref(c)


def block(**kw):
    c = Block(C.sizeof(Block), 1, 2, 8, 1, 64, 1e-5, 0.1, 1, 2)
    for k, v in kw.items():
        setattr(c, k, v)
    return C.byref(c)


def fake(p=0x1000, batch=4096, token=512, head=64):
    return C.byref(Rows(p, batch, token, head))


NONE, WORK = C.c_size_t(0), C.c_void_p(0x100)


def test_exports():
    assert {"per_gated_delta", "per_gated_delta_backward", "per_gated_delta_step", "per_layer_norm", "per_layer_norm_backward", "per_dropout"} <= set(seq.EXPORTS)
    assert {"gated_delta", "gated_delta_backward", "gated_delta_step", "layer_norm", "layer_norm_backward", "dropout"} <= set(dir(seq._calls()))


def test_delta_checks_before_any_work():
    lib, size = per._lib(), C.c_size_t(0)
    ask = lib.per_gated_delta_workspace
    assert ask(delta(), 0, C.byref(size)) == per.OK and size.value > 0
    forward = size.value
    assert ask(delta(), 1, C.byref(size)) == per.OK and size.value > forward
    for bad, code in [(dict(struct_size=8), per.EINVAL), (dict(dtype=3), per.EINVAL), (dict(dk=0), per.ERANGE), (dict(dk=129), per.ERANGE), (dict(dv=129), per.ERANGE),
                      (dict(q_heads=3), per.EINVAL), (dict(k_heads=0), per.EINVAL), (dict(v_heads=8), per.EINVAL), (dict(heads=0), per.EINVAL),
                      (dict(scale=math.inf), per.EINVAL), (dict(length=1 << 30), per.ERANGE), (dict(batch=1 << 22), per.ERANGE),
                      (dict(batch=1 << 20, length=1 << 10), per.ERANGE)]:
        assert ask(delta(**bad), 0, C.byref(size)) == code, bad
    assert ask(None, 0, C.byref(size)) == per.EINVAL and ask(delta(), 0, None) == per.EINVAL
    call, out = lib.per_gated_delta, fake(0x9000)
    good = [delta(), fake(), fake(), fake(), fake(0x2000), fake(0x3000), None, None, out, None, WORK, C.c_size_t(forward), None]

    def refused(code, at, with_):
        args = list(good)
        args[at] = with_
        assert call(*args) == code, (at, code)
    for at in (1, 2, 3, 4, 5, 8):
        refused(per.EINVAL, at, None)
        refused(per.EINVAL, at, fake(None))
        refused(per.EINVAL, at, fake(0x1001))
    refused(per.EINVAL, 6, C.c_void_p(0x1002))
    refused(per.EINVAL, 7, C.byref(States(None, 0, 0)))
    refused(per.EINVAL, 8, fake())                          # out is an input
    refused(per.EINVAL, 8, fake(0x9000, token=0))           # rows of out at one place
    refused(per.EINVAL, 9, C.byref(States(0x5000, 0, 4096)))
    refused(per.EINVAL, 10, None)
    refused(per.EINVAL, 10, C.c_void_p(0x110))
    refused(per.ENOMEM, 11, C.c_size_t(forward - 1))
    assert call(delta(batch=0), *[None] * 10, NONE, None) == per.OK
    back = lib.per_gated_delta_backward
    assert ask(delta(), 1, C.byref(size)) == per.OK
    good = [delta(), fake(0x8000), fake(), fake(), fake(), fake(0x2000), fake(0x3000), None, None, None, fake(0xa000), fake(0xb000), fake(0xc000),
            fake(0xd000), fake(0xe000), None, WORK, size, None]

    def refused_back(code, at, with_):
        args = list(good)
        args[at] = with_
        assert back(*args) == code, (at, code)
    for at in (1, 2, 3, 4, 5, 6, 10, 11, 12, 13, 14, 16):
        refused_back(per.EINVAL, at, None)
    refused_back(per.EINVAL, 10, fake(0xb000))             # two results at one place
    refused_back(per.EINVAL, 12, fake(0x8000))
    refused_back(per.EINVAL, 13, fake(0xe000))
    refused_back(per.EINVAL, 14, fake(0x2000))
    refused_back(per.EINVAL, 13, fake(0xd000, head=0))
    refused_back(per.ENOMEM, 17, C.c_size_t(size.value - 1))
    state = C.byref(States(0x5000, 4096, 4096))
    args = list(good)
    args[8] = args[15] = state
    assert back(*args) == per.EINVAL
    step = lib.per_gated_delta_step
    args = [fake(), fake(), fake(), fake(0x2000), fake(0x3000), None, state, out, None]
    assert step(delta(), *args) == per.ERANGE
    args[6] = None
    assert step(delta(length=1), *args) == per.EINVAL


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("sizes", [dict(heads=0, q_heads=0, k_heads=0, v_heads=0), dict(batch=0), dict(length=0)])
def test_empty_sizes_need_no_workspace(sizes, backward):
    size = C.c_size_t(1)
    assert per._lib().per_gated_delta_workspace(delta(**sizes), backward, C.byref(size)) == per.OK and size.value == 0


def test_block_checks_before_any_work():
    lib, size = per._lib(), C.c_size_t(0)
    norm, back, drop = lib.per_layer_norm, lib.per_layer_norm_backward, lib.per_dropout
    for bad, code in [(dict(struct_size=8), per.EINVAL), (dict(dtype=0), per.EINVAL), (dict(dim=0), per.ERANGE), (dict(dim=65537), per.ERANGE),
                      (dict(batch=1 << 31, length=2), per.ERANGE)]:
        assert norm(block(**bad), fake(), None, None, fake(), None) == code, bad
        assert "dim" in bad or drop(block(**bad), fake(), None, None, fake(), None) == code, bad
        assert lib.per_layer_norm_workspace(block(**bad), C.byref(size)) == code, bad
    assert drop(block(dim=0), fake(), None, None, fake(), None) == per.ERANGE
    for eps in (-1.0, math.nan, math.inf):
        assert norm(block(eps=eps), fake(), None, None, fake(), None) == per.EINVAL
    for p in (-0.5, 1.0, math.nan):
        assert drop(block(p=p), fake(), None, None, fake(), None) == per.EINVAL
    for call in (lambda x, out: norm(block(), x, None, None, out, None), lambda x, out: drop(block(), x, None, None, out, None)):
        assert call(None, fake()) == per.EINVAL and call(fake(), None) == per.EINVAL and call(fake(0x1001), fake()) == per.EINVAL
        assert call(fake(), fake(0x9000, token=0)) == per.EINVAL
    assert norm(block(), fake(), C.c_void_p(0x1002), None, fake(), None) == per.EINVAL
    assert drop(block(), fake(), None, C.c_void_p(0x1004), fake(), None) == per.EINVAL
    assert drop(block(), fake(), fake(0x1001), None, fake(), None) == per.EINVAL
    assert norm(block(batch=0), None, None, None, None, None) == per.OK and drop(block(length=0), None, None, None, None, None) == per.OK
    assert lib.per_layer_norm_workspace(block(), C.byref(size)) == per.OK and size.value > 0
    w, b = C.c_void_p(0x2000), C.c_void_p(0x3000)
    assert back(block(), fake(0x8000), fake(), None, fake(0x9000), w, b, None, size, None) == per.EINVAL
    assert back(block(), fake(0x8000), fake(), None, fake(0x9000), w, b, WORK, C.c_size_t(size.value - 1), None) == per.ENOMEM
    assert back(block(), fake(0x8000), fake(), None, fake(), w, b, WORK, size, None) == per.EINVAL            # dx is x
    assert back(block(), fake(0x8000), fake(), None, fake(0x9000), w, w, WORK, size, None) == per.EINVAL      # both at one place


def test_forward_mode_is_refused():
    """A tangent that a call does not know of would be lost without a word; every tensor of every call is asked, before anything else."""
    from torch.autograd import forward_ad
    t = torch.zeros(2, 4, 2, 8)
    s, g, w = torch.zeros(2, 2, 8, 8), torch.zeros(2, 4, 2), torch.zeros(8)
    calls = [(lambda x, f: seq.rotate(x, None, f), (t, w[:4])), (lambda q, k, a, b, f: seq.norm_rotate(q, k, a, b, None, f), (t, t, w, w, w[:4])),
             (lambda x, y, q, k, a, b, f: seq.norm_rotate_backward(x, y, q, k, a, b, None, f), (t, t, t, t, w, w, w[:4])), (seq.linear_attention, (t, t, t, w[:2], s)),
             (seq.linear_attention_backward, (t, t, t, t, w[:2], s)), (seq.linear_attention_step, (t, t, t, w[:2], s)), (seq.gated_delta, (t, t, t, g, g, s)),
             (seq.gated_delta_backward, (t, t, t, t, g, g, s, s)), (seq.gated_delta_step, (t, t, t, g, g, s)), (seq.layer_norm, (t, w, w)),
             (seq.layer_norm_backward, (t, t, w)), (lambda x, r: seq.dropout(x, 0.1, 0, residual=r), (t, t))]
    with forward_ad.dual_level():
        for call, args in calls:
            for i, a in enumerate(args):
                given = list(args)
                given[i] = forward_ad.make_dual(a, torch.ones_like(a))
                with pytest.raises(RuntimeError, match="forward"):
                    call(*given)


def test_views_that_stand_for_their_negative_are_refused():
    """torch keeps the imaginary part of a conjugate as a view of the memory that holds the opposite."""
    t, s, g = torch.zeros(2, 4, 2, 8), torch.zeros(2, 2, 8, 8), torch.zeros(2, 4, 2)
    lazy = torch.complex(g, g).conj().imag
    assert lazy.is_neg()
    for call in (lambda: seq.gated_delta(t, t, t, lazy, g), lambda: seq.gated_delta(t, t, t, g, lazy), lambda: seq.layer_norm(t._neg_view()),
                 lambda: seq.gated_delta_step(t[:, :1], t[:, :1], t[:, :1], g[:, :1], lazy[:, :1], s), lambda: seq.dropout(t, 0.1, 0, residual=t._neg_view())):
        with pytest.raises(ValueError, match="negative"):
            call()


def test_random_words():
    """Known answers of Philox4x32-10, as its authors publish them."""
    assert oracle.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert oracle.philox((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_the_rule_replaces_what_a_key_holds():
    """With strength 1, a key of length 1 and no decay, what is read back is what was written last, and other keys are left alone."""
    k = torch.eye(3, dtype=torch.float64)[[0, 1, 0, 2]].reshape(1, 4, 1, 3)
    v = torch.arange(8, dtype=torch.float64).reshape(1, 4, 1, 2)
    _, S = oracle.delta(k, k, v, torch.zeros(1, 4, 1, dtype=torch.float64), torch.ones(1, 4, 1, dtype=torch.float64))
    assert torch.equal(S[0, 0], v[0, [2, 1, 3], 0])
