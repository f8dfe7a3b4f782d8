"""CPU-only checks of the sequence operators' boundary: exports, argument checks of the C-ABI, frequencies (no kernel is launched)."""
import ctypes as C
import math
import os
import re

import pytest

from paper_2311_09445_amd import per, sequence as seq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Rows(C.Structure):
    _fields_ = [("d", C.c_void_p), ("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class States(C.Structure):
    _fields_ = [("d", C.c_void_p), ("batch", C.c_int64), ("head", C.c_int64)]


class Rotary(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "dtype", "batch", "length", "heads", "kv_heads", "dim", "rot", "layout", "inverse")] + \
               [("magnitude", C.c_float), ("eps", C.c_float)]


class Attention(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("struct_size", "dtype", "batch", "length", "heads", "kv_heads", "dk", "dv")] + [("scale", C.c_float)]


def rotary(**kw):
    c = Rotary(C.sizeof(Rotary), 1, 1, 2, 4, 2, 64, 64, 0, 0, 1.0, 1e-6)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def attention(**kw):
    c = Attention(C.sizeof(Attention), 1, 2, 8, 4, 2, 64, 64, 0.125)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "per_seq.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(per_[a-z_]+)\s*\(", text)))
    assert names == sorted(seq.EXPORTS)
    for n in names:
        assert hasattr(per._lib(), n), n


def test_binding_loads():
    assert {"linear_attention", "rotate", "norm_rotate"} <= set(dir(seq._calls()))


def fake(p=0x1000):
    return C.byref(Rows(p, 4096, 512, 64))


def test_attention_checks_before_any_work():
    lib = per._lib()
    size = C.c_size_t(0)
    ask = lib.per_linear_attention_workspace
    assert ask(C.byref(attention()), 0, C.byref(size)) == per.OK
    assert ask(C.byref(attention()), 1, C.byref(size)) == per.OK and size.value > 0     # shared heads: sums apart
    for bad, code in [(dict(struct_size=8), per.EINVAL), (dict(dtype=3), per.EINVAL), (dict(dk=0), per.ERANGE), (dict(dv=129), per.ERANGE),
                      (dict(kv_heads=3), per.EINVAL), (dict(kv_heads=0), per.EINVAL), (dict(scale=math.nan), per.EINVAL),
                      (dict(length=1 << 31), per.ERANGE), (dict(batch=1 << 24), per.ERANGE)]:
        assert ask(C.byref(attention(**bad)), 0, C.byref(size)) == code, bad
    assert ask(None, 0, C.byref(size)) == per.EINVAL and ask(C.byref(attention()), 0, None) == per.EINVAL
    call, decay = lib.per_linear_attention, C.c_void_p(0x2000)
    c = C.byref(attention())
    out = fake(0x9000)
    assert call(c, None, fake(), fake(), decay, None, None, out, None, None, C.c_size_t(0), None) == per.EINVAL
    assert call(c, fake(), fake(), fake(), None, None, None, out, None, None, C.c_size_t(0), None) == per.EINVAL
    assert call(c, fake(0x1001), fake(), fake(), decay, None, None, out, None, None, C.c_size_t(0), None) == per.EINVAL
    assert call(c, fake(), fake(), fake(), decay, None, None, fake(), None, None, C.c_size_t(0), None) == per.EINVAL     # out is an input
    assert call(c, fake(), fake(), fake(), decay, None, None, C.byref(Rows(0x9000, 0, 512, 64)), None, None, C.c_size_t(0), None) == per.EINVAL
    assert call(c, fake(), fake(), fake(), decay, None, C.byref(States(None, 0, 0)), out, None, None, C.c_size_t(0), None) == per.EINVAL
    back = lib.per_linear_attention_backward
    rest = (decay, None, None, None, fake(0xa000), fake(0xb000), fake(0xc000), None)
    assert back(c, fake(), fake(), fake(), fake(), *rest, None, C.c_size_t(0), None) == per.EINVAL                   # no workspace
    assert back(c, fake(), fake(), fake(), fake(), *rest, C.c_void_p(0x100), C.c_size_t(16), None) == per.ENOMEM
    assert lib.per_linear_attention_step(c, fake(), fake(), fake(), decay, None, C.byref(States(0x1000, 4096, 4096)), out, None) == per.ERANGE
    one = C.byref(attention(length=1))
    assert lib.per_linear_attention_step(one, fake(), fake(), fake(), decay, None, None, out, None) == per.EINVAL
    empty = C.byref(attention(batch=0))
    assert call(empty, None, None, None, None, None, None, None, None, None, C.c_size_t(0), None) == per.OK


def test_rotary_checks_before_any_work():
    lib = per._lib()
    f = C.c_void_p(0x2000)
    turn = lib.per_rotate
    for bad, code in [(dict(struct_size=8), per.EINVAL), (dict(dtype=0), per.EINVAL), (dict(dim=0), per.ERANGE), (dict(dim=257), per.ERANGE),
                      (dict(rot=63), per.EINVAL), (dict(rot=66), per.EINVAL), (dict(layout=2), per.EINVAL), (dict(magnitude=math.inf), per.EINVAL)]:
        assert turn(C.byref(rotary(**bad)), fake(), None, f, fake(), None) == code, bad
    c = C.byref(rotary())
    assert turn(None, fake(), None, f, fake(), None) == per.EINVAL
    assert turn(c, None, None, f, fake(), None) == per.EINVAL
    assert turn(c, fake(), None, None, fake(), None) == per.EINVAL
    assert turn(c, fake(), None, f, C.byref(Rows(0x1000, 0, 0, 64)), None) == per.EINVAL
    assert turn(C.byref(rotary(batch=0)), None, None, None, None, None) == per.OK
    assert lib.per_norm_rotate(C.byref(rotary(eps=-1.0)), fake(), fake(), None, None, None, f, fake(), fake(), None) == per.EINVAL
    assert lib.per_norm_rotate(c, fake(), None, None, None, None, f, fake(), fake(), None) == per.EINVAL
    size = C.c_size_t(0)
    assert lib.per_norm_rotate_workspace(c, C.byref(size)) == per.OK and size.value > 0
    back = lib.per_norm_rotate_backward
    args = (c, fake(), fake(), fake(), fake(), None, None, None, f, fake(), fake(), None, None)
    assert back(*args, None, size, None) == per.EINVAL
    assert back(*args, C.c_void_p(0x100), C.c_size_t(4), None) == per.ENOMEM


def test_frequencies():
    f, m = seq.rotary_frequencies(8, device="cpu")
    assert m == 1.0 and f.tolist() == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-6)
    g, _ = seq.rotary_frequencies(8, scaling="linear", factor=4.0, device="cpu")
    assert g.tolist() == pytest.approx([x / 4 for x in f.tolist()], rel=1e-6)
    g, _ = seq.rotary_frequencies(8, scaling="base", factor=4.0, device="cpu")
    assert g[0] == 1.0 and float(g[3]) == pytest.approx(float(f[3]) / 4, rel=1e-6)
    g, m = seq.rotary_frequencies(64, scaling="parts", factor=4.0, trained=4096, device="cpu")
    f, _ = seq.rotary_frequencies(64, device="cpu")
    assert g[0] == f[0] and float(g[-1]) == pytest.approx(float(f[-1]) / 4, rel=1e-6) and m == pytest.approx(0.1 * math.log(4) + 1)
    assert all(float(x) <= float(y) for x, y in zip(g, f))
    for bad in (dict(rot=7), dict(rot=0), dict(rot=8, factor=0.0), dict(rot=8, scaling="other"), dict(rot=8, scaling="parts")):
        with pytest.raises(ValueError):
            seq.rotary_frequencies(**{"device": "cpu", **bad})


def test_calls_without_their_tensors_raise():
    c = seq._calls()
    for call, n in ((c.rotate, 7), (c.norm_rotate, 11), (c.norm_rotate_backward, 14), (c.linear_attention, 10), (c.linear_attention_backward, 14),
                    (c.linear_attention_step, 8)):
        with pytest.raises(TypeError):
            call(*([None] * n))
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("sizes", [dict(heads=0, kv_heads=0), dict(batch=0), dict(length=0)])
def test_empty_sizes_need_no_workspace(sizes, backward):
    c, n = attention(**sizes), C.c_size_t(7)
    assert per._lib().per_linear_attention_workspace(C.byref(c), backward, C.byref(n)) == 0
    assert n.value == 0
