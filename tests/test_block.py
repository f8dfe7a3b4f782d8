"""Layer norm and dropout on the GPU against their definitions in 64 bits.

How far results may be off: sums of D values in fp32, of roundings of either sign (about sqrt(D) of 2^-24 of what is summed in 2-norm,
a row's mean and variance being sums of all its values), then one rounding to the result's type.  A mean that is far from zero leaves x - mean
off by 2^-24 of the mean, which is taken into account by its size in standard deviations."""
import math

import pytest
import torch

import block_oracle as oracle
from paper_2311_09445_amd import sequence as seq

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
UNIT = {BF16: oracle.U_BF16, F32: oracle.U_F32}


def normal(seed, *shape, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g, dtype=torch.float32).to(dtype).cuda()


def close(got, want, dtype, rel, what):
    """One rounding of the element, and `rel` of the tensor's root mean square 16 times over (elements), once (2-norm)."""
    got = oracle.f64(got)
    assert got.shape == want.shape and torch.isfinite(got).all(), what
    if not want.numel():
        return
    size = float(want.norm()) + 1e-30
    rms = size / math.sqrt(want.numel())
    off = (got - want).abs()
    assert float(off.norm()) <= (UNIT[dtype] + rel) * size, f"{what}: {float(off.norm()) / size:.3g}"
    worst = float((off - UNIT[dtype] * want.abs()).max())
    assert worst <= 16 * rel * rms, f"{what}: {worst / rms:.3g} of the root mean square"


def u32(n):
    return oracle.U_F32 * (4 + math.sqrt(n))


WIDTHS = [1, 3, 4, 7, 8, 9, 64, 255, 257, 511, 512, 513, 1024, 1025, 1537, 2047, 2048, 2049, 4096, 5000, 8191, 8192, 8193, 20001]


@TYPES
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("D", WIDTHS)
def test_layer_norm(D, weights, dtype):
    x = (normal(1, 3, 5, D) * (1 + normal(2, 3, 5, 1).abs()) + normal(3, D)).to(dtype)
    w, b = (1 + 0.1 * normal(4, D), 0.1 * normal(5, D)) if weights else (None, None)
    dout = normal(6, 3, 5, D, dtype=dtype)
    eps = 1e-3       # (a row of one or two values has next to no variance)
    close(seq.layer_norm(x, w, b, eps), oracle.norm(x, w, b, eps), dtype, u32(D), "out")
    dx, dw, db = seq.layer_norm_backward(dout, x, w, eps)
    wx, ww, wb = oracle.norm_backward(dout, x, w, eps)
    # h - mean h - y mean(h y): what is left may be smaller than what is taken apart, which is h / sqrt(variance) of its row
    size = float((oracle.f64(dout) * (1 if w is None else oracle.f64(w)) / torch.sqrt(oracle.f64(x).var(-1, unbiased=False, keepdim=True) + eps)).norm())
    off = (oracle.f64(dx) - wx).abs()
    assert float(off.norm()) <= UNIT[dtype] * float(wx.norm()) + 2 * u32(D) * size
    assert float((off - UNIT[dtype] * wx.abs()).max()) <= 32 * u32(D) * size / math.sqrt(wx.numel())
    close(dw, ww, F32, u32(15) + u32(D), "dweight")
    close(db, wb, F32, u32(15), "dbias")


@TYPES
@pytest.mark.parametrize("shape", [(70000, 24), (5000, 1536), (3000, 2500), (1100, 9000), (2, 700, 3, 40), (1, 1, 1, 16), (64,)])
def test_layer_norm_of_many_rows(shape, dtype):
    x, dout = normal(1, *shape, dtype=dtype), normal(2, *shape, dtype=dtype)
    w, b = 1 + 0.1 * normal(4, shape[-1]), 0.1 * normal(5, shape[-1])
    rows = x.numel() // shape[-1]
    close(seq.layer_norm(x, w, b), oracle.norm(x, w, b, 1e-5), dtype, u32(shape[-1]), "out")
    dx, dw, db = seq.layer_norm_backward(dout, x, w)
    wx, ww, wb = oracle.norm_backward(dout, x, w, 1e-5)
    close(dx, wx, dtype, 2 * u32(shape[-1]), "dx")
    close(dw, ww, F32, u32(rows) + u32(shape[-1]), "dweight")
    close(db, wb, F32, u32(rows), "dbias")
    again = seq.layer_norm_backward(dout, x, w)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))
    only, none, _ = seq.layer_norm_backward(dout, x, w, want_weights=False)
    assert none is None and torch.equal(only, dx)


@TYPES
@pytest.mark.parametrize("shape", [(70000, 16), (70000, 48), (20000, 40), (20000, 65), (20000, 100), (40000, 128), (20001, 200), (20000, 256), (5000, 129), (5000, 300),
                                   (5000, 600), (1100, 5000)])
def test_layer_norm_of_many_rows_of_every_shape(shape, dtype):
    """Rows for two turns of a loop over them, forward and against, in each number of lanes and pieces that widths are given."""
    test_layer_norm_of_many_rows(shape, dtype)


@TYPES
@pytest.mark.parametrize("D", [65, 100, 127, 128, 129, 200])
@pytest.mark.parametrize("weights", [True, False])
def test_layer_norm_of_rows_of_sixteen_lanes(D, weights, dtype):
    test_layer_norm(D, weights, dtype)


@TYPES
@pytest.mark.parametrize("D", [5, 40, 513, 2500, 9001])
def test_layer_norm_strides_and_in_place(D, dtype):
    pool = normal(1, 4, 3, 6, D + 3, dtype=dtype)
    x = pool[::2, :, 1:4, 1:D + 1]
    w, b = 1 + 0.1 * normal(4, D), 0.1 * normal(5, D)
    dout = normal(2, 3, 2, 3, D, dtype=dtype).transpose(0, 1)
    want = seq.layer_norm(x.contiguous(), w, b)
    back = seq.layer_norm_backward(dout.contiguous(), x.contiguous(), w)
    assert torch.equal(seq.layer_norm(x, w, b), want)
    assert all(torch.equal(p, q) for p, q in zip(seq.layer_norm_backward(dout, x, w), back))
    d = dout.clone()
    seq.layer_norm_backward(d, x, w, dx=d)
    assert torch.equal(d, back[0])
    before = pool.clone()
    seq.layer_norm(x, w, b, out=x)
    assert torch.equal(x, want)
    before[::2, :, 1:4, 1:D + 1] = want
    assert torch.equal(pool, before)


@TYPES
def test_layer_norm_of_rows_without_variance(dtype):
    x = torch.full((3, 100), 5.0, dtype=dtype, device="cuda")
    b = normal(5, 100)
    assert torch.equal(seq.layer_norm(x, None, b), b.to(dtype).expand(3, 100))
    # far from the origin: the variance is that of the differences
    x = (1000 + normal(1, 4, 1000)).to(dtype)
    close(seq.layer_norm(x), oracle.norm(x, None, None, 1e-5), dtype, u32(1000) + 1000 * oracle.U_F32, "far")
    # a row that is not finite stays by itself
    y = normal(1, 5, 700, dtype=dtype)
    want = seq.layer_norm(y)
    y[2, 3] = math.nan
    got = seq.layer_norm(y)
    assert got[2].isnan().all() and torch.equal(got[[0, 1, 3, 4]], want[[0, 1, 3, 4]])


def test_layer_norm_gradient_against_differences():
    x, w, b, dout = (normal(i, *s) for i, s in enumerate([(6, 50), (50,), (50,), (6, 50)]))
    grads = seq.layer_norm_backward(dout, x, w)
    for i in range(3):
        along = [torch.zeros(t.shape, dtype=torch.float64) for t in (x, w, b)]
        along[i] = torch.randn(along[i].shape, generator=torch.Generator().manual_seed(9), dtype=torch.float64)
        value = lambda s: float((oracle.norm(*(oracle.f64(t) + s * a for t, a in zip((x, w, b), along)), 1e-5) * oracle.f64(dout)).sum())  # noqa: E731
        want, step = (value(1e-4) - value(-1e-4)) / 2e-4, float(oracle.f64(grads[i]).norm())
        assert abs(float((oracle.f64(grads[i]) * along[i]).sum()) - want) <= 1e-5 * step + 1e-6 * abs(want)


def test_layer_norm_of_nothing():
    x = torch.zeros(0, 4, 30, device="cuda")
    dx, dw, db = seq.layer_norm_backward(x, x, None)
    assert seq.layer_norm(x).shape == x.shape and dx.shape == x.shape and not dw.any() and not db.any()


def test_rows_behind_2_to_31_elements():
    n, D = (1 << 31) // 64 + 3, 64
    x = torch.empty(n, D, dtype=BF16, device="cuda")
    x[:3] = normal(1, 3, D)
    x[-3:] = normal(2, 3, D)
    x[3:-3] = 1.0
    out = seq.layer_norm(x)
    close(out[-3:], oracle.norm(x[-3:], None, None, 1e-5), BF16, u32(D), "last rows")
    seq.dropout(x, 0.5, 3, 4, out=out)
    keep = oracle.kept(3 * D, 0.5, 3, 4, first=(n - 3) * D).reshape(3, D)
    assert torch.equal(oracle.f64(out[-3:]), torch.where(keep, 2 * oracle.f64(x[-3:]), torch.zeros(3, D, dtype=torch.float64)))


# ---------------------------------------------------------------------------------------------------------------- dropout
@TYPES
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("p,seed,offset", [(0.0, 0, 0), (0.1, 5, 7), (0.5, 2 ** 64 - 1, 2 ** 64 - 1), (1 - 2 ** -17, 2 ** 40 + 3, 2 ** 33)])
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5), (2, 3, 129), (2, 2, 3, 64)])
def test_dropout(shape, p, seed, offset, residual, dtype):
    x = normal(1, *shape, dtype=dtype)
    r = normal(2, *shape, dtype=dtype) if residual else None
    got = seq.dropout(x, p, seed, offset, residual=r)
    keep = oracle.kept(x.numel(), p, seed, offset).reshape(shape)
    factor = 65536 / (65536 - min(65535, math.floor(p * 65536 + 0.5)))
    want = torch.where(keep, oracle.f64(x) * factor, torch.zeros(shape, dtype=torch.float64)) + (oracle.f64(r) if residual else 0)
    # the factor, the product and the sum are rounded in fp32 (each to 2^-24 of itself), then the result
    inner = 3 * oracle.U_F32 * (oracle.f64(x).abs() * factor * keep + want.abs())
    assert ((oracle.f64(got) - want).abs() <= UNIT[dtype] * want.abs() * (1 + 2 ** -8) + inner).all()
    if not residual:
        assert not got.cpu()[~keep].any()
    # from the device
    if offset < 2 ** 63:
        at = torch.tensor([offset], dtype=torch.int64, device="cuda")
        assert torch.equal(seq.dropout(x, p, seed, at, residual=r), got)


@TYPES
def test_dropout_strides_and_in_place(dtype):
    """Places are counted over the shape, whatever the strides."""
    pool = normal(1, 6, 5, 40, dtype=dtype)
    x, r = pool[::2, :, 2:39], normal(2, 5, 3, 37, dtype=dtype).transpose(0, 1)
    want = seq.dropout(x.contiguous(), 0.3, 1, 2, residual=r.contiguous())
    assert torch.equal(seq.dropout(x, 0.3, 1, 2, residual=r), want)
    y, z = x.clone(), r.clone()
    assert seq.dropout(y, 0.3, 1, 2, residual=r, out=y) is not None and torch.equal(y, want)
    seq.dropout(x, 0.3, 1, 2, residual=z, out=z)
    assert torch.equal(z, want)
    before = pool.clone()
    seq.dropout(x, 0.3, 1, 2, residual=r, out=x)
    before[::2, :, 2:39] = want
    assert torch.equal(pool, before)
    assert seq.dropout(x[:0], 0.3, 1).shape == (0, 5, 37)


def test_dropped_places_may_hold_anything():
    x = torch.full((4000,), math.nan, device="cuda")
    keep = oracle.kept(4000, 0.5, 1, 2)
    x[keep.cuda()] = 1.0
    assert torch.equal(seq.dropout(x, 0.5, 1, 2).cpu(), 2.0 * keep.float())


def test_shares_next_to_one_and_next_to_half_a_step():
    """The share is taken to the nearest 1/65536 as it is given, in 64 bits: in fp32 one next to 1 would be 1, and one next to a tie the tie."""
    x = torch.ones(1 << 16, device="cuda")
    assert torch.equal(seq.dropout(x, 1 - 1e-12, 3), seq.dropout(x, 65535 / 65536, 3))
    tie = 100.5 / 65536
    assert torch.equal(seq.dropout(x, tie * (1 - 1e-12), 3), seq.dropout(x, 100 / 65536, 3))
    assert torch.equal(seq.dropout(x, tie, 3), seq.dropout(x, 101 / 65536, 3))
    assert not torch.equal(seq.dropout(x, 100 / 65536, 3), seq.dropout(x, 101 / 65536, 3))


def test_dropout_drops_its_share():
    """Of 2^20 elements; the count's standard deviation is sqrt(n p (1 - p)), and six of them are allowed."""
    n = 1 << 20
    for p in (0.1, 0.5, 0.9):
        for seed in (0, 1):
            kept = seq.dropout(torch.ones(n, device="cuda"), p, seed) != 0
            assert abs(int((~kept).sum()) - n * p) <= 6 * math.sqrt(n * p * (1 - p)) + n / 65536
            other = seq.dropout(torch.ones(n, device="cuda"), p, seed, 1) != 0
            both = int((~kept & ~other).sum())
            assert abs(both - n * p * p) <= 6 * math.sqrt(n * p * p * (1 - p * p)) + n / 32768


def test_autograd():
    x, w, b = normal(1, 6, 100).requires_grad_(), (1 + 0.1 * normal(2, 100)).requires_grad_(), normal(3, 100).requires_grad_()
    dout = normal(4, 6, 100)
    y = seq.dropout(seq.layer_norm(x, w, b), 0.2, 3, 4, residual=x)
    y.backward(dout)
    d = seq.dropout(dout, 0.2, 3, 4)
    dx, dw, db = seq.layer_norm_backward(d, x.detach(), w.detach())
    assert torch.equal(x.grad, dx + dout) and torch.equal(w.grad, dw) and torch.equal(b.grad, db)
    # a residual alone
    r = normal(5, 6, 100).requires_grad_()
    seq.dropout(x.detach(), 0.2, 3, residual=r).backward(dout)
    assert torch.equal(r.grad, dout)
    # dropout is linear: its gradient has one too; that of the norm does not
    z = normal(6, 6, 100).requires_grad_()
    (g,) = torch.autograd.grad(seq.dropout(z, 0.2, 3), z, dout.requires_grad_(), create_graph=True)
    g.sum().backward()
    assert torch.equal(dout.grad, seq.dropout(torch.ones_like(dout), 0.2, 3))
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(seq.layer_norm(x).sum(), x, create_graph=True)[0].sum(), x)
    with pytest.raises(RuntimeError):
        seq.layer_norm(x, out=torch.empty(6, 100, device="cuda"))
    # an offset that moved between a call and its gradient is noticed
    at = torch.zeros(1, dtype=torch.int64, device="cuda")
    y = seq.dropout(x, 0.2, 3, at)
    at += 1
    with pytest.raises(RuntimeError):
        y.sum().backward()


def test_refusals():
    x, w = normal(1, 4, 32), torch.ones(32, device="cuda")
    refused = [
        lambda: seq.layer_norm(x.half()), lambda: seq.layer_norm(x.cpu()), lambda: seq.layer_norm(x, w[:31]), lambda: seq.layer_norm(x, w.bfloat16()),
        lambda: seq.layer_norm(x, None, w.cpu()), lambda: seq.layer_norm(x, eps=-1.0), lambda: seq.layer_norm(x, eps=math.nan), lambda: seq.layer_norm(x.T),
        lambda: seq.layer_norm(x, out=x[:3]), lambda: seq.layer_norm(x, out=x.bfloat16()), lambda: seq.layer_norm(x[0, 0]),
        lambda: seq.layer_norm(x.expand(1, 1, 1, 4, 32)), lambda: seq.layer_norm(x, out=x[:1].expand(4, 32)), lambda: seq.layer_norm(x[:, :0]),
        lambda: seq.layer_norm(torch.zeros(1, 65537, device="cuda")), lambda: seq.layer_norm_backward(x[:3], x), lambda: seq.layer_norm_backward(x, x, dx=x),
        lambda: seq.dropout(x, 1.0, 0), lambda: seq.dropout(x, -0.1, 0), lambda: seq.dropout(x, math.nan, 0), lambda: seq.dropout(x, 0.1, -1),
        lambda: seq.dropout(x, 0.1, 2 ** 64), lambda: seq.dropout(x, 0.1, 0.5), lambda: seq.dropout(x, 0.1, 0, -1), lambda: seq.dropout(x, 0.1, 0, w[:1]),
        lambda: seq.dropout(x, 0.1, 0, torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: seq.dropout(x, 0.1, 0, torch.zeros(1, dtype=torch.int64)),
        lambda: seq.dropout(x, 0.1, 0, residual=x[:1]), lambda: seq.dropout(x, 0.1, 0, out=x[:, :31]), lambda: seq.dropout(x.double(), 0.1, 0),
        lambda: seq.dropout(x, 0.1, 0, out=x[:1].expand(4, 32)),
    ]
    for i, call in enumerate(refused):
        with pytest.raises((ValueError, TypeError, seq.PerError)):
            call()
            pytest.fail(f"call {i} was not refused")
