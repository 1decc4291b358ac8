"""Root-mean-square norm with its output in 8 bits, against its definition in 64
bits (quant_ref).

q and h are asked for exactly.  scale: a sum of D <= 65536 squares, no term of
which passes more than 64 + 16 additions of positive numbers, so at most
80 * 2^-24 relative if they are in fp32, half of it in r; the mean, the root,
the quotient and two products add 5: under 45 * 2^-24.  y has the same error and
a rounding to its type, half a step (finfo.eps / 2)."""
import pytest
import torch

import quant_ref as ref
from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
R = 45 * 2.0 ** -24


def _same(a, b):
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(torch.nan_to_num(a, nan=0.0), torch.nan_to_num(b, nan=0.0))


def _check(x, weight=None, residual=None, eps=1e-6, **kw):
    """Host tensors (x may be a strided view)."""
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    sum_, y, q, scale = bnn.bnn_rmsnorm(kw.pop("xd", dev(x)), dev(weight), kw.pop("rd", dev(residual)),
                                        eps, want_y=True, **kw)
    torch.cuda.synchronize()
    h, yr, qr, sr = ref.rmsnorm(x, weight, residual, eps)
    if residual is not None:
        _same(sum_.cpu().float(), h.float())
    else:
        assert sum_ is None or torch.equal(sum_.cpu(), x)
    assert q.stride(0) % 16 == 0 or q.shape[0] == 1 or "q" in kw
    assert torch.equal(q.cpu(), qr)
    nan = torch.isnan(sr)
    assert torch.equal(torch.isnan(scale.cpu()), nan)
    assert torch.equal(torch.isnan(y.cpu()).any(1), nan)
    torch.testing.assert_close(scale.cpu().double()[~nan], sr[~nan], rtol=R, atol=1e-44)
    half = torch.finfo(x.dtype).eps / 2
    tiny = torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps
    torch.testing.assert_close(y.cpu().double()[~nan], yr[~nan], rtol=R + half, atol=tiny)
    return y, q, scale


def _rows(g, M, D, kind, scale=1.0):
    return (scale * torch.randn(M, D, generator=g)).to(TYPES[kind])


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("M, D", [(1, 1), (3, 5), (7, 8), (5, 63), (4, 511), (9, 512), (2, 513), (1, 2048),
                                  (6, 2049), (3, 4096), (1100, 1100), (5, 4099), (2, 8192), (3, 8200),
                                  (2, 16384), (1, 16390), (2, 65536)])
def test_sizes(kind, M, D):
    g = torch.Generator().manual_seed(100 * D + M)
    _check(_rows(g, M, D, kind), _rows(g, 1, D, kind)[0], _rows(g, M, D, kind, 3.0))
    _check(_rows(g, M, D, kind), torch.randn(D, generator=g))
    _check(_rows(g, M, D, kind))


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 512, 1000, 1030, 1300, 1536, 4096])
def test_many_rows(kind, D):
    g = torch.Generator().manual_seed(D)
    _check(_rows(g, 4097, D, kind), _rows(g, 1, D, kind)[0], _rows(g, 4097, D, kind))


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_borders(kind):
    """Values that lie on a border between two 8-bit integers, and next to one:
    whole numbers over a largest one of 127 * 2, 127 * 3 and others."""
    g = torch.Generator().manual_seed(5)
    for most in (254, 127, 255, 1016, 2032):
        x = torch.randint(-most, most + 1, (64, 1030), generator=g).float()
        x[:, 7] = most
        x = x.to(TYPES[kind])
        x = torch.where(x.abs() > x[:1, 7:8].abs(), x[:1, 7:8], x)
        _check(x)
        _check(x, torch.full((1030,), 0.5).to(TYPES[kind]))
        _check(x * 2.0 ** -20 if kind != "fp16" else x * 2.0 ** -10)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_far_ends_of_the_range(kind):
    """Squares and products that leave fp32's range, rows of subnormals."""
    g = torch.Generator().manual_seed(6)
    x = torch.randn(12, 700, generator=g)
    for i, s in enumerate((1e-44, 1e-40, 1e-38, 1e-30, 1e-20, 1e-10, 1.0, 1e10, 1e18, 1e25, 1e36, 5e37)):
        x[i] *= s
    w = torch.randn(700, generator=g)
    for ws in (1.0, 1e-30, 1e30):
        for eps in (0.0, 1e-6):
            xk, wk = x.to(TYPES[kind]), (w * ws).to(TYPES[kind])
            q, scale = bnn.bnn_rmsnorm(xk.cuda(), wk.cuda(), eps=eps)[2:]
            _, _, qr, sr = ref.rmsnorm(xk, wk, None, eps)
            assert torch.equal(q.cpu(), qr)
            inside = (sr > 1e-37) & (sr < 3e38)
            torch.testing.assert_close(scale.cpu().double()[inside], sr[inside], rtol=R, atol=0)


@pytest.mark.parametrize("D", [40, 4096, 9000])
def test_zero_rows_and_bad_rows(D):
    g = torch.Generator().manual_seed(7)
    for eps in (0.0, 1e-5):
        for kind in TYPES:
            x = _rows(g, 9, D, kind)
            x[1] = 0
            x[3, D - 1] = float("nan")
            x[4, 0] = float("inf")
            x[5, D // 2] = -float("inf")
            x[6] = 0
            x[6, 3] = torch.finfo(TYPES[kind]).tiny
            _check(x, torch.randn(D, generator=g), eps=eps)
    x = torch.full((2, D), 60000.0, dtype=torch.float16)  # the sum leaves fp16's range
    _check(x, None, x.clone())


def test_strides_and_alignment():
    """Rows that start anywhere, and bytes between rows of q left as they are."""
    g = torch.Generator().manual_seed(8)
    for kind in TYPES:
        for D, first, stride in ((1029, 1, 1031), (64, 3, 70), (4096, 1, 4099), (7, 5, 13)):
            flat = _rows(g, 1, first + 11 * stride, kind)[0]
            flat2 = _rows(g, 1, first + 11 * stride, kind)[0]
            x = flat[first:].as_strided((11, D), (stride, 1))
            r = flat2[first:].as_strided((11, D), (stride, 1))
            xd = flat.cuda()[first:].as_strided((11, D), (stride, 1))
            rd = flat2.cuda()[first:].as_strided((11, D), (stride, 1))
            store = torch.full((2 + 11 * (D + 3),), 77, dtype=torch.int8, device="cuda")
            q = store[1:1 + 11 * (D + 3)].reshape(11, D + 3)[:, :D]
            _check(x, _rows(g, 1, D, kind)[0], r, xd=xd, rd=rd, q=q)
            left = store[1:1 + 11 * (D + 3)].reshape(11, D + 3)[:, D:]
            assert (left == 77).all() and store[0] == 77 and store[-1] == 77


@pytest.mark.parametrize("D", [96, 4096, 16384])
def test_in_place(D):
    g = torch.Generator().manual_seed(9)
    x, r, w = _rows(g, 70, D, "bf16"), _rows(g, 70, D, "bf16"), torch.randn(D, generator=g)
    h, y, q, scale = ref.rmsnorm(x, w, r)
    xd, rd = x.cuda(), r.cuda()
    out = bnn.bnn_rmsnorm(xd, w.cuda(), rd, sum=rd, y=xd)
    assert out[0] is rd and out[1] is xd
    assert torch.equal(rd.cpu(), h) and torch.equal(out[2].cpu(), q)
    torch.testing.assert_close(xd.cpu().double(), y, rtol=R + 2.0 ** -8, atol=1e-40)
    xd = x.cuda()
    assert bnn.bnn_rmsnorm(xd, w.cuda(), r.cuda(), sum=xd, want_q=False)[2:] == (None, None)
    assert torch.equal(xd.cpu(), h)


def test_single_outputs():
    g = torch.Generator().manual_seed(10)
    x, w = _rows(g, 33, 777, "fp16"), torch.randn(777, generator=g)
    full = bnn.bnn_rmsnorm(x.cuda(), w.cuda(), want_y=True)
    only_y = bnn.bnn_rmsnorm(x.cuda(), w.cuda(), want_y=True, want_q=False)
    only_q = bnn.bnn_rmsnorm(x.cuda(), w.cuda())
    assert torch.equal(full[1], only_y[1]) and only_y[2] is None
    assert torch.equal(full[2], only_q[2]) and torch.equal(full[3], only_q[3]) and only_q[1] is None
    empty = bnn.bnn_rmsnorm(x.cuda()[:0], w.cuda(), want_y=True)
    assert empty[1].shape == (0, 777) and empty[2].shape == (0, 777) and empty[3].shape == (0,)


@pytest.mark.parametrize("D", [1, 520])
def test_more_rows_than_a_launch_has(D):
    """Rows past 2^21 workgroups (of four rows each, and of one)."""
    M = (1 << 23) + 5 if D == 1 else (1 << 21) + 5
    x = torch.ones(M, D, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(15)
    ends = torch.cat([torch.arange(4), torch.arange(M - 9, M)])
    rows = _rows(g, len(ends), D, "bf16")
    x[ends.cuda()] = rows.cuda()
    w = _rows(g, 1, D, "bf16")[0]
    h, y, q, scale = bnn.bnn_rmsnorm(x, w.cuda(), x, want_y=True, sum=torch.empty_like(x))
    hr, yr, qr, sr = ref.rmsnorm(rows, w, rows)
    at = ends.cuda()
    assert torch.equal(h[at].cpu(), hr) and torch.equal(q[at].cpu(), qr)
    torch.testing.assert_close(scale[at].cpu().double(), sr, rtol=R, atol=0)
    torch.testing.assert_close(y[at].cpu().double(), yr, rtol=R + 2.0 ** -8, atol=0)
    assert (h[4:M - 9] == 2).all()
