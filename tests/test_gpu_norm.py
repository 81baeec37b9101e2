"""GPU: layer norm and RMS norm, forward and backward, through the C ABI, against the fp64 definition.

Tolerances, per element.  The result is rounded once to its type: eps(type) / 2 of the value (bf16 2^-8, fp32
2^-24).  Before that come fp32 operations.  A sum over a row is a chain of at most 32 additions in a thread (the
wide-row path: cols / 256) and at most 11 joins, so with the dozen roundings around it an error of K 2^-24, K =
64 + cols / 256, of the sum of magnitudes.  Forward: (x - mu) rstd w + b with mu within K 2^-24 of max |x| and
rstd within K 2^-24 of itself, so K 2^-24 (|w| rstd max |x| + |b|).  Backward: statistics are inputs; dx is a sum of
three terms, so K 2^-24 rstd (|u| + mean |u| + |xh| mean |u xh|).  Column sums: a chain of at most rows / 64 rows, 64
groups and 1,200 blocks whose sums are added, Kc = 1,280 + rows / 64, of the sum of magnitudes."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ops_oracle as oo
from paper_2602_01469_b200 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def rows_of(gen, rows, cols, pad, dtype, offset=0, std=1.0):
    """[rows, cols] view of a longer buffer: rows ``pad`` elements apart, the first ``offset`` elements in."""
    buf = torch.full((rows * (cols + pad) + offset,), float("nan"), dtype=dtype)
    v = buf[offset:].view(rows, cols + pad)[:, :cols] if rows else buf.view(0, cols + pad)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=gen) * std)
    out = torch.empty(buf.shape, dtype=dtype, device=DEV)
    out.copy_(buf)
    return out[offset:].view(rows, cols + pad)[:, :cols]


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def outside(got, want, bound):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.max((np.abs(got - want) / bound)[bad])))


def check_fwd(kind, x, w, b, eps, y, mean, rstd):
    want, wmean, wrstd = oo.norm_fwd(kind, f64(x), f64(w), f64(b), eps)
    K = 64 + x.shape[1] / 256
    top = np.abs(f64(x)).max(1, keepdims=True)
    wa = np.abs(f64(w)) if w is not None else np.ones(x.shape[1])
    ba = np.abs(f64(b)) if b is not None else np.zeros(x.shape[1])
    outside(f64(y), want, HALF[y.dtype] * np.abs(want) + K * U32 * (wa * wrstd[:, None] * top + ba))
    if rstd is not None:
        outside(f64(rstd), wrstd, K * U32 * wrstd)
    if mean is not None and kind == "layer":
        outside(f64(mean), wmean, K * U32 * top[:, 0])


def check_bwd(kind, x, w, mean, rstd, dy, dx, dw, dw0, db, db0):
    x64, dy64, m64, r64 = f64(x), f64(dy), f64(mean), f64(rstd)
    want, wdw, wdb = oo.norm_bwd(kind, x64, f64(w), m64, r64, dy64)
    K, Kc = 64 + x.shape[1] / 256, 1280 + x.shape[0] / 64
    xh = (x64 - m64[:, None] if kind == "layer" else x64) * r64[:, None]
    u = dy64 * f64(w) if w is not None else dy64
    au = np.abs(u)
    terms = r64[:, None] * (au + au.mean(1, keepdims=True) + np.abs(xh) * np.abs(u * xh).mean(1, keepdims=True))
    outside(f64(dx), want, HALF[dx.dtype] * np.abs(want) + K * U32 * terms)
    for got, first, add, mags in ((dw, dw0, wdw, np.abs(dy64 * xh).sum(0)), (db, db0, wdb, np.abs(dy64).sum(0))):
        if got is not None:
            outside(f64(got), f64(first) + add, Kc * U32 * (mags + np.abs(f64(first))))


CASES = [  # rows, cols, pad, offset, x dtype, w dtype, weight, bias
    (1, 1, 0, 0, BF16, BF16, True, True),
    (1, 2880, 0, 0, BF16, BF16, True, False),
    (3, 64, 0, 0, BF16, F32, True, True),
    (1025, 64, 0, 0, BF16, BF16, True, True),
    (700, 128, 0, 0, BF16, BF16, True, False),
    (130, 96, 8, 0, BF16, BF16, True, True),
    (333, 200, 0, 0, F32, F32, True, True),
    (67, 520, 0, 8, BF16, BF16, False, False),
    (301, 1001, 6, 0, F32, F32, True, True),
    (77, 1001, 0, 1, BF16, F32, True, True),
    (50, 2880, 8, 0, F32, BF16, True, False),
    (517, 2880, 0, 0, BF16, BF16, True, True),
    (40, 5120, 0, 3, BF16, BF16, True, True),
    (33, 4096, 0, 0, F32, F32, False, True),
    (9, 8192, 0, 0, BF16, BF16, True, True),
    (7, 16384, 0, 0, BF16, BF16, True, True),
    (5, 16384, 0, 0, F32, F32, True, True),
    (6, 20001, 5, 0, BF16, BF16, True, True),
    (4, 40000, 0, 0, F32, F32, True, True),
]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,cols,pad,offset,dtype,wdtype,weight,bias", CASES)
def test_forward_and_backward_match_the_definition(ctx, kind, rows, cols, pad, offset, dtype, wdtype, weight, bias):
    gen = torch.Generator().manual_seed(rows * 131 + cols)
    x = rows_of(gen, rows, cols, pad, dtype, offset, 2.0)
    w = (1 + 0.3 * torch.randn(cols, generator=gen)).to(wdtype).to(DEV) if weight else None
    b = torch.randn(cols, generator=gen).to(wdtype).to(DEV) if bias else None
    dy, y, dx = (rows_of(gen, rows, cols, pad, dtype, offset) for _ in range(3))
    beside = y._base.clone()
    mean, rstd = torch.full((rows,), float("nan"), device=DEV), torch.full((rows,), float("nan"), device=DEV)
    binding.peagle_norm_fwd(ctx, binding.NORM[kind], x, w, b, 1e-5, y, mean, rstd)
    torch.cuda.synchronize()
    check_fwd(kind, x, w, b, 1e-5, y, mean, rstd)
    # what lies between the rows is as it was
    gap = torch.ones(rows * (cols + pad) + offset, dtype=torch.bool, device=DEV)
    gap[offset:].view(rows, cols + pad)[:, :cols] = False
    assert torch.equal(y._base[gap].view(torch.int16), beside[gap].view(torch.int16))
    if kind == "rms":
        assert torch.isnan(mean).all()
        mean = None
    dw, db = torch.randn(cols, generator=gen).to(DEV), torch.randn(cols, generator=gen).to(DEV)
    dw0, db0 = dw.clone(), db.clone()
    binding.peagle_norm_bwd(ctx, binding.NORM[kind], x, w, mean, rstd, dy, dx, dw, db)
    torch.cuda.synchronize()
    check_bwd(kind, x, w, mean, rstd, dy, dx, dw, dw0, db, db0)
    assert binding.peagle_poll_status(ctx) == 0


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_many_rows(ctx, kind):
    """More rows than blocks have places, and an odd number of them."""
    gen = torch.Generator().manual_seed(8)
    x, dy = rows_of(gen, 20011, 72, 0, BF16, 0, 3.0), rows_of(gen, 20011, 72, 0, BF16)
    w = torch.randn(72, generator=gen).to(BF16).to(DEV)
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(20011, device=DEV), torch.empty(20011, device=DEV)
    binding.peagle_norm_fwd(ctx, binding.NORM[kind], x, w, None, 1e-6, y, mean, rstd)
    check_fwd(kind, x, w, None, 1e-6, y, mean, rstd)
    m = mean if kind == "layer" else None
    dw, zero = torch.zeros(72, device=DEV), torch.zeros(72, device=DEV)
    binding.peagle_norm_bwd(ctx, binding.NORM[kind], x, w, m, rstd, dy, dx, dw, None)
    check_bwd(kind, x, w, m, rstd, dy, dx, dw, zero, None, None)
    again, dx2 = torch.zeros(72, device=DEV), torch.empty_like(x)
    binding.peagle_norm_bwd(ctx, binding.NORM[kind], x, w, m, rstd, dy, dx2, again, None)
    assert torch.equal(again, dw) and torch.equal(dx2, dx)      # bit for bit


@pytest.mark.parametrize("cols", [64, 1001, 2880, 18000])
def test_in_place_and_without_optional_outputs(ctx, cols):
    gen = torch.Generator().manual_seed(cols)
    x, dy = rows_of(gen, 37, cols, 0, BF16), rows_of(gen, 37, cols, 0, BF16)
    w = torch.randn(cols, generator=gen).to(DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(37, device=DEV), torch.empty(37, device=DEV)
    binding.peagle_norm_fwd(ctx, 0, x, w, None, 1e-5, y, mean, rstd)
    z = x.clone()
    binding.peagle_norm_fwd(ctx, 0, z, w, None, 1e-5, z)
    assert torch.equal(z, y)
    dx, dw = torch.empty_like(x), torch.zeros(cols, device=DEV)
    binding.peagle_norm_bwd(ctx, 0, x, w, mean, rstd, dy, dx, dw, None)
    for overwritten in ("dy", "x"):
        a, b, dw2 = x.clone(), dy.clone(), torch.zeros(cols, device=DEV)
        out = b if overwritten == "dy" else a
        binding.peagle_norm_bwd(ctx, 0, a, w, mean, rstd, b, out, dw2, None)
        assert torch.equal(out, dx) and torch.equal(dw2, dw)
    only = torch.empty_like(x)
    binding.peagle_norm_bwd(ctx, 0, x, w, mean, rstd, dy, only)
    assert torch.equal(only, dx)


def test_a_mean_far_from_zero_and_a_constant_row(ctx):
    """fp32 rows around 1,000 with a spread of 1: the sum of squares alone would leave no digits."""
    gen = torch.Generator().manual_seed(5)
    x = (1000.0 + torch.randn(6, 2880, generator=gen)).to(DEV)
    x[2] = 7.0
    x[3] = 0.0
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device=DEV), torch.empty(6, device=DEV)
    binding.peagle_norm_fwd(ctx, 0, x, None, None, 1e-5, y, mean, rstd)
    check_fwd("layer", x, None, None, 1e-5, y, mean, rstd)
    assert float(y[3].abs().max()) == 0.0


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [72, 1001, 2880, 18000])
def test_rows_of_very_large_and_very_small_numbers(ctx, kind, dtype, cols):
    """The cube of rstd is no fp32 number for rows of 1e13 and larger, nor for rows of zeros with a tiny eps."""
    gen = torch.Generator().manual_seed(cols)
    w = (1 + 0.3 * torch.randn(cols, generator=gen)).to(dtype).to(DEV)
    size = torch.tensor([1e-14, 0.0, 1e-6, 1.0, 1e8, 1e12, 1e13, 3e13, 1e14, 1e15, 1e16, 1e17])
    x = (torch.randn(len(size), cols, generator=gen) * size[:, None]).to(dtype).to(DEV)
    dy = torch.randn(len(size), cols, generator=gen).to(dtype).to(DEV)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(len(size), device=DEV), torch.empty(len(size), device=DEV)
    binding.peagle_norm_fwd(ctx, binding.NORM[kind], x, w, None, 1e-30, y, mean, rstd)
    check_fwd(kind, x, w, None, float(np.float32(1e-30)), y, mean, rstd)
    m = mean if kind == "layer" else None
    dw, db, zero = torch.zeros(cols, device=DEV), torch.zeros(cols, device=DEV), torch.zeros(cols, device=DEV)
    binding.peagle_norm_bwd(ctx, binding.NORM[kind], x, w, m, rstd, dy, dx, dw, db)
    check_bwd(kind, x, w, m, rstd, dy, dx, dw, zero, db, zero)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [1001, 2880, 5120, 18000])
def test_the_mean_of_centred_and_shifted_rows(ctx, dtype, cols):
    """Rows around 0, spread s: an addition is off by U / sqrt(3) of its result in the mean square.  A thread's chains, in
    two halves, add up to 16 elements or cols / 256, a warp joins 32 and a block its warps: with partial sums that grow
    like the root of their number, an error of the mean of U s sqrt((11 / cols + 1 / 512) / 3), of which three times are
    allowed over 512 rows.  Around 1 and 1,000 the sum of the differences corrects the mean: its own rounding, U |mean|,
    and those of the differences, at most U of each, 4 U s with what their sum loses."""
    gen = torch.Generator().manual_seed(cols + 1)
    rows, s = 512, 2.2
    for middle in (0.0, 1.0, 1000.0):
        x = (middle + s * torch.randn(rows, cols, generator=gen)).to(dtype).to(DEV)
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        binding.peagle_norm_fwd(ctx, 0, x, None, None, 1e-5, y, mean, rstd)
        check_fwd("layer", x, None, None, 1e-5, y, mean, rstd)
        off = f64(mean) - f64(x).mean(1)
        if middle == 0.0:
            assert np.sqrt((off ** 2).mean()) <= 3 * U32 * s * np.sqrt((11 / cols + 1 / 512) / 3)
        else:
            assert np.abs(off).max() <= U32 * (1.01 * middle + 4 * s)


def test_nan_and_infinity_stay_in_their_rows(ctx):
    gen = torch.Generator().manual_seed(6)
    for cols in (128, 2880, 1001):
        x = torch.randn(9, cols, generator=gen).to(BF16).to(DEV)
        clean = torch.empty_like(x)
        binding.peagle_norm_fwd(ctx, 1, x, None, None, 1e-5, clean)
        x[4, 17], x[7, 3] = float("nan"), float("inf")
        y = torch.empty_like(x)
        binding.peagle_norm_fwd(ctx, 1, x, None, None, 1e-5, y)
        keep = [0, 1, 2, 3, 5, 6, 8]
        assert torch.equal(y[keep], clean[keep])
        assert torch.isnan(y[4]).all() and torch.isnan(y[7, 3])


def test_rows_past_two_to_the_31_elements(ctx):
    rows, ld = 70000, 32768
    buf = torch.empty(rows * ld, dtype=BF16, device=DEV)
    x = buf.view(rows, ld)[:, :64]
    x.copy_(torch.randn(rows, 64, device=DEV))
    first = x.clone()
    binding.peagle_norm_fwd(ctx, 1, x, None, None, 1e-5, x)
    torch.cuda.synchronize()
    at = [0, 1, 65535, 65536, 69999]
    check_fwd("rms", first[at], None, None, 1e-5, x[at], None, None)
    del buf, x


def test_another_stream_and_a_captured_graph(ctx):
    """A first call inside a capture, a larger call afterwards that outgrows the scratch, then replays."""
    gen = torch.Generator().manual_seed(7)
    own = binding.Context(0)
    try:
        x, dy = rows_of(gen, 300, 2880, 0, BF16), rows_of(gen, 300, 2880, 0, BF16)
        w = torch.randn(2880, generator=gen).to(BF16).to(DEV)
        rstd = torch.rand(300, generator=gen).to(DEV)
        want, dw = torch.empty_like(x), torch.zeros(2880, device=DEV)
        binding.peagle_norm_bwd(ctx, 1, x, w, None, rstd, dy, want, dw, None)
        torch.cuda.synchronize()
        dx, dw2 = torch.empty_like(x), torch.zeros(2880, device=DEV)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            dw2.zero_()
            binding.peagle_norm_bwd(own, 1, x, w, None, rstd, dy, dx, dw2, None)
        side = torch.cuda.Stream()
        bx = torch.randn(4096, 8192, device=DEV).to(BF16)
        br, bw = torch.rand(4096, device=DEV), torch.zeros(8192, device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            binding.peagle_norm_bwd(own, 1, bx, None, None, br, bx, torch.empty_like(bx), bw, None)
        side.synchronize()
        for _ in range(2):
            dx.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(dx, want) and torch.equal(dw2, dw)
        del g
    finally:
        own.close()


def test_no_rows_changes_nothing(ctx):
    x = torch.empty(0, 64, dtype=BF16, device=DEV)
    e = torch.empty(0, device=DEV)
    dw = torch.ones(64, device=DEV)
    binding.peagle_norm_fwd(ctx, 0, x, None, None, 1e-5, x.clone(), e, e)
    binding.peagle_norm_bwd(ctx, 0, x, None, e, e, x.clone(), x.clone(), dw, None)
    torch.cuda.synchronize()
    assert torch.equal(dw, torch.ones_like(dw))


def test_binding_refuses(ctx):
    x = torch.zeros(4, 64, dtype=BF16, device=DEV)
    r = torch.ones(4, device=DEV)

    def refused(status, f, *args):
        with pytest.raises(binding.PeagleError) as e:
            f(*args)
        assert e.value.status == binding.STATUS[status]

    fwd, bwd = binding.peagle_norm_fwd, binding.peagle_norm_bwd
    refused("BAD_SHAPE", fwd, ctx, 0, x, None, None, 0.0, x)                         # eps
    refused("BAD_SHAPE", fwd, ctx, 0, x, None, None, float("nan"), x)
    refused("BAD_SHAPE", fwd, ctx, 2, x, None, None, 1e-5, x)                        # kind
    refused("BAD_SHAPE", fwd, ctx, 0, x.half(), None, None, 1e-5, x.half())          # type
    refused("BAD_SHAPE", fwd, ctx, 0, x, None, None, 1e-5, x.float())                # Y of another type
    refused("BAD_SHAPE", fwd, ctx, 0, x, None, None, 1e-5, x[:, :32])                # Y of another shape
    refused("BAD_SHAPE", fwd, ctx, 0, x, x[0, :32], None, 1e-5, x)                   # weight of another length
    refused("BAD_SHAPE", fwd, ctx, 0, x.t(), None, None, 1e-5, x.t())                # columns apart
    refused("BAD_SHAPE", fwd, ctx, 0, x[:1].expand(4, 64), None, None, 1e-5, x)      # rows on top of each other
    refused("BAD_SHAPE", fwd, ctx, 0, x.cpu(), None, None, 1e-5, x)                  # host memory
    refused("NULL", bwd, ctx, 0, x, None, None, r, x, x.clone())                     # layer norm without its mean
    refused("NULL", bwd, ctx, 1, x, None, None, None, x, x.clone())
    refused("BAD_SHAPE", bwd, ctx, 1, x, None, None, r.double(), x, x.clone())
