"""Dropout (bnr_dropout_fwd / bnr_dropout_bwd) against its definition in float64 (oracle/dropout.py).

Tolerances: the scale is rounded to float32, its product with x and the sum once more (one operation), and the result
to the storage type: 2^-24 |x| scale + 2^-24 |y|, and half a step of the storage type of y where that is shorter.
What is dropped is exactly the added value."""
import numpy as np
import pytest
import torch

from oracle import dropout as D

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
MARK = 777.0


def _B():
    from paper_1807_01702_amd import bnr
    return bnr


def _view(t, dtype, pad=0, shift=0):
    """t [m, c] on the GPU as rows of a wider buffer (stride c + pad), its first element `shift` past a 16-byte
    boundary; the rest of the buffer holds a marker."""
    m, c = t.shape
    buf = torch.full((m * (c + pad) + shift + 8,), MARK, dtype=dtype, device="cuda")
    v = buf[shift:shift + m * (c + pad)].view(m, c + pad)[:, :c]
    v.copy_(t.to(dtype))
    return buf, v


def _untouched(buf, v, pad, shift):
    m, c = v.shape
    rest = buf.clone()
    rest[shift:shift + m * (c + pad)].view(m, c + pad)[:, :c] = MARK
    assert bool((rest == MARK).all()), "wrote outside the view"


def _np(t):
    return t.detach().double().cpu().numpy()


def _check(got, x, drop, step, dtype, add=None):
    ref = D.dropout(x, drop.p, drop.seed, drop.site, step, add)
    scaled = D.dropout(np.abs(x), drop.p, drop.seed, drop.site, step)
    tol = U * scaled + (U + HALF[dtype]) * np.abs(ref) * (1 + U) + 1e-300
    off = np.abs(_np(got) - ref)
    assert not np.any(~(off <= tol)), "%d values off, worst %.3g" % ((~(off <= tol)).sum(), (off / tol).max())


# m, c: one element, blocks of eight and their ends, odd widths, many narrow rows, one long row
SIZES = [(1, 1), (1, 7), (1, 8), (3, 9), (5, 24), (77, 63), (64, 64), (1000, 3), (33, 1001), (130, 264), (7, 4096),
         (4099, 8), (1, 100003), (2, 16385)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,c", SIZES)
def test_forward_and_backward(m, c, dtype):
    B = _B()
    g = torch.Generator().manual_seed(m * 7919 + c)
    x, r = (torch.randn(m, c, generator=g, dtype=torch.float64) for _ in range(2))
    for pad, shift, p in ((0, 0, 0.1), (5, 1, 0.5), (8, 0, 0.9)):
        bx, vx = _view(x, dtype, pad, shift)
        br, vr = _view(r, dtype, 0, shift)
        by, vy = _view(torch.zeros(m, c), dtype, pad, 3 * shift)
        drop = B.Dropout(p, 0x9E3779B97F4A7C15 ^ c, site=m, step=5)
        B.bnr_dropout_fwd(vx, drop, vy)
        _check(vy, _np(vx), drop, 5, dtype)
        _untouched(by, vy, pad, 3 * shift)
        B.bnr_dropout_fwd(vx, drop, vy, res=vr)
        _check(vy, _np(vx), drop, 5, dtype, _np(vr))
        B.bnr_dropout_bwd(vr, drop, vy)
        _check(vy, _np(vr), drop, 5, dtype)
        B.bnr_dropout_bwd(vr, drop, vy, dsum=vx)
        _check(vy, _np(vr), drop, 5, dtype, _np(vx))
        _untouched(by, vy, pad, 3 * shift)
        _untouched(bx, vx, pad, shift)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("p", [0.0, 1e-6, 2.0 ** -16, 1 - 2.0 ** -16, 1 - 1e-7, 1.0])
def test_ends_of_the_probability(p, dtype):
    B = _B()
    x = torch.randn(40, 100, device="cuda").to(dtype)
    y = torch.empty_like(x)
    drop = B.Dropout(p, 3)
    B.bnr_dropout_fwd(x, drop, y)
    _check(y, _np(x), drop, 0, dtype)
    if p == 0.0:
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_dropped_infinities_add_nothing(dtype):
    B = _B()
    m, c = 50, 40
    drop = B.Dropout(0.5, 11, site=1, step=2)
    gone = torch.from_numpy(D.bits(m, c, 11, 1, 2) < D.limit(0.5)).cuda()
    x, r = (torch.randn(m, c, device="cuda").to(dtype) for _ in range(2))
    bad = x.clone()
    bad[gone] = float("nan")
    bad[0][gone[0]] = float("inf")
    y, z = torch.empty_like(x), torch.empty_like(x)
    for add in (None, r):
        B.bnr_dropout_fwd(bad, drop, y, res=add)
        B.bnr_dropout_fwd(x, drop, z, res=add)
        assert torch.equal(y, z)
    B.bnr_dropout_fwd(x, drop, z, res=r)
    assert torch.equal(z[gone], r[gone])
    x[~gone] = float("inf")                               # what is kept stays what it is
    B.bnr_dropout_fwd(x, drop, y)
    assert bool(torch.isinf(y[~gone]).all()) and bool((y[gone] == 0).all())


def test_in_place_and_shared_inputs():
    B = _B()
    x, r = (torch.randn(301, 203, device="cuda").bfloat16() for _ in range(2))
    drop = B.Dropout(0.3, 5)
    want = torch.empty_like(x)
    B.bnr_dropout_fwd(x, drop, want, res=r)
    over_x, over_r = x.clone(), r.clone()
    B.bnr_dropout_fwd(over_x, drop, over_x, res=r)
    B.bnr_dropout_fwd(x, drop, over_r, res=over_r)
    assert torch.equal(over_x, want) and torch.equal(over_r, want)
    B.bnr_dropout_fwd(x, drop, want, res=x)               # one tensor as both
    y = x.clone()
    B.bnr_dropout_fwd(y, drop, y, res=y)
    assert torch.equal(y, want)


def test_gradient_is_the_formulas_and_the_differences():
    """sum(y dy) is linear in x: its difference quotient along any direction is the gradient's product with it."""
    B = _B()
    x, dy, d = (torch.randn(37, 51, device="cuda") for _ in range(3))
    drop = B.Dropout(0.25, 99, site=4, step=7)
    y0, y1, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    B.bnr_dropout_fwd(x, drop, y0)
    B.bnr_dropout_fwd(x + d, drop, y1)
    B.bnr_dropout_bwd(dy, drop, dx)
    terms = ((y1.double() - y0.double()) * dy.double())
    want = (dx.double() * d.double()).sum()
    # x + d, both y and dx are off by at most two roundings each of values up to |x| + |d|, scaled by 4 / 3
    tol = 8 * U * 4 / 3 * ((x.abs() + d.abs()).double() * dy.abs().double()).sum()
    assert abs(float(terms.sum() - want)) <= float(tol)


def test_step_on_the_device_and_captured():
    B = _B()
    x = torch.randn(100, 260, device="cuda")
    step = torch.tensor([41], dtype=torch.int32, device="cuda")
    drop = B.Dropout(0.2, 17, site=9, step=step)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.bnr_dropout_fwd(x, drop, y)
    torch.cuda.current_stream().wait_stream(side)
    _check(y, _np(x), drop, 41, torch.float32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.bnr_dropout_fwd(x, drop, y)
        B.bnr_dropout_bwd(x, drop, dx)
        step.add_(1)
    step.fill_(100)
    for k in range(4):                                    # every replay has its own mask
        graph.replay()
        other = torch.randn(1000, 1000, device="cuda").sum()
        torch.cuda.synchronize()
        _check(y, _np(x), drop, 100 + k, torch.float32)
        assert torch.equal(dx, y)
        x.add_(0.5 + 0 * other)
    step.fill_(-1)                                        # 2^32 - 1
    B.bnr_dropout_fwd(x, drop, y)
    _check(y, _np(x), drop, 0xFFFFFFFF, torch.float32)


def test_two_streams():
    B = _B()
    xs = [torch.randn(2000, 1024, device="cuda") for _ in range(2)]
    ys = [torch.empty_like(x) for x in xs]
    want = [torch.empty_like(x) for x in xs]
    drops = [B.Dropout(0.1, 1 + k) for k in range(2)]
    for x, w, d in zip(xs, want, drops):
        B.bnr_dropout_fwd(x, d, w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for x, y, d, s in zip(xs, ys, drops, streams):
            with torch.cuda.stream(s):
                B.bnr_dropout_fwd(x, d, y)
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for y, w in zip(ys, want))


def test_offsets_past_32_bits():
    """A row whose elements lie beyond 2^32 bytes, and 2^31 elements."""
    B = _B()
    c, ld = 24, 1 << 20
    m = (1 << 31) // ld + 3                               # float32: the last rows start past 8 GiB
    buf = torch.empty(m * ld, device="cuda")
    x = buf.view(m, ld)[:, :c]
    x.copy_(torch.randn(m, c, device="cuda"))
    y = buf.view(m, ld)[:, c:2 * c]
    drop = B.Dropout(0.4, 21)
    B.bnr_dropout_fwd(x, drop, y)
    _check(y, _np(x), drop, 0, torch.float32)


def test_more_threads_than_a_dimension_of_a_grid_holds():
    """2^31 - 5 rows of three blocks: past 2^32 threads (73 GB, in place), checked in windows of rows."""
    B = _B()
    m, c, p, seed, site, step = (1 << 31) - 5, 17, 0.3, 0x123456789ABCDEF, 6, 11
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 2 * m * c + (4 << 30):
        pytest.skip("74 GB of device memory are wanted")
    x = torch.empty(m, c, dtype=torch.bfloat16, device="cuda")
    n = 1000
    # the ends, the rows about the end of the grid's first dimension (2^29 threads), about 2^32 threads
    starts = [0, (1 << 29) // 3 - n // 2, (1 << 30) - 7, (1 << 32) // 3 - n // 2, m - n]
    before = []
    for s in starts:
        x[s:s + n] = torch.randn(n, c, device="cuda").bfloat16()
        before.append(_np(x[s:s + n]))
    B.bnr_dropout_fwd(x, B.Dropout(p, seed, site=site, step=step), x)
    for s, was in zip(starts, before):
        col, row = np.meshgrid(np.arange(3), s + np.arange(n))
        words = D.philox4x32((col, row, site, step), (seed & 0xFFFFFFFF, seed >> 32))
        words = np.stack([np.broadcast_to(w, col.shape) for w in words], 2).astype(np.int64)
        bits = np.stack((words & 0xFFFF, words >> 16), 3).reshape(n, 24)[:, :c]
        t = D.limit(p)
        ref = np.where(bits >= t, was * (65536 / (65536 - t)), 0.0)
        off, tol = np.abs(_np(x[s:s + n]) - ref), (2 * U + HALF[torch.bfloat16]) * np.abs(ref) * (1 + U)
        assert bool((off <= tol).all()), "rows from %d" % s
    del x
    torch.cuda.empty_cache()
