"""The linear layer with softmax cross entropy where its logits run in the large tiles (more than 64 rows and at least 128
tiles of 128 x 128), in pieces of few rows and past 4 GiB, and the accuracy that the header promises beyond the storage
type's.  The definitions and tolerances are those of test_gpu_linear_ce.py; where a test has a closer one, its head
derives it."""
import numpy as np
import pytest
import torch

from test_gpu_linear_ce import HALF, IGNORE, TINY, U, Case, _B, _close

pytestmark = pytest.mark.gpu

# 64 x 128 tiles in float32, 128 x 128 and 256 x 256 in bf16
TILES = [(torch.float32, 300, 72, 6001), (torch.bfloat16, 300, 72, 6001), (torch.bfloat16, 3100, 72, 4001)]


def _run(k, dloss=None, **kw):
    k.forward()
    k.check_forward()
    k.backward(dloss=dloss, **kw)
    k.check_backward(dloss)


@pytest.mark.parametrize("dtype,m,c,v", TILES)
@pytest.mark.parametrize("smoothing,z", [(0.1, 0.0), (0.0, 1e-3), (0.1, 1e-2)])
def test_smoothing_and_z_loss(dtype, m, c, v, smoothing, z):
    _run(Case(m, c, v, dtype, bias=True, smoothing=smoothing, z=z, ignored=0.2, pad=8), pad=8)


@pytest.mark.parametrize("dtype,m,c,v", TILES)
@pytest.mark.parametrize("dw_dtype", [torch.float32, torch.bfloat16])
def test_row_gradients_and_weight_gradient_types(dtype, m, c, v, dw_dtype):
    _run(Case(m, c, v, dtype, ignored=0.2), torch.randn(1 + m, device="cuda"), dw_dtype=dw_dtype)


@pytest.mark.parametrize("dtype,m,v", [(torch.bfloat16, 2100, 140001), (torch.float32, 1100, 130001)])
@pytest.mark.parametrize("want", [("dh",), ("dw", "dbias"), ("dbias",)])
def test_row_gradients_over_pieces(dtype, m, v, want):
    other = torch.float32 if dtype == torch.bfloat16 else torch.bfloat16
    _run(Case(m, 8, v, dtype, bias=True, smoothing=0.05, z=1e-3, ignored=0.2), torch.randn(1 + m, device="cuda"),
         dw_dtype=other, want=want)


@pytest.mark.parametrize("dtype,m,c,v", TILES)
@pytest.mark.parametrize("want", [("dh",), ("dw",), ("dbias",), ("dh", "dbias"), ("dh", "dw")])
def test_some_gradients(dtype, m, c, v, want):
    k = Case(m, c, v, dtype, bias=True)
    _run(k, want=want)
    assert "dbias" in want or bool((k.dbias == 777.0).all())


@pytest.mark.parametrize("dtype,m,c,v", TILES)
def test_labels_outside(dtype, m, c, v):
    for bad in (-1, v, (v // 128 + 1) * 128, 1 << 30, -(1 << 31)):
        k = Case(m, c, v, dtype)
        k.labels[7] = bad
        k.forward()
        k.backward()
        assert bool(torch.isnan(k.loss[8])) and bool(torch.isnan(k.loss[0])) and bool(torch.isnan(k.dh[7]).all())
        assert not bool(torch.isnan(torch.cat((k.loss[1:8], k.loss[9:]))).any())
        assert not bool(torch.isnan(torch.cat((k.dh[:7], k.dh[8:]))).any())
        assert bool(torch.isnan(k.dw).all()) and bool(torch.isnan(k.dbias).all())
        assert bool(torch.isfinite(k.ce.lse).all())


@pytest.mark.parametrize("dtype,m,c,v", TILES)
def test_classes_taken_out(dtype, m, c, v):
    k = Case(m, c, v, dtype, bias=True)
    out = torch.zeros(v, dtype=torch.bool, device="cuda")
    out[256:1024] = True                                  # whole tiles
    out[::7] = True
    keep = torch.nonzero(~out)[:, 0]
    k.labels.copy_(keep[k.labels.long() % len(keep)].int())
    k.bias[out] = float("-inf")
    _run(k)
    assert bool((k.dbias[out] == 0).all()) and bool((k.dw[out] == 0).all())


@pytest.mark.parametrize("dtype,m,c,v", TILES)
def test_infinities_stay_in_their_row(dtype, m, c, v):
    k, want = Case(m, c, v, dtype, ignored=0.3), Case(m, c, v, dtype, ignored=0.3)
    want.forward()
    pad, row = k.labels == IGNORE, int(torch.nonzero(k.labels != IGNORE)[20, 0])
    for value in (float("nan"), float("inf"), float("-inf")):
        k.h[pad] = value                                  # padding reaches nothing
        k.forward()
        assert torch.equal(k.loss, want.loss) and torch.equal(k.ce.lse, want.ce.lse)
    k.backward()
    want.backward()
    assert torch.equal(k.dh, want.dh) and torch.equal(k.dw, want.dw) and torch.equal(k.dbias, want.dbias)
    others = torch.arange(m, device="cuda") != row
    for value in (float("nan"), float("inf"), float("-inf")):
        k.h[row] = value
        k.forward()
        assert bool(torch.isnan(k.loss[1 + row])) and bool(torch.isnan(k.loss[0]))
        assert torch.equal(k.loss[1:][others], want.loss[1:][others])


@pytest.mark.parametrize("dtype,m,c,v", TILES)
def test_no_row_counts(dtype, m, c, v):
    k = Case(m, c, v, dtype, bias=True)
    k.labels.fill_(IGNORE)
    k.h[m // 2] = float("nan")
    k.forward()
    k.backward()
    for t in (k.loss, k.ce.lse, k.dh, k.dw, k.dbias):
        assert bool((t == 0).all())


@pytest.mark.parametrize("dtype,m,c,v", TILES)
def test_same_bits_streams_and_graph(dtype, m, c, v):
    B = _B()
    ks = [Case(m, c, v, dtype, seed=s, bias=True, ignored=0.2) for s in (1, 2)]
    results = lambda k: (k.loss, k.ce.lse, k.dh, k.dw, k.dbias)  # noqa: E731

    def both(k):
        B.bnr_linear_ce_fwd(k.h, k.w, k.ce, k.loss)
        B.bnr_linear_ce_bwd(k.h, k.w, k.ce, k.dh, k.dw, k.dbias)

    for k in ks:
        k.forward()
        k.backward()
        k.first = [t.clone() for t in results(k)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ks]
    for _ in range(3):
        for k, s in zip(ks, streams):
            with torch.cuda.stream(s):
                both(k)
    torch.cuda.synchronize()
    for k in ks:
        assert all(torch.equal(a, b) for a, b in zip(results(k), k.first))
    graphs = []
    for k in ks:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both(k)
        graphs.append(g)
    for turn in range(3):
        for k in ks:
            k.labels.copy_(torch.where(torch.rand(m, device="cuda") < 0.3 * turn, torch.full_like(k.labels, IGNORE),
                                       torch.randint_like(k.labels, 0, v)))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for k in ks:
            got = [t.clone() for t in results(k)]
            both(k)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(results(k), got))


@pytest.mark.parametrize("dtype,m", [(torch.bfloat16, 1), (torch.bfloat16, 20), (torch.bfloat16, 50), (torch.float32, 20)])
def test_pieces_of_few_rows(dtype, m):
    """Classes past 2^20 in two pieces; labels about their border and at the ends."""
    v = (1 << 20) + 300
    border = (v // 2 + 255) // 256 * 256
    k = Case(m, 8, v, dtype, bias=True, smoothing=0.05, ignored=0.2 if m > 1 else 0.0)
    at = torch.tensor([border, border - 1, 0, v - 1], dtype=torch.int32, device="cuda")[:m]
    k.labels[:len(at)] = at
    _run(k, torch.randn(1 + m, device="cuda"))


def test_offsets_past_32_bits():
    """Rows of h, dh, w and dw past 4 GiB in the large tiles."""
    m, c, v = 4200, 64, 5000
    k = Case(m, c, v, torch.bfloat16, bias=True, ignored=0.1)
    rows = torch.empty(m, 1 << 20, dtype=torch.bfloat16, device="cuda")
    h, dh = rows[:, -c:], rows[:, -3 * c:-2 * c]
    w, dw = (torch.empty(v, 1 << 19, dtype=torch.bfloat16, device="cuda")[:, -c:] for _ in range(2))
    h.copy_(k.h)
    w.copy_(k.w)
    k.h, k.w = h, w
    k.forward()
    k.check_forward()
    k.backward()
    want = (k.dh, k.dw, k.dbias.clone())
    k.check_backward()
    _B().bnr_linear_ce_bwd(k.h, k.w, k.ce, dh, dw, k.dbias)
    assert all(torch.equal(a, b) for a, b in zip((dh, dw, k.dbias), want))
    del rows, h, dh, w, dw, k
    torch.cuda.empty_cache()


# ---- promised accuracy ---------------------------------------------------------
def _gradient(k):
    """g in float64 and how far float32 leaves it off before it is rounded as an operand (Case.check_backward)."""
    n = int(k.counts.sum())
    p = torch.exp(k.l - k.lse[:, None])
    hot = torch.zeros_like(p).scatter_(1, k.at, 1.0)
    r = (k.counts / n)[:, None]
    rel = k.dl + (k.t + U * k.lse.abs())[:, None] + 16 * U
    return r * (p - hot), r * p * torch.expm1(rel) + 8 * U * r * (p + hot), n


@pytest.mark.parametrize("m,c,v", [(1, 64, 500), (16, 264, 3001), (17, 64, 900), (40, 136, 5000), (64, 64, 3000)])
def test_few_bf16_rows_keep_what_rounding_left(m, c, v):
    """Up to 64 bf16 rows g is two bf16 numbers: what the second one's rounding leaves is at most 2^-8 of 2^-8 of g."""
    k = Case(m, c, v, torch.bfloat16, bias=True, ignored=0.2 if m > 1 else 0.0)
    k.forward()
    k.check_forward()
    k.backward(dw_dtype=torch.float32)
    g, dg, _ = _gradient(k)
    operand = dg + 2.0 ** -16 * (g.abs() + dg) + TINY
    ga = g.abs() + operand
    h, w = k.h64, k.w64
    tol = (operand + (m + 66) * U * ga).t() @ h.abs()
    _close("dw", k.dw, g.t() @ h, tol + U * ((g.t() @ h).abs() + tol))
    tol = (operand + (2 * v + 66) * U * ga) @ w.abs()
    _close("dh", k.dh, g @ w, tol + HALF[torch.bfloat16] * ((g @ w).abs() + tol))


@pytest.mark.parametrize("m,c,v", [(300, 72, 6001), (300, 64, 700), (3100, 72, 4001)])
def test_the_means_significand_stays_outside_g(m, c, v):
    """g / f is what is rounded, f the significand of 1 / n: an entry x off by dx rounds to within |round(x) - x| + 2 dx of
    x.  Rounding g itself would leave 1 / 300 off by 2e-3, where most labels' x is next to -1."""
    k = Case(m, c, v, torch.bfloat16, std=0.5)
    k.forward()
    k.check_forward()
    k.backward(dw_dtype=torch.float32)
    g, dg, n = _gradient(k)
    f = float(np.frexp(np.float32(1.0) / np.float32(n))[0]) * 2.0
    operand = ((g / f).float().bfloat16().double() * f - g).abs() + 2 * dg + 4 * U * g.abs() + TINY
    ga = g.abs() + operand
    tol = (operand + (m + 66) * U * ga).t() @ k.h64.abs()
    ref = g.t() @ k.h64
    _close("dw", k.dw, ref, tol + U * (ref.abs() + tol))


@pytest.mark.parametrize("m,v", [(20, 300), (300, 6001)])
def test_float32_sums_in_two_levels(m, v):
    """4096 equal terms of 1 + 0.4 2^-13: one chain of additions loses 0.4 2^-13 in each from 1024 on, 600 steps of 2^-24 of
    the sum in all; 64 terms at a time and then those are at most 64 + 64 additions from a term to the sum."""
    c = 4096
    x = float(np.float32(1 + 0.4 * 2.0 ** -13))
    h, w = torch.ones(m, c, device="cuda"), torch.full((v, c), x, device="cuda")
    ce, loss = _B().CE(torch.zeros(m, dtype=torch.int32, device="cuda")), torch.empty(1 + m, device="cuda")
    _B().bnr_linear_ce_fwd(h, w, ce, loss)
    ref = torch.full((m,), c * x + np.log(v), dtype=torch.float64, device="cuda")
    _close("lse", ce.lse[1:], ref, (64 + 64 + 8) * U * c * x + 100 * U + U * ref)


@pytest.mark.parametrize("m,c,v", [(4096, 64, 40), (4096, 64, 6001)])
def test_float32_weight_gradient_in_two_levels(m, c, v):
    """The same rows 4096 times, none of them of label 1 and up: dw[v] is the sum of 4096 equal terms."""
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.rand(1, c, generator=g, device="cuda").add_(1.0).expand(m, c).contiguous()
    w = torch.randn(v, c, generator=g, device="cuda") * 0.05
    ce, loss = _B().CE(torch.zeros(m, dtype=torch.int32, device="cuda")), torch.empty(1 + m, device="cuda")
    dw = torch.empty_like(w)
    _B().bnr_linear_ce_fwd(h, w, ce, loss)
    _B().bnr_linear_ce_bwd(h, w, ce, dw=dw)
    l = h[:1].double() @ w.double().t()
    ref = (torch.softmax(l, 1).t() @ h[:1].double())[1:]
    # the probability's own error (of l and the stored lse), a product's and the additions' roundings
    dl = (c + 8) * U * (h[:1].double().abs() @ w.double().abs().t())
    rel = torch.expm1(dl + dl.amax() + 100 * U + U * torch.logsumexp(l, 1).abs() + 24 * U)
    _close("dw", dw[1:], ref, ref.abs() * (rel.t()[1:] + (64 + 64 + 64 + 4) * U))


@pytest.mark.parametrize("dtype,m,c,v", TILES + [(torch.float32, 60, 64, 700), (torch.bfloat16, 60, 64, 700)])
def test_classes_taken_out_keep_their_share_of_smoothing(dtype, m, c, v):
    k = Case(m, c, v, dtype, bias=True, smoothing=0.1)
    out = torch.zeros(v, dtype=torch.bool, device="cuda")
    out[100:300] = True
    keep = torch.nonzero(~out)[:, 0]
    k.labels.copy_(keep[k.labels.long() % len(keep)].int())
    k.bias[out] = float("-inf")
    k.forward()
    k.reference()
    assert bool((k.loss == float("inf")).all())
    _close("lse", k.ce.lse[1:], k.lse, k.t + U * k.lse.abs())
    k.backward()
    k.check_backward()
    share = -k.s / v                                      # the rows' r add up to 1
    assert bool(((k.dbias[out].double() - share).abs() <= (m + 70) * U * -share).all())
