"""Orthogonalised updates (bnr_orthogonalize, bnr_muon_update) against their
definition in float64.

Tolerance of the iteration.  The library holds every operand of a product with 22
bits and accumulates in float32.  Rounding makes a step's operands off by at most
e = 2^-21 of their Frobenius norms (2^-22 per operand, and as much again for the
accumulation, which adds at most q / 32 blocks of 32 terms: sqrt(q / 32) 2^-24 <
2^-21 for q <= 2048), and a step passes three products: it adds an error of
(|a| + 2 |b| + 3 |c|) e of X's norm.  An error in a direction of X whose singular
value is still small grows as that value does, by a = 3.45 a step, until the value
saturates near 1, where p(s) = a s + b s^3 + c s^5 has a slope between -1.6 and 1.2.
Relative to the weak singular values, which make up the result's norm, a rounding
therefore counts once: five steps add up to 5 (3.45 + 2 4.78 + 3 2.04) e = 95 e =
4.6e-5.  (The weak part of the matrices below holds at least a third of their
squared norm; the factor sqrt(3) is within the room between e and the roundings'
root mean square, 2^-23.)  REL bounds ||error||_F / ||result||_F.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
REL = 95 * 2.0 ** -21
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def _B():
    from paper_1807_01702_amd import bnr
    return bnr


def _rand(seed, r, c, low=2):
    """Noise with a few strong directions (float64)."""
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    low = min(low, r, c)
    return n(r, c) + n(r, low) @ n(low, c)


def _ns64(u, steps=5, coef=COEF, eps=1e-7):
    x = u if u.shape[0] <= u.shape[1] else u.t()
    x = x / (torch.sqrt((x * x).sum()) + eps)
    a, b, c = coef
    for _ in range(steps):
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x.contiguous()
    return x if u.shape[0] <= u.shape[1] else x.t()


def _d(t):
    return t.detach().double().cpu()


def _close(name, got, ref, dtype, rel=REL):
    err = float((_d(got) - ref).norm())
    tol = (rel + HALF[dtype]) * float(ref.norm())
    assert err <= tol, "%s: off by %.3g, tolerance %.3g" % (name, err, tol)


# lists whose tiles run whole and in pieces, in each tile size, and hang over the matrices' ends
LARGE = [[(1024, 1024)] * 8, [(2048, 2048)], [(2048, 2048)] * 4, [(1024, 4096)] * 6, [(1300, 2900)] * 3, [(1023, 4093)],
         [(520, 2000), (2700, 1100), (130, 4000)], [(700, 700), (64, 300), (200, 1900), (1500, 129)], [(4096, 1000)],
         [(3000, 2990)], [(64, 64), (700, 700), (20, 500)], [(60, 70), (3, 3), (128, 128), (30, 2000), (9, 9)],
         [(128, 100)] * 300]


@pytest.mark.parametrize("shapes", LARGE, ids=lambda s: "%dx%dx%d" % (len(s), *s[0]))
def test_large_lists(shapes):
    """The reference runs on the GPU in float64 (library products)."""
    B = _B()
    xs = [_rand(i * 31 + r, r, c).float().cuda() for i, (r, c) in enumerate(shapes)]
    outs = [torch.full_like(x, 5.0) for x in xs]
    B.bnr_orthogonalize(xs, outs)
    again = [torch.empty_like(x) for x in xs]
    B.bnr_orthogonalize(xs, again)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, again))
    for x, o in zip(xs, outs):
        ref = _ns64(x.double())
        err = float((o.double() - ref).norm() / ref.norm())
        # longer sums: sqrt(q / 32) 2^-24 per product past q = 2048
        tol = REL * max(1.0, (max(x.shape) / 2048) ** 0.5) + HALF[torch.float32]
        assert err <= tol, (tuple(x.shape), err)


def _strided(t, dtype, pad):
    r, c = t.shape
    buf = torch.full((r, c + pad), 777.0, dtype=dtype, device="cuda")
    buf[:, :c].copy_(t.to(dtype))
    return buf, buf[:, :c]


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (1, 5000), (16, 16), (17, 33), (31, 32), (33, 31), (64, 64), (65, 63),
          (96, 128), (128, 96), (127, 129), (128, 128), (129, 200), (1152, 32), (255, 257), (256, 256), (300, 40),
          (64, 1000), (513, 130), (260, 700), (1025, 515), (513, 1200), (100, 1500), (1100, 128), (20, 5000), (3000, 60),
          (128, 2100)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("r,c", SHAPES)
def test_shapes(r, c, dtype):
    B = _B()
    bx, x = _strided(_rand(r * 1000 + c, r, c), dtype, 3)
    bo, out = _strided(torch.zeros(r, c), dtype, 5)
    keep = bx.clone()
    B.bnr_orthogonalize(x, out)
    torch.cuda.synchronize()
    assert torch.equal(bx, keep), "the input changed"
    assert bool((bo[:, c:] == 777.0).all()), "wrote outside the view"
    _close("out", out, _ns64(_d(x)), dtype)


@pytest.mark.parametrize("steps,coef", [(1, COEF), (2, COEF), (7, COEF), (32, (1.5, -0.5, 0.0)), (12, (1.875, -1.25, 0.375)),
                                        (3, (2.0, -1.5, 0.5))])
def test_steps_and_coefficients(steps, coef):
    B = _B()
    for r, c in ((40, 90), (300, 130)):
        x = _rand(5, r, c).float().cuda()
        out = torch.empty_like(x)
        B.bnr_orthogonalize(x, out, steps=steps, coef=coef)
        ref = _ns64(_d(x), steps, coef)
        a, b, cc = (abs(v) for v in coef)
        _close("steps %d" % steps, out, ref, torch.float32, max(steps, 1) * (a + 2 * b + 3 * cc) * 2.0 ** -21)


def test_singular_values_and_vectors():
    """The result's singular values are p(p(..)) of the input's, with its singular vectors; apart from the reference
    above, from a matrix made of chosen factors."""
    B = _B()
    g = torch.Generator().manual_seed(11)
    u = torch.linalg.qr(torch.randn(60, 60, generator=g, dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn(150, 60, generator=g, dtype=torch.float64))[0]
    s = torch.logspace(0, -3, 60, dtype=torch.float64)
    x = (u * s) @ v.t()
    out = torch.empty(60, 150, device="cuda")
    xf = x.float()
    B.bnr_orthogonalize(xf.cuda(), out)
    t = s / s.norm()
    a, b, c = COEF
    for _ in range(5):
        t = t * (a + b * t ** 2 + c * t ** 4)
    # xf is x rounded: its rounding (2^-24 of every entry) passes 5 steps of slope 3.45 at the small values
    slack = 3.4445 ** 5 * 2.0 ** -24 * float(x.norm()) / float(s.norm()) * np.sqrt(60)
    err = float((_d(out) - (u * t) @ v.t()).norm())
    assert err <= REL * float(t.norm()) + slack, err
    # the smallest starts at 1e-3 / ||s|| = 4.5e-4 and grows by 3.4445^5 = 485
    assert 0.2 < float(t.min()) < 0.25 and float(t.max()) < 1.3


def test_scales_of_the_input():
    """The result does not depend on the input's scale, from the smallest to the largest squares."""
    B = _B()
    x = _rand(7, 70, 90).float().cuda()
    ref = torch.empty_like(x)
    B.bnr_orthogonalize(x, ref, eps=0.0)
    for k in (-100, -60, 20, 90):
        out = torch.empty_like(x)
        B.bnr_orthogonalize(x * 2.0 ** k, out, eps=0.0)
        assert torch.equal(out, ref), k
    # with eps, an input far below it stays far below 1
    out = torch.empty_like(x)
    tiny = x * 1e-12
    B.bnr_orthogonalize(tiny, out)
    want = _ns64(_d(tiny))
    # X is held to 2^-37 of 1 and grows by a per step; each step's factor a I + .. is held with 22 bits, off by up to
    # 2^-22 of the result itself (5 times: 1.2e-6, part of REL)
    assert float((_d(out) - want).abs().max()) <= COEF[0] ** 5 * 2.0 ** -36 + REL * float(want.abs().max())


def test_zero_and_non_finite_matrices_of_a_list():
    B = _B()
    shapes = [(40, 60), (128, 200), (33, 33), (70, 20), (5, 300)]
    xs = [_rand(i, *s).float().cuda() for i, s in enumerate(shapes)]
    clean = [torch.empty_like(x) for x in xs]
    B.bnr_orthogonalize(xs, clean)
    xs[1] = torch.zeros_like(xs[1])
    xs[2][3, 4] = float("nan")
    xs[3][0, 0] = float("inf")
    outs = [torch.full_like(x, 5.0) for x in xs]
    B.bnr_orthogonalize(xs, outs)
    torch.cuda.synchronize()
    assert bool((outs[1] == 0).all())
    assert bool(torch.isnan(outs[2]).all()) and bool(torch.isnan(outs[3]).all())
    assert torch.equal(outs[0], clean[0]) and torch.equal(outs[4], clean[4])


def test_list_equals_single_calls_in_place_and_again():
    """A matrix's result does not depend on the list around it, is the same on the next call, and may be written over
    the input."""
    B = _B()
    shapes = [(1152, 32), (64, 128), (256, 128), (31, 7), (300, 300), (1, 9), (700, 500)] + [(96 + 8 * i, 128) for i in range(70)]
    xs = [_rand(i, *s).float().cuda() for i, s in enumerate(shapes)]
    outs = [torch.empty_like(x) for x in xs]
    B.bnr_orthogonalize(xs, outs)
    again = [torch.empty_like(x) for x in xs]
    B.bnr_orthogonalize(xs, again)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))
    for i in (0, 1, 2, 3, 4, 5, 6, 40, 75):
        one = torch.empty_like(xs[i])
        B.bnr_orthogonalize(xs[i], one)
        _close("alone %d" % i, one, _d(outs[i]), torch.float32)
        _close("list %d" % i, outs[i], _ns64(_d(xs[i])), torch.float32)
    place = [x.clone() for x in xs]
    B.bnr_orthogonalize(place, place)
    assert all(torch.equal(a, b) for a, b in zip(outs, place))
    B.bnr_orthogonalize([], [])


def test_column_slices_of_one_matrix():
    """Several matrices as column slices of one buffer, read and written."""
    B = _B()
    x = _rand(3, 96, 300).float().cuda()
    out = torch.zeros_like(x)
    cuts = [(0, 100), (100, 164), (164, 300)]
    B.bnr_orthogonalize([x[:, a:b] for a, b in cuts], [out[:, a:b] for a, b in cuts])
    for a, b in cuts:
        _close("slice %d" % a, out[:, a:b], _ns64(_d(x[:, a:b])), torch.float32)


def _state(shapes, wdt, gdt, copies, seed=0):
    ws = [(_rand(seed + 10 * i, *s) * 0.05).to(wdt).cuda() for i, s in enumerate(shapes)]
    gs = [(_rand(seed + 10 * i + 1, *s) * 10.0 ** (i % 4 - 3)).to(gdt).cuda() for i, s in enumerate(shapes)]
    bs = [(_rand(seed + 10 * i + 2, *s) * 10.0 ** (i % 4 - 3)).float().cuda() for i, s in enumerate(shapes)]
    cs = [w.bfloat16().clone() for w in ws] if copies else None
    return ws, gs, bs, cs


def _update64(w, g, b, lr, mom, nesterov, wd, scale):
    b = mom * b + g
    u = g + mom * b if nesterov else b
    step = lr * scale * _ns64(u)
    return w * (1 - lr * wd) - step, b, step


@pytest.mark.parametrize("wdt,gdt,copies", [(torch.float32, torch.float32, True), (torch.float32, torch.bfloat16, False),
                                            (torch.bfloat16, torch.float32, False), (torch.bfloat16, torch.bfloat16, True)])
@pytest.mark.parametrize("nesterov,mom,wd", [(True, 0.95, 0.1), (False, 0.9, 0.0), (True, 0.0, 0.01)])
def test_update(wdt, gdt, copies, nesterov, mom, wd):
    B = _B()
    shapes = [(1152, 32), (64, 128), (130, 257), (1, 1), (40, 9), (300, 140)]
    ws, gs, bs, cs = _state(shapes, wdt, gdt, copies)
    scales = [1.0, 0.3, 2.0, 1.0, 0.5, 1.0]
    group = B.MuonGroup(ws, gs, bs, copies=cs, scales=scales)
    lr = 0.02
    before = [(_d(w), _d(g), _d(b)) for w, g, b in zip(ws, gs, bs)]
    B.bnr_muon_update(group, lr, momentum=mom, nesterov=nesterov, weight_decay=wd)
    torch.cuda.synchronize()
    u = 2.0 ** -24
    f32 = lambda v: float(np.float32(v))  # noqa: E731  (the numbers the call is given)
    for i, (w0, g0, b0) in enumerate(before):
        w, b, step = _update64(w0, g0, b0, f32(lr), f32(mom), nesterov, f32(wd), f32(scales[i]))
        # momentum: the product and the sum, each rounded at most once
        assert bool(((_d(bs[i]) - b).abs() <= u * (b.abs() + (f32(mom) * b0).abs() + g0.abs())).all()), i
        # weights: the step's error, three roundings of the factors and the sum, then the storage
        err = (_d(ws[i]) - w)
        tol = REL * float(step.norm()) + 4 * u * float(w0.norm() + step.norm()) + HALF[wdt] * float(w.norm())
        assert float(err.norm()) <= tol, (i, float(err.norm()), tol)
        if copies:
            assert torch.equal(cs[i], ws[i].bfloat16()), i
        assert torch.equal(gs[i].double().cpu(), g0)


def test_update_of_conv_filters_and_default_scale():
    """[k, k, c_in, c_out] filters are matrices [k k c_in, c_out]; the default factor is sqrt(max(1, out / in))."""
    B = _B()
    w = (torch.randn(3, 3, 16, 32, generator=torch.Generator().manual_seed(1)) * 0.1).cuda()
    w1 = (torch.randn(1, 1, 16, 64, generator=torch.Generator().manual_seed(2)) * 0.1).cuda()
    g, g1 = torch.randn_like(w), torch.randn_like(w1)
    b, b1 = torch.zeros_like(w), torch.zeros_like(w1)
    group = B.MuonGroup([w, w1], [g, g1], [b, b1])
    w0, w10 = _d(w).reshape(-1, 32), _d(w1).reshape(-1, 64)
    B.bnr_muon_update(group, 0.5, momentum=0.5, nesterov=False)
    for t, t0, gg, sc in ((w, w0, g, 1.0), (w1, w10, g1, 2.0)):
        step = 0.5 * sc * _ns64(_d(gg).reshape(t0.shape))
        err = float((_d(t).reshape(t0.shape) - (t0 - step)).norm())
        assert err <= REL * float(step.norm()) + 2.0 ** -22 * float(t0.norm() + step.norm())


def test_two_streams_graphs_and_device_rate():
    """Two updates at once on two streams; a captured step replayed with another learning rate in device memory,
    two graphs in turn, eager work between the replays."""
    B = _B()
    shapes = [(1152, 32), (200, 128), (300, 300), (64, 640)]

    def fresh(seed):
        ws, gs, bs, _ = _state(shapes, torch.float32, torch.float32, False, seed)
        return ws, gs, bs

    def steps(seed, lrs):
        ws, gs, bs = fresh(seed)
        group = B.MuonGroup(ws, gs, bs)
        for lr in lrs:
            B.bnr_muon_update(group, float(np.float32(lr)), weight_decay=0.1)
        torch.cuda.synchronize()
        return ws + bs

    rates = (0.02, 0.01, 0.03)
    want = [steps(0, rates), steps(1000, rates)]
    parts = [fresh(0), fresh(1000)]
    groups = [B.MuonGroup(*p) for p in parts]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for lr in rates:
        for grp, st in zip(groups, streams):
            with torch.cuda.stream(st):
                B.bnr_muon_update(grp, lr, weight_decay=0.1)
    torch.cuda.synchronize()
    for p, w in zip(parts, want):
        assert all(torch.equal(a, b) for a, b in zip(p[0] + p[2], w))
    parts = [fresh(0), fresh(1000)]
    groups = [B.MuonGroup(*p) for p in parts]
    lr = torch.zeros(1, device="cuda")
    graphs = []
    torch.cuda.synchronize()
    for grp in groups:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.bnr_muon_update(grp, lr, weight_decay=0.1)
        graphs.append(g)
    for rate in rates:
        lr.fill_(rate)
        for g in graphs:
            g.replay()
        steps(77, (0.1,))
        torch.cuda.synchronize()
    for p, w in zip(parts, want):
        assert all(torch.equal(a, b) for a, b in zip(p[0] + p[2], w))


def test_handle_refusals():
    B = _B()
    w = torch.zeros(8, 8, device="cuda")
    with pytest.raises(ValueError):
        B.MuonGroup([w], [w.clone()], [])
    with pytest.raises(ValueError):
        B.MuonGroup([w], [torch.zeros(8, 9, device="cuda")], [w.clone()])
    with pytest.raises(ValueError):
        B.MuonGroup([w], [w.clone()], [w.bfloat16()])
    with pytest.raises(ValueError):
        B.MuonGroup([w], [torch.zeros(8, 8)], [w.clone()])
    with pytest.raises(B.BnrError, match="shares memory"):
        B.bnr_muon_update(B.MuonGroup([w], [w.clone()], [w]), 0.1)
    with pytest.raises(B.BnrError, match="shares memory"):        # the same matrix twice
        B.bnr_muon_update(B.MuonGroup([w, w], [w.clone(), w.clone()], [w.clone(), w.clone()]), 0.1)
    with pytest.raises(B.BnrError, match="range"):
        B.bnr_orthogonalize(w, w.clone(), coef=(9.0, 0.0, 0.0))
    with pytest.raises(ValueError):
        B.bnr_muon_update(B.MuonGroup([w], [w.clone()], [w.clone()]), torch.zeros(1))
    assert bool((w == 0).all())
    B.bnr_muon_update(B.MuonGroup([], [], []), 0.1)


@pytest.mark.parametrize("wdt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("r,c", [(200, 333), (333, 200), (150, 256), (40, 150), (150, 41), (9, 7)])
def test_rows_of_every_alignment(r, c, wdt):
    """Weights, copies and outputs inside larger buffers: pitches and first elements that do and do not allow
    accesses of four columns give the contiguous matrices' bits, and nothing beside the rows changes."""
    B = _B()

    def inside(t, pitch, first):
        whole = torch.full((r * pitch + first + 8,), 7.0, dtype=t.dtype, device="cuda")
        view = whole[first:first + r * pitch].view(r, pitch)[:, :c]
        view.copy_(t)
        return whole, view

    (w,), (g,), (b,), (k,) = _state([(r, c)], wdt, torch.float32, True, seed=5)
    out = torch.empty_like(g)
    B.bnr_orthogonalize([g], [out])
    even = -(-c // 4) * 4
    places = [(even + 4, 0), (even, 4), (even + 4, 8), (even + 1, 0), (even + 2, 2), (even + 4, 1)]
    runs = [(w.clone(), b.clone(), k.clone())]
    fences = []
    for pitch, first in places:
        (ww, wv), (kw, kv), (ow, ov) = inside(w, pitch, first), inside(k, pitch + 4, first), inside(out * 0, pitch, first)
        B.bnr_orthogonalize([g], [ov])
        assert torch.equal(ov, out)
        runs.append((wv, b.clone(), kv))
        fences += [(ww, wv, first, pitch), (kw, kv, first, pitch + 4), (ow, ov, first, pitch)]
    for wv, bv, kv in runs:
        B.bnr_muon_update(B.MuonGroup([wv], [g], [bv], copies=[kv]), 0.02, weight_decay=0.1)
    assert not torch.equal(runs[0][0], w)
    for wv, bv, kv in runs[1:]:
        assert torch.equal(wv, runs[0][0]) and torch.equal(bv, runs[0][1]) and torch.equal(kv, runs[0][2])
    for whole, view, first, pitch in fences:
        out_of_rows = torch.ones_like(whole, dtype=torch.bool)
        out_of_rows[first:first + r * pitch].view(r, pitch)[:, :c] = False
        assert bool((whole[out_of_rows] == 7.0).all())


def test_one_input_for_several_outputs():
    """The same matrix, and the same gradient, twice in a list: they are only read."""
    B = _B()
    for r, c in ((40, 60), (90, 700), (200, 300)):
        x = _rand(7, r, c).float().cuda()
        keep, outs = x.clone(), [torch.empty_like(x) for _ in range(3)]
        B.bnr_orthogonalize([x, x, x], outs)
        _close("%dx%d" % (r, c), outs[0], _ns64(_d(x)), torch.float32)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and torch.equal(x, keep)
        w = [torch.ones_like(x) for _ in range(2)]
        B.bnr_muon_update(B.MuonGroup(w, [x, x], [torch.zeros_like(x) for _ in range(2)]), 0.1)
        assert torch.equal(w[0], w[1]) and torch.equal(x, keep) and not torch.equal(w[0], torch.ones_like(x))


@pytest.mark.parametrize("r,c", [(128, 512), (128, 513), (64, 2048), (2049, 64), (32, 16384), (20, 16385), (32, 2047)])
def test_narrow_blocks_around_the_sum(r, c):
    """Short sides whose blocks add the partial Gram matrices themselves, up to the largest number, and one more."""
    B = _B()
    x = _rand(11, r, c).float().cuda()
    out = torch.empty_like(x)
    B.bnr_orthogonalize(x, out)
    _close("alone", out, _ns64(_d(x)), torch.float32)
    y = _rand(12, 16, 24).float().cuda()
    outs = [torch.empty_like(x), torch.empty_like(y)]
    B.bnr_orthogonalize([x, y], outs)
    assert torch.equal(outs[0], out)
    _close("beside", outs[1], _ns64(_d(y)), torch.float32)


def test_copies_of_some_matrices():
    """A list where only some matrices have a bf16 copy: the others' results are those of a list without copies."""
    B = _B()
    shapes = [(40, 60), (300, 200), (9, 7), (128, 600)]
    ws, gs, bs, cs = _state(shapes, torch.float32, torch.float32, True)
    plain = [w.clone() for w in ws], [b.clone() for b in bs]
    B.bnr_muon_update(B.MuonGroup(plain[0], gs, plain[1]), 0.02)
    B.bnr_muon_update(B.MuonGroup(ws, gs, bs, copies=[cs[0], None, None, cs[3]]), 0.02)
    assert all(torch.equal(a, b) for a, b in zip(ws + bs, plain[0] + plain[1]))
    assert torch.equal(cs[0], ws[0].bfloat16()) and torch.equal(cs[3], ws[3].bfloat16())


# Further choices of the tile rule for X X^T, its square and R X, so that every kernel and every way to cut is run:
# tiles of 256 whole for all three (twelve of 1296 x 1489), R X in pieces only, of 128-tiles (1680 x 1256) and of
# 256-tiles (2360 x 2160).
@pytest.mark.parametrize("shapes", [[(1296, 1489)] * 12, [(1680, 1256)], [(2360, 2160)]], ids=lambda s: "%dx%dx%d" % (len(s), *s[0]))
def test_whole_and_cut_large_tiles(shapes):
    test_large_lists(shapes)


# (shapes, how R X, whose last one leaves the result, is tiled)
RESULTS = [([(1023, 4093)], "128 whole, ragged"), ([(4093, 1023)], "128 whole, turned"), ([(1680, 1256)], "128 in pieces"),
           ([(2360, 2160)], "256 in pieces"), ([(1300, 2900)] * 3, "256 whole, ragged"), ([(1024, 4096)] * 6, "256, some in pieces"),
           ([(3000, 2990)], "128, some in pieces"), ([(1000, 999)], "64"), ([(513, 300), (700, 260)], "32")]


@pytest.mark.parametrize("shapes,how", RESULTS, ids=[h.replace(" ", "-") for _, h in RESULTS])
def test_results_of_every_tile(shapes, how):
    """bf16 results, and weight steps with float32 weights and bf16 copies and with bf16 weights, from every kernel
    that leaves results.  The reference runs on the GPU in float64; longer sums as in test_large_lists."""
    B = _B()
    rel = REL * max(1.0, (max(max(s) for s in shapes) / 2048) ** 0.5)
    xs = [_rand(i * 17 + r, r, c).bfloat16().cuda() for i, (r, c) in enumerate(shapes)]
    outs = [torch.full_like(x, 5.0) for x in xs]
    B.bnr_orthogonalize(xs, outs)
    for x, o in zip(xs, outs):
        ref = _ns64(x.double())
        assert float((o.double() - ref).norm()) <= (rel + HALF[torch.bfloat16]) * float(ref.norm())
    lr, mom, wd = 0.125, 0.5, 0.25
    for wdt, gdt in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)):
        ws, gs, bs, cs = _state(shapes, wdt, gdt, True, seed=3)
        before = [(w.double(), g.double(), b.double()) for w, g, b in zip(ws, gs, bs)]
        scales = [0.5 + i for i in range(len(shapes))]
        B.bnr_muon_update(B.MuonGroup(ws, gs, bs, copies=cs, scales=scales), lr, momentum=mom, weight_decay=wd)
        for i, (w0, g0, b0) in enumerate(before):
            w, b, step = _update64(w0, g0, b0, lr, mom, True, wd, scales[i])
            u = 2.0 ** -24
            assert bool(((bs[i].double() - b).abs() <= u * (b.abs() + (mom * b0).abs() + g0.abs())).all()), i
            tol = rel * float(step.norm()) + 4 * u * float(w0.norm() + step.norm()) + HALF[wdt] * float(w.norm())
            assert float((ws[i].double() - w).norm()) <= tol, (wdt, i)
            assert torch.equal(cs[i], ws[i].bfloat16())


@pytest.mark.parametrize("shapes", [[(200, 300), (129, 200), (300, 140), (513, 130), (150, 257)], [(1000, 999)] * 5,
                                    [(1023, 4093), (1500, 700), (640, 1300), (900, 2000), (1100, 1030)],
                                    [(1296, 1489)] * 12, [(2360, 2160)] * 5], ids=lambda s: "%dx%dx%d" % (len(s), *s[0]))
def test_wide_zero_and_non_finite_matrices_of_a_list(shapes):
    """As test_zero_and_non_finite_matrices_of_a_list for short sides past 128, where a tile that hangs over a matrix
    reads its last rows again: a zero matrix gives zeros, a NaN in the last element and an infinity in the first make
    their own matrices NaN, and every other matrix keeps its bits."""
    B = _B()
    xs = [_rand(i, *s).float().cuda() for i, s in enumerate(shapes)]
    clean = [torch.empty_like(x) for x in xs]
    B.bnr_orthogonalize(xs, clean)
    xs[1] = torch.zeros_like(xs[1])
    xs[2][-1, -1] = float("nan")
    xs[3][0, 0] = float("-inf")
    outs = [torch.full_like(x, 5.0) for x in xs]
    B.bnr_orthogonalize(xs, outs)
    assert bool((outs[1] == 0).all())
    assert bool(torch.isnan(outs[2]).all()) and bool(torch.isnan(outs[3]).all())
    for i in [0] + list(range(4, len(shapes))):
        assert torch.equal(outs[i], clean[i]), i


@pytest.mark.parametrize("r,c", [(200, 300), (1000, 999), (1023, 4093), (2360, 2160), (100, 3000)])
def test_wide_scales_of_the_input(r, c):
    """Powers of two in front of the matrix leave the bits as they are."""
    B = _B()
    x = _rand(7, r, c).float().cuda()
    ref, out = torch.empty_like(x), torch.empty_like(x)
    B.bnr_orthogonalize(x, ref, eps=0.0)
    for k in (-90, -30, 60):
        B.bnr_orthogonalize(x * 2.0 ** k, out, eps=0.0)
        assert torch.equal(out, ref), k


def _kinds(r, c, seed):
    """Matrices whose singular values are far apart (float32, on the GPU)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    u = n(r, c)
    yield "direction 30", u + 30 * n(r, 1) @ n(1, c)
    yield "direction 1e4", u + 1e4 * n(r, 1) @ n(1, c)
    yield "rows of 1 to 1e-4", u * 1e-4 ** torch.rand(r, 1, generator=g, device="cuda")
    yield "rank 4", n(r, 4) @ n(4, c) + 1e-3 * u
    p = min(r, c)
    left, right = torch.linalg.qr(n(r, p))[0], torch.linalg.qr(n(c, p))[0]
    yield "decay over five decades", (left * torch.logspace(0, -5, p, device="cuda")) @ right.t()


@pytest.mark.parametrize("r,c", [(60, 90), (64, 576), (1152, 128), (300, 400), (512, 1024), (1023, 2047)])
def test_matrices_of_low_effective_rank(r, c):
    """A few directions hold almost all of the norm, so errors made beside them grow with the weak directions.  Step k
    adds an error of at most (|a| + 2 |b| + 3 |c|) e ||X_k||_F (head of this file, e = 2^-21), and no later step
    stretches a difference by more than its largest slope, p'(0) = a."""
    B = _B()
    a, b, cc = COEF
    for name, u in _kinds(r, c, r + c):
        out = torch.empty_like(u)
        B.bnr_orthogonalize(u, out)
        ud, tol = u.double(), 0.0
        for k in range(5):
            tol += (a - 2 * b + 3 * cc) * 2.0 ** -21 * float(_ns64(ud, k).norm()) * a ** (4 - k)
        ref = _ns64(ud)
        assert float((out.double() - ref).norm()) <= tol + HALF[torch.float32] * float(ref.norm()), name


@pytest.mark.parametrize("r,c", [(40, 60), (100, 900), (900, 100), (300, 400), (700, 300)])
def test_offsets_past_32_bits(r, c):
    """Rows so far apart that the last ones start past 2^31 elements, for every argument, and 4 columns beside every
    row: the contiguous matrices' bits, and nothing beside the rows changes."""
    B = _B()
    ld = -(-(1 << 31) // (r - 8)) // 8 * 8 + 8
    n = (r - 1) * ld + c + 8
    far = lambda dt: torch.as_strided(torch.empty(n, dtype=dt, device="cuda"), (r, c + 4), (ld, 1))  # noqa: E731

    def put(t):
        v = far(t.dtype)
        v[:, :c] = t
        v[:, c:] = 7.0
        return v

    assert (r - 1) * ld > 1 << 31
    (w,), (g,), (b,), (k,) = _state([(r, c)], torch.float32, torch.float32, True, seed=9)
    fw, fg, fb, fk = put(w), put(g), put(b), put(k)
    B.bnr_muon_update(B.MuonGroup([fw[:, :c]], [fg[:, :c]], [fb[:, :c]], copies=[fk[:, :c]]), 0.02, weight_decay=0.1)
    B.bnr_muon_update(B.MuonGroup([w], [g], [b], copies=[k]), 0.02, weight_decay=0.1)
    for f, t in ((fw, w), (fg, g), (fb, b), (fk, k)):
        assert torch.equal(f[:, :c], t) and bool((f[:, c:] == 7.0).all())
    out = torch.empty_like(g)
    B.bnr_orthogonalize(g, out)
    B.bnr_orthogonalize(fg[:, :c], fw[:, :c])
    assert torch.equal(fw[:, :c], out) and bool((fw[:, c:] == 7.0).all())


def _ns32(u):
    """The iteration in float32 products of the library, u [n, r, c] (r <= c)."""
    x = u / (u.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    a, b, c = COEF
    for _ in range(5):
        g = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * g + c * torch.bmm(g, g), x)
    return x


@pytest.mark.parametrize("r,c,n", [(8, 8, 64), (16, 40, 64), (31, 90, 64), (32, 2000, 16), (64, 64, 32), (64, 576, 16),
                                   (100, 300, 16), (128, 1152, 8), (150, 257, 8), (512, 1024, 4), (1023, 4093, 2)])
def test_error_beside_float32_products(r, c, n):
    """Root mean square over n matrices of the distance from float64, beside that of float32 products.  An operand's
    pair rounds hi's remainder, up to 2^-11 of the operand's binade, to 11 bits: steps of 2^-22 for half of the
    remainders, 2^-23 for a quarter and so on, root mean square 2^-22 / sqrt(12) times sqrt(1/2 + 1/16 + 1/128 + ..) =
    0.756; float32's is 2^-23 / sqrt(12).  Where operand roundings are all there is, the ratio is 1.51; sums that round
    no more often than the library's do not raise it."""
    B = _B()
    kinds = {}
    for i in range(n):
        g = torch.Generator(device="cuda").manual_seed(1000 + i)
        kinds.setdefault("noise", []).append(torch.randn(r, c, generator=g, device="cuda"))
        for name, u in _kinds(r, c, i):
            kinds.setdefault(name, []).append(u)
    for name, us in kinds.items():
        outs = [torch.empty_like(u) for u in us]
        B.bnr_orthogonalize([u.contiguous() for u in us], outs)
        own = lib = 0.0
        for u, o in zip(us, outs):
            ref = _ns64(u.double())
            own += float(((o.double() - ref).norm() / ref.norm()) ** 2)
            lib += float(((_ns32(u[None])[0].double() - ref).norm() / ref.norm()) ** 2)
        assert (own / lib) ** 0.5 <= 1.51, (name, (own / lib) ** 0.5)
