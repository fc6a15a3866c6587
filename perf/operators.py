"""Timed cases of the operators next to the BN path: layer normalisation of each
pixel's (token's) channels, and the orthogonalised update of weight matrices.

``ln_fwd``  y = (s - mean) rstd gamma + beta over the channels of each row, s = x or
            the stored sum x + res; also mean, rstd and s
``ln_bwd``  its gradients: dx (plus the gradient that reaches s by another way), and
            dgamma, dbeta summed over all rows
``orth``    the orthogonalised form of each matrix of a list, by Newton-Schulz products:
            X <- X / (||X||_F + eps), then five times
            X <- a X + b (X X^T) X + c (X X^T)^2 X   (on the shorter side)
``update``  the optimizer step built on it, for a list of weight matrices: momentum,
            orthogonalisation, weight decay and the step, in place

``run`` computes the plain forms in float32 torch operations, or calls the library
(``own``).  ``exact`` evaluates the definitions in float64.
"""
import math

import torch

own = False

EPS_LN = 1e-5
EPS_NS = 1e-7
COEF = (3.4445, -4.7750, 2.0315)
STEPS = 5
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


def _dense_filters(c0, layers, growth, width):
    """Filters of a dense block's composite layers: 1x1 [c, width], 3x3 [9 width, growth]."""
    return ["1x%dx%d" % (c0 + growth * i, width) for i in range(layers)] + ["%dx%dx%d" % (layers, 9 * width, growth)]


def _net_filters(blocks, c0=64, growth=32, width=128):
    """Every 1x1 and 3x3 filter of a DenseNet, transitions included, equal shapes together."""
    count, c = {}, c0
    for i, layers in enumerate(blocks):
        for part in _dense_filters(c, layers, growth, width):
            n, r, k = (int(v) for v in part.split("x"))
            count[r, k] = count.get((r, k), 0) + n
        c += layers * growth
        if i + 1 < len(blocks):
            count[c, c // 2] = count.get((c, c // 2), 0) + 1
            c //= 2
    return ["%dx%dx%d" % (n, r, k) for (r, k), n in sorted(count.items())]


def listed():
    return [
        # one token (or one pixel) at a time, where latency is everything
        dict(name="ln_fwd_one_row", op="ln_fwd", m=1, c=1024, ldc=1024, bf16=True, res=True),
        # a channel slice of the first dense block's concatenation buffer at batch 64 (56x56 images), float32
        dict(name="ln_fwd_block1_slice_f32", op="ln_fwd", m=64 * 56 * 56, c=96, ldc=256, bf16=False, res=False),
        # a batch of 8192 tokens, with the residual addition in front
        dict(name="ln_fwd_tokens_bf16", op="ln_fwd", m=8192, c=4096, ldc=4096, bf16=True, res=True),
        # a small odd batch of an odd width
        dict(name="ln_bwd_odd_f32", op="ln_bwd", m=77, c=1001, ldc=1001, bf16=False, res=False),
        # the way back through the 8192 tokens, the residual's gradient added
        dict(name="ln_bwd_tokens_bf16", op="ln_bwd", m=8192, c=4096, ldc=4096, bf16=True, res=True),
        # the output pixels of ResNet-50's conv2_x blocks at batch 128: many short rows
        dict(name="ln_bwd_stack_bf16", op="ln_bwd", m=128 * 56 * 56, c=256, ldc=256, bf16=True, res=True),
        # one small square matrix: launches and latency
        dict(name="orth_128_f32", op="orth", shapes="1x128x128", bf16=False),
        # an odd rectangle in bf16
        dict(name="orth_odd_bf16", op="orth", shapes="1x1023x4093", bf16=True),
        # a large square matrix: products only
        dict(name="orth_4096_f32", op="orth", shapes="1x4096x4096", bf16=False),
        # the filters of the benchmark's dense block and its transition, float32 weights with a bf16 copy
        dict(name="update_block1_f32", op="update", shapes=",".join(_dense_filters(64, 6, 32, 128) + ["1x256x128"]),
             bf16=False),
        # every 1x1 and 3x3 filter of DenseNet-121: 119 matrices
        dict(name="update_densenet121_f32", op="update", shapes=",".join(_net_filters((6, 12, 24, 16))), bf16=False),
        # the projections of several layers of one width, weights and gradients in bf16
        dict(name="update_wide_bf16", op="update", shapes="12x1024x4096", bf16=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "orth", "update"])
    bf16 = rng.random() < 0.5
    if op in ("ln_fwd", "ln_bwd"):
        c = rng.choice([_log(rng, 1, 16384), 8 * _log(rng, 1, 2048), 8 * _log(rng, 1, 2048)])
        m = _log(rng, 1, min(400_000, (100_000_000 if bf16 else 50_000_000) // c))
        return dict(op=op, m=m, c=c, ldc=c + rng.choice([0, 0, 8, 64]), bf16=bf16, res=rng.random() < 0.5)
    shapes, left = [], 3e11 if op == "orth" else 1.5e11          # p p q of one product of the largest listed cases: 6.9e10
    for _ in range(rng.choice([1, 1, 2, 3])):
        r, k = _log(rng, 1, 4096), _log(rng, 1, 4096)
        if rng.random() < 0.5:
            r, k = 8 * -(-r // 8), 8 * -(-k // 8)
        n = _log(rng, 1, 24)
        cost = min(r, k) ** 2 * max(r, k) * 4.0
        n = max(0, min(n, int(left / cost), int(2.5e7 / (r * k))))
        left -= n * cost
        if n:
            shapes.append("%dx%dx%d" % (n, r, k))
    return dict(op=op, shapes=",".join(shapes or ["1x64x576"]), bf16=bf16)


def _groups(case):
    return [tuple(int(v) for v in part.split("x")) for part in case["shapes"].split(",")]


def _type(case):
    return torch.bfloat16 if case["bf16"] else torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------ inputs ----
def _ln_inputs(case, seed):
    g, dt = _gen(seed), _type(case)
    m, c, ldc = case["m"], case["c"], case["ldc"]
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    # activations: every channel has its own mean and spread
    x = n(m, ldc).mul_(torch.rand(ldc, generator=g, device="cuda") * 1.2 + 0.4).add_(0.5 * n(ldc)).to(dt)[:, :c]
    t = dict(x=x, gamma=1 + 0.2 * n(c), beta=0.2 * n(c))
    if case["op"] == "ln_fwd":
        t["res"] = n(m, c).to(dt) if case["res"] else None
    else:
        t["dy"] = n(m, c).mul_(0.01).to(dt)
        t["dsum"] = n(m, c).mul_(0.01).to(dt) if case["res"] else None
    return t


def _matrices(case, seed):
    """Gradient-like matrices: noise with a few strong directions, each of its own scale.  One flat array; equal
    shapes lie together."""
    g = _gen(seed)
    parts = []
    for n, r, k in _groups(case):
        v = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        low = min(4, r, k)
        t = v(n, r, k) + torch.bmm(v(n, r, low) * 1.5, v(n, low, k))
        parts.append(t.mul_(10.0 ** (torch.rand(n, 1, 1, generator=g, device="cuda") * 3 - 4)).reshape(-1))
    return torch.cat(parts)


def _split(flat, case):
    """The [n, r, k] parts of a flat array."""
    out, at = [], 0
    for n, r, k in _groups(case):
        out.append(flat[at:at + n * r * k].view(n, r, k))
        at += n * r * k
    return out


def _list(flat, case):
    return [t for part in _split(flat, case) for t in part.unbind(0)]


def prepare(case, seed):
    dt = _type(case)
    if case["op"] in ("ln_fwd", "ln_bwd"):
        s = _ln_inputs(case, seed)
        s["case"] = case
        m, c = case["m"], case["c"]
        out = lambda: torch.empty((m, c), dtype=dt, device="cuda")  # noqa: E731
        if case["op"] == "ln_fwd":
            s["mean"] = s["rstd"] = None
            s["y"], s["sum"] = out(), out() if case["res"] else None
        else:                                            # what the forward left
            xd = s["x"].double()
            var, mean = torch.var_mean(xd, dim=1, correction=0)
            s["mean"], s["rstd"] = mean.float(), (var + EPS_LN).rsqrt().float()
            s["dx"], s["dgamma"], s["dbeta"] = out(), torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
        if own:
            from paper_1807_01702_amd import bnr as B
            s["ln"] = B.LN(s["gamma"], s["beta"], m, EPS_LN, mean=s["mean"], rstd=s["rstd"])
        return s
    u = _matrices(case, seed)
    if case["op"] == "orth":
        x = u.to(dt)
        return dict(case=case, x=x, out=torch.empty_like(x), xs=_list(x, case))
    # a run under way: weights, gradients, momentum of earlier steps
    s = dict(case=case, g=u.to(dt), buf=_matrices(case, seed + 500_000_003).mul_(3.0),
             w=(torch.randn(u.numel(), generator=_gen(seed + 7), device="cuda") * 0.05).to(dt))
    s["copy"] = None if case["bf16"] else s["w"].to(torch.bfloat16)
    if own:
        from paper_1807_01702_amd import bnr as B
        s["group"] = B.MuonGroup(_list(s["w"], case), _list(s["g"], case), _list(s["buf"], case),
                                 copies=None if s["copy"] is None else _list(s["copy"], case),
                                 scales=[_scale(r, k) for n, r, k in _groups(case) for _ in range(n)])
    return s


def _scale(r, k):
    return math.sqrt(max(1.0, k / r))                    # [inputs, outputs]: wider outputs, longer steps


# -------------------------------------------------------------- plain forms ----
def _ln_fwd(s):
    c, dt = s["case"], s["x"].dtype
    x = s["x"].float()
    if c["res"]:
        total = (x + s["res"].float()).to(dt)
        x = total.float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS_LN)
    out = dict(y=(d * rstd * s["gamma"] + s["beta"]).to(dt), mean=mean[:, 0], rstd=rstd[:, 0])
    if c["res"]:
        out["sum"] = total
    return out


def _ln_bwd(s):
    c, dt = s["case"], s["x"].dtype
    dy = s["dy"].float()
    rstd = s["rstd"][:, None]
    xhat = (s["x"].float() - s["mean"][:, None]) * rstd
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if c["res"]:
        dx = dx + s["dsum"].float()
    return dict(dx=dx.to(dt), dgamma=(dy * xhat).sum(0), dbeta=dy.sum(0))


def _newton_schulz(u):
    """u [n, r, k] float32."""
    x = u if u.shape[1] <= u.shape[2] else u.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS_NS)
    a, b, c = COEF
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x.contiguous())
    return x if u.shape[1] <= u.shape[2] else x.transpose(1, 2)


def _orth(s):
    dt = s["x"].dtype
    return torch.cat([_newton_schulz(t.float()).reshape(-1) for t in _split(s["x"], s["case"])]).to(dt)


def _update(s):
    c = s["case"]
    dt = s["w"].dtype
    s["buf"].mul_(MOMENTUM).add_(s["g"].float())
    u = s["g"].float() + MOMENTUM * s["buf"]
    step = torch.cat([_newton_schulz(t).reshape(-1) * _scale(t.shape[1], t.shape[2]) for t in _split(u, c)])
    s["w"].copy_((s["w"].float() * (1.0 - LR * DECAY) - LR * step).to(dt))
    if s["copy"] is not None:
        s["copy"].copy_(s["w"])
    return _updated(s)


def _updated(s):
    out = dict(w=s["w"], buf=s["buf"])
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    return out


# ---------------------------------------------------------------------- run ----
def _run_own(s):
    from paper_1807_01702_amd import bnr as B
    case = s["case"]
    op = case["op"]
    if op == "ln_fwd":
        B.bnr_layernorm_fwd(s["x"], s["ln"], s["y"], res=s["res"], sum=s["sum"])
        out = dict(y=s["y"], mean=s["ln"].mean, rstd=s["ln"].rstd)
        if case["res"]:
            out["sum"] = s["sum"]
        return out
    if op == "ln_bwd":
        B.bnr_layernorm_bwd(s["dy"], s["x"], s["ln"], s["dx"], s["dgamma"], s["dbeta"], dsum=s["dsum"])
        return dict(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    if op == "orth":
        B.bnr_orthogonalize(s["xs"], _list(s["out"], case), steps=STEPS, coef=COEF, eps=EPS_NS)
        return s["out"]
    B.bnr_muon_update(s["group"], LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY, steps=STEPS, coef=COEF,
                      eps=EPS_NS)
    return _updated(s)


def run(state):
    if own:
        return _run_own(state)
    return dict(ln_fwd=_ln_fwd, ln_bwd=_ln_bwd, orth=_orth, update=_update)[state["case"]["op"]](state)


# --------------------------------------------------------------------- work ----
def work(case):
    es = 2 if case["bf16"] else 4
    if case["op"] == "ln_fwd":
        n = case["m"] * case["c"]
        return {"bytes": n * es * (4 if case["res"] else 2) + 8 * case["m"] + 8 * case["c"], "flops": 8 * n}
    if case["op"] == "ln_bwd":
        n = case["m"] * case["c"]
        return {"bytes": n * es * (4 if case["res"] else 3) + 8 * case["m"] + 12 * case["c"], "flops": 14 * n}
    flops = values = 0
    for n, r, k in _groups(case):
        p, q = min(r, k), max(r, k)
        # X X^T and its square are symmetric: half of each product is enough
        flops += n * STEPS * (p * (p + 1) * q + p * p * (p + 1) + 2 * p * p * q)
        values += n * r * k
    if case["op"] == "orth":
        return {"bytes": 2 * es * values, "flops": flops}
    # gradient read, momentum and weight read and written, the bf16 copy written
    return {"bytes": values * (es + 8 + 2 * es + (0 if case["bf16"] else 2)), "flops": flops}


# -------------------------------------------------------------------- exact ----
def _orth64(u):
    """The iteration on the eigenvalues' side: with G = X X^T, every step multiplies X by q(G) = a + b G + c G^2 and
    G by q(G)^2, so the product of the q's is applied to X once, all in float64."""
    flip = u.shape[0] > u.shape[1]
    x = (u.t() if flip else u).contiguous()
    x = x / (torch.linalg.vector_norm(x) + EPS_NS)
    gram = x @ x.t().contiguous()
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=u.device)
    total = eye
    a, b, c = COEF
    for _ in range(STEPS):
        q = a * eye + gram @ (b * eye + c * gram)
        total, gram = q @ total, q @ gram @ q
    o = total @ x
    return o.t() if flip else o


def exact(case, seed):
    if case["op"] in ("ln_fwd", "ln_bwd"):
        s = _ln_inputs(case, seed)
        gamma, beta = s["gamma"].double().requires_grad_(), s["beta"].double().requires_grad_()
        x = s["x"].double()
        out = {}
        if case["op"] == "ln_fwd" and case["res"]:
            out["sum"] = x + s["res"].double()
            x = out["sum"].to(s["x"].dtype).double()     # what is normalised is the sum as it is stored
        x.requires_grad_()
        centre = x.sum(1, keepdim=True) / case["c"]
        spread = ((x - centre) ** 2).sum(1, keepdim=True) / case["c"] + EPS_LN
        y = gamma * (x - centre) / spread.sqrt() + beta
        if case["op"] == "ln_fwd":
            out.update(y=y, mean=centre[:, 0], rstd=1 / spread[:, 0].sqrt())
            return {k: v.detach() for k, v in out.items()}
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), s["dy"].double())
        if case["res"]:
            dx = dx + s["dsum"].double()
        return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)
    u = _matrices(case, seed)
    dt = _type(case)
    if case["op"] == "orth":
        return torch.cat([_orth64(t).reshape(-1) for t in _list(u.to(dt).double(), case)])
    g = u.to(dt).double()
    buf = MOMENTUM * _matrices(case, seed + 500_000_003).mul_(3.0).double() + g
    w = (torch.randn(u.numel(), generator=_gen(seed + 7), device="cuda") * 0.05).to(dt).double()
    step = torch.cat([(_orth64(t) * _scale(*t.shape)).reshape(-1) for t in _list(g + MOMENTUM * buf, case)])
    w = w - LR * DECAY * w - LR * step
    return dict(w=w, buf=buf, copy=None if case["bf16"] else w)
