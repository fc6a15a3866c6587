"""Timed cases of the operators at the end of a training step: dropout whose mask is
never stored, and the last linear layer with its softmax cross entropy over many
classes, whose logits are never kept.

``drop_fwd``  y = dropout(x) (+ res): element (row, ch) is kept where 16 bits of a
              counter-based generator are at least 65536 p, and scaled
``drop_bwd``  dx = the same elements of dy, scaled (+ the gradient that reaches x by
              another way)
``ce_fwd``    loss[0] the mean and loss[1 + i] the rows' softmax cross entropy of the
              logits h w^T + bias, and lse[1 + i] their log sum exp (lse[0]: the number
              of rows that count; loss and lse of the other rows, a batch's padding: 0)
``ce_bwd``    its gradients dh, dw (and dbias) from h, w, the labels and lse

The generator is Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers:
as easy as 1, 2, 3", 2011) with the counter (ch / 8, row, site, step) and the seed as its
key; its four words are the eight elements' 16 bits, low halves first.

``run`` computes the plain forms in float32 torch operations, or calls the library
(``own``).  ``exact`` evaluates the definitions in float64.
"""
import math

import torch

own = False

IGNORE = -100
SITE, STEP = 3, 1717


def listed():
    return [
        # scoring one token at a time against all classes: the weights are read once
        dict(name="ce_fwd_one_token_bf16", op="ce_fwd", m=1, c=2048, v=65536, bf16=True, bias=False, ignored=0.0,
             smoothing=0.0, z=0.0),
        # the classifier of DenseNet-121 at batch 128, float32: short launches
        dict(name="ce_fwd_classifier_f32", op="ce_fwd", m=128, c=1024, v=1000, bf16=False, bias=True, ignored=0.0,
             smoothing=0.1, z=0.0),
        # evaluating 4096 tokens over a large vocabulary
        dict(name="ce_fwd_tokens_bf16", op="ce_fwd", m=4096, c=4096, v=131072, bf16=True, bias=False, ignored=0.1,
             smoothing=0.0, z=0.0),
        # the way back through the same classifier
        dict(name="ce_bwd_classifier_f32", op="ce_bwd", m=128, c=1024, v=1000, bf16=False, bias=True, ignored=0.0,
             smoothing=0.1, z=0.0),
        # a padded batch of odd sizes with a bias
        dict(name="ce_bwd_odd_bf16", op="ce_bwd", m=1001, c=776, v=40961, bf16=True, bias=True, ignored=0.2,
             smoothing=0.0, z=0.0),
        # a handful of rows: what counts is reading the weights and writing their gradient
        dict(name="ce_bwd_few_rows_bf16", op="ce_bwd", m=16, c=2048, v=65536, bf16=True, bias=False, ignored=0.0,
             smoothing=0.0, z=0.0),
        # a batch of 8192 tokens over a large vocabulary: products only
        dict(name="ce_bwd_tokens_bf16", op="ce_bwd", m=8192, c=4096, v=131072, bf16=True, bias=False, ignored=0.1,
             smoothing=0.0, z=1e-4),
        # one token: latency
        dict(name="drop_fwd_one_row_bf16", op="drop_fwd", m=1, c=1024, ldc=1024, bf16=True, add=True, p=0.1),
        # a batch of 8192 tokens with the residual addition behind it
        dict(name="drop_fwd_tokens_bf16", op="drop_fwd", m=8192, c=4096, ldc=4096, bf16=True, add=True, p=0.1),
        # the new channels of one layer of the first dense block at batch 64, a slice of its buffer, float32
        dict(name="drop_bwd_block1_slice_f32", op="drop_bwd", m=64 * 56 * 56, c=32, ldc=256, bf16=False, add=False,
             p=0.2),
        # an odd batch of an odd width, another gradient added
        dict(name="drop_bwd_odd_bf16", op="drop_bwd", m=1003, c=1001, ldc=1001, bf16=True, add=True, p=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ce_fwd", "ce_bwd", "drop_fwd", "drop_bwd"])
    bf16 = rng.random() < 0.6
    if op in ("drop_fwd", "drop_bwd"):
        c = rng.choice([_log(rng, 1, 16384), 8 * _log(rng, 1, 2048), 8 * _log(rng, 1, 2048)])
        m = _log(rng, 1, min(400_000, (33_000_000 if bf16 else 16_000_000) // c))
        return dict(op=op, m=m, c=c, ldc=c + rng.choice([0, 0, 3, 8, 64]), bf16=bf16, add=rng.random() < 0.5,
                    p=rng.choice([0.1, 0.2, 0.5, rng.uniform(0.0, 0.9)]))
    c = 8 * _log(rng, 8, 512)
    v = _log(rng, 2, 131072)
    # products of at most 2e13 operations (float32: 2e12), 2^29 logits
    most = (2e13 if bf16 else 2e12) / (2.0 * c * v * (3 if op == "ce_bwd" else 1))
    m = _log(rng, 1, max(1, min(8192, int(most), (1 << 29) // v)))
    return dict(op=op, m=m, c=c, v=v, bf16=bf16, bias=rng.random() < 0.5, ignored=rng.choice([0.0, 0.0, 0.1, 0.5]),
                smoothing=rng.choice([0.0, 0.0, 0.1]), z=rng.choice([0.0, 0.0, 1e-4]))


def _type(case):
    return torch.bfloat16 if case["bf16"] else torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------ inputs ----
def _rows(g, m, c, ldc, dt, std=1.0):
    return (torch.randn(m, ldc, generator=g, device="cuda") * std).to(dt)[:, :c]


def _drop_inputs(case, seed):
    g, dt = _gen(seed), _type(case)
    m, c, ldc = case["m"], case["c"], case["ldc"]
    std = 1.0 if case["op"] == "drop_fwd" else 0.01
    return dict(x=_rows(g, m, c, ldc, dt, std), add=_rows(g, m, c, c, dt, std) if case["add"] else None,
                seed=(seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 64))


def _ce_inputs(case, seed):
    """A model under way: normalised features that lean towards their label's weights."""
    g, dt = _gen(seed), _type(case)
    m, c, v = case["m"], case["c"], case["v"]
    w = torch.randn(v, c, generator=g, device="cuda").mul_(1.5 / math.sqrt(c)).to(dt)
    labels = torch.randint(0, v, (m,), generator=g, device="cuda", dtype=torch.int32)
    lean = torch.rand(m, 1, generator=g, device="cuda") * 4.0
    h = torch.randn(m, c, generator=g, device="cuda").addcmul_(lean, w[labels.long()].float()).to(dt)
    if case["ignored"]:                                  # the padding of a batch; its first row is never padding
        pad = torch.rand(m, generator=g, device="cuda") < case["ignored"]
        pad[0] = False
        labels[pad] = IGNORE
    bias = torch.randn(v, generator=g, device="cuda").mul_(0.3) if case["bias"] else None
    return dict(h=h, w=w, labels=labels, bias=bias)


def prepare(case, seed):
    dt = _type(case)
    if case["op"] in ("drop_fwd", "drop_bwd"):
        s = _drop_inputs(case, seed)
        s["case"], s["out"] = case, torch.empty(case["m"], case["c"], dtype=dt, device="cuda")
        if own:
            from paper_1807_01702_amd import bnr as B
            s["drop"] = B.Dropout(case["p"], s["seed"], SITE, STEP)
        return s
    s = _ce_inputs(case, seed)
    s["case"], m, v = case, case["m"], case["v"]
    if case["op"] == "ce_bwd":                           # what the forward left
        logits = _logits(s)
        top = logits.amax(1, keepdim=True)
        total = torch.exp(logits.sub_(top)).sum(1, dtype=torch.float64)
        s["lse"] = torch.empty(1 + m, device="cuda")
        s["lse"][0] = (s["labels"] != IGNORE).sum()
        s["lse"][1:] = top[:, 0].double() + total.log()
        del logits
        s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
        s["dbias"] = torch.empty_like(s["bias"]) if case["bias"] else None
    else:
        s["loss"], s["lse"] = torch.empty(1 + m, device="cuda"), torch.empty(1 + m, device="cuda")
    if own:
        from paper_1807_01702_amd import bnr as B
        s["ce"] = B.CE(s["labels"], bias=s["bias"], ignore=IGNORE, smoothing=case["smoothing"], z_loss=case["z"],
                       lse=s["lse"])
    return s


# -------------------------------------------------------------- plain forms ----
def _words(rows, blocks, seed):
    """The generator's four words for every row and block of eight channels, as int64."""
    low = 0xFFFFFFFF
    x0 = torch.arange(blocks, device="cuda").expand(rows, blocks)
    x1 = torch.arange(rows, device="cuda")[:, None].expand(rows, blocks)
    x2, x3 = torch.full_like(x0, SITE), torch.full_like(x0, STEP)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57          # the products' 64 bits
        x0, x1, x2, x3 = ((b >> 32) & low) ^ x1 ^ k0, b & low, ((a >> 32) & low) ^ x3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((x0, x1, x2, x3), 2)


def _limit(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _drop(s):
    case, x = s["case"], s["x"].float()
    m, c = x.shape
    words = _words(m, (c + 7) // 8, s["seed"])
    bits = torch.stack((words & 0xFFFF, words >> 16), 3).reshape(m, -1)[:, :c]
    t = _limit(case["p"])
    y = torch.where(bits >= t, x * (65536.0 / (65536 - t)), torch.zeros_like(x))
    if case["add"]:
        y = y + s["add"].float()
    return y.to(s["x"].dtype)


def _logits(s):
    logits = s["h"].float() @ s["w"].float().t()
    return logits if s["bias"] is None else logits.add_(s["bias"])


def _ce_fwd(s):
    case, logits = s["case"], _logits(s)
    counts = s["labels"] != IGNORE
    top = logits.amax(1)
    lse = top + torch.exp(logits - top[:, None]).sum(1).log()
    picked = logits.gather(1, s["labels"].clamp_min(0).long()[:, None])[:, 0]
    rows = lse - (1 - case["smoothing"]) * picked + case["z"] * lse * lse
    if case["smoothing"]:
        rows = rows - case["smoothing"] * logits.mean(1)
    rows, lse = torch.where(counts, rows, torch.zeros_like(rows)), torch.where(counts, lse, torch.zeros_like(lse))
    n = counts.sum()
    mean = rows.double().sum() / n
    return dict(loss=torch.cat((mean.float()[None], rows)), lse=torch.cat((n.float()[None], lse)))


def _ce_bwd(s):
    case = s["case"]
    lse = s["lse"][1:, None]
    g = torch.exp(_logits(s).sub_(lse))
    if case["z"]:
        g *= 1 + 2 * case["z"] * lse
    if case["smoothing"]:
        g -= case["smoothing"] / case["v"]
    hot = s["labels"].clamp_min(0).long()[:, None]
    g.scatter_add_(1, hot, torch.full(hot.shape, case["smoothing"] - 1.0, device="cuda"))
    g *= ((s["labels"] != IGNORE) / s["lse"][0])[:, None]
    out = dict(dh=(g @ s["w"].float()).to(s["h"].dtype), dw=(g.t() @ s["h"].float()).to(s["w"].dtype))
    if case["bias"]:
        out["dbias"] = g.sum(0)
    return out


# ---------------------------------------------------------------------- run ----
def _run_own(s):
    from paper_1807_01702_amd import bnr as B
    op = s["case"]["op"]
    if op == "drop_fwd":
        B.bnr_dropout_fwd(s["x"], s["drop"], s["out"], res=s["add"])
        return s["out"]
    if op == "drop_bwd":
        B.bnr_dropout_bwd(s["x"], s["drop"], s["out"], dsum=s["add"])
        return s["out"]
    if op == "ce_fwd":
        B.bnr_linear_ce_fwd(s["h"], s["w"], s["ce"], s["loss"])
        return dict(loss=s["loss"], lse=s["lse"])
    B.bnr_linear_ce_bwd(s["h"], s["w"], s["ce"], s["dh"], s["dw"], dbias=s["dbias"])
    out = dict(dh=s["dh"], dw=s["dw"])
    if s["case"]["bias"]:
        out["dbias"] = s["dbias"]
    return out


def run(state):
    if own:
        return _run_own(state)
    return dict(drop_fwd=_drop, drop_bwd=_drop, ce_fwd=_ce_fwd, ce_bwd=_ce_bwd)[state["case"]["op"]](state)


# --------------------------------------------------------------------- work ----
def work(case):
    es = 2 if case["bf16"] else 4
    m, c = case["m"], case["c"]
    if case["op"] in ("drop_fwd", "drop_bwd"):
        # ten rounds of two products and six other operations for eight elements, two a kept one
        return {"bytes": m * c * es * (3 if case["add"] else 2), "flops": 12 * m * c}
    # rows that count, as drawn on average: the others need nothing read, and zeros written
    v, rows = case["v"], m * (1 - case["ignored"])
    values, bias = (rows * c + v * c) * es, 4 * v if case["bias"] else 0
    if case["op"] == "ce_fwd":                           # labels read, loss and lse written
        return {"bytes": values + bias + 12 * m, "flops": 2 * rows * c * v}
    # labels and lse read, a gradient written for each input; the logits are formed again: three products
    return {"bytes": 2 * (values + bias) + 8 * m + (m - rows) * c * es, "flops": 6 * rows * c * v}


# -------------------------------------------------------------------- exact ----
def _kept64(case, seed):
    """Which elements stay, from the generator's definition: one 32-bit half of each product at a time, so that no
    product passes 48 bits."""
    m, c = case["m"], case["c"]
    dev = torch.device("cuda")

    def halves(x, k):                                    # high and low word of x * k
        low = x * (k & 0xFFFF)
        mid = x * (k >> 16) + (low >> 16)
        return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    block = torch.arange((c + 7) // 8, device=dev)
    word = [block[None, :].repeat(m, 1), torch.arange(m, device=dev)[:, None].repeat(1, len(block)),
            torch.tensor(SITE, device=dev), torch.tensor(STEP, device=dev)]
    for turn in range(10):
        key = [(seed % (1 << 32) + turn * 0x9E3779B9) % (1 << 32), (seed // (1 << 32) + turn * 0xBB67AE85) % (1 << 32)]
        (ha, la), (hb, lb) = halves(word[0], 0xD2511F53), halves(word[2], 0xCD9E8D57)
        word = [hb ^ word[1] ^ key[0], lb, ha ^ word[3] ^ key[1], la]
    word = [x.broadcast_to(m, len(block)) for x in word]
    ch = torch.arange(c, device=dev)
    chosen = torch.stack(word)[(ch % 8) // 2, :, ch // 8].t()
    return (chosen >> (16 * (ch % 2))) % 65536 >= math.floor(case["p"] * 65536 + 0.5)


def exact(case, seed):
    if case["op"] in ("drop_fwd", "drop_bwd"):
        s = _drop_inputs(case, seed)
        share = 1.0 - math.floor(case["p"] * 65536 + 0.5) / 65536
        y = s["x"].double() / share * _kept64(case, s["seed"])
        return y + s["add"].double() if case["add"] else y
    s = _ce_inputs(case, seed)
    h, w = s["h"].double().requires_grad_(), s["w"].double().requires_grad_()
    bias = torch.zeros(case["v"], dtype=torch.float64, device="cuda") if s["bias"] is None else s["bias"].double()
    bias.requires_grad_()
    with torch.set_grad_enabled(case["op"] == "ce_bwd"):
        logits = torch.addmm(bias, h, w.t())
        total = torch.logsumexp(logits, 1)
        at = torch.nonzero(s["labels"] >= 0)[:, 0]
        right = logits[at, s["labels"][at].long()]
        e = case["smoothing"]
        rows = total[at] * (1 + case["z"] * total[at]) - (1 - e) * right
        if e:
            rows = rows - e * logits[at].sum(1) / case["v"]
        mean = rows.sum() / len(at)
    if case["op"] == "ce_bwd":
        grads = torch.autograd.grad(mean, (h, w, bias))
        return {k: t for k, t in zip(("dh", "dw", "dbias"), grads) if k != "dbias" or case["bias"]}
    loss, lse = total.new_zeros(1 + case["m"]), total.new_zeros(1 + case["m"])
    loss[0], lse[0] = mean, len(at)
    loss[1 + at], lse[1 + at] = rows, total[at]
    return dict(loss=loss, lse=lse)
