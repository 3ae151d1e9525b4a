"""The operators that stand between the node states of a training step and their cotangents, as cases that can be timed
and compared: the loss over classes or words with its gradient, layer norm with its backward pass, dropout.

  loss     jitdb_softmax_xent_forward (states, class weights, labels -> loss and log-sum-exp of every row) and
           jitdb_softmax_xent_backward (-> gradients of states, class weights and bias)
  eval     jitdb_softmax_xent_forward alone
  norm     jitdb_layernorm_forward (with dropout behind it where p > 0) and jitdb_layernorm_backward
  dropout  jitdb_dropout, forward pass and the same call on the cotangent
  head     all of them in a row: states -> norm, dropout -> loss, and back to the states' cotangent

Rows are the nodes of a forest; a row whose label is -1 takes no part in the loss (treebanks label some nodes, or the
roots alone).  Gradients of bf16 operands are asked for in bf16 or in fp32.
"""
import math

import torch

own = False

DTYPES = {"f32": (torch.float32, 4), "bf16": (torch.bfloat16, 2)}
EPS = 1e-5


def listed():
    def loss(name, n, labelled, H, C, dtype, grad, op="loss"):
        return dict(name=name, op=op, n=n, labelled=labelled, H=H, C=C, dtype=dtype, grad=grad)

    def norm(name, n, H, dtype, p):
        return dict(name=name, op="norm", n=n, H=H, dtype=dtype, p=p)

    def dropout(name, n, H, dtype, p):
        return dict(name=name, op="dropout", n=n, H=H, dtype=dtype, p=p)
    return [
        # a handful of short trees, five classes at every node: latency alone counts
        loss("loss-request-f32", 74, 74, 150, 5, "f32", "f32"),
        # sentiment over a large batch of trees: memory-bound, states in, cotangents out
        loss("loss-sentiment-bf16", 1179358, 1179358, 512, 5, "bf16", "f32"),
        # predicting a word at every node of 256 sentences, fp32
        loss("loss-words-f32", 4608, 4608, 150, 10007, "f32", "f32"),
        # the largest vocabulary and the widest state, gradients in bf16
        loss("loss-words-bf16", 32768, 32768, 512, 50021, "bf16", "bf16"),
        # labels at the roots of 4096 trees alone, gradients in fp32
        loss("loss-roots-bf16", 105003, 4096, 256, 8192, "bf16", "f32"),
        # loss of a held-out set: no gradient; half of the nodes carry a label
        loss("eval-words-bf16", 105003, 52501, 256, 20011, "bf16", "bf16", op="eval"),
        norm("norm-request-f32", 74, 150, "f32", 0.0),
        # states of half a million-node batch, normed and dropped in one pass
        norm("norm-large-bf16", 1179358, 512, "bf16", 0.1),
        # a width that fits no vector of four
        norm("norm-odd-f32", 105003, 203, "f32", 0.0),
        dropout("dropout-request-f32", 74, 300, "f32", 0.5),
        # word vectors of a large batch
        dropout("dropout-words-bf16", 1179358, 300, "bf16", 0.25),
        # the whole way from the states to their cotangent, on the batch of 256 sentences
        dict(name="head-sentences-f32", op="head", n=4608, labelled=2304, H=150, C=2003, dtype="f32", grad="f32", p=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: one node to a million, widths 24 to 1024, two classes to sixty thousand."""
    op = rng.choice(["loss", "loss", "loss", "eval", "norm", "norm", "dropout", "head"])
    dtype = "f32" if op == "head" else rng.choice(["f32", "bf16"])
    H = rng.choice([150, 256, 512, _log_int(rng, 24, 1024), 8 * _log_int(rng, 3, 128)])
    c = dict(op=op, H=H, dtype=dtype)
    if op in ("norm", "dropout"):
        c["n"] = _log_int(rng, 1, 1000000 * 512 // max(H, 512))
        c["p"] = rng.choice([0.0, 0.1, 0.5]) if op == "norm" else round(rng.uniform(0.05, 0.9), 3)
        return c
    C = rng.choice([2, 5, _log_int(rng, 2, 200), _log_int(rng, 200, 60000), _log_int(rng, 200, 60000)])
    # a quarter of the largest listed product in bf16, a sixteenth in fp32; at most 4e8 logits
    most = (2e11 if dtype == "bf16" else 5e10) / (H * C)
    n = _log_int(rng, 1, max(2, int(min(1e6, most, 4e8 / C))))
    c.update(n=n, labelled=max(1, int(n * rng.choice([1.0, 1.0, 0.5, 0.04]))), C=C,
             grad="f32" if dtype == "f32" else rng.choice(["f32", "bf16"]))
    if op == "head":
        c["p"] = rng.choice([0.0, 0.1, 0.5])
    return c


# ---- what a program has in hand before the call ---------------------------------------------
def prepare(case, seed):
    n, H, dt = case["n"], case["H"], DTYPES[case["dtype"]][0]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    st = {"case": case, "p": case.get("p", 0.0)}
    # seed and first word of the generator
    st["state"] = torch.randint(0, 1 << 62, (2,), generator=gen, device="cuda", dtype=torch.int64)
    # node states lie in (-1, 1)
    st["x"] = torch.tanh(randn(n, H).add_(0.2 * randn(H))).to(dt)
    if case["op"] in ("norm", "head"):
        st["gamma"], st["beta"] = 1 + 0.1 * randn(H), 0.1 * randn(H)
    if case["op"] in ("norm", "dropout"):
        st["gy"] = randn(n, H).to(dt)
        return st
    C = case["C"]
    st["V"] = (randn(C, H) * (2 / math.sqrt(H))).to(dt)
    st["b"] = 0.5 * randn(C)
    label = torch.randint(0, C, (n,), generator=gen, device="cuda", dtype=torch.int32)
    without = torch.randperm(n, generator=gen, device="cuda")[case["labelled"]:]
    label[without] = -1
    st["label"] = label
    # the weight of each row in the batch's loss: a mean, leaning on some rows more than on others
    st["gloss"] = (0.5 + torch.rand(n, generator=gen, device="cuda")) / case["labelled"]
    return st


# ---- the plain forms ------------------------------------------------------------------------
def _mix(z):
    """The output function of SplitMix64 on int64 values read as 64 unsigned bits."""
    z = (z ^ ((z >> 30) & 0x3FFFFFFFF)) * -0x40A7B892E31B1A47
    z = (z ^ ((z >> 27) & 0x1FFFFFFFFF)) * -0x6B2FB644ECCEEE15
    return z ^ ((z >> 31) & 0x1FFFFFFFF)


def _plain_keep(shape, p, state):
    """Element i is kept where half i % 2 of word state[1] + i / 2 of the stream with key mix(state[0]) is at least p 2^32."""
    n = shape[0] * shape[1]
    at = torch.arange((n + 1) // 2, device=state.device) + state[1]
    word = _mix(_mix(state[:1]) + at * -0x61C8864680B583EB)
    halves = torch.stack((word & 0xFFFFFFFF, (word >> 32) & 0xFFFFFFFF), 1).reshape(-1)[:n]
    return (halves >= int(_as_f32(p) * 4294967296.0)).view(shape)


def _as_f32(p):
    return float(torch.tensor(p, dtype=torch.float32))


def _plain_dropout(x, p, state, dt):
    zero = torch.zeros((), device=x.device)
    return torch.where(_plain_keep(x.shape, p, state), x.float() * (1.0 / (1.0 - _as_f32(p))), zero).to(dt)


def _plain_norm(x, gamma, beta, p, state, dt):
    x = x.float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = torch.rsqrt((d * d).mean(1) + EPS)
    y = d * rstd[:, None] * gamma + beta
    return (_plain_dropout(y, p, state, dt) if p > 0 else y.to(dt)), mean, rstd


def _plain_norm_back(x, gamma, mean, rstd, gy, p, state):
    g = _plain_dropout(gy, p, state, torch.float32) if p > 0 else gy.float()
    xhat = (x.float() - mean[:, None]) * rstd[:, None]
    dbeta = g.sum(0, dtype=torch.float64).float()
    dgamma = (g * xhat).sum(0, dtype=torch.float64).float()
    g = g * gamma
    dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * rstd[:, None]
    return dx, dgamma, dbeta


def _plain_loss(h, V, b, label):
    rows = (label >= 0).nonzero().flatten()
    z = h[rows].float() @ V.float().t() + b
    top = z.amax(1)
    lse_r = top + (z - top[:, None]).exp_().sum(1).log()
    loss, lse = torch.zeros(label.shape, device=h.device), torch.zeros(label.shape, device=h.device)
    loss[rows] = lse_r - z.gather(1, label[rows].long()[:, None]).flatten()
    lse[rows] = lse_r
    return loss, lse


def _plain_loss_back(h, V, b, label, lse, gloss, dt):
    rows = (label >= 0).nonzero().flatten()
    hr, V32 = h[rows].float(), V.float()
    dz = (hr @ V32.t() + b).sub_(lse[rows][:, None]).exp_()
    dz[torch.arange(rows.numel(), device=h.device), label[rows].long()] -= 1
    dz *= gloss[rows][:, None]
    dh = torch.zeros(h.shape, dtype=dt, device=h.device)
    dh[rows] = (dz @ V32).to(dt)
    return dh, (dz.t() @ hr).to(dt), dz.sum(0)


def run(st):
    case, p = st["case"], st["p"]
    op, dt, gdt = case["op"], DTYPES[case["dtype"]][0], DTYPES[case.get("grad", "f32")][0]
    if own:
        import paper_1904_07421_amd as J
        drop = dict(p=p, state=st["state"]) if p > 0 else {}
        if op == "dropout":
            return {"y": J.jitdb_dropout(st["x"], p, st["state"]), "dx": J.jitdb_dropout(st["gy"], p, st["state"])}
        if op in ("norm", "head"):
            y, mean, rstd = J.jitdb_layernorm_forward(st["x"], st["gamma"], st["beta"], eps=EPS, **drop)
        if op == "norm":
            dx, dgamma, dbeta = J.jitdb_layernorm_backward(st["x"], st["gamma"], mean, rstd, st["gy"], **drop)
            return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
        h = y if op == "head" else st["x"]
        loss, lse = J.jitdb_softmax_xent_forward(h, st["V"], st["label"], b=st["b"])
        if op == "eval":
            return {"loss": loss, "lse": lse}
        dh, dV, db = J.jitdb_softmax_xent_backward(h, st["V"], st["label"], lse, b=st["b"], gloss=st["gloss"], grad_dtype=gdt)
        if op == "loss":
            return {"loss": loss, "lse": lse, "dh": dh, "dV": dV, "db": db}
        dx, dgamma, dbeta = J.jitdb_layernorm_backward(st["x"], st["gamma"], mean, rstd, dh, **drop)
        return {"loss": loss, "dx": dx, "dgamma": dgamma, "dbeta": dbeta, "dV": dV, "db": db}
    if op == "dropout":
        return {"y": _plain_dropout(st["x"], p, st["state"], dt), "dx": _plain_dropout(st["gy"], p, st["state"], dt)}
    if op in ("norm", "head"):
        y, mean, rstd = _plain_norm(st["x"], st["gamma"], st["beta"], p, st["state"], dt)
    if op == "norm":
        dx, dgamma, dbeta = _plain_norm_back(st["x"], st["gamma"], mean, rstd, st["gy"], p, st["state"])
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    h = y if op == "head" else st["x"]
    loss, lse = _plain_loss(h, st["V"], st["b"], st["label"])
    if op == "eval":
        return {"loss": loss, "lse": lse}
    dh, dV, db = _plain_loss_back(h, st["V"], st["b"], st["label"], lse, st["gloss"], gdt)
    if op == "loss":
        return {"loss": loss, "lse": lse, "dh": dh, "dV": dV, "db": db}
    dx, dgamma, dbeta = _plain_norm_back(st["x"], st["gamma"], mean, rstd, dh, p, st["state"])
    return {"loss": loss, "dx": dx, "dgamma": dgamma, "dbeta": dbeta, "dV": dV, "db": db}


# ---- the operators' definitions in 64 bits --------------------------------------------------
def _exact_kept(n, H, p, state):
    """[n, H] of truth values, from 32-bit digits of the counter: nothing here relies on how 64-bit products wrap."""
    key, first = (int(v) % 2**64 for v in state.tolist())
    M = 2**64 - 1

    def mix(z):
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M
        return z ^ (z >> 31)
    start = (mix(key) + first * 0x9E3779B97F4A7C15) & M
    mask32, limit = 0xFFFFFFFF, int(_as_f32(p) * 2.0**32)

    def cross_fixed(u, k):
        return ((u & 0xFFFF) * (k & 0xFFFF) + ((((u >> 16) * (k & 0xFFFF) + (u & 0xFFFF) * (k >> 16)) & 0xFFFF) << 16)) & mask32

    def product(hi, lo, k):
        kl, kh = k & mask32, k >> 32
        a0, a1, k0, k1 = lo & 0xFFFF, lo >> 16, kl & 0xFFFF, kl >> 16
        low = a0 * k0
        mid = (low >> 16) + a1 * k0 + a0 * k1
        out_lo = (low & 0xFFFF) | ((mid & 0xFFFF) << 16)
        return ((mid >> 16) + a1 * k1 + cross_fixed(hi, kl) + cross_fixed(lo, kh)) & mask32, out_lo

    def xor_shift(hi, lo, s):                   # z ^ (z >> s), s < 32
        return hi ^ (hi >> s), lo ^ ((lo >> s) | ((hi << (32 - s)) & mask32))
    words = (n * H + 1) // 2
    out = torch.empty(2 * words, dtype=torch.bool, device=state.device)
    for at in range(0, words, 1 << 25):
        i = torch.arange(at, min(words, at + (1 << 25)), device=state.device)
        hi, lo = product(i >> 32, i & mask32, 0x9E3779B97F4A7C15)
        lo = lo + (start & mask32)
        hi = (hi + (start >> 32) + (lo >> 32)) & mask32
        lo = lo & mask32
        hi, lo = product(*xor_shift(hi, lo, 30), 0xBF58476D1CE4E5B9)
        hi, lo = product(*xor_shift(hi, lo, 27), 0x94D049BB133111EB)
        hi, lo = xor_shift(hi, lo, 31)
        out[2 * at:2 * (at + i.numel()):2] = lo >= limit
        out[2 * at + 1:2 * (at + i.numel()):2] = hi >= limit
    return out[:n * H].view(n, H)


def exact(case, seed):
    st = prepare(case, seed)
    op, n, H, p = case["op"], case["n"], case["H"], st["p"]
    if op == "dropout":
        f = _exact_kept(n, H, p, st["state"]).double() / (1 - _as_f32(p))
        return {"y": st["x"].double() * f, "dx": st["gy"].double() * f}
    f = _exact_kept(n, H, p, st["state"]).double() / (1 - _as_f32(p)) if p > 0 else None
    x = st["x"].double()
    if op in ("norm", "head"):
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        xhat = (x - mean[:, None]) * rstd[:, None]
        y = xhat * st["gamma"].double() + st["beta"].double()
        y = y if f is None else y * f

    def norm_back(gy):
        g = gy.double() if f is None else gy.double() * f
        dxhat = g * st["gamma"].double()
        dx = rstd[:, None] / H * (H * dxhat - dxhat.sum(1, keepdim=True) - xhat * (dxhat * xhat).sum(1, keepdim=True))
        return dx, (g * xhat).sum(0), g.sum(0)
    if op == "norm":
        dx, dgamma, dbeta = norm_back(st["gy"])
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    h, V, b, label = (y if op == "head" else x), st["V"].double(), st["b"].double(), st["label"].long()
    loss, lse = (torch.zeros(n, dtype=torch.float64, device=h.device) for _ in range(2))
    dh, dV, db = torch.zeros_like(h), torch.zeros_like(V), torch.zeros_like(b)
    step = max(1, (1 << 28) // case["C"])
    for at in range(0, n, step):
        part = slice(at, at + step)
        has = label[part] >= 0
        who = label[part].clamp(min=0)[:, None]
        z = torch.addmm(b, h[part], V.t())
        lse[part] = torch.logsumexp(z, 1) * has
        loss[part] = (torch.logsumexp(z, 1) - z.gather(1, who)[:, 0]) * has
        if op != "eval":
            dz = torch.softmax(z, 1).scatter_add_(1, who, torch.full(who.shape, -1.0, dtype=torch.float64, device=h.device))
            dz *= (st["gloss"][part].double() * has)[:, None]
            dh[part] = dz @ V
            dV += dz.t() @ h[part]
            db += dz.sum(0)
    if op == "eval":
        return {"loss": loss, "lse": lse}
    if op == "loss":
        return {"loss": loss, "lse": lse, "dh": dh, "dV": dV, "db": db}
    dx, dgamma, dbeta = norm_back(dh)
    return {"loss": loss, "dx": dx, "dgamma": dgamma, "dbeta": dbeta, "dV": dV, "db": db}


def work(case):
    n, H, (_, esz) = case["n"], case["H"], DTYPES[case["dtype"]]
    op = case["op"]
    if op == "dropout":                                     # two arrays in, two out
        return {"bytes": 4.0 * n * H * esz, "flops": 0.0}
    norm = n * H * (3.0 * esz + 4.0) + 8.0 * n + 16.0 * H   # x and gy in, y and the fp32 dx out
    if op == "norm":
        return {"bytes": norm, "flops": 0.0}
    gsz, C, rows = DTYPES[case["grad"]][1], case["C"], case["labelled"]
    nbytes = rows * H * esz + C * (H * esz + 4.0) + 12.0 * n
    if op == "eval":                                        # one product of [rows, H] and [H, C]
        return {"bytes": nbytes, "flops": 2.0 * rows * H * C}
    # the gradient's two products; gradients of all rows, of the class weights and of the bias out
    nbytes += n * H * gsz + C * (H * gsz + 4.0) + 4.0 * n
    if op == "head":
        nbytes += norm
    return {"bytes": nbytes, "flops": 6.0 * rows * H * C}
