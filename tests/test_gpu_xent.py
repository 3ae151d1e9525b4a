"""Softmax cross entropy and its gradients against the fp64 oracle."""
import numpy as np
import pytest

from gpu_util import bf16_tensor
from oracle import head_oracle as O

pytestmark = pytest.mark.gpu

U32, UB = 2.0 ** -24, 2.0 ** -8          # half a step of fp32 and bf16, relative


def _to(a, dtype):
    import torch
    a = np.ascontiguousarray(a, dtype=np.float32)
    return bf16_tensor(a) if dtype == "bf16" else (torch.from_numpy(a).cuda(), a)


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _f32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def _labels(kind, n, C, rng):
    label = rng.integers(0, C, n)
    if kind == "half":
        label[rng.random(n) < 0.5] = -1
    elif kind == "none":
        label[:] = -1
    elif kind == "last":
        label[:-1] = -1
    elif kind == "few":
        label[rng.random(n) < 0.96] = -1
    return label


def _tolerances(h, V, b, label, gloss, grad, dtype, loss, lse, g, p):
    """Bounds on the errors of loss and lse [N], dh, dV, db of an fp32 computation on exact inputs."""
    H, C, N = h.shape[1], V.shape[0], h.shape[0]
    bias = np.zeros(C) if b is None else np.where(np.isfinite(b), np.abs(b), 0)
    size = np.abs(h) @ np.abs(V).T + bias                    # sum of |terms| of every logit
    # H products of one rounding each (fp32 operands: what the parts leave out, 2^-23), H sums in any order, the bias
    z_err = ((H + 4) * U32 + (2.0 ** -23 if dtype == "f32" else 0)) * size
    seen = p > 0                                             # classes behind -inf have no error
    worst = np.where(seen, z_err, 0).max(1)
    # sums of C exponentials, each good to 2^-21 + 2^-23 |argument| relative; exp is at most 1, so arguments under -32 do not count
    lse_err = worst + (C + 4) * U32 + 2.0 ** -21 + 2.0 ** -23 * 32 + 4 * U32 * np.abs(lse)
    loss_err = lse_err + worst + 4 * U32 * np.abs(loss)
    rel_p = z_err + lse_err[:, None] + 2.0 ** -21 + 2.0 ** -22 * np.where(seen, -np.log(np.where(seen, p, 1)), 0)
    w = np.abs(gloss)[:, None] * (label != -1)[:, None]
    parts = U32 if grad == "f32" else UB
    onehot = np.zeros_like(p)
    onehot[np.arange(N), np.maximum(label, 0)] = 1
    g_err = w * (p * rel_p + 2 * U32 * (p + onehot)) + parts * np.abs(g)
    extra = 2.0 ** -22 if dtype == "f32" else 0              # parts left out of a product of fp32 operands
    out = UB if grad == "bf16" else U32
    dh = g_err @ np.abs(V) + ((C + 8) * U32 + extra) * (np.abs(g) @ np.abs(V))
    dV = g_err.T @ np.abs(h) + ((N + 8) * U32 + extra) * (np.abs(g).T @ np.abs(h))
    db = (g_err - parts * np.abs(g)).sum(0) + (N + 8) * U32 * np.abs(g).sum(0)
    return loss_err, lse_err, dh, dV, db, out


def _check(n, H, C, dtype, grad, kind="all", bias="random", scale=1.0):
    import torch
    import paper_1904_07421_amd as J
    print(f"xent n={n} H={H} C={C} {dtype}/{grad} labels={kind} bias={bias}", flush=True)
    rng = np.random.default_rng([n, H, C])
    h_t, h = _to(rng.uniform(-1, 1, (n, H)), dtype)
    V_t, V = _to(rng.standard_normal((C, H)) * scale * 2 / np.sqrt(H), dtype)
    label = _labels(kind, n, C, rng)
    h, V = h.astype(np.float64), V.astype(np.float64)
    b = None if bias == "none" else rng.standard_normal(C).astype(np.float32)
    if bias == "masked":
        b[rng.random(C) < 0.5] = -np.inf
        b[label[label >= 0]] = 0.25
    b_t = None if b is None else _f32(b)
    gloss = (rng.random(n) + 0.5).astype(np.float32)
    loss_t, lse_t = J.jitdb_softmax_xent_forward(h_t, V_t, _i32(label), b=b_t)
    gdt = torch.float32 if grad == "f32" else torch.bfloat16
    got = J.jitdb_softmax_xent_backward(h_t, V_t, _i32(label), lse_t, gloss=_f32(gloss), b=b_t, grad_dtype=gdt)
    again = J.jitdb_softmax_xent_backward(h_t, V_t, _i32(label), lse_t, gloss=_f32(gloss), b=b_t, grad_dtype=gdt)
    assert all(torch.equal(u, v) for u, v in zip(got, again))
    b64 = None if b is None else b.astype(np.float64)
    loss, lse = O.softmax_xent(h, V, b64, label)
    dh, dV, db, g, p = O.softmax_xent_backward(h, V, b64, label, gloss.astype(np.float64))
    loss_err, lse_err, dh_err, dV_err, db_err, out = _tolerances(h, V, b, label, gloss, grad, dtype, loss, lse, g, p)
    used = label != -1
    assert np.all(np.abs(_host(lse_t) - lse) <= np.where(used, lse_err, 0))
    assert np.all(np.abs(_host(loss_t) - loss) <= np.where(used, loss_err, 0))
    dh_t, dV_t, db_t = got
    assert dh_t.dtype == dV_t.dtype == gdt and db_t.dtype == torch.float32
    tiny = 1e-36                                             # below the range of normal values nothing is promised
    for name, t, want, err in (("dh", dh_t, dh, dh_err), ("dV", dV_t, dV, dV_err), ("db", db_t, db, db_err)):
        o = U32 if name == "db" else out
        diff, bound = np.abs(_host(t) - want), err * (1 + o) + o * np.abs(want) + tiny
        assert np.all(diff <= bound), (name, float((diff / bound).max()))
    assert not bool(dh_t[torch.from_numpy(~used).cuda()].any())


KINDS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")]


@pytest.mark.parametrize("dtype,grad", KINDS)
@pytest.mark.parametrize("n,H,C", [(1, 1, 1), (1, 8, 2), (3, 5, 7), (74, 150, 5), (1, 300, 1000), (256, 64, 128), (257, 65, 129), (300, 256, 1000),
                                   (1025, 99, 31), (600, 512, 2500), (2, 1030, 300), (70, 2050, 65), (4097, 24, 2), (130, 33, 4099)])
def test_sizes(n, H, C, dtype, grad):
    _check(n, H, C, dtype, grad)


@pytest.mark.parametrize("dtype,grad", KINDS)
@pytest.mark.parametrize("kind", ["half", "none", "last", "few"])
@pytest.mark.parametrize("n,H,C", [(700, 150, 5), (9000, 40, 70), (515, 96, 700)])
def test_rows_without_a_label(n, H, C, kind, dtype, grad):
    _check(n, H, C, dtype, grad, kind=kind)


@pytest.mark.parametrize("dtype,grad", KINDS)
@pytest.mark.parametrize("bias", ["none", "masked"])
@pytest.mark.parametrize("n,H,C", [(100, 50, 6), (300, 70, 900)])
def test_bias(n, H, C, bias, dtype, grad):
    _check(n, H, C, dtype, grad, bias=bias)


@pytest.mark.parametrize("dtype,grad", KINDS)
def test_large_logits(dtype, grad):
    """Logits of hundreds: exp alone would leave the range of fp32."""
    _check(200, 64, 500, dtype, grad, scale=120.0)
    _check(200, 64, 9, dtype, grad, scale=120.0)


@pytest.mark.parametrize("C", [5, 300])
def test_labels_that_name_no_class_and_rows_that_are_not_finite(C):
    import torch
    import paper_1904_07421_amd as J
    n, H = 600, 40
    rng = np.random.default_rng(5)
    h, V, label = _f32(rng.standard_normal((n, H))), _f32(rng.standard_normal((C, H))), rng.integers(0, C, n)
    good = J.jitdb_softmax_xent_forward(h, V, _i32(label))
    good_b = J.jitdb_softmax_xent_backward(h, V, _i32(label), good[1])
    for bad in (C, C + 7, -2, 2 ** 31 - 1, -2 ** 31):
        wrong = label.copy()
        wrong[17] = bad
        loss, lse = J.jitdb_softmax_xent_forward(h, V, _i32(wrong))
        dh, dV, db = J.jitdb_softmax_xent_backward(h, V, _i32(wrong), lse)
        rest = torch.arange(n, device="cuda") != 17
        assert bool(loss[17].isnan()) and torch.equal(loss[rest], good[0][rest]) and torch.equal(lse, good[1])
        assert bool(dh[17].isnan().all()) and torch.equal(dh[rest], good_b[0][rest])
        assert bool(dV.isnan().all()) and bool(db.isnan().all())
    # what a row without a label holds does not matter
    unlabelled = label.copy()
    unlabelled[[3, 255, 256, 599]] = -1
    dirty = h.clone()
    dirty[[3, 256]] = float("nan")
    dirty[[255, 599]] = float("inf")
    lab = _i32(unlabelled)
    clean_f, dirty_f = J.jitdb_softmax_xent_forward(h, V, lab), J.jitdb_softmax_xent_forward(dirty, V, lab)
    assert all(torch.equal(u, v) for u, v in zip(clean_f, dirty_f))
    clean_b, dirty_b = (J.jitdb_softmax_xent_backward(x, V, lab, clean_f[1]) for x in (h, dirty))
    assert all(torch.equal(u, v) for u, v in zip(clean_b, dirty_b))
    # a row that is not finite and has a label: its own loss and gradient are NaN, the other rows' are what they were
    one = h.clone()
    one[44, 3] = float("nan")
    loss, lse = J.jitdb_softmax_xent_forward(one, V, _i32(label))
    dh = J.jitdb_softmax_xent_backward(one, V, _i32(label), lse)[0]
    rest = torch.arange(n, device="cuda") != 44
    assert bool(loss[44].isnan()) and torch.equal(loss[rest], good[0][rest]) and torch.equal(dh[rest], good_b[0][rest])


@pytest.mark.parametrize("C", [4, 200])
def test_every_class_but_one_behind_minus_infinity(C):
    import torch
    import paper_1904_07421_amd as J
    n, H = 300, 33
    h, V = torch.randn(n, H, device="cuda"), torch.randn(C, H, device="cuda")
    b = torch.full((C,), -float("inf"), device="cuda")
    b[2] = 0.5
    label = torch.full((n,), 2, dtype=torch.int32, device="cuda")
    loss, lse = J.jitdb_softmax_xent_forward(h, V, label, b=b)
    z = (h.double() @ V[2].double() + 0.5)
    assert float((lse.double() - z).abs().max()) <= (H + 8) * U32 * float((h.abs() @ V[2].abs()).max() + 1)
    assert float(loss.abs().max()) <= 2 * (H + 8) * U32 * float((h.abs() @ V[2].abs()).max() + 1)
    dh, dV, db = J.jitdb_softmax_xent_backward(h, V, label, lse, b=b)
    assert not bool(dV[b == -float("inf")].any()) and not bool(db[b == -float("inf")].any())
    label[5] = 0                                             # a label behind -inf: the loss is infinite
    loss = J.jitdb_softmax_xent_forward(h, V, label, b=b)[0]
    assert float(loss[5]) == float("inf") and bool(loss[torch.arange(n, device="cuda") != 5].isfinite().all())


def test_gloss_of_none_is_ones():
    import torch
    import paper_1904_07421_amd as J
    h, V = torch.randn(90, 20, device="cuda"), torch.randn(40, 20, device="cuda")
    label = torch.randint(0, 40, (90,), dtype=torch.int32, device="cuda")
    _, lse = J.jitdb_softmax_xent_forward(h, V, label)
    a = J.jitdb_softmax_xent_backward(h, V, label, lse)
    b = J.jitdb_softmax_xent_backward(h, V, label, lse, gloss=torch.ones(90, device="cuda"), b=torch.zeros(40, device="cuda"))
    assert all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("dtype,grad", KINDS)
@pytest.mark.parametrize("C", [6, 150])
def test_views_that_start_anywhere_and_rows_behind_the_last(C, dtype, grad):
    import torch
    import paper_1904_07421_amd as J
    n, H = 67, 45
    dt, gdt = (torch.float32 if k == "f32" else torch.bfloat16 for k in (dtype, grad))
    h, V = torch.randn(n, H, device="cuda").to(dt), torch.randn(C, H, device="cuda").to(dt)
    label = torch.randint(-1, C, (n,), dtype=torch.int32, device="cuda")
    b, gloss = torch.randn(C, device="cuda"), torch.rand(n, device="cuda")

    def view(values, off):
        buf = torch.full((values.numel() + 40,), 9, dtype=values.dtype, device="cuda")
        v = buf[off:off + values.numel()].view(values.shape)
        v.copy_(values)
        return buf, v
    want = J.jitdb_softmax_xent_forward(h, V, label, b=b)
    want_b = J.jitdb_softmax_xent_backward(h, V, label, want[1], gloss=gloss, b=b, grad_dtype=gdt)
    for off in (1, 3):
        hv, Vv, lv, bv, gv = (view(t, off)[1] for t in (h, V, label, b, gloss))
        bufs = [view(torch.zeros_like(t), off) for t in (*want, *want_b)]
        outs = [v for _, v in bufs]
        J.jitdb_softmax_xent_forward(hv, Vv, lv, b=bv, out=tuple(outs[:2]))
        J.jitdb_softmax_xent_backward(hv, Vv, lv, outs[1], gloss=gv, b=bv, grad_dtype=gdt, out=tuple(outs[2:]))
        for (buf, got), ref in zip(bufs, (*want, *want_b)):
            assert torch.equal(got, ref)
            assert bool((buf[:off] == 9).all()) and bool((buf[off + ref.numel():] == 9).all())


def _reference(h, V, b, label, gloss, step=2048):
    """The same in fp64 on the GPU, a few rows at a time."""
    import torch
    h, V, b = h.double(), V.double(), b.double()
    loss, lse, dh, dV, db = torch.zeros_like(h[:, 0]), torch.zeros_like(h[:, 0]), torch.zeros_like(h), torch.zeros_like(V), torch.zeros_like(b)
    for at in range(0, len(label), step):
        rows = at + (label[at:at + step] >= 0).nonzero().flatten()
        z = h[rows] @ V.t() + b
        lse[rows] = torch.logsumexp(z, 1)
        who = label[rows].long()[:, None]
        loss[rows] = lse[rows] - z.gather(1, who)[:, 0]
        g = torch.softmax(z, 1)
        g.scatter_add_(1, who, torch.full(who.shape, -1.0, dtype=torch.float64, device="cuda"))
        g *= gloss[rows].double()[:, None]
        dh[rows] = g @ V
        dV += g.t() @ h[rows]
        db += g.sum(0)
    return loss, lse, dh, dV, db


# norm-wise bounds: fp32 values within 1e-5 (sums of 50 000 terms of random sign), bf16 within a rounding of operands and result
@pytest.mark.parametrize("dtype,grad,n,H,C,share", [
    ("f32", "f32", 20000, 40, 50021, 1.0),       # more rows than one chunk of the backward pass holds
    ("bf16", "bf16", 90112, 32, 50021, 0.97),    # ... than one chunk of the forward pass
    ("bf16", "f32", 30000, 64, 50021, 0.5),
    ("bf16", "f32", 300000, 256, 3, 1.0),
    ("f32", "f32", 200003, 150, 5, 0.9),
    ("bf16", "bf16", 150001, 99, 33, 0.6),
    ("f32", "f32", 70000, 64, 200, 0.02)])
def test_large(dtype, grad, n, H, C, share):
    import torch
    import paper_1904_07421_amd as J
    print(f"xent large n={n} H={H} C={C} {dtype}/{grad}", flush=True)
    dt, gdt = (torch.float32 if k == "f32" else torch.bfloat16 for k in (dtype, grad))
    torch.manual_seed(n)
    h, V = (torch.rand(n, H, device="cuda") * 2 - 1).to(dt), (torch.randn(C, H, device="cuda") * 2 / H ** 0.5).to(dt)
    b, gloss = torch.randn(C, device="cuda"), (torch.rand(n, device="cuda") + 0.5) / n
    label = torch.randint(0, C, (n,), dtype=torch.int32, device="cuda")
    label[torch.rand(n, device="cuda") >= share] = -1
    loss, lse = J.jitdb_softmax_xent_forward(h, V, label, b=b)
    got = (loss, lse) + J.jitdb_softmax_xent_backward(h, V, label, lse, gloss=gloss, b=b, grad_dtype=gdt)
    want = _reference(h, V, b, label, gloss)
    for name, a, w in zip(("loss", "lse", "dh", "dV", "db"), got, want):
        rel = float((a.double() - w).norm() / w.norm())
        assert rel <= (2 * UB if a.dtype == torch.bfloat16 else 1e-5), (name, rel)


def test_no_rows():
    import torch
    import paper_1904_07421_amd as J
    h, V, label = torch.empty((0, 30), device="cuda"), torch.ones(7, 30, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    loss, lse = J.jitdb_softmax_xent_forward(h, V, label)
    dh, dV, db = J.jitdb_softmax_xent_backward(h, V, label, lse)
    assert loss.shape == (0,) and dh.shape == (0, 30) and not bool(dV.any()) and not bool(db.any())


@pytest.mark.parametrize("C", [5, 300])
def test_on_another_stream_and_in_a_graph(C):
    """A captured loss and gradient, replayed with other labels (and another number of them), eager work in between."""
    import torch
    import paper_1904_07421_amd as J
    n, H = 900, 60
    h, V, b = torch.randn(n, H, device="cuda"), torch.randn(C, H, device="cuda"), torch.randn(C, device="cuda")
    label, gloss = torch.randint(-1, C, (n,), dtype=torch.int32, device="cuda"), torch.rand(n, device="cuda")

    def both(**kw):
        loss, lse = J.jitdb_softmax_xent_forward(h, V, label, b=b, **kw)
        return (loss, lse) + J.jitdb_softmax_xent_backward(h, V, label, lse, gloss=gloss, b=b, **kw)
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(stream=side)
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both()
    for k in range(4):
        h.copy_(torch.randn(n, H, device="cuda"))
        label.copy_(torch.randint(-1, C, (n,), device="cuda"))
        label[torch.rand(n, device="cuda") < 0.3 * k] = -1
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        assert all(torch.equal(u, v) for u, v in zip(got, both())), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_whole_training_step(dtype):
    """Forest -> states -> norm and dropout -> loss, and back to the gradients of the cell's weights, against the oracles."""
    import torch
    import paper_1904_07421_amd as J
    from oracle import treelstm_backward_oracle as B
    from gpu_util import dev_parent
    from workloads import make_workload
    _, parent, x, W, U, b = make_workload(1, bias="random")
    n, H, C = len(parent), U.shape[1], 11
    rng = np.random.default_rng(8)
    (x_t, x), (W_t, W), (U_t, U) = (_to(a, dtype) for a in (x, W, U))
    V_t, V = _to(rng.standard_normal((C, H)) * 0.3, dtype)
    gamma, beta, bias = (rng.standard_normal(k).astype(np.float32) for k in (H, H, C))
    label = rng.integers(-1, C, n)
    state = torch.tensor([3, 4], device="cuda")
    sched = J.jitdb_schedule(dev_parent(parent))
    h_t, c_t, gates, fgate = J.jitdb_treelstm_forward_train(x_t, W_t, U_t, _f32(b), sched)
    y_t, mean, rstd = J.jitdb_layernorm_forward(h_t, _f32(gamma), _f32(beta), p=0.2, state=state)
    loss_t, lse = J.jitdb_softmax_xent_forward(y_t, V_t, _i32(label), b=_f32(bias))
    gy, dV, db = J.jitdb_softmax_xent_backward(y_t, V_t, _i32(label), lse, b=_f32(bias))
    gh, dgamma, dbeta = J.jitdb_layernorm_backward(h_t, _f32(gamma), mean, rstd, gy, p=0.2, state=state)
    dx, dW, dU, d_bias = J.jitdb_treelstm_backward(x_t, W_t, U_t, sched, h_t, c_t, gates, fgate, gh)
    f = O.dropout(np.ones((n, H)), 0.2, 3, 4)
    h = _host(h_t)                                           # the states as they are; the cell has tests of its own
    y = O.layernorm(h, gamma.astype(np.float64), beta.astype(np.float64), 1e-5)[0] * f
    loss = O.softmax_xent(y, V, bias.astype(np.float64), label)[0]
    dy, dV64, db64, _, _ = O.softmax_xent_backward(y, V, bias.astype(np.float64), label, np.ones(n))
    gh64, dgamma64, dbeta64 = O.layernorm_backward(h, gamma.astype(np.float64), dy * f, 1e-5)
    # fp32 throughout: sums of a few hundred terms; bf16: y is rounded to 2^-8 (2^-8 / sqrt 3 as a norm) in front of the loss
    tol = 2e-5 if dtype == "f32" else 2.0 ** -7
    for name, got, want in (("loss", loss_t, loss), ("dV", dV, dV64), ("db", db, db64), ("dgamma", dgamma, dgamma64), ("dbeta", dbeta, dbeta64), ("gh", gh, gh64)):
        rel = np.linalg.norm(_host(got) - want) / np.linalg.norm(want)
        assert rel <= tol, (name, rel)
    _, _, *want = B.forward_backward(parent, x, W, U, b, _host(gh), np.zeros((n, H)))
    tol = 1e-4 if dtype == "f32" else 3e-2                   # the tree's own backward pass: its tests hold it tighter
    for name, got, ref in zip(("dx", "dW", "dU", "db"), (dx, dW, dU, d_bias), want):
        rel = np.linalg.norm(_host(got) - ref) / np.linalg.norm(ref)
        assert rel <= tol, (name, rel)


@pytest.mark.parametrize("dtype,grad", KINDS)
@pytest.mark.parametrize("H", [129, 160, 161, 300, 320, 321, 450])
def test_widths_around_the_tiles_of_160_features(H, dtype, grad):
    _check(70, H, 300, dtype, grad)


@pytest.mark.parametrize("dtype,grad", KINDS)
@pytest.mark.parametrize("H,C,first", [(150, 40, 20), (64, 500, 300), (150, 300, 40), (600, 500, 300)])
def test_first_classes_masked_and_the_others_far_below_zero(H, C, first, dtype, grad):
    """exp of the logits themselves is 0 in fp32: only a reference among the classes that count finds their sum."""
    import torch
    import paper_1904_07421_amd as J
    print(f"xent H={H} C={C} {first} masked {dtype}/{grad}", flush=True)
    n = 67
    rng = np.random.default_rng([H, C, first])
    h_t, h = _to(rng.uniform(-1, 1, (n, H)), dtype)
    V_t, V = _to(rng.standard_normal((C, H)) / np.sqrt(H), dtype)
    label = rng.integers(first, C, n)
    b = np.full(C, -200.0, np.float32)
    b[:first] = -np.inf
    h, V = h.astype(np.float64), V.astype(np.float64)
    loss_t, lse_t = J.jitdb_softmax_xent_forward(h_t, V_t, _i32(label), b=_f32(b))
    got = J.jitdb_softmax_xent_backward(h_t, V_t, _i32(label), lse_t, b=_f32(b), grad_dtype=torch.float32 if grad == "f32" else torch.bfloat16)
    gloss = np.ones(n)
    loss, lse = O.softmax_xent(h, V, b.astype(np.float64), label)
    dh, dV, db, g, p = O.softmax_xent_backward(h, V, b.astype(np.float64), label, gloss)
    loss_err, lse_err, dh_err, dV_err, db_err, out = _tolerances(h, V, b, label, gloss, grad, dtype, loss, lse, g, p)
    assert np.all(np.abs(_host(lse_t) - lse) <= lse_err)
    assert np.all(np.abs(_host(loss_t) - loss) <= loss_err)
    for name, t, want, err in zip(("dh", "dV", "db"), got, (dh, dV, db), (dh_err, dV_err, db_err)):
        o = U32 if name == "db" else out
        assert np.all(np.abs(_host(t) - want) <= err * (1 + o) + o * np.abs(want) + 1e-36), name
