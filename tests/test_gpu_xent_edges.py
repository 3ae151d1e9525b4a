"""Softmax cross entropy where its numbers leave the ordinary range."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,C", [("f32", 8, 4096), ("f32", 160, 700), ("f32", 200, 4096), ("f32", 8, 64), ("bf16", 8, 4096), ("bf16", 512, 300),
                                       ("bf16", 600, 4096), ("bf16", 8, 33)])
def test_probabilities_far_below_one(dtype, H, C):
    """The bias' gradient of one row whose logits and log-sum-exp are known exactly is e^b itself: the exponential good to a unit in the
    last place (2^-23), a correction or a product rounded (2^-24), and what both leave out."""
    import torch
    import paper_1904_07421_amd as J
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    b = -torch.arange(C, device="cuda").float() * (86 / C)
    h, V = torch.zeros(1, H, device="cuda", dtype=dt), torch.zeros(C, H, device="cuda", dtype=dt)
    _, _, db = J.jitdb_softmax_xent_backward(h, V, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda"), b=b)
    got, want = db.double().cpu().numpy()[1:], np.exp(b.double().cpu().numpy())[1:]
    assert np.abs(got / want - 1).max() <= 2.0 ** -23 + 2.0 ** -24 + 2.0 ** -26


SHAPES = [("f32", 40, 5), ("f32", 700, 20), ("bf16", 512, 64), ("f32", 150, 1000), ("f32", 200, 400), ("bf16", 256, 1000), ("bf16", 512, 5000),
          ("bf16", 600, 400)]             # few classes, resident operands, both operands streaming


@pytest.mark.parametrize("dtype,H,C", SHAPES)
@pytest.mark.parametrize("n", [3, 300])
def test_a_logit_of_plus_infinity(n, dtype, H, C):
    """log-sum-exp is +inf, and so is the loss of every other label; a NaN beside it stays one."""
    import torch
    import paper_1904_07421_amd as J
    print(f"xent +inf n={n} H={H} C={C} {dtype}", flush=True)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    torch.manual_seed(C)
    h, V = torch.randn(n, H, device="cuda").to(dt), torch.randn(C, H, device="cuda").to(dt)
    for where in ([0], [C // 2], [C - 1], [0, 1, C - 1]):
        b = torch.randn(C, device="cuda")
        b[2] = -float("inf")
        b[where] = float("inf")
        label = torch.full((n,), 3, dtype=torch.int32, device="cuda")
        label[1] = where[0]
        loss, lse = J.jitdb_softmax_xent_forward(h, V, label, b=b)
        want = torch.full((n,), float("inf"), device="cuda")
        assert torch.equal(lse, want), where
        assert bool(loss[1].isnan()) and torch.equal(loss[[0, *range(2, n)]], want[1:])
        b[C // 3] = float("nan")
        loss, lse = J.jitdb_softmax_xent_forward(h, V, label, b=b)
        assert bool(lse.isnan().all()) and bool(loss.isnan().all())


@pytest.mark.parametrize("dtype,H,C", SHAPES)
def test_every_class_behind_minus_infinity(dtype, H, C):
    """No class is left: log-sum-exp is -inf, and the loss has no value."""
    import torch
    import paper_1904_07421_amd as J
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    h, V = torch.randn(70, H, device="cuda").to(dt), torch.randn(C, H, device="cuda").to(dt)
    label = torch.full((70,), C - 1, dtype=torch.int32, device="cuda")
    label[5] = -1
    loss, lse = J.jitdb_softmax_xent_forward(h, V, label, b=torch.full((C,), -float("inf"), device="cuda"))
    rest = torch.arange(70, device="cuda") != 5
    assert bool((lse[rest] == -float("inf")).all()) and bool(loss[rest].isnan().all()) and float(lse[5]) == float(loss[5]) == 0


@pytest.mark.parametrize("C", [20, 100, 700])
@pytest.mark.parametrize("H", [4, 150, 200])
def test_fp32_values_above_the_largest_bf16(H, C):
    """The largest fp32 values, times class weights that bring them back: logits up to 60."""
    import torch
    import paper_1904_07421_amd as J
    from oracle import head_oracle as O
    from test_gpu_xent import _f32, _host, _i32, _tolerances
    print(f"xent largest values H={H} C={C}", flush=True)
    n = 6
    rng = np.random.default_rng([H, C])
    h, V = np.zeros((n, H), np.float32), np.zeros((C, H), np.float32)
    big = (2 - 2.0 ** -23) * 2.0 ** 127
    h[:4, H // 2] = big, -big, (2 - 2.0 ** -8) * 2.0 ** 127, (2 - 2.0 ** -7) * 2.0 ** 127      # ... half a step above the largest bf16, it itself
    h[4:] = rng.uniform(-1, 1, (2, H))
    V[:, H // 2] = (np.arange(C) % 16) * 2.0 ** -126
    label, gloss = rng.integers(0, C, n), rng.uniform(0.1, 0.4, n).astype(np.float32)
    loss_t, lse_t = J.jitdb_softmax_xent_forward(_f32(h), _f32(V), _i32(label))
    dh_t, dV_t, db_t = J.jitdb_softmax_xent_backward(_f32(h), _f32(V), _i32(label), lse_t, gloss=_f32(gloss))
    h, V = h.astype(np.float64), V.astype(np.float64)
    loss, lse = O.softmax_xent(h, V, None, label)
    dh, dV, db, g, p = O.softmax_xent_backward(h, V, None, label, gloss.astype(np.float64))
    loss_err, lse_err, dh_err, dV_err, db_err, out = _tolerances(h, V, None, label, gloss, "f32", "f32", loss, lse, g, p)
    for t, want, err in ((loss_t, loss, loss_err), (lse_t, lse, lse_err), (db_t, db, db_err), (dV_t, dV, dV_err), (dh_t, dh, dh_err)):
        assert np.all(np.abs(_host(t) - want) <= err * (1 + out) + out * np.abs(want) + 1e-36)


@pytest.mark.parametrize("C", [7, 300])
def test_more_than_2_to_32_elements(C):
    """Offsets past 32 bits in states, their layouts and gradients: the last rows of a batch are what they are alone."""
    import torch
    import paper_1904_07421_amd as J
    H = 512
    n = (1 << 32) // H + 5
    print(f"xent 2^32 elements C={C}", flush=True)
    torch.manual_seed(C)
    h = torch.zeros((n, H), dtype=torch.bfloat16, device="cuda")
    h[-7:] = torch.randn(7, H, device="cuda").bfloat16()
    V, b = (torch.randn(C, H, device="cuda") / 16).bfloat16(), torch.randn(C, device="cuda")
    label = torch.full((n,), 3, dtype=torch.int32, device="cuda")
    label[-7:] = torch.randint(0, C, (7,), device="cuda", dtype=torch.int32)
    gloss = torch.zeros(n, device="cuda")
    gloss[-7:] = torch.rand(7, device="cuda") + 0.5
    loss, lse = J.jitdb_softmax_xent_forward(h, V, label, b=b)
    dh, dV, db = J.jitdb_softmax_xent_backward(h, V, label, lse, gloss=gloss, b=b)
    tail = [t[-7:].contiguous() for t in (h, label, gloss)]
    loss7, lse7 = J.jitdb_softmax_xent_forward(tail[0], V, tail[1], b=b)
    dh7, dV7, db7 = J.jitdb_softmax_xent_backward(tail[0], V, tail[1], lse7, gloss=tail[2], b=b)
    assert bool((lse[:-7] == lse[0]).all()) and bool((loss[:-7] == loss[0]).all())
    want = float(torch.logsumexp(b.double(), 0))
    # of C exponentials and their logarithm, as in the tests of sizes; the rows alone are cut into other ranges, sums in another order
    close = (C + 8) * 2.0 ** -24 + 2.0 ** -20
    assert abs(float(lse[0]) - want) <= close + 4 * 2.0 ** -24 * abs(want)
    assert float((lse[-7:] - lse7).abs().max()) <= 2 * close + 8 * 2.0 ** -24 * float(lse7.abs().max())
    assert float((loss[-7:] - loss7).abs().max()) <= 2 * close + 8 * 2.0 ** -24 * float(lse7.abs().max() + loss7.abs().max())
    assert not bool(dh[:-7].any())
    for got, ref in ((dh[-7:], dh7), (dV, dV7), (db, db7)):
        # seven rows' terms, each good to 2^-18 (exponentials and what they are taken of), as a norm
        assert float((got - ref).norm() / ref.norm()) <= 2.0 ** -17


@pytest.mark.parametrize("dtype,H,C,grad", [(*s, g) for s in SHAPES for g in ("f32", "bf16") if s[0] == "bf16" or g == "f32"])
def test_a_mask_of_the_lowest_value_is_a_mask(dtype, H, C, grad):
    """Classes behind the type's lowest value, at the front, at the end and in between: what -inf gives, bit for bit."""
    import torch
    import paper_1904_07421_amd as J
    dt, gdt = (torch.float32 if k == "f32" else torch.bfloat16 for k in (dtype, grad))
    torch.manual_seed(C + H)
    n = 130
    h, V = torch.rand(n, H, device="cuda").to(dt), (torch.randn(C, H, device="cuda") / H ** 0.5).to(dt)
    out = torch.rand(C, device="cuda") < 0.3
    out[: C // 3] = out[-C // 5:] = True
    out[C // 2] = False
    classes = (~out).nonzero().flatten()
    label = classes[torch.randint(0, len(classes), (n,), device="cuda")].int()
    got = []
    for low in (-float("inf"), torch.finfo(torch.float32).min, -1e30):
        b = torch.randn(C, generator=torch.Generator().manual_seed(1)).cuda()
        b[out] = low
        loss, lse = J.jitdb_softmax_xent_forward(h, V, label, b=b)
        got.append((loss, lse) + J.jitdb_softmax_xent_backward(h, V, label, lse, b=b, grad_dtype=gdt))
        assert all(bool(t.isfinite().all()) for t in got[-1])
    for other in got[1:]:
        assert all(torch.equal(u, v) for u, v in zip(got[0], other))


@pytest.mark.parametrize("weights", ["alike", "one row"])
@pytest.mark.parametrize("n,H,C", [(40, 150, 3000), (2000, 512, 2500), (300, 600, 3000), (1500, 256, 4099)])
def test_weights_that_are_alike_are_not_rounded(n, H, C, weights):
    """Gradients in bf16 of improbable labels (p < 2^-9, so that p - 1 rounds to -1): the label's own derivative is then off by no more
    than p of it, whatever the weight that all rows have, or the only row.  The other classes' are rounded, 2^-8 of each."""
    import torch
    import paper_1904_07421_amd as J
    from oracle import head_oracle as O
    from test_gpu_xent import _f32, _host, _i32, _to
    print(f"xent weights n={n} H={H} C={C} {weights}", flush=True)
    U32, UB = 2.0 ** -24, 2.0 ** -8
    rng = np.random.default_rng([n, H, C])
    h_t, h = _to(rng.uniform(-1, 1, (n, H)), "bf16")
    V_t, V = _to(rng.standard_normal((C, H)) * 0.2 / np.sqrt(H), "bf16")
    h, V = h.astype(np.float64), V.astype(np.float64)
    label = rng.integers(0, C, n)
    if weights == "one row":
        label[np.arange(n) != n // 2] = -1
    for w in (1.0 / 3, 0.0021019, -1.7e-5, 1.99):
        gloss = np.full(n, w, np.float32)
        _, lse = J.jitdb_softmax_xent_forward(h_t, V_t, _i32(label))
        dh_t, dV_t, db_t = J.jitdb_softmax_xent_backward(h_t, V_t, _i32(label), lse, gloss=_f32(gloss), grad_dtype=torch.bfloat16)
        dh, dV, db, g, p = O.softmax_xent_backward(h, V, None, label, gloss.astype(np.float64))
        used = label != -1
        own = np.zeros_like(p)
        own[used, label[used]] = 1
        assert (p[used, label[used]] < 2.0 ** -9).all()
        size = np.abs(h) @ np.abs(V).T
        rel = ((H + 4) * U32 * size).max() * 2 + (C + 4) * U32 + 2.0 ** -20 + 2.0 ** -22 * 16       # of a probability, as in the tests of sizes
        g_err = abs(w) * (p * (rel + UB) * (1 + own))                                                # (p - 1 to -1 is off by p)
        total = np.abs(g)
        for name, t, want, err in (("dh", dh_t, dh, g_err @ np.abs(V) + (C + 8) * U32 * (total @ np.abs(V))),
                                   ("dV", dV_t, dV, g_err.T @ np.abs(h) + (n + 8) * U32 * (total.T @ np.abs(h)))):
            own_err = abs(w) * ((own * p) @ np.abs(V) if name == "dh" else (own * p).T @ np.abs(h))
            most = (err + own_err) * (1 + UB) + UB * np.abs(want) + 1e-36
            assert np.all(np.abs(_host(t) - want) <= most), (name, w, float((np.abs(_host(t) - want) / most).max()))
        db_err = abs(w) * (p * rel).sum(0) + (n + 16) * U32 * total.sum(0)
        assert np.all(np.abs(_host(db_t) - db) <= db_err + 1e-36), w


def test_weights_of_any_size():
    """Weights of every magnitude, 0 and none that counts: as the same call with fp32 gradients, rounded."""
    import torch
    import paper_1904_07421_amd as J
    torch.manual_seed(2)
    n, H, C = 700, 60, 300
    h, V = torch.randn(n, H, device="cuda").bfloat16(), torch.randn(C, H, device="cuda").bfloat16()
    label = torch.randint(-1, C, (n,), device="cuda", dtype=torch.int32)
    for scale in (0.0, 1e-41, 1e-30, 1.0, 1e30):
        gloss = torch.randn(n, device="cuda") * scale
        gloss[::5] = 0
        _, lse = J.jitdb_softmax_xent_forward(h, V, label)
        a = J.jitdb_softmax_xent_backward(h, V, label, lse, gloss=gloss, grad_dtype=torch.bfloat16)
        b = J.jitdb_softmax_xent_backward(h, V, label, lse, gloss=gloss)
        for u, v in zip(a, b):
            # products of rounded terms and a rounded result, as a norm (below the normal range nothing is promised)
            assert float((u.double() - v.double()).norm()) <= 2.0 ** -7 * float(v.double().norm()) + 1e-34
        assert not bool(a[0][::5].any())
