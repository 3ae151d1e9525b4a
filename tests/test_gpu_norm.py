"""Layer norm and dropout against the fp64 oracle."""
import numpy as np
import pytest

from gpu_util import bf16_tensor
from oracle import head_oracle as O

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24                         # half a step of fp32, relative
HALF = {"f32": U32, "bf16": 2.0 ** -8}   # of a stored value


def _to(a, dtype):
    """(CUDA tensor, the same values in fp32)."""
    import torch
    a = np.ascontiguousarray(a, dtype=np.float32)
    return bf16_tensor(a) if dtype == "bf16" else (torch.from_numpy(a).cuda(), a)


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _state(seed, first):
    import torch
    return torch.from_numpy(np.array([seed, first], dtype=np.uint64).view(np.int64)).cuda()


def _norm_bounds(x, gamma, beta, H):
    """Errors of mean, rstd (relative) and xhat of an fp32 computation: sums of H terms in trees no deeper than H."""
    depth = 2 + np.ceil(np.log2(H)) + 32                    # pieces of at most 32 in a row, then a tree over lanes
    mean_err = depth * U32 * np.abs(x).mean(1)
    _, mean, rstd = O.layernorm(x, gamma, beta, 1e-5)
    d = np.abs(x - mean[:, None])
    # a centred value is off by the mean's error and a rounding; the variance by twice that times the mean |d|, and its own sum
    d_err = mean_err[:, None] + U32 * (np.abs(x) + d)
    var_err = (2 * d * d_err).mean(1) + depth * U32 * (d ** 2).mean(1)
    rstd_rel = 0.5 * var_err * rstd ** 2 + 4 * U32
    xhat_err = rstd[:, None] * d_err + (rstd_rel[:, None] + 2 * U32) * d * rstd[:, None]
    return mean_err, rstd_rel, xhat_err


# one row, one column, widths off every vector, on both sides of each variant's limit, the longest
SHAPES = [(1, 1), (1, 2), (3, 5), (74, 150), (33, 64), (17, 129), (257, 203), (64, 256), (40, 512), (9, 513), (7, 1030), (5, 2048), (6, 2049),
          (2, 4100), (3, 16384)]


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n,H", SHAPES)
def test_layernorm_and_its_backward(n, H, dtype, grad, p):
    import torch
    import paper_1904_07421_amd as J
    print(f"layernorm n={n} H={H} {dtype}/{grad} p={p}", flush=True)
    rng = np.random.default_rng([n, H, 3])
    x_t, x = _to(rng.standard_normal((n, H)) + 3 * rng.standard_normal((n, 1)), dtype)
    gy_t, gy = _to(rng.standard_normal((n, H)), grad)
    gamma, beta = (rng.standard_normal(H).astype(np.float32) for _ in range(2))
    gamma_t, beta_t = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    drop = dict(p=p, state=_state(2 ** 63 + 11, 2 ** 64 - 5)) if p else {}
    y_t, mean_t, rstd_t = J.jitdb_layernorm_forward(x_t, gamma_t, beta_t, **drop)
    got = J.jitdb_layernorm_backward(x_t, gamma_t, mean_t, rstd_t, gy_t, **drop)
    again = J.jitdb_layernorm_backward(x_t, gamma_t, mean_t, rstd_t, gy_t, **drop)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    f = O.dropout(np.ones((n, H)), p, 2 ** 63 + 11, 2 ** 64 - 5) if p else np.ones((n, H))
    x, gy = x.astype(np.float64), gy.astype(np.float64)
    y, mean, rstd = O.layernorm(x, gamma.astype(np.float64), beta.astype(np.float64), 1e-5)
    mean_err, rstd_rel, xhat_err = _norm_bounds(x, gamma, beta, H)
    assert np.all(np.abs(_host(mean_t) - mean) <= mean_err + U32 * np.abs(mean))
    assert np.all(np.abs(_host(rstd_t) / rstd - 1) <= rstd_rel + U32)
    y_err = f * (np.abs(gamma) * xhat_err + 4 * U32 * (np.abs(y) + np.abs(beta)))
    assert np.all(np.abs(_host(y_t) - y * f) <= y_err + HALF[dtype] * np.abs(y * f) + 1e-30)
    g = gy * f
    dx, dgamma, dbeta = O.layernorm_backward(x, gamma.astype(np.float64), g, 1e-5)
    xhat = (x - mean[:, None]) * rstd[:, None]
    a = np.abs(g * gamma)
    depth = (2 + np.ceil(np.log2(H)) + 32) * U32
    mean_xa = (a * np.abs(xhat)).mean(1, keepdims=True)
    dx_err = rstd[:, None] * (depth * a.mean(1, keepdims=True) + np.abs(xhat) * (depth * mean_xa + (a * xhat_err).mean(1, keepdims=True))
                              + xhat_err * mean_xa + 6 * U32 * (a + a.mean(1, keepdims=True) + np.abs(xhat) * mean_xa)) + rstd_rel[:, None] * np.abs(dx)
    dx_t, dgamma_t, dbeta_t = got
    assert np.all(np.abs(_host(dx_t) - dx) <= dx_err + 1e-30)
    sums = (n + 4) * U32                                    # n terms in any order
    assert np.all(np.abs(_host(dgamma_t) - dgamma) <= sums * np.abs(g * xhat).sum(0) + (np.abs(g) * xhat_err).sum(0) + 1e-30)
    assert np.all(np.abs(_host(dbeta_t) - dbeta) <= sums * np.abs(g).sum(0) + 1e-30)


def test_many_rows_add_to_the_weight_gradients():
    """More rows than the backward pass has blocks, so that every block loops; no rounding: small whole numbers."""
    import torch
    import paper_1904_07421_amd as J
    for n, H in ((70001, 24), (20011, 130), (5003, 2050)):
        print(f"many rows n={n} H={H}", flush=True)
        gy = torch.randint(-2, 3, (n, H), device="cuda").float()
        x = torch.randint(-2, 3, (n, H), device="cuda").float()
        mean, rstd, gamma = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda"), torch.ones(H, device="cuda")
        _, dgamma, dbeta = J.jitdb_layernorm_backward(x, gamma, mean, rstd, gy)
        assert torch.equal(dbeta, gy.sum(0, dtype=torch.float64).float())
        assert torch.equal(dgamma, (gy * x).sum(0, dtype=torch.float64).float())


def test_rows_of_equal_values_and_rows_that_are_not_finite():
    import torch
    import paper_1904_07421_amd as J
    x = torch.randn(6, 300, device="cuda")
    x[1] = 7.25
    x[2, 5] = float("inf")
    x[3, 299] = float("nan")
    gamma, beta = torch.ones(300, device="cuda"), torch.full((300,), 0.5, device="cuda")
    y, mean, rstd = J.jitdb_layernorm_forward(x, gamma, beta)
    assert torch.equal(y[1], beta) and float(rstd[1]) == pytest.approx(1e-5 ** -0.5, rel=1e-6)
    assert bool(y[2].isnan().any()) and bool(y[3].isnan().all())
    clean = J.jitdb_layernorm_forward(x[[0, 1, 4, 5]].contiguous(), gamma, beta)[0]
    assert torch.equal(y[[0, 1, 4, 5]], clean)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.25, 0.9, 1.0])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 4095, 100003])
def test_dropout(n, p, dtype):
    import torch
    import paper_1904_07421_amd as J
    print(f"dropout n={n} p={p} {dtype}", flush=True)
    rng = np.random.default_rng(n)
    x_t, x = _to(rng.standard_normal(n), dtype)
    y_t = J.jitdb_dropout(x_t, p, _state(n, 2 ** 64 - 3))
    want = O.dropout(x, p, n, 2 ** 64 - 3)
    got = _host(y_t)
    assert np.array_equal(got == 0, want == 0)
    # the scale is rounded twice, the product once, the stored value once
    assert np.all(np.abs(got - want) <= (3 * U32 + HALF[dtype] * (p > 0)) * np.abs(want))
    if p == 0.0:
        assert torch.equal(y_t, x_t)
    in_place = x_t.clone()
    J.jitdb_dropout(in_place, p, _state(n, 2 ** 64 - 3), out=in_place)
    assert torch.equal(in_place, y_t)


def test_dropped_elements_are_zero_whatever_they_were():
    import torch
    import paper_1904_07421_amd as J
    x = torch.full((1000,), float("inf"), device="cuda")
    x[::2] = float("nan")
    y = J.jitdb_dropout(x, 0.5, _state(1, 0))
    keep = torch.from_numpy(O.kept(1000, 0.5, 1, 0)).cuda()
    assert bool((y[~keep] == 0).all()) and bool((~y[keep].isfinite()).all())
    assert bool((J.jitdb_dropout(x, 1.0, _state(1, 0)) == 0).all())


def test_layernorm_drops_what_dropout_drops():
    import torch
    import paper_1904_07421_amd as J
    x = torch.randn(37, 203, device="cuda")
    gamma, beta, st = torch.randn(203, device="cuda"), torch.randn(203, device="cuda"), _state(99, 12)
    plain, _, _ = J.jitdb_layernorm_forward(x, gamma, beta)
    fused, mean, rstd = J.jitdb_layernorm_forward(x, gamma, beta, p=0.4, state=st)
    assert torch.equal(fused, J.jitdb_dropout(plain, 0.4, st))
    gy = torch.randn(37, 203, device="cuda")
    a = J.jitdb_layernorm_backward(x, gamma, mean, rstd, gy, p=0.4, state=st)
    b = J.jitdb_layernorm_backward(x, gamma, mean, rstd, J.jitdb_dropout(gy, 0.4, st))
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    y = x.clone()
    J.jitdb_layernorm_forward(y, gamma, beta, out=(y, mean, rstd))
    assert torch.equal(y, plain)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_that_start_anywhere_and_rows_behind_the_last(dtype):
    """Tensors that start on any element of a buffer; nothing outside them is written."""
    import torch
    import paper_1904_07421_amd as J
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    n, H = 13, 75
    for off in (1, 3):
        def view(values, t=dt):
            buf = torch.full((values.numel() + 40,), 9.0, dtype=t, device="cuda")
            v = buf[off:off + values.numel()].view(values.shape)
            v.copy_(values)
            return buf, v
        x, gy = torch.randn(n, H, device="cuda").to(dt), torch.randn(n, H, device="cuda").to(dt)
        gamma, beta, st = torch.randn(H, device="cuda"), torch.randn(H, device="cuda"), _state(5, 6)
        drop = dict(p=0.2, state=st)
        want = J.jitdb_layernorm_forward(x, gamma, beta, **drop)
        want_b = J.jitdb_layernorm_backward(x, gamma, want[1], want[2], gy, **drop)
        (yb, y), (db, d) = view(torch.zeros(n, H)), view(torch.zeros(n, H), torch.float32)
        (mb, m), (rb, r), (gb, dg), (bb, dbt) = (view(torch.zeros(k), torch.float32) for k in (n, n, H, H))
        xv, gv, gav, bev = view(x)[1], view(gy)[1], view(gamma, torch.float32)[1], view(beta, torch.float32)[1]
        J.jitdb_layernorm_forward(xv, gav, bev, out=(y, m, r), **drop)
        J.jitdb_layernorm_backward(xv, gav, m, r, gv, out=(d, dg, dbt), **drop)
        for buf, got, ref in ((yb, y, want[0]), (mb, m, want[1]), (rb, r, want[2]), (db, d, want_b[0]), (gb, dg, want_b[1]), (bb, dbt, want_b[2])):
            assert torch.equal(got, ref)
            assert bool((buf[:off] == 9).all()) and bool((buf[off + ref.numel():] == 9).all())
        zb, z = view(torch.zeros(n, H))
        J.jitdb_dropout(xv, 0.2, st, out=z)
        assert torch.equal(z, J.jitdb_dropout(x, 0.2, st))
        assert bool((zb[:off] == 9).all()) and bool((zb[off + n * H:] == 9).all())


def test_more_than_2_to_32_elements():
    """Offsets past 32 bits: the last rows of a batch of 2^32 + elements equal those of a short one."""
    import torch
    import paper_1904_07421_amd as J
    H = 512
    n = (1 << 32) // H + 5
    x = torch.zeros((n, H), dtype=torch.bfloat16, device="cuda")
    x[-7:] = torch.randn(7, H, device="cuda").bfloat16()
    gamma, beta = torch.randn(H, device="cuda"), torch.randn(H, device="cuda")
    y, mean, rstd = J.jitdb_layernorm_forward(x, gamma, beta)
    y7, mean7, rstd7 = J.jitdb_layernorm_forward(x[-7:].contiguous(), gamma, beta)
    assert torch.equal(y[-7:], y7) and torch.equal(mean[-7:], mean7) and torch.equal(rstd[-7:], rstd7)
    assert torch.equal(y[0], beta.bfloat16()) and torch.equal(y[n // 2], beta.bfloat16())
    del y
    dx, dgamma, _ = J.jitdb_layernorm_backward(x, gamma, mean, rstd, x)
    dx7, dgamma7, _ = J.jitdb_layernorm_backward(x[-7:].contiguous(), gamma, mean7, rstd7, x[-7:].contiguous())
    assert torch.equal(dx[-7:], dx7) and not bool(dx[:-7].any())
    # the other rows add zeros: seven terms in another order
    assert float((dgamma - dgamma7).abs().max()) <= 14 * U32 * float((x[-7:].float() ** 2).sum(0).max()) * float(rstd7.max()) * 4
    del dx
    st = _state(4, 5)
    z = J.jitdb_dropout(x, 0.5, st)
    first = 5 + (n - 7) * H // 2
    assert torch.equal(z[-7:], J.jitdb_dropout(x[-7:].contiguous(), 0.5, _state(4, first)))


def test_no_rows():
    import torch
    import paper_1904_07421_amd as J
    x, gamma = torch.empty((0, 30), device="cuda"), torch.ones(30, device="cuda")
    y, mean, rstd = J.jitdb_layernorm_forward(x, gamma, gamma)
    dx, dgamma, dbeta = J.jitdb_layernorm_backward(x, gamma, mean, rstd, y)
    assert y.shape == (0, 30) and dx.shape == (0, 30)
    assert not bool(dgamma.any()) and not bool(dbeta.any())
    assert J.jitdb_dropout(x, 0.5, _state(1, 1)).numel() == 0


def test_on_another_stream_and_in_a_graph():
    """A captured forward and backward pass, replayed with other inputs and another state, with eager work in between."""
    import torch
    import paper_1904_07421_amd as J
    n, H = 501, 150
    x, gy = torch.randn(n, H, device="cuda"), torch.randn(n, H, device="cuda")
    gamma, beta, st = torch.randn(H, device="cuda"), torch.randn(H, device="cuda"), _state(1, 2)

    def both(x, gy, st):
        y, mean, rstd = J.jitdb_layernorm_forward(x, gamma, beta, p=0.3, state=st)
        return (J.jitdb_dropout(y, 0.3, st), y, mean, rstd) + J.jitdb_layernorm_backward(x, gamma, mean, rstd, gy, p=0.3, state=st)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2 = J.jitdb_layernorm_forward(x, gamma, beta, p=0.3, state=st, stream=side)[0]
    side.synchronize()
    assert torch.equal(y2, both(x, gy, st)[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both(x, gy, st)
    for k in range(4):
        x.copy_(torch.randn(n, H, device="cuda"))
        gy.copy_(torch.randn(n, H, device="cuda"))
        st.copy_(_state(k, 7 * k))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        assert all(torch.equal(a, b) for a, b in zip(got, both(x, gy, st))), k
