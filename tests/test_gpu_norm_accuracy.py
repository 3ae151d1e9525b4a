"""Layer norm of rows that lie far from zero: what is left of an fp32 mean comes off as well."""
import numpy as np
import pytest

from oracle import head_oracle as O

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24                         # half a step of fp32, relative
WIDTHS = [3, 150, 203, 300, 513, 2048, 2049, 5000]


def _norm(x, gamma, beta, eps=1e-5):
    import torch
    import paper_1904_07421_amd as J
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()  # noqa: E731
    return [t.cpu().numpy().astype(np.float64) for t in J.jitdb_layernorm_forward(to(x), to(gamma), to(beta), eps=eps)]


def _depth(H):
    """Additions in a row of a sum of H values: at most 32 of a lane, then a tree over lanes and waves."""
    return 34 + np.ceil(np.log2(H + 1))


@pytest.mark.parametrize("H", WIDTHS)
def test_rows_of_equal_values(H):
    """mean is the value itself; x - mean is what an fp32 correction of at most depth 2^-24 |x| may itself be off by."""
    values = np.array([0.1, -0.3, 7.25, 1e-20, 30000.1, 100000.1, -3.3e6, 1e15], np.float32)
    x = np.repeat(values[:, None], H, 1)
    gamma, beta = np.full(H, 1.5), np.full(H, 0.25)
    y, mean, rstd = _norm(x, gamma, beta)
    assert np.array_equal(mean, values.astype(np.float64))
    off = ((_depth(H) + 1) * U32) ** 2 * np.abs(values.astype(np.float64))      # of the correction of the correction
    assert np.all(np.abs(y - 0.25) <= (1.5 * off / np.sqrt(1e-5))[:, None] * (1 + 1e-3) + 2 * U32)
    # the variance is 0 up to the rounding of (what was corrected)^2
    d2 = ((_depth(H) + 1) * U32 * np.abs(values.astype(np.float64))) ** 2
    assert np.all(np.abs(rstd * np.sqrt(1e-5) - 1) <= (2 * _depth(H) + 4) * U32 * d2 / 1e-5 + 4 * U32)


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("far", [0.0, 1e2, 1e4, -1e5])
def test_rows_far_from_zero(H, far):
    rng = np.random.default_rng([H, int(abs(far))])
    x = (far + rng.standard_normal((40, H))).astype(np.float32)
    gamma, beta = (rng.standard_normal(H).astype(np.float32) for _ in range(2))
    y_t, mean_t, rstd_t = _norm(x, gamma, beta)
    x = x.astype(np.float64)
    y, mean, rstd = O.layernorm(x, gamma.astype(np.float64), beta.astype(np.float64), 1e-5)
    k = _depth(H) + 2
    first = k * U32 * np.abs(x).mean(1, keepdims=True)              # what the first mean may be off by
    d = np.abs(x - mean[:, None]) + first                           # the values that are summed, corrected and scaled
    corr = k * U32 * d.mean(1, keepdims=True)                       # error of the correction: its sum, the product with 1 / H
    assert np.all(np.abs(mean_t - mean)[:, None] <= corr * (1 + U32) + U32 * np.abs(mean)[:, None])
    d_err = corr + 2 * U32 * d                                      # both differences rounded
    # squares and what comes off them, each a sum of that depth, and twice the correction's error times what it multiplies
    var_err = (2 * k * U32 * (d ** 2).mean(1, keepdims=True) + 2 * first * corr)
    rstd_rel = 0.5 * var_err * rstd[:, None] ** 2 * (1 + 1e-3) + 4 * U32
    assert np.all(np.abs(rstd_t / rstd - 1)[:, None] <= rstd_rel)
    bound = np.abs(gamma) * rstd[:, None] * (d_err + d * (rstd_rel + 3 * U32)) + 4 * U32 * (np.abs(y) + np.abs(beta))
    assert np.all(np.abs(y_t - y) <= bound)


def test_rows_that_are_not_finite():
    import torch
    import paper_1904_07421_amd as J
    x = torch.randn(4, 203, device="cuda")
    x[0, 7], x[1, 9], x[2, 11] = float("inf"), -float("inf"), float("nan")
    one = torch.ones(203, device="cuda")
    y, mean, _ = J.jitdb_layernorm_forward(x, one, one)
    assert float(mean[0]) == float("inf") and float(mean[1]) == -float("inf") and bool(mean[2].isnan())
    assert bool(y[:3].isnan().any(1).all()) and bool(y[3].isfinite().all())


@pytest.mark.parametrize("H", [150, 203, 300, 1000, 2100])
def test_a_mean_whose_sum_is_exact_is_the_quotient(H):
    """Multiples of 1 / 128 around zero: their sum has no rounding, and the rounded differences may not add one."""
    import torch
    import paper_1904_07421_amd as J
    k = torch.randint(-127, 128, (5000, H), generator=torch.Generator().manual_seed(H))
    want = (k.sum(1).double() / 128 / H).float()
    one = torch.ones(H, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        _, mean, _ = J.jitdb_layernorm_forward((k.float() / 128).to("cuda", dtype), one, one)
        assert torch.equal(mean.cpu(), want)


@pytest.mark.parametrize("n,H,lanes,chain", [(1000000, 512, 4096, 16), (4000000, 24, 16384, 16), (300000, 1030, 4096, 16), (200000, 2049, 1024, 32)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_gradients_of_many_rows_alike(n, H, lanes, chain, dtype):
    """Terms that are all alike are rounded alike: each addition loses up to half a step of the sum so far, k of them (k + 1) / 2 half
    steps of the last.  A lane adds `chain` terms, then what it has of those before; at most 16 lanes are added in a block, the blocks in fp64."""
    import torch
    import paper_1904_07421_amd as J
    print(f"weight gradients n={n} H={H} {dtype}", flush=True)
    ones = torch.ones((n, H), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    mean, rstd, gamma = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda"), torch.ones(H, device="cuda")
    second = -(-(-(-n // lanes)) // chain)
    bound = ((chain + 1) / 2 + (second + 1) / 2 + (16 + 1) / 2 + 1) * U32
    for v in (0.9869921803474426, 0.5594824552536011, 0.7893792390823364):
        gy = torch.full((n, H), v, device="cuda")
        _, dgamma, dbeta = J.jitdb_layernorm_backward(ones, gamma, mean, rstd, gy)
        want = n * float(gy[0, 0])
        for name, got in (("dgamma", dgamma), ("dbeta", dbeta)):
            off = float((got.double() / want - 1).abs().max())
            assert off <= bound, (name, v, off, bound)
        del gy


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("far", [1e2, 1e4, -1e5])
def test_gradients_of_rows_far_from_zero(H, far):
    """dx and dgamma take the centred values: the mean that the forward pass returns is rounded, by 3e-3 of the spread at 1e5."""
    import torch
    import paper_1904_07421_amd as J
    n = 40
    rng = np.random.default_rng([H, int(abs(far)), 1])
    x = (far + rng.standard_normal((n, H))).astype(np.float32)
    gy, gamma = rng.standard_normal((n, H)).astype(np.float32), rng.standard_normal(H).astype(np.float32)
    x_t, gy_t, gamma_t = (torch.from_numpy(a).cuda() for a in (x, gy, gamma))
    _, mean_t, rstd_t = J.jitdb_layernorm_forward(x_t, gamma_t, gamma_t)
    got = [t.cpu().numpy().astype(np.float64) for t in J.jitdb_layernorm_backward(x_t, gamma_t, mean_t, rstd_t, gy_t)]
    x, gy, gamma = (a.astype(np.float64) for a in (x, gy, gamma))
    dx, dgamma, dbeta = O.layernorm_backward(x, gamma, gy, 1e-5)
    _, mean, rstd = O.layernorm(x, gamma, 0.0, 1e-5)
    rstd = rstd[:, None]
    k = _depth(H) + 2
    first = k * U32 * np.abs(x).mean(1, keepdims=True)              # of the first mean, forward; the second is closer than that
    d = np.abs(x - mean[:, None]) + first
    corr = k * U32 * d.mean(1, keepdims=True)
    rstd_rel = 0.5 * (2 * k * U32 * (d ** 2).mean(1, keepdims=True) + 2 * first * corr) * rstd ** 2 * (1 + 1e-3) + 4 * U32
    xhat = (x - mean[:, None]) * rstd
    xhat_err = rstd * (corr + 3 * U32 * d) + (rstd_rel + 2 * U32) * d * rstd
    a = np.abs(gy * gamma)
    mean_a, mean_xa = a.mean(1, keepdims=True), (a * np.abs(xhat)).mean(1, keepdims=True)
    dx_err = rstd * (k * U32 * mean_a + np.abs(xhat) * (k * U32 * mean_xa + (a * xhat_err).mean(1, keepdims=True)) + xhat_err * mean_xa
                     + 6 * U32 * (a + mean_a + np.abs(xhat) * mean_xa)) + rstd_rel * np.abs(dx)
    assert np.all(np.abs(got[0] - dx) <= dx_err)
    assert np.all(np.abs(got[1] - dgamma) <= (n + 4) * U32 * np.abs(gy * xhat).sum(0) + (np.abs(gy) * xhat_err).sum(0))
    assert np.all(np.abs(got[2] - dbeta) <= (n + 4) * U32 * np.abs(gy).sum(0))


@pytest.mark.parametrize("H", [20, 60, 100, 300, 2100])
def test_a_row_does_not_depend_on_its_neighbours(H):
    import torch
    import paper_1904_07421_amd as J
    torch.manual_seed(H)
    x, gy, gamma = torch.randn(64, H, device="cuda"), torch.randn(64, H, device="cuda"), torch.randn(H, device="cuda")
    near = torch.arange(64, device="cuda") % 3 != 1
    x[~near] += 3e4
    y, mean, rstd = J.jitdb_layernorm_forward(x, gamma, gamma)
    dx = J.jitdb_layernorm_backward(x, gamma, mean, rstd, gy)[0]
    x0 = x[near].contiguous()
    y0, mean0, rstd0 = J.jitdb_layernorm_forward(x0, gamma, gamma)
    dx0 = J.jitdb_layernorm_backward(x0, gamma, mean0, rstd0, gy[near].contiguous())[0]
    for a, b in ((y, y0), (mean, mean0), (rstd, rstd0), (dx, dx0)):
        assert torch.equal(a[near], b)
