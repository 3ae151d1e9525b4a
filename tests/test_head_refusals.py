"""What the calls of a training step's head refuse, before anything runs on a GPU."""
import ctypes

import numpy as np
import pytest

NULL, BADARG, WORKSPACE = -1, -2, -5


@pytest.fixture(scope="module")
def lib():
    import paper_1904_07421_amd as J
    return J.load_library()


@pytest.fixture(scope="module")
def at():
    """The address of host memory, 256-byte aligned: stands for device memory in calls that stop before using it."""
    buf = np.zeros(4096, dtype=np.uint8)
    a = (buf.ctypes.data + 255) // 256 * 256
    yield a
    del buf


def test_dropout(lib, at):
    call = lib.jitdb_dropout
    assert call(None, 0, 0, 0.5, None, None, None) == 0
    assert call(None, 4, 0, 0.5, at, at, None) == NULL
    assert call(at, 4, 0, 0.5, None, at, None) == NULL
    assert call(at, 4, 0, 0.5, at, None, None) == NULL
    for n, dtype, p in ((-1, 0, 0.5), (4, 2, 0.5), (4, 0, -0.1), (4, 0, 1.5), (4, 0, float("nan")), ((1 << 42) + 1, 0, 0.5)):
        assert call(at, n, dtype, p, at, at, None) == BADARG
    assert call(at + 2, 4, 0, 0.5, at, at, None) == BADARG
    assert call(at, 4, 1, 0.5, at, at + 1, None) == BADARG
    assert call(at, 4, 0, 0.5, at + 4, at, None) == BADARG


def test_layernorm_forward(lib, at):
    def call(x=at, gamma=at, beta=at, n=4, H=8, dtype=0, eps=1e-5, p=0.0, state=None, y=at, mean=at, rstd=at):
        return lib.jitdb_layernorm_forward(x, gamma, beta, n, H, dtype, eps, p, state, y, mean, rstd, None)
    assert call(n=0, x=None, y=None) == 0
    assert call(x=None) == call(gamma=None) == call(beta=None) == call(y=None) == call(p=0.5) == NULL
    bad = [dict(n=-1), dict(n=(1 << 28) + 1), dict(H=0), dict(H=16385), dict(dtype=5), dict(eps=-1.0), dict(eps=float("nan")),
           dict(eps=float("inf")), dict(p=2.0, state=at), dict(p=0.5, state=at + 4), dict(x=at + 1), dict(x=at + 2), dict(y=at + 1, dtype=1),
           dict(gamma=at + 2), dict(beta=at + 1), dict(mean=at + 3), dict(rstd=at + 2)]
    for b in bad:
        assert call(**b) == BADARG, b


def test_layernorm_backward(lib, at):
    import paper_1904_07421_amd as J
    need = J.jitdb_layernorm_backward_workspace_bytes(4, 8, 0)
    assert need > 0 and need % 256 == 0
    assert J.jitdb_layernorm_backward_workspace_bytes(0, 8, 0) > 0
    for n, H, dtype in ((-1, 8, 0), (4, 0, 0), (4, 16385, 0), (4, 8, 2)):
        assert J.jitdb_layernorm_backward_workspace_bytes(n, H, dtype) == 0

    def call(x=at, gamma=at, mean=at, rstd=at, gy=at, n=4, H=8, dtype=0, grad=0, p=0.0, state=None, dx=at, dgamma=at, dbeta=at, ws=at,
             size=need):
        return lib.jitdb_layernorm_backward(x, gamma, mean, rstd, gy, n, H, dtype, grad, p, state, dx, dgamma, dbeta, ws, size, None)
    for name in ("x", "gamma", "mean", "rstd", "gy", "dx", "dgamma", "dbeta", "ws"):
        assert call(**{name: None}) == NULL, name
    assert call(p=0.5) == NULL
    bad = [dict(n=-1), dict(H=0), dict(H=1 << 15), dict(dtype=-1), dict(grad=2), dict(p=-1.0), dict(x=at + 2), dict(gy=at + 2),
           dict(gy=at + 1, grad=1), dict(gamma=at + 1), dict(mean=at + 2), dict(rstd=at + 2), dict(dx=at + 2), dict(dgamma=at + 2), dict(dbeta=at + 2),
           dict(ws=at + 128), dict(p=0.5, state=at + 4)]
    for b in bad:
        assert call(**b) == BADARG, b
    assert call(size=need - 1) == WORKSPACE


def test_loss(lib, at):
    import paper_1904_07421_amd as J
    need, need_b = J.jitdb_softmax_xent_workspace_bytes(4, 8, 5, 0), J.jitdb_softmax_xent_backward_workspace_bytes(4, 8, 5, 0, 0)
    assert need > 0 and need_b > 0 and need % 256 == 0 and need_b % 256 == 0
    for n, H, C, dtype in ((-1, 8, 5, 0), ((1 << 28) + 1, 8, 5, 0), (4, 0, 5, 0), (4, 16385, 5, 0), (4, 8, 0, 0), (4, 8, (1 << 22) + 1, 0), (4, 8, 5, 3)):
        assert J.jitdb_softmax_xent_workspace_bytes(n, H, C, dtype) == 0
        assert J.jitdb_softmax_xent_backward_workspace_bytes(n, H, C, dtype, 0) == 0
    assert J.jitdb_softmax_xent_backward_workspace_bytes(4, 8, 5, J.JITDB_F32, J.JITDB_BF16) == 0
    assert J.jitdb_softmax_xent_backward_workspace_bytes(4, 8, 5, J.JITDB_BF16, J.JITDB_BF16) > 0

    def forward(h=at, V=at, b=None, label=at, n=4, H=8, C=5, dtype=0, loss=at, lse=at, ws=at, size=need):
        return lib.jitdb_softmax_xent_forward(h, V, b, label, n, H, C, dtype, loss, lse, ws, size, None)

    def backward(h=at, V=at, b=None, label=at, lse=at, gloss=None, n=4, H=8, C=5, dtype=0, grad=0, dh=at, dV=at, db=at, ws=at, size=need_b):
        return lib.jitdb_softmax_xent_backward(h, V, b, label, lse, gloss, n, H, C, dtype, grad, dh, dV, db, ws, size, None)
    assert forward(n=0, h=None) == 0
    for name in ("h", "V", "label", "loss", "lse", "ws"):
        assert forward(**{name: None}) == NULL, name
    for name in ("h", "V", "label", "lse", "dh", "dV", "db", "ws"):
        assert backward(**{name: None}) == NULL, name
    sizes = [dict(n=-1), dict(H=0), dict(H=16385), dict(C=0), dict(C=(1 << 22) + 1), dict(dtype=2)]
    for b in sizes + [dict(h=at + 2), dict(V=at + 1, dtype=1), dict(b=at + 2), dict(label=at + 2), dict(loss=at + 1), dict(lse=at + 2), dict(ws=at + 64)]:
        assert forward(**b) == BADARG, b
    for b in sizes + [dict(grad=1), dict(grad=2), dict(h=at + 2), dict(V=at + 2), dict(b=at + 1), dict(label=at + 1), dict(lse=at + 2), dict(gloss=at + 2),
                      dict(dh=at + 2), dict(dV=at + 2), dict(db=at + 2), dict(ws=at + 8)]:
        assert backward(**b) == BADARG, b
    assert forward(size=need - 1) == WORKSPACE and backward(size=need_b - 1) == WORKSPACE


def test_the_binding_refuses_what_is_not_on_a_gpu():
    import torch
    import paper_1904_07421_amd as J
    x, v, state = torch.zeros(4, 8), torch.zeros(8), torch.zeros(2, dtype=torch.int64)
    label = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: J.jitdb_dropout(x, 0.5, state), lambda: J.jitdb_layernorm_forward(x, v, v),
                 lambda: J.jitdb_layernorm_backward(x, v, v[:4], v[:4], x), lambda: J.jitdb_softmax_xent_forward(x, x, label),
                 lambda: J.jitdb_softmax_xent_backward(x, x, label, v[:4])):
        with pytest.raises(TypeError, match="CUDA"):
            call()
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        J.jitdb_dropout(x.half(), 0.5, state)
