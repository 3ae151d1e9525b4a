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
