"""What the layer norm calls refuse beside the cases of test_gpu_layer_norm.py."""
import pytest
import torch

import paper_2204_08211_b200 as co3
from paper_2204_08211_b200.session import Co3Session

pytestmark = pytest.mark.gpu


def test_session_refuses_layers_of_another_width():
    """A longer layer under a wrong index is no gain or bias of these rows."""
    sess = Co3Session([12, 12, 30, 5], [(4, 3, 0, 1.0, 1.0)] * 4, 1, 0.9)
    params = torch.ones(sess.n_elem, device="cuda")
    x = torch.randn(4, 12, device="cuda")
    y = torch.full_like(x, 7.0)
    for gain, bias in ((2, 1), (0, 2), (3, 1), (0, 3)):
        with pytest.raises(ValueError):
            sess.layer_norm(x, params, gain, bias, y)
    with pytest.raises(ValueError):
        sess.layer_norm(x[0], params, 0, 1, y[0])
    torch.cuda.synchronize()
    assert (y == 7.0).all()
    sess.layer_norm(x, params, 0, 1, y)
    torch.cuda.synchronize()
    want = torch.nn.functional.layer_norm(x.double(), (12,)) + 1.0
    assert (y.double() - want).abs().max() <= 1e-5          # twelve fp32 terms a sum, values of a few units


@pytest.mark.parametrize("stride", [-1, -64, -128, -2 ** 40])
def test_backward_refuses_negative_client_strides(stride):
    """They would pass the library's check as very large unsigned ones and place client 1 before the tensor."""
    x = torch.randn(4, 64, device="cuda")
    stats, w, dx = torch.ones(4, device="cuda"), torch.ones(64, device="cuda"), torch.full_like(x, 7.0)
    g = torch.full((512,), 7.0, device="cuda")
    ws = torch.empty(co3.co3_layer_norm_workspace_bytes(2, 64, 2), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        co3.co3_layer_norm_backward(x, x, w, stats, stats, dx, g[256:], g[320:], 2, stride, ws)
    torch.cuda.synchronize()
    assert (g == 7.0).all() and (dx == 7.0).all()
