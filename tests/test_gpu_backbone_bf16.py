"""The small network on decoded batches in bfloat16, the type it trains in: its gradients against automatic differentiation of its formula in 64 bits."""
import pytest
import torch

from paper_2306_16699_amd import backbone, rinr_nn as nn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_backbone_gradients_in_16_bits(dtype):
    """The formula takes the rounded weights and patches that the products take.  What differs: the 8 bits of what is kept (2e-2 of a gradient in the 32-bit test)
    and roundings to 16 bits, some twelve along the longest path, each at most half a unit (2^-8 in bfloat16) of a value, that is 2^-9 on average."""
    torch.manual_seed(1)
    net = backbone.Backbone(7, 96, 160, 2, 5, dtype=dtype, seed=4)
    images, d = torch.rand(6, 3, 28, 21, device="cuda"), torch.randn(6, 5, device="cuda").to(dtype).float()
    scores, tape = net.forward(images, keep=True)
    got = net.backward(tape, d)
    p = {k: (net.weights[k] if k in net.weights else v).double().requires_grad_() for k, v in net.params.items()}

    def norm(h, gain):
        return gain * h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6)

    def eight_bits(v):
        held = nn.unpack8(nn.pack8(v.detach().float()), torch.float32).double()
        return v + (held - v).detach()

    h = net.patches(images).double() @ p["w_in"].t() + p["b_in"]
    for k in range(2):
        z = eight_bits(norm(h, p[f"gain{k}"])) @ p[f"w1_{k}"].t() + p[f"b1_{k}"]
        h = h + torch.nn.functional.gelu(z) @ p[f"w2_{k}"].t() + p[f"b2_{k}"]
    want = norm(h, p["gain_out"]).view(6, -1, 96).mean(1) @ p["w_out"].t() + p["b_out"]
    (want * d.double()).sum().backward()
    rounding = 12 * torch.finfo(dtype).eps / 4
    assert float((scores.double() - want.detach()).norm() / want.detach().norm()) < 2e-3 + rounding
    assert set(got) == set(p)
    for k, v in got.items():
        off = float((v.double() - p[k].grad).norm() / p[k].grad.norm())
        assert off < 2e-2 + rounding, (k, off)
