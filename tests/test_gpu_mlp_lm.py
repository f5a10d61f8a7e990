"""The training step that runs the row operators, the compressed linears and the vocabulary cross entropy together."""
import pytest
import torch

from paper_2605_01255_b200 import binding as B
from paper_2605_01255_b200 import mlp_lm as M

pytestmark = pytest.mark.gpu


def _reference(model, h0, y):
    """Loss and gradients of the same network by autograd in float64."""
    s, dbl = model.s, torch.float64
    leaf = lambda t: t.detach().to(dbl).requires_grad_()  # noqa: E731
    p = {"h0": leaf(h0), "head": leaf(model.head), "w_pre": [leaf(t) for t in model.w_pre], "w_post": [leaf(t) for t in model.w_post],
         "gate": [leaf(t) for t in model.gate], "gu": [leaf(w["gu"]) for w in model.w], "dn": [leaf(w["dn"]) for w in model.w]}
    norm = lambda x, w: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s.eps) * w  # noqa: E731
    h, x = p["h0"], norm(p["h0"], p["w_pre"][0])
    for l in range(s.layers):
        g, u = (x @ p["gu"][l].T).split(s.inter, dim=1)
        b = (g * torch.sigmoid(g) * u) @ p["dn"][l].T
        h = h + s.alpha * p["gate"][l] * norm(b, p["w_post"][l])
        x = norm(h, p["w_pre"][l + 1])
    loss = torch.nn.functional.cross_entropy(x @ p["head"].T, y, ignore_index=-100)
    loss.backward()
    return loss, p


def _rel(a, b):
    return float((a.to(torch.float64) - b).norm() / b.norm())


def test_step_against_autograd():
    s = M.Sizes(tokens=333, d=136, inter=264, vocab=1003, layers=2, r=32, alpha=0.8)
    model = M.MlpLm(s)
    h0, y = M.synthetic_batch(s)
    total = model.forward(h0, y)
    dh0 = model.backward()
    assert B.acx_last_device_status() == B.ACX_OK
    loss, p = _reference(model, h0, y)
    # bf16 storage of every activation and gradient between the calls: 2^-9 each, some ten of them in a row, random: under
    # 1e-2; the 8-bit checkpoints: a step of max / 127 with max about 3.5 rms, 0.8 % of the rms each, four per layer: 2.5e-2
    assert abs(float(total[0] / total[1]) - float(loss.detach())) <= 1e-2 * float(loss.detach())
    tol = 4e-2
    assert _rel(dh0, p["h0"].grad) <= tol
    assert _rel(model.grads["head"][0], p["head"].grad) <= tol
    for k in ("w_pre", "w_post", "gate"):
        for a, b in zip(model.grads[k], p[k]):
            assert _rel(a, b.grad) <= tol, k


def test_training_lowers_the_loss_and_keeps_less_than_half():
    s = M.Sizes(tokens=512, d=256, inter=512, vocab=999, layers=2, r=64)
    model = M.MlpLm(s)
    h0, y = M.synthetic_batch(s)
    losses = []
    for _ in range(40):
        t = model.forward(h0, y)
        losses.append(float(t[0] / t[1]))
        model.backward(lr=2e-3)
    assert B.acx_last_device_status() == B.ACX_OK
    assert losses[-1] < 0.8 * losses[0], losses
    kept = model.kept_bytes()
    assert kept["kept"] < 0.5 * kept["bf16"]
