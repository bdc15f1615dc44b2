"""The example that runs group norm, gradient norm, AdamW and log-probabilities together: its gradients against a plain network in fp32 on the
CPU, and its training."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2112_10065_amd import train_gn
    assert torch.cuda.is_available()
    return train_gn


def reference(net, x, labels):
    """Loss and gradients of the same network by elementary torch operations, fp32 on the CPU, from the bf16 weights, with activations that are
    rounded to bf16 where the network stores them (which decides pooling's ties)."""
    F = torch.nn.functional
    r = lambda v: v + (v.to(torch.bfloat16).float() - v).detach()   # noqa: E731
    leaf = [p["view"].detach().cpu().clone() for p in net.params]
    for p, l in zip(net.params, leaf):
        if l.dim() > 1:
            l.copy_(p["w_bf16"].float().cpu().view(l.shape))
        l.requires_grad_(True)
    w1, g1, b1, w2, g2, b2, w3, b3 = leaf

    def norm(u, g, b):   # [n, c, h, w]
        n, c, h, w = u.shape
        v = u.reshape(n, 8, -1)
        v = (v - v.mean(dim=2, keepdim=True)) / torch.sqrt(v.var(dim=2, unbiased=False, keepdim=True) + 1e-5)
        return v.view(n, c, h, w) * g.view(1, -1, 1, 1) + b.view(1, -1, 1, 1)

    v = x.float().cpu().permute(0, 3, 1, 2)
    v = F.max_pool2d(r(torch.relu(norm(r(F.conv2d(v, w1.permute(0, 3, 1, 2), padding=1)), g1, b1))), 2)
    u = norm(r(F.conv2d(v, w2.permute(0, 3, 1, 2), padding=1)), g2, b2)
    v = F.max_pool2d(r(u * torch.sigmoid(u)), 2).permute(0, 2, 3, 1).reshape(len(x), -1)
    z = r(v @ w3.t() + b3)
    loss = -(z.log_softmax(dim=1)[torch.arange(len(x)), labels.long().cpu()]).mean()
    loss.backward()
    return loss.item(), [l.grad.view(-1).numpy() for l in leaf], z.detach().numpy()


@pytest.mark.parametrize("state", [0, 1], ids=["f32", "q8"])
def test_gradients_of_the_whole_step(G, state):
    """bf16 gradients between the layers, and sums in another order ahead of each rounding: 2^-9 relative, eight layers deep, and a rounding can
    move a pooling maximum: a few per cent of a gradient's norm."""
    net = G.GroupNormNet(8, 12, state)
    x, labels = G.Patterns(12).batch(8)
    net.x.copy_(x)
    loss, grads, z = reference(net, x, labels)
    old = [p["w32"].clone() for p in net.params]
    net.train_step(labels)
    torch.cuda.synchronize()
    assert abs(float(net.loss[0]) - loss) <= 0.02 * abs(loss)
    for p, g in zip(net.params, grads):
        got = p["grad"].cpu().numpy()
        assert np.linalg.norm(got - g) <= 0.08 * np.linalg.norm(g)
    norm = np.sqrt(sum((p["grad"].double() ** 2).sum().item() for p in net.params))
    assert abs(float(net.norm[0]) - norm) <= 1e-5 * norm
    # the first step moves a weight by about lr, against its gradient, decay apart
    for p, w in zip(net.params, old):
        moved = (p["w32"] - w * (1 - net.lr * p["weight_decay"])).cpu()
        big = p["grad"].abs().cpu() > 1e-4
        assert torch.all(torch.sign(moved[big]) == -torch.sign(p["grad"].cpu()[big])) and float(moved.abs().max()) <= 1.01 * net.lr
        assert torch.equal(p["w_bf16"], p["w32"].to(torch.bfloat16))
    net.evaluate(labels)
    logq = net.z.float().log_softmax(dim=1)
    assert torch.allclose(net.logp, logq[torch.arange(8), labels.long()], atol=1e-4)
    assert torch.allclose(net.entropy, -(logq.exp() * logq).sum(dim=1), atol=1e-4)


@pytest.mark.parametrize("state", ["f32", "q8"])
def test_it_learns(G, state, capsys):
    got = G.main(["--steps", "80", "--batch", "16", "--classes", "20", "--state", state])
    assert got["top1"] >= 0.9 and got["top5"] >= 0.98 and got["loss"] < 0.5   # chance: 0.05, 0.25, 3.0
    assert '"top1"' in capsys.readouterr().out


def test_a_gradient_that_is_not_finite_skips_the_step(G):
    net = G.GroupNormNet(4, 10)
    x, labels = G.Patterns(10).batch(4)
    net.x.copy_(x)
    net.x[1, 5, 5, 0] = float("nan")
    before = [p["w32"].clone() for p in net.params]
    net.train_step(labels)
    torch.cuda.synchronize()
    assert float(net.norm[1]) == 0.0
    assert all(torch.equal(p["w32"], w) and not p["m"].any() for p, w in zip(net.params, before))
