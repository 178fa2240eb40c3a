"""Steps of the trainable plain network whose gradients are not finite, and its gradients in binary16."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_train import IN_SHAPE, SPEC, _reference


class _Clip:
    """PlainContext's clip_grad_norm by its formula, on the CPU"""
    device = "cpu"

    def clip_grad_norm(self, grads, max_norm, eps=1e-6):
        norm = sum(g.double().square().sum() for g in grads).sqrt()
        for g in grads:
            g.mul_(torch.clamp(max_norm / (norm + eps), max=1.0))
        return norm.float()


def _network(ctx, dtype=torch.float32):
    from paper_1811_00778_amd import train
    return train.PlainNetwork(SPEC, IN_SHAPE, ctx, dtype)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_step_without_a_finite_norm_changes_nothing(bad):
    net, state = _network(_Clip()), {}
    g = torch.Generator().manual_seed(3)
    grads = [None if w is None else torch.randn(w.shape, generator=g) for w in net.weights]

    def step(poison, scale=8.0):
        given = [None if v is None else v.clone() * scale for v in grads]
        if poison is not None:
            given[0].view(-1)[5] = poison
        net.loss_and_gradients = lambda x, labels, s: (torch.tensor(1.0), given)
        return net.train_step(None, None, state, scale=scale)

    def held():
        return [v.clone() for v in [w for w in net.weights if w is not None] + state.get("moments", []) + state.get("master", [])]

    first = [w.clone() for w in net.weights if w is not None]
    assert not np.isfinite(float(step(bad)[1]))                # also as the first step of all
    assert all(torch.equal(a, b) for a, b in zip(first, held()))
    assert np.isfinite(float(step(None)[1]))
    before = held()
    assert not any(torch.equal(a, b) for a, b in zip(first, before))
    _, norm = step(bad)
    assert not np.isfinite(float(norm))
    assert all(torch.equal(a, b) for a, b in zip(before, held()))
    step(None)
    assert all(bool(torch.isfinite(v).all()) for v in held()) and not torch.equal(before[0], held()[0])


@pytest.mark.gpu
def test_network_gradients_in_binary16():
    """the loss times 1024; four layers' values and gradients rounded to 11 bits, about 2^-11 each"""
    from paper_1811_00778_amd import binding
    ctx = binding.PlainContext()
    net = _network(ctx, torch.float16)
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.random((33, 128))).to(ctx.device, net.dtype)
    labels = torch.from_numpy(rng.integers(0, 5, 33)).to(ctx.device)
    loss, grads = net.loss_and_gradients(x, labels, scale=1024.0)
    want, exact = _reference(net.weights, x, labels)
    assert abs(float(loss) - want) < 0.01 * want
    for g, e in zip(grads, exact):
        assert (g is None) == (e is None)
        if g is not None:
            assert float((g.double().cpu() / 1024 - e).norm()) < 0.01 * float(e.norm())
    ctx.close()


@pytest.mark.gpu
def test_a_step_that_overflows_leaves_the_weights():
    """a loss scale at which binary16 gradients overflow, then one at which they do not"""
    from paper_1811_00778_amd import binding
    ctx = binding.PlainContext()
    net, state = _network(ctx, torch.float16), {}
    rng = np.random.default_rng(6)
    x = torch.from_numpy(rng.random((33, 128))).to(ctx.device, net.dtype)
    labels = torch.from_numpy(rng.integers(0, 5, 33)).to(ctx.device)
    before = [w.clone() for w in net.weights if w is not None]
    _, norm = net.train_step(x, labels, state, scale=2.0 ** 30)
    assert not np.isfinite(float(norm))
    assert all(torch.equal(a, b) for a, b in zip(before, [w for w in net.weights if w is not None]))
    _, norm = net.train_step(x, labels, state, scale=64.0)
    assert np.isfinite(float(norm))
    for a, b in zip(before, [w for w in net.weights if w is not None]):
        assert bool(torch.isfinite(b).all()) and not torch.equal(a, b)
    ctx.close()
