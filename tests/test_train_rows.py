"""The trainable plain network with dropout before its last layer, and its answer from weights of four bits."""
import numpy as np
import pytest

import plain_rows_cases as rc

torch = pytest.importorskip("torch")

from test_train import IN_SHAPE, SPEC


def _network(ctx, **more):
    from paper_1811_00778_amd import train
    return train.PlainNetwork(SPEC, IN_SHAPE, ctx, torch.float32, seed=3, **more)


def _inputs(net):
    rng = np.random.default_rng(5)
    return torch.from_numpy(rng.random((33, 128))).to(net.ctx.device, net.dtype), torch.from_numpy(rng.integers(0, 5, 33)).to(net.ctx.device)


def _forward(x, ws, mask=None, round_weights=lambda w: w, round_rows=lambda r: r):
    """The network in 64 bits by torch; round_weights, round_rows: what the products' operands pass through"""
    F = torch.nn.functional
    h = x.double().cpu().reshape((-1,) + IN_SHAPE)
    for i, (layer, w) in enumerate(zip(SPEC, ws)):
        if layer[0] == "conv":
            rows = F.unfold(h, layer[2:4], stride=layer[4], padding=layer[5])                    # [B][terms][placements]
            side = (h.shape[2] + 2 * layer[5] - layer[2]) // layer[4] + 1
            flat = round_rows(rows.transpose(1, 2).reshape(-1, rows.shape[1]))
            y = (flat @ round_weights(w.reshape(w.shape[0], -1)).t()).reshape(rows.shape[0], -1, w.shape[0])
            h = y.transpose(1, 2).reshape(rows.shape[0], w.shape[0], side, side)
        elif layer[0] == "pool":
            h = F.avg_pool2d(h, layer[1])
        elif layer[0] == "square":
            h = h * h
        else:
            h = h.reshape(h.shape[0], -1)
            if mask is not None and i == len(SPEC) - 1:
                h = h * mask
            h = round_rows(h) @ round_weights(w).t()
    return h


@pytest.mark.gpu
def test_gradients_with_dropout():
    """32 bits: sums of up to 10^4 terms; the mask is that of the step"""
    from paper_1811_00778_amd import binding
    ctx = binding.PlainContext()
    net = _network(ctx, dropout=0.4)
    x, labels = _inputs(net)
    for step in (0, 1):
        net.steps = step
        loss, grads = net.loss_and_gradients(x, labels)
        ws = [None if w is None else w.double().cpu().requires_grad_() for w in net.weights]
        mask = torch.from_numpy(rc.kept(33, 7, 0.4, 3, step) / 0.6)
        want = torch.nn.functional.cross_entropy(_forward(x, ws, mask), labels.cpu())
        want.backward()
        assert abs(float(loss) - float(want.detach())) < 1e-5 * float(want.detach())
        for g, w in zip(grads, ws):
            if w is not None:
                assert float((g.double().cpu() - w.grad).norm()) < 1e-5 * float(w.grad.norm())
    before = net.steps
    net.train_step(x, labels, {})
    assert net.steps == before + 1
    ctx.close()


@pytest.mark.gpu
def test_no_dropout_by_default():
    from paper_1811_00778_amd import binding
    ctx = binding.PlainContext()
    net, same = _network(ctx), _network(ctx, dropout=0.0)
    x, labels = _inputs(net)
    a, b = net.loss_and_gradients(x, labels), same.loss_and_gradients(x, labels)
    assert torch.equal(a[0], b[0]) and all((g is None) == (f is None) and (g is None or torch.equal(g, f)) for g, f in zip(a[1], b[1]))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("format", ["mx4", "mx8"])
def test_few_bit_scores(format):
    """against the network in 64 bits whose products take the formats' numbers: rounded rows may differ by a step where 32-bit sums in front of them lie next to a border, so that
    rows of the first layer, which are the inputs', are compared exactly and the scores to a few steps' share"""
    from paper_1811_00778_amd import binding
    ctx = binding.PlainContext()
    net = _network(ctx)
    x, _ = _inputs(net)
    got = net.few_bit_scores(x, net.few_bit_weights(), format).double().cpu()

    def rounded(form):
        return lambda v: torch.from_numpy(rc.quantize(v.numpy(), form)[2][:, :v.shape[1]].copy())

    want = _forward(x, [None if w is None else w.double().cpu() for w in net.weights], None, rounded("mx4"), rounded(format))
    # a number next to a border moves by a step, 2^-1 or 2^-3 of itself; one in ten thousand does, in each of four layers
    step = 2.0 ** -1 if format == "mx4" else 2.0 ** -3
    assert float((got - want).norm()) < step * (4 * 1e-4) ** 0.5 * 4 * float(want.norm())
    ctx.close()
