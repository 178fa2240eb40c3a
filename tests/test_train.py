"""The trainable plain network: tables and integer evaluation on the CPU, gradients and the encrypted evaluation on the device."""
import numpy as np
import pytest

from paper_1811_00778_amd import layers, network

torch = pytest.importorskip("torch")

# padded convolution, square, pooling, strided convolution, square, two fully connected layers
SPEC = (("conv", 3, 3, 3, 1, 1), ("square",), ("pool", 2), ("conv", 4, 3, 3, 2, 0), ("square",), ("fc", 7), ("fc", 5))
IN_SHAPE = (2, 8, 8)


def test_inverse_table_lists_every_reader_once():
    from paper_1811_00778_amd import train
    idx, valid, _ = layers.conv_index_table(2, 8, 8, 3, 3, 1, 1)
    idx = np.where(valid, idx, 128)
    inverse = train._inverse_table(idx, 128)
    seen = inverse[inverse < idx.size]
    assert sorted(seen) == sorted(np.nonzero(idx.reshape(-1) < 128)[0])
    for i in range(128):
        assert all(idx.reshape(-1)[p] == i for p in inverse[i] if p < idx.size)


def test_integer_scores_are_the_plain_networks():
    from paper_1811_00778_amd import train
    rng = np.random.default_rng(4)
    weights = [None if s is None else rng.integers(-3, 4, size=s).astype(np.int32) for s in network.weight_shapes(SPEC, IN_SHAPE)]
    images = rng.integers(0, 4, size=(3, 128)).astype(np.int32)
    got = train.integer_scores(SPEC, IN_SHAPE, weights, images)
    for image, row in zip(images, got):
        x = image.reshape(IN_SHAPE).astype(object)
        for layer, w in zip(SPEC, weights):
            if layer[0] == "conv":
                _, f, fh, fw, stride, pad = layer
                x = np.pad(x, ((0, 0), (pad, pad), (pad, pad)))
                h, wd = (x.shape[1] - fh) // stride + 1, (x.shape[2] - fw) // stride + 1
                x = np.array([[[(x[:, r * stride:r * stride + fh, c * stride:c * stride + fw] * w[k].astype(object)).sum() for c in range(wd)]
                               for r in range(h)] for k in range(f)], dtype=object)
            elif layer[0] == "pool":
                e = layer[1]
                x = x.reshape(x.shape[0], x.shape[1] // e, e, x.shape[2] // e, e).sum(4).sum(2)
            elif layer[0] == "square":
                x = x * x
            else:
                x = (w.astype(object) @ x.reshape(-1)).reshape(-1, 1, 1)
        assert [int(v) for v in row] == [int(v) for v in x.reshape(-1)]


def _reference(weights, x, labels):
    """Loss and weight gradients in 64 bits by torch's own differentiation."""
    F = torch.nn.functional
    ws = [None if w is None else w.double().cpu().requires_grad_() for w in weights]
    h = x.double().cpu().reshape((-1,) + IN_SHAPE)
    for layer, w in zip(SPEC, ws):
        if layer[0] == "conv":
            h = F.conv2d(h, w, stride=layer[4], padding=layer[5])
        elif layer[0] == "pool":
            h = F.avg_pool2d(h, layer[1])
        elif layer[0] == "square":
            h = h * h
        else:
            h = h.reshape(h.shape[0], -1) @ w.t()
    loss = F.cross_entropy(h, labels.cpu())
    loss.backward()
    return float(loss.detach()), [None if w is None else w.grad for w in ws]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [("f32", 1e-5), ("bf16", 0.05)])
def test_network_gradients(dtype, tol):
    """32 bits: sums of up to 10^4 terms; bfloat16: four layers' values and gradients rounded to 8 bits, about 2^-8 each"""
    from paper_1811_00778_amd import binding, train
    ctx = binding.PlainContext()
    net = train.PlainNetwork(SPEC, IN_SHAPE, ctx, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.random((33, 128))).to(ctx.device, net.dtype)
    labels = torch.from_numpy(rng.integers(0, 5, 33)).to(ctx.device)
    loss, grads = net.loss_and_gradients(x, labels)
    want, exact = _reference(net.weights, x, labels)
    assert abs(float(loss) - want) < tol * want
    for g, e in zip(grads, exact):
        assert (g is None) == (e is None)
        if g is not None:
            assert float((g.double().cpu() - e).norm()) < tol * float(e.norm())
    ctx.close()


@pytest.mark.gpu
def test_training_and_the_encrypted_evaluation():
    from paper_1811_00778_amd import binding, train
    ctx = binding.PlainContext()
    net = train.PlainNetwork(SPEC, IN_SHAPE, ctx)
    rng = np.random.default_rng(6)
    protos, state, losses = None, {}, []
    for _ in range(40):
        images, labels, protos = train.made_up_images(64, IN_SHAPE, 5, rng, 4, protos)
        loss, norm = net.train_step(torch.from_numpy(images).to(ctx.device, torch.float32) / 3, torch.from_numpy(labels).to(ctx.device), state)
        losses.append(float(loss))
        assert np.isfinite(float(norm))
    assert losses[-1] < 0.5 * losses[0]
    weights = net.integer_weights(3)
    images, _, _ = train.made_up_images(2, IN_SHAPE, 5, rng, 4, protos)
    want = train.integer_scores(SPEC, IN_SHAPE, weights, images)
    got = train.encrypted_scores(SPEC, IN_SHAPE, weights, images, n=1024, k=11)
    assert [[int(v) for v in r] for r in got] == [[int(v) for v in r] for r in want]
    ctx.close()
