"""The plain network's answer from weights of four bits, layer by layer: what each product takes and gives."""
import numpy as np
import pytest

import plain_cases as pc
import plain_rows_cases as rc

torch = pytest.importorskip("torch")

from test_train import IN_SHAPE, SPEC


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("format", ["mx4", "mx8"])
def test_each_layer(format, dtype):
    """the inputs' and weights' codes are those of the definition, byte by byte, and the outputs the sums of their products, of 32 bits and rounded once"""
    from paper_1811_00778_amd import binding, train
    ctx = binding.PlainContext()
    kind = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    net = train.PlainNetwork(SPEC, IN_SHAPE, ctx, kind, seed=3)
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.random((33, 128))).to(ctx.device, kind)
    weights, seen = net.few_bit_weights(), []
    calls = {"quantize_mx": ctx.quantize_mx, "linear_mx": ctx.linear_mx}

    def quantize_mx(rows, form):
        m = calls["quantize_mx"](rows, form)
        seen.append([rows, m])
        return m

    def linear_mx(m, w, **more):
        y = calls["linear_mx"](m, w, **more)
        seen[-1] += [w, more["activation"], y]
        return y

    ctx.quantize_mx, ctx.linear_mx = quantize_mx, linear_mx
    scores = net.few_bit_scores(x, weights, format)
    values = lambda a: a.double().cpu().numpy()                                  # noqa: E731
    layers = [i for i, w in enumerate(net.weights) if w is not None]
    assert len(seen) == len(layers) and scores is seen[-1][-1]
    assert seen[0][0].shape[0] % 33 == 0 and seen[0][0].dtype == kind
    for i, (rows, m, w, act, y) in zip(layers, seen):
        assert w is weights[i] and m.format == format and w.format == "mx4"
        held = []
        for of, got in ((rows, m), (net.weights[i].reshape(net.weights[i].shape[0], -1), w)):
            code, scale, v = rc.quantize(values(of), got.format)
            rc.same_codes(rc.unpacked(got.codes.cpu().numpy(), got.format), code, got.format, "layer %d" % i)
            assert np.array_equal(got.scales.cpu().numpy(), scale)
            held.append(v)
        Z = held[0] @ held[1].T
        dz = (held[0].shape[1] + 4) * pc.E * (np.abs(held[0]) @ np.abs(held[1]).T)
        Y, _ = pc.act(Z, act)
        err = (2 * np.abs(Z) + dz) * dz if act == "square" else dz
        pc.within(values(y), Y, pc.U[dtype] * np.abs(Y) + err + 2 * pc.E * np.abs(Y) + pc.LEAST[dtype], "layer %d" % i)
    del ctx.quantize_mx, ctx.linear_mx
    ctx.close()
