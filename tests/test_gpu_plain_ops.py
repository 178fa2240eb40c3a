"""The training operators on the device: the CPU checker's cases and larger ones against 64-bit definitions, pieces and offsets
beyond 32 bits, streams and graphs, the same bits on every call."""
import numpy as np
import pytest

import plain_cases as pc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class Backend:
    def __init__(self):
        from paper_1811_00778_amd import binding
        self.ctx = binding.PlainContext()

    def make(self, a, dtype, strides=None):
        v = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(_DT[dtype]).cuda()
        if strides is None or v.dim() != 2:
            return v
        gap, shift = strides
        big = torch.full((shift + v.shape[0] * (v.shape[1] + gap),), float("nan"), dtype=v.dtype, device="cuda")
        view = big[shift:].as_strided(v.shape, (v.shape[1] + gap, 1))
        view.copy_(v)
        return view

    def ints(self, a, dtype):
        return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()

    def values(self, a):
        return a.double().cpu().numpy()


@pytest.fixture(scope="module")
def b():
    return Backend()


def say(*a):
    print("[plain]", *a, flush=True)


@pytest.mark.parametrize("case", pc.LINEAR + pc.LINEAR_LARGE, ids=str)
def test_linear(b, case):
    say("linear", case)
    pc.check_linear(b, *case)


@pytest.mark.parametrize("case", pc.GRAD + pc.GRAD_LARGE, ids=str)
def test_linear_grad(b, case):
    say("linear_grad", case)
    pc.check_grad(b, *case)


@pytest.mark.parametrize("case", pc.LOSS + pc.LOSS_LARGE, ids=str)
def test_cross_entropy(b, case):
    say("cross_entropy", case)
    pc.check_loss(b, *case)
    pc.check_loss(b, *case, wide=False, seed=1, junk=case[3] < 1000 and case[4] > 0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strides_and_alignment(b, dtype):
    for shape in ((37, 41, 19), (500, 300, 1100)):
        say("strides", dtype, shape)
        pc.check_linear(b, dtype, *shape, "silu", residual=True, keep=True, strides=(3, 1))
        pc.check_grad(b, dtype, *shape, "square", bias=True, strides=(3, 1))
        pc.check_loss(b, dtype, *shape, 0.3, strides=(3, 1))


def test_broadcast_rows(b):
    one = b.make(np.ones((1, 9)), "f32")
    pc.check_grad(b, "f32", 21, 12, 9, "none", bias=True, dy=one.expand(21, 9))


def test_large_scores(b):
    pc.check_loss(b, "f32", 40, 30, 50, 0.2, std=100.0)


@pytest.mark.parametrize("where", ["new", "place"])
@pytest.mark.parametrize("share", [0.3, 2.0])
def test_clip(b, where, share):
    say("clip", where, share)
    pc.check_clip(b, ["f32"], [1], share, where)
    pc.check_clip(b, ["f32", "bf16", "f16"], [125, 16385, 3], share, where)
    pc.check_clip(b, ["bf16", "f16", "f32"] * 67, [(7 * i) % 40 for i in range(201)], share, where)
    pc.check_clip(b, ["f32", "f32"], [40, 50], share, where, std=1e25)
    pc.check_clip(b, ["bf16", "f32", "bf16"], [3000001, 1500003, 17], share, where)


def test_clip_views_of_any_alignment(b):
    flat = b.make(pc.normal(np.random.default_rng(3), 5000), "bf16")
    before = b.values(flat)
    views = [flat[1:1000], flat[1000:1001], flat[1001:4444]]
    norm = b.ctx.clip_grad_norm(views, 1.0)
    want = np.sqrt((before[1:4444] ** 2).sum())
    pc.within(b.values(norm), want, 2.0 ** -23 * want, "norm")
    got, f = b.values(flat), 1.0 / (want + 1e-6)
    assert (got[:1] == before[:1]).all() and (got[4444:] == before[4444:]).all()
    pc.within(got[1:4444], before[1:4444] * f, (pc.U["bf16"] + 4 * pc.E) * np.abs(before[1:4444]) * f, "gradient")


def test_pieces_of_the_classes(b):
    """more scores than the library holds the gradients of at a time: 2^29 bytes"""
    M, D, V = 4099, 72, 70001
    say("pieces", M, D, V)
    x, w, t = pc.loss_inputs(b, "bf16", M, D, V, 0.2)
    loss, dx, dw = b.ctx.cross_entropy_grad(x, w, b.ints(t, np.int64))
    assert M * V * 2 > 2 ** 29
    keep = np.nonzero(t != pc.IGNORE)[0]
    n = len(keep)
    X, W = x.double()[torch.from_numpy(keep).cuda()], w.double()
    L = X @ W.t().contiguous()
    lse = torch.logsumexp(L, 1, keepdim=True)
    at = (torch.arange(n, device="cuda"), torch.from_numpy(t[keep]).cuda())
    want = float((lse[:, 0] - L[at]).mean())
    assert abs(float(loss) - want) < 1e-5 * want
    p = torch.exp(L - lse)
    p[at] -= 1
    p /= n
    # scores' gradients are rounded to 8 bits, each result once more; sums err by far less than either
    u, q = pc.U["bf16"], p.abs() * (pc.U["bf16"] * 1.1)
    for got, exact, slack in ((dx[torch.from_numpy(keep).cuda()], p @ W, q @ W.abs()), (dw, p.t().contiguous() @ X, q.t().contiguous() @ X.abs())):
        assert ((got.double() - exact).abs() <= u * exact.abs() + slack + 1e-30).all()
    assert float(dx[torch.from_numpy(np.nonzero(t == pc.IGNORE)[0]).cuda()].abs().max()) == 0


def test_offsets_beyond_32_bits(b):
    """an input whose rows lie 2^27 numbers apart: the last ones start beyond 2^32 bytes, and beyond 2^31 numbers"""
    M, K, N, gap = 20, 40, 24, 2 ** 27
    say("offsets", M, gap)
    big = torch.empty(M * gap, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(8)
    x = big.as_strided((M, K), (gap, 1))
    x.copy_(b.make(pc.normal(rng, M, K), "bf16"))
    w, dy = b.make(pc.normal(rng, N, K), "bf16"), b.make(pc.normal(rng, M, N), "bf16")
    near = x.contiguous()
    assert torch.equal(b.ctx.linear(x, w), b.ctx.linear(near, w))
    assert torch.equal(b.ctx.linear_grad(dy, x, w)[1], b.ctx.linear_grad(dy, near, w)[1])
    t = b.ints(rng.integers(0, N, M), np.int64)
    for u, v in zip(b.ctx.cross_entropy_grad(x, w, t), b.ctx.cross_entropy_grad(near, w, t)):
        assert torch.equal(u, v)
    y = big[64:].as_strided((M, N), (gap, 1))
    b.ctx.linear(near, w, out=y)
    assert torch.equal(y, b.ctx.linear(near, w))


def test_the_same_bits_every_time(b):
    rng = np.random.default_rng(9)
    x, w, t = pc.loss_inputs(b, "bf16", 3000, 256, 700, 0.3)
    targets, dy = b.ints(t, np.int64), b.make(pc.normal(rng, 3000, 700), "bf16")
    grads = [b.make(pc.normal(rng, n), "f32") for n in (100000, 7, 333)]
    out = [torch.empty_like(g) for g in grads]

    def step():
        y, z = b.ctx.linear(x, w, activation="square", keep=True)
        return [y, *b.ctx.linear_grad(dy, x, w, z, activation="square", bias=True), *b.ctx.cross_entropy_grad(x, w, targets),
                b.ctx.clip_grad_norm(grads, 0.5, out=out)] + [o.clone() for o in out]

    first = step()
    for _ in range(3):
        for u, v in zip(first, step()):
            assert torch.equal(u, v)


def test_stream_rule_and_graph(b):
    """a call on another stream than the handle's is refused; a recorded step, replayed between other work, gives the eager step's bits"""
    x, w, t = pc.loss_inputs(b, "f32", 900, 64, 40, 0.3)
    targets, bias = b.ints(t, np.int64), b.make(np.linspace(-1, 1, 64), "f32")
    w1 = b.make(pc.normal(np.random.default_rng(1), 64, 64, std=0.1), "f32")
    out = [torch.empty_like(w1), torch.empty_like(w)]

    def step():
        h, z = b.ctx.linear(x, w1, bias, activation="square", keep=True)
        loss, dh, dw = b.ctx.cross_entropy_grad(h, w, targets)
        _, dw1, db = b.ctx.linear_grad(dh, x, w1, z, activation="square", bias=True, need_dx=False)
        norm = b.ctx.clip_grad_norm([dw1, dw], 0.01, out=out)
        return loss, db, norm, out[0], out[1]

    want = [v.clone() for v in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with pytest.raises(RuntimeError):
            b.ctx.linear(x, w1)
    graph = torch.cuda.CUDAGraph()
    try:
        with torch.cuda.stream(side):
            b.ctx.use_stream()
            step()
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                got = step()
    finally:
        b.ctx.use_stream()
    for i in range(4):
        for v in got:
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(want, got):
            assert torch.equal(u, v), i
        say("replay", i)
        step()                                            # eager work in between, in the same work memory
        torch.cuda.synchronize()


def test_refusals(b):
    x, w = b.make(np.ones((6, 5)), "f32"), b.make(np.ones((4, 5)), "f32")
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    for bad in (lambda: b.ctx.linear(x.cpu(), w), lambda: b.ctx.linear(x.double(), w.double()), lambda: b.ctx.linear(x.t(), w),
                lambda: b.ctx.linear(x, w.half()), lambda: b.ctx.cross_entropy(x, w, t.cpu()), lambda: b.ctx.cross_entropy(x, w, t[::2]),
                lambda: b.ctx.clip_grad_norm([x.t()], 1.0)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: b.ctx.linear(x, w[:, :4]), lambda: b.ctx.linear(x, w, out=x[:, :4]), lambda: b.ctx.cross_entropy(x, w, t[:4])):
        with pytest.raises(ValueError):
            bad()
