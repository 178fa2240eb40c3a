"""The training operators on the device, at the edges of their numbers, memory and arguments."""
import numpy as np
import pytest

import plain_cases as pc
import plain_edge_cases as pe
from test_gpu_plain_ops import Backend, say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b():
    return Backend()


@pytest.mark.parametrize("case", pe.LOW, ids=str)
def test_classes_of_minus_infinity(b, case):
    say("minus infinity", case)
    pe.check_low_classes(b, *case)


@pytest.mark.parametrize("case", pe.RANGE, ids=str)
def test_range_of_binary16_gradients(b, case):
    pe.check_range(b, *case)


def test_range_of_each_row_and_column(b):
    pe.check_range_of_each_row(b)


def test_rows_that_are_not_finite(b):
    pe.check_rows_that_are_not_finite(b)


def test_recorded_step_after_larger_calls():
    """a step recorded at one size gives its bits after eager calls that need more work memory"""
    b = Backend()

    def inputs(rows):
        x, w, t = pc.loss_inputs(b, "bf16", rows, 96, 700, 0.3)
        w1 = b.make(pc.normal(np.random.default_rng(1), 96, 96, std=0.1), "bf16")
        return x, w, b.ints(t, np.int64), w1

    def step(x, w, targets, w1):
        h, z = b.ctx.linear(x, w1, activation="square", keep=True)
        loss, dh, dw = b.ctx.cross_entropy_grad(h, w, targets)
        _, dw1, db = b.ctx.linear_grad(dh, x, w1, z, activation="square", bias=True, need_dx=False)
        return loss, dh, dw, dw1, db

    small, side, graph = inputs(300), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    want = [v.clone() for v in step(*small)]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.ctx.use_stream()
        step(*small)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = step(*small)
    b.ctx.use_stream()
    held = b.ctx.scratch_bytes()
    for rows in (2000, 300, 9000):
        say("replay after", rows, "rows")
        step(*inputs(rows))
        others = [torch.full((1 << 24,), float("nan"), device="cuda") for _ in range(8)]      # what a freed block would be used for
        for v in got:
            v.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(want, got):
            assert torch.equal(u, v), rows
        assert all(bool(torch.isnan(o).all()) for o in others)
    assert b.ctx.scratch_bytes() > held
    del graph
    b.ctx.close()


def _within(got, want, bound, what):
    """|got - want| <= bound, number by number, on the device"""
    off = (got.double() - want).abs() - bound
    assert bool(torch.isfinite(got).all()) and float(off.max()) <= 0, (what, float(off.max()))


def _act(z, name):
    """(value, slope) in 64 bits"""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "square":
        return z * z, 2 * z
    cdf = torch.special.ndtr(z)
    return z * cdf, cdf + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5


def _wide_linear(b, dtype, M, K, N, strides):
    """linear with everything and linear_grad, at sizes whose 64-bit products belong on the device; plain_cases' bounds"""
    rng = np.random.default_rng([M, K, N])
    u, least, E, FN = pc.U[dtype], pc.LEAST[dtype], pc.E, pc.FN
    x, w = b.make(pc.normal(rng, M, K), dtype, strides), b.make(pc.normal(rng, N, K, std=K ** -0.5), dtype, strides)
    bias, r = b.make(pc.normal(rng, N), dtype), b.make(pc.normal(rng, M, N), dtype, strides)
    X, W, B, R = (v.double() for v in (x, w, bias, r))
    y, z = b.ctx.linear(x, w, bias, r, activation="gelu", keep=True)
    mag = X.abs() @ W.abs().t() + B.abs()
    Z = X @ W.t() + B
    dz = (K + 4) * E * mag
    _within(z, Z, u * Z.abs() + dz + least, "z")
    Y = _act(Z, "gelu")[0]
    _within(y, Y + R, u * (Y + R).abs() + 1.2 * dz + FN * (Z.abs() + 1e-30) * (2 + Z.abs()) + 2 * E * R.abs() + least, "y")
    assert torch.equal(b.ctx.linear(x, w, bias, r, activation="gelu"), y)
    for name in ("none", "square"):
        dy = b.make(pc.normal(rng, M, N), dtype, strides)
        dx, dw, db = b.ctx.linear_grad(dy, x, w, z, activation=name, bias=True)
        DY = dy.double()
        DZ = DY * _act(z.double(), name)[1]
        room = 0.0 if name == "none" else (u + 4 * E)
        low = 0.0 if name == "none" else least + (2.0 ** -39 * float(DZ.abs().max()) if dtype == "f16" else 0.0)
        err = room * DZ.abs() + low
        _within(dx, DZ @ W, u * (DZ @ W).abs() + (err + (N + 4) * E * DZ.abs()) @ W.abs() + least, "dx " + name)
        _within(dw, DZ.t() @ X, u * (DZ.t() @ X).abs() + (err + (M + 4) * E * DZ.abs()).t() @ X.abs() + least, "dw " + name)
        _within(db, DZ.sum(0), u * DZ.sum(0).abs() + ((M + 8) * E * DZ.abs()).sum(0) + least, "db " + name)


@pytest.mark.parametrize("case", pe.WIDE, ids=str)
def test_largest_tiles_with_ragged_edges(b, case):
    say("largest tiles", case)
    _wide_linear(b, *case, strides=None)


@pytest.mark.parametrize("case", pe.COPIED, ids=str)
@pytest.mark.parametrize("strides", [None, (3, 1)])
def test_copied_operands(b, case, strides):
    """odd rows, with NaN between them"""
    say("copied operands", case, strides)
    _wide_linear(b, *case, strides=strides)


@pytest.mark.parametrize("case", pe.COPIED_LOSS, ids=str)
@pytest.mark.parametrize("masked", [0.0, 0.3])
def test_copied_operands_of_the_loss(b, case, masked):
    dtype, M, K, V = case
    say("loss of copied operands", case, masked)
    u, least, E, FN = pc.U[dtype], pc.LEAST[dtype], pc.E, pc.FN
    x, w, t = pc.loss_inputs(b, dtype, M, K, V, masked, strides=(3, 1), junk=True)
    scale = 1024.0 if dtype == "f16" else 1.0
    loss, dx, dw = b.ctx.cross_entropy_grad(x, w, b.ints(t, np.int64), scale=scale)
    keep = torch.from_numpy(np.nonzero(t != pc.IGNORE)[0]).cuda()
    n = len(keep)
    X, W = x.double()[keep], w.double()
    L = X @ W.t()
    lse = torch.logsumexp(L, 1, keepdim=True)
    at = (torch.arange(n, device="cuda"), torch.from_numpy(t).cuda()[keep])
    rows = lse[:, 0] - L[at]
    row_err = 2 * (K + 4) * E * (X.abs() @ W.abs().t()).amax(1) + 8 * E * (L.abs().amax(1) + np.log(V) + 1) + FN
    assert abs(float(loss) - float(rows.mean())) <= float(row_err.mean()) + E * abs(float(rows.mean()))
    e = torch.exp(L - lse)
    q = (scale / n) * (e * (row_err[:, None] * 2 + FN * (1 + (L - lse).abs())) + least * (2.0 ** -15 if dtype == "f16" else 1.0))
    p = e.clone()
    p[at] -= 1
    p *= scale / n
    q += u * p.abs()
    DX, DW = p @ W, p.t() @ X
    _within(dx[keep], DX, u * DX.abs() + (q + (V + 8) * E * p.abs()) @ W.abs() + least, "dx")
    _within(dw, DW, u * DW.abs() + (q + (M + 8) * E * p.abs()).t() @ X.abs() + least, "dw")
    hidden = torch.from_numpy(np.nonzero(t == pc.IGNORE)[0]).cuda()
    assert not hidden.numel() or float(dx[hidden].abs().max()) == 0


def test_rows_beyond_one_launchs_threads(b):
    """2^26 rows and a few: with 64 threads each, more than a launch can have"""
    M, K, V = 2 ** 26 + 37, 2, 3
    say("rows", M)
    g = torch.Generator(device="cuda").manual_seed(4)
    t = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    w = torch.randn((V, K), generator=g, device="cuda").bfloat16()
    x = torch.randn((M, K), generator=g, device="cuda").bfloat16()
    hide = torch.rand(M, generator=g, device="cuda") < 0.1
    hide[-3] = True
    t[hide] = pc.IGNORE
    x[hide] = float("nan")
    loss, rows, lse = b.ctx.cross_entropy(x, w, t, rows=True)
    mean, dx, dw = b.ctx.cross_entropy_grad(x, w, t, scale=float(M))
    assert float(mean) == float(loss)
    n = int((~hide).sum())
    total, dws = 0.0, torch.zeros((V, K), dtype=torch.float64, device="cuda")
    for at in range(0, M, 2 ** 24):
        s = slice(at, min(M, at + 2 ** 24))
        keep = ~hide[s]
        X, T = x[s].double().nan_to_num(), t[s].long().clamp(min=0)
        L = X @ w.double().t()
        want = torch.logsumexp(L, 1)
        want_rows = (want - L.gather(1, T[:, None])[:, 0]) * keep
        # three scores of two products each: a few units of the last place of the largest
        err = 16 * pc.E * (1 + L.abs().amax(1)) + pc.FN
        assert bool(((rows[s].double() - want_rows).abs() <= err).all()) and bool(((lse[s].double() - want * keep).abs() <= err).all()), at
        p = torch.exp(L - want[:, None])
        p.scatter_add_(1, T[:, None], torch.full_like(L[:, :1], -1.0))
        p *= keep[:, None] * (float(M) / n)
        DX = p @ w.double()
        # the scores' gradients and the result are rounded to 8 bits each
        bound = pc.U["bf16"] * DX.abs() + (p.abs() @ w.double().abs().contiguous()) * (pc.U["bf16"] + 64 * pc.FN) + 64 * pc.FN
        assert bool(((dx[s].double() - DX).abs() <= bound).all()), at
        assert float(dx[s][hide[s]].abs().max()) == 0
        total, dws = total + float(want_rows.sum()), dws + p.t().contiguous() @ X
    assert abs(float(loss) - total / n) <= 1e-5 * total / n
    # 6 x 10^7 gradients of both signs: their roundings, 2^-9 each at most, add up to far less than 2^-9 of their magnitudes' sum
    assert float((dw.double() - dws).abs().max()) <= pc.U["bf16"] * (float(dws.abs().max()) + 2.0 ** -4 * M)


def test_copy_of_many_numbers(b):
    M, K, N = 20001, 7001, 2001
    say("copy of", M * K, "numbers")
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w = torch.randn((M, K), generator=g, device="cuda").bfloat16(), (torch.randn((N, K), generator=g, device="cuda") / K ** 0.5).bfloat16()
    y = b.ctx.linear(x, w)
    X, W = x.double(), w.double()
    Z = X @ W.t()
    _within(y, Z, pc.U["bf16"] * Z.abs() + (K + 4) * pc.E * (X.abs() @ W.abs().t()) + pc.LEAST["bf16"], "y")


@pytest.mark.parametrize("where", ["new", "place"])
@pytest.mark.parametrize("case", pe.TINY, ids=str)
def test_factors_below_the_normal_numbers(b, case, where):
    pe.check_tiny_factor(b, *case, where)


def test_tail_of_gelu(b):
    pe.check_gelu_tail(b)


@pytest.mark.parametrize("name", ["none", "square", "relu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_some_of_the_gradients(b, dtype, name):
    pe.check_some_of_the_gradients(b, dtype, name)


@pytest.mark.parametrize("shape", [(50, 20, 9), (70, 33, 300), (3, 0, 20), (1, 40, 1000)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_some_of_the_loss(b, dtype, shape):
    pe.check_some_of_the_loss(b, dtype, *shape)
