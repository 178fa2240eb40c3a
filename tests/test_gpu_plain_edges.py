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
