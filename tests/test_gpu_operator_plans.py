"""Every kernel of the products (operator_plans names the sizes that reach them) against 64 bits, element by element."""
import pytest
import torch

import paper_1906_12043_amd as P
from tests import operator_harness as oh
from tests import operator_plans as op
from tests.test_gpu_operators import close, generator

pytestmark = pytest.mark.gpu


def with_workspace(lay, direction):
    ws = torch.full((max(P.grouped_workspace(lay, direction), 16),), 255, dtype=torch.uint8, device="cuda")      # NaN in every word
    lay.set(workspace=ws, workspace_bytes=ws.numel())
    lay.ws = ws
    return lay


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", op.PRODUCTS)
def test_products(dtype, case):
    groups, rows, k, n = case
    t, gen, bounds = oh.TYPES[dtype][1], generator(rows + k + n), op.bounds_of(groups, rows)
    x, dy, w = oh.matrix(rows, k, 0, t, gen), oh.matrix(rows, n, 0, t, gen), oh.stack(groups, k, n, 0, 0, t, gen, std=max(k, n) ** -0.5)
    written = oh.inside(bounds, rows)
    for kind, direction in op.DIRECTIONS.items():
        buf, out = oh.output(dict(forward=(rows, n), input_grad=(rows, k), weight_grad=(groups, k, n))[kind], 0, torch.float32 if kind == "weight_grad" else t)
        given = dict(forward=dict(w=w, y=out), input_grad=dict(dy=dy, w=w, dx=out), weight_grad=dict(dy=dy, dw=out))[kind]
        lay = with_workspace(oh.layer(dtype, bounds, rows, k, n, x=x, flags=P.GROUPED_RELU_OUT | P.GROUPED_RELU_IN, **given), direction)
        assert P.debug_grouped_plan(lay, direction) == P.debug_grouped_plan(op.product_call(dtype, *case), direction)
        oh.CALLS[kind][0](torch.cuda.current_stream(), lay)
        want, mag, terms = oh.exact_product(kind, bounds, *dict(forward=(x, w), input_grad=(dy, w), weight_grad=(x, dy))[kind])
        bound = oh.product_bound(want, mag, terms, out.dtype)
        if kind == "weight_grad":
            close(out, want, bound)
        else:
            close(out[written], (want.clamp(min=0) if kind == "forward" else want * (x > 0))[written], bound[written])
            assert oh.untouched(buf, out, written)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", op.CODES)
def test_weight_gradients_from_codes(dtype, case):
    groups, rows, k, n = case
    (kind, t), gen, bounds = oh.TYPES[dtype], generator(rows + k + n), op.bounds_of(groups, rows)
    x, dy = torch.relu(oh.matrix(rows, k, 0, t, gen)), oh.matrix(rows, n, 0, t, gen)
    codes, scales = torch.empty((rows, k), dtype=torch.uint8, device="cuda"), torch.empty((rows, -(-k // 32)), dtype=torch.uint8, device="cuda")
    P.checkpoint_store(torch.cuda.current_stream(), kind, rows, k, x, k, codes, k, scales, scales.shape[1])
    back, dw = torch.empty_like(x), torch.empty((groups, k, n), device="cuda")
    P.checkpoint_load(torch.cuda.current_stream(), kind, rows, k, codes, k, scales, scales.shape[1], back, k)
    lay = with_workspace(oh.layer(dtype, bounds, rows, k, n, dy=dy, dw=dw, x_codes=codes, x_scales=scales), P.GROUPED_WEIGHT_GRAD)
    assert P.debug_grouped_plan(lay, P.GROUPED_WEIGHT_GRAD) == P.debug_grouped_plan(op.product_call(dtype, *case, codes=True), P.GROUPED_WEIGHT_GRAD)
    P.grouped_weight_grad(torch.cuda.current_stream(), lay)
    want, mag, terms = oh.exact_product("weight_grad", bounds, back, dy)
    close(dw, want, oh.product_bound(want, mag, terms, torch.float32))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", op.LOSSES)
def test_losses(dtype, case):
    groups, rows, dim, vocab, piece = case
    t, gen, bounds = oh.TYPES[dtype][1], generator(rows + dim + vocab), op.bounds_of(groups, rows)
    h, e = oh.matrix(rows, dim, 0, t, gen), oh.stack(groups, vocab, dim, 0, 0, t, gen, std=3.0 / dim ** 0.5)
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    target[::7] = -1
    h[::7] = float("nan")
    want = oh.exact_loss(bounds, h, e, target, grad_scale=3.0)
    bound, written = oh.loss_bounds(want, t, dim, vocab), oh.inside(bounds, rows)
    loss, (hbuf, dh), (ebuf, de) = torch.empty(rows, device="cuda"), oh.output((rows, dim), 0, t), oh.output((groups, vocab, dim), 0, t)
    call = oh.cross_entropy_call(dtype, bounds, h, e, target, dh, de, None, loss, grad_scale=3.0, piece=piece)
    assert P.debug_cross_entropy_plan(call) == P.debug_cross_entropy_plan(op.loss_call(dtype, *case))
    P.cross_entropy(torch.cuda.current_stream(), call)
    close(loss[written], want["loss"][written], bound["loss"][written])
    close(dh[written], want["dh"][written], bound["dh"][written])
    close(de, want["de"], bound["de"])
    assert oh.untouched(hbuf, dh, written)
