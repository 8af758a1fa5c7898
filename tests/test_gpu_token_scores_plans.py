"""Every product of the token scores (operator_plans names the sizes, test_token_scores_host asserts that they reach them) against 64 bits, and the loss's gradient beside theirs."""
import math

import pytest
import torch

import paper_1906_12043_amd as P
from tests import operator_harness as oh
from tests import operator_plans as op
from tests.scores_harness import exact_scores, scores_call
from tests.test_gpu_token_scores import check_scores, check_top
from tests.test_token_scores_host import planned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(oh.TYPES))
@pytest.mark.parametrize("case", op.LOSSES)
def test_scores_and_gradients(dtype, case):
    groups, rows, dim, vocab, piece = case
    t, bounds, gen = oh.TYPES[dtype][1], op.bounds_of(groups, rows), torch.Generator(device="cuda").manual_seed(rows + dim + vocab)
    h, e = oh.matrix(rows, dim, 0, t, gen), oh.stack(groups, vocab, dim, 0, 0, t, gen, std=2.0 / math.sqrt(dim))
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    target[::7] = -1
    h[::7] = float("nan")
    a, b = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda") * 0.1
    (hbuf, dh), (ebuf, de) = oh.output((rows, dim), 0, t), oh.output((groups, vocab, dim), 0, t)
    call, out = scores_call(dtype, bounds, h, e, target, grad=True, top=5, scale=0.75, d_logp=a, d_entropy=b, dh=dh, de=de, piece=piece)
    for direction in (P.TOKEN_SCORES_FORWARD, P.TOKEN_SCORES_GRAD):
        assert P.debug_token_scores_plan(call, direction) == P.debug_token_scores_plan(planned(dtype, *case), direction)
    P.token_scores(torch.cuda.current_stream(), call)
    P.token_scores_grad(torch.cuda.current_stream(), call)
    want, far = exact_scores(bounds, torch.where(torch.isnan(h), 0.0, h), e, target, 0.75, a, b)
    inside = check_scores(out, want, far, bounds, rows, target)
    for k in ("top_ids", "top_logp"):
        out[k] = out[k][inside]
    for k in ("part", "all", "z", "far_all"):
        want[k] = want[k][inside]
    check_top(out, want, 5, vocab, False)
    assert bool(((dh.double() - want["dh"]).abs() <= far["dh"])[inside].all())
    assert bool(((de.double() - want["de"]).abs() <= far["de"]).all())
    assert oh.untouched(hbuf, dh, inside) and oh.untouched(ebuf, de)


@pytest.mark.parametrize("dtype", list(oh.TYPES))
@pytest.mark.parametrize("rows, vocab, dim", [(130, 900, 64), (700, 2003, 136)])
def test_gradients_of_the_loss_are_those_of_minus_the_log_probability(dtype, rows, vocab, dim):
    t, bounds, gen = oh.TYPES[dtype][1], [0, rows // 3, rows], torch.Generator(device="cuda").manual_seed(rows)
    h, e = oh.matrix(rows, dim, 0, t, gen), oh.stack(2, vocab, dim, 0, 0, t, gen, std=2.0 / math.sqrt(dim))
    target = torch.randint(-1, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    one, dh, de, dh_loss, de_loss = torch.ones(rows, device="cuda"), torch.empty_like(h), torch.empty_like(e), torch.empty_like(h), torch.empty_like(e)
    call, out = scores_call(dtype, bounds, h, e, target, grad=True, d_logp=one, dh=dh, de=de)
    P.token_scores(torch.cuda.current_stream(), call)
    P.token_scores_grad(torch.cuda.current_stream(), call)
    loss = torch.empty(rows, device="cuda")
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, dh_loss, de_loss, loss=loss, flags=P.CROSS_ENTROPY_SUM))
    _, far = exact_scores(bounds, h, e, target, 1.0, one)
    far_loss = oh.loss_bounds(oh.exact_loss(bounds, h, e, target, total=True), t, dim, vocab)
    assert bool(((loss + out["logp"]).double().abs() <= far["logp"] + far_loss["loss"]).all())
    assert bool(((dh_loss.double() + dh.double()).abs() <= far["dh"] + far_loss["dh"]).all())
    assert bool(((de_loss.double() + de.double()).abs() <= far["de"] + far_loss["de"]).all())
