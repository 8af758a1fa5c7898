"""Token scores: what the host refuses, the workspace it plans and the layout of the description; no GPU call is made."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paper_1906_12043_amd as P
from tests import operator_plans as op
from tests.operator_harness import TYPES
from tests.scores_harness import exact_scores
from tests.test_gpu_token_scores import LARGE, SHAPES

A = 1 << 20            # addresses that no call below gets as far as using


def scores(**more):
    f = dict(dtype=P.BF16, groups=2, rows=100, dim=64, vocab=200, offsets=A, h=2 * A, ldh=64, e=3 * A, lde=64, e_stride=200 * 64, targets=4 * A, logp=5 * A, entropy=6 * A,
             top=4, top_ids=7 * A, top_logp=8 * A, ld_top=4, norms=9 * A, d_logp=10 * A, d_entropy=11 * A, dh=12 * A, lddh=64, de=13 * A, ldde=64, de_stride=200 * 64,
             workspace=1 << 40, workspace_bytes=1 << 30)
    f.update(more)
    return P.TokenScores(**f)


def refused(fn, *args, status=P.ERR_INVALID, text=""):
    with pytest.raises(P.CocodError) as err:
        fn(*args)
    assert err.value.status == status and text in str(err.value), str(err.value)


BOTH = (P.token_scores, P.token_scores_grad)


@pytest.mark.parametrize("change, text", [
    (dict(dtype=3), "element type"), (dict(flags=2), "flag"), (dict(groups=0), "groups"), (dict(groups=65536), "groups"), (dict(rows=1 << 26), "rows"), (dict(dim=0), "dim"),
    (dict(vocab=0), "vocab"), (dict(vocab=(1 << 30) + 1), "vocab"), (dict(top=33), "top"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale")])
def test_shape_is_checked_by_every_call(change, text):
    for fn in BOTH:
        refused(fn, None, scores(**change), text=text)
    refused(P.token_scores_workspace, scores(**change), P.TOKEN_SCORES_FORWARD, text=text)


@pytest.mark.parametrize("change, text", [
    (dict(offsets=None), "offsets"), (dict(offsets=A + 4), "offsets"), (dict(h=None), "h is NULL"), (dict(h=2 * A + 1), "h is not aligned"), (dict(ldh=63), "rows of h"),
    (dict(e=None), "e is NULL"), (dict(lde=63), "rows of e"), (dict(e_stride=64), "e: 64 elements"), (dict(targets=4 * A + 2), "targets is not aligned"),
    (dict(norms=9 * A + 8), "norms"), (dict(workspace=None), "workspace"), (dict(workspace=(1 << 40) + 128), "256-byte"), (dict(workspace_bytes=1000), "workspace holds"),
    (dict(workspace=2 * A), "overlap")])
def test_inputs_are_checked_by_both_directions(change, text):
    for fn in BOTH:
        refused(fn, None, scores(**change), text=text)


@pytest.mark.parametrize("fn, change, text", [
    (P.token_scores, dict(logp=None, entropy=None, norms=None, top=0), "no output"), (P.token_scores, dict(targets=None), "targets is NULL"),
    (P.token_scores, dict(top_ids=None), "top_ids is NULL"), (P.token_scores, dict(top_logp=None), "top_logp is NULL"), (P.token_scores, dict(ld_top=3), "rows of top_ids"),
    (P.token_scores, dict(logp=5 * A + 2), "logp is not aligned"), (P.token_scores, dict(entropy=6 * A + 1), "entropy is not aligned"),
    (P.token_scores, dict(logp=6 * A + 8), "logp and entropy overlap"), (P.token_scores, dict(norms=2 * A), "norms and h overlap"), (P.token_scores, dict(top_ids=8 * A), "overlap"),
    (P.token_scores, dict(top_logp=4 * A), "top_logp and targets overlap"), (P.token_scores, dict(entropy=A), "entropy and offsets overlap"),
    (P.token_scores_grad, dict(dh=None, de=None), "dh and de are NULL"), (P.token_scores_grad, dict(norms=None), "norms is NULL"),
    (P.token_scores_grad, dict(d_logp=10 * A + 1), "d_logp is not aligned"), (P.token_scores_grad, dict(d_entropy=11 * A + 2), "d_entropy is not aligned"),
    (P.token_scores_grad, dict(dh=12 * A + 1), "dh is not aligned"), (P.token_scores_grad, dict(lddh=63), "rows of dh"), (P.token_scores_grad, dict(ldde=63), "rows of de"),
    (P.token_scores_grad, dict(de_stride=0), "overlap"), (P.token_scores_grad, dict(dh=2 * A), "dh and h overlap"), (P.token_scores_grad, dict(de=3 * A), "de and e overlap"),
    (P.token_scores_grad, dict(dh=13 * A), "dh and de overlap"), (P.token_scores_grad, dict(dh=9 * A), "dh and norms overlap"), (P.token_scores_grad, dict(dh=10 * A), "dh and d_logp overlap")])
def test_arguments_are_refused(fn, change, text):
    refused(fn, None, scores(**change), text=text)


def test_struct_and_null():
    c = scores()
    c.struct_size -= 8
    for fn in BOTH:
        refused(fn, None, c, text="struct_size")
    for name in ("cocod_token_scores", "cocod_token_scores_grad"):
        assert getattr(P.lib(), name)(None, None) == P.ERR_INVALID
    assert P.lib().cocod_token_scores_workspace(C.byref(scores()), 0, None) == P.ERR_INVALID
    refused(P.token_scores_workspace, scores(), 2, text="direction")
    with pytest.raises(TypeError):
        P.TokenScores(no_such_field=1)
    with pytest.raises(ValueError):
        P.TokenScores(vocab=1 << 32)


def test_no_rows_need_no_gpu():
    P.token_scores(None, scores(rows=0))
    P.token_scores(None, scores(rows=0, h=None, targets=None, logp=None))


def test_workspace_follows_what_is_asked_for():
    small = P.token_scores_workspace(scores(top=0), P.TOKEN_SCORES_FORWARD)
    for top in (1, 32):
        need = P.token_scores_workspace(scores(top=top), P.TOKEN_SCORES_FORWARD)
        assert small + 100 * (256 + 8 * top + 8) <= need <= small + 100 * (256 + 8 * top + 8) + 3 * 256
    wide = dict(rows=8192, vocab=131072, dim=2048, groups=1)
    assert P.token_scores_workspace(scores(**wide), P.TOKEN_SCORES_GRAD) >= 2 ** 28 * 2
    assert P.token_scores_workspace(scores(piece=1024, **wide), P.TOKEN_SCORES_GRAD) < 2 ** 28


def test_results_of_more_tiles_than_a_launch_are_refused():
    # 2^16 rows by 2^30 entries: 2^8 x 2^22 tiles of 512 threads
    wide = scores(groups=1, rows=1 << 16, vocab=1 << 30, dim=1, ldh=1, lde=1, lddh=1, ldde=1, h=1 << 41, e=1 << 42, targets=1 << 43, logp=1 << 44, entropy=1 << 45, norms=1 << 46, top=0,
                  d_logp=1 << 47, d_entropy=1 << 48, dh=1 << 49, de=1 << 50, workspace=1 << 56, workspace_bytes=1 << 55)
    refused(P.token_scores, None, wide, status=P.ERR_UNSUPPORTED, text="tiles")


def test_description_matches_the_header(tmp_path):
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "cocod.h"', "int main(void) {", 'printf("%zu\\n", sizeof(cocod_token_scores_call));']
    lines += ['printf("%%zu\\n", offsetof(cocod_token_scores_call, %s));' % f for f, _ in P.TokenScores._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(P.TokenScores)] + [getattr(P.TokenScores, f).offset for f, _ in P.TokenScores._fields_]


def test_the_formulas_of_the_gradient_are_differences():
    """The plain implementation that the kernels are held to, against central differences: their error is below step^2 / 6 times third derivatives (below 100 here) and 1e-13 / step."""
    gen = torch.Generator().manual_seed(2)
    bounds, vocab, dim = [0, 3, 7], 11, 5
    h, e = torch.randn(7, dim, generator=gen, dtype=torch.float64), torch.randn(2, vocab, dim, generator=gen, dtype=torch.float64)
    target = torch.tensor([3, -1, 10, 0, 5, 11, 7], dtype=torch.int32)
    a, b = torch.randn(7, generator=gen), torch.randn(7, generator=gen)

    def value(h_, e_):
        out, _ = exact_scores(bounds, h_, e_, target, 0.75)
        return float((a * out["logp"] + b * out["entropy"]).sum())

    out, _ = exact_scores(bounds, h, e, target, 0.75, a, b)
    step = 2.0 ** -14
    for name, x in (("dh", h), ("de", e)):
        for i in range(0, x.numel(), 3):
            up, down = x.clone(), x.clone()
            up.view(-1)[i] += step
            down.view(-1)[i] -= step
            diff = (value(up, e) - value(down, e) if name == "dh" else value(h, up) - value(h, down)) / (2 * step)
            assert abs(diff - float(out[name].view(-1)[i])) <= step ** 2 / 6 * 100 + 1e-13 / step


def test_every_tile_is_reached():
    """The tiles that the shapes of the tests on the GPU run with (the plan depends on sizes alone, and is the loss's)."""
    seen = set()
    for dtype in TYPES:
        for bounds, rows, vocab, dim in SHAPES + [LARGE]:
            x = P.CrossEntropy(dtype=TYPES[dtype][0], groups=len(bounds) - 1, rows=rows, dim=dim, vocab=vocab, offsets=8, h=16, ldh=dim, e=16, lde=dim, e_stride=vocab * dim,
                               workspace=1 << 40)
            seen.add((dtype, P.debug_cross_entropy_plan(x)[0][0][0]))
    want = {("fp32", 1), ("fp32", 2), ("fp32", 5)} | {(d, t) for d in ("bf16", "fp16") for t in (0, 1, 2, 3)}
    assert want <= seen, want - seen


def planned(dtype, groups, rows, dim, vocab, piece=0):
    f = dict(dtype=TYPES[dtype][0], groups=groups, rows=rows, dim=dim, vocab=vocab, offsets=A, h=1 << 41, ldh=dim, e=1 << 42, lde=dim, e_stride=vocab * dim, targets=1 << 43,
             norms=1 << 44, dh=1 << 45, lddh=dim, de=1 << 46, ldde=dim, de_stride=vocab * dim, piece=piece, workspace=1 << 47, workspace_bytes=1 << 46)
    return P.TokenScores(**f)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_every_product_is_reached_by_the_plans_of_the_calls_themselves(dtype):
    """Tiles, sums whole and split, pieces and ways of the operands, as the calls would run at the sizes of operator_plans."""
    seen = set()
    for case in op.LOSSES:
        call = planned(dtype, *case)
        seen.add(("logits",) + P.debug_token_scores_plan(call, P.TOKEN_SCORES_FORWARD)[0][0][::2])
        (slopes, dh, de), pieces = P.debug_token_scores_plan(call, P.TOKEN_SCORES_GRAD)
        seen.add(("slopes",) + slopes[::2])
        if case[2] >= op.COLUMNS[dh[0]]:
            seen.add(("dh", dh[0], dh[1] > 1, pieces > 1, dh[2]))
        if case[2] >= op.COLUMNS[de[0]]:
            seen.add(("de", de[0], de[1] > 1))
    both, logits = (False, True), ("logits", "slopes")
    if dtype == "fp32":
        tiles = (op.MEDIUM, op.SMALL, op.SQUARE)
        want = {(k, tile, op.REGISTERS) for k in logits for tile in tiles} | {("dh", tile, split, pieces, op.REGISTERS) for tile in tiles for split in both for pieces in both}
        want |= {("de", tile, split) for tile in tiles for split in both}
    else:
        tiles, few = (op.LARGE, op.MEDIUM, op.SMALL, op.DEEP), (op.MEDIUM, op.SMALL)
        want = {(k, tile, op.DIRECT) for k in logits for tile in tiles} | {(k, tile, op.REGISTERS) for k in logits for tile in few}
        want |= {("dh", tile, split, pieces, op.DIRECT) for tile in tiles + (op.TALL,) for split in both for pieces in both}
        want |= {("dh", tile, split, pieces, op.REGISTERS) for tile in few for split in both for pieces in both} | {("de", tile, split) for tile in tiles for split in both}
    assert seen == want, (seen - want, want - seen)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_large_table_that_few_rows_read_goes_past_the_caches(dtype):
    def way(groups, rows, vocab, dim=520, **change):
        call = planned(dtype, groups, rows, dim, vocab)
        call.set(**change)
        return P.debug_token_scores_plan(call, P.TOKEN_SCORES_FORWARD)[0][0]
    assert way(1, 5, 300_001) == (op.SMALL, 1, 3) and way(2, 32, 150_000) == (op.SMALL, 1, 3)
    assert way(1, 33, 300_001)[2] == op.DIRECT and way(1, 5, 200_001) == (op.SMALL, 1, op.DIRECT)
    assert way(2, 32, 150_000, e_stride=0) == (op.SMALL, 1, op.DIRECT)                 # one table, within the caches
    assert way(1, 5, 300_001, e=(1 << 42) + 2) == (op.SMALL, 1, op.REGISTERS)


def test_plans_refuse_what_the_calls_refuse():
    refused(P.debug_token_scores_plan, planned("bf16", 0, 7, 8, 8), 0, text="groups")
    refused(P.debug_token_scores_plan, planned("bf16", 1, 7, 8, 8), 2, text="direction")
    assert P.lib().cocod_debug_token_scores_plan(None, 0, None, None) == P.ERR_INVALID
    assert P.debug_token_scores_plan(scores(dh=None, de=None), P.TOKEN_SCORES_GRAD)[0][1:] == [(0, 0, 0), (0, 0, 0)]


@pytest.mark.parametrize("rows, dim, vocab, top", [(4096, 4096, 1000, 8), (4096, 1024, 32003, 0), (4, 2048, 131072, 8), (509, 512, 5003, 5)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_the_header_says_how_much_workspace_a_forward_call_needs(dtype, rows, dim, vocab, top):
    size = 4 if dtype == "fp32" else 2
    need = P.token_scores_workspace(P.TokenScores(dtype=TYPES[dtype][0], groups=1, rows=rows, dim=dim, vocab=vocab, top=top), P.TOKEN_SCORES_FORWARD)
    least, most = (rows * (dim * size + 16 * -(-vocab // entries) + (vocab + 8 * top if top else 0)) for entries in (128, 64))
    assert least <= need <= most + rows * (20 + (256 if top else 0)) + 8 * 256            # (a little: five numbers a row, and quads of whole tiles)
