"""Grouped products, vocabulary loss, 8-bit checkpoints: what the host refuses, and the sizes it plans; no GPU call is made."""
import ctypes as C
import os
import subprocess

import pytest

import paper_1906_12043_amd as P

A = 1 << 20            # addresses that no call below gets as far as using


def grouped(**more):
    f = dict(dtype=P.BF16, groups=4, rows=100, inner=64, outer=32, offsets=A, x=2 * A, ldx=64, w=3 * A, ldw=32, w_stride=64 * 32,
             y=4 * A, ldy=32, dy=5 * A, lddy=32, dx=6 * A, lddx=64, dw=7 * A, lddw=32, dw_stride=64 * 32, dw_dtype=P.F32)
    f.update(more)
    return P.Grouped(**f)


def refused(fn, *args, status=P.ERR_INVALID, text=""):
    with pytest.raises(P.CocodError) as err:
        fn(*args)
    assert err.value.status == status and text in str(err.value), str(err.value)


COMMON = [
    (dict(dtype=3), "element type"), (dict(groups=0), "groups"), (dict(groups=65536), "groups"), (dict(flags=4), "flag"),
    (dict(rows=1 << 31), "rows"), (dict(inner=0), "inner"), (dict(outer=0), "inner"), (dict(inner=(1 << 30) + 1), "inner"),
    (dict(offsets=None), "offsets"), (dict(offsets=A + 4), "offsets"),
]


@pytest.mark.parametrize("change, text", COMMON)
def test_grouped_shape_is_checked_by_every_call(change, text):
    for fn in (P.grouped_forward, P.grouped_input_grad, P.grouped_weight_grad):
        refused(fn, None, grouped(**change), text=text)
    refused(P.grouped_workspace, grouped(**change), P.GROUPED_FORWARD, text=text)


@pytest.mark.parametrize("fn, change, text", [
    (P.grouped_forward, dict(x=None), "x is NULL"), (P.grouped_forward, dict(x=2 * A + 1), "x is not aligned"),
    (P.grouped_forward, dict(ldx=63), "rows of x"), (P.grouped_forward, dict(ldx=(1 << 30) + 1), "rows of x"),
    (P.grouped_forward, dict(w=None), "w is NULL"), (P.grouped_forward, dict(ldw=31), "rows of w"),
    (P.grouped_forward, dict(w_stride=64 * 32 - 1), "overlap"), (P.grouped_forward, dict(w_stride=(1 << 44) + 1), "2^44"),
    (P.grouped_forward, dict(y=None), "y is NULL"), (P.grouped_forward, dict(ldy=31), "rows of y"),
    (P.grouped_forward, dict(y=2 * A + 128), "y and x overlap"), (P.grouped_forward, dict(y=3 * A + 4 * 64 * 32 * 2 - 2), "y and w overlap"),
    (P.grouped_forward, dict(y=A + 38), "y and offsets overlap"),
    (P.grouped_forward, dict(dtype=P.F32, y=4 * A + 2), "y is not aligned"),
    (P.grouped_input_grad, dict(dy=None), "dy is NULL"), (P.grouped_input_grad, dict(dx=None), "dx is NULL"),
    (P.grouped_input_grad, dict(dx=5 * A), "dx and dy overlap"), (P.grouped_input_grad, dict(lddx=63), "rows of dx"),
    (P.grouped_input_grad, dict(flags=P.GROUPED_RELU_IN, x=None), "x_codes is NULL"),
    (P.grouped_input_grad, dict(flags=P.GROUPED_RELU_IN, x=6 * A), "dx and x overlap"),
    (P.grouped_weight_grad, dict(x=None), "x_codes is NULL"),
    (P.grouped_weight_grad, dict(x=None, x_codes=8 * A, ld_codes=64), "x_scales is NULL"),
    (P.grouped_weight_grad, dict(x=None, x_codes=8 * A, ld_codes=64, x_scales=9 * A, ld_scales=1), "rows of x_scales"),
    (P.grouped_weight_grad, dict(dw=None), "dw is NULL"), (P.grouped_weight_grad, dict(dw_dtype=P.F16), "dw_dtype"),
    (P.grouped_weight_grad, dict(dw_stride=0), "overlap"), (P.grouped_weight_grad, dict(dw=5 * A + 64), "dw and dy overlap"),
])
def test_grouped_arguments_are_refused(fn, change, text):
    refused(fn, None, grouped(**change), text=text)


def test_grouped_struct_and_null():
    g = grouped()
    g.struct_size -= 4
    for fn in (P.grouped_forward, P.grouped_input_grad, P.grouped_weight_grad):
        refused(fn, None, g, text="struct_size")
    for name in ("cocod_grouped_forward", "cocod_grouped_input_grad", "cocod_grouped_weight_grad", "cocod_cross_entropy"):
        assert getattr(P.lib(), name)(None, None) == P.ERR_INVALID
    assert P.lib().cocod_grouped_workspace(C.byref(grouped()), 0, None) == P.ERR_INVALID
    refused(P.grouped_workspace, grouped(), 3, text="direction")
    with pytest.raises(TypeError):
        P.Grouped(no_such_field=1)


def test_descriptions_match_the_header(tmp_path):
    """Size and place of every field, from a C compiler."""
    names = {"cocod_grouped": P.Grouped, "cocod_cross_entropy_call": P.CrossEntropy}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "cocod.h"', "int main(void) {"]
    for name, mirror in names.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in mirror._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include"), str(src), "-o", str(exe)], check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, mirror in names.items():
        assert int(got[name]) == C.sizeof(mirror)
        for f, _ in mirror._fields_:
            assert int(got["%s.%s" % (name, f)]) == getattr(mirror, f).offset, f


def test_grouped_workspace_is_needed_in_full_or_not_given():
    few = grouped(groups=1, rows=8192, inner=64, outer=64, ldx=64, lddy=64, lddw=64)
    need = P.grouped_workspace(few, P.GROUPED_WEIGHT_GRAD)
    assert need > 0 and need % (64 * 64 * 4) == 0
    few.set(workspace=16 * A, workspace_bytes=need - 1)
    refused(P.grouped_weight_grad, None, few, text="workspace holds")
    few.set(workspace=16 * A + 8, workspace_bytes=need)
    refused(P.grouped_weight_grad, None, few, text="16-byte")
    few.set(workspace=7 * A, workspace_bytes=need)
    refused(P.grouped_weight_grad, None, few, text="overlap")
    many = grouped(groups=16, rows=65536, inner=2048, outer=2048, ldx=2048, ldw=2048, ldy=2048, w_stride=1 << 22)
    assert P.grouped_workspace(many, P.GROUPED_FORWARD) == 0


def test_results_of_more_tiles_than_a_launch_are_refused():
    # 65535 groups of 15 rows, 2^14 columns: (983025 / 32 + 65535) * 256 tiles of 256 threads
    wide = grouped(groups=65535, rows=65535 * 15, inner=8, outer=1 << 14, ldx=8, ldw=1 << 14, ldy=1 << 14, w_stride=1 << 17,
                   x=1 << 50, w=1 << 52, y=1 << 54)
    refused(P.grouped_forward, None, wide, status=P.ERR_UNSUPPORTED, text="tiles")


def test_no_rows_need_no_gpu():
    P.grouped_forward(None, grouped(rows=0))
    P.grouped_input_grad(None, grouped(rows=0, dy=None, dx=None))
    P.checkpoint_store(None, P.BF16, 0, 40, A, 40, 2 * A, 40, 3 * A, 2)
    P.checkpoint_load(None, P.BF16, 0, 40, 2 * A, 40, 3 * A, 2, A, 40)


def loss_call(**more):
    f = dict(dtype=P.BF16, groups=2, rows=100, dim=64, vocab=1000, offsets=A, h=2 * A, ldh=64, e=3 * A, lde=64, e_stride=64000,
             targets=4 * A, loss=5 * A, group_loss=6 * A, dh=7 * A, lddh=64, de=8 * A, ldde=64, de_stride=64000,
             workspace=64 * A, workspace_bytes=1 << 40)
    f.update(more)
    return P.CrossEntropy(**f)


@pytest.mark.parametrize("change, text", [
    (dict(dtype=7), "element type"), (dict(groups=0), "groups"), (dict(flags=2), "flag"), (dict(rows=1 << 26), "rows"), (dict(dim=0), "dim"),
    (dict(vocab=0), "dim and vocab"), (dict(vocab=(1 << 30) + 1), "dim and vocab"), (dict(grad_scale=float("nan")), "grad_scale"),
    (dict(offsets=A + 2), "offsets"), (dict(h=None), "h is NULL"), (dict(ldh=63), "rows of h"), (dict(e=3 * A + 1), "e is not aligned"),
    (dict(e_stride=63999), "overlap"), (dict(targets=None), "targets"), (dict(targets=4 * A + 2), "targets"), (dict(loss=None), "loss"),
    (dict(group_loss=6 * A + 1), "group_loss"), (dict(lddh=63), "rows of dh"), (dict(ldde=63), "rows of de"), (dict(de_stride=0), "overlap"),
    (dict(workspace=None), "workspace"), (dict(workspace=64 * A + 16), "256-byte"), (dict(workspace_bytes=100), "workspace holds"),
    (dict(dh=2 * A + 64), "dh and h overlap"), (dict(de=3 * A + 64), "de and e overlap"), (dict(loss=4 * A), "loss and targets overlap"),
    (dict(workspace=2 * A), "overlap"), (dict(group_loss=5 * A + 4), "overlap"),
])
def test_loss_arguments_are_refused(change, text):
    refused(P.cross_entropy, None, loss_call(**change), text=text)


def test_loss_workspace_grows_with_what_is_asked_for():
    alone = P.cross_entropy_workspace(loss_call(dh=None, de=None))
    grads = P.cross_entropy_workspace(loss_call())
    pieces = P.cross_entropy_workspace(loss_call(vocab=100000, piece=256))
    whole = P.cross_entropy_workspace(loss_call(vocab=100000, piece=100000))
    assert 0 < alone < grads and pieces < whole
    # the logits of a large batch would take 2 GiB in 16 bits; the slopes of one piece take a quarter
    large = loss_call(groups=1, rows=8192, vocab=131072, dim=2048)
    assert P.cross_entropy_workspace(large) < 8192 * 131072 * 2 // 2
    c = loss_call()
    c.struct_size += 8
    refused(P.cross_entropy, None, c, text="struct_size")
    refused(P.cross_entropy_workspace, c, text="struct_size")


@pytest.mark.parametrize("args, text", [
    ((9, 4, 40, A, 40, 2 * A, 40, 3 * A, 2), "element type"), ((-1, 4, 40, A, 40, 2 * A, 40, 3 * A, 2), "element type"),
    ((P.BF16, 1 << 31, 40, A, 40, 2 * A, 40, 3 * A, 2), "rows"), ((P.BF16, 4, 0, A, 40, 2 * A, 40, 3 * A, 2), "cols"),
    ((P.BF16, 4, 40, None, 40, 2 * A, 40, 3 * A, 2), "x is NULL"), ((P.BF16, 4, 40, A + 1, 40, 2 * A, 40, 3 * A, 2), "x is not aligned"),
    ((P.BF16, 4, 40, A, 39, 2 * A, 40, 3 * A, 2), "rows of x"), ((P.BF16, 4, 40, A, 40, None, 40, 3 * A, 2), "codes is NULL"),
    ((P.BF16, 4, 40, A, 40, 2 * A, 39, 3 * A, 2), "rows of codes"), ((P.BF16, 4, 40, A, 40, 2 * A, 40, None, 2), "scales is NULL"),
    ((P.BF16, 4, 40, A, 40, 2 * A, 40, 3 * A, 1), "rows of scales"), ((P.BF16, 4, 40, A, 40, A + 100, 40, 3 * A, 2), "x and codes overlap"),
    ((P.BF16, 4, 40, A, 40, 2 * A, 40, 2 * A + 159, 2), "codes and scales overlap"),
])
def test_checkpoint_arguments_are_refused(args, text):
    refused(P.checkpoint_store, None, *args, text=text)
    dtype, rows, cols, x, ldx, codes, ldc, scales, lds = args
    refused(P.checkpoint_load, None, dtype, rows, cols, codes, ldc, scales, lds, x, ldx, text=text)


def test_the_loss_knows_its_flags():
    both = P.CROSS_ENTROPY_SUM | P.CROSS_ENTROPY_RELU_IN
    assert P.cross_entropy_workspace(loss_call(flags=both)) == P.cross_entropy_workspace(loss_call())
    for flags in (2, 8, both | 2, 1 << 31):
        refused(P.cross_entropy, None, loss_call(flags=flags), text="flag")
        refused(P.cross_entropy_workspace, loss_call(flags=flags), text="flag")


@pytest.mark.parametrize("dtype, rows, vocab, more", [
    (P.BF16, 1 << 22, 1 << 18, {}),                                       # 2^14 by 2^10 tiles of 256 x 256 for the logits
    (P.F32, 1 << 20, 1 << 18, dict(dh=None, de=None)),                    # 2^13 by 2^11 tiles of 128 x 128
    (P.BF16, 100, 1 << 30, dict(groups=16, de_stride=1 << 36, e_stride=0, dh=None, piece=1 << 30))])      # 2^24 row tiles of a table for each of 16 groups
def test_losses_of_more_tiles_than_a_launch_are_refused_before_anything_is_begun(dtype, rows, vocab, more):
    far = dict(e=1 << 44, targets=1 << 54, loss=1 << 55, h=1 << 56, dh=1 << 57, de=1 << 58, e_stride=0, groups=1, workspace=1 << 60, workspace_bytes=1 << 59)
    refused(P.cross_entropy, None, loss_call(dtype=dtype, rows=rows, vocab=vocab, **{**far, **more}), status=P.ERR_UNSUPPORTED, text="tiles")


def test_numbers_that_a_field_cannot_hold_are_refused():
    for field, value in (("inner", (1 << 32) + 64), ("outer", -1), ("groups", 1 << 32), ("rows", -1), ("rows", 1 << 64), ("ldx", (1 << 64) + 64)):
        with pytest.raises(ValueError, match=field):
            grouped(**{field: value})
        with pytest.raises(ValueError, match=field):
            grouped().set(**{field: value})
    with pytest.raises(ValueError, match="vocab"):
        loss_call(vocab=(1 << 32) + 1000)
    assert grouped(rows=(1 << 64) - 1).rows == (1 << 64) - 1 and loss_call(grad_scale=0.1).grad_scale == pytest.approx(0.1)
