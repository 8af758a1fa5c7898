"""The AdamW step: what the host refuses, the layout of its descriptions, and the terms that change from step to step; no GPU call is made."""
import ctypes as C
import math
import os
import subprocess

import pytest

import paper_1906_12043_amd as P

A = 1 << 20            # addresses that no call below gets as far as using
TENSOR = dict(n=1000, p=A, g=2 * A, m=3 * A, v=4 * A)
EIGHT = dict(TENSOR, m_scales=5 * A, v_scales=6 * A)


def adamw(tensors=(TENSOR,), **more):
    f = dict(dtype=P.F32, grad_dtype=P.F32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    f.update(more)
    return P.AdamW(tensors=tensors, **f)


def refused(call, text="", status=P.ERR_INVALID):
    with pytest.raises(P.CocodError) as err:
        P.adamw(None, call)
    assert err.value.status == status and text in str(err.value), str(err.value)


@pytest.mark.parametrize("change, text", [
    (dict(dtype=3), "element type"), (dict(grad_dtype=3), "element type"), (dict(copy_dtype=3), "element type"), (dict(state=2), "state"), (dict(flags=1), "flag"),
    (dict(workers=0), "workers"), (dict(workers=65536), "workers"), (dict(workers=2, stride=999), "overlap"), (dict(workers=2, stride=(1 << 44) + 1), "2^44"),
    (dict(beta1=1.0), "beta"), (dict(beta1=-0.1), "beta"), (dict(beta2=1.0), "beta"), (dict(beta2=float("nan")), "beta"), (dict(eps=-1e-9), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(lr=float("nan")), "lr"), (dict(grad_scale=float("inf")), "grad_scale"), (dict(step=0), "step"), (dict(now=A + 2), "now")])
def test_call_is_checked(change, text):
    refused(adamw(**change), text)


@pytest.mark.parametrize("change, more, text", [
    (dict(p=None), {}, "p is NULL"), (dict(g=None), {}, "g is NULL"), (dict(m=None), {}, "m is NULL"), (dict(v=None), {}, "v is NULL"),
    (dict(p=A + 2), {}, "p is not aligned"), (dict(g=2 * A + 1), dict(grad_dtype=P.BF16), "g is not aligned"), (dict(m=3 * A + 1), {}, "m is not aligned"),
    (dict(n=(1 << 40) + 1), {}, "2^40"), (dict(weight_decay=float("nan")), {}, "weight_decay"), (dict(lr_scale=float("inf")), {}, "lr_scale"),
    (dict(g=A), {}, "p and g overlap"), (dict(v=3 * A + 3996), {}, "m and v overlap"), (dict(m=A + 4), {}, "p and m overlap"),
    (dict(copy=7 * A), dict(copy_dtype=P.F32), "16 bits"), (dict(copy=7 * A), dict(dtype=P.BF16, copy_dtype=P.BF16), "16 bits"),
    (dict(copy=7 * A + 1), dict(copy_dtype=P.BF16), "copy is not aligned"), (dict(copy=A), dict(copy_dtype=P.BF16), "p and copy overlap"),
    (dict(p=8 * A), dict(now=8 * A + 400), "p and now overlap")])
def test_tensors_are_checked(change, more, text):
    refused(adamw([TENSOR, dict(TENSOR, **change)], **more), text)


@pytest.mark.parametrize("change, more, text", [
    (dict(m_scales=None), {}, "m_scales is NULL"), (dict(v_scales=None), {}, "v_scales is NULL"), (dict(v_scales=5 * A + 31), {}, "m_scales and v_scales overlap"),
    (dict(m_scales=3 * A), {}, "m and m_scales overlap"), ({}, dict(workers=2, stride=1008), "multiple of 32")])
def test_states_of_8_bits_are_checked(change, more, text):
    refused(adamw([dict(EIGHT, **change)], state=P.ADAMW_STATE_8BIT, **more), text)


@pytest.mark.parametrize("eps", [1e-45, 5e-39, 1.1754942e-38])
def test_an_eps_below_the_normal_numbers_is_refused(eps):
    refused(adamw(eps=eps), "eps must be 0 or at least 2^-126")
    for fine in (0.0, 2.0 ** -126):
        P.adamw(None, adamw([], eps=fine))


def test_struct_and_null():
    c = adamw()
    c.struct_size += 4
    refused(c, "struct_size")
    assert P.lib().cocod_adamw(None, None) == P.ERR_INVALID
    assert P.lib().cocod_adamw_now_of(C.byref(adamw()), None) == P.ERR_INVALID
    assert P.lib().cocod_adamw_now_of(None, C.byref(P.AdamWNow())) == P.ERR_INVALID
    c = adamw()
    c.tensors = None
    refused(c, "tensors is NULL")
    with pytest.raises(TypeError):
        P.AdamW(tensors=[dict(TENSOR, size=3)])
    with pytest.raises(ValueError):
        P.AdamW(tensors=[dict(TENSOR, n=-1)])
    with pytest.raises(ValueError):
        P.AdamW(seed=1 << 32)


def test_nothing_to_do_needs_no_gpu():
    P.adamw(None, adamw([]))
    P.adamw(None, adamw([dict(n=0), dict(n=0, p=A)]))


@pytest.mark.parametrize("step", [1, 2, 1000, 10 ** 9, 2 ** 63])
@pytest.mark.parametrize("beta1, beta2", [(0.9, 0.999), (0.0, 0.95), (0.99999994, 0.5)])
def test_terms_of_a_step(step, beta1, beta2):
    now = P.adamw_now(adamw(step=step, beta1=beta1, beta2=beta2, seed=7, grad_scale=0.25))
    assert (now.lr, now.grad_scale, now.seed, now.skip) == (C.c_float(1e-3).value, 0.25, 7, 0)
    for got, beta in ((now.bias1, beta1), (now.bias2, beta2)):
        beta = C.c_float(beta).value
        want = 1.0 if beta == 0 else -math.expm1(step * math.log(beta))
        assert abs(got - want) <= 2.0 ** -24 * want


def test_descriptions_match_the_header(tmp_path):
    names = {"cocod_adamw_call": P.AdamW, "cocod_adamw_tensor": P.AdamWTensor, "cocod_adamw_now": P.AdamWNow}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "cocod.h"', "int main(void) {"]
    for name, mirror in names.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f, _ in mirror._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for mirror in names.values():
        want += [C.sizeof(mirror)] + [getattr(mirror, f).offset for f, _ in mirror._fields_]
    assert got == want
