"""Grouped products, vocabulary loss and 8-bit checkpoints on the GPU against plain 64-bit implementations; every output is checked
element by element against a bound derived in operator_harness, and everything around the outputs has to stay as it was."""
import os
import re

import numpy as np
import pytest
import torch

import paper_1906_12043_amd as P
from tests import operator_harness as oh

pytestmark = pytest.mark.gpu


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def close(got, want, bound):
    got = got.to(torch.float64)
    worst = ((got - want).abs() / bound.clamp(min=1e-300)).max().item() if got.numel() else 0.0
    assert bool(((got - want).abs() <= bound).all()), "off by %.3g times the bound" % worst


# ---- checkpoints -------------------------------------------------------------------------------------------

def tricky(dtype, rows, cols, seed):
    r = np.random.default_rng(seed)
    x = r.standard_normal((rows, cols)) * np.exp(r.uniform(-6, 6, (rows, 1)))
    flat = x.reshape(-1)
    special = [0.0, -0.0, 448.0, 449.0, 2.0 ** -9, 1e-9, -3e-8, 6e-8, 1e-30, 464.0, 480.0, 65504.0, -65504.0, 3.3e38, -1e38, 1.2e-38, 1e-40,
               np.inf, -np.inf, np.nan, 17.0, 18.0, 19.0, 1.0625, 1.1875]
    for i, s in enumerate(special):
        flat[(i * 37) % flat.size] = s
    if rows > 2:
        x[1] = 0.0
        x[2] = np.where(np.arange(cols) % 2, 2.0 ** -16, -0.0)
    with np.errstate(over="ignore", invalid="ignore"):
        return torch.from_numpy(x.astype(np.float32)).to(oh.TYPES[dtype][1])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows, cols, pad", [(1, 1, 0), (3, 31, 0), (5, 32, 8), (4, 33, 0), (7, 100, 3), (33, 264, 0), (2, 1000, 24)])
def test_checkpoint_bit_for_bit(dtype, rows, cols, pad):
    kind, t = oh.TYPES[dtype]
    x = tricky(dtype, rows, cols, rows * cols)
    dev = torch.full((rows, cols + pad), 5.0, dtype=t, device="cuda")
    dev[:, :cols] = x.cuda()
    blocks = -(-cols // 32)
    codes = torch.full((rows, cols + pad), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, blocks + 2), 0xAA, dtype=torch.uint8, device="cuda")
    P.checkpoint_store(torch.cuda.current_stream(), kind, rows, cols, dev, cols + pad, codes, cols + pad, scales, blocks + 2)
    want_codes, want_scales = oh.encode(x.to(torch.float64).numpy(), dtype)
    assert np.array_equal(scales[:, :blocks].cpu().numpy(), want_scales)
    assert np.array_equal(codes[:, :cols].cpu().numpy(), want_codes)
    assert bool((codes[:, cols:] == 0xAA).all()) and bool((scales[:, blocks:] == 0xAA).all())
    buf, back = oh.output((rows, cols), pad, t)
    P.checkpoint_load(torch.cuda.current_stream(), kind, rows, cols, codes, cols + pad, scales, blocks + 2, back, cols + pad)
    got, want = back.to(torch.float64).cpu().numpy(), oh.decode(want_codes, want_scales)
    assert np.array_equal(got, want, equal_nan=True) and oh.untouched(buf, back)
    fine = np.isfinite(x.to(torch.float64).numpy())
    assert np.array_equal((got != 0)[fine], (x.to(torch.float64).numpy() != 0)[fine])


def test_checkpoint_of_more_chunks_than_one_launch_has_threads():
    rows, cols = 9, 1 << 28                        # 2.4 G values: offsets beyond 32 bits, and every thread takes two chunks
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, 31, 12345678, cols - 33, cols - 1], device="cuda")
    for r in range(rows):
        x[r, at] = torch.arange(1, 7, device="cuda").to(torch.bfloat16) * (r + 1)
    codes = torch.empty((rows, cols), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, cols // 32), dtype=torch.uint8, device="cuda")
    P.checkpoint_store(torch.cuda.current_stream(), P.BF16, rows, cols, x, cols, codes, cols, scales, cols // 32)
    back = torch.full_like(x, 3.0)
    P.checkpoint_load(torch.cuda.current_stream(), P.BF16, rows, cols, codes, cols, scales, cols // 32, back, cols)
    small = torch.zeros((rows * 6, 32), dtype=torch.bfloat16, device="cuda")
    small[:, 0] = x[:, at].reshape(-1)
    # 0, 1 and 31 share a block and its scale; 1 .. 54 are exact in every scale that 54 or less asks for up to 4 bits
    want_codes, want_scales = oh.encode(small.to(torch.float64).cpu().numpy(), "bf16")
    alone = oh.decode(want_codes, want_scales)[:, 0].reshape(rows, 6)
    assert np.array_equal(back[:, at].to(torch.float64).cpu().numpy(), alone)
    back[:, at] = 0
    assert not bool(back.any())


# ---- products ---------------------------------------------------------------------------------------------

SHAPES = [
    # bounds, rows in memory, inner, outer, pad of every pitch
    ([0, 1], 1, 1, 1, 0),
    ([0, 1, 2, 3, 4], 4, 64, 96, 0),
    ([0, 0, 0], 0, 40, 24, 0),
    ([2, 2, 5, 5, 9], 12, 33, 65, 1),
    ([0, 37, 37, 200], 203, 128, 72, 8),
    ([1, 130, 131, 300], 301, 129, 257, 0),
    ([0, 300, 700], 700, 264, 136, 0),
    ([0, 17, 17, 100, 513], 600, 520, 1032, 8),
    ([0] + [i * 5 % 11 + 11 * i for i in range(1, 70)], 11 * 71, 72, 40, 0),      # more groups than a wave has lanes
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
@pytest.mark.parametrize("workspace", [False, True])
def test_products(dtype, case, workspace):
    bounds, rows, k, n, pad = SHAPES[case]
    gen, t, groups = generator(case), oh.TYPES[dtype][1], len(bounds) - 1
    x, dy = oh.matrix(rows, k, pad, t, gen), oh.matrix(rows, n, pad, t, gen)
    w = oh.stack(groups, k, n, pad, pad, t, gen)
    written = oh.inside(bounds, rows)
    for relu in (False, True):
        buf, y = oh.output((rows, n), pad, t)
        oh.call("forward", oh.layer(dtype, bounds, rows, k, n, x=x, w=w, y=y, flags=P.GROUPED_RELU_OUT if relu else 0), workspace)
        out, mag, terms = oh.exact_product("forward", bounds, x, w)
        close(y[written], (out.clamp(min=0) if relu else out)[written], oh.product_bound(out, mag, terms, t)[written])
        assert oh.untouched(buf, y, written)
        buf, dx = oh.output((rows, k), pad, t)
        oh.call("input_grad", oh.layer(dtype, bounds, rows, k, n, x=x, dy=dy, w=w, dx=dx, flags=P.GROUPED_RELU_IN if relu else 0), workspace)
        out, mag, terms = oh.exact_product("input_grad", bounds, dy, w)
        close(dx[written], (out * (x > 0) if relu else out)[written], oh.product_bound(out, mag, terms, t)[written])
        assert oh.untouched(buf, dx, written)
    for to in {t, torch.float32}:
        buf, dw = oh.output((groups, k, n), pad, to, gap=pad)
        oh.call("weight_grad", oh.layer(dtype, bounds, rows, k, n, x=x, dy=dy, dw=dw), workspace)
        out, mag, terms = oh.exact_product("weight_grad", bounds, x, dy)
        close(dw, out, oh.product_bound(out, mag, terms, to))
        assert oh.untouched(buf, dw)
        empty = [g for g in range(groups) if bounds[g + 1] <= bounds[g]]
        assert not bool(dw[empty].any())


# enough tiles for the largest tile, ragged; and one group with few results and long sums (splits)
LARGE = [([0, 700, 700, 1956, 3000, 5120], 5120, 136, 2568), ([3, 9000], 9001, 200, 56), ([0, 40], 40, 9000, 72), ([0, 9, 12], 12, 4104, 520)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", range(len(LARGE)))
def test_large_tiles_and_splits(dtype, case):
    bounds, rows, k, n = LARGE[case]
    gen, t, groups = generator(100 + case), oh.TYPES[dtype][1], len(bounds) - 1
    x, dy = oh.matrix(rows, k, 0, t, gen), oh.matrix(rows, n, 0, t, gen)
    w = oh.stack(groups, k, n, 0, 0, t, gen)
    written = oh.inside(bounds, rows)
    for workspace in (False, True):
        buf, y = oh.output((rows, n), 0, t)
        oh.call("forward", oh.layer(dtype, bounds, rows, k, n, x=x, w=w, y=y, flags=P.GROUPED_RELU_OUT), workspace)
        out, mag, terms = oh.exact_product("forward", bounds, x, w)
        close(y[written], out.clamp(min=0)[written], oh.product_bound(out, mag, terms, t)[written])
        assert oh.untouched(buf, y, written)
        buf, dx = oh.output((rows, k), 0, t)
        oh.call("input_grad", oh.layer(dtype, bounds, rows, k, n, x=x, dy=dy, w=w, dx=dx, flags=P.GROUPED_RELU_IN), workspace)
        out, mag, terms = oh.exact_product("input_grad", bounds, dy, w)
        close(dx[written], (out * (x > 0))[written], oh.product_bound(out, mag, terms, t)[written])
        assert oh.untouched(buf, dx, written)
        buf, dw = oh.output((groups, k, n), 0, torch.float32)
        oh.call("weight_grad", oh.layer(dtype, bounds, rows, k, n, x=x, dy=dy, dw=dw), workspace)
        out, mag, terms = oh.exact_product("weight_grad", bounds, x, dy)
        close(dw, out, oh.product_bound(out, mag, terms, torch.float32))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("bounds, rows, k, n", [
    ([1, 2999], 3000, 72, 4104), ([1, 2999], 3000, 4104, 72), ([0, 5990], 6000, 72, 136), ([0, 5990], 6000, 136, 72), ([0, 690], 700, 73, 4101),
    ([0, 690], 700, 4101, 73), ([0, 100, 100, 390, 500, 700], 700, 4104, 520), ([0, 100, 100, 390, 500, 700], 700, 2056, 72)])
def test_every_tile(dtype, bounds, rows, k, n):
    """Sizes at which the three tiles are taken in each direction, with operands of whole and of odd rows."""
    gen, t, groups = generator(rows + k), oh.TYPES[dtype][1], len(bounds) - 1
    x, dy, w = oh.matrix(rows, k, 0, t, gen), oh.matrix(rows, n, 0, t, gen), oh.stack(groups, k, n, 0, 0, t, gen)
    written = oh.inside(bounds, rows)
    buf, y = oh.output((rows, n), 0, t)
    oh.call("forward", oh.layer(dtype, bounds, rows, k, n, x=x, w=w, y=y, flags=P.GROUPED_RELU_OUT))
    out, mag, terms = oh.exact_product("forward", bounds, x, w)
    close(y[written], out.clamp(min=0)[written], oh.product_bound(out, mag, terms, t)[written])
    assert oh.untouched(buf, y, written)
    buf, dx = oh.output((rows, k), 0, t)
    oh.call("input_grad", oh.layer(dtype, bounds, rows, k, n, x=x, dy=dy, w=w, dx=dx, flags=P.GROUPED_RELU_IN))
    out, mag, terms = oh.exact_product("input_grad", bounds, dy, w)
    close(dx[written], (out * (x > 0))[written], oh.product_bound(out, mag, terms, t)[written])
    assert oh.untouched(buf, dx, written)
    for to in {t, torch.float32}:
        buf, dw = oh.output((groups, k, n), 0, to)
        oh.call("weight_grad", oh.layer(dtype, bounds, rows, k, n, x=x, dy=dy, dw=dw))
        out, mag, terms = oh.exact_product("weight_grad", bounds, x, dy)
        close(dw, out, oh.product_bound(out, mag, terms, to))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("bounds, rows, wide, summed", [
    ([3, 195, 195, 900, 1092, 1993], 2000, 2056, 520), ([1, 1999], 2000, 2056, 520),              # rows of 192
    ([0, 1, 600, 600, 1700, 2999], 3000, 4104, 392), ([0, 100, 100, 390, 500, 700], 700, 2056, 392)])      # the large tile; four slices in flight
@pytest.mark.parametrize("direction", ["forward", "input_grad"])
@pytest.mark.parametrize("pad", [8, 3])
def test_rows_in_tiles_of_several_slices(dtype, bounds, rows, wide, summed, direction, pad):
    """The 16-bit tiles for many rows, with sums of several slices and a part of one: groups of exactly one tile, of a part of one, of none."""
    k, n = (summed, wide) if direction == "forward" else (wide, summed)
    gen, t, groups = generator(len(bounds)), oh.TYPES[dtype][1], len(bounds) - 1
    x, dy, w = oh.matrix(rows, k, 0, t, gen), oh.matrix(rows, n, 0, t, gen), oh.stack(groups, k, n, 0, 0, t, gen)
    written = oh.inside(bounds, rows)
    buf, got = oh.output((rows, wide), pad, t)
    if direction == "forward":
        oh.call("forward", oh.layer(dtype, bounds, rows, k, n, x=x, w=w, y=got, flags=P.GROUPED_RELU_OUT))
        out, mag, terms = oh.exact_product("forward", bounds, x, w)
        want = out.clamp(min=0)
    else:
        oh.call("input_grad", oh.layer(dtype, bounds, rows, k, n, x=x, dy=dy, w=w, dx=got, flags=P.GROUPED_RELU_IN))
        out, mag, terms = oh.exact_product("input_grad", bounds, dy, w)
        want = out * (x > 0)
    close(got[written], want[written], oh.product_bound(out, mag, terms, t)[written])
    assert oh.untouched(buf, got, written)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", [0, 1, 3, 4, 5, 7])
def test_products_from_codes(dtype, case):
    bounds, rows, k, n, pad = SHAPES[case]
    gen, (kind, t), groups = generator(case + 50), oh.TYPES[dtype], len(bounds) - 1
    x, dy = torch.relu(oh.matrix(rows, k, pad, t, gen)), oh.matrix(rows, n, pad, t, gen)
    w = oh.stack(groups, k, n, 0, 0, t, gen)
    blocks = -(-k // 32)
    codes = torch.full((rows, k + pad), 0x7f, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, blocks + pad), 0xff, dtype=torch.uint8, device="cuda")
    P.checkpoint_store(torch.cuda.current_stream(), kind, rows, k, x, x.stride(0), codes, k + pad, scales, blocks + pad)
    back = torch.empty((rows, k), dtype=t, device="cuda")
    P.checkpoint_load(torch.cuda.current_stream(), kind, rows, k, codes, k + pad, scales, blocks + pad, back, k)
    buf, dw = oh.output((groups, k, n), pad, torch.float32)
    oh.call("weight_grad", oh.layer(dtype, bounds, rows, k, n, x_codes=codes[:, :k], x_scales=scales[:, :blocks], dy=dy, dw=dw))
    out, mag, terms = oh.exact_product("weight_grad", bounds, back, dy)
    close(dw, out, oh.product_bound(out, mag, terms, torch.float32))
    assert oh.untouched(buf, dw)
    # the relu's mask survives in the codes: the same input gradient, bit for bit
    masks = dict(x=x), dict(x_codes=codes[:, :k], x_scales=scales[:, :blocks])
    got = []
    for m in masks:
        buf, dx = oh.output((rows, k), pad, t)
        oh.call("input_grad", oh.layer(dtype, bounds, rows, k, n, dy=dy, w=w, dx=dx, flags=P.GROUPED_RELU_IN, **m))
        got.append(buf)
    assert torch.equal(got[0], got[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_not_finite_and_extreme_operands(dtype):
    """Infinities and NaN reach exactly the results they belong to; the smallest and largest numbers of the type keep their accuracy."""
    t, gen = oh.TYPES[dtype][1], generator(7)
    bounds, rows, k, n = [0, 70, 140], 150, 96, 80
    x, w = oh.matrix(rows, k, 0, t, gen), oh.stack(2, k, n, 0, 0, t, gen)
    x[3, 5], x[75, 0], x[80, 7] = float("inf"), float("-inf"), float("nan")
    x[145] = float("nan")                          # behind the last group
    w[1, 3, 4] = float("inf")
    buf, y = oh.output((rows, n), 0, t)
    oh.call("forward", oh.layer(dtype, bounds, rows, k, n, x=x, w=w, y=y))
    want = torch.cat([x[:70].double() @ w[0].double(), x[70:140].double() @ w[1].double()])
    got = y[:140].double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isinf(got), torch.isinf(want)) and torch.equal(got[torch.isinf(got)], want[torch.isinf(want)])
    assert oh.untouched(buf, y, oh.inside(bounds, rows))
    # powers of two times small whole numbers: every product and sum is exact in fp32, so the result is exact
    lo, hi = {"bf16": (-100, 60), "fp16": (-14, 6), "fp32": (-120, 60)}[dtype]
    r = torch.randint(-3, 4, (rows, k), generator=gen, device="cuda").double()
    for a, b in ((lo, 10), (hi, 0), (lo + 1, hi)) if dtype != "fp16" else ((lo, 6), (hi, 0)):
        xs, ws = (r * 2.0 ** a).to(t), (torch.sign(torch.randn(1, k, n, generator=gen, device="cuda")).double() * 2.0 ** b).to(t)
        y = torch.empty((rows, n), dtype=torch.float32 if dtype == "fp32" else t, device="cuda")
        oh.call("forward", oh.layer(dtype, [0, rows], rows, k, n, x=xs, w=ws, y=y))
        assert torch.equal(y, (xs.double() @ ws[0].double()).to(t)), (a, b)


@pytest.mark.parametrize("dtype, lo, up", [("fp16", -24, 10), ("bf16", -133, 60), ("fp32", -149, 60)])
def test_subnormal_operands_and_results(dtype, lo, up):
    """The smallest numbers of a type, whose sums fp32 holds exactly, are neither lost as operands nor as results."""
    t, gen, rows, k, n = oh.TYPES[dtype][1], generator(11), 150, 96, 80
    r = torch.randint(-1, 2, (rows, k), generator=gen, device="cuda").double()
    sign = torch.sign(torch.randn(1, k, n, generator=gen, device="cuda")).double()
    for a, b in ((lo, up), (0, lo)):
        x, w = (r * 2.0 ** a).to(t), (sign * 2.0 ** b).to(t)
        y = torch.empty((rows, n), dtype=t, device="cuda")
        oh.call("forward", oh.layer(dtype, [0, rows], rows, k, n, x=x, w=w, y=y))
        assert bool(x.any()) and bool(w.any()) and torch.equal(y, (x.double() @ w[0].double()).to(t)), (a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("width", list(range(129, 137)) + [7, 9, 1023])
def test_widths_that_cut_a_chunk(dtype, width):
    """Rows of every length modulo 8, both as the axis that is summed over and as the one that is not; rows before, between and
    behind the groups; and the same layer with its activations in codes."""
    (kind, t), gen, bounds, rows = oh.TYPES[dtype], generator(width), [1, 60, 60, 205], 207
    other = 136
    for k, n in ((width, other), (other, width), (width, width)):
        x, dy, w = oh.matrix(rows, k, 0, t, gen), oh.matrix(rows, n, 0, t, gen), oh.stack(3, k, n, 0, 0, t, gen)
        written = oh.inside(bounds, rows)
        buf, y = oh.output((rows, n), 0, t)
        oh.call("forward", oh.layer(dtype, bounds, rows, k, n, x=x, w=w, y=y))
        out, mag, terms = oh.exact_product("forward", bounds, x, w)
        close(y[written], out[written], oh.product_bound(out, mag, terms, t)[written])
        assert oh.untouched(buf, y, written)
        buf, dx = oh.output((rows, k), 0, t)
        oh.call("input_grad", oh.layer(dtype, bounds, rows, k, n, x=x, dy=dy, w=w, dx=dx, flags=P.GROUPED_RELU_IN))
        out, mag, terms = oh.exact_product("input_grad", bounds, dy, w)
        close(dx[written], (out * (x > 0))[written], oh.product_bound(out, mag, terms, t)[written])
        codes = torch.empty((rows, k), dtype=torch.uint8, device="cuda")
        scales = torch.empty((rows, -(-k // 32)), dtype=torch.uint8, device="cuda")
        P.checkpoint_store(torch.cuda.current_stream(), kind, rows, k, x, k, codes, k, scales, scales.shape[1])
        back = torch.empty_like(x)
        P.checkpoint_load(torch.cuda.current_stream(), kind, rows, k, codes, k, scales, scales.shape[1], back, k)
        for source, value in ((dict(x=x), x), (dict(x_codes=codes, x_scales=scales), back)):
            buf, dw = oh.output((3, k, n), 0, torch.float32)
            oh.call("weight_grad", oh.layer(dtype, bounds, rows, k, n, dy=dy, dw=dw, **source))
            out, mag, terms = oh.exact_product("weight_grad", bounds, value, dy)
            close(dw, out, oh.product_bound(out, mag, terms, torch.float32))
            assert oh.untouched(buf, dw)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("bounds, rows, k, n", [([0, 900, 2100, 4000], 4000, 1304, 2568), ([5, 900, 2100, 4000], 4010, 1313, 2571), ([0, 3000], 3000, 96, 40), ([0, 2999], 3001, 65, 33)])
def test_codes_in_every_tile(dtype, bounds, rows, k, n):
    (kind, t), gen = oh.TYPES[dtype], generator(rows)
    x, dy = torch.relu(oh.matrix(rows, k, 0, t, gen)), oh.matrix(rows, n, 0, t, gen)
    codes = torch.empty((rows, k), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, -(-k // 32)), dtype=torch.uint8, device="cuda")
    P.checkpoint_store(torch.cuda.current_stream(), kind, rows, k, x, k, codes, k, scales, scales.shape[1])
    back = torch.empty_like(x)
    P.checkpoint_load(torch.cuda.current_stream(), kind, rows, k, codes, k, scales, scales.shape[1], back, k)
    for workspace in (False, True):
        dw = torch.empty((len(bounds) - 1, k, n), device="cuda")
        oh.call("weight_grad", oh.layer(dtype, bounds, rows, k, n, dy=dy, dw=dw, x_codes=codes, x_scales=scales), workspace)
        out, mag, terms = oh.exact_product("weight_grad", bounds, back, dy)
        close(dw, out, oh.product_bound(out, mag, terms, torch.float32))


def test_thousands_of_groups():
    t, gen, groups, k, n = torch.bfloat16, generator(12), 5000, 24, 40
    length = torch.randint(0, 4, (groups,), generator=gen, device="cuda")
    bounds = [0] + torch.cumsum(length, 0).tolist()
    rows = bounds[-1]
    x, dy, w = oh.matrix(rows, k, 0, t, gen), oh.matrix(rows, n, 0, t, gen), oh.stack(groups, k, n, 0, 0, t, gen)
    group = torch.repeat_interleave(torch.arange(groups, device="cuda"), length)
    y, dw = torch.empty((rows, n), dtype=t, device="cuda"), torch.empty((groups, k, n), device="cuda")
    oh.call("forward", oh.layer("bf16", bounds, rows, k, n, x=x, w=w, y=y))
    oh.call("weight_grad", oh.layer("bf16", bounds, rows, k, n, x=x, dy=dy, dw=dw))
    wide = w.double()[group]
    out = (x.double()[:, :, None] * wide).sum(1)
    close(y, out, oh.product_bound(out, (x.double()[:, :, None] * wide).abs().sum(1), k, t))
    each = x.double()[:, :, None] * dy.double()[:, None, :]
    out, mag = torch.zeros((groups, k, n), dtype=torch.float64, device="cuda"), torch.zeros((groups, k, n), dtype=torch.float64, device="cuda")
    out.index_add_(0, group, each)
    mag.index_add_(0, group, each.abs())
    close(dw, out, oh.product_bound(out, mag, 4, torch.float32))


def test_gradients_of_a_layer_against_differences():
    """f(x, w) = <x w, dy> is linear in either argument: differences are exact but for rounding.  fp32, |f| below 100: each value of f is a float64
    sum of fp32 results off by at most 72 2^-23 sum |x w| |dy| < 2e-3 at a step of one, so a quotient by 2e-3, and <dx, d> as much."""
    gen, t, bounds, rows, k, n = generator(13), torch.float32, [0, 20, 50], 50, 64, 48
    x, dy, w = oh.matrix(rows, k, 0, t, gen, 0.3), oh.matrix(rows, n, 0, t, gen, 0.3), oh.stack(2, k, n, 0, 0, t, gen, 0.3)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    oh.call("input_grad", oh.layer("fp32", bounds, rows, k, n, dy=dy, w=w, dx=dx))
    oh.call("weight_grad", oh.layer("fp32", bounds, rows, k, n, x=x, dy=dy, dw=dw))

    def f(xx, ww):
        y = torch.empty((rows, n), device="cuda")
        oh.call("forward", oh.layer("fp32", bounds, rows, k, n, x=xx, w=ww, y=y))
        return (y.double() * dy.double()).sum().item()

    for _ in range(3):
        d = torch.randn(rows, k, generator=gen, device="cuda") * 0.3
        assert abs((f(x + d, w) - f(x - d, w)) / 2 - (dx.double() * d.double()).sum().item()) < 4e-3
        d = torch.randn(2, k, n, generator=gen, device="cuda") * 0.3
        assert abs((f(x, w + d) - f(x, w - d)) / 2 - (dw.double() * d.double()).sum().item()) < 4e-3


def test_shared_weights_pitches_and_offsets_beyond_32_bits():
    t, gen = torch.bfloat16, generator(8)
    bounds, rows, k, n, pitch = [0, 3, 1030, 1040], 1040, 64, 48, 1 << 22         # 4.4 G elements from first to last row
    big = torch.empty((rows, pitch), dtype=t, device="cuda")
    x = big[:, :k]
    x.copy_(torch.randn(rows, k, generator=gen, device="cuda"))
    w = oh.stack(1, k, n, 0, 0, t, gen)
    y = big[:, pitch - n:]
    lay = oh.layer("bf16", bounds, rows, k, n, x=x, w=w.expand(3, k, n))
    lay.set(w_stride=0, ldw=n, y=y, ldy=pitch)
    # x and y lie interleaved in one buffer: their extents overlap, and the call says so
    with pytest.raises(P.CocodError):
        P.grouped_forward(torch.cuda.current_stream(), lay)
    y = torch.empty((rows, n), dtype=t, device="cuda")
    lay.set(y=y, ldy=n)
    P.grouped_forward(torch.cuda.current_stream(), lay)
    out, mag, terms = oh.exact_product("forward", bounds, x, w.expand(3, k, n))
    close(y, out, oh.product_bound(out, mag, terms, t))
    dw = torch.empty((3, k, n), device="cuda")
    dy = oh.matrix(rows, n, 0, t, gen)
    oh.call("weight_grad", oh.layer("bf16", bounds, rows, k, n, x=x, dy=dy, dw=dw))
    out, mag, terms = oh.exact_product("weight_grad", bounds, x, dy)
    close(dw, out, oh.product_bound(out, mag, terms, torch.float32))
    # one element more of pitch: no operand goes to LDS directly any more
    x = big.view(-1)[: (rows - 1) * (pitch + 1)].as_strided((rows - 1, k), (pitch + 1, 1))
    x.copy_(torch.randn(rows - 1, k, generator=gen, device="cuda"))
    y = torch.empty((rows - 1, n), dtype=t, device="cuda")
    oh.call("forward", oh.layer("bf16", [5, 1039], rows - 1, k, n, x=x, w=w, y=y))
    out, mag, terms = oh.exact_product("forward", [5, 1039], x, w)
    close(y[5:], out[5:], oh.product_bound(out, mag, terms, t)[5:])


def test_offsets_that_do_not_ascend_leave_the_arrays_alone_outside():
    t, gen, rows, k, n = torch.bfloat16, generator(9), 300, 64, 64
    x, w = oh.matrix(rows, k, 0, t, gen), oh.stack(4, k, n, 0, 0, t, gen)
    for bounds in ([0, 250, 10, 400, 300], [-5, 1 << 40, -(1 << 40), 7, 1 << 62], [300, 200, 100, 50, 0], [1 << 62] * 5, [-1] * 5):
        buf, y = oh.output((rows, n), 8, t)
        oh.call("forward", oh.layer("bf16", bounds, rows, k, n, x=x, w=w, y=y), True)
        assert bool((buf[:, n:] == oh.SENTINEL).all())
        buf, dw = oh.output((4, k, n), 8, t)
        oh.call("weight_grad", oh.layer("bf16", bounds, rows, k, n, x=x, dy=x[:, :n], dw=dw), True)
        assert oh.untouched(buf, dw)
        target = torch.randint(0, k, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        loss = torch.zeros(rows, device="cuda")
        dh, de = torch.zeros_like(x), torch.zeros_like(w)
        P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call("bf16", bounds, x, w, target, loss=loss, dh=dh, de=de))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [64, 1000])
@pytest.mark.parametrize("grads", [True, False])
def test_loss_of_groups_that_share_rows(dtype, dim, grads):
    """Offsets that do not ascend make groups share rows.  Groups of rows without a target beside long ones with most of theirs: their blocks mark
    the shared rows as gathered from nowhere while others gather them.  Results are undefined; nothing outside the arrays is touched.  With
    64 columns a group's block gathers its rows itself, with 1000 a launch of its own does."""
    t, gen, rows, vocab = oh.TYPES[dtype][1], generator(19), 300, 130
    bounds = [0, 250, 10, 12, 5, 300, 0, 300, 20, 22, 290, 3, 200, 100, 150, 40, 260, 10, 12, 0, 300]
    groups = len(bounds) - 1
    h, e = oh.matrix(rows, dim, 0, t, gen), oh.stack(1, vocab, dim, 0, 0, t, gen, std=dim ** -0.5).expand(groups, vocab, dim)
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    target[10:12], target[20:22], target[100:150:2], target[280:] = -100, vocab, -1, -1
    lbuf, loss = oh.output((1, rows), 3, torch.float32)
    hbuf, dh = oh.output((rows, dim), 8, t)
    ebuf, de = oh.output((groups, vocab, dim), 8, t)
    c = oh.cross_entropy_call(dtype, bounds, h, e, target, dh if grads else None, de if grads else None, None, loss)
    for _ in range(5):
        P.cross_entropy(torch.cuda.current_stream(), c)
    torch.cuda.synchronize()
    assert lbuf[0, rows:].tolist() == [oh.SENTINEL] * 3 and oh.untouched(hbuf, dh) and oh.untouched(ebuf, de)


# ---- loss ---------------------------------------------------------------------------------------------------

LOSSES = [
    # bounds, rows, dim, vocab, pad, piece, share of rows without a target
    ([0, 1], 1, 1, 1, 0, 0, 0.0),
    ([0, 1], 1, 24, 100, 0, 0, 0.0),
    ([0, 0], 0, 16, 40, 0, 0, 0.0),
    ([0, 3, 3, 20], 25, 33, 77, 1, 0, 0.4),
    ([2, 66, 130], 130, 64, 1000, 0, 256, 0.2),
    ([0, 200, 200, 333], 340, 120, 517, 8, 256, 0.1),
    ([0, 257], 257, 200, 2049, 0, 600, 0.5),
    ([0, 5, 10], 10, 40, 300, 0, 0, 1.0),
    ([0, 1500, 2100], 2100, 72, 5000, 0, 0, 0.05),
    ([3, 300], 310, 203, 3001, 0, 1024, 0.0),
    ([0, 10, 700, 2900, 4000], 4000, 136, 2000, 8, 1024, 0.3),
    # the large tile; the medium one, and it with odd rows
    ([1, 2999], 3000, 72, 4104, 0, 0, 0.1),
    ([0, 5990], 6000, 72, 136, 0, 0, 0.1),
    ([0, 690], 700, 73, 4101, 0, 0, 0.1),
    # four slices in flight, all at once and by pieces; the large tile with sums of several slices, the same; pieces with odd rows
    ([0, 100, 100, 390, 500, 700], 700, 264, 2056, 0, 0, 0.1),
    ([2, 400, 700], 700, 264, 5000, 0, 2560, 0.2),
    ([1, 1000, 2999], 3000, 264, 4104, 0, 0, 0.1),
    ([0, 1100, 3000], 3000, 264, 8200, 0, 4352, 0.1),
    ([0, 1200, 2500], 2500, 203, 4104, 0, 2304, 0.1),
]


def loss_inputs(dtype, case):
    bounds, rows, dim, vocab, pad, piece, out = LOSSES[case]
    gen, t, groups = generator(200 + case), oh.TYPES[dtype][1], len(bounds) - 1
    h, e = oh.matrix(rows, dim, pad, t, gen), oh.stack(groups, vocab, dim, pad, pad, t, gen, std=3.0 / dim ** 0.5)
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    gone = torch.rand(rows, generator=gen, device="cuda") < out
    target[gone] = torch.where(torch.arange(rows, device="cuda", dtype=torch.int32)[gone] % 2 == 0, -100, vocab).int()
    h[gone] = float("nan")                         # nothing of a row without a target is used
    return bounds, rows, dim, vocab, pad, piece, t, groups, h, e, target


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", range(len(LOSSES)))
@pytest.mark.parametrize("total", [False, True])
def test_loss_and_gradients(dtype, case, total):
    bounds, rows, dim, vocab, pad, piece, t, groups, h, e, target = loss_inputs(dtype, case)
    scale = 0.5 if total else 3.0
    want = oh.exact_loss(bounds, h, e, target, total, scale)
    bound = oh.loss_bounds(want, t, dim, vocab)
    written = oh.inside(bounds, rows)
    lbuf, loss = oh.output((1, rows), 3, torch.float32)
    gbuf, group_loss = oh.output((1, groups), 1, torch.float32)
    hbuf, dh = oh.output((rows, dim), pad, t)
    ebuf, de = oh.output((groups, vocab, dim), pad, t, gap=pad)
    c = oh.cross_entropy_call(dtype, bounds, h, e, target, dh, de, group_loss, loss, grad_scale=scale, piece=piece,
                              flags=P.CROSS_ENTROPY_SUM if total else 0)
    P.cross_entropy(torch.cuda.current_stream(), c)
    close(loss[0][written], want["loss"][written], bound["loss"][written])
    for g, s in oh.groups_of(bounds):
        n = int(((target[s] >= 0) & (target[s] < vocab)).sum())
        far = bound["loss"][s].sum() / (1 if total else max(n, 1)) + oh.STEP * want["group_loss"][g].abs()
        assert abs(group_loss[0, g].double() - want["group_loss"][g]) <= far
    close(dh[written], want["dh"][written], bound["dh"][written])
    close(de, want["de"], bound["de"])
    assert oh.untouched(hbuf, dh, written) and oh.untouched(ebuf, de)
    assert lbuf[0, rows:].tolist() == [oh.SENTINEL] * 3
    assert bool((loss[0][~written] == oh.SENTINEL).all())
    assert float(gbuf[0, groups]) == oh.SENTINEL
    # the loss alone, and one gradient alone, have the same bits
    only = torch.empty(rows, device="cuda")
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, loss=only))
    assert torch.equal(only[written], loss[0][written])
    one = torch.empty((rows, dim), dtype=t, device="cuda")
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, loss=only, dh=one, grad_scale=scale, piece=piece,
                                                                       flags=P.CROSS_ENTROPY_SUM if total else 0))
    assert torch.equal(one[written], dh[written])
    table = torch.empty_like(e)
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, loss=only, de=table, grad_scale=scale, piece=piece,
                                                                       flags=P.CROSS_ENTROPY_SUM if total else 0))
    assert torch.equal(table, de)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("bounds, rows, dim, vocab", [([2, 40, 40, 60, 71], 80, 64, 130), ([0, 200], 200, 264, 1000), ([0, 1], 1, 8, 1), ([5, 20, 30], 33, 128, 2500)])
@pytest.mark.parametrize("pad", [0, 8, 1])
@pytest.mark.parametrize("total", [False, True])
def test_loss_alone_of_few_rows(dtype, bounds, rows, dim, vocab, pad, total):
    """Without gradients: rows without a target between the others, a group without any, targets beside the vocabulary and at the ends of their type."""
    gen, t, groups = generator(rows + dim), oh.TYPES[dtype][1], len(bounds) - 1
    h, e = oh.matrix(rows, dim, pad, t, gen), oh.stack(groups, vocab, dim, pad, pad, t, gen, std=3.0 / dim ** 0.5)
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    for i, none in enumerate((-1, vocab, vocab + 1, -2 ** 31, 2 ** 31 - 1, -100)):
        if rows > 1:
            target[bounds[0] + 1 + 3 * i % (bounds[1] - bounds[0])] = none
    if groups > 1:
        target[bounds[-2]:bounds[-1]] = -100
    h[(target < 0) | (target >= vocab)] = float("nan")
    want = oh.exact_loss(bounds, h, e, target, total, 1.0)
    bound = oh.loss_bounds(want, t, dim, vocab)
    written = oh.inside(bounds, rows)
    lbuf, loss = oh.output((1, rows), 3, torch.float32)
    gbuf, group_loss = oh.output((1, groups), 1, torch.float32)
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, group_loss=group_loss, loss=loss,
                                                                       flags=P.CROSS_ENTROPY_SUM if total else 0))
    close(loss[0][written], want["loss"][written], bound["loss"][written])
    for g, s in oh.groups_of(bounds):
        n = int(((target[s] >= 0) & (target[s] < vocab)).sum())
        far = bound["loss"][s].sum() / (1 if total else max(n, 1)) + oh.STEP * want["group_loss"][g].abs()
        assert abs(group_loss[0, g].double() - want["group_loss"][g]) <= far
    assert lbuf[0, rows:].tolist() == [oh.SENTINEL] * 3 and bool((loss[0][~written] == oh.SENTINEL).all())
    assert float(gbuf[0, groups]) == oh.SENTINEL


def test_loss_of_as_many_rows_as_are_allowed():
    """2^26 - 1 rows: a wave a row would be 2^32 threads.  Two logits a row, exact in fp32: the loss is log1p(e^-x) of their difference x, below 8, to
    the exponential's (x + 2) steps, one of the logarithm, and one of each rounding: 16 steps of the loss."""
    rows, gen = (1 << 26) - 1, generator(31)
    h = torch.zeros((rows, 8), dtype=torch.bfloat16, device="cuda")
    h[:, 0] = (torch.randint(-64, 65, (rows,), generator=gen, device="cuda", dtype=torch.int32) / 16).to(torch.bfloat16)
    e = torch.zeros((1, 2, 8), dtype=torch.bfloat16, device="cuda")
    e[0, 0, 0], e[0, 1, 0] = 1.0, -1.0
    target = torch.arange(rows, device="cuda", dtype=torch.int32) % 5 - 1            # -1, 0, 1 and two beside the vocabulary
    loss, mean = torch.full((rows,), oh.SENTINEL, device="cuda"), torch.empty(1, device="cuda")
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call("bf16", [1, rows - 1], h, e, target, group_loss=mean, loss=loss))
    assert float(loss[0]) == oh.SENTINEL and float(loss[-1]) == oh.SENTINEL
    total, count = 0.0, 0
    for part in torch.arange(1, rows - 1, device="cuda").split(1 << 23):
        x = 2 * h[part, 0].double() * torch.where(target[part] == 0, 1.0, -1.0)
        want = torch.log1p(torch.exp(-x.abs())) + torch.clamp(-x, min=0)
        has = (target[part] == 0) | (target[part] == 1)
        want = torch.where(has, want, torch.zeros_like(want))
        close(loss[part], want, 16 * oh.STEP * want)
        total, count = total + want.sum().item(), count + int(has.sum())
    assert abs(mean.item() - total / count) <= 17 * oh.STEP * total / count


def test_loss_without_rows_of_groups_whose_tiles_no_launch_would_hold():
    """65535 groups by 200000 entries would be 2^27 tiles at the least, a tile begun per group; without rows there is no such product."""
    groups, vocab, dim = 65535, 200000, 8
    e = torch.zeros((1, vocab, dim), dtype=torch.bfloat16, device="cuda").expand(groups, vocab, dim)
    mean = torch.full((groups,), oh.SENTINEL, device="cuda")
    empty = torch.empty((0, dim), dtype=torch.bfloat16, device="cuda")
    call = oh.cross_entropy_call("bf16", [0] * (groups + 1), empty, e, torch.empty(0, dtype=torch.int32, device="cuda"), group_loss=mean, loss=torch.empty(0, device="cuda"))
    P.cross_entropy(torch.cuda.current_stream(), call)
    call.set(dh=torch.empty(16, dtype=torch.bfloat16, device="cuda"), lddh=dim)
    P.cross_entropy(torch.cuda.current_stream(), call)
    assert not bool(mean.any())


def test_loss_gradient_against_differences():
    """(L(h + s d) - L(h - s d)) / 2 s against <dh, d>, and the same for the table.  L in fp32 is off by the bound r of each row's loss, here
    below 4e-6; at s = 2^-6 that is 2.6e-4 in the quotient; the cubic term is s^2 / 6 max |L'''| |d . e|^3, with |d . e| <= 1 and
    |L'''| <= 1 below 4.1e-5."""
    dtype, bounds, rows, dim, vocab = "fp32", [0, 30, 64], 64, 32, 300
    gen, t = generator(5), torch.float32
    h, e = oh.matrix(rows, dim, 0, t, gen), oh.stack(2, vocab, dim, 0, 0, t, gen, std=2.0 / dim ** 0.5)
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    loss, mean = torch.empty(rows, device="cuda"), torch.empty(2, device="cuda")
    dh, de = torch.empty_like(h), torch.empty_like(e)
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, dh, de, mean, loss))

    def at(hh, ee):
        m = torch.empty(2, device="cuda")
        P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, hh, ee, target, loss=torch.empty(rows, device="cuda"), group_loss=m))
        return m.double().sum().item()

    s = 2.0 ** -6
    for _ in range(4):
        d = torch.randn(rows, dim, generator=gen, device="cuda")
        d /= torch.cat([(d[a:b] @ e[g].t()).abs().amax() * torch.ones(b - a, 1, device="cuda") for g, (a, b) in enumerate(((0, 30), (30, 64)))])
        assert abs((at(h + s * d, e) - at(h - s * d, e)) / (2 * s) - (dh * d).sum().item()) < 3.1e-4
        d = torch.randn(2, vocab, dim, generator=gen, device="cuda")
        d /= max((h[:30] @ d[0].t()).abs().amax(), (h[30:] @ d[1].t()).abs().amax())
        assert abs((at(h, e + s * d) - at(h, e - s * d)) / (2 * s) - (de * d).sum().item()) < 3.1e-4


def test_loss_with_a_shared_table_and_infinite_logits():
    t, gen, rows, dim, vocab = torch.bfloat16, generator(6), 40, 32, 200
    h, e = oh.matrix(rows, dim, 0, t, gen), oh.stack(1, vocab, dim, 0, 0, t, gen)
    h[:, 0], e[0, :, 0] = 1.0, 0.0
    e[0, 50:60, 0] = float("-inf")                 # entries that no row can choose: probability and slope zero
    target = torch.randint(0, 50, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    target[7] = 55                                 # the loss of an impossible target is infinite
    loss, dh, de = torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty((2, vocab, dim), dtype=t, device="cuda")
    two = e.expand(2, vocab, dim)
    c = oh.cross_entropy_call("bf16", [0, 8, rows], h, two, target, None, de, None, loss)
    P.cross_entropy(torch.cuda.current_stream(), c)
    z = h.double() @ torch.where(torch.isinf(e[0]), torch.zeros_like(e[0]), e[0]).double().t()
    z[:, 50:60] = -float("inf")
    want = torch.logsumexp(z, 1) - z[torch.arange(rows), target.long()]
    assert bool(torch.isposinf(loss[7]))
    keep = torch.arange(rows, device="cuda") != 7
    # logits off by (dim + 8) 2^-23 sum |h e| <= 40 * 2^-23 * 200 < 1e-3 for these inputs
    assert float((loss.double() - want)[keep].abs().max()) < 1e-3
    assert bool(torch.isfinite(de).all()) and not bool(de[1, 50:60].any())


# rows, dim, vocab, pad, piece: few rows (waves that share the terms), rows off 16 bytes, the larger tiles, one piece and several
CONFIDENT = [(40, 16, 700, 0, 0), (40, 16, 700, 0, 256), (41, 13, 700, 0, 256), (700, 264, 5000, 0, 0), (700, 16, 5000, 8, 2560), (2999, 72, 4104, 0, 1024)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", range(len(CONFIDENT)))
def test_confident_rows_keep_their_digits(dtype, case):
    """Rows whose target is almost certain, with logits of up to 600: loss and slopes to a relative bound that knows no size of the logits.

    Every logit is a sum of two products of a few bits, exact in fp32.  x = z - (a maximum) is then exact, too; an exponential of it is off by
    (|x| + 2) 2^-23 of itself, and what is below e^-90 of the largest of all does not count (2^-120, and the exponentials between the passes below).  Up
    to three factors of that kind, with the 300 + vocab / 64 additions of the others' sum: a slope, the sum of the others relative to the target and with it a loss
    below one are off by rel = (3 * 92 + 300 + vocab / 64) 2^-23, a loss above by its own roundings, too: 8 steps in all.  Slopes: half a step of a 16-bit type
    (fp16: not below steps of 2^-38); bf16 exponentials between the passes: 2^-11, not below steps of 2^-38 of their tile's largest.  Then the products.
    """
    rows, dim, vocab, pad, piece = CONFIDENT[case]
    t, gen = oh.TYPES[dtype][1], generator(400 + case)
    u, f = oh.half_step(t), torch.float64
    sure = torch.tensor([0, vocab // 2 + 5, vocab - 1], device="cuda")                     # entries that rows are sure of: in the first tile, within, in the last
    h, e = oh.matrix(rows, dim, pad, t, gen), oh.stack(1, vocab, dim, pad, 0, t, gen)
    h.zero_()
    e.zero_()
    e[0, :, :3] = torch.randint(-16, 17, (vocab, 3), generator=gen, device="cuda").to(t) / 8
    e[0, sure] = 0.0
    for i in range(3):
        e[0, sure[i], i] = 4.0
        e[0, sure[i], 4 + i] = 1.0                                                          # dh shows the slope of this entry by itself
    e[0, :, 3] = 1.0                                                                        # the size of all logits; dh shows the sum of all slopes
    e[0, :, 7] = 1.0
    e[0, sure, 7] = 0.0                                                                     #   and of the others'
    who = torch.arange(rows, device="cuda") % 3
    gaps = torch.tensor([1.0, 2.0, 3.0, 5.0, 7.0, 12.0, 30.0], device="cuda")
    h[torch.arange(rows), who] = gaps[torch.arange(rows, device="cuda") // 3 % 7].to(t)
    h[:, 3] = torch.tensor([0.0, 40.0, -100.0, 480.0], device="cuda")[torch.arange(rows, device="cuda") // 21 % 4].to(t)
    target = sure[who].int()
    target[5::11] = torch.randint(0, vocab, (len(target[5::11]),), generator=gen, device="cuda", dtype=torch.int32)       # and some that are wrong
    z = h.to(f) @ e[0].to(f).t()
    at = torch.arange(rows, device="cuda")
    ratio = torch.exp(z - z[at, target.long()][:, None])                                    # to the target's exponential
    ratio[at, target.long()] = 0.0
    others = ratio.sum(1)
    want = torch.log1p(others)
    dz = ratio / (1 + others)[:, None]
    dz[at, target.long()] = -others / (1 + others)
    rel = (3 * 92 + 300 + vocab / 64) * oh.STEP
    scale = 1.0 if dtype == "fp16" else 1024.0                                              # (the table's gradient stays within fp16)
    for grads in (True, False):
        loss, (hbuf, dh), (ebuf, de) = torch.empty(rows, device="cuda"), oh.output((rows, dim), pad, t), oh.output((1, vocab, dim), pad, t)
        mean = torch.empty(1, device="cuda")
        P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, [0, rows], h, e, target, dh if grads else None, de if grads else None, mean,
                                                                           loss, piece=piece, flags=P.CROSS_ENTROPY_SUM, grad_scale=scale))
        close(loss, want, (rel + 8 * oh.STEP) * want + 2.0 ** -120)
        assert abs(mean.double() - want.sum()) <= (rel + 9 * oh.STEP) * want.sum()
        if grads:
            off = dz.abs() * (rel + 8 * oh.STEP + (u if t != torch.float32 else 0.0) + (2.0 ** -11 if dtype == "bf16" else 0.0)) + 2.0 ** -120
            off += {"bf16": 2.0 ** -39, "fp16": 2.0 ** -39, "fp32": 0.0}[dtype] * (1.0 if dtype == "fp16" else (ratio / (1 + others)[:, None]).amax(1, keepdim=True))
            for got, left, right, terms in ((dh, (off, dz), e[0].to(f), vocab), (de[0], (off.t(), dz.t()), h.to(f), rows)):
                out = scale * (left[1] @ right)
                far = left[0] @ right.abs() + (terms + 8) * oh.STEP * ((left[1].abs() + left[0]) @ right.abs())
                close(got, out, scale * far * (1 + u) + (u + 4 * oh.STEP) * out.abs() + torch.finfo(t).smallest_normal * torch.finfo(t).eps)
            assert oh.untouched(hbuf, dh) and oh.untouched(ebuf, de)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("steps, piece", [(60, 0), (400, 0), (400, 256)])
def test_gradients_near_a_minimum(dtype, steps, piece):
    """A trained table, whose gradient is a small difference of large sums.  What the header says of 16 bits: every slope is off by half a step of the type
    (bf16: and 2^-11) of itself, so dE by that part of the sum of magnitudes and its own rounding; what fp32 adds is in loss_bounds, element by element."""
    t, gen, rows, vocab, dim, f = oh.TYPES[dtype][1], generator(21), 4096, 400, 64, torch.float64
    h = torch.randn(rows, dim, generator=gen, device="cuda").to(torch.bfloat16)
    true = torch.randn(vocab, dim, generator=gen, device="cuda", dtype=f) * 0.3
    target = torch.multinomial(torch.softmax(h.to(f) @ true.t(), 1), 1, generator=gen)[:, 0].int()
    e, m, v = (torch.zeros(vocab, dim, dtype=f, device="cuda") for _ in range(3))
    for step in range(1, steps + 1):
        dz = torch.softmax(h.to(f) @ e.t(), 1)
        dz[torch.arange(rows), target.long()] -= 1
        g = dz.t() @ h.to(f) / rows
        m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g * g
        e = e - 0.02 * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.999 ** step)).sqrt() + 1e-12)
    h, e = h.to(t), e[None].to(t)
    want = oh.exact_loss([0, rows], h, e, target)
    bound = oh.loss_bounds(want, t, dim, vocab)
    loss, dh, de = torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(e)
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, [0, rows], h, e, target, dh, de, None, loss, piece=piece))
    close(loss, want["loss"], bound["loss"])
    close(dh, want["dh"], bound["dh"])
    close(de, want["de"], bound["de"])
    dz = want["parts"][0][7]
    magnitude, u = (dz.abs().t() @ h.to(f).abs()) / rows, oh.half_step(t)
    # fp16: slopes are not below steps of 2^-38; fp32: the sums' (rows + 8) 2^-23 stand for everything
    part = {"bf16": u + 2.0 ** -11, "fp16": u, "fp32": 0.0}[dtype] + (rows + 8 + 400) * oh.STEP
    floor = (2.0 ** -39 * h.to(f).abs().mean(0) if dtype != "fp32" else 0.0) + torch.finfo(t).smallest_normal * torch.finfo(t).eps
    close(de[0], want["de"][0], part * (1 + u) * magnitude + u * want["de"][0].abs() + floor)


# bounds, rows, dim, vocab, pad, piece: one piece and several, rows in small and large tiles, joined splits, rows off 16 bytes
RELU_LOSSES = [([2, 40, 40, 71], 80, 64, 300, 0, 0), ([0, 200, 333], 340, 120, 700, 8, 256), ([0, 3], 3, 33, 77, 1, 0),
               ([1, 1000, 2999], 3000, 264, 2056, 0, 1024), ([0, 600], 600, 1032, 2500, 0, 0), ([0, 2990], 3000, 1032, 700, 0, 512)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", range(len(RELU_LOSSES)))
def test_loss_behind_a_relu(dtype, case):
    """dh is zero where h is not above zero, and else has the bits that it has without the relu; nothing else changes."""
    bounds, rows, dim, vocab, pad, piece = RELU_LOSSES[case]
    gen, t, groups = generator(300 + case), oh.TYPES[dtype][1], len(bounds) - 1
    h, e = oh.matrix(rows, dim, pad, t, gen), oh.stack(groups, vocab, dim, pad, pad, t, gen, std=2.0 / dim ** 0.5)
    h.copy_(torch.relu(h))
    h[::3, 1::7] = -0.0
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    target[1::5] = -1
    h[1::5] = float("nan")
    written, outs = oh.inside(bounds, rows), []
    for flags in (0, P.CROSS_ENTROPY_RELU_IN):
        loss = torch.zeros(rows, device="cuda")
        (hbuf, dh), (ebuf, de) = oh.output((rows, dim), pad, t), oh.output((groups, vocab, dim), pad, t)
        P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, dh, de, None, loss, piece=piece, flags=flags))
        assert oh.untouched(hbuf, dh, written)
        outs.append((loss, dh, ebuf))
    want = oh.exact_loss(bounds, h, e, target)
    close(outs[0][1][written], want["dh"][written], oh.loss_bounds(want, t, dim, vocab)["dh"][written])
    through = torch.where(h > 0, outs[0][1], torch.zeros_like(h))
    assert torch.equal(outs[1][1][written], through[written])
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][2], outs[1][2])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("each, dim, vocab, piece", [(9, 16, 600, 0), (9, 16, 600, 256), (10, 13, 600, 0), (160, 72, 2600, 0), (160, 72, 2600, 1024)])
def test_logits_that_are_not_finite(dtype, each, dim, vocab, piece):
    """Infinities and NaN in a group's table, at the target and beside it, alone and everywhere: loss and gradients are infinite or NaN where 64-bit
    arithmetic by the definition has them so, and finite where it does not; a group without them keeps its values."""
    inf, t, gen, f = float("inf"), oh.TYPES[dtype][1], generator(dim), torch.float64
    tables = [{}, {5: inf}, {7: -inf, vocab - 1: -inf}, "all but 2", "all", {vocab - 2: float("nan")}, {}]
    groups, rows = len(tables), len(tables) * each
    bounds = [g * each for g in range(groups + 1)]
    h, e = oh.matrix(rows, dim, 0, t, gen), oh.stack(groups, vocab, dim, 0, 0, t, gen, std=2.0 / dim ** 0.5)
    h[:, 0], e[:, :, 0] = 1.0, 0.0
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    for g, special in enumerate(tables):
        first = target[g * each:(g + 1) * each]
        if special == "all but 2":
            e[g, :, 0], e[g, 2, 0], first[0], first[1:] = -inf, 0.0, 2, 4
            first[2:5] = 2
        elif special == "all":
            e[g, :, 0] = -inf
        else:
            for v, x in special.items():
                e[g, v, 0] = x
            first[:4] = torch.tensor([5, 7, vocab - 1, vocab - 2], dtype=torch.int32)
    z = torch.cat([h[s].to(f) @ e[g].to(f).t() for g, s in oh.groups_of(bounds)])
    at = torch.arange(rows, device="cuda")
    want = -torch.log_softmax(z, 1)[at, target.long()]
    dz = torch.softmax(z, 1)
    dz[at, target.long()] -= 1
    loss, dh, de = torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(e)
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, dh, de, None, loss, piece=piece))
    only = torch.empty(rows, device="cuda")
    P.cross_entropy(torch.cuda.current_stream(), oh.cross_entropy_call(dtype, bounds, h, e, target, loss=only))
    assert torch.equal(torch.isnan(loss), torch.isnan(want)) and torch.equal(torch.isposinf(loss), torch.isposinf(want)) and not bool(torch.isneginf(loss).any())
    fine = torch.isfinite(want)
    assert torch.equal(only[fine], loss[fine]) and torch.equal(torch.isnan(only), torch.isnan(want)) and torch.equal(torch.isposinf(only), torch.isposinf(want))
    sure = 3 * each + torch.tensor([0, 2, 3, 4], device="cuda")
    assert not bool(loss[sure].any()) and bool(torch.isposinf(loss[3 * each + 1]))          # the only possible entry: loss 0; an impossible one: infinite
    magnitude = torch.cat([h[s].to(f).abs() @ torch.nan_to_num(e[g], nan=0.0, posinf=0.0, neginf=0.0).to(f).abs().t() for g, s in oh.groups_of(bounds)]).amax(1)
    bound = 2 * ((dim + 8) * oh.STEP * magnitude + (300 + vocab / 64) * oh.STEP) + 2 * oh.STEP * want.abs()
    close(loss[fine], want[fine], bound[fine])
    for g, s in oh.groups_of(bounds):
        for got, out in ((dh[s], dz[s] @ e[g].to(f)), (de[g], dz[s].t() @ h[s].to(f))):
            got = got.to(f)
            assert torch.equal(torch.isnan(got), torch.isnan(out)) and torch.equal(torch.isinf(got), torch.isinf(out)), g
            assert torch.equal(got[torch.isinf(got)], out[torch.isinf(out)]), g
    calm = oh.exact_loss(bounds[:2], h[:each], e[:1], target[:each])
    near = oh.loss_bounds(calm, t, dim, vocab)
    close(dh[:each], calm["dh"], near["dh"])
    close(de[:1], calm["de"], near["de"])


# ---- together ------------------------------------------------------------------------------------------------

def readme_example():
    """The README's block of Python, as it stands there."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    blocks = re.findall(r"```python\n(.*?)```", text, re.S)
    assert len(blocks) == 1
    return blocks[0]


def test_the_example_of_the_readme():
    """Run as it stands: every result against 64 bits from the inputs it was made of, and the weights' gradient against 64 bits from the first inputs:
    y, dz, dy and dW are rounded to bf16 once each (2^-8 of the value), y once more through the logits, dh and dE: 8 2^-8 in the norm."""
    bounds, R, K, N, V = [0, 60, 60, 200], 200, 96, 64, 500
    W, gen, t = len(bounds) - 1, generator(23), torch.bfloat16
    x, w, table = oh.matrix(R, K, 0, t, gen), oh.stack(W, K, N, 0, 0, t, gen, std=K ** -0.5), oh.stack(W, V, N, 0, 0, t, gen, std=2.0 * N ** -0.5)
    targets = torch.randint(0, V, (R,), generator=gen, device="cuda", dtype=torch.int32)
    targets[::5] = -1
    y, dy, dx = (torch.zeros((R, c), dtype=t, device="cuda") for c in (N, N, K))
    names = dict(torch=torch, W=W, R=R, K=K, N=N, V=V, offsets=torch.tensor(bounds, dtype=torch.int64, device="cuda"), x=x, w=w, y=y, dy=dy, dx=dx,
                 dw=torch.zeros((W, K, N), device="cuda"), table=table, targets=targets, loss=torch.zeros(R, device="cuda"),
                 group_loss=torch.zeros(W, device="cuda"), dtable=torch.zeros_like(table), stream=torch.cuda.current_stream())
    exec(compile(readme_example(), "README.md", "exec"), names)
    out, mag, terms = oh.exact_product("forward", bounds, x, w)
    close(y, out.clamp(min=0), oh.product_bound(out, mag, terms, t))
    want = oh.exact_loss(bounds, y, table, targets)
    bound = oh.loss_bounds(want, t, N, V)
    close(names["loss"], want["loss"], bound["loss"])
    close(names["dtable"], want["de"], bound["de"])
    close(dy, want["dh"] * (y > 0), bound["dh"])
    got, mag, terms = oh.exact_product("weight_grad", bounds, x, dy)
    close(names["dw"], got, oh.product_bound(got, mag, terms, torch.float32))
    first = oh.exact_loss(bounds, out.clamp(min=0), table, targets)
    dw, _, _ = oh.exact_product("weight_grad", bounds, x, first["dh"] * (out > 0))
    for g in range(W):
        assert float((names["dw"][g].double() - dw[g]).norm()) <= 2.0 ** -5 * float(dw[g].norm()), g



class Workers:
    """W workers with models of two layers and a vocabulary's table in one packed row each, trained by the framework's step with the caller's
    gradient: forward, checkpoints in 8 bits, loss, backward, cocod_external_step."""

    def __init__(self, dtype, bounds, dims, vocab, stream):
        self.dtype, self.t, self.W = dtype, oh.TYPES[dtype][1], len(bounds) - 1
        self.bounds, self.rows, self.dims, self.vocab = bounds, bounds[-1] + 3, dims, vocab
        a, b, c = dims
        sizes = [a * b, b * c, vocab * c]
        padded, self.at, _ = P.plan_layout(sum(sizes), sizes)
        gen = generator(17)
        W, rows, t = self.W, self.rows, self.t

        def zeros(*shape, dtype=torch.float32):
            return torch.zeros(shape, dtype=dtype, device="cuda")

        self.xA, self.xB, self.v, self.mean = zeros(W, padded), zeros(W, padded), zeros(W, padded), zeros(padded)
        for off, size, fan in zip(self.at, sizes, (a, b, c)):
            self.xA[:, off:off + size] = torch.randn(W, size, generator=gen, device="cuda") * fan ** -0.5
        self.shadow = zeros(W, padded, dtype=t)                  # the models in the element type
        self.G = zeros(W, padded, dtype=t)
        self.ctx = P.Context(W=W, d=sum(sizes), stride=padded, xA=self.xA, xB=self.xB, v=self.v, mean=self.mean, tensor_numel=sizes, lr=0.1,
                             momentum=0.9, grad=P.GRAD_EXTERNAL, compute_stream=stream, avg_stream=stream)
        self.x = oh.matrix(rows, a, 0, t, gen)
        self.target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        self.target[::5] = -1
        self.h1, self.h2, self.dh2, self.dh1 = zeros(rows, b, dtype=t), zeros(rows, c, dtype=t), zeros(rows, c, dtype=t), zeros(rows, b, dtype=t)
        self.codes, self.scales = zeros(rows, b, dtype=torch.uint8), zeros(rows, -(-b // 32), dtype=torch.uint8)
        self.loss, self.group_loss = zeros(rows), zeros(W)

        def part(buf, i, r, q):
            return buf[:, self.at[i]:self.at[i] + sizes[i]].unflatten(1, (r, q))

        w = [part(self.shadow, 0, a, b), part(self.shadow, 1, b, c), part(self.shadow, 2, vocab, c)]
        dw = [part(self.G, 0, a, b), part(self.G, 1, b, c), part(self.G, 2, vocab, c)]
        kind = oh.TYPES[dtype][0]
        self.first = oh.layer(dtype, bounds, rows, a, b, x=self.x, w=w[0], y=self.h1, dy=self.dh1, dw=dw[0], dw_dtype=kind, flags=P.GROUPED_RELU_OUT)
        self.second = oh.layer(dtype, bounds, rows, b, c, x=self.h1, w=w[1], y=self.h2)
        self.second_back = oh.layer(dtype, bounds, rows, b, c, x_codes=self.codes, x_scales=self.scales, w=w[1], dy=self.dh2, dx=self.dh1, dw=dw[1],
                                    dw_dtype=kind, flags=P.GROUPED_RELU_IN)
        self.head = oh.cross_entropy_call(dtype, bounds, self.h2, w[2], self.target, self.dh2, dw[2], self.group_loss, self.loss, piece=256)
        self.stream, self.kind = stream, kind

    def live(self):
        return self.xA if self.ctx.live_model() == self.xA.data_ptr() else self.xB

    def gradient(self):
        s, b = self.stream, self.dims[1]
        P.grouped_forward(s, self.first)
        P.grouped_forward(s, self.second)
        P.checkpoint_store(s, self.kind, self.rows, b, self.h1, b, self.codes, b, self.scales, self.scales.shape[1])
        self.h1.fill_(float("nan"))                              # the backward pass has nothing but the codes
        P.cross_entropy(s, self.head)
        P.grouped_weight_grad(s, self.second_back)
        P.grouped_input_grad(s, self.second_back)
        P.grouped_weight_grad(s, self.first)

    def step(self, close=False):
        self.shadow.copy_(self.live())
        self.gradient()
        (self.ctx.external_step if self.t == torch.float32 else self.ctx.external_step_bf16)(self.G, close)

    def exact_gradient(self):
        """The same pass in 64 bits from the same weights, with the checkpoint's definition."""
        a, b, c = self.dims
        f, out = torch.float64, []
        for g, s in oh.groups_of(self.bounds):
            row = self.shadow[g].to(f)
            w = [row[o:o + r * q].reshape(r, q) for o, (r, q) in zip(self.at, ((a, b), (b, c), (self.vocab, c)))]
            x, tt = self.x[s].to(f), self.target[s].long()
            h1 = torch.relu(x @ w[0])
            h2 = h1 @ w[1]
            keep = tt >= 0
            p = torch.softmax(h2 @ w[2].t(), 1)
            p[keep, tt[keep]] -= 1
            p *= keep[:, None] / max(int(keep.sum()), 1)
            d2 = p @ w[2]
            codes, scales = oh.encode(h1.cpu().numpy(), self.dtype)
            kept = torch.from_numpy(oh.decode(codes, scales)).cuda()
            d1 = (d2 @ w[1].t()) * (h1 > 0)
            out.append((x.t() @ d1, kept.t() @ d2, p.t() @ h2))
        return out


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_training_step_of_all_operators(dtype):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        k = Workers(dtype, [0, 60, 60, 200, 333], (48, 96, 64), 700, stream)
        k.shadow.copy_(k.live())
        k.gradient()
        want = k.exact_gradient()
        got = k.G.clone()
    stream.synchronize()
    a, b, c = k.dims
    for g in range(k.W):
        for i, (r, q) in enumerate(((a, b), (b, c), (k.vocab, c))):
            x = got[g, k.at[i]:k.at[i] + r * q].reshape(r, q).double()
            norm = want[g][i].norm()
            # bf16: every tensor of the chain (at most eight of them) is rounded by at most 2^-8 of its values, and a code may fall on the other side of
            # a rounding where h1 does (a step of 2^-3): 8 * 2^-8 in the norm, and as much again for the codes' 2^-4.  fp32: 2^-4 for
            # the rare code that falls on the other side, one in 10^4 of them: below 1e-3.
            assert float((x - want[g][i]).norm()) <= (2.0 ** -4 if dtype == "bf16" else 1e-3) * float(norm) + 1e-30, (g, i)
    # two rounds of CoCoD-SGD with these gradients: all workers end on different models around one mean, and everything stays finite
    with torch.cuda.stream(stream):
        for _ in range(2):
            k.ctx.average_begin()
            k.step()
            k.step(close=True)
    k.ctx.sync()
    assert bool(torch.isfinite(k.live()).all()) and bool(torch.isfinite(k.loss).all()) and k.ctx.get_step() == 4
    k.ctx.close()


def test_replays_of_a_captured_step_have_the_eager_bits():
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        k = Workers("bf16", [0, 60, 60, 200, 333], (48, 96, 64), 700, stream)
        k.shadow.copy_(k.live())
        k.gradient()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            k.gradient()
        moved = torch.tensor([0, 10, 100, 120, 300], dtype=torch.int64, device="cuda")
        for turn in range(4):
            offsets = k.first.keep[0]
            if turn == 2:                                        # other batches, without the host's part in it
                for lay in (k.first, k.second, k.second_back, k.head):
                    lay.keep[0].copy_(moved)
            k.shadow.mul_(1.0 + 0.125 * turn)
            k.G.fill_(float("nan"))
            k.gradient()
            eager = [t.clone() for t in (k.G, k.loss, k.group_loss, k.h2)]
            stream.synchronize()
            k.G.fill_(float("nan"))
            k.head.keep[-1].fill_(255)
            graph.replay()
            stream.synchronize()
            pads = torch.isnan(eager[0])
            assert torch.equal(torch.isnan(k.G), pads) and torch.equal(k.G[~pads], eager[0][~pads]), turn
            for t, e in zip((k.loss, k.group_loss, k.h2), eager[1:]):
                assert torch.equal(t, e), turn
    k.ctx.close()


def test_the_null_stream_and_another_thread():
    import threading
    gen, bounds, rows, k, n = generator(40), [0, 30, 90], 90, 64, 72
    x, w = oh.matrix(rows, k, 0, torch.bfloat16, gen), oh.stack(2, k, n, 0, 0, torch.bfloat16, gen)
    y = [torch.empty((rows, n), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    calls = [oh.layer("bf16", bounds, rows, k, n, x=x, w=w, y=out) for out in y]
    torch.cuda.synchronize()
    P.grouped_forward(None, calls[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()

    def other():
        P.grouped_forward(side, calls[1])
        with pytest.raises(P.CocodError, match="y is NULL"):
            calls[2].set(y=None)
            P.grouped_forward(side, calls[2])

    worker = threading.Thread(target=other)
    worker.start()
    worker.join()
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[1])


def test_two_streams_at_once():
    """Two calls at the same time, each with a workspace of its own, have the bits of each alone."""
    calls, alone = [], []
    for i in range(2):
        gen = generator(30 + i)
        h, e = oh.matrix(700, 64, 0, torch.bfloat16, gen), oh.stack(1, 3000, 64, 0, 0, torch.bfloat16, gen)
        target = torch.randint(0, 3000, (700,), generator=gen, device="cuda", dtype=torch.int32)
        c = oh.cross_entropy_call("bf16", [0, 700], h, e, target, torch.empty_like(h), torch.empty_like(e), None, torch.empty(700, device="cuda"))
        P.cross_entropy(torch.cuda.current_stream(), c)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in (c.keep[4], c.keep[6], c.keep[7])])
        calls.append(c)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(calls, streams):
            P.cross_entropy(s, c)
    torch.cuda.synchronize()
    for c, want in zip(calls, alone):
        for t, w in zip((c.keep[4], c.keep[6], c.keep[7]), want):
            assert torch.equal(t, w)
