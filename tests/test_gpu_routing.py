"""Routing between groups on the GPU, against counting and plain sums in 64 bits.

Bounds, u = eps / 2 of the type.  xs is a copy.  A sum over K choices is K fused multiply-adds in fp32: off by at most K 2^-24 sum |w ys| (1 + K 2^-24), then rounded once,
u |y|.  dys is one product in fp32 and one rounding: (2^-24 + u) |w dy| (fp32: the product alone).  dweights is `width` fused multiply-adds in some order and
six additions: (width + 8) 2^-24 sum |dy ys|.  Roundings below the normal range: half of the smallest step.
"""
import numpy as np
import pytest
import torch

import paper_1906_12043_amd as P
from tests.operator_harness import SENTINEL, TYPES, half_step, matrix, output, untouched

pytestmark = pytest.mark.gpu
E24 = 2.0 ** -24
NONE = -7777


def padded(rows, cols, pad, dtype, fill):
    buf = torch.full((max(rows, 1), cols + pad), fill, dtype=dtype, device="cuda")
    return buf, buf[:rows, :cols]


def pitch(t):
    return max(t.stride(0), t.shape[1])


def counted(experts, groups, capacity):
    """(offsets, place) by counting on the host."""
    flat = experts.cpu().numpy().reshape(-1).astype(np.int64)
    place, lists = np.full(flat.size, -1, np.int64), {}
    order = np.argsort(np.where((flat >= 0) & (flat < groups), flat, groups), kind="stable")
    order = order[(flat[order] >= 0) & (flat[order] < groups)]
    count = np.bincount(flat[order], minlength=groups)
    first = np.concatenate([[0], np.cumsum(count)])
    rank = np.arange(order.size) - first[flat[order]]
    taken = np.minimum(count, capacity) if capacity else count
    offsets = np.concatenate([[0], np.cumsum(taken)])
    keep = rank < (capacity or flat.size + 1)
    place[order[keep]] = offsets[flat[order[keep]]] + rank[keep]
    return offsets, place.reshape(experts.shape)


def sort(experts, groups, capacity=0, pad_place=0, stream=None):
    tokens, choices = experts.shape
    buf, place = padded(tokens, choices, pad_place, torch.int32, NONE)
    offsets = torch.full((groups + 2,), NONE, dtype=torch.int64, device="cuda")
    r = P.Route(groups=groups, choices=choices, tokens=tokens, capacity=capacity, experts=experts, ld_experts=pitch(experts), place=place, ld_place=choices + pad_place,
                offsets=offsets)
    ws = torch.full((max(P.route_workspace(r), 16),), 255, dtype=torch.uint8, device="cuda")
    r.set(workspace=ws, workspace_bytes=ws.numel())
    r.keep = (ws, buf, place, offsets, experts)
    P.route_sort(stream if stream is not None else torch.cuda.current_stream(), r)
    return r, buf, place, offsets


def random_experts(tokens, choices, groups, kind, seed, pad=0):
    gen = torch.Generator().manual_seed(seed)
    if kind == "even":
        e = torch.randint(0, groups, (tokens, choices), generator=gen)
    elif kind == "one":
        e = torch.full((tokens, choices), groups - 1)
    elif kind == "none":
        e = torch.randint(0, 2, (tokens, choices), generator=gen) * (2 ** 31 - 1 + groups) - 1
        e = torch.where(e >= 2 ** 31, 2 ** 31 - 1, e)
    elif kind == "few":                                       # some of a few groups, some of none, some out of range on either side
        e = torch.randint(-2, min(groups, 5) + 2, (tokens, choices), generator=gen)
        e = torch.where(e >= min(groups, 5), groups + e * 1000, e)
    else:                                                     # in descending runs
        e = (groups - 1) - (torch.arange(tokens * choices) * groups // max(1, tokens * choices)).reshape(tokens, choices)
    buf = torch.full((max(tokens, 1), choices + pad), 0, dtype=torch.int32, device="cuda")
    buf[:tokens, :choices] = e.to(torch.int32).cuda()
    return buf[:tokens, :choices]


SORTS = [(1, 1, 1), (16, 2, 8), (63, 1, 3), (65, 3, 512), (4096, 2, 512), (1024, 8, 511), (4097, 2, 8), (1000, 1, 513), (1, 1, 65535), (5000, 8, 128),
         (20_011, 6, 60), (3, 64, 4097), (30_000, 2, 8193), (70_001, 1, 65535), (600_000, 1, 2), (0, 2, 5), (0, 1, 600), (1 << 21, 2, 16)]


@pytest.mark.parametrize("tokens, choices, groups", SORTS)
@pytest.mark.parametrize("kind", ["even", "one", "few", "none", "runs"])
def test_sort(tokens, choices, groups, kind):
    pad = tokens % 3
    experts = random_experts(tokens, choices, groups, kind, tokens + groups, pad)
    for capacity in (0, max(1, tokens * choices // groups), 1 << 40):
        _, buf, place, offsets = sort(experts, groups, capacity, pad_place=pad)
        want_offsets, want_place = counted(experts, groups, min(capacity, 2 ** 31))
        assert np.array_equal(offsets.cpu().numpy()[:-1], want_offsets) and int(offsets[-1]) == NONE
        assert np.array_equal(place.cpu().numpy(), want_place)
        assert bool((buf[:, choices:] == NONE).all())


def rows_case(dtype, tokens, choices, width, seed, pad=0, drop=0.2, groups=7):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype][1]
    experts = torch.randint(0, groups, (tokens, choices), generator=gen, device="cuda", dtype=torch.int32)
    experts[torch.rand(tokens, choices, generator=gen, device="cuda") < drop] = -1
    _, _, place, offsets = sort(experts, groups, pad_place=pad % 2)
    place = place.long().cpu()
    used = int(offsets[groups])
    weights = matrix(tokens, choices, pad % 3, torch.float32, gen)
    weights[place.cuda() < 0] = float("nan")                   # nothing of the weight of a pair without a row is used
    return t, gen, place, used, weights


def description(dtype, place, width, **tensors):
    f = dict(dtype=TYPES[dtype][0], groups=7, tokens=place.shape[0], choices=place.shape[1], width=width, place=place, ld_place=pitch(place))
    names = {"x": "ldx", "xs": "ldxs", "ys": "ldys", "y": "ldy", "dy": "lddy", "dys": "lddys", "dxs": "lddxs", "dx": "lddx", "weights": "ld_weights", "dweights": "ld_dweights"}
    for name, t in tensors.items():
        if t is not None:
            f[name], f[names[name]] = t, pitch(t)
    r = P.Route(**f)
    r.keep = (place, tensors)
    return r


def on_gpu(place, pad=0):
    buf = torch.full((max(1, place.shape[0]), place.shape[1] + pad), NONE, dtype=torch.int32, device="cuda")
    buf[:place.shape[0], :place.shape[1]] = place.to(torch.int32).cuda()
    return buf[:place.shape[0], :place.shape[1]]


SHAPES = [(1, 1, 1), (5, 2, 7), (300, 2, 8), (33, 3, 9), (17, 8, 33), (64, 1, 64), (7, 64, 40), (300, 2, 1000), (5, 4, 2049), (257, 8, 512), (3, 2, 8200), (2, 1, 70_001), (5000, 2, 520)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens, choices, width", SHAPES)
@pytest.mark.parametrize("pad", [0, 8, 5])
def test_rows_to_groups_and_back(dtype, tokens, choices, width, pad):
    t, gen, place, used, weights = rows_case(dtype, tokens, choices, width, tokens * 31 + width, pad)
    u, tiny = half_step(t), torch.finfo(t).smallest_normal * half_step(t) * 2
    f64, stream, pairs = torch.float64, torch.cuda.current_stream(), tokens * choices
    at = on_gpu(place, pad % 4)
    has = place >= 0
    token = torch.arange(tokens)[:, None].expand(tokens, choices)[has].cuda()
    rows = place[has].cuda()

    x = matrix(tokens, width, pad, t, gen)
    buf, xs = output((pairs, width), pad, t)
    P.route_dispatch(stream, description(dtype, at, width, x=x, xs=xs))
    assert torch.equal(xs[rows], x[token]) and untouched(buf, xs, rows)

    def grouped_rows():
        m = matrix(pairs, width, pad, t, gen)
        m[used:] = float("nan")                                # rows that no pair has are not read
        return m

    ys = grouped_rows()
    w = torch.where(has.cuda(), weights, 0.0).to(f64)
    full = torch.zeros((tokens, choices, width), dtype=f64, device="cuda")
    full[has.cuda()] = ys[rows].to(f64)
    for weighted in (True, False):
        buf, y = output((tokens, width), pad, t)
        P.route_combine(stream, description(dtype, at, width, ys=ys, y=y, weights=weights if weighted else None))
        ww = w if weighted else has.cuda().to(f64)
        want, mag = (full * ww[:, :, None]).sum(1), (full * ww[:, :, None]).abs().sum(1)
        bound = u * want.abs() + (1 + u) * choices * E24 * mag * 1.001 + tiny
        assert bool(((y.to(f64) - want).abs() <= bound).all()) and untouched(buf, y)

    dxs = grouped_rows()
    buf, dx = output((tokens, width), pad, t)
    P.route_dispatch_grad(stream, description(dtype, at, width, dxs=dxs, dx=dx))
    full_d = torch.zeros((tokens, choices, width), dtype=f64, device="cuda")
    full_d[has.cuda()] = dxs[rows].to(f64)
    want, mag = full_d.sum(1), full_d.abs().sum(1)
    assert bool(((dx.to(f64) - want).abs() <= u * want.abs() + (1 + u) * choices * E24 * mag * 1.001 + tiny).all()) and untouched(buf, dx)

    dy = matrix(tokens, width, pad, t, gen)
    want_w = (full * dy.to(f64)[:, None, :]).sum(2)
    bound_w = (width + 8) * E24 * (full * dy.to(f64)[:, None, :]).abs().sum(2) * 1.001 + 2.0 ** -149
    for weighted, wanted in ((True, "both"), (False, "both"), (True, "rows"), (True, "weights")):
        buf, dys = output((pairs, width), pad, t)
        buf_w, dweights = output((tokens, choices), pad, torch.float32)
        P.route_combine_grad(stream, description(dtype, at, width, ys=ys if wanted != "rows" else None, dy=dy, weights=weights if weighted else None,
                                                 dys=dys if wanted != "weights" else None, dweights=dweights if wanted != "rows" else None))
        if wanted != "weights":
            ww = (w if weighted else torch.ones_like(w))[has.cuda()]
            want = dy.to(f64)[token] * ww[:, None]
            assert bool(((dys[rows].to(f64) - want).abs() <= (u + E24 + u * E24) * want.abs() + tiny).all())
        assert untouched(buf, dys, rows if wanted != "weights" else [])
        if wanted != "rows":
            assert bool(((dweights.to(f64) - want_w).abs() <= bound_w).all()) and bool((dweights[~has.cuda()] == 0).all())
        assert untouched(buf_w, dweights, slice(0, tokens if wanted != "rows" else 0))


def test_gradients_are_differences():
    """L = sum of y * dy is linear in weights and in ys; with small whole numbers every sum is exact, and so are the differences."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    tokens, choices, width = 40, 3, 72
    experts = torch.randint(-1, 5, (tokens, choices), generator=gen, device="cuda", dtype=torch.int32)
    _, _, place, _ = sort(experts, 5)
    whole = lambda *s: torch.randint(-4, 5, s, generator=gen, device="cuda").float()            # noqa: E731
    ys, dy, w, x = whole(tokens * choices, width), whole(tokens, width), whole(tokens, choices), whole(tokens, width)
    stream = torch.cuda.current_stream()

    def loss(w_, ys_):
        y = torch.empty(tokens, width, device="cuda")
        P.route_combine(stream, description("fp32", place, width, ys=ys_, y=y, weights=w_))
        return float((y.double() * dy.double()).sum())

    dys, dw = torch.zeros_like(ys), torch.empty_like(w)
    P.route_combine_grad(stream, description("fp32", place, width, ys=ys, dy=dy, weights=w, dys=dys, dweights=dw))
    base = loss(w, ys)
    for t, j in ((0, 0), (7, 1), (39, 2), (20, 0), (21, 1)):
        more = w.clone()
        more[t, j] += 1
        assert loss(more, ys) - base == float(dw[t, j])
    for r, c in ((0, 0), (13, 71), (60, 30)):
        more = ys.clone()
        more[r, c] += 1
        assert loss(w, more) - base == float(dys[r, c])

    def sent(x_):                                              # sum of xs * dxs
        xs = torch.zeros(tokens * choices, width, device="cuda")
        P.route_dispatch(stream, description("fp32", place, width, x=x_, xs=xs))
        return float((xs.double() * ys.double()).sum())

    dx = torch.empty_like(x)
    P.route_dispatch_grad(stream, description("fp32", place, width, dxs=ys, dx=dx))
    for t, c in ((0, 0), (17, 5), (39, 71)):
        more = x.clone()
        more[t, c] += 1
        assert sent(more) - sent(x) == float(dx[t, c])


def test_places_that_are_no_rows_count_as_none():
    place = torch.tensor([[0, 6], [-5, 2 ** 31 - 1], [3, -2 ** 31]], dtype=torch.int32, device="cuda")      # six rows
    ys = torch.arange(6 * 16, device="cuda", dtype=torch.float32).reshape(6, 16)
    y, xs = torch.full((3, 16), SENTINEL, device="cuda"), torch.full((6, 16), SENTINEL, device="cuda")
    stream = torch.cuda.current_stream()
    P.route_combine(stream, description("fp32", place, 16, ys=ys, y=y))
    assert torch.equal(y[0], ys[0]) and torch.equal(y[2], ys[3]) and bool((y[1] == 0).all())
    P.route_dispatch(stream, description("fp32", place, 16, x=y, xs=xs))
    assert torch.equal(xs[0], y[0]) and torch.equal(xs[3], y[2]) and bool((xs[[1, 2, 4, 5]] == SENTINEL).all())


def test_rows_beyond_4_gib():
    tokens, choices, width, ld = 33_000, 1, 40, 1 << 16       # 4.3 GB from first to last row
    x = torch.randn(tokens, width, device="cuda").to(torch.bfloat16)
    far = torch.zeros(tokens * ld, dtype=torch.bfloat16, device="cuda").as_strided((tokens, width), (ld, 1))
    place = torch.arange(tokens - 1, -1, -1, device="cuda", dtype=torch.int32)[:, None].contiguous()
    P.route_dispatch(torch.cuda.current_stream(), description("bf16", place, width, x=x, xs=far))
    assert torch.equal(far, x.flip(0))
    y = torch.empty_like(x)
    P.route_combine(torch.cuda.current_stream(), description("bf16", place, width, ys=far, y=y))
    assert torch.equal(y, x)


@pytest.mark.parametrize("tokens, groups", [(500, 8), (20_000, 8), (700, 600)])
def test_replays_follow_what_the_router_chose(tokens, groups):
    """Captured once, replayed with other choices in the same memory; eager work of the program between the replays."""
    width, choices = 96, 2
    side = torch.cuda.Stream()
    experts = torch.zeros((tokens, choices), dtype=torch.int32, device="cuda")
    x = torch.zeros((tokens, width), dtype=torch.bfloat16, device="cuda")
    weights = torch.zeros((tokens, choices), device="cuda")
    place, offsets = torch.zeros_like(experts), torch.zeros(groups + 1, dtype=torch.int64, device="cuda")
    xs, y = torch.zeros((tokens * choices, width), dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x)
    r = P.Route(dtype=P.BF16, groups=groups, choices=choices, tokens=tokens, width=width, capacity=tokens, experts=experts, ld_experts=choices, place=place, ld_place=choices,
                offsets=offsets, x=x, ldx=width, xs=xs, ldxs=width, ys=xs, ldys=width, y=y, ldy=width, weights=weights, ld_weights=choices)
    ws = torch.zeros(max(16, P.route_workspace(r)), dtype=torch.uint8, device="cuda")
    r.set(workspace=ws, workspace_bytes=ws.numel())

    def calls(stream):
        P.route_sort(stream, r)
        P.route_dispatch(stream, r)
        P.route_combine(stream, r)

    torch.cuda.synchronize()
    calls(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(side)
    for k in range(4):
        gen = torch.Generator(device="cuda").manual_seed(k)
        experts.copy_(torch.randint(-1, groups, experts.shape, generator=gen, device="cuda"))
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        weights.copy_(torch.rand(weights.shape, generator=gen, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (offsets, place, xs, y)]
        want_offsets, want_place = counted(experts, groups, tokens)
        assert np.array_equal(got[0].cpu().numpy(), want_offsets) and np.array_equal(got[1].cpu().numpy(), want_place)
        calls(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (offsets, place, xs, y)))


def test_two_streams_at_once():
    jobs = []
    for k, stream in enumerate((torch.cuda.Stream(), torch.cuda.Stream())):
        experts = random_experts(30_000, 4, 64, "even", k)
        torch.cuda.synchronize()
        for _ in range(5):
            out = sort(experts, 64, stream=stream)
        jobs.append((experts, out))
    torch.cuda.synchronize()
    for experts, (_, _, place, offsets) in jobs:
        want_offsets, want_place = counted(experts, 64, 0)
        assert np.array_equal(offsets.cpu().numpy()[:-1], want_offsets) and np.array_equal(place.cpu().numpy(), want_place)
