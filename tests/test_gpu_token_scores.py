"""Token scores on the GPU against the plain implementation in 64 bits; bounds: scores_harness."""
import math

import pytest
import torch

import paper_1906_12043_amd as P
from tests.operator_harness import STEP, TYPES, half_step, matrix, output, stack, untouched
from tests.scores_harness import exact_scores, scores_call

pytestmark = pytest.mark.gpu

# bounds of the groups (rows in front of the first and behind the last belong to none), rows, entries, columns
SHAPES = [([0, 1], 1, 1, 1), ([0, 3], 3, 3, 8), ([0, 4], 4, 5, 33), ([0, 0, 5, 5, 9], 12, 64, 40), ([2, 40], 50, 65, 64), ([0, 16], 16, 5000, 128), ([1, 33, 33, 70, 131], 140, 301, 72),
          ([0, 64], 64, 1000, 256), ([0, 200, 611], 620, 1003, 96), ([0, 513], 513, 2050, 136), ([0, 700, 1500], 1500, 4100, 64), ([0, 2100], 2100, 3000, 192),
          ([0, 100, 300], 300, 777, 515), ([0, 8], 8, 40_000, 520), ([0, 200, 500], 500, 3000, 136)]

LARGE = ([0, 700, 1500], 1500, 8000, 136)          # of the largest tile


def inputs(dtype, bounds, rows, vocab, dim, pad, seed, lattice=False, shared=False, std=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, groups = TYPES[dtype][1], 1 if shared else len(bounds) - 1
    h, e = matrix(rows, dim, pad, t, gen), stack(groups, vocab, dim, pad, pad * 3, t, gen, std / math.sqrt(dim))
    if lattice:
        h.copy_((torch.round(h.float() * 16) / 16).to(t))
        e.copy_((torch.round(e.float() * 256) / 256).to(t))
    target = torch.randint(-1, vocab + 1, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    return gen, h, e, target


def check_top(out, want, top, vocab, exact_order):
    part = want["part"]
    ids, lps = out["top_ids"], out["top_logp"]
    assert bool((ids[~part] == -1).all()) and bool((lps[~part] == -math.inf).all())
    ids, lps, n = ids[part].long(), lps[part].double(), min(top, vocab)
    assert bool((ids[:, n:] == -1).all()) and bool((lps[:, n:] == -math.inf).all())
    ids, lps = ids[:, :n], lps[:, :n]
    if not ids.numel():
        return
    assert bool(((ids >= 0) & (ids < vocab)).all()) and bool((torch.sort(ids, 1).values.diff(dim=1) > 0).all()) and bool((lps.diff(dim=1) <= 0).all())
    logp, z, far = want["all"][part], want["z"][part], want["far_all"][part][:, None]
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :n]
    if exact_order:
        assert torch.equal(ids, order)
    bound = far + 4 * STEP * logp.gather(1, ids).abs()
    assert bool(((lps - logp.gather(1, ids)).abs() <= bound).all())
    assert bool(((lps - logp.gather(1, order)).abs() <= bound + far).all())           # as large as the j-th largest


def check_scores(out, want, far, bounds, rows, target):
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    inside[bounds[0]:bounds[-1]] = True
    for k in ("logp", "entropy") if target is not None else ("entropy",):
        assert bool(torch.isnan(out[k][~inside]).all()), k                             # left as they were
        assert bool(((out[k].double() - want[k]).abs() <= far[k])[inside].all()), (k, float(((out[k].double() - want[k]).abs() / far[k].clamp(min=1e-30))[inside].max()))
    return inside


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("which", range(len(SHAPES)))
@pytest.mark.parametrize("pad, masked", [(0, True), (8, False), (3, True), (3, False)])
def test_scores(dtype, which, pad, masked):
    bounds, rows, vocab, dim = SHAPES[which]
    for lattice, top, scale in ((True, (1, 5, 8, 20, 32)[which % 5], 0.8125), (False, 3, 1.0 / 0.7)):
        gen, h, e, target = inputs(dtype, bounds, rows, vocab, dim, pad, 100 + which, lattice)
        if masked:
            h[(target < 0) | (target >= vocab)] = float("nan")                         # nothing of such a row is used
        target = target if masked else None
        c, out = scores_call(dtype, bounds, h, e, target, top=top, scale=scale)
        P.token_scores(torch.cuda.current_stream(), c)
        want, far = exact_scores(bounds, torch.where(torch.isnan(h), 0.0, h), e, target, scale)
        inside = check_scores(out, want, far, bounds, rows, target)
        out["top_ids"], out["top_logp"], want["part"] = out["top_ids"][inside], out["top_logp"][inside], want["part"][inside]
        for k in ("all", "z", "far_all"):
            want[k] = want.get(k, torch.zeros(rows, dtype=torch.float64, device="cuda"))[inside]
        check_top(out, want, top, vocab, lattice)
        assert bool((out["ids_buffer"][:rows][~inside] == -9).all()) and bool((out["ids_buffer"][:, top:] == -9).all()) and bool(torch.isnan(out["logp_buffer"][:, top:]).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("which", range(len(SHAPES)))
@pytest.mark.parametrize("pad, masked, relu", [(0, True, False), (8, True, True), (3, False, False)])
def test_gradients(dtype, which, pad, masked, relu):
    bounds, rows, vocab, dim = SHAPES[which]
    gen, h, e, target = inputs(dtype, bounds, rows, vocab, dim, pad, 300 + which)
    if relu:
        h.relu_()
    a, b = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda") * 0.1
    a[::5], b[::5] = 0.0, 0.0                                                          # rows without slopes
    a[1::7] *= 1e-4
    if masked:
        h[(target < 0) | (target >= vocab)] = float("nan")
    target = target if masked else None
    for piece, one, two in ((0, a, b), (256, a, None), (512, None, b)):
        buf_h, dh = output((rows, dim), pad, h.dtype)
        buf_e, de = output((e.shape[0], vocab, dim), pad, h.dtype, pad)
        c, out = scores_call(dtype, bounds, h, e, target, grad=True, scale=0.75, d_logp=one, d_entropy=two, dh=dh, de=de, piece=piece, flags=P.TOKEN_SCORES_RELU_IN if relu else 0)
        P.token_scores(torch.cuda.current_stream(), c)
        h_slopeless = h.clone()
        none = torch.zeros(rows, dtype=torch.bool, device="cuda")
        none[::5] = True
        h[none] = float("nan")                                                         # rows without slopes take no part in the gradient
        P.token_scores_grad(torch.cuda.current_stream(), c)
        torch.cuda.synchronize()
        h.copy_(h_slopeless)
        clean = torch.where(torch.isnan(h), 0.0, h)
        want, far = exact_scores(bounds, clean, e, target, 0.75, one, two)
        if relu:
            want["dh"], far["dh"] = torch.where(clean > 0, want["dh"], 0.0), torch.where(clean > 0, far["dh"], 0.0)
        inside = slice(bounds[0], bounds[-1])
        for k, got in (("dh", dh[inside]), ("de", de)):
            x, f = (want[k][inside], far[k][inside]) if k == "dh" else (want[k], far[k])
            assert bool(((got.double() - x).abs() <= f).all()), (k, piece, float(((got.double() - x).abs() / f.clamp(min=1e-300)).max()))
        assert untouched(buf_h, dh, torch.arange(rows, device="cuda")[inside]) and untouched(buf_e, de)


def test_only_one_gradient_is_wanted():
    gen, h, e, target = inputs("bf16", [0, 90], 90, 700, 64, 0, 1)
    a = torch.randn(90, generator=gen, device="cuda")
    both = {"dh": torch.empty_like(h), "de": torch.empty_like(e)}
    for wanted in ({"dh"}, {"de"}, {"dh", "de"}):
        got = {k: torch.zeros_like(v) for k, v in both.items() if k in wanted}
        c, _ = scores_call("bf16", [0, 90], h, e, target, grad=True, d_logp=a, **got)
        P.token_scores(torch.cuda.current_stream(), c)
        P.token_scores_grad(torch.cuda.current_stream(), c)
        if len(wanted) == 1:
            both.update(got)
        else:
            assert all(torch.equal(both[k], got[k]) for k in got)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_gradients_where_no_row_takes_part(dtype):
    """No slopes at all, slopes of zero, no row with a target, no rows: every gradient is zero."""
    t = TYPES[dtype][1]
    gen, h, e, target = inputs(dtype, [0, 20, 50], 50, 300, 40, 0, 3)
    h[:] = float("nan")
    for rows, a, targets in ((50, None, target), (50, torch.zeros(50, device="cuda"), target), (50, torch.ones(50, device="cuda"), torch.full_like(target, -1)), (0, None, None)):
        dh, de = torch.full((50, 40), 5.0, dtype=t, device="cuda"), torch.full((2, 300, 40), 5.0, dtype=t, device="cuda")
        c, out = scores_call(dtype, [0, 20, 50] if rows else [0, 0, 0], h, e, targets, grad=True, d_logp=a, dh=dh, de=de, rows=rows)
        out["norms"].zero_()
        P.token_scores_grad(torch.cuda.current_stream(), c)
        assert bool((de == 0).all()) and bool((dh == (0 if rows else 5.0)).all())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_one_table_for_all_groups(dtype):
    bounds = [0, 30, 30, 77]
    gen, h, e, target = inputs(dtype, bounds, 77, 900, 80, 0, 2, shared=True)
    c, out = scores_call(dtype, bounds, h, e, target, top=4)
    c.set(e_stride=0)
    P.token_scores(torch.cuda.current_stream(), c)
    want, far = exact_scores(bounds, h, e.expand(3, -1, -1), target)
    check_scores(out, want, far, bounds, 77, target)
    check_top(out, want, 4, 900, False)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("gap", [5.0, 20.0, 60.0, 120.0])
def test_rows_that_are_sure_keep_their_digits(dtype, gap):
    """One logit is `gap`, the others zero, exactly: log p of the first is -log1p((V - 1) e^-gap), to (gap + 40 + V / 64) steps of itself, and so are H = log1p(rest) + gap rest / (1 + rest)
    and, as differences from one, the slopes: of the first entry a (1 - p)."""
    vocab, dim, V = 3001, 16, 3001
    t = TYPES[dtype][1]
    h, e = torch.zeros(20, dim, dtype=t, device="cuda"), torch.zeros(1, vocab, dim, dtype=t, device="cuda")
    h[:, 0] = gap
    e[0, 1234, 0] = 1.0
    e[0, :, 1] = 1.0                                                                   # (h is zero there; dh reads it)
    target = torch.full((20,), 1234, dtype=torch.int32, device="cuda")
    a, dh = torch.ones(20, device="cuda"), torch.empty_like(h)
    c, out = scores_call(dtype, [0, 20], h, e, target, grad=True, top=2, d_logp=a, dh=dh)
    P.token_scores(torch.cuda.current_stream(), c)
    P.token_scores_grad(torch.cuda.current_stream(), c)
    rest = (V - 1) * math.exp(-gap)
    logp, H = -math.log1p(rest), math.log1p(rest) + gap * rest / (1 + rest)
    rel = (gap + 40 + V / 64) * STEP
    normal = rest > 2.0 ** -125                                                        # (below, exponentials lose digits of their own)
    for got, want in ((out["logp"], logp), (out["entropy"], H), (out["top_logp"][:, 0], logp)):
        assert bool(((got.double() - want).abs() <= rel * abs(want) * 1.01 + (0 if normal else 1e-44)).all())
    assert bool((out["top_ids"][:, 0] == 1234).all()) and bool((out["top_ids"][:, 1] == 0).all())
    # dh[0] = a (1 - p) e[1234][0]; in 16 bits rounded twice
    want = rest / (1 + rest)
    u = 2 * torch.finfo(t).eps if t != torch.float32 else 0.0
    low = 2.0 ** -38 if t == torch.float16 else 0.0 if t == torch.float32 else 1e-37
    assert bool(((dh[:, 0].double() - want).abs() <= (u + rel) * want * 1.01 + low + torch.finfo(t).smallest_normal * torch.finfo(t).eps + (0 if normal else 1e-37)).all())


def test_equal_logits_come_in_order():
    """Every entry is the largest: a row of zeros, and few distinct logits over several tiles."""
    for vocab in (3, 70, 1000, 20_000):
        h, e = torch.zeros(9, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(1, vocab, 64, dtype=torch.bfloat16, device="cuda")
        h[4:] = 1.0
        e[0, :, 0] = (torch.arange(vocab, device="cuda") % 3 == 2).to(torch.bfloat16)
        c, out = scores_call("bf16", [0, 9], h, e, None, top=32)
        P.token_scores(torch.cuda.current_stream(), c)
        n = min(32, vocab)
        assert bool((out["top_ids"][:4, :n] == torch.arange(n, device="cuda")).all()) and bool((out["top_ids"][:, n:] == -1).all())
        order = torch.sort((torch.arange(vocab, device="cuda") % 3 == 2).int(), descending=True, stable=True).indices[:n]
        assert bool((out["top_ids"][4:, :n] == order).all())
        assert bool(((out["entropy"][:4].double() - math.log(vocab)).abs() <= (300 + vocab / 64) * STEP * math.log(vocab + 1)).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows", [6, 300])
def test_values_that_are_not_finite(dtype, rows):
    """NaN and infinities stay in their rows; alternatives are entries of the vocabulary all the same, each once."""
    vocab, dim = 700, 64
    gen, h, e, target = inputs(dtype, [0, rows], rows, vocab, dim, 0, 7, lattice=True)
    h, e = h.clone(), e.clone()
    e[0, 10, 0] = 60000.0 if dtype == "fp16" else 3e38
    h[:, 0] = 0.0
    clean, _ = exact_scores([0, rows], h, e, None)
    h[1, 0], h[2, 5], h[3, 0], h[4, 0] = float("nan"), float("inf"), 60000.0, -60000.0          # NaN; infinities of both signs; one +inf; one -inf (fp16: large)
    c, out = scores_call(dtype, [0, rows], h, e, None, top=6)
    P.token_scores(torch.cuda.current_stream(), c)
    assert bool(torch.isnan(out["entropy"][[1, 2]]).all())
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[[1, 2, 3, 4]] = False
    assert bool(torch.isfinite(out["entropy"][good]).all())
    ids = out["top_ids"].long()
    assert bool(((ids >= 0) & (ids < vocab)).all()) and bool((torch.sort(ids, 1).values.diff(dim=1) > 0).all())
    assert torch.equal(ids[good], torch.sort(clean["z"], dim=1, descending=True, stable=True).indices[:, :6][good])
    assert int(ids[3, 0]) == 10 and not bool((ids[4] == 10).any())
    if dtype != "fp16":
        others = e.clone()
        others[0, 10] = 0.0
        z = exact_scores([0, 1], h[4:5], others, None)[0]["z"]
        z[0, 10] = -math.inf                                   # (counts as 0)
        p = torch.softmax(z, 1)
        H = float(-(p * torch.where(p > 0, torch.log(p.clamp(min=1e-300)), 0.0)).sum())
        assert math.isnan(float(out["entropy"][3])) and abs(float(out["entropy"][4]) - H) <= 1e-4


def test_calls_without_every_output():
    gen, h, e, target = inputs("bf16", [0, 50], 50, 600, 64, 0, 8)
    c, full = scores_call("bf16", [0, 50], h, e, target, top=3)
    P.token_scores(torch.cuda.current_stream(), c)
    for gone in (("logp",), ("entropy", "norms"), ("logp", "entropy", "norms"), ("top",)):
        c, out = scores_call("bf16", [0, 50], h, e, target, top=0 if "top" in gone else 3)
        c.set(**{k: None for k in gone if k != "top"})
        P.token_scores(torch.cuda.current_stream(), c)
        for k in ("logp", "entropy", "norms") + (() if "top" in gone else ("top_ids", "top_logp")):
            assert bool(torch.isnan(out[k]).all()) if k in gone else torch.equal(out[k], full[k])


def test_offsets_that_do_not_ascend_stay_inside():
    """Results are undefined; nothing but the outputs may be written (sentinels around), and every call comes back."""
    gen, h, e, target = inputs("bf16", [0, 100, 100, 200, 200], 200, 500, 64, 0, 9)
    a = torch.randn(200, device="cuda")
    buf_h, dh = output((200, 64), 8, h.dtype)
    buf_e, de = output((4, 500, 64), 8, h.dtype)
    c, out = scores_call("bf16", [50, 180, 20, 300, -4], h, e, target, grad=True, top=5, d_logp=a, dh=dh, de=de)
    P.token_scores(torch.cuda.current_stream(), c)
    P.token_scores_grad(torch.cuda.current_stream(), c)
    c2, _ = scores_call("bf16", [0, 180, 20, 300, 200], h, e, target, grad=True, top=5, d_logp=a, dh=dh, de=de)
    P.token_scores(torch.cuda.current_stream(), c2)
    P.token_scores_grad(torch.cuda.current_stream(), c2)
    torch.cuda.synchronize()
    assert untouched(buf_h, dh) and untouched(buf_e, de) and bool((out["ids_buffer"][:, 5:] == -9).all())


@pytest.mark.parametrize("rows, vocab", [(24, 3000), (600, 3000)])
def test_replays_follow_their_inputs(rows, vocab):
    """Forward and backward in one graph; offsets, targets and slopes change between the replays, eager calls of the same kind run between them."""
    gen, h, e, target = inputs("bf16", [0, rows // 2, rows], rows, vocab, 64, 0, 11, lattice=True)
    h, e = h.clone(), e.clone()
    a, b = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    dh, de = torch.zeros_like(h), torch.zeros_like(e)
    c, out = scores_call("bf16", [0, rows // 2, rows], h, e, target, grad=True, top=4, d_logp=a, d_entropy=b, dh=dh, de=de)
    offsets = c.keep[0]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def calls(stream):
        P.token_scores(stream, c)
        P.token_scores_grad(stream, c)

    calls(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(side)
    for k in range(4):
        g = torch.Generator(device="cuda").manual_seed(k)
        target.copy_(torch.randint(-1, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32))
        a.copy_(torch.randn(rows, generator=g, device="cuda"))
        offsets.copy_(torch.tensor([0, rows * (k + 1) // 5, rows - k], device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {n: v.clone() for n, v in {**out, "dh": dh, "de": de}.items()}
        calls(torch.cuda.current_stream())
        torch.cuda.synchronize()
        for n, v in {**out, "dh": dh, "de": de}.items():
            assert torch.equal(torch.nan_to_num(got[n].float(), 7.0), torch.nan_to_num(v.float(), 7.0)), (k, n)
        want, far = exact_scores(offsets.tolist(), h, e, target, 1.0, a, b)
        assert bool(((got["logp"].double() - want["logp"]).abs() <= far["logp"])[:rows - k].all())
        assert bool(((got["de"].double() - want["de"]).abs() <= far["de"]).all())


def test_two_graphs_with_a_workspace_each_at_once():
    graphs = []
    for k in range(2):
        gen, h, e, target = inputs("bf16", [0, 400, 900], 900, 3000, 64, 0, 60 + k, lattice=True)
        a = torch.randn(900, generator=gen, device="cuda")
        dh, de = torch.zeros_like(h), torch.zeros_like(e)
        c, out = scores_call("bf16", [0, 400, 900], h, e, target, grad=True, top=6, d_logp=a, dh=dh, de=de)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            P.token_scores(side, c)
            P.token_scores_grad(side, c)
        graphs.append((graph, side, c, out, h, e, target, a, dh, de))
    for _ in range(3):
        for graph, side, *_ in graphs:
            with torch.cuda.stream(side):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, c, out, h, e, target, a, dh, de in graphs:
        want, far = exact_scores([0, 400, 900], h, e, target, 1.0, a)
        check_scores(out, want, far, [0, 400, 900], 900, target)
        check_top(out, want, 6, 3000, True)
        for k, got in (("dh", dh), ("de", de)):
            assert bool(((got.double() - want[k]).abs() <= far[k]).all())


def test_two_streams_with_a_workspace_each():
    jobs = []
    for k, stream in enumerate((torch.cuda.Stream(), torch.cuda.Stream())):
        gen, h, e, target = inputs("bf16", [0, 700], 700, 5000, 128, 0, 20 + k, lattice=True)
        c, out = scores_call("bf16", [0, 700], h, e, target, top=8)
        torch.cuda.synchronize()
        for _ in range(3):
            P.token_scores(stream, c)
        jobs.append((c, out, h, e, target))
    torch.cuda.synchronize()
    for c, out, h, e, target in jobs:
        want, far = exact_scores([0, 700], h, e, target)
        check_scores(out, want, far, [0, 700], 700, target)
        check_top(out, want, 8, 5000, True)


def test_the_loss_is_minus_the_log_probability():
    """Beside the loss of the same head: loss = -log p, and its gradient (sum, scale -1) that of log p, within both bounds."""
    for dtype in TYPES:
        gen, h, e, target = inputs(dtype, [0, 130], 130, 900, 64, 0, 30)
        c, out = scores_call(dtype, [0, 130], h, e, target)
        P.token_scores(torch.cuda.current_stream(), c)
        loss = torch.empty(130, device="cuda")
        x = P.CrossEntropy(dtype=TYPES[dtype][0], groups=1, rows=130, dim=64, vocab=900, offsets=c.keep[0], h=h, ldh=64, e=e, lde=64, e_stride=e.stride(0), targets=target, loss=loss)
        ws = torch.empty(P.cross_entropy_workspace(x), dtype=torch.uint8, device="cuda")
        x.set(workspace=ws, workspace_bytes=ws.numel())
        P.cross_entropy(torch.cuda.current_stream(), x)
        _, far = exact_scores([0, 130], h, e, target)
        assert bool(((loss + out["logp"]).double().abs() <= 2 * far["logp"] + 1e-6).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("bounds", [[0, 5], [0, 20, 32]])
def test_a_table_larger_than_the_caches_and_few_rows(dtype, bounds):
    rows, groups, dim, vocab = bounds[-1], len(bounds) - 1, 520, 300_001 // (len(bounds) - 1)
    gen, h, e, target = inputs(dtype, bounds, rows, vocab, dim, 0, 50, lattice=True)
    c, out = scores_call(dtype, bounds, h, e, target, top=5)
    P.token_scores(torch.cuda.current_stream(), c)
    want, far = exact_scores(bounds, h, e, target)
    check_scores(out, want, far, bounds, rows, target)
    check_top(out, want, 5, vocab, True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_the_large_tile(dtype):
    bounds, rows, vocab, dim = LARGE
    gen, h, e, target = inputs(dtype, bounds, rows, vocab, dim, 0, 40, lattice=True)
    a, b = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda") * 0.1
    dh, de = torch.empty_like(h), torch.empty_like(e)
    c, out = scores_call(dtype, bounds, h, e, target, grad=True, top=8, d_logp=a, d_entropy=b, dh=dh, de=de)
    P.token_scores(torch.cuda.current_stream(), c)
    P.token_scores_grad(torch.cuda.current_stream(), c)
    want, far = exact_scores(bounds, h, e, target, 1.0, a, b)
    check_scores(out, want, far, bounds, rows, target)
    check_top(out, want, 8, e.shape[1], True)
    for k, got in (("dh", dh), ("de", de)):
        assert bool(((got.double() - want[k]).abs() <= far[k]).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows", [6, 300])
@pytest.mark.parametrize("slopes", ["logp", "entropy", "both"])
def test_gradients_where_the_target_has_no_probability(dtype, rows, slopes):
    """Entry 10 has the logit minus infinity in every other row, and is the target of some of these: log p is minus infinity, its slope a (1 - 0), that of the entropy 0.
    The other logits are sums of multiples of 1/8, exact.  A probability is then off by less than 500 steps of 2^-23 and D by 3e-4 (scores_harness), so a slope by 1e-3 (|dz| + |b| p), its
    rounding and, in fp16, two halves of 2^-38 (|a| + 32 |b|); for de h is rounded once more."""
    vocab, dim, t = 700, 64, TYPES[dtype][1]
    u = half_step(t) if t != torch.float32 else 0.0
    gen = torch.Generator(device="cuda").manual_seed(13)
    h = torch.randint(-1, 2, (rows, dim), generator=gen, device="cuda").to(t)
    e = (torch.randint(-4, 5, (1, vocab, dim), generator=gen, device="cuda") / 8).to(t)
    h[:, 0], e[0, :, 0] = 0.0, 0.0
    h[1::2, 0], e[0, 10, 0], scale = (2.0, -3e38, 1.0) if dtype != "fp16" else (2.0 ** 14, -2.0 ** 14, 2.0 ** 101)
    if dtype == "fp16":                                                                # (a scale that brings 2^28 to infinity: the others are zero)
        e[0, :, 1:] = 0.0
    target = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    target[1::4], target[2::4] = 10, 10
    a, b = (torch.empty(rows, device="cuda").uniform_(0.2, 0.4, generator=gen) / scale for _ in range(2))
    one, two = a if slopes != "entropy" else None, b if slopes != "logp" else None
    dh, de = torch.empty_like(h), torch.empty_like(e)
    c, out = scores_call(dtype, [0, rows], h, e, target, grad=True, scale=scale, d_logp=one, d_entropy=two, dh=dh, de=de)
    P.token_scores(torch.cuda.current_stream(), c)
    P.token_scores_grad(torch.cuda.current_stream(), c)
    assert bool((out["logp"][1::4] == -math.inf).all()) and bool(torch.isfinite(out["entropy"]).all())
    f = torch.float64
    hh, ee = h.to(f), e[0].to(f)
    z = scale * (hh @ ee.t())                                                          # (there is more room above here: p is 0, log p finite)
    p, x = torch.softmax(z, 1), z - z.amax(1, keepdim=True)
    off_mean = torch.where(p > 0, x - (p * x).sum(1, keepdim=True), 0.0)
    hot = torch.zeros_like(p)
    hot.scatter_(1, target.long()[:, None], 1.0)
    a64, b64 = (v.to(f)[:, None] * scale if v is not None else torch.zeros(rows, 1, dtype=f, device="cuda") for v in (one, two))
    dz = a64 * (hot - p) - b64 * p * off_mean
    off = 1e-3 * (dz.abs() + b64 * p)
    off = off + u * (dz.abs() + off) + (2.0 ** -38 * (a64 + 32 * b64).max() if t == torch.float16 else 0.0)
    for got, left, far, right, again in ((dh, dz, off, ee, 0.0), (de[0], dz.t(), off.t(), hh, u)):
        want, magnitude = left @ right, left.abs() @ right.abs()
        bound = (far @ right.abs() + again * magnitude + (max(vocab, rows) + 8) * STEP * magnitude) * (1 + 2 * u) + (half_step(t) + STEP) * want.abs()
        bound += torch.finfo(t).smallest_normal * torch.finfo(t).eps
        # (what lies beyond the type's largest number and half a step is infinite: 150 rows of 0.3 x 2^14 in fp16, above 65520)
        over = want.abs() - bound >= torch.finfo(t).max * (1 + torch.finfo(t).eps / 4)
        assert bool(torch.where(over, got.to(f) == torch.sign(want) * math.inf, (got.to(f) - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("which", range(len(SHAPES)))
def test_rows_without_a_target_change_no_bit_of_the_others(dtype, which):
    """Whatever such a row holds, NaN, infinities or numbers whose products overflow: the results of all others are the same."""
    bounds, rows, vocab, dim = SHAPES[which]
    gen, h, e, target = inputs(dtype, bounds, rows, vocab, dim, 0, 500 + which)
    target[::3] = torch.where(torch.arange(len(target[::3]), device="cuda") % 2 == 0, -1, vocab).to(torch.int32)
    gone = (target < 0) | (target >= vocab)
    seen = []
    for fill in (0.0, float("nan"), math.inf, torch.finfo(h.dtype).max):
        h[gone] = fill
        c, out = scores_call(dtype, bounds, h, e, target, top=4, scale=0.7)
        P.token_scores(torch.cuda.current_stream(), c)
        seen.append(out)
    for out in seen[1:]:
        for k in seen[0]:
            assert torch.equal(torch.nan_to_num(out[k].float(), 7.0), torch.nan_to_num(seen[0][k].float(), 7.0)), k


@pytest.mark.parametrize("bounds, rows, vocab, dim", [([0, 9], 9, 40, 128), ([0, 40, 40, 300], 310, 500, 64), ([0, 3000, 4000], 4000, 60, 40), ([0, 700, 1500], 1500, 4100, 64)])
@pytest.mark.parametrize("small", [1e-6, 1e-5, 1e-3])
def test_small_hidden_states_in_fp16(bounds, rows, vocab, dim, small):
    """Hidden states near the least numbers of the type, in whole groups (the first) or in single columns beside large ones (the last).  The factor that a row of h gets for de is rounded
    relative to the product (scores_harness) down to half of 2^-38 of the largest |h| of the group's rows that take part, which is added here.  Rows that take none hold the largest number."""
    gen = torch.Generator(device="cuda").manual_seed(17)
    h = torch.randn(rows, dim, generator=gen, device="cuda") * small
    h[bounds[-2]:, ::4] /= small
    h = h.half()
    e = torch.randn(len(bounds) - 1, vocab, dim, generator=gen, device="cuda").half()
    target = torch.randint(-1, max(2, vocab // 20), (rows,), generator=gen, device="cuda", dtype=torch.int32)
    a, b = torch.randn(rows, generator=gen, device="cuda") * 300, torch.randn(rows, generator=gen, device="cuda") * 100
    a[::6], b[::6] = 0.0, 0.0
    h[::6] = 65504.0
    h[target < 0] = 65504.0
    dh, de = torch.empty_like(h), torch.empty_like(e)
    part = (target >= 0) & ((a != 0) | (b != 0))
    for piece, one, two in ((0, a, None), (256, a, b)):
        c, out = scores_call("fp16", bounds, h, e, target, grad=True, scale=0.5, d_logp=one, d_entropy=two, dh=dh, de=de, piece=piece)
        P.token_scores(torch.cuda.current_stream(), c)
        P.token_scores_grad(torch.cuda.current_stream(), c)
        clean = torch.where(part[:, None], h, 0.0).half()
        want, far = exact_scores(bounds, clean, e, target, 0.5, one, two)
        for g, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
            if hi > lo:
                slopes = 0.5 * (one[lo:hi].abs().double() * 2 + (two[lo:hi].abs().double() * 32 if two is not None else 0.0))       # |dz| of a row in all is less
                far["de"][g] += 2.0 ** -39 * clean[lo:hi].abs().max() * slopes[part[lo:hi]].sum()
        inside = slice(bounds[0], bounds[-1])
        for k, got, x, f in (("dh", dh[inside], want["dh"][inside], far["dh"][inside]), ("de", de, want["de"], far["de"])):
            assert bool(((got.double() - x).abs() <= f).all()), (k, piece, float(((got.double() - x).abs() / f.clamp(min=1e-300)).max()))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows", [60, 240])
@pytest.mark.parametrize("which", [0, 5, 8])
def test_gradients_of_rows_in_one_of_nine_groups(dtype, rows, which):
    """One group holds them all, the others are empty: on both sides of the bound up to which the group's own block copies its rows."""
    bounds = [0] * (which + 1) + [rows] * (9 - which)
    gen, h, e, target = inputs(dtype, bounds, rows, 90, 520, 0, 600 + which)
    a, b = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda") * 0.1
    dh, de = torch.full_like(h, float("nan")), torch.full_like(e, float("nan"))
    c, out = scores_call(dtype, bounds, h, e, target, grad=True, d_logp=a, d_entropy=b, dh=dh, de=de)
    P.token_scores(torch.cuda.current_stream(), c)
    P.token_scores_grad(torch.cuda.current_stream(), c)
    want, far = exact_scores(bounds, h, e, target, 1.0, a, b)
    check_scores(out, want, far, bounds, rows, target)
    for k, got in (("dh", dh), ("de", de)):
        assert bool(((got.double() - want[k]).abs() <= far[k]).all()), k


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, vocab, dim", [(20, 3001, 16), (300, 3001, 16), (600, 2050, 136), (1500, 8000, 136)])
@pytest.mark.parametrize("gap, scale", [(20.3, 1.0 / 0.7), (33.1, 0.9), (12.7, 1.0 / 1.3)])
def test_rows_that_are_sure_keep_their_digits_at_any_scale(dtype, rows, vocab, dim, gap, scale):
    """As above, with a scale whose product with the largest logit is rounded (by half a step of itself, which moves the others' exponentials by gap / 2 steps), in every tile."""
    t, scale = TYPES[dtype][1], float(torch.tensor(scale, dtype=torch.float32))
    h, e = torch.zeros(rows, dim, dtype=t, device="cuda"), torch.zeros(1, vocab, dim, dtype=t, device="cuda")
    h[:, 0] = gap
    gap = float(h[0, 0]) * scale
    e[0, 1234, 0] = 1.0
    target = torch.full((rows,), 1234, dtype=torch.int32, device="cuda")
    a, dh = torch.ones(rows, device="cuda"), torch.empty_like(h)
    c, out = scores_call(dtype, [0, rows], h, e, target, grad=True, top=2, scale=scale, d_logp=a, dh=dh)
    P.token_scores(torch.cuda.current_stream(), c)
    P.token_scores_grad(torch.cuda.current_stream(), c)
    rest = (vocab - 1) * math.exp(-gap)
    logp, H = -math.log1p(rest), math.log1p(rest) + gap * rest / (1 + rest)
    rel = (2 * gap + 40 + vocab / 64) * STEP
    for got, want in ((out["logp"], logp), (out["entropy"], H), (out["top_logp"][:, 0], logp)):
        assert bool(((got.double() - want).abs() <= rel * abs(want) * 1.01).all())
    assert bool((out["top_ids"][:, 0] == 1234).all()) and bool((out["top_ids"][:, 1] == 0).all())
    # dh[0] = scale a (1 - p) e[1234][0]; in 16 bits rounded twice
    want = scale * rest / (1 + rest)
    u = 2 * torch.finfo(t).eps if t != torch.float32 else 0.0
    low = 2.0 ** -37 if t == torch.float16 else 0.0
    assert bool(((dh[:, 0].double() - want).abs() <= (u + rel + 4 * STEP) * want * 1.01 + low + torch.finfo(t).smallest_normal * torch.finfo(t).eps).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows, vocab, dim", [(20, 3001, 16), (300, 3001, 16), (600, 2050, 136), (1500, 8000, 136)])
@pytest.mark.parametrize("gap, scale", [(20.0, 1.0), (20.3, 1.0 / 0.7), (33.1, 0.9), (12.7, 1.0 / 1.3)])
def test_the_entropys_slope_of_a_sure_row_keeps_its_digits(dtype, rows, vocab, dim, gap, scale):
    """The largest entry's slope is b p D, D = -gap rest / (1 + rest), with the error of D (that of H above), of p and one rounding, after the mantissa of the target's."""
    t, scale = TYPES[dtype][1], float(torch.tensor(scale, dtype=torch.float32))
    h, e = torch.zeros(rows, dim, dtype=t, device="cuda"), torch.zeros(1, vocab, dim, dtype=t, device="cuda")
    h[:, 0] = gap
    gap = float(h[0, 0]) * scale
    e[0, 1234, 0] = 1.0
    target = torch.full((rows,), 77, dtype=torch.int32, device="cuda")
    b, dh = torch.ones(rows, device="cuda"), torch.empty_like(h)
    c, out = scores_call(dtype, [0, rows], h, e, target, grad=True, scale=scale, d_entropy=b, dh=dh)
    P.token_scores(torch.cuda.current_stream(), c)
    P.token_scores_grad(torch.cuda.current_stream(), c)
    rest = (vocab - 1) * math.exp(-gap)
    want = -scale * gap * rest / (1 + rest) ** 2
    rel = (2 * gap + 60 + vocab / 64) * STEP + (torch.finfo(t).eps if t != torch.float32 else 0.0)
    low = 32 * 2.0 ** -38 * scale if t == torch.float16 else 0.0
    assert bool(((dh[:, 0].double() - want).abs() <= rel * abs(want) * 1.01 + low + torch.finfo(t).smallest_normal * torch.finfo(t).eps).all())
