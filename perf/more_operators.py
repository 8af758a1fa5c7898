"""Timed cases of the routing between groups, the token scores and the AdamW step.

Routing takes every token's row to the rows of the groups that its router chose (the ragged batches of the grouped products) and
back.  Token scores are log probability, entropy and most probable alternatives at a vocabulary head whose logits are not kept, and
their gradients.  The AdamW step updates all tensors of all workers at a time.  Every case runs in two forms on the same inputs: the
plain one, elementary torch operations in fp32 rounded once at the end, and the calls a user makes of the library (`own`).  `exact`
is the definition in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = 32                                       # values of a tensor's state that share a scale
CAPACITY = 1.25                                  # rows that a group takes at most, times the mean, where a case limits them
SCALE = 0.8125                                   # logits over a temperature

# Cost of the largest listed case of each kind, which no drawn one exceeds (bytes; flops for the scores; parameters).
MOST_ROUTED = 16384 * 8 * 2048
MOST_SCORES = 2 * 8192 * 131072 * 2048
MOST_PARAMETERS = 16 * 11_200_000


def listed():
    return [
        # a decoding step: sixteen tokens to two of eight experts each, launches count
        dict(name="dispatch_decode", op="dispatch", dtype="bf16", tokens=16, choices=2, groups=8, width=1024, dropped=0.0, limited=False),
        # a training batch over many small experts, each with a capacity
        dict(name="dispatch_batch", op="dispatch", dtype="bf16", tokens=16384, choices=8, groups=128, width=2048, dropped=0.0, limited=True),
        # back from two of sixteen experts with weights, half precision, rows that are no multiple of a line, padded tokens
        dict(name="combine_ragged", op="combine", dtype="fp16", tokens=5003, choices=2, groups=16, width=1000, dropped=0.1, limited=False),
        # the training batch's way back through the weighted sum: gradients of the rows and of the weights
        dict(name="combine_grad_batch", op="combine_grad", dtype="bf16", tokens=16384, choices=8, groups=128, width=2048, dropped=0.0, limited=True),
        # the next token of four sequences: every entry of a large table read once, eight alternatives each
        dict(name="scores_decode", op="scores", dtype="bf16", groups=1, rows=4, dim=2048, vocab=131072, top=8, masked=0.0, grad=False),
        # a reference model's pass over a batch of texts with its alternatives, the largest
        dict(name="scores_large", op="scores", dtype="bf16", groups=1, rows=8192, dim=2048, vocab=131072, top=8, masked=0.0, grad=False),
        # a policy's training step with an entropy bonus: four workers, a quarter of the rows are prompt
        dict(name="scores_train", op="scores", dtype="bf16", groups=4, rows=4096, dim=1024, vocab=32003, top=0, masked=0.25, grad=True),
        # a model in 32 bits with sizes that no tile divides, five alternatives
        dict(name="scores_fp32", op="scores", dtype="fp32", groups=2, rows=509, dim=512, vocab=5003, top=5, masked=0.1, grad=True),
        # a small perceptron's six tensors: one launch's time
        dict(name="adamw_small", op="adamw", dtype="fp32", grad="fp32", copy="", bits=32, workers=1, tensors=6, parameters=70_000),
        # sixteen workers' models of 62 tensors with gradients and working copies in 16 bits
        dict(name="adamw_workers", op="adamw", dtype="fp32", grad="bf16", copy="bf16", bits=32, workers=16, tensors=62, parameters=11_200_000),
        # one large model, its states in 8 bits
        dict(name="adamw_8bit", op="adamw", dtype="fp32", grad="bf16", copy="bf16", bits=8, workers=1, tensors=32, parameters=138_000_000),
        # no copy in 32 bits at all: parameters and gradients in 16, states in 8, three workers
        dict(name="adamw_8bit_half", op="adamw", dtype="bf16", grad="bf16", copy="", bits=8, workers=3, tensors=40, parameters=1_000_003),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; a multiple of 8 about half the time (model widths are)."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n >= 16 and rng.random() < 0.5:
        n = n // 8 * 8
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(["dispatch", "combine", "combine_grad", "dispatch_grad", "scores", "scores", "scores", "adamw", "adamw", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    while True:
        if op == "scores":
            case = dict(op=op, dtype=dtype, groups=rng.choice([1, 1, 2, 4, 7]), rows=_spread(rng, 1, 8192), dim=_spread(rng, 32, 4096),
                        vocab=_spread(rng, 100, 131072), top=rng.choice([0, 1, 5, 8, 20]), masked=rng.choice([0.0, 0.0, 0.1, 0.5]),
                        grad=rng.random() < 0.5)
            if work(case)["flops"] <= MOST_SCORES / 4 and case["groups"] * case["vocab"] * case["dim"] <= 2 ** 28:
                return case
        elif op == "adamw":
            kind = rng.choice([("fp32", "fp32", ""), ("fp32", "bf16", "bf16"), ("fp32", "fp16", "fp16"), ("bf16", "bf16", ""), ("fp16", "fp16", "")])
            case = dict(op=op, dtype=kind[0], grad=kind[1], copy=kind[2], bits=rng.choice([32, 8]), workers=rng.choice([1, 1, 2, 4, 16]),
                        tensors=rng.choice([1, 2, 7, 62, 150, 400]), parameters=_spread(rng, 2000, 30_000_000))
            if case["workers"] * case["parameters"] <= MOST_PARAMETERS and case["tensors"] * 4 <= case["parameters"]:
                return case
        else:
            choices = rng.choice([1, 2, 2, 4, 8])
            case = dict(op=op, dtype=dtype, tokens=_spread(rng, 1, 65536), choices=choices, groups=max(choices, rng.choice([2, 8, 16, 60, 128, 512])),
                        width=_spread(rng, 32, 8192), dropped=rng.choice([0.0, 0.0, 0.1, 0.5]), limited=rng.random() < 0.3)
            if case["tokens"] * case["choices"] * case["width"] * SIZE[dtype] <= 2 * MOST_ROUTED:
                return case


def _valid(case):
    """Rows that take part."""
    return case["rows"] - int(case["rows"] * case["masked"])


def work(case):
    if case["op"] == "adamw":
        n = case["workers"] * case["parameters"]
        state = 16 if case["bits"] == 32 else 4 + 4 / BLOCK
        return {"bytes": n * (2 * SIZE[case["dtype"]] + SIZE[case["grad"]] + (SIZE[case["copy"]] if case["copy"] else 0) + state), "flops": 15 * n}
    s = SIZE[case["dtype"]]
    if case["op"] == "scores":
        rows = _valid(case)
        part = case["dim"] * case["vocab"] * min(case["groups"], max(1, rows))
        moved = s * (rows * case["dim"] + part) + case["rows"] * (12 + 8 * case["top"])
        if case["grad"]:
            moved += s * (case["rows"] * case["dim"] + case["groups"] * case["dim"] * case["vocab"])
        return {"bytes": moved, "flops": (6 if case["grad"] else 2) * rows * case["dim"] * case["vocab"]}
    pairs = case["tokens"] * case["choices"]
    one, all_ = s * case["tokens"] * case["width"], int(s * pairs * case["width"] * (1 - case["dropped"]))
    if case["op"] == "dispatch":
        return {"bytes": one + all_ + 8 * pairs + 8 * case["groups"], "flops": pairs}
    if case["op"] == "combine_grad":
        return {"bytes": one + 2 * all_ + 12 * pairs, "flops": 3 * pairs * case["width"]}
    return {"bytes": one + all_ + (8 if case["op"] == "combine" else 4) * pairs, "flops": 2 * pairs * case["width"]}


# ---- state ------------------------------------------------------------------------------------------

def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed * 1_000_003 + 29)
    st = {"case": case}
    if case["op"] == "adamw":
        _prepare_adamw(st, gen, dev, seed)
    elif case["op"] == "scores":
        _prepare_scores(st, gen, dev, seed)
    else:
        _prepare_route(st, gen, dev)
    if own:
        _prepare_own(st, dev)
    return st


def _prepare_route(st, gen, dev):
    """A router's choices: some experts more popular than others, no expert twice for a token, padded tokens without any."""
    case, t = st["case"], TYPES[st["case"]["dtype"]]
    tokens, k, groups, width = case["tokens"], case["choices"], case["groups"], case["width"]
    score = torch.randn(groups, generator=gen, device=dev) * 0.5 - torch.log(-torch.log(torch.rand(tokens, groups, generator=gen, device=dev).clamp(1e-9, 1 - 1e-6)))
    best, experts = torch.topk(score, k, dim=1)
    experts = experts.to(torch.int32)
    experts[torch.rand(tokens, generator=gen, device=dev) < case["dropped"]] = -1
    st["experts"] = experts.contiguous()
    st["capacity"] = int(math.ceil(CAPACITY * tokens * k / groups)) if case["limited"] else 0
    if case["op"] == "dispatch":
        st["x"] = torch.randn(tokens, width, generator=gen, device=dev).to(t)
        return
    st["place"] = _sort(st["experts"], groups, st["capacity"])[1]
    pairs = tokens * k
    if case["op"] != "dispatch_grad":
        st["weights"] = torch.softmax(best, dim=1).contiguous()
    if case["op"] != "combine":
        name = "dy" if case["op"] == "combine_grad" else "dxs"
        st[name] = (torch.randn(tokens if name == "dy" else pairs, width, generator=gen, device=dev) * 0.1).to(t)
    if case["op"] != "dispatch_grad":
        st["ys"] = torch.randn(pairs, width, generator=gen, device=dev).to(t)


def _bounds(case, seed):
    """Ragged row bounds of the groups."""
    g, rows = case["groups"], case["rows"]
    if rows <= g:
        return [min(i, rows) for i in range(g + 1)]
    r = random.Random(seed * 7919 + rows)
    share = [r.uniform(0.5, 1.5) for _ in range(g)]
    total, at, bounds = sum(share), 0.0, [0]
    for part in share:
        at += part
        bounds.append(int(round(rows * at / total)))
    bounds[-1] = rows
    return bounds


def _prepare_scores(st, gen, dev, seed):
    """Hidden states in steps of 1/16 and tables in steps of 2^-8: logits are then sums without rounding, in any order and type, so that the
    order of the alternatives (ties among them) is the same whatever adds them up."""
    case, t = st["case"], TYPES[st["case"]["dtype"]]
    rows, dim, vocab, g = case["rows"], case["dim"], case["vocab"], case["groups"]
    st["bounds"] = _bounds(case, seed)
    st["offsets"] = torch.tensor(st["bounds"], dtype=torch.int64, device=dev)
    st["h"] = (torch.round(torch.randn(rows, dim, generator=gen, device=dev) * 16) / 16).to(t)
    st["e"] = torch.empty((g, vocab, dim), dtype=t, device=dev)
    for one in st["e"]:
        one.copy_(torch.round(torch.randn(vocab, dim, generator=gen, device=dev) * (512 / math.sqrt(dim))) / 256)
    target = torch.randint(0, vocab, (rows,), generator=gen, device=dev, dtype=torch.int32)
    target[torch.randperm(rows, generator=gen, device=dev)[: rows - _valid(case)]] = -1
    st["target"] = target
    if case["grad"]:
        st["d_logp"] = torch.randn(rows, generator=gen, device=dev) / rows            # advantages
        st["d_entropy"] = torch.full((rows,), 0.01 / rows, device=dev)


def _sizes(case):
    """A list of tensor sizes, log-uniform, that sum to `parameters`; the same for every seed."""
    n, total = case["tensors"], case["parameters"]
    r = random.Random(n * 100_003 + total)
    raw = [math.exp(r.uniform(math.log(4.0), math.log(max(8.0, 4.0 * total / n)))) for _ in range(n)]
    sizes = [max(1, int(x * total / sum(raw))) for x in raw]
    at = sizes.index(max(sizes))
    sizes[at] += total - sum(sizes)
    return sizes


def _layout(case):
    """(sizes, first elements, elements from worker to worker): every tensor begins on a block."""
    sizes, at, first = _sizes(case), 0, []
    for n in sizes:
        first.append(at)
        at += -(-n // BLOCK) * BLOCK
    return sizes, first, at


def _prepare_adamw(st, gen, dev, seed):
    case = st["case"]
    sizes, first, stride = _layout(case)
    w = case["workers"]
    real = torch.zeros(stride, dtype=torch.bool, device=dev)
    for n, at in zip(sizes, first):
        real[at:at + n] = True

    def normal(std):
        return torch.randn(w, stride, generator=gen, device=dev) * std * real

    st["sizes"], st["first"], st["stride"] = sizes, first, stride
    st["decay"] = [0.1 if n >= 1024 else 0.0 for n in sizes]                   # biases and norms do not decay
    st["hyper"] = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1000, grad_scale=0.5, seed=(seed * 2_654_435_761 + 12345) % 2 ** 32)
    loud = torch.exp(torch.randn(w, stride // BLOCK, generator=gen, device=dev)).repeat_interleave(BLOCK, dim=1)     # gradients of unlike sizes
    st["p"] = normal(0.02).to(TYPES[case["dtype"]])
    st["g"] = (normal(0.01) * loud).to(TYPES[case["grad"]])
    m, v = normal(0.003) * loud, (normal(0.005) * loud).square() + 1e-9 * real
    if case["bits"] == 32:
        st["m"], st["v"] = m, v
    else:
        blocks = w * stride // BLOCK
        half = torch.full((blocks, BLOCK), 0x8000, dtype=torch.int64, device=dev)
        st["m"], st["m_scales"] = (x.view(w, -1) for x in _store_signed(m.view(blocks, BLOCK), half))
        st["v"], st["v_scales"] = (x.view(w, -1) for x in _store_square(v.view(blocks, BLOCK), half))
    if case["copy"]:
        st["copy"] = torch.zeros((w, stride), dtype=TYPES[case["copy"]], device=dev)


def _prepare_own(st, dev):
    """Output buffers and the description of the call, which a user's program keeps from step to step."""
    import paper_1906_12043_amd as P

    case = st["case"]
    kinds = {"bf16": P.BF16, "fp16": P.F16, "fp32": P.F32}
    if case["op"] == "adamw":
        tensors = []
        for n, at, decay in zip(st["sizes"], st["first"], st["decay"]):
            one = dict(n=n, p=st["p"][0, at:], g=st["g"][0, at:], m=st["m"][0, at:], v=st["v"][0, at:], weight_decay=decay, lr_scale=1.0)
            if case["bits"] == 8:
                one.update(m_scales=st["m_scales"][0, at // BLOCK:], v_scales=st["v_scales"][0, at // BLOCK:])
            if case["copy"]:
                one.update(copy=st["copy"][0, at:])
            tensors.append(one)
        more = dict(copy_dtype=kinds[case["copy"]]) if case["copy"] else {}
        st["call"] = P.AdamW(tensors=tensors, dtype=kinds[case["dtype"]], grad_dtype=kinds[case["grad"]], workers=case["workers"], stride=st["stride"],
                             state=P.ADAMW_STATE_F32 if case["bits"] == 32 else P.ADAMW_STATE_8BIT, **st["hyper"], **more)
        return
    t, kind = TYPES[case["dtype"]], kinds[case["dtype"]]
    if case["op"] == "scores":
        rows, dim, vocab, g, top = case["rows"], case["dim"], case["vocab"], case["groups"], case["top"]
        st["logp"], st["entropy"] = torch.zeros(rows, device=dev), torch.zeros(rows, device=dev)
        f = dict(dtype=kind, groups=g, rows=rows, dim=dim, vocab=vocab, offsets=st["offsets"], h=st["h"], ldh=dim, e=st["e"], lde=dim,
                 e_stride=vocab * dim, targets=st["target"], scale=SCALE, logp=st["logp"], entropy=st["entropy"])
        if top:
            st["top_ids"], st["top_logp"] = torch.zeros((rows, top), dtype=torch.int32, device=dev), torch.zeros((rows, top), device=dev)
            f.update(top=top, top_ids=st["top_ids"], top_logp=st["top_logp"], ld_top=top)
        if case["grad"]:
            st["norms"] = torch.empty((rows, 4), device=dev)
            st["dh"], st["de"] = torch.empty((rows, dim), dtype=t, device=dev), torch.empty((g, vocab, dim), dtype=t, device=dev)
            f.update(norms=st["norms"], d_logp=st["d_logp"], d_entropy=st["d_entropy"], dh=st["dh"], lddh=dim, de=st["de"], ldde=dim,
                     de_stride=vocab * dim)
        call = P.TokenScores(**f)
        need = P.token_scores_workspace(call, P.TOKEN_SCORES_FORWARD)
        if case["grad"]:
            need = max(need, P.token_scores_workspace(call, P.TOKEN_SCORES_GRAD))
        st["workspace"] = torch.empty(max(1, need), dtype=torch.uint8, device=dev)
        call.set(workspace=st["workspace"], workspace_bytes=st["workspace"].numel())
        st["call"] = call
        return
    tokens, k, groups, width = case["tokens"], case["choices"], case["groups"], case["width"]
    f = dict(dtype=kind, groups=groups, tokens=tokens, choices=k, width=width, capacity=st["capacity"])
    if case["op"] == "dispatch":
        st["offsets"], st["place"] = torch.zeros(groups + 1, dtype=torch.int64, device=dev), torch.zeros((tokens, k), dtype=torch.int32, device=dev)
        st["xs"] = torch.zeros((tokens * k, width), dtype=t, device=dev)
        f.update(experts=st["experts"], ld_experts=k, offsets=st["offsets"], x=st["x"], ldx=width, xs=st["xs"], ldxs=width)
    elif case["op"] == "combine":
        st["y"] = torch.empty((tokens, width), dtype=t, device=dev)
        f.update(weights=st["weights"], ld_weights=k, ys=st["ys"], ldys=width, y=st["y"], ldy=width)
    elif case["op"] == "combine_grad":
        st["dys"], st["dweights"] = torch.zeros((tokens * k, width), dtype=t, device=dev), torch.empty((tokens, k), device=dev)
        f.update(weights=st["weights"], ld_weights=k, ys=st["ys"], ldys=width, dy=st["dy"], lddy=width, dys=st["dys"], lddys=width,
                 dweights=st["dweights"], ld_dweights=k)
    else:
        st["dx"] = torch.empty((tokens, width), dtype=t, device=dev)
        f.update(dxs=st["dxs"], lddxs=width, dx=st["dx"], lddx=width)
    call = P.Route(place=st["place"], ld_place=k, **f)
    if case["op"] == "dispatch":
        st["workspace"] = torch.empty(max(1, P.route_workspace(call)), dtype=torch.uint8, device=dev)
        call.set(workspace=st["workspace"], workspace_bytes=st["workspace"].numel())
    st["call"] = call


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    import paper_1906_12043_amd as P

    case, stream = st["case"], torch.cuda.current_stream()
    if case["op"] == "adamw":
        P.adamw(stream, st["call"])
        return _adamw_outputs(st)
    if case["op"] == "scores":
        P.token_scores(stream, st["call"])
        out = {"logp": st["logp"], "entropy": st["entropy"]}
        if case["top"]:
            out.update(top_ids=st["top_ids"], top_logp=st["top_logp"])
        if case["grad"]:
            P.token_scores_grad(stream, st["call"])
            out.update(dh=st["dh"], de=st["de"])
        return out
    if case["op"] == "dispatch":
        P.route_sort(stream, st["call"])
        P.route_dispatch(stream, st["call"])
        return {"offsets": st["offsets"], "place": st["place"], "xs": st["xs"]}
    if case["op"] == "combine":
        P.route_combine(stream, st["call"])
        return st["y"]
    if case["op"] == "combine_grad":
        P.route_combine_grad(stream, st["call"])
        return {"dys": st["dys"], "dweights": st["dweights"]}
    P.route_dispatch_grad(stream, st["call"])
    return st["dx"]


def _run_plain(st):
    case = st["case"]
    if case["op"] == "adamw":
        return _adamw_plain(st)
    if case["op"] == "scores":
        return _scores_plain(st)
    return _route_plain(st)


# ---- routing, plainly ---------------------------------------------------------------------------------

def _sort(experts, groups, capacity):
    """(offsets, place): pairs in the order of group, token, choice; -1 for a pair without a group or beyond the group's capacity."""
    flat = experts.reshape(-1).to(torch.int64)
    key = torch.where((flat >= 0) & (flat < groups), flat, groups)
    count = torch.bincount(key, minlength=groups + 1)
    _, order = torch.sort(key, stable=True)
    rank = torch.empty_like(key)
    rank[order] = torch.arange(key.numel(), device=key.device) - (torch.cumsum(count, 0) - count)[key[order]]
    taken = torch.clamp(count[:groups], max=capacity) if capacity else count[:groups]
    offsets = torch.nn.functional.pad(torch.cumsum(taken, 0), (1, 0))
    kept = (key < groups) & ((rank < capacity) if capacity else (rank >= 0))
    place = torch.where(kept, offsets[torch.clamp(key, max=groups - 1)] + rank, -1).to(torch.int32)
    return offsets, place.view(experts.shape)


def _route_plain(st):
    case, f = st["case"], torch.float32
    t, k = TYPES[case["dtype"]], case["choices"]
    if case["op"] == "dispatch":
        offsets, place = _sort(st["experts"], case["groups"], st["capacity"])
        xs = torch.zeros((case["tokens"] * k, case["width"]), dtype=t, device=place.device)
        pair = torch.nonzero(place.view(-1) >= 0)[:, 0]
        xs[place.view(-1)[pair].to(torch.int64)] = st["x"][pair // k]
        return {"offsets": offsets, "place": place, "xs": xs}
    at = st["place"].to(torch.int64)
    has, at = (at >= 0)[:, :, None], torch.clamp(at, min=0)
    if case["op"] == "combine":
        return (torch.where(has, st["ys"][at].to(f), 0.0) * st["weights"][:, :, None]).sum(1).to(t)
    if case["op"] == "dispatch_grad":
        return torch.where(has, st["dxs"][at].to(f), 0.0).sum(1).to(t)
    dy = st["dy"].to(f)[:, None, :]
    dweights = (torch.where(has, st["ys"][at].to(f), 0.0) * dy).sum(2)
    pair = torch.nonzero(st["place"].view(-1) >= 0)[:, 0]
    dys = torch.zeros_like(st["ys"])
    dys[st["place"].view(-1)[pair].to(torch.int64)] = (dy * st["weights"][:, :, None]).to(t).view(-1, case["width"])[pair]
    return {"dys": dys, "dweights": dweights}


# ---- scores, plainly ----------------------------------------------------------------------------------

def _groups(st):
    return [(g, a, b) for g, (a, b) in enumerate(zip(st["bounds"], st["bounds"][1:])) if b > a]


def _scores_plain(st):
    case, f = st["case"], torch.float32
    t, dev, top = TYPES[case["dtype"]], st["h"].device, case["top"]
    rows = case["rows"]
    out = {"logp": torch.zeros(rows, device=dev), "entropy": torch.zeros(rows, device=dev)}
    if top:
        out["top_ids"], out["top_logp"] = torch.full((rows, top), -1, dtype=torch.int32, device=dev), torch.full((rows, top), float("-inf"), device=dev)
    if case["grad"]:
        out["dh"], out["de"] = torch.zeros_like(st["h"]), torch.zeros_like(st["e"])
    for g, a, b in _groups(st):
        keep = st["target"][a:b] >= 0
        at = torch.clamp(st["target"][a:b].to(torch.int64), min=0)[:, None]
        h, e = torch.where(keep[:, None], st["h"][a:b].to(f), 0.0), st["e"][g].to(f)
        z = (h @ e.t()).mul_(SCALE)
        most = z.amax(dim=1, keepdim=True)
        z -= most                                                              # distances below the largest
        p = torch.exp(z)
        total = p.sum(dim=1, keepdim=True, dtype=torch.float64)
        norm = torch.log(total).to(f)
        p /= total.to(f)
        mean = (p * z).sum(dim=1, keepdim=True, dtype=torch.float64).to(f)
        out["logp"][a:b] = torch.where(keep, (z.gather(1, at) - norm)[:, 0], 0.0)
        out["entropy"][a:b] = torch.where(keep, (norm - mean)[:, 0], 0.0)
        if case["grad"]:
            one, two = st["d_logp"][a:b, None], st["d_entropy"][a:b, None]
            dz = p * ((mean - z) * two - one)
            dz.scatter_add_(1, at, one)
            dz *= keep.to(f)[:, None] * SCALE
            out["dh"][a:b] = (dz @ e).to(t)
            out["de"][g] = (dz.t() @ h).to(t)
            del dz
        for j in range(min(top, case["vocab"])):                               # the largest left, the first of equal ones
            best = z.argmax(dim=1, keepdim=True)
            out["top_ids"][a:b, j] = torch.where(keep, best[:, 0], -1).to(torch.int32)
            out["top_logp"][a:b, j] = torch.where(keep, (z.gather(1, best) - norm)[:, 0], float("-inf"))
            z.scatter_(1, best, float("-inf"))
    return out


# ---- AdamW, plainly -----------------------------------------------------------------------------------

def _power(e):
    """2^e as fp32, e in -126 .. 127, put together from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _random(seed, sizes, first, stride, workers, dev):
    """32 random bits for every element, from the seed, the tensor's number, the worker and the element's place in the tensor."""
    word = 0xffffffff
    which = torch.repeat_interleave(torch.arange(len(sizes), device=dev), torch.tensor([-(-n // BLOCK) * BLOCK for n in sizes], device=dev))
    place = torch.arange(stride, device=dev) - torch.tensor(first, device=dev)[which]
    x = ((place * 0x9E3779B1) & word) + which * 0x632BE5AB
    x = (x[None, :] + seed + torch.arange(workers, device=dev)[:, None] * 0x85157AF5) & word
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & word
    x = ((x ^ (x >> 15)) * 0x846CA68B) & word
    return x ^ (x >> 16)


def _block_scale(size, low):
    """Smallest e, not below `low`, for which the largest finite magnitude of a block is at most 448 2^e."""
    mant, exp = torch.frexp(torch.where(torch.isfinite(size), size, 0.0).amax(dim=1))
    e = exp - torch.where(mant <= 0.875, 9, 8)
    return torch.where(mant == 0, low, e).clamp(min=low).to(torch.int32)


def _code_below(y):
    """(number, value and step to the next one) of the largest e4m3 magnitude not above y; y counts in the smallest one's units."""
    _, e = torch.frexp(y)
    step = _power((e - 4).clamp(min=0))
    low = torch.floor(y / step) * step
    code = torch.where(y < 8, low, low / step + 8 * (e - 4).to(torch.float32)).to(torch.int64)
    return code, low, step


def _store_signed(m, bits):
    """(codes, scales): rounded up where the way there, in 65536ths of the step, is above 16 random bits."""
    e = _block_scale(m.abs(), -117)
    fine = torch.isfinite(m)
    up = 9 - e
    y = torch.where(fine, m.abs(), 0.0) * _power(up // 2)[:, None] * _power(up - up // 2)[:, None]
    code, low, step = _code_below(y)
    code = code + ((y - low) / step * 65536.0 > bits.to(torch.float32)).to(torch.int64)
    code = torch.where(fine, code, 0x7f) | (torch.signbit(m).to(torch.int64) << 7)
    return code.to(torch.uint8), (e + 127).to(torch.uint8)


def _store_square(v, bits):
    """The square root's code, rounded so that the square of what is stored is v in the mean; what is not zero stays so."""
    r = torch.sqrt(v.double()).float()
    e = _block_scale(r, -51)
    fine = torch.isfinite(r)
    up = _power(9 - e)[:, None]
    y, w = torch.where(fine, r, 0.0) * up, torch.where(fine, v, 0.0) * up * up
    code, low, step = _code_below(y)
    code = code + (w - low * low > bits.to(torch.float32) * 2.0 ** -16 * (step * (2 * low + step))).to(torch.int64)
    code = torch.where((code == 0) & (r > 0), 1, code)
    return torch.where(fine, code, 0x7f).to(torch.uint8), (e + 127).to(torch.uint8)


def _load(codes, scales):
    e = scales.to(torch.int32) - 127
    return codes.view(torch.float8_e4m3fn).to(torch.float32) * _power(e // 2)[:, None] * _power(e - e // 2)[:, None]


def _adamw_plain(st):
    case, f, hy = st["case"], torch.float32, st["hyper"]
    dev, eight = st["p"].device, case["bits"] == 8
    blocks = st["p"].numel() // BLOCK
    b1, b2 = float(np.float32(hy["beta1"])), float(np.float32(hy["beta2"]))
    c1, c2 = float(np.float32(1.0 - b1)), float(np.float32(1.0 - b2))
    span = torch.tensor([-(-n // BLOCK) * BLOCK for n in st["sizes"]], device=dev)
    decay = torch.repeat_interleave(torch.tensor(st["decay"], device=dev), span)
    p, g = st["p"].to(f), st["g"].to(f) * hy["grad_scale"]
    m, v = st["m"], st["v"]
    if eight:
        m = _load(m.view(blocks, BLOCK), st["m_scales"].view(-1)).view(p.shape)
        v = _load(v.view(blocks, BLOCK), st["v_scales"].view(-1)).square().view(p.shape)
    m = m * b1 + g * c1
    v = v * b2 + (g * c2) * g
    bias1, bias2 = 1.0 - b1 ** hy["step"], 1.0 - b2 ** hy["step"]
    p = p * (1.0 - hy["lr"] * decay) - (hy["lr"] / bias1) * m / (torch.sqrt(v / bias2) + hy["eps"])
    st["p"].copy_(p)
    if case["copy"]:
        st["copy"].copy_(p)
    if not eight:
        st["m"].copy_(m)
        st["v"].copy_(v)
        return _adamw_outputs(st)
    bits = _random(hy["seed"], st["sizes"], st["first"], st["stride"], case["workers"], dev).view(blocks, BLOCK)
    for name, value, store, part in (("m", m, _store_signed, bits >> 16), ("v", v, _store_square, bits & 0xffff)):
        codes, scales = store(value.view(blocks, BLOCK), part)
        st[name].copy_(codes.view(p.shape))
        st[name + "_scales"].copy_(scales.view(st[name + "_scales"].shape))
    return _adamw_outputs(st)


def _adamw_outputs(st):
    out = {"p": st["p"]}
    if st["case"]["copy"]:
        out["copy"] = st["copy"]
    if st["case"]["bits"] == 32:
        return {**out, "m": st["m"], "v": st["v"]}
    # codes as the numbers they stand for, over their block's scale; scales by their exponent
    return {**out, "m": st["m"].view(torch.float8_e4m3fn), "v_root": st["v"].view(torch.float8_e4m3fn), "m_scales": st["m_scales"], "v_scales": st["v_scales"]}


# ---- the definition in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    return {"adamw": _exact_adamw, "scores": _exact_scores}.get(case["op"], _exact_route)(st)


def _exact_route(st):
    """By counting: a pair's row is the number of kept pairs of smaller groups and of earlier ones of its own."""
    case, d = st["case"], torch.float64
    k, dev = case["choices"], st["experts"].device
    if case["op"] == "dispatch":
        flat = st["experts"].cpu().numpy().reshape(-1)
        taken, rank = np.zeros(case["groups"], np.int64), np.full(flat.size, -1, np.int64)
        for g in range(case["groups"]):
            mine = np.flatnonzero(flat == g)
            mine = mine[: st["capacity"]] if st["capacity"] else mine
            taken[g] = mine.size
            rank[mine] = np.arange(mine.size)
        offsets = np.concatenate([[0], np.cumsum(taken)])
        place = np.where(rank >= 0, offsets[np.maximum(flat, 0)] + rank, -1)
        source = torch.zeros(flat.size, dtype=torch.int64, device=dev)
        kept = torch.from_numpy(np.flatnonzero(rank >= 0)).to(dev)
        source[torch.from_numpy(place[rank >= 0]).to(dev)] = kept // k
        xs = st["x"][source]
        xs[int(offsets[-1]):] = 0
        return {"offsets": torch.from_numpy(offsets), "place": torch.from_numpy(place.astype(np.int32)).view(-1, k), "xs": xs}
    rows = st["ys"] if "ys" in st else st["dxs"]
    y = torch.zeros((case["tokens"], case["width"]), dtype=d, device=dev)
    dys, dw = torch.zeros(rows.shape, dtype=d if case["op"] == "combine_grad" else torch.bool, device=dev), torch.zeros((case["tokens"], k), dtype=d, device=dev)
    for j in range(k):
        who = torch.nonzero(st["place"][:, j] >= 0)[:, 0]
        at = st["place"][who, j].to(torch.int64)
        if case["op"] == "combine_grad":
            dys[at] = st["dy"][who].to(d) * st["weights"][who, j].to(d)[:, None]
            dw[who, j] = (st["dy"][who].to(d) * rows[at].to(d)).sum(1)
        else:
            y[who] += rows[at].to(d) * (st["weights"][who, j].to(d)[:, None] if case["op"] == "combine" else 1.0)
    return {"dys": dys, "dweights": dw} if case["op"] == "combine_grad" else y


def _exact_scores(st):
    case, d = st["case"], torch.float64
    dev, top = st["h"].device, case["top"]
    rows = case["rows"]
    out = {"logp": torch.zeros(rows, dtype=d, device=dev), "entropy": torch.zeros(rows, dtype=d, device=dev)}
    if top:
        out["top_ids"], out["top_logp"] = torch.full((rows, top), -1, dtype=torch.int32, device=dev), torch.full((rows, top), float("-inf"), dtype=d, device=dev)
    if case["grad"]:
        out["dh"], out["de"] = torch.zeros(st["h"].shape, dtype=d, device=dev), torch.zeros(st["e"].shape, dtype=d, device=dev)
    number = torch.arange(rows, device=dev)
    for g, a, b in _groups(st):
        e = st["e"][g].to(d)
        mine = number[a:b][st["target"][a:b] >= 0]
        for part in mine.split(1024):
            h, t = st["h"][part].to(d), st["target"][part].to(torch.int64)
            z = torch.matmul(h, e.t()) * float(np.float32(SCALE))
            logp = z - torch.logsumexp(z, dim=1, keepdim=True)
            entropy = -(torch.exp(logp) * logp).sum(1)
            out["logp"][part], out["entropy"][part] = logp[torch.arange(len(part), device=dev), t], entropy
            if top:
                n = min(top, case["vocab"])
                edge = torch.topk(z, n, dim=1).values[:, -1:]
                for i, r in enumerate(part.tolist()):                          # those not below the last one, larger first, lower index first
                    who = torch.nonzero(z[i] >= edge[i])[:, 0]
                    who = who[torch.sort(z[i, who], descending=True, stable=True).indices[:n]]
                    out["top_ids"][r, :n], out["top_logp"][r, :n] = who.to(torch.int32), logp[i, who]
            if case["grad"]:
                one, two = st["d_logp"][part].to(d)[:, None], st["d_entropy"][part].to(d)[:, None]
                slope = -torch.exp(logp) * (one + two * (logp + entropy[:, None]))
                slope[torch.arange(len(part), device=dev), t] += one[:, 0]
                slope *= float(np.float32(SCALE))
                out["dh"][part] = torch.matmul(slope, e)
                out["de"][g] += torch.matmul(slope.t(), h)
    return out


def _round32(x):
    return x.to(torch.float32).to(torch.float64)


def _exact_adamw(st):
    """With states in 8 bits, m and v are fp32 numbers, rounded after each product and sum, before they are stored (their codes hang on it)."""
    case, d, hy = st["case"], torch.float64, st["hyper"]
    dev, eight = st["p"].device, case["bits"] == 8
    single = _round32 if eight else (lambda x: x)
    b1, b2 = float(np.float32(hy["beta1"])), float(np.float32(hy["beta2"]))
    lr, eps = float(np.float32(hy["lr"])), float(np.float32(hy["eps"]))
    table = torch.tensor([m / 512 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127], dtype=d, device=dev)
    names = ("p", "copy") if case["copy"] else ("p",)
    out = {n: torch.zeros(st["p"].shape, dtype=d, device=dev) for n in names + (("m", "v_root") if eight else ("m", "v"))}
    if eight:
        out.update(m_scales=torch.zeros_like(st["m_scales"]), v_scales=torch.zeros_like(st["v_scales"]))
    powers = torch.tensor([2.0 ** (k - 127) for k in range(256)], dtype=d, device=dev)

    def value(codes, scales):
        size = table[(codes & 0x7f).to(torch.int64)] * powers[scales.to(torch.int64)].repeat_interleave(BLOCK)[: codes.numel()]
        return torch.where(codes >= 128, -size, size)

    def scale_of(size, low):
        pad = torch.nn.functional.pad(size, (0, -size.numel() % BLOCK)).view(-1, BLOCK).amax(1)
        e = torch.ceil(torch.log2(torch.clamp(pad, min=2.0 ** -120) / 448.0)).to(torch.int64) + 127
        e = torch.where(448.0 * powers[e - 1] >= pad, e - 1, e)                         # the logarithm may be a hair off
        return torch.where(448.0 * powers[e] < pad, e + 1, e).clamp(min=low + 127)

    for w in range(case["workers"]):
        for i, (n, at, decay) in enumerate(zip(st["sizes"], st["first"], st["decay"])):
            s, b = slice(at, at + n), slice(at // BLOCK, at // BLOCK + -(-n // BLOCK))
            p, g = st["p"][w, s].to(d), st["g"][w, s].to(d) * float(np.float32(hy["grad_scale"]))
            m, v = st["m"][w, s], st["v"][w, s]
            m, v = (value(m, st["m_scales"][w, b]), value(v, st["v_scales"][w, b]) ** 2) if eight else (m.to(d), v.to(d))
            c1, c2 = float(np.float32(1.0 - b1)), float(np.float32(1.0 - b2))
            m = single(single(m * b1) + single(g * c1))
            v = single(single(v * b2) + single(single(g * c2) * g))
            p = p * (1.0 - lr * decay) - lr * (m / (1.0 - b1 ** hy["step"])) / (torch.sqrt(v / (1.0 - b2 ** hy["step"])) + eps)
            for name in names:
                out[name][w, s] = p
            if not eight:
                out["m"][w, s], out["v"][w, s] = m, v
                continue
            # (powers of two come from a table: a power function on the GPU may be a hair off, and a block's largest value may be a border)
            x = np.arange(n, dtype=np.uint32) * np.uint32(0x9E3779B1) + np.uint32((hy["seed"] + i * 0x632BE5AB + w * 0x85157AF5) % 2 ** 32)
            x = (x ^ (x >> np.uint32(16))) * np.uint32(0x7FEB352D)
            x = (x ^ (x >> np.uint32(15))) * np.uint32(0x846CA68B)
            x = torch.from_numpy((x ^ (x >> np.uint32(16))).astype(np.int64)).to(dev)
            for name, size, low, part in (("m", m.abs(), -117, x >> 16), ("v_root", single(torch.sqrt(v)), -51, x & 0xffff)):
                scales = scale_of(size, low)
                unit = powers[scales].repeat_interleave(BLOCK)[:n]
                q = size / unit
                below = torch.clamp(torch.searchsorted(table, q, right=True) - 1, max=125)
                lo, hi = table[below], table[below + 1]
                way, whole = (q - lo, hi - lo) if name == "m" else (v / unit ** 2 - lo ** 2, hi ** 2 - lo ** 2)
                code = table[below + (way * 65536 > part * whole).to(torch.int64)]
                if name == "m":
                    code = torch.where(torch.signbit(m), -code, code)
                else:
                    code = torch.where((code == 0) & (size > 0), table[1], code)
                out[name][w, s] = code
                out["m_scales" if name == "m" else "v_scales"][w, b] = scales.to(torch.uint8)
    return out
