"""Inputs, plain 64-bit implementations and error bounds for the tests of the grouped products, the loss and the checkpoints.

Bounds.  u = eps / 2 of a type is half a step relative to a value.  A sum of K products kept in fp32 takes at most K
additions (the matrix instruction adds sixteen at a time, in an order and with a rounding of its own: a whole step of 2^-23 each), so it is off by at
most (K + 8) 2^-23 sum |a b|; fp32 operands enter as three bf16 parts whose left-out products are below 2^-24 of sum |a b|, which the 8 covers.  The result is then rounded once: u |c|.
"""
import numpy as np
import torch

import paper_1906_12043_amd as P

TYPES = {"bf16": (P.BF16, torch.bfloat16), "fp16": (P.F16, torch.float16), "fp32": (P.F32, torch.float32)}
STEP = 2.0 ** -23
SENTINEL = 777.0


def half_step(t):
    return torch.finfo(t).eps / 2


def matrix(rows, cols, pad, t, gen, std=1.0, dev="cuda"):
    """A [rows, cols] view with a pitch of cols + pad inside a buffer full of NaN."""
    buf = torch.full((max(rows, 1), cols + pad), float("nan"), dtype=t, device=dev)
    buf[:rows, :cols] = (torch.randn(rows, cols, generator=gen, device=dev) * std).to(t)
    return buf[:rows, :cols]


def stack(groups, rows, cols, pad, gap, t, gen, std=1.0, dev="cuda"):
    """[groups, rows, cols] with pitch cols + pad and gap elements between the groups, NaN around."""
    stride = rows * (cols + pad) + gap
    buf = torch.full((groups * stride,), float("nan"), dtype=t, device=dev)
    view = buf.as_strided((groups, rows, cols), (stride, cols + pad, 1))
    view.copy_((torch.randn(groups, rows, cols, generator=gen, device=dev) * std).to(t))
    return view


def output(shape, pad, t, gap=0, dev="cuda"):
    """(buffer full of a sentinel, view of it) for an output of [rows, cols] or [groups, rows, cols]."""
    cols = shape[-1] + pad
    if len(shape) == 2:
        buf = torch.full((max(shape[0], 1), cols), SENTINEL, dtype=t, device=dev)
        return buf, buf[:shape[0], :shape[1]]
    stride = shape[1] * cols + gap
    buf = torch.full((shape[0] * stride,), SENTINEL, dtype=t, device=dev)
    return buf, buf.as_strided(shape, (stride, cols, 1))


def untouched(buf, view, written=None):
    """Everything of the buffer but the view (or the rows `written` of it) still holds the sentinel."""
    mark = torch.zeros_like(buf, dtype=torch.bool)
    mine = mark.as_strided(view.shape, view.stride(), view.storage_offset())
    if written is None:
        mine.fill_(True)
    else:
        mine[written] = True
    return bool((buf[~mark] == SENTINEL).all())


def groups_of(bounds):
    return [(g, slice(a, max(a, b))) for g, (a, b) in enumerate(zip(bounds, bounds[1:]))]


def inside(bounds, rows):
    mask = torch.zeros(rows, dtype=torch.bool, device="cuda")
    mask[bounds[0]:bounds[-1]] = True
    return mask


def exact_product(kind, bounds, a, b):
    """(result, sum of magnitudes, number of terms per group) in 64 bits; rows outside the groups are zero."""
    f = torch.float64
    if kind == "weight_grad":
        out = torch.stack([a[s].to(f).t() @ b[s].to(f) for _, s in groups_of(bounds)])
        mag = torch.stack([a[s].to(f).abs().t() @ b[s].to(f).abs() for _, s in groups_of(bounds)])
        return out, mag, max(s.stop - s.start for _, s in groups_of(bounds))
    cols = b.shape[2] if kind == "forward" else b.shape[1]
    out = torch.zeros((a.shape[0], cols), dtype=f, device=a.device)
    mag = torch.zeros_like(out)
    for g, s in groups_of(bounds):
        w = b[g].to(f) if kind == "forward" else b[g].to(f).t()
        out[s], mag[s] = a[s].to(f) @ w, a[s].to(f).abs() @ w.abs()
    return out, mag, a.shape[1]


def product_bound(out, mag, terms, t):
    return half_step(t) * out.abs() + (terms + 8) * STEP * mag * (1 + half_step(t)) + torch.finfo(t).smallest_normal * torch.finfo(t).eps


def layer(dtype, bounds, rows, inner, outer, **tensors):
    """P.Grouped from tensors (pitches and strides are read off them); keeps the offsets alive."""
    f = dict(dtype=TYPES[dtype][0], groups=len(bounds) - 1, rows=rows, inner=inner, outer=outer)
    pitch = {"x": "ldx", "x_codes": "ld_codes", "x_scales": "ld_scales", "w": "ldw", "y": "ldy", "dy": "lddy", "dx": "lddx", "dw": "lddw"}
    for name, t in tensors.items():
        if isinstance(t, torch.Tensor) and name in pitch:
            f[pitch[name]] = t.stride(-2) if t.shape[-2] > 1 else max(t.stride(-2), t.shape[-1])
            if name in ("w", "dw"):
                f[name + "_stride"] = t.stride(0)
        f[name] = t
    if "dw" in tensors:
        f.setdefault("dw_dtype", P.F32 if tensors["dw"].dtype == torch.float32 else TYPES[dtype][0])
    offsets = torch.tensor(bounds, dtype=torch.int64, device="cuda")
    out = P.Grouped(offsets=offsets, **f)
    out.keep = (offsets, tensors)
    return out


CALLS = {"forward": (P.grouped_forward, P.GROUPED_FORWARD), "input_grad": (P.grouped_input_grad, P.GROUPED_INPUT_GRAD),
         "weight_grad": (P.grouped_weight_grad, P.GROUPED_WEIGHT_GRAD)}


def call(kind, lay, workspace=False, stream=None):
    fn, direction = CALLS[kind]
    if workspace:
        need = P.grouped_workspace(lay, direction)
        ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")        # NaN in every word
        lay.set(workspace=ws, workspace_bytes=ws.numel())
        lay.ws = ws
    fn(stream if stream is not None else torch.cuda.current_stream(), lay)


# ---- checkpoints -------------------------------------------------------------------------------------

def e4m3_values():
    """Magnitude of the codes 0 .. 126, from the format's definition."""
    return np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def encode(x, dtype):
    """(codes, scales) of a [rows, cols] array of float64 values, value by value from the definition, on the CPU."""
    table = e4m3_values()
    low, most = (-15, 1.875 * 2.0 ** 15) if dtype == "fp16" else (-117, 1.875 * 2.0 ** 127)
    rows, cols = x.shape
    codes = np.zeros((rows, cols), np.uint8)
    scales = np.zeros((rows, -(-cols // 32)), np.uint8)
    for r in range(rows):
        for b in range(scales.shape[1]):
            v = x[r, 32 * b:32 * b + 32]
            fine = np.isfinite(v)
            top = np.max(np.abs(v[fine]), initial=0.0)
            e = low
            while 448.0 * 2.0 ** e < top:
                e += 1
            scales[r, b] = e + 127
            for i, val in enumerate(v):
                sign = 0x80 if np.signbit(val) else 0
                if not np.isfinite(val):
                    codes[r, 32 * b + i] = 0x7f | sign
                    continue
                q = min(abs(val), most) / 2.0 ** e
                at = int(np.searchsorted(table, q))                 # table[at - 1] < q <= table[at]
                if at == 0:
                    code = 0
                elif at > 126:
                    code = 126
                else:
                    below, above = q - table[at - 1], table[at] - q
                    code = at - 1 if below < above or (below == above and (at - 1) % 2 == 0) else at
                if code == 0 and val != 0:
                    code = 1
                codes[r, 32 * b + i] = code | sign
    return codes, scales


def decode(codes, scales):
    table = np.concatenate([e4m3_values(), [np.nan]])
    mag = table[codes & 0x7f] * np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, axis=1)[:, :codes.shape[1]]
    return np.where(codes & 0x80, -mag, mag)


# ---- loss ----------------------------------------------------------------------------------------------

def exact_loss(bounds, h, e, target, total=False, grad_scale=1.0):
    """Loss, group loss, gradients in 64 bits, and what the bounds need, group by group."""
    f = torch.float64
    rows, groups = h.shape[0], len(bounds) - 1
    out = {"loss": torch.zeros(rows, dtype=f, device=h.device), "group_loss": torch.zeros(groups, dtype=f, device=h.device),
           "dh": torch.zeros(h.shape, dtype=f, device=h.device), "de": torch.zeros(e.shape, dtype=f, device=h.device), "parts": []}
    for g, s in groups_of(bounds):
        ids = torch.arange(rows, device=h.device)[s]
        ids = ids[(target[ids] >= 0) & (target[ids] < e.shape[1])]
        if not len(ids):
            continue
        hh, ee, tt = h[ids].to(f), e[g].to(f), target[ids].long()
        z = hh @ ee.t()
        norm = torch.logsumexp(z, 1)
        pick = torch.arange(len(ids), device=h.device)
        prob = torch.exp(z - norm[:, None])
        dz = prob.clone()
        dz[pick, tt] -= 1
        scale = grad_scale * (1.0 if total else 1.0 / len(ids))
        out["loss"][ids] = norm - z[pick, tt]
        out["group_loss"][g] = out["loss"][ids].sum() if total else out["loss"][ids].mean()
        out["dh"][ids] = scale * (dz @ ee)
        out["de"][g] = scale * (dz.t() @ hh)
        out["parts"].append((g, ids, hh, ee, z, norm, prob, dz, scale))
    return out


def loss_bounds(out, t, dim, vocab):
    """Error bounds of loss, dh, de.

    A logit is off by d = (dim + 8) 2^-23 sum |h e|.  A row's sum of exponentials is a sum of positive terms: each is off by d, by the exponential's own
    error (|x| + 2 steps of 2^-23 at an argument x below the maximum, whose mean over the terms is below 32), and by the additions (a lane
    adds up to 128 values, then lanes, waves and tiles: fewer than 256 + vocab / 64).  So norm is off by at most
    r = d + (300 + vocab / 64) 2^-23 + |norm| 2^-23, the loss by r + d, and a probability by the factor r + d + 40 steps.
    Between two passes an exponential relative to its tile's maximum may be held in 11 bits (bf16, 2^-11 of it and not below steps of 2^-38) or 24,
    and is multiplied by a second exponential, with errors like the first's: 80 steps and 2^-11 of the probability.
    A slope is rounded by half a step of the type (fp16: times 2^14, not below steps of 2^-38).  The two products add what products add.
    """
    u = half_step(t)
    bound = {k: torch.zeros_like(out[k]) for k in ("loss", "dh", "de")}
    for g, ids, hh, ee, z, norm, prob, dz, scale in out["parts"]:
        d = (dim + 8) * STEP * (hh.abs() @ ee.abs().t()).amax(1)
        r = d + (300 + vocab / 64) * STEP + norm.abs() * STEP
        bound["loss"][ids] = r + d + STEP * (out["loss"][ids] + norm.abs())
        off = prob * (r + d + 80 * STEP + (2.0 ** -11 if t == torch.bfloat16 else 0.0))[:, None] * 1.01 + STEP
        off = off * (prob > 0) + (u if t != torch.float32 else STEP) * dz.abs() + (2.0 ** -39 if t != torch.float32 else 0.0)
        for key, at, left, right, terms in (("dh", ids, (off, dz), ee, vocab), ("de", g, (off.t(), dz.t()), hh, len(ids))):
            far = left[0] @ right.abs() + (terms + 8) * STEP * ((left[1].abs() + left[0]) @ right.abs())
            bound[key][at] = abs(scale) * far * (1 + u) + (u + 4 * STEP) * out[key][at].abs() + torch.finfo(t).smallest_normal * torch.finfo(t).eps
    return bound


def cross_entropy_call(dtype, bounds, h, e, target, dh=None, de=None, group_loss=None, loss=None, **more):
    offsets = torch.tensor(bounds, dtype=torch.int64, device="cuda")
    f = dict(dtype=TYPES[dtype][0], groups=len(bounds) - 1, rows=h.shape[0], dim=h.shape[1], vocab=e.shape[1], offsets=offsets,
             h=h, ldh=max(h.stride(0), h.shape[1]), e=e, lde=max(e.stride(1), e.shape[2]), e_stride=e.stride(0), targets=target, loss=loss,
             group_loss=group_loss)
    if dh is not None:
        f.update(dh=dh, lddh=max(dh.stride(0), dh.shape[1]))
    if de is not None:
        f.update(de=de, ldde=max(de.stride(1), de.shape[2]), de_stride=de.stride(0))
    c = P.CrossEntropy(**{**f, **more})
    need = P.cross_entropy_workspace(c)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")             # NaN in every word
    c.set(workspace=ws, workspace_bytes=ws.numel())
    c.keep = (offsets, h, e, target, loss, group_loss, dh, de, ws)
    return c
