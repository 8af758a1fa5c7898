"""A plain implementation of the token scores in 64 bits, and error bounds, for their tests.

A logit z = scale <h, e> is a sum of `dim` products in fp32, off by at most d = scale (dim + 8) 2^-23 sum |h e| + 2^-23 max |z| (see operator_harness).  `rest`, a sum of positive terms, each
with the error d, that of an exponential (|x| + 2 steps at a distance x) and of the additions (fewer than 300 + vocab / 64 on a path), is off by the factor
r = d + (300 + vocab / 64) 2^-23 + 2^-23 D of itself, with D = sum p |distance|; log(1 + rest) by at most r log(1 + rest), as rest / (1 + rest) <= log(1 + rest).
D is off by d-changes of p (sum p |x - D| d <= 2 D d), by d itself and by roundings, (300 + vocab / 64) 2^-23 D + 2^-22 sum p x^2.  H changes by at most 2 H d, and both roundings.
A probability is off by the factor q = r + 2 d + 80 steps + 2^-23 max |x| (x where it still counts: 104), so a slope a ([t] - p) - b p (x - D) by |a| p q + |b| p (|x - D| q + d + far D); then it is
rounded by half a step of the type (fp16: not below half of 2^-38 of the group's largest |a| + 32 |b|, times 2, as a power of two is taken), after a division by a number in 1/2 .. 1 by which
the result is multiplied again (two steps of 2^-23; twice the fp16 floor), for de by way of h, which is rounded to the type as well.  The products add what products add.
"""
import torch

import paper_1906_12043_amd as P
from tests.operator_harness import STEP, TYPES, groups_of, half_step


def exact_scores(bounds, h, e, target, scale=1.0, d_logp=None, d_entropy=None):
    """Scores, gradients and their bounds; rows that take no part as the call leaves them.  `order`: by row, entries from the largest logit on, lowest index first."""
    f, dev, rows, groups = torch.float64, h.device, h.shape[0], len(bounds) - 1
    t, vocab, dim = h.dtype, e.shape[1], h.shape[1]
    u = half_step(t)
    scale = float(torch.tensor(scale, dtype=torch.float32))
    zeros = lambda *s: torch.zeros(s, dtype=f, device=dev)     # noqa: E731
    out = {"logp": zeros(rows), "entropy": zeros(rows), "dh": zeros(*h.shape), "de": zeros(*e.shape), "all": zeros(rows, vocab), "z": zeros(rows, vocab)}
    far = {k: torch.zeros_like(out[k]) for k in ("logp", "entropy", "dh", "de")}
    part = torch.zeros(rows, dtype=torch.bool, device=dev)
    for g, s in groups_of(bounds):
        ids = torch.arange(rows, device=dev)[s]
        if target is not None:
            ids = ids[(target[ids] >= 0) & (target[ids] < vocab)]
        if not len(ids):
            continue
        part[ids] = True
        hh, ee = h[ids].to(f), e[g].to(f)
        z = scale * (hh @ ee.t())
        d = scale * (dim + 8) * STEP * (hh.abs() @ ee.abs().t()).amax(1) + STEP * z.abs().amax(1)
        logp = torch.log_softmax(z, 1)
        p = torch.exp(logp)
        x = z - z.amax(1, keepdim=True)
        mean = (p * x).sum(1)
        H = -(p * torch.where(p > 0, logp, 0.0)).sum(1)
        norm = H + mean                                        # log(1 + rest)
        adds = (300 + vocab / 64) * STEP
        r = d + adds - STEP * mean
        far_mean = d - 2 * mean * d - adds * mean + 2 * STEP * (p * x.clamp(min=-104) ** 2).sum(1)
        out["all"][ids], out["z"][ids] = logp, z
        out["entropy"][ids] = H
        far["entropy"][ids] = (2 * H * d + r * norm + (adds - STEP * mean) * norm + adds * -mean + 2 * STEP * (p * x.clamp(min=-104) ** 2).sum(1)) * 1.05 + STEP * H
        pick = torch.arange(len(ids), device=dev)
        at = target[ids].long() if target is not None else None
        if at is not None:
            out["logp"][ids] = logp[pick, at]
            far["logp"][ids] = (r * norm + 2 * d + 2 * STEP * logp[pick, at].abs()) * 1.05
        out.setdefault("far_all", zeros(rows))[ids] = (r * norm + 2 * d) * 1.05
        a = d_logp[ids].to(f)[:, None] if d_logp is not None and target is not None else zeros(len(ids), 1)
        b = d_entropy[ids].to(f)[:, None] if d_entropy is not None else zeros(len(ids), 1)
        off_mean = x - mean[:, None]
        dz = -p * (a + b * off_mean)
        if at is not None:
            dz[pick, at] += a[:, 0]
        q = (r + 2 * d + 184 * STEP)[:, None]
        off = p * (a.abs() * q + b.abs() * (off_mean.abs() * q + (d + far_mean)[:, None])) * 1.05 + (a.abs() + b.abs()) * 1e-37
        dz, off = dz * scale, off * scale
        off = off + (u if t != torch.float32 else 4 * STEP) * (dz.abs() + off)
        if t == torch.float16:
            off = off + 2.0 ** -38 * scale * (a.abs() + 32 * b.abs()).max()
        if t != torch.float32:
            off = off + 2 * STEP * (dz.abs() + off)
        tiny = torch.finfo(t).smallest_normal * torch.finfo(t).eps
        for key, where, left, right, terms in (("dh", ids, (off, dz), ee, vocab), ("de", g, (off.t(), dz.t()), hh, len(ids))):
            out[key][where] = left[1] @ right
            if key == "de" and t != torch.float32:
                left = (left[0] + u * (left[0] + left[1].abs()), left[1])
            total = left[0] @ right.abs() + (terms + 8) * STEP * ((left[1].abs() + left[0]) @ right.abs())
            far[key][where] = total * (1 + u) + (u + 4 * STEP) * out[key][where].abs() + tiny
    out["part"] = part
    return out, far


def scores_call(dtype, bounds, h, e, target, grad=False, top=0, scale=1.0, **more):
    """(call, outputs): everything that there is, outputs full of NaN (ids: -9)."""
    offsets = torch.tensor(bounds, dtype=torch.int64, device="cuda")
    rows, vocab = h.shape[0], e.shape[1]
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")                       # noqa: E731
    out = {"entropy": nan(rows), "norms": nan(rows, 4)}
    if target is not None:
        out["logp"] = nan(rows)
    f = dict(dtype=TYPES[dtype][0], groups=len(bounds) - 1, rows=rows, dim=h.shape[1], vocab=vocab, offsets=offsets, h=h, ldh=max(h.stride(0), h.shape[1]), e=e,
             lde=max(e.stride(1), e.shape[2]), e_stride=e.stride(0), targets=target, scale=scale)
    if top:
        ids, lps = torch.full((max(1, rows), top + 3), -9, dtype=torch.int32, device="cuda"), nan(max(1, rows), top + 3)
        f.update(top=top, top_ids=ids, top_logp=lps, ld_top=top + 3)
        out.update(top_ids=ids[:rows, :top], top_logp=lps[:rows, :top], ids_buffer=ids, logp_buffer=lps)
    f.update({k: out[k] for k in ("logp", "entropy", "norms") if k in out})
    f.update(more)
    for name, ld in (("dh", "lddh"), ("de", "ldde")):
        if f.get(name) is not None:
            f[ld] = max(f[name].stride(-2), f[name].shape[-1])
    if f.get("de") is not None:
        f["de_stride"] = f["de"].stride(0)
    c = P.TokenScores(**f)
    need = max(P.token_scores_workspace(c, P.TOKEN_SCORES_FORWARD), P.token_scores_workspace(c, P.TOKEN_SCORES_GRAD) if grad else 0)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")           # NaN in every word
    c.set(workspace=ws, workspace_bytes=ws.numel())
    c.keep = (offsets, f, ws, out)
    return c, out
