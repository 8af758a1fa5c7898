"""The AdamW step on the GPU: fp32 states against the formula in 64 bits, 8-bit states code by code.

Bounds of fp32 states, e = 2^-24 (one rounding), constants as the call holds them in fp32.  g' = s g: e.  m' = b1 m + (1 - b1) g': products e each, sum e: at most
e (|b1 m| + 2 |(1 - b1) g'| + |m'|).  v' likewise: (d c2) d has three roundings beside the two of d: e (|b2 v| + 5 |c2 g'^2| + |v'|).  The change of p is
lr / c1 * m' / (sqrt(v') / sqrt(c2) + eps): relative to itself the errors of m' and half of those of v', and roundings of the root (1), of 1 / sqrt(c2) (c2 itself 1/2, root 1,
quotient 1), product, sum, reciprocal (an instruction that is off by a whole step: 2), product, lr (1), lr / c1 (c1 1, quotient 1), product: below 14.  1 - lr wd: 2 |lr wd| + 1.
Then two products and a difference.  16-bit parameters are rounded once more, and a copy as they are.
"""
import math

import numpy as np
import pytest
import torch

import paper_1906_12043_amd as P
from tests.operator_harness import SENTINEL, TYPES, e4m3_values, half_step

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.98, eps=1e-6, step=3, grad_scale=0.75)
f32 = lambda v: float(np.float32(v))                          # noqa: E731


class Flat:
    """[workers][stride] arrays of a list of tensors, `shift` elements off 16 bytes, sentinels between the tensors."""

    def __init__(self, sizes, workers, dtype, gen, shift=0, std=1.0, fill=SENTINEL, gap=3, block=1):
        self.first, at = [], 0
        for n in sizes:
            self.first.append(at)
            at = -(-(at + n + gap) // block) * block
        self.stride = -(-max(1, at) // 32) * 32
        self.buf = torch.full((workers * self.stride + shift,), fill, dtype=dtype, device="cuda")
        self.all = self.buf[shift:].view(workers, self.stride)
        self.sizes = sizes
        if gen is not None:
            for i in range(len(sizes)):
                for w in range(workers):
                    self.part(i, w).copy_(torch.randn(sizes[i], generator=gen, device="cuda") * std)

    def part(self, i, w=0):
        return self.all[w, self.first[i]:self.first[i] + self.sizes[i]]

    def rest_untouched(self, value=SENTINEL):
        mark = torch.ones_like(self.all, dtype=torch.bool)
        for n, at in zip(self.sizes, self.first):
            mark[:, at:at + n] = False
        return bool((self.all[mark] == value).all())


def formula(p, g, m, v, decay, lr_scale, hyper):
    """(p, m, v) in 64 bits and their error bounds before p's rounding."""
    d = torch.float64
    p, g, m, v = (t.to(d) for t in (p, g, m, v))
    b1, b2, lr, eps, s = (f32(hyper[k]) for k in ("beta1", "beta2", "lr", "eps", "grad_scale"))
    c1, c2 = f32(1 - b1), f32(1 - b2)
    lr, decay = lr * f32(lr_scale), f32(decay)
    g = g * s
    m_new, v_new = b1 * m + c1 * g, b2 * v + c2 * g * g
    far_m = E * ((b1 * m).abs() + 2 * (c1 * g).abs() + m_new.abs()) * 1.01 + 2.0 ** -148
    far_v = E * ((b2 * v).abs() + 5 * c2 * g * g + v_new.abs()) * 1.01 + 2.0 ** -148
    bias1, bias2 = 1 - b1 ** hyper["step"], 1 - b2 ** hyper["step"]
    root = torch.sqrt(v_new / bias2)
    change = lr / bias1 * m_new / (root + eps)
    # (an error of v' near zero moves the root by at most its own root)
    far_root = torch.minimum(far_v / bias2 / (2 * root).clamp(min=1e-300), torch.sqrt(far_v / bias2)) / (root + eps)
    far = lr / bias1 * far_m / (root + eps) + change.abs() * (far_root + 14 * E)
    p_new = p * (1 - lr * decay) - change
    far = far * 1.02 + p.abs() * E * (2 * abs(lr * decay) + 2) + (change.abs() + p_new.abs()) * E + 2.0 ** -148
    return (p_new, m_new, v_new), (far, far_m, far_v)


KINDS = [("fp32", "fp32", None), ("fp32", "bf16", "bf16"), ("fp32", "fp16", "fp16"), ("fp32", "bf16", "fp16"), ("fp32", "fp16", None), ("bf16", "bf16", None), ("bf16", "fp32", None),
         ("fp16", "fp16", None), ("fp16", "fp32", None), ("bf16", "fp16", None), ("fp16", "bf16", None)]
LISTS = [[1], [7, 1, 0, 33], [2048, 2049, 31, 4100, 5], [3] * 45 + [5000] + [17] * 40, [200_003]]


def state_call(kind, sizes, workers, seed, shift, **more):
    p_type, g_type, copy_type = kind
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = {k: v[1] for k, v in TYPES.items()}
    p, g = Flat(sizes, workers, t[p_type], gen, shift), Flat(sizes, workers, t[g_type], gen, shift)
    m, v = Flat(sizes, workers, torch.float32, gen, shift, 0.1), Flat(sizes, workers, torch.float32, gen, shift)
    for i in range(len(sizes)):
        for w in range(workers):
            v.part(i, w).abs_()
            v.part(i, w)[::7] = 0
            m.part(i, w)[::7] = 0
            g.part(i, w)[::14] = 0
    copy = Flat(sizes, workers, t[copy_type], None, shift) if copy_type else None
    tensors = []
    for i, n in enumerate(sizes):
        one = dict(n=n, p=p.part(i), g=g.part(i), m=m.part(i), v=v.part(i), weight_decay=0.1 * (i % 3), lr_scale=1.0 if i % 2 == 0 else 0.5)
        if copy:
            one["copy"] = copy.part(i)
        tensors.append(one)
    call = P.AdamW(tensors=tensors, dtype=TYPES[p_type][0], grad_dtype=TYPES[g_type][0], copy_dtype=TYPES[copy_type][0] if copy_type else 0, workers=workers, stride=p.stride,
                   **{**HYPER, **more})
    return call, tensors, p, g, m, v, copy


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(str(x) for x in k))
@pytest.mark.parametrize("which", range(len(LISTS)))
@pytest.mark.parametrize("workers, shift", [(1, 0), (3, 1)])
def test_fp32_states(kind, which, workers, shift):
    sizes = LISTS[which]
    call, tensors, p, g, m, v, copy = state_call(kind, sizes, workers, which * 7 + workers, shift)
    before = [x.buf.clone() for x in (p, g, m, v)]
    old = [Flat(sizes, workers, x.all.dtype, None, shift) for x in (p, g, m, v)]
    for o, b in zip(old, before):
        o.buf.copy_(b)
    P.adamw(torch.cuda.current_stream(), call)
    torch.cuda.synchronize()
    assert torch.equal(g.buf, before[1])
    u = half_step(p.all.dtype) if p.all.dtype != torch.float32 else 0.0
    for i, one in enumerate(tensors):
        for w in range(workers):
            want, far = formula(*(o.part(i, w) for o in old), one["weight_decay"], one["lr_scale"], HYPER)
            tiny = torch.finfo(p.all.dtype).smallest_normal * torch.finfo(p.all.dtype).eps
            for got, x, f, r in ((p, want[0], far[0], u), (m, want[1], far[1], 0.0), (v, want[2], far[2], 0.0)):
                assert bool(((got.part(i, w).double() - x).abs() <= f * (1 + r) + r * x.abs() + (tiny if r else 0)).all()), (i, w)
            if copy:
                assert torch.equal(copy.part(i, w), p.part(i, w).to(copy.all.dtype))
    for x in (p, m, v) + ((copy,) if copy else ()):
        assert x.rest_untouched() and bool((x.buf[:shift] == SENTINEL).all())


def test_many_pairs_of_decay_and_rate_and_copies_of_some():
    """More pairs than a launch holds, tensors of no elements and tensors without a copy between the others."""
    sizes = [40 + 7 * (i % 9) if i % 11 else 0 for i in range(90)]
    _, tensors, p, g, m, v, copy = state_call(("fp32", "bf16", "bf16"), sizes, 2, 9, 0)
    old = [Flat(sizes, 2, x.all.dtype, None) for x in (p, g, m, v)]
    for o, x in zip(old, (p, g, m, v)):
        o.buf.copy_(x.buf)
    for i, one in enumerate(tensors):
        one["weight_decay"], one["lr_scale"] = 0.01 * (i % 37), 1.0 + 0.25 * (i % 5)
        if i % 4 == 1:
            one["copy"] = None
    P.adamw(torch.cuda.current_stream(), P.AdamW(tensors=tensors, dtype=P.F32, grad_dtype=P.BF16, copy_dtype=P.BF16, workers=2, stride=p.stride, **HYPER))
    for i, one in enumerate(tensors):
        for w in range(2):
            want, far = formula(*(o.part(i, w) for o in old), one["weight_decay"], one["lr_scale"], HYPER)
            for got, x, f in zip((p, m, v), want, far):
                assert bool(((got.part(i, w).double() - x).abs() <= f).all()), (i, w)
            assert torch.equal(copy.part(i, w), p.part(i, w).to(torch.bfloat16) if i % 4 != 1 else torch.full_like(copy.part(i, w), SENTINEL))


def test_gradients_that_are_not_finite_stay_with_their_element():
    call, tensors, p, g, m, v, _ = state_call(("fp32", "fp32", None), [4096], 1, 5, 0)
    g.part(0)[100], g.part(0)[200], g.part(0)[300] = float("nan"), float("inf"), float("-inf")
    P.adamw(torch.cuda.current_stream(), call)
    for x in (p, m, v):
        bad = ~torch.isfinite(x.part(0))
        assert set(torch.nonzero(bad)[:, 0].tolist()) <= {100, 200, 300}
    assert bool(torch.isnan(p.part(0)[[100, 200, 300]]).all()) and float(m.part(0)[200]) == math.inf and float(v.part(0)[300]) == math.inf


def test_zero_states_and_gradients_leave_parameters_that_do_not_decay():
    call, tensors, p, g, m, v, _ = state_call(("fp32", "fp32", None), [1000], 1, 5, 0)
    for x in (g, m, v):
        x.part(0).zero_()
    before = p.part(0).clone()
    P.adamw(torch.cuda.current_stream(), call)
    assert torch.equal(p.part(0), before) and not bool(m.part(0).any()) and not bool(v.part(0).any())


# ---- 8-bit states ------------------------------------------------------------------------------------

TABLE = e4m3_values()                                          # of the codes 0 .. 126


def random_words(n, seed, tensor, worker):
    at = np.arange(n, dtype=np.uint64)
    x = (at * np.uint64(0x9E3779B1) + np.uint64((seed + tensor * 0x632BE5AB + worker * 0x85157AF5) % 2 ** 32)) & np.uint64(0xffffffff)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x7FEB352D)) & np.uint64(0xffffffff)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x846CA68B)) & np.uint64(0xffffffff)
    return (x ^ (x >> np.uint64(16))).astype(np.int64)


def decoded(codes, scales):
    size = np.concatenate([TABLE, [np.nan]])[codes & 0x7f] * np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32)[:codes.size]
    return np.where(codes & 0x80, -size, size)


def stored(value, size, low, bits, square):
    """(codes, scales) of one tensor from the definition; value: m, or v whose root is `size`; 64 bits, exact."""
    n, blocks = size.size, -(-size.size // 32)
    fine = np.isfinite(size)
    pad = np.zeros(blocks * 32)
    pad[:n] = np.where(fine, size, 0.0)
    top = pad.reshape(blocks, 32).max(1)
    e = np.full(blocks, low)
    for k in range(low + 1, 140):
        e = np.where(448.0 * np.exp2(np.float64(k - 1)) < top, k, e)
    unit = np.repeat(np.exp2(e.astype(np.float64)), 32)[:n]
    q = np.where(fine, size, 0.0) / unit
    below = np.minimum(np.searchsorted(TABLE, q, side="right") - 1, 125)
    lo, hi = TABLE[below], TABLE[below + 1]
    if square:
        way, whole = np.where(fine, value, 0.0) / unit / unit - lo * lo, hi * hi - lo * lo
    else:
        way, whole = q - lo, hi - lo
    code = below + (way * 65536 > bits * whole)
    if square:
        code = np.where((code == 0) & (size > 0), 1, code)
        sign = np.zeros(n, np.int64)
    else:
        sign = np.where(np.signbit(value), 0x80, 0)
    return (np.where(fine, code, 0x7f) | sign).astype(np.uint8), (e + 127).astype(np.uint8)


def single(x):
    with np.errstate(over="ignore", invalid="ignore"):
        return x.astype(np.float32).astype(np.float64)


class Eight:
    """A list of tensors with 8-bit states; old states made of arbitrary codes."""

    def __init__(self, sizes, workers, seed, p_type="fp32", g_type="fp32", g_std=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t = {k: v[1] for k, v in TYPES.items()}
        self.sizes, self.workers = sizes, workers
        flat = dict(block=32, gap=0)
        self.p, self.g = Flat(sizes, workers, t[p_type], gen, **flat), Flat(sizes, workers, t[g_type], gen, std=g_std, **flat)
        self.stride = self.p.stride
        code = lambda top: torch.randint(0, top, (workers, self.stride), generator=gen, device="cuda").to(torch.uint8)          # noqa: E731
        self.m, self.v = code(127) | (code(2) << 7), code(127)
        exponent = lambda: torch.randint(110, 120, (workers, self.stride // 32), generator=gen, device="cuda").to(torch.uint8)   # noqa: E731
        self.m_scales, self.v_scales = exponent(), exponent()
        self.types = (p_type, g_type)

    def tensors(self):
        out = []
        for i, n in enumerate(self.sizes):
            at = self.p.first[i]
            out.append(dict(n=n, p=self.p.part(i), g=self.g.part(i), m=self.m[0, at:], v=self.v[0, at:], m_scales=self.m_scales[0, at // 32:], v_scales=self.v_scales[0, at // 32:],
                            weight_decay=0.1 * (i % 2)))
        return out

    def call(self, **more):
        return P.AdamW(tensors=self.tensors(), dtype=TYPES[self.types[0]][0], grad_dtype=TYPES[self.types[1]][0], state=P.ADAMW_STATE_8BIT, workers=self.workers, stride=self.stride,
                       **{**HYPER, "seed": 99, **more})

    def host(self):
        return [x.cpu().numpy() for x in (self.m, self.v, self.m_scales, self.v_scales)]

    def check(self, before, gradients, parameters, hyper, seed):
        """What a step made of the old states, code by code; parameters within their bound."""
        after = self.host()
        b1, b2, s = f32(hyper["beta1"]), f32(hyper["beta2"]), f32(hyper["grad_scale"])
        for w in range(self.workers):
            for i, n in enumerate(self.sizes):
                if n == 0:
                    continue
                at, sl, bl = self.p.first[i], slice(self.p.first[i], self.p.first[i] + n), slice(self.p.first[i] // 32, self.p.first[i] // 32 + -(-n // 32))
                m, root = decoded(before[0][w, sl], before[2][w, bl]), decoded(before[1][w, sl], before[3][w, bl])
                v = single(root * root)
                with np.errstate(over="ignore", invalid="ignore"):
                    g = single(gradients[w, sl].astype(np.float64) * s)
                    m_new = single(single(m * b1) + single(g * f32(1 - b1)))
                    v_new = single(single(v * b2) + single(single(g * f32(1 - b2)) * g))
                    bits = random_words(n, seed, i, w)
                    for k, (value, size, low, part, square) in enumerate(((m_new, np.abs(m_new), -117, bits >> 16, False), (v_new, single(np.sqrt(v_new)), -51, bits & 0xffff, True))):
                        codes, scales = stored(value, size, low, part, square)
                        assert np.array_equal(after[k][w, sl], codes), (i, w, k)
                        assert np.array_equal(after[2 + k][w, bl], scales), (i, w, k)
                fine = np.isfinite(m_new) & np.isfinite(v_new)
                to = lambda x: torch.from_numpy(np.ascontiguousarray(x[fine])).cuda()              # noqa: E731
                want, far = formula(to(parameters[w, sl].astype(np.float64)), to(gradients[w, sl].astype(np.float64)), to(m), to(v), 0.1 * (i % 2), 1.0, hyper)
                got = self.p.part(i, w).double()[torch.from_numpy(fine).cuda()]
                u = half_step(self.p.all.dtype) if self.types[0] != "fp32" else 0.0
                assert bool(((got - want[0]).abs() <= far[0] * (1 + u) + u * want[0].abs() + torch.finfo(self.p.all.dtype).smallest_normal * u).all()), (i, w)


def numbers(x):
    return x.float().cpu().numpy()


@pytest.mark.parametrize("types", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp16"), ("fp16", "fp32")])
@pytest.mark.parametrize("sizes, workers", [([1], 1), ([31, 32, 33, 0, 64, 7], 2), ([2048, 2049, 4097], 3), ([5] * 43 + [900], 1), ([100_003], 1)])
def test_states_of_8_bits(types, sizes, workers):
    x = Eight(sizes, workers, sum(sizes) + workers, *types)
    before, g, p = x.host(), numbers(x.g.all), numbers(x.p.all)
    P.adamw(torch.cuda.current_stream(), x.call())
    torch.cuda.synchronize()
    x.check(before, g, p, HYPER, 99)
    # what lies between the tensors stays
    mark = np.ones((workers, x.stride), bool)
    for n, at in zip(sizes, x.p.first):
        mark[:, at:at + n] = False
    after = x.host()
    assert np.array_equal(after[0][mark], before[0][mark]) and np.array_equal(after[1][mark], before[1][mark]) and x.p.rest_untouched()


@pytest.mark.parametrize("magnitude", [0.0, 1e-42, 1e-30, 3e-23, 1e-20, 1e-18, 1e-12, 1.0, 1e12, 1e18, 3e38])
def test_states_of_8_bits_over_the_range(magnitude):
    x = Eight([4096], 1, 3)
    x.g.part(0).mul_(magnitude)
    if magnitude > 1e30:
        x.g.part(0).copy_(torch.sign(x.g.part(0)) * 3e38)      # squares are infinite, m is not
    x.g.part(0)[::5] *= 1e-6
    x.g.part(0)[1::97] = 0.0
    for c in (x.m, x.v, x.m_scales, x.v_scales):
        c.zero_()
    hyper = {**HYPER, "grad_scale": 1.0}
    for seed in (1, 2 ** 32 - 1):
        before, g, p = x.host(), numbers(x.g.all), numbers(x.p.all)
        P.adamw(torch.cuda.current_stream(), x.call(grad_scale=1.0, seed=seed))
        torch.cuda.synchronize()
        x.check(before, g, p, hyper, seed)
        if magnitude == 0.0:
            assert not x.m.any() and not x.v.any()


def test_8_bit_states_that_are_not_finite_are_nan_and_leave_their_block_alone():
    x = Eight([256], 1, 4)
    x.g.part(0)[[3, 40, 70]] = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda")
    before, g, p = x.host(), numbers(x.g.all), numbers(x.p.all)
    for seed in (5, 6):                                        # and stay NaN
        P.adamw(torch.cuda.current_stream(), x.call(seed=seed))
        torch.cuda.synchronize()
        m, v, _, _ = x.host()
        assert [int(i) for i in np.flatnonzero((m[0, :256] & 0x7f) == 0x7f)] == [3, 40, 70] == [int(i) for i in np.flatnonzero(v[0, :256] == 0x7f)]
        if seed == 5:
            x.check(before, g, p, HYPER, seed)


def test_rounding_is_right_in_the_mean():
    """The same m and v in all elements: what is stored has their mean.  A code's distance from the value is below the step, so the mean of n of them is off by at most
    half a step / sqrt(n) as a standard deviation; six of them are allowed."""
    n = 1 << 18
    x = Eight([n], 1, 6)
    for c in (x.m, x.v, x.m_scales, x.v_scales):
        c.zero_()
    x.g.part(0).fill_(0.7)
    x.g.part(0)[::32] = 1.9                                    # the largest of its block, so that 0.7 lies between two codes
    P.adamw(torch.cuda.current_stream(), x.call(grad_scale=1.0))
    torch.cuda.synchronize()
    m, v, ms, vs = (a[0] for a in x.host())
    rest = np.arange(n) % 32 != 0
    got_m, got_v = decoded(m[:n], ms[:n // 32])[rest], decoded(v[:n], vs[:n // 32])[rest] ** 2
    b1, b2, d = f32(0.9), f32(0.98), f32(0.7)
    for got, want in ((got_m, f32(1 - b1) * d), (got_v, f32(1 - b2) * d * d)):
        values = np.unique(got)
        assert values.size == 2 and values[0] < want < values[1]
        assert abs(got.mean() - want) <= 6 * 0.5 * (values[1] - values[0]) / math.sqrt(rest.sum())


def test_checkpoint_load_reads_the_states():
    x = Eight([3000], 1, 8)
    P.adamw(torch.cuda.current_stream(), x.call())
    m, v, ms, vs = (a[0] for a in x.host())
    for codes, scales, c, s in ((x.m, x.m_scales, m, ms), (x.v, x.v_scales, v, vs)):
        out = torch.empty(3000, device="cuda")
        P.checkpoint_load(torch.cuda.current_stream(), P.F32, 1, 3000, codes, 3000, scales, 94, out, 3000)
        assert np.array_equal(out.cpu().numpy().astype(np.float64), decoded(c[:3000], s[:94]))


# ---- calls -------------------------------------------------------------------------------------------

def test_the_number_of_a_tensor_and_nothing_else_keys_its_bits():
    """One call with many tensors (several launches) and calls with the ones in front emptied: the same bits."""
    sizes = [300 + 32 * (i % 5) for i in range(90)]
    x, y = Eight(sizes, 2, 11), Eight(sizes, 2, 11)
    P.adamw(torch.cuda.current_stream(), x.call())
    whole = y.tensors()
    for lo, hi in ((0, 37), (37, 61), (61, 90)):
        part = [t if lo <= i < hi else dict(n=0) for i, t in enumerate(whole)]
        c = y.call()
        c.set_tensors(part)
        P.adamw(torch.cuda.current_stream(), c)
    torch.cuda.synchronize()
    assert torch.equal(x.p.all, y.p.all) and all(np.array_equal(a, b) for a, b in zip(x.host(), y.host()))


def device_now(now):
    return torch.frombuffer(bytearray(bytes(now)), dtype=torch.uint8).cuda()


@pytest.mark.parametrize("eight", [False, True])
def test_terms_on_the_device(eight):
    def make():
        if eight:
            x = Eight([5000, 77], 2, 12)
            return x, x.call, lambda: [x.p.all.clone()] + [torch.from_numpy(a) for a in x.host()]
        call, tensors, p, g, m, v, _ = state_call(("fp32", "bf16", None), [5000, 77], 2, 12, 0)

        def again(**more):
            return P.AdamW(tensors=tensors, dtype=P.F32, grad_dtype=P.BF16, workers=2, stride=p.stride, **{**HYPER, **more})
        return (p, g, m, v), again, lambda: [t.buf.clone() for t in (p, m, v)]

    keep_a, call_a, read_a = make()
    keep_b, call_b, read_b = make()
    steps = [dict(step=k + 1, lr=1e-2 / (k + 1), seed=1000 + k, grad_scale=1.0 / (k + 1)) for k in range(5)]
    now = device_now(P.adamw_now(call_b(**steps[0])))
    replayed = call_b(lr=float("nan"), step=0, grad_scale=float("nan"), now=now)       # (not read)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        P.adamw(side, replayed)
    for k, s in enumerate(steps):
        P.adamw(torch.cuda.current_stream(), call_a(**s))
        terms = P.adamw_now(call_b(**s))
        now.copy_(device_now(terms))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(read_a(), read_b())), k
        if k == 2:                                             # a step that overflowed
            terms.skip = 1
            now.copy_(device_now(terms))
            before = read_b()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(before, read_b()))


def test_more_than_4_gib_between_workers():
    stride = (1 << 31) + 64
    p = torch.zeros(stride + 5000, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros_like(p)
    m, v = torch.zeros(stride + 5000, dtype=torch.uint8, device="cuda"), torch.zeros(stride + 5000, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(stride // 32 + 200, dtype=torch.uint8, device="cuda"), torch.zeros(stride // 32 + 200, dtype=torch.uint8, device="cuda")
    for at in (0, stride):
        g[at:at + 5000] = torch.randn(5000, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(torch.bfloat16)
    P.adamw(torch.cuda.current_stream(), P.AdamW(tensors=[dict(n=5000, p=p, g=g, m=m, v=v, m_scales=ms, v_scales=vs)], dtype=P.BF16, grad_dtype=P.BF16, state=P.ADAMW_STATE_8BIT,
                                                 workers=2, stride=stride, **HYPER))
    torch.cuda.synchronize()
    assert torch.equal(p[:5000], p[stride:]) and bool(p[:5000].any()) and torch.equal(ms[:157], ms[stride // 32:stride // 32 + 157]) and bool(ms[:157].all())
    for x in (p, m, v):
        assert not bool(x[5000:stride].any())


def test_local_steps_of_workers_and_their_average():
    """Local SGD with AdamW as the local step: steps in place on the live model of an idle context, then the blocking average."""
    W, d = 4, 3001
    padded, _, _ = P.plan_layout(d)
    xA, xB = torch.zeros((W, padded), device="cuda"), torch.zeros((W, padded), device="cuda")
    mean, g = torch.zeros(padded, device="cuda"), torch.zeros((W, padded), device="cuda")
    m, v = torch.zeros((W, padded), device="cuda"), torch.zeros((W, padded), device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    xA[:, :d] = torch.randn(W, d, generator=gen, device="cuda")
    s_c, s_a = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    want = xA[:, :d].double()
    wm, wv = torch.zeros_like(want), torch.zeros_like(want)
    with P.Context(W=W, d=d, stride=padded, xA=xA, xB=xB, mean=mean, lr=0.0, grad=P.GRAD_EXTERNAL, compute_stream=s_c, avg_stream=s_a) as ctx:
        step = 0
        for _ in range(2):
            for _ in range(3):
                step += 1
                g[:, :d] = torch.randn(W, d, generator=gen, device="cuda")
                torch.cuda.synchronize()
                live = ctx.live_model()
                P.adamw(s_c, P.AdamW(tensors=[dict(n=d, p=live, g=g, m=m, v=v, weight_decay=0.01)], dtype=P.F32, grad_dtype=P.F32, workers=W, stride=padded, lr=1e-2, beta1=0.9, beta2=0.98,
                                     eps=1e-6, step=step))
                (want, wm, wv), _ = formula(want, g[:, :d], wm, wv, 0.01, 1.0, {**HYPER, "step": step, "grad_scale": 1.0})
            ctx.average_apply_fused()
            ctx.sync()
            want = want.mean(0, keepdim=True).expand(W, d).contiguous()
        x = xA if ctx.live_model() == xA.data_ptr() else xB
        # six steps and two means, each off by a few roundings of values up to 5
        assert float((x[:, :d].double() - want).abs().max()) <= 6 * 20 * E * 5
        assert not bool(x[:, d:].any())


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("gradient", [1e-17, 1e-19, 3e-20])
@pytest.mark.parametrize("n", [64, 2050])
def test_squares_below_the_normal_numbers(eight, gradient, n):
    """The first step without eps is lr whatever the gradient's size, its sign the gradient's; v of 1e-38 and less has steps of 2^-149, half of one moves its root by 2^-151 / v of itself."""
    g = torch.full((n,), gradient, device="cuda")
    g[1::2] *= -1
    p = torch.ones(n, device="cuda")
    block = -(-n // 32)
    m, v = (torch.zeros(n, dtype=torch.uint8 if eight else torch.float32, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(block, dtype=torch.uint8, device="cuda") for _ in range(2))
    one = dict(n=n, p=p, g=g, m=m, v=v, **(dict(m_scales=ms, v_scales=vs) if eight else {}))
    call = P.AdamW(tensors=[one], dtype=P.F32, grad_dtype=P.F32, state=P.ADAMW_STATE_8BIT if eight else P.ADAMW_STATE_F32, lr=0.125, beta1=0.9, beta2=0.95, eps=0.0, step=1, seed=3)
    P.adamw(torch.cuda.current_stream(), call)
    want = 1.0 - 0.125 * torch.sign(g).double()
    bound = 0.125 * (16 * E + 2 * 2.0 ** -151 / (0.05 * gradient ** 2)) + 2 * E
    assert bool(((p.double() - want).abs() <= bound).all())
    if eight:                                                  # (not zero is not stored as zero)
        assert bool((v > 0).all())
