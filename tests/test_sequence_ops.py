"""Sequence operators against their definitions in 64 bits (oracle/sequence.py), element by element.

Tolerances (fixed before the kernels first ran): an output may be off by one rounding to its type, u |ref| with u = 2^-24,
2^-11, 2^-8 for fp32, fp16, bf16, plus `scale` times the magnitude of what was summed (the same formula over absolute
values).  Convolution: (taps + 3) roundings and 2^-21 of the activation: 2^-19 (gradients: (tokens + 32) 2^-24, the length of
the longest sum).  Scan: 2^-16 per recurrence (see the oracle), 2^-14 for gradients, whose products hold two of them and
sums over tokens and channels.  Norm: the variance about a first element within four standard deviations loses a factor of
17 at most over chains of 64 sums: 2^-14 of (1 + |xhat|) |w|.
"""
import numpy as np
import pytest
import torch

from oracle import sequence as ref
from paper_2010_15884_b200 import sequence as seq
from paper_2010_15884_b200 import binding

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}


def close(got, want, mag, scale, what):
    u, tiny = UNIT[got.dtype], TINY[got.dtype]
    g = got.detach().cpu().double().numpy()
    assert g.shape == want.shape, (what, g.shape, want.shape)
    bound = u * np.abs(want) + scale * np.broadcast_to(mag, want.shape) + tiny
    off = np.abs(g - want) / bound
    assert np.isfinite(g).all(), what + ": not finite"
    assert g.size == 0 or off.max() <= 1.0, "%s: %.3g times the bound at %s (got %r, want %r)" % (
        what, off.max(), np.unravel_index(off.argmax(), off.shape), g.flat[off.argmax()], want.flat[off.argmax()])


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


class Draw:
    def __init__(self, seed, dtype):
        self.rng, self.dtype = np.random.default_rng(seed), dtype

    def __call__(self, *shape, scale=1.0, dtype=None):
        return torch.from_numpy(self.rng.standard_normal(shape) * scale).to(dtype or self.dtype).cuda()


def spans(lengths):
    at = np.concatenate([[0], np.cumsum(lengths)])
    return [(int(a), int(b)) for a, b in zip(at[:-1], at[1:])]


def offsets(lengths, kind=torch.int32):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=kind, device="cuda")


# ------------------------------------------------------------------------------------------ causal convolution

CONV = [  # type, lengths, channels, taps, bias, act, state, weight type, packed
    ("bf16", [37], 64, 4, True, True, True, "bf16", False),
    ("bf16", [1, 0, 2, 53, 0, 0, 3, 17, 1], 40, 4, True, True, True, "bf16", True),
    ("f32", [0, 0, 5, 130, 0], 33, 3, True, True, False, "f32", True),
    ("f16", [9, 9, 9], 24, 2, False, False, True, "f32", False),
    ("f32", [21, 21], 8, 1, True, True, False, "f32", False),
    ("bf16", [7, 7], 17, 8, True, True, True, "bf16", False),
    ("f32", [1], 4, 5, False, True, True, "f32", False),
    ("f16", [2, 3, 1, 1, 1, 4], 16, 6, True, True, True, "f16", True),
    ("bf16", [3, 70], 1, 7, True, False, True, "f32", True),
    ("bf16", [0, 0], 16, 4, True, True, True, "bf16", True),
]


def conv_case(case, seed=0):
    kind, lengths, d, k, bias, act, state, wkind, packed = case
    draw = Draw(seed + d * 7 + k, TYPES[kind])
    n, r = sum(lengths), len(lengths)
    x, dy = draw(n, d), draw(n, d)
    w = draw(d, k, scale=0.6, dtype=TYPES[wkind])
    b = draw(d, scale=0.3, dtype=TYPES[wkind]) if bias else None
    st = draw(r, k - 1, d) if state else None
    if not packed:
        x, dy = x.view(r, lengths[0], d), dy.view(r, lengths[0], d)
    return x, dy, w, b, st, "silu" if act else None, offsets(lengths) if packed else None


@pytest.mark.parametrize("case", CONV, ids=str)
def test_conv_forward_and_final_state(cuda_device, case):
    x, _, w, b, st, act, off = conv_case(case)
    y, final = seq.conv1d_causal(x, w, b, act, state=st, offsets=off, return_state=True)
    d = x.shape[-1]
    for i, (lo, hi) in enumerate(spans(case[1])):
        bb = np.zeros(d) if b is None else f64(b)
        want, last, mag = ref.conv_causal(f64(x.reshape(-1, d)[lo:hi]), f64(w), bb, None if st is None else f64(st[i]), act is not None)
        close(y.reshape(-1, d)[lo:hi], want, mag, 2.0 ** -19, "y")
        assert np.array_equal(f64(final[i]), last), "the final state is the inputs themselves"


@pytest.mark.parametrize("case", CONV, ids=str)
def test_conv_backward(cuda_device, case):
    x, dy, w, b, st, act, off = conv_case(case, 1)
    d, k, n = x.shape[-1], w.shape[1], sum(case[1])
    dfinal = Draw(5, x.dtype)(len(case[1]), k - 1, d) if st is not None else None
    dx, dw, db, ds = seq.conv1d_causal_backward(dy, x, w, b, act, state=st, offsets=off, dfinal=dfinal)
    assert (db is None) == (b is None) and (ds is None) == (st is None)
    scale = (n + 32) * 2.0 ** -24
    sw, swm, sb, sbm = 0.0, 0.0, 0.0, 0.0
    for i, (lo, hi) in enumerate(spans(case[1])):
        g = ref.conv_causal_backward(f64(dy.reshape(-1, d)[lo:hi]), f64(x.reshape(-1, d)[lo:hi]), f64(w), np.zeros(d) if b is None else f64(b),
                                     None if st is None else f64(st[i]), act is not None, None if dfinal is None else f64(dfinal[i]))
        close(dx.reshape(-1, d)[lo:hi], g["dx"], g["dx_mag"], scale, "dx")
        if ds is not None:
            close(ds[i], g["dstate"], g["dstate_mag"], scale, "dstate")
        sw, swm, sb, sbm = sw + g["dw"], swm + g["dw_mag"], sb + g["db"], sbm + g["db_mag"]
    close(dw, sw, swm, scale, "dweight")
    if db is not None:
        close(db, sb, sbm, scale, "dbias")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_conv_runs_meet_and_long_sums(cuda_device, kind):
    """Many runs per sequence (their windows overlap), and dweight as a sum over many blocks, against torch in 64 bits."""
    draw = Draw(3, TYPES[kind])
    x, dy, w, b, st = draw(3, 1501, 96), draw(3, 1501, 96), draw(96, 4, scale=0.5), draw(96), draw(3, 3, 96)
    xd, wd, bd, sd = (v.double().requires_grad_() for v in (x, w, b, st))
    line = torch.cat([sd, xd], 1).transpose(1, 2)
    pre = torch.nn.functional.conv1d(line, wd[:, None], bd, groups=96).transpose(1, 2)
    yd = torch.nn.functional.silu(pre)
    yd.backward(dy.double())
    y, final = seq.conv1d_causal(x, w, b, "silu", state=st, return_state=True)
    got = seq.conv1d_causal_backward(dy, x, w, b, "silu", state=st)
    mag = torch.nn.functional.conv1d(line.abs(), wd.abs()[:, None], bd.abs(), groups=96).transpose(1, 2)
    close(y, f64(yd), f64(mag), 2.0 ** -19, "y")
    assert torch.equal(final, x[:, -3:])
    for v, g, what in zip(got, (xd.grad, wd.grad, bd.grad, sd.grad), ("dx", "dweight", "dbias", "dstate")):
        # sums of up to 4503 products of terms of magnitude below 6 each, in chains of at most 64 and trees
        close(v, f64(g), np.full(g.shape, 4503.0 if what in ("dweight", "dbias") else 20.0), 2.0 ** -18, what)


def test_conv_strided_views(cuda_device):
    """x is one half of a wider projection, dy too; rows are not packed and (second form) not aligned."""
    for start in (0, 64, 3):
        wide, dwide = Draw(9, torch.bfloat16)(2, 29, 160), Draw(10, torch.bfloat16)(2, 29, 160)
        x, dy = wide[..., start: start + 64], dwide[..., start: start + 64]
        w, b = Draw(11, torch.bfloat16)(64, 4), Draw(12, torch.bfloat16)(64)
        assert torch.equal(seq.conv1d_causal(x, w, b, "silu"), seq.conv1d_causal(x.contiguous(), w, b, "silu"))
        got = seq.conv1d_causal_backward(dy, x, w, b, "silu")[:3]
        want = seq.conv1d_causal_backward(dy.contiguous(), x.contiguous(), w, b, "silu")[:3]
        assert torch.equal(got[0], want[0])
        for g, v in zip(got[1:], want[1:]):
            assert torch.allclose(g.float(), v.float(), rtol=2 ** -7, atol=1e-2)       # other runs, one rounding each


@pytest.mark.parametrize("kind,d,k,slots", [("bf16", 64, 4, True), ("f32", 33, 3, True), ("f16", 16, 2, False), ("bf16", 8, 1, False),
                                            ("bf16", 130, 8, True)])
def test_conv_step_follows_the_prompt(cuda_device, kind, d, k, slots):
    draw = Draw(d, TYPES[kind])
    rows, n = 5, 9
    x, w, b, st = draw(rows, n, d), draw(d, k, scale=0.5), draw(d), draw(rows, k - 1, d)
    want, last = seq.conv1d_causal(x, w, b, "silu", state=st, return_state=True)
    at = torch.tensor([6, 0, 3, 7, 2], dtype=torch.int32, device="cuda") if slots else None
    cache = draw(8 if slots else rows, k - 1, d)
    before = cache.clone()
    where = at.long() if slots else torch.arange(rows, device="cuda")
    cache[where] = st
    for t in range(n):
        y = seq.conv1d_causal_step(x[:, t], cache, w, b, "silu", slots=at)
        assert torch.equal(y, want[:, t]), "the same products in the same order"
    assert torch.equal(cache[where], last)
    if slots:
        rest = torch.tensor([1, 4, 5], device="cuda")
        assert torch.equal(cache[rest], before[rest])


def test_step_rows_without_a_slot(cuda_device):
    draw = Draw(1, torch.bfloat16)
    at = torch.tensor([2, -1, 0, 9], dtype=torch.int32, device="cuda")
    x, w, st = draw(4, 24), draw(24, 4), draw(3, 3, 24)
    before = st.clone()
    y = seq.conv1d_causal_step(x, st, w, None, "silu", slots=at)
    assert (y[1] == 0).all() and (y[3] == 0).all() and (y[0] != 0).any() and torch.equal(st[1], before[1])
    h = draw(3, 24, 16, dtype=torch.float32)
    before = h.clone()
    A = -Draw(2, torch.float32)(24, 16).abs()
    y = seq.state_scan_step(x, draw(4, 24), A, draw(4, 16), draw(4, 16), h, softplus=True, slots=at)
    assert (y[1] == 0).all() and (y[3] == 0).all() and (y[0] != 0).any() and torch.equal(h[1], before[1])


# ------------------------------------------------------------------------------------------ state space scan

SCAN = [  # type, lengths, channels, states, groups, D, z, bias, softplus, state, packed
    ("bf16", [37, 37], 24, 16, 1, True, True, True, True, True, False),
    ("f32", [1, 0, 2, 53, 0, 33, 17], 20, 16, 2, True, True, True, True, True, True),
    ("f16", [16], 9, 4, 1, False, False, False, True, False, False),
    ("f32", [31, 31], 6, 1, 3, True, False, True, False, True, False),
    ("f32", [65], 5, 2, 1, False, True, False, True, True, False),
    ("bf16", [48], 40, 8, 4, True, True, True, True, False, False),
    ("f32", [40, 3], 10, 19, 1, True, True, True, True, True, True),
    ("bf16", [35], 12, 32, 1, True, True, True, True, True, False),
    ("f32", [33], 6, 64, 1, True, True, True, True, True, False),
    ("f32", [20], 5, 128, 1, True, True, True, True, True, False),
    ("bf16", [18], 3, 100, 1, True, True, True, True, True, False),
    ("f16", [0, 0], 8, 16, 1, True, True, True, True, True, True),
    ("f32", [1], 1, 16, 1, True, True, True, True, True, False),
]


def scan_case(case, seed=0):
    kind, lengths, d, n, g, skip, gate, bias, plus, state, packed = case
    draw, f32 = Draw(seed + d * 7 + n, TYPES[kind]), torch.float32
    m, r = sum(lengths), len(lengths)
    v = {"u": draw(m, d), "delta": draw(m, d, scale=0.5) if plus else (draw(m, d).abs() * 0.1), "B": draw(m, g, n), "C": draw(m, g, n)}
    if gate:
        v["z"] = draw(m, d)
    dy = draw(m, d)
    p = {"A": -(draw(d, n, dtype=f32).abs() + 0.2) * 2.0}
    if skip:
        p["D"] = draw(d, dtype=f32)
    if bias:
        p["delta_bias"] = draw(d, dtype=f32) - 2.0 if plus else draw(d, dtype=f32).abs() * 0.05
    st = draw(r, d, n, dtype=f32) if state else None
    if not packed:
        v = {k: t.view((r, lengths[0]) + t.shape[1:]) for k, t in v.items()}
        dy = dy.view(r, lengths[0], d)
    return v, p, dy, st, plus, offsets(lengths) if packed else None


def scan_ref(case, v, p, st, plus, i, lo, hi):
    flat = {k: f64(t).reshape((-1,) + t.shape[-2:] if k in "BC" else (-1, t.shape[-1]))[lo:hi] for k, t in v.items()}
    return dict(u=flat["u"], delta=flat["delta"], A=f64(p["A"]), B=flat["B"], C=flat["C"], D=f64(p.get("D")), z=flat.get("z"),
                bias=f64(p.get("delta_bias")), plus=plus, state=None if st is None else f64(st[i]))


@pytest.mark.parametrize("case", SCAN, ids=str)
def test_scan_forward_and_final_state(cuda_device, case):
    v, p, _, st, plus, off = scan_case(case)
    y, final = seq.state_scan(**v, **p, softplus=plus, state=st, offsets=off, return_state=True)
    d = y.shape[-1]
    for i, (lo, hi) in enumerate(spans(case[1])):
        f = ref.scan(**scan_ref(case, v, p, st, plus, i, lo, hi))
        close(y.reshape(-1, d)[lo:hi], f["y"], f["y_mag"], 2.0 ** -16, "y")
        close(final[i], f["final"], f["final_mag"], 2.0 ** -16, "final state")


@pytest.mark.parametrize("case", SCAN, ids=str)
def test_scan_backward(cuda_device, case):
    v, p, dy, st, plus, off = scan_case(case, 1)
    d, r = dy.shape[-1], len(case[1])
    y, saved = seq.state_scan(**v, **p, softplus=plus, state=st, offsets=off, save=True)
    dfinal = Draw(4, torch.float32)(r, d, case[3])
    g = seq.state_scan_backward(dy, saved=saved, **v, **p, softplus=plus, offsets=off, dfinal=dfinal, state_grad=True)
    scale = 2.0 ** -14
    total = {}
    for i, (lo, hi) in enumerate(spans(case[1])):
        w = ref.scan_backward(f64(dy).reshape(-1, d)[lo:hi], **scan_ref(case, v, p, st, plus, i, lo, hi), dfinal=f64(dfinal[i]))
        for got, name in ((g.du, "du"), (g.ddelta, "dd"), (g.dz, "dz")):
            if got is not None:
                close(got.reshape(-1, d)[lo:hi], w[name], w[name + "_mag"], scale, name)
        for got, name in ((g.dB, "dB"), (g.dC, "dC")):
            close(got.reshape((-1,) + got.shape[-2:])[lo:hi], w[name], w[name + "_mag"], scale, name)
        close(g.dstate[i], w["dstate"], w["dstate_mag"], scale, "dstate")
        for name in ("dA", "dD", "dbias"):
            total[name] = total.get(name, 0.0) + w[name]
            total[name + "_mag"] = total.get(name + "_mag", 0.0) + w[name + "_mag"]
    for got, name in ((g.dA, "dA"), (g.dD, "dD"), (g.ddelta_bias, "dbias")):
        if got is not None:
            close(got, total[name], total[name + "_mag"], scale, name)


def _loop64(v, p, state, plus):
    """Dense sequences in torch float64 on the GPU, differentiable."""
    u, delta, B, C = (v[k].double() for k in ("u", "delta", "B", "C"))
    d, g = u.shape[-1], B.shape[2]
    dl = delta + p["delta_bias"].double()
    dl = torch.nn.functional.softplus(dl) if plus else dl
    h, ys = state.double(), []
    for t in range(u.shape[1]):
        b, c = (x[:, t].repeat_interleave(d // g, 1) for x in (B, C))
        h = torch.exp(dl[:, t, :, None] * p["A"].double()) * h + (dl[:, t] * u[:, t])[..., None] * b
        ys.append((h * c).sum(-1))
    y = torch.stack(ys, 1) + p["D"].double() * u
    return y * torch.nn.functional.silu(v["z"].double()), h


@pytest.mark.parametrize("length,d,n,batch", [(1500, 32, 16, 1), (2051, 6, 16, 2), (700, 40, 4, 1), (900, 3, 64, 1), (513, 24, 2, 1)])
def test_scan_split_over_tokens(cuda_device, length, d, n, batch):
    """Few channels and many tokens: the tokens are cut in chunks, forward and backward.  Bounds are relative to the 2-norm:
    1e-5 of it, for fp32 sums over up to 2051 tokens of positive and negative terms."""
    case = ("f32", [length] * batch, d, n, 1, True, True, True, True, True, False)
    v, p, dy, st, plus, _ = scan_case(case, 2)
    leaf = {k: t.double().requires_grad_() for k, t in {**v, **p, "state": st}.items()}
    yd, hd = _loop64(leaf, leaf, leaf["state"], plus)
    df = Draw(8, torch.float32)(batch, d, n)
    ((yd * dy.double()).sum() + (hd * df.double()).sum()).backward()
    before = binding.launch_count()
    y, final, saved = seq.state_scan(**v, **p, softplus=plus, state=st, return_state=True, save=True)
    assert binding.launch_count() - before == 3, "the split form was expected to run"
    g = seq.state_scan_backward(dy, saved=saved, **v, **p, softplus=plus, dfinal=df, state_grad=True)

    def near(got, want, what):
        e = float((got.double() - want).norm() / want.norm())
        assert e <= 1e-5, "%s: %.3g" % (what, e)

    near(y, yd, "y")
    near(final, hd, "final")
    for got, name in ((g.du, "u"), (g.ddelta, "delta"), (g.dA, "A"), (g.dB, "B"), (g.dC, "C"), (g.dD, "D"), (g.dz, "z"),
                      (g.ddelta_bias, "delta_bias"), (g.dstate, "state")):
        near(got, leaf[name].grad, name)


def test_scan_split_with_uneven_packed_lengths(cuda_device):
    """`longest` below the truth may cost time but never results: the last chunk of a sequence takes what is left."""
    lengths = [3, 1400, 0, 200, 1]
    case = ("f32", lengths, 8, 16, 1, True, True, True, True, True, True)
    v, p, dy, st, plus, off = scan_case(case, 3)
    runs = []
    for longest in (None, 1400, 600):
        y, final, saved = seq.state_scan(**v, **p, softplus=plus, state=st, offsets=off, longest=longest, return_state=True, save=True)
        g = seq.state_scan_backward(dy, saved=saved, **v, **p, softplus=plus, offsets=off, longest=longest, state_grad=True)
        runs.append((y, final) + tuple(g))
    alone = {k: t[3:1403].unsqueeze(0) for k, t in v.items()}
    y1 = seq.state_scan(**alone, **p, softplus=plus, state=st[1:2])
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert float((a - b).norm() / b.norm()) <= 1e-5
    assert float((runs[0][0][3:1403] - y1[0]).norm() / y1.norm()) <= 1e-5


def test_scan_gradient_against_differences(cuda_device):
    """<gradient, direction> from the kernels against central differences of the definition in 64 bits; step 1e-5: the
    difference's own error is about 1e-8 of the loss's terms, the kernels' about 1e-5."""
    case = ("f32", [21, 21], 10, 16, 2, True, True, True, True, True, False)
    v, p, dy, st, plus, _ = scan_case(case, 4)
    y, saved = seq.state_scan(**v, **p, softplus=plus, state=st, save=True)
    g = seq.state_scan_backward(dy, saved=saved, **v, **p, softplus=plus, state_grad=True)
    every = {**v, **p, "state": st}
    grads = {"u": g.du, "delta": g.ddelta, "A": g.dA, "B": g.dB, "C": g.dC, "D": g.dD, "z": g.dz, "delta_bias": g.ddelta_bias, "state": g.dstate}
    for name, t in every.items():
        w = Draw(len(name), torch.float64)(*t.shape)
        loss = []
        for sign in (1.0, -1.0):
            moved = {k: x.double() + (sign * 1e-5 * w if k == name else 0.0) for k, x in every.items()}
            loss.append(float((_loop64(moved, moved, moved["state"], plus)[0] * dy.double()).sum()))
        want, got = (loss[0] - loss[1]) / 2e-5, float((grads[name].double() * w).sum())
        size = float((grads[name].double() * w).abs().sum())
        assert abs(got - want) <= 1e-4 * size, (name, got, want, size)


@pytest.mark.parametrize("kind,d,n,g", [("bf16", 24, 16, 1), ("f32", 10, 19, 2), ("f16", 5, 4, 1), ("f32", 3, 128, 1), ("bf16", 7, 1, 7)])
def test_scan_step_follows_the_prompt(cuda_device, kind, d, n, g):
    case = (kind, [6, 6, 6], d, n, g, True, True, True, True, True, False)
    v, p, _, st, plus, _ = scan_case(case, 5)
    want, last = seq.state_scan(**v, **p, softplus=plus, state=st, return_state=True)
    at = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    cache = Draw(6, torch.float32)(5, d, n)
    untouched = cache[[1, 3]].clone()
    cache[at.long()] = st
    for t in range(6):
        y = seq.state_scan_step(v["u"][:, t], v["delta"][:, t], p["A"], v["B"][:, t], v["C"][:, t], cache, D=p["D"], z=v["z"][:, t],
                                delta_bias=p["delta_bias"], softplus=True, slots=at)
        # both within 2^-16 of magnitudes below 10 + 3 sqrt(states) of the same value, then one rounding each
        bound = 2 * UNIT[y.dtype] * want[:, t].double().abs() + 2.0 ** -15 * (10 + 3 * n ** 0.5) + TINY[y.dtype]
        assert ((y.double() - want[:, t].double()).abs() <= bound).all()
    assert float((cache[at.long()] - last).norm() / last.norm()) <= 1e-5
    assert torch.equal(cache[[1, 3]], untouched)


def test_scan_strided_views_and_64_bit_offsets(cuda_device):
    """u and z are halves of one projection, delta, B and C pieces of another, as a block has them."""
    draw, f32 = Draw(7, torch.bfloat16), torch.float32
    lengths = [11, 0, 40]
    for d, n in ((32, 16), (19, 5)):
        uz, dbc = draw(51, 2 * d), draw(51, d + 2 * n)
        v = dict(u=uz[:, :d], z=uz[:, d:], delta=dbc[:, :d], B=dbc[:, d: d + n], C=dbc[:, d + n:])
        A = -draw(d, n, dtype=f32).abs()
        packed = {k: t.contiguous() for k, t in v.items()}
        for kind in (torch.int32, torch.int64):
            off = offsets(lengths, kind)
            y, saved = seq.state_scan(**v, A=A, softplus=True, offsets=off, save=True)
            y0, saved0 = seq.state_scan(**packed, A=A, softplus=True, offsets=off, save=True)
            assert torch.equal(y, y0)
            g = seq.state_scan_backward(y, **v, A=A, saved=saved, softplus=True, offsets=off)
            g0 = seq.state_scan_backward(y0, **packed, A=A, saved=saved0, softplus=True, offsets=off)
            for a, b in zip(g[:5], g0[:5]):
                assert torch.equal(a, b)


def test_scan_states_never_mix(cuda_device):
    """A NaN or infinity in one channel, state or sequence stays there."""
    case = ("f32", [20, 20], 12, 16, 1, True, True, True, True, True, False)
    v, p, _, st, plus, _ = scan_case(case, 6)
    clean = seq.state_scan(**v, **p, softplus=plus, state=st)
    bad = v["u"].clone()
    bad[1, 3, 5] = float("nan")
    bad[0, 19, 2] = float("inf")
    y = seq.state_scan(**dict(v, u=bad), **p, softplus=plus, state=st)
    hit = torch.zeros_like(y, dtype=torch.bool)
    hit[1, 3:, 5] = True
    hit[0, 19:, 2] = True
    assert torch.equal(y[~hit], clean[~hit]) and (~torch.isfinite(y[hit])).all()
    strong = dict(p, A=p["A"].clone())
    strong["A"][4] = -float("inf")                                         # forgets everything at once
    y, final = seq.state_scan(**v, **strong, softplus=plus, state=st, return_state=True)
    assert torch.isfinite(y).all() and torch.isfinite(final).all()


def test_results_repeat_bit_for_bit(cuda_device):
    case = ("bf16", [300, 300], 64, 16, 1, True, True, True, True, True, False)
    v, p, dy, st, plus, _ = scan_case(case, 7)
    x, w = v["u"], Draw(1, torch.bfloat16)(64, 4)
    norm_w = Draw(2, torch.float32)(64)

    def all_of_it():
        y, saved = seq.state_scan(**v, **p, softplus=plus, state=st, save=True)
        g = seq.state_scan_backward(dy, saved=saved, **v, **p, softplus=plus, state_grad=True)
        yn, mean, rstd = seq.groupnorm(x, 4, norm_w, norm_w, activation="silu", return_stats=True)
        return (y, saved) + tuple(g) + seq.conv1d_causal_backward(dy, x, w)[:2] + (yn,) + seq.groupnorm_backward(
            dy, x, 4, mean, rstd, norm_w, norm_w, "silu")

    first = all_of_it()
    for _ in range(3):
        for a, b in zip(first, all_of_it()):
            assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------ group norm

NORM = [  # type, batch, space, channels, groups, affine, act
    ("bf16", 5, (1,), 64, 4, True, True),
    ("f32", 1, (1,), 512, 1, True, False),
    ("bf16", 700, (1,), 256, 8, True, False),
    ("f16", 3, (7, 5), 40, 4, True, True),
    ("f32", 2, (33, 17), 30, 3, True, True),
    ("bf16", 2, (64, 64), 96, 32, True, True),
    ("f32", 1, (1000,), 7, 7, True, True),
    ("bf16", 1, (3,), 1, 1, False, False),
    ("f32", 2, (11,), 2400, 2, True, True),
    ("bf16", 2, (9,), 5000, 1, True, True),
    ("f16", 9, (2,), 24, 24, True, False),
    ("f32", 3, (300, 21), 16, 1, False, True),
    ("bf16", 6, (1,), 9000, 3, True, True),
]


def norm_case(case, seed=0):
    kind, b, space, c, g, affine, act = case
    draw, f32 = Draw(seed + c, TYPES[kind]), torch.float32
    x = (draw(b, *space, c, dtype=f32) * 1.7 + draw(c, dtype=f32)).to(TYPES[kind])
    w, bias = (draw(c, dtype=f32), draw(c, dtype=f32)) if affine else (None, None)
    return x, draw(b, *space, c), g, w, bias, "silu" if act else None


@pytest.mark.parametrize("case", NORM, ids=str)
def test_norm_forward_and_backward(cuda_device, case):
    x, dy, g, w, b, act = norm_case(case)
    y, mean, rstd = seq.groupnorm(x, g, w, b, eps=1e-5, activation=act, return_stats=True)
    assert torch.equal(y, seq.groupnorm(x, g, w, b, eps=1e-5, activation=act))
    n, c = x.shape[0], x.shape[-1]
    x3, dy3 = f64(x).reshape(n, -1, c), f64(dy).reshape(n, -1, c)
    want, m, r, xhat, pre = ref.groupnorm(x3, g, f64(w), f64(b), 1e-5, act is not None)
    ww, bb = (1.0, 0.0) if w is None else (np.abs(f64(w)), np.abs(f64(b)))
    mag = (1.0 + np.abs(xhat)) * ww + bb
    close(y.reshape(n, -1, c), want, mag, 2.0 ** -14, "y")
    close(mean, m, 1.0 / r, 2.0 ** -14, "mean")
    close(rstd, r, r, 2.0 ** -14, "rstd")
    dx, dw, db = seq.groupnorm_backward(dy, x, g, mean, rstd, w, b, act)
    k = ref.groupnorm_backward(dy3, x3, g, f64(w), f64(b), 1e-5, act is not None)
    slope = 1.0 + (mag if act else 0.0)                                    # the slope moves by half an error of pre
    rs = np.repeat(r, c // g, axis=1)[:, None, :]
    close(dx.reshape(n, -1, c), k["dx"], k["dx_mag"] * slope + rs * np.abs(dy3) * ww * slope, 2.0 ** -13, "dx")
    assert (dw is None) == (w is None) and (db is None) == (b is None)
    if w is not None:
        close(dw, k["dw"], k["dw_mag"] * (1 + np.max(mag)), 2.0 ** -14, "dweight")
        close(db, k["db"], k["db_mag"] * (1 + np.max(mag)), 2.0 ** -14, "dbias")


NORM_TILES = [
    ("bf16", 3, (50,), 448, 7, True, True),         # tiles of four groups and of three
    ("f16", 200, (12,), 24, 1, True, True),
    ("bf16", 150, (13,), 440, 8, True, False),
    ("f32", 70, (100,), 600, 3, True, True),        # more than 64 KB a tile
    ("f16", 5, (31,), 9, 3, True, True),            # one channel an access, of 16 bits
    ("bf16", 2, (90, 80), 23, 1, True, True),       # slabs, one channel an access
    ("bf16", 1, (700,), 4096, 8, True, True),       # slabs, several tiles of channels
    ("f32", 2, (40, 40), 1030, 5, False, True),
]


@pytest.mark.parametrize("case", NORM_TILES, ids=str)
def test_norm_tiles_and_slabs(cuda_device, case):
    test_norm_forward_and_backward(cuda_device, case)


def test_norm_leaves_its_inputs(cuda_device):
    x, dy, g, w, b, act = norm_case(NORM_TILES[0])
    kept = x.clone(), dy.clone()
    y, mean, rstd = seq.groupnorm(x, g, w, b, activation=act, return_stats=True)
    seq.groupnorm_backward(dy, x, g, mean, rstd, w, b, act)
    assert torch.equal(x, kept[0]) and torch.equal(dy, kept[1])


def test_norm_mean_far_from_zero_and_constant_groups(cuda_device):
    """A mean 1000 deviations away costs no digits beyond those of the inputs; a constant group has variance 0."""
    x = (Draw(1, torch.float32)(3, 500, 32) + 1000.0)
    y = seq.groupnorm(x, 4)
    want = ref.groupnorm(f64(x), 4, None, None, 1e-5, False)[0]
    close(y, want, 1.0 + np.abs(want), 2.0 ** -14, "far mean")              # x - mean is exact to 2^-14 of a deviation
    flat = torch.full((2, 9, 16), 3.25, device="cuda")
    y, mean, rstd = seq.groupnorm(flat, 2, return_stats=True)
    assert (y == 0).all() and (mean == 3.25).all() and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5))


def test_norm_strided_views(cuda_device):
    wide = Draw(3, torch.bfloat16)(3, 50, 96)
    w, b = Draw(4, torch.float32)(64), Draw(5, torch.float32)(64)
    for start in (0, 32, 5):
        x = wide[..., start: start + 64]
        y, mean, rstd = seq.groupnorm(x, 4, w, b, activation="silu", return_stats=True)
        y0, m0, r0 = seq.groupnorm(x.contiguous(), 4, w, b, activation="silu", return_stats=True)
        assert torch.allclose(y.float(), y0.float(), rtol=2 ** -7, atol=1e-4) and torch.allclose(mean, m0, atol=1e-6)
        got, want = seq.groupnorm_backward(x, x, 4, mean, rstd, w, b, "silu"), seq.groupnorm_backward(x.contiguous(), x.contiguous(), 4, m0, r0, w, b, "silu")
        assert torch.allclose(got[0].float(), want[0].float(), rtol=2 ** -6, atol=1e-3)


def test_norm_gradient_against_differences(cuda_device):
    x, dy, g, w, b, act = norm_case(("f32", 2, (5, 3), 12, 3, True, True), 3)
    y, mean, rstd = seq.groupnorm(x, g, w, b, activation=act, return_stats=True)
    grads = dict(zip(("x", "w", "b"), seq.groupnorm_backward(dy, x, g, mean, rstd, w, b, act)))
    every = {"x": f64(x), "w": f64(w), "b": f64(b)}
    for name, t in every.items():
        v = np.random.default_rng(1).standard_normal(t.shape)
        loss = []
        for sign in (1.0, -1.0):
            m = dict(every, **{name: t + sign * 1e-5 * v})
            loss.append((ref.groupnorm(m["x"].reshape(2, -1, 12), g, m["w"], m["b"], 1e-5, True)[0] * f64(dy).reshape(2, -1, 12)).sum())
        got = (f64(grads[name]) * v).sum()
        assert abs(got - (loss[0] - loss[1]) / 2e-5) <= 1e-4 * np.abs(f64(grads[name]) * v).sum()


# ------------------------------------------------------------------------------------------ streams, large sizes, refusals


def test_another_stream_and_graph_replay(cuda_device):
    case = ("bf16", [40, 40], 32, 16, 1, True, True, True, True, True, False)
    v, p, dy, st, plus, _ = scan_case(case, 8)
    want = seq.state_scan(**v, **p, softplus=plus, state=st)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = seq.state_scan(**v, **p, softplus=plus, state=st, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    x, w, cache = v["u"][:, 0].contiguous(), Draw(1, torch.bfloat16)(32, 4), torch.zeros(2, 3, 32, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        seq.conv1d_causal_step(x, cache, w, None, "silu", out=out)
    cache.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    fresh = torch.zeros_like(cache)
    for _ in range(3):
        again = seq.conv1d_causal_step(x, fresh, w, None, "silu")
    assert torch.equal(out, again) and torch.equal(cache, fresh)


def test_offsets_past_32_bits(cuda_device):
    """Tokens and cache slots whose element offsets pass 2^31."""
    rows = 40000
    wide = torch.zeros(rows, 1, 65536, dtype=torch.bfloat16, device="cuda")          # 2.6 G elements, 5.2 GB
    wide[:, 0, :64] = torch.randn(rows, 64, device="cuda")
    x = wide[:, :, :64].transpose(0, 1)                                               # (1, rows, 64), time stride 65536
    w = Draw(2, torch.bfloat16)(64, 4)
    assert torch.equal(seq.conv1d_causal(x, w, None, "silu")[:, -50:], seq.conv1d_causal(x[:, -53:].contiguous(), w, None, "silu")[:, 3:])
    y = seq.groupnorm(x, 4)
    assert torch.equal(seq.groupnorm(x.contiguous(), 4), y)
    del wide, x, y
    slots = torch.zeros(34000, 64 * 16 * 64, dtype=torch.float32, device="cuda")      # 2.2 G elements, 8.9 GB
    cache = slots.as_strided((34000, 64, 16), (65536, 16, 1))
    at = torch.tensor([33999, 5], dtype=torch.int32, device="cuda")
    u, A, B = Draw(3, torch.bfloat16)(2, 64), -Draw(4, torch.float32)(64, 16).abs(), Draw(5, torch.bfloat16)(2, 16)
    y = seq.state_scan_step(u, u, A, B, B, cache, softplus=True, slots=at)
    small = torch.zeros(2, 64, 16, device="cuda")
    assert torch.equal(y, seq.state_scan_step(u, u, A, B, B, small, softplus=True))
    assert torch.equal(cache[at.long()], small) and float(slots.abs().sum()) == float(small.abs().sum())


def test_refusals_launch_nothing(cuda_device):
    x = torch.zeros(2, 5, 8, device="cuda")
    w = torch.zeros(8, 4, device="cuda")
    A, B = torch.zeros(8, 16, device="cuda"), torch.zeros(2, 5, 16, device="cuda")
    before = binding.launch_count()
    bad = [
        (TypeError, lambda: seq.conv1d_causal(x.double(), w)),
        (ValueError, lambda: seq.conv1d_causal(x, w[:7])),
        (TypeError, lambda: seq.conv1d_causal(x.bfloat16(), w.half())),
        (ValueError, lambda: seq.conv1d_causal(x, w, activation="gelu")),
        (ValueError, lambda: seq.conv1d_causal(x[0], w)),
        (ValueError, lambda: seq.conv1d_causal(x, w, state=torch.zeros(2, 4, 8, device="cuda"))),
        (ValueError, lambda: seq.conv1d_causal(x.transpose(1, 2), torch.zeros(5, 4, device="cuda"))),
        (TypeError, lambda: seq.conv1d_causal(x[0], w, offsets=torch.zeros(3, device="cuda"))),
        (ValueError, lambda: seq.conv1d_causal(x[0], w, offsets=torch.zeros(3, dtype=torch.int32))),
        (seq.SysconvError, lambda: seq.conv1d_causal(x, torch.zeros(8, 9, device="cuda"))),
        (seq.SysconvError, lambda: seq.conv1d_causal(x.cpu(), w.cpu())),
        (ValueError, lambda: seq.conv1d_causal_step(x[0], torch.zeros(4, 3, 8, device="cuda"), w)),
        (ValueError, lambda: seq.conv1d_causal_step(x[0], torch.zeros(5, 3, 8, device="cuda"), w, slots=torch.zeros(5, device="cuda"))),
        (ValueError, lambda: seq.state_scan(x, x, A[:, :8], B, B)),
        (ValueError, lambda: seq.state_scan(x, x, A, B, B[:, :4])),
        (ValueError, lambda: seq.state_scan(x, x, A, B.view(2, 5, 16, 1).expand(2, 5, 16, 3).transpose(2, 3), B)),
        (ValueError, lambda: seq.state_scan(x, x[:, :4], A, B, B)),
        (TypeError, lambda: seq.state_scan(x, x, A.half(), B, B)),
        (TypeError, lambda: seq.state_scan(x, x, A, B.half(), B.half())),
        (seq.SysconvError, lambda: seq.state_scan(x, x, torch.zeros(8, 129, device="cuda"), *[torch.zeros(2, 5, 129, device="cuda")] * 2)),
        (ValueError, lambda: seq.state_scan_backward(x, x, x, A, B, B, torch.zeros(1, 8, 16, device="cuda"))),
        (ValueError, lambda: seq.state_scan_backward(x, x, x, A, B, B, None)),
        (ValueError, lambda: seq.groupnorm(x, 3)),
        (ValueError, lambda: seq.groupnorm(x, 0)),
        (ValueError, lambda: seq.groupnorm(x, 2, weight=torch.zeros(7, device="cuda"))),
        (seq.SysconvError, lambda: seq.groupnorm(x, 2, eps=-1.0)),
        (seq.SysconvError, lambda: seq.groupnorm(x.cpu(), 2)),
    ]
    for i, (kind, call) in enumerate(bad):
        with pytest.raises(kind):
            call()
            print("case", i)
    assert binding.launch_count() == before


def test_nothing_to_do(cuda_device):
    x = torch.zeros(0, 5, 8, device="cuda")
    w = torch.zeros(8, 4, device="cuda")
    assert seq.conv1d_causal(x, w).shape == x.shape
    assert (seq.conv1d_causal_backward(x, x, w)[1] == 0).all()
    none = torch.zeros(0, 8, device="cuda")
    off = torch.zeros(1, dtype=torch.int32, device="cuda")
    A, B = torch.zeros(8, 16, device="cuda"), torch.zeros(0, 16, device="cuda")
    y, saved = seq.state_scan(none, none, A, B, B, offsets=off, save=True)
    g = seq.state_scan_backward(y, none, none, A, B, B, saved, offsets=off)
    assert (g.dA == 0).all()
    off = torch.zeros(4, dtype=torch.int32, device="cuda")                  # three empty sequences
    st = torch.randn(3, 8, 16, device="cuda")
    y, final, saved = seq.state_scan(none, none, A, B, B, offsets=off, state=st, return_state=True, save=True)
    assert torch.equal(final, st)
    df = torch.randn(3, 8, 16, device="cuda")
    g = seq.state_scan_backward(none, none, none, A, B, B, saved, offsets=off, dfinal=df, state_grad=True)
    assert torch.equal(g.dstate, df) and (g.dA == 0).all()
    assert seq.groupnorm(torch.zeros(0, 4, 8, device="cuda"), 2).shape == (0, 4, 8)


# ------------------------------------------------------------------------------------------ the block that uses them together


def test_block_trains_and_continues_prompts(cuda_device):
    """Gradients of the block against the same block in torch's own operators in 64 bits, fp32 matrix products included
    (1e-4 of the 2-norm); prompt and single tokens against whole sequences (fp32, 1e-5)."""
    from paper_2010_15884_b200 import scanblock
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        assert scanblock.main() <= 1e-5
        torch.manual_seed(1)
        b = scanblock.ScanBlock(width=48, channels=40, states=8, groups=4, dtype=torch.float32)
        x = torch.randn(2, 23, 48, device="cuda", requires_grad=True)
        dy = torch.randn(2, 23, 48, device="cuda")
        b(x).backward(dy)
        p = {k: v.detach().double().requires_grad_() for k, v in b.named_parameters()}
        xd = x.detach().double().requires_grad_()
        f = torch.nn.functional
        h = f.group_norm(xd.reshape(-1, 48), 4, p["norm_weight"], p["norm_bias"], 1e-5).reshape(xd.shape) @ p["into"].t()
        u, z = h[..., :40], h[..., 40:]
        u = f.silu(f.conv1d(f.pad(u.transpose(1, 2), (3, 0)), p["conv_weight"][:, None], p["conv_bias"], groups=40).transpose(1, 2))
        q = u @ p["params"].t()
        B, C = q[..., b.rank: b.rank + 8], q[..., b.rank + 8:]
        v = dict(u=u, delta=q[..., : b.rank] @ p["widen"].t(), z=z, B=B[:, :, None], C=C[:, :, None])
        y, _ = _loop64(v, dict(A=-torch.exp(p["log_A"]), D=p["D"], delta_bias=p["delta_bias"]), torch.zeros(2, 40, 8, device="cuda"), True)
        (xd + y @ p["out"].t()).backward(dy.double())
        for name, t in b.named_parameters():
            assert float((t.grad.double() - p[name].grad).norm() / p[name].grad.norm()) <= 1e-4, name
        assert float((x.grad.double() - xd.grad).norm() / xd.grad.norm()) <= 1e-4
    finally:
        torch.backends.cuda.matmul.allow_tf32 = before


def test_python_and_native_marshalling_agree(cuda_device, monkeypatch):
    """The calls by way of the C++ module and by way of the Python layer alone give the same bits."""
    assert seq._sequence is not None, "_sequence.so is not built"
    case = ("bf16", [5, 0, 33], 24, 16, 2, True, True, True, True, True, True)
    v, p, dy, st, plus, off = scan_case(case, 9)
    x, w, b = v["u"], Draw(1, torch.bfloat16)(24, 4), Draw(2, torch.bfloat16)(24)
    cs, nw = Draw(3, torch.bfloat16)(3, 3, 24), Draw(4, torch.float32)(24)

    def everything():
        y, final, saved = seq.state_scan(**v, **p, softplus=plus, state=st, offsets=off, return_state=True, save=True)
        g = seq.state_scan_backward(dy, saved=saved, **v, **p, softplus=plus, offsets=off, dfinal=final, state_grad=True)
        h, c = st.clone(), cs.clone()
        rows = {k: t[:3] for k, t in v.items()}
        ys = seq.state_scan_step(rows["u"], rows["delta"], p["A"], rows["B"], rows["C"], h, D=p["D"], z=rows["z"], softplus=True)
        yc = seq.conv1d_causal_step(x[:3], c, w, b, "silu")
        yn, mean, rstd = seq.groupnorm(x[None], 3, nw, nw, activation="silu", return_stats=True)
        # (`saved` itself has rows between packed sequences that nobody writes or reads)
        return (y, final, *g, h, c, ys, yc, yn, mean, rstd, *seq.conv1d_causal(x, w, b, "silu", cs, off, True),
                *seq.conv1d_causal_backward(dy, x, w, b, "silu", cs, off, cs), *seq.groupnorm_backward(dy[None], x[None], 3, mean, rstd, nw, nw, "silu"))

    native = everything()
    monkeypatch.setattr(seq, "_sequence", None)
    for a, c in zip(native, everything()):
        assert torch.equal(a, c)
