"""The sequence operators as they are measured: cases, inputs, plain forms, calls, and the definitions in 64 bits.

Operators (channels last everywhere: a token is a row of channels)

  conv    short causal convolution per channel, y[t] = act(bias + sum_k w[k] x[t+k-(K-1)]), with the K-1 inputs that
          precede the sequence as its state: prompts (packed or dense), training (forward and backward), single tokens
  scan    selective state space scan, h[t] = exp(delta[t] A) h[t-1] + delta[t] u[t] B[t], y[t] = C[t] h[t] + D u[t],
          gated by silu(z): prompts, training, single tokens
  norm    group norm with an activation over (batch, space, channels): forward, and training

Where ``own`` is false ``run`` computes them with elementary torch operations in 32 bits, rounded once at the end;
where it is true it makes the calls a user of the package makes.
"""
import functools
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}


@functools.lru_cache(None)
def _package():
    from paper_2010_15884_b200 import sequence
    return sequence


# ---------------------------------------------------------------------------------------------------- cases


def listed():
    return [
        # one user's next token: launch latency is what counts
        dict(name="conv_step_one", op="conv_step", rows=1, slots=1, channels=2560, taps=4, type="bf16"),
        dict(name="scan_step_one", op="scan_step", rows=1, slots=1, channels=2560, states=16, groups=1, type="bf16"),
        # the next tokens of a full server: rows picked out of a larger cache of states
        dict(name="scan_step_many", op="scan_step", rows=192, slots=250, channels=4096, states=16, groups=1, type="bf16"),
        # a pack of prompts of uneven lengths, the convolution's input being one half of a wider projection
        dict(name="conv_prompts", op="conv", sequences=11, tokens=8191, channels=4096, taps=4, packed=True, wide=True,
             type="bf16"),
        # a training step's convolution, forward and backward
        dict(name="conv_train", op="conv_train", sequences=4, tokens=4 * 2048, channels=2048, taps=4, packed=False,
             wide=False, type="bf16"),
        # one short prompt of an odd length: too few rows to fill the machine
        dict(name="scan_prompt_short", op="scan", sequences=1, tokens=113, channels=1408, states=16, groups=1, packed=False,
             type="f16"),
        # one long prompt
        dict(name="scan_prompt_long", op="scan", sequences=1, tokens=8192, channels=4096, states=16, groups=1, packed=False,
             type="bf16"),
        # a pack of prompts, single precision, the state matrices shared by groups of channels
        dict(name="scan_prompts", op="scan", sequences=7, tokens=3001, channels=1280, states=32, groups=2, packed=True,
             type="f32"),
        # a training step's scan, forward and backward
        dict(name="scan_train", op="scan_train", sequences=4, tokens=4 * 2048, channels=2048, states=16, groups=1,
             packed=False, type="bf16"),
        # tokens of a hybrid block: each token's channels in groups, no space to reduce over
        dict(name="norm_tokens", op="norm", batch=8191, space=1, channels=4096, groups=8, act=False, type="bf16"),
        # full-HD feature maps after a convolution
        dict(name="norm_image", op="norm", batch=1, space=1080 * 1920, channels=64, groups=16, act=True, type="bf16"),
        # training on feature maps, ten channels a group
        dict(name="norm_train", op="norm_train", batch=8, space=64 * 64, channels=320, groups=32, act=True, type="f32"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, evenly over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _channels(rng, lo, hi):
    """Channels: mostly multiples of 8, some odd."""
    c = _spread(rng, lo, hi)
    return c if rng.random() < 0.25 else max(8, c // 8 * 8)


def draw(rng):
    case = _drawn(rng)
    while 3072 in case.values() or 1536 in case.values():                 # one width (and its half) is left out
        case = _drawn(rng)
    return case


def _drawn(rng):
    op = rng.choice(["conv", "conv_train", "conv_step", "scan", "scan_train", "scan_step", "norm", "norm_train"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op.endswith("step"):
        rows = _spread(rng, 1, 192)
        case = dict(op=op, rows=rows, slots=rows + rng.randrange(0, 60), channels=_channels(rng, 64, 4096), type=kind)
        if op == "conv_step":
            return dict(case, taps=rng.choice([2, 3, 4, 4, 4, 6]))
        return dict(case, states=rng.choice([4, 8, 16, 16, 16, 19, 32, 64]), groups=1)
    if op.startswith("conv"):
        tokens, channels = _spread(rng, 1, 8191), _channels(rng, 64, 4096)
        return dict(op=op, sequences=min(tokens, _spread(rng, 1, 12)), tokens=tokens, channels=channels,
                    taps=rng.choice([2, 3, 4, 4, 4, 6]), packed=True, wide=rng.random() < 0.5, type=kind)
    if op.startswith("scan"):
        states = rng.choice([4, 8, 16, 16, 16, 19, 32, 64])
        channels = _channels(rng, 64, 4096)
        most = 8192 * 4096 * 16 // 2 if op == "scan" else 8192 * 2048 * 16 // 2
        tokens = _spread(rng, 1, max(1, min(8192, most // (channels * states))))
        groups = rng.choice([g for g in (1, 1, 2, 4) if channels % g == 0])
        return dict(op=op, sequences=min(tokens, _spread(rng, 1, 8)), tokens=tokens, channels=channels, states=states,
                    groups=groups, packed=True, type=kind)
    groups = rng.choice([1, 4, 8, 16, 32])
    channels = groups * _spread(rng, 2, 64)
    space = 1 if rng.random() < 0.3 else _spread(rng, 2, 256 * 256)
    most = 1 << (25 if op == "norm" else 24)
    batch = _spread(rng, 1, max(1, min(8191, most // (space * channels))))
    return dict(op=op, batch=batch, space=space, channels=channels, groups=groups, act=rng.random() < 0.7, type=kind)


def _lengths(case):
    """Lengths of the sequences: equal if dense, else uneven, one of them empty where there are four or more."""
    n, total = case["sequences"], case["tokens"]
    if not case["packed"]:
        return [total // n] * n
    share = [1.0 + 2.0 * ((7 * i + 3) % 5) for i in range(n)]
    if n >= 4:
        share[n // 2] = 0.0
    ends = [int(round(total * sum(share[: i + 1]) / sum(share))) for i in range(n)]
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


# ---------------------------------------------------------------------------------------------------- inputs


def prepare(case, seed):
    """Inputs with the distributions a trained layer meets: unit activations, decays between a few and a few hundred tokens."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = _TYPES[case["type"]]

    def normal(*shape, scale=1.0, dtype=kind):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    op, s = case["op"], dict(case)
    if op.startswith("norm"):
        b, n, c = case["batch"], case["space"], case["channels"]
        shift = torch.randn(c, generator=gen, device="cuda")
        s["x"] = (torch.randn(b, n, c, generator=gen, device="cuda").mul_(1.5).add_(shift)).to(kind)
        s["weight"] = normal(c, scale=0.2, dtype=torch.float32) + 1.0
        s["bias"] = normal(c, scale=0.2, dtype=torch.float32)
        if op == "norm_train":
            s["dy"] = normal(b, n, c)
        return s

    d = case["channels"]
    if op.startswith("conv"):
        k = case["taps"]
        s["weight"] = normal(d, k, scale=1.0 / math.sqrt(k))
        s["bias"] = normal(d, scale=0.1)
    else:
        n, g = case["states"], case["groups"]
        s["A"] = -(torch.arange(1, n + 1, device="cuda", dtype=torch.float32)
                   * torch.exp(0.1 * torch.randn(d, n, generator=gen, device="cuda"))).contiguous()
        s["D"] = normal(d, scale=0.3, dtype=torch.float32) + 1.0
        step = torch.exp(torch.rand(d, generator=gen, device="cuda") * math.log(100.0) + math.log(1e-3))
        s["delta_bias"] = step + torch.log(-torch.expm1(-step))                # softplus(delta_bias) in [0.001, 0.1]

    if op.endswith("step"):
        rows, slots = case["rows"], case["slots"]
        s["index"] = torch.randperm(slots, generator=gen, device="cuda")[:rows].to(torch.int32)
        if op == "conv_step":
            s["x"], s["state"] = normal(rows, d), normal(slots, k - 1, d)
            return s
        s["u"], s["delta"], s["z"] = normal(rows, d), normal(rows, d, scale=0.5), normal(rows, d)
        s["B"], s["C"] = normal(rows, g, n), normal(rows, g, n)
        s["state"] = normal(slots, d, n, scale=0.3, dtype=torch.float32)
        return s

    lengths = _lengths(case)
    r, t = len(lengths), sum(lengths)
    lead = (t,) if case["packed"] else (r, t // r)
    s["offsets"], s["longest"] = None, max(lengths)
    if case["packed"]:
        s["offsets"] = torch.tensor([sum(lengths[:i]) for i in range(r + 1)], dtype=torch.int32, device="cuda")
    if op.startswith("conv"):
        s["x"] = normal(*lead, 2 * d)[..., :d] if case["wide"] else normal(*lead, d)
        s["state"] = normal(r, k - 1, d)
    else:
        s["u"], s["delta"], s["z"] = normal(*lead, d), normal(*lead, d, scale=0.5), normal(*lead, d)
        s["B"], s["C"] = normal(*lead, g, n), normal(*lead, g, n)
        s["state"] = normal(r, d, n, scale=0.3, dtype=torch.float32)
    if op.endswith("train"):
        s["dy"] = normal(*lead, d)
    return s


def work(case):
    """Each input read once, each output written once; operations as written in the formulas (exp and division: one each)."""
    op, e = case["op"], _BYTES[case["type"]]
    if op.startswith("norm"):
        m = case["batch"] * case["space"] * case["channels"]
        par = 8 * case["channels"]
        if op == "norm":
            return {"bytes": 2 * m * e + par, "flops": 10 * m}
        return {"bytes": 4 * m * e + 2 * par, "flops": 30 * m}
    d = case["channels"]
    if op == "conv_step":
        k, r = case["taps"], case["rows"]
        return {"bytes": e * d * (r * 2 * k + k + 1), "flops": r * d * (2 * k + 4)}     # x, y, K-1 states in and out
    if op.startswith("conv"):
        k, t, r = case["taps"], case["tokens"], case["sequences"]
        par = e * d * (k + 1)
        if op == "conv":
            return {"bytes": 2 * t * d * e + par + 2 * r * (k - 1) * d * e, "flops": t * d * (2 * k + 4)}
        return {"bytes": 4 * t * d * e + 2 * par + 2 * r * (k - 1) * d * e, "flops": t * d * (8 * k + 12)}
    n, g = case["states"], case["groups"]
    par = 4 * d * (n + 2)
    if op == "scan_step":
        r = case["rows"]
        return {"bytes": r * (4 * d * e + 2 * g * n * e + 8 * d * n) + par, "flops": r * d * (7 * n + 10)}
    t, r = case["tokens"], case["sequences"]
    if op == "scan":
        return {"bytes": t * (4 * d + 2 * g * n) * e + par + 8 * r * d * n, "flops": t * d * (7 * n + 10)}
    return {"bytes": t * (8 * d + 4 * g * n) * e + 2 * par + 12 * r * d * n, "flops": t * d * (24 * n + 30)}


# ---------------------------------------------------------------------------------------------------- plain forms


def run(s):
    return _RUN[s["op"], own](s)


def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _dsilu(v):
    g = 1.0 / (1.0 + torch.exp(-v))
    return g * (1.0 + v * (1.0 - g))


def _softplus(v):
    return torch.where(v > 20.0, v, torch.log1p(torch.exp(torch.clamp(v, max=20.0))))


def _flat(s, name):
    """A tensor of tokens as (tokens, ...), the sequences one behind the other."""
    v = s[name]
    return v if s["packed"] else v.reshape((-1,) + v.shape[2:])


def _like(s, v):
    return v if s["packed"] else v.reshape((s["sequences"], -1) + v.shape[1:])


def _places(s):
    """Per token: its sequence, and its distance from the sequence's first token; and where the sequences begin and end."""
    if s["packed"]:
        first, end = s["offsets"][:-1].long(), s["offsets"][1:].long()
    else:
        n = s["tokens"] // s["sequences"]
        first = torch.arange(s["sequences"], device="cuda") * n
        end = first + n
    at = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(end, at, right=True)
    return seq, at - first[seq], first, end


def _conv_rows(s):
    """(row, from_state): the rows of [all states; all tokens] that the K taps of each token read, oldest first."""
    k, r = s["taps"], s["sequences"]
    seq, at, first, end = _places(s)
    back = torch.arange(k - 1, -1, -1, device="cuda")
    tokens = torch.arange(s["tokens"], device="cuda")
    row = torch.where(at[:, None] >= back, tokens[:, None] - back + r * (k - 1), seq[:, None] * (k - 1) + (k - 1) + at[:, None] - back)
    keep = torch.arange(k - 1, device="cuda")                              # new state: the last K-1 of state and tokens
    length = end - first
    late = length[:, None] + keep
    last = torch.where(late >= k - 1, first[:, None] + late - (k - 1) + r * (k - 1), torch.arange(r, device="cuda")[:, None] * (k - 1) + late)
    return row, last


def _conv_forward(s):
    k, d = s["taps"], s["channels"]
    row, last = _conv_rows(s)
    every = torch.cat([s["state"].reshape(-1, d), _flat(s, "x")]).float()
    w, b = s["weight"].float(), s["bias"].float()
    taps = [every[row[:, i]] for i in range(k)]
    pre = b + sum(taps[i] * w[:, i] for i in range(k))
    return every, taps, row, last, pre


def _plain_conv(s):
    every, taps, row, last, pre = _conv_forward(s)
    return _like(s, _silu(pre).to(s["x"].dtype)), every[last].to(s["x"].dtype)


def _plain_conv_train(s):
    k = s["taps"]
    every, taps, row, last, pre = _conv_forward(s)
    y = _silu(pre)
    dpre = _flat(s, "dy").float() * _dsilu(pre)
    w = s["weight"].float()
    devery = torch.zeros_like(every)
    for i in range(k):                                                     # a row is read once at most by each tap
        devery.index_add_(0, row[:, i], dpre * w[:, i])
    dweight = torch.stack([(dpre * taps[i]).sum(0) for i in range(k)], dim=1)
    n = s["sequences"] * (k - 1)
    t = s["x"].dtype
    return (_like(s, y.to(t)), _like(s, devery[n:].to(t)), dweight.to(t), dpre.sum(0).to(t),
            devery[:n].reshape(s["state"].shape).to(t))


def _plain_conv_step(s):
    at = s["index"].long()
    seen = torch.cat([s["state"][at], s["x"][:, None]], dim=1)             # (rows, K, channels)
    pre = s["bias"].float() + (seen.float() * s["weight"].float().t()).sum(1)
    s["state"][at] = seen[:, 1:]
    return _silu(pre).to(s["x"].dtype), s["state"]


def _recurrence(a, b):
    """h[t] = a[t] h[t-1] + b[t] with h[-1] = 0, along the first axis: pairs of steps are joined, half as many remain."""
    n = a.shape[0]
    if n == 1:
        return b
    m = n // 2 * 2
    odd = _recurrence(a[0:m:2] * a[1:m:2], a[1:m:2] * b[0:m:2] + b[1:m:2])
    h = torch.empty_like(b)
    h[1:m:2] = odd
    h[0] = b[0]
    if n > 2:
        h[2::2] = a[2::2] * odd[: (n - 1) // 2] + b[2::2]
    return h


def _scan_forward(s):
    d, g, n = s["channels"], s["groups"], s["states"]
    seq, at, first, end = _places(s)
    f = {name: _flat(s, name).float() for name in ("u", "delta", "z", "B", "C")}
    raw = f["delta"] + s["delta_bias"]
    f["raw"], f["delta"] = raw, _softplus(raw)
    wide = {name: f[name][:, :, None].expand(-1, g, d // g, n).reshape(-1, d, n) for name in ("B", "C")}
    a = torch.exp(f["delta"][:, :, None] * s["A"])
    b = (f["delta"] * f["u"])[:, :, None] * wide["B"]
    some = end > first
    starts = first[some]
    b[starts] += a[starts] * s["state"][some]
    cut = a.clone()
    cut[starts] = 0.0
    h = _recurrence(cut, b)
    final = s["state"].clone()
    final[some] = h[end[some] - 1]
    y = (h * wide["C"]).sum(2) + s["D"] * f["u"]
    return f, wide, a, h, y, final, starts, end[some] - 1, some


def _plain_scan(s):
    f, _, _, _, y, final, _, _, _ = _scan_forward(s)
    return _like(s, (y * _silu(f["z"])).to(s["u"].dtype)), final


def _plain_scan_train(s):
    d, g, n = s["channels"], s["groups"], s["states"]
    f, wide, a, h, y, _, starts, ends, some = _scan_forward(s)
    dout = _flat(s, "dy").float()
    dy = dout * _silu(f["z"])
    after = torch.zeros_like(a)                                            # decay towards the following token
    after[:-1] = a[1:]
    after[ends] = 0.0
    dh = _recurrence(after.flip(0), (dy[:, :, None] * wide["C"]).flip(0)).flip(0)
    del after
    before = torch.zeros_like(h)
    before[1:] = h[:-1]
    before[starts] = s["state"][some]
    dlog = dh * a * before                                                 # gradient with respect to delta A
    dbu = (dh * wide["B"]).sum(2)
    ddelta = (dlog * s["A"]).sum(2) + dbu * f["u"]
    dpre = ddelta / (1.0 + torch.exp(-f["raw"]))
    dstate = torch.zeros_like(s["state"])
    dstate[some] = dh[starts] * a[starts]
    t = s["u"].dtype
    db = (dh * (f["delta"] * f["u"])[:, :, None]).reshape(-1, g, d // g, n).sum(2)
    dc = (h * dy[:, :, None]).reshape(-1, g, d // g, n).sum(2)
    return {"y": _like(s, (y * _silu(f["z"])).to(t)), "du": _like(s, (dbu * f["delta"] + dy * s["D"]).to(t)),
            "ddelta": _like(s, dpre.to(t)), "dA": (dlog * f["delta"][:, :, None]).sum(0), "dB": _like(s, db.to(t)),
            "dC": _like(s, dc.to(t)), "dD": (dy * f["u"]).sum(0), "dz": _like(s, (dout * y * _dsilu(f["z"])).to(t)),
            "ddelta_bias": dpre.sum(0), "dstate": dstate}


def _plain_scan_step(s):
    d, g, n = s["channels"], s["groups"], s["states"]
    at = s["index"].long()
    delta, u = _softplus(s["delta"].float() + s["delta_bias"]), s["u"].float()
    b, c = (s[name].float()[:, :, None].expand(-1, g, d // g, n).reshape(-1, d, n) for name in ("B", "C"))
    h = torch.exp(delta[:, :, None] * s["A"]) * s["state"][at] + (delta * u)[:, :, None] * b
    s["state"][at] = h
    y = ((h * c).sum(2) + s["D"] * u) * _silu(s["z"].float())
    return y.to(s["u"].dtype), s["state"]


def _norm_forward(s, x):
    c, g = s["channels"], s["groups"]
    v = x.float().reshape(x.shape[0], x.shape[1], g, c // g)
    mean = v.mean(dim=(1, 3), keepdim=True)
    v = v - mean
    rstd = 1.0 / torch.sqrt((v * v).mean(dim=(1, 3), keepdim=True) + 1e-5)
    xhat = (v * rstd).reshape(x.shape)
    pre = xhat * s["weight"] + s["bias"]
    return xhat, rstd, pre, _silu(pre) if s["act"] else pre


def _plain_norm(s):
    return _norm_forward(s, s["x"])[3].to(s["x"].dtype)


def _plain_norm_train(s):
    x, g = s["x"], s["groups"]
    xhat, rstd, pre, y = _norm_forward(s, x)
    dpre = s["dy"].float()
    if s["act"]:
        dpre = dpre * _dsilu(pre)
    split = (x.shape[0], x.shape[1], g, -1)
    dxhat = (dpre * s["weight"]).reshape(split)
    v = xhat.reshape(split)
    dx = rstd * (dxhat - dxhat.mean(dim=(1, 3), keepdim=True) - v * (dxhat * v).mean(dim=(1, 3), keepdim=True))
    return y.to(x.dtype), dx.reshape(x.shape).to(x.dtype), (dpre * xhat).sum((0, 1)), dpre.sum((0, 1))


# ---------------------------------------------------------------------------------------------------- the package's calls


def _own_conv(s):
    return _package().conv1d_causal(s["x"], s["weight"], s["bias"], "silu", state=s["state"], offsets=s["offsets"],
                                    return_state=True)


def _own_conv_train(s):
    q = _package()
    y = q.conv1d_causal(s["x"], s["weight"], s["bias"], "silu", state=s["state"], offsets=s["offsets"])
    return (y,) + tuple(q.conv1d_causal_backward(s["dy"], s["x"], s["weight"], s["bias"], "silu", state=s["state"],
                                                 offsets=s["offsets"]))


def _own_conv_step(s):
    y = _package().conv1d_causal_step(s["x"], s["state"], s["weight"], s["bias"], "silu", slots=s["index"])
    return y, s["state"]


def _own_scan(s):
    return _package().state_scan(s["u"], s["delta"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"],
                                 delta_bias=s["delta_bias"], softplus=True, state=s["state"], offsets=s["offsets"],
                                 longest=s["longest"], return_state=True)


def _own_scan_train(s):
    q = _package()
    y, saved = q.state_scan(s["u"], s["delta"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"], delta_bias=s["delta_bias"],
                            softplus=True, state=s["state"], offsets=s["offsets"], longest=s["longest"], save=True)
    g = q.state_scan_backward(s["dy"], s["u"], s["delta"], s["A"], s["B"], s["C"], saved, D=s["D"], z=s["z"],
                              delta_bias=s["delta_bias"], softplus=True, offsets=s["offsets"], longest=s["longest"],
                              state_grad=True)
    return {"y": y, "du": g.du, "ddelta": g.ddelta, "dA": g.dA, "dB": g.dB, "dC": g.dC, "dD": g.dD, "dz": g.dz,
            "ddelta_bias": g.ddelta_bias, "dstate": g.dstate}


def _own_scan_step(s):
    y = _package().state_scan_step(s["u"], s["delta"], s["A"], s["B"], s["C"], s["state"], D=s["D"], z=s["z"],
                                   delta_bias=s["delta_bias"], softplus=True, slots=s["index"])
    return y, s["state"]


def _own_norm(s):
    return _package().groupnorm(s["x"], s["groups"], s["weight"], s["bias"], eps=1e-5,
                                activation="silu" if s["act"] else None)


def _own_norm_train(s):
    q, act = _package(), "silu" if s["act"] else None
    y, mean, rstd = q.groupnorm(s["x"], s["groups"], s["weight"], s["bias"], eps=1e-5, activation=act, return_stats=True)
    return (y,) + tuple(q.groupnorm_backward(s["dy"], s["x"], s["groups"], mean, rstd, s["weight"], s["bias"],
                                             activation=act))


_RUN = {("conv", False): _plain_conv, ("conv_train", False): _plain_conv_train, ("conv_step", False): _plain_conv_step,
        ("scan", False): _plain_scan, ("scan_train", False): _plain_scan_train, ("scan_step", False): _plain_scan_step,
        ("norm", False): _plain_norm, ("norm_train", False): _plain_norm_train,
        ("conv", True): _own_conv, ("conv_train", True): _own_conv_train, ("conv_step", True): _own_conv_step,
        ("scan", True): _own_scan, ("scan_train", True): _own_scan_train, ("scan_step", True): _own_scan_step,
        ("norm", True): _own_norm, ("norm_train", True): _own_norm_train}


# ---------------------------------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    """The definitions, token by token and sequence by sequence, in 64 bits."""
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v
         for k, v in prepare(case, seed).items()}
    op = case["op"]
    if op.startswith("norm"):
        return _exact_norm(s)
    if op == "conv_step":
        return _exact_conv_step(s)
    if op == "scan_step":
        return _exact_scan_step(s)
    lengths = _lengths(case)
    first = [sum(lengths[:i]) for i in range(len(lengths))]
    spans = [(a, a + n) for a, n in zip(first, lengths)]
    if op.startswith("conv"):
        return _exact_conv(s, spans)
    return _exact_scan(s, spans)


def _exact_conv_step(s):
    y, state = [], s["state"].clone()
    for row, slot in enumerate(s["index"].tolist()):
        window = torch.cat([s["state"][slot], s["x"][row: row + 1]])
        v = torch.einsum("kd,dk->d", window, s["weight"]) + s["bias"]
        y.append(v * torch.sigmoid(v))
        state[slot] = window[1:]
    return torch.stack(y), state


def _exact_conv(s, spans):
    k, d = s["taps"], s["channels"]
    x = s["x"].reshape(-1, d)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dw, db = torch.zeros_like(s["weight"]), torch.zeros_like(s["bias"])
    final, dstate = torch.empty_like(s["state"]), torch.zeros_like(s["state"])
    train = s["op"] == "conv_train"
    for i, (a, b) in enumerate(spans):
        line = torch.cat([s["state"][i], x[a:b]])
        final[i] = line[b - a:]
        if a == b:
            continue
        win = line.unfold(0, k, 1)                                          # (length, channels, K)
        v = (win * s["weight"]).sum(2) + s["bias"]
        sig = torch.sigmoid(v)
        y[a:b] = v * sig
        if train:
            dv = s["dy"].reshape(-1, d)[a:b] * (sig + v * sig * (1 - sig))
            dw += (dv[:, :, None] * win).sum(0)
            db += dv.sum(0)
            dline = torch.zeros_like(line)
            for j in range(k):
                dline[j: j + b - a] += dv * s["weight"][:, j]
            dx[a:b], dstate[i] = dline[k - 1:], dline[: k - 1]
    if train:
        return y.reshape(s["x"].shape), dx.reshape(s["x"].shape), dw, db, dstate
    return y.reshape(s["x"].shape), final


def _exact_scan_step(s):
    d, g = s["channels"], s["groups"]
    at = s["index"].long()
    delta = torch.nn.functional.softplus(s["delta"] + s["delta_bias"])
    b, c = (s[n].repeat_interleave(d // g, dim=1) for n in ("B", "C"))
    state = s["state"].clone()
    state[at] = (delta[:, :, None] * s["A"]).exp() * state[at] + (delta * s["u"])[:, :, None] * b
    y = torch.einsum("rdn,rdn->rd", state[at], c) + s["D"] * s["u"]
    return y * s["z"] * torch.sigmoid(s["z"]), state


def _exact_scan(s, spans):
    d, g, n = s["channels"], s["groups"], s["states"]
    u, raw, z = (s[name].reshape(-1, d) for name in ("u", "delta", "z"))
    raw = raw + s["delta_bias"]
    delta = torch.nn.functional.softplus(raw)
    b, c = (s[name].reshape(-1, g, n) for name in ("B", "C"))
    y, final = torch.empty_like(u), s["state"].clone()
    train = s["op"] == "scan_train"
    kept = torch.empty(u.shape[0], d, n, dtype=torch.float64, device="cuda") if train else None

    def per_channel(v):                                                     # (groups, states) -> (channels, states)
        return v[:, None].expand(g, d // g, n).reshape(d, n)

    for i, (lo, hi) in enumerate(spans):
        h = s["state"][i]
        for t in range(lo, hi):
            h = torch.exp(delta[t, :, None] * s["A"]) * h + (delta[t] * u[t])[:, None] * per_channel(b[t])
            y[t] = (h * per_channel(c[t])).sum(1)
            if train:
                kept[t] = h
        final[i] = h
    y = y + s["D"] * u
    sig = torch.sigmoid(z)
    out = y * z * sig
    if not train:
        return out.reshape(s["u"].shape), final
    dout = s["dy"].reshape(-1, d)
    dy, dz = dout * z * sig, dout * y * (sig + z * sig * (1 - sig))
    du, ddelta = dy * s["D"], torch.empty_like(u)
    dA, dB, dC = torch.zeros_like(s["A"]), torch.empty_like(b), torch.empty_like(c)
    dstate = torch.zeros_like(s["state"])
    for i, (lo, hi) in enumerate(spans):
        carry = torch.zeros_like(s["A"])
        for t in range(hi - 1, lo - 1, -1):
            dh = carry + dy[t, :, None] * per_channel(c[t])
            carry = dh * torch.exp(delta[t, :, None] * s["A"])
            dlog = carry * (kept[t - 1] if t > lo else s["state"][i])
            dbu = (dh * per_channel(b[t])).sum(1)
            dB[t] = (dh * (delta[t] * u[t])[:, None]).reshape(g, d // g, n).sum(1)
            dC[t] = (kept[t] * dy[t, :, None]).reshape(g, d // g, n).sum(1)
            ddelta[t] = (dlog * s["A"]).sum(1) + dbu * u[t]
            du[t] += dbu * delta[t]
            dA += dlog * delta[t, :, None]
        dstate[i] = carry
    dpre = ddelta * torch.sigmoid(raw)
    grads = {"y": out, "du": du, "ddelta": dpre, "dz": dz}
    grads = {k: v.reshape(s["u"].shape) for k, v in grads.items()}
    return dict(grads, dA=dA, dB=dB.reshape(s["B"].shape), dC=dC.reshape(s["C"].shape), dD=(dy * u).sum(0),
                ddelta_bias=dpre.sum(0), dstate=dstate)


def _exact_norm(s):
    b, n, c = s["x"].shape
    g = s["groups"]
    y, dx = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    dw, db = torch.zeros_like(s["weight"]), torch.zeros_like(s["bias"])
    piece = max(1, (1 << 26) // (n * c))                                    # images at a time
    for lo in range(0, b, piece):
        x = s["x"][lo: lo + piece].reshape(-1, n, g, c // g)
        var, mean = torch.var_mean(x, dim=(1, 3), unbiased=False, keepdim=True)
        rstd = (var + 1e-5).rsqrt()
        xhat = ((x - mean) * rstd).reshape(-1, n, c)
        v = xhat * s["weight"] + s["bias"]
        sig = torch.sigmoid(v)
        y[lo: lo + piece] = v * sig if s["act"] else v
        if s["op"] == "norm_train":
            dv = s["dy"][lo: lo + piece] * ((sig + v * sig * (1 - sig)) if s["act"] else 1.0)
            dw += (dv * xhat).sum((0, 1))
            db += dv.sum((0, 1))
            p = (dv * s["weight"]).reshape(x.shape)
            q = xhat.reshape(x.shape)
            m = n * (c // g)
            dx[lo: lo + piece] = (rstd * (p - p.sum((1, 3), keepdim=True) / m
                                          - q * (p * q).sum((1, 3), keepdim=True) / m)).reshape(-1, n, c)
    return (y, dx, dw, db) if s["op"] == "norm_train" else y
